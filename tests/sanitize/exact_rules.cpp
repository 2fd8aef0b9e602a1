// Prints which kernels calls of exact attention take, for sizes on stdin: bf16 batch q_len kv_len heads kv_heads causal
// window max_distance (0: no bias); then how many parts a bias gradient is joined from. Without a device the rules go by 256 CUs, an MI355X's.
#include <cstdio>
#include <cstring>

#include "exact.h"

int main() {
  static const char* names[] = {"32", "short", "128", "256"};
  int bf16, B, nq, nk, H, Hk, causal, window, D;
  while (std::scanf("%d %d %d %d %d %d %d %d %d", &bf16, &B, &nq, &nk, &H, &Hk, &causal, &window, &D) == 9) {
    mca::ExactParams p;
    std::memset(&p, 0, sizeof p);
    p.bf16 = bf16, p.B = B, p.nq = nq, p.nk = nk, p.H = H, p.Hk = Hk, p.G = H / Hk;
    p.causal = causal, p.window = window > 0, p.half = window / 2, p.D = D;
    p.table = D ? &p : nullptr;  // not read
    p.Gp = mca::exact_group(p);
    p.kv_splits = mca::exact_kv_splits(p);
    std::printf("%s %s %s %lld\n", names[(int)mca::exact_forward_kernel(p)], names[(int)mca::exact_dq_kernel(p)],
                names[(int)mca::exact_dkv_kernel(p)], (long long)mca::exact_bias_parts(p));
  }
  return 0;
}
