"""Exact attention in float64 torch, with bounds on a kernel's error derived from the inputs.

Error bounds (u = half a step of float32, 2^-24; h = half a step of the layer's type where it is
bfloat16, 2^-8, else u; every bound holds element by element; a float32 sum of k terms in any order
is off by at most k u times the sum of the terms' magnitudes):
  logit S_ij:   e_ij = scale 65 u sum_d |q_d k_d|  (products and their sum)
                + 3 u (|S_ij| + |b_ij|)            (scale and bias in base 2, their sum rounded)
  lse_i:        max_j e_ij + (n_k + 16) u          (sum of at most n_k terms, exp2 and log2 of a few
                steps, one more rescaling per key tile) + 5 u |lse_i| (subtractions, base change)
  P_ij:         relative eta_i = 2 max_j e_ij + (n_k + 16) u + 5 u |lse_i|, and, as the operand of a
                product, h more in bfloat16
                (backward in bfloat16: + 68 u |lse_i|, as the sums of S start at -lse_i / scale)
  y_i:          sum_j P_ij |v_j| (eta_i + [bf16] h + n_k u) + h |y_i|
  D_i:          sum_d |dy| (error of y_i) + 65 u sum_d |dy y|
  dS_ij:        P_ij (65 u sum_d |dy v| + error of D_i) + (eta_i + 4 u) P_ij (|dP_ij| + |D_i|), and, as
                the operand of a product, [bf16] h |dS_ij| more
  sums over dS: those errors times the other operand's magnitude, (terms) u of the sum of magnitudes,
                and h of the result
Second-order terms are covered by a factor of 1.01 and a floor of the smallest normal float32 (flushed
exp2 results).
"""
import math

import torch

U = 2.0 ** -24
TINY = 2.0 ** -126


def bucket(r, buckets, top, both):
    n = buckets // 2 if both else buckets
    e = n // 2
    m = n - e
    d = abs(r) if both else max(-r, 0)
    k = d if d < e else e + max(k for k in range(m) if d ** m * e ** k >= e ** m * top ** k)
    return k + (n if both and r > 0 else 0)


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


class Case:
    """Inputs of one call (tensors on any device) and the float64 results with their error bounds."""

    def __init__(self, Q, K, V, heads, kv_heads, dY=None, scale=0.125, q_lens=None, kv_lens=None, q_pos=None, causal=False,
                 window=0, table=None, max_distance=128, bidirectional=True):
        dt, dev = Q.dtype, Q.device
        B, nq, nk, G = Q.shape[0], Q.shape[1], K.shape[1], heads // kv_heads
        h = half_step(dt)
        hp = h if dt == torch.bfloat16 else 0.0
        i, j = torch.arange(nq, device=dev), torch.arange(nk, device=dev)
        ql = torch.full((B,), nq, device=dev) if q_lens is None else q_lens.to(dev).long().clamp(0, nq)
        kl = torch.full((B,), nk, device=dev) if kv_lens is None else kv_lens.to(dev).long().clamp(0, nk)
        pos = i[None] + (0 if q_pos is None else q_pos.to(dev).long()[:, None])  # [B, nq]
        rows, keys = i[None] < ql[:, None], j[None] < kl[:, None]
        ok = rows[:, :, None] & keys[:, None, :]
        rel = j[None, None, :] - pos[:, :, None]
        if causal:
            ok &= rel <= 0
        if window:
            ok &= (rel.abs() <= window // 2) | (pos == 0)[:, :, None] | (j == 0)[None, None, :]

        def split(x, valid, n):  # [B, heads, rows, 64], rows that are not read as zeros
            x = torch.where(valid[:, :, None], x.double(), torch.zeros((), dtype=torch.float64, device=dev))
            return x.reshape(B, x.shape[1], -1, 64).transpose(1, 2).repeat_interleave(n, 1)

        q, k, v = split(Q, rows, 1), split(K, keys, G), split(V, keys, G)
        kt, vt = k.transpose(2, 3), v.transpose(2, 3)
        S = scale * (q @ kt)
        E = scale * 65 * U * (q.abs() @ kt.abs()) + 3 * U * S.abs()
        okh = ok[:, None].expand(S.shape).clone()
        if table is not None:
            at = torch.tensor([bucket(r, table.shape[0], max_distance, bidirectional) for r in range(-max_distance, max_distance + 1)],
                              device=dev)
            idx = at[rel.clamp(-max_distance, max_distance) + max_distance]
            b = table.double()[idx].permute(0, 3, 1, 2)
            okh &= b > -1e30
            b = torch.where(okh, b, torch.zeros_like(b))
            S, E = S + b, E + 3 * U * b.abs()
        S = torch.where(okh, S, torch.full_like(S, -math.inf))
        E = torch.where(okh, E, torch.zeros_like(E)).amax(-1, keepdim=True)
        M = S.amax(-1, keepdim=True)
        M = torch.where(torch.isfinite(M), M, torch.zeros_like(M))
        P = torch.exp(S - M)
        L = P.sum(-1, keepdim=True)
        self.any = L[..., 0] > 0
        P = P / torch.where(L > 0, L, torch.ones_like(L))
        lse = M + torch.log(L)
        size = torch.where(L > 0, lse, torch.zeros_like(lse)).abs()

        def join(x):
            return x.transpose(1, 2).reshape(B, x.shape[2], -1)

        eta = 2 * E + (nk + 16) * U + 5 * U * size
        y = P @ v
        y_tol = (P @ v.abs()) * (eta + hp + nk * U) + h * y.abs()
        self.want = {"Y": join(y), "lse": lse[..., 0]}
        self.tol = {"Y": join(y_tol), "lse": (E + (nk + 16) * U + 5 * U * size)[..., 0]}
        if dY is not None:
            dy = split(dY, rows, 1)
            if hp:
                eta = eta + 68 * U * size
            dP = dy @ vt
            D = (dy * y).sum(-1, keepdim=True)
            D_tol = (dy.abs() * y_tol).sum(-1, keepdim=True) + 65 * U * (dy * y).abs().sum(-1, keepdim=True)
            dS = P * (dP - D)
            s_tol = P * (65 * U * (dy.abs() @ vt.abs()) + D_tol) + (eta + 4 * U) * P * (dP.abs() + D.abs())
            p_tol = P * (eta + hp)
            o_tol = s_tol + hp * dS.abs()

            def group(x):
                return join(x.reshape(B, kv_heads, G, x.shape[2], 64).sum(2))

            T = lambda x: x.transpose(2, 3)  # noqa: E731
            n_sum = G * nq * U
            self.want.update(dQ=join(scale * (dS @ k)), dK=group(scale * (T(dS) @ q)), dV=group(T(P) @ dy))
            self.tol.update(dQ=join(scale * ((o_tol + nk * U * dS.abs()) @ k.abs())),
                            dK=group(scale * (T(o_tol + n_sum * dS.abs()) @ q.abs())),
                            dV=group(T(p_tol + n_sum * P) @ dy.abs()))
            if table is not None:
                bh = idx[:, None].expand(S.shape).reshape(-1) * heads + torch.arange(heads, device=dev)[None, :, None, None].expand(S.shape).reshape(-1)
                new = lambda x: torch.zeros(table.numel(), dtype=torch.float64, device=dev).index_add_(0, bh, x.reshape(-1)).view(table.shape)  # noqa: E731
                # a sum passes at most: the entries of a half wave's array (one add per key tile of 32 and
                # row), the eight arrays, a bucket's entries, the blocks' parts by 64 lanes
                adds = nq + nk + 8 + 2 * max_distance + 129 + B * nq / 64 + 8
                self.want["dbias"] = new(dS)
                self.tol["dbias"] = new(s_tol + adds * U * dS.abs())
            for n in ("dQ", "dK", "dV", "dbias"):
                if n in self.want:
                    self.tol[n] = self.tol[n] + h * self.want[n].abs()

    def check(self, got):
        """got: results by name. Every element within its bound; empty rows exactly 0 and -inf."""
        for name, want in self.want.items():
            x = got[name].double()
            assert x.shape == want.shape, name
            if name == "lse":
                assert torch.equal(x == -math.inf, ~self.any), "rows without keys"
                x, want = x[self.any], want[self.any]
                tol = self.tol[name][self.any]
            else:
                tol = self.tol[name]
            assert torch.isfinite(x).all(), f"{name}: not finite"
            off = (x - want).abs() - (1.01 * tol + TINY)
            assert not (off > 0).any(), (f"{name}: {int((off > 0).sum())} of {off.numel()} elements off by more than their "
                                         f"bound, the worst by {float(off.max()):.3g}; error {float((x - want).norm() / want.norm()):.3g}")
        empty = ~self.any.transpose(1, 2).repeat_interleave(64, 2)  # [B, nq, heads 64]
        assert (got["Y"][empty] == 0).all()
        if "dQ" in self.want:
            assert (got["dQ"][empty] == 0).all()
