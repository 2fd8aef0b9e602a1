"""The stack's results and gradients with exact attention in norm: float32 against float64, bfloat16 against float64 that
is rounded where the stack holds bfloat16 tensors, so that what the backward pass rounds is left."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from exact_testutil import bucket  # noqa: E402
from paper_2201_12854_amd.stack import SyntheticEncoder  # noqa: E402

DEV = "cuda:0"


def _reference(enc, x, lens, window, d_out, rounding):
    """Result and gradients (x, then Wq, Wk, Wv of each layer, then the bias table) in float64; `rounding`: bfloat16 values
    of the projections, the attention's result and the hidden states, with the identity as its gradient."""
    B, n, d = x.shape
    leaves = [W.double().requires_grad_() for L in enc.layers for W in (L.Wq, L.Wk, L.Wv)]
    x = x.double().requires_grad_()
    i = torch.arange(n, device=x.device)
    rel = i[None, :] - i[:, None]
    ok = (i[None, :] < lens[:, None])[:, None, :] & (i[None, :] < lens[:, None])[:, :, None]
    if window:
        ok &= ((rel.abs() <= window // 2) | (i == 0)[:, None] | (i == 0)[None, :])[None]
    table, add = None, 0.0
    if enc.bias is not None:
        table = enc.bias.table.double().requires_grad_()
        top = enc.bias.max_distance
        at = torch.tensor([bucket(r, table.shape[0], top, True) for r in range(-top, top + 1)], device=x.device)
        add = table[at[rel.clamp(-top, top) + top]].permute(2, 0, 1)[None]

    def held(t):
        return t + (t.float().bfloat16().double() - t).detach() if rounding else t

    h = x
    for l in range(len(enc.layers)):
        q, k, v = (held(h @ W).reshape(B, n, -1, 64).transpose(1, 2) for W in leaves[3 * l:3 * l + 3])
        s = q @ k.transpose(2, 3).contiguous() / 8 + add
        p = torch.softmax(s.masked_fill(~ok[:, None], -1e300), -1) * ok[:, None]
        h = held(torch.nn.functional.layer_norm(h + held((p @ v).transpose(1, 2).reshape(B, n, d)), (d,)))
    grads = torch.autograd.grad(h, [x] + leaves + ([] if table is None else [table]), d_out.double())
    return h.detach(), grads


def _errors(dtype, window, buckets):
    B, n, d, layers = 3, 50, 256, 2
    enc = SyntheticEncoder(layers, d, 4, dtype, 5, relative_buckets=buckets, max_distance=20)
    g = torch.Generator().manual_seed(3)
    x, d_out = (torch.randn(B, n, d, generator=g).to(DEV).to(enc.dtype) for _ in range(2))
    lens = torch.tensor([50, 17, 1], dtype=torch.int32, device=DEV)
    want, grads = _reference(enc, x, lens.long(), window, d_out, dtype == "bf16")
    got = enc.gradients(x, d_out, lens, window=window)
    pairs = dict(out=(enc.exact_forward(x, lens, window=window), want), x=(got["x"], grads[0]))
    for l in range(layers):
        for k, name in enumerate(("Wq", "Wk", "Wv")):
            pairs[f"{name}{l}"] = (got[name][l], grads[1 + 3 * l + k])
    if buckets:
        pairs["bias"] = (got["bias"], grads[-1])
    return layers, {n: float((a.double() - b).norm() / b.norm()) for n, (a, b) in pairs.items()}


CASES = [(0, 0), (0, 32), (16, 8)]


@pytest.mark.parametrize("window,buckets", CASES)
def test_stack_float32(window, buckets):
    """A float32 sum of N terms of random signs is off by N independent roundings of partial sums, none of them larger in
    the mean than the result: at most sqrt(N) u in norm, u = 2^-24. N is at most 256 (widths, rows and keys), and a value
    passes at most six such sums a layer on its way forward and six back."""
    layers, off = _errors("f32", window, buckets)
    print(f"[case] stack f32 {window} {buckets}: {off}", flush=True)
    limit = 12 * layers * 16 * 2.0 ** -24
    assert all(v <= limit for v in off.values()), (off, limit)


@pytest.mark.parametrize("window,buckets", CASES)
def test_stack_bfloat16(window, buckets):
    """A layer's backward pass rounds dY, dS (or P) and its results to bfloat16, each by STEP in norm (derived in
    test_gpu_exact_precision): 3 STEP a layer. The forward pass rounds as the reference does (up to 128 keys P is
    multiplied to twice bfloat16's bits); a value next to a border that falls on its other side is one of thousands and
    moves the result by far less."""
    layers, off = _errors("bf16", window, buckets)
    print(f"[case] stack bf16 {window} {buckets}: {off}", flush=True)
    limit = 3 * layers * 1.05 * 0.78 * 2.0 ** -8 / 3 ** 0.5
    assert all(v <= limit for v in off.values()), (off, limit)
