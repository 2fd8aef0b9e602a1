"""The stack with exact attention, forward and gradients, against float64 torch and its automatic
gradient: the operators together, as a training step calls them."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from exact_testutil import bucket  # noqa: E402
from paper_2201_12854_amd.stack import SyntheticEncoder  # noqa: E402

DEV = "cuda:0"


def _float64(enc, x, lens, window, d_out):
    """The same stack in float64, its result and gradients."""
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
    h = x
    for l in range(len(enc.layers)):
        q, k, v = ((h @ W).reshape(B, n, -1, 64).transpose(1, 2) for W in leaves[3 * l:3 * l + 3])
        s = q @ k.transpose(2, 3).contiguous() / 8 + add
        p = torch.softmax(s.masked_fill(~ok[:, None], -1e300), -1) * ok[:, None]
        h = torch.nn.functional.layer_norm(h + (p @ v).transpose(1, 2).reshape(B, n, d), (d,))
    grads = torch.autograd.grad(h, [x] + leaves + ([] if table is None else [table]), d_out.double())
    return h.detach(), grads


@pytest.mark.parametrize("window,buckets", [(0, 0), (0, 32), (16, 8)])
def test_stack_gradients(window, buckets):
    B, n, d, layers = 3, 50, 256, 2
    print(f"[case] window {window} buckets {buckets}", flush=True)
    enc = SyntheticEncoder(layers, d, 4, "f32", 5, relative_buckets=buckets, max_distance=20)
    g = torch.Generator().manual_seed(3)
    x, d_out = (torch.randn(B, n, d, generator=g).to(DEV) for _ in range(2))
    lens = torch.tensor([50, 17, 1], dtype=torch.int32, device=DEV)
    want, grads = _float64(enc, x, lens.long(), window, d_out)
    # In norm: a float32 sum of N terms is off by N u of the terms' magnitudes, which are at most sqrt(N) times
    # their sum's for signs in no order; N is at most 256 here (widths, rows and keys). A value has at most six
    # such sums a layer on its way forward and six back.
    u, N = 2.0 ** -24, 256
    tol = 12 * layers * N ** 1.5 * u
    near = lambda a, b: float((a.double() - b).norm() / b.norm())  # noqa: E731
    assert near(enc.exact_forward(x, lens, window=window), want) <= tol
    got = enc.gradients(x, d_out, lens, window=window)
    assert near(got["x"], grads[0]) <= tol
    for l in range(layers):
        for k, name in enumerate(("Wq", "Wk", "Wv")):
            assert near(got[name][l], grads[1 + 3 * l + k]) <= tol, (name, l)
    assert (got["bias"] is None) == (buckets == 0)
    if buckets:
        assert near(got["bias"], grads[-1]) <= tol
        with pytest.raises(ValueError):
            enc.forward(x, lens, 0.4)


def test_stack_matches_regular_mode():
    """The exact stack against the stack that runs every token's encoding exactly through the estimator's
    kernels: the same layer, rounded to bfloat16 in other places (in norm at most half a step, 2^-8, for
    V, H~, P twice, Y and the state of each of the layers)."""
    enc = SyntheticEncoder(2, 256, 4, "bf16", 1)
    x = torch.randn(2, 90, 256, generator=torch.Generator().manual_seed(1)).to(DEV).bfloat16()
    lens = torch.full((2,), 90, dtype=torch.int32, device=DEV)
    a, b = enc.exact_forward(x, lens).float(), enc.forward(x, lens, 0.4, exact=True).float()
    assert float((a - b).norm() / b.norm()) <= 2 * 6 * 2.0 ** -8
    grads = enc.gradients(x, torch.randn(2, 90, 256, device=DEV), lens)
    assert all(torch.isfinite(t).all() for t in [grads["x"]] + grads["Wq"] + grads["Wk"] + grads["Wv"])
