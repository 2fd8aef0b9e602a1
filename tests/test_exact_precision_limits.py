"""The limits of test_gpu_exact_precision on the CPU: the arithmetic of the bfloat16 kernels, rounded where they
round and in float64 elsewhere, stays below them, and would not without the exact D or without the second products."""
import pytest

torch = pytest.importorskip("torch")

STEP = 1.05 * 0.78 * 2.0 ** -8 / 3 ** 0.5  # of one rounding, in norm


def _bf16(x):
    return x.float().bfloat16().double()


def _twice(x):  # the value and what its rounding took off, each in bfloat16
    return _bf16(x) + _bf16(x - _bf16(x))


def _attention(nq, nk, heads, q_scale, operand, exact_d, seed=0):
    """Errors in norm of Y, dQ, dK, dV: P and dS enter their products through `operand`, D comes from the rounded Y or
    from the sums of dS."""
    g = torch.Generator().manual_seed(seed)
    new = lambda n, s=1.0: _bf16(s * torch.randn(heads, n, 64, generator=g, dtype=torch.float64))  # noqa: E731
    q, k, v, dy = new(nq, q_scale), new(nk), new(nk), new(nq)
    P = torch.softmax(q @ k.transpose(1, 2) / 8, -1)
    T = lambda x: x.transpose(1, 2)  # noqa: E731
    dP = dy @ T(v)
    y = P @ v
    dS = P * (dP - (dy * y).sum(-1, keepdim=True))
    want = dict(Y=y, dQ=dS @ k / 8, dK=T(dS) @ q / 8, dV=T(P) @ dy)
    Y = _bf16(operand(P) @ v)
    D = (dy * Y).sum(-1, keepdim=True)
    dS = P * (dP - D)
    dQ = operand(dS) @ k
    if exact_d:
        rest = dS.sum(-1, keepdim=True)
        dQ = dQ - rest * (_bf16(P) @ k)
        dS = P * (dP - (D + rest))
    got = dict(Y=Y, dQ=_bf16(dQ / 8), dK=_bf16(T(operand(dS)) @ q / 8), dV=_bf16(T(operand(P)) @ dy))
    return {n: float((got[n] - want[n]).norm() / want[n].norm()) for n in want}


@pytest.mark.parametrize("width", [1.0, 1.3, 1.9])
def test_one_rounding(width):
    x = width * torch.randn(100000, generator=torch.Generator().manual_seed(1), dtype=torch.float64)
    for x in (x, x * x, x.sign() * x.abs().exp(), 2 * width * torch.rand(100000, generator=torch.Generator().manual_seed(2), dtype=torch.float64)):
        assert float((_bf16(x) - x).norm() / x.norm()) <= STEP


@pytest.mark.parametrize("nq,nk", [(300, 300), (128, 128)])
def test_exact_d(nq, nk):
    limit = 2 ** 0.5 * STEP
    assert all(v <= limit for v in _attention(nq, nk, 6, 4.0, _bf16, True).values())
    without = _attention(nq, nk, 6, 4.0, _bf16, False)
    assert min(without["dQ"], without["dK"]) > 1.3 * limit


@pytest.mark.parametrize("nq,nk", [(300, 2), (2, 300), (300, 7), (40, 2)])
def test_second_products(nq, nk):
    limit = STEP
    heads = 24
    off = _attention(nq, nk, heads, 0.25, _twice, True)
    assert all(v <= limit for v in off.values()), off
    once = _attention(nq, nk, heads, 0.25, _bf16, True)
    assert min(once.values()) > 1.2 * limit, once
