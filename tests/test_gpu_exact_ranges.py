"""Exact attention with values at the ends of their ranges, against
float64 element by element within the bounds of exact_testutil."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2201_12854_amd as mca  # noqa: E402
from exact_testutil import Case  # noqa: E402
from paper_2201_12854_amd import binding  # noqa: E402
from test_gpu_exact import _check, _make, _run  # noqa: E402

LARGE = [  # B, nq, nk, heads, kv_heads, options; query counts that are no multiple of 32 or 64
    (2, 50, 70, 4, 4, {}),
    (8, 200, 200, 8, 8, {}),  # in bfloat16 in blocks of 128 keys, as most below
    (8, 230, 200, 8, 8, dict(q_lens=[230, 1, 33, 95, 0, 129, 200, 64], kv_lens=[200, 1, 33, 95, 7, 129, 0, 64])),
    (4, 330, 330, 8, 2, dict(causal=True, bidirectional=False)),
    (3, 300, 300, 12, 12, dict(window=40)),
    (2, 1030, 300, 8, 2, {}),  # the query tiles of a key head in parts
    (64, 1, 5, 12, 12, {}),
    (6, 333, 333, 9, 9, dict(causal=True, bidirectional=False, q_lens=[333, 300, 97, 64, 1, 0], kv_lens=[333] * 6)),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", LARGE, ids=lambda s: "-".join(map(str, s[:5])) + "".join(f",{k}" for k in s[5]))
def test_large_bias(dtype, shape):
    """A softmax does not see a shift of its logits: a head all of whose biases are 100, or -100, has the gradients
    that it has without, and a bucket at 200 gets all of its rows' weight. (exp(89) is past float32.)"""
    B, nq, nk, heads, kv, kw = shape
    print(f"[case] large bias {dtype} {shape}", flush=True)
    t, kw, bias = _make(dtype, B, nq, nk, heads, kv, buckets=8, max_distance=20, **kw)
    t["table"][:, 0] += 100
    t["table"][:, 1] -= 100
    t["table"][1, 2] = 200  # near keys on one side
    t["table"][3, 3] = 150  # those further than 20 tokens
    _check(t, kw, bias)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [-1e9, 1e7, -2e29])
@pytest.mark.parametrize("shape", [LARGE[0], LARGE[1], LARGE[3], LARGE[4], LARGE[7], (64, 1, 5, 12, 12, {}), (2, 20, 20, 3, 3, {})],
                         ids=lambda s: "-".join(map(str, s[:5])) + "".join(f",{k}" for k in s[5]))
def test_rows_past_the_range_of_lse(dtype, shift, shape):
    """A head that is masked by a large finite bias instead of -1e30: float32 no longer has the log-sum-exp that the
    gradients start from. They are 0 there, not infinite, and what the other heads get of shared keys stays right."""
    B, nq, nk, heads, kv, kw = shape
    print(f"[case] lse past 2^22 {dtype} {shift} {shape}", flush=True)
    t, kw, bias = _make(dtype, B, nq, nk, heads, kv, buckets=8, max_distance=20, **kw)
    t["table"][:, 0] = shift
    got = _run(t, kw, bias)
    assert torch.isfinite(got["Y"]).all()
    assert (got["dQ"][..., :64] == 0).all() and (got["dbias"][:, 0] == 0).all()
    # the same call with that head masked altogether
    t["table"][:, 0] = -1e30
    case = Case(t["Q"], t["K"], t["V"], dY=t["dY"], table=t["table"], **kw, **bias)
    got.update(Y=got["Y"].clone(), lse=got["lse"].clone())
    got["Y"][..., :64] = 0
    got["lse"][:, 0] = float("-inf")
    case.check(got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", LARGE[:2] + LARGE[4:6], ids=lambda s: "-".join(map(str, s[:5])) + "".join(f",{k}" for k in s[5]))
def test_shift_of_ten_thousand(dtype, shape):
    B, nq, nk, heads, kv, kw = shape
    print(f"[case] shift of 1e4 {dtype} {shape}", flush=True)
    t, kw, bias = _make(dtype, B, nq, nk, heads, kv, buckets=8, max_distance=20, **kw)
    t["table"][:, 0] = -10000.0
    t["table"][:, 1] = 10000.0
    _check(t, kw, bias)


SCALED = [
    (2, 50, 70, 4, 4, {}),
    (3, 100, 100, 6, 6, dict(causal=True)),  # bfloat16: the gradients in one launch
    (30, 64, 64, 12, 12, {}),
    (8, 200, 200, 8, 8, {}),
    (3, 300, 300, 12, 12, dict(window=40)),
    (8, 200, 200, 8, 8, dict(buckets=8, max_distance=20)),
    (2, 3, 2100, 8, 2, dict(causal=True, q_pos=[2097, 5])),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [2.0 ** -100, 2.0 ** -20, 0.01, 1.0, 3.7])
@pytest.mark.parametrize("shape", SCALED, ids=lambda s: "-".join(map(str, s[:5])) + "".join(f",{k}" for k in s[5]))
def test_scales(dtype, scale, shape):
    B, nq, nk, heads, kv, kw = shape
    print(f"[case] scale {scale} {dtype} {shape}", flush=True)
    t, kw, bias = _make(dtype, B, nq, nk, heads, kv, **kw)
    kw["scale"] = scale
    case = Case(t["Q"], t["K"], t["V"], dY=t["dY"], table=t["table"], **kw, **bias)
    # Steep rows have P below the smallest normal number 2^-126, which exp2 may return as 0: an error of f = 2^-126
    # in each P, and so of f max|v| in each of y's nk terms, f max|dy| in each of dv's G nq; of f (|dP| + |D|) in
    # each dS, |dP| and |D| being at most 64 max|dy| max|v| (y is an average of v), hence in each of the nk terms of dq
    # and the G nq of dk that times scale max|k| and scale max|q|.
    f, G = 2.0 ** -126, heads // kv
    q, k, v, dy = (float(t[n].abs().max()) for n in ("Q", "K", "V", "dY"))
    lost = f * 128 * dy * v
    for name, x in dict(Y=nk * f * v, dV=G * nq * f * dy, dQ=scale * nk * lost * k, dK=scale * G * nq * lost * q,
                        dbias=B * nq * nk * lost).items():
        if name in case.tol:
            case.tol[name] = case.tol[name] + x
    case.check(_run(t, kw, bias))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_small_scales_refused(dtype):
    """Below 2^-100 (the bfloat16 backward pass starts its sums at -lse / scale)."""
    t, kw, bias = _make(dtype, 2, 32, 32, 4, 4)
    f = mca.exact_attention_forward(t["Q"], t["K"], t["V"], **kw)
    for scale in (2.0 ** -100 * (1 - 2.0 ** -52), 1e-35, 1e-38):
        for call in (lambda: mca.exact_attention_forward(t["Q"], t["K"], t["V"], **dict(kw, scale=scale)),
                     lambda: mca.exact_attention_backward(t["dY"], t["Q"], t["K"], t["V"], f.Y, f.lse, **dict(kw, scale=scale))):
            with pytest.raises(mca.MCAError) as e:
                call()
            assert e.value.status == binding.MCA_ERR_INVALID_ARGUMENT


def test_wide_window_refused():
    t, kw, bias = _make("bf16", 2, 32, 32, 4, 4)
    for window in (2**64, 2**64 + 2, -2**64 + 2):
        with pytest.raises(ValueError):
            mca.exact_attention_forward(t["Q"], t["K"], t["V"], **dict(kw, window=window))
        with pytest.raises(ValueError):
            mca.ExactPlan(t["Q"], t["K"], t["V"], **dict(kw, window=window))
    with pytest.raises(mca.MCAError):
        mca.exact_attention_forward(t["Q"], t["K"], t["V"], **dict(kw, window=2**63 - 1))
