"""Exact attention in bfloat16: errors in norm, which show roundings that the element bounds of
test_gpu_exact (every rounding at its worst) leave room for.

A bfloat16 value m 2^e, 1 <= m < 2, is off by an error that is uniform in +-2^-8 2^e, in the root mean square
2^-8 / sqrt(3) of 2^e. Over values spread like a normal distribution of any width that is 0.737 of 2^-8 / sqrt(3) of
their norm, over uniform ones at most 0.78: STEP. One independent rounding of every term of a sum adds as much to the
sum's error in norm (terms of random signs), so a result that is rounded itself and is a sum of terms of which each was
rounded once is off by sqrt(2) STEP. 5% more for a sample of some thousand values; what is done in float32 is far
below. (test_exact_precision_limits has the same arithmetic on the CPU.)
"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from exact_testutil import Case  # noqa: E402
from test_gpu_exact import _make, _run  # noqa: E402

STEP = 1.05 * 0.78 * 2.0 ** -8 / 3 ** 0.5


def _errors(t, kw, bias, train=True):
    case = Case(t["Q"], t["K"], t["V"], dY=t["dY"] if train else None, table=t["table"], **kw, **bias)
    got = _run(t, kw, bias, train)
    case.check(got)
    # (a table's gradient has few elements, whose own rounding's root mean square is no sample of many)
    return {n: float((got[n].double() - w).norm() / w.norm()) for n, w in case.want.items() if n not in ("lse", "dbias")}


FEW = [  # B, nq, nk, heads, kv_heads, options: the same few keys or queries in calls of few and of many rows
    (2, 40, 2, 4, 4, {}),
    (300, 2, 2, 4, 4, {}),
    (64, 2, 2, 12, 12, {}),
    (64, 70, 3, 12, 12, {}),
    (32, 300, 2, 12, 12, {}),  # more queries than a block of 128
    (32, 300, 7, 12, 4, {}),
    (8, 600, 32, 8, 8, dict(window=16)),
    (64, 33, 5, 12, 3, dict(causal=True, q_pos=[b % 9 for b in range(64)])),
    (64, 2, 2, 12, 12, dict(buckets=8, max_distance=5)),
    (32, 200, 6, 12, 12, dict(buckets=8, max_distance=5)),
    (32, 200, 31, 12, 12, dict(buckets=32, window=10)),
    (24, 200, 30, 12, 12, dict(window=16, q_pos=[-70, 5, -33, 0] * 6)),  # a global query within a block
    (24, 200, 30, 12, 4, dict(window=16, q_pos=[-70, 5, -33, 0] * 6, buckets=8, max_distance=5)),
    (32, 30, 200, 12, 12, dict(window=16, q_pos=[-15, 40, 0, 150] * 8)),
    (1, 4100, 20, 2, 2, dict(window=16)),  # the query tiles in parts
    (1, 4100, 31, 4, 2, dict(buckets=8, max_distance=20, window=16)),
    (2, 2100, 9, 4, 1, dict(buckets=8, max_distance=20)),
    (2, 3, 100, 4, 4, {}),  # few queries
    (64, 3, 100, 12, 12, {}),
    (32, 2, 300, 12, 4, {}),
    (32, 32, 200, 12, 12, dict(window=16)),
    (32, 5, 300, 12, 12, dict(buckets=16, max_distance=100)),
    (16, 20, 520, 16, 4, dict(causal=True, buckets=16, max_distance=100, bidirectional=False, q_pos=[500] * 16)),
]


@pytest.mark.parametrize("q_scale", [0.25, 2.0])
@pytest.mark.parametrize("shape", FEW, ids=lambda s: "-".join(map(str, s[:5])) + "".join(f",{k}" for k in s[5]))
def test_few_keys_or_queries(shape, q_scale):
    """Up to 32 keys or queries P and dS enter the backward products with twice bfloat16's bits, up to 128 keys P the
    forward product, whatever the size of the batch: what is left is the results' own rounding."""
    B, nq, nk, heads, kv, kw = shape
    print(f"[case] few {shape} {q_scale}", flush=True)
    off = _errors(*_make("bf16", B, nq, nk, heads, kv, q_scale=q_scale, **kw))
    limits = {n: STEP for n in off}
    if nk > 128:
        limits["Y"] = 2 ** 0.5 * STEP
    print(off, flush=True)
    assert all(off[n] <= limits[n] for n in off), (off, limits)


@pytest.mark.parametrize("shape", [
    (2, 9, 128, 4, 4, {}),
    (64, 128, 128, 12, 12, {}),
    (40, 61, 50, 12, 3, {}),
    (16, 300, 100, 12, 12, {}),
    (16, 600, 128, 16, 16, {}),
    (16, 300, 90, 8, 8, dict(window=30)),
    (32, 128, 128, 12, 12, dict(buckets=32)),
    (16, 300, 65, 12, 12, dict(buckets=32, window=30)),
], ids=lambda s: "-".join(map(str, s[:5])) + "".join(f",{k}" for k in s[5]))
@pytest.mark.parametrize("q_scale", [0.25, 2.0])
def test_forward_of_128_keys(shape, q_scale):
    B, nq, nk, heads, kv, kw = shape
    print(f"[case] 128 keys {shape} {q_scale}", flush=True)
    off = _errors(*_make("bf16", B, nq, nk, heads, kv, q_scale=q_scale, **kw), train=False)
    print(off, flush=True)
    assert off["Y"] <= STEP, off


@pytest.mark.parametrize("shape", [
    (2, 300, 300, 3, 3, {}),  # blocks of 32 rows
    (2, 300, 300, 4, 1, {}),
    (8, 300, 300, 12, 12, {}),  # of 128
    (8, 300, 300, 12, 12, dict(causal=True)),
    (4, 700, 700, 12, 12, dict(window=256)),
    (8, 300, 300, 12, 12, dict(buckets=32)),
    (8, 128, 128, 12, 12, {}),  # one launch
    (3, 100, 100, 4, 4, {}),
], ids=lambda s: "-".join(map(str, s[:5])) + "".join(f",{k}" for k in s[5]))
def test_sharp_rows(shape):
    """Logits of standard deviation 4: with the D of the rounded Y the gradients of Q and K would be 4e-3 off."""
    B, nq, nk, heads, kv, kw = shape
    print(f"[case] sharp {shape}", flush=True)
    off = _errors(*_make("bf16", B, nq, nk, heads, kv, q_scale=4.0, **kw))
    print(off, flush=True)
    assert all(v <= 2 ** 0.5 * STEP for v in off.values()), off
