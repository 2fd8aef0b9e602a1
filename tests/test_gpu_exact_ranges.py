"""Exact attention with values at the ends of their ranges, against
float64 element by element within the bounds of exact_testutil."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_exact import _check, _make  # noqa: E402

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
