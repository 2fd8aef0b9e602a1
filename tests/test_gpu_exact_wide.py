"""Exact attention, bfloat16, forward in blocks of 256 queries, against float64 element by element (the sizes are
checked against the launch rules in test_exact_launch_rules)."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_exact import _check, _make  # noqa: E402

WIDE = [  # B, nq, nk, heads, kv_heads, options
    (16, 256, 300, 16, 16, {}),
    (16, 250, 333, 16, 4, {}),
    (16, 256, 129, 16, 2, dict(kv_lens=[129, 1, 0, 64, 65, 33, 128, 2] * 2)),
    (8, 300, 300, 16, 16, dict(q_lens=[300, 257, 256, 255, 129, 1, 0, 299], kv_lens=[300, 7, 256, 64, 0, 300, 33, 299])),
    (16, 200, 400, 16, 8, dict(causal=True, q_pos=[200, 0, -60, 390] * 4)),
    (42, 129, 200, 6, 6, dict(causal=True)),
]


@pytest.mark.parametrize("shape", WIDE, ids=lambda s: "-".join(map(str, s[:5])) + "".join(f",{k}" for k in s[5]))
def test_wide_blocks(shape):
    B, nq, nk, heads, kv, kw = shape
    print(f"[case] wide {shape}", flush=True)
    _check(*_make("bf16", B, nq, nk, heads, kv, **kw), train=False)


SHARP = [(16, 256, 300, 16, 16, {}), (16, 250, 300, 16, 4, dict(kv_lens=[300, 250, 201, 1] * 4)), (16, 256, 300, 16, 16, dict(causal=True, q_pos=[44] * 16))]


@pytest.mark.parametrize("shape", SHARP, ids=lambda s: "-".join(map(str, s[:5])) + "".join(f",{k}" for k in s[5]))
def test_wide_blocks_redone(shape):
    """Logits far above those of a row's first 32 keys, for some of the rows: their sums pass 2^64, and their blocks take
    the pass again with a running maximum."""
    B, nq, nk, heads, kv, kw = shape
    print(f"[case] wide, sharp {shape}", flush=True)
    t, kw, bias = _make("bf16", B, nq, nk, heads, kv, q_scale=8.0, **kw)
    t["K"][:, 200:] *= 4
    t["K"][:, 299] *= 4
    _check(t, kw, bias, train=False)
