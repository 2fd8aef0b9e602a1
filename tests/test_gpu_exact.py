"""Exact attention, forward and backward, on the GPU against float64, element by element within
bounds derived from the inputs (exact_testutil)."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2201_12854_amd as mca  # noqa: E402
from exact_testutil import Case  # noqa: E402

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _make(dtype, B, nq, nk, heads, kv_heads, *, q_lens=None, kv_lens=None, q_pos=None, causal=False, window=0, buckets=0,
          max_distance=128, bidirectional=True, seed=0, q_scale=1.0):
    g = torch.Generator().manual_seed(seed + 7919 * nq + 104729 * nk + heads)
    new = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    dt = TYPES[dtype]
    t = dict(Q=q_scale * new(B, nq, heads * 64), K=new(B, nk, kv_heads * 64), V=new(B, nk, kv_heads * 64), dY=new(B, nq, heads * 64))
    t = {k: v.to(dt).to(DEV) for k, v in t.items()}
    ints = lambda v: None if v is None else torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    t["table"] = new(buckets, heads).to(dt).to(DEV) if buckets else None
    kw = dict(heads=heads, kv_heads=kv_heads, q_lens=ints(q_lens), kv_lens=ints(kv_lens), q_pos=ints(q_pos), causal=causal,
              window=window)
    return t, kw, dict(max_distance=max_distance, bidirectional=bidirectional)


def _run(t, kw, bias, train=True):
    b = None if t["table"] is None else mca.RelativeBias(t["table"], **bias)
    f = mca.exact_attention_forward(t["Q"], t["K"], t["V"], bias=b, **kw)
    got = dict(Y=f.Y, lse=f.lse)
    if train:
        g = mca.exact_attention_backward(t["dY"], t["Q"], t["K"], t["V"], f.Y, f.lse, bias=b, **kw)
        got.update(dQ=g.dQ, dK=g.dK, dV=g.dV)
        if b is not None:
            got["dbias"] = g.dbias
    torch.cuda.synchronize()
    return got


def _check(t, kw, bias, train=True):
    case = Case(t["Q"], t["K"], t["V"], dY=t["dY"] if train else None, table=t["table"], **kw, **bias)
    got = _run(t, kw, bias, train)
    case.check(got)
    return got


SHAPES = [  # B, nq, nk, heads, kv_heads, options
    (1, 1, 1, 1, 1, {}),
    (2, 1, 33, 4, 4, {}),
    (1, 31, 1, 3, 3, {}),
    (2, 32, 32, 4, 2, {}),
    (2, 33, 31, 2, 2, {}),
    (3, 65, 64, 6, 2, dict(kv_lens=[64, 1, 33])),
    (2, 128, 128, 12, 12, dict(q_lens=[128, 77], kv_lens=[128, 77])),
    (3, 100, 100, 4, 1, dict(q_lens=[100, 0, 3], kv_lens=[0, 100, 50])),
    (2, 97, 131, 5, 5, dict(causal=True)),
    (2, 130, 130, 8, 2, dict(causal=True, q_lens=[130, 50], kv_lens=[130, 50])),
    (2, 7, 300, 6, 2, dict(causal=True, q_pos=[293, 100], kv_lens=[300, 107])),
    (2, 40, 64, 4, 4, dict(causal=True, q_pos=[-20, 500])),
    (2, 200, 200, 4, 4, dict(window=32)),
    (3, 333, 333, 3, 3, dict(window=64, q_lens=[333, 120, 1], kv_lens=[333, 120, 1])),
    (2, 129, 257, 4, 2, dict(window=2, q_pos=[0, 128])),
    (2, 70, 200, 4, 4, dict(window=16, q_pos=[-30, 90])),
    (2, 150, 150, 2, 2, dict(window=30, causal=True)),
    (2, 40, 200, 2, 2, dict(window=30, causal=True, q_pos=[-10, 100])),
    (1, 513, 511, 2, 1, {}),
    # more than eight tiles to a block and a CU to each: eight waves
    (1, 1, 297, 4, 4, {}),
    (2, 330, 330, 4, 4, dict(kv_lens=[330, 290], q_lens=[330, 289])),
    (1, 300, 289, 6, 2, dict(causal=True)),
    (1, 500, 500, 3, 3, dict(window=40)),
    # up to 128 queries and keys, more of them than the card has CUs
    (30, 128, 128, 12, 12, dict(kv_lens=[128, 1, 0, 33, 64, 100] * 5, q_lens=[128, 1, 40, 0, 65, 97] * 5)),
    (60, 33, 64, 8, 8, dict(causal=True, q_pos=[0, 31, -40] * 20)),
    (40, 70, 90, 9, 9, dict(window=20, q_pos=[0, 15, -30, 60] * 10)),
    (300, 1, 2, 2, 2, {}),
    (40, 61, 50, 12, 3, dict(causal=True, kv_lens=[50, 7] * 20)),
    # up to 128 queries and keys: one launch for the gradients in bfloat16
    (3, 128, 100, 4, 4, dict(window=16, q_lens=[128, 33, 1], kv_lens=[100, 64, 2])),
    (2, 100, 128, 3, 3, dict(window=30, causal=True, q_pos=[28, -40])),
    (3, 127, 128, 5, 5, dict(causal=True, q_lens=[127, 96, 0], kv_lens=[128, 0, 65])),
    (2, 65, 97, 4, 4, dict(window=6, q_pos=[-33, 20])),
    (2, 1057, 1057, 2, 2, dict(window=256, q_lens=[1057, 353], kv_lens=[1057, 353])),
    # more blocks of 32 rows than CUs: bfloat16 in blocks of 128 rows
    (9, 129, 127, 8, 8, {}),
    (24, 1, 90, 12, 12, {}),
    (40, 33, 65, 8, 4, dict(kv_lens=[1 + b * 64 // 39 for b in range(40)])),
    (5, 321, 321, 8, 8, dict(causal=True, q_lens=[321, 200, 1, 0, 129], kv_lens=[321, 200, 1, 77, 0])),
    (4, 250, 400, 12, 4, dict(causal=True, q_pos=[150, 0, -60, 390])),
    (4, 333, 333, 9, 3, dict(window=64, q_lens=[333, 120, 1, 200], kv_lens=[333, 120, 1, 200])),
    (4, 300, 290, 9, 9, dict(window=30, causal=True, q_pos=[0, -10, 100, 5])),
    (3, 260, 520, 12, 12, dict(window=100, q_pos=[0, 260, -100])),
    # and of 256 queries: two rounds of 128 would not fill the card better
    (8, 256, 640, 16, 8, {}),
    (6, 500, 500, 16, 16, dict(causal=True, q_lens=[500, 100, 257, 256, 1, 499], kv_lens=[500, 100, 257, 256, 1, 499])),
    (6, 511, 333, 16, 16, dict(window=128)),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s[:5])) + "".join(f",{k}" for k in s[5]))
def test_against_float64(dtype, shape):
    B, nq, nk, heads, kv, kw = shape
    print(f"[case] {dtype} {shape}", flush=True)
    _check(*_make(dtype, B, nq, nk, heads, kv, **kw))


BIAS = [
    (1, 1, 1, 1, 1, dict(buckets=4, max_distance=8)),
    (2, 64, 64, 4, 4, dict(buckets=32)),
    (2, 201, 201, 8, 2, dict(buckets=16, max_distance=100, bidirectional=False, causal=True, q_lens=[201, 77], kv_lens=[201, 77])),
    (2, 90, 90, 2, 2, dict(buckets=8, max_distance=5, bidirectional=False)),  # keys ahead share bucket 0
    (2, 300, 310, 3, 1, dict(buckets=64, max_distance=256, q_pos=[0, 10])),
    (1, 700, 700, 2, 2, dict(buckets=32, max_distance=64)),  # tiles past max_distance on both sides
    (2, 5, 333, 8, 8, dict(buckets=32, bidirectional=False, causal=True, q_pos=[328, 35], kv_lens=[333, 40])),
    (2, 160, 160, 12, 1, dict(buckets=128, max_distance=256)),  # a group whose tables do not fit at once
    (2, 260, 260, 4, 4, dict(buckets=6, max_distance=216, window=64)),
    (3, 40, 40, 4, 4, dict(buckets=32, q_lens=[40, 0, 7], kv_lens=[40, 12, 0])),
    # more blocks of 32 rows than CUs
    (8, 200, 200, 8, 8, dict(buckets=32)),
    (3, 600, 500, 6, 2, dict(buckets=16, max_distance=40)),
    (4, 330, 330, 8, 2, dict(buckets=32, bidirectional=False, causal=True, q_lens=[330, 77, 1, 200], kv_lens=[330, 77, 1, 200])),
    (3, 300, 300, 12, 12, dict(buckets=64, max_distance=256, window=40, q_pos=[0, 3, 290])),
    (1, 1030, 1030, 12, 12, dict(buckets=32)),
    (3, 150, 190, 24, 1, dict(buckets=128, max_distance=256)),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", BIAS, ids=lambda s: "-".join(map(str, s[:5])) + f",D{s[5].get('max_distance', 128)}")
def test_relative_bias(dtype, shape):
    B, nq, nk, heads, kv, kw = shape
    print(f"[case] {dtype} {shape}", flush=True)
    _check(*_make(dtype, B, nq, nk, heads, kv, **kw))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,nq,nk,heads,kv,opt", [
    (1, 1, 1, 2, 2, {}),
    (2, 1, 1, 8, 2, dict(buckets=8)),
    (64, 1, 1, 12, 12, dict(buckets=32)),  # in bfloat16, blocks of 128 rows
    (64, 1, 1, 12, 3, {}),
    (3, 200, 130, 4, 4, dict(kv_lens=[1, 130, 0])),
    (4, 1, 300, 4, 2, dict(causal=True, buckets=8, bidirectional=False, q_pos=[0, 0, -3, 5])),
    (20, 300, 300, 8, 8, dict(causal=True)),
    (4, 40, 70, 3, 3, dict(window=10, q_pos=[-60, 75, 70, -20])),
    (80, 40, 70, 4, 4, dict(window=10, buckets=8, q_pos=[-60, 75, 70, -20] * 20)),
])
def test_rows_with_one_key(dtype, B, nq, nk, heads, kv, opt):
    """A row that attends one key has no gradient but dV's, and leaves no rounding in the others."""
    t, kw, bias = _make(dtype, B, nq, nk, heads, kv, **opt)
    print(f"[case] one key {dtype} {B} {nq} {nk} {heads} {kv} {opt}", flush=True)
    got = _check(t, kw, bias)
    i, j = torch.arange(nq, device=DEV), torch.arange(nk, device=DEV)
    pos = i[None] + (0 if kw["q_pos"] is None else kw["q_pos"][:, None])
    rel = j[None, None] - pos[:, :, None]
    ok = torch.ones(B, nq, nk, dtype=torch.bool, device=DEV)
    if kw["kv_lens"] is not None:
        ok &= (j[None] < kw["kv_lens"][:, None])[:, None]
    if kw["causal"]:
        ok &= rel <= 0
    if kw["window"]:
        ok &= (rel.abs() <= kw["window"] // 2) | (pos == 0)[:, :, None] | (j == 0)[None, None]
    one = ok.sum(-1) <= 1
    assert one.any()
    assert (got["dQ"][one] == 0).all()
    still = ~(ok & ~one[:, :, None]).any(1)  # keys that no other row attends
    assert (got["dK"][still] == 0).all()
    if one.all() and "dbias" in got:
        assert (got["dbias"] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("low", [float("-inf"), -1e30, "lowest"])
@pytest.mark.parametrize("B,heads", [(2, 3), (14, 5)])  # blocks of 32 and, in bfloat16, of 128 rows
def test_bias_that_masks(dtype, low, B, heads):
    """Buckets at -inf, -1e30 or the type's lowest value mask their pairs, whole rows among them."""
    t, kw, bias = _make(dtype, B, 150, 150, heads, heads, buckets=8, max_distance=20)
    low = torch.finfo(TYPES[dtype]).min if low == "lowest" else low
    t["table"][2] = low
    t["table"][:, 1] = low  # every pair of one head
    t["table"][4:, 2] = low  # the keys ahead of the query, and those that share its far bucket
    got = _check(t, kw, bias)
    assert (got["lse"][:, 1] == float("-inf")).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,kv,nq,nk", [(8, 2, 1, 5000), (4, 4, 3, 2049), (16, 1, 2, 4100), (1, 1, 1, 16384)])
def test_keys_split_over_blocks(dtype, heads, kv, nq, nk):
    print(f"[case] {dtype} {heads} {kv} {nq} {nk}", flush=True)
    pos = [nk - nq, nk // 3]
    _check(*_make(dtype, 2, nq, nk, heads, kv, causal=True, q_pos=pos, kv_lens=[nk, nk // 3 + nq]), train=False)
    _check(*_make(dtype, 2, nq, nk, heads, kv, kv_lens=[0, nk], buckets=32), train=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,heads,buckets", [(2, 2, 0), (18, 6, 0), (18, 6, 32), (18, 16, 0)])
def test_sharp_and_large_logits(dtype, B, heads, buckets):
    """Running maxima that rise late and far: logits of tens to hundreds, in blocks of 32, 128 and 256
    rows (there the sums pass 2^64 and the pass is taken again)."""
    nq = 256 if heads == 16 else 70
    t, kw, bias = _make(dtype, B, nq, 300, heads, heads, q_scale=8.0, buckets=buckets)
    t["K"][:, 200:] *= 4
    t["K"][:, 299] *= 4
    _check(t, kw, bias)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nan_behind_the_lengths(dtype):
    """Rows past the valid lengths are not read, whatever they hold; their results are 0."""
    t, kw, bias = _make(dtype, 3, 70, 90, 4, 2, q_lens=[70, 33, 0], kv_lens=[41, 90, 64], buckets=32)
    for b in range(3):
        t["Q"][b, kw["q_lens"][b]:] = float("nan")
        t["dY"][b, kw["q_lens"][b]:] = float("nan")
        t["K"][b, kw["kv_lens"][b]:] = float("nan")
        t["V"][b, kw["kv_lens"][b]:] = float("inf")
    got = _check(t, kw, bias)
    for b in range(3):
        assert (got["dK"][b, kw["kv_lens"][b]:] == 0).all() and (got["dV"][b, kw["kv_lens"][b]:] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides(dtype):
    """Slices of one projected tensor in and out, rows of a longer cache, one key set for the batch, and
    the [n, B, width] order; nothing outside the outputs' rows is written."""
    dt, B, n, H = TYPES[dtype], 2, 75, 4
    w = H * 64
    t, kw, bias = _make(dtype, B, n, n, H, H)
    packed = torch.cat([t["Q"], t["K"], t["V"]], -1)
    q, k, v = packed.split(w, -1)
    want = _check(t, kw, bias)
    f = mca.exact_attention_forward(q, k, v, **kw)
    assert torch.equal(f.Y, want["Y"]) and torch.equal(f.lse, want["lse"])
    dpacked = torch.full((B, n + 3, 3 * w + 16), 7.0, dtype=dt, device=DEV)
    outs = tuple(dpacked[:, :n, i * w:(i + 1) * w] for i in range(3))
    mca.exact_attention_backward(t["dY"], q, k, v, f.Y, f.lse, out=outs + (None,), **kw)
    for x, name in zip(outs, ("dQ", "dK", "dV")):
        assert torch.equal(x, want[name]), name
    assert (dpacked[:, n:] == 7).all() and (dpacked[:, :, 3 * w:] == 7).all()
    # sequence first
    s = {m: t[m].transpose(0, 1).contiguous().transpose(0, 1) for m in ("Q", "K", "V", "dY")}
    y = torch.empty(n, B, w, dtype=dt, device=DEV).transpose(0, 1)
    f = mca.exact_attention_forward(s["Q"], s["K"], s["V"], out=(y, torch.empty(B, H, n, device=DEV)), **kw)
    assert torch.equal(f.Y, want["Y"])
    # one set of keys for the whole batch: gradients come per batch row
    t["K"], t["V"] = t["K"][:1].expand(B, -1, -1), t["V"][:1].expand(B, -1, -1)
    assert t["K"].stride(0) == 0
    _check(t, kw, bias)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_offsets_past_32_bits(dtype):
    """A cache whose rows and batch rows start more than 4 GiB behind its beginning."""
    dt, H, n = TYPES[dtype], 2, 70
    pitch = (1 << 23) // dt.itemsize  # 8 MiB from row to row
    store = torch.empty((2 * 600 * pitch,), dtype=dt, device=DEV)
    K = store.as_strided((2, 600, H * 64), (600 * pitch, pitch, 1))
    V = store.as_strided((2, 600, H * 64), (600 * pitch, pitch, 1), H * 64)
    t, kw, bias = _make(dtype, 2, n, 600, H, H)
    K.copy_(t["K"])
    V.copy_(t["V"])
    t["K"], t["V"] = K, V
    _check(t, kw, bias)


def test_same_bits_again():
    """The same call gives the same bits, and a batch row's results do not depend on what the others hold
    (on how many there are they may: the sizes choose how sums are split)."""
    for dtype, heads in (("f32", 6), ("bf16", 6), ("bf16", 12)):
        t, kw, bias = _make(dtype, 3, 300, 300, heads, 2, buckets=32)
        a, b = _run(t, kw, bias), _run(t, kw, bias)
        for k in a:
            assert torch.equal(a[k], b[k]), k
        for k in ("Q", "K", "V", "dY"):
            t[k][::2] = t[k][::2].flip(1) * 3
        c = _run(t, kw, bias)
        for k in ("Y", "lse", "dQ", "dK", "dV"):
            assert torch.equal(a[k][1], c[k][1]), k


def test_differences():
    """Directional derivatives of sum(dY * Y) against central differences of the forward pass. Each
    difference quotient is off by its roundings (the bound of Y over 2 h) and by its truncation, which
    the step of twice the size shows (three times that of h, plus higher orders)."""
    t, kw, bias = _make("f32", 2, 37, 45, 4, 2, causal=True, q_pos=[8, 8], buckets=8, max_distance=16, bidirectional=False)
    case = Case(t["Q"], t["K"], t["V"], dY=t["dY"], table=t["table"], **kw, **bias)
    got = _run(t, kw, bias)
    g = torch.Generator().manual_seed(5)

    def loss(name, d, step):
        x = dict(t)
        x[name] = t[name] + step * d
        return float((_run(x, kw, bias, train=False)["Y"].double() * t["dY"].double()).sum())

    noise = 2 * float((case.tol["Y"] * t["dY"].double().abs()).sum())
    for name, grad in (("Q", "dQ"), ("K", "dK"), ("V", "dV"), ("table", "dbias")):
        # multiples of 2^-10 of one sign pattern: t + step d rounds, by at most half a step of t, which
        # moves the loss by the gradient times it
        d = (torch.randint(-8, 9, t[name].shape, generator=g).float() / 8).to(DEV)
        want = float((got[grad].double() * d.double()).sum())
        size = float((got[grad].double().abs() * (t[name].abs().double() + 1) * 2.0 ** -24).sum())
        h = 2.0 ** -6
        quotient = [(loss(name, d, s) - loss(name, d, -s)) / (2 * s) for s in (h, 2 * h)]
        off = abs(quotient[0] - want)
        assert off <= abs(quotient[1] - quotient[0]) + (noise + 2 * size) / (2 * h), (name, quotient, want)


def test_streams_and_graphs():
    """A side stream; a captured forward and backward pass replayed with new inputs and eager work
    between the replays."""
    t, kw, bias = _make("bf16", 2, 200, 200, 4, 4, buckets=32)
    want = _run(t, kw, bias)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _run(t, kw, bias)
    torch.cuda.current_stream().wait_stream(side)
    for k in want:
        assert torch.equal(got[k], want[k]), k
    plan = mca.ExactPlan(t["Q"], t["K"], t["V"], t["dY"], bias=mca.RelativeBias(t["table"], **bias), **kw)
    few = mca.ExactPlan(t["Q"][:, :1], t["K"], t["V"], **kw)
    graph = torch.cuda.CUDAGraph()
    plan.forward()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        plan.forward()
        plan.backward()
        few.forward()
    for seed in range(4):
        new, _, _ = _make("bf16", 2, 200, 200, 4, 4, buckets=32, seed=seed)
        for k in ("Q", "K", "V", "dY", "table"):
            t[k].copy_(new[k])
        graph.replay()
        torch.cuda.synchronize()
        want = _run(t, kw, bias)  # eager work between the replays
        for k in want:
            assert torch.equal(getattr(plan, k), want[k]), (seed, k)
        first = mca.exact_attention_forward(t["Q"][:, :1], t["K"], t["V"], **kw)
        torch.cuda.synchronize()
        assert torch.equal(few.Y, first.Y) and torch.equal(few.lse, first.lse)


def test_plan_matches_calls():
    for dtype in ("f32", "bf16"):
        t, kw, bias = _make(dtype, 2, 90, 90, 6, 3, causal=True)
        want = _run(t, kw, bias)
        plan = mca.ExactPlan(t["Q"], t["K"], t["V"], t["dY"], **kw)
        plan.forward()
        plan.backward()
        torch.cuda.synchronize()
        for k in want:
            assert torch.equal(getattr(plan, k), want[k]), k
        with pytest.raises(ValueError):
            p = mca.ExactPlan(t["Q"], t["K"], t["V"], **kw)
            p.backward()


def test_refusals():
    t, kw, bias = _make("bf16", 2, 32, 32, 4, 2)
    q, k, v = t["Q"], t["K"], t["V"]
    f = mca.exact_attention_forward(q, k, v, **kw)
    bad = [(q.float(), k, v, {}), (q, k.cpu(), v, {}), (q, k, v[:, :31], {}), (q[..., :-64], k, v, {}), (q.half(), k.half(), v.half(), {}),
           (q, k.transpose(1, 2), v, {}), (q[0], k, v, {}), (q, k, v, dict(kv_lens=torch.ones(3, dtype=torch.int32, device=DEV))),
           (q, k, v, dict(q_lens=torch.ones(2, dtype=torch.int64, device=DEV))), (q, k, v, dict(q_pos=torch.ones(2, dtype=torch.int32))),
           (q, k, v, dict(bias=mca.RelativeBias(torch.zeros(32, 4, device=DEV)))),
           (q, k, v, dict(bias=mca.RelativeBias(torch.zeros(32, 3, dtype=torch.bfloat16, device=DEV)))),
           (q, k, v, dict(out=(torch.empty_like(q), torch.empty(2, 4, 31, device=DEV))))]
    for a, b, c, more in bad:
        with pytest.raises((ValueError, TypeError)):
            mca.exact_attention_forward(a, b, c, **dict(kw, **more))
    with pytest.raises(mca.MCAError):  # rows that do not start at whole 16 bytes
        mca.exact_attention_forward(torch.zeros(2, 32, 260, dtype=torch.bfloat16, device=DEV)[..., :256], k, v, **kw)
    with pytest.raises(mca.MCAError):
        mca.exact_attention_forward(q, k, v, **dict(kw, scale=0.0))
    one = torch.empty(1, 32, 256, dtype=torch.bfloat16, device=DEV).expand(2, -1, -1)
    with pytest.raises(mca.MCAError):  # one set of rows for two results
        mca.exact_attention_forward(q, k, v, out=(one, f.lse), **kw)
    with pytest.raises(ValueError):
        mca.exact_attention_backward(t["dY"], q, k, v, f.Y, f.lse, **dict(kw, out=(q, k, v, q)))
    with pytest.raises(ValueError):
        mca.exact_attention_backward(t["dY"][:1], q, k, v, f.Y, f.lse, **kw)
