"""Exact softmax attention with its gradient, and the learned relative position bias, as cases
that can be timed and checked.

The operators are the attention layer that MCA approximates, as it is trained and as single tokens
are served: ``Y_h = softmax(scale Q_h K_h^T + bias_h) V_h`` with the row log-sum-exp, its backward
pass (dQ, dK, dV and the bias table's gradient) and the form for few queries over many keys. A case
is one call, or for ``do`` "train" a forward and a backward call. Where ``own`` is false ``run``
takes the plain form: the probabilities as a matrix, in float32 torch. ``exact`` is float64 torch
with its own automatic gradient.

The bias adds ``table[bucket(j - p), h]`` to the logit of the query at position p and the key at j:
half of the buckets for j > p where it is bidirectional; the first half of those (E) for single
distances, the rest (m of them) logarithmically up to ``max_distance`` D: distance d >= E is in the
largest bucket E + k, k < m, with d >= E (D / E)^(k / m).
"""
import math

import torch

own = False

D_HEAD = 64

DEFAULTS = dict(do="forward", entry="plan", dtype="bf16", batch=1, q=128, k=128, heads=12, kv_heads=12, causal=False,
                window=0, len_lo=0, len_hi=0, packed=False, buckets=0, max_distance=128, bidirectional=True, q_scale=1.0)


def _case(name, **kw):
    c = dict(DEFAULTS)
    c.update(kw)
    if name:
        c = dict(name=name, **c)
    return c


def listed():
    return [
        # one new token of one sequence against its keys: the latency of a served token
        _case("row_bf16_b1_k701", q=1, k=701, causal=True),
        # a served batch of long sequences of different lengths with shared key heads: the cache is
        # read once
        _case("row_bf16_b32_k16384_kv4", batch=32, q=1, k=16384, heads=16, kv_heads=4, causal=True, len_lo=2048,
              len_hi=16384),
        # a few tokens at a time behind a cached prefix, with the causal position bias, through the
        # plain call
        _case("rows_f32_b4_q5_k333_bias", entry="call", dtype="f32", batch=4, q=5, k=333, heads=8, kv_heads=8,
              causal=True, len_lo=40, len_hi=333, buckets=32, bidirectional=False),
        # the smallest layer of the benchmark, in float32
        _case("forward_f32_b1_s128", dtype="f32"),
        # a batch of sentences of very different lengths padded to 128
        _case("forward_bf16_b64_padded", batch=64, len_lo=16, len_hi=128),
        # the benchmark's long layer
        _case("forward_bf16_b4_s4096", batch=4, q=4096, k=4096),
        # a fine-tuning step's attention in float32, ragged documents of an odd padded length
        _case("train_f32_b2_s333", do="train", dtype="f32", batch=2, q=333, k=333, len_lo=100, len_hi=333),
        # the BERT-base classification batch, Q, K and V in one projected tensor
        _case("train_bf16_b32_s128", do="train", batch=32, packed=True),
        # documents through a local window of 256 keys with a global first token
        _case("train_bf16_b8_s1057_window", do="train", batch=8, q=1057, k=1057, window=256, len_lo=353, len_hi=1057),
        # an encoder with a bidirectional position bias
        _case("train_bf16_b16_s512_bias", do="train", batch=16, q=512, k=512, buckets=32),
        # a small decoder with shared key heads and a causal position bias, float32, odd lengths
        _case("train_f32_b4_s201_bias", do="train", dtype="f32", batch=4, q=201, k=201, heads=8, kv_heads=2, causal=True,
              len_lo=77, len_hi=201, buckets=16, max_distance=100, bidirectional=False),
        # the benchmark's long layer, trained
        _case("train_bf16_b4_s4096", do="train", batch=4, q=4096, k=4096),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Another call of the same ranges: 1 to 4096 queries (a few of them against up to 16384 keys),
    1 to 64 rows of a batch, 1 to 16 heads with 1 to 16 key heads."""
    f32 = rng.random() < 0.3
    heads, kv = rng.choice([(12, 12), (12, 12), (16, 16), (16, 4), (8, 2), (8, 1), (12, 3), (4, 4), (5, 5), (6, 2)])
    do = rng.choice(["row", "forward", "train", "train"])
    c = dict(dtype="f32" if f32 else "bf16", heads=heads, kv_heads=kv, q_scale=rng.choice([0.5, 1.0, 2.0]))
    if do == "row":
        c["q"] = rng.choice([1, 1, 1, 2, 3, 7, 16])
        c["k"] = _log_uniform(rng, 16, 16384)
        c["causal"] = True
        # at most the largest listed cache
        most = 32 * 16384 * 4 // (c["k"] * kv * (2 if f32 else 1))
        c["batch"] = max(1, min(most, _log_uniform(rng, 1, 64)))
    else:
        c["do"] = do
        c["q"] = c["k"] = _log_uniform(rng, 1, 4096 if not f32 else 1024)
        # at most the largest listed case's pairs (a sixteenth of them in float32)
        most = 4 * 4096 * 4096 * 12 // (c["q"] * c["k"] * heads * (16 if f32 else 1))
        c["batch"] = max(1, min(most, 16384 // c["q"], _log_uniform(rng, 1, 64)))
        c["causal"] = rng.random() < 0.3
        if not c["causal"] and c["q"] >= 100 and rng.random() < 0.25:
            c["window"] = rng.choice([32, 64, 256])
        c["packed"] = kv == heads and rng.random() < 0.3
    if rng.random() < 0.5 and c["k"] >= 16:
        c["len_lo"], c["len_hi"] = max(c["q"] if do == "row" else 1, c["k"] // rng.randint(2, 8)), c["k"]
        c["len_lo"] = min(c["len_lo"], c["len_hi"])
    if rng.random() < 0.35 and c["q"] * c["k"] <= 1024 * 1024:
        c["buckets"] = rng.choice([8, 16, 32, 32, 64])
        c["max_distance"] = rng.choice([64, 100, 128, 128, 256])
        c["bidirectional"] = not c["causal"]
    if c["batch"] * c["q"] <= 512 and rng.random() < 0.5:
        c["entry"] = "call"
    return _case(None, **c)


def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _lengths(case):
    """The valid lengths of the batch's rows: spread evenly over len_lo .. len_hi."""
    B, lo, hi = case["batch"], case["len_lo"], case["len_hi"]
    if not hi:
        return [case["k"]] * B
    return [hi if B == 1 else hi - (hi - lo) * b // (B - 1) for b in range(B)]


def _inputs(case, seed):
    """Q, K, V of the layer's type (slices of one tensor where they are packed), dY, the bias table and
    the rows' lengths and first positions."""
    dev, dt = torch.device("cuda:0"), _type(case)
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    B, nq, nk, wq, wk = case["batch"], case["q"], case["k"], case["heads"] * D_HEAD, case["kv_heads"] * D_HEAD

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev, dtype=torch.float32)

    t = {"case": case}
    if case["packed"]:
        x = normal(B, nq, wq + 2 * wk)
        x[..., :wq] *= case["q_scale"]
        t["Q"], t["K"], t["V"] = x.to(dt).split([wq, wk, wk], dim=-1)
    else:
        t["Q"] = (case["q_scale"] * normal(B, nq, wq)).to(dt)
        t["K"], t["V"] = normal(B, nk, wk).to(dt), normal(B, nk, wk).to(dt)
    t["dY"] = normal(B, nq, wq).to(dt) if case["do"] == "train" else None
    t["table"] = normal(case["buckets"], case["heads"]).to(dt) if case["buckets"] else None
    order = torch.randperm(B, generator=g, device=dev)
    lens = torch.tensor(_lengths(case), dtype=torch.int32, device=dev)[order].contiguous()
    ragged = case["len_hi"] > 0
    t["kv_lens"] = lens if ragged else None
    if nq == nk:
        t["q_lens"], t["q_pos"] = t["kv_lens"], None
    else:  # the queries are the last ones of their rows
        t["q_lens"], t["q_pos"] = None, lens - nq
    return t


def prepare(case, seed):
    t = _inputs(case, seed)
    if own and case["entry"] == "plan":
        import paper_2201_12854_amd as mca

        t["plan"] = mca.ExactPlan(t["Q"], t["K"], t["V"], t["dY"], **_arguments(t))
    return t


def _arguments(t):
    import paper_2201_12854_amd as mca

    c = t["case"]
    bias = None
    if t["table"] is not None:
        bias = mca.RelativeBias(t["table"], c["max_distance"], c["bidirectional"])
    return dict(heads=c["heads"], kv_heads=c["kv_heads"], q_lens=t["q_lens"], kv_lens=t["kv_lens"], q_pos=t["q_pos"],
                causal=c["causal"], window=c["window"], bias=bias)


def run(t):
    if not own:
        return _plain(t)
    train = t["case"]["do"] == "train"
    if "plan" in t:
        p = t["plan"]
        p.forward()
        if train:
            p.backward()
        got = {"Y": p.Y, "lse": p.lse}
        grads = p
    else:
        import paper_2201_12854_amd as mca

        kw = _arguments(t)
        f = mca.exact_attention_forward(t["Q"], t["K"], t["V"], **kw)
        got = {"Y": f.Y, "lse": f.lse}
        if train:
            grads = mca.exact_attention_backward(t["dY"], t["Q"], t["K"], t["V"], f.Y, f.lse, **kw)
    if train:
        got.update(dQ=grads.dQ, dK=grads.dK, dV=grads.dV)
        if t["table"] is not None:
            got["dbias"] = grads.dbias
    return got


# ------------------------------------------------------------------ the plain form
def _pairs(t):
    """Which (query, key) pairs attend, [B, nq, nk], and their key minus query positions."""
    c, dev = t["case"], t["Q"].device
    i = torch.arange(c["q"], device=dev)[None, :, None]
    j = torch.arange(c["k"], device=dev)[None, None, :]
    p = i if t["q_pos"] is None else i + t["q_pos"].long()[:, None, None]
    ok = (j >= 0) & (p == p)
    if t["kv_lens"] is not None:
        ok = ok & (j < t["kv_lens"][:, None, None])
    if t["q_lens"] is not None:
        ok = ok & (i < t["q_lens"][:, None, None])
    if c["causal"]:
        ok = ok & (j <= p)
    if c["window"]:
        ok = ok & (((p - j).abs() <= c["window"] // 2) | (p == 0) | (j == 0))
    return ok, j - p


def _bucket(rel, buckets, max_distance, bidirectional):
    n = buckets // 2 if bidirectional else buckets
    side = (rel > 0).long() * n if bidirectional else 0
    d = rel.abs() if bidirectional else (-rel).clamp(min=0)
    e = n // 2
    # in 64 bits, with a little on top: distances on a border belong to the bucket that begins there
    far = torch.log(d.clamp(min=1).double() / e) / math.log(max_distance / e) * (n - e) + 1e-9
    far = (e + far.floor().long()).clamp(max=n - 1)
    return side + torch.where(d < e, d, far)


def _heads(x, heads):
    B, n, _ = x.shape
    return x.float().reshape(B, n, -1, D_HEAD).transpose(1, 2).repeat_interleave(heads // (x.shape[2] // D_HEAD), 1).contiguous()


def _rows(x):
    return x.transpose(1, 2).reshape(x.shape[0], x.shape[2], -1)


def _plain(t):
    c, dt = t["case"], t["Q"].dtype
    H, G, scale = c["heads"], c["heads"] // c["kv_heads"], 1.0 / math.sqrt(D_HEAD)
    Q, K, V = (_heads(t[k], H) for k in ("Q", "K", "V"))
    ok, rel = _pairs(t)
    S = torch.matmul(Q, K.transpose(2, 3).contiguous()) * scale
    if t["table"] is not None:
        bucket = _bucket(rel, c["buckets"], c["max_distance"], c["bidirectional"])
        S = S + t["table"].float()[bucket].permute(0, 3, 1, 2)
    S = S.masked_fill(~ok[:, None], -math.inf)
    M = S.amax(-1, keepdim=True)
    P = torch.exp(S - M.masked_fill(M == -math.inf, 0.0))
    L = P.sum(-1, keepdim=True)
    P = P / L.masked_fill(L == 0, 1.0)
    del S
    got = {"Y": _rows(torch.matmul(P, V)).to(dt), "lse": (M + torch.log(L)).squeeze(-1)}
    if c["do"] != "train":
        return got
    dY = _heads(t["dY"], H)
    if t["q_lens"] is not None:  # padded queries have no gradient
        dY = dY * (torch.arange(c["q"], device=dY.device)[None, :] < t["q_lens"][:, None])[:, None, :, None]
    dV = torch.matmul(P.transpose(2, 3), dY)
    dP = torch.matmul(dY, V.transpose(2, 3).contiguous())
    dS = P * (dP - (P * dP).sum(-1, keepdim=True))
    del P, dP
    got["dQ"] = _rows(torch.matmul(dS, K) * scale).to(dt)
    dK = torch.matmul(dS.transpose(2, 3), Q) * scale
    B, nk = c["batch"], c["k"]
    got["dK"] = _rows(dK.reshape(B, H // G, G, nk, D_HEAD).sum(2)).to(dt)
    got["dV"] = _rows(dV.reshape(B, H // G, G, nk, D_HEAD).sum(2)).to(dt)
    if t["table"] is not None:  # the positions are the same in every row of the batch; a long sum
        one = torch.nn.functional.one_hot(bucket[0].reshape(-1), c["buckets"]).double()
        got["dbias"] = torch.matmul(dS.double().sum(0).reshape(H, -1), one).t().contiguous().to(dt)
    return got


# ------------------------------------------------------------------ work and float64
def _attended(case):
    """Attended (query, key) pairs of one head over the batch."""
    nq, total = case["q"], 0
    for n in _lengths(case):
        if nq != case["k"]:
            first = n - nq  # causal: query i of the last nq sees first + i + 1 keys
            total += sum(min(n, first + i + 1) for i in range(nq)) if case["causal"] else nq * n
        elif case["window"]:
            h = case["window"] // 2
            for p in range(n):
                lo, hi = (max(0, p - h), min(n - 1, p + h)) if p else (0, n - 1)
                total += hi - lo + 1 + (1 if lo > 0 else 0)
        else:
            total += n * (n + 1) // 2 if case["causal"] else n * n
    return total


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    keys = sum(_lengths(case))
    queries = keys if case["q"] == case["k"] else case["q"] * case["batch"]
    qrow, krow = case["heads"] * D_HEAD * es, case["kv_heads"] * D_HEAD * es
    # Q, K, V read, Y and the log-sum-exp written
    nbytes = 2 * queries * qrow + 2 * keys * krow + 4 * queries * case["heads"]
    flops = 4.0 * D_HEAD * case["heads"] * _attended(case)
    if case["do"] == "train":  # Q, K, V, Y, dY and the log-sum-exp read, dQ, dK, dV written; five products
        nbytes += 4 * queries * qrow + 4 * keys * krow + 4 * queries * case["heads"]
        flops *= 3.5
    if case["buckets"]:
        nbytes += case["buckets"] * case["heads"] * es * (3 if case["do"] == "train" else 1)
    return {"bytes": nbytes, "flops": flops}


def _bucket_of(d, n, max_distance):
    """Bucket of distance d among n one-sided buckets, in whole numbers."""
    e = n // 2
    if d < e:
        return d
    m, k = n - e, 0
    while k + 1 < m and d ** m * e ** (k + 1) >= e ** m * max_distance ** (k + 1):
        k += 1
    return e + k


def exact(case, seed):
    t = _inputs(case, seed)
    c, dev = case, t["Q"].device
    H, Hk, nq, nk = c["heads"], c["kv_heads"], c["q"], c["k"]
    train = c["do"] == "train"
    out = {"Y": [], "lse": []}
    if train:
        out.update(dQ=[], dK=[], dV=[])
    table = t["table"].double().requires_grad_(train) if t["table"] is not None else None
    if table is not None:
        n = c["buckets"] // 2 if c["bidirectional"] else c["buckets"]
        near = [_bucket_of(d, n, c["max_distance"]) for d in range(c["max_distance"] + 1)]
        left = torch.tensor(near, device=dev)
    dbias = 0.0
    for b in range(c["batch"]):
        x = {k: t[k][b].double().requires_grad_(train) for k in ("Q", "K", "V")}
        pos = torch.arange(nq, device=dev) + (0 if t["q_pos"] is None else int(t["q_pos"][b]))
        key = torch.arange(nk, device=dev)
        keys = nk if t["kv_lens"] is None else int(t["kv_lens"][b])
        rows = nq if t["q_lens"] is None else int(t["q_lens"][b])
        ok = (key < keys)[None, :] & (torch.arange(nq, device=dev) < rows)[:, None]
        back = pos[:, None] - key[None, :]
        if c["causal"]:
            ok &= back >= 0
        if c["window"]:
            ok &= (back.abs() <= c["window"] // 2) | (pos == 0)[:, None] | (key == 0)[None, :]
        q = x["Q"].reshape(nq, Hk, H // Hk, D_HEAD).permute(1, 2, 0, 3)
        k = x["K"].reshape(nk, Hk, D_HEAD).permute(1, 2, 0)[:, None]
        v = x["V"].reshape(nk, Hk, D_HEAD).permute(1, 0, 2)[:, None]
        s = (q / 8.0) @ k  # [Hk, G, nq, nk]
        if table is not None:
            if c["bidirectional"]:
                bucket = left[back.abs().clamp(max=c["max_distance"])] + (back < 0) * n
            else:
                bucket = left[back.clamp(0, c["max_distance"])]
            s = s + table[bucket].permute(2, 0, 1).reshape(Hk, H // Hk, nq, nk)
        s = torch.where(ok, s, torch.full_like(s, -1e300))
        y = ((torch.softmax(s, -1) * ok) @ v).permute(2, 0, 1, 3).reshape(nq, H * D_HEAD)
        lse = torch.logsumexp(s.detach(), -1).reshape(H, nq)
        out["Y"].append(y.detach())
        out["lse"].append(torch.where(ok.any(-1), lse, torch.full_like(lse, -math.inf)))
        if train:
            leaves = [x["Q"], x["K"], x["V"]] + ([table] if table is not None else [])
            grads = torch.autograd.grad(y, leaves, t["dY"][b].double())
            for name, g in zip(("dQ", "dK", "dV"), grads):
                out[name].append(g)
            if table is not None:
                dbias = dbias + grads[3]
    got = {name: torch.stack(v) for name, v in out.items()}
    if train and table is not None:
        got["dbias"] = dbias
    return got
