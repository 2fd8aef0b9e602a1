"""Exact attention's host side (no GPU): bucket borders, workspace sizes, refusals of the C entries
before any device work."""
import ctypes
import os
import re

import pytest

import paper_2201_12854_amd as mca
from paper_2201_12854_amd import binding

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "mca.h")
FAKE = 1 << 20  # aligned, never dereferenced: the checks run before device work


@pytest.mark.parametrize("struct,name", [(binding.ExactDesc, "mca_exact_desc"), (binding.Rows, "mca_rows")])
def test_structs_match_header(struct, name):
    body = re.search(rf"typedef struct {name} \{{(.*?)\}} {name};", open(HEADER).read(), re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    assert re.findall(r"(\w+);", body) == [f for f, _ in struct._fields_]


def _bucket(d, n, top):
    """Bucket of distance d among n one-sided buckets, in whole numbers."""
    e = n // 2
    m = n - e
    if d < e:
        return d
    return e + max(k for k in range(m) if d ** m * e ** k >= e ** m * top ** k)


@pytest.mark.parametrize("buckets,top,both", [(32, 128, True), (32, 128, False), (2, 2, False), (4, 2, True), (4, 256, True),
                                              (128, 256, False), (128, 256, True), (128, 65, False), (17, 81, False),
                                              (16, 100, False), (64, 256, False), (6, 216, True), (9, 64, False)])
def test_relative_buckets(buckets, top, both):
    got = mca.relative_buckets(buckets, top, both)
    n = buckets // 2 if both else buckets
    want = [_bucket(abs(r) if both else max(-r, 0), n, top) + (n if both and r > 0 else 0) for r in range(-top, top + 1)]
    assert got == want
    assert got[top] == 0 and got[0] == n - 1


@pytest.mark.parametrize("buckets,top,both", [(1, 128, False), (0, 128, False), (2, 128, True), (5, 128, True), (129, 256, False),
                                              (130, 256, True), (32, 16, False), (32, 8, True), (32, 257, True), (-4, 8, True)])
def test_bucket_sizes_refused(buckets, top, both):
    with pytest.raises(binding.MCAError) as e:
        mca.relative_buckets(buckets, top, both)
    assert e.value.status == binding.MCA_ERR_INVALID_ARGUMENT


def _desc(**kw):
    d = binding.ExactDesc()
    base = dict(batch=2, q_len=128, kv_len=160, heads=12, kv_heads=4, d_head=64, dtype=1, scale=0.125)
    for k, v in dict(base, **kw).items():
        setattr(d, k, v)
    return d


def _size(d, backward):
    out = ctypes.c_size_t(0)
    st = mca.load_library().mca_exact_workspace_size(ctypes.byref(d), backward, ctypes.byref(out))
    return st, out.value


def test_workspace_sizes():
    assert _size(_desc(), 0) == (binding.MCA_OK, 0)  # enough rows: no block shares another's keys
    st, n = _size(_desc(), 1)
    assert st == binding.MCA_OK and n >= 8 * 2 * 12 * 128
    st, with_bias = _size(_desc(bias_table=FAKE, bias_buckets=32, bias_max_distance=128, bias_bidirectional=1), 1)
    assert st == binding.MCA_OK and with_bias > n
    st, few = _size(_desc(q_len=1, kv_len=16384), 0)
    assert st == binding.MCA_OK and few > 0
    short = dict(dtype=binding.MCA_BF16, q_len=128, kv_len=128, heads=12)
    assert _size(_desc(kv_heads=12, **short), 1) == (binding.MCA_OK, 0)  # one launch
    for more in (dict(kv_heads=4), dict(kv_heads=12, kv_len=129), dict(kv_heads=12, dtype=binding.MCA_F32)):
        assert _size(_desc(**dict(short, **more)), 1)[1] > 0


REFUSED = [dict(batch=0), dict(q_len=0), dict(kv_len=0), dict(heads=0), dict(kv_heads=0), dict(kv_heads=5), dict(kv_heads=24),
           dict(heads=2048, kv_heads=1), dict(dtype=2), dict(dtype=-1), dict(causal=2), dict(window=-2), dict(window=3),
           dict(window=1 << 26), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
           dict(scale=1e300), dict(scale=1e-300), dict(reserved=1), dict(q_lens=FAKE + 2), dict(kv_lens=FAKE + 1),
           dict(q_pos=FAKE + 3), dict(bias_table=FAKE), dict(bias_table=FAKE + 4, bias_buckets=32, bias_max_distance=128),
           dict(bias_table=FAKE, bias_buckets=32, bias_max_distance=300),
           dict(bias_table=FAKE, bias_buckets=33, bias_max_distance=128, bias_bidirectional=1),
           dict(bias_table=FAKE, bias_buckets=32, bias_max_distance=128, bias_bidirectional=2),
           dict(q_len=1 << 25), dict(kv_len=1 << 25), dict(batch=1 << 25), dict(batch=1 << 20, q_len=1 << 20),
           dict(batch=1 << 20, kv_len=1 << 20)]


@pytest.mark.parametrize("kw", REFUSED, ids=lambda kw: ",".join(f"{k}={v}" for k, v in kw.items()))
@pytest.mark.parametrize("backward", [0, 1])
def test_desc_refused(kw, backward):
    assert _size(_desc(**kw), backward)[0] == binding.MCA_ERR_INVALID_ARGUMENT
    assert mca.load_library().mca_last_error().decode()


def test_unsupported_head_width():
    assert _size(_desc(d_head=128), 0)[0] == binding.MCA_ERR_UNSUPPORTED


def _rows(data=FAKE, batch=1 << 20, row=1024):
    return binding.Rows(data, batch, row)


def _forward(d, lse=FAKE, ws=None, ws_bytes=0, **rows):
    t = {n: _rows(FAKE + (k + 1 << 44)) for k, n in enumerate(("Q", "K", "V", "Y"))}
    t.update(rows)
    return mca.load_library().mca_exact_attention_forward(d, t["Q"], t["K"], t["V"], t["Y"], lse, ws, ws_bytes, None)


def _backward(d, lse=FAKE, dbias=None, ws=FAKE + (1 << 43), ws_bytes=1 << 40, **rows):
    t = {n: _rows(FAKE + (k + 1 << 44)) for k, n in enumerate(("dY", "Q", "K", "V", "Y", "dQ", "dK", "dV"))}
    t.update(rows)
    return mca.load_library().mca_exact_attention_backward(d, t["dY"], t["Q"], t["K"], t["V"], t["Y"], lse, t["dQ"], t["dK"],
                                                           t["dV"], dbias, ws, ws_bytes, None)


BAD_ROWS = [_rows(data=None), _rows(data=FAKE + 8), _rows(row=1020), _rows(row=128), _rows(batch=4), _rows(batch=-8),
            _rows(row=1 << 25), None]


@pytest.mark.parametrize("bad", range(len(BAD_ROWS)))
def test_rows_refused(bad):
    for name in ("Q", "K", "V", "Y"):
        assert _forward(_desc(), **{name: BAD_ROWS[bad]}) == binding.MCA_ERR_INVALID_ARGUMENT, name
    for name in ("dY", "Q", "K", "V", "Y", "dQ", "dK", "dV"):
        assert _backward(_desc(), **{name: BAD_ROWS[bad]}) == binding.MCA_ERR_INVALID_ARGUMENT, name


def test_overlapping_outputs_refused():
    once = _rows(batch=0)  # one set of rows for the whole batch: fine to read only
    assert _forward(_desc(), Y=once) == binding.MCA_ERR_INVALID_ARGUMENT
    for name in ("dQ", "dK", "dV"):
        assert _backward(_desc(), **{name: once}) == binding.MCA_ERR_INVALID_ARGUMENT, name
        # half of the rows of the next batch row
        assert _backward(_desc(), **{name: _rows(batch=1024 * 64)}) == binding.MCA_ERR_INVALID_ARGUMENT, name


def test_results_in_place_refused():
    at = lambda k: _rows(FAKE + (k << 44))  # noqa: E731
    said = lambda: mca.load_library().mca_last_error().decode()  # noqa: E731
    for k in (1, 2, 3):  # Y in Q, K, V
        assert _forward(_desc(), Y=at(k)) == binding.MCA_ERR_INVALID_ARGUMENT and "operand" in said()
    assert _forward(_desc(), lse=at(4).data) == binding.MCA_ERR_INVALID_ARGUMENT and "two results" in said()
    for n, name in enumerate(("dQ", "dK", "dV")):
        for k in range(1, 6):
            assert _backward(_desc(), **{name: at(k)}) == binding.MCA_ERR_INVALID_ARGUMENT and "operand" in said(), name
        other = at(6 + (n + 1) % 3)
        assert _backward(_desc(), **{name: other}) == binding.MCA_ERR_INVALID_ARGUMENT and "two results" in said(), name
    d = _desc(bias_table=FAKE, bias_buckets=32, bias_max_distance=128, bias_bidirectional=1)
    assert _backward(d, lse=FAKE + (1 << 42), dbias=FAKE) == binding.MCA_ERR_INVALID_ARGUMENT and "operand" in said()


def test_wide_integers_refused():
    for args in ((8, 2**32 + 20), (2**32 + 8, 20), (8, 10**15)):
        with pytest.raises(ValueError):
            mca.relative_buckets(*args)
    with pytest.raises(binding.MCAError):
        mca.relative_buckets(8, 2**31 - 1)


def test_other_arguments_refused():
    few = _desc(q_len=1, kv_len=16384)
    need = _size(few, 0)[1]
    assert _forward(few) == binding.MCA_ERR_INVALID_ARGUMENT  # no workspace
    assert _forward(few, ws=FAKE + 8, ws_bytes=need) == binding.MCA_ERR_INVALID_ARGUMENT
    assert _forward(few, ws=FAKE, ws_bytes=need - 1) == binding.MCA_ERR_WORKSPACE_TOO_SMALL
    assert _forward(_desc(), lse=None) == binding.MCA_ERR_INVALID_ARGUMENT
    assert _forward(_desc(), lse=FAKE + 4) == binding.MCA_ERR_INVALID_ARGUMENT
    d = _desc()
    assert _backward(d, ws_bytes=_size(d, 1)[1] - 1) == binding.MCA_ERR_WORKSPACE_TOO_SMALL
    assert _backward(d, lse=None) == binding.MCA_ERR_INVALID_ARGUMENT
    assert _backward(d, dbias=FAKE) == binding.MCA_ERR_INVALID_ARGUMENT  # no table
    with_bias = _desc(bias_table=FAKE, bias_buckets=32, bias_max_distance=128, bias_bidirectional=1)
    assert _backward(with_bias) == binding.MCA_ERR_INVALID_ARGUMENT  # no gradient
    assert _backward(with_bias, dbias=FAKE + 2) == binding.MCA_ERR_INVALID_ARGUMENT
    lib = mca.load_library()
    assert lib.mca_exact_attention_forward(None, _rows(), _rows(), _rows(), _rows(), FAKE, None, 0, None) == \
        binding.MCA_ERR_INVALID_ARGUMENT
    assert lib.mca_exact_workspace_size(_desc(), 0, None) == binding.MCA_ERR_INVALID_ARGUMENT
    assert lib.mca_relative_buckets(32, 128, 1, None) == binding.MCA_ERR_INVALID_ARGUMENT
