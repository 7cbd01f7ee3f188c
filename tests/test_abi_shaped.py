"""Host-side refusals of attention with shaped scores, of the packed cache and of
eviction: bad arguments are refused before any HIP call (so these run without a
GPU), and calls with nothing to do succeed."""
import ctypes
import os
import re

import pytest

import paper_2411_01142_amd as neo
from paper_2411_01142_amd.shaped import _ScoreShape

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
FAKE = 1 << 20  # non-null, aligned; never dereferenced on these paths


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(neo.library_path()):
        import __graft_entry__
        __graft_entry__.build()
    return neo.load_library()


BASE = dict(q=FAKE, k=FAKE, v=FAKE, cache=FAKE, table=FAKE, lens=FAKE, hq=32, hkv=8, d=128, bs=16, scale=0.1,
            softcap=0.0, slopes=None, starts=None, prefix=None, out=FAKE, lse=None, batch=4, mbps=8, nb=100,
            stride=0, ws=FAKE, ws_bytes=1 << 40, kn=FAKE, vn=FAKE, row_starts=None, rows=4, strides=(1024, 128) * 2,
            sums=FAKE, sums_out=FAKE, sums_stride=128, lse_in=FAKE, budgets=FAKE, recent=0, new_table=FAKE, new_mbps=4,
            new_lens=FAKE, kept=FAKE, new_sums=FAKE, k_out=FAKE, v_out=FAKE)


def call(lib, op, **kw):
    a = {**BASE, **kw}
    shape = _ScoreShape(a["softcap"], a["slopes"], a["starts"], a["prefix"])
    heads = (a["hq"], a["hkv"], a["d"], a["bs"], a["scale"], shape)
    rows = (a["table"], a["lens"], a["batch"], a["mbps"], a["hkv"], a["d"], a["bs"], a["nb"], a["stride"])
    caches = (a["k"], a["v"]) if op in ("shaped", "evict") else (a["cache"],)
    if op in ("shaped", "packed"):
        fn = lib.neo_shaped_decode_attention if op == "shaped" else lib.neo_packed_decode_attention
        return fn(a["q"], *caches, a["table"], a["lens"], *heads, a["out"], a["lse"], a["batch"], a["mbps"], a["nb"],
                  a["stride"], a["ws"], a["ws_bytes"], None)
    if op in ("weights", "packed_weights"):
        fn = lib.neo_add_attention_weights if op == "weights" else lib.neo_packed_add_attention_weights
        return fn(a["sums"], a["sums_out"], a["sums_stride"], a["lse_in"], a["q"], a["k" if op == "weights" else "cache"],
                  a["table"], a["lens"], *heads, a["batch"], a["mbps"], a["nb"], a["stride"], None)
    if op == "append":
        return lib.neo_packed_append(a["cache"], a["kn"], a["vn"], a["row_starts"], a["rows"], *a["strides"], *rows, None)
    if op == "gather":
        return lib.neo_packed_gather(a["cache"], a["row_starts"], a["rows"], *rows, a["k_out"], a["v_out"], None)
    fn = lib.neo_kv_evict if op == "evict" else lib.neo_packed_evict
    return fn(*caches, a["table"], a["lens"], a["sums"], a["sums_stride"], a["budgets"], a["recent"], a["new_table"],
              a["new_mbps"], a["new_lens"], a["kept"], a["new_sums"], *rows[2:], None)


ATTENDS = ["shaped", "packed"]
SCORES = ATTENDS + ["weights", "packed_weights"]
EVERY = SCORES + ["append", "gather", "evict", "packed_evict"]


@pytest.mark.parametrize("op", EVERY)
@pytest.mark.parametrize("kw,code,needle", [
    (dict(batch=-1, rows=-1), INVALID, "batch"), (dict(hkv=0), INVALID, "positive"),
    (dict(d=64), UNSUPPORTED, "head_dim"), (dict(bs=32), UNSUPPORTED, "block_size"),
    (dict(table=None), INVALID, "block_table"), (dict(lens=None), INVALID, "seq_lens"),
    (dict(mbps=0), INVALID, "positive"), (dict(nb=0), INVALID, "positive"), (dict(mbps=1 << 27), INVALID, "too large"),
    (dict(batch=1 << 20, rows=1 << 20, mbps=1 << 12, sums_stride=1 << 20), INVALID, "2^31"),
    (dict(table=FAKE + 2), INVALID, "4-byte"), (dict(lens=FAKE + 1), INVALID, "4-byte"),
    (dict(stride=-16), INVALID, "stride"), (dict(stride=8), INVALID, "stride"), (dict(stride=(1 << 40) + 16), INVALID, "stride"),
    (dict(stride=1 << 40, nb=1 << 22), INVALID, "stride"),
])
def test_every_call_refuses_bad_sizes(lib, op, kw, code, needle):
    assert call(lib, op, **kw) == code
    assert needle in lib.neo_last_error().decode()


@pytest.mark.parametrize("op", SCORES)
@pytest.mark.parametrize("kw,code,needle", [
    (dict(hkv=7), INVALID, "multiple"), (dict(hq=0), INVALID, "positive"), (dict(hq=24), UNSUPPORTED, "group"),
    (dict(scale=float("nan")), INVALID, "scale"), (dict(scale=float("inf")), INVALID, "scale"),
    (dict(softcap=-1.0), INVALID, "softcap"), (dict(softcap=float("nan")), INVALID, "softcap"),
    (dict(softcap=float("inf")), INVALID, "softcap"), (dict(softcap=3e38), INVALID, "softcap"),
    (dict(softcap=1e-40), INVALID, "softcap"), (dict(q=None), INVALID, "q is NULL"), (dict(q=FAKE + 8), INVALID, "16-byte"),
    (dict(slopes=FAKE + 2), INVALID, "slopes"), (dict(starts=FAKE + 2), INVALID, "starts"),
    (dict(prefix=FAKE + 2), INVALID, "prefix_lens"), (dict(k=None, cache=None), INVALID, "cache"),
    (dict(k=FAKE + 4, cache=FAKE + 4), INVALID, "16-byte"),
])
def test_scores_are_refused(lib, op, kw, code, needle):
    assert call(lib, op, **kw) == code
    assert needle in lib.neo_last_error().decode()


@pytest.mark.parametrize("op", ATTENDS)
@pytest.mark.parametrize("kw,code", [
    (dict(out=None), INVALID), (dict(out=FAKE + 4), INVALID), (dict(lse=FAKE + 2), INVALID), (dict(ws=None), WORKSPACE),
    (dict(ws_bytes=1000), WORKSPACE), (dict(ws=FAKE + 64), INVALID),
])
def test_attention_is_refused(lib, op, kw, code):
    assert call(lib, op, **kw) == code
    assert lib.neo_last_error().decode()


def test_the_bf16_value_cache_is_checked_where_it_is_read(lib):
    for op in ("shaped", "evict"):
        assert call(lib, op, v=None) == INVALID and "v_cache" in lib.neo_last_error().decode()
        assert call(lib, op, v=FAKE + 8) == INVALID


@pytest.mark.parametrize("op", ["weights", "packed_weights"])
@pytest.mark.parametrize("kw", [dict(sums=None), dict(sums_out=None), dict(lse_in=None), dict(sums=FAKE + 2),
                                dict(sums_stride=127), dict(sums_stride=-1)])
def test_weights_are_refused(lib, op, kw):
    assert call(lib, op, **kw) == INVALID
    assert lib.neo_last_error().decode()


@pytest.mark.parametrize("kw,needle", [
    (dict(rows=5), "row_starts"), (dict(rows=-1, row_starts=FAKE), "negative"), (dict(row_starts=FAKE + 2), "row_starts"),
    (dict(row_starts=FAKE, rows=1 << 29), "2^31"), (dict(cache=None), "cache"), (dict(cache=FAKE + 8), "16-byte"),
])
@pytest.mark.parametrize("op", ["append", "gather"])
def test_rows_are_refused(lib, op, kw, needle):
    assert call(lib, op, **kw) == INVALID
    assert needle in lib.neo_last_error().decode()


@pytest.mark.parametrize("kw", [dict(kn=None), dict(vn=None), dict(kn=FAKE + 2), dict(vn=FAKE + 8),
                                dict(strides=(1020, 128, 1024, 128)), dict(strides=(1024, -8, 1024, 128)),
                                dict(strides=(1024, 128, (1 << 30) + 8, 128)), dict(strides=(1024, 128, 1024, 4))])
def test_append_is_refused(lib, kw):
    assert call(lib, "append", **kw) == INVALID
    assert lib.neo_last_error().decode()


def test_gather_is_refused(lib):
    assert call(lib, "gather", k_out=None) == INVALID
    assert call(lib, "gather", v_out=FAKE + 8) == INVALID


@pytest.mark.parametrize("op", ["evict", "packed_evict"])
@pytest.mark.parametrize("kw", [dict(sums=None), dict(budgets=None), dict(new_table=None), dict(new_lens=None),
                                dict(kept=None), dict(new_sums=None), dict(recent=-1), dict(new_mbps=0),
                                dict(new_mbps=1 << 27), dict(sums_stride=100), dict(kept=FAKE + 2),
                                dict(k=FAKE + 8, cache=FAKE + 8)])
def test_eviction_is_refused(lib, op, kw):
    assert call(lib, op, **kw) == INVALID
    assert lib.neo_last_error().decode()


@pytest.mark.parametrize("op", EVERY)
def test_an_empty_batch_is_a_noop(lib, op):
    nothing = {k: None for k in ("q", "k", "v", "cache", "table", "lens", "out", "ws", "kn", "vn", "sums", "sums_out",
                                 "lse_in", "budgets", "new_table", "new_lens", "kept", "new_sums", "k_out", "v_out")}
    assert call(lib, op, batch=0, rows=0, **nothing) == OK
    assert lib.neo_last_error().decode() == ""


def test_a_shape_may_be_left_out(lib):
    null = ctypes.POINTER(_ScoreShape)()
    assert lib.neo_shaped_decode_attention(FAKE, FAKE, FAKE, FAKE, FAKE, 32, 8, 128, 16, 0.1, null, FAKE, None, 4, 8, 100,
                                           0, None, 0, None) == WORKSPACE


def test_the_record_size_matches_the_header():
    text = open(os.path.join(ROOT, "include", "libneoattn.h")).read()
    assert int(re.search(r"#define NEO_PACKED_RECORD_BYTES (\d+)", text).group(1)) == neo.PACKED_RECORD_BYTES


def test_bindings_refuse_cpu_tensors():
    import torch
    i32 = torch.int32
    q = torch.zeros(2, 8, 128, dtype=torch.bfloat16)
    k, v = torch.zeros(4, 2, 16, 16, 8, dtype=torch.bfloat16), torch.zeros(4, 2, 128, 16, dtype=torch.bfloat16)
    p = torch.zeros(4, 2, 2176, dtype=torch.uint8)
    bt, sl = torch.zeros(2, 2, dtype=i32), torch.ones(2, dtype=i32)
    sums, lse = torch.zeros(2, 2, 32), torch.zeros(2, 8)
    for fn, args in [(neo.shaped_decode_attention, (q, k, v, bt, sl)), (neo.packed_decode_attention, (q, p, bt, sl)),
                     (neo.packed_append, (p, q[:, :2], q[:, :2], bt, sl)), (neo.packed_gather, (p, bt, sl)),
                     (neo.add_attention_weights, (sums, lse, q, k, bt, sl)),
                     (neo.packed_add_attention_weights, (sums, lse, q, p, bt, sl)),
                     (neo.kv_evict, (k, v, bt, sl, sums, sl, bt)), (neo.packed_evict, (p, bt, sl, sums, sl, bt))]:
        with pytest.raises(ValueError, match="GPU"):
            fn(*args)
