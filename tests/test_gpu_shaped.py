"""GPU tests of attention with shaped scores over bf16 and packed caches, and of the
sums of its weights, against the plain implementation in 64 bits."""
import numpy as np
import pytest

import paper_2411_01142_amd as neo
import shaped_ref as R

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

# A softmax weight enters the second product with 16 bits or more: off by at most
# 2^-17 of itself. A score is a sum of 128 products of bf16 values, exact in fp32, in
# fp32 steps, times the scale, and its bias, distances counted from the token where
# it is largest: with |score| below 64 off by less than 64 * 2^-24 * 8 = 2^-15. A row is
# an average of value rows, so it is off by at most 2 * 2^-15 + 2^-17 of the largest
# value it averages.
TOL = 2.0 ** -13.8
# A log-sum-exp is off by a score's error and its own roundings, 2^-24 of it.
LSE_TOL = 2.0 ** -14


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    neo.load_library()
    yield


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def dev_bf16(x):
    return torch.from_numpy(R.bits(x).view(np.int16)).cuda().view(torch.bfloat16)


class Case:
    """A batch with one of the cache types; k, v are the values that the cache stands for."""

    def __init__(self, kind, lens, hkv, group, seed, layout="dense", extra_cols=0, new_cols=0):
        rng = self.rng = np.random.default_rng(seed)
        self.kind, self.hkv, self.hq = kind, hkv, hkv * group
        self.lens = np.asarray(lens, np.int32)
        self.table, self.new_table, self.pool = R.make_table(lens, rng, extra_cols=extra_cols,
                                                             new_cols=new_cols)
        k, v = R.make_rows(self.pool, hkv, rng)
        self.q = R.bf16(rng.standard_normal((len(lens), self.hq, R.D)))
        if kind == "packed":
            kq, vq = R.quantise(k), R.quantise(v)
            self.k, self.v = R.values(*kq), R.values(*vq)
            rec = R.pack(*kq, *vq)
            if layout == "padded":
                buf = torch.full((self.pool, hkv * R.RECORD + 48), 255, dtype=torch.uint8, device="cuda")
                c = buf[:, :hkv * R.RECORD].view(self.pool, hkv, R.RECORD)
                c.copy_(dev(rec))
            else:
                c = dev(rec)
            self.cache = (c,)
        else:
            self.k, self.v = k, v
            kk = dev_bf16(k.reshape(self.pool, hkv, R.BS, 16, 8).transpose(0, 1, 3, 2, 4))
            vv = dev_bf16(v.transpose(0, 1, 3, 2))
            if layout != "dense":
                a, b = neo.new_kv_cache(self.pool, hkv)
                a.copy_(kk), b.copy_(vv)
                kk, vv = a, b
            self.cache = (kk, vv)
        self.gpu = [dev_bf16(self.q), *self.cache, dev(self.table), dev(self.lens)]

    def ranges(self, mask):
        """(starts, prefix lengths) of a kind of mask."""
        L, r = np.maximum(self.lens, 0), self.rng
        return {
            "none": (None, None),
            "window": (np.maximum(L - 40, 0).astype(np.int32), np.full(len(L), 5, np.int32)),
            "document": ((L * r.random(len(L))).astype(np.int32),
                         (L * r.random(len(L)) * 0.5).astype(np.int32)),
            "starts": ((L * r.random(len(L))).astype(np.int32), None),
            "last": (L - 1, None),
            "first": (L + 100, np.ones(len(L), np.int32)),
            "nothing": (np.where(np.arange(len(L)) % 2 == 0, L, 0).astype(np.int32),
                        np.where(np.arange(len(L)) % 2 == 0, -3, 2).astype(np.int32)),
            "overlap": (L // 3, L // 2),
        }[mask]

    def attend(self, scale=None, cap=None, slopes=None, starts=None, prefix=None, **kw):
        lse = torch.full((len(self.lens), self.hq), float("nan"), device="cuda")
        out = torch.full((len(self.lens), self.hq, R.D), float("nan"), device="cuda")
        fn = neo.packed_decode_attention if self.kind == "packed" else neo.shaped_decode_attention
        fn(*self.gpu, scale, out, softcap=cap, slopes=None if slopes is None else dev(slopes, torch.float32),
           starts=None if starts is None else dev(starts, torch.int32),
           prefix_lens=None if prefix is None else dev(prefix, torch.int32), lse=lse, **kw)
        torch.cuda.synchronize()
        return out.cpu().double().numpy(), lse.cpu().double().numpy()

    def check(self, scale=None, cap=None, slopes=None, starts=None, prefix=None, tol=TOL, **kw):
        out, lse = self.attend(scale, cap, slopes, starts, prefix, **kw)
        want, want_lse = R.attention(self.q, self.k, self.v, self.table, self.lens, scale, cap,
                                     slopes, starts, prefix)
        assert np.array_equal(np.isneginf(lse), np.isneginf(want_lse))
        fine = ~np.isneginf(want_lse)
        assert np.all(out[~fine] == 0)
        top = np.abs(self.v).max()
        err = np.abs(out - want).max() if out.size else 0.0
        lerr = (np.abs(lse[fine] - want_lse[fine]) / np.maximum(1, np.abs(want_lse[fine]))).max() if fine.any() else 0.0
        print(f"[shaped] {self.kind} B={len(self.lens)} {self.hq}/{self.hkv}: {err / top:.1e} of the largest value, "
              f"lse {lerr:.1e}", flush=True)
        assert err <= tol * top and lerr <= LSE_TOL
        return out, lse


KINDS = ["bf16", "packed"]
LENGTHS = {
    "edges": [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 79, 80, 81, -4],
    "ragged": [700, 3, 129, 1000, 0, 511, 512, 513, 64, 1],
    "one": [1234],
    "long": [20011, 5],
}


@pytest.mark.parametrize("group", [1, 2, 4, 8, 16])
@pytest.mark.parametrize("lens", LENGTHS)
@pytest.mark.parametrize("kind", KINDS)
def test_plain_scores(kind, lens, group):
    Case(kind, LENGTHS[lens], 2, group, seed=group).check()


@pytest.mark.parametrize("hkv,group", [(1, 16), (3, 4), (5, 1), (8, 8)])
@pytest.mark.parametrize("mask", ["none", "window", "document", "starts", "last", "first", "nothing",
                                  "overlap"])
@pytest.mark.parametrize("kind", KINDS)
def test_masks(kind, mask, hkv, group):
    c = Case(kind, LENGTHS["edges"] + LENGTHS["ragged"], hkv, group, seed=7, extra_cols=3)
    c.check(None, None, None, *c.ranges(mask))


@pytest.mark.parametrize("group", [1, 4, 8, 16])
@pytest.mark.parametrize("cap,slope,mask", [(5.0, 0, "none"), (30.0, 0, "window"), (None, 0.3, "document"),
                                            (20.0, 0.01, "window"), (None, -0.02, "document"),
                                            (2.0, -0.3, "none")])
@pytest.mark.parametrize("kind", KINDS)
def test_caps_and_biases(kind, cap, slope, mask, group):
    c = Case(kind, LENGTHS["ragged"] + [33, 48], 2, group, seed=11)
    slopes = (slope * c.rng.uniform(0.3, 1, c.hq)).astype(np.float32) if slope else None
    starts, prefix = c.ranges(mask)
    # Distances reach 1000 tokens of bias 0.3: the scores' origin keeps those that count small.
    out, lse = c.attend(None, cap, slopes, starts, prefix)
    c.check(None, cap, slopes, starts, prefix)


def test_both_signs_of_slopes_in_one_group():
    c = Case("packed", [900, 1, 17], 1, 8, seed=12)
    c.check(slopes=np.array([0.5, -0.5, 0, 0.01, -0.01, 2, -2, 1e-4], np.float32))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("cap", [None, 3.0])
def test_large_scores(kind, cap):
    # Scores up to about 60 in magnitude, where a softmax is one token; scale negative too.
    c = Case(kind, LENGTHS["ragged"], 2, 4, seed=13)
    for scale in (1.2, -1.2):
        c.check(scale, cap)


@pytest.mark.parametrize("kind,layout", [("bf16", "interleaved"), ("packed", "padded")])
def test_block_strides(kind, layout):
    a = Case(kind, LENGTHS["ragged"], 3, 4, seed=14, layout=layout)
    b = Case(kind, LENGTHS["ragged"], 3, 4, seed=14)
    for x, y in zip(a.check(cap=9.0), b.check(cap=9.0)):
        assert np.array_equal(x, y)


@pytest.mark.parametrize("kind", KINDS)
def test_what_lies_behind_a_request_and_in_masked_places_is_not_read_into_it(kind):
    c = Case(kind, [5, 40, 100, 64], 2, 4, seed=15)
    starts = np.array([2, 20, 0, 50], np.int32)
    prefix = np.array([1, 3, 0, 0], np.int32)
    want = c.attend(None, None, None, starts, prefix)
    used = np.zeros((c.pool, R.BS), bool)
    for b, L in enumerate(c.lens):
        t = R.seen_tokens(L, starts[b], prefix[b])
        used[c.table[b, t // R.BS], t % R.BS] = True
    for bad in (np.inf, -np.inf, np.nan):
        for blk, slot in np.argwhere(~used):
            if kind == "packed":
                rec = c.cache[0][blk]
                pk, pv, pke, pve = R._places()
                for at in (pke, pve):
                    rec[:, torch.from_numpy(at[slot]).cuda()] = 255
                for at in (pk, pv):
                    rec[:, torch.from_numpy(at[slot]).cuda()] = 0x77
            else:
                c.cache[0][blk, :, :, slot] = bad
                c.cache[1][blk, :, :, slot] = bad
        got = c.attend(None, None, None, starts, prefix)
        assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])


def test_keys_of_minus_infinity_weigh_nothing():
    # A key with an infinite entry masks its token (bf16 caches; a packed group would be NaN).
    c = Case("bf16", [300, 64, 33, 1000], 2, 4, seed=16)
    c.q[:, :, 0] = 1.0
    c.gpu[0] = dev_bf16(c.q)
    start = np.array([48, 16, 32, 999], np.int32)
    for b, L in enumerate(c.lens):
        t = np.arange(start[b])
        c.k[c.table[b, t // 16], :, t % 16, 0] = -np.inf
        c.cache[0][torch.from_numpy(c.table[b, t // 16]).long(), :, 0, torch.from_numpy(t % 16).long(), 0] = -np.inf
    out, lse = c.attend()
    c.k = np.where(np.isinf(c.k), 0, c.k)
    want, want_lse = R.attention(c.q, c.k, c.v, c.table, c.lens, starts=start)
    assert np.abs(out - want).max() <= TOL * np.abs(c.v).max()
    assert np.abs(lse - want_lse).max() <= LSE_TOL * 16


@pytest.mark.parametrize("kind", KINDS)
def test_a_nan_reaches_its_own_request_and_head_alone(kind):
    c = Case(kind, [100, 300, 50], 2, 4, seed=17)
    want, _ = c.attend()
    blk, slot = c.table[1, 7], 3
    if kind == "packed":
        c.cache[0][blk, 1, 2048 + 16 * 2 + slot] = 255
    else:
        c.cache[0][blk, 1, 4, slot, 2] = float("nan")
    out, lse = c.attend()
    assert np.isnan(out[1, 4:]).all() and np.isnan(lse[1, 4:]).all()
    out[1, 4:] = want[1, 4:]
    assert np.array_equal(out, want)


def test_values_of_every_packed_number_and_many_exponents():
    # One token: the output is its value row, exactly; all 16 codes, exponents 2 .. 252.
    B = 12
    c = Case("packed", [1] * B, 1, 1, seed=18)
    code = c.rng.integers(0, 16, (c.pool, 1, 16, R.D)).astype(np.uint8)
    byte = c.rng.integers(2, 253, (c.pool, 1, 16, 4)).astype(np.uint8)
    kc, kb = R.quantise(c.k)
    c.cache[0].copy_(dev(R.pack(kc, kb, code, byte)))
    out, _ = c.attend()
    want = R.values(code, byte)[c.table[:, 0], :, 0]
    assert np.array_equal(out, want.astype(np.float32).astype(np.float64))


@pytest.mark.parametrize("kind", KINDS)
def test_lengths_past_the_table_and_bad_ids_are_clamped(kind):
    c = Case(kind, [100, 40, 20], 1, 4, seed=19)
    c.lens[:] = [5000, -7, 20]
    c.gpu[-1] = dev(c.lens)
    last = c.table.copy()
    last[0] = np.where(last[0] < 0, c.pool - 1, last[0])
    table = last.copy()
    table[2, 1] = c.pool + 12345  # read as the last block
    table[0, -1] = -5             # likewise (unsigned)
    last[2, 1] = last[0, -1] = c.pool - 1
    c.gpu[-2] = dev(table)
    c.table = last
    c.check()


@pytest.mark.parametrize("kind", KINDS)
def test_addresses_past_four_gigabytes(kind):
    hkv = 8
    lens = [70, 300]
    c = Case(kind, lens, hkv, 4, seed=20)
    per = hkv * (R.RECORD if kind == "packed" else 8192)
    blocks = (1 << 32) // per + 5000
    shift = blocks - c.pool
    if kind == "packed":
        big = (torch.empty((blocks, hkv, R.RECORD), dtype=torch.uint8, device="cuda"),)
    else:
        big = neo.new_kv_cache(blocks, hkv)
    for a, b in zip(big, c.cache):
        a[shift:] = b
    table = np.where(c.table >= 0, c.table + shift, -1).astype(np.int32)
    want = c.attend()
    c.gpu = [c.gpu[0], *big, dev(table), c.gpu[-1]]
    for x, y in zip(c.attend(), want):
        assert np.array_equal(x, y)


def test_a_shaped_call_without_shape_agrees_with_decode_attention():
    c = Case("bf16", LENGTHS["ragged"], 8, 4, seed=21)
    out, _ = c.check()
    plain = neo.decode_attention(*c.gpu).cpu().double().numpy()
    assert np.abs(out - plain).max() <= 2 * TOL * np.abs(c.v).max()


# ------------------------------------------------------------- many requests

BATCHES = {
    # name: (requests' lengths, kv heads): few pairs, about as many as compute units, many.
    "pairs_100": ([(i * 353) % 1500 for i in range(50)], 2),
    "pairs_270": ([(i * 353) % 900 + 1 for i in range(90)], 3),
    "pairs_1200": ([(i * 97) % 300 for i in range(600)], 2),
    "one_long_among_short": ([20000] + [(i * 31) % 70 for i in range(400)], 1),
    "pairs_4000_short": ([(i * 7) % 40 for i in range(1000)], 4),
    "nobody": ([0] * 700, 1),
    "few_with_tokens": ([0] * 500 + [77] + [0] * 600 + [3000] + [0] * 100, 1),
}


@pytest.mark.parametrize("name", BATCHES)
@pytest.mark.parametrize("kind", KINDS)
def test_batches(kind, name):
    lens, hkv = BATCHES[name]
    c = Case(kind, lens, hkv, 4, seed=22)
    c.check()
    c.check(None, 8.0, None, *c.ranges("document"))
    c.check(None, None, None, *c.ranges("window"))


@pytest.mark.parametrize("group", [1, 8, 16])
@pytest.mark.parametrize("kind", KINDS)
def test_a_large_batch_of_every_group(kind, group):
    lens = [(i * 353) % 700 for i in range(300)]
    c = Case(kind, lens, 2, group, seed=23)
    c.check(None, None, (np.arange(c.hq) / c.hq).astype(np.float32), *c.ranges("document"))


# ------------------------------------------------------- streams and graphs

@pytest.mark.parametrize("kind", KINDS)
def test_results_do_not_depend_on_the_run_or_the_stream(kind):
    c = Case(kind, LENGTHS["ragged"] + [9000], 4, 8, seed=24)
    first = c.attend()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for x, y in zip(c.attend(), first):
            assert np.array_equal(x, y)
        for x, y in zip(c.attend(stream=side), first):
            assert np.array_equal(x, y)
    ws = neo.new_workspace(len(c.lens), c.hq, c.hkv)
    for x, y in zip(c.attend(workspace=ws), first):
        assert np.array_equal(x, y)
    # The same workspace serves plain decode attention in between.
    if kind == "bf16":
        plain = neo.decode_attention(*c.gpu, workspace=ws)
        for x, y in zip(c.attend(workspace=ws), first):
            assert np.array_equal(x, y)
        assert torch.equal(neo.decode_attention(*c.gpu, workspace=ws), plain)


@pytest.mark.parametrize("lens,hkv", [([900, 17, 3000, 1, 0, 64], 8), ([(i * 53) % 500 for i in range(400)], 2)])
@pytest.mark.parametrize("kind", KINDS)
def test_graph_replays_follow_the_inputs(kind, lens, hkv):
    c = Case(kind, lens, hkv, 4, seed=25)
    fn = neo.packed_decode_attention if kind == "packed" else neo.shaped_decode_attention
    ws = neo.new_workspace(len(lens), c.hq, hkv)
    out = torch.empty((len(lens), c.hq, R.D), device="cuda")
    lse = torch.empty((len(lens), c.hq), device="cuda")
    fn(*c.gpu, out=out, lse=lse, softcap=7.0, workspace=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fn(*c.gpu, out=out, lse=lse, softcap=7.0, workspace=ws)
    for i in range(4):
        c.gpu[0].copy_(torch.randn_like(c.gpu[0]))
        c.gpu[-1].copy_(dev((c.lens * (i + 1) // 4).astype(np.int32)))
        torch.randn(1 << 18, device="cuda").sum().item()
        g.replay()
        torch.cuda.synchronize()
        eager, eager_lse = torch.empty_like(out), torch.empty_like(lse)
        fn(*c.gpu, out=eager, lse=eager_lse, softcap=7.0)
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.equal(lse, eager_lse)


def test_a_captured_call_needs_its_own_workspace():
    c = Case("packed", [40], 1, 4, seed=26)
    neo.packed_decode_attention(*c.gpu)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with pytest.raises(ValueError, match="workspace"):
        with torch.cuda.graph(g):
            neo.packed_decode_attention(*c.gpu)
    torch.cuda.synchronize()
    c.check()


# ------------------------------------------------------------------ weights

# A weight exp(score - lse) is off by the score's error, the log-sum-exp's (2^-24 of it) and
# its exponential's, relatively; 2^-15 for scores below 64 as above.
WEIGHT_TOL = 2.0 ** -14


def check_weights(c, cap=None, slopes=None, starts=None, prefix=None, in_place=False):
    _, lse = c.attend(None, cap, slopes, starts, prefix)
    lse = lse.astype(np.float32)
    S = c.table.shape[1] * 16 + 5
    sums = c.rng.random((len(c.lens), c.hkv, S)).astype(np.float32)
    dsums = dev(sums)
    dout = dsums if in_place else torch.full_like(dsums, 7.0)
    fn = neo.packed_add_attention_weights if c.kind == "packed" else neo.add_attention_weights
    fn(dsums, dev(lse), c.gpu[0], c.cache[0], *c.gpu[-2:], out=None if in_place else dout, softcap=cap,
       slopes=None if slopes is None else dev(slopes, torch.float32),
       starts=None if starts is None else dev(starts, torch.int32),
       prefix_lens=None if prefix is None else dev(prefix, torch.int32))
    torch.cuda.synchronize()
    want = R.weight_sums(sums, lse.astype(np.float64), c.q, c.k, c.table, c.lens, None, cap, slopes, starts, prefix)
    seen = np.zeros(sums.shape, bool)
    for b, L in enumerate(c.lens):
        t = R.seen_tokens(min(L, S - 5), 0 if starts is None else starts[b], 0 if prefix is None else prefix[b])
        seen[b][:, t] = True
    got = dout.cpu().numpy()
    assert np.array_equal(got[~seen], (sums if in_place else np.full_like(sums, 7.0))[~seen])
    added = want - sums
    err = np.abs(got - want)[seen] - 2.0 ** -23 * np.abs(want)[seen]
    assert np.all(err <= WEIGHT_TOL * np.abs(added)[seen])
    if not in_place:
        assert np.array_equal(dsums.cpu().numpy(), sums)


@pytest.mark.parametrize("group", [1, 2, 4, 8, 16])
@pytest.mark.parametrize("kind", KINDS)
def test_weights(kind, group):
    c = Case(kind, LENGTHS["edges"] + LENGTHS["ragged"], 3, group, seed=30)
    check_weights(c)
    check_weights(c, in_place=True)
    check_weights(c, 6.0, (0.05 * c.rng.standard_normal(c.hq)).astype(np.float32), *c.ranges("document"))
    check_weights(c, None, None, *c.ranges("nothing"))


@pytest.mark.parametrize("name", BATCHES)
@pytest.mark.parametrize("kind", KINDS)
def test_weights_of_batches(kind, name):
    lens, hkv = BATCHES[name]
    check_weights(Case(kind, lens, hkv, 2, seed=31))


def test_a_tokens_weights_sum_to_its_heads():
    c = Case("packed", [1000, 3], 2, 8, seed=32)
    sums = torch.zeros((2, 2, c.table.shape[1] * 16), device="cuda")
    _, lse = c.attend()
    neo.packed_add_attention_weights(sums, dev(lse, torch.float32), c.gpu[0], c.cache[0], *c.gpu[-2:])
    assert torch.allclose(sums.sum(-1), torch.full((2, 2), 8.0, device="cuda"), rtol=2.0 ** -14)


# ----------------------------------------------------------------- refusals

def test_refusals():
    for kind in KINDS:
        c = Case(kind, [40, 20], 2, 4, seed=40)
        q, *cache, table, lens = c.gpu
        fn = neo.packed_decode_attention if kind == "packed" else neo.shaped_decode_attention
        ok = dict(slopes=torch.zeros(8, device="cuda"), starts=torch.zeros(2, dtype=torch.int32, device="cuda"))
        fn(q, *cache, table, lens, **ok)
        with pytest.raises(ValueError):
            fn(q, *cache, table, lens, slopes=torch.zeros(7, device="cuda"))
        with pytest.raises(TypeError):
            fn(q, *cache, table, lens, starts=torch.zeros(2, dtype=torch.int64, device="cuda"))
        with pytest.raises(ValueError):
            fn(q, *cache, table, lens, prefix_lens=torch.zeros(3, dtype=torch.int32, device="cuda"))
        with pytest.raises(ValueError, match="GPU"):
            fn(q, *cache, table, lens.cpu())
        with pytest.raises(ValueError):
            fn(q, *cache, table, lens, lse=torch.zeros(2, 7, device="cuda"))
        with pytest.raises(ValueError):
            fn(q[:1], *cache, table, lens)
        with pytest.raises(ValueError, match="contiguous"):
            fn(q.transpose(0, 1).contiguous().transpose(0, 1), *cache, table, lens)
        for bad in (-1.0, float("nan"), float("inf")):
            with pytest.raises(neo.NeoError, match="softcap"):
                fn(q, *cache, table, lens, softcap=bad)
        with pytest.raises(neo.NeoError, match="scale"):
            fn(q, *cache, table, lens, float("nan"))
        with pytest.raises(neo.NeoError, match="group"):
            fn(q[:, :6].contiguous(), *cache, table, lens)
        with pytest.raises(neo.NeoError):
            fn(q, *cache, table, lens, workspace=torch.zeros(256, dtype=torch.uint8, device="cuda"))
        empty = fn(q[:0], *cache, table[:0], lens[:0])
        assert empty.shape == (0, 8, 128)
    with pytest.raises(ValueError, match="2176"):
        neo.packed_decode_attention(q, cache[0][..., :2000], table, lens)
    with pytest.raises(TypeError, match="uint8"):
        neo.packed_decode_attention(q, cache[0].view(torch.int8), table, lens)
    with pytest.raises(ValueError, match="dense"):
        neo.packed_decode_attention(q, cache[0].repeat_interleave(2, 1)[:, ::2], table, lens)
    torch.cuda.synchronize()


def test_weights_refusals():
    c = Case("packed", [40, 20], 2, 4, seed=41)
    q, cache, table, lens = c.gpu
    S = table.shape[1] * 16
    lse = torch.zeros((2, 8), device="cuda")
    fn = neo.packed_add_attention_weights
    with pytest.raises(ValueError):
        fn(torch.zeros((2, 2, S - 1), device="cuda"), lse, q, cache, table, lens)
    with pytest.raises(ValueError):
        fn(torch.zeros((2, 3, S), device="cuda"), lse, q, cache, table, lens)
    with pytest.raises(TypeError):
        fn(torch.zeros((2, 2, S), device="cuda", dtype=torch.float64), lse, q, cache, table, lens)
    buf = torch.zeros(3 * 2 * S, device="cuda")
    with pytest.raises(ValueError, match="overlap"):
        fn(buf[:4 * S].view(2, 2, S), lse, q, cache, table, lens, out=buf[S:5 * S].view(2, 2, S))
    torch.cuda.synchronize()
