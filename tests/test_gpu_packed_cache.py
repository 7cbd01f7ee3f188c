"""GPU tests of the packed cache's append and read-back and of eviction: bit for bit
against the plain implementations, and a decoding program that uses all of it."""
import numpy as np
import pytest

import paper_2411_01142_amd as neo
import shaped_ref as R
from test_gpu_shaped import TOL, Case, dev, dev_bf16

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    neo.load_library()
    yield


def host_f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def same(a, b):
    """Equal values, NaN where NaN."""
    return np.array_equal(a, b, equal_nan=True)


def expected_rows(counts, lens, width):
    """(row, request, token) of rows that have a place."""
    row = 0
    for b, n in enumerate(counts):
        L = min(max(int(lens[b]), 0), width * 16)
        for i in range(n):
            t = L - n + i
            if t >= 0:
                yield row + i, b, t
        row += n


def odd_values(rng, shape):
    """bf16 rows of many magnitudes, with ties, zeros, denormals and large values."""
    x = R.bf16(rng.standard_normal(shape) * 2.0 ** rng.integers(-30, 30, (*shape[:-1], 1)))
    pick = rng.random(shape)
    x = np.where(pick < 0.2, rng.choice([0, -0.0, 0.25, 0.75, 2.5, -5, 6, 7, -1.75], shape), x)
    x = np.where(pick > 0.995, rng.choice([1e-40, 3e38, -3e38, 2.0 ** -126], shape), x)
    return R.bf16(x)


@pytest.mark.parametrize("hkv", [1, 3, 8])
@pytest.mark.parametrize("counts,lens", [
    (None, [1, 2, 15, 16, 17, 0, 300, 33, -1, 64]),
    ([1, 0, 16, 33, 5, 0, 100, 1], [1, 40, 16, 33, 60, 0, 100, 64]),
    ([7], [7]),
    ([0, 0, 500, 0, 1], [3, 0, 777, 5, 1]),
    ([20, 3], [12, 3]),              # more rows than tokens: the first eight have no place
    ([1] * 150, list(range(1, 151))),
    ([(i * 7) % 5 for i in range(130)], [(i * 7) % 5 + i for i in range(130)]),
])
def test_append_and_gather(counts, lens, hkv):
    rng = np.random.default_rng(len(lens) + hkv)
    table, _, pool = R.make_table(lens, rng, extra_cols=1)
    B = len(lens)
    n = B if counts is None else sum(counts)
    extra = 0 if counts is None else 6  # rows behind the last request's
    x = [odd_values(rng, (n + extra, hkv, R.D)) for _ in range(2)]
    cache = torch.from_numpy(rng.integers(0, 256, (pool, hkv, R.RECORD), dtype=np.uint8)).cuda()
    want = cache.cpu().numpy()
    starts = None if counts is None else dev(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32))
    neo.packed_append(cache, dev_bf16(x[0]), dev_bf16(x[1]), dev(table), dev(np.array(lens, np.int32)), starts)
    (kc, kb), (vc, vb) = R.quantise(x[0]), R.quantise(x[1])
    pk, pv, pke, pve = R._places()
    place = list(expected_rows([1] * B if counts is None else counts, lens, table.shape[1]))
    sign = np.uint8(0x77)  # numbers without their sign bits, for zeros
    for r, b, t in place:
        rec = want[table[b, t // 16]]
        for code, byte, at, ex in ((kc, kb, pk, pke), (vc, vb, pv, pve)):
            rec[:, at[t % 16, ::2]] = code[r][:, ::2] | (code[r][:, 1::2] << 4)
            rec[:, ex[t % 16]] = byte[r]
    got = cache.cpu().numpy()
    exps = np.r_[2048:2176]
    assert np.array_equal(got[..., exps], want[..., exps])
    assert np.array_equal(got[..., :2048] & sign, want[..., :2048] & sign)
    for a, b in zip(R.unpack(got), R.unpack(want)):
        assert same(a, b)
    # and back
    k_out = torch.full((n + extra, hkv, R.D), 3.0, dtype=torch.bfloat16, device="cuda")
    v_out = torch.full_like(k_out, 5.0)
    neo.packed_gather(cache, dev(table), dev(np.array(lens, np.int32)), starts, k_out, v_out)
    wk, wv = np.full(x[0].shape, 3.0), np.full(x[1].shape, 5.0)
    for r, b, t in place:
        wk[r], wv[r] = R.values(kc, kb)[r], R.values(vc, vb)[r]
    assert same(host_f64(k_out), wk) and same(host_f64(v_out), wv)


def test_infinities_and_nans_spoil_their_group_alone():
    rng = np.random.default_rng(3)
    x = R.bf16(rng.standard_normal((5, 2, R.D)))
    x[0, 0, 3], x[1, 1, 127], x[2, 0, 64] = np.inf, np.nan, -np.inf
    cache = neo.new_packed_kv_cache(5, 2).zero_()
    table = dev(np.arange(5, dtype=np.int32)[:, None])
    lens = dev(np.full(5, 16, np.int32))
    neo.packed_append(cache, dev_bf16(x), dev_bf16(x), table, lens)
    k, v = neo.packed_gather(cache, table, lens)
    want = R.values(*R.quantise(x))
    assert same(host_f64(k), want) and same(host_f64(v), want)
    assert np.isnan(want).sum() == 3 * 32


def test_rows_of_a_fused_projection():
    # q, k and v of one projection's output: rows and heads strided.
    B, hkv = 6, 4
    qkv = torch.randn(B, 8 + 2 * hkv, 128, device="cuda").to(torch.bfloat16)
    k, v = qkv[:, 8:8 + hkv], qkv[:, 8 + hkv:]
    other = torch.randn(hkv, B, 128, device="cuda").to(torch.bfloat16).transpose(0, 1)
    table = dev(np.arange(2 * B, dtype=np.int32).reshape(B, 2))
    lens = dev(np.arange(1, B + 1, dtype=np.int32) * 5)
    for a, b in ((k, v), (other, k), (k[:1].expand(B, hkv, 128), other)):
        c1, c2 = (neo.new_packed_kv_cache(2 * B, hkv).zero_() for _ in range(2))
        neo.packed_append(c1, a, b, table, lens)
        neo.packed_append(c2, a.contiguous(), b.contiguous(), table, lens)
        assert torch.equal(c1, c2) and int(c1.to(torch.int32).sum()) > 0


def test_bad_ids_skip_their_rows_and_reads_are_clamped():
    cache = neo.new_packed_kv_cache(4, 1).zero_()
    table = dev(np.array([[9], [-1], [2]], np.int32))
    lens = dev(np.array([3, 3, 3], np.int32))
    x = torch.ones(3, 1, 128, dtype=torch.bfloat16, device="cuda")
    neo.packed_append(cache, x, x, table, lens)
    assert int(cache[[0, 1, 3]].to(torch.int32).sum()) == 0
    k, _ = neo.packed_gather(cache, table, lens)
    assert torch.equal(k[2], x[2]) and int(k[:2].abs().sum()) == 0  # the clamped last block holds zeros


def test_append_past_four_gigabytes():
    hkv = 8
    blocks = (1 << 32) // (hkv * R.RECORD) + 100
    cache = neo.new_packed_kv_cache(blocks, hkv)
    table = dev(np.array([[blocks - 1], [1]], np.int32))
    lens = dev(np.array([16, 16], np.int32))
    x = torch.randn(2, hkv, 128, device="cuda").to(torch.bfloat16)
    neo.packed_append(cache, x, 2 * x, table, lens)
    k, v = neo.packed_gather(cache, table, lens)
    want = R.values(*R.quantise(host_f64(x)))
    assert same(host_f64(k), want) and same(host_f64(v), 2 * want)


def test_append_refusals():
    cache = neo.new_packed_kv_cache(4, 2)
    table = torch.zeros((3, 1), dtype=torch.int32, device="cuda")
    lens = torch.zeros(3, dtype=torch.int32, device="cuda")
    x = torch.zeros(3, 2, 128, dtype=torch.bfloat16, device="cuda")
    neo.packed_append(cache, x, x, table, lens)
    bad = [(dict(k_new=x[:2]), ValueError), (dict(k_new=x.float()), TypeError), (dict(v_new=x[:, :1]), ValueError),
           (dict(k_new=torch.zeros(3, 2, 132, dtype=torch.bfloat16, device="cuda")[..., 2:130]), ValueError),
           (dict(k_new=x.transpose(1, 2).contiguous().transpose(1, 2)), ValueError),
           (dict(v_new=x.cpu()), ValueError), (dict(row_starts=torch.zeros(3, dtype=torch.int32, device="cuda")), ValueError),
           (dict(row_starts=torch.zeros(4, dtype=torch.int64, device="cuda")), TypeError),
           (dict(cache=cache.float()), TypeError), (dict(cache=cache[:, :, :100]), ValueError),
           (dict(cache=cache.cpu()), ValueError)]
    for kw, error in bad:
        a = dict(cache=cache, k_new=x, v_new=x, block_table=table, seq_lens=lens)
        a.update(kw)
        with pytest.raises(error):
            neo.packed_append(**a)
    with pytest.raises(ValueError, match="rows"):
        neo.packed_gather(cache, table, lens, torch.zeros(4, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        neo.packed_gather(cache, table, lens, k_out=x[:, :1].contiguous())
    # nothing to do
    none = torch.zeros(0, 2, 128, dtype=torch.bfloat16, device="cuda")
    neo.packed_append(cache, none, none, table, lens, torch.zeros(4, dtype=torch.int32, device="cuda"))
    neo.packed_append(cache, none, none, table[:0], lens[:0])
    torch.cuda.synchronize()


# ------------------------------------------------------------------ eviction

def evict_case(kind, lens, budgets, recent, hkv, sums_of, seed, new_cols=None, extra=0):
    if new_cols is None:
        new_cols = max(1, (max(list(budgets) + [1]) + 15) // 16)
    c = Case(kind, lens, hkv, 2, seed=seed, new_cols=new_cols)
    S = c.table.shape[1] * 16 + extra
    sums = sums_of(c.rng, (len(lens), hkv, S)).astype(np.float32)
    before = [x.clone() for x in c.cache]
    fn = neo.packed_evict if kind == "packed" else neo.kv_evict
    new_lens, kept, new_sums = fn(*c.cache, *c.gpu[-2:], dev(sums), dev(np.array(budgets, np.int32)),
                                  dev(c.new_table), recent=recent)
    torch.cuda.synchronize()
    N = 16 * new_cols
    old_blocks = np.setdiff1d(np.arange(c.pool), c.new_table.ravel())
    for x, y in zip(c.cache, before):  # old blocks are only read
        assert torch.equal(x[torch.from_numpy(old_blocks)].view(torch.uint8), y[torch.from_numpy(old_blocks)].view(torch.uint8))
    rows = [x.cpu().numpy() for x in c.cache] if kind == "packed" else None
    for b in range(len(lens)):
        L = max(0, lens[b])
        n = min(L, max(0, budgets[b]), N)
        assert int(new_lens[b]) == n
        for g in range(hkv):
            want = R.kept_tokens(sums[b, g], L, n, recent)
            got = kept[b, g].cpu().numpy()
            assert np.array_equal(got[:n], want) and np.all(got[n:] == -1), (b, g)
            s = new_sums[b, g].cpu().numpy()
            assert same(s[:n], sums[b, g][want]) and np.all(s[n:] == 0)
            used = (n + 15) // 16
            blk = torch.from_numpy(c.new_table[b, :used].astype(np.int64))
            pad = used * 16 - n
            if kind == "packed":
                k, v = R.unpack(rows[0][c.new_table[b, :used]][:, g])
                k, v = k.reshape(-1, R.D), v.reshape(-1, R.D)
            else:
                k = host_f64(c.cache[0][blk, g]).transpose(0, 2, 1, 3).reshape(-1, R.D)
                v = host_f64(c.cache[1][blk, g]).transpose(0, 2, 1).reshape(-1, R.D)
            src = c.table[b, want // 16], g, want % 16
            assert same(k[:n], c.k[src]) and same(v[:n], c.v[src])
            assert pad == 0 or (np.all(k[n:] == 0) and np.all(v[n:] == 0))
    # new blocks past the last kept token keep what they held
    for b in range(len(lens)):
        n = int(new_lens[b])
        rest = torch.from_numpy(c.new_table[b, (n + 15) // 16:].astype(np.int64))
        for x, y in zip(c.cache, before):
            assert torch.equal(x[rest].view(torch.uint8), y[rest].view(torch.uint8))


def few_values(rng, shape):
    return rng.integers(0, 4, shape) * 0.25  # many ties


def heavy(rng, shape):
    x = rng.random(shape)
    return np.where(x < 0.1, 0, x ** 8 * 100)


def signed(rng, shape):
    x = rng.standard_normal(shape)
    x[rng.random(shape) < 0.05] = -0.0
    x[rng.random(shape) < 0.02] = np.inf
    x[rng.random(shape) < 0.02] = -np.inf
    x[rng.random(shape) < 0.02] = np.nan
    return x


@pytest.mark.parametrize("kind", ["bf16", "packed"])
@pytest.mark.parametrize("sums_of", [few_values, heavy, signed])
@pytest.mark.parametrize("lens,budgets,recent,hkv", [
    ([100, 64, 17, 1, 0, 300], [50, 64, 16, 1, 5, 37], 0, 2),
    ([100, 64, 17, 1, 0, 300], [50, 10, 20, 0, 5, 299], 8, 3),
    ([1000, 999, 33, -2], [160, 1, 1, 3], 500, 1),
    ([40, 50], [7, -3], 3, 1),
])
def test_evict(kind, lens, budgets, recent, hkv, sums_of):
    evict_case(kind, lens, budgets, recent, hkv, sums_of, seed=recent, extra=3)


@pytest.mark.parametrize("kind", ["bf16", "packed"])
@pytest.mark.parametrize("L,n", [(1023, 500), (1024, 1000), (1025, 16), (5000, 4999), (20011, 3001), (40000, 100)])
def test_evict_one_long_request(kind, L, n):
    evict_case(kind, [L], [n], 13, 1, heavy, seed=L)
    evict_case(kind, [L], [n], 0, 1, few_values, seed=L)


@pytest.mark.parametrize("kind", ["bf16", "packed"])
def test_evict_into_a_narrow_table_and_of_a_large_batch(kind):
    evict_case(kind, [100, 30], [64, 64], 4, 2, heavy, seed=50, new_cols=2)
    evict_case(kind, [(i * 37) % 200 for i in range(150)], [(i * 11) % 90 for i in range(150)], 5, 2, heavy, seed=51)


def test_evict_from_shared_blocks_with_bad_new_ids():
    # Two requests with the same table row; the second's new block is out of range.
    c = Case("packed", [40, 40], 1, 1, seed=52, new_cols=1)
    table = c.table.copy()
    table[1] = table[0]
    new = c.new_table.copy()
    new[1, 0] = c.pool + 7
    before = c.cache[0].clone()
    sums = c.rng.random((2, 1, 48)).astype(np.float32)
    new_lens, kept, _ = neo.packed_evict(c.cache[0], dev(table), dev(c.lens), dev(sums),
                                         dev(np.array([9, 9], np.int32)), dev(new))
    assert new_lens.tolist() == [9, 9]
    changed = (c.cache[0] != before).flatten(1).any(1).nonzero().flatten().tolist()
    assert changed == [int(new[0, 0])]
    for b in range(2):
        assert kept[b, 0, :9].tolist() == R.kept_tokens(sums[b, 0], 40, 9, 0).tolist()


def test_evict_refusals():
    c = Case("bf16", [40, 20], 2, 2, seed=53, new_cols=1)
    k, v = c.cache
    table, lens = c.gpu[-2:]
    sums = torch.zeros((2, 2, table.shape[1] * 16), device="cuda")
    budgets = torch.full((2,), 9, dtype=torch.int32, device="cuda")
    new = dev(c.new_table)
    neo.kv_evict(k, v, table, lens, sums, budgets, new)
    for kw, error in [(dict(sums=sums[..., 1:].contiguous()), ValueError), (dict(budgets=budgets[:1]), ValueError),
                      (dict(new_table=new.long()), TypeError), (dict(new_table=new[:1]), ValueError),
                      (dict(recent=-1), neo.NeoError), (dict(new_table=new[:, :0]), neo.NeoError),
                      (dict(v_cache=v[:, :1]), ValueError)]:
        a = dict(k_cache=k, v_cache=v, block_table=table, seq_lens=lens, sums=sums, budgets=budgets, new_table=new)
        a.update(kw)
        with pytest.raises(error):
            neo.kv_evict(**a)
    torch.cuda.synchronize()


# ------------------------------------------------------- all of it, together

@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("kind", ["bf16", "packed"])
def test_a_decoding_program_that_evicts(kind, graph):
    """Prompts, then tokens: append, attend with log-sum-exps, add the weights; after four
    tokens evict to a budget, then four more from the new blocks. The attention of every step
    against the plain implementation over the tokens that are left."""
    rng = np.random.default_rng(60)
    hkv, G, cap, budget, recent = 2, 4, 20.0, 40, 6
    prompts = [50, 7, 90, 33]
    B, width = len(prompts), 7
    order = rng.permutation(2 * B * width).astype(np.int32)
    tables = [dev(order[:B * width].reshape(B, width)), dev(order[B * width:].reshape(B, width))]
    if kind == "packed":
        cache = (neo.new_packed_kv_cache(2 * B * width, hkv),)
        attend, add, evict = neo.packed_decode_attention, neo.packed_add_attention_weights, neo.packed_evict
        stands = lambda x: R.values(*R.quantise(x))  # noqa: E731
    else:
        cache = neo.new_kv_cache(2 * B * width, hkv)
        attend, add, evict = neo.shaped_decode_attention, neo.add_attention_weights, neo.kv_evict
        stands = lambda x: x  # noqa: E731
    rows = {b: [[], []] for b in range(B)}  # per request: K and V rows [hkv, 128] by head, as lists
    lens = torch.tensor(prompts, dtype=torch.int32, device="cuda")
    sums = torch.zeros((B, hkv, width * 16), device="cuda")
    ref_sums = np.zeros((B, hkv, width * 16))
    ws = neo.new_workspace(B, hkv * G, hkv)
    q, kn, vn = (torch.empty((B, h, 128), dtype=torch.bfloat16, device="cuda") for h in (hkv * G, hkv, hkv))
    out, lse = torch.empty((B, hkv * G, 128), device="cuda"), torch.empty((B, hkv * G), device="cuda")
    heads = [[[] for _ in range(hkv)] for _ in range(B)]  # (k, v) per kept token

    # The prompts.
    n = sum(prompts)
    x = [R.bf16(rng.standard_normal((n, hkv, 128))) for _ in range(2)]
    starts = dev(np.concatenate([[0], np.cumsum(prompts)]).astype(np.int32))
    if kind == "packed":
        neo.packed_append(*cache, dev_bf16(x[0]), dev_bf16(x[1]), tables[0], lens, starts)
    else:
        for t in range(max(prompts)):
            at = [sum(prompts[:b]) + min(t, p - 1) for b, p in enumerate(prompts)]
            step = dev(np.array([min(t + 1, p) for p in prompts], np.int32))
            neo.kv_append(*cache, dev_bf16(x[0][at]), dev_bf16(x[1][at]), tables[0], step)
    y = [stands(a) for a in x]
    for b, p in enumerate(prompts):
        r0 = sum(prompts[:b])
        for g in range(hkv):
            heads[b][g] = [(y[0][r0 + t, g], y[1][r0 + t, g]) for t in range(p)]

    def token(table):
        if kind == "packed":
            neo.packed_append(*cache, kn, vn, table, lens)
        else:
            neo.kv_append(*cache, kn, vn, table, lens)
        attend(q, *cache, table, lens, out=out, lse=lse, softcap=cap, workspace=ws)
        add(sums, lse, q, cache[0], table, lens, softcap=cap)

    for phase in range(2):
        table, g = tables[phase], None
        for step in range(4):
            new = [R.bf16(rng.standard_normal((B, h, 128))) for h in (hkv * G, hkv, hkv)]
            for t, v in zip((q, kn, vn), new):
                t.copy_(dev_bf16(v))
            lens += 1
            if graph and step == 1:
                torch.cuda.synchronize()
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g):
                    token(table)
            if g is not None:
                g.replay()
            else:
                token(table)
            torch.cuda.synchronize()
            ky, vy = stands(new[1]), stands(new[2])
            got, got_lse = out.cpu().double().numpy(), lse.cpu().double().numpy()
            for b in range(B):
                for h in range(hkv):
                    heads[b][h].append((ky[b, h], vy[b, h]))
                    K, V = (np.array([r[i] for r in heads[b][h]]) for i in (0, 1))
                    s = cap * np.tanh(new[0][b, h * G:(h + 1) * G] @ K.T * 128 ** -0.5 / cap)
                    w = np.exp(s)
                    want = w @ V / w.sum(-1, keepdims=True)
                    assert np.abs(got[b, h * G:(h + 1) * G] - want).max() <= TOL * np.abs(V).max()
                    assert np.abs(got_lse[b, h * G:(h + 1) * G] - np.log(w.sum(-1))).max() <= 2.0 ** -12
                    ref_sums[b, h, :len(K)] += (w / w.sum(-1, keepdims=True)).sum(0)
            assert np.abs(sums.cpu().numpy() - ref_sums).max() <= 2.0 ** -10
        if phase == 0:
            new_lens, kept, new_sums = evict(*cache, tables[0], lens, sums,
                                             torch.full((B,), budget, dtype=torch.int32, device="cuda"),
                                             tables[1], recent=recent)
            torch.cuda.synchronize()
            host = sums.cpu().numpy()
            for b in range(B):
                for h in range(hkv):
                    L = len(heads[b][h])
                    stay = R.kept_tokens(host[b, h], L, min(L, budget), recent)
                    assert kept[b, h, :len(stay)].tolist() == stay.tolist()
                    heads[b][h] = [heads[b][h][t] for t in stay]
                    ref_sums[b, h, :len(stay)] = ref_sums[b, h][stay]
                    ref_sums[b, h, len(stay):] = 0
            lens.copy_(new_lens)
            sums.zero_()
            sums[..., :new_sums.shape[2]] = new_sums
