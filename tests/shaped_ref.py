"""Plain implementations, in numpy and 64 bits, of attention with shaped scores, of
the packed cache and of eviction, and the inputs that their tests share. Caches are
kept as logical rows [blocks, kv heads, 16 tokens, 128]; only pack and unpack know
the packed layout."""
import numpy as np

from paper_2411_01142_amd import workloads as W

D, BS, RECORD = 128, 16, 2176
NUMBERS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], np.float64)


def bf16(x):
    """float64 values of x rounded to bf16."""
    return W.bf16_to_f32(W.to_bf16(np.asarray(x, np.float32))).astype(np.float64)


def bits(x):
    """bf16 bits (uint16) of values that bf16 holds."""
    return W.to_bf16(np.asarray(x, np.float32))


# ---------------------------------------------------------------- packed cache

def quantise(x):
    """(codes, exponent bytes) of bf16 values [..., 128], by the definition: numbers are
    looked for in the list of all of them."""
    x = np.asarray(x, np.float64).reshape(*x.shape[:-1], D // 32, 32)
    top = np.max(np.where(np.isfinite(x), np.abs(x), 0), axis=-1)
    e = np.full(top.shape, -125, np.int64)
    while True:
        more = (top >= 7 * 2.0 ** e) & (e < 125)
        if not more.any():
            break
        e = e + more
    with np.errstate(invalid="ignore"):
        t = x / 2.0 ** e[..., None]
        off = np.abs(np.abs(t)[..., None] - NUMBERS)       # distance to each number
        best = off.min(-1, keepdims=True)
        near = off == best
        even = near & (np.arange(8) % 2 == 0)
        code = np.where(even.any(-1), even.argmax(-1), near.argmax(-1))
    code = code + 8 * (t < 0)
    byte = np.where(top == 0, 0, e + 127)
    bad = ~np.isfinite(x).all(-1)
    byte = np.where(bad, 255, byte)
    code = np.where(bad[..., None], 0, code)
    return code.reshape(*code.shape[:-2], D).astype(np.uint8), byte.astype(np.uint8)


def values(code, byte):
    """float64 values of codes [..., 128] and exponent bytes [..., 4]."""
    v = np.where(code >= 8, -1.0, 1.0) * NUMBERS[code & 7]
    s = np.where(byte == 0, 0.0, 2.0 ** (byte.astype(np.float64) - 127))
    s = np.where(byte == 255, np.nan, s)
    return v * np.repeat(s, 32, axis=-1)


def _places():
    """Byte offsets in a record: of each token's and dim's K and V code, and exponent."""
    t, d = np.arange(BS)[:, None], np.arange(D)[None, :]
    k = (d // 32) * 256 + t * 16 + (d % 32) // 2
    v = 1024 + (t // 4) * 256 + (d // 8) * 16 + (t % 4) * 4 + (d % 8) // 2
    g = np.arange(4)[None, :]
    return k, v, 2048 + g * 16 + t, 2112 + (t // 4) * 16 + g * 4 + t % 4


def pack(kc, kb, vc, vb):
    """Records uint8 [..., 2176] of codes [..., 16, 128] and exponent bytes [..., 16, 4]."""
    rec = np.zeros((*kc.shape[:-2], RECORD), np.uint8)
    pk, pv, pke, pve = _places()
    for c, at in ((kc, pk), (vc, pv)):
        rec[..., at[:, 0::2]] = c[..., 0::2] | (c[..., 1::2] << 4)
    rec[..., pke], rec[..., pve] = kb, vb
    return rec


def unpack(rec):
    """(k, v) float64 [..., 16, 128] of records."""
    pk, pv, pke, pve = _places()
    out = []
    for at, ex in ((pk, pke), (pv, pve)):
        byte = rec[..., at]
        code = np.where(np.arange(D) % 2 == 1, byte >> 4, byte & 15)
        out.append(values(code, rec[..., ex]))
    return out


# ------------------------------------------------------------------- attention

def seen_tokens(L, start, prefix):
    t = np.arange(max(L, 0))
    return t[(t < prefix) | (t >= start)]


def rows_of(cache, table_row, t):
    """Rows [kv heads, len(t), 128] of tokens t from logical blocks."""
    return cache[table_row[t // BS], :, t % BS].transpose(1, 0, 2)


def scores(q, K, t, L, scale, cap, slopes):
    """float64 [hkv, G, len(t)]."""
    hkv = K.shape[0]
    x = scale * np.matmul(q.reshape(hkv, -1, D), K.transpose(0, 2, 1))
    if cap:
        x = cap * np.tanh(x / cap)
    if slopes is not None:
        x = x + slopes.reshape(hkv, -1, 1) * (t - (L - 1)).astype(np.float64)
    return x


def attention(q, k, v, table, lens, scale=None, cap=0.0, slopes=None, starts=None, prefix=None):
    """(out [B, hq, 128], lse [B, hq]) in float64; k, v logical blocks."""
    B, hq, _ = q.shape
    out, lse = np.zeros((B, hq, D)), np.full((B, hq), -np.inf)
    for b in range(B):
        L = min(max(int(lens[b]), 0), table.shape[1] * BS)
        t = seen_tokens(L, 0 if starts is None else starts[b], 0 if prefix is None else prefix[b])
        if len(t) == 0:
            continue
        x = scores(q[b], rows_of(k, table[b], t), t, L, scale or D ** -0.5, cap, slopes)
        top = x.max(-1, keepdims=True)
        w = np.exp(x - top)
        z = w.sum(-1, keepdims=True)
        out[b] = np.matmul(w / z, rows_of(v, table[b], t)).reshape(hq, D)
        lse[b] = (top + np.log(z)).reshape(hq)
    return out, lse


def weight_sums(sums, lse, q, k, table, lens, scale=None, cap=0.0, slopes=None, starts=None,
                prefix=None):
    out = sums.astype(np.float64).copy()
    for b in range(q.shape[0]):
        L = min(max(int(lens[b]), 0), table.shape[1] * BS)
        t = seen_tokens(L, 0 if starts is None else starts[b], 0 if prefix is None else prefix[b])
        if len(t) == 0:
            continue
        x = scores(q[b], rows_of(k, table[b], t), t, L, scale or D ** -0.5, cap, slopes)
        out[b][:, t] += np.exp(x - lse[b].reshape(k.shape[1], -1, 1)).sum(1)
    return out


def kept_tokens(sums, L, n, recent):
    """Positions that stay, ascending: the newest, then the largest sums, ties to the lower."""
    recent = min(recent, n)
    old = L - recent
    key = np.where(np.isnan(sums[:old]), np.inf, sums[:old])
    nan = np.isnan(sums[:old])
    order = sorted(range(old), key=lambda i: (not nan[i], -key[i], i))
    return np.array(sorted(order[:n - recent]) + list(range(old, L)), np.int64)


# --------------------------------------------------------------------- inputs

def make_table(lens, rng, spare=5, extra_cols=0, new_cols=0):
    """(table with -1 where unused, new table, blocks in the pool), blocks scattered."""
    need = [(max(int(L), 0) + BS - 1) // BS for L in lens]
    B = len(lens)
    pool = sum(need) + spare + B * new_cols
    order = rng.permutation(pool).astype(np.int32)
    table = np.full((B, max(max(need), 1) + extra_cols), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    new = order[at:at + B * new_cols].reshape(B, new_cols)
    return table, new, pool


def make_rows(pool, hkv, rng):
    """Logical K and V blocks of N(0, 1) bf16 values."""
    return [bf16(rng.standard_normal((pool, hkv, BS, D))) for _ in range(2)]
