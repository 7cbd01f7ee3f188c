"""Operators around decode attention, as timed cases, with their plain forms.

A serving program that decodes from a paged KV cache needs, beside plain decode
attention: scores that are capped by a tanh, biased by distance or masked by
documents and prefixes; a cache held in 4 bits, with its append, its read-back
and the attention that reads it; and, where memory ends, the sums of the
attention weights by which tokens are evicted, with the eviction itself. The
cases cover those through the package's public entry points.

A case is a dict of plain values:

* ``op``: ``attend`` (one attention call, with its log-sum-exps), ``append``
  (new rows into a 4-bit cache, and their values read back), ``weights``
  (attention weights added to sums) or ``evict`` (the lightest tokens left out);
* ``cache``: ``bf16`` (K ``[NB, Hkv, 16, 16, 8]``, V ``[NB, Hkv, 128, 16]``) or
  ``packed`` (uint8 ``[NB, Hkv, 2176]``, below);
* ``hq``, ``hkv``: query and kv heads; head_dim is 128 and a block 16 tokens;
* ``batch``, ``lo``, ``hi``: requests and their cached lengths, uniform in
  [lo, hi], drawn from ``lens_seed``;
* ``cap`` (0: none), ``slopes`` (a bias by distance), ``mask`` (``none``;
  ``window``: the newest ``span`` tokens and the first 4; ``document``: from a
  drawn token on, and a drawn prefix, one request in nine seeing nothing);
* ``rows``: for ``append``, ``one`` (a token a request) or ``all`` (prompts);
* ``budget``, ``recent``: for ``evict``, the tokens kept, and how many of them
  are the newest ones.

A score is ``s = scale * q.k``, then ``s = cap * tanh(s / cap)``, then
``s += slope * (t - (L - 1))``, for the tokens t that the request sees:
``t < prefix`` or ``t >= start``, below its length L.

The packed cache holds 4-bit numbers (a sign, 0, 0.5, 1, 1.5, 2, 3, 4 or 6)
with one power of two for every 32 dims of a token. The 2176 bytes of a block
and kv head are

* K: ``[4 dim groups][16 tokens][16 bytes]``, byte j dims 2j (low half), 2j + 1;
* V: ``[4 token groups][16 dim octets][4 tokens][4 bytes]``, likewise;
* the exponents (plus 127) of K ``[4 dim groups][16 tokens]`` and of
  V ``[4 token groups][4 dim groups][4 tokens]``.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False  # True: the package's operators, False: plain torch

D = 128     # head dim
BS = 16     # tokens per block
GROUP = 32  # dims that share an exponent
RECORD = 2176


def _attend(name, cache, hq, hkv, batch, lo, hi, cap=0.0, slopes=False, mask="none", span=0,
            op="attend"):
    return {"name": name, "op": op, "cache": cache, "hq": hq, "hkv": hkv, "batch": batch,
            "lo": lo, "hi": hi, "lens_seed": 11, "cap": cap, "slopes": slopes, "mask": mask,
            "span": span}


def listed():
    return [
        # One interactive user of a model with capped scores, a chat of under a
        # thousand tokens: the smallest call, launch and latency.
        _attend("cap_one_877", "bf16", 32, 8, 1, 877, 877, cap=30.0),
        # A serving batch with distance biases, each request a document behind a
        # shared prefix.
        _attend("bias_documents_64", "bf16", 32, 8, 64, 512, 2048, slopes=True, mask="document"),
        # A 70B-shaped layer whose requests see a window and the first tokens.
        _attend("window_cap_256", "bf16", 64, 8, 256, 256, 4096, cap=50.0, mask="window",
                span=1500),
        # 4-bit caches: a small batch without grouped heads, one long document,
        # and the largest, a 70B-shaped layer.
        _attend("packed_mha_small", "packed", 32, 32, 4, 64, 512, slopes=True),
        _attend("packed_one_long", "packed", 32, 8, 1, 50021, 50021),
        _attend("packed_layer70b_512", "packed", 64, 8, 512, 256, 4096),
        # Writing into a 4-bit cache: the new token of each request of a batch, and
        # the prompts of five requests (ragged).
        {"name": "append_256", "op": "append", "cache": "packed", "hq": 32, "hkv": 8,
         "batch": 256, "lo": 64, "hi": 1024, "lens_seed": 13, "rows": "one"},
        {"name": "append_prompts", "op": "append", "cache": "packed", "hq": 32, "hkv": 8,
         "batch": 5, "lo": 1000, "hi": 6000, "lens_seed": 14, "rows": "all"},
        # The weights of a step added to the sums by which tokens are evicted.
        _attend("weights_64", "bf16", 32, 8, 64, 512, 2048, op="weights"),
        _attend("weights_packed_256", "packed", 64, 8, 256, 256, 4096, cap=50.0, op="weights"),
        # One conversation cut from 4099 tokens to 1024, and a batch of long ones.
        {"name": "evict_one", "op": "evict", "cache": "bf16", "hq": 32, "hkv": 8, "batch": 1,
         "lo": 4099, "hi": 4099, "lens_seed": 15, "budget": 1024, "recent": 64},
        {"name": "evict_packed_96", "op": "evict", "cache": "packed", "hq": 64, "hkv": 8,
         "batch": 96, "lo": 2048, "hi": 8192, "lens_seed": 16, "budget": 1500, "recent": 128},
    ]


def draw(rng):
    """One more case of the ranges above."""
    def logu(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choices(["attend", "append", "weights", "evict"], [6, 2, 2, 2])[0]
    cache = "packed" if op == "append" else rng.choice(["bf16", "packed"])
    hkv = rng.choice([1, 2, 4, 8, 8, 8, 16, 32])
    group = rng.choice([g for g in (1, 2, 4, 4, 8, 8, 16) if hkv * g <= 128])
    most = {"attend": 6e6, "append": 3e5, "weights": 3e6, "evict": 2e6}[op]  # tokens x kv heads
    batch = logu(1, {"attend": 600, "append": 300, "weights": 300, "evict": 100}[op])
    mean = min(logu(20, 60000), most / (batch * hkv))
    mean = max(mean, 5)
    spread = rng.choice([0.0, 0.5, 0.9])
    case = {"op": op, "cache": cache, "hq": hkv * group, "hkv": hkv, "batch": batch,
            "lo": max(1, int(mean * (1 - spread))), "hi": int(mean * (1 + spread)),
            "lens_seed": rng.randrange(1 << 20)}
    if op in ("attend", "weights"):
        case["cap"] = rng.choice([0.0, 0.0, 15.0, 50.0])
        case["slopes"] = rng.random() < 0.4
        case["mask"] = rng.choice(["none", "none", "window", "document"])
        case["span"] = max(1, int(mean * rng.uniform(0.1, 1.0))) if case["mask"] == "window" else 0
    elif op == "append":
        case["rows"] = rng.choice(["one", "all"])
    else:
        case["budget"] = max(1, int(mean * rng.uniform(0.1, 0.9)))
        case["recent"] = rng.choice([0, 1, case["budget"] // 8, case["budget"]])
    return case


# ------------------------------------------------------------------ inputs

def _lens(case):
    """Cached length of each request, the token being decoded included."""
    r = np.random.default_rng(case["lens_seed"])
    return r.integers(case["lo"], case["hi"], size=case["batch"], endpoint=True).astype(np.int32)


def _ranges(case):
    """(starts, prefix lengths), or (None, None)."""
    lens, mask = _lens(case).astype(np.int64), case["mask"]
    if mask == "none":
        return None, None
    if mask == "window":
        return np.maximum(lens - case["span"], 0).astype(np.int32), np.full(len(lens), 4, np.int32)
    r = np.random.default_rng(case["lens_seed"] + 1)
    start = np.floor(lens * r.random(len(lens))).astype(np.int32)
    prefix = np.floor(lens * r.random(len(lens)) * 0.3).astype(np.int32)
    nothing = r.random(len(lens)) < 1 / 9
    start[nothing], prefix[nothing] = lens[nothing] + 3, 0
    return start, prefix


def _seen(case):
    """Tokens that each request sees, and the blocks that hold them."""
    lens = _lens(case).astype(np.int64)
    start, prefix = _ranges(case)
    if start is None:
        return lens, (lens + BS - 1) // BS
    p = np.minimum(prefix, lens)
    s = np.minimum(np.maximum(start, p), lens)
    first = np.minimum(np.maximum(s // BS, (p + BS - 1) // BS), (lens + BS - 1) // BS)
    blocks = (p + BS - 1) // BS + np.where(s < lens, (lens + BS - 1) // BS - first, 0)
    return p + lens - s, blocks


def _table(lens, seed, extra=0):
    """(block table, its first spare block's number in the order of the pool, the order):
    the requests' blocks scattered over the pool, -1 where unused, and ``extra`` spare blocks."""
    nblk = (lens.astype(np.int64) + BS - 1) // BS
    used = int(nblk.sum())
    pool = used + math.ceil(0.05 * used) + extra
    order = np.random.default_rng(seed).permutation(pool).astype(np.int32)
    table = np.full((len(lens), int(nblk.max())), -1, np.int32)
    table[np.arange(table.shape[1])[None, :] < nblk[:, None]] = order[:used]
    return table, used, order


def _normal(shape, gen):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)


def _filled(cache, blocks, hkv, gen):
    """The caches' tensors, filled with N(0, 1) values: K and V views of one buffer, or one of bytes."""
    if cache == "bf16":
        buf = torch.empty((blocks, 2, hkv, D * BS), dtype=torch.bfloat16, device="cuda")
    else:
        buf = torch.empty((blocks, hkv, RECORD), dtype=torch.uint8, device="cuda")
    for i in range(0, blocks, 16384):
        part = buf[i:i + 16384]
        if cache == "bf16":
            part.copy_(_normal(part.shape, gen))
        else:
            shape = (part.shape[0], hkv, BS, D)
            part.copy_(_pack(*_quantise(_normal(shape, gen).float()),
                             *_quantise(_normal(shape, gen).float())))
    if cache == "bf16":
        return [buf[:, 0].view(blocks, hkv, D // 8, BS, 8), buf[:, 1].view(blocks, hkv, D, BS)]
    return [buf]


def _gpu(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    lens = _lens(case)
    B, hq, hkv, op = case["batch"], case["hq"], case["hkv"], case["op"]
    new_blocks = (case["budget"] + BS - 1) // BS if op == "evict" else 0
    table, used, order = _table(lens, seed, B * new_blocks)
    s = {"op": op, "kind": case["cache"], "lens": _gpu(lens), "table": _gpu(table),
         "cache": _filled(case["cache"], len(order), hkv, gen)}
    if op in ("attend", "weights"):
        start, prefix = _ranges(case)
        slopes = None
        if case["slopes"]:  # 2^-8 .. 2^-0.5 or thereabouts, a geometric row over the heads
            slopes = torch.exp2(-8.0 * torch.arange(1, hq + 1, device="cuda") / hq)
        s.update(q=_normal((B, hq, D), gen), cap=case["cap"] or None, slopes=slopes,
                 starts=_gpu(start), prefix=_gpu(prefix))
    if op == "attend":
        s.update(out=torch.empty((B, hq, D), device="cuda"), lse=torch.empty((B, hq), device="cuda"))
    elif op == "weights":
        s["lse"] = _plain_attend(s)[1]
        s["sums"] = torch.rand((B, hkv, table.shape[1] * BS), generator=gen, device="cuda")
        s["out"] = s["sums"].clone()
    elif op == "append":
        counts = lens.astype(np.int64) if case["rows"] == "all" else np.ones(B, np.int64)
        rows = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        s["row_starts"] = _gpu(rows) if case["rows"] == "all" else None
        shape = (int(rows[-1]), hkv, D)
        # Values of several magnitudes, as keys have by channel.
        gain = torch.exp2(torch.randint(-3, 4, (1, hkv, D), generator=gen, device="cuda").float())
        s["k_new"] = (_normal(shape, gen) * gain).to(torch.bfloat16)
        s["v_new"] = _normal(shape, gen)
        s["k_out"], s["v_out"] = torch.empty_like(s["k_new"]), torch.empty_like(s["v_new"])
    else:
        # Sums of attention weights: few heavy tokens, many light ones, some never seen.
        x = torch.rand((B, hkv, table.shape[1] * BS), generator=gen, device="cuda")
        s["sums"] = torch.where(x < 0.1, torch.zeros_like(x), x.pow(12) * 40)
        s["new_table"] = _gpu(order[used:used + B * new_blocks].reshape(B, new_blocks))
        s["budgets"] = torch.full((B,), case["budget"], dtype=torch.int32, device="cuda")
        s["recent"] = case["recent"]
    return s


def run(s):
    if own:
        return _own(s)
    if s["op"] == "attend":
        return list(_plain_attend(s))
    if s["op"] == "append":
        return _plain_append(s)
    if s["op"] == "weights":
        return _plain_weights(s)
    return _plain_evict(s)


def _own(s):
    """The same through the package."""
    import paper_2411_01142_amd as neo
    op, packed = s["op"], s["kind"] == "packed"
    if op == "attend":
        attend = neo.packed_decode_attention if packed else neo.shaped_decode_attention
        attend(s["q"], *s["cache"], s["table"], s["lens"], out=s["out"], lse=s["lse"],
               softcap=s["cap"], slopes=s["slopes"], starts=s["starts"], prefix_lens=s["prefix"])
        return [s["out"], s["lse"]]
    if op == "append":
        neo.packed_append(*s["cache"], s["k_new"], s["v_new"], s["table"], s["lens"],
                          s["row_starts"])
        neo.packed_gather(*s["cache"], s["table"], s["lens"], s["row_starts"], k_out=s["k_out"],
                          v_out=s["v_out"])
        return [s["k_out"], s["v_out"]]
    if op == "weights":
        add = neo.packed_add_attention_weights if packed else neo.add_attention_weights
        add(s["sums"], s["lse"], s["q"], *s["cache"][:1], s["table"], s["lens"], out=s["out"],
            softcap=s["cap"], slopes=s["slopes"], starts=s["starts"], prefix_lens=s["prefix"])
        return s["out"]
    evict = neo.packed_evict if packed else neo.kv_evict
    new_lens, kept, sums = evict(*s["cache"], s["table"], s["lens"], s["sums"], s["budgets"],
                                 s["new_table"], recent=s["recent"])
    return [new_lens, kept, sums, *s["cache"]]


# ------------------------------------------------------------- plain forms

_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _quantise(x):
    """(codes uint8, exponents + 127 uint8) of x, fp32 [..., 128]: per 32 dims the smallest
    power of two under which the largest magnitude is below 7 (it then rounds to at most 6),
    within [-125, 125]; every value to the nearest of the eight magnitudes, ties to the even
    one. A group of zeros has exponent byte 0, one with an infinity or NaN 255."""
    g = x.unflatten(-1, (D // GROUP, GROUP))
    top = g.abs().amax(-1)
    m, e = torch.frexp(top)
    e = (e - 3 + (m >= 0.875).to(e.dtype)).clamp(-125, 125)
    t = torch.ldexp(g, -e.unsqueeze(-1))
    a = t.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75).to(torch.uint8) + (a > 1.25).to(torch.uint8)
            + (a >= 1.75).to(torch.uint8) + (a > 2.5).to(torch.uint8) + (a >= 3.5).to(torch.uint8)
            + (a > 5).to(torch.uint8))
    code = code + 8 * (t < 0).to(torch.uint8)
    scale = torch.where(top == 0, torch.zeros_like(e), e + 127)
    scale = torch.where(torch.isfinite(top), scale, torch.full_like(e, 255))
    return code.flatten(-2), scale.to(torch.uint8)


def _pack(kc, ks, vc, vs):
    """Whole blocks [n, Hkv, 16 tokens, 128] of codes, and [n, Hkv, 16, 4] exponents, as records."""
    n, h = kc.shape[:2]
    k, v = ((c[..., 0::2] + 16 * c[..., 1::2]) for c in (kc, vc))  # [n, h, token, 64 bytes]
    return torch.cat([
        k.view(n, h, BS, 4, 16).transpose(2, 3).reshape(n, h, -1),
        v.view(n, h, 4, 4, 16, 4).transpose(3, 4).reshape(n, h, -1),
        ks.transpose(2, 3).reshape(n, h, -1),
        vs.view(n, h, 4, 4, 4).transpose(3, 4).reshape(n, h, -1)], dim=-1)


def _unpacked(rec):
    """(k, v) fp32 [n, Hkv, 16, 128] of whole records [n, Hkv, 2176]."""
    n, h = rec.shape[:2]
    k = rec[..., :1024].view(n, h, 4, BS, 16).transpose(2, 3).reshape(n, h, BS, 64)
    v = rec[..., 1024:2048].view(n, h, 4, 16, 4, 4).transpose(3, 4).reshape(n, h, BS, 64)
    ks = rec[..., 2048:2112].view(n, h, 4, BS).transpose(2, 3)
    vs = rec[..., 2112:].view(n, h, 4, 4, 4).transpose(3, 4).reshape(n, h, BS, 4)
    return _dequantise(k, ks), _dequantise(v, vs)


def _dequantise(b, e):
    """fp32 [..., 128] of bytes [..., 64] and exponent bytes [..., 4]."""
    code = torch.stack([b & 15, b >> 4], dim=-1).flatten(-2)
    exp, odd = (code >> 1) & 3, (code & 1).float()
    mag = torch.where(exp == 0, 0.5 * odd, (1 + 0.5 * odd) * torch.exp2(exp.float() - 1))
    val = torch.where(code >= 8, -mag, mag).unflatten(-1, (D // GROUP, GROUP))
    scale = torch.exp2(e.float() - 127).masked_fill(e == 0, 0.0).masked_fill(e == 255, float("nan"))
    return (val * scale.unsqueeze(-1)).flatten(-2)


def _dense(s, want=(0, 1)):
    """K and/or V as fp32 [B, Hkv, table width x 16, 128]."""
    table = s["table"].clamp(min=0).long()
    B, M = table.shape
    if s["kind"] == "packed":
        rec = s["cache"][0][table.flatten()]
        both = _unpacked(rec)
    else:
        both = []
        for i in want:
            c = s["cache"][i][table.flatten()]
            both.append((c.permute(0, 1, 3, 2, 4) if i == 0 else c.transpose(2, 3))
                        .reshape(B * M, c.shape[1], BS, D).float())
        both = both if len(want) == 2 else both * 2
    return [both[i].view(B, M, -1, BS, D).transpose(1, 2).reshape(B, -1, M * BS, D) for i in want]


def _plain_scores(s, k):
    """fp32 scores [B, Hkv, G, T], minus infinity where a token is not seen, and who sees it."""
    B, hkv, T, _ = k.shape
    hq = s["q"].shape[1]
    q = s["q"].float().view(B, hkv, hq // hkv, D)
    x = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(D)
    if s["cap"]:
        x = s["cap"] * torch.tanh(x / s["cap"])
    L = s["lens"].view(B, 1, 1, 1)
    t = torch.arange(T, device=x.device).view(1, 1, 1, T)
    if s["slopes"] is not None:
        x = x + s["slopes"].view(1, hkv, -1, 1) * (t - (L - 1)).float()
    seen = t < L
    if s["starts"] is not None:
        seen = seen & ((t < s["prefix"].view(B, 1, 1, 1)) | (t >= s["starts"].view(B, 1, 1, 1)))
    return x.masked_fill(~seen, -math.inf), seen


def _plain_attend(s):
    k, v = _dense(s)
    x, _ = _plain_scores(s, k)
    B, hkv, G, _ = x.shape
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    w = torch.exp(x - top)
    z = w.sum(-1, keepdim=True)
    out = torch.matmul(w, v) / torch.where(z == 0, torch.ones_like(z), z)
    lse = (top + torch.log(z)).view(B, hkv * G)
    return out.view(B, hkv * G, D), lse


def _plain_weights(s):
    k, = _dense(s, (0,))
    x, seen = _plain_scores(s, k)
    B, hkv, G, T = x.shape
    lse = s["lse"].view(B, hkv, G, 1)
    w = torch.where(seen, torch.exp(x - lse), torch.zeros_like(x)).sum(2)
    return torch.where(seen[:, 0], s["sums"] + w, s["out"])


def _rows(s):
    """Request and token of each new row."""
    n = s["k_new"].shape[0]
    r = torch.arange(n, device="cuda")
    if s["row_starts"] is None:
        return r, s["lens"].long() - 1
    ends = s["row_starts"][1:].long()
    b = torch.searchsorted(ends, r, right=True)
    return b, s["lens"].long()[b] - (ends[b] - r)


def _plain_append(s):
    b, t = _rows(s)
    blk, slot = s["table"].long()[b, t // BS], t % BS
    cache = s["cache"][0]
    nb, h, _ = cache.shape
    outs = []
    for which, new in enumerate((s["k_new"], s["v_new"])):
        code, e = _quantise(new.float())
        byte = code[..., 0::2] + 16 * code[..., 1::2]
        at = cache[..., 1024 * which:1024 * which + 1024]
        sc = cache[..., 2048 + 64 * which:2112 + 64 * which]
        if which == 0:  # [blk, h, dim group, token, 16]
            at.unflatten(-1, (4, BS, 16))[blk, :, :, slot] = byte.view(-1, h, 4, 16)
            sc.unflatten(-1, (4, BS))[blk, :, :, slot] = e
        else:           # [blk, h, token group, octet, token, 4]
            at.unflatten(-1, (4, 16, 4, 4))[blk, :, slot // 4, :, slot % 4] = byte.view(-1, h, 16, 4)
            sc.unflatten(-1, (4, 4, 4))[blk, :, slot // 4, :, slot % 4] = e
        outs.append(_dequantise(byte, e).to(torch.bfloat16))
    return outs


def _plain_evict(s):
    sums, lens, table, new = s["sums"], s["lens"].long(), s["table"].clamp(min=0).long(), s["new_table"]
    B, hkv, T = sums.shape
    N = new.shape[1] * BS
    keep = torch.minimum(lens, s["budgets"].long().clamp(0, N))
    recent = keep.clamp(max=s["recent"])
    t = torch.arange(T, device="cuda").view(1, 1, T)
    L = lens.view(B, 1, 1)
    key = torch.where(t >= L - recent.view(B, 1, 1), torch.full_like(sums, math.inf), sums)
    key = key.masked_fill(t >= L, -math.inf)
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(2, order, t.expand(B, hkv, T).contiguous())
    kept = torch.where(rank < keep.view(B, 1, 1), t, torch.full_like(order, T))
    kept = torch.sort(kept, dim=-1).values[..., :N]
    if kept.shape[2] < N:
        kept = torch.nn.functional.pad(kept, (0, N - kept.shape[2]), value=T)
    valid = kept < T
    src = kept.clamp(max=T - 1)
    new_sums = torch.where(valid, torch.gather(sums, 2, src), torch.zeros_like(src, dtype=sums.dtype))
    blk = torch.gather(table.view(B, 1, -1).expand(B, hkv, -1), 2, src // BS)
    head = torch.arange(hkv, device="cuda").view(1, hkv, 1)
    slot = src % BS
    full = (torch.arange(N // BS, device="cuda").view(1, -1) * BS < keep.view(B, 1))
    ids = new[full].long()

    def blocks(x):  # [B, Hkv, N, ...] -> the written blocks [n, Hkv, 16, ...]
        x = x * valid.view(*valid.shape, *[1] * (x.dim() - 3)).to(x.dtype)
        return x.unflatten(2, (N // BS, BS)).transpose(1, 2)[full]

    if s["kind"] == "packed":
        rec, = s["cache"]
        part = [rec[..., :1024].unflatten(-1, (4, BS, 16))[blk, head, :, slot],
                rec[..., 1024:2048].unflatten(-1, (4, 16, 4, 4))[blk, head, slot // 4, :, slot % 4],
                rec[..., 2048:2112].unflatten(-1, (4, BS))[blk, head, :, slot],
                rec[..., 2112:].unflatten(-1, (4, 4, 4))[blk, head, slot // 4, :, slot % 4]]
        k, v, ks, vs = (blocks(x) for x in part)
        n = k.shape[0]
        rec[ids] = torch.cat([
            k.transpose(2, 3).reshape(n, hkv, -1),
            v.view(n, hkv, 4, 4, 16, 4).transpose(3, 4).reshape(n, hkv, -1),
            ks.transpose(2, 3).reshape(n, hkv, -1),
            vs.view(n, hkv, 4, 4, 4).transpose(3, 4).reshape(n, hkv, -1)], dim=-1)
    else:
        k_cache, v_cache = s["cache"]
        k_cache[ids] = blocks(k_cache[blk, head, :, slot]).transpose(2, 3)
        v_cache[ids] = blocks(v_cache[blk, head, :, slot]).transpose(2, 3)
    kept = torch.where(valid, kept, torch.full_like(kept, -1)).to(torch.int32)
    return [keep.to(torch.int32), kept, new_sums, *s["cache"]]


# -------------------------------------------------------------- accounting

def work(case):
    lens = _lens(case).astype(np.int64)
    B, hq, hkv, op = case["batch"], case["hq"], case["hkv"], case["op"]
    token = 2 * D * 2 if case["cache"] == "bf16" else 2 * (D // 2 + D // GROUP)  # K and V of a head
    if op == "append":
        rows = int(lens.sum()) if case["rows"] == "all" else B
        # bf16 rows in, 4-bit rows out, and the way back
        return {"bytes": rows * hkv * 2 * (token + 2 * D * 2) + 8 * B, "flops": 0}
    if op == "evict":
        keep = int(np.minimum(lens, case["budget"]).sum())
        slots = B * hkv * ((case["budget"] + BS - 1) // BS * BS)
        return {"bytes": int(lens.sum()) * hkv * 4 + keep * hkv * 2 * token + slots * 8, "flops": 0}
    seen, blocks = (int(x.sum()) for x in _seen(case))
    small = B * hq * (2 * D + 4) + 4 * blocks + 4 * B
    if op == "weights":
        return {"bytes": seen * hkv * (token // 2 + 8) + small, "flops": seen * hq * D * 2}
    return {"bytes": seen * hkv * token + small + B * hq * D * 4, "flops": seen * hq * D * 4}


# ------------------------------------------------------------- in 64 bits

def _exact_rows(s, b, L):
    """K and V of a request's tokens, fp64 [Hkv, L, 128], read token by token from the layouts."""
    n = (L + BS - 1) // BS
    ids = s["table"][b, :n].long()
    if s["kind"] == "bf16":
        k, v = s["cache"]
        K = k[ids].permute(1, 0, 3, 2, 4).reshape(k.shape[1], n * BS, D)
        V = v[ids].permute(1, 0, 3, 2).reshape(v.shape[1], n * BS, D)
        return K[:, :L].double(), V[:, :L].double()
    rec = s["cache"][0][ids].transpose(0, 1).contiguous()  # [Hkv, n, 2176]
    d = torch.arange(D, device="cuda").view(1, D)
    t = torch.arange(BS, device="cuda").view(BS, 1)
    lut = torch.tensor(_VALUES + tuple(-x for x in _VALUES), dtype=torch.float64, device="cuda")
    places = ((d // 32) * 256 + t * 16 + (d % 32) // 2, 2048 + (d // 32) * 16 + t), \
        (1024 + (t // 4) * 256 + (d // 8) * 16 + (t % 4) * 4 + (d % 8) // 2,
         2112 + (t // 4) * 16 + (d // 32) * 4 + t % 4)
    out = []
    for byte_at, exp_at in places:
        byte, e = rec[..., byte_at], rec[..., exp_at]
        code = torch.where(d % 2 == 1, byte >> 4, byte & 15).long()
        val = lut[code] * torch.exp2(e.double() - 127) * (e > 0)
        out.append(val.reshape(rec.shape[0], n * BS, D)[:, :L])
    return out


def exact(case, seed):
    """What ``run`` returns for these inputs, in 64 bits, request by request; None for data
    that only moves."""
    op = case["op"]
    if op == "evict":
        return None
    s = prepare(case, seed)
    if op == "append":
        outs = []
        for new in (s["k_new"], s["v_new"]):
            x = new.double().view(*new.shape[:2], D // GROUP, GROUP)
            top = x.abs().amax(-1, keepdim=True)
            e = torch.floor(torch.log2(top / 7)) + 1           # smallest e with top < 7 * 2^e
            e = torch.where(top >= 7 * torch.exp2(e), e + 1, e)
            e = torch.where(top < 7 * torch.exp2(e - 1), e - 1, e).clamp(-125, 125)
            y = x / torch.exp2(e)
            # One mantissa bit from 1 on, steps of a half below: round half to even by steps.
            step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=1))) - 1)
            y = (torch.round(y / step) * step).clamp(-6, 6)
            outs.append(torch.where(top > 0, y * torch.exp2(e), 0.0).view(new.shape))
        return outs
    lens = _lens(case)
    B, hq, hkv = case["batch"], case["hq"], case["hkv"]
    G = hq // hkv
    outs = torch.zeros((B, hq, D), dtype=torch.float64, device="cuda")
    lse = torch.full((B, hq), -math.inf, dtype=torch.float64, device="cuda")
    sums = s["out"].double() if op == "weights" else None
    start, prefix = _ranges(case)
    for b in range(B):
        L = int(lens[b])
        K, V = _exact_rows(s, b, L)
        t = torch.arange(L, device="cuda")
        Q = s["q"][b].double().view(hkv, G, D)
        x = torch.matmul(Q, K.transpose(1, 2).contiguous()) / math.sqrt(D)
        if s["cap"]:
            x = s["cap"] * torch.tanh(x / s["cap"])
        if s["slopes"] is not None:
            x = x + s["slopes"].double().view(hkv, G, 1) * (t - (L - 1)).double()
        at = t
        if start is not None:
            at = t[(t < int(prefix[b])) | (t >= int(start[b]))]
        if at.numel() == 0:
            continue
        x, V = x[..., at], V[:, at]
        if op == "weights":
            w = torch.exp(x - s["lse"][b].double().view(hkv, G, 1)).sum(1)
            sums[b][:, at] = s["sums"][b][:, at].double() + w
            continue
        lse[b] = torch.logsumexp(x, -1).view(hq)
        outs[b] = torch.matmul(torch.softmax(x, -1), V.contiguous()).view(hq, D)
    return sums if op == "weights" else [outs, lse]
