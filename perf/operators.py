"""The 8-bit cache's operators, as a serving program calls them: append to the cache, attention over it, eviction from it.

A case is a dict of plain values; `op` names the operator:
  append  quantises new keys and values (16-bit) and writes them into the cache, which holds one scale per 64 tokens and head
  attend  attention of n_q new tokens per sequence over the cache: 1 = a decode step, more = a chunk of a prompt (causal) or the
          tokens of a decoder over an encoder's states (not causal); with `weights` it also adds up every token's attention weights
  evict   keeps the first and the most recent tokens of each head and those with the largest weights, and closes the gaps
Lengths are uniform in [len_lo, len_hi], drawn with len_seed (part of the case, not of the inputs).  Places of the cache that hold no token
are filled with random bytes.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

BLOCK = 64               # tokens that share a scale
_BASE = dict(batch=1, q_heads=32, kv_heads=8, head_dim=128, code="int8", io="fp16", page=0, len_lo=1024, len_hi=1024, len_seed=0)


def _append(name=None, **kw):
    c = dict(_BASE, op="append", n_lo=1, n_hi=1)
    c.update(kw)
    return dict(c, name=name) if name else c


def _attend(name=None, **kw):
    c = dict(_BASE, op="attend", n_q=1, causal=False, q_ragged=False, weights=False)
    c.update(kw)
    return dict(c, name=name) if name else c


def _evict(name=None, **kw):
    c = dict(_BASE, op="evict", first=4, recent=64)
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # every decode step of eight conversations: one token each, anywhere inside a 64-token block
        _append("append_token", batch=8, len_lo=512, len_hi=8000, len_seed=1),
        # chunks of prompts of 32 requests of very different lengths, continuing part-filled pages
        _append("append_chunks_paged", batch=32, len_lo=0, len_hi=4000, len_seed=2, n_lo=1, n_hi=701, page=256, code="e4m3", io="bf16"),
        # prefill of eight long prompts into an empty cache
        _append("append_prompts", batch=8, len_lo=0, len_hi=0, n_lo=8192, n_hi=8192),
        # one short conversation on one head pair: the smallest call, where only latency counts
        _attend("decode_tiny", q_heads=1, kv_heads=1, len_lo=77, len_hi=77),
        # the ordinary decode step of a grouped-query model: 8 sequences of 8192 tokens
        _attend("decode_gqa", batch=8, len_lo=8192, len_hi=8192),
        # continuous batching: 32 requests of very different lengths in pages
        _attend("decode_ragged_paged", batch=32, len_lo=512, len_hi=16384, len_seed=4, page=256, code="e4m3", io="bf16"),
        # one very long context whose tokens' weights are added up for a later eviction
        _attend("decode_long_weights", len_lo=131072, len_hi=131072, weights=True),
        # a chunk of a long prompt of a grouped-query model: the matrix cores' rate counts
        _attend("chunk_causal", n_q=2048, len_lo=10240, len_hi=10240, causal=True, io="bf16"),
        # a prompt whose tokens' weights are added up, two sequences of different lengths (the shorter one padded)
        _attend("chunk_weights", batch=2, n_q=1000, len_lo=1200, len_hi=4200, len_seed=3, causal=True, q_ragged=True, weights=True,
                code="e4m3"),
        # a decoder's tokens over the states of an encoder, 64-channel heads, padded on both sides
        _attend("cross_heads64", batch=16, q_heads=12, kv_heads=12, head_dim=64, n_q=197, len_lo=300, len_hi=1500, len_seed=5, q_ragged=True),
        # a cache that has grown by 64 tokens beyond its budget
        _evict("evict_small", kv_heads=8, len_lo=1088, len_hi=1088, keep=1024),
        # prompts of different lengths cut down to their budget, in pages
        _evict("evict_prompts_paged", batch=8, len_lo=5000, len_hi=16384, len_seed=6, keep=4096, recent=512, page=256, code="e4m3"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    c = dict(head_dim=rng.choice((64, 128, 128)), code=rng.choice(("int8", "e4m3")), io=rng.choice(("fp16", "bf16")),
             page=rng.choice((0, 0, 64, 256)), len_seed=rng.randrange(1000))
    op = rng.choice(("append", "attend", "attend", "attend", "evict"))
    batch, kv = _log(rng, 1, 32), rng.choice((1, 2, 3, 4, 8, 12, 16))
    if op == "append":
        n = _log(rng, 1, min(8192, 65536 * 8 // (batch * kv)))
        return _append(batch=batch, kv_heads=kv, q_heads=kv, n_lo=rng.randint(1, n), n_hi=n, len_lo=0, len_hi=rng.randint(0, 5000), **c)
    if op == "evict":
        hi = _log(rng, 70, min(16384, 131072 * 8 // (batch * kv)))
        keep = _log(rng, 16, max(17, hi - 1))
        return _evict(batch=batch, kv_heads=kv, q_heads=kv, len_lo=rng.randint(1, hi), len_hi=hi, keep=keep, recent=rng.randint(0, keep // 2),
                      first=rng.randint(0, min(8, keep // 2)), **c)
    ratio = rng.choice((1, 2, 3, 4, 5, 8))
    form = rng.choice(("decode", "few", "chunk", "cross"))
    hi = _log(rng, 1, min(131072, 277000 * 8 // (batch * kv)))
    n_q = 1 if form == "decode" else _log(rng, 2, 16) if form == "few" else _log(rng, 17, 1500)
    rows = lambda: batch * kv * ratio * n_q * c["head_dim"]  # noqa: E731
    while form in ("chunk", "cross") and (rows() * hi > 6e10 or rows() > 4e7):  # below the largest listed ones
        hi, n_q, batch = max(n_q, hi // 2), max(17, n_q * 3 // 4), max(1, batch * 3 // 4)
    return _attend(batch=batch, q_heads=kv * ratio, kv_heads=kv, n_q=n_q, causal=form in ("few", "chunk"), q_ragged=n_q > 1 and rng.random() < 0.5,
                   weights=rng.random() < 0.35, len_lo=rng.randint(max(1, hi // 8), hi), len_hi=hi, **c)


def _lengths(case):
    """Tokens in the cache, and new tokens, per sequence."""
    r = random.Random(case["len_seed"])
    lens = [r.randint(case["len_lo"], case["len_hi"]) for _ in range(case["batch"])]
    if case["op"] == "append":
        new = [r.randint(case["n_lo"], case["n_hi"]) for _ in range(case["batch"])]
        new[0] = case["n_hi"]
    elif case["op"] == "attend":
        new = [r.randint(1, case["n_q"]) if case["q_ragged"] else case["n_q"] for _ in range(case["batch"])]
        new[0] = case["n_q"]
    else:
        new = [0] * case["batch"]
        lens[0] = case["len_hi"]
    return lens, new


def _dtype(case):
    return torch.float16 if case["io"] == "fp16" else torch.bfloat16


def _up(n, m):
    return (n + m - 1) // m * m


# ---- the cache's format, in elementary operations ------------------------------------------------------------------------------

def _level(code, amax):
    """The scale of a block whose largest magnitude is amax."""
    if code == "int8":
        return amax / torch.full_like(amax, 127.0)   # (by a number, torch multiplies by its reciprocal)
    m, e = torch.frexp(amax)                   # amax = m 2^e, 1/2 <= m < 1; 448 = 0.875 2^9
    return torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), e - 9 + (m > 0.875)), torch.zeros_like(amax))


def _round(code, y):
    """The nearest code to y, as the value it stands for before the scale."""
    if code == "int8":
        return y.round().clamp(-127, 127)
    return y.clamp(-448, 448).to(torch.float8_e4m3fn).to(y.dtype)


def _inverse(s):
    return torch.where(s > 0, torch.ones_like(s) / s, torch.zeros_like(s))


def _to_bytes(code, c):
    return c.to(torch.int8).view(torch.uint8) if code == "int8" else c.to(torch.float8_e4m3fn).view(torch.uint8)


def _from_bytes(code, u):
    c = u.view(torch.int8).float() if code == "int8" else u.view(torch.float8_e4m3fn).float()
    return torch.where(torch.isnan(c), torch.zeros_like(c), c)


def _cells(x):
    """V rows [.., T, D] in the cache's order: cells of 16 bytes that hold D / 16 channels of 256 / D tokens."""
    *lead, T, D = x.shape
    return x.reshape(*lead, T * D // 256, 256 // D, 16, D // 16).transpose(-3, -2).reshape(*lead, T, D)


def _rows(x):
    *lead, T, D = x.shape
    return x.reshape(*lead, T * D // 256, 16, 256 // D, D // 16).transpose(-3, -2).reshape(*lead, T, D)


def _logical(case, u, table):
    """Bytes [unit, head, tokens, ...] of a cache by sequence: [batch, head, max_len, ...]."""
    if not case["page"]:
        return u
    x = u[table.clamp(min=0).long()]           # [batch, pages, head, page, ...]
    x = x.transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], -1, *x.shape[4:])


def _physical(case, u, table, x):
    """Writes x [batch, head, max_len, ...] to the places of the cache that the table names."""
    if not case["page"]:
        u.copy_(x)
        return
    b, h, n = x.shape[0], x.shape[1], u.shape[2]
    x = x.reshape(b, h, -1, n, *x.shape[3:]).transpose(1, 2)
    at = table >= 0
    u[table[at].long()] = x[at]


def _by_token(scales):
    return scales.repeat_interleave(BLOCK, dim=-1)


# ---- inputs --------------------------------------------------------------------------------------------------------------------

def _generator(seed, *more):
    return torch.Generator("cuda").manual_seed((seed * 1000003 + sum(m * 7919 ** i for i, m in enumerate(more, 1))) % (1 << 62))


def _states(g, case, tokens, kind):
    """Keys: a scale and an offset per channel, two channels with large offsets; values: normal; both with a level per token."""
    B, H, D = case["batch"], case["kv_heads"], case["head_dim"]
    x = torch.randn((B, H, tokens, D), generator=g, device="cuda")
    if kind == "k":
        x *= torch.randn((H, 1, D), generator=g, device="cuda").mul(0.5).exp()
        off = torch.randn((H, 1, D), generator=g, device="cuda")
        off[..., 3] += 12.0
        off[..., D // 2 + 5] -= 9.0
        x += off
    else:
        x *= torch.randn((B, H, tokens, 1), generator=g, device="cuda").mul(0.3).exp()
    return x.to(_dtype(case))


def _quantised(case, x):
    """Codes (bytes) and scales of x [B, H, T, D], T a multiple of 64."""
    B, H, T, D = x.shape
    y = x.float().view(B, H, T // BLOCK, BLOCK, D)
    s = _level(case["code"], y.abs().amax(dim=(3, 4)))
    c = _round(case["code"], y * _inverse(s)[..., None, None])
    return _to_bytes(case["code"], c).view(B, H, T, D), s


def _max_len(case):
    """Capacity of a sequence's cache."""
    most = case["len_hi"] + (case["n_hi"] if case["op"] == "append" else 0)
    return _up(max(most, 1), max(BLOCK, case["page"]))


def _cache(g, case, kind, lens, table, n_pages):
    """One tensor kind's codes, scales and block table; places without a token hold random bytes."""
    B, H, D, L = case["batch"], case["kv_heads"], case["head_dim"], _max_len(case)
    codes, scales = _quantised(case, _states(g, case, L, kind))
    noise = torch.randint(0, 256, codes.shape, generator=g, device="cuda", dtype=torch.uint8)
    there = (torch.arange(L, device="cuda")[None, :] < torch.tensor(lens, device="cuda")[:, None])[:, None, :, None]
    codes = torch.where(there, codes, noise)
    if kind == "v":
        codes = _cells(codes)
    if not case["page"]:
        return dict(codes=codes, scales=scales, table=None)
    p = case["page"]
    pool = torch.randint(0, 256, (n_pages, H, p, D), generator=g, device="cuda", dtype=torch.uint8)
    levels = torch.ones((n_pages, H, p // BLOCK), device="cuda")
    _physical(case, pool, table, codes)
    _physical(dict(case), levels, table, scales)
    return dict(codes=pool, scales=levels, table=table)


def _tables(case, seed, lens, spare):
    """Random pages for every sequence (-1 where it needs none), twice for an eviction: where from and where to."""
    p, L, B = case["page"], _max_len(case), case["batch"]
    if not p:
        return None, None, 0
    r = np.random.RandomState((seed * 31 + 7) % (1 << 31))
    need = [-(-n // p) for n in lens]
    more = [-(-n // p) for n in spare]
    free = r.permutation(sum(need) + sum(more) + 3)
    out, at = [], 0
    for counts in (need, more):
        t = np.full((B, L // p), -1, np.int32)
        for b, n in enumerate(counts):
            t[b, :n] = free[at:at + n]
            at += n
        out.append(torch.from_numpy(t).cuda())
    return out[0], out[1], len(free)


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    B, Hq, H, D, L = case["batch"], case["q_heads"], case["kv_heads"], case["head_dim"], _max_len(case)
    lens, new = _lengths(case)
    g = _generator(seed, B, L)
    spare = [min(n, case["keep"]) for n in lens] if case["op"] == "evict" else [0] * B
    table, to, n_pages = _tables(case, seed, [a + b for a, b in zip(lens, new)] if case["op"] == "append" else lens, spare)
    s = dict(case=case, n_pages=n_pages, lens=_int32(lens), new=_int32(new), max_seq=max(lens),
             k=_cache(g, case, "k", lens, table, n_pages), v=_cache(g, case, "v", lens, table, n_pages))
    if case["op"] == "append":
        n = case["n_hi"]
        # as a model's projection leaves them, token by token: [B, n, H, D] seen as [B, H, n, D]
        s["k_new"], s["v_new"] = (_states(g, case, n, kind).transpose(1, 2).contiguous().transpose(1, 2) for kind in "kv")
    elif case["op"] == "attend":
        q = torch.randn((B, case["n_q"], Hq, D), generator=g, device="cuda")
        s["q"] = (q * torch.randn((B, 1, Hq, 1), generator=g, device="cuda").mul(0.3).exp()).to(_dtype(case))
        s["out"] = torch.zeros((B, case["n_q"], Hq, D), dtype=_dtype(case), device="cuda")
        s["lse"] = torch.zeros((B, case["n_q"], Hq), device="cuda")
        if case["weights"]:
            s["weights"] = torch.rand((B, H, L), generator=g, device="cuda")
            s["added"] = torch.zeros((B, H, L), device="cuda")
    else:
        # what attention adds up: few tokens hold most of it, many the same least amount; beyond a sequence's end anything
        w = torch.randn((B, H, L), generator=g, device="cuda").mul(2.0).exp()
        w = torch.where(torch.rand((B, H, L), generator=g, device="cuda") < 0.2, torch.zeros_like(w), w)
        there = torch.arange(L, device="cuda")[None, None, :] < s["lens"][:, None, None]
        s["weights"] = torch.where(there, w, torch.full_like(w, float("nan")))
        s["kept"] = torch.zeros((B, H, case["keep"]), dtype=torch.int32, device="cuda")
        s["new_lens"] = torch.zeros(B, dtype=torch.int32, device="cuda")
        s["moved"] = torch.zeros((B, H, L), device="cuda")
        if case["page"]:
            s["k_to"], s["v_to"] = (dict(s[kind], table=to) for kind in "kv")
        else:
            s["k_to"], s["v_to"] = ({"codes": torch.zeros_like(s[kind]["codes"]), "scales": torch.zeros_like(s[kind]["scales"]), "table": None}
                                    for kind in "kv")
    return s


# ---- the plain forms -----------------------------------------------------------------------------------------------------------

def _plain_append(s):
    case = s["case"]
    code, B, H, D = case["code"], case["batch"], case["kv_heads"], case["head_dim"]
    n_blocks = case["n_hi"] // BLOCK + 2
    L = _max_len(case)
    start, n = s["lens"].long(), s["new"].long()
    b0 = start // BLOCK
    blocks = b0[:, None] + torch.arange(n_blocks, device="cuda")                         # [B, n_blocks]
    t = (blocks[:, :, None] * BLOCK + torch.arange(BLOCK, device="cuda")).view(B, -1)    # tokens of those blocks
    fresh = (t >= start[:, None]) & (t < (start + n)[:, None]) & (t < L)
    old = (t < start[:, None])
    touched = fresh.view(B, n_blocks, BLOCK).any(-1)
    at = t.clamp(max=L - 1)
    for kind in "kv":
        c = s[kind]
        codes = _logical(case, c["codes"], c["table"])
        codes = codes.clone() if not case["page"] else codes
        rows = _rows(codes) if kind == "v" else codes
        scales = _logical(case, c["scales"], c["table"])
        scales = scales.clone() if not case["page"] else scales
        pick = at[:, None, :, None].expand(B, H, -1, D)
        bytes_ = rows.gather(2, pick)
        was = _from_bytes(code, bytes_) * old[:, None, :, None]
        x = s[kind + "_new"].gather(2, (t - start[:, None]).clamp(0, case["n_hi"] - 1)[:, None, :, None].expand(B, H, -1, D)).float()
        x = torch.where(fresh[:, None, :, None], x, torch.zeros_like(x))
        at_block = blocks.clamp(max=L // BLOCK - 1)[:, None, :].expand(B, H, -1)
        before = scales.gather(2, at_block) * old.view(B, 1, n_blocks, BLOCK).any(-1)
        level = torch.maximum(before, _level(code, x.view(B, H, n_blocks, BLOCK * D).abs().amax(-1)))
        ratio = torch.where(level > 0, before / level, torch.zeros_like(level))
        y = torch.where(fresh[:, None, :, None], x * _by_token(_inverse(level))[..., None], was * _by_token(ratio)[..., None])
        y = _to_bytes(code, _round(code, y))
        # (the last blocks' indices were held back to the cache's end: those are written by no one)
        put = (fresh | old) & touched.repeat_interleave(BLOCK, dim=1)
        b, tt = put.nonzero(as_tuple=True)
        rows[b, :, t[b, tt]] = y[b, :, tt]
        b, j = touched.nonzero(as_tuple=True)
        scales[b, :, blocks[b, j]] = level[b, :, j]
        _physical(case, c["codes"], c["table"], _cells(rows) if kind == "v" else rows)
        _physical(case, c["scales"], c["table"], scales)


def _values(case, c, kind):
    """The cache's values by sequence, in 32 bits: [B, H, max_len, D]."""
    rows = _logical(case, c["codes"], c["table"])
    rows = _rows(rows) if kind == "v" else rows
    return _from_bytes(case["code"], rows) * _by_token(_logical(case, c["scales"], c["table"]))[..., None]


def _plain_attend(s):
    case = s["case"]
    B, Hq, H, D, n_q = case["batch"], case["q_heads"], case["kv_heads"], case["head_dim"], case["n_q"]
    ratio, L = Hq // H, s["max_seq"]
    k, v = (_values(case, s[kind], kind)[:, :, :L].contiguous() for kind in "kv")
    t = torch.arange(L, device="cuda")
    there = t[None, :] < s["lens"][:, None]                                               # [B, L]
    v = torch.where(there[:, None, :, None], v, torch.zeros_like(v))
    q = s["q"].float().view(B, n_q, H, ratio, D).permute(0, 2, 1, 3, 4).reshape(B, H, n_q * ratio, D)
    p = torch.matmul(q, k.transpose(2, 3).contiguous())
    p *= 1.0 / math.sqrt(D)
    i = torch.arange(n_q, device="cuda")
    asked = i[None, :] < s["new"][:, None]                                                # [B, n_q]
    seen = there[:, None, :] & asked[:, :, None]
    if case["causal"]:
        seen = seen & (t[None, None, :] <= (s["lens"] - s["new"])[:, None, None] + i[None, :, None])
    seen = seen.repeat_interleave(ratio, dim=1)[:, None]                                  # [B, 1, rows, L]
    p.masked_fill_(~seen, -math.inf)
    m = p.amax(-1, keepdim=True)
    m = torch.where(m > -math.inf, m, torch.zeros_like(m))
    p -= m
    p.exp_()
    total = p.sum(-1, keepdim=True)
    lse = torch.where(total > 0, m + total.log(), torch.full_like(m, -math.inf)).squeeze(-1)
    p /= torch.where(total > 0, total, torch.ones_like(total))
    o = torch.matmul(p, v).view(B, H, n_q, ratio, D).permute(0, 2, 1, 3, 4).reshape(B, n_q, Hq, D)
    lse = lse.view(B, H, n_q, ratio).permute(0, 2, 1, 3).reshape(B, n_q, Hq)
    out = {"out": torch.where(asked[:, :, None, None], o.to(s["out"].dtype), s["out"]), "lse": torch.where(asked[:, :, None], lse, s["lse"])}
    if case["weights"]:
        out["weights"] = s["added"].clone()
        out["weights"][:, :, :L] = torch.where(there[:, None], s["weights"][:, :, :L] + p.sum(2), s["added"][:, :, :L])
    return out


def _plain_evict(s):
    case = s["case"]
    B, H, D, keep, L = case["batch"], case["kv_heads"], case["head_dim"], case["keep"], s["max_seq"]
    t, lens = torch.arange(L, device="cuda"), s["lens"].long()
    there = (t[None, :] < lens[:, None])[:, None].expand(B, H, L)
    sure = ((t < case["first"])[None, :] | (t[None, :] >= (lens - case["recent"])[:, None]))[:, None].expand(B, H, L)
    w = s["weights"][:, :, :L]
    w = torch.where(sure, torch.full_like(w, math.inf), w)
    w = torch.where(there, w, torch.full_like(w, -math.inf))
    order = w.sort(dim=-1, descending=True, stable=True).indices[..., :min(keep, L)]
    new_lens = lens.clamp(max=keep)
    live = (torch.arange(order.shape[-1], device="cuda")[None, :] < new_lens[:, None])[:, None]
    order = torch.where(live, order, torch.full_like(order, L)).sort(dim=-1).values
    s["kept"].fill_(-1)
    s["kept"][..., :order.shape[-1]] = torch.where(live, order, torch.full_like(order, -1)).int()
    s["new_lens"].copy_(new_lens)
    order = order.clamp(max=L - 1)
    n = order.shape[-1]
    s["moved"][:, :, :L] = 0
    s["moved"][:, :, :n] = torch.where(live, s["weights"].gather(2, order), torch.zeros((), device="cuda"))
    pad = _up(n, BLOCK)
    for kind in "kv":
        c, d = s[kind], s[kind + "_to"]
        rows, to = _logical(case, c["codes"], c["table"]), _logical(case, d["codes"], d["table"])
        to = to.clone() if not case["page"] else to
        if kind == "v":
            rows, to = _rows(rows), _rows(to).contiguous()
        scale = _by_token(_logical(case, c["scales"], c["table"])).gather(2, order) * live
        scale = torch.nn.functional.pad(scale, (0, pad - n)).view(B, H, pad // BLOCK, BLOCK)
        level = scale.amax(-1)
        ratio = torch.where(level[..., None] > 0, scale / level[..., None], torch.zeros_like(scale)).view(B, H, pad)[..., :n]
        x = _from_bytes(case["code"], rows.gather(2, order[..., None].expand(-1, -1, -1, D)))
        y = _to_bytes(case["code"], _round(case["code"], x * ratio[..., None]))
        to[:, :, :n] = torch.where(live[..., None], y, to[:, :, :n])
        levels = _logical(case, d["scales"], d["table"])
        levels = levels.clone() if not case["page"] else levels
        used = (torch.arange(pad // BLOCK, device="cuda")[None, :] * BLOCK < new_lens[:, None])[:, None]
        levels[:, :, :pad // BLOCK] = torch.where(used, level, levels[:, :, :pad // BLOCK])
        _physical(case, d["codes"], d["table"], _cells(to) if kind == "v" else to)
        _physical(case, d["scales"], d["table"], levels)


# ---- a user's calls ------------------------------------------------------------------------------------------------------------

_scratch = {}


def _workspace(api, shape, op, batch, n, max_seq):
    """One workspace for every call of an operator, as a program with many layers keeps it (zero-filled when it is made)."""
    need = api.nsn_q8_workspace_bytes(shape, op, batch, n, max_seq)
    if op not in _scratch or _scratch[op].numel() < need:
        _scratch[op] = torch.zeros(max(need, 256), dtype=torch.uint8, device="cuda")
    return _scratch[op]


def _handles(api, s):
    if "shape" not in s:
        case = s["case"]
        s["shape"] = api.make_q8_shape(case["head_dim"], case["q_heads"], case["kv_heads"], _max_len(case), case["page"], s["n_pages"],
                                       api.NSN_Q8_INT8 if case["code"] == "int8" else api.NSN_Q8_E4M3, _dtype(case))
        for kind in ("k", "v", "k_to", "v_to"):
            if kind in s:
                s[kind + "_cache"] = api.Q8Cache(s[kind]["codes"], s[kind]["scales"], s[kind]["table"])
    return s["shape"], s["k_cache"], s["v_cache"]


def _own(s):
    from paper_2505_18231_amd import api
    case = s["case"]
    shape, kc, vc = _handles(api, s)
    if case["op"] == "append":
        api.nsn_q8_append(shape, s["k_new"], s["v_new"], s["lens"], s["new"], kc, vc)
        return None
    if case["op"] == "attend":
        ws = _workspace(api, shape, api.NSN_OP_Q8_ATTENTION, case["batch"], case["n_q"], s["max_seq"])
        api.nsn_q8_attention(shape, s["q"], kc, vc, s["lens"], s["max_seq"], 1.0 / math.sqrt(case["head_dim"]), causal=case["causal"],
                             q_lens=s["new"] if case["q_ragged"] else None, weights_in=s.get("weights"), weights_out=s.get("added"),
                             out=s["out"], lse=s["lse"], workspace=ws)
        out = {"out": s["out"], "lse": s["lse"]}
        return dict(out, weights=s["added"]) if case["weights"] else out
    ws = _workspace(api, shape, api.NSN_OP_Q8_EVICT, case["batch"], case["keep"], s["max_seq"])
    api.nsn_q8_evict(shape, s["weights"], s["lens"], s["max_seq"], case["keep"], kc, vc, s["k_to_cache"], s["v_to_cache"], first=case["first"],
                     recent=case["recent"], kept=s["kept"], new_lens=s["new_lens"], weights_out=s["moved"], workspace=ws)
    return None


def _codes(case, c):
    """A cache's codes as the values they stand for, before the scale."""
    return c["codes"].view(torch.int8 if case["code"] == "int8" else torch.float8_e4m3fn)


def _cache_out(case, s, names):
    return {n: {"codes": _codes(case, s[n]), "scales": s[n]["scales"]} for n in names}


def run(s):
    case = s["case"]
    if own:
        out = _own(s)
    else:
        out = {"append": _plain_append, "attend": _plain_attend, "evict": _plain_evict}[case["op"]](s)
    if case["op"] == "append":
        return _cache_out(case, s, ("k", "v"))
    if case["op"] == "evict":
        return {"kept": s["kept"], "new_lens": s["new_lens"], "weights": s["moved"], **_cache_out(case, s, ("k_to", "v_to"))}
    return out


def work(case):
    lens, new = _lengths(case)
    B, Hq, H, D = case["batch"], case["q_heads"], case["kv_heads"], case["head_dim"]
    if case["op"] == "append":
        n, blocks = sum(new), sum(-(-(a + c) // BLOCK) - a // BLOCK for a, c in zip(lens, new))
        return {"bytes": 2 * H * (3 * D * n + 4 * blocks) + 8 * B, "flops": 2 * 2 * H * D * n}
    if case["op"] == "attend":
        t = sum(lens)
        if case["causal"]:
            pairs = sum(sum(max(0, n - m + i + 1) for i in range(m)) for n, m in zip(lens, new))
        else:
            pairs = sum(n * m for n, m in zip(lens, new))
        moved = H * t * (2 * D + 8.0 / BLOCK) + Hq * sum(new) * (4 * D + 4)
        return {"bytes": moved + (8 * H * t if case["weights"] else 0), "flops": 4 * D * Hq * pairs}
    kept = sum(min(n, case["keep"]) for n in lens)
    return {"bytes": H * (4 * sum(lens) + 4 * B * max(lens) + 4 * B * case["keep"] + kept * (4 * D + 16.0 / BLOCK)), "flops": 2 * 2 * H * D * kept}


# ---- from the definitions, in 64 bits ------------------------------------------------------------------------------------------

def _exact_codes(case, rows, kind):
    """Bytes [T, D] of one head of a unit as numbers, written from the format: sign, exponent and fraction of e4m3; the order of V's cells."""
    T, D = rows.shape
    if kind == "v":
        t, c = torch.arange(T, device="cuda")[:, None], torch.arange(D, device="cuda")[None, :]
        n, m = 256 // D, D // 16
        rows = rows.reshape(-1)[t // n * 256 + c // m * 16 + t % n * m + c % m]
    u = rows.long()
    if case["code"] == "int8":
        return (u - 256 * (u >= 128)).double()
    e, f = (u >> 3) & 15, (u & 7).double()
    x = torch.where(e > 0, (8 + f) * torch.exp2((e - 10).double()), f * 2.0 ** -9)
    return torch.where(u >= 128, -x, x)


def _exact_unit(case, c, b, h, n, kind):
    """Values [n, D] of sequence b, head h."""
    if case["page"]:
        pages = c["table"][b, :-(-n // case["page"])].long()
        x = torch.cat([_exact_codes(case, c["codes"][p, h], kind) for p in pages])
        s = torch.cat([c["scales"][p, h] for p in pages])
    else:
        x, s = _exact_codes(case, c["codes"][b, h], kind), c["scales"][b, h]
    return (x * s.double().repeat_interleave(BLOCK)[:, None])[:n]


def _exact_scales(case, c, b, h):
    if case["page"]:
        return torch.cat([c["scales"][p, h] for p in c["table"][b].clamp(min=0).long()]).double()
    return c["scales"][b, h].double()


def _exact_empty(case, c):
    """What lies in a cache before the call: codes where they are floating values (None for whole ones), scales."""
    return (_codes(case, c).double() if case["code"] == "e4m3" else None), c["scales"].double()


def _exact_put(case, codes, scales, table, b, h, first, rows, level, kind):
    """Rows [n, D] from block `first` on, and those blocks' scales, into the places of sequence b, head h."""
    n, D = rows.shape
    t = torch.arange(first * BLOCK, first * BLOCK + n, device="cuda")
    blocks = torch.arange(first, first + level.shape[0], device="cuda")
    unit, tu, bu, ub = b, t, blocks, b
    if case["page"]:
        unit, tu = table[b].long()[t // case["page"]], t % case["page"]
        ub, bu = table[b].long()[blocks * BLOCK // case["page"]], blocks % (case["page"] // BLOCK)
    scales[ub, h, bu] = level
    if codes is None:
        return
    c = torch.arange(D, device="cuda")[None, :]
    at = tu[:, None] * D + c
    if kind == "v":
        m, k = 256 // D, D // 16
        at = tu[:, None] // m * 256 + c // k * 16 + tu[:, None] % m * k + c % k
    flat = codes.view(codes.shape[0], codes.shape[1], -1)
    flat[unit if isinstance(unit, int) else unit[:, None], h, at] = rows


def _exact_level(case, amax):
    if case["code"] == "int8":
        return amax / 127
    return torch.where(amax > 0, torch.exp2(torch.ceil(torch.log2(amax / 448))), torch.zeros_like(amax))


def _exact_round(case, y):
    if case["code"] == "int8":
        return y.round().clamp(-127, 127)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return ((y / step).round() * step).clamp(-448, 448)


def exact(case, seed):
    s = prepare(case, seed)
    lens, new = _lengths(case)
    B, Hq, H, D = case["batch"], case["q_heads"], case["kv_heads"], case["head_dim"]
    if case["op"] == "attend":
        ratio = Hq // H
        out, lse = s["out"].double(), s["lse"].double()
        weights = s["added"].double() if case["weights"] else None
        for b in range(B):
            n, m = lens[b], new[b]
            for h in range(H):
                k, v = _exact_unit(case, s["k"], b, h, n, "k"), _exact_unit(case, s["v"], b, h, n, "v")
                for g in range(ratio):
                    x = s["q"][b, :m, h * ratio + g].double() @ k.T / math.sqrt(D)
                    if case["causal"]:
                        x = x.masked_fill(torch.arange(n, device="cuda")[None, :] > n - m + torch.arange(m, device="cuda")[:, None], -math.inf)
                    z = torch.logsumexp(x, dim=1)
                    p = torch.exp(x - torch.where(z > -math.inf, z, torch.zeros_like(z))[:, None])
                    out[b, :m, h * ratio + g], lse[b, :m, h * ratio + g] = p @ v, z
                    if weights is not None:
                        weights[b, h, :n] = p.sum(0) + (weights[b, h, :n] if g else s["weights"][b, h, :n].double())
        got = {"out": out, "lse": lse}
        return dict(got, weights=weights) if case["weights"] else got
    got = {}
    if case["op"] == "append":
        for kind in "kv":
            codes, scales = _exact_empty(case, s[kind])
            for b in range(B):
                a, m = lens[b], min(new[b], _max_len(case) - lens[b])
                first, last = a // BLOCK, -(-(a + m) // BLOCK)
                for h in range(H):
                    old, was = _exact_unit(case, s[kind], b, h, a, kind)[first * BLOCK:], _exact_scales(case, s[kind], b, h)
                    x = torch.cat([old, s[kind + "_new"][b, h, :m].double()])
                    wide = torch.nn.functional.pad(x, (0, 0, 0, (last - first) * BLOCK - x.shape[0])).view(last - first, -1)
                    fresh = torch.where(torch.arange(wide.numel(), device="cuda").view(wide.shape) < old.numel(), torch.zeros_like(wide), wide)
                    level = _exact_level(case, fresh.abs().amax(1))
                    if old.numel():
                        level[0] = torch.maximum(level[0], was[first])
                    y = wide / torch.where(level > 0, level, torch.ones_like(level))[:, None]
                    _exact_put(case, codes, scales, s[kind]["table"], b, h, first, _exact_round(case, y).view(-1, D)[:x.shape[0]], level, kind)
            got[kind] = {"codes": codes, "scales": scales}
        return got
    order = []
    for b in range(B):
        w, n = s["weights"][b, :, :lens[b]].double().cpu().numpy(), lens[b]
        sure = [t < case["first"] or t >= n - case["recent"] for t in range(n)]
        order.append([np.sort(np.lexsort((np.arange(n), np.where(sure, -np.inf, -w[h])))[:case["keep"]]) for h in range(H)])
    got = {"kept": s["kept"], "new_lens": s["new_lens"], "weights": s["moved"].double()}
    got["kept"].fill_(-1)
    got["weights"][:, :, :s["max_seq"]] = 0
    for b in range(B):
        got["new_lens"][b] = len(order[b][0])
        for h in range(H):
            got["kept"][b, h, :len(order[b][h])] = torch.from_numpy(order[b][h]).int()
            got["weights"][b, h, :len(order[b][h])] = s["weights"][b, h, torch.from_numpy(order[b][h]).cuda()].double()
    for kind in "kv":
        codes, scales = _exact_empty(case, s[kind + "_to"])
        for b in range(B):
            for h in range(H):
                at = torch.from_numpy(order[b][h]).cuda()
                x, n = _exact_unit(case, s[kind], b, h, lens[b], kind)[at], len(at)
                sc = torch.nn.functional.pad(_exact_scales(case, s[kind], b, h)[at // BLOCK], (0, _up(n, BLOCK) - n))
                level = sc.view(-1, BLOCK).amax(1)
                y = x / torch.where(level > 0, level, torch.ones_like(level)).repeat_interleave(BLOCK)[:n, None]
                _exact_put(case, codes, scales, s[kind + "_to"]["table"], b, h, 0, _exact_round(case, y), level, kind)
        got[kind + "_to"] = {"codes": codes, "scales": scales}
    return got
