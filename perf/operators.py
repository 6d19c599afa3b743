"""The operators of the KV cache held in 8 bits, as a user of the package calls them, beside their plain forms.

  append    mc_kv8_append: new K/V of a ragged batch, rounded to e4m3 codes with one power-of-two
            scale per block (16 tokens of K or of V of one kv head of one layer).
  attend    mc_attn8_plan once, then for every layer mc_prefix_prefill_attn8: attention of the new
            tokens over the 8-bit cache, with grouped heads, output and log-sum-exp.
  step      both, as a decode step or a prefill of an engine runs them: plan once, then for every
            layer the append and the attention that reads it.
  compress, restore
            mc_kv8_compress_range, mc_kv8_restore_range: a token range of every layer, from the
            pages of a 16-bit pool to those of an 8-bit one and back.
  pack, unpack
            mc_kv8_pack_range, mc_kv8_unpack_range: the pages of a range, codes and scales, to one
            contiguous buffer and back: what one engine sends another.

Layout: codes [layer][page][2: K, V][kv_head][2048 bytes], a K block [slot][128], a V block [128][slot];
scales [layer][page][kv_head][2: K, V] float32.  A block's scale is 2^k with the least k for which its
largest finite magnitude is at most 448 * 2^k, within [-15, 8] (fp16 tokens) or [-100, 120] (bf16).

A case holds sizes only; token counts are drawn from them by the case's own "lens" number, the values
and the page placement by the seed handed to prepare().
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
P, D = 16, 128                     # page size (tokens), head dim: the cache's only ones
LIMITS = {"fp16": (-15, 8), "bf16": (-100, 120)}
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}

_BATCH = dict(dtype="bf16", hq=32, hkv=8, layers=1, lens=0, decodes=0, ctx_lo=0, ctx_hi=0,
              prefills=0, n_lo=0, n_hi=0, cached_lo=0.0, cached_hi=0.0)
_RANGE = dict(dtype="bf16", hkv=8, layers=1, n=0, begin=0)


def listed():
    return [
        # a decode step of a small batch over four layers: all latency
        dict(_BATCH, kind="step", name="step-decode-8", layers=4, decodes=8, ctx_lo=1024, ctx_hi=4096, lens=1),
        # the new K/V of a full decode batch: one token into each of 256 partly filled pages
        dict(_BATCH, kind="append", name="append-decode-256", decodes=256, ctx_lo=1024, ctx_hi=4096, lens=2),
        # the new K/V of a prefill batch: ragged ranges that begin and end inside pages
        dict(_BATCH, kind="append", name="append-prompts-8", prefills=8, n_lo=1024, n_hi=4096, cached_hi=0.5, lens=3),
        # a full decode batch: every sequence's codes are read once
        dict(_BATCH, kind="attend", name="attend-decode-256", decodes=256, ctx_lo=1024, ctx_hi=4096, lens=4),
        # 500 new tokens over 4500 cached ones
        dict(_BATCH, kind="attend", name="attend-500-over-4500", prefills=1, n_lo=5000, n_hi=5000, cached_lo=0.9,
             cached_hi=0.9, lens=5),
        # the ordinary prefill batch: 8 prompts of 1024..4096 tokens, up to 75 % cached
        dict(_BATCH, kind="attend", name="attend-prompts-8", prefills=8, n_lo=1024, n_hi=4096, cached_hi=0.75, lens=6),
        # long context: 16384 new tokens over 16384 cached ones
        dict(_BATCH, kind="attend", name="attend-32k", prefills=1, n_lo=32768, n_hi=32768, cached_lo=0.5,
             cached_hi=0.5, lens=7),
        # decode steps fused with the rest of a prompt: fp16, 64 query heads
        dict(_BATCH, kind="attend", name="attend-mixed-fp16", dtype="fp16", hq=64, decodes=24, ctx_lo=700, ctx_hi=2500,
             prefills=1, n_lo=1777, n_hi=1777, cached_lo=0.4, cached_hi=0.4, lens=8),
        # a cached prompt leaves the 16-bit pool for the 8-bit one, all layers
        dict(_RANGE, kind="compress", name="compress-4k", layers=32, n=4096),
        # ... and an odd part of one comes back, in fp16
        dict(_RANGE, kind="restore", name="restore-odd-fp16", dtype="fp16", layers=32, n=1999, begin=37),
        # a whole 32768-token sequence leaves for another engine
        dict(_RANGE, kind="pack", name="pack-32k", layers=32, n=32768),
        # four layers of a prompt arrive, behind a prefix that was there
        dict(_RANGE, kind="unpack", name="unpack-2500", layers=4, n=2500, begin=512),
    ]


# ---------------------------------------------------------------- sizes ------
def _logint(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    """One more case: 1..256 decode rows over 100..8192 tokens, 1..8 prefills of up to 8192 tokens (one of
    up to 32768), mixtures, ranges of 16..32768 tokens in 1..32 layers; the heads of an 8-billion and of a
    70-billion-parameter model, whole or as one of several GPUs holds them, and as many q as kv heads."""
    while True:
        kind = rng.choice(("append", "append", "attend", "attend", "attend", "step", "compress", "restore", "pack", "unpack"))
        dtype = rng.choice(("bf16", "bf16", "fp16"))
        if kind in ("append", "attend", "step"):
            c = dict(_BATCH, kind=kind, dtype=dtype, lens=rng.randrange(1 << 20), layers=rng.randint(1, 4))
            c["hq"], c["hkv"] = rng.choice(((32, 8), (32, 8), (64, 8), (8, 8), (16, 8), (8, 2), (8, 1), (16, 4)))
            form = rng.choice(("decode", "prefill", "mixed"))
            if form != "prefill":
                c["ctx_hi"] = _logint(rng, 128, 8192)
                c["ctx_lo"] = _logint(rng, 100, c["ctx_hi"])
                c["decodes"] = _logint(rng, 1, 256 if form == "decode" else 64)
            if form != "decode":
                c["n_hi"] = _logint(rng, 17, 32768 if form == "prefill" else 2048)
                c["n_lo"] = rng.randint(max(1, c["n_hi"] // 4), c["n_hi"])
                c["prefills"] = _logint(rng, 1, 8) if c["n_hi"] <= 8192 else 1
                c["cached_lo"] = rng.uniform(0.0, 0.9)
                c["cached_hi"] = rng.uniform(c["cached_lo"], 0.95)
        else:
            c = dict(_RANGE, kind=kind, dtype=dtype, layers=_logint(rng, 1, 32), n=_logint(rng, 16, 32768),
                     hkv=rng.choice((1, 2, 4, 8, 8)))
            c["begin"] = rng.randrange(c["n"])
            if kind != "restore":
                c["begin"] = c["begin"] // P * P
        w = work(c)
        # no dearer than the listed ones, and small enough to be held three times beside the plain form's scores
        if w["flops"] <= 6e12 and w["bytes"] <= 4e9 and _room(c) <= 1:
            return c


def _room(c):
    """What the plain form keeps of scores at a time, as a part of what it may."""
    if "hq" not in c:
        return 0
    begin, new = _lengths(c)
    return len(new) * (c["hq"] // c["hkv"]) * int(new.max()) * int((begin + new).max()) / 2.4e9


def _lengths(c):
    """(tokens cached, new tokens) of every sequence of a case."""
    r, begin, new = random.Random(c["lens"]), [], []
    for _ in range(c["decodes"]):
        begin.append(r.randint(c["ctx_lo"], c["ctx_hi"]) - 1)
        new.append(1)
    for _ in range(c["prefills"]):
        n = r.randint(c["n_lo"], c["n_hi"])
        begin.append(min(n - 1, round(n * r.uniform(c["cached_lo"], c["cached_hi"]))))
        new.append(n - begin[-1])
    return np.array(begin, dtype=np.int64), np.array(new, dtype=np.int64)


def work(c):
    if "hq" in c:
        begin, new = _lengths(c)
        tq, total, last = int(new.sum()), int((begin + new).sum()), int((-(-(begin + new) // P)).sum())
        first = int((begin // P).sum())
        append = tq * c["hkv"] * D * 2 * (2 + 1) + (last - first) * c["hkv"] * 2 * 4
        attend = tq * c["hq"] * (D * 2 * 2 + 4) + total * c["hkv"] * D * 2 + last * c["hkv"] * 2 * 4
        flops = 4 * D * c["hq"] * int((new * begin + new * (new + 1) // 2).sum())
        return {"bytes": c["layers"] * ((append if c["kind"] != "attend" else 0) + (attend if c["kind"] != "append" else 0)),
                "flops": c["layers"] * flops if c["kind"] != "append" else 0}
    tokens, pages = c["n"] - c["begin"], -(-c["n"] // P) - c["begin"] // P
    scales = pages * 2 * 4
    if c["kind"] in ("compress", "restore"):
        return {"bytes": c["layers"] * c["hkv"] * (tokens * 2 * D * (2 + 1) + scales), "flops": 0}
    return {"bytes": c["layers"] * c["hkv"] * 2 * (pages * 2 * D * P + scales), "flops": 0}


# -------------------------------------------------------------- prepare ------
def _up(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).to(DEV)


def _pool8(g, layers, pages, hkv, dtype):
    """An 8-bit pool in use: blocks of N(0, s) tokens, s around 1 for K and from 1/8 to 8 for V; every slot
    holds something."""
    codes = torch.empty((layers, pages, 2, hkv, P * D), dtype=torch.uint8, device=DEV)
    scales = torch.empty((layers, pages, hkv, 2), dtype=torch.float32, device=DEV)
    some = max(1, (1 << 26) // (2 * hkv * P * D))             # pages at a time
    for i in range(layers):
        for p in range(0, pages, some):
            n = min(some, pages - p)
            x = torch.randn((n, 2, hkv, P * D), generator=g, device=DEV)
            power = torch.randint(-3, 4, (n, hkv, 2), generator=g, device=DEV)
            power[..., 0].clamp_(-1, 1)
            big = x.abs().amax(3).permute(0, 2, 1)
            k = torch.ceil(torch.log2(big / 448))
            codes[i, p:p + n] = (x / torch.exp2(k).permute(0, 2, 1)[..., None]).clamp(-448, 448).to(
                torch.float8_e4m3fn).view(torch.uint8)
            scales[i, p:p + n] = torch.exp2((k + power).clamp(*LIMITS[dtype]))
    return codes, scales


def prepare(c, seed):
    rng, g = np.random.default_rng(seed), torch.Generator(DEV).manual_seed(seed)
    return _prepare_batch(c, rng, g) if "hq" in c else _prepare_range(c, rng, g)


def _prepare_batch(c, rng, g):
    begin, new = _lengths(c)
    L, hq, hkv, tq = c["layers"], c["hq"], c["hkv"], int(new.sum())
    need = -(-(begin + new) // P)
    pages = int(need.sum()) + 8
    s = dict(c, B=len(new), tq=tq, pages=pages, q_most=int(new.max()), n_most=int((begin + new).max()))
    s["codes"], s["scales"] = _pool8(g, L, pages, hkv, c["dtype"])
    randn = lambda h: torch.randn((L, tq, h, D), generator=g, dtype=TYPES[c["dtype"]], device=DEV)  # noqa: E731
    s["q"], s["k"], s["v"] = randn(hq), randn(hkv), randn(hkv)
    s["out"] = torch.zeros((L, tq, hq, D), dtype=TYPES[c["dtype"]], device=DEV)
    s["lse"] = torch.zeros((L, tq, hq), dtype=torch.float32, device=DEV)
    s["cu_q"], s["begin"] = _up(np.concatenate([[0], np.cumsum(new)])), _up(begin)
    s["table"] = _up(rng.permutation(pages)[:int(need.sum())])           # pages scattered over the pool
    s["cu_pages"] = _up(np.concatenate([[0], np.cumsum(need)]))
    return s


def _prepare_range(c, rng, g):
    L, hkv, n = c["layers"], c["hkv"], -(-c["n"] // P)
    pages = n + 5
    s = dict(c, pages=pages, entries=n)
    s["codes"], s["scales"] = _pool8(g, L, pages, hkv, c["dtype"])
    s["pages8"] = _up(rng.permutation(pages)[:n])
    if c["kind"] in ("compress", "restore"):
        s["pool"] = torch.randn((L, pages, 2, hkv, P, D), generator=g, dtype=TYPES[c["dtype"]], device=DEV)
        s["pages16"] = _up(rng.permutation(pages)[:n])
    else:
        moved = L * (n - c["begin"] // P) * hkv
        s["codes_bytes"] = moved * 2 * P * D
        s["buf"] = torch.zeros(moved * (2 * P * D + 8), dtype=torch.uint8, device=DEV)
        if c["kind"] == "unpack":
            s["buf"][:s["codes_bytes"]] = s["codes"].view(-1)[-s["codes_bytes"]:]
            s["buf"][s["codes_bytes"]:] = s["scales"].view(torch.uint8).view(-1)[-8 * moved:]
    return s


# ------------------------------------------------------------------ run ------
def run(s):
    return _run_own(s) if own else _PLAIN[s["kind"]](s)


def _state8(s):
    """The 8-bit pool: the codes as the e4m3 numbers they are, and the scales."""
    return [s["codes"].view(torch.float8_e4m3fn), s["scales"]]


def _run_own(s):
    import paper_2412_12488_amd as mc
    if "pool8" not in s:               # descriptors and workspace of the pool's owner, made once
        code = mc.MC_BF16 if s["dtype"] == "bf16" else mc.MC_F16
        s["pool8"] = mc.pool8_desc(s["codes"], s["scales"], s["layers"], s["pages"], s["hkv"], code)
        if "pool" in s:
            s["pool16"] = mc.pool_desc(s["pool"], s["layers"], s["pages"], s["hkv"], code)
        if s["kind"] in ("attend", "step"):
            s["ws_bytes"] = mc.mc_attn8_workspace_size(s["B"], s["tq"], s["hq"], s["hkv"])
            s["ws"] = torch.empty(s["ws_bytes"], dtype=torch.uint8, device=DEV)
        if "q" in s:
            s["of_layer"] = [[s[x][i] for x in ("k", "v", "q", "out", "lse")] for i in range(s["layers"])]
    pool, L, kind = s["pool8"], s["layers"], s["kind"]
    if "q" in s:
        batch = (s["B"], s["tq"], s["cu_q"], s["begin"], s["table"], s["cu_pages"])
        if kind != "append":
            mc.mc_attn8_plan(pool, s["hq"], *batch, s["ws"], s["ws_bytes"])
        for i, (k, v, q, out, lse) in enumerate(s["of_layer"]):
            if kind != "attend":
                mc.mc_kv8_append(pool, i, k, v, *batch)
            if kind != "append":
                mc.mc_prefix_prefill_attn8(pool, i, q, s["hq"], *batch, 0.0, out, lse, s["ws"], s["ws_bytes"])
        return ([s["out"], s["lse"]] if kind != "append" else []) + (_state8(s) if kind != "attend" else [])
    n, s0, s1 = s["entries"], s["begin"], s["n"]
    if kind == "compress":
        mc.mc_kv8_compress_range(s["pool16"], pool, 0, L, s["pages16"], n, s["pages8"], n, s0, s1)
        return _state8(s)
    if kind == "restore":
        mc.mc_kv8_restore_range(pool, s["pool16"], 0, L, s["pages8"], n, s["pages16"], n, s0, s1)
        return [s["pool"]]
    if kind == "pack":
        mc.mc_kv8_pack_range(pool, 0, L, s["pages8"], n, s0, s1, s["buf"])
        return _buffer(s)
    mc.mc_kv8_unpack_range(pool, 0, L, s["pages8"], n, s0, s1, s["buf"])
    return _state8(s)


def _buffer(s):
    return [s["buf"][:s["codes_bytes"]].view(torch.float8_e4m3fn), s["buf"][s["codes_bytes"]:].view(torch.float32)]


# ---- the plain forms ----
def _power(x):
    """2^x of whole x, exactly."""
    return ((x + 127) << 23).view(torch.float32)


def _exponent(big, dtype):
    """The exponent of a block's scale from its largest finite magnitude."""
    m, e = torch.frexp(big)
    k = e - 9 + (m > 0.875)
    lo, hi = LIMITS[dtype]
    return torch.where(big > 0, k, lo).clamp(lo, hi).int()


def _codes(x, k, dtype):
    """e4m3 codes of x with scales 2^k: round to nearest even, at most the type's largest value, NaN for what is no number."""
    most = torch.where(k == LIMITS[dtype][1], 240.0, 448.0)
    y = torch.minimum(torch.maximum(x / _power(k), -most), most)
    return torch.where(torch.isfinite(x), y, math.nan).to(torch.float8_e4m3fn).view(torch.uint8)


def _magnitude(x):
    return torch.where(torch.isfinite(x), x.abs(), 0.0)


def _values(codes):
    return codes.view(torch.float8_e4m3fn).float()


def _plain_append(s, layer):
    begin, cu_q, dtype, hkv = s["begin"].long(), s["cu_q"].long(), s["dtype"], s["hkv"]
    token = torch.arange(s["tq"], device=DEV)
    seq = torch.searchsorted(cu_q, token, right=True) - 1
    pos = begin[seq] + token - cu_q[seq]
    page = s["table"].long()[s["cu_pages"].long()[seq] + pos // P]
    touched, at = torch.unique(page, return_inverse=True)
    n = len(touched)
    # slots below the first new one of a page held tokens before
    first = torch.full((n,), P, device=DEV).scatter_reduce(0, at, pos % P, "amin")
    x = torch.stack([s["k"][layer], s["v"][layer]], 1).float()                      # [token][K, V][head][D]
    big = torch.zeros((n, 2, hkv), device=DEV).scatter_reduce(
        0, at[:, None, None].expand(-1, 2, hkv), _magnitude(x).amax(3), "amax")
    k = _exponent(big, dtype)
    old_scale = s["scales"][layer][touched].permute(0, 2, 1)                        # [page][K, V][head]
    old_k = (old_scale.contiguous().view(torch.int32) >> 23) - 127
    k = torch.where(first[:, None, None] > 0, torch.maximum(k, old_k), k)
    # every block as [slot][D]
    old = s["codes"][layer][touched]
    old = torch.stack([old[:, 0].view(n, hkv, P, D), old[:, 1].view(n, hkv, D, P).transpose(2, 3)], 1)
    slot = torch.arange(P, device=DEV)
    kept = (slot < first[:, None])[:, None, None, :, None] & (k > old_k)[..., None, None]
    moved = _values(old) * _power((old_k - k).clamp(min=-120))[..., None, None]
    new = torch.where(kept, moved.to(torch.float8_e4m3fn).view(torch.uint8), old)
    new[at, :, :, pos % P] = _codes(x, k[at][..., None], dtype)
    s["codes"][layer][touched] = torch.stack(
        [new[:, 0].reshape(n, hkv, P * D), new[:, 1].transpose(2, 3).reshape(n, hkv, P * D)], 1)
    s["scales"][layer][touched] = _power(k).permute(0, 2, 1)


def _plain_attend(s, layer):
    B, hq, hkv, G, pages = s["B"], s["hq"], s["hkv"], s["hq"] // s["hkv"], -(-s["n_most"] // P)
    begin, cu_q, cu_pages, Q = s["begin"].long(), s["cu_q"].long(), s["cu_pages"].long(), s["q_most"]
    entry = cu_pages[:-1, None] + torch.arange(pages, device=DEV)
    page = s["table"].long()[torch.minimum(entry, cu_pages[1:, None] - 1)]
    row = torch.arange(Q, device=DEV)
    live = row < (cu_q[1:] - cu_q[:-1])[:, None]
    at = torch.minimum(cu_q[:-1, None] + row, cu_q[1:, None] - 1)
    pos = begin[:, None] + row
    key = torch.arange(pages * P, device=DEV)
    hidden = key > pos[..., None]                                                   # [B][row][key]
    stale = (key >= (begin + cu_q[1:] - cu_q[:-1])[:, None])[:, None, :, None]
    some = max(1, min(hkv, int(2.5e9 / (B * G * Q * pages * P)), int(1e9 / (B * pages * P * D))))
    for h in range(0, hkv, some):
        e = min(hkv, h + some)
        c, scale = s["codes"][layer][page, :, h:e], s["scales"][layer][page, h:e]
        k = _values(c[:, :, 0]).view(B, pages, e - h, P, D) * scale[..., 0, None, None]
        k = k.transpose(1, 2).reshape(B, e - h, pages * P, D)
        v = _values(c[:, :, 1]).view(B, pages, e - h, D, P) * scale[..., 1, None, None]
        v = v.permute(0, 2, 1, 4, 3).reshape(B, e - h, pages * P, D).masked_fill_(stale, 0.0)
        q = s["q"][layer][at, h * G:e * G].float().view(B, Q, e - h, G, D)
        q = q.permute(0, 2, 1, 3, 4).reshape(B, e - h, Q * G, D)
        score = torch.matmul(q, k.transpose(2, 3).contiguous()).view(B, e - h, Q, G, pages * P)
        score.mul_(D ** -0.5).masked_fill_(hidden[:, None, :, None], -math.inf)
        top = score.amax(4, keepdim=True)
        total = score.sub_(top).exp_().sum(4, keepdim=True)
        o = torch.matmul(score.view(B, e - h, Q * G, pages * P), v).view(B, e - h, Q, G, D) / total
        o, lse = o.permute(0, 2, 1, 3, 4), (top + total.log())[..., 0].permute(0, 2, 1, 3)
        s["out"][layer][:, h * G:e * G] = o[live].flatten(1, 2).to(s["out"].dtype)
        s["lse"][layer][:, h * G:e * G] = lse[live].flatten(1, 2)


def _run_plain_batch(s):
    kind = s["kind"]
    for layer in range(s["layers"]):
        if kind != "attend":
            _plain_append(s, layer)
        if kind != "append":
            _plain_attend(s, layer)
    return ([s["out"], s["lse"]] if kind != "append" else []) + (_state8(s) if kind != "attend" else [])


def _run_plain_compress(s):
    p0, last = s["begin"] // P, s["n"] % P or P
    src, dst = s["pages16"].long()[p0:], s["pages8"].long()[p0:]
    L, n, hkv = s["layers"], len(src), s["hkv"]
    x = s["pool"][:, src].float()                                                   # [layer][page][K, V][head][slot][D]
    empty = torch.zeros((n, 1, 1, P, 1), dtype=torch.bool, device=DEV)
    empty[-1, :, :, last:] = True
    k = _exponent(_magnitude(x).masked_fill_(empty, 0.0).flatten(4).amax(4), s["dtype"])
    new = _codes(x, k[..., None, None], s["dtype"])
    old = s["codes"][:, dst]
    old = torch.stack([old[:, :, 0].view(L, n, hkv, P, D), old[:, :, 1].view(L, n, hkv, D, P).transpose(3, 4)], 2)
    new = torch.where(empty, old, new)
    s["codes"][:, dst] = torch.stack([new[:, :, 0].flatten(3), new[:, :, 1].transpose(3, 4).flatten(3)], 2)
    s["scales"][:, dst] = _power(k).transpose(2, 3)
    return _state8(s)


def _run_plain_restore(s):
    s0, s1, L, hkv = s["begin"], s["n"], s["layers"], s["hkv"]
    p0 = s0 // P
    src, dst = s["pages8"].long()[p0:], s["pages16"].long()[p0:]
    n = len(src)
    x = _values(s["codes"][:, src]) * s["scales"][:, src].transpose(2, 3)[..., None]
    x = torch.stack([x[:, :, 0].view(L, n, hkv, P, D), x[:, :, 1].view(L, n, hkv, D, P).transpose(3, 4)], 2)
    token = p0 * P + torch.arange(n * P, device=DEV).view(n, 1, 1, P, 1)
    s["pool"][:, dst] = torch.where((token >= s0) & (token < s1), x.to(s["pool"].dtype), s["pool"][:, dst])
    return [s["pool"]]


def _run_plain_pack(s):
    pages = s["pages8"].long()[s["begin"] // P:]
    s["buf"][:s["codes_bytes"]] = s["codes"][:, pages].view(-1)
    s["buf"][s["codes_bytes"]:] = s["scales"][:, pages].view(-1).view(torch.uint8)
    return _buffer(s)


def _run_plain_unpack(s):
    pages, moved = s["pages8"].long()[s["begin"] // P:], s["codes_bytes"]
    L, n, hkv = s["layers"], len(pages), s["hkv"]
    s["codes"][:, pages] = s["buf"][:moved].view(L, n, 2, hkv, P * D)
    s["scales"][:, pages] = s["buf"][moved:].view(torch.float32).view(L, n, hkv, 2)
    return _state8(s)


_PLAIN = {"append": _run_plain_batch, "attend": _run_plain_batch, "step": _run_plain_batch,
          "compress": _run_plain_compress, "restore": _run_plain_restore, "pack": _run_plain_pack,
          "unpack": _run_plain_unpack}


# ---------------------------------------------------------------- exact ------
def exact(c, seed):
    s = prepare(c, seed)
    codes, scales = s["codes"].view(torch.float8_e4m3fn), s["scales"].double()
    if c["kind"] in ("pack", "unpack"):
        return _exact_moved(c, s, codes.double(), scales)
    if c["kind"] == "restore":
        return [_exact_restore(s, codes, scales)]
    values = codes.double() if c["kind"] != "attend" else None
    if c["kind"] == "compress":
        for i in range(-(-c["begin"] // P), s["entries"]):
            src, dst, filled = int(s["pages16"][i]), int(s["pages8"][i]), min(P, c["n"] - P * i)
            x = s["pool"][:, src, :, :, :filled].double()                           # [layer][K, V][head][slot][D]
            scale = _exact_scale(x.abs().amax((3, 4)), c["dtype"])
            y = _exact_round(x / scale[..., None, None], scale, c["dtype"])
            values[:, dst, 0].view(-1, c["hkv"], P, D)[:, :, :filled] = y[:, 0]
            values[:, dst, 1].view(-1, c["hkv"], D, P)[..., :filled] = y[:, 1].transpose(2, 3)
            scales[:, dst] = scale.transpose(1, 2)
        return [values, scales]
    out, lse = torch.zeros_like(s["out"], dtype=torch.float64), torch.zeros_like(s["lse"], dtype=torch.float64)
    begin, new = _lengths(c)
    cu_q, cu_pages, table = s["cu_q"].tolist(), s["cu_pages"].tolist(), s["table"].long()
    for i in range(c["layers"]):
        for b, (n0, n) in enumerate(zip(begin.tolist(), new.tolist())):
            pages = table[cu_pages[b]:cu_pages[b + 1]]
            if c["kind"] != "attend":
                for p in range(n0 // P, (n0 + n - 1) // P + 1):
                    lo, hi = max(n0, p * P), min(n0 + n, p * P + P)                 # the page's new tokens
                    at = slice(cu_q[b] + lo - n0, cu_q[b] + hi - n0)
                    x = torch.stack([s["k"][i, at], s["v"][i, at]]).double().transpose(1, 2)   # [K, V][head][slot][D]
                    scale, dst, lo, hi = _exact_scale(x.abs().amax((2, 3)), c["dtype"]), int(pages[p]), lo - p * P, hi - p * P
                    k_block, v_block = values[i, dst, 0].view(-1, P, D), values[i, dst, 1].view(-1, D, P).transpose(1, 2)
                    if lo:
                        had = scales[i, dst].transpose(0, 1)
                        scale = torch.maximum(scale, had)
                        by = (had / scale)[..., None, None]
                        k_block[:, :lo] = _exact_round(k_block[:, :lo] * by[0])
                        v_block[:, :lo] = _exact_round(v_block[:, :lo] * by[1])
                    y = _exact_round(x / scale[..., None, None], scale, c["dtype"])
                    k_block[:, lo:hi], v_block[:, lo:hi] = y[0], y[1]
                    scales[i, dst] = scale.transpose(0, 1)
            if c["kind"] != "append":
                _exact_attend(c, s, i, b, n0, n, cu_q[b], pages, (codes if values is None else values)[i], scales[i], out, lse)
    return ([out, lse] if c["kind"] != "append" else []) + ([values, scales] if c["kind"] != "attend" else [])


def _exact_scale(big, dtype):
    lo, hi = LIMITS[dtype]
    k = torch.ceil(torch.log2(big / 448)).clamp(lo, hi)
    k += (big > 448 * torch.exp2(k)) & (k < hi)                                     # (a logarithm rounded down to a whole one)
    return torch.exp2(k)


def _exact_round(x, scale=None, dtype=None):
    """To the nearest e4m3 number, ties to even, from the spacing of those numbers at x."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    y = torch.round(x / step) * step
    if scale is None:
        return y
    most = torch.where(scale == 2.0 ** LIMITS[dtype][1], 240.0, 448.0)[..., None, None]
    return torch.minimum(torch.maximum(y, -most), most)


def _exact_moved(c, s, values, scales):
    moved, first = s["codes_bytes"], c["begin"] // P
    buf, buf_scales = s["buf"][:moved].view(torch.float8_e4m3fn).double(), s["buf"][moved:].view(torch.float32).double()
    each, n = 2 * c["hkv"] * P * D, s["entries"] - first                            # codes of a page; pages
    buf, buf_scales = buf.view(c["layers"], n, each), buf_scales.view(c["layers"], n, 2 * c["hkv"])
    for i, page in enumerate(s["pages8"].tolist()[first:]):
        if c["kind"] == "pack":
            buf[:, i], buf_scales[:, i] = values[:, page].flatten(1), scales[:, page].flatten(1)
        else:
            values[:, page] = buf[:, i].view_as(values[:, page])
            scales[:, page] = buf_scales[:, i].view_as(scales[:, page])
    return [buf.view(-1), buf_scales.view(-1)] if c["kind"] == "pack" else [values, scales]


def _exact_restore(s, codes, scales):
    pool = s["pool"].double()
    for i in range(s["begin"] // P, s["entries"]):
        lo, hi = max(0, s["begin"] - P * i), min(P, s["n"] - P * i)
        src, dst = int(s["pages8"][i]), int(s["pages16"][i])
        block, scale = codes[:, src].double(), scales[:, src]
        k = block[:, 0].view(-1, s["hkv"], P, D) * scale[..., 0, None, None]
        v = block[:, 1].view(-1, s["hkv"], D, P).transpose(2, 3) * scale[..., 1, None, None]
        pool[:, dst, 0, :, lo:hi], pool[:, dst, 1, :, lo:hi] = k[:, :, lo:hi], v[:, :, lo:hi]
    return pool


def _exact_attend(c, s, layer, b, n0, n, q0, pages, codes, scales, out, lse):
    G, total = c["hq"] // c["hkv"], n0 + n
    for h in range(c["hkv"]):
        k = (codes.view(torch.uint8)[pages, 0, h].view(torch.float8_e4m3fn).double() if codes.dtype != torch.float64
             else codes[pages, 0, h]) * scales[pages, h, 0, None]
        v = (codes.view(torch.uint8)[pages, 1, h].view(torch.float8_e4m3fn).double() if codes.dtype != torch.float64
             else codes[pages, 1, h]) * scales[pages, h, 1, None]
        k, v = k.view(-1, D)[:total], v.view(-1, D, P).transpose(1, 2).reshape(-1, D)[:total]
        for r in range(0, n, 1024):
            e = min(n, r + 1024)
            seen = n0 + e
            q = s["q"][layer, q0 + r:q0 + e, h * G:(h + 1) * G].double()
            x = torch.mm(q.reshape(-1, D), k[:seen].t().contiguous()).view(e - r, G, seen) / math.sqrt(D)
            later = torch.arange(seen, device=DEV) > torch.arange(n0 + r, seen, device=DEV)[:, None]
            x.masked_fill_(later[:, None], -math.inf)
            l = torch.logsumexp(x, 2)
            out[layer, q0 + r:q0 + e, h * G:(h + 1) * G] = torch.mm(x.sub_(l[..., None]).exp_().view(-1, seen), v[:seen]).view(e - r, G, D)
            lse[layer, q0 + r:q0 + e, h * G:(h + 1) * G] = l
