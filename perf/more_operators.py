"""The paged cache held in 4 bits, as it is timed: new tokens stored as E2M1 with a power-of-two scale for each token, KV head
and 32 features and what the cache then holds of them read back (`append`), cached tokens of any 8- or 4-bit cache read back
as bf16 rows (`read`), and the drafting step that reads a 4-bit cache (`draft`).

With `own` false, run() computes them in elementary torch operations, in 32 bits; with `own` true it makes the library's
calls.  A page is 64 consecutive tokens of one request, all KV heads, as for the other caches.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

PAGE = 64
BLOCK = 32                           # features that share a scale in a 4-bit cache
HEADS = {64: (64, 8), 128: (32, 4)}  # query / KV heads of the two drafter shapes
MIN_EXPONENT = -100                  # of a scale
FP4 = torch.float4_e2m1fn_x2         # two codes a byte, the lower feature in the lower half
F8 = {"e4m3": (torch.float8_e4m3fn, 448.0), "e5m2": (torch.float8_e5m2, 57344.0)}  # 8-bit types, largest values


# ------------------------------------------------------------------------------------------- cases

def _append(C, ctx_lo, ctx_hi, new_lo, new_hi, D, fused):
    return {"kind": "append", "C": C, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi, "new_lo": new_lo, "new_hi": new_hi, "Hkv": HEADS[D][1],
            "D": D, "fused": fused}


def _read(C, lo, hi, D, type_, fused, pad):
    return {"kind": "read", "C": C, "lo": lo, "hi": hi, "Hkv": HEADS[D][1], "D": D, "type": type_, "fused": fused, "pad": pad}


def _draft(C, K, D, ctx_lo, ctx_hi, heads=None):
    Hq, Hkv = heads or HEADS[D]
    return {"kind": "draft", "C": C, "K": K, "Hq": Hq, "Hkv": Hkv, "D": D, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi}


def listed():
    return [
        # The paper's serving setting: four requests, each keeps up to eight tokens of a verified draft. Latency only.
        _append(4, 2048, 4096, 1, 8, 64, True) | {"name": "append_serving"},
        # The same of a full batch, larger heads.
        _append(256, 512, 8192, 1, 8, 128, False) | {"name": "append_batch"},
        # One prompt of the median training length (odd); K and V stand in the rows of a fused projection. Its own attention
        # runs on what the cache holds of it, so that it sees the values that later steps will see.
        _append(1, 0, 0, 3891, 3891, 64, True) | {"name": "append_prompt"},
        # Prompts of many lengths as one ragged batch, some after a cached prefix.
        _append(16, 0, 1000, 203, 16001, 128, False) | {"name": "append_prompts"},
        # A short prefix that another request shares, before its next chunk is computed. Latency only.
        _read(1, 77, 77, 64, "e2m1", False, 3) | {"name": "read_short"},
        # A long prefix (P90 to P99 of the training lengths), K and V side by side in each row.
        _read(1, 13701, 13701, 64, "e2m1", True, 0) | {"name": "read_prefix"},
        # A batch that moves from an 8-bit cache to another machine, in a buffer for the most tokens there may be.
        _read(32, 512, 8192, 128, "e4m3", False, 4000) | {"name": "read_batch"},
        # One request, one token: plain decoding on a short context; launches count.
        _draft(1, 1, 64, 77, 77) | {"name": "draft_one_token"},
        # The paper's serving setting: concurrency 4, K = 7.
        _draft(4, 7, 64, 2048, 4096) | {"name": "draft_serving"},
        # Two requests with contexts of the P90 to P99 length, larger heads.
        _draft(2, 5, 128, 10800, 20000) | {"name": "draft_long_d128"},
        # A full batch of requests of all lengths.
        _draft(64, 7, 64, 512, 8192) | {"name": "draft_batch"},
        # The same on the larger heads, K = 8 and sixteen query heads a KV head: 128 query rows share a cache row.
        _draft(48, 8, 128, 500, 8191, (64, 4)) | {"name": "draft_batch_wide_d128"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "append", "read", "read", "draft", "draft", "draft"])
    D = rng.choice([64, 128])
    if kind == "draft":
        C = _log_int(rng, 1, 64)
        hi = _log_int(rng, 1, 20000 if C <= 16 else 8192)
        heads = HEADS[D] if rng.random() < 0.6 else rng.choice([(4, 4), (9, 3), (16, 1), (32, 2)])
        return _draft(C, rng.choice([1, 3, 4, 5, 7, 8]), D, int(hi * rng.random()), hi, heads)
    fused = rng.random() < 0.5
    if kind == "read":
        C = _log_int(rng, 1, 32)
        hi = _log_int(rng, 1, 8000)
        return _read(C, int(hi * rng.random()), hi, D, rng.choice(["e2m1", "e2m1", "e4m3", "e5m2"]), fused, rng.choice([0, 1, 500]))
    if rng.random() < 0.5:  # a step
        C = _log_int(rng, 1, 256)
        hi = _log_int(rng, 16, 8192)
        return _append(C, int(hi * rng.random()), hi, 1, rng.choice([1, 4, 8]), D, fused)
    C = _log_int(rng, 1, 16)
    hi = _log_int(rng, 16, 8000)
    return _append(C, 0, rng.choice([0, 0, 1000]), max(1, int(hi * rng.random())), hi, D, fused)


def _spread(lo, hi, n, seed):
    """n whole numbers from lo to hi, both ends present, in a mixed order."""
    v = [hi] if n == 1 else [lo + (hi - lo) * i // (n - 1) for i in range(n)]
    random.Random(seed * 1000003 + n).shuffle(v)
    return v


def _lengths(case):
    """(cached tokens, new tokens) of each request."""
    C = case["C"]
    return _spread(case["ctx_lo"], case["ctx_hi"], C, 1), _spread(case["new_lo"], case["new_hi"], C, 2)


def _pages(n):
    return (n + PAGE - 1) // PAGE


def work(case):
    Hkv, D = case["Hkv"], case["D"]
    token = 2 * Hkv * (D // 2 + D // BLOCK)  # bytes of a token's keys and values in 4 bits, with their scales
    if case["kind"] == "draft":
        C, K, Hq = (case[n] for n in ("C", "K", "Hq"))
        ctx, rows = _spread(case["ctx_lo"], case["ctx_hi"], C, 1), C * K
        return {"bytes": sum(ctx) * token + 4 * sum(_pages(n) for n in ctx) + 4 * C + 2 * rows * (Hq + Hkv) * D * 2 + rows * Hq * 4 + 4 * C,
                "flops": 4 * D * Hq * sum(K * n + K * (K + 1) // 2 for n in ctx)}
    if case["kind"] == "append":
        n = sum(_lengths(case)[1])
        return {"bytes": n * (8 + token + 2 * 4 * Hkv * D), "flops": 4 * n * Hkv * D}
    n = _spread(case["lo"], case["hi"], case["C"], 1)
    held = sum(n) * token if case["type"] == "e2m1" else sum(n) * 2 * Hkv * D + sum(_pages(x) for x in n) * 2 * Hkv
    rows = sum(n) + case["pad"]
    return {"bytes": held + rows * (8 + 4 * Hkv * D), "flops": 2 * sum(n) * Hkv * D}


# ---------------------------------------------------------------------------------------------- states

def _random(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _keys(g, *shape):
    """Keys have channels that are several times as large as the others."""
    gain = torch.where(torch.rand(shape[-1], generator=g, device="cuda") < 0.06, 6.0, 1.0)
    return _random(g, *shape) * gain


def _power(e):
    """2^e, exactly; e a whole number in [-126, 127]."""
    return ((e + 127).to(torch.int32) << 23).view(torch.float32)


def _exponent(amax, top, part):
    """The smallest e, at least MIN_EXPONENT, with amax <= part * 2^top * 2^e; part in [0.5, 1)."""
    m, p = torch.frexp(amax)
    e = p - top + (m > part).to(p.dtype)
    return torch.where(amax > 0, e, torch.full_like(e, MIN_EXPONENT)).clamp(min=MIN_EXPONENT)


def _scales(e):
    return (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _narrow(x):
    """(codes, two a byte; exponents of the scales) of x [..., D] in 4 bits."""
    x = x.float().unflatten(-1, (-1, BLOCK))
    e = _exponent(x.abs().amax(-1), 3, 0.75)                 # the largest value is 6 = 0.75 * 2^3
    y = x * _power(-e)[..., None]
    size = y.abs()
    step = torch.where(size < 2.0, 0.5, torch.where(size < 4.0, 1.0, 2.0))
    size = torch.round(size / step) * step                   # (to even, as the codes are)
    code = torch.where(size < 2.0, 2.0 * size, torch.where(size < 4.0, size + 2.0, size / 2.0 + 4.0)).to(torch.uint8)
    code = (code + 8 * torch.signbit(y)).to(torch.uint8).flatten(-2)
    return code[..., ::2] | (code[..., 1::2] << 4), e


def _widen(codes, scale):
    """The values (float32) of packed codes [..., D / 2] and scales [..., D / BLOCK]."""
    raw = codes.view(torch.uint8)
    c = torch.stack([raw & 15, raw >> 4], -1).flatten(-2)
    half = (c & 7).float()
    size = torch.where(half < 4.0, 0.5 * half, torch.where(half < 6.0, half - 2.0, 2.0 * half - 8.0))
    x = torch.where(c > 7, -size, size).unflatten(-1, (-1, BLOCK))
    return (x * _power(scale.view(torch.uint8).to(torch.int32) - 127)[..., None]).flatten(-2)


def _pool(x, type_):
    """Pages and scales of a cache that holds x [pages, Hkv, 64, D]."""
    if type_ == "e2m1":
        codes, e = _narrow(x)
        return codes.view(FP4), _scales(e)
    dtype, largest = F8[type_]
    e = _exponent(x.abs().amax((2, 3)), int(math.log2(largest / 0.875)), 0.875)
    return (x * _power(-e)[:, :, None, None]).to(dtype), _scales(e)


def _table(g, held, n_pages):
    """A pool in use: the block table of requests of `held` tokens, pages in any order."""
    perm = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    counts = torch.tensor([_pages(n) for n in held], device="cuda")
    col = torch.arange(max(1, _pages(max(held))), device="cuda")
    at = (counts.cumsum(0) - counts)[:, None] + col
    return torch.where(col < counts[:, None], perm[at.clamp(max=n_pages - 1)], -1)


def _slots(table, ctx, new):
    """Slots of tokens [ctx, ctx + new) of each request, one after another."""
    request = np.repeat(np.arange(len(new)), new)
    first = np.cumsum([0] + list(new))[:-1]
    pos = torch.from_numpy(np.asarray(ctx)[request] + np.arange(sum(new)) - first[request]).cuda()
    return table[torch.from_numpy(request).cuda(), pos // PAGE].long() * PAGE + pos % PAGE


def _prepare_append(case, g):
    ctx, new = _lengths(case)
    n, Hkv, D = sum(new), case["Hkv"], case["D"]
    n_pages = sum(_pages(a + b) for a, b in zip(ctx, new)) + 3
    slots = _slots(_table(g, [a + b for a, b in zip(ctx, new)], n_pages), ctx, new)
    kp, ks = _pool(_keys(g, n_pages, Hkv, PAGE, D), "e2m1")
    vp, vs = _pool(_random(g, n_pages, Hkv, PAGE, D), "e2m1")
    if case["fused"]:  # rows of a fused projection: 2 * Hkv query heads' values stand before the keys
        rows = _keys(g, n, 4 * Hkv * D).to(torch.bfloat16)
        k = rows[:, 2 * Hkv * D:3 * Hkv * D].unflatten(1, (Hkv, D))
        v = rows[:, 3 * Hkv * D:].unflatten(1, (Hkv, D))
    else:
        k, v = _keys(g, n, Hkv, D).to(torch.bfloat16), _random(g, n, Hkv, D).to(torch.bfloat16)
    return {"k": k, "v": v, "slots": slots, "k_pages": kp, "v_pages": vp, "k_scale": ks, "v_scale": vs,
            "k_out": torch.empty((n, Hkv, D), dtype=torch.bfloat16, device="cuda"),
            "v_out": torch.empty((n, Hkv, D), dtype=torch.bfloat16, device="cuda")}


def _prepare_read(case, g):
    lens = _spread(case["lo"], case["hi"], case["C"], 1)
    n, Hkv, D = sum(lens) + case["pad"], case["Hkv"], case["D"]
    n_pages = sum(_pages(x) for x in lens) + 3
    slots = _slots(_table(g, lens, n_pages), [0] * len(lens), lens)
    kp, ks = _pool(_keys(g, n_pages, Hkv, PAGE, D), case["type"])
    vp, vs = _pool(_random(g, n_pages, Hkv, PAGE, D), case["type"])
    if case["fused"]:
        rows = torch.empty((n, 2, Hkv, D), dtype=torch.bfloat16, device="cuda")
        k, v = rows[:, 0], rows[:, 1]
    else:
        k, v = (torch.empty((n, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    return {"slots": torch.cat([slots, slots.new_full((case["pad"],), -1)]), "k_pages": kp, "v_pages": vp, "k_scale": ks, "v_scale": vs,
            "k_out": k, "v_out": v}


def _prepare_draft(case, g):
    C, K, Hq, Hkv, D = (case[n] for n in ("C", "K", "Hq", "Hkv", "D"))
    ctx = _spread(case["ctx_lo"], case["ctx_hi"], C, 1)
    n_pages = sum(_pages(n) for n in ctx) + 1
    table = _table(g, ctx, n_pages)
    kp, ks = _pool(_keys(g, n_pages, Hkv, PAGE, D), "e2m1")
    vp, vs = _pool(_random(g, n_pages, Hkv, PAGE, D), "e2m1")
    q, k, v = _random(g, C, K, Hq, D), _keys(g, C, K, Hkv, D), _random(g, C, K, Hkv, D)
    return {"q": q.to(torch.bfloat16), "k": k.to(torch.bfloat16), "v": v.to(torch.bfloat16), "k_pages": kp, "v_pages": vp,
            "k_scale": ks, "v_scale": vs, "table": table, "ctx": torch.tensor(ctx, dtype=torch.int32, device="cuda"),
            "o": torch.empty((C, K, Hq, D), dtype=torch.bfloat16, device="cuda"), "lse": torch.empty((C, Hq, K), device="cuda"),
            "status": torch.empty((C,), dtype=torch.int32, device="cuda")}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"append": _prepare_append, "read": _prepare_read, "draft": _prepare_draft}[case["kind"]](case, g) | {"case": case}
    if own:  # what a serving program keeps beside its buffers: the call's shape, and scratch of the size that the library names
        import paper_2602_01469_amd as pe
        n_pages = s["k_pages"].shape[0]
        if case["kind"] == "draft":
            s["shape"] = pe.DecodeShape(case["C"], case["K"], case["Hq"], case["Hkv"], case["D"], n_pages, s["table"].shape[1])
            s["ws"] = torch.empty(pe.peagle_draft_decode_block_scaled_workspace_bytes(s["shape"]), dtype=torch.uint8, device="cuda")
        else:
            s["shape"] = pe.CacheShape(s["slots"].numel(), case["Hkv"], case["D"], n_pages)
    return s


# --------------------------------------------------------------------------------------------- plain forms

def _plain_store(x, pages, scale, slots):
    codes, e = _narrow(x)
    page, off = slots // PAGE, slots % PAGE
    pages.view(torch.uint8)[page, :, off] = codes
    scale.view(torch.uint8)[page, :, off] = (e + 127).to(torch.uint8)


def _plain_read(pages, scale, slots):
    there = slots >= 0
    page, off = slots.clamp(min=0) // PAGE, slots.clamp(min=0) % PAGE
    raw = pages.view(torch.uint8)[page, :, off]
    if pages.dtype is FP4:
        x = _widen(raw, scale.view(torch.uint8)[page, :, off])
    else:
        x = raw.view(pages.dtype).float() * _power(scale.view(torch.uint8)[page].to(torch.int32) - 127)[..., None]
    return torch.where(there[:, None, None], x, 0.0).to(torch.bfloat16)


def _plain_draft(s):
    q, table, ctx = s["q"].float(), s["table"].clamp(min=0).long(), s["ctx"]
    C, K, Hq, D = q.shape
    Hkv = s["k"].shape[2]
    T = table.shape[1] * PAGE
    cached = torch.arange(T, device=q.device) < ctx[:, None]

    def rows(pages, scale, new):
        x = _widen(pages.view(torch.uint8)[table], scale.view(torch.uint8)[table])
        x = x.transpose(2, 3).reshape(C, T, Hkv, D)
        x = torch.where(cached[:, :, None, None], x, 0.0)
        return torch.cat([x, new.float()], 1).transpose(1, 2).contiguous()

    k, v = rows(s["k_pages"], s["k_scale"], s["k"]), rows(s["v_pages"], s["v_scale"], s["v"])
    q = q.view(C, K, Hkv, Hq // Hkv, D).transpose(1, 2).reshape(C, Hkv, -1, D)
    own_chain = torch.ones((K, K), dtype=torch.bool, device=q.device).tril()
    seen = torch.cat([cached[:, None].expand(C, K, T), own_chain.expand(C, K, K)], 2).repeat_interleave(Hq // Hkv, 1)[:, None]
    x = torch.where(seen, torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(D), -math.inf)
    m = x.amax(-1, keepdim=True)
    x = torch.exp(x - m)
    total = x.sum(-1, keepdim=True)
    o = (torch.matmul(x, v) / total).view(C, Hkv, K, Hq // Hkv, D).transpose(1, 2).reshape(C, K, Hq, D)
    lse = (m + total.log()).view(C, Hkv, K, Hq // Hkv).transpose(2, 3).reshape(C, Hq, K)
    return {"o": o.to(torch.bfloat16), "lse": lse, "status": torch.zeros_like(ctx)}


# ------------------------------------------------------------------------------------------------------ runs

def _run_own(s):
    import paper_2602_01469_amd as pe
    kind = s["case"]["kind"]
    cache = s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"]
    if kind == "draft":
        pe.peagle_draft_decode_block_scaled(s["shape"], s["q"], s["k"], s["v"], *cache, s["table"], s["ctx"], s["o"], s["lse"], s["status"], s["ws"])
        return {n: s[n] for n in ("o", "lse", "status")}
    if kind == "append":
        pe.peagle_cache_append_block_scaled(s["shape"], s["k"], s["v"], s["slots"], *cache)
    pe.peagle_cache_read(s["shape"], s["slots"], *cache, s["k_out"], s["v_out"])
    return {n: s[n] for n in (("k_out", "v_out", "k_scale", "v_scale") if kind == "append" else ("k_out", "v_out"))}


def run(s):
    """One pass.  A second append of the same tokens writes the same codes and scales."""
    if own:
        return _run_own(s)
    kind = s["case"]["kind"]
    if kind == "draft":
        return _plain_draft(s)
    if kind == "append":
        _plain_store(s["k"], s["k_pages"], s["k_scale"], s["slots"])
        _plain_store(s["v"], s["v_pages"], s["v_scale"], s["slots"])
    out = {"k_out": _plain_read(s["k_pages"], s["k_scale"], s["slots"]), "v_out": _plain_read(s["v_pages"], s["v_scale"], s["slots"])}
    return out | ({n: s[n] for n in ("k_scale", "v_scale")} if kind == "append" else {})


# -------------------------------------------------------------------------------------------- from the definitions

VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # of the codes 0 to 7; 8 to 15 are their negatives


def _values64(pages, scale):
    """What a 4-bit cache holds, as 64-bit numbers."""
    raw = pages.view(torch.uint8).long()
    both = torch.tensor([*VALUES, *(-v for v in VALUES)], dtype=torch.float64, device=raw.device)
    x = torch.stack([both[raw % 16], both[raw // 16]], -1).flatten(-2)
    return x * scale.double().repeat_interleave(BLOCK, -1)


def _stored64(x):
    """(values, scales) that x [tokens, Hkv, D] becomes in the cache."""
    x = x.double().unflatten(-1, (-1, BLOCK))
    amax = x.abs().amax(-1)
    scale = torch.full_like(amax, 2.0 ** MIN_EXPONENT)
    while bool((amax > VALUES[-1] * scale).any()):
        scale = torch.where(amax > VALUES[-1] * scale, 2.0 * scale, scale)
    size = (x / scale[..., None]).abs()
    code = torch.zeros_like(size, dtype=torch.int64)
    for c in range(1, 8):  # halfway goes to the even code
        middle = (VALUES[c - 1] + VALUES[c]) / 2
        code += (size > middle) if c % 2 else (size >= middle)
    values = torch.tensor(VALUES, dtype=torch.float64, device=x.device)[code]
    return (torch.copysign(values, x) * scale[..., None]).flatten(-2), scale


def _exact_append(s):
    out = {}
    for n in "kv":
        scales = s[n + "_scale"].double()
        parts = []
        for at in range(0, s["slots"].numel(), 16384):
            slots = s["slots"][at:at + 16384]
            values, scale = _stored64(s[n][at:at + 16384])
            scales[slots // PAGE, :, slots % PAGE] = scale
            parts.append(values)
        out |= {n + "_out": torch.cat(parts), n + "_scale": scales}
    return out


def _exact_read(s, type_):
    out = {}
    for n in "kv":
        pages, scale, parts = s[n + "_pages"], s[n + "_scale"], []
        for at in range(0, s["slots"].numel(), 16384):
            slots = s["slots"][at:at + 16384]
            page, off = slots.clamp(min=0) // PAGE, slots.clamp(min=0) % PAGE
            raw = pages.view(torch.uint8)[page, :, off]
            if type_ == "e2m1":
                x = _values64(raw, scale.view(torch.uint8)[page, :, off].view(scale.dtype))
            else:
                x = raw.view(pages.dtype).double() * scale.double()[page][..., None]
            x[slots < 0] = 0.0
            parts.append(x)
        out[n + "_out"] = torch.cat(parts)
    return out


def _exact_draft(s):
    q, ctx = s["q"].double(), s["ctx"].tolist()
    C, K, Hq, D = q.shape
    Hkv = s["k"].shape[2]
    o, lse = torch.empty_like(q), torch.empty((C, Hq, K), dtype=torch.float64, device=q.device)
    for c, n in enumerate(ctx):
        pages = s["table"][c, :_pages(n)].long()
        for h in range(Hkv):
            rows = lambda x: torch.cat([_values64(s[x + "_pages"].view(torch.uint8)[pages, h], s[x + "_scale"].view(torch.uint8)[pages, h]
                                                  .view(torch.float8_e8m0fnu)).reshape(-1, D)[:n], s[x][c, :, h].double()])
            k, v = rows("k"), rows("v")
            heads = slice(h * (Hq // Hkv), (h + 1) * (Hq // Hkv))
            for d in range(K):
                x = q[c, d, heads] @ k[:n + d + 1].T / math.sqrt(D)
                lse[c, heads, d] = torch.logsumexp(x, 1)
                o[c, d, heads] = torch.exp(x - lse[c, heads, d][:, None]) @ v[:n + d + 1]
    return {"o": o, "lse": lse, "status": None}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "append":
        return _exact_append(s)
    return _exact_read(s, case["type"]) if case["kind"] == "read" else _exact_draft(s)
