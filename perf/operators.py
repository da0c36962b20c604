"""The serving operators around a paged cache that is held in 8 bits, as they are timed: block tables and slot maps built on
the GPU from request lengths (`plan`), new tokens' keys and values stored with one power-of-two scale for each page and KV
head (`append`), and the drafting step that reads such a cache (`draft`).

With `own` false, run() computes them in elementary torch operations, in 32 bits; with `own` true it makes the library's
calls.  A page is 64 consecutive tokens of one request, all KV heads, as for the bf16 cache.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

PAGE = 64
HEADS = {64: (64, 8), 128: (32, 4)}  # query / KV heads of the two drafter shapes
MIN_EXPONENT = -100                  # of a scale
TYPES = {  # type of the cache: largest finite value, stored significand bits, exponent of the smallest normal value
    "e4m3": (torch.float8_e4m3fn, 448.0, 3, -6),
    "e5m2": (torch.float8_e5m2, 57344.0, 2, -14),
}
LARGEST_PROMPTS = 131072             # rows of a slot map


# ------------------------------------------------------------------------------------------- cases

def _plan(C, ctx_lo, ctx_hi, new_lo, new_hi, ended, pad):
    return {"kind": "plan", "C": C, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi, "new_lo": new_lo, "new_hi": new_hi, "ended": ended, "pad": pad}


def _append(C, ctx_lo, ctx_hi, new_lo, new_hi, D, type_, fused):
    return {"kind": "append", "C": C, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi, "new_lo": new_lo, "new_hi": new_hi, "Hkv": HEADS[D][1],
            "D": D, "type": type_, "fused": fused}


def _draft(C, K, D, ctx_lo, ctx_hi, type_, heads=None):
    Hq, Hkv = heads or HEADS[D]
    return {"kind": "draft", "C": C, "K": K, "Hq": Hq, "Hkv": Hkv, "D": D, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi, "type": type_}


def listed():
    return [
        # The paper's serving setting: four requests, each keeps up to eight tokens of a verified draft. Latency only.
        _plan(4, 2048, 4096, 1, 8, 0, 32) | {"name": "plan_serving"},
        # A full batch between two steps, some requests of which have ended and give their pages back.
        _plan(256, 512, 8192, 1, 8, 32, 2048) | {"name": "plan_batch"},
        # Admission of prompts of the training distribution's long end: a slot for each of their tokens.
        _plan(16, 0, 0, 2469, 13701, 0, 131072) | {"name": "plan_prompts"},
        # The tokens that a serving step keeps: most land in a page that others have begun, whose scale may have to grow.
        _append(4, 2048, 4096, 1, 8, 64, "e4m3", True) | {"name": "append_serving"},
        # The same of a full batch, larger heads.
        _append(256, 512, 8192, 1, 8, 128, "e5m2", False) | {"name": "append_batch"},
        # One prompt of the median training length (odd), whole pages but the last; K and V stand in the rows of a fused projection.
        _append(1, 0, 0, 3891, 3891, 64, "e4m3", True) | {"name": "append_prompt"},
        # Prompts of many lengths as one ragged batch, some after a cached prefix.
        _append(16, 0, 1000, 203, 16001, 128, "e4m3", False) | {"name": "append_prompts"},
        # One request, one token: plain decoding on a short context; launches count.
        _draft(1, 1, 64, 77, 77, "e4m3") | {"name": "draft_one_token"},
        # The paper's serving setting: concurrency 4, K = 7.
        _draft(4, 7, 64, 2048, 4096, "e4m3") | {"name": "draft_serving"},
        # Two requests with contexts of the P90 to P99 length, larger heads.
        _draft(2, 5, 128, 10800, 20000, "e4m3") | {"name": "draft_long_d128"},
        # A full batch of requests of all lengths: the cache read fills the memory system.
        _draft(64, 7, 64, 512, 8192, "e4m3") | {"name": "draft_batch"},
        # The same on the larger heads, K = 8 and sixteen query heads a KV head: 128 query rows share a cache row.
        _draft(48, 8, 128, 500, 8191, "e5m2", (64, 4)) | {"name": "draft_batch_wide_d128"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["plan", "append", "append", "draft", "draft", "draft"])
    type_ = rng.choice(["e4m3", "e4m3", "e5m2"])
    D = rng.choice([64, 128])
    if kind == "draft":
        C = _log_int(rng, 1, 64)
        hi = _log_int(rng, 1, 20000 if C <= 16 else 8192)
        heads = HEADS[D] if rng.random() < 0.6 else rng.choice([(4, 4), (9, 3), (16, 1), (32, 2)])
        K = rng.choice([1, 3, 4, 5, 7, 8])
        return _draft(C, K, D, int(hi * rng.random()), hi, type_, heads)
    if rng.random() < 0.5:  # a step
        C = _log_int(rng, 1, 512 if kind == "plan" else 256)
        hi = _log_int(rng, 16, 8192)
        step = (C, int(hi * rng.random()), hi, 1, rng.choice([1, 4, 8]))
        if kind == "plan":
            return _plan(*step, rng.randint(0, C // 4), 8 * C)
        return _append(*step, D, type_, rng.random() < 0.5)
    C = _log_int(rng, 1, 16)
    hi = _log_int(rng, 16, LARGEST_PROMPTS // C if kind == "plan" else 8000)
    hi = min(hi, 20000)
    lo = max(1, int(hi * rng.random()))
    if kind == "plan":
        return _plan(C, 0, rng.choice([0, 100]), lo, hi, 0, C * hi)
    return _append(C, 0, rng.choice([0, 0, 1000]), lo, hi, D, type_, rng.random() < 0.5)


def _spread(lo, hi, n, seed):
    """n whole numbers from lo to hi, both ends present, in a mixed order."""
    v = [hi] if n == 1 else [lo + (hi - lo) * i // (n - 1) for i in range(n)]
    random.Random(seed * 1000003 + n).shuffle(v)
    return v


def _lengths(case):
    """(cached tokens, new tokens, tokens whose pages are held) of each request."""
    C = case["C"]
    ctx, new = _spread(case["ctx_lo"], case["ctx_hi"], C, 1), _spread(case["new_lo"], case["new_hi"], C, 2)
    held = list(ctx)
    for c in range(0, case.get("ended", 0)):  # a request that has ended still holds its pages
        ctx[c] = new[c] = 0
    return ctx, new, held


def _pages(n):
    return (n + PAGE - 1) // PAGE


def work(case):
    if case["kind"] == "draft":
        C, K, Hq, Hkv, D = (case[n] for n in ("C", "K", "Hq", "Hkv", "D"))
        ctx, rows = _spread(case["ctx_lo"], case["ctx_hi"], C, 1), C * K
        pages = sum(_pages(n) for n in ctx)
        return {"bytes": 2 * sum(ctx) * Hkv * D + pages * (2 * Hkv + 4) + 4 * C + 2 * rows * (Hq + Hkv) * D * 2 + rows * Hq * 4 + 4 * C,
                "flops": 4 * D * Hq * sum(K * n + K * (K + 1) // 2 for n in ctx)}
    ctx, new, held = _lengths(case)
    if case["kind"] == "append":
        n = sum(new)
        touched = sum(_pages(a + b) - a // PAGE for a, b in zip(ctx, new))
        return {"bytes": 2 * n * case["Hkv"] * case["D"] * 3 + 8 * n + 2 * touched * case["Hkv"], "flops": 4 * n * case["Hkv"] * case["D"]}
    taken = sum(max(0, _pages(a + b) - _pages(h)) for a, b, h in zip(ctx, new, held))
    given = sum(max(0, _pages(h) - _pages(a + b)) for a, b, h in zip(ctx, new, held))
    C = case["C"]
    return {"bytes": 8 * case["pad"] + 12 * C + 16 * C + 4 * C + 8 * (taken + given) + 8, "flops": case["pad"] + C}


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


def _exponent(amax, type_):
    """The smallest e with amax <= largest * 2^e; the largest value of either type is 0.875 times a power of two."""
    largest = TYPES[type_][1]
    top = int(math.log2(largest / 0.875))
    m, p = torch.frexp(amax)
    e = p - top + (m > 0.875).to(p.dtype)
    return torch.where(amax > 0, e, torch.full_like(e, MIN_EXPONENT)).clamp(min=MIN_EXPONENT)


def _codes(e):
    return (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _cache(x, type_):
    """Pages and scales of a cache that holds x [pages, Hkv, 64, D]."""
    e = _exponent(x.abs().amax((2, 3)), type_)
    return (x * _power(-e)[:, :, None, None]).to(TYPES[type_][0]), _codes(e)


def _table(g, held, max_pages, n_pages):
    """A pool in use: pages in any order; (block table, the pages that no request holds)."""
    perm = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    counts = torch.tensor([_pages(n) for n in held], device="cuda")
    col = torch.arange(max_pages, device="cuda")
    at = (counts.cumsum(0) - counts)[:, None] + col
    table = torch.where(col < counts[:, None], perm[at.clamp(max=n_pages - 1)], -1)
    total = sum(_pages(n) for n in held)
    free = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
    free[:n_pages - total] = perm[total:]
    return table, free, counts.to(torch.int32), n_pages - total


def _prepare_plan(case, g):
    ctx, new, held = _lengths(case)
    C, most = case["C"], max(max(a + b, h) for a, b, h in zip(ctx, new, held))
    max_pages = _pages(most) + 1
    n_pages = sum(_pages(max(a + b, h)) for a, b, h in zip(ctx, new, held)) + 8
    table, free, counts, n_free = _table(g, held, max_pages, n_pages)
    i32 = lambda *shape: torch.empty(shape, dtype=torch.int32, device="cuda")
    s = {"ctx": torch.tensor(ctx, dtype=torch.int32, device="cuda"), "new": torch.tensor(new, dtype=torch.int32, device="cuda"),
         "held": counts, "free": free, "free_count": torch.tensor([n_free], dtype=torch.int32, device="cuda"), "table": table,
         "token_start": i32(C + 1), "slots": torch.empty((case["pad"],), dtype=torch.int64, device="cuda"), "seq_len": i32(C),
         "status": i32(C), "held_out": i32(C), "free_count_out": i32(1)}
    if own:
        import paper_2602_01469_amd as pe
        s["shape"] = pe.PlanShape(C, max_pages, n_pages, case["pad"])
        s["ws"] = torch.empty(pe.peagle_cache_plan_workspace_bytes(s["shape"]), dtype=torch.uint8, device="cuda")
    return s


def _prepare_append(case, g):
    ctx, new, _ = _lengths(case)
    n, Hkv, D = sum(new), case["Hkv"], case["D"]
    n_pages = sum(_pages(a + b) for a, b in zip(ctx, new)) + 3
    table, _, _, _ = _table(g, [a + b for a, b in zip(ctx, new)], max(_pages(a + b) for a, b in zip(ctx, new)), n_pages)
    request = np.repeat(np.arange(case["C"]), new)
    first = np.cumsum([0] + new)[:-1]
    pos = torch.from_numpy(np.asarray(ctx)[request] + np.arange(n) - first[request]).cuda()
    slots = table[torch.from_numpy(request).cuda(), pos // PAGE].long() * PAGE + pos % PAGE
    kp, ks = _cache(_keys(g, n_pages, Hkv, PAGE, D), case["type"])
    vp, vs = _cache(_random(g, n_pages, Hkv, PAGE, D), case["type"])
    if case["fused"]:  # rows of a fused projection: 2 * Hkv query heads' values stand before the keys
        rows = _keys(g, n, 4 * Hkv * D).to(torch.bfloat16)
        k = rows[:, 2 * Hkv * D:3 * Hkv * D].unflatten(1, (Hkv, D))
        v = rows[:, 3 * Hkv * D:].unflatten(1, (Hkv, D))
    else:
        k, v = _keys(g, n, Hkv, D).to(torch.bfloat16), _random(g, n, Hkv, D).to(torch.bfloat16)
    s = {"k": k, "v": v, "slots": slots, "first": torch.from_numpy(first).cuda(), "k_pages": kp, "v_pages": vp, "k_scale": ks,
         "v_scale": vs}
    if own:
        import paper_2602_01469_amd as pe
        s["shape"] = pe.CacheShape(n, Hkv, D, n_pages)
    return s


def _prepare_draft(case, g):
    C, K, Hq, Hkv, D = (case[n] for n in ("C", "K", "Hq", "Hkv", "D"))
    ctx = _spread(case["ctx_lo"], case["ctx_hi"], C, 1)
    max_pages, n_pages = max(1, _pages(max(ctx))), sum(_pages(n) for n in ctx) + 1
    table, _, _, _ = _table(g, ctx, max_pages, n_pages)
    kp, ks = _cache(_keys(g, n_pages, Hkv, PAGE, D), case["type"])
    vp, vs = _cache(_random(g, n_pages, Hkv, PAGE, D), case["type"])
    q, k, v = _random(g, C, K, Hq, D), _keys(g, C, K, Hkv, D), _random(g, C, K, Hkv, D)
    s = {"q": q.to(torch.bfloat16), "k": k.to(torch.bfloat16), "v": v.to(torch.bfloat16), "k_pages": kp, "v_pages": vp,
         "k_scale": ks, "v_scale": vs, "table": table, "ctx": torch.tensor(ctx, dtype=torch.int32, device="cuda"),
         "o": torch.empty((C, K, Hq, D), dtype=torch.bfloat16, device="cuda"), "lse": torch.empty((C, Hq, K), device="cuda"),
         "status": torch.empty((C,), dtype=torch.int32, device="cuda")}
    if own:
        import paper_2602_01469_amd as pe
        s["shape"] = pe.DecodeShape(C, K, Hq, Hkv, D, n_pages, max_pages)
        s["ws"] = torch.empty(pe.peagle_draft_decode_scaled_workspace_bytes(s["shape"]), dtype=torch.uint8, device="cuda")
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    make = {"plan": _prepare_plan, "append": _prepare_append, "draft": _prepare_draft}[case["kind"]]
    return make(case, g) | {"case": case}


# --------------------------------------------------------------------------------------------- plain forms

def _plain_plan(s):
    ctx, new, held, table = s["ctx"].long(), s["new"].long(), s["held"].long(), s["table"]
    C, max_pages = table.shape
    n_pages, rows = s["free"].numel(), s["slots"].numel()
    end = new.clamp(min=0).cumsum(0)
    start = end - new.clamp(min=0)
    ok = (ctx >= 0) & (new >= 0) & (ctx + new <= PAGE * max_pages) & (held >= (ctx + PAGE - 1) // PAGE) & (held <= max_pages) & (end <= rows)
    want = torch.where(ok, (ctx + new + PAGE - 1) // PAGE, held)
    surplus, need = (held - want).clamp(min=0), (want - held).clamp(min=0)
    col = torch.arange(max_pages, device=table.device)
    # what requests no longer need goes on the list, so that the first request's first page ends up on top
    count, given = s["free_count"].long().clamp(0, n_pages), surplus.sum()
    k = (surplus.cumsum(0) - surplus - want)[:, None] + col
    at = torch.where((col >= want[:, None]) & (col < held[:, None]), count + given - 1 - k, n_pages).clamp(max=n_pages)
    free = torch.cat([s["free"], s["free"].new_zeros(1)])
    free[at.reshape(-1)] = table.reshape(-1)
    free = free[:n_pages]
    # what they lack comes off its end, in order, for as long as it lasts
    there = (count + given).clamp(max=n_pages)
    need_end = need.cumsum(0)
    served = ok & ((need == 0) | (need_end <= there))
    j = (need_end - need - held)[:, None] + col
    takes = served[:, None] & (col >= held[:, None]) & (col < want[:, None])
    table = torch.where(takes, free[(there - 1 - j).clamp(0, n_pages - 1)], table)
    t = torch.arange(rows, device=table.device)
    c = torch.searchsorted(end, t, right=True)
    cc = c.clamp(max=C - 1)
    pos = ctx[cc] + t - start[cc]
    page = table[cc, (pos // PAGE).clamp(0, max_pages - 1)].long()
    slots = torch.where((c < C) & served[cc] & (page >= 0) & (page < n_pages), page * PAGE + pos % PAGE, -1)
    i32 = lambda x: x.to(torch.int32)
    return {"table": table, "free": free, "held": i32(torch.where(served, want, held)),
            "free_count": i32(there - torch.where(served, need, 0).sum()),
            "token_start": i32(torch.cat([end.new_zeros(1), end]).clamp(max=rows)), "slots": slots,
            "seq_len": i32(torch.where(served, ctx + new, ctx)), "status": i32(torch.where(ok, torch.where(served, 0, 2), 1))}


def _plain_store(x, pages, scale, slots, first, type_):
    """Stores x [tokens, Hkv, D] in place; `first`: each request's first token, the only one whose page may hold others."""
    x, codes = x.float(), scale.view(torch.uint8)
    page, off, e_old = slots // PAGE, slots % PAGE, codes.to(torch.int32) - 127
    size = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1)
    amax = torch.zeros_like(e_old, dtype=torch.float32).scatter_reduce(0, page[:, None].expand_as(size), size, "amax")
    start = torch.full((pages.shape[0],), PAGE, device=x.device).scatter_reduce(0, page, off, "amin")[:, None]
    e_new = _exponent(amax, type_)
    e = torch.where(start == 0, e_new, torch.where(start < PAGE, torch.maximum(e_new, e_old), e_old))
    begun = page[first]
    before = (torch.arange(PAGE, device=x.device) < start[begun])[:, None, :, None]
    turned = (pages[begun].float() * _power((e_old - e).clamp(min=-126))[begun][:, :, None, None]).to(pages.dtype).view(torch.uint8)
    raw = pages.view(torch.uint8)
    raw[begun] = torch.where(before, turned, raw[begun])
    raw[page, :, off] = (x * _power(-e)[page][:, :, None]).to(pages.dtype).view(torch.uint8)
    codes.copy_((e + 127).to(torch.uint8))


def _plain_draft(s):
    q, table, ctx = s["q"].float(), s["table"].clamp(min=0).long(), s["ctx"]
    C, K, Hq, D = q.shape
    Hkv = s["k"].shape[2]
    T = table.shape[1] * PAGE
    cached = torch.arange(T, device=q.device) < ctx[:, None]

    def rows(pages, scale, new):
        x = pages[table].float() * _power(scale.view(torch.uint8)[table].to(torch.int32) - 127)[..., None, None]
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
    if kind == "plan":
        pe.peagle_cache_plan(s["shape"], s["ctx"], s["new"], s["held"], s["free"], s["free_count"], s["table"], s["token_start"],
                             s["slots"], s["seq_len"], s["status"], s["ws"], s["held_out"], s["free_count_out"])
        return {n: s[n] for n in ("table", "free", "token_start", "slots", "seq_len", "status")} | {
            "held": s["held_out"], "free_count": s["free_count_out"]}
    if kind == "append":
        pe.peagle_cache_append_scaled(s["shape"], s["k"], s["v"], s["slots"], s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"])
        return {n: s[n] for n in ("k_pages", "v_pages", "k_scale", "v_scale")}
    pe.peagle_draft_decode_scaled(s["shape"], s["q"], s["k"], s["v"], s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"],
                                  s["table"], s["ctx"], s["o"], s["lse"], s["status"], s["ws"])
    return {n: s[n] for n in ("o", "lse", "status")}


def run(s):
    """One pass.  A plan of the same state takes the same pages again (the counts that it starts from are kept); a second
    append of the same tokens writes the same values, and finds the page's scale large enough."""
    if own:
        return _run_own(s)
    kind = s["case"]["kind"]
    if kind == "plan":
        return _plain_plan(s)
    if kind == "draft":
        return _plain_draft(s)
    for n in "kv":
        _plain_store(s[n], s[n + "_pages"], s[n + "_scale"], s["slots"], s["first"], s["case"]["type"])
    return {n: s[n] for n in ("k_pages", "v_pages", "k_scale", "v_scale")}


# -------------------------------------------------------------------------------------------- from the definitions

def _exact_plan(s):
    """Request by request, as a host's scheduler would do it."""
    host = lambda n: s[n].cpu().numpy().astype(np.int64)
    ctx, new, held, table, free = host("ctx"), host("new"), host("held"), host("table"), host("free")
    n_pages, rows, max_pages = len(free), s["slots"].numel(), table.shape[1]
    count, at = min(max(int(host("free_count")[0]), 0), n_pages), 0
    status, seq_len, slots, starts, want = np.zeros_like(ctx), ctx.copy(), np.full(rows, -1), [0], held.copy()
    for c in range(len(ctx)):
        at += max(int(new[c]), 0)
        starts.append(at)
        fits = ctx[c] >= 0 and new[c] >= 0 and ctx[c] + new[c] <= PAGE * max_pages and _pages(ctx[c]) <= held[c] <= max_pages
        status[c] = 0 if fits and at <= rows else 1
        if status[c] == 0:
            want[c] = _pages(ctx[c] + new[c])
    for c in reversed(range(len(ctx))):
        for b in reversed(range(want[c], held[c])):
            if count < n_pages:
                free[count] = table[c, b]
            count += 1
    count, out = min(count, n_pages), False
    for c in range(len(ctx)):
        lacks = max(int(want[c] - held[c]), 0)
        out = out or lacks > count
        if status[c] or (lacks and out):
            status[c], want[c] = status[c] or 2, held[c]
            continue
        for b in range(held[c], want[c]):
            count -= 1
            table[c, b] = free[count]
        seq_len[c] = ctx[c] + new[c]
        pos = np.arange(ctx[c], seq_len[c])
        page = table[c, pos // PAGE]
        slots[starts[c]:starts[c + 1]] = np.where((page >= 0) & (page < n_pages), page * PAGE + pos % PAGE, -1)
    return {"table": table, "free": free, "held": want, "free_count": np.array([count]),
            "token_start": np.minimum(starts, rows), "slots": slots, "seq_len": seq_len, "status": status}


def _power64(e):
    """2^e, exactly (a power function need not be)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _to_grid(x, type_):
    """x rounded to the type's values, ties to even, as 64-bit numbers; |x| at most the largest one."""
    _, _, bits, low = TYPES[type_]
    step = _power64(torch.clamp(torch.frexp(x)[1] - 1, min=low) - bits)
    return torch.round(x / step) * step


def _exact_append(s, type_):
    out = {}
    largest = TYPES[type_][1]
    slots = s["slots"].cpu().numpy()
    cuts = [0] + [t for t in range(1, len(slots)) if slots[t] != slots[t - 1] + 1 or slots[t] % PAGE == 0] + [len(slots)]
    for n in "kv":
        pages = s[n + "_pages"].double()
        scale = s[n + "_scale"].double()
        x = s[n].double()
        for a, b in zip(cuts, cuts[1:]):
            page, off = int(slots[a]) // PAGE, int(slots[a]) % PAGE
            new = x[a:b].transpose(0, 1)
            amax = new.abs().amax((1, 2))
            e = torch.ceil(torch.log2(amax / largest)).clamp(min=MIN_EXPONENT - 1)
            e = torch.where(amax > largest * _power64(e), e + 1, torch.where(amax <= largest * _power64(e - 1), e - 1, e))
            now = _power64(e.clamp(min=MIN_EXPONENT))
            if off:
                now = torch.maximum(now, scale[page])
                pages[page, :, :off] = _to_grid(pages[page, :, :off] * (scale[page] / now)[:, None, None], type_)
            pages[page, :, off:off + b - a] = _to_grid(new / now[:, None, None], type_)
            scale[page] = now
        out[n + "_pages"], out[n + "_scale"] = pages, scale
    return out


def _exact_draft(s):
    q, ctx = s["q"].double(), s["ctx"].tolist()
    C, K, Hq, D = q.shape
    Hkv = s["k"].shape[2]
    o, lse = torch.empty_like(q), torch.empty((C, Hq, K), dtype=torch.float64, device=q.device)
    for c, n in enumerate(ctx):
        pages = s["table"][c, :_pages(n)].long()
        for h in range(Hkv):
            rows = lambda x: torch.cat([(s[x + "_pages"][pages, h].double() * s[x + "_scale"][pages, h].double()[:, None, None])
                                        .reshape(-1, D)[:n], s[x][c, :, h].double()])
            k, v = rows("k"), rows("v")
            heads = slice(h * (Hq // Hkv), (h + 1) * (Hq // Hkv))
            for d in range(K):
                x = q[c, d, heads] @ k[:n + d + 1].T / math.sqrt(D)
                lse[c, heads, d] = torch.logsumexp(x, 1)
                o[c, d, heads] = torch.exp(x - lse[c, heads, d][:, None]) @ v[:n + d + 1]
    return {"o": o, "lse": lse, "status": None}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "plan":
        return _exact_plan(s)
    return _exact_append(s, case["type"]) if case["kind"] == "append" else _exact_draft(s)
