"""GPU tests of the paged cache between the drafting steps against the oracle (numpy, 64 bits): block tables and slot maps
(whole numbers: equal), and tokens stored in 8 bits with a power-of-two scale for each page and KV head (codes, scales and
untouched places: equal; every rounding is defined)."""
import numpy as np
import pytest
import torch

import paper_2602_01469_amd as pe
from gpu_harness import bf16_to_f64
from oracle import peagle_oracle as orc
from test_gpu_guards import Guarded

pytestmark = pytest.mark.gpu

TYPES = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
E8M0 = torch.float8_e8m0fnu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# ---------------------------------------------------------------------------------------------------------- plan

class Plan:
    """Device buffers of one plan and the call."""

    def __init__(self, ctx, new, held, free, count, table, max_tokens):
        i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()
        self.host = [np.array(x) for x in (ctx, new, held, free)] + [count, np.array(table), max_tokens]
        self.shape = pe.PlanShape(len(ctx), np.shape(table)[1], len(free), max_tokens)
        self.ctx, self.new, self.held, self.free, self.table = i32(ctx), i32(new), i32(held), i32(free), i32(table)
        self.count = i32([count])
        C = len(ctx)
        self.start, self.seq_len, self.status = i32(np.full(C + 1, -9)), i32(np.full(C, -9)), i32(np.full(C, -9))
        self.slots = torch.full((max_tokens,), -9, dtype=torch.int64, device="cuda")
        self.ws = torch.empty(pe.peagle_cache_plan_workspace_bytes(self.shape), dtype=torch.uint8, device="cuda")

    def call(self, held_out=None, count_out=None):
        pe.peagle_cache_plan(self.shape, self.ctx, self.new, self.held, self.free, self.count, self.table, self.start, self.slots,
                             self.seq_len, self.status, self.ws, held_out, count_out)

    def check(self, what, held=None, count=None):
        torch.cuda.synchronize()
        want = orc.cache_plan(*self.host)
        got = {"pages_held": self.held if held is None else held, "free_pages": self.free, "free_count": self.count if count is None else count,
               "block_table": self.table, "token_start": self.start, "slots": self.slots, "seq_len": self.seq_len, "status": self.status}
        for n, x in got.items():
            assert np.array_equal(x.cpu().numpy(), want[n]), (what, n)
        return want


def _pages(n):
    return -(-np.asarray(n) // 64)


def _state(rng, C, ctx_hi, new_hi, spare, extra_columns=2, ended=0.1, rolled_back=0.1):
    """A pool in use: requests that go on, that ended, and that hold a page more than they need."""
    ctx, new = rng.integers(0, ctx_hi + 1, C), rng.integers(0, new_hi + 1, C)
    held = _pages(ctx)
    over = rng.random(C) < ended
    ctx[over] = new[over] = 0
    max_pages = int(_pages(ctx_hi + new_hi)) + extra_columns
    held = held + (rng.random(C) < rolled_back)
    n_pages = int(held.sum() + np.maximum(_pages(ctx + new) - held, 0).sum()) + spare
    perm = rng.permutation(n_pages)
    table = np.full((C, max_pages), -1)
    at = 0
    for c in range(C):
        table[c, :held[c]] = perm[at:at + held[c]]
        at += held[c]
    free = np.full(n_pages, -3)
    free[:n_pages - at] = perm[at:]
    return ctx, new, held, free, n_pages - at, table


PLANS = [
    # name, requests, longest context, most new tokens, spare pages, rows behind the last token; 4,096 rows or fewer and up to
    # 1,024 requests go in one launch, more requests in rounds of 1,024
    ("one_request_one_token", 1, 0, 1, 0, 0), ("one_request", 1, 500, 8, 3, 5), ("serving", 4, 4096, 8, 0, 32),
    ("sixty_four", 64, 300, 8, 1, 0), ("sixty_five", 65, 300, 70, 1, 100), ("prompts", 9, 0, 700, 0, 3),
    ("prompts_two_launches", 7, 100, 3001, 4, 1), ("thousand", 1000, 900, 8, 9, 0), ("one_round", 1024, 200, 4, 0, 0),
    ("two_rounds", 1025, 200, 4, 2, 17), ("three_rounds_many_rows", 2500, 70, 40, 5, 1000), ("no_new_tokens", 33, 400, 0, 0, 7),
]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("name,C,ctx_hi,new_hi,spare,pad", PLANS, ids=[p[0] for p in PLANS])
def test_plan(name, C, ctx_hi, new_hi, spare, pad, in_place):
    print(f"case plan {name} in_place={in_place}", flush=True)
    rng = np.random.default_rng(C + new_hi)
    state = _state(rng, C, ctx_hi, new_hi, spare)
    p = Plan(*state, max(1, int(state[1].sum()) + pad))
    if in_place:
        p.call()
        want = p.check(name)
    else:
        held, count = torch.full_like(p.held, -9), torch.full_like(p.count, -9)
        for _ in range(2):  # what a call starts from is kept: the second does the same again
            p.call(held, count)
            want = p.check(name, held, count)
        assert np.array_equal(p.held.cpu().numpy(), state[2]) and p.count.item() == state[4]
    assert (want["status"] == 0).all()


@pytest.mark.parametrize("C,rows", [(40, 1000), (40, 5000), (1500, 20000)])
def test_plan_with_requests_that_cannot_be_served(C, rows):
    """Lengths out of range, tables too short, pages held outside what the length allows, page ids outside the pool, rows
    beyond the slot map, a list that runs out."""
    print(f"case plan bad C={C}", flush=True)
    rng = np.random.default_rng(C)
    ctx, new, held, free, count, table = _state(rng, C, 600, 40, 0)
    bad = rng.permutation(C)
    new[bad[0]], ctx[bad[1]], ctx[bad[2]], new[bad[3]] = -5, -1, 64 * table.shape[1] + 1, 64 * table.shape[1]
    new[bad[4]], ctx[bad[4]] = 2**31 - 1, 2**31 - 1
    held[bad[5]] = 0 if ctx[bad[5]] else -1
    held[bad[6]] = table.shape[1] + 1
    table[bad[7], :] = len(free) + 7
    table[bad[8], :] = -4
    ctx[bad[9]], new[bad[9]], held[bad[9]] = 64, 1, 0
    total = int(np.maximum(new, 0).astype(np.int64).sum())
    for left in (count, count // 2, 1, 0, -7, len(free) + 99):
        for max_tokens in (rows, max(1, int(np.maximum(new[:C // 2], 0).astype(np.int64).sum()) % rows)):
            p = Plan(ctx, new, held, free, left, table, max_tokens)
            p.call()
            want = p.check((left, max_tokens))
            assert (want["status"] == 1).sum() >= 6 and total > max_tokens
    assert (want["status"] == 2).any() or left > 0


@pytest.mark.parametrize("C,first_short,ended,pad", [(50, 20, 0.0, 40), (50, 0, 0.0, 6000), (50, 40, 0.05, 40), (1024, 900, 0.1, 0),
                                                     (1500, 600, 0.0, 10), (1500, 1200, 0.0, 10), (2500, 1800, 0.1, 3000), (2500, 2200, 0.0, 10)])
def test_plan_when_the_pages_run_out(C, first_short, ended, pad):
    """The list ends inside the pages that one request lacks, in a launch that writes the slots itself, in two, and in each of
    several rounds of 1,024 requests: that request and all later ones that lack any get none, those that lack none are served."""
    print(f"case plan short C={C} at {first_short}", flush=True)
    rng = np.random.default_rng(C + first_short)
    ctx, new, held, free, count, table = _state(rng, C, 300, 130, 0, ended=ended, rolled_back=0.0)
    still = (rng.random(C) < 0.3) & (ctx > 0) & (ctx % 64 != 0)
    new[still] = 1                                        # lacks no page
    lacks, given = np.maximum(_pages(ctx + new) - held, 0), int(np.maximum(held - _pages(ctx + new), 0).sum())
    f = next(c for c in range(first_short, C) if lacks[c] > 0)
    there = int(lacks[:f].sum()) + int(lacks[f]) - 1 - given
    assert 0 <= there < count
    p = Plan(ctx, new, held, free, there, table, int(new.sum()) + pad)
    p.call()
    want = p.check((C, f))
    assert (want["status"][:f] == 0).all() and want["status"][f] == 2
    assert ((want["status"] == 2) == ((lacks > 0) & (np.arange(C) >= f))).all() and (want["status"][f + 1:] == 0).any()
    assert want["free_count"][0] == lacks[f] - 1


def test_plan_over_the_life_of_a_batch():
    """Admission, steps with accepted and rejected drafts, ends: the pool's pages are at every moment either held or free, each
    once, and when all requests have ended the list holds all of them."""
    print("case plan life", flush=True)
    rng = np.random.default_rng(9)
    C, n_pages, cols = 20, 150, 12
    ctx, held, table = np.zeros(C, int), np.zeros(C, int), np.full((C, cols), -1)
    free, count = rng.permutation(n_pages), n_pages
    p = Plan(ctx, np.zeros(C, int), held, free, count, table, 4000)
    for step in range(12):
        new = rng.integers(1, 200, C) if step == 0 else rng.integers(1, 9, C) if step < 11 else np.zeros(C, int)
        if 4 <= step < 11:
            over = rng.random(C) < 0.2
            ctx[over] = 0
            new[over] = rng.integers(0, 2, int(over.sum())) * 100
        if step == 11:
            ctx[:] = 0
        p.ctx.copy_(torch.from_numpy(ctx.astype(np.int32)))
        p.new.copy_(torch.from_numpy(new.astype(np.int32)))
        p.host = [ctx.copy(), new, p.held.cpu().numpy(), p.free.cpu().numpy(), p.count.item(), p.table.cpu().numpy(), 4000]
        p.call()
        want = p.check(step)
        assert (want["status"] == 0).all()
        in_use = [x for c in range(C) for x in want["block_table"][c, :want["pages_held"][c]]]
        assert sorted(in_use + want["free_pages"][:want["free_count"][0]].tolist()) == list(range(n_pages))
        ctx = np.maximum(want["seq_len"] - rng.integers(0, 5, C) * (new > 4) * (step < 11), 0)
    assert want["free_count"][0] == n_pages


def test_plan_replays_from_a_graph():
    print("case plan graph", flush=True)
    rng = np.random.default_rng(3)
    state = _state(rng, 30, 500, 8, 40)
    for rows in (300, 6000):  # one launch, two
        p = Plan(*state, rows)
        p.call()
        start = [x.clone() for x in (p.held, p.free, p.count, p.table)]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            p.call()
        for rep in range(4):
            new = np.minimum(rng.integers(0, 9, 30), 64 * p.shape.max_pages - state[0])
            for x, y in zip((p.held, p.free, p.count, p.table), start):
                x.copy_(y)
            p.new.copy_(torch.from_numpy(new.astype(np.int32)))
            p.host = [state[0], new] + [x.cpu().numpy() for x in start[:2]] + [start[2].item(), start[3].cpu().numpy(), rows]
            graph.replay()
            p.check(("replay", rep))


@pytest.mark.parametrize("C,ctx_hi,new_hi,pad", [(5, 300, 9, 3), (70, 900, 8, 700), (1100, 300, 8, 9001)])
def test_plan_stays_inside_its_buffers(C, ctx_hi, new_hi, pad):
    print(f"case plan guards C={C}", flush=True)
    rng = np.random.default_rng(C)
    state = _state(rng, C, ctx_hi, new_hi, 1, extra_columns=1)  # (a request may hold one page more than it needs)
    p = Plan(*state, int(state[1].sum()) + pad)
    g = Guarded()
    for name in ("held", "free", "table", "count", "start", "seq_len", "status", "slots", "ws"):
        x = getattr(p, name)
        setattr(p, name, g.tensor(name, tuple(x.shape), x.dtype).copy_(x))
    p.call()
    g.check("plan")
    p.check("guards")


def test_plans_on_two_streams_at_once():
    """Two pools with workspaces of their own, on streams of their own: neither call sees the other's."""
    print("case plans on two streams", flush=True)
    rng = np.random.default_rng(77)
    plans = []
    for C in (300, 1300):
        state = _state(rng, C, 500, 20, 5)
        plans.append(Plan(*state, int(state[1].sum()) + 100))
    torch.cuda.synchronize()
    for p, stream in zip(plans, (torch.cuda.Stream(), torch.cuda.Stream())):
        with torch.cuda.stream(stream):
            p.call()
    for i, p in enumerate(plans):
        p.check(i)


# -------------------------------------------------------------------------------------------------------- append

class Cache:
    """A cache whose places hold arbitrary finite values, its 64-bit image, and the call."""

    def __init__(self, rng, n_pages, Hkv, D, fmt, exps=(-8, 4)):
        self.fmt, self.Hkv, self.D, self.n_pages = fmt, Hkv, D, n_pages
        codes = torch.from_numpy(rng.integers(0, 256, (2, n_pages, Hkv, 64, D), dtype=np.uint8))
        values = codes.view(TYPES[fmt]).double()
        codes = torch.where(torch.isfinite(values), codes.int(), 0).to(torch.uint8)
        self.pages = [c.contiguous().cuda().view(TYPES[fmt]) for c in codes]
        self.exps = [rng.integers(*exps, (n_pages, Hkv)) for _ in range(2)]
        self.scales = [torch.from_numpy((e + 127).astype(np.uint8)).cuda().view(E8M0) for e in self.exps]
        self.values = [p.double().cpu().numpy() for p in self.pages]

    def append(self, k, v, slots):
        shape = pe.CacheShape(k.shape[0], self.Hkv, self.D, self.n_pages)
        pe.peagle_cache_append_scaled(shape, k, v, torch.from_numpy(np.asarray(slots, dtype=np.int64)).cuda(), *self.pages, *self.scales)
        for x, values, exps in zip((k, v), self.values, self.exps):
            orc.cache_append(bf16_to_f64(x.contiguous()), slots, values, exps, self.fmt)

    def check(self, what):
        torch.cuda.synchronize()
        for i, n in enumerate("kv"):
            assert np.array_equal(self.scales[i].view(torch.uint8).cpu().numpy().astype(int) - 127, self.exps[i]), (what, n, "scale")
            assert np.array_equal(self.pages[i].double().cpu().numpy(), self.values[i], equal_nan=True), (what, n)


def _rand(g, *shape, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(torch.bfloat16)


def _slots(rng, n_pages, runs):
    """Slots of runs (place, tokens) in pages of their own, in any order."""
    pages = rng.permutation(n_pages)[:len(runs)]
    return np.concatenate([p * 64 + at + np.arange(n) for p, (at, n) in zip(pages, runs)])


RUNS = [
    ("one_token", [(0, 1)]), ("one_token_inside", [(37, 1)]), ("last_place", [(63, 1)]), ("a_page", [(0, 64)]),
    ("all_but_one", [(1, 63)]), ("pages", [(0, 64)] * 9 + [(0, 5)]), ("steps", [(5, 7), (60, 4), (0, 3), (62, 2), (63, 1), (1, 8), (16, 16)]),
    ("ragged", [(40, 24), (0, 64), (0, 64), (0, 11), (0, 33), (7, 57), (0, 64), (0, 1)]), ("many", [(i % 64, 1) for i in range(200)]),
]


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("Hkv,D", [(1, 64), (8, 64), (3, 128), (4, 128)])
@pytest.mark.parametrize("name,runs", RUNS, ids=[r[0] for r in RUNS])
def test_append(name, runs, Hkv, D, fmt):
    print(f"case append {name} Hkv={Hkv} D={D} {fmt}", flush=True)
    rng = np.random.default_rng(len(runs) + D + Hkv)
    g = torch.Generator(device="cuda").manual_seed(len(runs) + Hkv)
    cache = Cache(rng, max(len(runs), 4) + 3, Hkv, D, fmt)
    for scale in (1.0, 300.0, 1e-3):  # the second call's values make every scale grow, the third's none
        slots = _slots(rng, cache.n_pages, runs)
        cache.append(_rand(g, len(slots), Hkv, D, scale=scale), _rand(g, len(slots), Hkv, D, scale=7 * scale), slots)
        cache.check((name, scale))


@pytest.mark.parametrize("n_tokens,C,Hkv,D", [(3891, 1, 8, 64), (9000, 5, 4, 128), (40000, 3, 8, 64), (1500, 700, 8, 128)])
def test_append_of_many_tokens(n_tokens, C, Hkv, D):
    """Enough tokens for each number of tokens that a wave may look through, for requests at any place of a page."""
    print(f"case append many {n_tokens} C={C} Hkv={Hkv} D={D}", flush=True)
    rng = np.random.default_rng(n_tokens)
    g = torch.Generator(device="cuda").manual_seed(n_tokens)
    new = rng.multinomial(n_tokens, np.ones(C) / C)
    ctx = rng.integers(0, 64, C)
    pages = _pages(ctx + new)
    perm = rng.permutation(int(pages.sum()))
    first = np.concatenate([[0], np.cumsum(pages)])
    slots = np.concatenate([perm[first[c] + (ctx[c] + np.arange(new[c])) // 64] * 64 + (ctx[c] + np.arange(new[c])) % 64 for c in range(C)])
    cache = Cache(rng, int(pages.sum()), Hkv, D, "e4m3")
    cache.append(_rand(g, n_tokens, Hkv, D, scale=3), _rand(g, n_tokens, Hkv, D), slots)
    cache.check(n_tokens)


def test_append_finds_few_slots_among_many_tokens():
    """More tokens than one dimension of the launch holds workgroups for; slots in the first, the middle and the last of them."""
    n = 32768 * 256 + 1000
    print(f"case append few of {n}", flush=True)
    rng = np.random.default_rng(5)
    g = torch.Generator(device="cuda").manual_seed(5)
    cache = Cache(rng, 9, 1, 64, "e4m3")
    k, v = _rand(g, n, 1, 64), _rand(g, n, 1, 64)
    at = np.concatenate([np.arange(70), n // 2 + np.arange(130), n - 90 + np.arange(90)])
    places = np.concatenate([7 * 64 + 5 + np.arange(59), 0 * 64 + np.arange(11), 3 * 64 + np.arange(64), 4 * 64 + np.arange(64), 2 * 64 + np.arange(2),
                             5 * 64 + np.arange(64), 6 * 64 + np.arange(26)])
    slots = np.full(n, -1, dtype=np.int64)
    slots[at] = places
    pe.peagle_cache_append_scaled(pe.CacheShape(n, 1, 64, 9), k, v, torch.from_numpy(slots).cuda(), *cache.pages, *cache.scales)
    rows = torch.from_numpy(at).cuda()
    for x, values, exps in zip((k, v), cache.values, cache.exps):
        orc.cache_append(bf16_to_f64(x[rows]), places, values, exps, "e4m3")
    cache.check("few of many")


@pytest.mark.parametrize("Hkv,D,n_tokens", [(1, 64, 1), (3, 128, 77), (2, 64, 700)])
def test_append_stays_inside_its_buffers(Hkv, D, n_tokens):
    print(f"case append guards Hkv={Hkv} D={D}", flush=True)
    rng = np.random.default_rng(n_tokens)
    gen = torch.Generator(device="cuda").manual_seed(n_tokens)
    cache = Cache(rng, -(-n_tokens // 64) + 1, Hkv, D, "e5m2")
    g = Guarded()
    cache.pages = [g.tensor(f"pages {i}", tuple(x.shape), x.dtype).copy_(x) for i, x in enumerate(cache.pages)]
    cache.scales = [g.tensor(f"scales {i}", tuple(x.shape), torch.uint8).copy_(x.view(torch.uint8)).view(E8M0) for i, x in enumerate(cache.scales)]
    last = cache.n_pages * 64
    slots = np.arange(last - n_tokens, last)
    cache.append(_rand(gen, n_tokens, Hkv, D, scale=50), _rand(gen, n_tokens, Hkv, D), slots)
    g.check("append")
    cache.check("guards")


def test_append_skips_tokens_without_a_slot():
    """Padding (-1) at both ends and between, slots outside the pool; what stands behind a gap in the slots is another run."""
    print("case append skips", flush=True)
    rng, g = np.random.default_rng(5), torch.Generator(device="cuda").manual_seed(5)
    cache = Cache(rng, 6, 2, 64, "e4m3")
    slots = np.array([-1, -1, 64, 65, 66, -1, 130, -1, 6 * 64, 6 * 64 + 1, 2**40, -2**40, 0, 1, 3 * 64 + 62, 3 * 64 + 63, 4 * 64, -1, -1])
    cache.append(_rand(g, len(slots), 2, 64), _rand(g, len(slots), 2, 64), slots)
    cache.check("skips")
    cache.append(_rand(g, 3, 2, 64), _rand(g, 3, 2, 64), np.array([-1, -1, -1]))
    cache.check("nothing")
    cache.append(_rand(g, 0, 2, 64), _rand(g, 0, 2, 64), np.zeros(0))
    cache.check("no tokens")


def test_append_of_rows_of_a_fused_projection():
    """K and V are views of wider rows; a distance between tokens that no whole number of heads makes."""
    print("case append strides", flush=True)
    rng, g = np.random.default_rng(6), torch.Generator(device="cuda").manual_seed(6)
    for D, width in ((64, 64 * 20), (128, 128 * 9 + 8)):
        cache = Cache(rng, 9, 3, D, "e5m2")
        rows = _rand(g, 150, width)
        k, v = rows[:, 2 * D:5 * D].unflatten(1, (3, D)), rows[:, 5 * D + 8:8 * D + 8].unflatten(1, (3, D))
        assert not k.is_contiguous()
        cache.append(k, v, np.concatenate([128 + 30 + np.arange(34), np.arange(64), 320 + np.arange(52)]))
        cache.check(D)
    with pytest.raises(ValueError, match="contiguous"):
        pe.peagle_cache_append_scaled(pe.CacheShape(4, 2, 64, 9), rows[:4, :128].view(4, 64, 2).transpose(1, 2), rows[:4, :128].unflatten(1, (2, 64)),
                                      torch.zeros(4, dtype=torch.int64, device="cuda"), *Cache(rng, 9, 2, 64, "e4m3").pages,
                                      *Cache(rng, 9, 2, 64, "e4m3").scales)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_append_of_values_at_the_edges(fmt):
    """Zeros, the largest and smallest bf16 values, values next to a change of scale, halfway cases, infinities and NaN, alone
    in their page, beside ordinary values, and added to a page that holds them."""
    print(f"case append edges {fmt}", flush=True)
    rng = np.random.default_rng(7)
    top = orc.F8[fmt][2]
    big = 3.3895313892515355e38
    rows = [[0.0], [-0.0, 0.0], [big, -big], [2.0**-126, -2.0**-126], [2.0**-133, 2.0**-100], [top, -1.0], [top * 1.0078125, 1.0], [top * 2, 0.5],
            [np.inf, 1.0], [-np.inf, np.nan], [np.nan], [17.0, 19.0, 18.0, 448.0], [2.0**-9, 2.0**-10, 3 * 2.0**-10, 3 * 2.0**-11, 448.0, 2.0**-16, 2.0**-17],
            [1e-30, 2e-30], [np.inf, big], [2.0**-92, 2.0**-110, 448 * 2.0**-100]]
    x = torch.zeros(len(rows), 1, 64)
    for i, r in enumerate(rows):
        x[i, 0] = torch.tensor(r, dtype=torch.float64).repeat(64)[:64].float()
    x = x.to(torch.bfloat16).cuda()
    cache = Cache(rng, len(rows), 1, 64, fmt)
    at = np.arange(len(rows)) * 64
    cache.append(x, x.flip(0), at)
    cache.check("alone")
    for step in range(1, 5):
        cache.append(x.roll(step, 0), x.roll(-step, 0), at + step)
        cache.check(("added", step))


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_append_behind_the_largest_scales(fmt):
    """Pages from elsewhere whose scales are above what an append makes: kept, with the new values rounded to them; behind the codes
    254 and 255 finite values become zeros and others NaN."""
    print(f"case append large scales {fmt}", flush=True)
    rng, big = np.random.default_rng(14), 3.3895313892515355e38
    x = torch.tensor([big, -big, 1.5 * 2.0**120, 2.0**112, 1.0, 0.0, float("nan"), float("inf")]).repeat(8)[None, None].to(torch.bfloat16).cuda()
    for e in range(121, 127):                                  # codes 248 to 253
        cache = Cache(rng, 2, 1, 64, fmt, exps=(e, e + 1))
        cache.append(x, x.flip(2), [64 + 5])
        cache.check(e)
        assert (cache.exps[0] == e).all()
    for e in (127, 128):                                       # codes 254, 255
        cache = Cache(rng, 2, 1, 64, fmt, exps=(e, e + 1))
        pe.peagle_cache_append_scaled(pe.CacheShape(1, 1, 64, 2), x, x, torch.tensor([64 + 5], device="cuda"), *cache.pages, *cache.scales)
        for values in cache.values:
            values[1, 0, 5] = np.where(np.isfinite(bf16_to_f64(x)[0, 0]), 0.0, np.nan)
        cache.check(e)


def test_append_adds_one_token_at_a_time():
    """A page filled by 64 calls with values that grow and shrink: the scale only grows, what is held is rounded again."""
    print("case append token by token", flush=True)
    for fmt in ("e4m3", "e5m2"):
        rng, g = np.random.default_rng(8), torch.Generator(device="cuda").manual_seed(8)
        cache = Cache(rng, 3, 2, 128, fmt)
        for i in range(64):
            size = float(np.exp2(rng.uniform(-6, 6)))
            cache.append(_rand(g, 1, 2, 128, scale=size), _rand(g, 1, 2, 128, scale=1 / size), np.array([64 + i]))
            if i % 9 == 0 or i == 63:
                cache.check((fmt, i))


def test_append_replays_from_a_graph():
    print("case append graph", flush=True)
    rng, g = np.random.default_rng(10), torch.Generator(device="cuda").manual_seed(10)
    cache = Cache(rng, 12, 4, 64, "e4m3")
    runs = [(0, 64), (9, 8), (0, 3)]
    n = sum(r[1] for r in runs)
    k, v = _rand(g, n, 4, 64), _rand(g, n, 4, 64)
    slots = torch.empty(n, dtype=torch.int64, device="cuda")
    shape = pe.CacheShape(n, 4, 64, 12)
    slots.copy_(torch.from_numpy(_slots(rng, 12, runs)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        pe.peagle_cache_append_scaled(shape, k, v, slots, *cache.pages, *cache.scales)
    for rep in range(4):
        at = _slots(rng, 12, runs)
        k.copy_(_rand(g, n, 4, 64, scale=rep + 1))
        v.copy_(_rand(g, n, 4, 64))
        slots.copy_(torch.from_numpy(at))
        graph.replay()
        for x, values, exps in zip((k, v), cache.values, cache.exps):
            orc.cache_append(bf16_to_f64(x), at, values, exps, "e4m3")
        cache.check(rep)


def test_append_beyond_four_gigabytes():
    """Pools of 4.3 GB: pages and scales on both sides of byte 2^32."""
    print("case append beyond 2^32", flush=True)
    Hkv, D = 8, 128
    per_page = Hkv * 64 * D
    n_pages = 2**32 // per_page + 3
    g = torch.Generator(device="cuda").manual_seed(12)
    pages = [torch.zeros((n_pages, Hkv, 64, D), dtype=torch.uint8, device="cuda").view(TYPES["e4m3"]) for _ in range(2)]
    scales = [torch.full((n_pages, Hkv), 9, dtype=torch.uint8, device="cuda").view(E8M0) for _ in range(2)]
    k, v = _rand(g, 130, Hkv, D), _rand(g, 130, Hkv, D)
    where = [n_pages - 1, 0, n_pages - 4]
    slots = np.concatenate([where[0] * 64 + np.arange(64), where[1] * 64 + np.arange(64), where[2] * 64 + np.arange(2)])
    pe.peagle_cache_append_scaled(pe.CacheShape(130, Hkv, D, n_pages), k, v, torch.from_numpy(slots).cuda(), *pages, *scales)
    torch.cuda.synchronize()
    for x, p, s in zip((k, v), pages, scales):
        values, exps = np.zeros((3, Hkv, 64, D)), np.zeros((3, Hkv), dtype=int)
        orc.cache_append(bf16_to_f64(x), np.concatenate([np.arange(64), 64 + np.arange(64), 128 + np.arange(2)]), values, exps, "e4m3")
        at = torch.tensor(where, device="cuda")
        assert np.array_equal(p.view(torch.uint8)[at].view(TYPES["e4m3"]).double().cpu().numpy(), values)
        assert np.array_equal(s.view(torch.uint8)[at].cpu().numpy().astype(int) - 127, exps)
        others = torch.ones(n_pages, dtype=torch.bool, device="cuda")
        others[at] = False
        assert bool((s.view(torch.uint8)[others] == 9).all())
        assert int(p.view(torch.uint8).view(torch.int64).ne(0).sum()) <= 130 * Hkv * D // 8
