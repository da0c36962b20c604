"""GPU tests of the drafting step on a paged cache held in 8 bits, against the 64-bit oracle on the values that the cache stands
for.  Tolerances: what the cache holds is exact in bf16, so that the arithmetic's roundings are those of the probabilities and of
the output (half a step of bf16 each, 2^-9 relative: O rel-L2 at most 2 * 2^-9 < 5e-3, elements as in the bf16 step's tests) and fp32
sums (scores of D products: D * 2^-24 of sum |q k| scale, below 1e-3 for the inputs here, which bounds the LSE's error too)."""
import numpy as np
import pytest
import torch

import paper_2602_01469_amd as pe
from gpu_harness import bf16_to_f64, max_abs, rel_l2, to_dev_bf16
from oracle import peagle_oracle as orc
from peagle_inputs import bf16_bits_to_f64, f32_to_bf16_bits
from test_gpu_guards import Guarded
from test_gpu_parity import _check_o_abs

pytestmark = pytest.mark.gpu

TYPES = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
E8M0 = torch.float8_e8m0fnu
REL, LSE_ABS = 5e-3, 1e-3


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _cache(x, fmt, rng):
    """8-bit pages and scale codes for x [n_pages, Hkv, 64, D] (float32), some scales larger than they have to be."""
    amax = np.abs(x).max((2, 3))
    e = np.ceil(np.log2(amax / orc.F8[fmt][2])).astype(int)
    e += amax > orc.F8[fmt][2] * np.exp2(e)
    e += rng.integers(0, 3, e.shape)
    return torch.from_numpy(x * np.exp2(-e)[..., None, None].astype(np.float32)).to(TYPES[fmt]), torch.from_numpy((e + 127).astype(np.uint8))


class ScaledRun:
    """Inputs of one drafting step on a shuffled pool: unused places hold NaN, unused pages' scales too, unused table entries -1.
    shared: that many pages that all requests use in any order, for long contexts in a small pool."""

    def __init__(self, ctx_lens, K, Hq, Hkv, D, fmt, seed, shared=0, scale=None, spare=3, gain=1.0):
        rng = np.random.default_rng(seed)
        C = len(ctx_lens)
        pages_of = [-(-n // 64) for n in ctx_lens]
        max_pages = max(1, max(pages_of))
        used = shared or sum(pages_of)
        n_pages = max(1, used + spare)
        perm = rng.permutation(n_pages)
        x = rng.standard_normal((2, n_pages, Hkv, 64, D), dtype=np.float32)
        x[0] *= np.where(rng.random(D) < 0.05, 4.0, 1.0).astype(np.float32) * gain
        table = np.full((C, max_pages), -1, dtype=np.int32)
        at = 0
        for c, n in enumerate(pages_of):
            table[c, :n] = rng.choice(perm[:shared], n) if shared else perm[at:at + n]
            at += n
        self.pages, self.scales = [], []
        for i in range(2):
            codes, scales = _cache(x[i], fmt, rng)
            raw = codes.view(torch.uint8)
            if not shared:
                for c, n in enumerate(ctx_lens):
                    if n % 64:
                        raw[table[c, n // 64], :, n % 64:] = 0x7F  # NaN of either type
                raw[torch.from_numpy(perm[used:])] = 0x7F
                scales[torch.from_numpy(perm[used:])] = 255
            self.pages.append(codes.cuda())
            self.scales.append(scales.cuda().view(E8M0))
        bits = lambda *shape: f32_to_bf16_bits(rng.standard_normal(shape, dtype=np.float32))
        self.host = [bits(C, K, Hq, D), bits(C, K, Hkv, D), bits(C, K, Hkv, D)]
        self.table, self.lens = table, list(ctx_lens)
        self.shape = pe.DecodeShape(C, K, Hq, Hkv, D, n_pages, max_pages, scale)
        self.q, self.k, self.v = (to_dev_bf16(x) for x in self.host)
        self.bt, self.cl = torch.from_numpy(table).cuda(), torch.tensor(ctx_lens, dtype=torch.int32, device="cuda")
        self.o = torch.full((C, K, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full((C, Hq, K), float("nan"), device="cuda")
        self.status = torch.full((C,), -7, dtype=torch.int32, device="cuda")
        self.ws = torch.empty(pe.peagle_draft_decode_scaled_workspace_bytes(self.shape), dtype=torch.uint8, device="cuda").fill_(0x7F)

    def call(self, stream=None):
        pe.peagle_draft_decode_scaled(self.shape, self.q, self.k, self.v, *self.pages, *self.scales, self.bt, self.cl, self.o, self.lse,
                                      self.status, self.ws, stream)

    def run(self):
        self.call()
        torch.cuda.synchronize()
        return bf16_to_f64(self.o), self.lse.double().cpu().numpy(), self.status.cpu().numpy()

    def context(self, c):
        n = self.lens[c]
        pages = torch.from_numpy(self.table[c, :-(-n // 64)].astype(np.int64)).cuda()
        out = []
        for p, s in zip(self.pages, self.scales):
            x = p.view(torch.uint8)[pages].view(p.dtype).double() * s.view(torch.uint8)[pages].view(E8M0).double()[..., None, None]
            out.append(x.transpose(1, 2).reshape(-1, p.shape[1], p.shape[3])[:n].cpu().numpy())
        return out

    def oracle(self, c):
        k, v = self.context(c)
        return orc.draft_decode(*(bf16_bits_to_f64(x[c]) for x in self.host), k, v, self.shape.scale)

    def check(self, o, lse, what, requests=None):
        for c in range(len(self.lens)) if requests is None else requests:
            ro, rl = self.oracle(c)
            assert np.isfinite(o[c]).all() and np.isfinite(lse[c]).all(), (what, c)
            assert rel_l2(o[c], ro) <= REL, (what, c, rel_l2(o[c], ro))
            _check_o_abs(o[c], ro, f"{what} request {c}")
            assert max_abs(lse[c], rl) <= LSE_ABS, (what, c, max_abs(lse[c], rl))


CASES = [
    # name, contexts, K, Hq, Hkv, D; rows K * Hq / Hkv of one to four blocks of 32
    ("one_token", (77,), 1, 64, 8, 64), ("no_context", (0,), 1, 4, 4, 128), ("one_key", (1,), 1, 1, 1, 64), ("empty_and_short", (0, 1, 0), 5, 8, 2, 64),
    ("page_edges", (0, 1, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 192, 193), 4, 8, 2, 64),
    ("page_edges_d128", (0, 1, 31, 32, 33, 63, 64, 65, 95, 96, 97, 127, 128, 129, 191, 192, 193), 4, 8, 2, 128),
    ("paper_k7", (900, 1500, 333, 2048), 7, 64, 8, 64), ("paper_k3_d128", (513, 1200), 3, 32, 4, 128), ("paper_k7_d128", (1000, 257, 5), 7, 32, 4, 128),
    ("odd_group", (300, 1000), 7, 9, 3, 64), ("odd_group_d128", (300, 1000), 7, 9, 3, 128),
    ("three_blocks", (400, 70, 0), 6, 32, 2, 64), ("three_blocks_d128", (400, 70, 0), 6, 32, 2, 128),
    ("four_blocks", (300, 10, 64), 8, 16, 1, 64), ("four_blocks_d128", (300, 10, 64), 8, 16, 1, 128),
    ("most_new_keys", (130, 0), 64, 4, 2, 64), ("most_new_keys_d128", (130, 0), 64, 2, 1, 128), ("thirty_three_new_keys", (200,), 33, 3, 1, 64),
    ("seventeen_new_keys_d128", (64,), 17, 2, 2, 128), ("long", (20000, 4096), 7, 64, 8, 64), ("long_d128", (10800, 20000), 5, 32, 4, 128),
    ("mixed_batch", (2371, 0, 77, 1257, 1000, 64, 192, 3, 4097, 129, 0, 600, 384, 511, 2048, 65), 5, 32, 8, 64),
]


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("name,ctx_lens,K,Hq,Hkv,D", CASES, ids=[c[0] for c in CASES])
def test_draft_scaled_matches_oracle(name, ctx_lens, K, Hq, Hkv, D, fmt):
    print(f"case scaled {name} {fmt}", flush=True)
    r = ScaledRun(ctx_lens, K, Hq, Hkv, D, fmt, 3000 + len(name))
    o, lse, status = r.run()
    assert (status == 0).all()
    r.check(o, lse, name)
    o2, lse2, _ = r.run()
    assert np.array_equal(o, o2) and np.array_equal(lse, lse2)


@pytest.mark.parametrize("C,ctx,K,Hq,Hkv,D", [(64, 20000, 2, 16, 8, 64), (64, 5000, 8, 128, 8, 128), (130, 9000, 4, 64, 4, 64),
                                              (256, 500, 7, 16, 2, 64), (70, 2000, 4, 8, 8, 128)])
def test_draft_scaled_batches_on_a_shared_pool(C, ctx, K, Hq, Hkv, D):
    """Many requests whose tables point into a few pages: one piece a request and more, more than 64 pages for a wave, unequal
    lengths; a few of them against the oracle.  Then one request's table is spoiled: it alone is flagged and changes."""
    rng = np.random.default_rng(C)
    lens = rng.integers(0, ctx, C)
    lens[3] = ctx
    print(f"case scaled batch C={C} ctx={ctx} D={D}", flush=True)
    r = ScaledRun(tuple(int(x) for x in lens), K, Hq, Hkv, D, "e4m3", C, shared=40)
    o, lse, status = r.run()
    assert (status == 0).all()
    r.check(o, lse, "batch", (0, 3, C // 2, C - 1))
    spoiled = 3
    r.bt[spoiled, 1] = r.shape.n_pages
    o2, lse2, status2 = r.run()
    others = np.arange(C) != spoiled
    assert status2[spoiled] == 1 and (status2[others] == 0).all()
    assert np.array_equal(o2[others], o[others]) and np.array_equal(lse2[others], lse[others]) and np.isfinite(o2).all()


@pytest.mark.parametrize("C,ctx,K,Hq,Hkv,D", [(70, 900, 7, 32, 4, 64), (130, 5000, 4, 64, 4, 64), (100, 2500, 7, 24, 4, 128), (40, 1500, 16, 64, 8, 64),
                                              (40, 6000, 4, 256, 8, 64), (64, 5000, 3, 16, 8, 128), (64, 4000, 8, 64, 4, 128), (40, 1500, 3, 32, 4, 128),
                                              (50, 2000, 7, 32, 4, 128), (33, 1900, 16, 32, 4, 128)])
def test_draft_scaled_batches_in_e5m2(C, ctx, K, Hq, Hkv, D):
    """More workgroups than compute units, by request and in shares: two to four blocks of rows."""
    rng = np.random.default_rng(C + ctx)
    lens = rng.integers(0, ctx, C)
    lens[C // 3] = ctx
    lens[C // 2] = 0
    print(f"case scaled e5m2 batch C={C} ctx={ctx} D={D}", flush=True)
    r = ScaledRun(tuple(int(x) for x in lens), K, Hq, Hkv, D, "e5m2", C, shared=50)
    o, lse, status = r.run()
    assert (status == 0).all()
    r.check(o, lse, "batch", (0, C // 3, C // 2, C - 1))
    o2, lse2, _ = r.run()
    assert np.array_equal(o, o2) and np.array_equal(lse, lse2)


@pytest.mark.parametrize("D", [64, 128])
def test_draft_scaled_flags_bad_tables_and_lengths(D):
    """Page ids on both sides of the pool, lengths below zero and beyond the table: flagged, skipped or clamped as the bf16
    step does, the other requests exact."""
    print(f"case scaled bad tables D={D}", flush=True)
    r = ScaledRun((300, 200, 100, 130, 64), 3, 8, 2, D, "e5m2", 3100)
    good = r.run()
    r.bt[1, 2] = r.shape.n_pages + 5
    r.bt[3, 0] = -2**31
    r.cl[2] = 64 * r.shape.max_pages + 1
    r.bt[2, :] = r.bt[2, 0].clone()
    r.cl[4] = -3
    o, lse, status = r.run()
    assert status.tolist() == [0, 1, 1, 1, 1] and np.array_equal(o[0], good[0][0]) and np.array_equal(lse[0], good[1][0])
    assert np.isfinite(lse[1:]).all()
    k, v = r.context(1)                                       # (request 1: without the bad page's keys)
    ro, rl = orc.draft_decode(*(bf16_bits_to_f64(x[1]) for x in r.host), np.delete(k, slice(128, 192), 0), np.delete(v, slice(128, 192), 0), r.shape.scale)
    assert rel_l2(o[1], ro) <= REL and max_abs(lse[1], rl) <= LSE_ABS
    ro, rl = orc.draft_decode(*(bf16_bits_to_f64(x[4]) for x in r.host), k[:0], v[:0], r.shape.scale)
    assert rel_l2(o[4], ro) <= REL and max_abs(lse[4], rl) <= LSE_ABS


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("K", [5, 40])
def test_draft_scaled_keeps_masked_values_out(K, D):
    """NaN and infinities in the keys and values of new positions that a row does not see leave the row as it is, bit for
    bit; rows that see them show them."""
    print(f"case scaled masked NaN K={K} D={D}", flush=True)
    r = ScaledRun((150, 0), K, 6, 2, D, "e4m3", 3200)
    clean, clean_lse, _ = r.run()
    at = K - 2
    r.k[0, at, 0, 3], r.v[0, at, 1, 5] = float("nan"), float("inf")
    r.v[1, at, 0, 7], r.v[1, at + 1, 1, D - 1] = float("nan"), -float("inf")
    o, lse, _ = r.run()
    assert np.array_equal(o[:, :at], clean[:, :at]) and np.array_equal(lse[:, :, :at], clean_lse[:, :, :at])
    assert np.isnan(o[0, at:, :3]).all() and np.isnan(lse[0, :3, at:]).all()          # heads 0..2 use KV head 0
    assert np.isposinf(o[0, at:, 3:, 5]).all() and np.isfinite(np.delete(o[0, at:, 3:], 5, 2)).all() and np.isfinite(lse[0, 3:]).all()
    assert np.isnan(o[1, at:, :3, 7]).all() and np.isfinite(np.delete(o[1, :, :3], 7, 2)).all()
    assert np.isneginf(o[1, at + 1, 3:, D - 1]).all() and np.isfinite(o[1, at, 3:]).all()


def test_draft_scaled_shows_nan_that_the_cache_holds():
    print("case scaled NaN in the cache", flush=True)
    r = ScaledRun((100, 100, 100), 2, 4, 2, 64, "e4m3", 3300)
    clean, _, _ = r.run()
    page = int(r.table[1, 0])
    r.pages[1].view(torch.uint8)[page, 1, 10, 20] = 0x7F
    r.scales[0].view(torch.uint8)[int(r.table[2, 1]), 0] = 255
    o, lse, status = r.run()
    assert (status == 0).all() and np.array_equal(o[0], clean[0])
    assert np.isnan(o[1, :, 2:, 20]).all() and np.isfinite(np.delete(o[1, :, 2:], 20, 2)).all() and np.array_equal(o[1, :, :2], clean[1, :, :2])
    assert np.isnan(o[2, :, :2]).all() and np.isnan(lse[2, :2]).all() and np.array_equal(o[2, :, 2:], clean[2, :, 2:])


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("D", [64, 128])
def test_draft_scaled_reads_every_code_and_scale(D, fmt):
    """Keys of zero weigh all values alike: each output is the mean of one feature's codes.  Every finite code stands in every
    feature's column once, with scales far apart from page to page and head to head."""
    print(f"case scaled codes D={D} {fmt}", flush=True)
    every = np.arange(256, dtype=np.uint8)
    every = every[np.isfinite(torch.from_numpy(every).view(TYPES[fmt]).double().numpy())]
    n, Hkv = len(every), 2
    r = ScaledRun((n,), 1, 2, Hkv, D, fmt, 3400, spare=0)
    for codes in ([127, 127, 127, 127], [100, 140, 110, 130], [30, 27, 33, 29], [220, 190, 221, 200]):
        raw = torch.from_numpy(np.resize(every, 256)).view(4, 64)
        for b in range(4):
            r.pages[0].view(torch.uint8)[int(r.table[0, b])] = 0
            for d in range(D):
                r.pages[1].view(torch.uint8)[int(r.table[0, b]), :, :, d] = raw.roll(d, 1)[b].cuda()
            r.scales[1].view(torch.uint8)[int(r.table[0, b])] = torch.tensor([codes[b], codes[b] + 1], dtype=torch.uint8).cuda()
        r.k.zero_()
        r.v.zero_()
        r.host[1][:], r.host[2][:] = 0, 0
        o, lse, _ = r.run()
        ro, rl = r.oracle(0)
        size = np.abs(r.context(0)[1]).mean(0)                # [Hkv, D]: what the mean's terms add up to
        # fp32 sums of 255 terms and one rounding to bf16 (a probability of 1 is exact)
        assert (np.abs(o[0, 0] - ro[0]) <= 2.0**-8 * np.abs(ro[0]) + 2.0**-15 * size).all()
        assert max_abs(lse, rl) <= 1e-5


def test_draft_scaled_large_logits():
    print("case scaled large logits", flush=True)
    for D in (64, 128):
        r = ScaledRun((700, 90), 5, 16, 2, D, "e4m3", 3500, gain=8.0)
        o, lse, status = r.run()
        for c in range(2):
            ro, rl = r.oracle(c)
            assert rel_l2(o[c], ro) <= REL and max_abs(lse[c], rl) <= 8 * LSE_ABS and (status == 0).all()


def test_draft_scaled_equals_the_bf16_step_on_the_same_values():
    """The values that the cache stands for are bf16 numbers: both steps on them agree to their roundings of probabilities and
    outputs (two of 2^-9 each)."""
    print("case scaled against bf16", flush=True)
    for D, Hq, Hkv in ((64, 64, 8), (128, 32, 4)):
        r = ScaledRun((1000, 64, 333, 0), 7, Hq, Hkv, D, "e5m2", 3600, spare=0)
        o, lse, _ = r.run()
        wide = [(p.float() * s.float()[..., None, None]).to(torch.bfloat16) for p, s in zip(r.pages, r.scales)]
        ws = torch.empty(pe.peagle_draft_decode_workspace_bytes(r.shape), dtype=torch.uint8, device="cuda")
        pe.peagle_draft_decode(r.shape, r.q, r.k, r.v, *wide, r.bt, r.cl, r.o, r.lse, r.status, ws)
        torch.cuda.synchronize()
        assert rel_l2(o, bf16_to_f64(r.o)) <= 4 * 2.0**-9 and max_abs(lse, r.lse.double().cpu().numpy()) <= 4e-3 + LSE_ABS


def test_draft_scaled_replays_from_a_graph_and_runs_on_other_streams():
    """One graph of two calls that share a workspace, replayed with new queries, lengths and tables between the replays; and the
    same call on a stream of its own."""
    print("case scaled graph", flush=True)
    r = ScaledRun((1500, 70, 640), 5, 16, 2, 64, "e4m3", 3700)
    r.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o2 = torch.empty_like(r.o)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        r.call(torch.cuda.current_stream())
        o2.copy_(r.o)
        r.call()
    rng = np.random.default_rng(1)
    for rep in range(3):
        r.q.copy_(torch.randn_like(r.q.float()))
        r.cl[0] = 1500 - 400 * rep
        r.bt[0, :5] = r.bt[0, torch.from_numpy(rng.permutation(5)).cuda()].clone()
        r.o.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        o_graph, lse_graph = r.o.clone(), r.lse.clone()
        eager = r.run()
        assert np.array_equal(bf16_to_f64(o_graph), eager[0]) and np.array_equal(bf16_to_f64(o2), eager[0])
        assert np.array_equal(lse_graph.double().cpu().numpy(), eager[1])
        r.o.fill_(float("nan"))
        side.wait_stream(torch.cuda.current_stream())
        r.call(side)
        side.synchronize()
        assert np.array_equal(bf16_to_f64(r.o), eager[0])


@pytest.mark.parametrize("K,Hq,Hkv,D,lens", [(5, 12, 4, 64, (130, 0, 63, 1000)), (3, 8, 2, 128, (700, 20)), (8, 16, 1, 128, (90, 200)), (1, 1, 1, 64, (5,))])
def test_draft_scaled_stays_inside_its_buffers(K, Hq, Hkv, D, lens):
    print(f"case scaled guards K={K} D={D}", flush=True)
    r = ScaledRun(lens, K, Hq, Hkv, D, "e4m3", 3800)
    g = Guarded()
    C = len(lens)
    r.o = g.tensor("o", (C, K, Hq, D), torch.bfloat16)
    r.lse = g.tensor("lse", (C, Hq, K), torch.float32)
    r.status = g.tensor("status", (C,), torch.int32)
    r.ws = g.tensor("workspace", (pe.peagle_draft_decode_scaled_workspace_bytes(r.shape),), torch.uint8)
    o, lse, status = r.run()
    g.check("scaled drafting step")
    r.check(o, lse, "guards")
    r.status = None
    r.call()
    g.check("without status")


def test_draft_scaled_beyond_four_gigabytes():
    """Pools of 4.3 GB with the context's pages on both sides of byte 2^32."""
    print("case scaled beyond 2^32", flush=True)
    r = ScaledRun((400,), 3, 8, 8, 128, "e4m3", 3900, spare=0)
    o, lse, _ = r.run()
    n_pages = 2**32 // (8 * 64 * 128) + 9
    where = torch.tensor([n_pages - 1, 3, n_pages - 9, 0, n_pages - 12, n_pages - 2, 70], device="cuda")
    for i in range(2):
        pages = torch.full((n_pages, 8, 64, 128), 0x7F, dtype=torch.uint8, device="cuda")
        scales = torch.full((n_pages, 8), 255, dtype=torch.uint8, device="cuda")
        order = r.bt[0].long()
        pages[where], scales[where] = r.pages[i].view(torch.uint8)[order], r.scales[i].view(torch.uint8)[order]
        r.pages[i], r.scales[i] = pages.view(TYPES["e4m3"]), scales.view(E8M0)
    r.bt[0] = where.int()
    r.shape = pe.DecodeShape(1, 3, 8, 8, 128, n_pages, 7)
    o2, lse2, status = r.run()
    assert (status == 0).all() and np.array_equal(o, o2) and np.array_equal(lse, lse2)


def test_plan_append_and_draft_as_a_serving_loop_runs_them():
    """Prompts admitted, stored and drafted from; accepted tokens appended, rejected ones rolled back, a request replaced: at
    every step the draft equals the oracle on the cache as the oracle holds it, and what that holds is off from the tokens
    themselves by no more than E4M3's rounding (2^-4, in norm)."""
    print("case serving loop", flush=True)
    rng = np.random.default_rng(11)
    C, K, Hq, Hkv, D, n_pages, cols = 3, 4, 8, 2, 64, 40, 10
    dev = lambda x, t: torch.from_numpy(np.asarray(x)).to(t).cuda()
    plan = pe.PlanShape(C, cols, n_pages, 512)
    held, free, count = dev([0] * C, torch.int32), dev(rng.permutation(n_pages), torch.int32), dev([n_pages], torch.int32)
    table = torch.full((C, cols), -1, dtype=torch.int32, device="cuda")
    start, slots = dev([0] * (C + 1), torch.int32), dev([0] * 512, torch.int64)
    seq_len, status = dev([0] * C, torch.int32), dev([0] * C, torch.int32)
    ws = torch.empty(pe.peagle_cache_plan_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
    pages = [torch.zeros((n_pages, Hkv, 64, D), dtype=torch.uint8, device="cuda").view(TYPES["e4m3"]) for _ in range(2)]
    scales = [torch.zeros((n_pages, Hkv), dtype=torch.uint8, device="cuda").view(E8M0) for _ in range(2)]
    shape = pe.DecodeShape(C, K, Hq, Hkv, D, n_pages, cols)
    draft_ws = torch.empty(pe.peagle_draft_decode_scaled_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    o, lse = torch.empty((C, K, Hq, D), dtype=torch.bfloat16, device="cuda"), torch.empty((C, Hq, K), device="cuda")
    values, exps = [np.zeros((n_pages, Hkv, 64, D)) for _ in range(2)], [np.full((n_pages, Hkv), -127) for _ in range(2)]
    kept = [[np.zeros((0, Hkv, D)) for _ in range(C)] for _ in range(2)]   # unrounded tokens of each request
    new_lens = [[70, 200, 5], [4, 1, 3], [0, 60, 4], [64, 2, 100], [1, 1, 1]]
    for step, new in enumerate(new_lens):
        if step == 3:
            kept = [[x[:max(0, len(x) - 2)] if c != 1 else x[:0] for c, x in enumerate(side)] for side in kept]
        ctx = [len(x) for x in kept[0]]
        pe.peagle_cache_plan(plan, dev(ctx, torch.int32), dev(new, torch.int32), held, free, count, table, start, slots, seq_len, status, ws)
        bits = [f32_to_bf16_bits(rng.standard_normal((512, Hkv, D), dtype=np.float32) * (step + 1)) for _ in range(2)]
        rows = [to_dev_bf16(b) for b in bits]
        pe.peagle_cache_append_scaled(pe.CacheShape(512, Hkv, D, n_pages), *rows, slots, *pages, *scales)
        q, kn, vn = (f32_to_bf16_bits(rng.standard_normal(s, dtype=np.float32)) for s in ((C, K, Hq, D), (C, K, Hkv, D), (C, K, Hkv, D)))
        draft_status = torch.full((C,), -1, dtype=torch.int32, device="cuda")
        pe.peagle_draft_decode_scaled(shape, to_dev_bf16(q), to_dev_bf16(kn), to_dev_bf16(vn), *pages, *scales, table, seq_len, o, lse, draft_status,
                                      draft_ws)
        torch.cuda.synchronize()
        assert status.tolist() == [0] * C and draft_status.tolist() == [0] * C and start.tolist() == [0, *np.cumsum(new)]
        at, host_table = slots.cpu().numpy(), table.cpu().numpy()
        for i in range(2):
            orc.cache_append(bf16_bits_to_f64(bits[i]), at, values[i], exps[i], "e4m3")
            for c in range(C):
                kept[i][c] = np.concatenate([kept[i][c], bf16_bits_to_f64(bits[i][sum(new[:c]):sum(new[:c + 1])])])
        assert seq_len.tolist() == [len(x) for x in kept[0]]
        for c in range(C):
            n = len(kept[0][c])
            p = host_table[c, :-(-n // 64)]
            held_k, held_v = ((values[i][p] * np.exp2(exps[i][p])[..., None, None]).transpose(0, 2, 1, 3).reshape(-1, Hkv, D)[:n] for i in range(2))
            args = [bf16_bits_to_f64(x[c]) for x in (q, kn, vn)]
            ro, rl = orc.draft_decode(*args, held_k, held_v, shape.scale)
            got, got_lse = bf16_to_f64(o[c]), lse[c].double().cpu().numpy()
            assert rel_l2(got, ro) <= REL and max_abs(got_lse, rl) <= 8 * LSE_ABS, (step, c)
            assert rel_l2(held_v, kept[1][c]) <= 2.0**-4 and rel_l2(held_k, kept[0][c]) <= 2.0**-4


ROWS = [(1, 2, 2), (7, 16, 2), (6, 32, 2), (8, 16, 1)]  # K, Hq, Hkv: one to four blocks of rows


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("K,Hq,Hkv", ROWS)
def test_draft_scaled_shows_infinities_of_the_last_cached_token(K, Hq, Hkv, D):
    """An infinity of E5M2 in V of the last cached token reaches that feature's outputs as an infinity of its sign, whether the
    places behind the token are masked (lengths off a multiple of 32) or not; every other feature stays as the oracle has it."""
    print(f"case scaled last token infinite K={K} Hq={Hq} D={D}", flush=True)
    r = ScaledRun((64, 65, 95, 96, 97, 127, 1, 31, 33, 1000), K, Hq, Hkv, D, "e5m2", 4000 + K)
    for c, n in enumerate(r.lens):
        raw, page, at = r.pages[1].view(torch.uint8), int(r.table[c, (n - 1) // 64]), (n - 1) % 64
        raw[page, 0, at, 5], raw[page, Hkv - 1, at, D - 1] = 0x7C, 0xFC
    o, lse, status = r.run()
    assert (status == 0).all() and np.isfinite(lse).all()
    group = Hq // Hkv
    for c in range(len(r.lens)):
        ro, rl = r.oracle(c)
        assert np.isposinf(ro[:, :group, 5]).all() and np.isneginf(ro[:, -group:, D - 1]).all()
        finite = np.isfinite(ro)
        assert np.array_equal(o[c][~finite], ro[~finite]), (c, r.lens[c])
        assert rel_l2(o[c][finite], ro[finite]) <= REL and max_abs(lse[c], rl) <= LSE_ABS, (c, r.lens[c])


@pytest.mark.parametrize("D", [64, 128])
def test_draft_scaled_masks_codes_that_widen_to_infinity(D):
    """A code and scale beyond bf16 in the last cached token: infinite in its own feature, and nowhere else."""
    print(f"case scaled widened infinity D={D}", flush=True)
    r = ScaledRun((65, 97, 64), 3, 8, 2, D, "e4m3", 4100)
    for c, n in enumerate(r.lens):
        page, at = int(r.table[c, (n - 1) // 64]), (n - 1) % 64
        raw = r.pages[1].view(torch.uint8)
        raw[page, :, :at + 1] = 0
        raw[page, :, at, 5] = 0x7E                    # 448 * 2^127
        r.scales[1].view(torch.uint8)[page] = 254
    o, lse, status = r.run()
    assert (status == 0).all() and np.isfinite(lse).all()
    assert np.isposinf(o[..., 5]).all() and np.isfinite(np.delete(o, 5, 3)).all()


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("K,Hq,Hkv", ROWS)
def test_draft_scaled_large_values_under_keys_that_stand_out(K, Hq, Hkv, D, fmt):
    """Values up to 2^101 whose keys score 28 or 32 powers of two above those before them: outputs are their weighted means, far
    from what fp32 holds at most, and so must be what is summed for them.  Some pages' values are small, on either side of them."""
    print(f"case scaled large values K={K} Hq={Hq} D={D} {fmt}", flush=True)
    r = ScaledRun((64 * 30, 100, 64 * 3 + 50), K, Hq, Hkv, D, fmt, 4200 + K, scale=float(np.log(2)), spare=0)
    keys = torch.zeros(r.pages[0].shape)
    keys[0::2, :, 40, 0], keys[1::2, :, 40, 0] = 28.0, 32.0
    r.pages[0].copy_(keys.to(TYPES[fmt]).cuda())
    r.scales[0].view(torch.uint8).fill_(127)
    top = 101 - (9 if fmt == "e4m3" else 16)
    r.scales[1].view(torch.uint8).copy_(torch.where(torch.arange(r.shape.n_pages) % 3 == 0, 120, 127 + top)[:, None].to(torch.uint8).cuda())
    q, k, _ = (bf16_bits_to_f64(x).astype(np.float32) for x in r.host)
    q[..., 0] = 1.0
    r.host[0], r.host[1] = f32_to_bf16_bits(q), f32_to_bf16_bits(np.zeros_like(k))
    r.q, r.k = to_dev_bf16(r.host[0]), to_dev_bf16(r.host[1])
    o, lse, status = r.run()
    assert (status == 0).all()
    for c in range(len(r.lens)):
        ro, rl = r.oracle(c)
        assert np.isfinite(o[c]).all() and (c != 0 or np.abs(ro).max() > 2.0**90), c
        assert rel_l2(o[c], ro) <= REL and max_abs(lse[c], rl) <= LSE_ABS, (c, rel_l2(o[c], ro))


@pytest.mark.parametrize("D", [64, 128])
def test_draft_scaled_large_new_values_under_keys_that_stand_out(D):
    """The same of new keys beyond the first sixteen."""
    print(f"case scaled large new values D={D}", flush=True)
    r = ScaledRun((0, 40), 40, 4, 2, D, "e4m3", 4300, scale=float(np.log(2)), spare=0)
    r.pages[0].view(torch.uint8).zero_()
    q, k, v = (bf16_bits_to_f64(x).astype(np.float32) for x in r.host)
    q[..., 0] = 1.0
    k[:] = 0.0
    k[:, 20, :, 0], k[:, 33, :, 0] = 28.0, 32.0
    v *= 2.0**100
    r.host = [f32_to_bf16_bits(x) for x in (q, k, v)]
    r.q, r.k, r.v = (to_dev_bf16(x) for x in r.host)
    o, lse, status = r.run()
    assert (status == 0).all()
    for c in range(2):
        ro, rl = r.oracle(c)
        assert np.isfinite(o[c]).all() and rel_l2(o[c], ro) <= REL and max_abs(lse[c], rl) <= LSE_ABS, c


class OneTokenEach:
    """Requests of one cached token each, in a page of its own, which has all the weight: O is its value.  It scores 300 above the
    new key."""

    def __init__(self, C, Hkv, D, fmt):
        q = torch.zeros((C, 1, Hkv, D), dtype=torch.bfloat16, device="cuda")
        k, self.v_new = torch.zeros_like(q), torch.zeros_like(q)
        q[..., 0], k[..., 0] = 300.0, -1.0
        self.q, self.k, self.fmt, self.shape = q, k, fmt, pe.DecodeShape(C, 1, Hkv, Hkv, D, C, 1, 1.0)
        keys = torch.zeros((C, Hkv, 64, D), device="cuda")
        keys[..., 0] = 1.0
        self.pages = [keys.to(TYPES[fmt]), torch.full(keys.shape, 0x7F, dtype=torch.uint8, device="cuda").view(TYPES[fmt])]
        self.scales = [torch.full((C, Hkv), 127, dtype=torch.uint8, device="cuda").view(E8M0) for _ in range(2)]

    def run(self):
        s = self.shape
        table, lens = torch.arange(s.C, dtype=torch.int32, device="cuda")[:, None].contiguous(), torch.ones(s.C, dtype=torch.int32, device="cuda")
        o, lse, status = torch.empty_like(self.q), torch.empty((s.C, s.Hq, 1), device="cuda"), torch.empty_like(lens)
        ws = torch.empty(pe.peagle_draft_decode_scaled_workspace_bytes(s), dtype=torch.uint8, device="cuda")
        pe.peagle_draft_decode_scaled(s, self.q, self.k, self.v_new, *self.pages, *self.scales, table, lens, o, lse, status, ws)
        torch.cuda.synchronize()
        assert not status.any()
        return bf16_to_f64(o)[:, 0]


def _as_widened(x):
    """Products of codes and scales as the step uses them: zero below bf16's normal numbers, infinite beyond them."""
    return np.where(np.abs(x) >= 2.0**128, np.copysign(np.inf, x), np.where(np.abs(x) < 2.0**-126, 0.0, x))


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("D", [64, 128])
def test_draft_scaled_widens_every_code_with_every_scale(D, fmt):
    """All 256 codes of values under all 256 codes of scales: exact wherever the product is a normal bf16 number."""
    print(f"case scaled every code and scale D={D} {fmt}", flush=True)
    r = OneTokenEach(256, 256 // D, D, fmt)
    every = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    r.pages[1].view(torch.uint8)[:, :, 0, :] = every.view(256 // D, D).cuda()
    r.scales[1].view(torch.uint8).copy_(every[:, None].cuda())
    o = r.run().reshape(256, 256)
    codes = every.view(TYPES[fmt]).double().numpy()
    exact = np.ldexp(codes[None], np.arange(256)[:, None] - 127)
    exact[255] = np.nan
    assert np.array_equal(o, _as_widened(exact), equal_nan=True)
    finite, (low, high) = codes[np.isfinite(codes)], {"e4m3": (10, 246), "e5m2": (17, 239)}[fmt]
    inside = np.ldexp(finite[None], np.arange(low, high + 1)[:, None] - 127)
    assert np.array_equal(_as_widened(inside), inside)
    for beyond in (low - 1, high + 1):  # (the range that the header names is the largest)
        outside = np.ldexp(finite, beyond - 127)
        assert not np.array_equal(_as_widened(outside), outside)


@pytest.mark.parametrize("fmt,first", [("e4m3", 1.9375), ("e5m2", 1.875)])
def test_append_and_draft_of_the_largest_values(fmt, first):
    """The largest bf16 values are rounded to 2^128 from `first` * 2^127 on, which the drafting step shows as an infinity; what is
    smaller stays finite."""
    print(f"case scaled largest values {fmt}", flush=True)
    x = np.array([1.75, 1.7578125, first - 2.0**-7, first, 1.9921875, -1.9921875, -1.75]) * 2.0**127
    r = OneTokenEach(len(x), 2, 64, fmt)
    rows = torch.from_numpy(x).float().to(torch.bfloat16).cuda()[:, None, None].expand(len(x), 2, 64).contiguous()
    slots = torch.arange(len(x), device="cuda") * 64
    pools, scales = [r.pages[0].clone(), r.pages[1]], [r.scales[0].clone(), r.scales[1]]  # (the keys stay what they are)
    pe.peagle_cache_append_scaled(pe.CacheShape(len(x), 2, 64, len(x)), rows, rows, slots, *pools, *scales)
    o = r.run()
    exps = np.array([orc.scale_exponent(abs(v), fmt) for v in x])
    assert np.array_equal(r.scales[1].view(torch.uint8).cpu().numpy().astype(int) - 127, np.stack([exps, exps], 1))
    assert exps.max() == {"e4m3": 120, "e5m2": 113}[fmt]
    want = _as_widened(np.array([orc.f8_round(v * 2.0**-e, fmt) * 2.0**e for v, e in zip(x, exps)]))
    assert np.array_equal(o, np.broadcast_to(want[:, None, None], o.shape))
    assert np.array_equal(np.isinf(want), np.abs(x) >= first * 2.0**127)


@pytest.mark.parametrize("C,ctx,columns,K,Hq,Hkv,D", [(16, 1000, 320, 7, 64, 8, 64), (3, 70, 1024, 5, 32, 4, 128), (1, 0, 300, 1, 4, 2, 64), (70, 300, 90, 8, 16, 1, 128)])
def test_draft_scaled_on_tables_wider_than_any_context(C, ctx, columns, K, Hq, Hkv, D):
    """Tables as wide as the longest context that a server permits: the division of the work sees the width, the results do not."""
    print(f"case scaled wide table C={C} columns={columns} D={D}", flush=True)
    rng = np.random.default_rng(columns)
    r = ScaledRun(tuple(int(x) for x in rng.integers(0, ctx + 1, C)), K, Hq, Hkv, D, "e4m3", 4400 + C)
    r.table = np.pad(r.table, ((0, 0), (0, columns - r.shape.max_pages)), constant_values=-1)
    r.bt = torch.from_numpy(r.table).cuda()
    r.shape = pe.DecodeShape(C, K, Hq, Hkv, D, r.shape.n_pages, columns)
    r.ws = torch.empty(pe.peagle_draft_decode_scaled_workspace_bytes(r.shape), dtype=torch.uint8, device="cuda").fill_(0x7F)
    o, lse, status = r.run()
    assert (status == 0).all()
    r.check(o, lse, "wide", range(0, C, max(1, C // 8)))


@pytest.mark.parametrize("C", [999, 1024, 1025])
def test_draft_scaled_of_a_thousand_requests(C):
    """The most requests whose pages are shared among workgroups, and one more, which take a workgroup each."""
    print(f"case scaled C={C}", flush=True)
    rng = np.random.default_rng(C)
    lens = rng.integers(0, 200, C)
    lens[0], lens[500], lens[C - 1] = 5000, 4700, 4321
    r = ScaledRun(tuple(int(x) for x in lens), 2, 2, 1, 64, "e5m2", C, shared=30)
    o, lse, status = r.run()
    assert (status == 0).all()
    r.check(o, lse, "thousand", (0, 1, 15, 16, 17, 499, 500, 501, C // 2, C - 2, C - 1))
