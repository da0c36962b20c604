"""GPU tests of the operators on a paged cache held in 4 bits, against the oracle (numpy, 64 bits): tokens stored as E2M1 with a
power-of-two scale for each token, KV head and 32 features, caches read back as bf16 rows, and the drafting step on such a cache.

What is stored and read is defined to the bit: codes, scales, rows and untouched places are compared for equality.

The drafting step: what the cache holds is exact in bf16.  A rounding to bf16 is off by at most 2^-8 of the value.  Rounded
probabilities p (1 + d) weigh the values and are summed for the division: to first order an output is off by at most
2 * 2^-8 sum p |v|, by fp32 scores that are each off by less than 1e-3 (D products: D * 2^-24 of sum |q k| scale, for the inputs
here) by another 2e-3 sum p |v|, and by its own rounding, 2^-8 of itself.  In norm the roundings are random: one of them has a mean
square of (2^-8 / sqrt 3)^2 times that of a significand's place in [1, 2), 1.7e-3 together, and the two of the probabilities and
the output's are below 1.7e-3 * sqrt 3 = 2.9e-3 < 5e-3.  The LSE takes unrounded probabilities: off by what the scores are."""
import threading
from types import SimpleNamespace

import numpy as np
import pytest
import torch

import paper_2602_01469_amd as pe
from gpu_harness import bf16_to_f64, max_abs, rel_l2, to_dev_bf16
from oracle import peagle_oracle as orc
from peagle_inputs import bf16_bits_to_f64, f32_to_bf16_bits
from test_gpu_draft_scaled import CASES, LSE_ABS, REL, ROWS, ScaledRun
from test_gpu_guards import Guarded

pytestmark = pytest.mark.gpu

F4, E8M0 = torch.float4_e2m1fn_x2, torch.float8_e8m0fnu
TYPES = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _packed(codes):
    """Codes [..., D] two a byte, the lower feature in the lower half."""
    c = np.asarray(codes, dtype=np.uint8)
    return torch.from_numpy(c[..., ::2] | c[..., 1::2] << 4)


def _unpacked(pages):
    raw = pages.view(torch.uint8).cpu().numpy()
    return np.stack([raw & 15, raw >> 4], -1).reshape(*raw.shape[:-1], 2 * raw.shape[-1])


def _rand(g, *shape, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(torch.bfloat16)


def _slots_on(slots):
    return torch.from_numpy(np.asarray(slots, dtype=np.int64)).cuda()


class Cache:
    """A 4-bit cache on the GPU and in the oracle, from random codes and scales."""

    def __init__(self, rng, n_pages, Hkv, D):
        self.n_pages, self.Hkv, self.D = n_pages, Hkv, D
        self.codes = [rng.integers(0, 16, (n_pages, Hkv, 64, D)) for _ in range(2)]
        self.exps = [rng.integers(90, 150, (n_pages, Hkv, 64, D // 32)) for _ in range(2)]
        self.pages = [_packed(c).cuda().view(F4) for c in self.codes]
        self.scales = [torch.from_numpy(e.astype(np.uint8)).cuda().view(E8M0) for e in self.exps]

    def append(self, k, v, slots):
        pe.peagle_cache_append_block_scaled(pe.CacheShape(len(slots), self.Hkv, self.D, self.n_pages), k, v, _slots_on(slots), *self.pages, *self.scales)
        for x, codes, exps in zip((k, v), self.codes, self.exps):
            orc.cache_append_blocks(bf16_to_f64(x.contiguous()), slots, codes, exps)

    def check(self, what):
        torch.cuda.synchronize()
        for i, n in enumerate("kv"):
            assert np.array_equal(self.scales[i].view(torch.uint8).cpu().numpy(), self.exps[i]), (what, n, "scale")
            assert np.array_equal(_unpacked(self.pages[i]), self.codes[i]), (what, n)

    def read(self, slots, k=None, v=None):
        n = len(slots)
        if k is None:
            k, v = (torch.full((n, self.Hkv, self.D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        pe.peagle_cache_read(pe.CacheShape(n, self.Hkv, self.D, self.n_pages), _slots_on(slots), *self.pages, *self.scales, k, v)
        return k, v

    def values(self, i, slots):
        slots = np.asarray(slots)
        there = (slots >= 0) & (slots < 64 * self.n_pages)
        at = np.where(there, slots, 0)
        x = orc.cache_values_blocks(self.codes[i], self.exps[i])[at // 64, :, at % 64]
        return np.where(there[:, None, None], x, 0.0)

    def check_read(self, slots, what):
        for i, x in enumerate(self.read(slots)):
            assert np.array_equal(bf16_to_f64(x), self.values(i, slots), equal_nan=True), (what, "kv"[i])


# -------------------------------------------------------------------------------------------------------- append, read

@pytest.mark.parametrize("Hkv,D", [(1, 64), (8, 64), (3, 128), (4, 128)])
@pytest.mark.parametrize("n", [1, 2, 3, 7, 8, 9, 31, 33, 64, 65, 127, 128, 129, 300])
def test_append_and_read(n, Hkv, D):
    """Numbers of tokens around those that a load, a wave and a workgroup take; any places of the pool; sizes far apart."""
    print(f"case block append n={n} Hkv={Hkv} D={D}", flush=True)
    rng, g = np.random.default_rng(n + D + Hkv), torch.Generator(device="cuda").manual_seed(n)
    cache = Cache(rng, 9, Hkv, D)
    for scale in (1.0, 300.0, 1e-3):
        slots = rng.permutation(9 * 64)[:n]
        cache.append(_rand(g, n, Hkv, D, scale=scale), _rand(g, n, Hkv, D, scale=7 * scale), slots)
        cache.check((n, scale))
        cache.check_read(slots, (n, scale))
    cache.check_read(rng.integers(-3, 9 * 64 + 3, 2 * n), "any slots")


@pytest.mark.parametrize("n_tokens,Hkv,D", [(3891, 8, 64), (9000, 4, 128), (5000, 1, 64)])
def test_append_and_read_of_many_tokens(n_tokens, Hkv, D):
    print(f"case block append many {n_tokens} Hkv={Hkv} D={D}", flush=True)
    rng, g = np.random.default_rng(n_tokens), torch.Generator(device="cuda").manual_seed(n_tokens)
    n_pages = -(-n_tokens // 64) + 2
    pages = rng.permutation(n_pages)
    slots = pages[(np.arange(n_tokens) + 40) // 64] * 64 + (np.arange(n_tokens) + 40) % 64
    k, v = _rand(g, n_tokens, Hkv, D, scale=3), _rand(g, n_tokens, Hkv, D)
    cache = Cache(rng, n_pages, Hkv, D)
    before = [s.view(torch.uint8).clone() for s in cache.scales]
    pe.peagle_cache_append_block_scaled(pe.CacheShape(n_tokens, Hkv, D, n_pages), k, v, _slots_on(slots), *cache.pages, *cache.scales)
    k2, v2 = cache.read(slots)
    some = rng.permutation(n_tokens)[:200]
    for x, y, scales, old in zip((k, v), (k2, v2), cache.scales, before):
        codes, exps = np.zeros((4, Hkv, 64, D), dtype=int), np.zeros((4, Hkv, 64, D // 32), dtype=int)
        orc.cache_append_blocks(bf16_to_f64(x[torch.from_numpy(some).cuda()]), np.arange(200), codes, exps)
        want = orc.cache_values_blocks(codes, exps).transpose(0, 2, 1, 3).reshape(256, Hkv, D)[:200]
        assert np.array_equal(bf16_to_f64(y[torch.from_numpy(some).cuda()]), want)
        free = np.setdiff1d(np.arange(n_pages * 64), slots)
        new = scales.view(torch.uint8).cpu().numpy()
        assert np.array_equal(new[free // 64, :, free % 64], old.cpu().numpy()[free // 64, :, free % 64])
        # a block's largest value is kept to half a step of its code, between 3 and 6 two powers of two below 8: 2^-2 relative at most
        assert float((y.float() - x.float()).abs().max() / x.float().abs().max()) <= 0.25


def test_append_and_read_find_few_slots_among_many_tokens():
    """More tokens than one dimension of the launch holds workgroups for; slots in the first, the middle and the last of them."""
    n = 32768 * 128 + 1000
    print(f"case block append few of {n}", flush=True)
    rng, g = np.random.default_rng(5), torch.Generator(device="cuda").manual_seed(5)
    cache = Cache(rng, 5, 1, 64)
    k, v = _rand(g, n, 1, 64), _rand(g, n, 1, 64)
    at = np.concatenate([np.arange(70), n // 2 + np.arange(130), n - 90 + np.arange(90)])
    places = rng.permutation(5 * 64)[:len(at)]
    slots = np.full(n, -1, dtype=np.int64)
    slots[at] = places
    pe.peagle_cache_append_block_scaled(pe.CacheShape(n, 1, 64, 5), k, v, _slots_on(slots), *cache.pages, *cache.scales)
    rows = torch.from_numpy(at).cuda()
    for x, codes, exps in zip((k, v), cache.codes, cache.exps):
        orc.cache_append_blocks(bf16_to_f64(x[rows]), places, codes, exps)
    cache.check("few of many")
    for i, x in enumerate(cache.read(slots)):
        assert np.array_equal(bf16_to_f64(x[rows]), cache.values(i, places))
        x[rows] = 0
        assert not bool(x.any())


def test_append_and_read_skip_slots_outside_the_pool():
    print("case block skips", flush=True)
    rng, g = np.random.default_rng(6), torch.Generator(device="cuda").manual_seed(6)
    cache = Cache(rng, 6, 2, 64)
    slots = np.array([-1, -1, 64, 65, 66, -1, 130, -1, 6 * 64, 6 * 64 + 1, 2**40, -2**40, 2**62, -2**63, 0, 1, 6 * 64 - 1, -1])
    cache.append(_rand(g, len(slots), 2, 64), _rand(g, len(slots), 2, 64), slots)
    cache.check("skips")
    cache.check_read(slots, "skips")
    for n in (3, 0):
        cache.append(_rand(g, n, 2, 64), _rand(g, n, 2, 64), np.full(n, -1))
        cache.check("nothing")
        cache.check_read(np.full(n, -1), "nothing")


def test_read_gives_a_slot_as_often_as_it_is_named():
    print("case block read repeats", flush=True)
    cache = Cache(np.random.default_rng(7), 3, 2, 128)
    cache.check_read(np.array([5] * 70 + [191, 0, 191]), "repeats")


@pytest.mark.parametrize("D", [64, 128])
def test_append_of_two_tokens_with_one_slot(D):
    """Each piece of the slot is one of the two tokens'; nothing else is touched."""
    print(f"case block one slot D={D}", flush=True)
    rng = np.random.default_rng(77)
    rows = torch.from_numpy(rng.standard_normal((40, 2, D))).bfloat16().cuda()
    slots = np.arange(40) + 30
    slots[37] = slots[2]                                      # (of other steps, waves)
    slots[1] = slots[0]                                       # (of one step)
    firsts, lasts = np.sort(np.unique(slots, return_index=True)[1]), 39 - np.sort(np.unique(slots[::-1], return_index=True)[1])
    held = []
    for keep in (np.arange(40), firsts, lasts):
        cache = Cache(np.random.default_rng(5), 3, 2, D)
        x = rows[torch.from_numpy(keep)]
        pe.peagle_cache_append_block_scaled(pe.CacheShape(len(keep), 2, D, 3), x, x, _slots_on(slots[keep]), *cache.pages, *cache.scales)
        held.append([x.view(torch.uint8).cpu().numpy() for x in (*cache.pages, *cache.scales)])
    for both, a, b in zip(*held):
        assert ((both == a) | (both == b)).all()


def test_rows_that_stand_apart():
    """K and V of wider rows, to be stored and as results; what stands between the results stays."""
    print("case block strides", flush=True)
    rng, g = np.random.default_rng(8), torch.Generator(device="cuda").manual_seed(8)
    for D, width in ((64, 64 * 20), (128, 128 * 9 + 8)):
        cache = Cache(rng, 4, 3, D)
        rows = _rand(g, 150, width)
        views = lambda x: (x[:, 2 * D:5 * D].unflatten(1, (3, D)), x[:, 5 * D + 8:8 * D + 8].unflatten(1, (3, D)))
        slots = rng.permutation(256)[:150]
        cache.append(*views(rows), slots)
        cache.check(D)
        out = torch.full_like(rows, 3.0)
        for i, x in enumerate(cache.read(slots, *views(out))):
            assert np.array_equal(bf16_to_f64(x.contiguous()), cache.values(i, slots))
            x.fill_(3.0)
        assert bool((out == 3.0).all())
    with pytest.raises(ValueError, match="contiguous"):
        cache.read(np.arange(4), rows[:4, :3 * 128].view(4, 128, 3).transpose(1, 2), rows[:4, :3 * 128].unflatten(1, (3, 128)))


def test_append_of_values_at_the_edges():
    """Zeros of both signs, halfway cases, the largest and smallest bf16 values, values next to a change of scale, infinities and NaN
    alone and among ordinary values, in one block and in the other."""
    print("case block append edges", flush=True)
    big, tiny = 3.3895313892515355e38, 2.0**-133
    rows = [[0.0], [-0.0, 0.0], [big, -big], [2.0**-126, -2.0**-126], [tiny, 2.0**-100], [6.0, -1.0], [6.03125, 1.0], [5.96875, 1.0], [12.0, 0.5],
            [np.inf, 1.0], [-np.inf, np.nan], [np.nan], [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], [-0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, 6.0],
            [1e-30, 2e-30], [np.inf, big], [2.0**-92, 2.0**-110, 6 * 2.0**-100], [2.0**-100, 2.0**-101, 2.0**-102, 3 * 2.0**-102, -2.0**-103],
            [1.75 * 2.0**127, 2.0**126, 2.0**127], [1.7421875 * 2.0**127, 1.5 * 2.0**127], [1.5 * 2.0**127], [6 * 2.0**-100], [6.03125 * 2.0**-100]]
    x = torch.zeros(len(rows), 1, 64)
    for i, r in enumerate(rows):
        x[i, 0] = torch.tensor(r, dtype=torch.float64).repeat(64)[:64].float()
        if i % 2:
            x[i, 0, 32:] = torch.arange(32) / 8.0  # (its other block is an ordinary one)
    x = x.to(torch.bfloat16).cuda()
    cache = Cache(np.random.default_rng(9), 1, 1, 64)
    with np.errstate(over="ignore"):
        cache.append(x, x.flip(0).flip(2), np.arange(len(rows)) + 20)
        cache.check("edges")
        assert cache.exps[0].min() == 27 and set(cache.exps[0][cache.exps[0] > 253]) == {255} and cache.exps[0][cache.exps[0] < 255].max() == 253
        got = [bf16_to_f64(y) for y in cache.read(np.arange(64))]
    for i, y in enumerate(got):
        want = cache.values(i, np.arange(64))
        assert np.array_equal(y, np.where(np.abs(want) >= 2.0**128, np.copysign(np.inf, want), want), equal_nan=True)


def _as_bf16(x):
    """The bf16 number that exact 64-bit x with at most four significant bits is; infinite from 2^128 on."""
    return np.where(np.abs(x) >= 2.0**128, np.copysign(np.inf, x), x)


@pytest.mark.parametrize("D", [64, 128])
def test_read_of_every_code_with_every_scale(D):
    print(f"case block read every code D={D}", flush=True)
    cache = Cache(np.random.default_rng(10), 4, 2, D)
    every = np.arange(16)
    cache.codes = [np.broadcast_to(np.resize(every, D), (4, 2, 64, D)).copy(), np.broadcast_to(np.resize(every[::-1], D), (4, 2, 64, D)).copy()]
    scales = np.broadcast_to(np.arange(256).reshape(4, 1, 64, 1), (4, 2, 64, D // 32)).copy()
    scales[:, 1], scales[..., 1] = 255 - scales[:, 1], (scales[..., 1] + 100) % 256
    cache.exps = [scales, scales[::-1].copy()]
    cache.pages = [_packed(c).cuda().view(F4) for c in cache.codes]
    cache.scales = [torch.from_numpy(e.astype(np.uint8)).cuda().view(E8M0) for e in cache.exps]
    for i, x in enumerate(cache.read(np.arange(256))):
        assert np.array_equal(bf16_to_f64(x), _as_bf16(cache.values(i, np.arange(256))), equal_nan=True)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("D", [64, 128])
def test_read_of_every_8_bit_code_with_every_scale(D, fmt):
    """Exact wherever the product is a normal bf16 number; NaN, infinities and what is infinite in bf16 as they are."""
    print(f"case block read 8 bits D={D} {fmt}", flush=True)
    every = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    Hkv = 256 // D
    pages = every.view(1, Hkv, 1, D).expand(256, Hkv, 64, D).contiguous().cuda().view(TYPES[fmt])
    scales = every[:, None].expand(256, Hkv).contiguous().cuda().view(E8M0)
    slots = torch.arange(256, device="cuda") * 64 + torch.arange(256, device="cuda") % 64
    k, v = (torch.empty((256, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pe.peagle_cache_read(pe.CacheShape(256, Hkv, D, 256), slots, pages, pages, scales, scales.flip(0), k, v)
    codes = every.view(TYPES[fmt]).double().numpy()
    want = np.ldexp(codes[None], np.arange(256)[:, None] - 127)
    want[255] = np.nan
    for x, w in ((k, want), (v, want[::-1])):
        x = bf16_to_f64(x).reshape(256, 256)
        normal = ~(np.abs(w) < 2.0**-126) | (w == 0)
        assert np.array_equal(x[normal], _as_bf16(w)[normal], equal_nan=True)
        assert (np.abs(x[~normal] - w[~normal]) <= 2.0**-126).all()


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("Hkv,D,n", [(8, 64, 500), (3, 128, 77), (1, 64, 1)])
def test_read_of_what_an_8_bit_append_stored(Hkv, D, n, fmt):
    print(f"case block read after 8 bits Hkv={Hkv} D={D} {fmt}", flush=True)
    rng, g = np.random.default_rng(n), torch.Generator(device="cuda").manual_seed(n)
    n_pages = -(-n // 64) + 2
    pages = [torch.zeros((n_pages, Hkv, 64, D), dtype=torch.uint8, device="cuda").view(TYPES[fmt]) for _ in range(2)]
    scales = [torch.zeros((n_pages, Hkv), dtype=torch.uint8, device="cuda").view(E8M0) for _ in range(2)]
    slots = rng.permutation(n_pages)[np.arange(n) // 64] * 64 + np.arange(n) % 64
    k, v = _rand(g, n, Hkv, D), _rand(g, n, Hkv, D, scale=100)
    shape = pe.CacheShape(n, Hkv, D, n_pages)
    pe.peagle_cache_append_scaled(shape, k, v, _slots_on(slots), *pages, *scales)
    out = torch.full((n, 2, Hkv, D), 3.0, dtype=torch.bfloat16, device="cuda")
    pe.peagle_cache_read(shape, _slots_on(slots), *pages, *scales, out[:, 0], out[:, 1])
    for i, x in enumerate((k, v)):
        values, exps = np.zeros((n_pages, Hkv, 64, D)), np.zeros((n_pages, Hkv), dtype=int)
        orc.cache_append(bf16_to_f64(x), slots, values, exps, fmt)
        assert np.array_equal(bf16_to_f64(out[:, i].contiguous()), (values * np.exp2(exps)[..., None, None])[slots // 64, :, slots % 64])


@pytest.mark.parametrize("Hkv,D,n", [(1, 64, 1), (3, 128, 77), (2, 64, 700)])
def test_append_and_read_stay_inside_their_buffers(Hkv, D, n):
    print(f"case block guards Hkv={Hkv} D={D}", flush=True)
    rng, gen = np.random.default_rng(n), torch.Generator(device="cuda").manual_seed(n)
    cache = Cache(rng, -(-n // 64) + 1, Hkv, D)
    g = Guarded()
    cache.pages = [g.tensor(f"pages {i}", tuple(x.shape), torch.uint8).copy_(x.view(torch.uint8)).view(F4) for i, x in enumerate(cache.pages)]
    cache.scales = [g.tensor(f"scales {i}", tuple(x.shape), torch.uint8).copy_(x.view(torch.uint8)).view(E8M0) for i, x in enumerate(cache.scales)]
    slots = np.arange(cache.n_pages * 64 - n, cache.n_pages * 64)
    cache.append(_rand(gen, n, Hkv, D, scale=50), _rand(gen, n, Hkv, D), slots)
    out = [g.tensor(f"rows {i}", (n, Hkv, D), torch.bfloat16) for i in range(2)]
    cache.read(slots, *out)
    g.check("append and read")
    cache.check("guards")
    for i, x in enumerate(out):
        assert np.array_equal(bf16_to_f64(x), cache.values(i, slots))


def test_append_and_read_replay_from_a_graph_and_run_on_other_streams():
    print("case block append graph", flush=True)
    rng, g = np.random.default_rng(11), torch.Generator(device="cuda").manual_seed(11)
    cache = Cache(rng, 6, 4, 64)
    n = 75
    k, v, slots = _rand(g, n, 4, 64), _rand(g, n, 4, 64), _slots_on(np.arange(n))
    out = [torch.empty((n, 4, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    shape = pe.CacheShape(n, 4, 64, 6)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        pe.peagle_cache_append_block_scaled(shape, k, v, slots, *cache.pages, *cache.scales)
        pe.peagle_cache_read(shape, slots, *cache.pages, *cache.scales, *out)
    for rep in range(4):
        at = rng.permutation(6 * 64)[:n]
        k.copy_(_rand(g, n, 4, 64, scale=rep + 1))
        v.copy_(_rand(g, n, 4, 64))
        slots.copy_(_slots_on(at))
        graph.replay()
        for x, codes, exps in zip((k, v), cache.codes, cache.exps):
            orc.cache_append_blocks(bf16_to_f64(x), at, codes, exps)
        cache.check(rep)
        for i, x in enumerate(out):
            assert np.array_equal(bf16_to_f64(x), cache.values(i, at))
            x.fill_(5.0)
        side.wait_stream(torch.cuda.current_stream())
        pe.peagle_cache_read(shape, slots, *cache.pages, *cache.scales, *out, stream=side)
        side.synchronize()
        assert all(np.array_equal(bf16_to_f64(x), cache.values(i, at)) for i, x in enumerate(out))


def test_append_and_read_beyond_four_gigabytes():
    """Pools of 4.3 GB: pages on both sides of byte 2^32."""
    print("case block beyond 2^32", flush=True)
    Hkv, D = 8, 128
    n_pages = 2**32 // (Hkv * 64 * D // 2) + 3
    g = torch.Generator(device="cuda").manual_seed(12)
    pages = [torch.zeros((n_pages, Hkv, 64, D // 2), dtype=torch.uint8, device="cuda").view(F4) for _ in range(2)]
    scales = [torch.full((n_pages, Hkv, 64, D // 32), 9, dtype=torch.uint8, device="cuda").view(E8M0) for _ in range(2)]
    k, v = _rand(g, 130, Hkv, D), _rand(g, 130, Hkv, D)
    slots = _slots_on(np.concatenate([(n_pages - 1) * 64 + np.arange(64), np.arange(64), (n_pages - 4) * 64 + np.arange(2)]))
    shape = pe.CacheShape(130, Hkv, D, n_pages)
    pe.peagle_cache_append_block_scaled(shape, k, v, slots, *pages, *scales)
    out = [torch.empty((130, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    pe.peagle_cache_read(shape, slots, *pages, *scales, *out)
    for x, y, p, s in zip((k, v), out, pages, scales):
        codes, exps = np.zeros((3, Hkv, 64, D), dtype=int), np.full((3, Hkv, 64, D // 32), 9)
        orc.cache_append_blocks(bf16_to_f64(x), np.arange(130), codes, exps)
        at = torch.tensor([n_pages - 1, 0, n_pages - 4], device="cuda")
        assert np.array_equal(_unpacked(p.view(torch.uint8)[at]), codes) and np.array_equal(s.view(torch.uint8)[at].cpu().numpy(), exps)
        assert np.array_equal(bf16_to_f64(y), orc.cache_values_blocks(codes, exps).transpose(0, 2, 1, 3).reshape(192, Hkv, D)[:130])
        others = torch.ones(n_pages, dtype=torch.bool, device="cuda")
        others[at] = False
        assert bool((s.view(torch.uint8)[others] == 9).all())
        assert int(p.view(torch.uint8).view(torch.int64).ne(0).sum()) <= 130 * Hkv * D // 16


# ------------------------------------------------------------------------------------------------------ drafting step

class BlockRun(ScaledRun):
    """Inputs of one drafting step on a 4-bit cache: scales of their own for every token and 32 features, some larger than they have
    to be; unused places hold a scale of NaN and any codes.  shared: that many pages that all requests use in any order."""

    def __init__(self, ctx_lens, K, Hq, Hkv, D, seed, shared=0, scale=None, spare=3, gain=1.0):
        rng = np.random.default_rng(seed)
        C = len(ctx_lens)
        pages_of = [-(-n // 64) for n in ctx_lens]
        max_pages = max(1, max(pages_of))
        used = shared or sum(pages_of)
        n_pages = max(1, used + spare)
        perm = rng.permutation(n_pages)
        table = np.full((C, max_pages), -1, dtype=np.int32)
        at = 0
        for c, n in enumerate(pages_of):
            table[c, :n] = rng.choice(perm[:shared], n) if shared else perm[at:at + n]
            at += n
        self.pages, self.scales = [], []
        for i in range(2):
            codes = rng.integers(0, 256, (n_pages, Hkv, 64, D // 2), dtype=np.uint8)
            exps = rng.integers(123, 128, (n_pages, Hkv, 64, D // 32)) + (0 if i else int(np.log2(gain)))
            if not shared:
                for c, n in enumerate(ctx_lens):
                    if n % 64:
                        exps[table[c, n // 64], :, n % 64:] = 255
                exps[perm[used:]] = 255
            self.pages.append(torch.from_numpy(codes).cuda().view(F4))
            self.scales.append(torch.from_numpy(exps.astype(np.uint8)).cuda().view(E8M0))
        bits = lambda *shape: f32_to_bf16_bits(rng.standard_normal(shape, dtype=np.float32))
        self.host = [bits(C, K, Hq, D), bits(C, K, Hkv, D), bits(C, K, Hkv, D)]
        self.table, self.lens = table, list(ctx_lens)
        self.shape = pe.DecodeShape(C, K, Hq, Hkv, D, n_pages, max_pages, scale)
        self.q, self.k, self.v = (to_dev_bf16(x) for x in self.host)
        self.bt, self.cl = torch.from_numpy(table).cuda(), torch.tensor(ctx_lens, dtype=torch.int32, device="cuda")
        self.o = torch.full((C, K, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full((C, Hq, K), float("nan"), device="cuda")
        self.status = torch.full((C,), -7, dtype=torch.int32, device="cuda")
        self.ws = torch.empty(pe.peagle_draft_decode_block_scaled_workspace_bytes(self.shape), dtype=torch.uint8, device="cuda").fill_(0x7F)

    def call(self, stream=None):
        pe.peagle_draft_decode_block_scaled(self.shape, self.q, self.k, self.v, *self.pages, *self.scales, self.bt, self.cl, self.o, self.lse,
                                            self.status, self.ws, stream)

    def context(self, c):
        n = self.lens[c]
        pages = torch.from_numpy(np.maximum(self.table[c, :-(-n // 64)], 0).astype(np.int64)).cuda()
        out = []
        for p, s in zip(self.pages, self.scales):
            x = orc.cache_values_blocks(_unpacked(p.view(torch.uint8)[pages]), s.view(torch.uint8)[pages].cpu().numpy())
            out.append(x.transpose(0, 2, 1, 3).reshape(-1, x.shape[1], x.shape[3])[:n])
        return out

    def check(self, o, lse, what, requests=None):
        for c in range(len(self.lens)) if requests is None else requests:
            k, v = self.context(c)
            q, kn, vn = (bf16_bits_to_f64(x[c]) for x in self.host)
            ro, rl = orc.draft_decode(q, kn, vn, k, v, self.shape.scale)
            weighed, _ = orc.draft_decode(q, kn, np.abs(vn), k, np.abs(v), self.shape.scale)  # sum p |v|
            assert np.isfinite(o[c]).all() and np.isfinite(lse[c]).all(), (what, c)
            over = np.abs(o[c] - ro) - 2.0**-8 * np.abs(ro) - (2.0**-7 + 2e-3) * weighed
            assert over.max() <= 0, (what, c, over.max())
            assert rel_l2(o[c], ro) <= REL, (what, c, rel_l2(o[c], ro))
            assert max_abs(lse[c], rl) <= LSE_ABS, (what, c, max_abs(lse[c], rl))


@pytest.mark.parametrize("name,ctx_lens,K,Hq,Hkv,D", CASES, ids=[c[0] for c in CASES])
def test_draft_matches_oracle(name, ctx_lens, K, Hq, Hkv, D):
    print(f"case block {name}", flush=True)
    r = BlockRun(ctx_lens, K, Hq, Hkv, D, 3000 + len(name))
    o, lse, status = r.run()
    assert (status == 0).all()
    r.check(o, lse, name)
    o2, lse2, _ = r.run()
    assert np.array_equal(o, o2) and np.array_equal(lse, lse2)


@pytest.mark.parametrize("C,ctx,K,Hq,Hkv,D", [(64, 20000, 2, 16, 8, 64), (64, 5000, 8, 128, 8, 128), (130, 9000, 4, 64, 4, 64), (256, 500, 7, 16, 2, 64),
                                              (70, 2000, 4, 8, 8, 128), (70, 900, 7, 32, 4, 64), (100, 2500, 7, 24, 4, 128), (40, 1500, 16, 64, 8, 64),
                                              (40, 6000, 4, 256, 8, 64), (64, 5000, 3, 16, 8, 128), (64, 4000, 8, 64, 4, 128), (40, 1500, 3, 32, 4, 128),
                                              (50, 2000, 7, 32, 4, 128), (33, 1900, 16, 32, 4, 128),
                                              (30, 2000, 7, 64, 8, 64), (20, 5000, 16, 32, 4, 128), (9, 300, 16, 32, 4, 128)])
def test_draft_batches_on_a_shared_pool(C, ctx, K, Hq, Hkv, D):
    """Many requests whose tables point into a few pages: by request and in shares, one to four blocks of rows, more than 64 pages for
    a wave, unequal lengths; some of them against the oracle.  Then one request's table is spoiled: it alone is flagged and changes."""
    rng = np.random.default_rng(C + ctx)
    lens = rng.integers(0, ctx, C)
    lens[3], lens[C // 2] = ctx, 0
    print(f"case block batch C={C} ctx={ctx} D={D}", flush=True)
    r = BlockRun(tuple(int(x) for x in lens), K, Hq, Hkv, D, C, shared=40)
    o, lse, status = r.run()
    assert (status == 0).all()
    r.check(o, lse, "batch", (0, 3, C // 2, C - 1))
    r.bt[3, 1] = r.shape.n_pages
    o2, lse2, status2 = r.run()
    others = np.arange(C) != 3
    assert status2[3] == 1 and (status2[others] == 0).all()
    assert np.array_equal(o2[others], o[others]) and np.array_equal(lse2[others], lse[others]) and np.isfinite(o2).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("K,Hq,Hkv", ROWS)
def test_draft_flags_bad_tables_and_lengths(K, Hq, Hkv, D):
    """Page ids on both sides of the pool, lengths below zero and beyond the table: flagged, skipped or clamped; what is left of such a
    request, and the other requests, exact."""
    print(f"case block bad tables K={K} Hq={Hq} D={D}", flush=True)
    r = BlockRun((300, 200, 100, 130, 64), K, Hq, Hkv, D, 3100)
    good = r.run()
    r.bt[1, 2] = r.shape.n_pages + 5
    r.bt[3, 0] = -2**31
    r.cl[2] = 64 * r.shape.max_pages + 1
    r.bt[2, :] = int(r.table[0, 0])   # (all of its tokens are there)
    r.cl[4] = -3
    o, lse, status = r.run()
    assert status.tolist() == [0, 1, 1, 1, 1] and np.array_equal(o[0], good[0][0]) and np.array_equal(lse[0], good[1][0])
    assert np.isfinite(lse[1:]).all()
    for c, bad in ((1, slice(128, 192)), (3, slice(0, 64)), (4, slice(0, None))):   # without the keys of the bad page, or any
        k, v = (np.delete(x, bad, 0) for x in r.context(c))
        ro, rl = orc.draft_decode(*(bf16_bits_to_f64(x[c]) for x in r.host), k, v, r.shape.scale)
        assert rel_l2(o[c], ro) <= REL and max_abs(lse[c], rl) <= LSE_ABS, c


@pytest.mark.parametrize("C,ctx,K,Hq,Hkv,D", [(256, 20000, 7, 64, 8, 64), (256, 20000, 2, 16, 8, 64), (256, 20000, 16, 64, 8, 64), (64, 20000, 8, 128, 8, 128),
                                              (64, 20000, 7, 64, 8, 128), (128, 20000, 3, 64, 8, 128)])
def test_draft_runs_of_more_pages_than_lanes(C, ctx, K, Hq, Hkv, D):
    """Shares in which a wave has more than 64 pages of one request, whose ids a wave's lanes hold: two of the requests against the
    oracle, and all of them the same twice."""
    print(f"case block long runs C={C} K={K} Hq={Hq} D={D}", flush=True)
    rng = np.random.default_rng(C + K)
    lens = rng.integers(ctx // 2, ctx, C)
    lens[1] = ctx
    r = BlockRun(tuple(int(x) for x in lens), K, Hq, Hkv, D, C + K, shared=30)
    o, lse, status = r.run()
    assert (status == 0).all()
    r.check(o, lse, "long runs", (1, C // 2))
    o2, lse2, _ = r.run()
    assert np.array_equal(o, o2) and np.array_equal(lse, lse2)


@pytest.mark.parametrize("lens,K,Hq,Hkv,D", [((40000,), 5, 16, 1, 128), ((12000,), 7, 8, 2, 128), ((10800, 20000), 5, 32, 4, 128), ((9000, 0, 70, 2000), 8, 16, 1, 64),
                                             ((30000, 1), 3, 4, 1, 64), ((5000,), 64, 2, 1, 128), ((7000, 300, 8000), 1, 1, 1, 64)])
def test_draft_of_many_records(lens, K, Hq, Hkv, D):
    """Few long requests, whose merge four waves make for each row: up to 200 records a request, and requests of one or none.  A page
    outside the pool, in the middle, is flagged, and its keys count for nothing."""
    print(f"case block records {lens} K={K} Hq={Hq} D={D}", flush=True)
    r = BlockRun(lens, K, Hq, Hkv, D, 5100 + K + len(lens))
    o, lse, status = r.run()
    assert (status == 0).all()
    r.check(o, lse, "records")
    o2, lse2, _ = r.run()
    assert np.array_equal(o, o2) and np.array_equal(lse, lse2)
    bad = -(-lens[0] // 64) // 2
    r.bt[0, bad] = r.shape.n_pages
    o2, lse2, status = r.run()
    assert status.tolist() == [1] + [0] * (len(lens) - 1)
    assert np.array_equal(o[1:], o2[1:]) and np.array_equal(lse[1:], lse2[1:])
    k, v = (np.delete(x, slice(64 * bad, 64 * bad + 64), 0) for x in r.context(0))
    ro, rl = orc.draft_decode(*(bf16_bits_to_f64(x[0]) for x in r.host), k, v, r.shape.scale)
    assert rel_l2(o2[0], ro) <= REL and max_abs(lse2[0], rl) <= LSE_ABS


@pytest.mark.parametrize("K,Hq,D", [(2, 8, 64), (5, 8, 64), (16, 8, 64), (2, 8, 128), (5, 8, 128), (16, 8, 128)])
def test_draft_of_more_than_a_thousand_requests(K, Hq, D):
    """The first number of requests that take a workgroup each whatever they are long; one of them has more pages than lanes for every
    stream."""
    print(f"case block thousand K={K} D={D}", flush=True)
    C = 1025
    rng = np.random.default_rng(K)
    lens = rng.integers(0, 150, C)
    lens[0], lens[700] = 0, 40000
    r = BlockRun(tuple(int(x) for x in lens), K, Hq, 1, D, 5000 + K, shared=30)
    o, lse, status = r.run()
    assert (status == 0).all()
    r.check(o, lse, "thousand", (0, 1, 500, 700, 701, C - 1))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("K", [5, 40])
def test_draft_keeps_masked_values_out(K, D):
    """NaN and infinities of new positions that a row does not see leave the row as it is, bit for bit; rows that see them show them."""
    print(f"case block masked NaN K={K} D={D}", flush=True)
    r = BlockRun((150, 0), K, 6, 2, D, 3200)
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


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("K,Hq,Hkv", ROWS)
def test_draft_shows_nan_that_the_cache_holds(K, Hq, Hkv, D):
    """A scale of NaN in V is NaN in its 32 features and in no others, in K it is NaN in all of the head's rows; also of the last
    token, whether the places behind it are masked or not."""
    print(f"case block NaN in the cache K={K} Hq={Hq} D={D}", flush=True)
    r = BlockRun((100, 100, 100, 64, 65, 95, 96, 1), K, Hq, Hkv, D, 3300)
    clean, clean_lse, _ = r.run()
    r.scales[1].view(torch.uint8)[int(r.table[1, 0]), Hkv - 1, 10, 1] = 255
    r.scales[0].view(torch.uint8)[int(r.table[2, 1]), 0, 3, D // 32 - 1] = 255
    for c in range(3, len(r.lens)):
        n = r.lens[c]
        r.scales[1].view(torch.uint8)[int(r.table[c, (n - 1) // 64]), 0, (n - 1) % 64, 0] = 255
    o, lse, status = r.run()
    group = Hq // Hkv
    assert (status == 0).all() and np.array_equal(o[0], clean[0]) and np.array_equal(lse[1], clean_lse[1])
    assert np.isnan(o[1, :, -group:, 32:64]).all() and np.isfinite(np.delete(o[1, :, -group:], slice(32, 64), 2)).all()
    assert np.array_equal(np.delete(o[1], slice(32, 64), 2), np.delete(clean[1], slice(32, 64), 2)) and np.array_equal(o[1, :, :-group], clean[1, :, :-group])
    assert np.isnan(o[2, :, :group]).all() and np.isnan(lse[2, :group]).all() and np.array_equal(o[2, :, group:], clean[2, :, group:])
    for c in range(3, len(r.lens)):
        assert np.isnan(o[c, :, :group, :32]).all() and np.array_equal(o[c, ..., 32:], clean[c, ..., 32:]) and np.array_equal(lse[c], clean_lse[c]), c


@pytest.mark.parametrize("D", [64, 128])
def test_draft_reads_every_code_and_scale(D):
    """Keys of zero weigh all values alike: each output is the mean of one feature's codes times their scales.  All codes stand in every
    feature's column, scales differ from token to token and block to block."""
    print(f"case block codes D={D}", flush=True)
    n, Hkv = 256, 2
    rng = np.random.default_rng(3400)
    r = BlockRun((n,), 1, 2, Hkv, D, 3400, spare=0)
    for low, high in ((127, 128), (120, 134), (27, 31), (220, 224), (40, 43)):
        r.pages[0].view(torch.uint8).zero_()
        codes = (np.arange(n).reshape(4, 1, 64, 1) + np.arange(D) + np.arange(Hkv)[:, None, None]) % 16
        r.pages[1] = _packed(codes).cuda().view(F4)
        r.scales[1] = torch.from_numpy(rng.integers(low, high, (4, Hkv, 64, D // 32)).astype(np.uint8)).cuda().view(E8M0)
        r.scales[0].view(torch.uint8).fill_(127)
        r.k.zero_()
        r.v.zero_()
        r.host[1][:], r.host[2][:] = 0, 0
        o, lse, _ = r.run()
        ro, rl = r.oracle(0)
        size = np.abs(r.context(0)[1]).mean(0)                # [Hkv, D]: what the mean's terms add up to
        # fp32 sums of 256 terms and one rounding to bf16 (a probability of 1 is exact)
        assert (np.abs(o[0, 0] - ro[0]) <= 2.0**-8 * np.abs(ro[0]) + 2.0**-15 * size).all(), (low, high)
        assert max_abs(lse, rl) <= 1e-5


@pytest.mark.parametrize("D", [64, 128])
def test_draft_widens_every_code_with_every_scale(D):
    """One cached token a request has all the weight, so that O is its value: every code under every scale, in every block."""
    print(f"case block every code and scale D={D}", flush=True)
    C, Hkv = 256, 2
    shape = pe.DecodeShape(C, 1, Hkv, Hkv, D, C, 1, 1.0)
    q = torch.zeros((C, 1, Hkv, D), dtype=torch.bfloat16, device="cuda")
    k, v_new = torch.zeros_like(q), torch.zeros_like(q)
    q[..., 0], k[..., 0] = 300.0, -1.0
    keys, codes = np.zeros((C, Hkv, 64, D), dtype=np.uint8), np.full((C, Hkv, 64, D), 7, dtype=np.uint8)
    keys[..., 0] = 2                                           # 1: 300 above the new key
    codes[:, :, 0] = (np.arange(D) + np.arange(Hkv)[:, None]) % 16
    scales = np.full((C, Hkv, 64, D // 32), 255, dtype=np.uint8)
    scales[:, :, 0] = (np.arange(C)[:, None, None] + 37 * np.arange(D // 32)) % 256
    ones = torch.full(scales.shape, 127, dtype=torch.uint8, device="cuda").view(E8M0)
    table, lens = torch.arange(C, dtype=torch.int32, device="cuda")[:, None].contiguous(), torch.ones(C, dtype=torch.int32, device="cuda")
    o, lse, status = torch.empty_like(q), torch.empty((C, Hkv, 1), device="cuda"), torch.empty_like(lens)
    ws = torch.empty(pe.peagle_draft_decode_block_scaled_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    pe.peagle_draft_decode_block_scaled(shape, q, k, v_new, _packed(keys).cuda().view(F4), _packed(codes).cuda().view(F4), ones,
                                        torch.from_numpy(scales).cuda().view(E8M0), table, lens, o, lse, status, ws)
    want = orc.cache_values_blocks(codes[:, :, 0], scales[:, :, 0])
    got = bf16_to_f64(o)[:, 0]
    assert not status.any()
    assert np.array_equal(got, np.where(np.abs(want) < 2.0**-126, 0.0, _as_bf16(want)), equal_nan=True)
    inside = (scales[:, :, 0] >= 2) & (scales[:, :, 0] <= 252)  # (the range that the header names)
    inside = np.repeat(inside, 32, -1)
    assert np.array_equal(got[inside], want[inside]) and not np.array_equal(got[~inside], want[~inside], equal_nan=True)


def test_draft_large_logits():
    print("case block large logits", flush=True)
    for D in (64, 128):
        r = BlockRun((700, 90), 5, 16, 2, D, 3500, gain=8.0)
        o, lse, status = r.run()
        for c in range(2):
            ro, rl = r.oracle(c)
            assert rel_l2(o[c], ro) <= REL and max_abs(lse[c], rl) <= 8 * LSE_ABS and (status == 0).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("K,Hq,Hkv", ROWS)
def test_draft_large_values_under_keys_that_stand_out(K, Hq, Hkv, D):
    """Values up to 2^101 whose keys score 24 or 32 powers of two above those before them: what is summed for them must stay far from
    what fp32 holds at most.  Most tokens' values are small, on either side of them."""
    print(f"case block large values K={K} Hq={Hq} D={D}", flush=True)
    r = BlockRun((64 * 30, 100, 64 * 3 + 50), K, Hq, Hkv, D, 4200 + K, scale=float(np.log(2)), spare=0)
    keys = np.zeros((r.shape.n_pages, Hkv, 64, D), dtype=np.uint8)
    keys[0::2, :, 40, 0], keys[1::2, :, 40, 0] = 5, 6          # 3 * 2^3 and 4 * 2^3
    r.pages[0] = _packed(keys).cuda().view(F4)
    r.scales[0].view(torch.uint8).fill_(130)
    scales = torch.full(r.scales[1].shape, 120, dtype=torch.uint8)
    scales[:, :, 35:41] = 127 + 98
    r.scales[1] = scales.cuda().view(E8M0)
    q, k, _ = (bf16_bits_to_f64(x).astype(np.float32) for x in r.host)
    q[..., 0] = 1.0
    r.host[0], r.host[1] = f32_to_bf16_bits(q), f32_to_bf16_bits(np.zeros_like(k))
    r.q, r.k = to_dev_bf16(r.host[0]), to_dev_bf16(r.host[1])
    o, lse, status = r.run()
    assert (status == 0).all()
    for c in range(len(r.lens)):
        ro, rl = r.oracle(c)
        assert np.isfinite(o[c]).all() and np.abs(ro).max() > 2.0**90, c
        assert rel_l2(o[c], ro) <= REL and max_abs(lse[c], rl) <= LSE_ABS, (c, rel_l2(o[c], ro))


def test_draft_replays_from_a_graph_and_runs_on_other_streams():
    """One graph of two calls that share a workspace, replayed with new queries, lengths and tables; the same on another stream."""
    print("case block draft graph", flush=True)
    r = BlockRun((1500, 70, 640), 5, 16, 2, 64, 3700)
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
def test_draft_stays_inside_its_buffers(K, Hq, Hkv, D, lens):
    print(f"case block draft guards K={K} D={D}", flush=True)
    r = BlockRun(lens, K, Hq, Hkv, D, 3800)
    g = Guarded()
    C = len(lens)
    r.o, r.lse, r.status = g.tensor("o", (C, K, Hq, D), torch.bfloat16), g.tensor("lse", (C, Hq, K), torch.float32), g.tensor("status", (C,), torch.int32)
    r.ws = g.tensor("workspace", (pe.peagle_draft_decode_block_scaled_workspace_bytes(r.shape),), torch.uint8)
    o, lse, status = r.run()
    g.check("drafting step")
    r.check(o, lse, "guards")
    r.status = None
    r.call()
    g.check("without status")


def test_draft_beyond_four_gigabytes():
    """Pools of 4.3 GB with the context's pages on both sides of byte 2^32."""
    print("case block draft beyond 2^32", flush=True)
    r = BlockRun((400,), 3, 8, 8, 128, 3900, spare=0)
    o, lse, _ = r.run()
    n_pages = 2**32 // (8 * 64 * 64) + 9
    where = torch.tensor([n_pages - 1, 3, n_pages - 9, 0, n_pages - 12, n_pages - 2, 70], device="cuda")
    order = r.bt[0].long()
    for i in range(2):
        pages = torch.full((n_pages, 8, 64, 64), 0x77, dtype=torch.uint8, device="cuda")
        scales = torch.full((n_pages, 8, 64, 4), 255, dtype=torch.uint8, device="cuda")
        pages[where], scales[where] = r.pages[i].view(torch.uint8)[order], r.scales[i].view(torch.uint8)[order]
        r.pages[i], r.scales[i] = pages.view(F4), scales.view(E8M0)
    r.bt[0] = where.int()
    r.shape = pe.DecodeShape(1, 3, 8, 8, 128, n_pages, 7)
    o2, lse2, status = r.run()
    assert (status == 0).all() and np.array_equal(o, o2) and np.array_equal(lse, lse2)


@pytest.mark.parametrize("C,ctx,columns,K,Hq,Hkv,D", [(16, 1000, 320, 7, 64, 8, 64), (3, 70, 1024, 5, 32, 4, 128), (1, 0, 300, 1, 4, 2, 64), (70, 300, 90, 8, 16, 1, 128)])
def test_draft_on_tables_wider_than_any_context(C, ctx, columns, K, Hq, Hkv, D):
    print(f"case block wide table C={C} columns={columns} D={D}", flush=True)
    rng = np.random.default_rng(columns)
    r = BlockRun(tuple(int(x) for x in rng.integers(0, ctx + 1, C)), K, Hq, Hkv, D, 4400 + C)
    r.table = np.pad(r.table, ((0, 0), (0, columns - r.shape.max_pages)), constant_values=-1)
    r.bt = torch.from_numpy(r.table).cuda()
    r.shape = pe.DecodeShape(C, K, Hq, Hkv, D, r.shape.n_pages, columns)
    r.ws = torch.empty(pe.peagle_draft_decode_block_scaled_workspace_bytes(r.shape), dtype=torch.uint8, device="cuda").fill_(0x7F)
    o, lse, status = r.run()
    assert (status == 0).all()
    r.check(o, lse, "wide", range(0, C, max(1, C // 8)))


def test_two_drafting_steps_at_once():
    """Two streams, a workspace each: as one after the other."""
    print("case block two streams", flush=True)
    a, b = BlockRun((900, 70, 640, 2000), 7, 64, 8, 64, 4500), BlockRun((300, 1800), 8, 64, 4, 128, 4501)
    want = a.run(), b.run()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for x, stream in zip((a, b), streams):
        x.o.fill_(float("nan"))
        stream.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        for x, stream in zip((a, b), streams):
            x.call(stream)
    torch.cuda.synchronize()
    for x, w in zip((a, b), want):
        assert np.array_equal(bf16_to_f64(x.o), w[0]) and np.array_equal(x.lse.double().cpu().numpy(), w[1])


def test_calls_from_two_threads():
    """Each on a stream of its own, all three calls: as one after the other."""
    print("case block two threads", flush=True)
    runs = BlockRun((900, 70, 640, 2000), 7, 64, 8, 64, 4510), BlockRun((300, 1800), 8, 64, 4, 128, 4511)
    want = [r.run() for r in runs]
    rng = np.random.default_rng(19)
    rows = [torch.from_numpy(rng.standard_normal((90, 4, D))).bfloat16().cuda() for D in (64, 128)]
    torch.cuda.synchronize()
    got, errors = [None, None], []

    def work(i):
        try:
            stream, D, r = torch.cuda.Stream(), (64, 128)[i], runs[i]
            cache = Cache(np.random.default_rng(20 + i), 3, 4, D)
            with torch.cuda.stream(stream):
                k, v = torch.empty_like(rows[i]), torch.empty_like(rows[i])
                for n in range(30):
                    slots = _slots_on((np.arange(90) * 2 + n) % 192)
                    shape = pe.CacheShape(90, 4, D, 3)
                    pe.peagle_cache_append_block_scaled(shape, rows[i], rows[i], slots, *cache.pages, *cache.scales)
                    pe.peagle_cache_read(shape, slots, *cache.pages, *cache.scales, k, v)
                    r.call(stream)
                stream.synchronize()
            got[i] = k.clone(), v.clone(), bf16_to_f64(r.o), r.lse.double().cpu().numpy()
        except Exception as e:  # noqa: BLE001  (shown by the assertion below)
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    assert not errors and all(g is not None for g in got), errors
    for i, (k, v, o, lse) in enumerate(got):
        held = np.zeros((2, 4, 64, (64, 128)[i]), np.int64), np.zeros((2, 4, 64, (64, 128)[i] // 32), np.int64)
        orc.cache_append_blocks(bf16_to_f64(rows[i]), np.arange(90), *held)
        ref = orc.cache_values_blocks(*held).transpose(0, 2, 1, 3).reshape(128, 4, -1)[:90]
        assert np.array_equal(bf16_to_f64(k), ref) and np.array_equal(bf16_to_f64(v), ref)
        assert np.array_equal(o, want[i][0]) and np.array_equal(lse, want[i][1])


def test_binding_says_what_is_wrong_with_a_call():
    """Arguments that are not what the shape says are refused with their names before anything is launched; sizes may be any whole
    numbers."""
    print("case block binding", flush=True)
    cache = Cache(np.random.default_rng(13), 3, 2, 64)
    k = torch.zeros(5, 2, 64, dtype=torch.bfloat16, device="cuda")
    slots, shape = _slots_on(np.arange(5)), pe.CacheShape(5, 2, 64, 3)
    pools = *cache.pages, *cache.scales
    for call in (lambda s=shape, x=k, at=slots, p=pools, stream=None: pe.peagle_cache_append_block_scaled(s, x, x, at, *p, stream),
                 lambda s=shape, x=k, at=slots, p=pools, stream=None: pe.peagle_cache_read(s, at, *p, x, x, stream)):
        call()
        call(s=pe.CacheShape(np.int64(5), np.int32(2), 64, 3))
        for change, error, name in (({"x": k.float()}, TypeError, "k_"), ({"x": k[:4]}, ValueError, "k_"), ({"x": k.cpu()}, ValueError, "k_"),
                                    ({"x": torch.zeros(5, 64, 2, dtype=torch.bfloat16, device="cuda").transpose(1, 2)}, ValueError, "k_"),
                                    ({"at": slots.int()}, TypeError, "slots"), ({"at": slots[:3]}, ValueError, "slots"), ({"at": slots.cpu()}, ValueError, "slots"),
                                    ({"p": (pools[0].view(torch.uint8), *pools[1:])}, TypeError, "k_pages"),
                                    ({"p": (pools[0], pools[1][:2], *pools[2:])}, ValueError, "v_pages"),
                                    ({"p": (*pools[:2], pools[2].view(torch.uint8), pools[3])}, TypeError, "k_scale"),
                                    ({"p": (*pools[:3], pools[3].transpose(2, 3).contiguous())}, ValueError, "v_scale")):
            with pytest.raises(error, match=name):
                call(**change)
        with pytest.raises(pe.PeagleError):
            call(s=pe.CacheShape(5, 2, 64, 3), x=torch.zeros(5 * 132, dtype=torch.bfloat16, device="cuda").as_strided((5, 2, 64), (132, 64, 1)))
        with pytest.raises(ValueError, match="cuda:1"):
            call(stream=SimpleNamespace(cuda_stream=torch.cuda.current_stream().cuda_stream, device_index=1))
        call(stream=SimpleNamespace(cuda_stream=torch.cuda.current_stream().cuda_stream))
    cache.check_read(np.arange(5, 192), "untouched")
    r = BlockRun((70, 3), 3, 8, 2, 64, 4600)
    good = r.run()
    for name, x, error in (("q", r.q.float(), TypeError), ("k", r.k[:1], ValueError), ("o", r.o.transpose(1, 2).contiguous(), ValueError),
                           ("bt", r.bt.long(), TypeError), ("cl", r.cl.cpu(), ValueError), ("lse", r.lse.half(), TypeError), ("ws", r.ws.int(), TypeError),
                           ("status", r.status.long(), TypeError)):
        kept = getattr(r, name)
        setattr(r, name, x)
        with pytest.raises(error):
            r.call()
        setattr(r, name, kept)
    kept, r.ws = r.ws, r.ws[:16]
    with pytest.raises(pe.PeagleError):
        r.call()
    r.ws = kept
    again = r.run()
    assert all(np.array_equal(x, y) for x, y in zip(good, again))


def test_draft_equals_the_bf16_step_on_what_the_cache_reads_as():
    """A request that moves to the bf16 cache: both steps on the same values agree to their roundings of probabilities and outputs."""
    print("case block against bf16", flush=True)
    for D, Hq, Hkv in ((64, 64, 8), (128, 32, 4)):
        r = BlockRun((1000, 64, 333, 0), 7, Hq, Hkv, D, 3600, spare=0)
        o, lse, _ = r.run()
        n_pages = r.shape.n_pages
        wide = [torch.empty((n_pages * 64, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        pe.peagle_cache_read(pe.CacheShape(n_pages * 64, Hkv, D, n_pages), torch.arange(n_pages * 64, device="cuda"), *r.pages, *r.scales, *wide)
        pools = [x.view(n_pages, 64, Hkv, D).transpose(1, 2).contiguous() for x in wide]
        ws = torch.empty(pe.peagle_draft_decode_workspace_bytes(r.shape), dtype=torch.uint8, device="cuda")
        pe.peagle_draft_decode(r.shape, r.q, r.k, r.v, *pools, r.bt, r.cl, r.o, r.lse, r.status, ws)
        torch.cuda.synchronize()
        assert rel_l2(o, bf16_to_f64(r.o)) <= 4 * 2.0**-9 and max_abs(lse, r.lse.double().cpu().numpy()) <= 4e-3 + LSE_ABS


def test_plan_append_read_and_draft_as_a_serving_loop_runs_them():
    """Prompts admitted, stored, read back and drafted from; accepted tokens appended, rejected ones rolled back, a request replaced:
    the rows read are the oracle's to the bit, every draft equals the oracle on them, and they are off from the tokens themselves by
    no more than E2M1's rounding (half a step of its values, 2^-2 relative, in norm)."""
    print("case block serving loop", flush=True)
    rng = np.random.default_rng(11)
    C, K, Hq, Hkv, D, n_pages, cols = 3, 4, 8, 2, 64, 40, 10
    dev = lambda x, t: torch.from_numpy(np.asarray(x)).to(t).cuda()
    plan = pe.PlanShape(C, cols, n_pages, 512)
    held, free, count = dev([0] * C, torch.int32), dev(rng.permutation(n_pages), torch.int32), dev([n_pages], torch.int32)
    table = torch.full((C, cols), -1, dtype=torch.int32, device="cuda")
    start, slots = dev([0] * (C + 1), torch.int32), dev([0] * 512, torch.int64)
    seq_len, status = dev([0] * C, torch.int32), dev([0] * C, torch.int32)
    ws = torch.empty(pe.peagle_cache_plan_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
    cache = Cache(rng, n_pages, Hkv, D)
    shape = pe.DecodeShape(C, K, Hq, Hkv, D, n_pages, cols)
    draft_ws = torch.empty(pe.peagle_draft_decode_block_scaled_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    o, lse = torch.empty((C, K, Hq, D), dtype=torch.bfloat16, device="cuda"), torch.empty((C, Hq, K), device="cuda")
    kept = [[np.zeros((0, Hkv, D)) for _ in range(C)] for _ in range(2)]   # unrounded tokens of each request
    new_lens = [[70, 200, 5], [4, 1, 3], [0, 60, 4], [64, 2, 100], [1, 1, 1]]
    for step, new in enumerate(new_lens):
        if step == 3:
            kept = [[x[:max(0, len(x) - 2)] if c != 1 else x[:0] for c, x in enumerate(side)] for side in kept]
        ctx = [len(x) for x in kept[0]]
        pe.peagle_cache_plan(plan, dev(ctx, torch.int32), dev(new, torch.int32), held, free, count, table, start, slots, seq_len, status, ws)
        bits = [f32_to_bf16_bits(rng.standard_normal((512, Hkv, D), dtype=np.float32) * (step + 1)) for _ in range(2)]
        pe.peagle_cache_append_block_scaled(pe.CacheShape(512, Hkv, D, n_pages), *(to_dev_bf16(b) for b in bits), slots, *cache.pages, *cache.scales)
        q, kn, vn = (f32_to_bf16_bits(rng.standard_normal(s, dtype=np.float32)) for s in ((C, K, Hq, D), (C, K, Hkv, D), (C, K, Hkv, D)))
        draft_status = torch.full((C,), -1, dtype=torch.int32, device="cuda")
        pe.peagle_draft_decode_block_scaled(shape, to_dev_bf16(q), to_dev_bf16(kn), to_dev_bf16(vn), *cache.pages, *cache.scales, table, seq_len, o, lse,
                                            draft_status, draft_ws)
        torch.cuda.synchronize()
        assert status.tolist() == [0] * C and draft_status.tolist() == [0] * C and start.tolist() == [0, *np.cumsum(new)]
        at, host_table = slots.cpu().numpy(), table.cpu().numpy()
        for i in range(2):
            orc.cache_append_blocks(bf16_bits_to_f64(bits[i]), at, cache.codes[i], cache.exps[i])
            for c in range(C):
                kept[i][c] = np.concatenate([kept[i][c], bf16_bits_to_f64(bits[i][sum(new[:c]):sum(new[:c + 1])])])
        cache.check(step)
        for c in range(C):
            n = len(kept[0][c])
            pos = np.arange(n)
            there = host_table[c, pos // 64].astype(np.int64) * 64 + pos % 64
            rows = [bf16_to_f64(x) for x in cache.read(there)]
            assert all(np.array_equal(x, cache.values(i, there)) for i, x in enumerate(rows))
            ro, rl = orc.draft_decode(*(bf16_bits_to_f64(x[c]) for x in (q, kn, vn)), *rows, shape.scale)
            assert rel_l2(bf16_to_f64(o[c]), ro) <= REL and max_abs(lse[c].double().cpu().numpy(), rl) <= 8 * LSE_ABS, (step, c)
            assert all(rel_l2(rows[i], kept[i][c]) <= 2.0**-2 for i in range(2))
