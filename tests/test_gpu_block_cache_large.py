"""GPU tests of appends to and reads from a paged cache on both sides of the size from which rows no longer stay in the device's
caches: dense rows of both head sizes, all three types, some hundred of them against the oracle (numpy, 64 bits) to the bit."""
import numpy as np
import pytest
import torch

import paper_2602_01469_amd as pe
from gpu_harness import bf16_to_f64
from oracle import peagle_oracle as orc
from test_gpu_block_cache import E8M0, F4, TYPES, _rand, _slots_on, _unpacked

pytestmark = pytest.mark.gpu

LINE = 72 << 20  # bytes of K and V


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _some(rng, n):
    """Tokens at the ends, around multiples of what a wave and a workgroup take, and anywhere."""
    at = np.concatenate([np.arange(70), n - 1 - np.arange(70), n // 2 + np.arange(-40, 40), rng.integers(0, n, 400)])
    return np.unique(at)


def _slots(rng, n, spare):
    """Places of n tokens in pages in any order, from within a page on; number of pages."""
    n_pages = (n + 40 + 63) // 64 + spare
    pos = np.arange(n) + 40
    return rng.permutation(n_pages)[pos // 64] * 64 + pos % 64, n_pages


SIZES = [pytest.param(Hkv, D, LINE // (Hkv * D * 4) + more, id=f"{Hkv}x{D}{more:+d}") for Hkv, D in ((4, 128), (8, 64), (1, 128)) for more in (0, 1)]
SIZES += [pytest.param(4, 128, 65600, id="4x128, 134 MB"), pytest.param(8, 64, 65601, id="8x64, 134 MB")]


@pytest.mark.parametrize("Hkv,D,n", SIZES)
def test_append_and_read_of_dense_rows(Hkv, D, n):
    """Codes, scales and rows of some tokens are the oracle's; every block of every other token's row is off by at most a rounding;
    places of no token stay."""
    print(f"case dense rows n={n} Hkv={Hkv} D={D}", flush=True)
    rng, g = np.random.default_rng(n), torch.Generator(device="cuda").manual_seed(n)
    slots, n_pages = _slots(rng, n, 2)
    pages = [torch.full((n_pages, Hkv, 64, D // 2), 0x55, dtype=torch.uint8, device="cuda").view(F4) for _ in range(2)]
    scales = [torch.full((n_pages, Hkv, 64, D // 32), 9, dtype=torch.uint8, device="cuda").view(E8M0) for _ in range(2)]
    k, v, at = _rand(g, n, Hkv, D, scale=3), _rand(g, n, Hkv, D), _slots_on(slots)
    out = [torch.full_like(k, 7.0) for _ in range(2)]
    shape = pe.CacheShape(n, Hkv, D, n_pages)
    pe.peagle_cache_append_block_scaled(shape, k, v, at, *pages, *scales)
    pe.peagle_cache_read(shape, at, *pages, *scales, *out)
    some = _some(rng, n)
    rows = torch.from_numpy(some).cuda()
    free = torch.from_numpy(np.setdiff1d(np.arange(n_pages * 64), slots)).cuda()
    for x, y, p, s in zip((k, v), out, pages, scales):
        m = -(-len(some) // 64)
        codes, exps = np.zeros((m, Hkv, 64, D), dtype=int), np.zeros((m, Hkv, 64, D // 32), dtype=int)
        orc.cache_append_blocks(bf16_to_f64(x[rows]), np.arange(len(some)), codes, exps)
        flat = lambda a: a.transpose(0, 2, 1, 3).reshape(m * 64, Hkv, -1)[:len(some)]
        held_p, held_s = (t.view(torch.uint8).transpose(1, 2).flatten(0, 1) for t in (p, s))
        assert np.array_equal(held_s[at[rows]].cpu().numpy(), flat(exps)) and np.array_equal(_unpacked(held_p[at[rows]]), flat(codes))
        assert np.array_equal(bf16_to_f64(y[rows]), flat(orc.cache_values_blocks(codes, exps)))
        assert bool((held_s[free] == 9).all()) and bool((held_p[free] == 0x55).all())
        # between 3 and 6 scales two codes are at most two scales apart, and the block's largest value is above 3 scales: half of two
        # scales is less than a third of it
        x, y = (t.float().unflatten(-1, (-1, 32)) for t in (x, y))
        assert bool(((y - x).abs() <= x.abs().amax(-1, keepdim=True) / 3).all())


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2", "e2m1"])
@pytest.mark.parametrize("Hkv,D,n", SIZES)
def test_read_of_dense_rows(Hkv, D, n, fmt):
    """Any codes and scales that are normal numbers in bf16, tokens in any order, some outside the pool; K and V side by side."""
    print(f"case dense reads n={n} Hkv={Hkv} D={D} {fmt}", flush=True)
    rng, g = np.random.default_rng(n + 1), torch.Generator(device="cuda").manual_seed(n + 1)
    four = fmt == "e2m1"
    n_pages = 700
    width, blocks = (D // 2, (64, D // 32)) if four else (D, ())
    pages, scales = [], []
    for _ in range(2):
        raw = torch.randint(0, 256, (n_pages, Hkv, 64, width), generator=g, device="cuda", dtype=torch.uint8)
        if not four:
            raw &= 0xBB  # (no infinity, no NaN)
        pages.append(raw.view(F4 if four else TYPES[fmt]))
        scales.append(torch.randint(60, 180, (n_pages, Hkv, *blocks), generator=g, device="cuda", dtype=torch.uint8).view(E8M0))
    slots = rng.integers(0, 64 * n_pages, n)
    slots[rng.integers(0, n, 50)] = -1
    out = torch.full((n, 2, Hkv, D), 7.0, dtype=torch.bfloat16, device="cuda")
    pe.peagle_cache_read(pe.CacheShape(n, Hkv, D, n_pages), _slots_on(slots), *pages, *scales, out[:, 0], out[:, 1])
    some = np.unique(np.concatenate([_some(rng, n), np.flatnonzero(slots < 0)]))
    there, at = slots[some] >= 0, np.maximum(slots[some], 0)
    page, off = torch.from_numpy(at // 64).cuda(), torch.from_numpy(at % 64).cuda()
    for i in range(2):
        raw, s = pages[i].view(torch.uint8)[page, :, off], scales[i].view(torch.uint8)
        if four:
            want = orc.f4_widen(_unpacked(raw)).astype(np.float64) * np.exp2(np.repeat(s[page, :, off].cpu().numpy().astype(np.float64), 32, -1) - 127)
        else:
            want = raw.view(TYPES[fmt]).double().cpu().numpy() * np.exp2(s[page].cpu().numpy().astype(np.float64) - 127)[..., None]
        assert np.array_equal(bf16_to_f64(out[torch.from_numpy(some).cuda(), i]), np.where(there[:, None, None], want, 0.0))
    assert not bool((out == 7.0).all(-1).any())
