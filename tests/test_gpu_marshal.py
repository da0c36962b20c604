"""GPU tests of the binding's compiled part: it makes the calls that are as they have to be by itself, hands others back without
launching anything, and gives what the calls marshalled in Python give."""
import numpy as np
import pytest
import torch

import paper_2602_01469_amd as pe
from paper_2602_01469_amd import binding
from test_gpu_block_cache import BlockRun, Cache, _rand, _slots_on

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _bytes(*tensors):
    torch.cuda.synchronize()
    return [t.view(torch.uint8).cpu().numpy() for t in tensors]


def _same(a, b):
    return all(np.array_equal(x, y) for x, y in zip(a, b))


def _cache_call(D, n=75):
    g = torch.Generator(device="cuda").manual_seed(D)
    cache = Cache(np.random.default_rng(D), 4, 3, D)
    rows = _rand(g, n, 6 * D)  # (K and V side by side)
    k, v = rows[:, :3 * D].unflatten(1, (3, D)), rows[:, 3 * D:].unflatten(1, (3, D))
    return cache, pe.CacheShape(n, 3, D, 4), k, v, _slots_on(np.random.default_rng(1).permutation(256)[:n]), torch.empty_like(rows)


@pytest.mark.parametrize("D", [64, 128])
def test_well_formed_calls_are_made_by_the_compiled_part(D, monkeypatch):
    """With stream None and a stream; K and V contiguous or in wider rows; with and without `status`."""
    print(f"case marshal accepts D={D}", flush=True)
    fast = binding._fast()
    assert fast is not binding._Unmarshalled
    side = torch.cuda.Stream()
    cache, shape, k, v, slots, out = _cache_call(D)
    ko, vo = out[:, :3 * D].unflatten(1, (3, D)), out[:, 3 * D:].unflatten(1, (3, D))
    r = BlockRun((130, 0, 64), 5, 6, 3, D, 6000)
    draft = lambda status, stream: fast.draft_decode(r.shape, r.q, r.k, r.v, *r.pages, *r.scales, r.bt, r.cl, r.o, r.lse, status, r.ws, stream)
    held = [x.clone() for x in (*cache.pages, *cache.scales)]
    got = []
    for stream in (None, side, torch.cuda.current_stream()):
        for x, old in zip((*cache.pages, *cache.scales), held):
            x.view(torch.uint8).copy_(old.view(torch.uint8))
        out.fill_(3.0)
        r.o.fill_(float("nan"))
        torch.cuda.synchronize()
        assert fast.cache_append(shape, k, v, slots, *cache.pages, *cache.scales, stream) == 0
        assert fast.cache_read(shape, slots, *cache.pages, *cache.scales, ko, vo, stream) == 0
        assert draft(None, stream) == 0 and draft(r.status, stream) == 0
        got.append(_bytes(*cache.pages, *cache.scales, out, r.o, r.lse, r.status))
    monkeypatch.setattr(binding, "_marshal", binding._Unmarshalled)
    for x, old in zip((*cache.pages, *cache.scales), held):
        x.view(torch.uint8).copy_(old.view(torch.uint8))
    pe.peagle_cache_append_block_scaled(shape, k, v, slots, *cache.pages, *cache.scales)
    pe.peagle_cache_read(shape, slots, *cache.pages, *cache.scales, ko, vo)
    r.call()
    want = _bytes(*cache.pages, *cache.scales, out, r.o, r.lse, r.status)
    assert all(_same(x, want) for x in got)
    assert fast.cache_append(pe.CacheShape(0, 3, D, 4), k[:0], v[:0], slots[:0], *cache.pages, *cache.scales, None) == 0
    assert fast.cache_append(pe.CacheShape(1, 3, D, 4), k[:1], v[:1], slots[:1], *cache.pages, *cache.scales, None) == 0


@pytest.mark.parametrize("fmt", [torch.float8_e4m3fn, torch.float8_e5m2])
def test_reads_of_8_bit_caches_are_made_by_the_compiled_part(fmt):
    print(f"case marshal reads {fmt}", flush=True)
    pages = torch.zeros((3, 2, 64, 64), dtype=torch.uint8, device="cuda").view(fmt)
    scales = torch.full((3, 2), 127, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
    out = torch.full((2, 9, 2, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    shape, slots = pe.CacheShape(9, 2, 64, 3), torch.arange(9, device="cuda") * 20
    assert binding._fast().cache_read(shape, slots, pages, pages, scales, scales, out[0], out[1], None) == 0
    assert not bool(out.any())
    # (an append stores no such codes through this entry)
    assert binding._fast().cache_append(shape, out[0], out[1], slots, pages, pages, scales, scales, None) is None


def test_malformed_calls_are_handed_back_and_launch_nothing():
    print("case marshal hands back", flush=True)
    fast = binding._fast()
    D = 64
    cache, shape, k, v, slots, out = _cache_call(D)
    pools = (*cache.pages, *cache.scales)
    ko, vo = torch.full((75, 3, D), 3.0, dtype=torch.bfloat16, device="cuda"), torch.full((75, 3, D), 3.0, dtype=torch.bfloat16, device="cuda")
    r = BlockRun((130, 0, 64), 5, 6, 3, D, 6001)
    good = [r.shape, r.q, r.k, r.v, *r.pages, *r.scales, r.bt, r.cl, r.o, r.lse, r.status, r.ws, None]
    before = _bytes(*pools, ko, vo, r.o, r.lse, r.status)
    wrongs = lambda x: [x.cpu(), x[:-1], x.unsqueeze(0), x.float(), x.cpu().tolist(), None]
    plain = lambda x: x.view(torch.uint8)
    for i, x, more in ((1, k, [k.transpose(0, 2), k.transpose(1, 2).contiguous().transpose(1, 2)]), (2, v, [v[..., :32]]), (3, slots, [slots.repeat(2)[::2]])):
        for w in wrongs(x) + more:
            a = [shape, k, v, slots, *pools, None]
            a[i] = w
            assert fast.cache_append(*a) is None, i
    for i, x in ((1, slots), (6, ko), (7, vo)):
        for w in wrongs(x):
            a = [shape, slots, *pools, ko, vo, None]
            a[i] = w
            assert fast.cache_read(*a) is None, i
    for i in range(4):
        for w in (plain(pools[i]), pools[i].cpu(), pools[i][:3], pools[(i + 2) % 4], None):
            p = list(pools)
            p[i] = w
            assert fast.cache_append(shape, k, v, slots, *p, None) is None and fast.cache_read(shape, slots, *p, ko, vo, None) is None, i
    for i in range(1, 14):
        for w in (good[i].cpu(), plain(good[i].contiguous())[:1] if i != 13 else good[i].int(), "x"):
            a = list(good)
            a[i] = w
            assert fast.draft_decode(*a) is None, i
    for i in (1, 10):
        a = list(good)
        a[i] = good[i].transpose(1, 2).contiguous().transpose(1, 2)
        assert fast.draft_decode(*a) is None, i
    assert _same(_bytes(*pools, ko, vo, r.o, r.lse, r.status), before)
