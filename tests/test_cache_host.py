"""Host-only tests of the serving operators around the paged cache: the oracle's 8-bit rounding against the library type
conversions, its plan on hand-made examples, and the refusals of the C ABI and of the binding (arguments are validated before
anything is launched, so no GPU is needed)."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2602_01469_amd as pe
from oracle import peagle_oracle as orc
from paper_2602_01469_amd import binding

EINVAL, ENULL, EUNSUPPORTED, EWORKSPACE = -1, -2, -5, -6
TYPES = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
PTR = C.c_void_p(256)  # never dereferenced: every call below is refused first


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_oracle_rounds_as_the_type_conversion_does(fmt):
    rng = np.random.default_rng(1)
    largest = orc.F8[fmt][2]
    x = np.concatenate([rng.standard_normal(20000) * np.exp2(rng.uniform(-24, 7, 20000)), [0.0, largest, -largest],
                        np.exp2(np.arange(-20.0, 8)), 1.5 * np.exp2(np.arange(-20.0, 8)), np.arange(-33, 34) / 1024])
    x = x.astype(np.float32)
    got, want = orc.f8_round(x, fmt), torch.from_numpy(x).to(TYPES[fmt]).double().numpy()
    assert np.array_equal(got, want)
    odd = np.array([np.nan, np.inf, -np.inf], dtype=np.float32)
    assert np.array_equal(orc.f8_round(odd, fmt), torch.from_numpy(odd).to(TYPES[fmt]).double().numpy(), equal_nan=True)
    every = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(TYPES[fmt]).double().numpy()
    every = every[np.isfinite(every)]
    assert np.array_equal(orc.f8_round(every, fmt), every) and np.abs(every).max() == largest


def test_oracle_scale_is_the_smallest_power_of_two_that_holds_the_largest_value():
    for fmt, largest in (("e4m3", 448.0), ("e5m2", 57344.0)):
        assert orc.scale_exponent(largest, fmt) == 0 and orc.scale_exponent(np.nextafter(largest, np.inf), fmt) == 1
        assert orc.scale_exponent(largest / 2, fmt) == -1 and orc.scale_exponent(0.0, fmt) == -100
        assert largest * 2.0 ** orc.scale_exponent(3.3895313892515355e38, fmt) >= 3.3895313892515355e38


def test_oracle_append_on_a_page_in_two_runs():
    pages, exps = np.full((2, 1, 64, 1), 7.0), np.array([[5], [9]])
    orc.cache_append(np.array([[[448.0]], [[-3.0]]]), np.array([64, 65]), pages, exps, "e4m3")
    assert exps.tolist() == [[5], [0]] and pages[1, 0, :2, 0].tolist() == [448.0, -3.0] and (pages[1, 0, 2:] == 7).all()
    orc.cache_append(np.array([[[900.0]]]), np.array([66]), pages, exps, "e4m3")           # 900 needs 2^2
    assert exps.tolist() == [[5], [2]] and pages[1, 0, :3, 0].tolist() == [112.0, -0.75, 224.0]  # 225: halfway, to even
    orc.cache_append(np.array([[[0.25]]]), np.array([67]), pages, exps, "e4m3")
    assert exps.tolist() == [[5], [2]] and pages[1, 0, 3, 0] == 0.0625 and (pages[0] == 7).all()


def test_oracle_plan_takes_gives_back_and_restores():
    table = np.full((3, 4), -1)
    table[0, :2] = [5, 6]
    free = np.array([9, 8, 7, 4, 3, 2, 0, 0, 0, 0])
    r = orc.cache_plan([100, 0, 0], [29, 1, 65], [2, 0, 0], free, 6, table, 100)
    assert r["status"].tolist() == [0, 0, 0] and r["pages_held"].tolist() == [3, 1, 2] and r["free_count"][0] == 2
    assert r["block_table"].tolist() == [[5, 6, 2, -1], [3, -1, -1, -1], [4, 7, -1, -1]]
    assert r["token_start"].tolist() == [0, 29, 30, 95] and r["seq_len"].tolist() == [129, 1, 65]
    assert r["slots"][:30].tolist() == [6 * 64 + 36 + i for i in range(28)] + [2 * 64, 3 * 64]
    assert r["slots"][94] == 7 * 64 and (r["slots"][95:] == -1).all()
    back = orc.cache_plan([100, 0, 0], [0, 0, 0], r["pages_held"], r["free_pages"], int(r["free_count"][0]), r["block_table"], 100)
    assert back["free_count"][0] == 6 and np.array_equal(back["free_pages"], free) and back["pages_held"].tolist() == [2, 0, 0]
    short = orc.cache_plan([100, 0, 0], [29, 65, 0], [2, 0, 0], free, 2, table, 100)       # one page, then two where one is left
    assert short["status"].tolist() == [0, 2, 0] and short["free_count"][0] == 1 and short["seq_len"].tolist() == [129, 0, 0]


def _plan_call(shape, **change):
    names = ["ctx_len", "new_len", "pages_held", "pages_held_out", "free_pages", "free_count", "free_count_out", "block_table",
             "token_start", "slots", "seq_len", "status", "workspace"]
    args = [change.get(n, PTR) for n in names]
    c = binding._PlanShapeC(*shape)
    need = pe.load_library().peagle_cache_plan_workspace_bytes(C.byref(c))
    return pe.load_library().peagle_cache_plan(C.byref(c), *args, change.get("ws_bytes", need), None)


@pytest.mark.parametrize("shape,rc", [((0, 4, 8, 8), EINVAL), ((-1, 4, 8, 8), EINVAL), ((4, 0, 8, 8), EINVAL), ((4, 4, 0, 8), EINVAL),
                                      ((4, 4, 8, 0), EINVAL), ((65536, 4, 8, 8), EUNSUPPORTED), ((4, (1 << 24) + 1, 8, 8), EUNSUPPORTED),
                                      ((4, 4, (1 << 30) + 1, 8), EUNSUPPORTED), ((4, 4, 8, (1 << 30) + 1), EUNSUPPORTED)])
def test_plan_refuses_shapes(shape, rc):
    assert _plan_call(shape) == rc
    with pytest.raises(pe.PeagleError):
        pe.peagle_cache_plan_workspace_bytes(pe.PlanShape(*shape))


def test_plan_refuses_missing_arguments_and_short_workspaces():
    lib = pe.load_library()
    assert lib.peagle_cache_plan(None, *[PTR] * 13, 1 << 20, None) == ENULL
    for n in ("ctx_len", "new_len", "pages_held", "pages_held_out", "free_pages", "free_count", "free_count_out", "block_table",
              "token_start", "slots", "seq_len", "status"):
        assert _plan_call((4, 4, 8, 8), **{n: None}) == ENULL, n
    assert _plan_call((4, 4, 8, 8), workspace=None) == EWORKSPACE
    assert _plan_call((20, 4, 8, 8), ws_bytes=255) == EWORKSPACE
    assert _plan_call((4, 4, 8, 8), workspace=C.c_void_p(264)) == EINVAL
    assert pe.peagle_cache_plan_workspace_bytes(pe.PlanShape(20, 4, 8, 8)) == 512


def _append_call(change=None, k=PTR, v=PTR, slots=PTR, kp=PTR, vp=PTR, ks=PTR, vs=PTR):
    f = {"n_tokens": 5, "Hkv": 2, "D": 64, "n_pages": 8, "format": 0, "k_stride": 128, "v_stride": 128} | (change or {})
    c = binding._CacheShapeC(*f.values())
    return pe.load_library().peagle_cache_append_scaled(C.byref(c), k, v, slots, kp, vp, ks, vs, None)


@pytest.mark.parametrize("change,rc", [({"n_tokens": -1}, EINVAL), ({"Hkv": 0}, EINVAL), ({"n_pages": 0}, EINVAL), ({"D": 96}, EUNSUPPORTED),
                                       ({"format": 2}, EUNSUPPORTED), ({"format": -1}, EUNSUPPORTED), ({"n_tokens": (1 << 28) + 1}, EUNSUPPORTED),
                                       ({"Hkv": 65536, "k_stride": 1 << 23, "v_stride": 1 << 23}, EUNSUPPORTED),
                                       ({"n_pages": (1 << 30) + 1}, EUNSUPPORTED), ({"k_stride": 120}, EINVAL), ({"v_stride": 127}, EINVAL),
                                       ({"k_stride": 132}, EINVAL), ({"v_stride": -128}, EINVAL), ({"k_stride": 0}, EINVAL)])
def test_append_refuses_shapes(change, rc):
    assert _append_call(change) == rc


def test_append_refuses_missing_and_unaligned_pointers():
    assert pe.load_library().peagle_cache_append_scaled(None, *[PTR] * 7, None) == ENULL
    for n in ("k", "v", "slots", "kp", "vp", "ks", "vs"):
        assert _append_call(**{n: None}) == ENULL, n
    for n in ("k", "v", "kp", "vp"):
        assert _append_call(**{n: C.c_void_p(264)}) == EINVAL, n
    assert _append_call({"n_tokens": 0}, k=None, v=None, slots=None) == 0   # nothing to store: nothing is launched


def test_binding_refuses_tensors_that_are_not_what_the_shape_says():
    e4, e8, bf = torch.float8_e4m3fn, torch.float8_e8m0fnu, torch.bfloat16
    k = torch.zeros(5, 2, 64, dtype=bf)
    pool, scale, slots = torch.zeros(3, 2, 64, 64, dtype=e4), torch.zeros(3, 2, dtype=torch.uint8).view(e8), torch.zeros(5, dtype=torch.int64)
    shape = pe.CacheShape(5, 2, 64, 3)
    call = pe.peagle_cache_append_scaled
    with pytest.raises(TypeError, match="k_pages"):
        call(shape, k, k, slots, pool.to(bf), pool, scale, scale)
    with pytest.raises(TypeError, match="v_pages"):
        call(shape, k, k, slots, pool, pool.to(torch.float8_e5m2), scale, scale)
    with pytest.raises(ValueError, match="must live on the GPU"):
        call(shape, k, k, slots, pool, pool, scale, scale)
    plan = pe.PlanShape(2, 3, 4, 5)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    with pytest.raises(TypeError, match="workspace"):
        pe.peagle_cache_plan(plan, i32(2), i32(2), i32(2), i32(4), i32(1), i32(2, 3), i32(3), torch.zeros(5, dtype=torch.int64), i32(2),
                             i32(2), torch.zeros(256, dtype=torch.uint8))


def _draft_call(change=None, format_=0, **ptrs):
    f = {"C": 2, "K": 3, "Hq": 8, "Hkv": 2, "D": 64, "scale": 0.125, "n_pages": 8, "max_pages": 40} | (change or {})
    c = binding._DecodeShapeC(*f.values())
    lib = pe.load_library()
    names = ["q_new", "k_new", "v_new", "k_pages", "v_pages", "k_scale", "v_scale", "block_table", "ctx_len", "o", "lse", "status", "workspace"]
    need = lib.peagle_draft_decode_scaled_workspace_bytes(C.byref(c))
    return lib.peagle_draft_decode_scaled(C.byref(c), format_, *[ptrs.get(n, PTR) for n in names], ptrs.get("ws_bytes", need), None)


@pytest.mark.parametrize("change,rc", [({"C": 0}, EINVAL), ({"K": 0}, EINVAL), ({"Hkv": 0}, EINVAL), ({"Hkv": 3}, EINVAL), ({"n_pages": 0}, EINVAL),
                                       ({"max_pages": 0}, EINVAL), ({"scale": 0.0}, EINVAL), ({"scale": float("nan")}, EINVAL), ({"D": 96}, EUNSUPPORTED),
                                       ({"K": 33, "Hq": 8}, EUNSUPPORTED), ({"K": 65, "Hq": 2}, EUNSUPPORTED), ({"C": 65536}, EUNSUPPORTED),
                                       ({"max_pages": (1 << 24) + 1}, EUNSUPPORTED)])
def test_scaled_draft_refuses_shapes(change, rc):
    assert _draft_call(change) == rc
    f = {"C_": 2, "K": 3, "Hq": 8, "Hkv": 2, "D": 64, "n_pages": 8, "max_pages": 40}
    if "scale" not in change and "Hkv" not in change:
        shape = pe.DecodeShape(**(f | {("C_" if n == "C" else n): x for n, x in change.items()}))
        with pytest.raises(pe.PeagleError):
            pe.peagle_draft_decode_scaled_workspace_bytes(shape)


def test_scaled_draft_refuses_formats_pointers_and_workspaces():
    assert _draft_call(format_=2) == EUNSUPPORTED and _draft_call(format_=-1) == EUNSUPPORTED
    for n in ("q_new", "k_new", "v_new", "k_pages", "v_pages", "k_scale", "v_scale", "block_table", "ctx_len", "o", "lse"):
        assert _draft_call(**{n: None}) == ENULL, n
    for n in ("q_new", "k_new", "v_new", "k_pages", "v_pages", "o", "workspace"):
        assert _draft_call(**{n: C.c_void_p(264)}) == EINVAL, n
    assert _draft_call(workspace=None) == EWORKSPACE and _draft_call(ws_bytes=16) == EWORKSPACE


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows", [1, 32, 33, 64, 96, 97, 128])
def test_scaled_draft_workspaces_up_to_the_largest_shapes(rows, D):
    """What a workspace holds, at the ends of every dimension: two records of rows x (D + 4) floats for each workgroup that shares a
    KV head's work, and eight bytes a request.  There are no more workgroups than two for each of 256 compute units, or one a head."""
    pad256 = lambda n: -(-n // 256) * 256
    rows_pad = -(-rows // 32) * 32
    for C_ in (1, 2, 64, 1024, 1025, 65535):
        for Hkv in (1, 3, 8, 513, 65535):
            for max_pages in (1, 16, 17, 64, 65, 1023, 1 << 20, 1 << 24):
                shape = pe.DecodeShape(C_, 1, rows * Hkv, Hkv, D, 1 << 30, max_pages)
                total = pe.peagle_draft_decode_scaled_workspace_bytes(shape)
                size = lambda shares: pad256(2 * Hkv * shares * rows_pad * D * 4) + pad256(2 * Hkv * shares * rows_pad * 16) + pad256(8 * C_)
                most = -(-512 // Hkv)
                assert any(total == size(s) for s in range(most + 1)), (C_, Hkv, max_pages, total)
                if C_ > 1024 or max_pages == 1 or C_ * max_pages > 1 << 30:
                    assert total == size(0), (C_, Hkv, max_pages)


def test_plan_workspaces_up_to_the_largest_shapes():
    for C_ in (1, 16, 17, 1024, 65535):
        for other in (1, 1 << 24):
            assert pe.peagle_cache_plan_workspace_bytes(pe.PlanShape(C_, other, 1 << 30, 1 << 30)) == -(-16 * C_ // 256) * 256
