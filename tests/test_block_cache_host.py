"""Host-only tests of the operators on a paged cache held in 4 bits: the oracle's rounding and append on hand-made examples, and the
refusals of the C ABI and of the binding (arguments are validated before anything is launched, so no GPU is needed)."""
import ctypes as C
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2602_01469_amd as pe
from oracle import peagle_oracle as orc
from paper_2602_01469_amd import binding

EINVAL, ENULL, EUNSUPPORTED, EWORKSPACE = -1, -2, -5, -6
PTR, OFF = C.c_void_p(256), C.c_void_p(264)  # never dereferenced: every call below is refused first
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_oracle_rounds_halfway_to_the_even_code():
    x = [0.0, 0.25, 0.2500001, 0.5, 0.75, 0.7499999, 1.25, 1.2500001, 1.75, 2.5, 2.4999, 2.5001, 3.5, 3.4999, 5.0, 5.0001, 6.0]
    want = [0, 0, 1, 1, 2, 1, 2, 3, 4, 4, 4, 5, 6, 5, 6, 7, 7]
    assert orc.f4_codes(np.array(x)).tolist() == want
    assert orc.f4_codes(-np.array(x)).tolist() == [c + 8 for c in want]
    assert np.array_equal(orc.f4_codes(orc.f4_widen(np.arange(16))), np.arange(16))


def test_oracle_appends_block_by_block():
    codes, scales = np.full((2, 1, 64, 64), 5), np.full((2, 1, 64, 2), 9)
    x = np.zeros((3, 1, 64))
    x[0, 0, 0], x[0, 0, 1], x[0, 0, 40] = 6.0, -0.75, 6.01       # 2^0; 2^1 for the second block: 3.005 -> 3
    x[1, 0, 3], x[1, 0, 63] = np.nan, -2.0**-104
    orc.cache_append_blocks(x, np.array([64 + 7, 3, 128]), codes, scales)
    assert scales[1, 0, 7].tolist() == [127, 128] and codes[1, 0, 7, [0, 1, 2, 40]].tolist() == [7, 10, 0, 5]
    assert scales[0, 0, 3].tolist() == [255, 27] and codes[0, 0, 3, [3, 63]].tolist() == [0, 8]
    values = orc.cache_values_blocks(codes, scales)
    assert values[1, 0, 7, [0, 1, 40]].tolist() == [6.0, -1.0, 6.0] and np.isnan(values[0, 0, 3, :32]).all() and not values[0, 0, 3, 32:].any()
    untouched = np.ones((2, 64), dtype=bool)
    untouched[1, 7] = untouched[0, 3] = False
    assert (codes[:, 0][untouched] == 5).all() and (scales[:, 0][untouched] == 9).all()


def _shape(change):
    f = {"n_tokens": 5, "Hkv": 2, "D": 64, "n_pages": 8, "format": 2, "k_stride": 128, "v_stride": 128} | (change or {})
    return C.byref(binding._CacheShapeC(*f.values()))


def _append_call(change=None, **ptrs):
    names = ["k", "v", "slots", "kp", "vp", "ks", "vs"]
    return pe.load_library().peagle_cache_append_block_scaled(_shape(change), *[ptrs.get(n, PTR) for n in names], None)


def _read_call(change=None, **ptrs):
    names = ["slots", "kp", "vp", "ks", "vs", "k", "v"]
    return pe.load_library().peagle_cache_read(_shape(change), *[ptrs.get(n, PTR) for n in names], None)


SHAPES = [({"n_tokens": -1}, EINVAL), ({"Hkv": 0}, EINVAL), ({"n_pages": 0}, EINVAL), ({"D": 96}, EUNSUPPORTED), ({"D": 32}, EUNSUPPORTED),
          ({"format": 3}, EUNSUPPORTED), ({"format": -1}, EUNSUPPORTED), ({"n_tokens": (1 << 28) + 1}, EUNSUPPORTED),
          ({"Hkv": 65536, "k_stride": 1 << 23, "v_stride": 1 << 23}, EUNSUPPORTED), ({"n_pages": (1 << 30) + 1}, EUNSUPPORTED),
          ({"k_stride": 120}, EINVAL), ({"v_stride": 127}, EINVAL), ({"k_stride": 132}, EINVAL), ({"v_stride": -128}, EINVAL), ({"k_stride": 0}, EINVAL)]


@pytest.mark.parametrize("change,rc", SHAPES)
def test_append_and_read_refuse_shapes(change, rc):
    assert _append_call(change) == rc and _read_call(change) == rc


def test_append_and_read_refuse_missing_and_unaligned_pointers():
    lib = pe.load_library()
    assert lib.peagle_cache_append_block_scaled(None, *[PTR] * 7, None) == ENULL and lib.peagle_cache_read(None, *[PTR] * 7, None) == ENULL
    for n in ("k", "v", "slots", "kp", "vp", "ks", "vs"):
        assert _append_call(**{n: None}) == ENULL and _read_call(**{n: None}) == ENULL, n
    for n in ("k", "v", "kp", "vp", "ks", "vs"):
        assert _append_call(**{n: OFF}) == EINVAL and _read_call(**{n: OFF}) == EINVAL, n
    for n in ("k", "v", "kp", "vp"):
        assert _read_call({"format": 0}, **{n: OFF}) == EINVAL and _read_call({"format": 1}, **{n: OFF}) == EINVAL, n
    for f in (0, 1):  # the append of 4-bit codes stores no others
        assert _append_call({"format": f}) == EUNSUPPORTED
    none = {"n_tokens": 0}  # nothing to store or read: nothing is launched
    assert _append_call(none, k=None, v=None, slots=None) == 0 and _read_call(none, k=None, v=None, slots=None) == 0


def test_binding_refuses_tensors_that_are_not_what_the_shape_says():
    f4, e8, bf = torch.float4_e2m1fn_x2, torch.float8_e8m0fnu, torch.bfloat16
    raw = lambda *s: torch.zeros(s, dtype=torch.uint8)
    k, slots = torch.zeros(5, 2, 64, dtype=bf), torch.zeros(5, dtype=torch.int64)
    pool, scale = raw(3, 2, 64, 32).view(f4), raw(3, 2, 64, 2).view(e8)
    shape = pe.CacheShape(5, 2, 64, 3)
    with pytest.raises(TypeError, match="k_pages"):
        pe.peagle_cache_append_block_scaled(shape, k, k, slots, raw(3, 2, 64, 32), pool, scale, scale)
    with pytest.raises(ValueError, match="k_pages"):
        pe.peagle_cache_append_block_scaled(shape, k, k, slots, raw(3, 2, 64, 64).view(f4), pool, scale, scale)
    with pytest.raises(ValueError, match="must live on the GPU"):
        pe.peagle_cache_append_block_scaled(shape, k, k, slots, pool, pool, scale, scale)
    with pytest.raises(TypeError, match="k_pages"):
        pe.peagle_cache_read(shape, slots, k, k, scale, scale, k, k)
    with pytest.raises(ValueError, match="must live on the GPU"):
        pe.peagle_cache_read(shape, slots, pool, pool, scale, scale, k, k)
    draft = pe.DecodeShape(2, 3, 8, 2, 64, 3, 1)
    with pytest.raises(TypeError, match="workspace"):
        pe.peagle_draft_decode_block_scaled(draft, *[k] * 3, pool, pool, scale, scale, slots, slots, k, k, None, raw(256))


def _draft_call(change=None, **ptrs):
    f = {"C": 2, "K": 3, "Hq": 8, "Hkv": 2, "D": 64, "scale": 0.125, "n_pages": 8, "max_pages": 40} | (change or {})
    c = binding._DecodeShapeC(*f.values())
    lib = pe.load_library()
    names = ["q_new", "k_new", "v_new", "k_pages", "v_pages", "k_scale", "v_scale", "block_table", "ctx_len", "o", "lse", "status", "workspace"]
    need = lib.peagle_draft_decode_block_scaled_workspace_bytes(C.byref(c))
    return lib.peagle_draft_decode_block_scaled(C.byref(c), *[ptrs.get(n, PTR) for n in names], ptrs.get("ws_bytes", need), None)


@pytest.mark.parametrize("change,rc", [({"C": 0}, EINVAL), ({"K": 0}, EINVAL), ({"Hkv": 0}, EINVAL), ({"Hkv": 3}, EINVAL), ({"n_pages": 0}, EINVAL),
                                       ({"max_pages": 0}, EINVAL), ({"scale": 0.0}, EINVAL), ({"scale": float("nan")}, EINVAL),
                                       ({"scale": float("inf")}, EINVAL), ({"D": 96}, EUNSUPPORTED), ({"K": 33, "Hq": 8}, EUNSUPPORTED),
                                       ({"K": 65, "Hq": 2}, EUNSUPPORTED), ({"C": 65536}, EUNSUPPORTED), ({"max_pages": (1 << 24) + 1}, EUNSUPPORTED)])
def test_draft_refuses_shapes(change, rc):
    assert _draft_call(change) == rc
    f = {"C_": 2, "K": 3, "Hq": 8, "Hkv": 2, "D": 64, "n_pages": 8, "max_pages": 40}
    if "scale" not in change and "Hkv" not in change:
        shape = pe.DecodeShape(**(f | {("C_" if n == "C" else n): x for n, x in change.items()}))
        with pytest.raises(pe.PeagleError):
            pe.peagle_draft_decode_block_scaled_workspace_bytes(shape)


def test_draft_refuses_pointers_and_workspaces():
    for n in ("q_new", "k_new", "v_new", "k_pages", "v_pages", "k_scale", "v_scale", "block_table", "ctx_len", "o", "lse"):
        assert _draft_call(**{n: None}) == ENULL, n
    for n in ("q_new", "k_new", "v_new", "k_pages", "v_pages", "k_scale", "v_scale", "o", "workspace"):
        assert _draft_call(**{n: OFF}) == EINVAL, n
    assert _draft_call(workspace=None) == EWORKSPACE and _draft_call(ws_bytes=16) == EWORKSPACE


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows", [1, 32, 33, 64, 96, 97, 128])
def test_draft_workspaces_up_to_the_largest_shapes(rows, D):
    """Two records of rows x (D + 4) floats for each workgroup that shares a KV head's work, and eight bytes a request, at the ends of
    every dimension; no more workgroups than two for each of 256 compute units, or one a head."""
    pad256 = lambda n: -(-n // 256) * 256
    rows_pad = -(-rows // 32) * 32
    for C_ in (1, 2, 64, 1024, 1025, 65535):
        for Hkv in (1, 3, 8, 513, 65535):
            for max_pages in (1, 16, 17, 64, 65, 1023, 1 << 20, 1 << 24):
                total = pe.peagle_draft_decode_block_scaled_workspace_bytes(pe.DecodeShape(C_, 1, rows * Hkv, Hkv, D, 1 << 30, max_pages))
                size = lambda shares: pad256(2 * Hkv * shares * rows_pad * D * 4) + pad256(2 * Hkv * shares * rows_pad * 16) + pad256(8 * C_)
                assert any(total == size(s) for s in range(-(-512 // Hkv) + 1)), (C_, Hkv, max_pages, total)


def test_host_code_is_clean_under_asan_and_ubsan(tmp_path_factory):
    """The tests above once more, on a build of the library whose host code carries both sanitizers."""
    if "PEAGLE_ATTN_LIB" in os.environ:
        pytest.skip("this is that run")
    from paper_2602_01469_amd import build as _build
    clang = "/opt/rocm/llvm/bin/clang"
    if not os.path.exists(clang):
        pytest.skip("no ROCm clang: cannot locate the sanitizer runtime")
    runtime = subprocess.run([clang, "-print-file-name=libclang_rt.asan-x86_64.so"], stdout=subprocess.PIPE, text=True, check=True).stdout.strip()
    if not os.path.isabs(runtime) or not os.path.exists(runtime):
        pytest.skip("AddressSanitizer runtime not found")
    # (a build takes two minutes: another test has left one where it ran before this one in this session)
    built = sorted(tmp_path_factory.getbasetemp().glob("**/libpeagle_attn_hostsan.so"))
    lib = str(built[-1]) if built else _build.build(sanitize_host_to=str(tmp_path_factory.mktemp("hostsan") / "libpeagle_attn_hostsan.so"))
    env = os.environ | {"PEAGLE_ATTN_LIB": lib, "LD_PRELOAD": " ".join(x for x in (os.environ.get("LD_PRELOAD", ""), runtime) if x),
                        "ASAN_OPTIONS": "detect_leaks=0:abort_on_error=0:exitcode=86", "UBSAN_OPTIONS": "print_stacktrace=1:halt_on_error=1:exitcode=87"}
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.abspath(__file__), "-x", "-q", "-p", "no:cacheprovider"], cwd=ROOT, env=env,
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=1500)
    assert "AddressSanitizer" not in r.stdout and "runtime error:" not in r.stdout, r.stdout[-4000:]
    assert r.returncode == 0 and " passed" in r.stdout, r.stdout[-4000:]
