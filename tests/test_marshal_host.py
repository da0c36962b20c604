"""Host-only tests of the binding's compiled part: what happens where it is missing or cannot be loaded, and that it hands calls
that are not as they have to be back, leaving no error and no reference behind."""
import ctypes as C
import importlib.machinery
import importlib.util
import os
import subprocess
import sys
import warnings
from types import SimpleNamespace

import numpy as np
import pytest
import torch

import paper_2602_01469_amd as pe
from paper_2602_01469_amd import binding
from paper_2602_01469_amd import build as _build

F4, E8M0, BF16 = torch.float4_e2m1fn_x2, torch.float8_e8m0fnu, torch.bfloat16


@pytest.fixture
def folder(monkeypatch, tmp_path):
    """The compiled part is looked for in an empty folder, and has not been loaded."""
    monkeypatch.setattr(pe, "__path__", [str(tmp_path)])
    monkeypatch.delattr(pe, "_marshal", raising=False)
    monkeypatch.delitem(sys.modules, pe.__name__ + "._marshal", raising=False)
    monkeypatch.setattr(binding, "_marshal", None)
    return tmp_path


def _calls():
    """The three calls, each with tensors that are not on a GPU."""
    raw = lambda *s: torch.zeros(s, dtype=torch.uint8)
    k, slots = torch.zeros(5, 2, 64, dtype=BF16), torch.zeros(5, dtype=torch.int64)
    cache = *[raw(3, 2, 64, 32).view(F4)] * 2, *[raw(3, 2, 64, 2).view(E8M0)] * 2
    shape, draft = pe.CacheShape(5, 2, 64, 3), pe.DecodeShape(2, 3, 8, 2, 64, 3, 1)
    return (lambda: pe.peagle_cache_append_block_scaled(shape, k, k, slots, *cache), lambda: pe.peagle_cache_read(shape, slots, *cache, k, k),
            lambda: pe.peagle_draft_decode_block_scaled(draft, k, k, k, *cache, slots, slots, k, k, None, raw(256)))


def _refused_by_the_checks():
    for call in _calls():
        with pytest.raises((TypeError, ValueError), match="GPU"):
            call()


def test_calls_do_without_the_compiled_part(folder):
    with pytest.warns(RuntimeWarning, match="_marshal.so is missing.*marshalled in Python") as said:
        _refused_by_the_checks()
    assert len(said) == 1


def test_a_file_that_cannot_be_loaded_is_not_called_missing(folder):
    (folder / "_marshal.so").write_bytes(b"no library")
    with pytest.warns(RuntimeWarning, match=r"_marshal.so cannot be loaded \(.*_marshal.so.*\): rebuild") as said:
        _refused_by_the_checks()
    assert len(said) == 1


@pytest.mark.parametrize("error", [RuntimeError("g++ failed"), FileNotFoundError("g++"), ImportError("torch")])
def test_the_library_is_built_without_it(monkeypatch, tmp_path, error):
    """A build without a host compiler, torch or its headers ends with the library, and leaves no older compiled part beside it."""
    def run(cmd, what):
        if what == "g++":
            raise error
        return ""

    old = tmp_path / "_marshal.so"
    old.write_bytes(b"older")
    monkeypatch.setattr(_build, "_run", run)
    monkeypatch.setattr(_build, "MARSHAL", str(old))
    with pytest.warns(RuntimeWarning, match="_marshal.so is not built"):
        assert _build.build() == _build.LIB
    assert not old.exists()


def test_one_built_for_another_torch_is_not_used(monkeypatch):
    """Its reads of tensors would be of another layout."""
    if not os.path.exists(os.path.join(os.path.dirname(pe.__file__), "_marshal.so")):
        pytest.skip("not built")
    monkeypatch.setattr(binding, "_marshal", None)
    monkeypatch.setattr(torch, "__version__", "1.0.0")
    with pytest.warns(RuntimeWarning, match=r"cannot be loaded \(built for torch .*, this is torch 1.0.0, .*\): rebuild"):
        _refused_by_the_checks()
    assert binding._marshal is not sys.modules[pe.__name__ + "._marshal"]


def test_the_built_one_is_taken():
    if not os.path.exists(os.path.join(os.path.dirname(pe.__file__), "_marshal.so")):
        pytest.skip("not built")
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        _refused_by_the_checks()
    assert binding._marshal is sys.modules[pe.__name__ + "._marshal"]


@pytest.fixture(scope="module")
def module():
    """The compiled part by itself, bound to the library's entry points."""
    path = os.environ.get("PEAGLE_MARSHAL", _build.MARSHAL)
    if not os.path.exists(path):
        pytest.skip("not built")
    loader = importlib.machinery.ExtensionFileLoader("_marshal", path)
    m = importlib.util.module_from_spec(importlib.util.spec_from_loader("_marshal", loader))
    lib = pe.load_library()
    m.bind(*(C.cast(f, C.c_void_p).value for f in (lib.peagle_cache_append_block_scaled, lib.peagle_cache_read, lib.peagle_draft_decode_block_scaled)))
    return m


class Raises:
    """A shape whose sizes cannot be read."""

    def __getattr__(self, name):
        raise ValueError(name)


def _cache_arguments():
    raw = lambda *s: torch.zeros(s, dtype=torch.uint8)
    k = torch.zeros(5, 2, 64, dtype=BF16)
    return pe.CacheShape(5, 2, 64, 3), k, torch.zeros(5, dtype=torch.int64), (*[raw(3, 2, 64, 32).view(F4)] * 2, *[raw(3, 2, 64, 2).view(E8M0)] * 2)


STREAMS = [None, 0, 7, "default", Raises(), SimpleNamespace(cuda_stream=0), SimpleNamespace(cuda_stream=0, device_index=0), SimpleNamespace(cuda_stream="0", device_index=0),
           SimpleNamespace(cuda_stream=2**70, device_index=0), SimpleNamespace(cuda_stream=0, device_index=2**40), SimpleNamespace(device_index=0)]
SIZES = [5, 0, -1, 2**31, -2**31 - 1, 2**70, -2**70, 5.0, "5", None, True, np.int64(5)]


def test_calls_that_are_not_as_they_have_to_be_are_handed_back(module):
    """None, and no exception, for tensors that are not on a GPU, sizes and streams that are none, too few and too many arguments."""
    shape, k, slots, cache = _cache_arguments()
    sums, none = torch.zeros(2, 8, 3), torch.zeros(2, dtype=torch.int32)
    draft = (k, k, k, *cache, none, none, k, sums, None, torch.zeros(256, dtype=torch.uint8))
    for n in SIZES:
        s = SimpleNamespace(n_tokens=n, Hkv=2, D=64, n_pages=n)
        d = SimpleNamespace(C=n, K=3, Hq=8, Hkv=2, D=64, scale=0.125 if n != 5.0 else n, n_pages=3, max_pages=n)
        assert module.cache_append(s, k, k, slots, *cache, None) is None and module.cache_read(s, slots, *cache, k, k, None) is None
        assert module.draft_decode(d, *draft, None) is None
    for n in (1, "0.125", None, np.float32(0.125)):  # not a float
        assert module.draft_decode(SimpleNamespace(C=2, K=3, Hq=8, Hkv=2, D=64, scale=n, n_pages=3, max_pages=1), *draft, None) is None
    for stream in STREAMS:
        assert module.cache_append(shape, k, k, slots, *cache, stream) is None and module.cache_read(shape, slots, *cache, k, k, stream) is None
        assert module.draft_decode(pe.DecodeShape(2, 3, 8, 2, 64, 3, 1), *draft, stream) is None
    for other in (None, 3, [], Raises(), np.zeros(3), k.float(), k.to_sparse()):
        for i in range(8):
            a, r = [shape, k, k, slots, *cache, None], [shape, slots, *cache, k, k, None]
            a[i] = r[i] = other
            assert module.cache_append(*a) is None and module.cache_read(*r) is None
        for i in range(len(draft)):
            assert module.draft_decode(pe.DecodeShape(2, 3, 8, 2, 64, 3, 1), *draft[:i], other, *draft[i + 1:], None) is None
    for f in (module.cache_append, module.cache_read, module.draft_decode):
        assert f() is None and f(shape) is None and f(*[shape] * 40) is None
    for wrong in ((), (1, 2), ("a", "b", "c"), (1, 2, 2**70)):
        with pytest.raises((TypeError, OverflowError)):
            module.bind(*wrong)


def test_calls_leave_no_reference_behind(module):
    _, k, slots, cache = _cache_arguments()
    sizes, scale = [100000 + i for i in range(4)], 1.0 / 3.0
    shape = SimpleNamespace(n_tokens=sizes[0], Hkv=sizes[1], D=sizes[2], n_pages=sizes[3], C=sizes[0], K=sizes[1], Hq=sizes[2], max_pages=sizes[3], scale=scale)
    stream = SimpleNamespace(cuda_stream=sizes[0], device_index=sizes[1])
    held = [*sizes, scale, shape, stream, k, slots, *cache]
    before = [sys.getrefcount(x) for x in held]
    for s in (None, stream):
        for _ in range(100):
            module.cache_append(shape, k, k, slots, *cache, s)
            module.cache_read(shape, slots, *cache, k, k, s)
            module.draft_decode(shape, k, k, k, *cache, slots, slots, k, k, None, slots, s)
    del s
    assert [sys.getrefcount(x) for x in held] == before


def test_it_is_clean_under_asan_and_ubsan(tmp_path):
    """The two tests above once more, with both sanitizers in it."""
    if "PEAGLE_MARSHAL" in os.environ:
        pytest.skip("this is that run")
    llvm = "/opt/rocm/llvm/bin/"
    if not os.path.exists(llvm + "clang++"):
        pytest.skip("no ROCm clang: cannot locate the sanitizer runtime")
    runtime = subprocess.run([llvm + "clang", "-print-file-name=libclang_rt.asan-x86_64.so"], stdout=subprocess.PIPE, text=True, check=True).stdout.strip()
    if not os.path.isabs(runtime) or not os.path.exists(runtime):
        pytest.skip("AddressSanitizer runtime not found")
    out = _build.build_marshal(str(tmp_path / "_marshal.so"), llvm + "clang++", ("-O1", "-g", "-fno-omit-frame-pointer", "-shared-libsan", "-fsanitize=address",
                               "-fsanitize=undefined", "-fno-sanitize=vptr,function", "-fno-sanitize-recover=undefined"))
    env = os.environ | {"PEAGLE_MARSHAL": out, "LD_PRELOAD": " ".join(x for x in (os.environ.get("LD_PRELOAD", ""), runtime) if x),
                        "ASAN_OPTIONS": "detect_leaks=0:abort_on_error=0:exitcode=86", "UBSAN_OPTIONS": "print_stacktrace=1:halt_on_error=1:exitcode=87"}
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.abspath(__file__), "-x", "-q", "-p", "no:cacheprovider", "-k", "handed_back or no_reference"],
                       cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), env=env, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600)
    assert "AddressSanitizer" not in r.stdout and "runtime error:" not in r.stdout, r.stdout[-4000:]
    assert r.returncode == 0 and "2 passed" in r.stdout, r.stdout[-4000:]
