"""Host-only tests of the binding's compiled part: what happens where it is missing or cannot be loaded."""
import os
import sys
import warnings

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
