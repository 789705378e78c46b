"""The Python layer without a GPU: what it does where a part of it is absent."""
import ctypes
import importlib.util
import sys

import pytest

import paper_1712_02912_amd
from paper_1712_02912_amd import binding

VIEWS = "paper_1712_02912_amd.tensor_views"


class Refusing:
    """Finds no extension module that can be imported."""

    @staticmethod
    def find_spec(name, path=None, target=None):
        if name == VIEWS:
            raise ImportError("tensor_views.so: undefined symbol: of_another_torch")


def test_the_search_goes_without_the_extension_module(monkeypatch):
    monkeypatch.delattr(paper_1712_02912_amd, "tensor_views", raising=False)
    monkeypatch.delitem(sys.modules, VIEWS, raising=False)
    monkeypatch.setattr(sys, "meta_path", [Refusing] + sys.meta_path)
    spec = importlib.util.spec_from_file_location("binding_alone", binding.__file__)
    alone = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(alone)
    assert alone.load().pq_version().decode().startswith("pqadc")
    ctx = alone.Context.__new__(alone.Context)
    ctx.lib, ctx.handle, ctx._address = alone.load(), ctypes.c_void_p(), None
    none = [None] * 6
    for call in (lambda: ctx.pq_kv_plan(*none, out=()), lambda: ctx.pq_kv_append(None, *none), lambda: ctx.pq_kv_attention(*none, 1, out=1, lse=1),
                 lambda: ctx.pq_sample_tokens(None, None, out=())):
        with pytest.raises(RuntimeError, match="undefined symbol: of_another_torch") as e:
            call()
        assert isinstance(e.value.__cause__, ImportError)
