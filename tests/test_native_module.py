"""The native Python module belongs to the prompt calls alone: a reader works without it, and it is compiled anew for another
torch."""
import os

import pytest
import torch

from paper_2508_09072_b200 import binding, build


class Library:
    """What Reader's constructor and destructor ask of the library."""

    def reader_create(self, out, device):
        return binding.OK

    def reader_destroy(self, handle):
        pass


@pytest.fixture
def no_module(monkeypatch):
    """A machine with a GPU and the library, where the module cannot be loaded."""
    def missing():
        raise ImportError("no module")
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(torch.cuda, "set_device", lambda d: None)
    monkeypatch.setattr(torch, "zeros", lambda *a, **kw: None)
    monkeypatch.setattr(binding, "load_library", Library)
    monkeypatch.setattr(binding, "load_native", missing)


def test_a_reader_does_not_need_the_module(no_module):
    rd = binding.Reader(0)
    for call in (rd.prompt_append, rd.tree_rotate):
        with pytest.raises((ImportError, TypeError)):
            call()
    cache = binding.KvCache(None, None, None, None)
    with pytest.raises(ImportError):
        rd.prompt_append(None, None, None, cache, None)
    rd.close()


def test_the_module_is_compiled_anew_for_another_torch(monkeypatch):
    build.build()
    assert build._library_is_current() and build._marshal_is_current()
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    assert build._library_is_current() and not build._marshal_is_current()


def test_a_compiler_that_fails_leaves_what_is_there(monkeypatch):
    build.build()
    before = [os.path.getmtime(f) for f in (build.LIB, build.MARSHAL, build.MARSHAL_MADE_FOR)]
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    monkeypatch.setenv("CXX", "/bin/false")
    with pytest.raises(RuntimeError, match="g\\+\\+"):
        build.build()
    assert [os.path.getmtime(f) for f in (build.LIB, build.MARSHAL, build.MARSHAL_MADE_FOR)] == before
    monkeypatch.undo()
    assert build._marshal_is_current()
