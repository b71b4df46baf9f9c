"""The 4-bit cache and the page calls without a GPU: what the library and its native module refuse before anything is launched."""
import ctypes
from types import SimpleNamespace

import pytest
import torch


@pytest.fixture(scope="module")
def native():
    from paper_2508_09072_b200 import binding, build
    build.build()
    return binding.load_native()


def test_the_library_refuses_a_missing_context(native):
    from paper_2508_09072_b200 import binding
    lib = binding.load_library()
    n, i, f, size, bad = ctypes.c_void_p(None), ctypes.c_int32(1), ctypes.c_float(1.0), ctypes.c_size_t(16), binding.ERR_INVALID_ARG
    assert lib.reader_q4_workspace_bytes(None, 128) == 0
    assert lib.reader_set_q4_give_up(None, 0) == bad
    assert lib.reader_q4_store(n, n, n, i, i, n, n, n, n) == bad
    assert lib.reader_q4_load(n, n, n, i, i, n, n, n, n) == bad
    assert lib.reader_q4_commit(n, n, n, n, i, i, i, n, n, i, i, n, n, n) == bad
    assert lib.reader_q4_verify_attn(n, n, i, n, n, n, n, f, n, n, n, size, n, n) == bad
    assert lib.reader_pages_fork(n, n, n, n, i, n, size, n, n) == bad
    assert lib.reader_pages_reserve(n, n, n, n, i, n, size, n, n) == bad
    assert lib.reader_pages_free(n, n, n, n, i, n, n) == bad
    assert lib.reader_pages_compact(n, n, n, n, size, n) == bad
    assert lib.reader_pages_copy(n, n, i, n, i, i, size, n, n, i, n, n) == bad


def test_workspace_sizes(native):
    from paper_2508_09072_b200 import binding
    f = binding.load_library().reader_pages_workspace_bytes
    assert f(100, 10, 8, 4) > 0 and f(100, 10, 8, 400) > f(100, 10, 8, 4) and f(10000, 10, 8, 4) > f(100, 10, 8, 4)
    for wrong in ((0, 10, 8, 4), (100, 0, 8, 4), (100, 10, 0, 4), (100, 10, 8, -1), (100, 10, 1 << 20, 1 << 12)):
        assert f(*wrong) == 0


def cache(**changed):
    a = dict(k_pool=torch.zeros(2, 2, 36 * 64, dtype=torch.uint8), v_pool=torch.zeros(2, 2, 36 * 64, dtype=torch.uint8),
             page_table=torch.zeros(1, 2, dtype=torch.int32), seq_lens=torch.zeros(1, dtype=torch.int32), shared_prefix_len=0)
    a.update(changed)
    return SimpleNamespace(**a)


def test_the_native_module_takes_cuda_tensors_only(native):
    one = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(TypeError, match="CUDA"):
        native.q4_convert(0, 0, True, [cache()], [cache()], one, one, None)
    with pytest.raises(TypeError, match="CUDA"):
        native.q4_commit(0, 0, [cache()], [], [], torch.zeros(1, 2, dtype=torch.int32), one, True, None, None)
    with pytest.raises(TypeError, match="CUDA"):
        native.q4_verify_attn(0, 0, one, one, one, cache(), one, 0.1, None, None, None, None, one)
    with pytest.raises(TypeError, match="no such attribute"):
        native.q4_verify_attn(0, 0, one, one, one, object(), one, 0.1, None, None, None, None, one)
    pages = SimpleNamespace(refs=one, page_table=one, seq_lens=one, pools=[])
    for call in (native.pages_fork, native.pages_reserve):
        with pytest.raises(TypeError, match="CUDA"):
            call(0, 0, pages, one, one, one, None)
    with pytest.raises(TypeError, match="CUDA"):
        native.pages_free(0, 0, pages, one, None, None)
    with pytest.raises(TypeError, match="CUDA"):
        native.pages_compact(0, 0, pages, one, None)
    with pytest.raises(TypeError, match="CUDA"):
        native.pages_copy(0, 0, [one], [one], one, one, None)
    with pytest.raises(TypeError, match="list"):
        native.pages_copy(0, 0, 3, [one], one, one, None)
    with pytest.raises(ValueError, match="one pool"):
        native.pages_copy(0, 0, [], [], one, one, None)
    for f in (native.q4_convert, native.q4_commit, native.q4_verify_attn, native.pages_fork, native.pages_reserve, native.pages_free, native.pages_compact,
              native.pages_copy):
        with pytest.raises(TypeError, match="arguments"):
            f(1, 2, 3)
