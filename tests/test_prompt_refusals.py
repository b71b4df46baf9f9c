"""The prompt calls without a GPU: what the library and its native Python module refuse before anything is launched."""
import ctypes

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
    lib.reader_prompt_workspace_bytes.restype = ctypes.c_size_t
    assert lib.reader_prompt_workspace_bytes(None, 128) == 0
    none = ctypes.c_void_p(None)
    n64, n32, f32, size = ctypes.c_int64(0), ctypes.c_int32(0), ctypes.c_float(1.0), ctypes.c_size_t(0)
    assert lib.reader_prompt_append(none, none, none, none, n64, n64, n64, n32, none, none, none, none, none, none) == binding.ERR_INVALID_ARG
    assert lib.reader_tree_rotate(none, none, none, none, n64, n64, n64, n32, n32, n32, none, none, none, none, none, none, none,
                                  none) == binding.ERR_INVALID_ARG
    assert lib.reader_prompt_attn(none, none, n32, none, none, f32, n32, none, none, none, size, none, none) == binding.ERR_INVALID_ARG


def args(**changed):
    bf, i32 = torch.bfloat16, torch.int32
    a = dict(handle=0, device=0, q=torch.zeros(5, 4, 64, dtype=bf), k_pool=torch.zeros(2, 2, 64, 64, dtype=bf),
             v_pool=torch.zeros(2, 2, 64, 64, dtype=bf), page_table=torch.zeros(1, 2, dtype=i32), seq_lens=torch.zeros(1, dtype=i32), prefix=0,
             token_start=torch.zeros(2, dtype=i32), scale=0.1, update=False, out=None, lse=None, workspace=None, status=None)
    a.update(changed)
    return list(a.values())


def test_the_native_module_takes_cuda_tensors_only(native):
    with pytest.raises(TypeError, match="CUDA"):
        native.prompt_attn(*args())
    with pytest.raises(TypeError, match="tensor"):
        native.prompt_attn(*args(k_pool=[1, 2]))
    with pytest.raises(TypeError, match="arguments"):
        native.prompt_attn(1, 2, 3)
    with pytest.raises(TypeError, match="arguments"):
        native.prompt_append(*args())
    with pytest.raises(TypeError, match="arguments"):
        native.tree_rotate()
    with pytest.raises(TypeError, match="integer"):
        native.prompt_attn(*args(device="cuda"))


def test_the_testing_aid_refuses_a_missing_context(native):
    from paper_2508_09072_b200 import binding
    assert binding.load_library().reader_set_prompt_give_up(None, 0) == binding.ERR_INVALID_ARG
