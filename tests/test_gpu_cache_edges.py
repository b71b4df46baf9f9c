"""The 4-bit cache's attention and the page calls where they can go wrong quietly.  Tolerances as in test_gpu_q4 unless a test derives its own."""
import numpy as np
import pytest
import torch

from test_gpu_q4 import attend, binding, i32, make, rd  # noqa: F401 (rd: a fixture)

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------------------------- bad pages in the form of one launch
@pytest.mark.parametrize("T,group,d", [(1, 4, 64), (1, 4, 128), (4, 4, 64), (20, 2, 128)])
def test_every_bad_page_is_reported_on_every_call(rd, T, group, d):
    """Whichever warp of a small call's thread blocks finds the page, and however soon: sequence b's only bad page is its b-th, and the calls follow one another."""
    b = binding()
    rng = np.random.default_rng(60)
    lens = [64 * 12] * 6
    both, cache, q, kt, vt, parent = make(rng, lens, T, 1, group, d)
    table = both.t4.copy()
    for s in range(6):
        table[s, 2 * s] = both.n16 if s & 1 else -1
    cache = b.Q4Cache(both.k4, both.v4, i32(table), i32(lens))
    out, lse, st = attend(rd, cache, q, kt, vt, parent, 0.1)
    assert st == [b.ERR_BAD_PAGE] * 6 and not out.any() and not lse.any()
    q, kt, vt, parent = q.cuda(), kt.cuda(), vt.cuda(), i32(parent)
    out, status = torch.ones_like(q), torch.zeros(500, 6, dtype=torch.int32, device="cuda")
    for i in range(500):
        rd.q4_verify_attn(q, kt, vt, cache, parent, 0.1, out=out, status=status[i])
    assert (status == b.ERR_BAD_PAGE).all() and not out.any()
