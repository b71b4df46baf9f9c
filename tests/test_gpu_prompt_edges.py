"""Prompt attention and append where they can go wrong quietly: NaN in units that are cut and merged, rows that belong to
nobody beside rows that count, the long forms at both head dimensions, in-place calls.  Tolerances as in test_gpu_prompt."""
import numpy as np
import pytest
import torch

from test_gpu_prompt import HALF, PAGE, bf16, check_attn, make_cache, plain_attn, rd, starts, within  # noqa: F401 (rd: a fixture)

pytestmark = pytest.mark.gpu


def run(rd, q, cache, ns, scale):
    tokens, Hq, D = q.shape
    out = torch.full((tokens, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((tokens, Hq), 7.0, dtype=torch.float32, device="cuda")
    rd.prompt_workspace().fill_(0xFF)
    _, st = rd.prompt_attn(q, cache, starts(ns), scale, out=out, lse=lse)
    assert st.tolist() == [0] * len(ns)
    return out.cpu(), lse.cpu()


def nan_rows_only(got, want, nan):
    """Rows where `nan` [tokens, heads] holds are NaN throughout, the others are what they are without the NaN."""
    (out, lse), (o, z, tol, ltol) = got, want
    assert torch.isnan(out[nan]).all() and torch.isnan(lse[nan]).all()
    within(out[~nan], o[~nan], tol[~nan])
    assert ((lse.double() - z).abs()[~nan] <= ltol[~nan]).all()


# ---------------------------------------------------------------------------------------------- NaN in units that are cut
@pytest.mark.parametrize("D", [64, 128])
def test_nan_keys_from_a_tile_boundary_on_reach_every_row_that_sees_them(rd, D):
    """Units of two 128-row tiles cut into a few pieces.  In the tile where the NaN begin, a row sees NaN keys and keys that
    are masked, nothing else: a piece that holds only this tile for it has the maximum -inf and a NaN sum."""
    rng = np.random.default_rng(60 + D)
    n, L, scale = 1500, 1300, 0.09
    cache = make_cache(rng, [L], [L + n], 2, D)
    q = bf16(rng, n, 2, D).cuda()
    want = plain_attn(q, cache, [n], [L], scale)
    pos = torch.arange(L + n)
    page = cache.page_table[0].cpu()[pos // PAGE].long().cuda()
    clean = cache.k_pool.clone()
    for t in range(0, (L + n) // 128 + 1):
        cache.k_pool.copy_(clean)
        first = 128 * t
        cache.k_pool[page[first:], 1, pos[first:].cuda() % PAGE] = float("nan")
        nan = torch.zeros(n, 2, dtype=torch.bool)
        nan[max(0, first - L):, 1] = True
        nan_rows_only(run(rd, q, cache, [n], scale), want, nan)


@pytest.mark.parametrize("D", [64, 128])
def test_nan_keys_over_whole_pieces_of_a_long_history(rd, D):
    """Few rows over a long history: twenty pieces to a unit, some of them NaN from end to end."""
    rng = np.random.default_rng(62 + D)
    n, L, scale = 3, 20000, 0.09
    cache = make_cache(rng, [L], [L + n], 2, D)
    q = bf16(rng, n, 4, D).cuda()
    want = plain_attn(q, cache, [n], [L], scale)
    pos = torch.arange(L + n)
    page = cache.page_table[0].cpu()[pos // PAGE].long().cuda()
    clean = cache.k_pool.clone()
    for lo, hi in ((4096, 8192), (0, 2048), (16384, L + n), (0, L + n), (12800, 12801)):
        cache.k_pool.copy_(clean)
        cache.k_pool[page[lo:hi], 0, pos[lo:hi].cuda() % PAGE] = float("nan")
        nan = torch.zeros(n, 4, dtype=torch.bool)
        nan[:, :2] = True
        nan_rows_only(run(rd, q, cache, [n], scale), want, nan)


@pytest.mark.parametrize("ns,L", [((1500,), 1300), ((3,), 20000), ((40,), 10), ((1,), 100)])
def test_a_nan_query_is_nan_in_output_and_lse(rd, ns, L):
    rng = np.random.default_rng(64)
    n = ns[0]
    cache = make_cache(rng, [L], [L + n], 2, 128)
    q = bf16(rng, n, 4, 128)
    want = plain_attn(q, cache, ns, [L], 0.09)
    nan = torch.zeros(n, 4, dtype=torch.bool)
    nan[n // 2, 1] = nan[n - 1, 2] = True
    q[nan] = float("nan")
    nan_rows_only(run(rd, q.cuda(), cache, ns, 0.09), want, nan)


# ---------------------------------------------------------------------------------------------- rows that belong to nobody
@pytest.mark.parametrize("ns,lens,extra", [((37, 60), (700, 0), 0), ((37, 60), (700, 0), 200), ((1, 1, 1, 1), (900, 3, 40, 17), 0),
                                           ((1, 1, 1, 1), (900, 3, 40, 17), 300), ((300, 90), (2300, 0), 0)])
@pytest.mark.parametrize("D", [64, 128])
def test_a_sequences_bits_do_not_depend_on_its_neighbour(rd, ns, lens, extra, D):
    """A query tile that a sequence does not fill holds the next sequence's queries behind it."""
    rng = np.random.default_rng(70)
    cache = make_cache(rng, lens, [a + b for a, b in zip(ns, lens)], 2, D)
    if extra:   # a wide page table: the call is cut into ranges
        wide = torch.full((len(ns), extra), -1, dtype=torch.int32, device="cuda")
        wide[:, :cache.page_table.shape[1]] = cache.page_table
        cache.page_table = wide
    q = bf16(rng, sum(ns), 8, D)
    calm, calm_lse = run(rd, q.cuda(), cache, ns, 0.09)
    for by in (40.0, -40.0, float("nan"), float("inf"), 2.0 ** 100):
        other = q.clone()
        other[ns[0]:] *= by
        out, lse = run(rd, other.cuda(), cache, ns, 0.09)
        assert torch.equal(out[:ns[0]], calm[:ns[0]]) and torch.equal(lse[:ns[0]], calm_lse[:ns[0]]), by


@pytest.mark.parametrize("Hq", [3, 5, 7])
def test_bits_do_not_depend_on_what_an_earlier_call_left_in_shared_memory(rd, Hq):
    """Groups that do not divide 128 leave rows of the query tile that no copy writes."""
    rng = np.random.default_rng(71)
    B, n, L = 200, 2 * (128 // Hq), 400
    filler = make_cache(rng, [0] * B, [256] * B, 1, 64)
    cache = make_cache(rng, [L] * 3, [L + n] * 3, 1, 64)
    q = bf16(rng, 3 * n, Hq, 64).cuda()
    seen = []
    for by in (1.0, 50.0, 2.0 ** 100):
        rd.prompt_attn(bf16(rng, 256 * B, 1, 64, scale=by).cuda(), filler, starts([256] * B), 0.125)   # every SM's query tiles
        seen.append(run(rd, q, cache, [n] * 3, 0.125))
    for out, lse in seen[1:]:
        assert torch.equal(out, seen[0][0]) and torch.equal(lse, seen[0][1])


@pytest.mark.parametrize("D", [64, 128])
def test_the_largest_batch(rd, D):
    """As many sequences as a call takes: the partition's words fill the whole ring before its first copy."""
    from paper_2508_09072_b200 import binding
    B = 32768
    g = torch.Generator(device="cuda").manual_seed(72)
    lens = torch.randint(0, PAGE - 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    ns = (torch.rand(B, generator=g, device="cuda") < 0.9).int()
    start = torch.cat([ns.new_zeros(1), ns.cumsum(0)]).int()
    tokens = int(start[-1])
    k, v = (torch.randn(B, 1, PAGE, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    cache = binding.KvCache(k, v, torch.randperm(B, generator=g, device="cuda").int()[:, None].contiguous(), lens)
    q = torch.randn(tokens, 2, D, generator=g, device="cuda").to(torch.bfloat16)
    out, st = rd.prompt_attn(q, cache, start, 0.1)
    assert not st.any()
    seq = ns.nonzero().flatten()
    page = cache.page_table[seq, 0].long()
    for lo in range(0, tokens, 4096):
        at = slice(lo, min(lo + 4096, tokens))
        kk, vv, qq = k[page[at], 0].double(), v[page[at], 0].double(), q[at].double()
        seen = torch.arange(PAGE, device="cuda") <= lens[seq[at], None]
        s = (torch.einsum("thd,tkd->thk", qq, kk) * 0.1).masked_fill(~seen[:, None], float("-inf"))
        mag = (torch.einsum("thd,tkd->thk", qq.abs(), kk.abs()) * 0.1).amax(-1, keepdim=True)
        w = torch.softmax(s, -1)
        want = torch.einsum("thk,tkd->thd", w, vv)
        tol = (HALF + 4 * (D * 2.0 ** -23 * mag + 1e-6)) * torch.einsum("thk,tkd->thd", w, vv.abs()) + HALF * 1.01 * want.abs() + 1e-30
        assert ((out[at].double() - want).abs() <= tol).all()
    with pytest.raises(binding.ReaderError) as e:   # one more is refused
        more = binding.KvCache(k, v, torch.zeros(B + 1, 1, dtype=torch.int32, device="cuda"), torch.zeros(B + 1, dtype=torch.int32, device="cuda"))
        rd.prompt_attn(q, more, torch.zeros(B + 2, dtype=torch.int32, device="cuda"), 0.1)
    assert e.value.code == binding.ERR_UNSUPPORTED
