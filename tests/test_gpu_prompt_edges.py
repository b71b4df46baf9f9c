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


# ---------------------------------------------------------------------------------------------- a thread block that gives up
# (no wait runs out in these tests: a thread block says so when its work is done, or the host leaves the note that one would)
@pytest.fixture
def give_up(rd):
    yield rd.set_prompt_give_up
    rd.set_prompt_give_up(-1)


def unit_of(cta, ns, Hkv, tokens_per_unit):
    """(sequence, block, head) of a single-launch call's thread block."""
    for b, n in enumerate(ns):
        units = -(-n // tokens_per_unit) * Hkv
        if cta < units:
            return b, cta // Hkv, cta % Hkv
        cta -= units


@pytest.mark.parametrize("D", [64, 128])
def test_one_that_gives_up_in_the_single_launch_form(rd, give_up, D):
    from paper_2508_09072_b200 import binding
    rng = np.random.default_rng(75)
    ns, lens, Hq, Hkv = [100, 0, 1, 64], [70, 3, 200, 0], 8, 2     # 64 tokens a unit: 2 + 0 + 1 + 1 blocks of 2 heads
    cache = make_cache(rng, lens, [a + b for a, b in zip(ns, lens)], Hkv, D)
    q = bf16(rng, sum(ns) + 1, Hq, D).cuda()
    good, good_lse = check_attn(rd, q, cache, ns, lens, 0.1)
    at = np.concatenate([[0], np.cumsum(ns)])
    ws = torch.full_like(rd.prompt_workspace(), 0xFF)

    def call():
        out, lse = torch.full_like(q, 7.0), torch.full((len(q), Hq), 7.0, device="cuda")
        _, st = rd.prompt_attn(q, cache, starts(ns), 0.1, out=out, lse=lse, workspace=ws)
        return out, lse, st.tolist()
    for cta in range(9):
        give_up(cta)
        out, lse, st = call()
        want, want_lse, want_st = good.clone(), good_lse.clone(), [0] * 4
        if cta < 8:
            b, block, h = unit_of(cta, ns, Hkv, 64)
            rows = slice(at[b] + 64 * block, min(at[b] + 64 * block + 64, at[b + 1]))
            want[rows, 4 * h:4 * h + 4] = 0
            want_lse[rows, 4 * h:4 * h + 4] = 0
            want_st[b] = binding.ERR_TIMEOUT
        assert st == want_st, cta
        assert torch.equal(out, want) and torch.equal(lse, want_lse), cta
        give_up(-1)
        out, lse, st = call()      # the event may be reported once more, with the right rows
        assert all(x in (0, y) for x, y in zip(st, want_st)) and torch.equal(out, good)
        out, lse, st = call()
        assert st == [0] * 4 and torch.equal(out, good) and torch.equal(lse, good_lse)
    # the note of one that gave up before the first unit's thread block began
    ws.view(torch.int64).fill_(0x9d6b2f04c18e73a5 - 2 ** 64)
    out, lse, st = call()
    assert st == [binding.ERR_TIMEOUT, 0, binding.ERR_TIMEOUT, binding.ERR_TIMEOUT] and torch.equal(out, good)
    assert call()[2] == [0] * 4
    # a bad page is still reported, and the one that gives up has the last word
    cache.page_table[3, 0] = -1
    assert call()[2] == [0, 0, 0, binding.ERR_BAD_PAGE]
    give_up(7)
    out, lse, st = call()
    assert st == [0, 0, 0, binding.ERR_TIMEOUT] and not out[at[3]:at[4]].any() and torch.equal(out[:at[3]], good[:at[3]])


@pytest.mark.parametrize("form", ["ranges", "counter", "advancing"])
def test_one_that_gives_up_in_the_other_forms(rd, give_up, form):
    from paper_2508_09072_b200 import binding
    rng = np.random.default_rng(76)
    ns, lens = [300, 0, 40, 310], [70, 5, 10, 1900]
    Hq, Hkv, D = (128, 16, 64) if form == "counter" else (4, 2, 128)
    cache = make_cache(rng, lens, [a + b for a, b in zip(ns, lens)], Hkv, D)
    q = bf16(rng, sum(ns) + 1, Hq, D).cuda()
    update = form == "advancing"
    good, _ = rd.prompt_attn(q, cache, starts(ns), 0.1)
    for cta in (0, 5):
        out, lse = torch.full_like(q, 7.0), torch.full((len(q), Hq), 7.0, device="cuda")
        give_up(cta)
        _, st = rd.prompt_attn(q, cache, starts(ns), 0.1, out=out, lse=lse, update_seq_lens=update)
        assert st.tolist() == [binding.ERR_TIMEOUT] * 4 and cache.seq_lens.tolist() == lens
        assert not out[:-1].any() and not lse[:-1].any() and (out[-1] == 7.0).all() and (lse[-1] == 7.0).all()
        give_up(-1)
        out, st = rd.prompt_attn(q, cache, starts(ns), 0.1)
        assert st.tolist() == [0] * 4 and torch.equal(out[:-1], good[:-1])
    assert cache.seq_lens.tolist() == lens
    with pytest.raises(binding.ReaderError) as e:
        give_up(-2)
    assert e.value.code == binding.ERR_INVALID_ARG


# ---------------------------------------------------------------------------------------------- arguments
def test_a_value_that_is_neither_true_nor_false_is_refused(rd):
    rng = np.random.default_rng(78)
    cache = make_cache(rng, [3], [8], 2, 64)
    q, k = bf16(rng, 5, 4, 64).cuda(), bf16(rng, 5, 2, 64).cuda()
    neither = torch.tensor([True, False])
    before = cache.k_pool.clone()
    with pytest.raises(TypeError, match="interleaved"):
        rd.prompt_append(q, k, k, cache, starts([5]), interleaved=neither)
    with pytest.raises(TypeError, match="update_seq_lens"):
        rd.prompt_attn(q, cache, starts([5]), 0.1, update_seq_lens=neither)
    with pytest.raises(TypeError, match="interleaved"):
        rd.tree_rotate(q[None], k[None], k[None], cache.seq_lens, torch.tensor([[-1, 0, 1, 2, 3]], dtype=torch.int32, device="cuda"), interleaved=neither)
    assert torch.equal(cache.k_pool.view(torch.int16), before.view(torch.int16)) and cache.seq_lens.tolist() == [3]
    _, st = rd.prompt_append(q, k, k, cache, starts([5]), interleaved=np.bool_(False))
    assert not st.any()
