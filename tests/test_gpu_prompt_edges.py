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


# ---------------------------------------------------------------------------------------------- long forms, both head dimensions
@pytest.mark.parametrize("D", [64, 128])
def test_units_from_the_counter(rd, D):
    rng = np.random.default_rng(80 + D)
    ns, lens = [500, 0, 333, 1, 8, 700, 9, 400], [0, 5, 100, 300, 0, 2900, 77, 40]
    cache = make_cache(rng, lens, [a + b for a, b in zip(ns, lens)], 8, D)
    q = bf16(rng, sum(ns) + 2, 64, D).cuda()
    for _ in range(2):   # the counter starts anew
        check_attn(rd, q, cache, ns, lens, 0.09)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("L", [1500, 2700])   # pieces of 12 and of 20 key tiles and more
def test_infinities_in_long_pieces(rd, D, L):
    rng = np.random.default_rng(82 + D)
    ns, lens = [300, 300, 301], [L + 200, L + 503, L]
    cache = make_cache(rng, lens, [a + b for a, b in zip(ns, lens)], 16, D)   # NaN and inf behind the last keys
    q = bf16(rng, sum(ns), 32, D).cuda()
    check_attn(rd, q, cache, ns, lens, 0.1)
    for b, j in ((0, 0), (0, 37), (2, 300), (2, 150)):
        pos = lens[b] + j
        page = cache.page_table[b, pos // PAGE].long()
        cache.v_pool[page, ::3, pos % PAGE, 9::13] = float("inf")
        cache.v_pool[page, 1, pos % PAGE, 4] = float("nan")
    check_attn(rd, q, cache, ns, lens, 0.1)


@pytest.mark.parametrize("D,Hq", [(64, 32), (128, 32), (128, 48)])
def test_whole_long_units(rd, D, Hq):
    """Wide units of 20 key tiles and more that one CTA does from end to end: three or so to an equal range (two heads to a
    group), from the counter (three)."""
    rng = np.random.default_rng(84 + D)
    ns, lens = [2600, 700], [1000, 2300]
    cache = make_cache(rng, lens, [a + b for a, b in zip(ns, lens)], 16, D)
    check_attn(rd, bf16(rng, sum(ns), Hq, D).cuda(), cache, ns, lens, 0.09)


def test_long_histories_begun_in_the_middle_at_head_dim_128(rd):
    """Whole units of more than 64 key tiles at four ring stages; sampled heads."""
    from paper_2508_09072_b200 import binding
    rng = np.random.default_rng(86)
    B, Hkv, D = 10, 32, 128
    ns, lens = [256] * B, [int(x) for x in rng.integers(8200, 8500, B)]
    ns[3], ns[7] = 100, 77
    pages = [(a + b + PAGE - 1) // PAGE for a, b in zip(ns, lens)]
    g = torch.Generator(device="cuda").manual_seed(86)
    order = torch.from_numpy(rng.permutation(sum(pages)).astype(np.int32)).cuda()
    table = torch.full((B, max(pages)), -1, dtype=torch.int32, device="cuda")
    for b in range(B):
        table[b, :pages[b]] = order[sum(pages[:b]):sum(pages[:b + 1])]
    k, v = (torch.randn(sum(pages), Hkv, PAGE, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    cache = binding.KvCache(k, v, table, torch.tensor(lens, dtype=torch.int32).cuda())
    q = torch.randn(sum(ns), Hkv, D, generator=g, device="cuda").to(torch.bfloat16)
    out, st = rd.prompt_attn(q, cache, starts(ns), D ** -0.5)
    assert st.tolist() == [0] * B
    for b in range(B):
        at = sum(ns[:b])
        for h in (b, 31 - b, 15):
            one = binding.KvCache(k[:, h:h + 1], v[:, h:h + 1], table[b:b + 1], cache.seq_lens[b:b + 1])
            want, _, tol, _ = plain_attn(q[at:at + ns[b], h:h + 1], one, [ns[b]], [lens[b]], D ** -0.5)
            within(out[at:at + ns[b], h:h + 1], want, tol)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("case", [((40,), (10,), 8, 2), ((300, 1, 77), (2000, 5000, 0), 8, 2), ((1,) * 5, (900, 0, 7, 4000, 64), 8, 2),
                                  ((4000, 3300), (0, 50), 16, 16), ((43, 85), (700, 0), 6, 2)])
def test_attn_in_place(rd, case, D):
    """out may be q, in every form of the call: the result is that of a call with an output of its own, every time."""
    ns, lens, Hq, Hkv = case
    rng = np.random.default_rng(87)
    cache = make_cache(rng, lens, [a + b for a, b in zip(ns, lens)], Hkv, D)
    q = bf16(rng, sum(ns), Hq, D).cuda()
    want, _ = rd.prompt_attn(q, cache, starts(ns), 0.125)
    for _ in range(3):
        again = q.clone()
        out, st = rd.prompt_attn(again, cache, starts(ns), 0.125, out=again)
        assert out is again and not st.any() and torch.equal(out, want)


@pytest.mark.parametrize("tokens", [5, 3000])   # several warps to a token, and one
@pytest.mark.parametrize("D,Hq,Hkv,inter,rot", [(128, 32, 8, False, 128), (64, 6, 2, True, 32)])
def test_append_in_place(rd, tokens, D, Hq, Hkv, inter, rot):
    rng = np.random.default_rng(88)
    ns, lens = [tokens // 2, 0, tokens - tokens // 2], [70, 3, 0]
    angle = np.arange(tokens + 80)[:, None] * 10000.0 ** (-np.arange(0, rot, 2) / rot)
    rope = torch.from_numpy(np.stack([np.cos(angle), np.sin(angle)], 1).astype(np.float32)).cuda()
    caches = [make_cache(np.random.default_rng(89), lens, [a + b for a, b in zip(ns, lens)], Hkv, D) for _ in range(2)]
    q, k, v = (bf16(rng, tokens + 1, h, D).cuda() for h in (Hq, Hkv, Hkv))
    qw, kw = bf16(rng, D).cuda(), bf16(rng, D).cuda()
    kw_args = dict(rope=rope, q_weight=qw, k_weight=kw, interleaved=inter)
    want = torch.full_like(q, 7.0)
    rd.prompt_append(q, k, v, caches[0], starts(ns), out=want, **kw_args)
    last = q[-1].clone()
    out, st = rd.prompt_append(q, k, v, caches[1], starts(ns), out=q, **kw_args)
    assert out is q and not st.any() and torch.equal(q[:-1], want[:-1]) and torch.equal(q[-1], last)
    for pool in ("k_pool", "v_pool"):
        assert torch.equal(*(getattr(c, pool).view(torch.int16) for c in caches))


# ---------------------------------------------------------------------------------------------- a shared prefix
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("ns,lens,prefix", [((1,) * 6, (512, 700, 513, 900, 640, 512), 512), ((33, 1, 0, 300), (256, 300, 256, 1000), 256),
                                            ((1,) * 4, (4096, 4100, 4500, 4097), 4096)])
def test_attention_behind_a_shared_prefix(rd, ns, lens, prefix, D):
    rng = np.random.default_rng(90)
    cache = make_cache(rng, lens, [a + b for a, b in zip(ns, lens)], 2, D)
    cache.page_table[:, :prefix // PAGE] = cache.page_table[0, :prefix // PAGE]
    q = bf16(rng, sum(ns), 8, D).cuda()
    plain, _ = rd.prompt_attn(q, cache, starts(ns), 0.09)
    cache.shared_prefix_len = prefix
    out, _ = check_attn(rd, q, cache, ns, lens, 0.09)
    assert torch.equal(out, plain)


# ---------------------------------------------------------------------------------------------- large pools
@pytest.mark.parametrize("D,Hkv", [(64, 8), (128, 8)])
def test_pages_whose_offsets_pass_32_bits(rd, D, Hkv):
    """Pools of more than 2^32 elements; the call's pages lie at both ends and around 2^31 and 2^32."""
    from paper_2508_09072_b200 import binding
    rng = np.random.default_rng(92)
    row = Hkv * PAGE * D
    total = 2 ** 32 // row + 40
    k_pool, v_pool = (torch.empty(total, Hkv, PAGE, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ns, lens = [300, 1, 70], [1500, 90, 0]
    pages = [(a + b + PAGE - 1) // PAGE for a, b in zip(ns, lens)]
    some = [total - 1, 0, 2 ** 31 // row, 2 ** 32 // row, 2 ** 31 // row - 1, 2 ** 32 // row - 1]
    some += [x for x in range(total - 30, total - 1) if x not in some]
    table = torch.full((3, max(pages)), -1, dtype=torch.int32)
    for b in range(3):
        table[b, :pages[b]] = torch.tensor(some[sum(pages[:b]):sum(pages[:b + 1])])
    cache = binding.KvCache(k_pool, v_pool, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    used = torch.tensor(some[:sum(pages)]).cuda()
    for pool in (k_pool, v_pool):
        pool[used] = bf16(rng, len(used), Hkv, PAGE, D).cuda()
    tokens = sum(ns)
    q, k, v = (bf16(rng, tokens, h, D).cuda() for h in (2 * Hkv, Hkv, Hkv))
    v[5, 1, 3], v[250, 0, D - 1] = float("inf"), float("nan")
    q2, st = rd.prompt_append(q, k, v, cache, starts(ns))
    assert not st.any() and torch.equal(q2, q)
    pos = torch.cat([torch.arange(L, L + n) for n, L in zip(ns, lens)])
    seq = torch.cat([torch.full((n,), b) for b, n in enumerate(ns)])
    page, at = table[seq, pos // PAGE].long().cuda(), (pos % PAGE).cuda()
    assert torch.equal(k_pool[page, :, at], k) and torch.equal(v_pool[page, :, at].view(torch.int16), v.view(torch.int16))
    check_attn(rd, q, cache, ns, lens, 0.1)


# ---------------------------------------------------------------------------------------------- many calls
@pytest.mark.parametrize("D,Hq,Hkv,ns,lens", [(64, 8, 8, (1,), (511,)), (128, 8, 2, (40, 1, 130), (10, 300, 0)),       # a single launch
                                              (128, 32, 8, (1,) * 16, tuple(range(500, 2100, 100))), (128, 4, 2, (700, 3), (900, 3000)),
                                              (64, 128, 16, (300, 90, 310), (70, 5, 1000)), (128, 96, 16, (500, 300), (0, 40))])   # counter
def test_thousands_of_calls_never_give_up_a_wait(rd, D, Hq, Hkv, ns, lens):
    """Every wait of the kernel is bounded: a lost wake-up would show as READER_ERR_TIMEOUT in one call of many."""
    rng = np.random.default_rng(95)
    cache = make_cache(rng, lens, [a + b for a, b in zip(ns, lens)], Hkv, D)
    q, ts = bf16(rng, sum(ns), Hq, D).cuda(), starts(ns)
    first, st = rd.prompt_attn(q, cache, ts, 0.1)
    out, status = torch.empty_like(q), torch.empty_like(st)
    worst, differs = torch.zeros_like(st), torch.zeros((), dtype=torch.bool, device="cuda")
    for i in range(2000):
        rd.prompt_attn(q, cache, ts, 0.1, out=out, status=status)
        worst = torch.maximum(worst, status)
        if i % 20 == 0:
            differs |= (out != first).any()
    assert not worst.any() and not differs


# ---------------------------------------------------------------------------------------------- calls that the documentation allows
@pytest.mark.parametrize("Hq,Hkv,D,ns,lens,width", [(8, 2, 128, (40, 0, 3), (10, 5, 300), 0), (8, 2, 128, (40, 0, 3), (10, 5, 300), 100),
                                                    (128, 16, 64, (300, 0, 310), (70, 5, 100), 0)])
def test_rows_in_front_of_the_first_sequence(rd, Hq, Hkv, D, ns, lens, width):
    """token_start need not begin at 0: rows in front are nobody's, like those behind."""
    rng = np.random.default_rng(97)
    cache = make_cache(rng, lens, [a + b for a, b in zip(ns, lens)], Hkv, D)
    if width:
        wide = torch.full((len(ns), width), -1, dtype=torch.int32, device="cuda")
        wide[:, :cache.page_table.shape[1]] = cache.page_table
        cache.page_table = wide
    q = bf16(rng, sum(ns) + 7, Hq, D).cuda()
    k, v = bf16(rng, sum(ns) + 7, Hkv, D).cuda(), bf16(rng, sum(ns) + 7, Hkv, D).cuda()
    ts = starts(ns) + 5
    q2 = torch.full_like(q, 7.0)
    _, st = rd.prompt_append(q, k, v, cache, ts, out=q2)
    assert not st.any() and torch.equal(q2[5:-2], q[5:-2]) and (q2[:5] == 7.0).all() and (q2[-2:] == 7.0).all()
    out, lse = torch.full_like(q, 7.0), torch.full((len(q), Hq), 7.0, device="cuda")
    _, st = rd.prompt_attn(q2, cache, ts, 0.1, out=out, lse=lse)
    assert not st.any() and (out[:5] == 7.0).all() and (out[-2:] == 7.0).all() and (lse[:5] == 7.0).all() and (lse[-2:] == 7.0).all()
    want, wlse, tol, ltol = plain_attn(q[5:-2], cache, ns, lens, 0.1)
    within(out[5:-2], want, tol)
    assert ((lse[5:-2].double().cpu() - wlse).abs() <= ltol).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,ns,lens", [(128, (300,), (200,)), (65, (70, 1), (0, 900)), (127, (9, 40), (130, 3)), (63, (50,), (64,)), (43, (90,), (1,))])
def test_wide_groups(rd, D, G, ns, lens):
    rng = np.random.default_rng(98)
    cache = make_cache(rng, lens, [a + b for a, b in zip(ns, lens)], 1, D)
    check_attn(rd, bf16(rng, sum(ns) + 1, G, D).cuda(), cache, ns, lens, D ** -0.5)


def test_append_and_tree_captured_and_replayed_on_another_stream(rd):
    rng = np.random.default_rng(99)
    Hq, Hkv, D, T, B = 8, 2, 128, 9, 3
    room = [400, 300, 200]
    cache = make_cache(rng, [0] * B, room, Hkv, D)
    angle = np.arange(500)[:, None] * 10000.0 ** (-np.arange(0, D, 2) / D)
    rope = torch.from_numpy(np.stack([np.cos(angle), np.sin(angle)], 1).astype(np.float32)).cuda()
    q, k, v = (bf16(rng, 120, h, D).cuda() for h in (Hq, Hkv, Hkv))
    tq, tk, tv = (bf16(rng, B, T, h, D).cuda() for h in (Hq, Hkv, Hkv))
    parent = torch.tensor([[-1, 0, 0, 1, 2, 3, 3, 0, 7]] * B, dtype=torch.int32).cuda()
    ts, out, st = starts([1, 1, 1]), torch.empty_like(q), torch.empty(B, dtype=torch.int32, device="cuda")
    touts = [torch.empty_like(x) for x in (tq, tk, tv)]
    tst = torch.empty_like(st)

    def calls():
        rd.prompt_append(q, k, v, cache, ts, rope=rope, out=out, status=st)
        rd.tree_rotate(tq, tk, tv, cache.seq_lens, parent, rope=rope, out=touts[0], k_tree=touts[1], v_tree=touts[2], status=tst)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            calls()
    torch.cuda.synchronize()
    for ns, lens in (([70, 1, 33], [5, 200, 0]), ([0, 0, 0], [1, 2, 3]), ([1, 100, 19], [399, 150, 181])):
        ts.copy_(starts(ns))
        cache.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (out, cache.k_pool, cache.v_pool, *touts, st, tst)]
        out.fill_(7.0)
        calls()
        assert all(torch.equal(a.view(torch.int16) if a.dtype == torch.bfloat16 else a, b.view(torch.int16) if b.dtype == torch.bfloat16 else b)
                   for a, b in zip(got, (out, cache.k_pool, cache.v_pool, *touts, st, tst)))
        assert not st.any() and not tst.any() and (out[sum(ns):] == 7.0).all()


def test_empty_calls(rd):
    from paper_2508_09072_b200 import binding
    rng = np.random.default_rng(100)
    cache = make_cache(rng, [5, 0, 64], [5, 0, 64], 2, 64)
    cache.seq_lens[1] = -1
    none = lambda h: torch.empty(0, h, 64, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    out, st = rd.prompt_append(none(4), none(2), none(2), cache, starts([0, 0, 0]))
    assert out.shape == (0, 4, 64) and st.tolist() == [0, binding.ERR_CAPACITY, 0]
    out, st = rd.prompt_attn(none(4), cache, starts([0, 0, 0]), 0.1)
    assert st.tolist() == [0, binding.ERR_CAPACITY, 0]
    nobody = binding.KvCache(cache.k_pool, cache.v_pool, cache.page_table[:0], cache.seq_lens[:0])
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert rd.prompt_append(none(4), none(2), none(2), nobody, one)[1].numel() == 0
    assert rd.prompt_attn(none(4), nobody, one, 0.1)[1].numel() == 0
    tree = lambda h: torch.empty(0, 3, h, 64, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    got = rd.tree_rotate(tree(4), tree(2), tree(2), one[:0], torch.empty(0, 3, dtype=torch.int32, device="cuda"))
    assert got[0].shape == (0, 3, 4, 64) and got[3].numel() == 0


@pytest.mark.parametrize("B,T", [(3000, 1), (700, 5)])
def test_tree_rotate_of_many_trees(rd, B, T):
    rng = np.random.default_rng(101)
    Hq, Hkv, D = 6, 2, 64
    parent = torch.tensor([[-1, 0, 1, 0, 3][:T]] * B, dtype=torch.int32)
    level = torch.tensor([0, 1, 2, 1, 2][:T])
    lens = torch.from_numpy(rng.integers(0, 90, B).astype(np.int32))
    angle = np.arange(100)[:, None] * 10000.0 ** (-np.arange(0, D, 2) / D)
    rope = torch.from_numpy(np.stack([np.cos(angle), np.sin(angle)], 1).astype(np.float32))
    q, k, v = (bf16(rng, B, T, h, D) for h in (Hq, Hkv, Hkv))
    got = rd.tree_rotate(q.cuda(), k.cuda(), v.cuda(), lens.cuda(), parent.cuda(), rope=rope.cuda())
    assert not got[3].any() and torch.equal(got[2].cpu(), v)
    row = rope[(lens[:, None] + level).long()].double()
    for x, y in ((q, got[0]), (k, got[1])):
        x = x.double()
        a, b, c, s = x[..., :D // 2], x[..., D // 2:], row[:, :, None, 0], row[:, :, None, 1]
        want = torch.cat([a * c - b * s, b * c + a * s], -1)
        mag = torch.cat([a.abs() + b.abs()] * 2, -1)
        within(y, want, HALF * want.abs() + 2.0 ** -20 * mag)


def test_values_that_the_call_before_has_just_written(rd):
    """Decoding steps back to back, each of which brings an infinity into one column of one head: the attention looks at value
    rows that the append right before it wrote, next to rows that the attention before that has looked at."""
    rng = np.random.default_rng(103)
    Hq, Hkv, D, L, steps = 16, 8, 128, 1700, 300
    cache = make_cache(rng, [L], [L + steps], Hkv, D, poison=False)
    q, k, v = (bf16(rng, steps, h, D) for h in (Hq, Hkv, Hkv))
    where = torch.from_numpy(rng.permutation(Hkv * D)[:steps])
    v.view(steps, -1)[torch.arange(steps), where] = float("inf")
    q, k, v, ts = q.cuda(), k.cuda(), v.cuda(), starts([1])
    outs, worst = torch.empty_like(q), torch.zeros(1, dtype=torch.int32, device="cuda")
    for i in range(steps):
        one = slice(i, i + 1)
        _, st = rd.prompt_append(q[one], k[one], v[one], cache, ts)
        _, st2 = rd.prompt_attn(q[one], cache, ts, 0.09, out=outs[one], update_seq_lens=True)
        worst = torch.maximum(worst, torch.maximum(st, st2))
    assert not worst.any() and cache.seq_lens.tolist() == [L + steps]
    seen = torch.zeros(steps, Hkv * D, dtype=torch.bool)
    seen[torch.arange(steps), where] = True
    seen = (seen.cumsum(0) > 0).view(steps, Hkv, 1, D).expand(steps, Hkv, Hq // Hkv, D).reshape(steps, Hq, D)
    got = outs.cpu()
    assert torch.isfinite(got[~seen]).all() and not torch.isfinite(got[seen]).any()
