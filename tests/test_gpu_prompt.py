"""Prompt append, tree rotation and prompt attention against plain implementations in 64 bits.

Tolerances (bf16 rounds by at most 2^-8 of the value):
  rotation   one rounding at the end of an fp32 computation: 2^-8 |y| + 2^-20 times the sum of the terms' magnitudes
             (a norm, two products and a sum, each with a few fp32 roundings of 2^-24).
  attention  the weights of the value product are rounded once (2^-8 of each), the output once (2^-8), everything else
             is fp32: a score is off by at most D 2^-23 of the sum of its products' magnitudes, which moves a weight by
             that factor and the log of the denominator by that amount.
"""
import numpy as np
import pytest
import torch

from paper_2508_09072_b200 import workloads as W

pytestmark = pytest.mark.gpu
PAGE = 64
HALF = 2.0 ** -8     # half a step of bf16


@pytest.fixture(scope="module")
def rd():
    from paper_2508_09072_b200 import binding
    r = binding.Reader(0)
    yield r
    r.close()


def bf16(rng, *shape, scale=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(torch.bfloat16)


def make_cache(rng, lens, room, Hkv, D, spare=2, poison=True):
    """A cache with room[b] positions for sequence b, `lens` of them committed; every byte beyond room is NaN."""
    from paper_2508_09072_b200 import binding
    pages = [(r + PAGE - 1) // PAGE for r in room]
    total, width = sum(pages) + spare, max(max(pages), 1)
    order = rng.permutation(total).astype(np.int32)
    table = np.full((len(lens), width), -1, np.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at:at + n]
        at += n
    k, v = bf16(rng, total, Hkv, PAGE, D), bf16(rng, total, Hkv, PAGE, D)
    if poison:
        real = torch.zeros(total, PAGE, dtype=torch.bool)
        for b, r in enumerate(room):
            for p in range(pages[b]):
                real[table[b, p], :max(0, min(PAGE, r - p * PAGE))] = True
        k.transpose(1, 2)[~real] = float("nan")
        v.transpose(1, 2)[~real] = float("inf")
    return binding.KvCache(k.cuda(), v.cuda(), torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32).cuda())


def starts(ns):
    return torch.from_numpy(np.concatenate([[0], np.cumsum(ns)]).astype(np.int32)).cuda()


def rows_of(cache, b, n):
    """K and V of positions 0 .. n-1 of sequence b, float64 [n, Hkv, D]."""
    pages = cache.page_table[b, :(n + PAGE - 1) // PAGE].long()
    take = lambda pool: pool[pages].transpose(1, 2).reshape(-1, pool.shape[1], pool.shape[3])[:n].double().cpu()  # noqa: E731
    return take(cache.k_pool), take(cache.v_pool)


def plain_attn(q, cache, ns, lens, scale):
    """out, lse, and the tolerances of both, float64."""
    tokens, Hq, D = q.shape
    Hkv = cache.k_pool.shape[1]
    out, tol = torch.zeros(tokens, Hq, D, dtype=torch.float64), torch.zeros(tokens, Hq, D, dtype=torch.float64)
    lse, ltol = torch.zeros(tokens, Hq, dtype=torch.float64), torch.zeros(tokens, Hq, dtype=torch.float64)
    q = q.double().cpu()
    at = 0
    for b, (n, L) in enumerate(zip(ns, lens)):
        if n == 0:
            continue
        k, v = rows_of(cache, b, L + n)
        for h in range(Hq):
            kk, vv, qq = k[:, h * Hkv // Hq], v[:, h * Hkv // Hq], q[at:at + n, h]
            seen = torch.arange(L + n)[None] <= L + torch.arange(n)[:, None]
            s = (qq @ kk.T * scale).masked_fill(~seen, float("-inf"))
            mag = (qq.abs() @ kk.abs().T * scale).masked_fill(~seen, 0).amax(-1)
            z = torch.logsumexp(s, -1)
            w = (s - z[:, None]).exp()
            delta = D * 2.0 ** -23 * mag + 1e-6
            vv0 = torch.where(torch.isfinite(vv), vv, 0.0)
            o = w @ vv0
            for j in (~torch.isfinite(vv)).any(-1).nonzero().flatten().tolist():   # only for the rows that see them
                bad = torch.where(torch.isfinite(vv[j]), 0.0, vv[j])
                o[max(0, j - L):] += bad
            out[at:at + n, h], lse[at:at + n, h], ltol[at:at + n, h] = o, z, delta + 2.0 ** -22 * z.abs()
            tol[at:at + n, h] = (HALF + 4 * delta[:, None]) * (w @ vv0.abs()) + HALF * 1.01 * o.abs() + 1e-30
        at += n
    return out, lse, tol, ltol


def check_attn(rd, q, cache, ns, lens, scale, status=None, **kw):
    tokens, Hq, D = q.shape
    out = torch.full((tokens, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((tokens, Hq), 7.0, dtype=torch.float32, device="cuda")
    ws = rd.prompt_workspace()
    ws.fill_(0xFF)   # scratch that is read without having been written must show
    want, wlse, tol, ltol = plain_attn(q, cache, ns, lens, scale)
    out, st = rd.prompt_attn(q, cache, starts(ns), scale, out=out, lse=lse, **kw)
    torch.cuda.synchronize()
    assert st.tolist() == (status or [0] * len(ns))
    used = sum(ns)
    assert (out[used:] == 7.0).all() and (lse[used:] == 7.0).all()
    got = out[:used].double().cpu()
    fin = torch.isfinite(want[:used])
    assert torch.equal(torch.isfinite(got), fin)
    assert torch.equal(torch.isnan(got), torch.isnan(want[:used]))
    err = torch.where(fin, (got - want[:used]).abs() / tol[:used], 0.0)
    assert err.max() <= 1 if err.numel() else True, float(err.max())
    lerr = (lse[:used].double().cpu() - wlse[:used]).abs() / ltol[:used]
    assert lerr.max() <= 1 if lerr.numel() else True, float(lerr.max())
    return out, lse


# ---------------------------------------------------------------------------------------------- attention
ATTN = [
    # Hq, Hkv, D, new tokens, committed
    (8, 8, 64, (1,), (0,)),
    (8, 8, 64, (1,), (511,)),
    (4, 1, 128, (1,), (63,)),
    (32, 8, 128, (1, 1, 1), (1000, 64, 0)),
    (4, 2, 128, (127,), (0,)),
    (4, 4, 128, (128,), (0,)),
    (4, 4, 64, (129,), (0,)),
    (4, 4, 128, (256,), (0,)),
    (4, 4, 128, (257,), (0,)),
    (8, 2, 128, (64, 65, 31, 33, 0, 1), (0, 0, 0, 0, 0, 0)),
    (8, 2, 128, (200, 0, 77), (61, 5, 130)),
    (6, 2, 64, (90, 43), (10, 0)),          # 3 heads to a group: 42 tokens in a tile
    (5, 1, 128, (70,), (33,)),
    (7, 1, 64, (19, 300), (0, 129)),
    (16, 1, 128, (40,), (1,)),
    (128, 1, 64, (5,), (70,)),              # one token in a tile
    (100, 1, 64, (3,), (0,)),
    (2, 2, 64, (700,), (0,)),
    (2, 1, 128, (3,), (5000,)),             # few rows, long history: split over many CTAs
    (2, 2, 128, (1500,), (1300,)),
    (1, 1, 64, (2, 1, 1), (2047, 2048, 2049)),
]


@pytest.mark.parametrize("case", range(len(ATTN)))
def test_attn_against_64_bits(rd, case):
    Hq, Hkv, D, ns, lens = ATTN[case]
    rng = np.random.default_rng(100 + case)
    cache = make_cache(rng, lens, [a + b for a, b in zip(ns, lens)], Hkv, D)
    q = bf16(rng, sum(ns) + 3, Hq, D).cuda()   # three rows behind the last sequence
    check_attn(rd, q, cache, ns, lens, D ** -0.5)


@pytest.mark.parametrize("D", [64, 128])
def test_attn_random_shapes(rd, D):
    rng = np.random.default_rng(7 + D)
    for _ in range(12):
        Hkv, G, B = int(rng.integers(1, 4)), int(rng.integers(1, 10)), int(rng.integers(1, 7))
        ns = [int(2 ** rng.uniform(0, 8.5)) * int(rng.random() > 0.1) for _ in range(B)]
        lens = [int(2 ** rng.uniform(0, 10)) * int(rng.random() > 0.4) for _ in range(B)]
        cache = make_cache(rng, lens, [a + b for a, b in zip(ns, lens)], Hkv, D)
        q = bf16(rng, sum(ns) + 1, Hkv * G, D).cuda()
        check_attn(rd, q, cache, ns, lens, 0.11)


def test_attn_units_from_the_counter(rd):
    """Enough units that they are handed out whole: ragged prompts, with and without a history, an empty one, rows behind."""
    rng = np.random.default_rng(17)
    ns, lens = [500, 0, 333, 1, 8, 700, 9, 400], [0, 5, 100, 300, 0, 0, 77, 40]
    cache = make_cache(rng, lens, [a + b for a, b in zip(ns, lens)], 8, 64)
    q = bf16(rng, sum(ns) + 2, 128, 64).cuda()
    for _ in range(2):   # the counter starts anew
        check_attn(rd, q, cache, ns, lens, 0.125)


# one sequence of each kind that is turned down, in every form of the call: a single launch (short pages tables), equal
# ranges (a wide page table), units from the counter (many heads)
FORMS = [(4, 2, 64, 0), (4, 2, 64, 200), (128, 16, 64, 0)]


@pytest.mark.parametrize("form", range(3))
def test_attn_rejections_in_every_form(rd, form):
    from paper_2508_09072_b200 import binding
    Hq, Hkv, D, extra = FORMS[form]
    rng = np.random.default_rng(40 + form)
    ns, lens = [300, 40, 0, 310, 20, 300], [70, 10, 0, 100, 30, 0]
    cache = make_cache(rng, lens, [a + b for a, b in zip(ns, lens)], Hkv, D, poison=False)
    if extra:
        wide = torch.full((len(ns), extra), -1, dtype=torch.int32, device="cuda")
        wide[:, :cache.page_table.shape[1]] = cache.page_table
        cache.page_table = wide
    q = bf16(rng, sum(ns) + 1, Hq, D).cuda()
    good, st = rd.prompt_attn(q, cache, starts(ns), 0.125)
    assert st.tolist() == [0] * 6
    good = good.clone()
    cache.page_table[1, 0], cache.page_table[3, 6] = -1, cache.k_pool.shape[0]
    cache.seq_lens[4] = 2 ** 30
    lse = torch.full((sum(ns) + 1, Hq), 7.0, device="cuda")
    out = torch.full_like(q, 7.0)
    _, st = rd.prompt_attn(q, cache, starts(ns), 0.125, out=out, lse=lse)
    assert st.tolist() == [0, binding.ERR_BAD_PAGE, 0, binding.ERR_BAD_PAGE, binding.ERR_CAPACITY, 0]
    at = np.concatenate([[0], np.cumsum(ns)])
    for b in range(6):
        rows = slice(at[b], at[b + 1])
        if st[b]:
            assert not out[rows].any() and not lse[rows].any(), b
        else:
            assert torch.equal(out[rows], good[rows]), b
    assert (out[-1] == 7.0).all() and (lse[-1] == 7.0).all()
    for bad in ([0, 300, 340, 330, 650, 670, 970], [0, 300, 340, 340, 650, 670, sum(ns) + 2], [-3, 300, 340, 340, 650, 670, 970]):
        out.fill_(3.0)
        _, st = rd.prompt_attn(q, cache, torch.tensor(bad, dtype=torch.int32).cuda(), 0.125, out=out)
        assert st.tolist() == [binding.ERR_INVALID_ARG] * 6 and (out == 3.0).all()


def test_attn_infinities_in_long_pieces(rd):
    """The same as above where the values are looked at ahead of their tiles, and on garbage behind the last key."""
    rng = np.random.default_rng(43)
    ns, lens = [300, 300, 301], [1700, 2003, 1500]
    cache = make_cache(rng, lens, [a + b for a, b in zip(ns, lens)], 16, 64)   # NaN and inf behind the last keys
    for b, j in ((0, 0), (0, 37), (2, 300), (2, 150)):
        pos = lens[b] + j
        page = cache.page_table[b, pos // PAGE].long()
        cache.v_pool[page, ::3, pos % PAGE, 9::13] = float("inf")
        cache.v_pool[page, 1, pos % PAGE, 4] = float("nan")
    check_attn(rd, bf16(rng, sum(ns), 32, 64).cuda(), cache, ns, lens, 0.1)
    ns = [100] * 3
    lens = [x + 200 for x in lens[:2]] + [1701]
    cache.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
    check_attn(rd, bf16(rng, 300, 32, 64).cuda(), cache, ns, lens, 0.1)


@pytest.mark.parametrize("case", [((40,), (10,), 8, 2), ((300, 1, 77), (2000, 5000, 0), 8, 2), ((1,) * 5, (900, 0, 7, 4000, 64), 8, 2),
                                  ((4000, 3300), (0, 50), 16, 16)])
def test_attn_in_place(rd, case):
    """out may be q: a unit's queries have been read before its rows are written, in every form of the call."""
    ns, lens, Hq, Hkv = case
    rng = np.random.default_rng(47)
    cache = make_cache(rng, lens, [a + b for a, b in zip(ns, lens)], Hkv, 64)
    q = bf16(rng, sum(ns), Hq, 64).cuda()
    want, _ = rd.prompt_attn(q, cache, starts(ns), 0.125)
    out, st = rd.prompt_attn(q, cache, starts(ns), 0.125, out=q)
    assert out is q and not st.any() and torch.equal(out, want)


def test_attn_very_large_batch(rd):
    rng = np.random.default_rng(44)
    B = 3000
    lens = [int(x) for x in rng.integers(0, 40, B)]
    ns = [int(x) for x in rng.integers(0, 3, B)]
    cache = make_cache(rng, lens, [64] * B, 1, 64, poison=False)
    q = bf16(rng, sum(ns), 2, 64).cuda()
    check_attn(rd, q, cache, ns, lens, 0.125)
    k, v = bf16(rng, sum(ns), 1, 64).cuda(), bf16(rng, sum(ns), 1, 64).cuda()
    _, st = rd.prompt_append(q, k, v, cache, starts(ns))
    assert not st.any()
    pos = torch.cat([torch.arange(L, L + n) for n, L in zip(ns, lens)])
    seq = torch.cat([torch.full((n,), b) for b, n in enumerate(ns)])
    page = cache.page_table.cpu()[seq, 0].long()
    assert torch.equal(cache.k_pool.cpu()[page, :, pos], k.cpu()) and torch.equal(cache.v_pool.cpu()[page, :, pos], v.cpu())


def test_calls_at_once_on_two_streams(rd):
    """Two readers, two streams, workspaces of their own."""
    from paper_2508_09072_b200 import binding
    rng = np.random.default_rng(45)
    other = binding.Reader(0)
    try:
        work = []
        for r, ns, lens in ((rd, [400, 30], [100, 900]), (other, [1, 1, 1, 600], [700, 5, 0, 64])):
            cache = make_cache(rng, lens, [a + b for a, b in zip(ns, lens)], 2, 128)
            work.append((r, ns, lens, cache, bf16(rng, sum(ns), 8, 128).cuda(), torch.cuda.Stream(), starts(ns)))
        torch.cuda.synchronize()
        outs = []
        for _ in range(20):
            outs = []
            for r, ns, lens, cache, q, stream, ts in work:
                with torch.cuda.stream(stream):
                    outs.append(r.prompt_attn(q, cache, ts, 0.09)[0])
        torch.cuda.synchronize()
        for (r, ns, lens, cache, q, stream, ts), out in zip(work, outs):
            want, _, tol, _ = plain_attn(q, cache, ns, lens, 0.09)
            within(out, want, tol)
    finally:
        other.close()


def test_attn_long_histories_begun_in_the_middle(rd):
    """Whole units of more than 64 key tiles, which different CTAs begin at different tiles; sampled heads."""
    rng = np.random.default_rng(18)
    B, Hkv, D = 10, 32, 64
    ns, lens = [256] * B, [int(x) for x in rng.integers(8200, 8500, B)]
    ns[3], ns[7] = 100, 77
    pages = [(a + b + PAGE - 1) // PAGE for a, b in zip(ns, lens)]
    g = torch.Generator(device="cuda").manual_seed(18)
    from paper_2508_09072_b200 import binding
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
            kk, vv = rows_of(cache, b, lens[b] + ns[b])
            kk, vv, qq = kk[:, h], vv[:, h], q[at:at + ns[b], h].double().cpu()
            seen = torch.arange(len(kk))[None] <= lens[b] + torch.arange(ns[b])[:, None]
            w = torch.softmax((qq @ kk.T * D ** -0.5).masked_fill(~seen, float("-inf")), -1)
            want = w @ vv
            delta = D * 2.0 ** -23 * (qq.abs() @ kk.abs().T * D ** -0.5).amax(-1, keepdim=True) + 1e-6
            tol = (HALF + 4 * delta) * (w @ vv.abs()) + HALF * 1.01 * want.abs()
            within(out[at:at + ns[b], h], want, tol)


def test_attn_many_single_tokens(rd):
    rng = np.random.default_rng(3)
    B = 200
    lens = [int(x) for x in rng.integers(0, 300, B)]
    ns = [1] * B
    cache = make_cache(rng, lens, [x + 1 for x in lens], 2, 64)
    check_attn(rd, bf16(rng, B, 8, 64).cuda(), cache, ns, lens, 0.125)


def test_attn_rising_scores_are_rescaled(rd):
    """Keys whose scores grow by far more than 2^8 from tile to tile, in both directions."""
    rng = np.random.default_rng(4)
    for sign in (1.0, -1.0):
        n, D = 600, 128
        cache = make_cache(rng, [0], [n], 1, D, poison=False)
        ramp = torch.linspace(0.0, 30.0 * sign, n).repeat_interleave(1)
        pages = cache.page_table[0].long()
        k = (ramp[:, None] * torch.ones(D) / D ** 0.5).to(torch.bfloat16)
        flat = torch.zeros(pages.numel() * PAGE, D, dtype=torch.bfloat16)
        flat[:n] = k
        cache.k_pool[pages, 0] = flat.view(-1, PAGE, D).cuda()
        q = (torch.ones(n, 2, D) * 3).to(torch.bfloat16).cuda()
        check_attn(rd, q, cache, [n], [0], 1.0)


def test_attn_scores_beyond_the_exponents_range(rd):
    """Scores of 10^12, where the rounding of a maximum is many times what an exponential can hold, after ordinary ones.

    Every key of a head has its own score: a row's largest lies 10^9 above the rest, so its weight is 1 and the others' 0.
    q and k are powers of two times at most 8 bits, and the products of a row are alike, so a score's sum is exact; its
    scaling and the maximum's move the log of the denominator by a few 2^-24 of it."""
    rng = np.random.default_rng(46)
    n, D = 600, 128
    cache = make_cache(rng, [0], [n], 2, D)
    pos = torch.arange(n)
    page = cache.page_table[0].cpu()[pos // PAGE].long()
    size = torch.stack([torch.tensor(f)[pos // 128] * (1 + pos % 128 / 128) for f in
                        ([2.0 ** -40, 1, 0.125, 2, 0.5], [1, 0.125, 2, 0.5, 4])])          # [head, position]
    k = (size * 2.0 ** 18).to(torch.bfloat16)
    assert torch.equal(k.float(), size * 2.0 ** 18)
    pool = cache.k_pool.cpu()
    for h in range(2):
        pool[page, h, pos % PAGE] = k[h][:, None].expand(n, D)
    cache.k_pool.copy_(pool)
    sign = torch.tensor([1.0, -1.0, 1.0, -1.0])
    q = (sign * 2.0 ** 18)[None, :, None].expand(n, 4, D).to(torch.bfloat16).contiguous()
    for pieces in ([n], [1] * 3, [300]):
        m = sum(pieces)
        lens = [n - m]
        if len(pieces) > 1:      # single tokens of three sequences that share the pages
            lens = [n - 1, 200, 5]
            many = type(cache)(cache.k_pool, cache.v_pool, cache.page_table.repeat(3, 1), torch.tensor(lens, dtype=torch.int32).cuda())
        else:
            many = cache
            many.seq_lens.fill_(lens[0])
        lse = torch.empty(m, 4, device="cuda")
        out, st = rd.prompt_attn(q[:m].cuda(), many, starts(pieces), 0.125, lse=lse)
        assert not st.any()
        want, wlse, _, _ = plain_attn(q[:m], many, pieces, lens, 0.125)
        out, lse = out.double().cpu(), lse.double().cpu()
        last = torch.cat([torch.arange(L, L + c) for c, L in zip(pieces, lens)])
        ordinary = torch.zeros(m, 4, dtype=torch.bool)
        ordinary[:, 1] = True                  # the small scores are the largest ones
        ordinary[last < 128, 0] = True         # nothing else is seen
        assert torch.equal(out[~ordinary], want[~ordinary])
        assert ((lse - wlse)[~ordinary].abs() <= 2.0 ** -21 * wlse[~ordinary].abs()).all()
        v = rows_of(cache, 0, 128)[1][:, 0]
        delta = D * 2.0 ** -23 * 2 + 1e-6      # scores of at most 2
        s = 0.125 * D * 2.0 ** 36 * size[0, :128].double()
        for i, h in ordinary.nonzero().tolist():
            w = torch.softmax((sign[h] * s)[:int(last[i]) + 1], 0)
            o, top = w @ v[:len(w)], w @ v[:len(w)].abs()
            assert ((out[i, h] - o).abs() <= (HALF + 4 * delta) * top + HALF * 1.01 * o.abs()).all()
    from paper_2508_09072_b200 import binding
    with pytest.raises(binding.ReaderError) as e:   # times log2(e) it is infinite
        rd.prompt_attn(q.cuda(), cache, starts([n]), 2.5e38)
    assert e.value.code == binding.ERR_UNSUPPORTED


def test_attn_infinities_in_later_tokens_do_not_reach_earlier_rows(rd):
    rng = np.random.default_rng(5)
    for ns, lens, where in [((200,), (0,), (0, 3, 64, 150, 199)), ((50, 90), (70, 20), (10, 33)), ((300,), (100,), (299,)), ((1,), (90,), (90 - 1,))]:
        cache = make_cache(rng, lens, [a + b for a, b in zip(ns, lens)], 2, 128)
        for b in range(len(ns)):
            for j in where:
                pos = min(lens[b] + j, lens[b] + ns[b] - 1) if ns[b] > 1 else j
                page = cache.page_table[b, pos // PAGE].long()
                cache.v_pool[page, :, pos % PAGE, 5::17] = float("inf")
                cache.v_pool[page, 1, pos % PAGE, 100] = float("nan")
                cache.v_pool[page, 0, pos % PAGE, 7] = float("-inf")
        check_attn(rd, bf16(rng, sum(ns), 8, 128).cuda(), cache, ns, lens, 0.09)


def test_attn_nan_keys_reach_only_the_rows_that_see_them(rd):
    rng = np.random.default_rng(6)
    n = 300
    cache = make_cache(rng, [0], [n], 1, 64)
    q = bf16(rng, n, 2, 64).cuda()
    clean, _ = rd.prompt_attn(q, cache, starts([n]), 0.125)
    clean = clean.clone()
    page = cache.page_table[0, 170 // PAGE].long()
    cache.k_pool[page, 0, 170 % PAGE] = float("nan")
    out, st = rd.prompt_attn(q, cache, starts([n]), 0.125)
    assert torch.equal(out[:170], clean[:170]) and torch.isnan(out[170:]).all() and st.tolist() == [0]


def test_attn_same_bits_every_time_and_pieces_agree_with_the_whole(rd):
    rng = np.random.default_rng(8)
    n, Hq, Hkv, D = 777, 8, 2, 128
    cache = make_cache(rng, [0], [n], Hkv, D)
    q = bf16(rng, n, Hq, D).cuda()
    a, lse = check_attn(rd, q, cache, [n], [0], 0.09)
    b, _ = rd.prompt_attn(q, cache, starts([n]), 0.09)
    assert torch.equal(a, b)
    at = 0
    for piece in (1, 300, 63, 1, 412):
        rd.prompt_attn(q[at:at + piece].contiguous(), cache, starts([piece]), 0.09, update_seq_lens=True)
        at += piece
        assert cache.seq_lens.tolist() == [at]
    cache.seq_lens.fill_(n - 412)
    check_attn(rd, q[n - 412:].contiguous(), cache, [412], [n - 412], 0.09)


def test_attn_agrees_with_verify_attn_on_a_chain(rd):
    """A single token against a one-node tree: the same query, the same keys."""
    rng = np.random.default_rng(9)
    lens = [130, 700, 64]
    cache = make_cache(rng, lens, [x + 1 for x in lens], 2, 128)
    q = bf16(rng, 3, 8, 128).cuda()
    kv = [rows_of(cache, b, lens[b] + 1) for b in range(3)]
    k_tree, v_tree = (torch.stack([x[i][-1:] for x in kv]).to(torch.bfloat16).cuda() for i in (0, 1))
    want, st = rd.verify_attn(q[:, None].contiguous(), k_tree, v_tree, cache, torch.full((3, 1), -1, dtype=torch.int32, device="cuda"), 0.09)
    got, st2 = rd.prompt_attn(q, cache, starts([1, 1, 1]), 0.09)
    ref, _, tol, _ = plain_attn(q, cache, [1, 1, 1], lens, 0.09)
    assert ((got.double().cpu() - ref).abs() <= tol).all() and ((want[:, 0].double().cpu() - ref).abs() <= tol).all()


def test_attn_status_words(rd):
    from paper_2508_09072_b200 import binding
    rng = np.random.default_rng(10)
    ns, lens = [40, 30, 20, 5], [10, 0, 100, 0]
    q = bf16(rng, 95, 4, 64).cuda()
    cache = make_cache(rng, lens, [a + b for a, b in zip(ns, lens)], 2, 64)
    good, _ = rd.prompt_attn(q, cache, starts(ns), 0.125)
    good = good.clone()
    cache.page_table[1, 0] = 10 ** 6
    lse = torch.full((95, 4), 7.0, device="cuda")
    out, st = rd.prompt_attn(q, cache, starts(ns), 0.125, lse=lse, update_seq_lens=True)
    assert st.tolist() == [0, binding.ERR_BAD_PAGE, 0, 0]
    assert not out[40:70].any() and not lse[40:70].any()
    keep = [i for i in range(95) if not 40 <= i < 70]
    assert torch.equal(out[keep], good[keep])
    assert cache.seq_lens.tolist() == [50, 0, 120, 5]
    cache.page_table[1, 0] = -5
    cache.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
    _, st = rd.prompt_attn(q, cache, starts(ns), 0.125)
    assert st.tolist() == [0, binding.ERR_BAD_PAGE, 0, 0]
    cache.page_table[1, 0] = 0
    cache.seq_lens[0] = -1
    cache.seq_lens[2] = 2 ** 31 - 1
    out, st = rd.prompt_attn(q, cache, starts(ns), 0.125)
    assert st.tolist() == [binding.ERR_CAPACITY, 0, binding.ERR_CAPACITY, 0] and not out[:40].any() and not out[70:90].any()
    for bad in ([0, 40, 30, 90, 95], [-1, 40, 70, 90, 95], [0, 40, 70, 90, 96]):
        out.fill_(3.0)
        _, st = rd.prompt_attn(q, cache, torch.tensor(bad, dtype=torch.int32).cuda(), 0.125, out=out)
        assert st.tolist() == [binding.ERR_INVALID_ARG] * 4 and (out == 3.0).all()


def test_attn_without_tokens(rd):
    rng = np.random.default_rng(11)
    cache = make_cache(rng, [5, 0], [5, 0], 2, 64)
    out, st = rd.prompt_attn(torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda"), cache, starts([0, 0]), 0.125, update_seq_lens=True)
    assert st.tolist() == [0, 0] and out.shape[0] == 0 and cache.seq_lens.tolist() == [5, 0]
    out = torch.full((4, 4, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    _, st = rd.prompt_attn(torch.ones_like(out), cache, starts([0, 0]), 0.125, out=out)
    assert st.tolist() == [0, 0] and (out == 3.0).all()


def test_attn_captured_and_replayed_and_on_another_stream(rd):
    rng = np.random.default_rng(12)
    ns, lens = [70, 1, 33], [5, 200, 0]
    cache = make_cache(rng, lens, [a + b + 64 for a, b in zip(ns, lens)], 2, 128)
    q, ts = bf16(rng, 120, 8, 128).cuda(), starts(ns)
    out, status = torch.empty_like(q), torch.empty(3, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        rd.prompt_attn(q, cache, ts, 0.09, out=out, status=status)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            rd.prompt_attn(q, cache, ts, 0.09, out=out, status=status, update_seq_lens=True)
    torch.cuda.synchronize()
    # other lengths in the same buffers: the captured call follows what is on the device
    for ns in ([70, 1, 33], [1, 60, 2], [0, 0, 9]):
        before = cache.seq_lens.tolist()
        cache.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        ts.copy_(starts(ns))
        graph.replay()
        torch.cuda.synchronize()
        assert status.tolist() == [0, 0, 0] and cache.seq_lens.tolist() == [a + b for a, b in zip(ns, lens)]
        want, _, tol, _ = plain_attn(q, cache, ns, lens, 0.09)
        assert ((out[:sum(ns)].double().cpu() - want[:sum(ns)]).abs() <= tol[:sum(ns)]).all(), before


def test_attn_refusals(rd):
    from paper_2508_09072_b200 import binding
    rng = np.random.default_rng(13)
    cache = make_cache(rng, [0], [64], 1, 64)
    q, ts = bf16(rng, 4, 129, 64).cuda(), starts([4])

    def refused(code, *a, **kw):
        with pytest.raises(binding.ReaderError) as e:
            rd.prompt_attn(*a, **kw)
        assert e.value.code == code
    refused(binding.ERR_UNSUPPORTED, q, cache, ts, 0.1)                                # 129 heads to a group
    q = bf16(rng, 4, 2, 64).cuda()
    refused(binding.ERR_UNSUPPORTED, q, cache, ts, 0.0)
    refused(binding.ERR_UNSUPPORTED, q, cache, ts, -1.0)
    refused(binding.ERR_UNSUPPORTED, q, cache, ts, float("inf"))
    refused(binding.ERR_INVALID_ARG, q, cache, ts, float("nan"))
    refused(binding.ERR_WORKSPACE, q, cache, ts, 0.1, workspace=torch.empty(1024, dtype=torch.uint8, device="cuda"))
    refused(binding.ERR_INVALID_ARG, q, cache, ts, 0.1, workspace=rd.prompt_workspace()[16:])
    two = make_cache(rng, [0], [64], 2, 64)
    refused(binding.ERR_UNSUPPORTED, bf16(rng, 4, 3, 64).cuda(), two, ts, 0.1)         # 3 heads over 2
    with pytest.raises(ValueError):
        rd.prompt_attn(bf16(rng, 4, 2, 128).cuda(), cache, ts, 0.1)
    with pytest.raises(TypeError):
        rd.prompt_attn(q.float(), cache, ts, 0.1)
    with pytest.raises(ValueError):
        rd.prompt_attn(q, cache, starts([2, 2]), 0.1)


# ---------------------------------------------------------------------------------------------- append and tree
def make_rope(positions, rot, base=10000.0):
    f = base ** (-np.arange(0, rot, 2, dtype=np.float64) / rot)
    a = np.arange(positions, dtype=np.float64)[:, None] * f
    return torch.from_numpy(np.stack([np.cos(a), np.sin(a)], 1).astype(np.float32))


def plain_turn(x, pos, rope, weight, eps, interleaved):
    """x bf16 [tokens, heads, D], pos [tokens] -> value and tolerance, float64."""
    y = x.double()
    if weight is not None:
        y = y / (y.square().mean(-1, keepdim=True) + eps).sqrt() * weight.double()
    z, mag = y.clone(), y.abs()
    if rope is not None:
        half = rope.shape[2]
        for j in range(half):
            a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
            c, s = rope[pos, 0, j].double()[:, None], rope[pos, 1, j].double()[:, None]
            z[..., a] = y[..., a] * c - y[..., b] * s
            z[..., b] = y[..., b] * c + y[..., a] * s
            mag[..., a] = mag[..., b] = (y[..., a].abs() + y[..., b].abs())
    return z, HALF * z.abs() + 2.0 ** -20 * mag


TURN = [
    # Hq, Hkv, D, norm, rot (0: none), interleaved, fused
    (8, 8, 64, True, 64, False, True),
    (32, 8, 128, True, 128, False, True),
    (6, 2, 64, False, 48, False, False),
    (4, 4, 128, True, 96, True, True),
    (5, 1, 128, False, 64, True, False),
    (1, 1, 64, True, 16, False, True),
    (3, 1, 64, True, 0, False, True),
    (2, 1, 128, False, 0, False, False),
    (70, 14, 64, True, 32, True, True),      # more heads than a pass of a block holds
]


def projection(rng, lead, Hq, Hkv, D, fused):
    if fused:
        x = bf16(rng, *lead, Hq + 2 * Hkv, D).cuda()
        return x[..., :Hq, :], x[..., Hq:Hq + Hkv, :], x[..., Hq + Hkv:, :]
    return bf16(rng, *lead, Hq, D).cuda(), bf16(rng, *lead, Hkv, D).cuda(), bf16(rng, *lead, Hkv, D).cuda()


def weights(rng, D, norm):
    return (bf16(rng, D).cuda(), bf16(rng, D).cuda()) if norm else (None, None)


def within(got, want, tol):
    err = (got.double().cpu() - want).abs()
    assert (err <= tol).all(), float((err / tol.clamp(min=1e-300)).max())


@pytest.mark.parametrize("case", range(len(TURN)))
@pytest.mark.parametrize("ns,lens", [((1,), (0,)), ((70, 0, 1, 130), (3, 64, 127, 0)), ((1,) * 9, (0, 63, 64, 65, 1, 2, 3, 200, 5))])
def test_append_against_64_bits(rd, case, ns, lens):
    Hq, Hkv, D, norm, rot, inter, fused = TURN[case]
    rng = np.random.default_rng(200 + case)
    cache = make_cache(rng, lens, [a + b for a, b in zip(ns, lens)], Hkv, D)
    used = sum(ns)
    q, k, v = projection(rng, (used + 2,), Hq, Hkv, D, fused)
    qw, kw = weights(rng, D, norm)
    rope = make_rope(max(a + b for a, b in zip(ns, lens)), rot) if rot else None
    k0, v0 = cache.k_pool.clone(), cache.v_pool.clone()
    out = torch.full((used + 2, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    out, st = rd.prompt_append(q, k, v, cache, starts(ns), rope=None if rope is None else rope.cuda(), q_weight=qw, k_weight=kw,
                               eps=1e-5, interleaved=inter, out=out)
    assert st.tolist() == [0] * len(ns) and (out[used:] == 7.0).all() and cache.seq_lens.tolist() == list(lens)
    pos = torch.cat([torch.arange(L, L + n) for n, L in zip(ns, lens)])
    seq = torch.cat([torch.full((n,), b) for b, n in enumerate(ns)])
    cpu = lambda t: None if t is None else t.cpu()  # noqa: E731
    within(out[:used], *plain_turn(q[:used].cpu(), pos, rope, cpu(qw), 1e-5, inter))
    page = cache.page_table.cpu()[seq, pos // PAGE].long()
    want, tol = plain_turn(k[:used].cpu(), pos, rope, cpu(kw), 1e-5, inter)
    within(cache.k_pool.cpu()[page, :, pos % PAGE], want, tol)
    assert torch.equal(cache.v_pool.cpu()[page, :, pos % PAGE], v[:used].cpu())
    # nothing else in the pools has changed
    for now, before in ((cache.k_pool, k0), (cache.v_pool, v0)):
        now = now.clone()
        now[page.cuda(), :, (pos % PAGE).cuda()] = before[page.cuda(), :, (pos % PAGE).cuda()]
        assert torch.equal(now.view(torch.int16), before.view(torch.int16))


@pytest.mark.parametrize("case", range(len(TURN)))
@pytest.mark.parametrize("T", [1, 2, 37, 128])
def test_tree_rotate_against_64_bits(rd, case, T):
    Hq, Hkv, D, norm, rot, inter, fused = TURN[case]
    rng = np.random.default_rng(300 + case)
    parent = np.stack([W.chain_tree(T), W.star_tree(T), W.capped_recursive_tree(rng, T, 12, 4)]).astype(np.int32)
    level = np.zeros_like(parent)
    for b in range(3):
        for j in range(1, T):
            level[b, j] = level[b, parent[b, j]] + 1
    lens = torch.tensor([0, 700, 33], dtype=torch.int32)
    q, k, v = projection(rng, (3, T), Hq, Hkv, D, fused)
    qw, kw = weights(rng, D, norm)
    rope = make_rope(701 + T, rot) if rot else None
    got = rd.tree_rotate(q, k, v, lens.cuda(), torch.from_numpy(parent).cuda(), rope=None if rope is None else rope.cuda(),
                         q_weight=qw, k_weight=kw, eps=1e-5, interleaved=inter)
    assert got[3].tolist() == [0, 0, 0]
    pos = (lens[:, None] + torch.from_numpy(level)).long().flatten()
    for x, y, w in ((q, got[0], qw), (k, got[1], kw)):
        want, tol = plain_turn(x.cpu().reshape(3 * T, -1, D), pos, rope, None if w is None else w.cpu(), 1e-5, inter)
        within(y.reshape(3 * T, -1, D), want, tol)
    assert torch.equal(got[2], v)


def test_rotation_in_place(rd):
    rng = np.random.default_rng(20)
    lens, T = torch.tensor([5, 9], dtype=torch.int32).cuda(), 17
    parent = torch.from_numpy(np.stack([W.chain_tree(T), W.star_tree(T)]).astype(np.int32)).cuda()
    q, k, v = projection(rng, (2, T), 12, 4, 128, False)
    rope, (qw, kw) = make_rope(64, 128).cuda(), weights(rng, 128, True)
    want = rd.tree_rotate(q, k, v, lens, parent, rope=rope, q_weight=qw, k_weight=kw)
    got = rd.tree_rotate(q, k, v, lens, parent, rope=rope, q_weight=qw, k_weight=kw, out=q, k_tree=k, v_tree=v)
    assert got[0] is q and all(torch.equal(a, b) for a, b in zip(got, want))


def test_append_status_words(rd):
    from paper_2508_09072_b200 import binding
    rng = np.random.default_rng(21)
    ns, lens = [40, 30, 100, 5], [10, 0, 100, 0]
    q, k, v = projection(rng, (175,), 4, 2, 64, True)
    rope = make_rope(200, 64).cuda()

    def run(cache, ts=None, **kw):
        k0, v0 = cache.k_pool.clone(), cache.v_pool.clone()
        out = torch.full((175, 4, 64), 3.0, dtype=torch.bfloat16, device="cuda")
        _, st = rd.prompt_append(q, k, v, cache, starts(ns) if ts is None else ts, rope=kw.get("rope", rope), out=out)
        same = torch.equal(cache.k_pool.view(torch.int16), k0.view(torch.int16)) and torch.equal(cache.v_pool.view(torch.int16), v0.view(torch.int16))
        return out, st.tolist(), same
    fresh = lambda: make_cache(np.random.default_rng(22), lens, [a + b for a, b in zip(ns, lens)], 2, 64)  # noqa: E731
    good, st, _ = run(fresh())
    assert st == [0] * 4
    c = fresh()
    c.page_table[2, 3] = c.k_pool.shape[0]      # the last page of the third sequence
    out, st, _ = run(c)
    assert st == [0, 0, binding.ERR_BAD_PAGE, 0] and not out[70:170].any()
    assert torch.equal(out[:70], good[:70]) and torch.equal(out[170:], good[170:])
    c = fresh()
    c.page_table[2, 0] = -7                     # a page that is not written
    assert run(c)[1] == [0] * 4
    c = fresh()
    c.seq_lens[0], c.seq_lens[1] = -1, 2 ** 31 - 1
    out, st, _ = run(c)
    assert st == [binding.ERR_CAPACITY, binding.ERR_CAPACITY, 0, 0] and not out[:70].any()
    out, st, _ = run(fresh(), rope=rope[:199].contiguous())
    assert st == [0, 0, binding.ERR_CAPACITY, 0]
    c = fresh()
    c.shared_prefix_len = 64
    assert run(c)[1] == [binding.ERR_CAPACITY, binding.ERR_CAPACITY, 0, binding.ERR_CAPACITY]
    for bad in ([0, 40, 30, 90, 95], [-1, 40, 70, 90, 95], [0, 40, 70, 90, 176]):
        out, st, same = run(fresh(), torch.tensor(bad, dtype=torch.int32).cuda())
        assert st == [binding.ERR_INVALID_ARG] * 4 and same and (out == 3.0).all()


def test_tree_rotate_status_words(rd):
    from paper_2508_09072_b200 import binding
    rng = np.random.default_rng(23)
    T = 9
    parent = np.stack([W.chain_tree(T)] * 5).astype(np.int32)
    parent[1, 4], parent[2, 0] = 4, 0
    lens = torch.tensor([3, 0, 0, -1, 4], dtype=torch.int32).cuda()
    q, k, v = projection(rng, (5, T), 4, 2, 64, True)
    *got, st = rd.tree_rotate(q, k, v, lens, torch.from_numpy(parent).cuda(), rope=make_rope(12, 64).cuda())
    assert st.tolist() == [0, binding.ERR_BAD_TREE, binding.ERR_BAD_TREE, binding.ERR_CAPACITY, binding.ERR_CAPACITY]
    for x in got:
        assert not x[1:].any() and x[0].any()


def test_rotation_refusals(rd):
    from paper_2508_09072_b200 import binding
    rng = np.random.default_rng(24)
    cache = make_cache(rng, [0], [64], 2, 64)
    q, k, v = projection(rng, (5,), 4, 2, 64, True)
    ts = starts([5])

    def refused(code, **kw):
        with pytest.raises(binding.ReaderError) as e:
            rd.prompt_append(kw.pop("q", q), k, v, cache, ts, **kw)
        assert e.value.code == code
    w = bf16(rng, 64).cuda()
    refused(binding.ERR_INVALID_ARG, q_weight=w)
    refused(binding.ERR_INVALID_ARG, q_weight=w, k_weight=w, eps=-1.0)
    refused(binding.ERR_INVALID_ARG, q_weight=w, k_weight=w, eps=float("nan"))
    refused(binding.ERR_UNSUPPORTED, rope=make_rope(64, 40).cuda())
    refused(binding.ERR_INVALID_ARG, rope=make_rope(64, 80).cuda())
    refused(binding.ERR_UNSUPPORTED, q=projection(rng, (5,), 3, 2, 64, False)[0])
    odd = torch.empty(5 * (4 * 64 + 4), dtype=torch.bfloat16, device="cuda").as_strided((5, 4, 64), (4 * 64 + 4, 64, 1))
    refused(binding.ERR_INVALID_ARG, q=odd)
    with pytest.raises(ValueError):
        rd.prompt_append(q.transpose(0, 1).contiguous().transpose(0, 1), k, v, cache, ts)
    with pytest.raises(ValueError):
        rd.prompt_append(q, k[:, :1], v, cache, ts)
    with pytest.raises(TypeError):
        rd.prompt_append(q.half(), k, v, cache, ts)
    with pytest.raises(ValueError):
        rd.prompt_append(q, k, v, cache, ts, q_weight=w[:32].contiguous(), k_weight=w)


# ---------------------------------------------------------------------------------------------- all of it together
def test_prompt_then_decoding_steps(rd):
    """Two layers: a prompt in two pieces, a token without a draft, then a step with a draft tree and its commit; every
    attention against the plain one over what the caches hold."""
    rng = np.random.default_rng(30)
    Hq, Hkv, D, B, T, layers = 8, 2, 128, 3, 11, 2
    room = [400, 150, 90]
    first = make_cache(rng, [0] * B, room, Hkv, D)
    caches = [first]
    for _ in range(layers - 1):
        c = make_cache(rng, [0] * B, room, Hkv, D)
        c.page_table, c.seq_lens = first.page_table, first.seq_lens
        c.k_pool, c.v_pool = bf16(rng, *first.k_pool.shape).cuda(), bf16(rng, *first.k_pool.shape).cuda()
        caches.append(c)
    rope, (qw, kw) = make_rope(512, 128), weights(rng, D, True)
    lens = [0] * B
    for ns in ([200, 64, 0], [90, 1, 63], [1, 1, 1]):
        for i, c in enumerate(caches):
            q, k, v = projection(rng, (sum(ns),), Hq, Hkv, D, True)
            q2, st = rd.prompt_append(q, k, v, c, starts(ns), rope=rope.cuda(), q_weight=qw, k_weight=kw)
            out, st2 = rd.prompt_attn(q2, c, starts(ns), D ** -0.5, update_seq_lens=i == layers - 1)
            assert st.tolist() == st2.tolist() == [0] * B
            want, _, tol, _ = plain_attn(q2, c, ns, lens, D ** -0.5)
            within(out, want, tol)
        lens = [a + b for a, b in zip(lens, ns)]
        assert first.seq_lens.tolist() == lens
    parent = np.stack([W.capped_recursive_tree(rng, T, 6, 3) for _ in range(B)]).astype(np.int32)
    dev_parent = torch.from_numpy(parent).cuda()
    path = torch.full((B, 4), -1, dtype=torch.int32)
    path[:, 0] = 0
    kids = [int(np.nonzero(parent[b] == 0)[0][0]) for b in range(B)]
    path[:, 1] = torch.tensor(kids)
    n_acc = torch.full((B,), 2, dtype=torch.int32)
    for i, c in enumerate(caches):
        q, k, v = projection(rng, (B, T), Hq, Hkv, D, True)
        q2, k2, v2, st = rd.tree_rotate(q, k, v, c.seq_lens, dev_parent, rope=rope.cuda(), q_weight=qw, k_weight=kw)
        out, st2 = rd.verify_attn(q2, k2, v2, c, dev_parent, D ** -0.5)
        assert st.tolist() == st2.tolist() == [0] * B
        rd.kv_commit(c, k2, v2, path.cuda(), n_acc.cuda(), update_seq_lens=i == layers - 1)
        # the accepted child is what plain decoding gives at its position: the same key, the same attention
        chain = torch.stack([q2[b, [0, kids[b]]] for b in range(B)]).reshape(2 * B, Hq, D)
        view = type(c)(c.k_pool, c.v_pool, c.page_table, torch.tensor(lens, dtype=torch.int32).cuda())
        got, _ = rd.prompt_attn(chain.contiguous(), view, starts([2] * B), D ** -0.5)
        want, _, tol, _ = plain_attn(chain, view, [2] * B, lens, D ** -0.5)
        within(got, want, tol)
        within(torch.stack([out[b, [0, kids[b]]] for b in range(B)]).reshape(2 * B, Hq, D), want, tol)
    assert first.seq_lens.tolist() == [x + 2 for x in lens]
