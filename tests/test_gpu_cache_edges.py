"""The 4-bit cache's attention and the page calls where they can go wrong quietly.  Tolerances as in test_gpu_q4 unless a test derives its own."""
import numpy as np
import pytest
import torch

from test_gpu_q4 import attend, binding, held, i32, make, plain_attn, rd, rows_of, sees_of, widened, within  # noqa: F401 (rd: a fixture)

from test_gpu_pages import Model, pages

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


# ---------------------------------------------------------------------------------------------- infinite values
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,group", [(5, 1), (16, 1), (40, 4), (100, 3), (128, 2)])
@pytest.mark.parametrize("masks", [False, True])
def test_infinite_values_of_several_nodes_add_up(rd, d, T, group, masks):
    """A column has what all the nodes that a row sees add to it: their sum in fp32, infinite or NaN (of +inf and -inf), in one column or in many."""
    rng = np.random.default_rng(61)
    lens = [70, 0, 200]
    both, cache, q, kt, vt, parent = make(rng, lens, T, 2, group, d)
    for s in range(3):   # (a path down half of the nodes, so that rows see several)
        parent[s, 1:T // 2] = np.arange(T // 2 - 1)
    want = plain_attn(both, lens, q, kt, vt, parent, 0.1)
    x = vt.clone()
    for s in range(3):
        for h in range(2):
            for n in rng.permutation(T)[:max(3, T // 4)]:
                for e in rng.permutation(d)[:3].tolist() + [1, d - 1]:
                    x[s, n, h, e] = float(rng.choice([np.inf, -np.inf, np.inf, np.nan] if s == 1 else [np.inf, -np.inf] if s == 0 else [np.inf]))
    kw = {"anc_mask": rd.tree_encode(i32(parent))[0]} if masks else {}
    out, lse, st = attend(rd, cache, q, kt, x, parent, 0.1, **kw)
    assert st == [0] * 3
    seen = torch.from_numpy(np.stack([sees_of(p) for p in parent]))                       # [b, rows, nodes]
    count = lambda which: torch.einsum("btn,bnhd->bthd", seen.double(), which(x.double()).double()).repeat_interleave(group, 2)  # noqa: E731
    plus, minus, nan = count(lambda y: y == np.inf), count(lambda y: y == -np.inf), count(torch.isnan)
    assert (plus > 1).any() and ((plus > 0) & (minus > 0)).any()
    is_nan, is_plus, is_minus = (nan > 0) | (plus > 0) & (minus > 0), (plus > 0) & (minus == 0) & (nan == 0), (minus > 0) & (plus == 0) & (nan == 0)
    assert torch.isnan(out[is_nan]).all() and (out[is_plus] == np.inf).all() and (out[is_minus] == -np.inf).all()
    rest = ~(is_nan | is_plus | is_minus)
    assert ((out.double() - want[0]).abs() <= want[2])[rest].all() and ((lse.double() - want[1]).abs() <= want[3]).all()


# ---------------------------------------------------------------------------------------------- scores and scales at the ends of fp32
FP32_MAX = torch.finfo(torch.float32).max


def one_hot(rng, shape, value):
    """Queries with one element that is not 0: a score is that times an element of a key, which fp32 holds exactly."""
    q = torch.zeros(shape, dtype=torch.bfloat16)
    at = torch.from_numpy(rng.integers(0, shape[-1], shape[:-1]))
    return q.scatter_(-1, at[..., None], torch.full((*shape[:-1], 1), value, dtype=torch.bfloat16))


@pytest.mark.parametrize("columns", [None, 700])
@pytest.mark.parametrize("T", [1, 4, 40])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("size,scale", [(2.0 ** 100, 2.0 ** 30), (2.0 ** 118, 64.0), (1.0, 1.9e38)])
def test_scaled_scores_beyond_fp32(rd, size, scale, sign, T, columns):
    """Finite scores whose products with the scale are not: a row's largest keys share it, whatever the largest score's sign.  Scores are exact and differ by 0 or by
    far more than 2^10 scaled, so that weights are exact, too: what is left are the roundings to bf16 of 1 / n (its sum: n terms in fp32) and of the output."""
    rng = np.random.default_rng(50)
    lens = [300, 65, 2000]
    both, cache, q, kt, vt, parent = make(rng, lens, T, 2, 2, 64, scale=16.0)
    if sign < 0:   # keys below 0 alone, far enough that none is held as 0
        both.k.copy_(-both.k.abs() - 16)
        rd.q4_store([both.wide], [both.narrow], torch.zeros(3, dtype=torch.int32, device="cuda"), cache.seq_lens)
        kt = -kt.abs() - 16
    q = one_hot(rng, tuple(q.shape), size)
    out, lse, st = attend(rd, cache if columns is None else widened(cache, columns), q, kt, vt, parent, scale)
    assert st == [0] * 3
    o, z, mag = plain_rows(both, lens, q, kt, vt, parent, scale)
    far = z.abs() > FP32_MAX
    assert far.any() and (lse[far] == torch.where(z[far] > 0, torch.inf, -torch.inf)).all()
    assert ((lse.double() - z).abs() <= z.abs() * 2.0 ** -22)[z.abs() < FP32_MAX / 2].all()
    assert ((out.double() - o).abs() <= 2.0 ** -8 * (mag + o.abs()) * 1.01 + 1e-30).all()


def plain_rows(both, lens, q, kt, vt, parent, scale):
    """out, lse and the sums of weights times magnitudes in 64 bits, the maximum taken off before the exponentials (beside scores of 2^128 a logarithm is lost in 64 bits, too)."""
    out, mag, lse = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape[:3], dtype=torch.float64)
    group = q.shape[2] // kt.shape[2]
    for b, n in enumerate(lens):
        k = torch.cat([held(rows_of(both.k, both.t16, b, 0, n)), kt[b].double()])
        v = torch.cat([held(rows_of(both.v, both.t16, b, 0, n)), vt[b].double()])
        mask = torch.ones(q.shape[1], len(k), dtype=torch.bool)
        mask[:, n:] = torch.from_numpy(sees_of(parent[b]))
        for h in range(q.shape[2]):
            s = (q[b, :, h].double() @ k[:, h // group].T * scale).masked_fill(~mask, -torch.inf)
            p = s.softmax(-1)
            out[b, :, h], mag[b, :, h], lse[b, :, h] = p @ v[:, h // group], p @ v[:, h // group].abs(), s.logsumexp(-1)
    return out, lse, mag


@pytest.mark.parametrize("columns", [None, 700])
@pytest.mark.parametrize("T", [1, 4, 40])
@pytest.mark.parametrize("size,scale", [(2.0 ** 118, 1e-38), (2.0 ** 118, 1e-39), (1.0, 1.5e-38), (1.0, 1e-45)])
def test_the_smallest_scales(rd, size, scale, T, columns):
    """Scales down to the smallest number: weights go by the scaled scores, 0.1 to 1 where the scores are near the end of fp32."""
    rng = np.random.default_rng(51)
    lens = [300, 65, 4000]
    both, cache, q, kt, vt, parent = make(rng, lens, T, 2, 2, 64, scale=16.0)
    q = one_hot(rng, tuple(q.shape), size)
    out, lse, st = attend(rd, cache if columns is None else widened(cache, columns), q, kt, vt, parent, scale)
    assert st == [0] * 3
    o, z, tol, ltol = plain_attn(both, lens, q, kt, vt, parent, float(np.float32(scale)))
    # (a subnormal scale times log2 e is off by half of 2^-149, a score is below 2^125 by far: an exponent by 2^-24 at most)
    within((out, lse), (o, z, tol + 2.0 ** -23 * 8, ltol + 2.0 ** -23))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,group,columns", [(1, 4, None), (1, 4, 700), (4, 4, None), (4, 4, 700), (40, 2, None), (100, 3, None)])
def test_a_readers_first_call_may_be_captured(T, group, columns, d):
    """What a context asks about its kernels once, it may ask while a graph is captured."""
    from paper_2508_09072_b200 import binding as b
    rng = np.random.default_rng(67)
    lens = [300, 5]
    both, cache, q, kt, vt, parent = make(rng, lens, T, 1, group, d)
    if columns:
        cache = widened(cache, columns)
    args = q.cuda(), kt.cuda(), vt.cuda(), cache, i32(parent), 0.1
    out, status = torch.empty_like(args[0]), torch.full((2,), 7, dtype=torch.int32, device="cuda")
    reader = b.Reader(0)
    ws = torch.empty_like(reader.q4_workspace())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        reader.q4_verify_attn(*args, out=out, status=status, workspace=ws)
    graph.replay()
    torch.cuda.synchronize()
    o, _, tol, _ = plain_attn(both, lens, q, kt, vt, parent, 0.1)
    assert status.tolist() == [0, 0] and ((out.cpu().double() - o).abs() <= tol).all()
    del graph
    reader.close()


@pytest.mark.parametrize("d,group,T,lens", [(64, 4096, 1, [70]), (64, 4095, 7, [0, 200]), (128, 4093, 33, [130]), (64, 4095, 128, [64]), (128, 257, 1, [1000, 3])])
def test_the_widest_groups(rd, d, group, T, lens):
    rng = np.random.default_rng(group + T)
    both, cache, q, kt, vt, parent = make(rng, lens, T, 1, group, d)
    got = attend(rd, cache, q, kt, vt, parent, 0.1)
    assert got[2] == [0] * len(lens)
    within(got[:2], plain_attn(both, lens, q, kt, vt, parent, 0.1))


@pytest.mark.parametrize("T,group", [(1, 4), (40, 2), (100, 3)])
@pytest.mark.parametrize("big", [2048.0, 4096.0, 6144.0, 8192.0, 65536.0])
def test_shares_with_large_maxima_of_their_own(rd, big, T, group):
    """One long sequence cut into many shares whose largest scores differ by a few units beside 2^14 to 2^19 (scaled, in log2 units).  Scores have two terms and are rounded
    once at most: what counts is the exponents' 2^-23 of the largest scaled score, and 2^-8 for the roundings to bf16 of a probability and of the output."""
    rng = np.random.default_rng(66)
    L, d = 9000, 64
    both, cache, q, kt, vt, parent = make(rng, [L], T, 1, group, d)
    pos = torch.arange(L)
    page, at = torch.from_numpy(both.t16[0])[pos // 64].long().cuda(), (pos % 64).cuda()
    level = torch.from_numpy(rng.integers(-3, 4, L // 512 + 1)).repeat_interleave(512)[:L] + torch.from_numpy(rng.integers(-4, 1, L))
    both.k.zero_()
    both.k[page, 0, at, 3] = 7.0                                        # (7 of a scale of 1)
    both.k[page, 0, at, 20] = (level / 4).to(torch.bfloat16).cuda()     # (whole numbers up to 7 of a scale of 1 / 4 or less)
    rd.q4_store([both.wide], [both.narrow], i32([0]), i32([L]))
    kt = torch.zeros_like(kt)
    kt[..., 3], kt[..., 20] = 7.0, 0.25
    q = torch.zeros_like(q)
    q[..., 3], q[..., 20] = big, 2.0
    out, lse, st = attend(rd, cache, q, kt, vt, parent, 1.0)
    assert st == [0]
    o, z, mag = plain_rows(both, [L], q, kt, vt, parent, 1.0)
    off = 2.0 ** -23 * 7 * big * 1.4427 * 2 * np.log(2)     # of a weight, and of the sum that it is divided by
    off += (L + T) * 2.0 ** -23
    assert ((out.double() - o).abs() <= 2.0 ** -8 * (mag + o.abs()) * 1.01 + mag * off).all()
    assert ((lse.double() - z).abs() <= off + z * 2.0 ** -23).all()


# ---------------------------------------------------------------------------------------------- pages
@pytest.mark.parametrize("rows", [7, 70])
def test_rows_without_a_committed_page_get_none(rd, rows):
    """Wherever the missing page is; other requests are served, and pages that nothing is written to need not be in the pool."""
    b = binding()
    rng = np.random.default_rng(62)
    m = Model(rng, 60 * rows, rows, 50, 1, 16)
    free = rng.permutation(60 * rows).tolist()
    for r in range(rows):
        m.lens[r] = [64 * 40, 64 * 40 + 1, 1, 64, 0, 64 * 33 + 7, 64 * 40][r % 7]
        for e in range(pages(m.lens[r])):
            m.table[r][e] = free.pop()
            m.refs[m.table[r][e]] = 1
    want = []
    for r in range(rows):
        hole = [0, 39, None, 0, None, 32, 35][r % 7]
        if hole is not None:
            m.refs[m.table[r][hole]] = 0
            m.table[r][hole] = -1
        want.append(0 if hole is None else b.ERR_BAD_PAGE)
    m.table[2][49] = -7
    p = m.device()
    before = [list(x) for x in m.table]
    assert rd.pages_reserve(p, i32(range(rows)), i32([0] * rows)).tolist() == [0] * rows
    assert rd.pages_reserve(p, i32(range(rows)), i32([70] * rows)).tolist() == want
    table, refs = p.page_table.tolist(), p.refs.tolist()
    served = [r for r in range(rows) if want[r] == 0]
    fresh = [table[r][e] for r in served for e in range(m.lens[r] // 64, pages(m.lens[r] + 70)) if before[r][e] < 0]
    assert fresh == [page for page, n in enumerate(m.refs) if n == 0][:len(fresh)] and all(refs[page] == 1 for page in fresh)
    for r in range(rows):
        if r in served:
            n = pages(m.lens[r])
            assert table[r][:n] == before[r][:n]
        else:
            assert table[r] == before[r]
    assert sum(refs) == sum(m.refs) + len(fresh) and p.seq_lens.tolist() == m.lens


@pytest.mark.parametrize("num_pages", [60, 4096, 4097, 9000])
@pytest.mark.parametrize("share", [0.0, 0.3, 0.9, 1.0])
def test_a_compaction_tells_where_pages_went(rd, num_pages, share):
    """Pages that no entry names (a count of the caller's own) and a second table over the same pools are found again."""
    rng = np.random.default_rng(63)
    m = Model(rng, num_pages, 10, 20, 2, 16)
    used = rng.permutation(num_pages)[:int(num_pages * share)].tolist()
    for i, page in enumerate(used):
        m.refs[page] = 1
        if i < 150:
            m.table[i // 20][i % 20] = page
    p = m.device()
    data = [x.clone() for x in p.pools]
    new_ids = torch.full((num_pages,), 7, dtype=torch.int32, device="cuda")
    assert rd.pages_compact(p, new_ids=new_ids).tolist() == [m.compact()] == [len(used)]
    m.same(p)
    ids = new_ids.cpu().long()
    held = torch.zeros(num_pages, dtype=torch.bool)
    held[used] = True
    assert (ids[~held] == -1).all() and sorted(ids[held].tolist()) == list(range(len(used)))
    for was, now in zip(data, p.pools):
        assert torch.equal(now[ids[held].cuda()], was[held.cuda()])
    again = torch.empty_like(new_ids)   # nothing moves a second time
    rd.pages_compact(p, new_ids=again)
    assert again.tolist() == list(range(len(used))) + [-1] * (num_pages - len(used))


def test_new_ids_that_cannot_be(rd):
    m = Model(np.random.default_rng(64), 20, 2, 4, 1, 16)
    p = m.device()
    for wrong, error in ((torch.zeros(19, dtype=torch.int32, device="cuda"), ValueError), (torch.zeros(20, dtype=torch.int64, device="cuda"), TypeError),
                         (torch.zeros(20, dtype=torch.int32), TypeError), (torch.zeros(40, dtype=torch.int32, device="cuda")[::2], TypeError)):
        with pytest.raises(error, match="new_ids"):
            rd.pages_compact(p, new_ids=wrong)


def test_workspaces_of_growing_calls_take_little_room():
    """Calls that have a few requests more each time: all the buffers together are less than twice what the largest call may be given."""
    from paper_2508_09072_b200 import binding as b
    reader = b.Reader(0)
    p = Model(np.random.default_rng(65), 20, 4, 4000, 1, 16).device()
    for n in range(1, 400, 3):
        ws = reader.pages_workspace(p, n)
        need = reader.lib.reader_pages_workspace_bytes(20, 4, 4000, n)
        assert need <= ws.numel() <= max(2 * need, reader._pages_ws[0].numel())
        assert sum(x.numel() for x in reader._pages_ws) <= 2 * ws.numel()
    reader.close()
