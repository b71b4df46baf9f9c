"""The 4-bit cache against its definition in 64 bits: stored and loaded values (exact), commits, attention.

Tolerance of the attention, counted from its roundings: a probability is rounded to bf16 (2^-8 of itself), the output too, and
sums of n products in fp32 are off by at most n 2^-24 of the sum of magnitudes; 2^-8 (sum p |v| + |out|) and the scores' own
error, (D + 4) 2^-24 sum |q k| scale, which moves a probability by that much of itself."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

PAGE = 64


@pytest.fixture(scope="module")
def rd():
    from paper_2508_09072_b200 import binding
    r = binding.Reader(0)
    yield r
    r.close()


def binding():
    from paper_2508_09072_b200 import binding as b
    return b


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


def bf16(rng, *shape, scale=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(torch.bfloat16)


def scales():
    c = np.arange(255)
    return (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 18)


def held(x):
    """What a tensor [..., d] is after a stay in 4 bits (float64): the definition, by comparing with every scale and rounding x / s."""
    y = x.double().numpy()
    y = y.reshape(*y.shape[:-1], x.shape[-1] // 16, 16)
    top = np.abs(y).max(-1)
    finite = np.isfinite(y).all(-1)
    s = scales()
    code = np.minimum((7.5 * s[None] < np.where(finite, top, 0).reshape(-1, 1)).sum(-1), 254).reshape(top.shape)
    step = s[code][..., None]
    q = np.clip(np.rint(np.where(finite[..., None], y, 0) / step), -7, 7)   # (x / s in 64 bits rounds no quotient to a tie)
    v = np.where(finite[..., None], q * step, np.nan)
    return torch.from_numpy(v.reshape(x.shape))


def table_of(rng, counts, spare=2, shuffle=True):
    """Page table for these numbers of pages; returns it and the pool's size."""
    total = sum(counts) + spare
    order = rng.permutation(total) if shuffle else np.arange(total)
    t = np.full((len(counts), max(max(counts), 1)), -1)
    at = 0
    for b, n in enumerate(counts):
        t[b, :n] = order[at:at + n]
        at += n
    return t, total


def pages(n):
    return (n + PAGE - 1) // PAGE


def rows_of(pool, table, b, lo, hi):
    """Rows [lo .. hi) of sequence b: [n, heads, d] on the host."""
    pos = np.arange(lo, hi)
    return pool.cpu()[torch.from_numpy(table[b][pos // PAGE].astype(np.int64)), :, torch.from_numpy(pos % PAGE)]


class Both:
    """A bf16 cache with random rows and an empty 4-bit one, with page tables of their own."""

    def __init__(self, rng, lens, heads, d, scale=1.0, spare=2):
        b = binding()
        self.t16, n16 = table_of(rng, [pages(x) for x in lens], spare)
        self.t4, n4 = table_of(rng, [pages(x) for x in lens], spare)
        self.k, self.v = (bf16(rng, n16, heads, PAGE, d, scale=scale).cuda() for _ in range(2))
        self.k4, self.v4 = (torch.from_numpy(rng.integers(0, 256, (n4, heads, 36 * d), dtype=np.uint8)).cuda() for _ in range(2))
        lens = i32(lens)
        self.wide = b.KvCache(self.k, self.v, i32(self.t16), lens)
        self.narrow = b.Q4Cache(self.k4, self.v4, i32(self.t4), lens)
        self.out16, self.n16 = torch.full_like(self.k, 3.0), n16
        self.out = b.KvCache(self.out16, torch.full_like(self.v, 3.0), self.wide.page_table, lens)


# ---------------------------------------------------------------------------------------------- store and load
@pytest.mark.parametrize("heads,d", [(1, 64), (8, 64), (2, 128), (8, 128)])
@pytest.mark.parametrize("ranges", [[(0, 64)], [(0, 1)], [(63, 65)], [(5, 6), (6, 7), (0, 0)], [(0, 130), (1, 200), (127, 129), (64, 64)], [(3, 1000)]])
def test_stored_values_are_the_definitions(rd, heads, d, ranges):
    rng = np.random.default_rng(1)
    both = Both(rng, [max(b, 1) for _, b in ranges], heads, d, scale=2.0)
    before = both.k4.clone(), both.v4.clone()
    first, last = i32([a for a, _ in ranges]), i32([b for _, b in ranges])
    assert rd.q4_store([both.wide], [both.narrow], first, last).tolist() == [0] * len(ranges)
    assert rd.q4_load([both.narrow], [both.out], first, last).tolist() == [0] * len(ranges)
    for src, out in ((both.k, both.out.k_pool), (both.v, both.out.v_pool)):
        want = torch.full(src.shape, 3.0, dtype=torch.float64)
        for b, (lo, hi) in enumerate(ranges):
            pos = np.arange(lo, hi)
            page = torch.from_numpy(both.t16[b][pos // PAGE].astype(np.int64))
            want[page, :, torch.from_numpy(pos % PAGE)] = held(rows_of(src, both.t16, b, lo, hi))
        assert torch.equal(out.cpu().double(), want)
    # positions outside the ranges read as they did before
    for was, now, is_key in ((before[0], both.k4, True), (before[1], both.v4, False)):
        touched = np.zeros(was.shape[0], bool)
        for b, (lo, hi) in enumerate(ranges):
            if hi > lo:
                touched[both.t4[b][lo // PAGE:pages(hi)]] = True
        assert torch.equal(was.cpu()[~touched], now.cpu()[~touched])


@pytest.mark.parametrize("d", [64, 128])
def test_neighbouring_positions_keep_their_values(rd, d):
    """Every position by itself, in an order that visits even before odd ones and back: each store leaves the others."""
    rng = np.random.default_rng(2)
    both = Both(rng, [PAGE], 2, d)
    for p in list(range(0, 64, 2)) + list(range(63, 0, -2)):
        rd.q4_store([both.wide], [both.narrow], i32([p]), i32([p + 1]))
    rd.q4_load([both.narrow], [both.out], i32([0]), i32([PAGE]))
    page = both.t16[0][0]
    assert torch.equal(both.out.k_pool[page].cpu().double(), held(both.k[page].cpu()))
    assert torch.equal(both.out.v_pool[page].cpu().double(), held(both.v[page].cpu()))


@pytest.mark.parametrize("d", [64, 128])
def test_values_at_the_borders(rd, d):
    """Zeros, ties, the smallest and largest magnitudes, subnormals, infinities and NaN; every mantissa of every size."""
    rng = np.random.default_rng(3)
    both = Both(rng, [PAGE * 4], 1, d)
    every = torch.arange(0, 0x7f80, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)   # all finite magnitudes
    x = both.k.cpu()
    flat = torch.zeros(x.shape[0] * PAGE, d, dtype=torch.bfloat16)
    n = flat.numel() // 16
    # one block per magnitude as its largest element, the other elements whole eighths of it
    pick = torch.from_numpy(rng.integers(0, every.numel(), n))
    blocks = (every[pick].float()[:, None] * torch.from_numpy(rng.integers(-16, 17, (n, 16)) / 16.0).float()).to(torch.bfloat16)
    blocks[:, 0] = every[pick]
    # ties: odd multiples of half a scale
    s = torch.from_numpy(scales()[rng.integers(0, 255, n // 4)])
    blocks[:n // 4] = (s[:, None] * torch.from_numpy(rng.integers(-15, 16, (n // 4, 16)) / 2.0)).to(torch.bfloat16)
    blocks[:n // 4, 3] = (7.5 * s).to(torch.bfloat16)
    blocks[n // 4, :] = 0
    blocks[n // 4 + 1, 5] = float("inf")
    blocks[n // 4 + 2, 15] = float("-inf")
    blocks[n // 4 + 3, 0] = float("nan")
    blocks[n // 4 + 4] = torch.finfo(torch.bfloat16).max
    blocks[n // 4 + 5] = -torch.finfo(torch.bfloat16).tiny
    perm = torch.from_numpy(rng.permutation(n))
    flat = blocks[perm].reshape(x.shape)
    for pool in (both.k, both.v):
        pool.copy_(flat)
    rd.q4_store([both.wide], [both.narrow], i32([0]), i32([PAGE * 4]))
    rd.q4_load([both.narrow], [both.out], i32([0]), i32([PAGE * 4]))
    used = torch.from_numpy(both.t16[0].astype(np.int64))
    want = held(flat)[used]
    for pool in (both.out.k_pool, both.out.v_pool):
        got = pool.cpu()[used].double()
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))
    # what the header promises of the values
    x = flat[used].double()
    ok = ~torch.isnan(want) & (x.abs() <= 107520)
    top = torch.from_numpy(np.abs(np.where(np.isfinite(x.numpy()), x.numpy(), 0)).reshape(*x.shape[:-1], -1, 16).max(-1))
    s = torch.from_numpy(scales()[np.minimum((7.5 * scales()[None] < top.numpy().reshape(-1, 1)).sum(-1), 254)].reshape(top.shape)).repeat_interleave(16, -1)
    assert ((x - want).abs()[ok] <= s[ok] / 2).all()


def test_many_layers_in_one_call(rd):
    b = binding()
    rng = np.random.default_rng(4)
    n = 35
    both = [Both(np.random.default_rng(7), [70, 3], 2, 64) for _ in range(n)]
    for x in both:   # one table for all, pools of their own
        x.k.copy_(bf16(rng, *x.k.shape)), x.v.copy_(bf16(rng, *x.v.shape))
    wide = [b.KvCache(x.k, x.v, both[0].wide.page_table, both[0].wide.seq_lens) for x in both]
    narrow = [b.Q4Cache(x.k4, x.v4, both[0].narrow.page_table, both[0].wide.seq_lens) for x in both]
    out = [b.KvCache(x.out.k_pool, x.out.v_pool, both[0].wide.page_table, both[0].wide.seq_lens) for x in both]
    first, last = i32([2, 0]), i32([70, 3])
    assert rd.q4_store(wide, narrow, first, last).tolist() == [0, 0]
    assert rd.q4_load(narrow, out, first, last).tolist() == [0, 0]
    for x, o in zip(both, out):
        for seq, lo, hi in ((0, 2, 70), (1, 0, 3)):
            assert torch.equal(rows_of(o.k_pool, x.t16, seq, lo, hi).double(), held(rows_of(x.k, x.t16, seq, lo, hi)))
            assert torch.equal(rows_of(o.v_pool, x.t16, seq, lo, hi).double(), held(rows_of(x.v, x.t16, seq, lo, hi)))


def test_convert_status_words(rd):
    b = binding()
    rng = np.random.default_rng(5)
    both = Both(rng, [128] * 6, 2, 64)
    t16, t4 = both.t16.copy(), both.t4.copy()
    t16[1, 1] = both.n16          # outside the pool
    t4[2, 0] = -1
    wide = b.KvCache(both.k, both.v, i32(t16), both.wide.seq_lens)
    narrow = b.Q4Cache(both.k4, both.v4, i32(t4), both.wide.seq_lens)
    before = both.k4.clone()
    st = rd.q4_store([wide], [narrow], i32([0, 0, 0, -1, 100, 100]), i32([128, 128, 128, 5, 129, 128]))
    assert st.tolist() == [0, b.ERR_BAD_PAGE, b.ERR_BAD_PAGE, b.ERR_CAPACITY, b.ERR_CAPACITY, 0]
    keep = np.concatenate([both.t4[1], both.t4[3], both.t4[4]])
    assert torch.equal(both.k4[keep], before[keep])
    # a bad page outside the range does not matter
    assert rd.q4_store([wide], [narrow], i32([0] * 6), i32([1, 64, 0, 1, 1, 1])).tolist() == [0] * 6
    # nothing is written below a shared prefix
    narrow.shared_prefix_len = 64
    assert rd.q4_store([wide], [narrow], i32([63, 64, 64, 64, 64, 64]), i32([65, 64, 65, 64, 64, 64])).tolist() == [b.ERR_CAPACITY, 0, 0, 0, 0, 0]
    # (the other way the prefix is only read)
    assert rd.q4_load([narrow], [wide], i32([0] * 6), i32([1, 1, 0, 1, 1, 1])).tolist() == [0] * 6


# ---------------------------------------------------------------------------------------------- commit
@pytest.mark.parametrize("d,heads,layers", [(64, 1, 1), (128, 8, 1), (64, 8, 3), (128, 2, 34)])
def test_commit_writes_the_rows_of_the_path(rd, d, heads, layers):
    b = binding()
    rng = np.random.default_rng(6)
    lens = [0, 1, 63, 64, 62, 127]
    n_acc = [1, 5, 4, 0, 3, 7]
    T, max_path, B = 9, 7, len(lens)
    counts = [pages(x + max_path) for x in lens]
    table, total = table_of(rng, counts)
    seq_lens = i32(lens)
    k4, v4 = ([torch.from_numpy(rng.integers(0, 255, (total, heads, 36 * d), dtype=np.uint8)).cuda() for _ in range(layers)] for _ in range(2))
    caches = [b.Q4Cache(k, v, i32(table), seq_lens) for k, v in zip(k4, v4)]
    for c in caches:
        c.page_table = caches[0].page_table
    path = np.full((B, max_path), -1)
    for s in range(B):
        path[s, :n_acc[s]] = np.sort(rng.permutation(T)[:n_acc[s]])
    kt, vt = ([bf16(rng, B, T, heads, d).cuda() for _ in range(layers)] for _ in range(2))
    whole = [(0, c * PAGE) for c in counts]
    load = lambda: [rd_load(rd, c, total, whole) for c in caches]  # noqa: E731
    before = load()
    slots, st = rd.q4_commit(caches, kt, vt, i32(path), i32(n_acc))
    assert st.tolist() == [0] * B and seq_lens.tolist() == [a + n for a, n in zip(lens, n_acc)]
    after = load()
    for s in range(B):
        pos = np.arange(lens[s], lens[s] + n_acc[s])
        assert slots[s].tolist() == (table[s][pos // PAGE] * PAGE + pos % PAGE).tolist() + [-1] * (max_path - n_acc[s])
    for i in range(layers):
        for was, now, tree in ((before[i][0], after[i][0], kt[i]), (before[i][1], after[i][1], vt[i])):
            want = was.double()
            for s in range(B):
                pos = np.arange(lens[s], lens[s] + n_acc[s])
                if len(pos):
                    want[torch.from_numpy(table[s][pos // PAGE].astype(np.int64)), :, torch.from_numpy(pos % PAGE)] = held(tree[s, path[s, :n_acc[s]]].cpu())
            assert torch.equal(torch.nan_to_num(now.double()), torch.nan_to_num(want))


def rd_load(rd, cache, total, ranges):
    """Everything a 4-bit cache's sequences hold, as bf16 pools on the host under the same page table."""
    b = binding()
    d = cache.k_pool.shape[2] // 36
    out = b.KvCache(*(torch.zeros(total, cache.k_pool.shape[1], PAGE, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)), cache.page_table, cache.seq_lens)
    assert set(rd.q4_load([cache], [out], i32([a for a, _ in ranges]), i32([e for _, e in ranges])).tolist()) <= {0}
    return out.k_pool.cpu(), out.v_pool.cpu()


def test_commit_status_words(rd):
    b = binding()
    rng = np.random.default_rng(7)
    table, total = table_of(rng, [2] * 6)
    table[2, 1] = total
    lens = [126, 10, 63, 0, -1, 10]
    cache = b.Q4Cache(*(torch.zeros(total, 2, 36 * 64, dtype=torch.uint8, device="cuda") for _ in range(2)), i32(table), i32(lens))
    kt = bf16(rng, 6, 4, 2, 64).cuda()
    path = i32([[0, 1, 2], [0, 4, 2], [0, 1, 2], [0, 1, 2], [0, 1, 2], [0, 1, 2]])
    slots, st = rd.q4_commit([cache], [kt], [kt], path, i32([3, 2, 2, 4, 1, 0]))
    assert st.tolist() == [b.ERR_CAPACITY] * 5 + [0] and (slots == -1).all() and cache.seq_lens.tolist() == lens
    assert not cache.k_pool.any() and not cache.v_pool.any()
    cache.shared_prefix_len = 64
    _, st = rd.q4_commit([cache], [kt], [kt], path, i32([0, 1, 0, 0, 0, 1]))
    assert st.tolist() == [0, b.ERR_CAPACITY, 0, 0, 0, b.ERR_CAPACITY]


# ---------------------------------------------------------------------------------------------- attention
def random_parents(rng, B, T):
    p = np.full((B, T), -1)
    for j in range(1, T):
        p[:, j] = rng.integers(max(0, j - 6), j, B)
    return p


def sees_of(parent):
    T = len(parent)
    s = np.zeros((T, T), bool)
    for j in range(T):
        if parent[j] >= 0:
            s[j] = s[parent[j]]
        s[j, j] = True
    return s


def make(rng, lens, T, heads, group, d, extra_pages=0, scale=1.0):
    b = binding()
    both = Both(rng, [max(x, 1) for x in lens], heads, d, scale=scale)
    st = rd_store(both, lens)
    B = len(lens)
    q, kt, vt = bf16(rng, B, T, heads * group, d), bf16(rng, B, T, heads, d), bf16(rng, B, T, heads, d)
    parent = random_parents(rng, B, T)
    cache = b.Q4Cache(both.k4, both.v4, both.narrow.page_table, i32(lens))
    assert st
    return both, cache, q, kt, vt, parent


_rd = None


def rd_store(both, lens):
    global _rd
    if _rd is None:
        _rd = binding().Reader(0)
    first = i32([0] * len(lens))
    return set(_rd.q4_store([both.wide], [both.narrow], first, i32(lens)).tolist()) == {0}


def plain_attn(both, lens, q, kt, vt, parent, scale, sees=None):
    """out, lse and their tolerances in 64 bits."""
    B, T, hq, d = q.shape
    heads = kt.shape[2]
    group = hq // heads
    out, tol = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    lse, ltol = torch.zeros(q.shape[:3], dtype=torch.float64), torch.zeros(q.shape[:3], dtype=torch.float64)
    for b in range(B):
        k = torch.cat([held(rows_of(both.k, both.t16, b, 0, lens[b])), kt[b].double()])
        v = torch.cat([held(rows_of(both.v, both.t16, b, 0, lens[b])), vt[b].double()])
        mask = torch.ones(T, lens[b] + T, dtype=torch.bool)
        mask[:, lens[b]:] = torch.from_numpy(sees_of(parent[b]) if sees is None else sees[b])
        for h in range(heads):
            x = q[b, :, h * group:(h + 1) * group].double()
            s = torch.einsum("tgd,kd->tgk", x, k[:, h]) * scale
            err = torch.einsum("tgd,kd->tgk", x.abs(), k[:, h].abs()) * scale * (d + 4) * 2.0 ** -24
            s = s.masked_fill(~mask[:, None], -torch.inf)
            z = torch.logsumexp(s, -1)
            p = (s - z[..., None]).exp()
            worst = torch.where(mask[:, None], err, 0.0).amax(-1)
            o = torch.einsum("tgk,kd->tgd", p, v[:, h])
            mag = torch.einsum("tgk,kd->tgd", p, v[:, h].abs())
            rows = slice(h * group, (h + 1) * group)
            out[b, :, rows], lse[b, :, rows] = o, z
            n = lens[b] + T
            tol[b, :, rows] = 2.0 ** -8 * (mag + o.abs()) * 1.01 + mag * (2 * worst[..., None] + n * 2.0 ** -23 + 2.0 ** -20) + 1e-30
            ltol[b, :, rows] = 2 * worst + n * 2.0 ** -23 + 2.0 ** -20 + z.abs() * 2.0 ** -22
    return out, lse, tol, ltol


def attend(rd, cache, q, kt, vt, parent, scale, **kw):
    B, T, hq, d = q.shape
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((B, T, hq), 7.0, dtype=torch.float32, device="cuda")
    rd.q4_workspace().fill_(0xFF)
    _, st = rd.q4_verify_attn(q.cuda(), kt.cuda(), vt.cuda(), cache, i32(parent), scale, out=out, lse=lse, **kw)
    return out.cpu(), lse.cpu(), st.tolist()


def within(got, want):
    (out, lse), (o, z, tol, ltol) = got, want
    bad = (out.double() - o).abs() > tol
    assert not bad.any(), ((out.double() - o).abs() / tol).max()
    assert ((lse.double() - z).abs() <= ltol).all(), ((lse.double() - z).abs() / ltol).max()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,group", [(1, 1), (2, 4), (8, 1), (3, 7), (1, 16), (2, 5)])
@pytest.mark.parametrize("T", [1, 2, 16, 33])
def test_attention_is_that_of_the_values(rd, d, heads, group, T):
    rng = np.random.default_rng(d + 10 * heads + group + 100 * T)
    lens = [0, 1, 63, 64, 65, 200, 517]
    both, cache, q, kt, vt, parent = make(rng, lens, T, heads, group, d)
    scale = d ** -0.5
    got = attend(rd, cache, q, kt, vt, parent, scale)
    assert got[2] == [0] * len(lens)
    within(got[:2], plain_attn(both, lens, q, kt, vt, parent, scale))


@pytest.mark.parametrize("d,heads,group,T,lens", [
    (128, 8, 4, 128, [700, 64]), (64, 2, 8, 128, [130]), (128, 1, 1, 65, [64, 0, 3]), (64, 1, 128, 3, [100, 1]), (128, 2, 3, 100, [900, 31, 257]),
    (128, 1, 4, 1, [20000]), (64, 1, 1, 1, [70000]), (128, 2, 2, 20, [5000, 10, 4000]), (128, 8, 4, 32, [1500, 64, 900, 2500])])
def test_attention_of_large_trees_and_long_caches(rd, d, heads, group, T, lens):
    rng = np.random.default_rng(sum(lens) + T)
    both, cache, q, kt, vt, parent = make(rng, lens, T, heads, group, d)
    scale = d ** -0.5
    got = attend(rd, cache, q, kt, vt, parent, scale)
    assert got[2] == [0] * len(lens)
    within(got[:2], plain_attn(both, lens, q, kt, vt, parent, scale))


def test_large_batches(rd):
    """More sequences than the prefix table has entries, most of them short, some empty."""
    rng = np.random.default_rng(11)
    for B, T, group in ((1500, 1, 2), (2100, 3, 1), (1030, 40, 4)):
        lens = rng.integers(0, 80, B).tolist()
        lens[7], lens[B - 1], lens[B // 2] = 0, 400, 1
        both, cache, q, kt, vt, parent = make(rng, lens, T, 1, group, 64)
        got = attend(rd, cache, q, kt, vt, parent, 0.125)
        assert got[2] == [0] * B
        some = [0, 7, 31, 32, 33, B // 2, B - 2, B - 1] + rng.integers(0, B, 12).tolist()
        pick = lambda x: x[torch.tensor(some)]  # noqa: E731
        sub = Both.__new__(Both)
        sub.k, sub.v, sub.t16 = both.k, both.v, both.t16[some]
        within((pick(got[0]), pick(got[1])), plain_attn(sub, [lens[i] for i in some], pick(q), pick(kt), pick(vt), parent[some], 0.125))


@pytest.mark.parametrize("T,group", [(1, 4), (40, 4)])
def test_bytes_that_are_not_committed_have_no_influence(rd, T, group):
    rng = np.random.default_rng(12)
    for d in (64, 128):
        lens = [1, 40, 64, 100, 0, 33]
        both, cache, q, kt, vt, parent = make(rng, lens, T, 2, group, d)
        want = attend(rd, cache, q, kt, vt, parent, 0.1)
        b = binding()
        bad = b.KvCache(torch.full_like(both.k, float("nan")), torch.full_like(both.v, float("inf")), both.wide.page_table, both.wide.seq_lens)
        width = both.t4.shape[1] * PAGE
        ends = [pages(max(x, 1)) * PAGE for x in lens]
        for fill in ("nan", "ff", "zero"):
            if fill == "nan":
                assert set(rd.q4_store([bad], [both.narrow], i32(lens), i32(ends)).tolist()) == {0}
            else:   # whole pools of these bytes, the committed rows stored again
                both.k4.fill_(255 if fill == "ff" else 0)
                both.v4.fill_(255 if fill == "ff" else 0)
                assert rd_store(both, lens)
            got = attend(rd, cache, q, kt, vt, parent, 0.1)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert width


@pytest.mark.parametrize("T", [1, 40])
@pytest.mark.parametrize("where", [0, 64, 777, 4000])
def test_a_nan_that_is_committed_reaches_the_rows_that_see_it(rd, T, where):
    """In keys: all elements of the head's rows.  In values: the block's 16 elements.  Whatever pieces the sequence is cut into."""
    rng = np.random.default_rng(13)
    lens = [4001, 50]
    both, cache, q, kt, vt, parent = make(rng, lens, T, 2, 4, 128)
    want = plain_attn(both, lens, q, kt, vt, parent, 0.1)
    page, at = both.t16[0][where // PAGE], where % PAGE
    for pool, key in ((both.k, True), (both.v, False)):
        was = pool[page, 1, at].clone()
        pool[page, 1, at, 37] = float("nan")
        rd_store(both, lens)
        out, lse, st = attend(rd, cache, q, kt, vt, parent, 0.1)
        assert st == [0, 0]
        hit = torch.zeros(out.shape, dtype=torch.bool)
        hit[0, :, 4:, slice(None) if key else slice(32, 48)] = True
        assert torch.isnan(out[hit]).all() and (torch.isnan(lse[0, :, 4:]).all() == key)
        assert ((out.double() - want[0]).abs() <= want[2])[~hit].all()
        pool[page, 1, at] = was
    rd_store(both, lens)


def test_nan_over_whole_pieces(rd):
    """Pieces in which a row sees nothing but NaN have the maximum -inf and a NaN sum: the merge keeps it."""
    rng = np.random.default_rng(14)
    lens = [8192]
    both, cache, q, kt, vt, parent = make(rng, lens, 1, 1, 4, 64)
    clean = both.k.clone()
    for lo, hi in ((0, 1024), (3000, 8192), (8191, 8192), (0, 8192)):
        both.k.copy_(clean)
        pos = np.arange(lo, hi)
        both.k[torch.from_numpy(both.t16[0][pos // PAGE].astype(np.int64)).cuda(), 0, torch.from_numpy(pos % PAGE).cuda()] = float("nan")
        rd_store(both, lens)
        out, lse, _ = attend(rd, cache, q, kt, vt, parent, 0.1)
        assert torch.isnan(out).all() and torch.isnan(lse).all()


@pytest.mark.parametrize("T", [1, 40])
def test_scores_of_any_size(rd, T):
    """Large keys and queries: the scores' differences decide, however large the scores."""
    rng = np.random.default_rng(15)
    lens = [300, 65]
    for qs in (1.0, 64.0, 2.0 ** 20, 2.0 ** 60):
        both, cache, q, kt, vt, parent = make(rng, lens, T, 2, 2, 64, scale=16.0)
        # one-hot queries: a score is one element of a key, so fp32 holds it exactly
        hot = torch.zeros_like(q)
        at = torch.from_numpy(rng.integers(0, 64, q.shape[:3]))
        hot.scatter_(3, at[..., None], torch.full((*q.shape[:3], 1), qs, dtype=torch.bfloat16))
        got = attend(rd, cache, hot, kt, vt, parent, 0.125)
        o, z, tol, ltol = plain_attn(both, lens, hot, kt, vt, parent, 0.125)
        assert ((got[0].double() - o).abs() <= tol).all()
        assert ((got[1].double() - z).abs() <= ltol).all()


@pytest.mark.parametrize("T", [1, 40])
def test_status_words(rd, T):
    b = binding()
    rng = np.random.default_rng(16)
    lens = [100, 200, 130, 64, 90, 10]
    both, cache, q, kt, vt, parent = make(rng, lens, T, 2, 4, 128)
    want = plain_attn(both, lens, q, kt, vt, parent, 0.1)
    table, now, par = both.t4.copy(), list(lens), parent.copy()
    table[1, 3] = both.n16              # the last page of sequence 1
    now[2] = table.shape[1] * PAGE + 1
    par[4, 0] = 0
    table[5, 1:] = -5                   # behind its only page: not looked at
    cache = b.Q4Cache(both.k4, both.v4, i32(table), i32(now))
    out, lse, st = attend(rd, cache, q, kt, vt, par, 0.1)
    assert st == [0, b.ERR_BAD_PAGE, b.ERR_CAPACITY, 0, b.ERR_BAD_TREE, 0]
    for i in (1, 2, 4):
        assert not out[i].any() and not lse[i].any()
    good = torch.tensor([0, 3, 5])
    within((out[good], lse[good]), tuple(x[good] for x in want))
    now[2] = -1
    cache = b.Q4Cache(both.k4, both.v4, i32(table), i32(now))
    assert attend(rd, cache, q, kt, vt, par, 0.1)[2] == st
    # every length wrong: no unit at all
    cache = b.Q4Cache(both.k4, both.v4, i32(table), i32([-1] * 6))
    out, lse, st = attend(rd, cache, q, kt, vt, parent, 0.1)
    assert st == [b.ERR_CAPACITY] * 6 and not out.any() and not lse.any()


@pytest.mark.parametrize("T", [1, 40])
def test_an_empty_pool(rd, T):
    b = binding()
    rng = np.random.default_rng(17)
    none = torch.empty(0, 2, 36 * 64, dtype=torch.uint8, device="cuda")
    some = torch.empty(1, 2, 36 * 64, dtype=torch.uint8, device="cuda")
    q, kt, vt, parent = bf16(rng, 2, T, 4, 64), bf16(rng, 2, T, 2, 64), bf16(rng, 2, T, 2, 64), random_parents(rng, 2, T)
    # (an empty tensor has no address; a pool without pages is refused like a missing one)
    with pytest.raises(b.ReaderError):
        attend(rd, b.Q4Cache(none, none, i32([[0], [0]]), i32([0, 0])), q, kt, vt, parent, 0.1)
    out, lse, st = attend(rd, b.Q4Cache(some, some, i32([[-1], [-1]]), i32([0, 0])), q, kt, vt, parent, 0.1)
    assert st == [0, 0]
    both = Both.__new__(Both)
    both.k = both.v = torch.zeros(1, 2, PAGE, 64)
    both.t16 = np.zeros((2, 1), int)
    within((out, lse), plain_attn(both, [0, 0], q, kt, vt, parent, 0.1))


@pytest.mark.parametrize("T", [1, 40, 100])
def test_given_masks_are_used(rd, T):
    rng = np.random.default_rng(18)
    lens = [70, 0, 300]
    both, cache, q, kt, vt, parent = make(rng, lens, T, 2, 4, 64)
    anc, _, _ = rd.tree_encode(i32(parent))
    a = attend(rd, cache, q, kt, vt, parent, 0.1)
    b = attend(rd, cache, q, kt, vt, parent, 0.1, anc_mask=anc)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    # masks of the caller's own: the node alone; nothing at all
    alone = torch.zeros(3, T, 2, dtype=torch.int64)
    for j in range(T):
        alone[:, j, j // 64] = 1 << (j % 64) if j % 64 < 63 else -(1 << 63)
    got = attend(rd, cache, q, kt, vt, parent, 0.1, anc_mask=alone.cuda())
    within(got[:2], plain_attn(both, lens, q, kt, vt, parent, 0.1, sees=[np.eye(T, dtype=bool)] * 3))
    out, lse, st = attend(rd, cache, q, kt, vt, parent, 0.1, anc_mask=torch.zeros(3, T, 2, dtype=torch.int64, device="cuda"))
    assert st == [0, 0, 0] and not out[1].any() and (lse[1] == -float("inf")).all()
    want = plain_attn(both, [70, 1, 300], q, kt, vt, parent, 0.1, sees=[np.zeros((T, T), bool)] * 3)
    within((out[::2], lse[::2]), tuple(x[::2] for x in want))


@pytest.mark.parametrize("T", [1, 40])
def test_the_same_bits_on_every_call_and_captured_calls_follow_the_lengths(rd, T):
    rng = np.random.default_rng(19)
    lens = [4000, 10, 700, 2500]
    both, cache, q, kt, vt, parent = make(rng, lens, T, 2, 4, 128)
    args = q.cuda(), kt.cuda(), vt.cuda(), cache, i32(parent), 0.1
    first = attend(rd, cache, q, kt, vt, parent, 0.1)
    for _ in range(20):
        assert torch.equal(attend(rd, cache, q, kt, vt, parent, 0.1)[0], first[0])
    out, status = torch.empty_like(q, device="cuda"), torch.empty(4, dtype=torch.int32, device="cuda")
    ws = torch.empty_like(rd.q4_workspace())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rd.q4_verify_attn(*args, out=out, status=status, workspace=ws)
    for now in (lens, [1, 0, 64, 2500], [3999, 3, 2, 1], lens):
        cache.seq_lens.copy_(i32(now))
        ws.fill_(0xAB)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.cpu(), attend(rd, cache, q, kt, vt, parent, 0.1)[0]) and status.tolist() == [0] * 4


def test_two_streams_with_workspaces_of_their_own(rd):
    rng = np.random.default_rng(20)
    jobs = []
    for T in (1, 40):
        both, cache, q, kt, vt, parent = make(rng, [3000, 100, 900], T, 2, 4, 128)
        want = attend(rd, cache, q, kt, vt, parent, 0.1)[0]
        jobs.append((torch.cuda.Stream(), torch.empty_like(rd.q4_workspace()), (q.cuda(), kt.cuda(), vt.cuda(), cache, i32(parent), 0.1), want, []))
    torch.cuda.synchronize()
    for _ in range(50):
        for stream, ws, args, _, got in jobs:
            with torch.cuda.stream(stream):
                got.append(rd.q4_verify_attn(*args, workspace=ws)[0])
    torch.cuda.synchronize()
    for _, _, _, want, got in jobs:
        assert all(torch.equal(x.cpu(), want) for x in got)


@pytest.mark.parametrize("T", [1, 40])
def test_a_worker_that_gives_up_is_reported(rd, T):
    b = binding()
    rng = np.random.default_rng(21)
    lens = [4000, 3000]
    both, cache, q, kt, vt, parent = make(rng, lens, T, 2, 4, 128)
    want = attend(rd, cache, q, kt, vt, parent, 0.1)
    try:
        for worker in (0, 3, 11):
            rd.set_q4_give_up(worker)
            out, lse, st = attend(rd, cache, q, kt, vt, parent, 0.1)
            assert b.ERR_TIMEOUT in st and set(st) <= {0, b.ERR_TIMEOUT}
            zero = ~(out != 0).any(-1)
            assert zero.any() and torch.equal(out[~zero], want[0][~zero])
            assert all(st[s] == b.ERR_TIMEOUT for s in range(2) if zero[s].any())
    finally:
        rd.set_q4_give_up(-1)
    got = attend(rd, cache, q, kt, vt, parent, 0.1)
    assert got[2] == [0, 0] and torch.equal(got[0], want[0])


def test_pools_beyond_32_bit_offsets(rd):
    """Pages on either side of 2^31 and 2^32 bytes."""
    b = binding()
    rng = np.random.default_rng(22)
    heads, d = 8, 128
    per = heads * 36 * d
    n = (1 << 32) // per + 40
    k4, v4 = (torch.zeros(n, heads, 36 * d, dtype=torch.uint8, device="cuda") for _ in range(2))
    ids = [n - 1, (1 << 31) // per, (1 << 32) // per, 0, (1 << 32) // per + 1, 5]
    lens = [384]
    both = Both(rng, lens, heads, d)
    table = i32([ids])
    narrow = b.Q4Cache(k4, v4, table, i32(lens))
    assert rd.q4_store([both.wide], [narrow], i32([0]), i32(lens)).tolist() == [0]
    for T in (1, 40):
        q, kt, vt, parent = bf16(rng, 1, T, 16, d), bf16(rng, 1, T, heads, d), bf16(rng, 1, T, heads, d), random_parents(rng, 1, T)
        out, lse, st = attend(rd, narrow, q, kt, vt, parent, 0.1)
        within((out, lse), plain_attn(both, lens, q, kt, vt, parent, 0.1))


# ---------------------------------------------------------------------------------------------- together
def test_a_prompt_and_decoding_steps_on_a_4_bit_cache(rd):
    """Prompt into a bf16 cache, stored in 4 bits, then steps: pages reserved, attention, acceptance, commit."""
    b = binding()
    rng = np.random.default_rng(23)
    B, heads, group, d, T, max_path, n_pages = 3, 2, 2, 64, 8, 4, 40
    lens = [70, 5, 130]
    seq_lens = i32([0] * B)
    k4, v4 = (torch.zeros(n_pages, heads, 36 * d, dtype=torch.uint8, device="cuda") for _ in range(2))
    pages_ = b.Pages(torch.zeros(n_pages, dtype=torch.int32, device="cuda"), torch.full((B, 8), -1, dtype=torch.int32, device="cuda"), seq_lens, [k4, v4])
    cache = b.Q4Cache(k4, v4, pages_.page_table, seq_lens)
    t16, n16 = table_of(rng, [4] * B)
    wide = b.KvCache(*(torch.zeros(n16, heads, PAGE, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)), i32(t16), seq_lens)
    rows = i32(range(B))
    assert rd.pages_reserve(pages_, rows, i32(lens)).tolist() == [0] * B
    tokens = sum(lens)
    q, k, v = bf16(rng, tokens, heads * group, d).cuda(), bf16(rng, tokens, heads, d).cuda(), bf16(rng, tokens, heads, d).cuda()
    start = i32(np.concatenate([[0], np.cumsum(lens)]))
    assert set(rd.prompt_append(q, k, v, wide, start)[1].tolist()) == {0}
    assert set(rd.prompt_attn(q, wide, start, 0.1)[1].tolist()) == {0}
    assert set(rd.q4_store([wide], [cache], i32([0] * B), i32(lens)).tolist()) == {0}
    seq_lens.copy_(i32(lens))
    ks, vs = ([held(x[sum(lens[:s]):sum(lens[:s + 1])].cpu()) for s in range(B)] for x in (k, v))
    for step in range(12):
        assert rd.pages_reserve(pages_, rows, i32([max_path] * B)).tolist() == [0] * B
        qt, kt, vt, parent = bf16(rng, B, T, heads * group, d), bf16(rng, B, T, heads, d), bf16(rng, B, T, heads, d), random_parents(rng, B, T)
        out, st = rd.q4_verify_attn(qt.cuda(), kt.cuda(), vt.cuda(), cache, i32(parent), 0.1)
        assert st.tolist() == [0] * B
        for s in range(B):
            kk, vv = torch.cat([ks[s], kt[s].double()]), torch.cat([vs[s], vt[s].double()])
            mask = torch.ones(T, len(kk), dtype=torch.bool)
            mask[:, len(ks[s]):] = torch.from_numpy(sees_of(parent[s]))
            for h in range(heads):
                x = torch.einsum("tgd,kd->tgk", qt[s, :, h * group:(h + 1) * group].double(), kk[:, h]) * 0.1
                p = x.masked_fill(~mask[:, None], -torch.inf).softmax(-1)
                want, mag = torch.einsum("tgk,kd->tgd", p, vv[:, h]), torch.einsum("tgk,kd->tgd", p, vv[:, h].abs())
                err = (out[s, :, h * group:(h + 1) * group].cpu().double() - want).abs()
                assert (err <= 2.0 ** -8 * (mag + want.abs()) * 1.01 + mag * 1e-4).all()
        tok = rng.integers(0, 3, (B, T))
        acc = rd.accept(i32(parent), i32(tok), max_path, target_ids=i32(rng.integers(0, 3, (B, T))))
        path, n_acc = acc["path"].cpu().numpy(), acc["n_acc"].tolist()
        assert rd.q4_commit([cache], [kt.cuda()], [vt.cuda()], acc["path"], acc["n_acc"])[1].tolist() == [0] * B
        for s in range(B):
            ks[s] = torch.cat([ks[s], held(kt[s, path[s, :n_acc[s]]])])
            vs[s] = torch.cat([vs[s], held(vt[s, path[s, :n_acc[s]]])])
        assert seq_lens.tolist() == [len(x) for x in ks]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,group", [(5, 1), (40, 4), (100, 3)])
def test_infinite_values_of_nodes_reach_the_rows_that_see_them_alone(rd, d, T, group):
    rng = np.random.default_rng(24)
    lens = [70, 0]
    both, cache, q, kt, vt, parent = make(rng, lens, T, 2, group, d)
    want = plain_attn(both, lens, q, kt, vt, parent, 0.1)
    sees = np.stack([sees_of(x) for x in parent])
    for value in (float("inf"), float("-inf"), float("nan")):
        for key, what in ((False, vt), (True, kt)):
            x = what.clone()
            node = T // 2
            x[0, node, 1, 3] = value
            x[1, T - 1, 0, d - 1] = value
            out, lse, st = attend(rd, cache, q, x if key else kt, vt if key else x, parent, 0.1)
            assert st == [0, 0]
            hit = torch.zeros(out.shape, dtype=torch.bool)
            for b, h, n, e in ((0, 1, node, 3), (1, 0, T - 1, d - 1)):
                rows = torch.from_numpy(np.nonzero(sees[b][:, n])[0])
                hit[b, rows, h * group:(h + 1) * group] |= True if key else (torch.arange(d) == e)
            if key:   # (a score of -inf is a key that is not seen: only NaN is NaN throughout)
                if np.isnan(value):
                    assert torch.isnan(out[hit]).all()
            else:
                assert (torch.isnan(out[hit]) if np.isnan(value) else out[hit] == value).all()
            assert ((out.double() - want[0]).abs() <= want[2])[~hit].all()


# ---------------------------------------------------------------------------------------------- forms of the calls
@pytest.mark.parametrize("store", [True, False])
@pytest.mark.parametrize("d", [64, 128])
def test_bf16_pools_on_any_16_byte_border(rd, store, d):
    """Blocks of 32 bytes are moved whole only where they lie on such a border."""
    b = binding()
    rng = np.random.default_rng(41)
    lens = [0, 77, 130]
    both = Both(rng, [max(x, 1) for x in lens], 2, d)
    first, last = i32([0, 5, 0]), i32(lens)

    def shifted(t):
        room = torch.empty(t.numel() + 8, dtype=t.dtype, device="cuda")
        out = room[8:].view(t.shape)
        assert out.data_ptr() % 32 == 16
        return out.copy_(t)

    if store:
        rd.q4_store([both.wide], [both.narrow], first, last)
        want = both.k4.clone(), both.v4.clone()
        moved = b.KvCache(shifted(both.k), shifted(both.v), both.wide.page_table, both.wide.seq_lens)
        for pool in (both.k4, both.v4):
            pool.random_(0, 256)
        assert rd.q4_store([moved], [both.narrow], first, last).tolist() == [0] * 3
        rd.q4_load([both.narrow], [both.out], first, last)
        again = both.out.k_pool.clone(), both.out.v_pool.clone()
        both.k4.copy_(want[0])
        both.v4.copy_(want[1])
        rd.q4_load([both.narrow], [both.out], first, last)
        assert torch.equal(again[0], both.out.k_pool) and torch.equal(again[1], both.out.v_pool)
    else:
        rd.q4_store([both.wide], [both.narrow], first, last)
        rd.q4_load([both.narrow], [both.out], first, last)
        moved = b.KvCache(shifted(torch.full_like(both.k, 3.0)), shifted(torch.full_like(both.v, 3.0)), both.wide.page_table, both.wide.seq_lens)
        assert rd.q4_load([both.narrow], [moved], first, last).tolist() == [0] * 3
        assert torch.equal(moved.k_pool, both.out.k_pool) and torch.equal(moved.v_pool, both.out.v_pool)


def widened(cache, columns):
    """The same cache with more columns in its page table (a call's form goes by their number)."""
    b = binding()
    t = torch.full((cache.page_table.shape[0], columns), -1, dtype=torch.int32, device="cuda")
    t[:, :cache.page_table.shape[1]] = cache.page_table
    return b.Q4Cache(cache.k_pool, cache.v_pool, t, cache.seq_lens)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,group,T", [
    (1, 1, 1), (2, 4, 2), (1, 1, 17), (1, 2, 64), (1, 1, 128), (2, 3, 43), (1, 8, 17), (1, 2, 100), (1, 2, 128), (1, 3, 100), (1, 4, 97), (1, 3, 128), (1, 5, 128), (3, 5, 26)])
@pytest.mark.parametrize("lens", [[517, 0, 1], [64, 127, 128, 129], [3000]])
def test_attention_with_wide_page_tables(rd, d, heads, group, T, lens):
    """Lists of work whatever the call's size: units of up to 128 rows, of more, both (257 to 384 rows of a head), ends inside a tile."""
    rng = np.random.default_rng(d + heads + 10 * group + T + sum(lens))
    both, cache, q, kt, vt, parent = make(rng, lens, T, heads, group, d)
    want = plain_attn(both, lens, q, kt, vt, parent, 0.09)
    got = attend(rd, widened(cache, 700), q, kt, vt, parent, 0.09)
    assert got[2] == [0] * len(lens)
    within(got[:2], want)


@pytest.mark.parametrize("d,heads,group,T,L", [(128, 1, 2, 128, 20000), (128, 1, 4, 32, 30000), (64, 1, 4, 4, 40000), (128, 1, 1, 1, 50000), (64, 2, 3, 100, 9000)])
def test_units_that_many_ranges_share(rd, d, heads, group, T, L):
    rng = np.random.default_rng(L)
    both, cache, q, kt, vt, parent = make(rng, [L], T, heads, group, d)
    got = attend(rd, cache, q, kt, vt, parent, 0.09)
    assert got[2] == [0]
    within(got[:2], plain_attn(both, [L], q, kt, vt, parent, 0.09))


@pytest.mark.parametrize("T,group", [(1, 4), (4, 4), (40, 3), (100, 4)])
def test_many_calls_in_a_row_do_not_give_up(rd, T, group):
    """Calls overlap at their ends (the next one is set up while one is under way); all of them answer the same."""
    rng = np.random.default_rng(43)
    lens = rng.integers(0, 1500, 24).tolist()
    both, cache, q, kt, vt, parent = make(rng, lens, T, 2, group, 128)
    want = attend(rd, cache, q, kt, vt, parent, 0.1)
    assert want[2] == [0] * 24
    q, kt, vt, parent = q.cuda(), kt.cuda(), vt.cuda(), i32(parent)
    outs = [torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    status = torch.full((300, 24), 9, dtype=torch.int32, device="cuda")
    for i in range(300):
        rd.q4_verify_attn(q, kt, vt, cache, parent, 0.1, out=outs[i % 4], status=status[i])
    assert not status.any()
    assert all(torch.equal(x.cpu(), want[0]) for x in outs)


@pytest.mark.parametrize("T", [1, 40, 100])
def test_statuses_with_wide_page_tables(rd, T):
    """Lengths that cannot be, pages that are not there and parents that are no tree, each in a sequence of its own among good ones."""
    b = binding()
    rng = np.random.default_rng(45)
    lens = [300, 200, 500, 64, 0]
    both, cache, q, kt, vt, parent = make(rng, lens, T, 2, 3, 64)
    wide = widened(cache, 900)
    want = plain_attn(both, lens, q, kt, vt, parent, 0.1)
    wide.seq_lens = i32([300, -1, 500, 900 * PAGE + 1, 0])
    wide.page_table[2, 3] = both.k4.shape[0]
    parent = parent.copy()
    parent[4][0] = 0
    out, lse, st = attend(rd, wide, q, kt, vt, parent, 0.1)
    assert st == [0, b.ERR_CAPACITY, b.ERR_BAD_PAGE, b.ERR_CAPACITY, b.ERR_BAD_TREE]
    within((out[:1], lse[:1]), [x[:1] for x in want])   # (where the list is cut goes by all lengths: not the bits of another batch)
    assert not out[1:].any() and not lse[1:].any()


@pytest.mark.parametrize("heads,d", [(1, 64), (8, 64), (3, 128), (8, 128)])
@pytest.mark.parametrize("columns", [4, 900])
def test_ranges_of_few_positions(rd, heads, d, columns):
    """One to seventeen positions (up to sixteen take another form behind a wide page table), at both ends of pages and over them; several layers at once."""
    b = binding()
    rng = np.random.default_rng(47)
    ranges = [(a, a + n) for n in (1, 2, 3, 8, 15, 16, 17) for a in (0, 1, 47, 48, 49, 62, 63, 64, 120)]
    both = [Both(rng, [x for _, x in ranges], heads, d) for _ in range(3)]
    for x in both[1:]:   # (the layers of a call have their tables in common)
        x.t16, x.t4 = both[0].t16, both[0].t4
    tables = [torch.full((len(ranges), columns), -1, dtype=torch.int32, device="cuda") for _ in range(2)]
    for t, now in zip(tables, (both[0].wide.page_table, both[0].narrow.page_table)):
        t[:, :now.shape[1]] = now
    for x in both:
        x.wide.page_table, x.narrow.page_table, x.out.page_table = tables[0], tables[1], tables[0]
    first, last = i32([a for a, _ in ranges]), i32([x for _, x in ranges])
    assert not rd.q4_store([x.wide for x in both], [x.narrow for x in both], first, last).any()
    assert not rd.q4_load([x.narrow for x in both], [x.out for x in both], first, last).any()
    for x in both:
        for src, out in ((x.k, x.out.k_pool), (x.v, x.out.v_pool)):
            want = torch.full(src.shape, 3.0, dtype=torch.float64)
            for s, (lo, hi) in enumerate(ranges):
                pos = np.arange(lo, hi)
                page = torch.from_numpy(x.t16[s][pos // PAGE].astype(np.int64))
                want[page, :, torch.from_numpy(pos % PAGE)] = held(rows_of(src, x.t16, s, lo, hi))
            assert torch.equal(out.cpu().double(), want)
    assert b.ERR_CAPACITY in rd.q4_store([both[0].wide], [both[0].narrow], first - 1, last).tolist()


@pytest.mark.parametrize("B,T,group", [(65536, 1, 1), (65536, 1, 12), (9000, 20, 2)])
def test_the_largest_batches(rd, B, T, group):
    """As many sequences as a call may have, with empty ones and ones of a few pages; one page for all that are short."""
    b = binding()
    rng = np.random.default_rng(B + T)
    lens = np.where(rng.random(B) < 0.2, 0, rng.integers(1, PAGE, B))
    long_ones = [3, 64, B // 2, B - 2]
    lens[long_ones] = 200
    both = Both(rng, [200], 1, 64)
    assert not rd.q4_store([both.wide], [both.narrow], i32([0]), i32([200])).any()
    table = np.tile(both.t4[0][:4], (B, 1))
    cache = b.Q4Cache(both.k4, both.v4, i32(table), i32(lens))
    q, kt, vt = bf16(rng, B, T, group, 64), bf16(rng, B, T, 1, 64), bf16(rng, B, T, 1, 64)
    parent = random_parents(rng, B, T)
    got = attend(rd, cache, q, kt, vt, parent, 0.125)
    assert not any(got[2])
    some = long_ones + [0, 1, 31, 32, 255, 256, 257, B - 1] + rng.integers(0, B, 20).tolist()
    pick = lambda x: x[torch.tensor(some)]  # noqa: E731
    sub = Both.__new__(Both)
    sub.k, sub.v, sub.t16 = both.k, both.v, np.tile(both.t16[0][:4], (len(some), 1))
    within((pick(got[0]), pick(got[1])), plain_attn(sub, [int(lens[i]) for i in some], pick(q), pick(kt), pick(vt), parent[some], 0.125))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,group", [(77, 5), (100, 3), (32, 4)])
def test_the_same_bits_behind_other_work(rd, T, group, d):
    """Calls that begin with cold caches, whose first pages come late and in any order: one call in some hundreds once took values before they were there."""
    rng = np.random.default_rng(49)
    lens = rng.integers(379, 610, 31).tolist()
    both, cache, q, kt, vt, parent = make(rng, lens, T, 2, group, d)
    want = attend(rd, cache, q, kt, vt, parent, d ** -0.5)
    within(want[:2], plain_attn(both, lens, q, kt, vt, parent, d ** -0.5))
    q, kt, vt, parent, expect = q.cuda(), kt.cuda(), vt.cuda(), i32(parent), want[0].cuda()
    out, wide, differ = torch.empty_like(expect), expect.double(), 0
    for i in range(1500):
        rd.q4_verify_attn(q, kt, vt, cache, parent, d ** -0.5, out=out)
        off = (out.double() - wide).norm(dim=-1) / wide.norm(dim=-1)
        differ += len((off != 0).nonzero())
    assert differ == 0
