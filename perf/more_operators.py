"""The 4-bit cache and the page calls of the library as cases that can be run and timed.

Five operators: ``convert`` (rows of a bf16 paged cache to 4 bits and their values back), ``commit`` (accepted tree rows of
several layers into 4-bit caches, and their values back), ``attn`` (tree-masked attention over a 4-bit cache; one node is
plain decoding), ``branch`` (rows of a page table freed, forked from others and given pages to write to) and ``compact``
(pages in use moved to the front of the pools).  ``run`` computes them in elementary torch operations, or through the
library where ``own`` is true; ``exact`` computes what has numbers in 64 bits.

The 4-bit values: 16 consecutive elements of a head share the scale (1 + (c & 7) / 8) 2^((c >> 3) - 18) of a code c < 255, the
smallest with 7.5 scales >= the largest magnitude; an element is a whole number of scales from -7 to 7, held as that plus 8.
"""
import random

import torch

own = False

PAGE = 64
_DEV = "cuda:0"


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    small, big = dict(hkv=8, d=64), dict(hkv=8, d=128)
    return [
        # the next piece of two short prompts, from and to the middle of pages
        dict(name="convert_pieces", op="convert", batch=2, n_min=131, n_max=517, l_min=0, l_max=90, **small),
        # a batch of whole prompts after their attention
        dict(name="convert_prompts", op="convert", batch=16, n_min=100, n_max=4096, l_min=0, l_max=0, **big),
        # the accepted path of a single prompt's tree, one layer
        dict(name="commit_one", op="commit", batch=1, layers=1, nodes=16, max_path=6, l_min=512, l_max=512, **small),
        # the accepted paths of a batch in all layers of a model
        dict(name="commit_layers", op="commit", batch=16, layers=16, nodes=32, max_path=8, l_min=0, l_max=1024, **big),
        # plain decoding of one short context: latency
        dict(name="attn_one_token", op="attn", batch=1, nodes=1, l_min=511, l_max=511, hq=8, **small, lse=False),
        # plain decoding of a served batch
        dict(name="attn_single_tokens", op="attn", batch=32, nodes=1, l_min=1024, l_max=4096, hq=32, **big, lse=True),
        # draft trees of a served batch
        dict(name="attn_trees", op="attn", batch=32, nodes=32, l_min=1024, l_max=4096, hq=32, **big, lse=False),
        # the largest: large trees over long contexts
        dict(name="attn_long", op="attn", batch=4, nodes=128, l_min=32768, l_max=32768, hq=32, **big, lse=False),
        # four answers to one prompt, one layer of a bf16 cache
        dict(name="branch_one", op="branch", parents=1, children=4, tokens=8, l_min=700, l_max=700, pools=2, page_bytes=65536, spare=64),
        # four answers each to a batch of prompts, eight layers of a 4-bit cache
        dict(name="branch_batch", op="branch", parents=32, children=4, tokens=64, l_min=256, l_max=1024, pools=16, page_bytes=36864,
             spare=200),
        # a small pool, one layer of a bf16 cache
        dict(name="compact_small", op="compact", pages=256, rows=24, width=16, held=0.5, pools=2, page_bytes=65536),
        # a pool after hours of serving, four layers of a 4-bit cache
        dict(name="compact_served", op="compact", pages=4096, rows=160, width=32, held=0.6, pools=8, page_bytes=36864),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(lo * (hi / lo) ** rng.random())))


def draw(rng):
    ops = ("convert", "commit", "attn", "branch", "compact")
    limit = {op: max(_cost(c) for c in listed() if c["op"] == op) for op in ops}
    while True:
        op = rng.choice(ops + ("attn",))
        c = dict(op=op)
        if op in ("convert", "commit", "attn"):
            c.update(batch=_log_int(rng, 1, 64), hkv=rng.choice([1, 2, 4, 8]), d=rng.choice([64, 128, 128]))
        if op == "convert":
            c["n_max"] = _log_int(rng, 1, 8192)
            c["n_min"] = rng.randint(0, c["n_max"])
            c["l_max"] = rng.choice([0, _log_int(rng, 1, 4096)])
            c["l_min"] = rng.randint(0, c["l_max"])
        elif op == "commit":
            c.update(layers=_log_int(rng, 1, 32), nodes=_log_int(rng, 1, 128))
            c["max_path"] = rng.randint(1, min(16, c["nodes"]))
            c["l_max"] = _log_int(rng, 1, 2048)
            c["l_min"] = rng.randint(0, c["l_max"])
        elif op == "attn":
            c["hq"] = c["hkv"] * rng.choice([1, 2, 3, 4, 5, 7, 8])
            c["nodes"] = rng.choice([1, _log_int(rng, 1, 128)])
            c["l_max"] = _log_int(rng, 1, 32768)
            c["l_min"] = rng.randint(0, c["l_max"])
            c["lse"] = rng.random() < 0.5
        elif op == "branch":
            c.update(parents=_log_int(rng, 1, 64), children=_log_int(rng, 1, 8), tokens=_log_int(rng, 1, 300))
            c["l_max"] = _log_int(rng, 1, 4096)
            c["l_min"] = rng.randint(0, c["l_max"])
            c.update(pools=2 * _log_int(rng, 1, 28), page_bytes=rng.choice([2304, 4608, 16384, 36864, 65536, 131072]),
                     spare=_log_int(rng, 1, 1000))
        else:
            c.update(pages=_log_int(rng, 16, 8192), width=_log_int(rng, 4, 128), held=round(rng.uniform(0.1, 0.95), 2))
            c["rows"] = max(1, int(c["pages"] * c["held"] * 1.2 / c["width"]))
            c.update(pools=2 * _log_int(rng, 1, 28), page_bytes=rng.choice([2304, 4608, 16384, 36864, 65536, 131072]))
        if 0 < _cost(c) <= limit[op] and _room(c) <= 4 << 30:
            return c


def _lengths(c):
    """New tokens and committed lengths per sequence: a property of the case, not of the seed."""
    count = c["parents"] if c["op"] == "branch" else c["batch"]
    rng = random.Random("%s %s %s" % (count, c.get("n_max"), c["l_max"]))
    past = [rng.randint(c["l_min"], c["l_max"]) for _ in range(count)]
    if c["op"] == "convert":
        n = [rng.randint(c["n_min"], c["n_max"]) for _ in range(count)]
        n[0] = max(1, n[0])
    elif c["op"] == "commit":
        n = [rng.randint(1, c["max_path"]) for _ in range(count)]
    else:
        n = [0] * count
    return n, past


def _pages(tokens):
    return (tokens + PAGE - 1) // PAGE


def _branch_pages(c):
    """Pages the parents hold, pages the children get, pages copied among those."""
    _, past = _lengths(c)
    held = sum(_pages(x) for x in past)
    fresh = sum(_pages(x + c["tokens"]) - x // PAGE for x in past) * c["children"]
    return held, fresh, sum(1 for x in past if x % PAGE) * c["children"]


def _moved(c):
    """Pages in use and those of them that stand behind as many places: a property of the case."""
    rng = random.Random("%s %s" % (c["pages"], c["held"]))
    used = sorted(rng.sample(range(c["pages"]), min(c["pages"], max(1, int(c["pages"] * c["held"])), c["rows"] * c["width"])))
    return used, sum(1 for p in used if p >= len(used))


def _room(c):
    """Bytes of the pools a case needs."""
    if c["op"] == "branch":
        held, fresh, _ = _branch_pages(c)
        return (held + fresh + c["spare"]) * c["pools"] * c["page_bytes"]
    if c["op"] == "compact":
        return c["pages"] * c["pools"] * c["page_bytes"]
    n, past = _lengths(c)
    rows = sum(_pages(a + b) + 2 for a, b in zip(n, past)) * PAGE * c["hkv"] * c["d"]
    if c["op"] == "commit":
        return rows * 2 * c["layers"] + 2 * c["batch"] * PAGE * c["hkv"] * c["d"] * 4 * c["layers"]
    return rows * (10 if c["op"] == "convert" else 2)


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 6e12, w["flops"] / 1.5e15)


def _row_bytes(c):
    """K and V of one position: in bf16, in 4 bits."""
    return 4 * c["hkv"] * c["d"], 2 * c["hkv"] * c["d"] * 9 // 16


def work(c):
    if c["op"] == "branch":
        held, fresh, copied = _branch_pages(c)
        # what a table entry costs: read in the parent's row, written and read in the child's, a count on either side
        return {"bytes": 2 * copied * c["pools"] * c["page_bytes"] + 4 * (5 * held * c["children"] + 3 * fresh), "flops": 0}
    if c["op"] == "compact":
        _, moved = _moved(c)
        return {"bytes": 2 * moved * c["pools"] * c["page_bytes"] + 8 * c["pages"] + 4 * c["rows"] * c["width"], "flops": 0}
    n, past = _lengths(c)
    wide, narrow = _row_bytes(c)
    if c["op"] == "convert":   # read, written in 4 bits; read in 4 bits, written
        return {"bytes": 2 * sum(n) * (wide + narrow), "flops": 0}
    if c["op"] == "commit":
        return {"bytes": 2 * c["layers"] * sum(n) * (wide + narrow), "flops": 0}
    rows, tree = c["batch"] * c["nodes"], c["batch"] * c["nodes"] * wide
    pairs = sum(c["nodes"] * x for x in past) + rows * (c["nodes"] + 1) // 2
    return {"bytes": 4 * rows * c["hq"] * c["d"] + tree + sum(past) * narrow + (4 * rows * c["hq"] if c["lse"] else 0),
            "flops": 4 * c["d"] * c["hq"] * pairs}


# ------------------------------------------------------------------------------------------------ the 4-bit values
def _scales():
    """The scales of the codes 0 .. 254."""
    c = torch.arange(255, device=_DEV)
    return (1 + (c & 7).float() / 8) * torch.exp2((c >> 3).float() - 18)


def _quantise(x):
    """Whole numbers [..., d] (int32) and scale codes [..., d / 16] (int32) of x [..., d]; finite values."""
    scales = _scales()
    blocks = x.float().unflatten(-1, (-1, 16))
    code = torch.searchsorted(7.5 * scales, blocks.abs().amax(-1).contiguous()).clamp(max=254)
    number = torch.round(blocks / scales[code][..., None]).clamp(-7, 7)
    return number.flatten(-2).to(torch.int32), code.to(torch.int32)


def _held(x):
    """What x [..., d] is after a stay in 4 bits."""
    number, code = _quantise(x)
    return (number.unflatten(-1, (-1, 16)) * _scales()[code.long()][..., None]).flatten(-2)


def _k_scale_places(d, g, j, u):
    """Bytes of the scales of position 8 j + g and block u in a K tile."""
    return ((g * 4 + u // (d // 64)) * 8 + j) * (d // 64) + u % (d // 64)


def _v_chunk(d, t, q):
    """Place among its row's eight chunks of chunk q of the position pair t in a V tile."""
    return q ^ (2 * (t & 3) if d == 128 else 4 * ((t >> 1) & 1))


def _words(nibbles):
    """Eight nibbles [..., 8] to a 32-bit word, rotated left by three bits."""
    w = sum(nibbles[..., i].long() << (4 * i) for i in range(8))
    w = ((w << 3) | (w >> 29)) & 0xffffffff
    return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)


def _nibbles(words):
    w = words.long() & 0xffffffff
    w = (w >> 3) | (w << 29)
    return torch.stack([(w >> (4 * i)) & 15 for i in range(8)], -1)


def _pack(x, kind):
    """Tiles x [tiles, 64, d] as bytes [tiles, 36 d]."""
    tiles, _, d = x.shape
    number, code = _quantise(x)
    n = number + 8
    if kind == "k":     # a word: elements 8 w .. 8 w + 7 of a position, the even ones below the odd ones
        words = _words(n.view(tiles, PAGE, d // 8, 4, 2).transpose(-1, -2).reshape(tiles, PAGE, d // 8, 8))
        places = _k_scale_places(d, torch.arange(PAGE, device=_DEV)[:, None] & 7, torch.arange(PAGE, device=_DEV)[:, None] >> 3,
                                 torch.arange(d // 16, device=_DEV))
    else:               # a word: elements 4 w .. 4 w + 3 of a position pair, the even position below the odd one
        words = _words(n.view(tiles, PAGE // 2, 2, d // 4, 4).transpose(2, 3).reshape(tiles, PAGE // 2, d // 4, 8))
        t, q = torch.arange(PAGE // 2, device=_DEV)[:, None], torch.arange(8, device=_DEV)
        chunks = words.view(tiles, PAGE // 2, 8, d // 32)
        words = torch.empty_like(chunks)
        words[:, t, _v_chunk(d, t, q)] = chunks
        r = torch.arange(PAGE, device=_DEV)[:, None]
        places = ((torch.arange(d // 16, device=_DEV) * 4 + ((r >> 1) & 3)) * 8 + (r >> 3)) * 2 + (r & 1)
    scale = torch.empty(tiles, 4 * d, dtype=torch.uint8, device=_DEV)
    scale[:, places.flatten()] = code.view(tiles, -1).to(torch.uint8)
    return torch.cat([words.reshape(tiles, -1).view(torch.uint8), scale], 1)


def _unpack(tiles, d, kind):
    """Values [tiles, 64, d] (32 bits) of tiles [tiles, 36 d]."""
    count = tiles.shape[0]
    words = tiles[:, :32 * d].contiguous().view(torch.int32)
    if kind == "k":
        n = _nibbles(words.view(count, PAGE, d // 8)).view(count, PAGE, d // 8, 2, 4).transpose(-1, -2).reshape(count, PAGE, d)
        places = _k_scale_places(d, torch.arange(PAGE, device=_DEV)[:, None] & 7, torch.arange(PAGE, device=_DEV)[:, None] >> 3,
                                 torch.arange(d // 16, device=_DEV))
    else:
        t, q = torch.arange(PAGE // 2, device=_DEV)[:, None], torch.arange(8, device=_DEV)
        chunks = words.view(count, PAGE // 2, 8, d // 32)[:, t, _v_chunk(d, t, q)]
        n = _nibbles(chunks.reshape(count, PAGE // 2, d // 4)).view(count, PAGE // 2, d // 4, 2, 4).transpose(2, 3).reshape(count, PAGE, d)
        r = torch.arange(PAGE, device=_DEV)[:, None]
        places = ((torch.arange(d // 16, device=_DEV) * 4 + ((r >> 1) & 3)) * 8 + (r >> 3)) * 2 + (r & 1)
    scale = _scales()[tiles[:, 32 * d:][:, places].long()]
    return ((n - 8).unflatten(-1, (-1, 16)) * scale[..., None]).flatten(-2)


# ------------------------------------------------------------------------------------------------ inputs
def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=_DEV, dtype=torch.float32).to(torch.bfloat16)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=_DEV)


def _table(g, ranges, spare=1):
    """A page table whose rows have pages for the positions of their (first, last); the pool's pages in random order."""
    counts = [(a // PAGE, _pages(b)) for a, b in ranges]
    total = sum(b - a for a, b in counts) + spare
    order = torch.randperm(total, generator=g, device=_DEV).to(torch.int32)
    table = torch.full((len(ranges), max(max(b for _, b in counts), 1)), -1, dtype=torch.int32, device=_DEV)
    at = 0
    for row, (a, b) in enumerate(counts):
        table[row, a:b] = order[at:at + b - a]
        at += b - a
    return table, total


def _trees(g, batch, nodes):
    """Parent arrays: every node hangs under a random earlier one, the last few at most."""
    back = torch.randint(1, 9, (batch, nodes), generator=g, device=_DEV)
    parent = (torch.arange(nodes, device=_DEV) - back).clamp(min=0)
    parent[:, 0] = -1
    return parent.to(torch.int32)


def _packed_pool(g, pages, hkv, d, kind):
    pool = torch.empty(pages, hkv, 36 * d, dtype=torch.uint8, device=_DEV)
    step = max(1, (64 << 20) // (hkv * PAGE * d))
    for lo in range(0, pages, step):
        hi = min(pages, lo + step)
        pool[lo:hi] = _pack(_normal(g, (hi - lo) * hkv, PAGE, d), kind).view(hi - lo, hkv, 36 * d)
    return pool


def prepare(c, seed):
    g = torch.Generator(device=_DEV)
    g.manual_seed(seed)
    return dict({"convert": _prepare_convert, "commit": _prepare_commit, "attn": _prepare_attn, "branch": _prepare_branch,
                 "compact": _prepare_compact}[c["op"]](c, g), case=c)


def _prepare_convert(c, g):
    n, past = _lengths(c)
    hkv, d = c["hkv"], c["d"]
    ranges = [(b, a + b) for a, b in zip(n, past)]
    s = dict(first=_ints(past), last=_ints([b for _, b in ranges]))
    s["table"], total = _table(g, ranges)
    s["k_pool"], s["v_pool"] = _normal(g, total, hkv, PAGE, d), _normal(g, total, hkv, PAGE, d)
    s["q4_table"], total = _table(g, ranges)
    s["k4"], s["v4"] = (torch.zeros(total, hkv, 36 * d, dtype=torch.uint8, device=_DEV) for _ in range(2))
    s["out_table"], total = _table(g, ranges)
    s["k_out"], s["v_out"] = (torch.zeros(total, hkv, PAGE, d, dtype=torch.bfloat16, device=_DEV) for _ in range(2))
    return s


def _prepare_commit(c, g):
    n, past = _lengths(c)
    hkv, d = c["hkv"], c["d"]
    s = dict(first=_ints(past), last=_ints([a + b for a, b in zip(n, past)]), n_acc=_ints(n))
    # any increasing chain of nodes from the root
    rank = torch.rand(c["batch"], c["nodes"], generator=g, device=_DEV)
    rank[:, 0] = -1
    chain = rank.argsort(1)[:, :c["max_path"]].sort(1).values.to(torch.int32)
    s["path"] = torch.where(torch.arange(c["max_path"], device=_DEV) < s["n_acc"][:, None], chain, -1).contiguous()
    s["q4_table"], total = _table(g, [(0, b + c["max_path"]) for b in past])
    s["k4"], s["v4"] = ([torch.zeros(total, hkv, 36 * d, dtype=torch.uint8, device=_DEV) for _ in range(c["layers"])] for _ in range(2))
    s["k_tree"], s["v_tree"] = ([_normal(g, c["batch"], c["nodes"], hkv, d) for _ in range(c["layers"])] for _ in range(2))
    s["out_table"], total = _table(g, [(b, a + b) for a, b in zip(n, past)])
    s["k_out"], s["v_out"] = ([torch.zeros(total, hkv, PAGE, d, dtype=torch.bfloat16, device=_DEV) for _ in range(c["layers"])] for _ in range(2))
    return s


def _prepare_attn(c, g):
    _, past = _lengths(c)
    hkv, d, hq, rows = c["hkv"], c["d"], c["hq"], (c["batch"], c["nodes"])
    s = dict(past=past, seq_lens=_ints(past), scale=d ** -0.5)
    s["q4_table"], total = _table(g, [(0, x) for x in past])
    s["k4"], s["v4"] = _packed_pool(g, total, hkv, d, "k"), _packed_pool(g, total, hkv, d, "v")
    s["parent"] = _trees(g, *rows)
    s["q"], s["k_tree"], s["v_tree"] = _normal(g, *rows, hq, d), _normal(g, *rows, hkv, d), _normal(g, *rows, hkv, d)
    s["out"] = torch.empty(*rows, hq, d, dtype=torch.bfloat16, device=_DEV)
    s["lse"] = torch.empty(*rows, hq, dtype=torch.float32, device=_DEV) if c["lse"] else None
    return s


def _bytes_pools(g, count, pages, page_bytes):
    return [torch.randint(0, 256, (pages, page_bytes), generator=g, device=_DEV, dtype=torch.uint8) for _ in range(count)]


def _prepare_branch(c, g):
    _, past = _lengths(c)
    held, fresh, _ = _branch_pages(c)
    rows, pages = c["parents"] * (1 + c["children"]), held + fresh + c["spare"]
    width = max(_pages(x + c["tokens"]) for x in past) + 1
    parents, total = _table(g, [(0, x) for x in past], fresh + c["spare"])
    assert total == pages
    table = torch.full((rows, width), -1, dtype=torch.int32, device=_DEV)
    table[:c["parents"], :parents.shape[1]] = parents
    refs = torch.zeros(pages, dtype=torch.int32, device=_DEV)
    refs[parents[parents >= 0].long()] = 1
    # the children's rows stand behind the parents', those of one parent together
    src = torch.arange(c["parents"], device=_DEV, dtype=torch.int32).repeat_interleave(c["children"])
    dst = torch.arange(c["parents"], rows, device=_DEV, dtype=torch.int32)
    return dict(table=table, refs=refs, seq_lens=_ints(past + [0] * (rows - c["parents"])), src=src, dst=dst,
                tokens=torch.full_like(dst, c["tokens"]), pools=_bytes_pools(g, c["pools"], pages, c["page_bytes"]))


def _prepare_compact(c, g):
    used, _ = _moved(c)
    ids = _ints(used)[torch.randperm(len(used), generator=g, device=_DEV)]
    places = torch.randperm(c["rows"] * c["width"], generator=g, device=_DEV)
    flat = torch.full((c["rows"] * c["width"],), -1, dtype=torch.int32, device=_DEV)
    flat[places[:len(used)]] = ids
    # some places that are left name a page of another row: a shared prefix
    shared = places[len(used):len(used) + len(used) // 8]
    flat[shared] = ids[:shared.numel()]
    refs = torch.bincount(flat[flat >= 0].long(), minlength=c["pages"]).to(torch.int32)
    table = flat.view(c["rows"], c["width"])
    return dict(table=table.clone(), refs=refs.clone(), found_table=table, found_refs=refs, n_used=torch.zeros(1, dtype=torch.int32, device=_DEV),
                seq_lens=torch.zeros(c["rows"], dtype=torch.int32, device=_DEV),
                pools=_bytes_pools(g, c["pools"], c["pages"], c["page_bytes"]))


# ------------------------------------------------------------------------------------------------ plain forms
def _positions(first, last, total):
    """Sequence and position of each of the `total` rows in the ranges first .. last - 1."""
    count = (last - first).long()
    seq = torch.repeat_interleave(torch.arange(count.numel(), device=_DEV), count, output_size=total)
    return seq, first.long()[seq] + torch.arange(total, device=_DEV) - (count.cumsum(0) - count)[seq]


def _plain_convert(s):
    seq, pos = _positions(s["first"], s["last"], sum(_lengths(s["case"])[0]))
    page, to = s["table"].long()[seq, pos // PAGE], s["out_table"].long()[seq, pos // PAGE]
    for src, dst in (("k_pool", "k_out"), ("v_pool", "v_out")):
        s[dst][to, :, pos % PAGE] = _held(s[src][page, :, pos % PAGE]).to(torch.bfloat16)
    return {"k": s["k_out"], "v": s["v_out"]}


def _plain_commit(s):
    seq, pos = _positions(s["first"], s["last"], sum(_lengths(s["case"])[0]))
    node, to = s["path"].long()[seq, pos - s["first"].long()[seq]], s["out_table"].long()[seq, pos // PAGE]
    for src, dst in (("k_tree", "k_out"), ("v_tree", "v_out")):
        for tree, pool in zip(s[src], s[dst]):
            pool[to, :, pos % PAGE] = _held(tree[seq, node]).to(torch.bfloat16)
    return {"k": s["k_out"], "v": s["v_out"]}


def _ancestors(parent):
    """Which nodes [b, query, key] a node sees: itself and those above it."""
    nodes = parent.shape[1]
    up = parent.long()
    seen = torch.eye(nodes, dtype=torch.bool, device=_DEV).expand(parent.shape[0], nodes, nodes).clone()
    hop = torch.cat([torch.where(up < 0, nodes, up), torch.full_like(up[:, :1], nodes)], 1)   # `nodes`: above the root
    seen = torch.nn.functional.pad(seen, (0, 1, 0, 1))
    # by doubling: what a node sees within 2^i steps, and where 2^i steps lead
    for _ in range(7):
        seen = seen | seen.gather(1, hop[..., None].expand_as(seen))
        hop = hop.gather(1, hop)
    return seen[:, :nodes, :nodes]


def _plain_attn_of(s, lo, hi):
    """Sequences lo .. hi - 1, padded to their longest; writes their rows of the outputs."""
    c = s["case"]
    d, hkv, nodes, group = c["d"], c["hkv"], c["nodes"], c["hq"] // c["hkv"]
    k_max = max(s["past"][lo:hi])
    page = s["q4_table"][lo:hi, :_pages(k_max)].long().clamp(min=0)
    values = []
    for pool, tree, kind in ((s["k4"], s["k_tree"], "k"), (s["v4"], s["v_tree"], "v")):
        tiles = _unpack(pool[page].view(-1, 36 * d), d, kind).view(hi - lo, -1, hkv, PAGE, d)
        committed = tiles.permute(0, 2, 1, 3, 4).reshape(hi - lo, hkv, -1, d)
        values.append(torch.cat([committed, tree[lo:hi].float().transpose(1, 2)], 2))
    k, v = values
    t = torch.arange(k.shape[2] - nodes, device=_DEV)
    seen = torch.cat([(t < s["seq_lens"][lo:hi, None])[:, None].expand(-1, nodes, -1), _ancestors(s["parent"][lo:hi])], 2)
    q = s["q"][lo:hi].float().view(hi - lo, nodes, hkv, group, d).permute(0, 2, 1, 3, 4).reshape(hi - lo, hkv, nodes * group, d)
    score = (q @ k.transpose(-1, -2)).mul_(s["scale"]).view(hi - lo, hkv, nodes, group, -1)
    score = score.masked_fill_(~seen[:, None, :, None], float("-inf"))
    top = score.amax(-1, keepdim=True)
    weight = score.sub_(top).exp_()
    total = weight.sum(-1, keepdim=True)
    out = (weight.view(hi - lo, hkv, nodes * group, -1) @ v).view(hi - lo, hkv, nodes, group, d) / total
    s["out"][lo:hi] = out.transpose(1, 2).reshape(hi - lo, nodes, hkv * group, d).to(torch.bfloat16)
    if s["lse"] is not None:
        s["lse"][lo:hi] = (top + total.log()).squeeze(-1).transpose(1, 2).reshape(hi - lo, nodes, hkv * group)


def _plain_attn(s):
    # as many sequences at a time as keep the padded scores and the unpacked keys within 1 Gi values
    c = s["case"]
    step = max(1, (1 << 30) // ((max(s["past"]) + PAGE + c["nodes"]) * max(c["hq"] * c["nodes"], 8 * c["hkv"] * c["d"])))
    for lo in range(0, c["batch"], step):
        _plain_attn_of(s, lo, min(lo + step, c["batch"]))
    return {"out": s["out"]} if s["lse"] is None else {"out": s["out"], "lse": s["lse"]}


def _count(refs, pages, by):
    """refs[page] += by for every page that is one."""
    refs.index_add_(0, pages.clamp(min=0).flatten().long(), torch.where(pages >= 0, by, 0).to(torch.int32).flatten())


def _plain_branch(s):
    table, refs, lens, src, dst = s["table"], s["refs"], s["seq_lens"], s["src"].long(), s["dst"].long()
    column = torch.arange(table.shape[1], device=_DEV)
    # the rows that are to be reused are freed
    _count(refs, table[dst], -1)
    table[dst] = -1
    # they become what others are
    table[dst] = torch.where(column < (lens[src] + PAGE - 1)[:, None] // PAGE, table[src], -1)
    _count(refs, table[dst], 1)
    lens[dst] = lens[src]
    # and get pages of their own for what they will write: the free ones with the lowest ids, in order
    length, now = lens[dst], table[dst]
    first = length // PAGE
    wanted = (column >= first[:, None]) & (column < ((length + s["tokens"] + PAGE - 1) // PAGE)[:, None])
    fresh = wanted & ((now < 0) | (refs[now.clamp(min=0).long()] > 1))
    free = (refs != 0).to(torch.uint8).argsort(stable=True).to(torch.int32)
    rank = fresh.flatten().long().cumsum(0).view(fresh.shape) - 1
    new = torch.where(fresh, free[rank.clamp(min=0)], now)
    # a page that is begun is copied (a row whose last page is full copies one of its new pages to itself)
    begun = (length % PAGE != 0) & fresh.gather(1, first[:, None].long())[:, 0]
    to = new.gather(1, first[:, None].long())[:, 0].long()
    of = torch.where(begun, now.gather(1, first[:, None].long())[:, 0].long(), to)
    _count(refs, torch.where(fresh, now, -1), -1)
    _count(refs, torch.where(fresh, new, -1), 1)
    table[dst] = new
    for pool in s["pools"]:
        pool[to] = pool[of]
    return {"table": table, "refs": refs, "seq_lens": lens, "pools": s["pools"]}


def _as_found(s):
    """The fragmented pool as a program finds it (the data behind the front are still in place)."""
    s["table"].copy_(s["found_table"])
    s["refs"].copy_(s["found_refs"])


def _plain_compact(s):
    _as_found(s)
    table, refs, count = s["table"], s["refs"], _moved(s["case"])[1]
    page = torch.arange(refs.numel(), device=_DEV)
    held = refs > 0
    used = held.sum()
    # the k-th page behind the front goes to the k-th free one in it
    movers = (held & (page >= used)).to(torch.uint8).argsort(stable=True, descending=True)[:count]
    holes = (~held & (page < used)).to(torch.uint8).argsort(stable=True, descending=True)[:count]
    for pool in s["pools"]:
        pool[holes] = pool[movers]
    name = page.to(torch.int32)
    name[movers] = holes.to(torch.int32)
    refs[holes] = refs[movers]
    refs[movers] = 0
    table.copy_(torch.where(table >= 0, name[table.clamp(min=0).long()], table))
    s["n_used"].copy_(used[None])
    return {"table": table, "refs": refs, "n_used": s["n_used"], "pools": s["pools"]}


# ------------------------------------------------------------------------------------------------ the library
_reader = None


def _library(s):
    """The handle and the objects that a program keeps."""
    global _reader
    from paper_2508_09072_b200 import binding
    if _reader is None:
        _reader = binding.Reader(0)
    if "objects" in s:
        return _reader
    s["objects"] = True
    op, lens = s["case"]["op"], s.get("seq_lens", s.get("first"))
    if op == "convert":
        s["from"] = [binding.KvCache(s["k_pool"], s["v_pool"], s["table"], lens)]
        s["caches"] = [binding.Q4Cache(s["k4"], s["v4"], s["q4_table"], lens)]
        s["to"] = [binding.KvCache(s["k_out"], s["v_out"], s["out_table"], lens)]
    elif op == "commit":
        s["caches"] = [binding.Q4Cache(k, v, s["q4_table"], lens) for k, v in zip(s["k4"], s["v4"])]
        s["to"] = [binding.KvCache(k, v, s["out_table"], lens) for k, v in zip(s["k_out"], s["v_out"])]
    elif op == "attn":
        s["cache"] = binding.Q4Cache(s["k4"], s["v4"], s["q4_table"], lens)
    else:
        s["pages"] = binding.Pages(s["refs"], s["table"], lens, s["pools"])
    return _reader


def _own_convert(s):
    rd = _library(s)
    rd.q4_store(s["from"], s["caches"], s["first"], s["last"])
    rd.q4_load(s["caches"], s["to"], s["first"], s["last"])
    return {"k": s["k_out"], "v": s["v_out"]}


def _own_commit(s):
    rd = _library(s)
    # (a decoding loop advances the lengths; here the same positions are written again and again)
    rd.q4_commit(s["caches"], s["k_tree"], s["v_tree"], s["path"], s["n_acc"], update_seq_lens=False)
    rd.q4_load(s["caches"], s["to"], s["first"], s["last"])
    return {"k": s["k_out"], "v": s["v_out"]}


def _own_attn(s):
    rd = _library(s)
    rd.q4_verify_attn(s["q"], s["k_tree"], s["v_tree"], s["cache"], s["parent"], s["scale"], out=s["out"], lse=s["lse"])
    return {"out": s["out"]} if s["lse"] is None else {"out": s["out"], "lse": s["lse"]}


def _own_branch(s):
    rd = _library(s)
    rd.pages_free(s["pages"], s["dst"])
    rd.pages_fork(s["pages"], s["src"], s["dst"])
    rd.pages_reserve(s["pages"], s["dst"], s["tokens"])
    return {"table": s["table"], "refs": s["refs"], "seq_lens": s["seq_lens"], "pools": s["pools"]}


def _own_compact(s):
    rd = _library(s)
    _as_found(s)
    rd.pages_compact(s["pages"], n_used=s["n_used"])
    return {"table": s["table"], "refs": s["refs"], "n_used": s["n_used"], "pools": s["pools"]}


def run(s):
    op = s["case"]["op"]
    if own:
        return {"convert": _own_convert, "commit": _own_commit, "attn": _own_attn, "branch": _own_branch, "compact": _own_compact}[op](s)
    return {"convert": _plain_convert, "commit": _plain_commit, "attn": _plain_attn, "branch": _plain_branch,
            "compact": _plain_compact}[op](s)


# ------------------------------------------------------------------------------------------------ in 64 bits
def _held64(x):
    """The value in 4 bits, by looking for the scale from above and for the nearest number among all fifteen."""
    y = x.double().unflatten(-1, (-1, 16))
    top = y.abs().amax(-1)
    scale = torch.full_like(top, 1.75 * 2.0 ** 13)
    for exponent in range(13, -19, -1):
        for eighths in range(15, 7, -1):
            size = eighths / 8 * 2.0 ** exponent
            if size < 1.75 * 2.0 ** 13:
                scale = torch.where(7.5 * size >= top, torch.full_like(top, size), scale)
    best, near = torch.zeros_like(y), y.abs()
    for number in (-2, 2, -4, 4, -6, 6, -1, 1, -3, 3, -5, 5, -7, 7):   # (between two of them the even one wins: it comes first)
        value = number * scale[..., None]
        nearer = (y - value).abs() < near
        best, near = torch.where(nearer, value, best), torch.where(nearer, (y - value).abs(), near)
    return best.flatten(-2)


def _unpack64(tile, d, kind):
    """Values [64, d] of one tile, element by element from the places of its bits."""
    raw = tile.to(torch.int64)
    word = raw[0:32 * d:4] | raw[1:32 * d:4] << 8 | raw[2:32 * d:4] << 16 | raw[3:32 * d:4] << 24
    r = torch.arange(PAGE, device=_DEV)[:, None].expand(PAGE, d)
    x = torch.arange(d, device=_DEV)[None].expand(PAGE, d)
    if kind == "k":
        index, bit = r * (d // 8) + x // 8, 4 * ((x % 8) // 2) + 16 * (x % 2) + 3
        lane = (r % 8) * 4 + x // (d // 4)
        place = (lane * 8 + r // 8) * (d // 64) + (x // 16) % (d // 64)
    else:
        pair, per = r // 2, d // 32
        turn = 2 * (pair % 4) if d == 128 else 4 * (pair // 2 % 2)
        index, bit = pair * (d // 4) + torch.bitwise_xor(x // 4 // per, turn) * per + x // 4 % per, 4 * (x % 4) + 16 * (r % 2) + 3
        place = ((x // 16 * 4 + pair % 4) * 8 + pair // 4) * 2 + r % 2
    twice = word | word << 32                      # so that a number that wraps around the word lies in one piece
    number = torch.where(bit < 32, twice[index] >> bit, twice[index] >> (bit - 32)) & 15
    code = raw[32 * d + place]
    return (number - 8).double() * (1 + (code % 8).double() / 8) * torch.pow(2.0, (code // 8 - 18).double())


def _exact_attn(s):
    c = s["case"]
    d, hkv, nodes = c["d"], c["hkv"], c["nodes"]
    group = c["hq"] // hkv
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=_DEV)
    lse = torch.zeros(s["q"].shape[:3], dtype=torch.float64, device=_DEV)
    parents = s["parent"].tolist()
    unpack = torch.vmap(lambda tile, kind: _unpack64(tile, d, kind), in_dims=(0, None))
    for b, length in enumerate(s["past"]):
        sees = torch.zeros(nodes, nodes, dtype=torch.bool)
        for j, p in enumerate(parents[b]):
            if p >= 0:
                sees[j] = sees[p]
            sees[j, j] = True
        sees = sees.to(_DEV)
        pages = s["q4_table"][b, :_pages(length)].long()
        for h in range(hkv):
            heads = slice(h * group, (h + 1) * group)
            q = s["q"][b, :, heads].double()
            k, v = (unpack(s[name][pages, h], kind).reshape(-1, d)[:length] for name, kind in (("k4", "k"), ("v4", "v")))
            near = torch.einsum("jgd,td->jgt", q, s["k_tree"][b, :, h].double()) * s["scale"]
            near = near.masked_fill(~sees[:, None], float("-inf"))
            score = torch.cat([torch.einsum("jgd,td->jgt", q, k) * s["scale"], near], -1)
            total = torch.logsumexp(score, -1)
            weight = (score - total[..., None]).exp()
            out[b, :, heads] = (torch.einsum("jgt,td->jgd", weight[..., :length], v)
                                + torch.einsum("jgt,td->jgd", weight[..., length:], s["v_tree"][b, :, h].double()))
            lse[b, :, heads] = total
    return {"out": out} if s["lse"] is None else {"out": out, "lse": lse}


def exact(c, seed):
    if c["op"] in ("branch", "compact"):
        return None   # pages and counts: whole numbers, no computed ones
    s = prepare(c, seed)
    if c["op"] == "attn":
        return _exact_attn(s)
    n, past = _lengths(c)
    at = [(b, past[b] + i, i) for b in range(len(n)) for i in range(n[b])]
    table, out_table = s.get("table", s["q4_table"]).tolist(), s["out_table"].tolist()
    to = torch.tensor([out_table[b][p // PAGE] * PAGE + p % PAGE for b, p, _ in at], device=_DEV)

    def placed(rows, pool):
        pages, hkv, _, d = pool.shape
        flat = torch.zeros(pages * PAGE, hkv, d, dtype=torch.float64, device=_DEV)
        flat[to] = _held64(rows)
        return flat.view(pages, PAGE, hkv, d).transpose(1, 2).contiguous()

    if c["op"] == "convert":
        of = torch.tensor([table[b][p // PAGE] * PAGE + p % PAGE for b, p, _ in at], device=_DEV)
        rows = [s[x].transpose(1, 2).reshape(-1, c["hkv"], c["d"])[of] for x in ("k_pool", "v_pool")]
        return {"k": placed(rows[0], s["k_out"]), "v": placed(rows[1], s["v_out"])}
    path = s["path"].tolist()
    seq, node = torch.tensor([b for b, _, _ in at], device=_DEV), torch.tensor([path[b][i] for b, _, i in at], device=_DEV)
    return {"k": [placed(t[seq, node], o) for t, o in zip(s["k_tree"], s["k_out"])],
            "v": [placed(t[seq, node], o) for t, o in zip(s["v_tree"], s["v_out"])]}
