"""The prompt-side operators of the library as cases that can be run and timed.

Three operators: ``append`` (norms of queries and keys, position rotation and the write of K and V into the paged
cache), ``tree`` (the same for the nodes of draft trees) and ``attn`` (causal attention of packed prompts, prompt
pieces and single tokens over the paged cache).  ``run`` computes them in elementary torch operations, or through
the library where ``own`` is true; ``exact`` computes them in 64 bits.
"""
import functools
import random

import torch

own = False

PAGE = 64
_DEV = "cuda:0"


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    small, big = dict(hq=8, hkv=8, d=64), dict(hq=32, hkv=8, d=128)
    return [
        # one decoding step of 32 sequences without a draft: one new row each
        dict(name="append_single_tokens", op="append", batch=32, n_min=1, n_max=1, l_min=1024, l_max=4096, **big,
             norm=True, rot=128, interleaved=False),
        # two short prompts of odd lengths on the small head layout, no norms, a part of each head rotated in pairs
        dict(name="append_short_pairs", op="append", batch=2, n_min=131, n_max=517, l_min=0, l_max=90, **small,
             norm=False, rot=32, interleaved=True),
        # a batch of whole prompts of different lengths
        dict(name="append_prompts", op="append", batch=8, n_min=100, n_max=4096, l_min=0, l_max=0, **big,
             norm=True, rot=128, interleaved=False),
        # the draft tree of a single prompt
        dict(name="tree_one", op="tree", batch=1, nodes=16, l_min=512, l_max=512, **small, norm=True, rot=64,
             interleaved=False),
        # large draft trees in a large batch
        dict(name="tree_batch", op="tree", batch=64, nodes=128, l_min=256, l_max=4096, **big, norm=True, rot=128,
             interleaved=False),
        # plain decoding of one short context: latency
        dict(name="attn_one_token", op="attn", batch=1, n_min=1, n_max=1, l_min=511, l_max=511, **small, lse=False),
        # plain decoding of a served batch
        dict(name="attn_single_tokens", op="attn", batch=32, n_min=1, n_max=1, l_min=1024, l_max=4096, **big, lse=True),
        # short prompts with equal numbers of query and KV heads behind a short history
        dict(name="attn_short_heads64", op="attn", batch=5, n_min=33, n_max=700, l_min=0, l_max=300, **small, lse=True),
        # a batch of prompts of different lengths, an empty one possible
        dict(name="attn_ragged", op="attn", batch=16, n_min=0, n_max=2048, l_min=0, l_max=0, **big, lse=False),
        # one prompt of ordinary length
        dict(name="attn_prompt", op="attn", batch=1, n_min=4096, n_max=4096, l_min=0, l_max=0, **big, lse=False),
        # the next piece of two long prompts whose beginnings are in the cache
        dict(name="attn_piece", op="attn", batch=2, n_min=777, n_max=1024, l_min=30000, l_max=32768, **big, lse=False),
        # the largest: long prompts
        dict(name="attn_long", op="attn", batch=4, n_min=6001, n_max=8192, l_min=0, l_max=0, **big, lse=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(lo * (hi / lo) ** rng.random())))


def draw(rng):
    limit = {op: max(_cost(c) for c in listed() if c["op"] == op) for op in ("append", "tree", "attn")}
    while True:
        op = rng.choice(["append", "tree", "attn", "attn"])
        d = rng.choice([64, 128, 128])
        hkv, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 5, 7, 8])
        c = dict(op=op, batch=_log_int(rng, 1, 64), hq=hkv * group, hkv=hkv, d=d)
        if op == "tree":
            c["nodes"] = _log_int(rng, 1, 128)
            c["l_min"] = rng.choice([0, _log_int(rng, 1, 4096)])
            c["l_max"] = c["l_min"] + rng.choice([0, _log_int(rng, 1, 1024)])
        else:
            form = rng.choice(["single", "prompt", "piece"])
            c["n_max"] = 1 if form == "single" else _log_int(rng, 2, 8192 if form == "prompt" else 1024)
            c["n_min"] = 1 if form == "single" else rng.randint(0, c["n_max"])
            c["l_max"] = 0 if form == "prompt" else _log_int(rng, 1, 32768 if op == "attn" else 8192)
            c["l_min"] = rng.randint(0, c["l_max"])
        if op == "attn":
            c["lse"] = rng.random() < 0.5
        else:
            c["norm"] = rng.random() < 0.6
            c["interleaved"] = rng.random() < 0.4
            c["rot"] = rng.choice([d, d, d // 2, d // 4 * 3])
        if 0 < _cost(c) <= limit[op] and _room(c) <= 12 << 30:
            return c


def _lengths(c):
    """New tokens and committed lengths per sequence: a property of the case, not of the seed."""
    rng = random.Random("%s %s %s" % (c["batch"], c.get("n_max"), c["l_max"]))
    spread = lambda lo, hi: [rng.randint(lo, hi) for _ in range(c["batch"])]  # noqa: E731
    n = [c["nodes"]] * c["batch"] if c["op"] == "tree" else spread(c["n_min"], c["n_max"])
    if c["op"] != "tree" and sum(n) == 0:
        n[0] = max(1, c["n_max"])
    return n, spread(c["l_min"], c["l_max"])


def _room(c):
    """Bytes of the pools a case needs."""
    n, past = _lengths(c)
    return 0 if c["op"] == "tree" else sum((a + b + PAGE) for a, b in zip(n, past)) * c["hkv"] * c["d"] * 4


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 6e12, w["flops"] / 1.5e15) if c["op"] == "attn" else w["bytes"]


def work(c):
    n, past = _lengths(c)
    tokens, row = sum(n), c["d"] * 2
    if c["op"] == "attn":
        keys = sum(a + b for a, b in zip(n, past) if a)
        pairs = sum(a * b + a * (a + 1) // 2 for a, b in zip(n, past))
        return {"bytes": 2 * tokens * c["hq"] * row + 2 * keys * c["hkv"] * row + (4 * tokens * c["hq"] if c["lse"] else 0),
                "flops": 4 * c["d"] * c["hq"] * pairs}
    heads = c["hq"] + 2 * c["hkv"]
    return {"bytes": 2 * tokens * heads * row + 4 * c["rot"] * tokens + 4 * tokens,
            "flops": tokens * (c["hq"] + c["hkv"]) * ((4 * c["d"] if c["norm"] else 0) + 3 * c["rot"])}


# ------------------------------------------------------------------------------------------------ inputs
def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=_DEV, dtype=torch.float32).to(torch.bfloat16)


def _trees(g, batch, nodes):
    """Parent arrays: every node hangs under a random earlier one, the last few at most."""
    back = torch.randint(1, 9, (batch, nodes), generator=g, device=_DEV)
    parent = (torch.arange(nodes, device=_DEV) - back).clamp(min=0)
    parent[:, 0] = -1
    return parent.to(torch.int32)


def prepare(c, seed):
    g = torch.Generator(device=_DEV)
    g.manual_seed(seed)
    n, past = _lengths(c)
    d, hq, hkv, tokens = c["d"], c["hq"], c["hkv"], sum(n)
    s = dict(case=c, n=n, past=past, seq_lens=torch.tensor(past, dtype=torch.int32, device=_DEV),
             token_start=torch.tensor([0] + [sum(n[:i + 1]) for i in range(len(n))], dtype=torch.int32, device=_DEV))
    if c["op"] != "tree":
        pages = [(a + b + PAGE - 1) // PAGE for a, b in zip(n, past)]
        width, total = max(max(pages), 1), sum(pages) + 1
        order = torch.randperm(total, generator=g, device=_DEV).to(torch.int32)
        table = torch.full((c["batch"], width), -1, dtype=torch.int32, device=_DEV)
        for b, used in enumerate(pages):
            table[b, :used] = order[sum(pages[:b]):sum(pages[:b]) + used]
        s["page_table"] = table
        s["k_pool"], s["v_pool"] = _normal(g, total, hkv, PAGE, d), _normal(g, total, hkv, PAGE, d)
    if c["op"] == "attn":
        s["q"], s["out"] = _normal(g, tokens, hq, d), torch.empty(tokens, hq, d, dtype=torch.bfloat16, device=_DEV)
        s["lse"] = torch.empty(tokens, hq, dtype=torch.float32, device=_DEV) if c["lse"] else None
        s["scale"] = d ** -0.5
        return s
    # the output of one fused projection: queries, keys and values of a token side by side
    lead = (c["batch"], c["nodes"]) if c["op"] == "tree" else (tokens,)
    qkv = _normal(g, *lead, hq + 2 * hkv, d)
    s["q"], s["k"], s["v"] = qkv[..., :hq, :], qkv[..., hq:hq + hkv, :], qkv[..., hq + hkv:, :]
    s["q_out"] = torch.empty(*lead, hq, d, dtype=torch.bfloat16, device=_DEV)
    if c["op"] == "tree":
        s["parent"] = _trees(g, c["batch"], c["nodes"])
        s["k_tree"], s["v_tree"] = (torch.empty(*lead, hkv, d, dtype=torch.bfloat16, device=_DEV) for _ in range(2))
    s["q_weight"] = s["k_weight"] = None
    if c["norm"]:
        s["q_weight"], s["k_weight"] = ((1 + 0.1 * torch.randn(d, generator=g, device=_DEV)).to(torch.bfloat16) for _ in range(2))
    positions = max(a + b for a, b in zip(n, past))
    freq = 10000.0 ** (-torch.arange(0, c["rot"], 2, device=_DEV, dtype=torch.float64) / c["rot"])
    angle = torch.arange(positions, device=_DEV, dtype=torch.float64)[:, None] * freq
    s["rope"] = torch.stack([angle.cos(), angle.sin()], 1).float().contiguous()   # [positions, 2, rot / 2]
    s["eps"], s["interleaved"] = 1e-6, c["interleaved"]
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _rotated(x, rows, s, weight):
    """Norm and rotation of x [..., heads, d] in 32 bits; rows [..., 2, rot / 2] are the positions' table rows."""
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"]) * weight.float()
    rot = 2 * rows.shape[-1]
    cos, sin = rows[..., None, 0, :], rows[..., None, 1, :]
    part, rest = x[..., :rot], x[..., rot:]
    if s["interleaved"]:
        a, b = part[..., 0::2], part[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = part[..., :rot // 2], part[..., rot // 2:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, rest], -1).to(torch.bfloat16)


def _plain_append(s):
    start = s["token_start"].long()
    token = torch.arange(s["q"].shape[0], device=_DEV)
    seq = torch.searchsorted(start, token, right=True) - 1
    pos = s["seq_lens"].long()[seq] + token - start[seq]
    rows = s["rope"][pos]
    page, at = s["page_table"].long()[seq, pos // PAGE], pos % PAGE
    s["q_out"].copy_(_rotated(s["q"], rows, s, s["q_weight"]))
    s["k_pool"][page, :, at] = _rotated(s["k"], rows, s, s["k_weight"])
    s["v_pool"][page, :, at] = s["v"]
    return {"q": s["q_out"], "k_pool": s["k_pool"], "v_pool": s["v_pool"]}


def _plain_tree(s):
    parent = s["parent"].long()
    nodes = parent.shape[1]
    # depth by doubling: after step i, hop[j] is j's ancestor 2^i levels up and depth[j] the nodes on the way to it
    # (above the root is a node `nodes` of depth 0, its own ancestor); 2^7 levels are the most a tree can have
    hop = torch.cat([torch.where(parent < 0, nodes, parent), torch.full_like(parent[:, :1], nodes)], 1)
    depth = (torch.arange(nodes + 1, device=_DEV) < nodes).long().expand_as(hop)
    depth, hop = functools.reduce(lambda x, _: (x[0] + x[0].gather(1, x[1]), x[1].gather(1, x[1])), range(7), (depth, hop))
    pos = s["seq_lens"].long()[:, None] + depth[:, :-1] - 1
    rows = s["rope"][pos]
    s["q_out"].copy_(_rotated(s["q"], rows, s, s["q_weight"]))
    s["k_tree"].copy_(_rotated(s["k"], rows, s, s["k_weight"]))
    s["v_tree"].copy_(s["v"])
    return {"q": s["q_out"], "k_tree": s["k_tree"], "v_tree": s["v_tree"]}


def _plain_attn_of(s, lo, hi):
    """Sequences lo .. hi-1, padded to their longest; writes their rows of the outputs."""
    n_list, past_list = s["n"][lo:hi], s["past"][lo:hi]
    n_max = max(n_list)
    if n_max == 0:
        return
    k_max = max(a + b for a, b in zip(n_list, past_list))
    hkv, d = s["k_pool"].shape[1], s["k_pool"].shape[3]
    group = s["q"].shape[1] // hkv
    start, n = s["token_start"][lo:hi].long(), (s["token_start"][lo + 1:hi + 1] - s["token_start"][lo:hi]).long()
    i, t = torch.arange(n_max, device=_DEV), torch.arange(k_max, device=_DEV)
    live = i < n[:, None]                                                     # [b, i]
    token = torch.where(live, start[:, None] + i, start[:, None]).clamp(max=s["q"].shape[0] - 1)
    page = s["page_table"][lo:hi].long()[:, t // PAGE].clamp(min=0)
    k, v = (s[x][page, :, t % PAGE].permute(0, 2, 1, 3).float() for x in ("k_pool", "v_pool"))   # [b, hkv, t, d]
    q = s["q"][token].float().view(hi - lo, n_max, hkv, group, d).permute(0, 2, 3, 1, 4).reshape(hi - lo, hkv, group * n_max, d)
    score = (q @ k.transpose(-1, -2)).view(hi - lo, hkv, group, n_max, k_max) * s["scale"]
    seen = t <= (s["seq_lens"][lo:hi].long()[:, None] + i)[..., None]          # [b, i, t]
    score = score.masked_fill_(~seen[:, None, None], float("-inf"))
    top = score.amax(-1, keepdim=True)
    weight = score.sub_(top).exp_()
    total = weight.sum(-1, keepdim=True)
    out = (weight.view(hi - lo, hkv, group * n_max, k_max) @ v).view(hi - lo, hkv, group, n_max, d) / total
    out = out.permute(0, 3, 1, 2, 4).reshape(hi - lo, n_max, hkv * group, d)
    s["out"][token[live]] = out[live].to(torch.bfloat16)
    if s["lse"] is not None:
        lse = (top + total.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(hi - lo, n_max, hkv * group)
        s["lse"][token[live]] = lse[live]


def _plain_attn(s):
    # as many sequences at a time as keep the padded scores and the gathered keys within 2 Gi values
    k_max = max(a + b for a, b in zip(s["n"], s["past"]))
    one = max(1, s["q"].shape[1] * max(s["n"]) * k_max, 2 * s["k_pool"].shape[1] * s["k_pool"].shape[3] * k_max)
    step = max(1, (2 << 30) // one)
    [_plain_attn_of(s, lo, min(lo + step, len(s["n"]))) for lo in range(0, len(s["n"]), step)]
    return {"out": s["out"]} if s["lse"] is None else {"out": s["out"], "lse": s["lse"]}


# ------------------------------------------------------------------------------------------------ the library
_reader = None


def _library(s):
    """The handle and the cache object that a program keeps."""
    global _reader
    from paper_2508_09072_b200 import binding
    if _reader is None:
        _reader = binding.Reader(0)
    if "cache" not in s and "k_pool" in s:
        s["cache"] = binding.KvCache(s["k_pool"], s["v_pool"], s["page_table"], s["seq_lens"])
    return _reader


def _own_append(s):
    _library(s).prompt_append(s["q"], s["k"], s["v"], s["cache"], s["token_start"], rope=s["rope"], q_weight=s["q_weight"],
                              k_weight=s["k_weight"], eps=s["eps"], interleaved=s["interleaved"], out=s["q_out"])
    return {"q": s["q_out"], "k_pool": s["k_pool"], "v_pool": s["v_pool"]}


def _own_tree(s):
    _library(s).tree_rotate(s["q"], s["k"], s["v"], s["seq_lens"], s["parent"], rope=s["rope"], q_weight=s["q_weight"],
                            k_weight=s["k_weight"], eps=s["eps"], interleaved=s["interleaved"], out=s["q_out"],
                            k_tree=s["k_tree"], v_tree=s["v_tree"])
    return {"q": s["q_out"], "k_tree": s["k_tree"], "v_tree": s["v_tree"]}


def _own_attn(s):
    _library(s).prompt_attn(s["q"], s["cache"], s["token_start"], s["scale"], out=s["out"], lse=s["lse"])
    return {"out": s["out"]} if s["lse"] is None else {"out": s["out"], "lse": s["lse"]}


def run(s):
    op = s["case"]["op"]
    if own:
        return {"append": _own_append, "tree": _own_tree, "attn": _own_attn}[op](s)
    return {"append": _plain_append, "tree": _plain_tree, "attn": _plain_attn}[op](s)


# ------------------------------------------------------------------------------------------------ in 64 bits
def _turn64(row, table, s, weight):
    """One token's heads [heads, d], from the definition."""
    y = row.double()
    if weight is not None:
        y = y / torch.sqrt(y.square().sum(-1, keepdim=True) / y.shape[-1] + s["eps"]) * weight.double()
    half = table.shape[-1]
    cos, sin = table[0].double(), table[1].double()
    first = torch.arange(half, device=_DEV) * (2 if s["interleaved"] else 1)
    second = first + (1 if s["interleaved"] else half)
    z = y.clone()
    z[..., first] = y[..., first] * cos - y[..., second] * sin
    z[..., second] = y[..., first] * sin + y[..., second] * cos
    return z


def _turn64_many(x, table, s, weight):
    return torch.vmap(lambda r, t: _turn64(r, t, s, weight))(x, table) if x.shape[0] else x.double()


def exact(c, seed):
    s = prepare(c, seed)
    n, past = s["n"], s["past"]
    if c["op"] == "attn":
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device=_DEV)
        lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device=_DEV)
        hkv = s["k_pool"].shape[1]
        group = s["q"].shape[1] // hkv
        begin = 0
        for b in range(len(n)):
            keys = past[b] + n[b]
            pages = s["page_table"][b, :(keys + PAGE - 1) // PAGE].long()
            for h in range(hkv if n[b] else 0):
                k = s["k_pool"][pages, h].reshape(-1, s["q"].shape[2])[:keys].double()
                v = s["v_pool"][pages, h].reshape(-1, s["q"].shape[2])[:keys].double()
                for i in range(0, n[b], 1024):
                    j = min(i + 1024, n[b])
                    sees = past[b] + j
                    q = s["q"][begin + i:begin + j, h * group:(h + 1) * group].double()
                    score = torch.einsum("igd,td->igt", q, k[:sees]) * s["scale"]
                    later = torch.arange(sees, device=_DEV)[None, :] > torch.arange(past[b] + i, past[b] + j, device=_DEV)[:, None]
                    score = score.masked_fill(later[:, None, :], float("-inf"))
                    total = torch.logsumexp(score, -1)
                    out[begin + i:begin + j, h * group:(h + 1) * group] = torch.einsum("igt,td->igd", (score - total[..., None]).exp(), v[:sees])
                    lse[begin + i:begin + j, h * group:(h + 1) * group] = total
            begin += n[b]
        return {"out": out} if s["lse"] is None else {"out": out, "lse": lse}
    if c["op"] == "tree":
        parents = s["parent"].tolist()
        pos = []
        for b, par in enumerate(parents):
            level = []
            for p in par:
                level.append(0 if p < 0 else level[p] + 1)
            pos += [past[b] + lv for lv in level]
        rows = s["rope"][torch.tensor(pos, device=_DEV)]
        flat = lambda x: x.reshape(-1, *x.shape[-2:])  # noqa: E731
        q = _turn64_many(flat(s["q"]), rows, s, s["q_weight"]).view(s["q"].shape)
        k = _turn64_many(flat(s["k"]), rows, s, s["k_weight"]).view(s["k"].shape)
        return {"q": q, "k_tree": k, "v_tree": s["v"].double()}
    at = [(b, past[b] + i) for b in range(len(n)) for i in range(n[b])]
    table = s["page_table"].tolist()
    rows = s["rope"][torch.tensor([p for _, p in at], device=_DEV)]
    slot = torch.tensor([table[b][p // PAGE] * PAGE + p % PAGE for b, p in at], device=_DEV)
    pools = {}
    for name, x in (("k_pool", _turn64_many(s["k"], rows, s, s["k_weight"])), ("v_pool", s["v"].double())):
        pages, hkv, _, d = s[name].shape
        flat = s[name].double().transpose(1, 2).reshape(pages * PAGE, hkv, d)
        flat[slot] = x
        pools[name] = flat.view(pages, PAGE, hkv, d).transpose(1, 2).contiguous()
    return {"q": _turn64_many(s["q"], rows, s, s["q_weight"]), **pools}
