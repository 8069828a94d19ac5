"""Performance cases of the operators on a paged cache: attention for a tree of drafted tokens, the commit of its
accepted path, accumulated attention weights, eviction by them, and attention over selected pages.

The cache is that of the decoding path: pages of 64 positions, a pool per layer and a page table per sequence.  A step of
a program that drafts trees of tokens runs, per layer, one of the two attentions over the cache and the drafted nodes,
then looks at the base model's predictions for all nodes and commits the accepted path to the caches of all layers.  A
program that bounds its cache adds up the attention weight of the accepted tokens and evicts by it.

Where ``own`` is false a pass computes the operators in elementary torch operations; where it is true it makes the
library's calls.
"""
import math

import torch

own = False

PAGE = 64


def listed():
    def tree(name, batch, nodes, heads, kv_heads, dim, lo, hi, dtype, shape):
        return {"name": name, "kind": "tree", "batch": batch, "nodes": nodes, "heads": heads, "kv_heads": kv_heads, "dim": dim,
                "len_lo": lo, "len_hi": hi, "dtype": dtype, "shape": shape}

    def commit(name, layers, batch, nodes, kv_heads, dim, lo, hi, dtype):
        return {"name": name, "kind": "commit", "layers": layers, "batch": batch, "nodes": nodes, "kv_heads": kv_heads, "dim": dim,
                "len_lo": lo, "len_hi": hi, "dtype": dtype}

    def weights(name, batch, nodes, heads, kv_heads, dim, lo, hi, dtype):
        return {"name": name, "kind": "weights", "batch": batch, "nodes": nodes, "heads": heads, "kv_heads": kv_heads, "dim": dim,
                "len_lo": lo, "len_hi": hi, "dtype": dtype}

    def evict(name, layers, batch, kv_heads, dim, lo, hi, budget, recent, dtype):
        return {"name": name, "kind": "evict", "layers": layers, "batch": batch, "kv_heads": kv_heads, "dim": dim, "len_lo": lo,
                "len_hi": hi, "budget": budget, "recent": recent, "dtype": dtype}

    def pages(name, batch, nodes, heads, kv_heads, dim, lo, hi, select, fresh, dtype):
        return {"name": name, "kind": "pages", "batch": batch, "nodes": nodes, "heads": heads, "kv_heads": kv_heads, "dim": dim,
                "len_lo": lo, "len_hi": hi, "select": select, "fresh": fresh, "dtype": dtype}
    return [
        # the smallest call: one token of one sentence, base translation model, nothing but latency
        tree("tree_one_token", 1, 1, 8, 8, 64, 57, 57, "bf16", "chain"),
        # offline translation: blocks of ten proposals for 32 ragged sentences, big model
        tree("tree_blocks32", 32, 10, 16, 16, 64, 1, 128, "bf16", "chain"),
        # fp32 model, small trees over caches of odd lengths, four query heads to a key head
        tree("tree_fp32", 4, 13, 8, 2, 64, 500, 2500, "fp32", "tree"),
        # large trees over long ragged caches: what a server of a large model drafts
        tree("tree_long", 8, 32, 32, 8, 128, 2000, 16000, "bf16", "tree"),
        # one sentence's block goes to the caches of six layers
        commit("commit_sentence", 6, 1, 8, 8, 64, 40, 40, "bf16"),
        # a server's batch of trees, all layers of a large model
        commit("commit_batch", 24, 24, 32, 8, 128, 20, 220, "bf16"),
        # the weights of a few accepted tokens of one sequence
        weights("weights_one", 1, 4, 8, 8, 64, 501, 501, "bf16"),
        # the same for a server's batch over long caches
        weights("weights_long", 16, 8, 32, 8, 128, 4000, 16000, "bf16"),
        # every step of a bounded cache: a block over the budget leaves, few entries move
        evict("evict_step", 6, 1, 8, 64, 517, 522, 512, 64, "fp32"),
        # after a long prompt: most of the cache leaves at once
        evict("evict_prompt", 4, 8, 8, 128, 4000, 8000, 1024, 128, "bf16"),
        # one token over a long cache, of which a few pages are read
        pages("pages_one_token", 1, 1, 32, 8, 128, 30000, 30000, 16, False, "bf16"),
        # a server's batch of small trees right after the prompts: the pages' means are built, then used
        pages("pages_batch", 8, 8, 32, 8, 128, 8000, 60000, 32, True, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["tree", "tree", "commit", "weights", "evict", "pages"])
    dim = rng.choice([16, 32, 64, 64, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16]) if dim < 128 else rng.choice([1, 2, 4, 8])
    heads = kv_heads * rng.choice([1, 1, 2, 3, 4, 8])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    batch = _log_int(rng, 1, 32)
    # positions of all sequences together, so that no case costs more than the largest listed one
    room = 16000 * 4 * 1024 // (batch * kv_heads * dim * (2 if dtype == "fp32" else 1))
    hi = _log_int(rng, 1, max(2, min(16000, room)))
    case = {"kind": kind, "batch": batch, "kv_heads": kv_heads, "dim": dim, "len_hi": hi, "len_lo": max(1, hi // rng.randint(1, 8)), "dtype": dtype}
    if kind == "tree":
        return {**case, "heads": heads, "nodes": _log_int(rng, 1, 64 * kv_heads // heads if heads > kv_heads else 64), "shape": rng.choice(["chain", "tree", "tree"])}
    if kind == "commit":
        hi = rng.randint(1, 200)
        return {**case, "layers": rng.randint(1, 12), "nodes": _log_int(rng, 1, 64), "len_hi": hi, "len_lo": rng.randint(0, hi)}
    if kind == "weights":
        return {**case, "heads": heads, "nodes": _log_int(rng, 1, 16)}
    if kind == "evict":
        budget = rng.randint(1, hi + hi // 4 + 1)
        return {**case, "layers": rng.randint(1, 3), "budget": budget, "recent": rng.randint(0, budget)}
    return {**case, "heads": heads, "nodes": _log_int(rng, 1, 8), "select": _log_int(rng, 1, 32), "fresh": rng.choice([False, True])}


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


# ---------------------------------------------------------------------- inputs
def _lengths(case, gen):
    lo, hi, b = case["len_lo"], case["len_hi"], case["batch"]
    lens = torch.randint(lo, hi + 1, (b,), generator=gen, dtype=torch.int32)
    lens[int(torch.randint(0, b, (1,), generator=gen))] = hi
    return lens


def _trees(case, gen):
    """parents [batch, nodes] (-1: the last committed token), nodes of each sequence."""
    b, t = case["batch"], case["nodes"]
    index = torch.arange(t)
    if case.get("shape") == "chain":
        parents = (index - 1).expand(b, t)
    else:
        # nodes come level by level, as proposal heads draft them: a node's parent is one of the last few before it
        back = 1 + (torch.rand(b, t, generator=gen) ** 2 * min(t, 6)).long()
        parents = (index - back).clamp(min=-1)
    nodes = torch.full((b,), t, dtype=torch.int32)
    if b > 1 and t > 1:
        nodes = torch.randint(max(1, t // 2), t + 1, (b,), generator=gen, dtype=torch.int32)
        nodes[0] = t
    return parents.int().contiguous(), nodes


def _pools(case, layers, capacity, gen, dev_gen):
    """Pools of all layers and a page table that gives out their pages in no order."""
    per_row = -(-capacity // PAGE)
    n = case["batch"] * per_row
    table = torch.randperm(n, generator=gen).view(case["batch"], per_row).int().cuda()
    shape = (layers, n, PAGE, case["kv_heads"], case["dim"])
    k, v = (torch.empty(shape, dtype=_type(case), device="cuda").normal_(generator=dev_gen) for _ in range(2))
    return k, v, table


def _randn(shape, dtype, gen, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)


def prepare(case, seed):
    gen = torch.Generator().manual_seed(seed)
    dev = torch.Generator("cuda").manual_seed(seed)
    kind, b, hk, d, dt = case["kind"], case["batch"], case["kv_heads"], case["dim"], _type(case)
    lens = _lengths(case, gen)
    st = {"case": case, "lens": lens.cuda(), "max_len": int(lens.max())}
    if kind in ("tree", "pages", "weights", "commit"):
        t = case["nodes"]
        parents, nodes = _trees(case, gen)
        st.update(parents=parents.cuda(), nodes=nodes.cuda())
        layers = case.get("layers", 1)
        st["k"], st["v"], st["table"] = _pools(case, layers, case["len_hi"] + t, gen, dev)
    if kind in ("tree", "pages"):
        h = case["heads"]
        st["q"] = _randn((b, t, h, d), dt, dev, 1.5)
        st["k_new"], st["v_new"] = _randn((b, t, hk, d), dt, dev), _randn((b, t, hk, d), dt, dev)
    if kind == "pages":
        per_row = st["table"].shape[1]
        # what the pages filled in earlier steps left; a step fills the pages of its last 200 positions at most
        start = torch.zeros_like(lens) if case["fresh"] else (lens - torch.randint(0, 200, (b,), generator=gen, dtype=torch.int32)).clamp(min=0)
        st["from"] = start.int().cuda()
        st["means"] = torch.zeros(1, b, per_row, hk, d, device="cuda")
        if not case["fresh"]:
            st["means"] = _plain_means(st["k"], st["table"], st["means"], torch.zeros_like(st["from"]), st["from"])
    if kind == "commit":
        st["k_new"], st["v_new"] = (_randn((layers, b, t, hk, d), dt, dev) for _ in range(2))
        # a few token ids only, so that paths of several nodes come up as with drafts that are often right
        st["tokens"] = torch.randint(0, 2, (b, t), generator=gen, dtype=torch.int32).cuda()
        st["top1"] = torch.randint(0, 2, (b, t), generator=gen, dtype=torch.int32).cuda()
        st["last_top1"] = torch.randint(0, 2, (b,), generator=gen, dtype=torch.int32).cuda()
    if kind == "weights":
        h = case["heads"]
        st["q"] = _randn((b, t, h, d), dt, dev, 1.5)
        # one accepted path: some of the nodes in ascending order
        accepted = torch.stack([torch.randint(1, int(n) + 1, (), generator=gen) for n in nodes]).int()
        order = torch.rand(b, t, generator=gen).masked_fill(torch.arange(t) >= nodes[:, None], 2.0).argsort(1)
        path = order.masked_fill(torch.arange(t) >= accepted[:, None], t).sort(1).values
        path = path.masked_fill(path == t, -1).int()
        st.update(path=path.cuda(), accepted=accepted.cuda(), seen=(st["lens"] * 2 + 5).int())
        cap = st["table"].shape[1] * PAGE
        st["weights"] = torch.rand(1, b, hk, cap, generator=dev, device="cuda") ** 4
        st["positions"] = torch.arange(cap, dtype=torch.int32, device="cuda").expand(1, b, hk, cap).contiguous()
        # the attention that went before left the logarithm of every query's softmax sum
        st["lse"] = _path_lse(st)
    if kind == "evict":
        layers = case["layers"]
        st["k"], st["v"], st["table"] = _pools(case, layers, case["len_hi"], gen, dev)
        cap = st["table"].shape[1] * PAGE
        st["weights"] = torch.rand(layers, b, hk, cap, generator=dev, device="cuda") ** 4
        # positions lie in no order once entries have moved
        st["positions"] = torch.rand(layers, b, hk, cap, generator=dev, device="cuda").masked_fill(
            torch.arange(cap, device="cuda") >= st["lens"][:, None, None], 2.0).argsort(-1).argsort(-1).int()
        st["seen"] = st["lens"].clone()
    return st


def _path_lse(st):
    """log of the softmax sum of every node on the path, over the cache as it is after the commit; 0 elsewhere."""
    q, path, lens = st["q"].float(), st["path"], st["lens"]
    b, t, h, d = q.shape
    hk = st["k"].shape[3]
    keys = _gather(st["k"][0], st["table"], st["table"].shape[1] * PAGE)
    at = path.clamp(min=0).long()
    rows = q.gather(1, at[:, :, None, None].expand(b, t, h, d)).view(b, t, hk, h // hk, d).permute(0, 2, 1, 3, 4).reshape(b, hk, -1, d)
    s = (rows @ keys.permute(0, 2, 3, 1)).view(b, hk, t, h // hk, -1) / math.sqrt(d)
    limit = lens[:, None] + torch.arange(t, device="cuda")
    s.masked_fill_((torch.arange(s.shape[-1], device="cuda") > limit[..., None])[:, None, :, None], -math.inf)
    found = s.logsumexp(-1).permute(0, 2, 1, 3).reshape(b, t, h)
    lse = torch.zeros(b, t + 1, h, device="cuda")
    lse.scatter_(1, path.masked_fill(path < 0, t).long()[..., None].expand(b, t, h), found)
    return lse[:, :t].contiguous()


# ---------------------------------------------------------------------- the plain forms
def _gather(pool, table, n):
    """The first n positions of every sequence as [batch, n, kv_heads, dim] in 32 bits."""
    s = torch.arange(n, device=pool.device)
    return pool[table[:, s // PAGE].long(), s % PAGE].float()


def _ancestors(parents, nodes):
    """[batch, t, u]: node u is t itself or above it."""
    t = parents.shape[1]
    index = torch.arange(t, device=parents.device)
    m = (parents[..., None] == index) | (index[:, None] == index)
    for _ in range(max(1, (t - 1).bit_length())):
        m = (m.float() @ m.float()) > 0
    return m & (index < nodes[:, None])[:, None, :]


def _softmax_rows(s, values):
    """s [..., r, n] with -inf where masked, values [..., n, d]: outputs, and log of the sums."""
    top = s.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    p = (s - top).exp()
    total = p.sum(-1, keepdim=True)
    out = (p @ values) / torch.where(total == 0, torch.ones_like(total), total)
    return out, (total.log() + top).squeeze(-1)


def _plain_tree(st):
    q, parents, nodes, lens = st["q"].float(), st["parents"], st["nodes"], st["lens"]
    b, t, h, d = q.shape
    hk, n = st["k"].shape[3], st["max_len"]
    keys = torch.cat([_gather(st["k"][0], st["table"], n), st["k_new"].float()], 1).permute(0, 2, 1, 3)
    values = torch.cat([_gather(st["v"][0], st["table"], n), st["v_new"].float()], 1).permute(0, 2, 1, 3)
    rows = q.view(b, t, hk, h // hk, d).permute(0, 2, 1, 3, 4).reshape(b, hk, -1, d)
    s = (rows @ keys.transpose(-1, -2)).view(b, hk, t, h // hk, n + t) / math.sqrt(d)
    cached = (torch.arange(n, device=q.device) < lens[:, None])[:, None].expand(b, t, n)
    seen = torch.cat([cached, _ancestors(parents, nodes)], -1) & (torch.arange(t, device=q.device) < nodes[:, None])[..., None]
    s = s.masked_fill(~seen[:, None, :, None], -math.inf).view(b, hk, -1, n + t)
    out, lse = _softmax_rows(s, values)
    out = out.view(b, hk, t, h // hk, d).permute(0, 2, 1, 3, 4).reshape(b, t, h, d)
    return {"out": out.to(st["q"].dtype), "lse": lse.view(b, hk, t, h // hk).permute(0, 2, 1, 3).reshape(b, t, h)}


def _plain_commit(st):
    parents, tokens, top1, nodes, lens = (st[x] for x in ("parents", "tokens", "top1", "nodes", "lens"))
    b, t = parents.shape
    index = torch.arange(t, device=parents.device)
    room = st["table"].shape[1] * PAGE
    at, want = torch.full_like(lens, -1), st["last_top1"].clone()
    path, accepted = torch.full_like(parents, -1), torch.zeros_like(lens)
    for i in range(t):
        child = (parents == at[:, None]) & (tokens == want[:, None]) & (index < nodes[:, None])
        step = child.any(1) & (accepted == i) & (lens + i < room)
        nxt = child.int().argmax(1).int()
        path[:, i] = torch.where(step, nxt, path[:, i])
        at, accepted = torch.where(step, nxt, at), accepted + step.int()
        want = torch.where(step, top1.gather(1, nxt[:, None].long())[:, 0], want)
    rows, cols = (path >= 0).nonzero(as_tuple=True)
    slot = lens[rows].long() + cols
    page, node = st["table"][rows, slot // PAGE].long(), path[rows, cols].long()
    st["k"][:, page, slot % PAGE] = st["k_new"][:, rows, node]
    st["v"][:, page, slot % PAGE] = st["v_new"][:, rows, node]
    return {"lens": lens + accepted, "accepted": accepted, "path": path, "next": want, "k": st["k"], "v": st["v"]}


def _plain_weights(st):
    q, path, accepted, lens = st["q"].float(), st["path"], st["accepted"], st["lens"]
    b, t, h, d = q.shape
    hk, n = st["k"].shape[3], st["table"].shape[1] * PAGE
    at = path.clamp(min=0).long()
    rows = q.gather(1, at[:, :, None, None].expand(b, t, h, d)).view(b, t, hk, h // hk, d).permute(0, 2, 1, 3, 4).reshape(b, hk, -1, d)
    lse = st["lse"].gather(1, at[:, :, None].expand(b, t, h)).view(b, t, hk, h // hk).permute(0, 2, 1, 3)
    s = (rows @ _gather(st["k"][0], st["table"], n).permute(0, 2, 3, 1)).view(b, hk, t, h // hk, n) / math.sqrt(d)
    slot, step = torch.arange(n, device=q.device), torch.arange(t, device=q.device)
    seen = (slot <= (lens[:, None] + step)[..., None]) & (step < accepted[:, None])[..., None]
    got = (s - lse[..., None]).exp().masked_fill(~seen[:, None, :, None], 0.0).sum((2, 3))
    weights, positions = st["weights"].clone(), st["positions"].clone()
    old, new = (slot < lens[:, None])[:, None], ((slot >= lens[:, None]) & (slot < (lens + accepted)[:, None]))[:, None]
    weights[0] = torch.where(old, weights[0] + got, torch.where(new, got, weights[0]))
    positions[0] = torch.where(new, (st["seen"][:, None] + slot - lens[:, None])[:, None].int(), positions[0])
    return {"weights": weights, "positions": positions}


def _plain_evict(st):
    case, lens = st["case"], st["lens"]
    weights, positions = st["weights"].clone(), st["positions"].clone()
    layers, b, hk, n = weights.shape
    slot = torch.arange(n, device=lens.device)
    there = (slot < lens[:, None])[:, None].expand(b, hk, n)
    recent = positions >= (st["seen"] - case["recent"])[:, None, None]
    # by weight, ties to the lower slot; then the recent ones before the rest, and what is not there behind all
    order = weights.masked_fill(~there, -math.inf).argsort(dim=-1, descending=True, stable=True)
    group = torch.where(there, torch.where(recent, 0, 1), 2).gather(-1, order)
    order = order.gather(-1, group.argsort(dim=-1, stable=True))
    left = lens.clamp(max=case["budget"])
    kept = torch.zeros_like(recent).scatter_(-1, order, (slot < left[:, None])[:, None].expand(layers, b, hk, n))
    low = slot < left[:, None, None]
    holes, fill = (~kept & low), (kept & ~low)
    to = holes.nonzero()
    src = fill.nonzero()            # as many per list, both in ascending order
    la, ro, he, s0, s1 = src[:, 0], src[:, 1], src[:, 2], src[:, 3], to[:, 3]
    p0, p1 = st["table"][ro, s0 // PAGE].long(), st["table"][ro, s1 // PAGE].long()
    for pool in (st["k"], st["v"]):
        pool[la, p1, s1 % PAGE, he] = pool[la, p0, s0 % PAGE, he]
    weights[la, ro, he, s1] = weights[la, ro, he, s0]
    positions[la, ro, he, s1] = positions[la, ro, he, s0]
    return {"lens": left, "weights": weights, "positions": positions, "k": st["k"], "v": st["v"]}


def _plain_means(k, table, means, start, lens):
    pages = torch.arange(table.shape[1], device=k.device)
    new = (pages >= (start // PAGE)[:, None]) & (pages < (lens // PAGE)[:, None])
    rows, cols = new.nonzero(as_tuple=True)
    means = means.clone()
    means[:, rows, cols] = k[:, table[rows, cols].long()].double().mean(2).float()     # in 64 bits: selections go by them
    return means


def _plain_pages(st):
    case, q, parents, nodes, lens = st["case"], st["q"], st["parents"], st["nodes"], st["lens"]
    b, t, h, d = q.shape
    hk, table, g = st["k"].shape[3], st["table"], case["heads"] // st["k"].shape[3]
    means = _plain_means(st["k"], table, st["means"], st["from"], lens)
    per_row, dev = table.shape[1], q.device
    full = lens // PAGE
    # the scores in 64 bits: the border of a selection is often close
    sums = q.double().view(b, t, hk, g, d).sum(3).permute(0, 2, 1, 3)
    score = (sums @ means[0].double().permute(0, 2, 3, 1)).permute(0, 2, 1, 3)          # [b, t, hk, pages]
    page = torch.arange(per_row, device=dev)
    there = (page < full[:, None])[:, None, None].expand(b, t, hk, per_row)
    n = min(case["select"], per_row)
    order = score.masked_fill(~there, -math.inf).argsort(dim=-1, descending=True, stable=True)[..., :n]
    alive = (torch.arange(t, device=dev) < nodes[:, None])
    chosen = order.where(there.gather(-1, order) & alive[..., None, None], per_row).sort(-1).values
    valid = chosen < per_row
    rows = torch.arange(b, device=dev)[:, None, None, None]
    phys = table[rows, chosen.clamp(max=per_row - 1)].long()                           # [b, t, hk, n]
    head = torch.arange(hk, device=dev)[None, None, :, None]
    open_page = table.gather(1, full.clamp(max=per_row - 1)[:, None].long())[:, 0].long()
    tree = _ancestors(parents, nodes)

    def keys_of(pool, new):
        far = pool[0][phys[..., None], torch.arange(PAGE, device=dev), head[..., None]].float().reshape(b, t, hk, n * PAGE, d)
        near = pool[0][open_page].float().permute(0, 2, 1, 3)[:, None].expand(b, t, hk, PAGE, d)
        return torch.cat([far, near, new.float().permute(0, 2, 1, 3)[:, None].expand(b, t, hk, t, d)], 3)

    keys, values = keys_of(st["k"], st["k_new"]), keys_of(st["v"], st["v_new"])
    s = (q.float().view(b, t, hk, g, d) @ keys.transpose(-1, -2)) / math.sqrt(d)
    near = (torch.arange(PAGE, device=dev) < (lens % PAGE)[:, None])[:, None, None].expand(b, t, hk, PAGE)
    seen = torch.cat([valid.repeat_interleave(PAGE, -1), near, tree[:, :, None].expand(b, t, hk, t)], -1) & alive[..., None, None]
    out, lse = _softmax_rows(s.masked_fill(~seen[..., None, :], -math.inf), values)
    chosen = torch.nn.functional.pad(chosen.masked_fill(~valid, -1), (0, case["select"] - n), value=-1)
    return {"out": out.reshape(b, t, h, d).to(q.dtype), "lse": lse.reshape(b, t, h), "pages": chosen.int(), "means": means}


# ---------------------------------------------------------------------- a pass
def run(st):
    kind = st["case"]["kind"]
    if not own:
        return {"tree": _plain_tree, "commit": _plain_commit, "weights": _plain_weights, "evict": _plain_evict, "pages": _plain_pages}[kind](st)
    import paper_1811_03115_b200 as bpd
    k, v, table, lens = st["k"], st["v"], st["table"], st["lens"]
    if kind == "tree":
        out, lse = bpd.bpd_op_tree_attention(st["q"], st["k_new"], st["v_new"], k[0], v[0], table, lens, st["parents"], st["nodes"], want_lse=True)
        return {"out": out, "lse": lse}
    if kind == "commit":
        lens, accepted, path, nxt = bpd.bpd_op_tree_commit(st["k_new"], st["v_new"], k, v, table, lens, st["parents"], st["tokens"],
                                                           st["top1"], st["last_top1"], st["nodes"])
        return {"lens": lens, "accepted": accepted, "path": path, "next": nxt, "k": k, "v": v}
    if kind == "weights":
        # the sums of the step before are kept, as a program does that may still take the step back
        weights, positions = st["weights"].clone(), st["positions"].clone()
        bpd.bpd_op_cache_weights(st["q"], st["lse"], st["path"], st["accepted"], k[0], table, lens, st["seen"], weights[0], positions[0])
        return {"weights": weights, "positions": positions}
    if kind == "evict":
        weights, positions = st["weights"].clone(), st["positions"].clone()
        lens = bpd.bpd_op_cache_evict(weights, positions, k, v, table, lens, st["seen"], st["case"]["budget"], st["case"]["recent"])
        return {"lens": lens, "weights": weights, "positions": positions, "k": k, "v": v}
    means = st["means"].clone()
    bpd.bpd_op_page_means(k, table, st["from"], lens, means)
    out, lse, chosen = bpd.bpd_op_page_attention(st["q"], st["k_new"], st["v_new"], k[0], v[0], table, means[0], lens, st["parents"],
                                                 st["case"]["select"], st["nodes"], want_lse=True, want_pages=True)
    return {"out": out, "lse": lse, "pages": chosen, "means": means}


# ---------------------------------------------------------------------- work
def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    b, hk, d = case["batch"], case["kv_heads"], case["dim"]
    mean_len = (case["len_lo"] + case["len_hi"]) / 2 if b > 1 else case["len_hi"]
    row = 2 * hk * d * e                       # a position's keys and values
    t = case.get("nodes", 0)
    live = t if b == 1 or t == 1 else 0.75 * t
    if case["kind"] == "commit":
        path = min(live, 2)
        return {"bytes": 2 * case["layers"] * b * path * row + 16 * b * t, "flops": 0}
    if case["kind"] == "evict":
        left = min(case["budget"], mean_len)
        stay = left * left / mean_len
        lists = case["layers"] * b * hk
        return {"bytes": lists * (8 * mean_len + 2 * (left - stay) * (2 * d * e + 8)), "flops": 0}
    h = case["heads"]
    own_rows = b * live * (2 * h * d * e + row + 4 * h)
    if case["kind"] == "weights":
        rows = (live + 1) / 2 * h
        return {"bytes": b * (mean_len * (row / 2 + 8 * hk) + rows * (d * e + 4)), "flops": 2 * b * mean_len * rows * d}
    if case["kind"] == "tree":
        return {"bytes": b * mean_len * row + own_rows, "flops": 4 * b * mean_len * live * h * d}
    full = mean_len / PAGE
    n = min(case["select"], full)
    apart = full * (1 - (1 - n / max(1, full)) ** live)      # pages that some node of a sequence selects, drawn at random
    new = mean_len if case["fresh"] else min(100, mean_len)
    return {"bytes": b * (new * row / 2 + full * hk * d * 4 + (apart + 1) * PAGE * row) + own_rows,
            "flops": b * live * (2 * full * hk * d + 4 * (n * PAGE + PAGE / 2) * h * d)}


# ---------------------------------------------------------------------- 64 bits
def _exact_rows(q, keys, values, scale):
    """One query over the keys that it sees, in 64 bits."""
    s = (keys @ q) * scale
    w = torch.exp(s - s.max())
    return (w / w.sum()) @ values, s.max() + torch.log(w.sum())


def _exact_position(pool, table, row, positions):
    positions = torch.as_tensor(positions, dtype=torch.int64, device=pool.device)
    return pool[table[row][positions // PAGE].long(), positions % PAGE].double()


def _chain_of(parents, t):
    found = []
    while t >= 0:
        found.append(t)
        t = parents[t]
    return found[::-1]


def exact(case, seed):
    """The operators from their definition, sequence by sequence and node by node, in 64 bits."""
    st = prepare(case, seed)
    kind, b, hk, d = case["kind"], case["batch"], case["kv_heads"], case["dim"]
    lens = st["lens"].tolist()
    scale = d ** -0.5
    if kind == "commit":
        return _exact_commit(st, lens)
    if kind == "evict":
        return _exact_evict(st, lens)
    q = st["q"].double()
    t_all, h = q.shape[1], q.shape[2]
    g = h // hk
    if kind == "weights":
        weights, positions = st["weights"].double(), st["positions"].clone()
        for r in range(b):
            n, got = lens[r], int(st["accepted"][r])
            keys = _exact_position(st["k"][0], st["table"], r, range(n + got))
            weights[0, r, :, n:n + got] = 0
            positions[0, r, :, n:n + got] = torch.arange(got, dtype=torch.int32, device="cuda") + int(st["seen"][r])
            for i in range(got):
                node = int(st["path"][r, i])
                for j in range(hk):
                    s = keys[:n + i + 1, j] @ q[r, node, j * g:(j + 1) * g].T * scale
                    weights[0, r, j, :n + i + 1] += torch.exp(s - st["lse"][r, node, j * g:(j + 1) * g].double()).sum(1)
        return {"weights": weights, "positions": positions}
    out = torch.zeros(b, t_all, h, d, dtype=torch.float64, device="cuda")
    lse = torch.full((b, t_all, h), -math.inf, dtype=torch.float64, device="cuda")
    parents, nodes = st["parents"].tolist(), st["nodes"].tolist()
    if kind == "pages":
        per_row = st["table"].shape[1]
        means = st["means"].double()
        chosen = torch.full((b, t_all, hk, case["select"]), -1, dtype=torch.int32, device="cuda")
    for r in range(b):
        n = lens[r]
        keys, values = (_exact_position(st[x][0], st["table"], r, range(n)) for x in ("k", "v"))
        if kind == "pages":
            done, first = n // PAGE, int(st["from"][r]) // PAGE
            if done > first:
                means[0, r, first:done] = keys[first * PAGE:done * PAGE].view(done - first, PAGE, hk, d).sum(1) / PAGE
        for t in range(nodes[r]):
            line = _chain_of(parents[r], t)
            k_line, v_line = st["k_new"][r, line].double(), st["v_new"][r, line].double()
            for j in range(hk):
                see = slice(0, n)
                if kind == "pages" and done > 0:
                    # the operator scores with the means as they are held, in 32 bits
                    score = means[0, r, :done, j].float().double() @ q[r, t, j * g:(j + 1) * g].sum(0)
                    best = torch.sort(score, descending=True, stable=True).indices[:case["select"]].sort().values
                    chosen[r, t, j, :len(best)] = best.int()
                    see = torch.cat([(best[:, None] * PAGE + torch.arange(PAGE, device="cuda")).view(-1), torch.arange(done * PAGE, n, device="cuda")])
                ks, vs = torch.cat([keys[see, j], k_line[:, j]]), torch.cat([values[see, j], v_line[:, j]])
                s = (ks @ q[r, t, j * g:(j + 1) * g].T) * scale
                top = s.max(0).values
                w = torch.exp(s - top)
                out[r, t, j * g:(j + 1) * g] = (w / w.sum(0)).T @ vs
                lse[r, t, j * g:(j + 1) * g] = top + torch.log(w.sum(0))
    if kind == "tree":
        return {"out": out, "lse": lse}
    return {"out": out, "lse": lse, "pages": chosen, "means": means}


def _exact_commit(st, lens):
    parents, tokens, top1, nodes = (st[x].tolist() for x in ("parents", "tokens", "top1", "nodes"))
    last, room = st["last_top1"].tolist(), st["table"].shape[1] * PAGE
    k, v = st["k"].clone(), st["v"].clone()
    b, t = st["parents"].shape
    path = torch.full((b, t), -1, dtype=torch.int32)
    accepted, following = [], []
    for r in range(b):
        want, at, count = last[r], -1, 0
        while lens[r] + count < room:
            child = [u for u in range(nodes[r]) if parents[r][u] == at and tokens[r][u] == want]
            if not child:
                break
            at = child[0]
            slot = lens[r] + count
            page = int(st["table"][r, slot // PAGE])
            k[:, page, slot % PAGE], v[:, page, slot % PAGE] = st["k_new"][:, r, at], st["v_new"][:, r, at]
            path[r, count] = at
            count, want = count + 1, top1[r][at]
        accepted.append(count)
        following.append(want)
    as_i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"lens": as_i32([n + a for n, a in zip(lens, accepted)]), "accepted": as_i32(accepted), "path": path.cuda(), "next": as_i32(following), "k": k, "v": v}


def _exact_evict(st, lens):
    case = st["case"]
    k, v, weights, positions = (st[x].clone() for x in ("k", "v", "weights", "positions"))
    layers, b, hk, _ = weights.shape
    table = st["table"].long()
    for layer in range(layers):
        for r in range(b):
            left = min(lens[r], case["budget"])
            for j in range(hk):
                w, p = st["weights"][layer, r, j, :lens[r]].cpu(), st["positions"][layer, r, j, :lens[r]].cpu()
                recent = p >= int(st["seen"][r]) - case["recent"]
                a, c = recent.nonzero()[:, 0], (~recent).nonzero()[:, 0]
                a = a[torch.sort(w[a], descending=True, stable=True).indices]
                c = c[torch.sort(w[c], descending=True, stable=True).indices]
                keep = torch.cat([a, c])[:left].sort().values
                to = torch.ones(left, dtype=torch.bool)
                to[keep[keep < left]] = False
                dst, src = to.nonzero()[:, 0].cuda(), keep[keep >= left].cuda()
                for pool, was in ((k, st["k"]), (v, st["v"])):
                    pool[layer, table[r, dst // PAGE], dst % PAGE, j] = was[layer, table[r, src // PAGE], src % PAGE, j]
                weights[layer, r, j, dst], positions[layer, r, j, dst] = st["weights"][layer, r, j, src], st["positions"][layer, r, j, src]
    return {"lens": torch.tensor([min(n, case["budget"]) for n in lens], dtype=torch.int32, device="cuda"), "weights": weights, "positions": positions, "k": k, "v": v}
