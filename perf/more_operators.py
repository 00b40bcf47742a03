"""Drafted tokens in a constrained decoder, as measurable cases: a tree of drafted tokens runs through the model in one
step, and the cache keeps the path that the model confirms.

* ``tree``: from each drafted token's parent, which tokens of its tree it attends to, and its depth;
* ``append``: the new tokens' K (rotated by their positions) and V into a paged cache, and their rotated queries;
* ``attend``: attention of the drafted tokens over the cache and over those of their tree that they see;
* ``accept``: the path through the tree that the model's choices follow stays in the cache, the rest is cut off;
* ``top``: the ``k`` best tokens of each row of logits with their log probabilities, what is drafted and confirmed with.

With ``own`` false each operator is computed in its plain form from torch's elementary operations, in 32 bits (the angles of
the rotation in 64).
"""
import math
import random

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    def cached(name, kind, B, chunk, ragged, ctx, heads, kv, dim, page, dtype, **more):
        return dict(name=name, kind=kind, B=B, chunk=chunk, ragged=ragged, ctx=ctx, heads=heads, kv=kv, dim=dim, page=page,
                    dtype=dtype, **more)

    def accept(name, B, chunk, ragged, ctx, layers, kv, dim, page):
        return dict(name=name, kind="accept", B=B, chunk=chunk, ragged=ragged, ctx=ctx, heads=kv, layers=layers, kv=kv, dim=dim,
                    page=page, dtype="bf16")

    def top(name, B, V, pad, dtype, k, masked):
        return dict(name=name, kind="top", B=B, V=V, pad=pad, dtype=dtype, k=k, masked=masked)
    return [
        # one request's small tree: latency
        dict(name="tree-one", kind="tree", B=1, chunk=16, ragged=False),
        # a full batch of large trees of different sizes
        dict(name="tree-batch", kind="tree", B=256, chunk=256, ragged=True),
        # one request's next token, far into a long text: latency, and the angles of far positions
        cached("append-one", "append", 1, 1, False, 100000, 32, 8, 128, 16, "bf16", rot=128, pairs="halves"),
        # trees of a batch: positions by depth, half of a smaller head rotated, in adjacent pairs
        cached("append-tree", "append", 32, 33, True, 8192, 16, 2, 64, 32, "fp16", rot=32, pairs="adjacent"),
        # the prompt parts of a batch
        cached("append-prompt", "append", 8, 1024, True, 4096, 32, 8, 128, 16, "bf16", rot=128, pairs="halves"),
        # one request's tree over a short text: latency
        cached("attend-one", "attend", 1, 16, False, 700, 32, 8, 128, 16, "bf16", mask="tree"),
        # a batch's trees over long texts, idle rows among them: the cache is read once
        cached("attend-step", "attend", 32, 32, True, 8192, 32, 8, 128, 16, "bf16", mask="tree"),
        # large trees over a few long documents, smaller heads
        cached("attend-large", "attend", 4, 250, True, 60000, 16, 2, 64, 32, "fp16", mask="tree"),
        # one request's path through a few layers: launches
        accept("accept-one", 1, 24, False, 120, 4, 8, 128, 16),
        # a batch's paths
        accept("accept-batch", 128, 64, True, 500, 8, 8, 128, 16),
        # one request over the smallest vocabulary of the configurations: the call's own cost
        top("top-one", 1, 32000, 0, "fp32", 4, False),
        # a full batch of constrained requests over the largest vocabulary
        top("top-batch", 256, 262144, 0, "bf16", 8, True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Sizes over the listed cases' ranges, odd ones among them; every kind, head layout, pairing and type."""
    kind = rng.choice(["tree", "append", "append", "attend", "attend", "attend", "accept", "top", "top"])
    most = [work(c) for c in listed() if c["kind"] == kind]
    while True:
        case = _draw(rng, kind)
        w = work(case)
        if all(w[x] <= max(m[x] for m in most) for x in w):
            return case


def _draw(rng, kind):
    if kind == "top":
        V = _log(rng, 32000, 262144)
        return dict(kind=kind, B=_log(rng, 1, 256), V=V if rng.random() < 0.6 else V // 64 * 64, pad=rng.choice([0, 0, 1, 6, 8]),
                    dtype=rng.choice(["bf16", "fp32"]), k=rng.choice([1, _log(rng, 2, 64)]), masked=rng.random() < 0.6)
    B, chunk, ragged = _log(rng, 1, 256), _log(rng, 1, 256), rng.random() < 0.7
    if kind == "tree":
        return dict(kind=kind, B=B, chunk=_log(rng, 4, 256), ragged=ragged)
    heads, kv = rng.choice([(32, 8), (16, 2), (8, 8), (12, 4), (24, 8), (16, 1), (7, 7)])
    dim, page = rng.choice([64, 96, 128, 128]), rng.choice([8, 16, 32, 64])
    case = dict(kind=kind, B=B, chunk=chunk, ragged=ragged, heads=heads, kv=kv, dim=dim, page=page,
                dtype=rng.choice(["bf16", "bf16", "fp16"]))
    if kind == "accept":
        return dict(case, B=_log(rng, 1, 128), chunk=_log(rng, 1, 64), ctx=_log(rng, 64, 500), heads=min(kv, 8), kv=min(kv, 8),
                    layers=rng.randint(1, 8), page=rng.choice([8, 16]))
    case["ctx"] = max(chunk, _log(rng, 16, 100000))
    if kind == "append":
        if rng.random() < 0.3:
            case["chunk"] = _log(rng, 1, 1024)
            case["ctx"] = max(case["ctx"], case["chunk"])
        return dict(case, rot=rng.choice([dim, dim, dim // 2, 24]), pairs=rng.choice(["halves", "adjacent"]))
    return dict(case, mask=rng.choice(["tree", "tree", "any"]))


# -------------------------------------------------------------------- sizes ---

def _up(a, b):
    return -(-a // b)


def _random(case):
    return random.Random(" ".join("%s=%s" % x for x in sorted(case.items()) if x[0] not in ("name", "kind", "dtype")))


def _rows(case):
    """(new tokens, tokens in the cache with them) of each sequence: by the case alone."""
    r, B, chunk, ctx = _random(case), case["B"], case["chunk"], case.get("ctx", case["chunk"])
    if not case["ragged"]:
        return [chunk] * B, [ctx] * B
    n = [chunk if chunk == 1 else r.choice([1, r.randint(0, chunk), r.randint(1, chunk), chunk]) for _ in range(B)]
    n[r.randrange(B)] = chunk
    return n, [max(x, r.randint(_up(ctx, 4), ctx)) for x in n]


DEEPEST = 10  # tokens after a tree's root on any path


def _forests(case, seed):
    """Parents and depths of each row's tokens, the shapes by the seed: any token, or none, is followed, the first ones most."""
    r = random.Random(seed)
    trees = []
    for n in _rows(case)[0]:
        parents, depth = [], []
        while len(parents) < n:
            p = int((len(parents) + 1) * r.random() ** 1.5) - 1
            if p < 0 or depth[p] < DEEPEST:
                parents.append(p)
                depth.append(depth[p] + 1 if p >= 0 else 0)
        trees.append((parents, depth))
    return trees


def _trees(case):
    """Each row's tree, by the case alone: the parents and depths of its tokens.  The root is the last chosen token, its
    children the best candidates for the next one; the likelier a token, the lower its number, and the more follow it."""
    r = _random(case)
    trees = []
    for n in _rows(case)[0]:
        deepest = max(1, min(DEEPEST, n // 3))
        wide = min(n - 1, deepest + 1 + r.randint(0, _up(n, 8)))
        parents, depth = [-1] * min(n, 1) + [0] * wide, [0] * min(n, 1) + [1] * wide
        # what the root's candidates but the first lead to comes after the places that a path can take (see _paths)
        open_ = [j for j in range(1, n) if j < len(parents) and (j == 1 or j > deepest)]
        while len(parents) < n:
            on = [j for j in open_ if depth[j] < deepest]
            p = on[int(len(on) * r.random() ** 2)] if on else 0
            open_.append(len(parents))
            parents.append(p)
            depth.append(depth[p] + 1)
        trees.append((parents, depth))
    return trees


def _paths(case):
    """The path of each row that the model confirms, by the case alone.  A token that stays moves to the place of
    its depth; the paths are such that no place moved to is one moved from, so that a pass can be repeated."""
    r = _random(case)
    paths = []
    for parents, depth in _trees(case):
        n, deepest = len(parents), max(1, min(DEEPEST, len(parents) // 3))
        path = [0] if n else []
        while path:
            then = [j for j in range(n) if parents[j] == path[-1] and (j == len(path) or j > deepest)]
            if not then or r.random() < 0.2:
                break
            path.append(then[int(len(then) * r.random() ** 2)])
        paths.append(path)
    return paths


def work(case):
    kind, size = case["kind"], 4 if case.get("dtype") == "fp32" else 2
    if kind == "top":
        return {"bytes": case["B"] * (case["V"] * size + 8 * case["k"]), "flops": 3 * case["B"] * case["V"]}
    n, lens = _rows(case)
    if kind == "tree":
        return {"bytes": sum(n) * (8 + 8 * _up(case["chunk"], 64)), "flops": 0}
    line = case["kv"] * case["dim"] * size  # one token's K or V
    if kind == "append":
        q = case["heads"] * case["dim"] * size
        return {"bytes": sum(n) * (2 * q + 4 * line + 4), "flops": 3 * sum(n) * (case["heads"] + case["kv"]) * case["rot"]}
    if kind == "attend":
        seen = sum(x * (length - x) for x, length in zip(n, lens)) + (
            sum(1 + d for _, depth in _trees(case) for d in depth) if case["mask"] == "tree" else sum(x * x for x in n) // 2)
        rows = sum(n) * case["heads"]
        return {"bytes": 2 * line * sum(length for x, length in zip(n, lens) if x) + rows * (2 * case["dim"] * size + 4) +
                8 * sum(n) * _up(case["chunk"], 64), "flops": 4 * case["dim"] * case["heads"] * seen}
    moved = sum(j != d for path in _paths(case) for d, j in enumerate(path))
    return {"bytes": 2 * moved * 2 * case["layers"] * line + 16 * sum(n), "flops": 0}


# ------------------------------------------------------------------- inputs ---

def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _pool(case, planes, pages, g):
    data = torch.empty((planes, pages, case["kv"], case["page"], case["dim"]), device="cuda", dtype=DTYPES[case["dtype"]])
    for plane in data:
        plane.copy_(torch.randn(plane.shape, generator=g, device="cuda"))
    return data


def _prepare_top(case, seed, g):
    B, V = case["B"], case["V"]
    kw = dict(generator=g, device="cuda")
    x = torch.randn((B, V + case["pad"]), **kw) * 3
    if case["masked"]:  # as a grammar leaves them: from one valid token to all, and a dead row now and then
        share = torch.exp(torch.rand((B, 1), **kw) * math.log(V)) / V
        x = torch.where(torch.rand((B, V + case["pad"]), **kw) < share, x, -math.inf)
        x[B // 2: B // 2 + B // 64] = -math.inf
    return {"logits": x.to(DTYPES[case["dtype"]])[:, :V], "k": case["k"]}


def _prepare_tree(case, seed, g):
    trees = _forests(case, seed)
    n = [len(p) for p, _ in trees]
    return {"offsets": _ints([sum(n[:i]) for i in range(len(n) + 1)]), "parents": _ints([p for up, _ in trees for p in up]),
            "longest": max(n), "deepest": max(d for _, depth in trees for d in depth + [0])}


def _tables(case, spare, g):
    """The sequences' pages, which lie in any order, and ``spare`` free ones."""
    n, lens = _rows(case)
    page = case["page"]
    width = max(_up(x, page) for x in lens) + 1
    held = torch.tensor([_up(x, page) for x in lens], device="cuda")
    pages = sum(_up(x, page) for x in lens) + spare
    ids = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    at = torch.arange(width, device="cuda")
    first = (held.cumsum(0) - held)[:, None]
    table = torch.where(at < held[:, None], ids[(first + at).clamp_(max=pages - 1)], -1).contiguous()
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    refs[table[table >= 0].long()] = 1
    s = {"table": table, "length": _ints(lens), "refs": refs, "longest": max(n), "offsets": None}
    if case["chunk"] > 1 or case["ragged"]:
        s["offsets"] = _ints([sum(n[:i]) for i in range(len(n) + 1)])
    return s, pages, n


def _prepare_chunks(case, seed, g):
    s, pages, n = _tables(case, 0, g)
    heads, kv, dim = case["heads"], case["kv"], case["dim"]
    # q, k and v as a projection leaves them: side by side in one row per token
    qkv = torch.randn((sum(n), (heads + 2 * kv) * dim), generator=g, device="cuda").to(DTYPES[case["dtype"]])
    q, k, v = qkv.split([heads * dim, kv * dim, kv * dim], 1)
    s["q"], s["k"], s["v"] = q.unflatten(1, (heads, dim)), k.unflatten(1, (kv, dim)), v.unflatten(1, (kv, dim))
    s["data"] = _pool(case, 2, pages, g)
    trees = _trees(case) if case["kind"] == "attend" or case["chunk"] <= 256 else None
    if case["kind"] == "append":
        s["adjacent"] = case["pairs"] == "adjacent"
        s["frequencies"] = (500000.0 ** -(torch.arange(0, case["rot"], 2, device="cuda").double() / case["rot"])).float()
        s["depth"] = None if trees is None or s["offsets"] is None else _ints([d for _, depth in trees for d in depth])
        return s
    s["scale"] = dim ** -0.5
    parents = _ints([p for parents, _ in trees for p in parents])
    deepest = max(d for _, depth in trees for d in depth + [0])
    offsets = s["offsets"] if s["offsets"] is not None else torch.arange(case["B"] + 1, dtype=torch.int32, device="cuda")
    s["seen"] = _plain_tree(dict(parents=parents, offsets=offsets, longest=s["longest"], deepest=deepest))["seen"]
    if case["mask"] == "any":  # any mask over the row's own tokens; some see none of them
        bits = torch.randint(-2 ** 62, 2 ** 62, s["seen"].shape, generator=g, device="cuda") * 2
        s["seen"] = torch.where(torch.rand((s["seen"].shape[0], 1), generator=g, device="cuda") < 0.1, 0, bits)
    return s


def _prepare_accept(case, seed, g):
    s, pages, n = _tables(case, case["B"], g)
    r = random.Random(seed)
    tokens, picks, parents = [], [], []
    for (up, _), path in zip(_trees(case), _paths(case)):
        # even tokens, so that an odd choice ends a path
        row = [2 * t for t in r.sample(range(16000), len(up))]
        choice = [2 * r.randrange(16000) + 1 for _ in up]
        for a, b in zip(path, path[1:]):
            choice[a] = row[b]
        for j, p in enumerate(up):  # choices off the path follow their trees too
            if j and p not in path and r.random() < 0.5:
                choice[p] = row[j]
        tokens, picks, parents = tokens + row, picks + choice, parents + up
    s["tokens"], s["picks"], s["parents"] = _ints(tokens), _ints(picks), _ints(parents)
    s["deepest"] = max(len(p) for p in _paths(case))
    for name in ("table", "length", "refs"):
        s[name + "0"] = s[name].clone()
    s["data"] = _pool(case, 2 * case["layers"], pages, g)
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind = case["kind"]
    made = {"top": _prepare_top, "tree": _prepare_tree, "append": _prepare_chunks, "attend": _prepare_chunks,
            "accept": _prepare_accept}[kind](case, seed, g)
    made["kind"] = kind
    if own and "data" in made:  # the framework's cache over the pool and its tables
        import paper_2608_12574_amd as tam
        made["cache"] = tam.PageCache(made["data"], made["table"], made["length"], made["refs"])
    return made


# -------------------------------------------------------------------- passes ---

def run(s):
    return (_own if own else _plain)[s["kind"]](s)


def _own_top(s):
    import paper_2608_12574_amd as tam
    tokens, logprobs, lse = tam.top_tokens(s["logits"], s["k"], return_lse=True)
    return {"tokens": tokens, "logprobs": logprobs, "lse": lse}


def _own_tree(s):
    import paper_2608_12574_amd as tam
    seen, depth = tam.tree_masks(s["parents"], s["offsets"], longest=s["longest"])
    return {"seen": seen, "depth": depth}


def _own_append(s):
    q = s["cache"].append(0, s["q"], s["k"], s["v"], s["frequencies"], offsets=s["offsets"], longest=s["longest"],
                          depth=s["depth"], adjacent=s["adjacent"])
    return {"q": q, "data": s["data"]}


def _own_attend(s):
    out, lse = s["cache"].attend(0, s["q"], offsets=s["offsets"], longest=s["longest"], scale=s["scale"], seen=s["seen"],
                                 return_lse=True)
    return {"out": out, "lse": lse}


def _back(s):
    # a step that is tried and taken back: each pass begins with the tree in the cache
    for name in ("table", "length", "refs"):
        s[name].copy_(s[name + "0"])


def _own_accept(s):
    _back(s)
    path, count, last = s["cache"].accept(s["tokens"], s["picks"], s["parents"], offsets=s["offsets"], longest=s["longest"])
    return dict(path=path, count=count, last=last, **{x: s[x] for x in ("data", "table", "length", "refs")})


_own = {"top": _own_top, "tree": _own_tree, "append": _own_append, "attend": _own_attend, "accept": _own_accept}


def _plain_top(s):
    x, k = s["logits"].float(), s["k"]
    top = x.amax(1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    lse = torch.log(torch.exp(x - top).sum(1, keepdim=True)) + top
    y, at = torch.sort(x, dim=1, descending=True, stable=True)  # of equal logits the lower token first
    y, at = y[:, :k], at[:, :k]
    there = y > -math.inf
    return {"tokens": torch.where(there, at, -1).to(torch.int32), "logprobs": torch.where(there, y - lse, -math.inf),
            "lse": lse[:, 0]}


def _where(s):
    """(row, place in its row) of each new token."""
    T = (s["parents"] if "parents" in s else s["q"]).shape[0]
    t = torch.arange(T, device="cuda")
    if s["offsets"] is None:
        return t, torch.zeros_like(t)
    off = s["offsets"].long()
    row = torch.searchsorted(off, t, right=True) - 1
    return row, t - off[row]


def _plain_tree(s):
    parents = s["parents"].long()
    T, words = parents.shape[0], _up(s["longest"], 64)
    row, at = _where(s)
    first = torch.arange(T, device="cuda") - at
    bits = torch.zeros((T, words * 64), dtype=torch.int64, device="cuda")
    depth = torch.zeros(T, dtype=torch.int32, device="cuda")
    of = at
    for _ in range(s["deepest"] + 1):  # of: each token's next ancestor in its row, -1 past the root
        bits.scatter_add_(1, of.clamp(min=0)[:, None], (of >= 0).long()[:, None])
        of = torch.where(of >= 0, parents[(first + of).clamp(min=0)], -1)
        depth += of >= 0
    return {"seen": (bits.view(T, words, 64) << torch.arange(64, device="cuda")).sum(2), "depth": depth}


def _positions(s):
    row, at = _where(s)
    length = s["length"].long()[row]
    n = 1 if s["offsets"] is None else (s["offsets"][1:] - s["offsets"][:-1]).long()[row]
    return row, length - n, length - n + at  # rows, where they begin, the tokens' places


def _plain_append(s):
    row, begin, place = _positions(s)
    position = place if s["depth"] is None else begin + s["depth"]
    angle = position.double()[:, None] * s["frequencies"].double()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    rot = 2 * s["frequencies"].shape[0]

    def rotate(x):
        y = x.float()
        if s["adjacent"]:
            a, b = y[..., 0:rot:2], y[..., 1:rot:2]
            turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        else:
            a, b = y[..., :rot // 2], y[..., rot // 2:rot]
            turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        return torch.cat([turned, y[..., rot:]], -1).to(x.dtype)
    data, page = s["data"], s["data"].shape[3]
    to = s["table"][row, place // page].long()
    data[0][to, :, place % page] = rotate(s["k"])
    data[1][to, :, place % page] = s["v"]
    return {"q": rotate(s["q"]), "data": data}


def _plain_attend(s):
    q, data, table = s["q"], s["data"], s["table"]
    T, heads, dim = q.shape
    B, n, kv, page = table.shape[0], s["longest"], data.shape[2], data.shape[3]
    row, begin, place = _positions(s)
    at = place - begin
    pad = torch.zeros((B, n, heads, dim), device="cuda")
    pad[row, at] = q.float()
    k, v = (data[p][table.clamp(min=0).long()].permute(0, 2, 1, 3, 4).reshape(B, kv, -1, dim).float() for p in (0, 1))
    key = torch.arange(k.shape[2], device="cuda")
    # a token sees what lies before its row's new tokens, and those of them that its bits name
    sees = torch.zeros((B, n, k.shape[2]), dtype=torch.bool, device="cuda")
    bits = ((s["seen"][:, :, None] >> torch.arange(64, device="cuda")) & 1).flatten(1) != 0
    count = s["length"].long()[row] - begin
    rel = key - begin[:, None]
    named = bits.gather(1, rel.clamp(0, bits.shape[1] - 1)) & (rel < torch.minimum(count, count.new_tensor(bits.shape[1]))[:, None])
    sees[row, at] = torch.where(rel < 0, True, named)
    x = torch.matmul(pad.view(B, n, kv, heads // kv, dim).permute(0, 2, 1, 3, 4).reshape(B, kv, -1, dim),
                     k.transpose(2, 3).contiguous()) * s["scale"]
    x = torch.where(sees.repeat_interleave(heads // kv, 1)[:, None], x, -math.inf)
    top = x.amax(3, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    p = torch.exp(x - top)
    total = p.sum(3, keepdim=True)
    out = torch.matmul(p, v) / total.clamp(min=torch.finfo(torch.float32).tiny)
    lse = (torch.log(total) + top)[..., 0]
    lse = torch.where(total[..., 0] > 0, lse, -math.inf)
    out = out.view(B, kv, n, heads // kv, dim).transpose(1, 2).reshape(B, n, heads, dim)[row, at]
    lse = lse.view(B, kv, n, heads // kv).transpose(1, 2).reshape(B, n, heads)[row, at]
    return {"out": out.to(q.dtype), "lse": lse}


def _plain_accept(s):
    _back(s)
    data, table, length, refs = s["data"], s["table"], s["length"], s["refs"]
    tokens, picks, parents, page = s["tokens"], s["picks"], s["parents"].long(), data.shape[3]
    T, B, most = tokens.shape[0], table.shape[0], s["longest"]
    off = s["offsets"].long() if s["offsets"] is not None else torch.arange(B + 1, device="cuda")
    n = off[1:] - off[:-1]
    at = torch.arange(most, device="cuda")
    t = (off[:-1, None] + at).clamp(max=T - 1)  # the rows' tokens, side by side
    inside = at < n[:, None]
    here = torch.where(n > 0, 0, -1)  # the last token that stays
    count = (n > 0).int()
    last = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    path = torch.full((B, most), -1, dtype=torch.int64, device="cuda")
    path[:, 0] = here
    i = torch.arange(B, device="cuda")
    for d in range(1, s["deepest"] + 1):
        want = picks[(off[:-1] + here.clamp(min=0)).clamp(max=T - 1)]
        last = torch.where(here >= 0, want, last)
        fits = inside & (parents[t] == here[:, None]) & (here >= 0)[:, None] & (tokens[t] == want[:, None])
        then = torch.where(fits, at, most).amin(1)
        here = torch.where(then < most, then, -1)
        if d < most:
            path[:, d] = here
        count += here >= 0
    begin = length.long() - n
    # all moves at once, from what was there; a place past the path takes what it has
    src = torch.where(path >= 0, path, at) + begin[:, None]
    dst = at + begin[:, None]
    on = inside.nonzero(as_tuple=True)
    src, dst, row = src[on], dst[on], i[:, None].expand(-1, most)[on]
    data[:, table[row, dst // page].long(), :, dst % page] = data[:, table[row, src // page].long(), :, src % page]
    held = (length.long() + page - 1) // page
    keep = (begin + count + page - 1) // page
    col = torch.arange(table.shape[1], device="cuda")
    gone = (col >= keep[:, None]) & (col < held[:, None])
    refs.index_add_(0, table.clamp(min=0).flatten().long(), -gone.flatten().int())
    table.copy_(torch.where(col >= keep[:, None], -1, table))
    length.copy_(begin + count)
    flat = torch.where(at < count[:, None], path, -1)[on].to(torch.int32)
    return dict(path=flat, count=count, last=last, data=data, table=table, length=length, refs=refs)


_plain = {"top": _plain_top, "tree": _plain_tree, "append": _plain_append, "attend": _plain_attend, "accept": _plain_accept}


# --------------------------------------------------------------------- exact ---

def exact(case, seed):
    """From the definitions, sequence by sequence, in 64 bits."""
    s = prepare(case, seed)
    return {"top": _exact_top, "tree": _exact_tree, "append": _exact_append, "attend": _exact_attend,
            "accept": _exact_accept}[case["kind"]](case, s)


def _exact_top(case, s):
    x = s["logits"].double()
    lse = torch.logsumexp(x, 1)
    tokens = torch.full((x.shape[0], case["k"]), -1, dtype=torch.int32)
    logprobs = torch.full((x.shape[0], case["k"]), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(x.shape[0]):
        # every logit from the k-th largest up, in the order of the tokens
        low = x[b].topk(case["k"]).values[-1]
        ids = ((x[b] >= low) & (x[b] > -math.inf)).nonzero().flatten()
        best = sorted(zip((-x[b, ids]).tolist(), ids.tolist()))[:case["k"]]
        for i, (y, v) in enumerate(best):
            tokens[b, i] = v
            logprobs[b, i] = -y - lse[b]
    return {"tokens": tokens.cuda(), "logprobs": logprobs, "lse": lse}


def _exact_tree(case, s):
    off, parents = s["offsets"].tolist(), s["parents"].tolist()
    words = _up(s["longest"], 64)
    seen, depth = [], []
    for a, b in zip(off, off[1:]):
        of = []
        for j, p in enumerate(parents[a:b]):
            of.append((of[p] if p >= 0 else 0) | 1 << j)
            depth.append(bin(of[-1]).count("1") - 1)
        for x in of:
            row = [x >> 64 * w & (1 << 64) - 1 for w in range(words)]
            seen.append([w - (1 << 64) if w >> 63 else w for w in row])
    return {"seen": torch.tensor(seen, dtype=torch.int64, device="cuda").view(-1, words), "depth": _ints(depth)}


def _exact_append(case, s):
    n, lens = _rows(case)
    page, half = case["page"], case["rot"] // 2
    q, k, data = s["q"].double(), s["k"].double(), s["data"].double()
    depth = None if s["depth"] is None else s["depth"].tolist()
    table = s["table"].tolist()
    t, angle, to = 0, [], []
    for b, x in enumerate(n):
        for j in range(x):
            p = lens[b] - x + j
            to.append((table[b][p // page], p % page))
            angle.append(lens[b] - x + (j if depth is None else depth[t]))
            t += 1
    turn = torch.polar(torch.ones((t, half), dtype=torch.float64, device="cuda"),
                       torch.tensor(angle, dtype=torch.float64, device="cuda")[:, None] * s["frequencies"].double())[:, None]
    for x in (q, k):
        first, second = ((slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if s["adjacent"] else
                         (slice(0, half), slice(half, 2 * half)))
        z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
        x[..., first], x[..., second] = z.real, z.imag
    pages, places = (torch.tensor(x, device="cuda") for x in zip(*to))
    data[0][pages, :, places] = k
    data[1][pages, :, places] = s["v"].double()
    return {"q": q, "data": data}


def _exact_attend(case, s):
    n, lens = _rows(case)
    group, dim = case["heads"] // case["kv"], case["dim"]
    if sum(x * length for x, length in zip(n, lens)) * case["heads"] * dim > 2 ** 39:
        return None
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    t = 0
    for b, (x, length) in enumerate(zip(n, lens)):
        if not x:
            continue
        ids = s["table"][b, :_up(length, case["page"])].long()
        k, v = (s["data"][p][ids].transpose(0, 1).reshape(case["kv"], -1, dim)[:, :length].double() for p in (0, 1))
        hidden = torch.zeros((x, length), dtype=torch.bool, device="cuda")
        for j in range(x):
            word = s["seen"][t:t + x, j // 64]
            hidden[:, length - x + j] = (word >> j % 64) & 1 == 0
        for h in range(case["heads"]):
            score = s["q"][t:t + x, h].double() @ k[h // group].T * s["scale"]
            score[hidden] = -math.inf
            sums = torch.logsumexp(score, 1)
            lse[t:t + x, h] = sums
            out[t:t + x, h] = torch.exp(score - sums.clamp(min=-1e300)[:, None]) @ v[h // group]
        t += x
    return {"out": out, "lse": lse}


def _exact_accept(case, s):
    table, length, refs, page = s["table"].tolist(), s["length"].tolist(), s["refs"].tolist(), case["page"]
    off = s["offsets"].tolist() if s["offsets"] is not None else list(range(case["B"] + 1))
    tokens, picks, parents = (s[x].tolist() for x in ("tokens", "picks", "parents"))
    paths, count, last = [], [], []
    was = s["data"].clone()
    for b, (a, z) in enumerate(zip(off, off[1:])):
        path = [0] if z > a else []
        while path:
            then = [j for j in range(z - a) if parents[a + j] == path[-1] and tokens[a + j] == picks[a + path[-1]]]
            if not then:
                break
            path.append(then[0])
        begin = length[b] - (z - a)
        for d, j in enumerate(path):
            to, of = begin + d, begin + j
            if j != d:
                s["data"][:, table[b][to // page], :, to % page] = was[:, table[b][of // page], :, of % page]
        for x in range(_up(begin + len(path), page), len(table[b])):
            if table[b][x] >= 0:
                refs[table[b][x]] -= 1
                table[b][x] = -1
        length[b] = begin + len(path)
        paths += path + [-1] * (z - a - len(path))
        count.append(len(path))
        last.append(picks[a + path[-1]] if path else -1)
    return dict(path=_ints(paths), count=_ints(count), last=_ints(last), data=s["data"], table=_ints(table),
                length=_ints(length), refs=_ints(refs))
