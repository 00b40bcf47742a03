"""The operators beside the token mask, as measurable cases: what one step of a constrained decoder runs
around ``apply_mask`` and ``advance``.

* ``adjust``: penalties for repeated tokens, biases and the grammar's mask on ``[B, V]`` logits, in place;
* ``attend``: attention of a chunk of new tokens per sequence over a paged K/V cache;
* ``store``: the new tokens' K and V into their pages;
* ``beam``: one step of beams over the cache: fork from the surviving parents, room for the next tokens
  (shared last pages are copied);
* ``compact``: the used pages of a fragmented pool moved to its front.

With ``own`` false each operator is computed in its plain form from torch's elementary operations, in 32 bits.
"""
import math
import random

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    def adjust(name, B, V, pad, dtype, history, biases, masked):
        return dict(name=name, kind="adjust", B=B, V=V, pad=pad, dtype=dtype, history=history, biases=biases,
                    masked=masked)

    def attend(name, B, chunk, ragged, ctx, heads, kv, dim, page, dtype):
        return dict(name=name, kind="attend", B=B, chunk=chunk, ragged=ragged, ctx=ctx, heads=heads, kv=kv, dim=dim,
                    page=page, dtype=dtype)

    def beam(name, groups, width, ctx, count, layers, kv, dim, page):
        return dict(name=name, kind="beam", groups=groups, width=width, ctx=ctx, count=count, layers=layers, kv=kv,
                    dim=dim, page=page, dtype="bf16")
    return [
        # one request over the smallest vocabulary of the configurations: the call's own cost
        adjust("adjust-one", 1, 32000, 0, "fp32", 64, 8, True),
        # a batch with long histories and no grammar, rows of odd length and stride: only named tokens change
        adjust("adjust-free", 64, 128255, 3, "fp32", 8192, 300, False),
        # a full batch of constrained requests over the largest vocabulary
        adjust("adjust-batch", 256, 262144, 0, "bf16", 2048, 32, True),
        # one sequence's next token: latency
        attend("attend-one", 1, 1, False, 700, 32, 8, 128, 16, "bf16"),
        # the decode step of a batch: the cache is read once
        attend("attend-step", 64, 1, True, 8192, 32, 8, 128, 16, "bf16"),
        # two long documents, a forced run of a few tokens each: few rows, a long axis
        attend("attend-long", 2, 5, True, 131072, 16, 2, 128, 64, "bf16"),
        # a mixed batch: short chunks, single tokens and idle rows, smaller heads
        attend("attend-ragged", 24, 96, True, 3000, 16, 2, 64, 32, "fp16"),
        # one part of a long prompt, behind what is cached already
        attend("attend-prompt", 1, 4096, False, 16384, 32, 8, 128, 16, "bf16"),
        # the K and V of a batch of prompt parts
        dict(name="store-prompt", kind="store", B=8, chunk=1024, ragged=True, ctx=4096, heads=32, kv=8, dim=128,
             page=16, dtype="bf16"),
        # four beams of one request: launches
        beam("beam-one", 1, 4, 100, 1, 4, 8, 128, 16),
        # 32 requests of eight beams, half of the beams survive
        beam("beam-batch", 32, 8, 500, 1, 8, 8, 128, 16),
        # a pool of which half is free
        dict(name="compact-half", kind="compact", pages=2048, used=1024, slots=128, layers=8, kv=8, dim=128, page=16,
             dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Sizes over the listed cases' ranges, odd ones among them; every kind, head layout and type."""
    kind = rng.choice(["adjust", "adjust", "attend", "attend", "attend", "store", "beam", "compact"])
    if kind == "adjust":
        V = _log(rng, 32000, 262144)
        return dict(kind=kind, B=_log(rng, 1, 256), V=V if rng.random() < 0.6 else V // 64 * 64,
                    pad=rng.choice([0, 0, 1, 6, 8]), dtype=rng.choice(["bf16", "fp32"]), history=_log(rng, 16, 8192),
                    biases=rng.choice([0, 8, _log(rng, 1, 300)]), masked=rng.random() < 0.7)
    heads, kv = rng.choice([(32, 8), (16, 2), (8, 8), (12, 4), (24, 8), (16, 1), (7, 7)])
    dim, page = rng.choice([64, 96, 128, 128]), rng.choice([8, 16, 32, 64])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    if kind in ("attend", "store"):
        while True:
            B, chunk, ctx = _log(rng, 1, 64), rng.choice([1, _log(rng, 1, 64), _log(rng, 1, 4096)]), _log(rng, 16, 131072)
            if chunk > ctx or B * ctx * kv > 64 * 8192 * 8 or B * chunk * max(ctx * heads, 16384 * 8) > 4096 * 16384 * 32:
                continue
            if kind == "store" and B * chunk > 8192:
                continue
            return dict(kind=kind, B=B, chunk=chunk, ragged=rng.random() < 0.7, ctx=ctx, heads=heads, kv=kv, dim=dim,
                        page=page, dtype=dtype)
    if kind == "beam":
        width = rng.randint(2, 8)
        return dict(kind=kind, groups=_log(rng, 1, 256 // width), width=width, ctx=_log(rng, 10, 500),
                    count=rng.choice([1, 1, rng.randint(2, 20)]), layers=rng.randint(1, 8), kv=min(kv, 8), dim=dim,
                    page=rng.choice([8, 16]), dtype=dtype)
    pages = _log(rng, 32, 2048)
    used = rng.randint(1, pages)
    return dict(kind=kind, pages=pages, used=used, slots=rng.randint(1, min(128, used)), layers=rng.randint(1, 8),
                kv=min(kv, 8), dim=dim, page=rng.choice([8, 16]), dtype=dtype)


# -------------------------------------------------------------------- sizes ---

def _up(a, b):
    return -(-a // b)


def _rows(case):
    """(tokens in the chunk, tokens in the cache with them) of each sequence: by the case alone."""
    r = random.Random("%(B)d %(chunk)d %(ctx)d %(heads)d %(page)d" % case)
    B, chunk, ctx = case["B"], case["chunk"], case["ctx"]
    if not case["ragged"]:
        return [chunk] * B, [ctx] * B
    n = [chunk if chunk == 1 else r.choice([1, r.randint(0, chunk), r.randint(1, chunk)]) for _ in range(B)]
    n[r.randrange(B)] = chunk
    return n, [max(x, r.randint(_up(ctx, 4), ctx)) for x in n]


def _beams(case):
    """(prompt tokens, tokens so far) of each group: by the case alone."""
    r = random.Random("%(groups)d %(width)d %(ctx)d" % case)
    lens = []
    for _ in range(case["groups"]):
        prompt = r.randint(_up(case["ctx"], 2), case["ctx"])
        lens.append((prompt, prompt + r.randint(0, 2 * case["page"])))
    return lens


def work(case):
    kind, size = case["kind"], 4 if case["dtype"] == "fp32" else 2
    if kind == "adjust":
        B, V, named = case["B"], case["V"], case["history"] // 2 + case["biases"]
        touched = min(V, named) * (0.1 if case["masked"] else 1.0)
        return {"bytes": B * ((V / 8 + V * size * 0.85 if case["masked"] else 0) + 2 * case["history"] + 8 * case["biases"]
                              + 2 * touched * size), "flops": B * 6 * touched}
    line = case["kv"] * case["dim"] * size  # one token's K or V
    if kind in ("attend", "store"):
        n, lens = _rows(case)
        if kind == "store":
            return {"bytes": 4 * line * sum(n), "flops": 0}
        pairs = sum(x * (length - x) + x * (x + 1) // 2 for x, length in zip(n, lens))
        rows = sum(n) * case["heads"]
        return {"bytes": 2 * line * sum(length for x, length in zip(n, lens) if x) + rows * (2 * case["dim"] * size + 4),
                "flops": 4 * case["dim"] * case["heads"] * pairs}
    page = 2 * case["layers"] * line * case["page"]
    if kind == "beam":
        lens, w = _beams(case), case["width"]
        copies = sum(w - max(1, w // 2) for _, length in lens if length % case["page"])
        table = sum(w * _up(length + case["count"], case["page"]) for _, length in lens)
        return {"bytes": 2 * copies * page + 16 * table, "flops": 0}
    moved = case["used"] * (case["pages"] - case["used"]) / case["pages"]
    return {"bytes": 2 * moved * page + 8 * (case["pages"] + case["used"]), "flops": 0}


# ------------------------------------------------------------------- inputs ---

def _pool(case, planes, pages, g):
    data = torch.empty((planes, pages, case["kv"], case["page"], case["dim"]), device="cuda",
                       dtype=DTYPES[case["dtype"]])
    for plane in data:
        plane.copy_(torch.randn(plane.shape, generator=g, device="cuda"))
    return data


def _counts(table, pages):
    flat = torch.bincount(table.reshape(-1).long() + 1, minlength=pages + 1)
    return flat[1:].to(torch.int32).contiguous()


def _prepare_adjust(case, seed, g):
    B, V, L, nb = case["B"], case["V"], case["history"], case["biases"]
    kw = dict(generator=g, device="cuda")
    s = {"logits": (torch.randn((B, V + case["pad"]), **kw) * 3).to(DTYPES[case["dtype"]])[:, :V]}
    # text repeats its frequent tokens: ids skewed to one end, then spread over the vocabulary
    ids = (torch.rand((B, L), **kw) ** 4 * V).long().clamp_(max=V - 1)
    s["tokens"] = (ids * 7919 % V).to(torch.int32)
    s["length"] = torch.randint(L // 2, L + 1, (B,), dtype=torch.int32, **kw)
    s["prompt"] = (s["length"] * torch.rand(B, **kw)).to(torch.int32)
    s["repetition"] = 1 + 0.3 * torch.rand(B, **kw)
    s["frequency"] = 0.5 * torch.rand(B, **kw)
    s["presence"] = 0.5 * torch.rand(B, **kw)
    s["bias_ids"] = s["bias"] = s["rows"] = s["row_ids"] = None
    if nb:  # a token may be named twice (the later entry stands); -1 fills shorter lists
        s["bias_ids"] = torch.randint(-1, V, (B, nb), dtype=torch.int32, **kw)
        s["bias_ids"][:, : nb // 4] = s["tokens"][:, : nb // 4] if L >= nb // 4 else -1
        s["bias"] = 4 * torch.randn((B, nb), **kw)
    if case["masked"]:  # from one valid token to all of them, as by depth in a trie, and a dead row now and then
        R, W = B, _up(V, 64)
        share = torch.exp(torch.rand((R, 1), **kw) * math.log(V)) / V
        bits = torch.rand((R, W * 64), **kw) < share
        bits[:, V:] = False
        bits[: R // 16, :V] = True
        s["rows"] = (bits.view(R, W, 64).long() << torch.arange(64, device="cuda")).sum(2)
        s["row_ids"] = torch.randint(0, R, (B,), dtype=torch.int32, **kw)
        s["row_ids"][B // 2: B // 2 + B // 64] = -1
    return s


def _prepare_chunks(case, seed, g):
    n, lens = _rows(case)
    B, page, kv, dim, heads = case["B"], case["page"], case["kv"], case["dim"], case["heads"]
    width = max(_up(x, page) for x in lens)
    held = torch.tensor([_up(x, page) for x in lens], device="cuda")
    pages = sum(_up(x, page) for x in lens)
    ids = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)  # pages lie in any order
    at = torch.arange(width, device="cuda")
    first = (held.cumsum(0) - held)[:, None]
    table = torch.where(at < held[:, None], ids[(first + at).clamp_(max=pages - 1)], -1).contiguous()
    s = {"table": table, "length": torch.tensor(lens, dtype=torch.int32, device="cuda"),
         "refs": torch.ones(pages, dtype=torch.int32, device="cuda"), "longest": max(n), "scale": dim ** -0.5,
         "offsets": None}
    if case["chunk"] > 1:
        s["offsets"] = torch.tensor([sum(n[:i]) for i in range(B + 1)], dtype=torch.int32, device="cuda")
    # q, k and v as a projection leaves them: side by side in one row per token
    qkv = torch.randn((sum(n), (heads + 2 * kv) * dim), generator=g, device="cuda").to(DTYPES[case["dtype"]])
    q, k, v = qkv.split([heads * dim, kv * dim, kv * dim], 1)
    s["q"], s["k"], s["v"] = q.unflatten(1, (heads, dim)), k.unflatten(1, (kv, dim)), v.unflatten(1, (kv, dim))
    s["data"] = _pool(case, 2, pages, g)
    return s


def _prepare_beam(case, seed, g):
    lens, w, page = _beams(case), case["width"], case["page"]
    n = case["groups"] * w
    width = max(_up(b + case["count"], page) for _, b in lens) + 1
    rows, used = [], 0
    for prompt, length in lens:  # the prompt's whole pages are shared, what follows is each beam's own
        shared, own_ = prompt // page, _up(length, page) - prompt // page
        for b in range(w):
            at = used + shared + b * own_
            rows.append([*range(used, used + shared), *range(at, at + own_)] + [-1] * (width - shared - own_))
        used += shared + w * own_
    pages = used + 2 * n + n * _up(case["count"], page)
    ids = torch.cat([torch.randperm(pages, generator=g, device="cuda").to(torch.int32),
                     torch.full((1,), -1, dtype=torch.int32, device="cuda")])
    table = ids[torch.tensor(rows, device="cuda")].contiguous()
    r = random.Random(seed)
    parents = []
    for j in range(case["groups"]):
        alive = r.sample(range(w), max(1, w // 2))
        of = [j * w + alive[b % len(alive)] for b in range(w)]
        r.shuffle(of)
        parents += of
    length = torch.tensor([b for _, b in lens for _ in range(w)], dtype=torch.int32, device="cuda")
    s = {"table": table, "length": length.clone(), "refs": _counts(table, pages), "keep": length,
         "slots": torch.arange(n, dtype=torch.int32, device="cuda"),
         "parents": torch.tensor(parents, dtype=torch.int32, device="cuda"),
         "counts": torch.full((n,), case["count"], dtype=torch.int32, device="cuda"), "most": case["count"]}
    s["data"] = _pool(case, 2 * case["layers"], pages, g)
    return s


def _prepare_compact(case, seed, g):
    P, U, S, page = case["pages"], case["used"], case["slots"], case["page"]
    held = [U // S + (i < U % S) for i in range(S)]
    width = max(held) + 1
    rows, at = [], 0
    for h in held:
        rows.append([*range(at, at + h)] + [-1] * (width - h))
        at += h
    ids = torch.randperm(P, generator=g, device="cuda").to(torch.int32)
    ids[U:] = -1
    ids = torch.cat([ids[:U], torch.full((1,), -1, dtype=torch.int32, device="cuda")])
    table = ids[torch.tensor(rows, device="cuda")].contiguous()
    r = random.Random(seed)
    length = torch.tensor([h * page - r.randrange(page) if h else 0 for h in held], dtype=torch.int32, device="cuda")
    s = {"table": table, "length": length, "refs": _counts(table, P)}
    s["table0"], s["refs0"] = table.clone(), s["refs"].clone()
    s["data"] = _pool(case, 2 * case["layers"], P, g)
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind = case["kind"]
    made = {"adjust": _prepare_adjust, "attend": _prepare_chunks, "store": _prepare_chunks, "beam": _prepare_beam,
            "compact": _prepare_compact}[kind](case, seed, g)
    made["kind"] = kind
    if own and "data" in made:  # the framework's cache over the pool and its tables
        import paper_2608_12574_amd as tam
        made["cache"] = tam.PageCache(made["data"], made["table"], made["length"], made["refs"])
    return made


# -------------------------------------------------------------------- passes ---

def run(s):
    return (_own if own else _plain)[s["kind"]](s)


def _state(s, **more):
    return dict(data=s["data"], table=s["table"], length=s["length"], refs=s["refs"], **more)


def _own_adjust(s):
    import paper_2608_12574_amd as tam
    return tam.adjust_logits(s["logits"], tokens=s["tokens"], length=s["length"], prompt=s["prompt"],
                             repetition=s["repetition"], frequency=s["frequency"], presence=s["presence"],
                             bias_ids=s["bias_ids"], bias=s["bias"], rows=s["rows"], row_ids=s["row_ids"])


def _own_attend(s):
    out, lse = s["cache"].attend(0, s["q"], offsets=s["offsets"], longest=s["longest"], scale=s["scale"],
                                 return_lse=True)
    return {"out": out, "lse": lse}


def _own_store(s):
    s["cache"].store(0, s["k"], s["v"], offsets=s["offsets"], longest=s["longest"])
    return s["data"]


def _own_beam(s):
    # a step that is tried and taken back: each pass forks from the tokens before the last one's
    s["cache"].fork(s["slots"], s["parents"], s["keep"])
    info = s["cache"].extend(s["slots"], s["counts"])
    return _state(s, info=info)


def _own_compact(s):
    s["table"].copy_(s["table0"])
    s["refs"].copy_(s["refs0"])
    info, moved = s["cache"].compact()
    return _state(s, info=info, moved=moved)


_own = {"adjust": _own_adjust, "attend": _own_attend, "store": _own_store, "beam": _own_beam, "compact": _own_compact}


def _plain_adjust(s):
    logits, tokens = s["logits"], s["tokens"].long()
    B, V = logits.shape
    x = logits.float()
    at = torch.arange(tokens.shape[1], device="cuda")
    inside = at < s["length"][:, None]
    output = inside & (at >= s["prompt"][:, None])
    seen = torch.zeros((B, V), dtype=torch.int32, device="cuda").scatter_add_(1, tokens, inside.int()) > 0
    count = torch.zeros((B, V), dtype=torch.float32, device="cuda").scatter_add_(1, tokens, output.float())
    rep = s["repetition"][:, None]
    y = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
    y = y - s["frequency"][:, None] * count
    y = y - torch.where(count > 0, s["presence"][:, None], 0.0)
    if s["bias_ids"] is not None:
        ids = s["bias_ids"].long()
        entry = torch.arange(1, ids.shape[1] + 1, device="cuda").expand_as(ids)
        last = torch.zeros((B, V + 1), dtype=torch.int64, device="cuda")
        last = last.scatter_reduce_(1, torch.where(ids >= 0, ids, V), entry, "amax")[:, :V]
        bias = torch.cat([torch.zeros((B, 1), device="cuda"), s["bias"]], 1)
        y = y + bias.gather(1, last)
    if s["rows"] is not None:
        rows = s["rows"][s["row_ids"].clamp(min=0).long()]
        valid = ((rows[:, :, None] >> torch.arange(64, device="cuda")) & 1).reshape(B, -1)[:, :V] != 0
        valid = valid & (s["row_ids"] >= 0)[:, None]
        y = torch.where(valid, y, -math.inf)
    logits.copy_(y)
    return logits


def _new_tokens(s):
    """(sequence, position) of each new token."""
    T = s["q"].shape[0]
    t = torch.arange(T, device="cuda")
    if s["offsets"] is None:
        return t, s["length"].long() - 1
    off = s["offsets"].long()
    row = torch.searchsorted(off, t, right=True) - 1
    return row, s["length"].long()[row] - (off[row + 1] - off[row]) + t - off[row]


def _plain_attend(s):
    q, data, table = s["q"], s["data"], s["table"]
    T, heads, dim = q.shape
    B, n, kv, page = table.shape[0], s["longest"], data.shape[2], data.shape[3]
    row, pos = _new_tokens(s)
    off = s["offsets"].long()[:B] if s["offsets"] is not None else torch.arange(B, device="cuda")
    at = torch.arange(T, device="cuda") - off[row]  # place in the chunk
    pad = torch.zeros((B, n, heads, dim), device="cuda")
    pad[row, at] = q.float()
    where = torch.full((B, n), -1, device="cuda")
    where[row, at] = pos
    k, v = (data[p][table.clamp(min=0).long()].permute(0, 2, 1, 3, 4).reshape(B, kv, -1, dim).float() for p in (0, 1))
    qq = pad.view(B, n, kv, heads // kv, dim).permute(0, 2, 1, 3, 4).reshape(B, kv, -1, dim)
    x = torch.matmul(qq, k.transpose(2, 3).contiguous()) * s["scale"]
    key = torch.arange(k.shape[2], device="cuda")
    seen = (key <= where[:, :, None]).repeat_interleave(heads // kv, 1)[:, None]
    x = torch.where(seen, x, -math.inf)
    top = x.amax(3, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    p = torch.exp(x - top)
    total = p.sum(3, keepdim=True)
    out = torch.matmul(p, v) / total.clamp(min=torch.finfo(torch.float32).tiny)
    lse = (torch.log(total) + top)[..., 0]
    out = out.view(B, kv, n, heads // kv, dim).transpose(1, 2).reshape(B, n, heads, dim)[row, at]
    lse = lse.view(B, kv, n, heads // kv).transpose(1, 2).reshape(B, n, heads)[row, at]
    return {"out": out.to(q.dtype), "lse": lse}


def _plain_store(s):
    row, pos = _new_tokens(s)
    page = s["data"].shape[3]
    to = s["table"][row, pos // page].long()
    s["data"][0][to, :, pos % page] = s["k"]
    s["data"][1][to, :, pos % page] = s["v"]
    return s["data"]


def _names(table, length, page):
    """Which entries of the table name a page."""
    return torch.arange(table.shape[1], device="cuda") < (length[:, None] + page - 1) // page


def _plain_fork(s):
    table, length, refs, page = s["table"], s["length"], s["refs"], s["data"].shape[3]
    slots, parents = s["slots"].long(), s["parents"].long()
    one = torch.ones((), dtype=torch.int32, device="cuda")
    old, old_len = table[slots], length[slots]
    new_len = torch.minimum(length[parents], s["keep"])
    held = _names(old, new_len, page)
    new = torch.where(held, table[parents], -1)
    refs.index_add_(0, new.clamp(min=0).reshape(-1).long(), (held * one).reshape(-1))
    refs.index_add_(0, old.clamp(min=0).reshape(-1).long(), -(_names(old, old_len, page) * one).reshape(-1))
    table[slots] = new
    length[slots] = new_len


def _plain_extend(s):
    data, table, length, refs = s["data"], s["table"], s["length"], s["refs"]
    page, P, M = data.shape[3], refs.shape[0], table.shape[1]
    slots, c = s["slots"].long(), s["counts"]
    n = slots.shape[0]
    length_, i = length[slots], torch.arange(n, device="cuda")
    have, total = (length_ + page - 1) // page, (length_ + c + page - 1) // page
    last = table[slots, (have - 1).clamp(min=0).long()].clamp(min=0).long()
    part = (length_ % page != 0) & (c > 0)
    sharers = torch.zeros(P, dtype=torch.int32, device="cuda").index_add_(0, last, part.int())
    final = torch.full((P,), -1, device="cuda").scatter_reduce_(0, last, torch.where(part, i, -1), "amax")
    copy = part & ~((refs[last] == sharers[last]) & (final[last] == i))
    need = copy.int() + torch.where(c > 0, total - have, 0)
    ends = need.cumsum(0)
    free = torch.argsort((refs > 0).int(), stable=True)  # the free pages in order, then the others
    nfree, narrow = (refs <= 0).sum(), ((c > 0) & (total > M)).sum()
    done = (ends[-1] <= nfree) & (narrow == 0)
    step = torch.arange(s["most"] // page + 3, device="cuda")
    took = done & (step < need[:, None])
    got = free[((ends - need)[:, None] + step).clamp(max=P - 1)]
    # the pages themselves; a row that copies none writes its own page again
    src = last
    dst = torch.where(copy & done, got[:, 0], src)
    data[:, dst] = data[:, src]
    refs.index_add_(0, src, -(copy & done).int())
    refs.index_add_(0, torch.where(took, got, 0).reshape(-1), took.int().reshape(-1))
    col = torch.arange(M, device="cuda")
    from_ = have - copy.int()
    nth = (col - from_[:, None]).clamp(0, step.shape[0] - 1)
    fresh = done & (col >= from_[:, None]) & (col < (from_ + need)[:, None])
    table[slots] = torch.where(fresh, got.gather(1, nth).int(), table[slots])
    length[slots] = torch.where(done, length_ + c.clamp(min=0), length_)
    return torch.stack([done.int(), ends[-1].int(), nfree.int(), narrow.int()]).int()


def _plain_beam(s):
    _plain_fork(s)
    return _state(s, info=_plain_extend(s))


def _plain_compact(s):
    s["table"].copy_(s["table0"])
    s["refs"].copy_(s["refs0"])
    data, table, refs = s["data"], s["table"], s["refs"]
    P = refs.shape[0]
    used = refs > 0
    ids = torch.arange(P, device="cuda")
    U = used.sum()
    free = torch.argsort(used.int(), stable=True)  # the k-th page to move goes to the k-th free page
    out = used & (ids >= U)
    nth = torch.cumsum(out.int(), 0) - 1
    to = torch.where(out, free[nth.clamp(min=0)], torch.where(used, ids, -1))
    src = torch.argsort((~out).int(), stable=True)[:P // 2 + 1]
    src = torch.where(out[src], src, src[0])  # past the last move, the first one again
    data[:, torch.where(out[src], to[src], src)] = data[:, src]
    moved = to.to(torch.int32)
    keep = _names(table, s["length"], data.shape[3])
    table.copy_(torch.where(keep, moved[table.clamp(min=0).long()], -1))
    refs.copy_(torch.where(ids < U, torch.zeros_like(refs).scatter_add_(0, to.clamp(min=0), refs * used), 0))
    return _state(s, info=torch.stack([U, out.sum()]).int(), moved=moved)


_plain = {"adjust": _plain_adjust, "attend": _plain_attend, "store": _plain_store, "beam": _plain_beam,
          "compact": _plain_compact}


# --------------------------------------------------------------------- exact ---

def exact(case, seed):
    """From the definitions, sequence by sequence, in 64 bits."""
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "adjust":
        return _exact_adjust(s)
    if kind == "attend":
        return _exact_attend(case, s)
    table, length = s["table"].tolist(), s["length"].tolist()
    page = case["page"]
    if kind == "store":
        n, _ = _rows(case)
        t = 0
        for b, x in enumerate(n):
            for j in range(x):
                p = length[b] - x + j
                s["data"][0, table[b][p // page], :, p % page] = s["k"][t]
                s["data"][1, table[b][p // page], :, p % page] = s["v"][t]
                t += 1
        return s["data"]
    refs = s["refs"].tolist()
    if kind == "compact":
        U = sum(r > 0 for r in refs)
        holes = [p for p in range(len(refs)) if p < U and refs[p] == 0]
        moves = dict(zip([p for p in range(len(refs)) if p >= U and refs[p] > 0], holes))
        for a, b in moves.items():
            s["data"][:, b] = s["data"][:, a]
    else:
        old, old_len = [list(r) for r in table], list(length)
        for i, p in enumerate(s["parents"].tolist()):
            length[i] = min(old_len[p], s["keep"].tolist()[i])
            table[i] = [x if j < _up(length[i], page) else -1 for j, x in enumerate(old[p])]
        holders = {}
        for i, row in enumerate(table):
            for x in row:
                if x >= 0:
                    holders.setdefault(x, []).append(i)
        spare = [p for p in range(len(refs)) if p not in holders]
        for i, row in enumerate(table):
            have = _up(length[i], page)
            if length[i] % page and holders[row[have - 1]][-1] != i:
                to = spare.pop(0)
                s["data"][:, to] = s["data"][:, row[have - 1]]
            for _ in range(_up(length[i] + case["count"], page) - have):
                spare.pop(0)
    return dict(data=s["data"], table=None, length=None, refs=None, info=None)


def _exact_adjust(s):
    y = s["logits"].double()
    B, V = y.shape
    for b in range(B):
        length, prompt = int(s["length"][b]), int(s["prompt"][b])
        row = s["tokens"][b].long()
        seen = row[:length].unique()
        x = y[b, seen]
        rep = s["repetition"][b].double()
        y[b, seen] = torch.where(x > 0, x / rep, x * rep)
        ids, count = row[prompt:length].unique(return_counts=True)
        y[b, ids] -= s["frequency"][b].double() * count + s["presence"][b].double()
        if s["bias_ids"] is not None:
            named = dict(zip(s["bias_ids"][b].tolist(), s["bias"][b].tolist()))
            named.pop(-1, None)
            y[b, torch.tensor(list(named), dtype=torch.long, device="cuda")] += torch.tensor(
                list(named.values()), dtype=torch.float64, device="cuda")
        if s["rows"] is not None:
            r = int(s["row_ids"][b])
            word = s["rows"][max(r, 0)].repeat_interleave(64)[:V]
            bit = (word >> (torch.arange(V, device="cuda") % 64)) & 1
            y[b][(bit == 0) | (r < 0)] = -math.inf
    return y


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
        hidden = torch.arange(length, device="cuda") > torch.arange(length - x, length, device="cuda")[:, None]
        for h in range(case["heads"]):
            score = s["q"][t:t + x, h].double() @ k[h // group].T * s["scale"]
            score[hidden] = -math.inf
            lse[t:t + x, h] = torch.logsumexp(score, 1)
            out[t:t + x, h] = torch.exp(score - lse[t:t + x, h, None]) @ v[h // group]
        t += x
    return {"out": out, "lse": lse}
