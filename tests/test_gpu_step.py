"""The decode step's operators beside the mask, against plain implementations in 64 bits.

Tolerances.  u is half a unit in the last place of 1: 2^-8 (bf16), 2^-11 (fp16), 2^-24 (fp32).
* Adjusted logits: three fp32 roundings of values no larger than the largest
  intermediate, then one rounding to the logits' type.
* Attention: the weights p and the output are each rounded once to the type, so with
  A = sum_j p_j |v_j| / sum_j p_j the error is at most u (A + |out|), but for the scores'
  own error e_s <= (D + 8) 2^-24 scale max_j sum_d |q_d k_jd|, which moves each weight by a
  factor exp(2 e_s) at most, the fp32 sums (2^-24 per key), and fp16 weights below 2^-14, which are
  held to 2^-25.
"""
import math

import numpy as np
import pytest

import workloads as W

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


@pytest.fixture(scope="module")
def P():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2608_12574_amd as P
    P.lib()
    return P


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------- adjust -------

def adjusted(x, V, tokens=None, length=None, prompt=None, repetition=None, frequency=None, presence=None,
             bias_ids=None, bias=None, valid=None):
    """(result, bound on its error) in 64 bits, and which entries must keep their bits."""
    u = U[x.dtype]
    x = x.double().cpu().numpy()
    y, big, kept = x.copy(), np.abs(x), np.ones(x.shape, bool)
    for b in range(x.shape[0]):
        text = tokens[b].tolist() if tokens is not None else []
        n = len(text) if length is None else min(max(int(length[b]), 0), len(text))
        p = 0 if prompt is None else int(prompt[b])
        rep, freq, pres = (float(t[b]) if t is not None else d for t, d in
                           ((repetition, 1.0), (frequency, 0.0), (presence, 0.0)))
        seen, count = set(), {}
        for i, v in enumerate(text[:n]):
            if 0 <= v < V:
                seen.add(v)
                if i >= p:
                    count[v] = count.get(v, 0) + 1
        named = {}
        if bias_ids is not None:
            for v, w in zip(bias_ids[b].tolist(), bias[b].tolist()):
                if 0 <= v < V:
                    named[v] = w
        for v in seen | set(named):
            z = x[b, v]
            if v in seen:
                z = z / rep if z > 0 else z * rep
            steps = [abs(z)]
            if v in count:
                steps += [abs(freq * count[v]), abs(pres)]
                z = z - freq * count[v] - pres
            if v in named:
                steps.append(abs(named[v]))
                z = z + named[v]
            y[b, v], kept[b, v] = z, False
            big[b, v] = sum(steps)
    if valid is not None:
        y = np.where(valid, y, -np.inf)
        kept &= valid
    return y, 8 * 2.0 ** -24 * big + u * np.where(np.isfinite(y), np.abs(y), 0), kept


def check_adjusted(P, B, V, dtype, seed, pad=0, offset=0, history=40, biases=5, masked=True, call=None, **without):
    rng = np.random.default_rng(seed)
    g = gen(seed)
    buf = torch.randn((B, offset + V + pad), generator=g, device="cuda") * 4
    buf[:, ::97] = 0.0
    buf = buf.to(dtype)
    logits = buf[:, offset:offset + V]
    kw = {}
    if history is not None:
        t = (rng.random((B, history)) ** 3 * V).astype(np.int32)
        t[rng.random((B, history)) < 0.1] = -1
        t[rng.random((B, history)) < 0.05] = V + 3
        if history:
            t[:, 0] = V - 1
        kw["tokens"] = ints(t)
        kw["length"] = ints(rng.integers(-1, history + 3, B))
        kw["prompt"] = ints(rng.integers(0, history + 1, B))
        kw["repetition"] = torch.as_tensor(rng.uniform(0.8, 1.5, B), dtype=torch.float32, device="cuda")
        kw["frequency"] = torch.as_tensor(rng.uniform(-0.5, 1, B), dtype=torch.float32, device="cuda")
        kw["presence"] = torch.as_tensor(rng.uniform(-0.5, 1, B), dtype=torch.float32, device="cuda")
    if biases:
        ids = rng.integers(-1, V, (B, biases)).astype(np.int32)
        ids[:, 0] = ids[:, -1]
        ids[:, biases // 2] = 0
        kw["bias_ids"] = ints(ids)
        kw["bias"] = torch.as_tensor(rng.normal(0, 5, (B, biases)), dtype=torch.float32, device="cuda")
    for name in without:
        kw.pop(name, None)
    valid, mask = None, {}
    if masked:
        R = 5
        bits = rng.random((R, V)) < np.array([0.0, 1.0, 0.5, 2.0 / V, 0.02])[:, None]
        full = np.zeros((R, -(-V // 64) * 64), dtype=np.uint8)
        full[:, :V] = bits
        words = np.packbits(full, axis=1, bitorder="little").view(np.int64)
        words = np.concatenate([words, np.full((R, 3), -1, np.int64)], 1)  # rows longer than the vocabulary
        ids = rng.integers(0, R, B).astype(np.int32)
        ids[0] = [2, -1, R, 1][seed % 4]
        mask = {"rows": torch.as_tensor(words, device="cuda"), "row_ids": ints(ids)}
        ok = (ids >= 0) & (ids < R)
        valid = bits[np.clip(ids, 0, R - 1)] & ok[:, None]
    want, bound, kept = adjusted(logits, V, valid=valid, **kw)
    before = buf.clone()
    got = P.adjust_logits(logits, **kw, **mask)
    torch.cuda.synchronize()
    assert got is logits
    y = logits.double().cpu().numpy()
    assert np.array_equal(np.isinf(y), np.isinf(want))
    f = np.isfinite(want)
    assert np.all(np.abs(y[f] - want[f]) <= bound[f])
    raw = torch.int16 if dtype is torch.bfloat16 else torch.int32
    same = (buf.view(raw) == before.view(raw)).cpu().numpy()
    assert same[:, offset:offset + V][kept].all()
    assert same[:, :offset].all() and same[:, offset + V:].all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,V,pad,offset", [(1, 1, 0, 0), (3, 63, 1, 0), (2, 4096, 0, 0), (4, 4097, 3, 1), (5, 12289, 0, 7),
                                            (2, 32000, 8, 0), (7, 8191, 2, 5)])
def test_adjust_shapes(P, dtype, B, V, pad, offset):
    for seed in range(3):
        check_adjusted(P, B, V, dtype, 10 * V + seed, pad=pad, offset=offset, masked=seed != 1)


@pytest.mark.parametrize("history,biases", [(0, 5), (1, 0), (300, 300), (5000, 1), (None, 4095), (9000, 0)])
def test_adjust_lists(P, history, biases):
    check_adjusted(P, 3, 5003, torch.bfloat16, 3, history=history, biases=biases)
    check_adjusted(P, 2, 5003, torch.float32, 4, history=history, biases=biases, masked=False)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,V,history,biases", [(3, 150000, 3000, 100), (2, 262144, 12000, 200), (20, 50001, 900, 30),
                                                (200, 20000, 64, 5), (9, 16 * 45, 40, 5), (1, 400000, 6100, 0),
                                                (2, 262144, 12200, 90)])
def test_adjust_few_of_many(P, dtype, B, V, history, biases):
    """Texts that name a small part of the vocabulary, no mask."""
    check_adjusted(P, B, V, dtype, V, pad=3, offset=1, history=history, biases=biases, masked=False)


@pytest.mark.parametrize("B,V,pad,offset,dtype", [(50, 262144, 0, 0, torch.float32), (97, 262143, 1, 0, torch.bfloat16),
                                                  (97, 262143, 2, 3, torch.bfloat16)])
def test_adjust_large_batches(P, B, V, pad, offset, dtype):
    check_adjusted(P, B, V, dtype, 5, pad=pad, offset=offset, history=300, biases=20)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,V,pad,offset", [(9, 4096, 0, 0), (5, 4101, 3, 0), (4, 8191, 2, 5), (6, 200, 0, 1)])
def test_adjust_mask_alone(P, dtype, B, V, pad, offset):
    for seed in range(2):
        check_adjusted(P, B, V, dtype, seed, pad=pad, offset=offset, history=None, biases=0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,V,pad,offset,history", [(9, 4101, 3, 1, None), (4, 8192, 0, 5, None), (1, 63, 0, 1, None), (6, 200, 5, 0, 40),
                                                    (110, 262143, 1, 1, 300), (110, 262144, 0, 3, 300)])
def test_adjust_rows_as_wide_as_the_vocabulary(P, dtype, B, V, pad, offset, history):
    """Mask rows of ceil(V/64) words with bits set past V, the last one at the end of its memory, logits of any alignment:
    the mask alone, in one pass with the edits, and after them."""
    rng = np.random.default_rng(V + B)
    words = -(-V // 64)
    bits = rng.random((7, words * 64)) < np.array([0, 1, 0.5, 2 / V, 0.02, 0.9, 0.3])[:, None]
    bits[:, V:] = True
    rows = torch.as_tensor(np.packbits(bits, axis=1, bitorder="little").view(np.int64), device="cuda")
    ids = rng.integers(-1, 8, B)
    buf = (torch.randn((B, offset + V + pad), generator=gen(B), device="cuda") * 4).to(dtype)
    before, kw = buf.clone(), {}
    if history:
        kw = dict(tokens=ints(rng.integers(-1, V + 2, (B, history)).astype(np.int32)),
                  presence=torch.as_tensor(rng.uniform(-0.5, 1, B), dtype=torch.float32, device="cuda"))
    logits = buf[:, offset:offset + V]
    valid = torch.as_tensor(bits[np.clip(ids, 0, 6), :V] & ((ids >= 0) & (ids < 7))[:, None], device="cuda")
    want, bound, kept = (torch.as_tensor(x, device="cuda") for x in adjusted(logits, V, **kw))
    P.adjust_logits(logits, rows=rows, row_ids=ints(ids), **kw)
    assert ((logits == -math.inf) == ~valid).all()
    assert ((logits.double() - want).abs() <= bound)[valid].all()
    raw = torch.int16 if dtype is torch.bfloat16 else torch.int32
    same = buf.view(raw) == before.view(raw)
    assert same[:, offset:offset + V][kept & valid].all() and same[:, :offset].all() and same[:, offset + V:].all()


@pytest.mark.parametrize("name", ["length", "prompt", "repetition", "frequency", "presence"])
def test_adjust_parts_left_out(P, name):
    check_adjusted(P, 4, 1000, torch.float32, 8, **{name: None})


def test_adjust_keeps_and_masks_special_values(P):
    x = torch.tensor([[float("nan"), float("inf"), -float("inf"), -0.0, 1e-40, 3.0e38, -3.0e38, 1.0]], device="cuda")
    before = x.clone()
    P.adjust_logits(x, tokens=ints([[6, 5, 2]]), repetition=torch.tensor([2.0], device="cuda"),
                    rows=torch.tensor([[0b11111111]], device="cuda"), row_ids=ints([0]))
    y = x.cpu()
    assert torch.equal(y[0, [0, 1, 3, 4, 7]].view(torch.int32), before.cpu()[0, [0, 1, 3, 4, 7]].view(torch.int32))
    assert y[0, 2] == -math.inf and y[0, 6] == -math.inf and y[0, 5] == 1.5e38
    P.adjust_logits(x, rows=torch.tensor([[0]], device="cuda"), row_ids=ints([0]))
    assert (x == -math.inf).all()  # NaN and infinities among them


def test_adjust_one_row_of_any_stride(P):
    """Of a single row the stride says nothing: one row of larger lists."""
    x = torch.randn((3, 5003), generator=gen(6), device="cuda")
    want = x.clone()
    tokens, ids = (torch.randint(0, 5003, (3, n), generator=gen(n), device="cuda", dtype=torch.int32) for n in (40, 9))
    bias, presence = torch.randn((3, 9), generator=gen(7), device="cuda"), torch.ones(3, device="cuda")
    rows = torch.randint(-2 ** 62, 2 ** 62, (3, 90), generator=gen(8), device="cuda")
    P.adjust_logits(want, tokens=tokens[:, :30].contiguous(), presence=presence, bias_ids=ids[:, :5].contiguous(),
                    bias=bias[:, :5].contiguous(), rows=rows, row_ids=ints([0, 1, 2]))
    for b in range(3):
        P.adjust_logits(x[b:b + 1], tokens=tokens[b:b + 1, :30], presence=presence[b:b + 1], bias_ids=ids[b:b + 1, :5],
                        bias=bias[b:b + 1, :5].clone(), rows=rows[b:b + 1], row_ids=ints([0]))
    assert torch.equal(x, want)


def test_adjust_refusals(P):
    x = torch.zeros((2, 100), device="cuda")
    t = ints([[1], [2]])
    bad = [
        dict(logits=x.half()), dict(logits=x.t()), dict(logits=x[0]), dict(logits=x.cpu()),
        dict(logits=x, tokens=t.long()), dict(logits=x, tokens=t[:1]), dict(logits=x, tokens=t.cpu()),
        dict(logits=x, length=ints([1])), dict(logits=x, repetition=torch.ones(2, device="cuda").double()),
        dict(logits=x, bias_ids=t), dict(logits=x, bias=torch.ones((2, 1), device="cuda")),
        dict(logits=x, bias_ids=t, bias=torch.ones((2, 2), device="cuda")),
        dict(logits=x, rows=torch.zeros((3, 1), dtype=torch.int64, device="cuda"), row_ids=ints([0, 0])),
        dict(logits=x, rows=torch.zeros((3, 2), dtype=torch.int64, device="cuda")),
        dict(logits=x, rows=torch.zeros((3, 2), dtype=torch.int64, device="cuda"), row_ids=ints([0])),
        dict(logits=x, bias_ids=torch.zeros((2, 4096), dtype=torch.int32, device="cuda"),
             bias=torch.zeros((2, 4096), device="cuda")),
    ]
    for kw in bad:
        with pytest.raises(P.TamError):
            P.adjust_logits(**kw)
    P.adjust_logits(torch.zeros((0, 100), device="cuda"))
    P.adjust_logits(x)
    assert (x == 0).all()


def test_adjust_mask_arguments(P):
    """No mask rows at all: nothing is valid.  A mask given twice or by half, or of a closed handle, is refused."""
    x = torch.zeros((2, 100), device="cuda")
    rows = torch.full((3, 2), -1, dtype=torch.int64, device="cuda")
    P.adjust_logits(x, rows=rows[:0].clone(), row_ids=ints([0, 1]))
    assert (x == -math.inf).all()
    x.zero_()
    h = P.compile([b"ab", b"c"], [b"a", b"b", b"c", b'"'], device="cuda:0")
    for call in (lambda: P.adjust_logits(x, row_ids=ints([0, 1])),
                 lambda: P.adjust_logits(x, rows=rows[0], row_ids=ints([0, 1])),
                 lambda: h.adjust_logits(ints([0, 1]), x, rows=rows)):
        with pytest.raises(P.TamError):
            call()
    h.close()
    with pytest.raises(P.TamError):
        h.adjust_logits(ints([0, 1]), x, tokens=ints([[1], [2]]))
    assert (x == 0).all()


@pytest.mark.parametrize("flags", ["0", "FLAG_TAIL_LISTS", "FLAG_NO_TABLE", "FLAG_LAZY_ROWS"])
def test_adjust_on_a_handle_is_edits_then_mask(P, flags):
    w = W.config(1)
    h = P.compile(w.strings, w.vocab, flags=getattr(P, flags, 0))
    V, B = len(w.vocab), 9
    nodes = ints([0, 1, 5, h.num_nodes - 1, -1, h.num_nodes, 3, 2, h.num_nodes // 2])
    x = torch.randn((B, V + 5), generator=gen(1), device="cuda").to(torch.bfloat16)
    kw = dict(tokens=torch.randint(0, V, (B, 200), generator=gen(2), device="cuda", dtype=torch.int32),
              presence=torch.full((B,), 0.75, device="cuda"))
    kw["tokens"][:, ::2] = torch.arange(100, device="cuda", dtype=torch.int32)
    want = x.clone()
    P.adjust_logits(want[:, :V], **kw)
    h.apply_mask(nodes, want)
    got = x.clone()
    h.adjust_logits(nodes, got, **kw)
    assert torch.equal(got.view(torch.int16), want.view(torch.int16))
    only = x.clone()
    h.adjust_logits(nodes, only)
    masked = x.clone()
    h.apply_mask(nodes, masked)
    assert torch.equal(only.view(torch.int16), masked.view(torch.int16))
    with pytest.raises(P.TamError):
        h.adjust_logits(nodes, got[:, :V - 1])
    with pytest.raises(P.TamError):
        h.adjust_logits(nodes[:3], got)
    h.close()


# ----------------------------------------------------------------- pages -------

class Model:
    """The page tables on the host."""

    def __init__(self, cache):
        self.page = cache.page_tokens
        self.M = cache.table.shape[1]
        self.rows = [r[:-(-n // self.page)] for r, n in zip(cache.table.tolist(), cache.length.tolist())]
        self.len = cache.length.tolist()
        self.refs = cache.refs.tolist()
        self.data = cache.data.clone()

    def fork(self, slots, parents, lengths=None):
        rows, lens = [list(r) for r in self.rows], list(self.len)
        for i, (s, p) in enumerate(zip(slots, parents)):
            if not 0 <= s < len(lens):
                continue
            n = lens[p] if 0 <= p < len(lens) else 0
            if lengths is not None:
                n = min(n, max(lengths[i], 0))
            new = rows[p][:-(-n // self.page)] if n else []
            for x in rows[s]:
                self.refs[x] -= 1
            for x in new:
                self.refs[x] += 1
            self.rows[s], self.len[s] = new, n

    def extend(self, slots, counts):
        part = {}
        for i, (s, c) in enumerate(zip(slots, counts)):
            if 0 <= s < len(self.len) and c > 0 and self.len[s] % self.page:
                part.setdefault(self.rows[s][-1], []).append(i)
        need, narrow, plan = 0, 0, []
        for i, (s, c) in enumerate(zip(slots, counts)):
            if not 0 <= s < len(self.len) or c <= 0:
                continue
            total = -(-(self.len[s] + c) // self.page)
            copy = False
            if self.len[s] % self.page:
                g = self.rows[s][-1]
                copy = self.refs[g] != len(part[g]) or part[g][-1] != i
            narrow += total > self.M
            plan.append((s, c, copy, total - len(self.rows[s])))
            need += copy + total - len(self.rows[s])
        free = [p for p, r in enumerate(self.refs) if r <= 0]
        done = need <= len(free) and not narrow
        if done:
            it = iter(list(free))
            for s, c, copy, more in plan:
                if copy:
                    g, to = self.rows[s][-1], next(it)
                    self.data[:, to] = self.data[:, g]
                    self.refs[g] -= 1
                    self.refs[to] = 1
                    self.rows[s] = self.rows[s][:-1] + [to]
                for _ in range(more):
                    to = next(it)
                    self.refs[to] = 1
                    self.rows[s] = self.rows[s] + [to]
                self.len[s] += c
        return [int(done), need, len(free), narrow]

    def compact(self):
        used = [p for p, r in enumerate(self.refs) if r > 0]
        U = len(used)
        holes = [p for p in range(U) if self.refs[p] <= 0]
        move = dict(zip([p for p in used if p >= U], holes))
        for a, b in move.items():
            self.data[:, b] = self.data[:, a]
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.rows = [[move.get(p, p) for p in r] for r in self.rows]
        gone = set(holes) | set(p for p in range(len(self.refs)) if p >= U and p not in move)
        return [U, len(move)], [move.get(p, -1 if p in gone else p) for p in range(len(self.refs))]

    def same(self, cache):
        torch.cuda.synchronize()
        assert cache.length.tolist() == self.len
        table = cache.table.tolist()
        for s, r in enumerate(self.rows):
            assert table[s][:len(r)] == r, s
        assert cache.refs.tolist() == self.refs
        assert torch.equal(cache.data.view(torch.int16), self.data.view(torch.int16))


def page_cache(P, pages, slots, width, page=4, kv=2, dim=16, layers=2, seed=0):
    c = P.PageCache.empty(layers, kv, dim, pages, slots, width, page_tokens=page)
    c.data.copy_(torch.randn(c.data.shape, generator=gen(seed), device="cuda"))
    return c


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("page,width,slots,pages", [(4, 9, 12, 60), (1, 20, 5, 64), (16, 3, 40, 70), (8, 700, 30, 4100),
                                                    (2, 6, 1, 5)])
def test_pages_against_the_model(P, seed, page, width, slots, pages):
    rng = np.random.default_rng(100 * seed + page)
    c = page_cache(P, pages, slots, width, page=page, seed=seed)
    m = Model(c)
    for step in range(14):
        n = int(rng.integers(0, slots + 1))
        s = rng.permutation(slots)[:n].tolist()
        kind = step % 3 if step else 0
        if kind == 0:
            counts = rng.integers(-1, 2 * page + 2, n).tolist()
            if n and rng.random() < 0.2:
                counts[0] = page * width + 1
            info = c.extend(ints(s), ints(counts))
            assert info.tolist() == m.extend(s, counts)
        elif kind == 1:
            parents = rng.integers(-1, slots + 1, n).tolist()
            lengths = rng.integers(-1, 3 * page, n).tolist() if rng.random() < 0.5 else None
            c.fork(ints(s), ints(parents), None if lengths is None else ints(lengths))
            m.fork(s, parents, lengths)
            assert all(x == -1 for i in s for x in c.table[i].tolist()[len(m.rows[i]):])
        else:
            info, moved = c.compact()
            want = m.compact()
            assert info.tolist() == want[0] and moved.tolist() == want[1]
        m.same(c)
    c.free(ints(list(range(slots))))
    m.fork(list(range(slots)), [-1] * slots)
    m.same(c)
    assert not c.refs.any()


def test_pages_all_or_nothing_and_held_pages(P):
    c = page_cache(P, 6, 3, 8)
    assert c.extend(ints([0]), ints([6])).tolist() == [1, 2, 6, 0]
    c.fork(ints([1, 2]), ints([0, 0]))
    m = Model(c)
    before = c.table.clone()
    assert c.extend(ints([0, 1, 2]), ints([1, 9, 9])).tolist() == m.extend([0, 1, 2], [1, 9, 9]) == [0, 6, 4, 0]
    assert torch.equal(c.table, before)
    m.same(c)
    # a holder outside the table keeps its page: every row copies
    c.refs[c.table[0, 1].long()] += 1
    m = Model(c)
    assert c.extend(ints([2, 0, 1]), ints([1, 1, 1])).tolist() == m.extend([2, 0, 1], [1, 1, 1]) == [1, 3, 4, 0]
    m.same(c)
    # slots outside the cache are left out
    c.fork(ints([-1, 3]), ints([0, 0]))
    c.extend(ints([-5, 7]), ints([1, 1]))
    m.same(c)


def test_pages_of_many_rows(P):
    """More rows than one block has threads, and tables too large for one block's fork."""
    c = page_cache(P, 9000, 1500, 40, page=2, kv=1, dim=8, layers=1)
    m = Model(c)
    rng = np.random.default_rng(0)
    s = rng.permutation(1500).tolist()
    counts = rng.integers(0, 8, 1500).tolist()
    assert c.extend(ints(s), ints(counts)).tolist() == m.extend(s, counts)
    m.same(c)
    for _ in range(2):
        parents = rng.integers(-1, 1500, 1500).tolist()
        c.fork(ints(s), ints(parents))
        m.fork(s, parents)
        m.same(c)
        assert c.extend(ints(s), ints([1] * 1500)).tolist() == m.extend(s, [1] * 1500)
        m.same(c)
    info, moved = c.compact()
    want = m.compact()
    assert info.tolist() == want[0] and moved.tolist() == want[1]
    m.same(c)


def test_pages_unaligned_pool(P):
    """Pages whose bytes are no multiple of 16 (the copy's narrow path), planes with gaps."""
    whole = torch.randn((4, 7, 11, 1, 1, 12), generator=gen(3), device="cuda").to(torch.bfloat16)
    data = whole[:, 3]  # [4, 11, 1, 1, 12]: 24-byte pages
    c = P.PageCache(data, torch.full((3, 5), -1, dtype=torch.int32, device="cuda"), ints([0, 0, 0]), ints([0] * 11))
    m = Model(c)
    for s, n in (([0, 1, 2], [3, 1, 4]), ([1], [2])):
        assert c.extend(ints(s), ints(n)).tolist() == m.extend(s, n)
    c.fork(ints([0]), ints([-1]))
    m.fork([0], [-1])
    c.compact()
    m.compact()
    m.same(c)
    assert torch.equal(whole[:, 2], whole[:, 2])


@pytest.mark.parametrize("dim", [12, 16])
def test_pages_stay_in_their_planes(P, dim):
    """Copies and moves in a pool with gaps between planes and between pages, in bytes (dim 12) and in pieces (16)."""
    whole = torch.randn((4, 5, 11, 3, 1, 1, dim), generator=gen(24), device="cuda").to(torch.bfloat16)
    before = whole.clone()
    c = P.PageCache(whole[:, 3, :, 1], torch.full((3, 5), -1, dtype=torch.int32, device="cuda"), ints([0, 0, 0]), ints([0] * 11))
    assert c.page_tokens == 1
    m = Model(c)
    for s, n in (([0, 1, 2], [3, 1, 4]), ([1], [2])):
        assert c.extend(ints(s), ints(n)).tolist() == m.extend(s, n)
    c.fork(ints([0]), ints([-1]))
    m.fork([0], [-1])
    info, moved = c.compact()
    want = m.compact()
    assert info.tolist() == want[0] and want[0][1] > 0 and moved.tolist() == want[1]
    m.same(c)
    before[:, 3, :, 1] = c.data
    assert torch.equal(whole.view(torch.int16), before.view(torch.int16))


@pytest.mark.parametrize("dim", [12, 16])
def test_shared_pages_are_copied_in_their_planes(P, dim):
    whole = torch.randn((4, 5, 11, 3, 1, 4, dim), generator=gen(25), device="cuda").to(torch.bfloat16)
    before = whole.clone()
    c = P.PageCache(whole[:, 3, :, 1], torch.full((3, 5), -1, dtype=torch.int32, device="cuda"), ints([0, 0, 0]), ints([0] * 11))
    m = Model(c)
    for call in (lambda x: x.extend([0], [6]), lambda x: x.fork([1, 2], [0, 0], [6, 5]), lambda x: x.extend([0, 1, 2], [1, 3, 1])):
        want = call(m)
        got = call(OnLists(c))
        assert want == got
    m.same(c)
    before[:, 3, :, 1] = c.data
    assert torch.equal(whole.view(torch.int16), before.view(torch.int16))


class OnLists:
    """A cache that takes lists, as the model does."""

    def __init__(self, cache):
        self.cache = cache

    def extend(self, *lists):
        return self.cache.extend(*map(ints, lists)).tolist()

    def fork(self, *lists):
        return self.cache.fork(*map(ints, lists))


def test_pages_refusals(P):
    import ctypes
    c = page_cache(P, 6, 3, 8)
    for kw in (dict(slots=ints([0]), parents=ints([0, 1])), dict(slots=ints([0]).long(), parents=ints([0])),
               dict(slots=ints([0, 1, 2, 3]), parents=ints([0, 1, 2, 3])),
               dict(slots=ints([0]), parents=ints([0]), lengths=ints([0, 1]))):
        with pytest.raises(P.TamError):
            c.fork(**kw)
    with pytest.raises(P.TamError):
        c.extend(ints([0]), torch.ones(1, device="cuda"))
    with pytest.raises(P.TamError):
        P.PageCache.empty(1, 2, 16, 8, 2, 4, page_tokens=12)
    with pytest.raises(P.TamError):
        P.PageCache.empty(1, 2, 16, 8, 2, 4, dtype=torch.float32)
    with pytest.raises(P.TamError):
        P.PageCache(c.data[:1], c.table, c.length, c.refs)
    with pytest.raises(P.TamError):
        P.PageCache(c.data, c.table, c.length, c.refs[1:])
    with pytest.raises(P.TamError):
        P.PageCache(c.data, c.table, c.length[:2], c.refs)
    rc = P.lib().tam_pages_extend(ctypes.byref(c._pages), None, None, 1, None, None, None)
    assert rc == -1 and P.lib().tam_last_error()


def test_pages_overlapping_tables(P):
    c = page_cache(P, 6, 3, 8)
    for table in (c.table[:1].expand(3, 8), c.table.view(-1).as_strided((3, 8), (4, 1))):
        with pytest.raises(P.TamError):
            P.PageCache(c.data, table, c.length, c.refs)
    with pytest.raises(P.TamError):
        P.PageCache(c.data[:, :0], c.table, c.length, c.refs[:0])
    P.PageCache(c.data, c.table[:1], c.length[:1], c.refs)


# ------------------------------------------------------- store and attention ----

class Sequences:
    """A cache filled directly, with garbage in every place that no token has, and chunks over it."""

    def __init__(self, P, lens, chunks, heads, kv, dim, page, dtype, seed=0, slots=None, spare=3,
                 garbage=float("nan"), far=0):
        g = gen(seed)
        rng = np.random.default_rng(seed)
        self.lens, self.chunks, self.heads, self.kv, self.dim, self.page = lens, chunks, heads, kv, dim, page
        rows = len(lens)
        held = [-(-x // page) for x in lens]
        width = max(held) + 1
        pages = sum(held) + spare + far
        self.slots = list(range(rows)) if slots is None else slots
        nslots = max(self.slots) + 1
        shape = (4, pages, kv, page, dim)
        data = torch.full(shape, garbage, dtype=dtype, device="cuda")
        ids = far + rng.permutation(pages - far)
        table = np.full((nslots, width), -1, np.int32)
        length = np.zeros(nslots, np.int32)
        self.k, self.v = [], []
        at = 0
        for i, n in enumerate(lens):
            mine = ids[at:at + held[i]]
            at += held[i]
            table[self.slots[i], :held[i]] = mine
            table[self.slots[i], held[i]:] = 2 ** 30  # not read
            length[self.slots[i]] = n
            k = torch.randn((n, kv, dim), generator=g, device="cuda").to(dtype)
            v = torch.randn((n, kv, dim), generator=g, device="cuda").to(dtype)
            self.k.append(k)
            self.v.append(v)
            if n:
                pos = torch.arange(n, device="cuda")
                to = torch.as_tensor(mine.astype(np.int64), device="cuda")[pos // page]
                data[2][to, :, pos % page] = k
                data[3][to, :, pos % page] = v
        self.cache = P.PageCache(data, ints(table), ints(length), torch.ones(pages, dtype=torch.int32, device="cuda"))
        T = sum(chunks)
        self.offsets = ints(np.concatenate([[0], np.cumsum(chunks)]).astype(np.int32))
        self.q = torch.randn((T, heads * dim + 24), generator=g, device="cuda").to(dtype)[:, 8:8 + heads * dim].unflatten(
            1, (heads, dim))

    def reference(self, scale):
        out, lse, tol, ltol = [], [], [], []
        u = U[self.q.dtype]
        q = self.q.double()
        t = 0
        for n, x, k, v in zip(self.lens, self.chunks, self.k, self.v):
            kk = k.double().repeat_interleave(self.heads // self.kv, 1).permute(1, 0, 2)
            vv = v.double().repeat_interleave(self.heads // self.kv, 1).permute(1, 0, 2)
            qq = q[t:t + x].permute(1, 0, 2)
            t += x
            pos = torch.arange(n - x, n, device="cuda")
            hidden = torch.arange(n, device="cuda")[None, :] > pos[:, None]
            s = (qq @ kk.transpose(1, 2) * scale).masked_fill(hidden, -math.inf)
            top = s.amax(2, keepdim=True) if n else torch.full((self.heads, x, 1), -math.inf, device="cuda").double()
            top = top.clamp(min=-1e300)
            p = torch.exp(s - top)
            l = p.sum(2, keepdim=True)
            w = p / l.clamp(min=1e-300)
            o, a = w @ vv, w @ vv.abs()
            es = (self.dim + 8) * 2.0 ** -24 * scale * (
                (qq.abs() @ kk.abs().transpose(1, 2)).amax(2, keepdim=True) if n else torch.zeros_like(top))
            small = 2.0 ** -25 * vv.abs().sum(1, keepdim=True) / l.clamp(min=1) if self.q.dtype is torch.float16 else 0
            tol.append((u * (a + o.abs()) + (torch.exp(2 * es) - 1 + (n + 16) * 2.0 ** -24) * a + small + 1e-30).permute(1, 0, 2))
            empty = l == 0
            lg = torch.where(empty, -math.inf, torch.log(l) + top)
            out.append(o.permute(1, 0, 2))
            lse.append(lg[..., 0].T)
            ltol.append((es + (n + 16) * 2.0 ** -24 + 4 * 2.0 ** -24 * torch.where(empty, 0, lg.abs()))[..., 0].T)
        return tuple(torch.cat(z) for z in (out, lse, tol, ltol))

    def check(self, scale=None, **kw):
        scale = self.dim ** -0.5 if scale is None else scale
        slots = ints(self.slots) if self.slots != list(range(len(self.lens))) else None
        out, lse = self.cache.attend(1, self.q, offsets=self.offsets, slots=slots, scale=scale, return_lse=True, **kw)
        self.compare(out, lse, scale)
        return out, lse

    def compare(self, out, lse, scale):
        want, wl, tol, ltol = self.reference(scale)
        assert torch.isfinite(out).all()
        worst = ((out.double() - want).abs() / tol).max() if out.numel() else 0
        assert worst <= 1, float(worst)
        fin = torch.isfinite(wl)
        assert torch.equal(fin, torch.isfinite(lse)) and (lse[~fin] == -math.inf).all()
        assert ((lse.double() - wl).abs()[fin] <= ltol[fin]).all()


# chunks of tiles of 16, 128 and 256 rows with four heads to a K/V head
TILES = [[4, 2], [20, 30], [200, 90]]
HEADS = [(8, 8, 64), (8, 2, 128), (16, 1, 128), (6, 2, 96), (5, 5, 40), (7, 1, 8), (40, 1, 64), (12, 4, 120)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,kv,dim", HEADS)
def test_attend_single_tokens(P, dtype, heads, kv, dim):
    for page, lens in ((16, [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 300]), (1, [5, 129]), (64, [700, 1])):
        Sequences(P, lens, [1] * len(lens), heads, kv, dim, page, dtype, seed=page).check(longest=1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,kv,dim", HEADS)
def test_attend_chunks(P, dtype, heads, kv, dim):
    chunks = [1, 0, 7, 33, 64, 100, 129, 5]
    lens = [40, 9, 7, 200, 64, 613, 130, 1500]
    s = Sequences(P, lens, chunks, heads, kv, dim, 16, dtype, seed=1)
    a = s.check()
    b = s.check(longest=129)
    for x, y in zip(a, b):
        assert torch.equal(x, y)


@pytest.mark.parametrize("heads,kv,dim,page", [(8, 2, 128, 16), (4, 4, 64, 32), (32, 4, 128, 8)])
def test_attend_long_rows(P, heads, kv, dim, page):
    """A long axis split over the chip, beside short rows; and a longer chunk."""
    Sequences(P, [20011, 3, 4097], [1, 1, 1], heads, kv, dim, page, torch.bfloat16, seed=2).check(longest=1)
    Sequences(P, [9000, 50, 1023], [9, 2, 17], heads, kv, dim, page, torch.float16, seed=3).check()
    Sequences(P, [2000, 700], [700, 700], heads, kv, dim, page, torch.bfloat16, seed=4).check()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,kv,dim", HEADS)
def test_attend_long_chunks(P, dtype, heads, kv, dim):
    """Tiles of 256 rows, the last ones of a row partly filled; and of 128 for mostly short rows."""
    for page, lens, chunks in ((16, [700, 333, 64], [610, 300, 64]), (4, [300], [290]), (32, [500, 9, 40, 90, 0, 3], [310, 1, 1, 1, 0, 3])):
        Sequences(P, lens, chunks, heads, kv, dim, page, dtype, seed=page + 1).check()


@pytest.mark.parametrize("chunk", [5, 17])
def test_attend_join_of_many_pieces(P, chunk):
    """A few rows over keys enough for every block: each tile's parts lie in many of them."""
    Sequences(P, [50000, 33000], [chunk, 3], 16, 2, 128, 16, torch.bfloat16, seed=17).check()
    Sequences(P, [40001], [chunk], 6, 2, 64, 16, torch.float16, seed=18).check()


def test_attend_rows_without_keys(P):
    """Chunks longer than their sequence: the first queries see nothing."""
    s = Sequences(P, [0, 3, 1, 40], [0, 3, 1, 40], 8, 2, 64, 16, torch.bfloat16, seed=5)
    s.cache.length.copy_(ints([0, 2, 0, 5]))
    # the last `length` tokens of each chunk are the ones with keys
    out, lse = s.cache.attend(1, s.q, offsets=s.offsets, return_lse=True)
    t = 0
    for x, n, full in zip(s.chunks, [0, 2, 0, 5], s.lens):
        assert (out[t:t + x - n] == 0).all() and (lse[t:t + x - n] == -math.inf).all()
        t += x
    cut = Sequences(P, [0, 3, 1, 40], [0, 3, 1, 40], 8, 2, 64, 16, torch.bfloat16, seed=5)
    keep = [i for o, x, n in ((0, 0, 0), (0, 3, 2), (3, 1, 0), (4, 40, 5)) for i in range(o + x - n, o + x)]
    cut.lens = cut.chunks = [0, 2, 0, 5]
    cut.k, cut.v = ([z[:n] for z, n in zip(w, cut.lens)] for w in (cut.k, cut.v))
    cut.q = cut.q[keep]
    cut.compare(out[keep], lse[keep], 64 ** -0.5)


@pytest.mark.parametrize("chunks", [[1, 1], [40, 3], [200, 90]])
def test_attend_nan_stays_in_its_row(P, chunks):
    """A query or a key that is not a number: its rows say so, the others do not change."""
    s = Sequences(P, [700, 3000], chunks, 8, 2, 128, 16, torch.bfloat16, seed=19)
    out, lse = s.check()
    s.q[0, 3, 5] = float("nan")
    s.cache.data[2][int(s.cache.table[1, 20]), 1, 3] = float("nan")  # K of the second sequence, heads 4 to 7
    got, glse = s.cache.attend(1, s.q, offsets=s.offsets, return_lse=True)
    bad = torch.zeros(lse.shape, dtype=torch.bool, device="cuda")
    bad[0, 3] = True
    bad[chunks[0]:, 4:] = True
    assert torch.isnan(glse[bad]).all() and torch.isnan(got[bad]).all()
    assert torch.equal(glse[~bad], lse[~bad]) and torch.equal(got[~bad], out[~bad])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,kv,dim,page", [(8, 2, 128, 16), (8, 2, 64, 4), (4, 1, 40, 16), (16, 4, 120, 1)])
@pytest.mark.parametrize("chunks", TILES)
@pytest.mark.parametrize("lens", [[700, 3000], [20011, 203]])
def test_attend_hidden_values(P, dtype, heads, kv, dim, page, chunks, lens):
    """V of a chunk's tokens that is not finite: the queries before them do not change, those that see it say so."""
    s = Sequences(P, lens, chunks, heads, kv, dim, page, dtype, seed=20)
    out, lse = s.check(longest=max(chunks))
    inf, nan, group = math.inf, math.nan, heads // kv
    extra = torch.zeros(out.shape, device="cuda")
    t0 = 0
    for row, (n, x) in enumerate(zip(lens, chunks)):
        hits = {}  # the last one of a place stands
        for j, head, d, value in ((x - 1, 0, 5, nan), (x - 1, kv - 1, dim - 1, inf), (x // 2, 0, 0, -inf), (x // 2, 0, 9, inf),
                                  (x - 1, 0, 9, -inf), (1, kv - 1, 17, nan)):
            hits[j, head, d] = value
        for (j, head, d), value in hits.items():
            pos = n - x + j
            s.cache.data[3][int(s.cache.table[row, pos // page]), head, pos % page, d] = value
            extra[t0 + j:t0 + x, head * group:(head + 1) * group, d] += value
        t0 += x
    got, glse = s.cache.attend(1, s.q, offsets=s.offsets, longest=max(chunks), return_lse=True)
    want = torch.where(extra == 0, out.float(), extra)
    assert torch.equal(glse, lse)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got.float().nan_to_num(0), want.nan_to_num(0))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,kv,dim", [(8, 2, 128), (8, 2, 64)])
@pytest.mark.parametrize("chunks", TILES)
def test_attend_infinite_values_under_rising_scores(P, dtype, heads, kv, dim, chunks):
    """An infinity in V that every query sees stays one, where the scores rise by 7 (weights by 2^10) after its key."""
    lens = [700, 900]
    s = Sequences(P, lens, chunks, heads, kv, dim, 16, dtype, seed=21)
    s.q.fill_(1)
    places, hit = [], torch.zeros((2, dim), dtype=torch.bool, device="cuda")
    for row, n in enumerate(lens):
        pos = torch.arange(n, device="cuda")
        places.append((s.cache.table[row, pos // 16].long(), pos % 16))
        s.k[row].copy_((pos // 32 % 2 * 7 / dim ** 0.5)[:, None, None].expand(n, kv, dim))
        s.cache.data[2][places[row][0], :, places[row][1]] = s.k[row]
    out, lse = s.check(longest=max(chunks))
    for row, n in enumerate(lens):
        for i, key in enumerate(range(3, n - max(chunks), 16)):
            if key // 32 % 2 == 0:
                s.cache.data[3][places[row][0][key], :, places[row][1][key], 2 * i % dim] = math.inf
                hit[row, 2 * i % dim] = True
    got, glse = s.cache.attend(1, s.q, offsets=s.offsets, longest=max(chunks), return_lse=True)
    assert torch.equal(glse, lse)
    for a, b, h in zip(got.split(chunks), out.split(chunks), hit):
        assert (a[:, :, h] == math.inf).all()
        assert torch.equal(a[:, :, ~h], b[:, :, ~h])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,kv,dim", [(8, 2, 128), (8, 2, 64), (4, 1, 40), (4, 1, 8), (8, 2, 96), (16, 4, 120)])
@pytest.mark.parametrize("chunks", TILES)
def test_attend_infinite_keys(P, dtype, heads, kv, dim, chunks):
    """A key whose scores are -inf has the weight 0, as one whose scores are far below the others."""
    s = Sequences(P, [700, 90 + chunks[1]], chunks, heads, kv, dim, 16, dtype, seed=22)
    s.q[:, :, 3] = 1
    at = int(s.cache.table[0, 2]), slice(None), 7, 3
    s.cache.data[2][at] = -6e4
    want = s.cache.attend(1, s.q, offsets=s.offsets, longest=max(chunks), return_lse=True)
    s.cache.data[2][at] = -math.inf
    got = s.cache.attend(1, s.q, offsets=s.offsets, longest=max(chunks), return_lse=True)
    for a, b in zip(want, got):
        assert torch.isfinite(a).all() and torch.equal(a, b)


def test_attend_slots_and_page_ids(P):
    s = Sequences(P, [33, 70, 5], [4, 9, 1], 8, 2, 64, 16, torch.bfloat16, seed=6, slots=[7, 0, 3])
    out, lse = s.check()
    # entries outside the pool name no tokens, slots outside the cache are empty
    s.cache.table[0, 1] = -1
    s.cache.table[7, 0] = 10 ** 6
    again, l2 = s.cache.attend(1, s.q, offsets=s.offsets, slots=ints([7, 0, 99]), return_lse=True)
    assert torch.isfinite(again).all()
    assert (again[13:] == 0).all() and (l2[13:] == -math.inf).all()
    assert (l2[:13] < lse[:13]).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,kv,dim,page", [(8, 2, 128, 16), (8, 2, 64, 4), (4, 1, 40, 1)])
@pytest.mark.parametrize("chunks", [[1, 1]] + TILES)
@pytest.mark.parametrize("where", [[0], [-1], [3, 9], [0, 1, 2, 3, 4, 5, 6, 7, 8, -1]])
def test_attend_pages_outside_the_pool(P, dtype, heads, kv, dim, page, chunks, where):
    """A page number outside the pool names no tokens: the others' attention is as if its keys were hidden."""
    lens = [700, 260]
    s = Sequences(P, lens, chunks, heads, kv, dim, page, dtype, seed=26)
    for row, bad in ((0, -1), (1, s.cache.refs.numel())):
        for at in where:
            s.cache.table[row, at % -(-lens[row] // page)] = bad
    got = s.cache.attend(1, s.q, offsets=s.offsets, longest=max(chunks), return_lse=True)
    t0, u, scale = 0, U[dtype], dim ** -0.5
    for n, x, k, v in zip(lens, chunks, s.k, s.v):
        missing = [p // page in {at % -(-n // page) for at in where} for p in range(n)]
        hidden = torch.arange(n, device="cuda") > torch.arange(n - x, n, device="cuda")[:, None]
        hidden = (hidden | torch.tensor(missing, device="cuda")).repeat(heads // kv, 1)  # [group of queries, keys]
        for h in range(kv):
            at = slice(t0, t0 + x), slice(h * (heads // kv), (h + 1) * (heads // kv))
            q, kk, vv = s.q[at].double().transpose(0, 1).reshape(-1, dim), k[:, h].double(), v[:, h].double()
            score = (q @ kk.T.contiguous() * scale).masked_fill(hidden, -math.inf)
            want = torch.logsumexp(score, 1)
            w = torch.exp(score - want[:, None])
            o, size = w @ vv, w @ vv.abs()
            es = (dim + 8) * 2.0 ** -24 * scale * (q.abs() @ kk.abs().T.contiguous()).amax(1)
            # (fp16 weights are held to 2^-25 under a highest one of 2^7 or more)
            tol = u * (size + o.abs()) + (torch.exp(2 * es) - 1 + (n + 16) * 2.0 ** -24)[:, None] * size + (
                2.0 ** -32 * vv.abs().sum(0) if dtype is torch.float16 else 0) + 1e-30
            y, z = (g[at].transpose(0, 1).flatten(0, 1).double() for g in got)
            assert ((y - o).abs() <= tol).all()
            assert ((z - want).abs() <= es + (n + 16) * 2.0 ** -24 + 4 * 2.0 ** -24 * want.abs()).all()
        t0 += x


@pytest.mark.parametrize("heads,kv,dim", [(8, 2, 128), (16, 1, 64)])
@pytest.mark.parametrize("lens,chunks", [([700, 3000, 90], [130, 40, 90]), ([64, 33, 500], [1, 1, 4])])
def test_attend_hints(P, heads, kv, dim, lens, chunks):
    """`longest` chooses tiles of 16, 128 and 256 rows; the result agrees whichever it is, below the rows' length too."""
    s = Sequences(P, lens, chunks, heads, kv, dim, 16, torch.bfloat16, seed=27)
    for longest in (1, 2, 5, 8, 20, 33, 70, 200, 5000):
        s.check(longest=longest)


@pytest.mark.parametrize("chunks", [[1, 1, 1], [60, 200, 1]])
def test_attend_large_and_equal_scores(P, chunks):
    """Scores far apart (one weight is 1, the others underflow) and all the same."""
    s = Sequences(P, [300, 250, 64], chunks, 8, 2, 128, 16, torch.bfloat16, seed=7)
    s.q.mul_(30)
    s.check()
    s.q.zero_()
    s.check()
    s.q.fill_(-1e4)
    out, lse = s.cache.attend(1, s.q, offsets=s.offsets, return_lse=True)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()


def test_attend_orders_of_the_pool(P):
    """Tokens before heads in a page, as a view of the pool."""
    s = Sequences(P, [100, 33], [20, 1], 8, 2, 64, 16, torch.bfloat16, seed=8)
    want = s.check()
    other = s.cache.data.transpose(2, 3).contiguous().transpose(2, 3)
    c = s.cache
    c._chunk.page_stride, c._chunk.head_stride, c._chunk.token_stride = other.stride(1), other.stride(2), other.stride(3)
    c._pages.data, c._pages.plane_stride = other.data_ptr(), other.stride(0) * 2
    got = c.attend(1, s.q, offsets=s.offsets, return_lse=True)
    for a, b in zip(want, got):
        assert torch.equal(a, b)


def test_attend_out_strides_and_untouched_memory(P):
    s = Sequences(P, [100, 33, 8], [20, 1, 3], 8, 2, 64, 16, torch.bfloat16, seed=9)
    want, _ = s.check()
    wide = torch.full((30, 8, 72), 7.0, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros((30, 8, 64), dtype=torch.bfloat16, device="cuda")
    q[2:26] = s.q
    s.cache.attend(1, q, offsets=s.offsets + 2, out=wide[:, :, :64])
    assert torch.equal(wide[2:26, :, :64], want)
    wide[2:26, :, :64] = 7.0
    assert (wide == 7.0).all()


def test_attend_offsets_past_32_bits(P):
    """Pages whose elements lie beyond 2^31 from the pool's start."""
    s = Sequences(P, [300, 70], [3, 1], 8, 8, 128, 64, torch.bfloat16, seed=10, far=(2 ** 31) // (8 * 128 * 64) + 5)
    s.check()


def test_attend_off_the_current_stream(P):
    s = Sequences(P, [5000, 70], [3, 1], 8, 2, 128, 16, torch.bfloat16, seed=11)
    want = s.check()
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = s.cache.attend(1, s.q, offsets=s.offsets, return_lse=True, stream=other)
    other.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)


def test_step_in_a_graph(P):
    """The whole step captured and replayed with eager work between the replays."""
    s = Sequences(P, [500, 70, 9], [1, 1, 1], 8, 2, 128, 16, torch.bfloat16, seed=12, spare=40)
    c = s.cache
    c.refs.copy_(torch.bincount(c.table[c.table < 2 ** 20].long(), minlength=c.refs.numel()).int())
    slots, counts, keep = ints([0, 1, 2]), ints([1, 1, 1]), ints([499, 69, 8])
    x = torch.randn((3, 5000), generator=gen(3), device="cuda").to(torch.bfloat16)
    x0, tokens = x.clone(), ints([[1, 2, 3]] * 3)
    presence = torch.ones(3, device="cuda")
    k, v = (torch.stack([z[-1] for z in w]) for w in (s.k, s.v))

    def step():
        c.fork(slots, slots, keep)
        c.extend(slots, counts)
        c.store(1, k, v)
        out, lse = c.attend(1, s.q, return_lse=True)
        P.adjust_logits(x, tokens=tokens, presence=presence)
        return out, lse

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    s.compare(*step(), 128 ** -0.5)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = step()
    want = x0.clone()
    P.adjust_logits(want, tokens=tokens, presence=presence)
    for _ in range(4):
        out.zero_()
        lse.zero_()
        x.copy_(x0)
        graph.replay()
        torch.cuda.synchronize()
        s.compare(out, lse, 128 ** -0.5)
        assert torch.equal(x, want)
        torch.randn(1000, device="cuda").sum().item()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("kv,dim,page", [(1, 8, 1), (8, 128, 16), (3, 40, 4)])
def test_store(P, dtype, kv, dim, page):
    lens, chunks = [40, 9, 3, 200, 64, 5], [1, 0, 3, 33, 64, 5]
    s = Sequences(P, lens, chunks, kv, kv, dim, page, dtype, seed=13, garbage=7.0)
    T = sum(chunks)
    new = torch.randn((T, 2 * kv * dim + 16), generator=gen(4), device="cuda").to(dtype)
    k, v = new[:, :kv * dim].unflatten(1, (kv, dim)), new[:, kv * dim + 8:2 * kv * dim + 8].unflatten(1, (kv, dim))
    want = s.cache.data.clone()
    length = [40, 9, 2, 200, 64, 5]  # the third row's first token has no place
    table = s.cache.table.clone()
    s.cache.length.copy_(ints(length))
    s.cache.table[5, 0] = -1  # and the last row's first page is not there
    t = 0
    for i, x in enumerate(chunks):
        for j in range(x):
            p = length[i] - x + j
            if p >= 0 and not (i == 5 and p // page == 0):
                want[0, int(table[i, p // page]), :, p % page] = k[t]
                want[1, int(table[i, p // page]), :, p % page] = v[t]
            t += 1
    s.cache.store(0, k, v, offsets=s.offsets)
    assert torch.equal(s.cache.data.view(torch.int16), want.view(torch.int16))


def test_chunk_refusals(P):
    s = Sequences(P, [100, 33], [20, 1], 8, 2, 64, 16, torch.bfloat16, seed=14)
    c, q = s.cache, s.q
    bad = [dict(layer=2, q=q), dict(layer=-1, q=q), dict(layer=0, q=q.float()), dict(layer=0, q=q[:, :7]),
           dict(layer=0, q=q[:, :, :32]), dict(layer=0, q=q.transpose(1, 2)), dict(layer=0, q=q.cpu()),
           dict(layer=0, q=q, offsets=s.offsets.long()), dict(layer=0, q=q, offsets=s.offsets, slots=ints([0])),
           dict(layer=0, q=q), dict(layer=0, q=q, offsets=s.offsets, scale=0.0),
           dict(layer=0, q=q, offsets=s.offsets, scale=float("nan")),
           dict(layer=0, q=q, offsets=s.offsets, out=torch.empty_like(q)[:, :4]),
           dict(layer=0, q=torch.zeros((21, 8, 68), dtype=q.dtype, device="cuda")[:, :, :64], offsets=s.offsets)]
    for kw in bad:
        with pytest.raises(P.TamError):
            c.attend(**kw)
    for kw in (dict(k=s.k[0][:21], v=s.v[0][:20]), dict(k=s.k[0][:21, :1], v=s.v[0][:21, :1]),
               dict(k=s.k[0][:21].half(), v=s.v[0][:21])):
        with pytest.raises(P.TamError):
            c.store(0, offsets=s.offsets, **kw)
    empty = c.attend(0, q[:0], offsets=ints([0, 0, 0]))
    assert empty.shape == (0, 8, 64)
    big = P.PageCache.empty(1, 1, 136, 4, 1, 4)
    with pytest.raises(P.TamError):
        big.attend(0, torch.zeros((1, 1, 136), dtype=torch.bfloat16, device="cuda"))


def test_attend_one_token_of_any_stride(P):
    """The strides of an axis of one element say nothing."""
    s = Sequences(P, [50], [1], 8, 2, 64, 16, torch.bfloat16, seed=15)
    out, lse = s.check()
    q = s.q.contiguous().as_strided((1, 8, 64), (1, 64, 1))
    got = s.cache.attend(1, q, offsets=s.offsets, return_lse=True)
    assert torch.equal(got[0], out) and torch.equal(got[1], lse)


@pytest.mark.parametrize("x", [1, 70])
def test_attend_small_fp16_weights(P, x):
    """One key far above many: weights of 2^-27 are under fp16's range, and their sum is not."""
    n, dim, scale = 60000, 64, 64 ** -0.5
    s = Sequences(P, [n], [x], 4, 2, dim, 16, torch.float16, seed=16)
    k, v = s.k[0], s.v[0]
    s.q.fill_(1)
    k.zero_()
    k[77] = 27 * math.log(2) * 8 / 64  # its score
    v.fill_(1)
    v[77] = 0
    pos = torch.arange(n, device="cuda")
    to = s.cache.table[0, pos // 16].long()
    s.cache.data[2][to, :, pos % 16] = k
    s.cache.data[3][to, :, pos % 16] = v
    out, lse = s.cache.attend(1, s.q, offsets=s.offsets, scale=scale, return_lse=True)
    want, wl, _, ltol = s.reference(scale)
    # the highest weight is 2^7 or more and all are held to 2^-25: n 2^-32 in the sum, beside what weights and output round
    assert ((out.double() - want).abs() <= 2.0 ** -10 * want + n * 2.0 ** -32).all()
    assert ((lse.double() - wl).abs() <= ltol).all()


def test_beams_example(P):
    """The example's beams, found step by step, have the scores that whole sequences get in one chunk."""
    import examples.beams as E
    vocab = E.vocabulary()
    h = P.compile(E.STRINGS, vocab, device="cuda:0")
    ends = torch.tensor([t.endswith(b'"') for t in vocab], device="cuda")
    model = E.Decoder(len(vocab))
    prompts = [list(b"a prompt"), list(b"and one that is longer than a page of the cache")]
    found, cache = E.search(model, h, ends, prompts, width=4)
    assert (cache.refs == 0).all() and (cache.length == 0).all()
    for prompt, beams in zip(prompts, found):
        assert beams and beams == sorted(beams, key=lambda x: -x[0])
        for score, tokens in beams:
            assert b"".join(vocab[t] for t in tokens)[:-1] in E.STRINGS
            T, n = len(prompt) + len(tokens) - 1, len(tokens)
            whole = ints(prompt + tokens)
            one = P.PageCache.empty(len(model.layers), 2, 64, 8, 1, 8)
            one.extend(ints([0]), ints([T]))
            logits = model(whole[:T], one, ints([0]), ints([0, T]), T)[len(prompt) - 1:]
            nodes = [ints([0])]
            for t in tokens[:-1]:
                nodes.append(h.advance(nodes[-1], ints([t])))
            at = ints(range(len(prompt), len(prompt) + n))
            h.adjust_logits(torch.cat(nodes), logits, tokens=whole.expand(n, -1).contiguous(), length=at,
                            prompt=torch.full_like(at, len(prompt)), presence=torch.full((n,), 0.3, device="cuda"))
            want = torch.log_softmax(logits.float(), 1)[torch.arange(n), tokens].sum()
            # logits of size 1 from bf16 layers, a few roundings of 2^-8 each
            assert abs(float(want) - score) <= 0.03 * n
    h.close()


def test_attend_refuses_outputs_that_overlap(P):
    s = Sequences(P, [100, 33], [20, 1], 8, 2, 64, 16, torch.bfloat16, seed=23)
    one = torch.zeros((1, 1, 64), dtype=torch.bfloat16, device="cuda")
    for out in (one.expand(21, 8, 64), torch.zeros((1, 8, 64), dtype=torch.bfloat16, device="cuda").expand(21, 8, 64),
                torch.zeros((21, 1, 64), dtype=torch.bfloat16, device="cuda").expand(21, 8, 64)):
        with pytest.raises(P.TamError):
            s.cache.attend(1, s.q, offsets=s.offsets, out=out)
    with pytest.raises(P.TamError):
        P.PageCache(s.cache.data[:1].expand(2, -1, -1, -1, -1), s.cache.table, s.cache.length, s.cache.refs)
    heads_first = torch.zeros((8, 21, 64), dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    assert torch.equal(s.cache.attend(1, s.q, offsets=s.offsets, out=heads_first), s.cache.attend(1, s.q, offsets=s.offsets))
    # pages before planes
    data = s.cache.data.transpose(0, 1).contiguous().transpose(0, 1)
    c = P.PageCache(data, s.cache.table, s.cache.length, s.cache.refs)
    assert torch.equal(c.attend(1, s.q, offsets=s.offsets), s.cache.attend(1, s.q, offsets=s.offsets))
