"""Trees of drafted tokens and the best tokens, against plain implementations in 64 bits.

Tolerances.  u is half a step of the type relative to the value: 2^-8 (bf16), 2^-11 (fp16), 2^-24 (fp32).
* Rotation: the fraction of a turn is at most half a turn, rounded to fp32: 2^-26 turns, so 2 pi 2^-26 < 2^-23 radians;
  sine and cosine add 4 ulp of values up to 1, 2^-22; two products and their sum 3 roundings of 2^-24.  So each of
  x cos - y sin and y cos + x sin is off by less than (|x| + |y|) 2^-21 before it is rounded to the type, and half of
  fp16's smallest step is 2^-25.
* Attention: as for attention without a mask (test_gpu_step.py), over the keys that are seen.
* Log probabilities: the exponentials (2 ulp and the argument's rounding, |x - m| <= 2^7 where they count: 2^-16 of
  what is under e^-88, less than 2^-20 weighted by e^(x - m)) and their sums in a tree of 2^8 levels at most (each thread
  adds up to 128 in turn): (128 + 32) 2^-24 of the sum; log, its sum with the maximum and the difference: 3 roundings
  of the largest of them.
"""
import math

import numpy as np
import pytest

from test_gpu_step import HEADS, TILES, U, P, Sequences, gen, ints  # noqa: F401 (P: a fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DTYPES = [torch.bfloat16, torch.float16]


def forest(rng, n, bushy=1.0, odd=0.0):
    """Parents of n tokens; `odd`: the share that names no earlier token."""
    p = [-1] + [int(rng.integers(max(0, int(j * (1 - bushy))), j)) for j in range(1, n)]
    for j in range(n):
        if rng.random() < odd:
            p[j] = int(rng.choice([-1, -7, j, j + 1, n, 2 ** 31 - 1, -2 ** 31]))
    return p[:n]


def sees(parents):
    """[n, n]: which tokens each one sees, and their depths."""
    n = len(parents)
    m, depth = np.zeros((n, n), bool), [0] * n
    for j, p in enumerate(parents):
        if 0 <= p < j:
            m[j] = m[p]
            depth[j] = depth[p] + 1
        m[j, j] = True
    return m, depth


def packed(m, words):
    """Bits of a [n, any] matrix in rows of int64 words."""
    out = np.zeros((m.shape[0], words * 64), np.uint8)
    w = min(m.shape[1], words * 64)
    out[:, :w] = m[:, :w]
    return np.packbits(out, axis=1, bitorder="little").view(np.int64)


# ----------------------------------------------------------------- masks -------

@pytest.mark.parametrize("rows", [[1], [0], [5], [64], [65, 0, 1, 63], [130, 2, 300, 7, 0], [257] * 3, [1] * 200, [0, 0, 3]])
@pytest.mark.parametrize("bushy,odd", [(1.0, 0.0), (0.05, 0.0), (1.0, 0.2)])
def test_tree_masks(P, rows, bushy, odd):
    rng = np.random.default_rng(sum(rows) + int(10 * bushy))
    trees = [forest(rng, n, bushy, odd) for n in rows]
    off = ints(np.concatenate([[0], np.cumsum(rows)]).astype(np.int32))
    up = ints(sum(trees, []))
    for longest in (None, max(rows), 700, 64):
        seen, depth = P.tree_masks(up, off, longest=longest)
        words = max(1, -(-(sum(rows) if longest is None else longest) // 64))
        assert seen.shape == (sum(rows), words) and seen.dtype is torch.int64 and depth.dtype is torch.int32
        t = 0
        for p in trees:
            m, d = sees(p)
            assert np.array_equal(seen[t:t + len(p)].cpu().numpy(), packed(m, words))
            assert depth[t:t + len(p)].tolist() == d
            t += len(p)


def test_tree_masks_of_long_rows(P):
    """Rows that LDS does not hold, one of them a single chain."""
    rng = np.random.default_rng(0)
    trees = [forest(rng, 4097), list(range(-1, 4999))]
    off = ints([0, 4097, 4097 + 5000])
    seen, depth = P.tree_masks(ints(trees[0] + trees[1]), off, longest=5000)
    for p, lo in zip(trees, (0, 4097)):
        m, d = sees(p)
        assert np.array_equal(seen[lo:lo + len(p)].cpu().numpy(), packed(m, seen.shape[1]))
        assert depth[lo:lo + len(p)].tolist() == d


def test_tree_masks_without_rows_and_outside_them(P):
    seen, depth = P.tree_masks(ints([-1, 0, 5]))
    assert seen.tolist() == [[1]] * 3 and depth.tolist() == [0] * 3
    up = ints([-1, 0, -1, 0, 1, 0])
    out, deep = torch.full((6, 2), 77, dtype=torch.int64, device="cuda"), ints([77] * 6)
    off = ints([1, 4])
    rc = P.lib().tam_tree_masks(up.data_ptr(), off.data_ptr(), 1, 6, out.data_ptr(), 2, deep.data_ptr(),
                                torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    assert out.tolist() == [[77, 77], [1, 0], [2, 0], [5, 0], [77, 77], [77, 77]] and deep.tolist() == [77, 0, 0, 1, 77, 77]
    seen, depth = P.tree_masks(up[:0], ints([0, 0]))
    assert seen.shape == (0, 1) and depth.numel() == 0


# ---------------------------------------------------------------- append -------

def turned(x, position, frequencies, adjacent):
    """(turned, bound on the error before it is rounded) of x [T, heads, dim], in 64 bits."""
    x = x.double()
    n = frequencies.numel()
    angle = (position.double()[:, None] * frequencies.double())[:, None]
    c, s = torch.cos(angle), torch.sin(angle)
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if adjacent else (slice(0, n), slice(n, 2 * n))
    y, bound = x.clone(), torch.zeros_like(x)
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    bound[..., first] = bound[..., second] = (a.abs() + b.abs()) * 2.0 ** -21
    return y, bound


def close(got, want, bound, dtype):
    small = 2.0 ** -25 if dtype is torch.float16 else 1e-38
    return bool(((got.double() - want).abs() <= bound + U[dtype] * (want.abs() + bound) + small).all())


def check_append(P, heads, kv, dim, page, dtype, pairs, adjacent, chunks, lens, depth=True, in_place=False, queries=True, seed=0):
    s = Sequences(P, lens, chunks, heads, kv, dim, page, dtype, seed=seed, garbage=0.5)
    c, T = s.cache, sum(chunks)
    g = gen(seed + 1)
    rng = np.random.default_rng(seed)
    k = torch.randn((T, kv * dim + 8), generator=g, device="cuda").to(dtype)[:, 8:].unflatten(1, (kv, dim))
    v = torch.randn((kv, T, dim), generator=g, device="cuda").to(dtype).transpose(0, 1)
    f = torch.as_tensor(10000.0 ** -(np.arange(pairs) / max(pairs, 1)), dtype=torch.float32, device="cuda")
    begin = torch.tensor([n - x for n, x in zip(lens, chunks) for _ in range(x)], device="cuda")
    at = torch.tensor([j for x in chunks for j in range(x)], device="cuda")
    deep = ints(rng.integers(0, 40, T).astype(np.int32)) if depth else None
    if depth and T > 2:
        deep[1], deep[2] = 2 ** 30, -5
    before = c.data.clone()
    q = s.q.clone() if in_place else s.q
    out = c.append(0, q if queries else None, k, v, f, depth=deep, adjacent=adjacent, offsets=s.offsets,
                   out=q if in_place else None)
    position = begin + (deep if depth else at)
    if queries:
        want, bound = turned(s.q, position, f, adjacent)
        assert out.shape == s.q.shape and (not in_place or out is q)
        assert close(out, want, bound, dtype)
        assert torch.equal(out[..., 2 * pairs:], s.q[..., 2 * pairs:])
    else:
        assert out is None
    want, bound = turned(k, position, f, adjacent)
    table = c.table.long()
    row = torch.tensor([i for i, x in enumerate(chunks) for _ in range(x)], device="cuda")
    place = begin + at
    to = table[row, place // page]
    assert close(c.data[0][to, :, place % page], want, bound, dtype)
    assert torch.equal(c.data[0][to, :, place % page][..., 2 * pairs:], k[..., 2 * pairs:])
    assert torch.equal(c.data[1][to, :, place % page], v)
    after = c.data.clone()
    for plane in (0, 1):
        after[plane][to, :, place % page] = before[plane][to, :, place % page]
    assert torch.equal(after.view(torch.int16), before.view(torch.int16))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("heads,kv,dim,pairs", [(8, 8, 64, 32), (8, 2, 128, 64), (16, 1, 128, 32), (6, 2, 96, 48), (5, 5, 40, 20), (7, 1, 8, 4),
                                                (12, 4, 120, 12), (3, 3, 64, 0), (40, 1, 64, 28), (1, 1, 8, 0)])
def test_append(P, dtype, adjacent, heads, kv, dim, pairs):
    chunks = [1, 0, 7, 33, 64, 0, 5]
    lens = [40, 9, 7, 200, 64, 0, 1500]
    check_append(P, heads, kv, dim, 16, dtype, pairs, adjacent, chunks, lens)
    check_append(P, heads, kv, dim, 1, dtype, pairs, adjacent, [3, 1], [90, 1], depth=False, in_place=True, seed=3)
    check_append(P, heads, kv, dim, 64, dtype, pairs, adjacent, [2], [70], queries=False, seed=4)


def test_append_single_tokens_and_many_rows(P):
    lens = [1, 2, 17, 300, 5]
    s = Sequences(P, lens, [1] * 5, 8, 2, 64, 4, torch.bfloat16, garbage=0.25)
    f = torch.rand(32, generator=gen(2), device="cuda")
    k = torch.randn((5, 2, 64), generator=gen(3), device="cuda").to(torch.bfloat16)
    out = s.cache.append(1, s.q, k, k, f)
    want, bound = turned(s.q, torch.tensor(lens, device="cuda") - 1, f, False)
    assert close(out, want, bound, torch.bfloat16)
    rng = np.random.default_rng(1)
    for rows in (65, 300, 5000):  # offsets found in several turns, empty rows among them
        chunks = rng.integers(0, 3, rows).tolist()
        chunks[0] = chunks[-1] = 0
        check_append(P, 2, 1, 16, 8, torch.float16, 8, False, chunks, [x + int(rng.integers(0, 4)) for x in chunks], seed=rows)


def test_append_tokens_without_a_place(P):
    """A position under 0, a page outside the pool, a slot outside the cache, tokens of no row: nothing is stored, and
    queries of a row's tokens turn all the same."""
    s = Sequences(P, [3, 40, 20, 8], [5, 4, 2, 2], 4, 2, 32, 16, torch.bfloat16, garbage=1.0)
    c, T = s.cache, 13 + 3
    c.table[1, 2] = 99
    q, k, v = (torch.randn((T, h, 32), generator=gen(h), device="cuda").to(torch.bfloat16) for h in (4, 2, 2))
    c.length[0] = 3
    slots = ints([0, 1, -1, 4])
    off = ints([1, 6, 10, 12, 14])
    out = torch.full_like(q, 7.0)
    before = c.data.clone()
    f = torch.rand(16, generator=gen(5), device="cuda")
    c.append(0, q, k, v, f, offsets=off, slots=slots, out=out)
    assert (out[0] == 7).all() and (out[14:] == 7).all()
    position = torch.tensor([0, -2, -1, 0, 1, 2, 36, 37, 38, 39, -2, -1, -2, -1, 0, 0], device="cuda")
    want, bound = turned(q, position, f, False)
    assert close(out[1:14], want[1:14], bound[1:14], torch.bfloat16)
    page = int(c.table[0, 0])
    kk, kb = turned(k, position, f, False)
    assert close(c.data[0, page, :, :3].transpose(0, 1), kk[3:6], kb[3:6], torch.bfloat16)
    assert torch.equal(c.data[1, page, :, :3].transpose(0, 1), v[3:6])
    after = c.data.clone()
    after[:2, page, :, :3] = before[:2, page, :, :3]
    assert torch.equal(after, before)


def test_append_is_store_without_pairs(P):
    s = Sequences(P, [100, 33], [20, 1], 8, 2, 64, 16, torch.float16, seed=14, garbage=0.0)
    k, v = (torch.randn((21, 2, 64), generator=gen(i), device="cuda").half() for i in (1, 2))
    s.cache.store(0, k, v, offsets=s.offsets)
    want = s.cache.data.clone()
    s.cache.data[:2] = 0
    out = s.cache.append(0, s.q, k, v, torch.empty(0, device="cuda"), offsets=s.offsets)
    # (what lay in the places of no token was 0)
    assert torch.equal(s.cache.data[:2], want[:2]) and torch.equal(out, s.q)


def test_append_far_positions_and_special_values(P):
    s = Sequences(P, [64], [64], 1, 1, 16, 16, torch.float16, garbage=0.0)
    f = torch.tensor([1.0, 0.7, 1e-3, 3.0, 0.0, 100.0, -1.0, 1e-30], device="cuda")
    depth = ints([int(x) for x in np.random.default_rng(0).integers(-2 ** 30, 2 ** 30, 64)])
    x = torch.randn((64, 1, 16), generator=gen(1), device="cuda").half()
    out = s.cache.append(0, x, x, x, f, depth=depth, offsets=s.offsets)
    # a turn of 2^30 * 100 radians is known to 2^37 2^-53 turns
    want, bound = turned(x, depth, f, False)
    assert close(out, want, bound + 2.0 ** -15 * 6.3, torch.float16)
    assert close(out[..., [1, 2, 4, 9, 10, 12]], want[..., [1, 2, 4, 9, 10, 12]], bound[..., [1, 2, 4, 9, 10, 12]] + 2.0 ** -20, torch.float16)
    x[0, 0, 3], x[1, 0, 5], x[2, 0, 0] = math.inf, math.nan, 6e-8
    out = s.cache.append(0, x, x, x, f, offsets=s.offsets)
    assert not torch.isfinite(out[0, 0, [3, 11]]).any() and torch.isfinite(out[0, 0, [0, 1, 2, 4, 5, 6, 7, 8, 9, 10]]).all()
    assert out[1, 0, [5, 13]].isnan().all() and torch.isfinite(out[2:]).all()


# ------------------------------------------------------------- attention -------

class Trees(Sequences):
    """Sequences whose chunks are seen through a mask."""

    def __init__(self, P, lens, chunks, *args, mask="tree", words=None, seed=0, **kw):
        super().__init__(P, lens, chunks, *args, seed=seed, **kw)
        rng = np.random.default_rng(seed + 99)
        self.m = []
        for n in chunks:
            if mask == "tree":
                m = sees(forest(rng, n, rng.choice([0.1, 1.0])))[0]
            elif mask == "chain":
                m = np.tril(np.ones((n, n), bool))
            else:
                m = rng.random((n, n)) < rng.choice([0.0, 0.1, 0.5, 1.0], (n, 1))
            self.m.append(m)
        words = words or max(1, -(-max(chunks + [1]) // 64))
        # bits of tokens that a row does not have are set
        full = [np.pad(m, ((0, 0), (0, max(0, 64 * words - m.shape[1]))), constant_values=True) for m in self.m]
        self.seen = torch.as_tensor(np.concatenate([packed(m, words) for m in full] + [np.zeros((0, words), np.int64)]), device="cuda")
        for m in self.m:
            m[:, 64 * words:] = False

    def reference(self, scale):
        out, lse, tol, ltol = [], [], [], []
        u = U[self.q.dtype]
        q = self.q.double()
        t = 0
        for n, x, k, v, m in zip(self.lens, self.chunks, self.k, self.v, self.m):
            kk = k.double().repeat_interleave(self.heads // self.kv, 1).permute(1, 0, 2)
            vv = v.double().repeat_interleave(self.heads // self.kv, 1).permute(1, 0, 2)
            qq = q[t:t + x].permute(1, 0, 2)
            t += x
            seen = torch.ones((x, n), dtype=torch.bool, device="cuda")
            # token j of the row lies at n - x + j; those under 0 lie nowhere
            some = min(n, x)
            seen[:, n - some:] = torch.as_tensor(m[:, x - some:], device="cuda")
            s = (qq @ kk.transpose(1, 2) * scale).masked_fill(~seen, -math.inf)
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

    def check(self, **kw):
        return super().check(seen=self.seen, **kw)


# rows under 17, 33, 65, 129 and 257 of a K/V head's tile, and more
CHUNKS = [[1, 1], [4, 2], [3, 7, 8], [20, 30], [64, 1, 0, 33], [200, 90], [129, 257]]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,kv,dim", HEADS)
@pytest.mark.parametrize("mask", ["tree", "any"])
def test_attend_seen(P, dtype, heads, kv, dim, mask):
    for i, chunks in enumerate(CHUNKS):
        lens = [x + [0, 40, 513, 7][(i + j) % 4] for j, x in enumerate(chunks)]
        s = Trees(P, lens, chunks, heads, kv, dim, [16, 1, 64, 8][i % 4], dtype, mask=mask, seed=i)
        s.check()
        s.check(longest=max(chunks))


@pytest.mark.parametrize("heads,kv,dim,page", [(8, 2, 128, 16), (4, 4, 64, 32), (32, 4, 128, 8)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_attend_seen_over_long_rows(P, heads, kv, dim, page, dtype):
    """The tree beyond the cuts of a long axis, and cuts inside the tree."""
    Trees(P, [20011, 9, 4097], [4, 2, 1], heads, kv, dim, page, dtype, seed=2).check(longest=4)
    Trees(P, [9000, 50, 1023, 3000], [30, 50, 17, 0], heads, kv, dim, page, dtype, seed=3).check(longest=50)
    Trees(P, [3000, 900], [500, 900], heads, kv, dim, page, dtype, mask="any", seed=4).check()


@pytest.mark.parametrize("chunks", CHUNKS)
def test_attend_seen_chain_is_causal(P, chunks):
    s = Trees(P, [x + 100 for x in chunks], chunks, 8, 2, 64, 16, torch.bfloat16, mask="chain", seed=5)
    out, lse = s.check()
    plain = s.cache.attend(1, s.q, offsets=s.offsets, return_lse=True)
    s.compare(*plain, s.dim ** -0.5)


@pytest.mark.parametrize("chunks", CHUNKS)
@pytest.mark.parametrize("dim", [64, 128])
def test_attend_seen_rows_that_see_nothing(P, chunks, dim):
    s = Trees(P, chunks, chunks, 8, 2, dim, 16, torch.float16, mask="any", seed=6)
    for m in s.m:
        m[::2] = False
    s.seen = torch.as_tensor(np.concatenate([packed(m, s.seen.shape[1]) for m in s.m]), device="cuda")
    out, lse = s.check()
    t = 0
    for m in s.m:
        assert not out[t:t + len(m):2].any() and (lse[t:t + len(m):2] == -math.inf).all()
        t += len(m)


@pytest.mark.parametrize("chunks,words", [([100, 70], 1), ([300, 3], 2), ([10, 5], 4)])
def test_attend_seen_words_and_strides(P, chunks, words):
    """Masks narrower and wider than the rows, and rows of a wider tensor."""
    s = Trees(P, [x + 33 for x in chunks], chunks, 8, 2, 64, 16, torch.bfloat16, mask="any", words=words, seed=7)
    a = s.check()
    wide = torch.full((s.seen.shape[0], words + 3), -1, dtype=torch.int64, device="cuda")
    wide[:, 1:1 + words] = s.seen
    s.seen = wide[:, 1:1 + words]
    for x, y in zip(a, s.check()):
        assert torch.equal(x, y)


def test_attend_seen_sequences_shorter_than_their_rows(P):
    """A length below the row's tokens: the first ones lie nowhere and see what the mask says of the rest."""
    for chunks in ([6, 4], [40, 9], [300, 5]):
        s = Trees(P, [x + 20 for x in chunks], chunks, 8, 2, 64, 16, torch.bfloat16, mask="any", seed=8)
        short = [chunks[0] - 2, 0]
        s.cache.length.copy_(ints(short))
        s.k, s.v = [k[:n] for k, n in zip(s.k, short)], [v[:n] for v, n in zip(s.v, short)]
        s.lens = short
        s.check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,kv,dim,page", [(8, 2, 128, 16), (8, 2, 64, 4), (4, 1, 40, 16), (16, 4, 120, 1)])
@pytest.mark.parametrize("chunks", TILES)
def test_attend_seen_hidden_values(P, dtype, heads, kv, dim, page, chunks):
    """K and V of a token that some see and others do not, and of one that nobody sees: NaN and infinities reach those alone
    that see them."""
    lens = [x + 517 for x in chunks]
    s = Trees(P, lens, chunks, heads, kv, dim, page, dtype, mask="tree", seed=9)
    clean, _ = s.check()
    row, n = 0, chunks[0]
    hidden = n - 1  # no parent: only itself sees it
    for kind, j, value in (("v", 1, math.inf), ("v", hidden, math.nan), ("k", hidden, math.nan), ("v", 1, -math.inf)):
        p = lens[row] - n + j
        plane = 2 if kind == "k" else 3
        place = (plane, int(s.cache.table[row, p // page]), slice(None), p % page, 3)
        keep = s.cache.data[place].clone()
        s.cache.data[place] = value
        out, lse = s.cache.attend(1, s.q, offsets=s.offsets, return_lse=True, seen=s.seen)
        reaches = torch.as_tensor(s.m[row][:, j], device="cuda")
        got = out[:n]
        if kind == "v":
            assert not torch.isfinite(got[reaches][..., 3]).any()
            others = [d for d in range(dim) if d != 3]
            assert torch.isfinite(got[reaches][..., others]).all()
        assert torch.equal(got[~reaches].view(torch.int16), clean[:n][~reaches].view(torch.int16))
        assert torch.equal(out[n:].view(torch.int16), clean[n:].view(torch.int16))
        s.cache.data[place] = keep


@pytest.mark.parametrize("chunks", [[1, 1]] + TILES)
def test_attend_seen_pages_outside_the_pool(P, chunks):
    """Keys in pages that are not there are not seen, among the row's tokens too."""
    s = Trees(P, [x + 200 for x in chunks], chunks, 8, 2, 64, 16, torch.bfloat16, mask="any", seed=10)
    s.cache.table[0, 3] = -1
    last = (s.lens[0] - 1) // 16
    s.cache.table[0, last] = 10 ** 6
    gone = [p for p in range(s.lens[0]) if p // 16 in (3, last)]
    out, lse = s.cache.attend(1, s.q, offsets=s.offsets, return_lse=True, seen=s.seen)
    # the same without those keys: their scores are -inf
    n, x = s.lens[0], chunks[0]
    keep = [p for p in range(n) if p not in gone]
    seen = np.concatenate([np.ones((x, n - x), bool), s.m[0]], 1)[:, keep]
    q, k, v = s.q[:x].double(), s.k[0][keep].double(), s.v[0][keep].double()
    for h in range(8):
        score = (q[:, h] @ k[:, h // 4].T * 64 ** -0.5).masked_fill(~torch.as_tensor(seen, device="cuda"), -math.inf)
        want = torch.softmax(score, 1) @ v[:, h // 4]
        a = torch.softmax(score, 1) @ v[:, h // 4].abs()
        assert ((out[:x, h].double() - want).abs() <= 2.0 ** -8 * (a + want.abs()) + 2.0 ** -13 * a).all()


def test_attend_seen_slots_and_far_pages(P):
    s = Trees(P, [300, 40, 77], [20, 1, 30], 8, 2, 128, 16, torch.bfloat16, seed=11, slots=[4, 0, 2])
    s.check()
    Trees(P, [500, 90], [17, 40], 8, 8, 128, 64, torch.bfloat16, seed=12, far=70000).check()


def test_attend_seen_off_the_current_stream(P):
    s = Trees(P, [300, 40], [20, 9], 8, 2, 64, 16, torch.bfloat16, seed=13)
    want = s.check()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    up = ints(forest(np.random.default_rng(0), 29))
    masks = P.tree_masks(up, ints([0, 29]), stream=side)
    best = P.top_tokens(s.q.float().flatten(1), 5, stream=side)
    got = s.cache.attend(1, s.q, offsets=s.offsets, return_lse=True, seen=s.seen, stream=side)
    torch.cuda.synchronize()
    for x, y in zip(got, want):
        assert torch.equal(x, y)
    for x, y in zip(masks, P.tree_masks(up, ints([0, 29]))):
        assert torch.equal(x, y)
    for x, y in zip(best, P.top_tokens(s.q.float().flatten(1), 5)):
        assert torch.equal(x, y)


# ---------------------------------------------------------------- accept -------

def accepted(parents, tokens, picks):
    path = [0] if parents else []
    while path:
        here = path[-1]
        then = [j for j in range(here + 1, len(parents)) if parents[j] == here and tokens[j] == picks[here] >= 0]
        if not then:
            break
        path.append(then[0])
    return path


def check_accept(P, rng, chunks, befores, page, kv=2, dim=16, layers=2, slots=None, bushy=1.0, likely=0.8, odd=0.0, spare=2):
    rows = len(chunks)
    slots = list(range(rows)) if slots is None else slots
    nslots = max(slots + [rows - 1]) + 1
    lens = [0] * nslots
    for s, n, b in zip(slots, chunks, befores):
        if s >= 0:
            lens[s] = n + b
    held = [-(-x // page) for x in lens]
    c = P.PageCache.empty(layers, kv, dim, sum(held) + spare, nslots, max(held) + 2, page_tokens=page)
    c.data.copy_(torch.randn(c.data.shape, generator=gen(int(rng.integers(1 << 30))), device="cuda"))
    ids = rng.permutation(sum(held) + spare)
    table, at = np.full((nslots, max(held) + 2), -1, np.int32), 0
    for s, h in enumerate(held):
        table[s, :h] = ids[at:at + h]
        at += h
    c.table.copy_(ints(table))
    c.length.copy_(ints(lens))
    refs = np.zeros(len(ids), np.int32)
    refs[ids[:at]] = 1
    if len(held) > 1 and held[0] > 1 and befores[0] >= page:  # a page of the text that others hold too
        refs[table[slots[0], 0]] = 3
    c.refs.copy_(ints(refs))
    trees, tokens, picks = [], [], []
    for n in chunks:
        p = forest(rng, n, bushy, odd)
        t = rng.integers(-1, 6, n).tolist()
        pick = rng.integers(-1, 6, n).tolist()
        for j in range(1, n):
            if 0 <= p[j] < j and rng.random() < likely:
                pick[p[j]] = t[j]
        trees.append(p), tokens.append(t), picks.append(pick)
    want = c.data.clone()
    paths, count, last = [], [], []
    for i, s in enumerate(slots):
        n = chunks[i]
        if s < 0 or s >= nslots:
            paths += [-1] * n
            count.append(0)
            last.append(-1)
            continue
        path = accepted(trees[i], tokens[i], picks[i])
        base = lens[s] - n
        for d, j in enumerate(path):
            a, b = base + j, base + d
            want[:, table[s, b // page], :, b % page] = c.data[:, table[s, a // page], :, a % page]
        if n:
            now = base + len(path)
            for x in range(-(-now // page), held[s]):
                refs[table[s, x]] -= 1
                table[s, x] = -1
            lens[s] = now
        paths += path + [-1] * (n - len(path))
        count.append(len(path))
        last.append(picks[i][path[-1]] if path else -1)
    off = ints(np.concatenate([[0], np.cumsum(chunks)]).astype(np.int32))
    got = c.accept(*(ints(sum(x, [])) for x in (tokens, picks, trees)), offsets=off, slots=ints(slots))
    assert got[0].tolist() == paths and got[1].tolist() == count and got[2].tolist() == last
    assert c.table.tolist() == table.tolist() and c.length.tolist() == lens and c.refs.tolist() == refs.tolist()
    assert torch.equal(c.data.view(torch.int16), want.view(torch.int16))
    return count


@pytest.mark.parametrize("page", [1, 4, 16, 64])
@pytest.mark.parametrize("bushy,likely,odd", [(1.0, 0.9, 0.0), (0.02, 0.99, 0.0), (0.3, 0.9, 0.2), (1.0, 0.2, 0.0)])
def test_accept(P, page, bushy, likely, odd):
    rng = np.random.default_rng(page + int(100 * bushy))
    most = 0
    for chunks in ([1], [9], [16, 0, 64, 1, 5], [65, 130, 7], [300, 2], [40] * 20):
        most = max(most, *check_accept(P, rng, chunks, rng.integers(0, 70, len(chunks)).tolist(), page, bushy=bushy, likely=likely, odd=odd))
    assert most > 3 or likely < 0.5


@pytest.mark.parametrize("kv,dim,layers", [(1, 8, 1), (8, 128, 3), (3, 40, 2), (7, 120, 1)])
def test_accept_layouts_and_slots(P, kv, dim, layers):
    rng = np.random.default_rng(dim)
    check_accept(P, rng, [30, 50, 3], [20, 5, 0], 8, kv=kv, dim=dim, layers=layers, slots=[4, 1, 2], bushy=0.1, likely=0.95)
    check_accept(P, rng, [12, 50], [20, 5], 16, kv=kv, dim=dim, layers=layers, slots=[-1, 0], bushy=0.1, likely=0.95)


@pytest.mark.parametrize("kv,dim,layers", [(8, 128, 9), (7, 120, 15), (136, 128, 64)])
def test_accept_of_many_layers(P, kv, dim, layers):
    """Caches whose walk and moves are launches of their own, from 2,049 pieces of 16 bytes per token on: in whole blocks of 256,
    with a last one that is not full, and more than 1,024 blocks, so that a thread takes several.  Of a row's tokens every
    second one stays (0, 2, 4, ..., the others are leaves), or all of them."""
    pieces = 2 * layers * kv * dim // 8
    assert pieces in (9 * 256, 3150) or pieces > 1024 * 256
    page = 8 if layers < 64 else 2
    rows = [(150, 5, 2), (0, 7, 2), (9, 0, 1), (1, 3, 2), (33, 12, 2)] if layers < 64 else [(17, 3, 2), (2, 0, 2), (5, 1, 1)]
    slots = [3, 0, 5, 1, 2] if layers < 64 else [2, 0, 1]
    c = P.PageCache.empty(layers, kv, dim, sum(-(-(n + b) // page) for n, b, _ in rows) + 1, 6, 20, page_tokens=page)
    for plane in c.data:
        plane.copy_(torch.randn(plane.shape, generator=gen(0), device="cuda"))
    ids = np.random.default_rng(layers).permutation(c.data.shape[1])
    table, length, refs, at = np.full((6, 20), -1, np.int32), np.zeros(6, np.int32), np.zeros(len(ids), np.int32), 0
    for s, (n, b, _) in zip(slots, rows):
        length[s] = n + b
        held = -(-(n + b) // page)
        table[s, :held] = ids[at:at + held]
        refs[ids[at:at + held]] = 1
        at += held
    c.table.copy_(ints(table))
    c.length.copy_(ints(length))
    c.refs.copy_(ints(refs))
    want, tokens, picks, up, path, count, last = c.data.clone(), [], [], [], [], [], []
    for s, (n, b, each) in zip(slots, rows):
        stay = list(range(0, n, each))
        up += [-1 if j == 0 else j - 1 - (j - 1) % each for j in range(n)]
        tokens += list(range(n))
        picks += [j + each if j % each == 0 else 3 for j in range(n)]
        path += stay + [-1] * (n - len(stay))
        count.append(len(stay))
        last.append(stay[-1] + each if n else -1)
        for d, j in enumerate(stay):
            want[:, table[s, (b + d) // page], :, (b + d) % page] = c.data[:, table[s, (b + j) // page], :, (b + j) % page]
        if n:
            length[s] = b + len(stay)
            for x in table[s, -(-length[s] // page):]:
                refs[x] -= x >= 0
            table[s, -(-length[s] // page):] = -1
    off = ints(np.concatenate([[0], np.cumsum([n for n, _, _ in rows])]).astype(np.int32))
    got = c.accept(ints(tokens), ints(picks), ints(up), offsets=off, slots=ints(slots))
    assert got[0].tolist() == path and got[1].tolist() == count and got[2].tolist() == last
    assert c.table.tolist() == table.tolist() and c.length.tolist() == length.tolist() and c.refs.tolist() == refs.tolist()
    assert torch.equal(c.data.view(torch.int16), want.view(torch.int16))


def test_accept_whole_chains_and_none(P):
    """A chain that stays whole moves nothing; a path longer than a wave; a root whose choice was not drafted."""
    c = P.PageCache.empty(1, 1, 8, 60, 3, 20, page_tokens=8)
    c.data.copy_(torch.randn(c.data.shape, generator=gen(0), device="cuda"))
    c.extend(ints([0, 1, 2]), ints([105, 33, 1]))
    before, table, refs = c.data.clone(), c.table.tolist(), c.refs.tolist()
    up = list(range(-1, 99)) + [-1] + [0] * 29 + [-1]
    token = [j + 1 for j in range(100)] + [7] * 30 + [3]
    pick = [j + 2 for j in range(100)] + [8] * 30 + [5]
    path, count, last = c.accept(ints(token), ints(pick), ints(up), offsets=ints([0, 100, 130, 131]))
    assert count.tolist() == [100, 1, 1] and last.tolist() == [101, 8, 5] and c.length.tolist() == [105, 4, 1]
    assert path.tolist() == list(range(100)) + [0] + [-1] * 29 + [0]
    assert torch.equal(c.data, before) and c.table[0].tolist() == table[0] and c.table[1].tolist()[:5] == table[1][:1] + [-1] * 4
    assert sum(c.refs.tolist()) == sum(refs) - 4
    # one token per row, without offsets
    path, count, last = c.accept(ints([1, 2, 3]), ints([4, 5, 6]), ints([-1, -1, -1]))
    assert path.tolist() == [0] * 3 and count.tolist() == [1] * 3 and last.tolist() == [4, 5, 6] and c.length.tolist() == [105, 4, 1]


def test_accept_places_that_are_not_there(P):
    """Lengths under the row's tokens and past the table, pages outside the pool: such tokens do not move."""
    c = P.PageCache.empty(1, 1, 8, 8, 3, 3, page_tokens=4)
    c.data.copy_(torch.randn(c.data.shape, generator=gen(1), device="cuda"))
    c.table.copy_(ints([[0, 1, 2], [3, 99, 4], [5, 6, 7]]))
    c.refs.fill_(1)
    c.length.copy_(ints([3, 12, 2 ** 30]))
    before = c.data.clone()
    up, token, pick = [-1, 0, 0, 2, 3] * 3, [0, 1, 2, 3, 4] * 3, [2, 0, 3, 4, 9] * 3
    path, count, last = c.accept(ints(token), ints(pick), ints(up), offsets=ints([0, 5, 10, 15]))
    assert path.tolist() == [0, 2, 3, 4, -1] * 3 and count.tolist() == [4] * 3 and last.tolist() == [9] * 3
    # row 0: its tokens lie at -2 .. 2; 2 -> place 1 of the row and so on: to -1, 0, 1 from 0, 1, 2
    want = before.clone()
    want[:, 0, :, 0], want[:, 0, :, 1] = before[:, 0, :, 1], before[:, 0, :, 2]
    # row 1: at 7 .. 11, the first of them in a page that is not there: to 8, 9, 10 from 9, 10, 11
    want[:, 4, :, :3] = before[:, 4, :, 1:]
    # row 2: a length of 12 at most
    want[:, 7, :, :3] = before[:, 7, :, 1:]
    assert torch.equal(c.data, want)
    assert c.length.tolist() == [2, 11, 11] and c.table.tolist() == [[0, 1, 2], [3, 99, 4], [5, 6, 7]]


def test_accept_of_millions_of_rows(P):
    """More rows than blocks of 1,024 threads in a launch, one token each and some in trees of three."""
    rows = 2 ** 22 + 3
    c = P.PageCache.empty(1, 1, 8, rows, rows, 1, page_tokens=4)
    page = torch.randperm(rows, generator=gen(0), device="cuda")
    c.data.copy_(torch.randn(c.data.shape, generator=gen(1), device="cuda"))
    c.table[:, 0] = page
    c.refs.fill_(1)
    n = torch.ones(rows, dtype=torch.int64, device="cuda")
    trees = torch.tensor([0, 1234567, rows - 1], device="cuda")
    n[trees] = 3
    c.length.copy_(n)
    off = torch.zeros(rows + 1, dtype=torch.int64, device="cuda")
    off[1:] = n.cumsum(0)
    first = off[:-1]
    tokens, picks, up = (torch.full((rows + 6,), x, dtype=torch.int32, device="cuda") for x in (5, 6, -1))
    for j, (token, pick, parent) in enumerate(((5, 8, -1), (7, 1, 0), (8, 9, 0))):  # the root's choice is token 2
        for x, y in zip((tokens, picks, up), (token, pick, parent)):
            x[first[trees] + j] = y
    want = c.data.clone()
    want[:, page[trees], :, 1] = c.data[:, page[trees], :, 2]
    path, count, last = c.accept(tokens, picks, up, offsets=off.int())
    assert torch.equal(c.data, want)
    in_tree = torch.zeros(rows, dtype=torch.bool, device="cuda")
    in_tree[trees] = True
    assert torch.equal(count, torch.where(in_tree, 2, 1).int()) and torch.equal(last, torch.where(in_tree, 9, 6).int())
    assert torch.equal(c.length, count) and torch.equal(c.table[:, 0].long(), page) and bool((c.refs == 1).all())
    want = torch.zeros_like(path)
    want[first[trees] + 1], want[first[trees] + 2] = 2, -1
    assert torch.equal(path, want)


def test_append_and_accept_past_32_bits(P):
    """Pages past 2^31 elements of a plane, and a move from one to another."""
    c = P.PageCache.empty(1, 8, 128, 70000, 2, 4, page_tokens=64)
    c.table.copy_(ints([[69999, 3, 69000, -1], [2, 69998, -1, -1]]))
    c.length.copy_(ints([130, 70]))
    c.refs[[69999, 3, 69000, 2, 69998]] = 1
    k, v = (torch.randn((70, 8, 128), generator=gen(i), device="cuda").to(torch.bfloat16) for i in (1, 2))
    off = ints([0, 67, 70])
    c.append(0, None, k, v, torch.zeros(64, device="cuda"), offsets=off)
    # row 0's tokens lie at 63 .. 129: the first in page 69999, the last two in page 69000; row 1's at 67 .. 69, in page 69998
    for t, page, place in ((0, 69999, 63), (1, 3, 0), (64, 3, 63), (65, 69000, 0), (66, 69000, 1), (67, 69998, 3), (69, 69998, 5)):
        assert torch.equal(c.data[0, page, :, place], k[t]) and torch.equal(c.data[1, page, :, place], v[t])
    up = ints([-1] + [0] * 65 + [65] + [-1, 0, 0])
    token = ints([0] + [1] * 64 + [2, 3] + [0, 1, 2])
    pick = ints([2] + [9] * 64 + [3, 7] + [2, 9, 5])
    path, count, last = c.accept(token, pick, up, offsets=off)
    assert count.tolist() == [3, 2] and last.tolist() == [7, 5] and c.length.tolist() == [66, 69]
    for t, page, place in ((0, 69999, 63), (65, 3, 0), (66, 3, 1), (67, 69998, 3), (69, 69998, 4)):
        assert torch.equal(c.data[0, page, :, place], k[t]) and torch.equal(c.data[1, page, :, place], v[t])
    assert c.table.tolist() == [[69999, 3, -1, -1], [2, 69998, -1, -1]] and int(c.refs[69000]) == 0


def test_append_and_accept_off_the_current_stream(P):
    rng = np.random.default_rng(5)
    s = Sequences(P, [300, 40], [20, 9], 8, 2, 64, 16, torch.bfloat16, seed=13, garbage=0.25)
    k, v = (torch.randn((29, 2, 64), generator=gen(i), device="cuda").to(torch.bfloat16) for i in (1, 2))
    f = torch.rand(32, generator=gen(3), device="cuda")
    up, token, pick = (ints(x) for x in (forest(rng, 20) + forest(rng, 9), rng.integers(0, 3, 29), rng.integers(0, 3, 29)))
    c = s.cache
    kept = [x.clone() for x in (c.data, c.table, c.length)]

    def step(**kw):
        return [c.append(0, s.q, k, v, f, offsets=s.offsets, **kw), *c.accept(token, pick, up, offsets=s.offsets, **kw)]
    want = step() + [x.clone() for x in (c.data, c.table, c.length)]
    for x, y in zip((c.data, c.table, c.length), kept):
        x.copy_(y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(stream=side) + [c.data, c.table, c.length]
    torch.cuda.synchronize()
    for x, y in zip(got, want):
        assert torch.equal(x, y)


# ------------------------------------------------------------------- top -------

def check_top(P, x, k):
    B, V = x.shape
    tokens, logprobs, lse = P.top_tokens(x, k, return_lse=True)
    assert tokens.shape == logprobs.shape == (B, k) and lse.shape == (B,)
    y = x.double()
    order = torch.sort(y, dim=1, descending=True, stable=True)
    want = torch.where(order.values[:, :k] > -math.inf, order.indices[:, :k], -1)
    if V < k:
        want = torch.cat([want, torch.full((B, k - V), -1, device="cuda")], 1)
    assert torch.equal(tokens.long(), want)
    top = y.amax(1)
    sums = torch.logsumexp(y, 1)
    tol = 170 * 2.0 ** -24 + 3 * 2.0 ** -24 * torch.where(sums.isfinite(), top.abs() + sums.abs(), 0)
    dead = sums == -math.inf
    assert torch.equal(dead, lse == -math.inf) and ((lse.double() - sums).abs()[~dead] <= tol[~dead]).all()
    none = tokens < 0
    assert (logprobs[none] == -math.inf).all()
    lp = y.gather(1, tokens.clamp(min=0).long()) - sums[:, None]
    err = (logprobs.double() - lp).abs()
    assert (err <= tol[:, None] + 2.0 ** -24 * lp.abs())[~none].all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,V,pad,offset", [(1, 1, 0, 0), (3, 63, 1, 0), (2, 4096, 0, 0), (4, 4097, 3, 1), (5, 12289, 0, 7),
                                            (2, 32000, 8, 0), (7, 8191, 2, 5), (1, 262144, 0, 0), (3, 100003, 0, 0), (130, 9001, 1, 3),
                                            (300, 33000, 0, 1), (40, 128255, 1, 0)])
def test_top_shapes(P, dtype, B, V, pad, offset):
    g = gen(V + B)
    buf = torch.randn((B, offset + V + pad), generator=g, device="cuda") * 4
    buf[:, :offset] = math.inf  # what lies beside the rows is not looked at
    buf[:, offset + V:] = math.nan
    x = buf.to(dtype)[:, offset:offset + V]
    for k in (1, 2, 5, 16, 33, 64):
        check_top(P, x, k)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [50, 1000, 40007, 262144])
def test_top_ties_and_masks(P, dtype, V):
    """Equal logits by the thousand, rows with few or no logits left, signs of 0, orders that rise and fall."""
    g = gen(V)
    n = torch.arange(V, device="cuda").float()
    rows = [torch.zeros(V, device="cuda"), -torch.zeros(V, device="cuda"), torch.where(n % 2 == 0, -0.0, 0.0), n, -n,
            torch.full((V,), -math.inf, device="cuda"), torch.where(n == V - 1, 2.0, -math.inf),
            torch.where(n % 7 == 3, -1e38, -math.inf), torch.randint(-2, 3, (V,), generator=g, device="cuda").float(),
            torch.full((V,), 3.0e38, device="cuda"), torch.full((V,), -3.0e38, device="cuda"), (n % 512 == 5).float(), (n % 4096 < 8).float(),
            torch.where(torch.rand(V, generator=g, device="cuda") < 20 / V, torch.randn(V, generator=g, device="cuda"), -math.inf),
            1e-40 * (n % 3), n % 100]
    x = torch.stack(rows).to(dtype)
    for k in (1, 4, 64):
        check_top(P, x, k)
        check_top(P, x[3:5], k)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("at", [1e4, -1e4, 1e6, 1e9, -1e9, 1e12, 1e20, -1e20, 1e30, 8e37, 3e38, -3e38])
def test_top_far_from_zero(P, dtype, at):
    """Logits around a large number, a few steps of its type apart."""
    step = abs(at) * torch.finfo(dtype).eps
    for V in (700, 40001):
        n = torch.randint(0, 7, (3, V), generator=gen(V), device="cuda").double()
        x = (at + n * step).to(dtype)
        assert torch.isfinite(x).all() and x.unique().numel() > 1
        check_top(P, x, 5)


def test_top_infinities_and_nan(P):
    for dtype in (torch.float32, torch.bfloat16):
        for V in (70, 5000, 70000):
            x = torch.randn((5, V), generator=gen(V), device="cuda").to(dtype)
            x[0, 30] = x[0, 50] = math.inf
            x[1, 40] = math.nan
            x[2, 60] = -torch.tensor(math.nan, device="cuda").to(dtype)  # with a sign
            x[3] = -math.inf
            x[3, 20] = -torch.tensor(math.nan, device="cuda").to(dtype)
            bits = x.view(torch.int32 if dtype is torch.float32 else torch.int16)
            bits[2, 60] = bits[3, 20] = -1
            tokens, logprobs, lse = P.top_tokens(x, 3, return_lse=True)
            assert tokens[0, :2].tolist() == [30, 50] and lse[0] == math.inf
            assert logprobs[0, :2].isnan().all() and logprobs[0, 2] == -math.inf
            for b, v in ((1, 40), (2, 60), (3, 20)):
                assert tokens[b, 0] == v and lse[b].isnan() and logprobs[b, 0].isnan()
            y = x.float()
            y[1, 40] = y[2, 60] = -math.inf
            assert torch.equal(tokens[1:3, 1:].long(), torch.sort(y[1:3], dim=1, descending=True, stable=True).indices[:, :2])
            assert tokens[3, 1:].tolist() == [-1, -1]
            check_top(P, x[4:], 3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_top_of_wide_rows_and_many(P, dtype):
    """Rows of more parts than 256 threads hold, as wide as they may be, and more rows than there are CUs."""
    for B, V in ((2, 1500001), (1, 2 ** 21), (3000, 50), (1000, 5000)):
        x = torch.randn((B, V), generator=gen(V), device="cuda").to(dtype)
        for k in (1, 7, 64):
            check_top(P, x, k)
    with pytest.raises(P.TamError):
        P.top_tokens(torch.zeros((1, 2 ** 21 + 1), dtype=dtype, device="cuda"), 1)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [900, 32000, 262144])
def test_top_many_nan(P, dtype, V):
    """NaN of both signs, few and by the thousand: first, the lowest token first, and the numbers behind them."""
    for share in (3 / V, 0.01, 1.0):
        x = torch.randn((4, V), generator=gen(V), device="cuda").to(dtype)
        at = torch.rand((4, V), generator=gen(V + 1), device="cuda") < share
        at[:, 7] = True
        x[at] = math.nan
        bits = x.view(torch.int32 if dtype is torch.float32 else torch.int16)
        bits[:, 1::2] = torch.where(at[:, 1::2], torch.full_like(bits[:, 1::2], -1), bits[:, 1::2])
        for k in (1, 5, 64):
            tokens, logprobs, lse = P.top_tokens(x, k, return_lse=True)
            y = torch.where(at, math.inf, x.double())
            want = torch.sort(y, dim=1, descending=True, stable=True).indices[:, :k]
            assert torch.equal(tokens.long(), want) and lse.isnan().all() and logprobs.isnan().all()


def test_top_of_a_view_and_empty(P):
    x = torch.randn((6, 5003), generator=gen(6), device="cuda")
    check_top(P, x[1:2, 3:], 7)
    check_top(P, x[::2], 7)
    check_top(P, x[:1].expand(4, -1), 3)
    tokens, logprobs = P.top_tokens(x[:0], 7)
    assert tokens.shape == logprobs.shape == (0, 7)
    w = P.top_tokens(x, 9)
    h = P.compile([b"ab", b"c"], [b"a", b"b", b"c", b'"'], device="cuda:0")
    y = torch.randn((2, 4), generator=gen(7), device="cuda")
    h.apply_mask(ints([0, -1]), y)
    check_top(P, y, 3)
    h.close()
    assert torch.equal(w[0], P.top_tokens(x, 9)[0])


# --------------------------------------------------------------- together -------

def test_tree_step_in_a_graph(P):
    """A whole step over drafted trees captured, and replayed with eager work between the replays."""
    rng = np.random.default_rng(3)
    chunks, lens = [9, 20, 0, 33], [300, 90, 12, 33]
    s = Trees(P, lens, chunks, 8, 2, 64, 16, torch.bfloat16, seed=14, garbage=0.5)
    c = s.cache
    T = sum(chunks)
    trees = [forest(rng, n) for n in chunks]
    up = ints(sum(trees, []))
    tokens = ints([t for n in chunks for t in rng.integers(0, 4, n)])
    k, v = (torch.randn((T, 2, 64), generator=gen(i), device="cuda").to(torch.bfloat16) for i in (1, 2))
    logits = torch.randn((T, 5003), generator=gen(3), device="cuda").to(torch.bfloat16)
    logits[:, 4:] -= 8  # mostly one of the first four tokens
    f = torch.rand(32, generator=gen(4), device="cuda")
    kept = [x.clone() for x in (c.data, c.table, c.length, c.refs)]

    def step():
        for x, y in zip((c.data, c.table, c.length, c.refs), kept):
            x.copy_(y)
        seen, depth = P.tree_masks(up, s.offsets, longest=40)
        q = c.append(1, s.q, k, v, f, depth=depth, offsets=s.offsets, longest=40)
        out, lse = c.attend(1, q, offsets=s.offsets, longest=40, seen=seen, return_lse=True)
        best, logprobs, sums = P.top_tokens(logits, 5, return_lse=True)
        path, count, last = c.accept(tokens, best[:, 0].contiguous(), up, offsets=s.offsets)
        return seen, depth, q, out, lse, best, logprobs, sums, path, count, last

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    want = [x.clone() for x in step()]
    state = [x.clone() for x in (c.data, c.table, c.length, c.refs)]
    assert int(want[9].max()) > 1 and not torch.equal(state[2], kept[2])
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    got = []
    for g in graphs:
        with torch.cuda.graph(g):
            got.append(step())
    for i in range(6):
        for x in got[i % 2]:
            x.zero_()
        c.data.zero_()
        c.length.zero_()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        for x, y in zip((*got[i % 2], c.data, c.table, c.length, c.refs), (*want, *state)):
            assert torch.equal(x, y)
        torch.randn(1000, device="cuda").sum().item()
        P.top_tokens(logits, 3)


def test_calls_on_two_streams_at_once(P):
    logits = [torch.randn((40, 70001), generator=gen(i), device="cuda") for i in (1, 2)]
    s = [Trees(P, [4000, 900], [40, 25], 8, 2, 128, 16, torch.bfloat16, seed=i) for i in (1, 2)]
    want = [(*P.top_tokens(x, 9), *y.cache.attend(1, y.q, offsets=y.offsets, seen=y.seen, return_lse=True)) for x, y in zip(logits, s)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, on in enumerate(streams):
            got[i].append((*P.top_tokens(logits[i], 9, stream=on),
                           *s[i].cache.attend(1, s[i].q, offsets=s[i].offsets, seen=s[i].seen, return_lse=True, stream=on)))
    torch.cuda.synchronize()
    for i in range(2):
        for calls in got[i]:
            for x, y in zip(calls, want[i]):
                assert torch.equal(x, y)


def plain_decoder(model, tokens):
    """The example's decoder over one text, in 64 bits: [tokens, vocab] logits."""
    x = model.embed[torch.tensor(tokens, device="cuda")].double()
    norm = lambda x: x * torch.rsqrt((x * x).mean(-1, keepdim=True) + torch.finfo(torch.bfloat16).eps)
    T, heads, kv, dim = len(tokens), model.heads, model.kv_heads, model.head_dim
    position = torch.arange(T, device="cuda")
    hidden = position[None, :] > position[:, None]
    for qkv, out, up, down in model.layers:
        y = norm(x) @ qkv.double().T
        q, k, v = y[:, :heads * dim].view(T, heads, dim), y[:, heads * dim:(heads + kv) * dim].view(T, kv, dim), y[:, (heads + kv) * dim:].view(T, kv, dim)
        q, k = (turned(z, position, model.frequencies, False)[0] for z in (q, k))
        a = torch.empty((T, heads, dim), dtype=torch.float64, device="cuda")
        for h in range(heads):
            score = (q[:, h] @ k[:, h // (heads // kv)].T.contiguous() * dim ** -0.5).masked_fill(hidden, -math.inf)
            a[:, h] = torch.softmax(score, 1) @ v[:, h // (heads // kv)]
        x = x + a.flatten(1) @ out.double().T
        gate, y = (norm(x) @ up.double().T).chunk(2, 1)
        x = x + (torch.nn.functional.silu(gate) * y) @ down.double().T
    return norm(x) @ model.head.double().T


@pytest.mark.parametrize("levels", [(), (4, 2, 1), (2, 1, 1, 1, 1), (16, 2)])
def test_drafts_example(P, levels):
    """What the example finds with drafts is the greedy continuation: at each token the model's best one, up to the rounding of
    its logits.  Those are of size 1; bf16 activations of two layers take about 16 roundings of 2^-9 (a half step is at most
    2^-8 of a value, 2^-9 on average) times the layers' gains of about 2: 16^0.5 2^-9 2 = 0.016, 4 times that for the worst
    of thousands."""
    import examples.drafts as E
    vocab = E.beams.vocabulary()
    h = P.compile(E.beams.STRINGS, vocab, device="cuda:0")
    prior = torch.tensor([float(len(t)) for t in vocab], device="cuda")
    prompts = [list(b"a prompt"), list(b"and one that is longer than a page of the cache"), list(b"x")]
    model = E.Decoder(len(vocab))
    found, steps, cache = E.generate(model, h, prior, prompts, levels)
    assert not cache.refs.any() and not cache.length.any()
    assert steps == max(len(t) for t in found) if not levels else steps < max(len(t) for t in found)
    for prompt, tokens in zip(prompts, found):
        assert b"".join(vocab[t] for t in tokens)[:-1] in E.beams.STRINGS
        logits = plain_decoder(model, prompt + tokens)
        node = ints([0])
        for i, t in enumerate(tokens):
            row = logits[len(prompt) - 1 + i:len(prompt) + i].float()
            h.apply_mask(node, row)
            assert row[0, t] >= row.max() - 2 * 0.064
            node = h.advance(node, ints([t]))
    h.close()


@pytest.mark.parametrize("levels,most", [((4, 2, 1), 32), ((1, 1, 1, 1, 1), 20), ((), 110)])
def test_drafts_example_of_long_strings(P, monkeypatch, levels, most):
    """Strings as long as the steps allow: the cache has room for every tree, and the tokens of each."""
    import examples.drafts as E
    made = []
    monkeypatch.setattr(P.PageCache, "extend", lambda c, *a, real=P.PageCache.extend, **kw: made.append(real(c, *a, **kw)) or made[-1])
    vocab = E.beams.vocabulary()
    strings = [bytes(65 + (i * i + k * (i > 90)) % 26 for i in range(107)) for k in (0, 1)]
    h = P.compile(strings, vocab, device="cuda:0")
    prior = torch.ones(len(vocab), device="cuda")
    prompts = [list(b"short"), list(b"a prompt that is longer than a page")]
    found, steps, cache = E.generate(E.Decoder(len(vocab)), h, prior, prompts, levels, most=most)
    assert len(made) == steps + 1 and [x[0].item() for x in made] == [1] * len(made)
    assert steps <= most and not cache.refs.any() and not cache.length.any()
    for tokens in found:
        assert b"".join(vocab[t] for t in tokens)[:-1] in strings
    h.close()
