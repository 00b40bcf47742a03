"""Trees of drafted tokens and the best tokens without a GPU: what the entry points refuse before anything is launched.

Pointers here are made up, so nothing of this runs where a launch could reach them.
"""
import ctypes
from types import SimpleNamespace

import pytest

from test_step_host import AT, INVAL, Launched, On, P, chunk, two_gpus  # noqa: F401 (P, two_gpus: fixtures)

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up pointers: only where there is no GPU to follow them")


def refused(L, rc, word):
    assert rc == INVAL and word in L.tam_last_error().decode(), (rc, L.tam_last_error())


def test_tree_masks_refusals(P):
    L = P.lib()
    good = dict(parents=AT, offsets=AT, rows=3, tokens=7, seen=AT, words=1, depth=AT)

    def call(**kw):
        a = dict(good, **kw)
        return L.tam_tree_masks(a["parents"], a["offsets"], a["rows"], a["tokens"], a["seen"], a["words"], a["depth"], None)
    for kw, word in ((dict(rows=-1), "rows"), (dict(rows=2 ** 23 + 1), "rows"), (dict(tokens=-1), "rows"), (dict(tokens=2 ** 31 - 1), "rows"),
                     (dict(words=0), "words"), (dict(words=2 ** 25 + 1), "words"), (dict(parents=None), "null"), (dict(seen=None), "null"),
                     (dict(depth=None), "null"), (dict(parents=AT + 2), "aligned"), (dict(offsets=AT + 1), "aligned"),
                     (dict(seen=AT + 4), "aligned"), (dict(depth=AT + 2), "aligned")):
        refused(L, call(**kw), word)
    assert call(tokens=0, parents=None, seen=None, depth=None) == 0 and call(rows=0) == 0


def test_append_refusals(P):
    L = P.lib()
    turn = dict(frequencies=AT, pairs=32, adjacent=0, depth=AT)
    good = dict(k=AT, k_token=256, k_head=64, v=AT, v_token=256, v_head=64, q=AT, q_token=512, q_head=64, heads=8, out=AT, out_token=512,
                out_head=64)

    def call(c=None, r=True, **kw):
        c = chunk(P) if c is None else c
        t = P.tam.Rotation(*[kw.pop(n, turn[n]) for n in ("frequencies", "pairs", "adjacent", "depth")])
        return L.tam_pages_append(ctypes.byref(c), ctypes.byref(t) if r else None, *dict(good, **kw).values(), None)
    for kw, word in ((dict(pairs=-4), "pairs"), (dict(pairs=6), "pairs"), (dict(pairs=36), "pairs"), (dict(adjacent=2), "adjacent"),
                     (dict(frequencies=None), "frequencies"), (dict(frequencies=AT + 2), "aligned"), (dict(depth=AT + 1), "aligned"),
                     (dict(heads=-1), "heads"), (dict(heads=65536), "heads"), (dict(q=None), "null"), (dict(out=None), "null"),
                     (dict(q=AT + 8), "aligned"), (dict(out_token=4 * 512 + 4), "multiples of 8"), (dict(out_token=0), "overlap"),
                     (dict(out_head=56), "overlap"), (dict(k=None), "null"), (dict(v=AT + 2), "aligned"), (dict(k_token=12), "multiples of 8"),
                     (dict(r=False), "rotation"), (dict(c=chunk(P, token=56)), "overlap"), (dict(c=chunk(P, tokens=-1)), "tokens")):
        refused(L, call(**kw), word)
    # nothing to do: no tokens; without queries theirs are not looked at
    assert call(c=chunk(P, tokens=0)) == 0 and call(c=chunk(P, tokens=0), heads=0, q=None, out=None, out_token=0, frequencies=None, pairs=0) == 0


def test_append_refuses_more_tokens_than_blocks(P):
    L = P.lib()
    turn = P.tam.Rotation(AT, 32, 0, None)

    def call(tokens, heads, q):
        c = chunk(P, tokens=tokens)
        return L.tam_pages_append(ctypes.byref(c), ctypes.byref(turn), AT, 256, 64, AT, 256, 64, q, 512, 64, heads, q, 512, 64, None)
    for tokens in (2 ** 24, 2 ** 24 + 7, 2 ** 31 - 2):
        refused(L, call(tokens, 8, AT), "2^24")
        refused(L, call(tokens, 0, None), "2^24")
    refused(L, call(2 ** 24 - 1, 8, None), "null")  # as many are looked at further


def test_attend_seen_refusals(P):
    L = P.lib()
    good = dict(q=AT, q_token=512, q_head=64, heads=8, scale=0.1, seen=AT, words=2, stride=2, out=AT, out_token=512, out_head=64, lse=None,
                work=AT)

    def call(c=None, **kw):
        return L.tam_attend_seen(ctypes.byref(chunk(P) if c is None else c), *dict(good, **kw).values(), None)
    for kw, word in ((dict(seen=None), "seen"), (dict(seen=AT + 4), "seen"), (dict(words=0), "words"), (dict(words=2 ** 31), "words"),
                     (dict(stride=1), "seen_stride"), (dict(heads=6), "heads"), (dict(scale=0.0), "scale"), (dict(scale=float("inf")), "scale"),
                     (dict(q=None), "null"), (dict(out_token=64), "overlap"), (dict(work=None), "work"), (dict(lse=AT + 2), "lse")):
        refused(L, call(**kw), word)
    assert call(c=chunk(P, tokens=0), seen=None) == 0


def test_accept_refusals(P):
    L = P.lib()
    page = 4 * 16 * 64 * 2
    lists = dict(tokens=AT, picks=AT, parents=AT, path=AT, count=AT, last=AT, work=AT)

    def call(pages=(), c=None, **kw):
        a = dict(data=AT, planes=4, plane_stride=10 * page, page_stride=page, page_bytes=page, num_pages=10, page_tokens=16, table=AT, slots=3,
                 max_pages=5, table_stride=5, length=AT, refs=AT)
        a.update(pages)
        return L.tam_pages_accept(ctypes.byref(P.tam.Pages(*a.values())), ctypes.byref(chunk(P) if c is None else c),
                                  *dict(lists, **kw).values(), None)
    for kw, word in [(dict(pages=dict([x])), "tables") for x in dict(num_pages=9, page_tokens=8, table=AT + 64, slots=4, max_pages=4, table_stride=6,
                                                                     length=AT + 4).items()] + [
            (dict(pages=dict(page_bytes=page - 16)), "fit"), (dict(pages=dict(data=AT + 8)), "aligned"), (dict(pages=dict(data=None)), "data"),
            (dict(pages=dict(plane_stride=10 * page + 8)), "multiples"), (dict(pages=dict(refs=None)), "refs"),
            (dict(c=chunk(P, token=56)), "overlap"), (dict(c=chunk(P, head=0)), "overlap"), (dict(c=chunk(P, token=128, head=2048)), "fit"),
            (dict(tokens=AT + 2), "aligned"), (dict(work=AT + 8), "aligned")] + [(dict([(x, None)]), "null") for x in lists]:
        refused(L, call(**kw), word)
    c = chunk(P)
    c.slot_ids, c.rows = AT, 4
    refused(L, call(c=c), "rows")
    c = chunk(P, tokens=0)
    c.rows = 0
    assert call(c=c) == 0
    assert L.tam_pages_accept_work(ctypes.byref(chunk(P))) >= 7 * 16 + 3 * 4
    refused(L, L.tam_pages_accept_work(ctypes.byref(chunk(P, tokens=-1))), "tokens")


def test_accept_does_not_look_at_k_and_v(P):
    """The vectors lie in the cache's planes: the chunk's own k and v may be anything."""
    L = P.lib()
    page = 4 * 16 * 64 * 2
    pages = P.tam.Pages(AT, 4, 10 * page, page, page, 10, 16, AT, 3, 5, 5, AT, AT)
    for at in (None, AT + 2):
        c = chunk(P)
        c.k = c.v = at
        assert L.tam_pages_accept_work(ctypes.byref(c)) >= 7 * 16 + 3 * 4
        c.rows = 0
        assert L.tam_pages_accept(ctypes.byref(pages), ctypes.byref(c), AT, AT, AT, AT, AT, AT, AT, None) == 0
        refused(L, L.tam_attend_work(ctypes.byref(c), 8), "k")


def test_accept_refuses_more_rows_than_blocks(P):
    L = P.lib()
    page = 4 * 16 * 64 * 2

    def call(rows, path):
        pages = P.tam.Pages(AT, 4, 10 * page, page, page, 10, 16, AT, 2 ** 30, 5, 5, AT, AT)
        c = chunk(P)
        c.slots, c.rows = 2 ** 30, rows
        return L.tam_pages_accept(ctypes.byref(pages), ctypes.byref(c), AT, AT, AT, path, AT, AT, AT, None)
    for rows in (2 ** 24, 2 ** 30):
        refused(L, call(rows, AT), "2^24")
    refused(L, call(2 ** 24 - 1, None), "null")  # as many are looked at further


def test_top_tokens_refusals(P):
    L = P.lib()
    good = dict(logits=AT, dtype=P.DTYPE_BF16, B=4, V=100000, stride=100000, k=8, tokens=AT, logprobs=AT, lse=AT, work=AT)

    def call(**kw):
        return L.tam_top_tokens(*dict(good, **kw).values(), None)
    for kw, word in ((dict(dtype=P.DTYPE_FP16), "dtype"), (dict(dtype=7), "dtype"), (dict(B=-1), "B"), (dict(B=65536), "B"), (dict(V=0), "V"),
                     (dict(V=2 ** 21 + 1, stride=2 ** 22), "V"), (dict(k=0), "k"), (dict(k=65), "k"), (dict(stride=-1), "row_stride"),
                     (dict(logits=None), "null"), (dict(tokens=None), "null"), (dict(logprobs=None), "null"), (dict(work=None), "null work"),
                     (dict(logits=AT + 1), "aligned"), (dict(dtype=P.DTYPE_FP32, logits=AT + 2), "aligned"), (dict(lse=AT + 2), "aligned"),
                     (dict(work=AT + 8), "aligned")):
        refused(L, call(**kw), word)
    assert call(B=0, logits=None, tokens=None, logprobs=None, work=None) == 0
    # the join holds the best of all parts
    for V in (1, 63, 4096, 131072, 2 ** 20, 2 ** 21):
        for B in (0, 1, 2, 63, 64, 1000, 65535):
            for dtype in (P.DTYPE_FP32, P.DTYPE_BF16):
                size = L.tam_top_tokens_work(B, V, 64, dtype)
                assert 0 <= size <= B * 128 * (64 * 8 + 8)
    refused(L, L.tam_top_tokens_work(1, 0, 1, 0), "V")


@pytest.fixture
def fake(P, two_gpus, monkeypatch):
    """`two_gpus` with the calls of this file, which say so when they would launch."""
    def launch(*args):
        raise Launched
    lib = SimpleNamespace(tam_top_tokens=launch, tam_tree_masks=launch, tam_top_tokens_work=lambda *a: 0)
    real = P.tam.lib
    monkeypatch.setattr(P.tam, "lib", lambda: lib)
    from paper_2608_12574_amd import step
    monkeypatch.setattr(step, "_scratch", lambda dtype, device, stream, *shape: On(torch.empty(*shape, dtype=dtype), 0))

    def cache(gpu):
        monkeypatch.setattr(P.tam, "lib", real)  # the size of the pages' scratch
        c = two_gpus(gpu)
        monkeypatch.setattr(P.tam, "lib", lambda: lib)
        c._lib = SimpleNamespace(tam_attend_work=lambda *a: 0, tam_pages_accept_work=lambda *a: 16,
                                 **{"tam_" + n: launch for n in ("pages_append", "attend_seen", "pages_accept", "attend")})
        return c
    return cache


def test_arguments_of_the_cache(P, fake):
    c = fake(0)
    ints = lambda n, gpu=0: On(torch.zeros(n, dtype=torch.int32), gpu)
    vec = lambda gpu=0, n=3: On(torch.zeros((n, 1, 8), dtype=torch.bfloat16), gpu)
    f = lambda n=4, gpu=0, dtype=torch.float32: On(torch.zeros(n, dtype=dtype), gpu)
    bits = lambda *shape, gpu=0, dtype=torch.int64: On(torch.zeros(shape, dtype=dtype), gpu)
    other = SimpleNamespace(cuda_stream=0, device_index=1)

    def append(q=None, k=None, v=None, fr=None, **kw):
        return c.append(0, q, k if k is not None else vec(), v if v is not None else vec(), fr if fr is not None else f(), **kw)
    for call in (append, lambda: append(q=vec(), depth=ints(3)), lambda: append(q=vec(), out=vec()),
                 lambda: c.attend(0, vec(), seen=bits(3, 1)), lambda: c.attend(0, vec(), seen=On(torch.zeros((3, 5), dtype=torch.int64)[:, 1:3], 0)),
                 lambda: c.accept(ints(3), ints(3), ints(3)), lambda: c.accept(ints(3), ints(3), ints(3), offsets=ints(3), slots=ints(2))):
        with pytest.raises(Launched):
            call()
    for call in (lambda: append(q=vec(1)), lambda: append(k=vec(1)), lambda: append(v=vec(1)), lambda: append(fr=f(gpu=1)),
                 lambda: append(depth=ints(3, 1)), lambda: append(depth=ints(2)), lambda: append(q=vec(n=2)), lambda: append(v=vec(n=2)),
                 lambda: append(fr=f(dtype=torch.float64)), lambda: append(fr=On(torch.zeros((2, 2)), 0)), lambda: append(out=vec()),
                 lambda: append(fr=On(torch.zeros(8)[::2], 0)), lambda: append(q=vec(), out=vec(n=2)), lambda: append(q=vec(), out=vec(1)),
                 lambda: append(stream=other), lambda: c.append(1, None, vec(), vec(), f()),
                 lambda: c.attend(0, vec(), seen=bits(3, 1, gpu=1)), lambda: c.attend(0, vec(), seen=bits(2, 1)),
                 lambda: c.attend(0, vec(), seen=bits(3, 1, dtype=torch.int32)), lambda: c.attend(0, vec(), seen=bits(3)),
                 lambda: c.attend(0, vec(), seen=On(torch.zeros((1, 3), dtype=torch.int64).t().expand(3, 4), 0)),
                 lambda: c.accept(ints(3), ints(2), ints(3)), lambda: c.accept(ints(3), ints(3), ints(3, 1)),
                 lambda: c.accept(On(torch.zeros(3, dtype=torch.int64), 0), ints(3), ints(3)), lambda: c.accept(ints(3), ints(3), ints(3), offsets=ints(0)),
                 lambda: c.accept(ints(3), ints(3), ints(3), offsets=ints(3, 1)), lambda: c.accept(ints(3), ints(3), ints(3), slots=ints(2)),
                 lambda: c.accept(ints(3), ints(3), ints(3), stream=other)):
        with pytest.raises(P.TamError):
            call()
    for call in (lambda c: c.append(0, None, vec(1), vec(1), f(gpu=1)), lambda c: c.accept(ints(3, 1), ints(3, 1), ints(3, 1)),
                 lambda c: c.attend(0, vec(1), seen=bits(3, 1, gpu=1))):
        with pytest.raises(P.TamError):  # a cache on another GPU than the current one
            call(fake(1))


def test_attend_takes_its_stream_by_place(P, two_gpus):
    """The mask came after the other arguments: calls that give them by place are what they were."""
    c, on = two_gpus(0), []
    c._lib.tam_attend = lambda *a: on.append(a[-1]) or 0
    q = On(torch.zeros((3, 1, 8), dtype=torch.bfloat16), 0)
    c.attend(0, q, None, None, None, None, On(torch.zeros((3, 1, 8), dtype=torch.bfloat16), 0), False, SimpleNamespace(cuda_stream=77, device_index=0))
    assert on == [77]


def test_arguments_of_the_functions(P, fake):
    ints = lambda n, gpu=0: On(torch.zeros(n, dtype=torch.int32), gpu)
    x = lambda *shape, gpu=0, dtype=torch.float32: On(torch.zeros(shape, dtype=dtype), gpu)
    other = SimpleNamespace(cuda_stream=0, device_index=1)
    for call in (lambda: P.top_tokens(x(2, 9), 3), lambda: P.top_tokens(x(2, 9, dtype=torch.bfloat16), 3, return_lse=True),
                 lambda: P.tree_masks(ints(5)), lambda: P.tree_masks(ints(5), ints(3), longest=2)):
        with pytest.raises(Launched):
            call()
    for call in (lambda: P.top_tokens(x(2, 9, gpu=1), 3), lambda: P.top_tokens(x(2, 9, dtype=torch.float16), 3), lambda: P.top_tokens(x(9), 3),
                 lambda: P.top_tokens(On(torch.zeros((9, 2)).t(), 0), 3), lambda: P.top_tokens(torch.zeros((2, 9)), 3),
                 lambda: P.top_tokens(x(2, 9), 3, stream=other), lambda: P.tree_masks(ints(5, 1)), lambda: P.tree_masks(ints(5), ints(3, 1)),
                 lambda: P.tree_masks(ints(5), ints(0)), lambda: P.tree_masks(x(5)), lambda: P.tree_masks(torch.zeros(5, dtype=torch.int32)),
                 lambda: P.tree_masks(ints(5), stream=other)):
        with pytest.raises(P.TamError):
            call()
