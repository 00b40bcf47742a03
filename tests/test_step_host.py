"""The decode step's entry points without a GPU: what they refuse before anything is launched.

Pointers here are made up, so nothing of this runs where a launch could reach them.
"""
import ctypes

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up pointers: only where there is no GPU to follow them")


@pytest.fixture(scope="module")
def P():
    import paper_2608_12574_amd as P
    try:
        P.lib()
    except RuntimeError:
        from paper_2608_12574_amd import build
        build.build()
    return P


AT = 1 << 20  # an aligned address
INVAL = -1


def chunk(P, page=4 * 16 * 64, head=16 * 64, token=64, pages=10, heads=4, tokens=7):
    return P.tam.Chunk(AT, AT, page, head, token, pages, 16, heads, 64, P.DTYPE_BF16, AT, 3, 5, 5, AT, 3, tokens, AT, None, 0)


@pytest.mark.parametrize("token,head", [(0, 64), (64, 64), (512, 0), (256, 64), (512, 56), (8 * 64 - 8, 64), (64, 64 * 6), (-64, 64)])
def test_attend_refuses_outputs_that_overlap(P, token, head):
    c = chunk(P)
    L = P.lib()
    assert L.tam_attend_work(ctypes.byref(c), 8) > 0
    assert L.tam_attend(ctypes.byref(c), AT, 512, 64, 8, 0.1, AT, token, head, None, AT, None) == INVAL
    assert b"overlap" in L.tam_last_error()


@pytest.mark.parametrize("kw", [dict(page=0), dict(head=0), dict(token=0), dict(page=4 * 16 * 64 - 8), dict(head=64, token=64),
                                dict(token=56), dict(page=64, head=640, token=64 * 40 - 8)])
def test_store_refuses_pools_that_overlap(P, kw):
    c = chunk(P, **kw)
    L = P.lib()
    assert L.tam_pages_store(ctypes.byref(c), AT, 256, 64, AT, 256, 64, None) == INVAL
    assert b"overlap" in L.tam_last_error()


def test_pages_refuse_pools_that_overlap(P):
    L = P.lib()

    def work(planes, plane, page):
        c = P.tam.Pages(AT, planes, plane, page, 1024, 10, 16, AT, 3, 5, 5, AT, AT)
        return L.tam_pages_work(ctypes.byref(c), 3)
    for planes, plane, page in ((4, 10 * 1024, 1024), (4, 1024, 4096), (4, 1040, 8192), (1, 0, 1024), (2, 99999, 1040)):
        assert work(planes, plane, page) > 0
    for planes, plane, page in ((4, 0, 1024), (4, 10 * 1024 - 16, 1024), (4, 1024, 1024), (4, 1024, 4080), (4, 512, 4096)):
        assert work(planes, plane, page) == INVAL
        assert b"overlap" in L.tam_last_error()


class On:
    """A tensor of the CPU that says it lies on a GPU."""

    is_cuda = True

    def __init__(self, t, gpu):
        self.t, self.gpu = t, gpu

    def get_device(self):
        return self.gpu

    def __getattr__(self, name):
        return getattr(self.t, name)

    def __getitem__(self, at):
        return self.t[at]


class Launched(Exception):
    pass


@pytest.fixture
def two_gpus(P, monkeypatch):
    """As on a machine with two GPUs, the first of them current: calls that would launch say so."""
    from types import SimpleNamespace

    from paper_2608_12574_amd import step, tam

    def launch(*args):
        raise Launched
    calls = SimpleNamespace(stream=lambda: 0, stream_of=lambda gpu: 0, device=lambda: 0, adjust=launch,
                            dtypes={torch.float32: P.DTYPE_FP32, torch.bfloat16: P.DTYPE_BF16})
    monkeypatch.setattr(tam, "_calls_made", calls)
    monkeypatch.setattr(step, "_int", torch.int32)
    monkeypatch.setattr(step, "_float", torch.float32)
    monkeypatch.setattr(step, "_long", torch.int64)

    def cache(gpu, table=None, refs=None):
        ints = lambda *shape: torch.zeros(shape, dtype=torch.int32)
        c = P.PageCache(On(torch.zeros((2, 4, 1, 16, 8), dtype=torch.bfloat16), gpu), On(ints(3, 2), gpu if table is None else table),
                        On(ints(3), gpu), On(ints(4), gpu if refs is None else refs))
        c._lib = SimpleNamespace(tam_attend_work=lambda *a: 0, **{"tam_" + n: launch for n in (
            "pages_fork", "pages_extend", "pages_compact", "pages_store", "attend")})
        return c
    return cache


def test_tensors_of_another_gpu_are_refused(P, two_gpus):
    from types import SimpleNamespace
    ints = lambda n, gpu: On(torch.zeros(n, dtype=torch.int32), gpu)
    vec = lambda gpu: On(torch.zeros((3, 1, 8), dtype=torch.bfloat16), gpu)
    here, there = two_gpus(0), two_gpus(1)

    def calls(c, gpu, **kw):
        return [lambda: c.fork(ints(1, gpu), ints(1, gpu), **kw), lambda: c.extend(ints(1, gpu), ints(1, gpu), **kw),
                lambda: c.store(0, vec(gpu), vec(gpu), **kw), lambda: c.attend(0, vec(gpu), out=vec(gpu), **kw)]
    for call in calls(here, 0) + [here.compact]:  # all of it on the current one
        with pytest.raises(Launched):
            call()
    stream = SimpleNamespace(cuda_stream=0, device_index=1)
    for call in (calls(there, 1) + calls(there, 0) + calls(here, 1) + [there.compact] +
                 [lambda: here.attend(0, vec(0), out=vec(1)), lambda: here.attend(0, vec(0), slots=ints(3, 1), out=vec(0)),
                  lambda: here.attend(0, vec(0), offsets=ints(4, 1), out=vec(0)), lambda: here.store(0, vec(0), vec(1)),
                  lambda: here.fork(ints(1, 0), ints(1, 1)), lambda: here.fork(ints(1, 0), ints(1, 0), ints(1, 1)),
                  lambda: here.store(0, vec(0), vec(0), stream=stream)]):
        with pytest.raises(P.TamError):
            call()
    for kw in (dict(table=0), dict(refs=0)):
        with pytest.raises(P.TamError):
            two_gpus(1, **kw)


def test_adjust_takes_one_row_of_any_stride(P, two_gpus):
    """Of a single row the stride says nothing: a bias beside ids that are part of a larger list."""
    ids, bias = torch.zeros((4, 9), dtype=torch.int32)[2:3, :3], torch.zeros((1, 3))
    with pytest.raises(Launched):
        P.adjust_logits(On(torch.zeros((1, 128)), 0), bias_ids=On(ids, 0), bias=On(bias, 0))
    with pytest.raises(P.TamError):
        P.adjust_logits(On(torch.zeros((2, 128)), 0), bias_ids=On(torch.zeros((4, 9), dtype=torch.int32)[:2, :3], 0),
                        bias=On(torch.zeros((2, 3)), 0))


def test_logits_of_another_gpu_are_refused(P, two_gpus):
    from types import SimpleNamespace

    def call(**gpus):
        gpu = lambda name: gpus.get(name, gpus.get("all", 0))
        ints = lambda name, *shape: On(torch.zeros(shape, dtype=torch.int32), gpu(name))
        P.adjust_logits(On(torch.zeros((2, 128)), gpu("logits")), tokens=ints("tokens", 2, 5), length=ints("length", 2),
                        prompt=ints("prompt", 2), repetition=On(torch.ones(2), gpu("repetition")), bias_ids=ints("bias_ids", 2, 3),
                        bias=On(torch.zeros((2, 3)), gpu("bias")), rows=On(torch.zeros((4, 2), dtype=torch.int64), gpu("rows")),
                        row_ids=ints("row_ids", 2), stream=gpus.get("stream"))
    with pytest.raises(Launched):
        call()
    for name in ("all", "logits", "tokens", "length", "prompt", "repetition", "bias_ids", "bias", "rows", "row_ids"):
        with pytest.raises(P.TamError):
            call(**{name: 1})
    with pytest.raises(P.TamError):
        call(stream=SimpleNamespace(cuda_stream=0, device_index=1))
    from paper_2608_12574_amd.step import _adjust
    for gpu in (0, 1):
        handle = SimpleNamespace(_raw=1, vocab_size=128, host_only=False, device=torch.device("cuda", gpu))
        with pytest.raises(P.TamError if gpu else Launched):
            _adjust(On(torch.zeros((2, 128)), 0), None, handle=handle, ids=On(torch.zeros(2, dtype=torch.int32), 0))
