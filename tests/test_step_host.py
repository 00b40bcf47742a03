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
