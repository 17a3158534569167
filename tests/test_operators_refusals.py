"""Calls of the operators' C entries that are refused before anything is enqueued: no kernel is launched, no address is read."""
import pytest

OK, ARG, ALIGN, SIZE = 0, -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    from paper_1807_06629_b200 import _build
    _build.build_library()
    from paper_1807_06629_b200 import binding
    return binding.lib


def route(lib, **kw):
    a = dict(x=4096, ty=1, rs=64, gs=6400, live=None, G=2, T=100, E=64, k=4, norm=0, coef=0.01, e=256, w=256, c=256, m=256, l=256,
             work=65536, bytes=1 << 30)
    a.update(kw)
    return lib.prsgd_route(*a.values(), None)


def grad(lib, **kw):
    a = dict(x=4096, ty=1, rs=64, gs=6400, live=None, G=2, T=100, E=64, k=4, norm=0, coef=0.01, e=256, c=256, dw=256, dl=256,
             d=8192, drs=64, dgs=6400)
    a.update(kw)
    return lib.prsgd_route_grad(*a.values(), None)


@pytest.mark.parametrize("off", [1, 2, 3])
def test_arrays_of_words_are_aligned_to_them(lib, off):
    for name in "ewcml":
        assert route(lib, **{name: 256 + off}) == ALIGN, name
    for name in ("e", "c", "dw", "dl"):
        assert grad(lib, **{name: 256 + off}) == ALIGN, name
    assert lib.prsgd_last_error(None)
