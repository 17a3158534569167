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


def orthogonalize(lib, **kw):
    a = dict(G=4096, gt=0, gr=64, gb=4096, out=8192, ot=0, orow=64, ob=4096, batch=3, rows=64, cols=64, steps=5, coefs=None,
             scale=1.0, eps=1e-7, precision=1, work=65536, bytes=1 << 30)
    a.update(kw)
    return lib.prsgd_orthogonalize(*a.values(), None)


def test_rows_of_an_output_that_overlap(lib):
    for kw in (dict(ob=0), dict(ob=63), dict(ob=64), dict(ob=64, orow=191), dict(ob=4095, orow=64), dict(ob=63, orow=4096), dict(ob=100, orow=263)):
        assert orthogonalize(lib, **kw) == ARG, kw
    for kw in (dict(dgs=64), dict(dgs=64, drs=127), dict(dgs=63, drs=6400), dict(dgs=6399), dict(dgs=0), dict(G=3, dgs=100, drs=263)):
        assert grad(lib, **kw) == ARG, kw
    big = (1 << 62) + (1 << 61)                        # (a row stride whose product with the rows passes 64 bits)
    assert orthogonalize(lib, ob=63, orow=big) == ARG


def test_in_place_calls_keep_type_and_strides(lib):
    """Written while rows that lie elsewhere are still to be read, the result would depend on the order of the blocks."""
    for kw in (dict(ot=1, gt=2), dict(orow=65, ob=65 * 64), dict(ob=4097), dict(gb=0), dict(gr=65)):
        assert orthogonalize(lib, **{**dict(G=8192, out=8192), **kw}) == ARG, kw
    for kw in (dict(drs=65, dgs=6500), dict(dgs=6401), dict(gs=0), dict(rs=65)):
        assert grad(lib, **{**dict(x=8192, d=8192), **kw}) == ARG, kw


def test_muon_arrays_are_three(lib):
    def call(**kw):
        a = dict(W=4096, wt=0, wr=64, wb=4096, V=8192, vr=64, vb=4096, G=12288, gt=0, gr=64, gb=4096, batch=2, rows=64, cols=64,
                 lr=0.1, mu=0.9, nesterov=1, wd=0.0, steps=5, coefs=None, scale=1.0, eps=1e-7, precision=0, work=65536, bytes=1 << 30)
        a.update(kw)
        return lib.prsgd_muon_step(*a.values(), None)
    for kw in (dict(V=4096), dict(G=4096), dict(G=8192)):
        assert call(**kw) == ARG, kw
