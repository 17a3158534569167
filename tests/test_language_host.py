"""Embedding, dropout and vocabulary loss without a GPU: the checks of their C entries, the generator, the references that the
GPU tests compare with, and the Python functions' own checks.  No kernel is launched, no address is read."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest
import torch

import language_reference as ref

OK, ARG, ALIGN, SIZE = 0, -1, -2, -3
CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1807_06629_b200", "csrc")


@pytest.fixture(scope="module")
def b():
    from paper_1807_06629_b200 import _build
    _build.build_library()
    from paper_1807_06629_b200 import binding
    return binding


def embed(lib, **kw):
    a = dict(t=4096, ty=1, rs=64, gs=6400, ids=256, G=2, T=50, V=100, D=64, scale=1.0, o=8192, ot=1, ors=64, ogs=3200)
    a.update(kw)
    return lib.prsgd_embed(*a.values(), None)


def embed_grad(lib, **kw):
    a = dict(d=4096, ty=1, rs=64, gs=3200, ids=256, G=2, T=50, V=100, D=64, scale=1.0, o=8192, ot=0, ors=64, ogs=6400, acc=0, work=65536, bytes=1 << 30)
    a.update(kw)
    return lib.prsgd_embed_grad(*a.values(), None)


def dropout(lib, **kw):
    a = dict(x=4096, ty=1, rs=64, gs=640, r=None, rrs=0, rgs=0, o=8192, ors=64, ogs=640, G=2, R=10, Cn=64, p=0.1, seed=1, step=0, dstep=None, g0=0)
    a.update(kw)
    return lib.prsgd_dropout(*a.values(), None)


def loss(lib, **kw):
    a = dict(H=4096, hr=64, hg=640, W=8192, wr=64, wg=6400, ty=1, y=256, G=2, T=10, V=100, D=64, l=256, s=256, work=65536, bytes=1 << 30)
    a.update(kw)
    return lib.prsgd_vocab_loss(*a.values(), None)


def loss_grad(lib, **kw):
    a = dict(H=4096, hr=64, hg=640, W=8192, wr=64, wg=6400, ty=1, y=256, G=2, T=10, V=100, D=64, s=256, dl=256, ds=256,
             dH=12288, dhr=64, dhg=640, dW=16384, dwt=1, dwr=64, dwg=6400, acc=0, work=65536, bytes=1 << 30)
    a.update(kw)
    return lib.prsgd_vocab_loss_grad(*a.values(), None)


TOKENS = [(dict(G=-1), ARG), (dict(T=-1), ARG), (dict(V=0), ARG), (dict(D=-1), ARG), (dict(G=65536), SIZE), (dict(T=(1 << 24) + 1), SIZE),
          (dict(V=(1 << 24) + 1), SIZE), (dict(D=65537), SIZE), (dict(ids=None), ARG), (dict(ids=258), ALIGN), (dict(ty=3), ARG), (dict(ot=-1), ARG),
          (dict(scale=float("nan")), ARG), (dict(scale=float("inf")), ARG), (dict(rs=63), ARG), (dict(gs=-1), ARG), (dict(ors=63), ARG),
          (dict(ogs=0), ARG), (dict(ogs=63), ARG), (dict(o=None), ARG), (dict(o=8193), ALIGN), (dict(o=4096), ARG)]


def test_embed_refusals(b):
    for kw, want in TOKENS + [(dict(t=None), ARG), (dict(t=4097), ALIGN)]:
        assert embed(b.lib, **kw) == want, kw
        assert b.lib.prsgd_last_error(None)
    for kw in (dict(G=0), dict(T=0), dict(D=0)):
        assert embed(b.lib, t=None, o=None, ids=None, **kw) == OK


def test_embed_grad_refusals(b):
    for kw, want in TOKENS + [(dict(d=None), ARG), (dict(d=4097), ALIGN), (dict(work=None), SIZE), (dict(bytes=256), SIZE), (dict(work=65536 + 64), ALIGN)]:
        assert embed_grad(b.lib, **kw) == want, kw
        assert b.lib.prsgd_last_error(None)
    for kw in (dict(G=0), dict(D=0), dict(T=0, acc=1)):
        assert embed_grad(b.lib, **{**dict(d=None, o=None, ids=None, work=None), **kw}) == OK
    n = C.c_size_t()
    assert b.lib.prsgd_embed_grad_workspace_bytes(1, 1, 1, 1, None) == ARG
    assert b.lib.prsgd_embed_grad_workspace_bytes(1, 1, 0, 1, C.byref(n)) == ARG


def test_dropout_refusals(b):
    for kw, want in [(dict(p=-0.1), ARG), (dict(p=1.0), ARG), (dict(p=float("nan")), ARG), (dict(p=1 - 2.0 ** -18), ARG), (dict(ty=7), ARG),
                     (dict(G=-1), ARG), (dict(R=-1), ARG), (dict(Cn=-1), ARG), (dict(G=65536), SIZE), (dict(R=1 << 31), SIZE), (dict(x=None), ARG),
                     (dict(o=None), ARG), (dict(x=4097), ALIGN), (dict(rs=63), ARG), (dict(ors=63), ARG), (dict(ogs=0), ARG), (dict(ogs=63), ARG),
                     (dict(o=4096, ors=65, ogs=650), ARG), (dict(r=8192, rrs=65, rgs=650), ARG), (dict(r=16384, rrs=60, rgs=640), ARG),
                     (dict(r=16385, rrs=64, rgs=640), ALIGN), (dict(dstep=1028), ALIGN)]:
        assert dropout(b.lib, **kw) == want, kw
        assert b.lib.prsgd_last_error(None)
    for kw in (dict(G=0), dict(R=0), dict(Cn=0)):
        assert dropout(b.lib, x=None, o=None, **kw) == OK


VOCAB = [(dict(ty=3), ARG), (dict(G=-1), ARG), (dict(T=-1), ARG), (dict(V=0), ARG), (dict(D=0), ARG), (dict(G=4097), SIZE), (dict(T=(1 << 22) + 1), SIZE),
         (dict(V=(1 << 24) + 1), SIZE), (dict(D=65537), SIZE), (dict(H=None), ARG), (dict(W=None), ARG), (dict(H=4097), ALIGN), (dict(W=8193), ALIGN),
         (dict(hr=63), ARG), (dict(wr=63), ARG), (dict(hg=-1), ARG), (dict(wg=-1), ARG), (dict(y=None), ARG), (dict(y=257), ALIGN), (dict(s=None), ARG),
         (dict(s=258), ALIGN), (dict(work=None), SIZE), (dict(bytes=256), SIZE), (dict(work=65536 + 128), ALIGN)]


def test_vocab_loss_refusals(b):
    for kw, want in VOCAB + [(dict(l=None), ARG), (dict(l=257), ALIGN)]:
        assert loss(b.lib, **kw) == want, kw
        assert b.lib.prsgd_last_error(None)
    for kw in (dict(G=0), dict(T=0)):
        assert loss(b.lib, **{**dict(H=None, W=None, y=None, l=None, s=None, work=None), **kw}) == OK


@pytest.mark.parametrize("T", [1, 10])
def test_vocab_loss_outputs_apart(b, T):
    for l, s in [(4096, 4096), (4096, 4096 + 4 * 2 * T - 4), (4096 + 8 * 2 * T - 4, 4096)]:
        assert loss(b.lib, T=T, l=l, s=s) == ARG


def test_dropout_of_almost_all(b):
    """65536 p is rounded to even: below 1 - 2^-17 something may stay."""
    assert b.lib.prsgd_dropout_keep(1, 0, 0, 0, 0, 1 - 2.0 ** -17 - 2.0 ** -40) in (0, 1)
    assert b.lib.prsgd_dropout_keep(1, 0, 0, 0, 0, 1 - 2.0 ** -17) == ARG
    assert dropout(b.lib, p=1 - 2.0 ** -17) == ARG


def test_vocab_loss_grad_refusals(b):
    for kw, want in VOCAB + [(dict(dl=257), ALIGN), (dict(ds=257), ALIGN), (dict(dH=12289), ALIGN), (dict(dW=16385), ALIGN), (dict(dhr=63), ARG), (dict(dwr=63), ARG),
                             (dict(dhg=0), ARG), (dict(dwg=0), ARG), (dict(dwg=63), ARG), (dict(dwt=2), ARG), (dict(dH=4096), ARG), (dict(dH=8192), ARG),
                             (dict(dH=16384), ARG), (dict(dW=8192), ARG), (dict(dW=4096), ARG)]:
        assert loss_grad(b.lib, **kw) == want, kw
        assert b.lib.prsgd_last_error(None)
    for kw in (dict(G=0), dict(T=0, acc=1), dict(T=0, dW=None)):
        assert loss_grad(b.lib, **{**dict(H=None, W=None, y=None, s=None, dH=None, work=None), **kw}) == OK
    for call, size in ((loss, b.prsgd_vocab_loss_workspace_bytes), (loss_grad, b.prsgd_vocab_loss_grad_workspace_bytes)):
        small = size(1, 2, 10, 100, 64, 1)                  # (of a W whose rows begin on 16-byte boundaries; these do not)
        for kw in (dict(W=8194), dict(wr=65, wg=6500), dict(wg=6401)):
            assert call(b.lib, bytes=small, **kw) == SIZE, kw
    huge = dict(T=1 << 22, V=1 << 24, D=65536, hr=65536, wr=65536, hg=1 << 38, wg=1 << 40, dhr=65536, dwr=65536, dhg=1 << 38, dwg=1 << 40, bytes=1 << 62)
    assert loss_grad(b.lib, **huge) == SIZE and b"tiles" in b.lib.prsgd_last_error(None)
    for fn in (b.lib.prsgd_vocab_loss_workspace_bytes, b.lib.prsgd_vocab_loss_grad_workspace_bytes):
        n = C.c_size_t()
        assert fn(1, 1, 1, 1, 1, 1, None) == ARG and fn(5, 1, 1, 1, 1, 1, C.byref(n)) == ARG and fn(1, 1, 1, 1, 0, 1, C.byref(n)) == ARG


def test_philox_known_answers(tmp_path):
    """The generator's published known answers, for the library's own code compiled for the host and for the reference's."""
    cases = [((0, 0, 0, 0), (0, 0), "6627e8d5 e169c58d bc57ac4c 9b00dbd8"),
             ((0xffffffff,) * 4, (0xffffffff, 0xffffffff), "408f276d 41c83b0e a20bc7c6 6d5451fd"),
             ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0), "d16cfe09 94fdcceb 5001e420 24126ea1")]
    src = tmp_path / "p.cpp"
    src.write_text('#include <cstdio>\n#include <cstdlib>\n#include "philox.h"\nint main(int n, char** v) { uint32_t c[6]; for (int i = 0; i < 6; ++i) '
                   'c[i] = strtoul(v[i + 1], 0, 16); auto w = prsgd::philox4x32_10({c[0], c[1], c[2], c[3]}, (uint64_t)c[5] << 32 | c[4]); '
                   'printf("%08x %08x %08x %08x", w.x, w.y, w.z, w.w); }\n')
    subprocess.run(["g++", "-O1", "-I" + CSRC, str(src), "-o", str(tmp_path / "p")], check=True)
    for c, k, want in cases:
        out = subprocess.run([str(tmp_path / "p")] + ["%x" % w for w in c + k], capture_output=True, text=True, check=True).stdout
        assert out == want
        assert " ".join("%08x" % int(w) for w in ref.philox(c, k[1] << 32 | k[0])) == want


@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.9, 1 - 2.0 ** -16])
def test_keep_of_one_element(b, p):
    for seed, step, g0 in ((0, 0, 0), (2 ** 64 - 1, 2 ** 33 + 5, 3), (0x123456789ABCDEF, -1, 2 ** 32 - 1)):
        want = ref.dropout_keep(2, 3, 21, p, seed, step, g0)
        got = [[[b.prsgd_dropout_keep(seed, g0 + g, r, c, step, p) for c in range(21)] for r in range(3)] for g in range(2)]
        assert np.array_equal(want, np.array(got))
    with pytest.raises(b.PRSGDError):
        b.prsgd_dropout_keep(0, 0, 0, -1, 0, p)


def test_share_of_kept_elements():
    """Binomial: five deviations of 1e6 draws."""
    for p in (0.1, 0.5):
        keep = ref.dropout_keep(2, 500, 1000, p, 99, 7)
        assert abs(keep.mean() - (1 - p)) < 5 * (p * (1 - p) / keep.size) ** 0.5 + 2.0 ** -17
        assert abs((keep[0] & keep[1]).mean() - (1 - p) ** 2) < 5 * 0.5 / (keep.size / 2) ** 0.5


def test_reference_gradients_by_differences():
    """vocab_grad against central differences of vocab_loss, embed_grad against embed's linearity."""
    g = torch.Generator().manual_seed(3)
    H, W = torch.randn(2, 5, 6, generator=g, dtype=torch.float64), torch.randn(2, 9, 6, generator=g, dtype=torch.float64)
    y = torch.tensor([[0, 8, -1, 3, 3], [2, 2, 9, 1, 0]], dtype=torch.int32)
    dl, ds = torch.randn(2, 5, generator=g, dtype=torch.float64), torch.randn(2, 5, generator=g, dtype=torch.float64)

    def f(H, W):
        loss, stats = ref.vocab_loss(H, W, y)
        return (loss * dl).sum() + (stats.sum(-1) * ds * ref.live_tokens(y, 9)).sum()
    dH, dW = ref.vocab_grad(H, W, y, dl, ds)[:2]
    h = 1e-6
    for x, d, other in ((H, dH, False), (W, dW, True)):
        for i in range(0, x.numel(), 7):
            e = torch.zeros_like(x)
            e.view(-1)[i] = h
            num = (f(H, W + e) - f(H, W - e) if other else f(H + e, W) - f(H - e, W)) / (2 * h)
            assert abs(num - d.view(-1)[i]) < 1e-8 * (1 + abs(num))
    ids, dout = torch.tensor([[1, 1, -3, 4], [0, 7, 4, 4]], dtype=torch.int32), torch.randn(2, 4, 3, generator=g, dtype=torch.float64)
    table = torch.randn(2, 5, 3, generator=g, dtype=torch.float64)
    assert torch.allclose((ref.embed(table, ids, 0.5) * dout).sum(), (ref.embed_grad(dout, ids, 5, 0.5)[0] * table).sum())


def test_python_checks(b):
    x = torch.zeros(2, 3, 4)
    for call in (lambda: b.prsgd_embed(x, torch.zeros(2, 3, dtype=torch.int32)), lambda: b.prsgd_dropout(x, 0.1, 1),
                 lambda: b.prsgd_vocab_loss(x, x, torch.zeros(2, 3, dtype=torch.int32)), lambda: b.prsgd_embed_grad(x, torch.zeros(2, 3, dtype=torch.int32), x)):
        with pytest.raises(ValueError, match="on the GPU"):
            call()
    W = torch.zeros(2, 10, 16, dtype=torch.bfloat16)
    assert b._rows_aligned is not None and b.TYPES[W.dtype] == 1
    small = b.prsgd_vocab_loss_grad_workspace_bytes(1, 1, 4096, 32000, 1024, 1)
    assert 0 < small <= b.prsgd_vocab_loss_grad_workspace_bytes(1, 1, 4096, 32000, 1024, 0)
