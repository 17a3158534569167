"""The training operators' checks of arguments, and the references the GPU tests compare with: no kernel is launched."""
import ctypes as C

import pytest
import torch

import operator_reference as ref

OK, ARG, ALIGN, SIZE = 0, -1, -2, -3


@pytest.fixture(scope="module")
def binding():
    from paper_1807_06629_b200 import _build
    _build.build_library()
    from paper_1807_06629_b200 import binding as b
    return b


def ortho(lib, **kw):
    a = dict(G=4096, gt=0, gr=64, gb=4096, out=8192, ot=0, orow=64, ob=4096, batch=2, rows=64, cols=64, steps=5, coefs=None,
             scale=1.0, eps=1e-7, precision=1, work=65536, bytes=1 << 30)
    a.update(kw)
    return lib.prsgd_orthogonalize(*a.values(), None)


def test_orthogonalize_refusals(binding):
    lib = binding.lib
    for kw, want in [(dict(G=None), ARG), (dict(out=None), ARG), (dict(gt=3), ARG), (dict(ot=-1), ARG), (dict(gr=63), ARG),
                     (dict(orow=63), ARG), (dict(gb=-1), ARG), (dict(ob=4095), ARG), (dict(batch=-1), ARG), (dict(rows=-1), ARG),
                     (dict(cols=-2), ARG), (dict(batch=65536), SIZE), (dict(rows=65537), SIZE), (dict(steps=0), ARG), (dict(steps=17), ARG),
                     (dict(scale=float("nan")), ARG), (dict(scale=float("inf")), ARG), (dict(eps=-1.0), ARG), (dict(eps=float("nan")), ARG),
                     (dict(precision=2), ARG), (dict(work=None), SIZE), (dict(bytes=256), SIZE), (dict(work=65536 + 128), ALIGN),
                     (dict(G=4098), ALIGN), (dict(out=8193, ot=1), ALIGN), (dict(coefs=(C.c_float * 3)(1.0, 17.0, 0.0)), ARG),
                     (dict(coefs=(C.c_float * 3)(1.0, float("nan"), 0.0)), ARG)]:
        assert ortho(lib, **kw) == want, kw
        assert lib.prsgd_last_error(None)
    for kw in (dict(batch=0), dict(rows=0), dict(cols=0)):          # nothing to do: not even the pointers are looked at
        assert ortho(lib, G=None, out=None, work=None, **kw) == OK


def test_orthogonalize_workspace_covers_what_a_call_holds(binding):
    for rows, cols in ((1, 1), (10, 1024), (777, 300)):
        s = min(rows, cols)
        small = binding.prsgd_orthogonalize_workspace_bytes(3, rows, cols, binding.PRECISION_BF16)
        big = binding.prsgd_orthogonalize_workspace_bytes(3, rows, cols, binding.PRECISION_FP32)
        assert small >= 3 * 2 * (4 * rows * cols + 2 * s * s) and big >= 3 * 2 * (4 * rows * cols + 4 * s * s)
    n = C.c_size_t()
    assert binding.lib.prsgd_orthogonalize_workspace_bytes(1, 2, 3, 0, None) == ARG
    assert binding.lib.prsgd_orthogonalize_workspace_bytes(1, 2, 3, 5, C.byref(n)) == ARG
    assert binding.lib.prsgd_orthogonalize_workspace_bytes(1, 1 << 17, 3, 0, C.byref(n)) == SIZE


def test_muon_refusals(binding):
    def call(**kw):
        a = dict(W=4096, wt=0, wr=64, wb=4096, V=8192, vr=64, vb=4096, G=12288, gt=0, gr=64, gb=4096, batch=2, rows=64, cols=64,
                 lr=0.1, mu=0.9, nesterov=1, wd=0.0, steps=5, coefs=None, scale=1.0, eps=1e-7, precision=0, work=65536, bytes=1 << 30)
        a.update(kw)
        return binding.lib.prsgd_muon_step(*a.values(), None)
    for kw, want in [(dict(W=None), ARG), (dict(V=None), ARG), (dict(G=None), ARG), (dict(mu=1.0), ARG), (dict(mu=-0.1), ARG),
                     (dict(mu=float("nan")), ARG), (dict(lr=float("inf")), ARG), (dict(wd=float("nan")), ARG), (dict(lr=0.5, wd=2.0), ARG),
                     (dict(vb=64), ARG), (dict(wb=64), ARG), (dict(vr=1), ARG), (dict(V=8194), ALIGN), (dict(work=None), SIZE),
                     (dict(steps=0), ARG), (dict(precision=9), ARG)]:
        assert call(**kw) == want, kw
    assert call(batch=0, W=None, V=None, G=None, work=None) == OK


def test_route_refusals(binding):
    lib = binding.lib

    def call(**kw):
        a = dict(x=4096, ty=1, rs=64, gs=6400, live=None, G=2, T=100, E=64, k=4, norm=0, coef=0.01, e=256, w=256, c=256, m=256, l=256,
                 work=65536, bytes=1 << 30)
        a.update(kw)
        return lib.prsgd_route(*a.values(), None)

    def grad(**kw):
        a = dict(x=4096, ty=1, rs=64, gs=6400, live=None, G=2, T=100, E=64, k=4, norm=0, coef=0.01, e=256, c=256, dw=256, dl=256,
                 d=8192, drs=64, dgs=6400)
        a.update(kw)
        return lib.prsgd_route_grad(*a.values(), None)

    common = [(dict(x=None), ARG), (dict(ty=7), ARG), (dict(rs=63), ARG), (dict(gs=-1), ARG), (dict(G=-1), ARG), (dict(T=-1), ARG),
              (dict(E=0), ARG), (dict(k=0), ARG), (dict(k=65), ARG), (dict(E=100, rs=100, k=33), ARG), (dict(E=1025, rs=1025), SIZE),
              (dict(G=65536), SIZE), (dict(T=(1 << 24) + 1), SIZE), (dict(x=4097), ALIGN)]
    for kw, want in common + [(dict(e=None), ARG), (dict(w=None), ARG), (dict(c=None), ARG), (dict(m=None), ARG), (dict(l=None), ARG),
                              (dict(work=None), SIZE), (dict(bytes=16), SIZE), (dict(work=65540), ALIGN)]:
        assert call(**kw) == want, kw
    for kw, want in common + [(dict(d=None), ARG), (dict(c=None), ARG), (dict(e=None), ARG), (dict(drs=63), ARG), (dict(dgs=64), ARG),
                              (dict(d=8193), ALIGN)]:
        assert grad(**kw) == want, kw
    assert call(G=0, x=None, c=None, work=None) == OK
    assert grad(G=0, x=None, c=None, d=None) == OK and grad(T=0, x=None, d=None, c=None) == OK
    n = C.c_size_t()
    assert lib.prsgd_route_workspace_bytes(1, 1, 8, None) == ARG
    assert lib.prsgd_route_workspace_bytes(1, 1, 2000, C.byref(n)) == ARG


def test_the_binding_checks_tensors(binding):
    x = torch.zeros(2, 8, 8)
    with pytest.raises(ValueError):
        binding._matrices(x, "G")                                   # not on the GPU
    with pytest.raises(ValueError):
        binding._dense(torch.zeros(3), "loss", torch.float32, 2, -1)


# ---- the references themselves ---------------------------------------------------------------------------
def test_reference_newton_schulz_is_the_polynomial_of_the_singular_values():
    g = torch.Generator().manual_seed(0)
    for shape in ((6, 9), (9, 6), (5, 5), (1, 4)):
        G = torch.randn(2, *shape, generator=g, dtype=torch.float64)
        u, s, v = torch.linalg.svd(G, full_matrices=False)
        t = s / (s.square().sum(-1, keepdim=True).sqrt() + 1e-7)
        a, b, c = ref.COEFS
        for _ in range(5):
            t = a * t + b * t ** 3 + c * t ** 5
        assert torch.allclose(ref.orthogonalize(G), u @ torch.diag_embed(t) @ v, rtol=0, atol=1e-11)


def test_reference_route_by_hand():
    x = torch.tensor([[[0.0, 2.0, 2.0, -1.0], [float("-inf")] * 4, [1.0, 1.0, 1.0, 1.0]]])
    live = torch.tensor([[1, 1, 1]], dtype=torch.uint8)
    chosen, w, counts, mean, loss = ref.route(x, 2, 0.5, live=live)
    assert chosen.tolist() == [[[1, 2], [-1, -1], [0, 1]]] and counts.tolist() == [[1, 2, 1, 0]]
    p = torch.softmax(x[0, 0].double(), 0)
    assert torch.allclose(mean[0], (p + 0.25) / 2) and torch.allclose(w[0, 0], p[1:3])
    assert loss.item() == pytest.approx(0.5 * 4 * sum(f * m for f, m in zip([.25, .5, .25, 0], mean[0].tolist())))


def test_reference_route_gradient_against_differences():
    g = torch.Generator().manual_seed(1)
    x = torch.randn(2, 5, 6, generator=g, dtype=torch.float64)
    live = torch.tensor([[1, 1, 0, 1, 1], [0, 0, 0, 0, 0]], dtype=torch.uint8)
    dw, dl = torch.randn(2, 5, 3, generator=g, dtype=torch.float64), torch.rand(2, generator=g, dtype=torch.float64)
    for normalize in (False, True):
        chosen, _, counts, _, _ = ref.route(x, 3, 0.1, normalize, live)
        grad = ref.route_grad(x, chosen, counts, 0.1, normalize, live, dw, dl)
        on = ref.alive(x, live)
        for t in range(5):
            for e in range(6):
                h = torch.zeros_like(x)
                h[0, t, e] = 1e-5
                f = [ref.route_objective(x + s * h, chosen, counts, on, 0.1, normalize, dw, dl).item() for s in (1, -1)]
                assert (f[0] - f[1]) / 2e-5 == pytest.approx(grad[0, t, e].item(), abs=1e-9)
        assert (grad[1] == 0).all() and (grad[0, 2] == 0).all()
