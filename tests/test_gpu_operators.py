"""The stand-alone training operators on the GPU against their formulas in 64 bits (tests/operator_reference.py).

Tolerances (2-norm of the difference over the result's norm unless said otherwise), with half-steps bf16 2^-8,
fp16 2^-11, fp32 2^-24:
 * Newton-Schulz, 32-bit precision.  X, A and P are pairs of fp16 values (relative 2^-22 each).  A step's polynomial
   weighs them with 1, |b| and 2 |c|: a relative perturbation of rms (1 + 4.8 + 4.1) 2^-22 / sqrt(3) = 1.4e-6, which
   later steps multiply by at most |f'| = 2.3 on the singular values the iteration holds; random errors add in
   square, sqrt(sum_{k<5} 2.3^2k) = 26 at most: 3.6e-5, allowed 5e-5.
 * 16-bit precision.  Single fp16 operands: rms rounding 2^-11 / sqrt(3) = 2.8e-4 where the pairs have 2^-22 / sqrt(3).
   The same worst growth would allow 7e-2; rounding errors of single elements are spread over all singular
   directions, of which few sit where |f'| is large, and an emulation in numpy over Gaussian, low-rank and decaying spectra
   (sides 10 to 2048) stays below 2.6e-3: allowed 6e-3, plus the half-step of the output's type.
 * Router: expf within 2 ulp, sums of E <= 1024 terms and of T <= 2^12 tokens in fp32 by lanes and blocks (each
   partial sum is at most 2^7 long): 2^7 2^-24 = 8e-6 relative at worst, typically a tenth; allowed 5e-6 by element
   for the weights (no long sums), 1e-5 for mean and loss.
 * Router gradient: the same over p, then a difference h - sum p h of terms of one size: 2e-5 of the largest gradient of
   the token by element, plus the half-step of the output's type.
"""
import math

import numpy as np
import pytest
import torch

import operator_reference as ref

pytestmark = pytest.mark.gpu

TOL = {0: 5e-5, 1: 6e-3}
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def b():
    from paper_1807_06629_b200 import _build
    _build.build_library()
    from paper_1807_06629_b200 import binding
    assert torch.cuda.is_available()
    return binding


def gen(seed):
    g = torch.Generator(device="cuda:0")
    g.manual_seed(seed)
    return g


def matrices(seed, batch, rows, cols, rank=None, dtype=F32):
    g = gen(seed)
    if rank is None:
        return torch.randn(batch, rows, cols, generator=g, device="cuda:0").to(dtype)
    return (torch.randn(batch, rows, rank, generator=g, device="cuda:0") @ torch.randn(batch, rank, cols, generator=g, device="cuda:0")).to(dtype)


def rel(got, want):
    return ((got.double() - want).norm() / want.norm()).item()


def half_step(dtype):
    return torch.finfo(dtype).eps / 2 if dtype != F32 else 0.0


def poisoned(n_bytes):
    """A workspace whose contents are NaN whatever they are read as."""
    return torch.full((n_bytes,), 0xFF, dtype=torch.uint8, device="cuda:0")


def workspace(b, G, precision):
    return poisoned(b.prsgd_orthogonalize_workspace_bytes(*G.shape, precision))


SHAPES = [(1, 1, 1), (2, 1, 7), (2, 7, 1), (3, 5, 5), (16, 10, 1024), (1, 64, 64), (2, 63, 65), (1, 128, 128), (2, 129, 257),
          (1, 128, 700), (1, 300, 77), (3, 100, 2100), (2, 2100, 90), (2, 256, 512), (1, 515, 300), (2, 257, 1030), (5, 520, 520), (1, 1000, 700)]


# ---- orthogonalisation -------------------------------------------------------------------------------------
@pytest.mark.parametrize("precision", [0, 1])
@pytest.mark.parametrize("shape", SHAPES)
def test_orthogonalize_matches_the_formula(b, shape, precision):
    G = matrices(1, *shape)
    got = b.prsgd_orthogonalize(G, precision=precision, workspace=(w := workspace(b, G, precision)))
    b.prsgd_work_status(w)
    want = ref.orthogonalize(G)
    assert rel(got, want) <= TOL[precision]
    for i in range(shape[0]):                          # every matrix by itself
        assert rel(got[i], want[i]) <= TOL[precision] * 2


@pytest.mark.parametrize("shape", [(2, 300, 515), (1, 700, 260), (2, 60, 90)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_orthogonalize_of_a_type_is_as_exact_as_the_type(b, dtype, shape):
    """Without a precision asked for: a half-step of the result's type beside what the chain allows, single operands for
    bfloat16, pairs for float16 and float32."""
    G = matrices(29, *shape, dtype=dtype)
    got = b.prsgd_orthogonalize(G)
    assert got.dtype == dtype
    assert rel(got, ref.orthogonalize(G)) <= half_step(dtype) + (TOL[1] if dtype == BF16 else TOL[0])
    assert torch.equal(got, b.prsgd_orthogonalize(G, workspace=b.orthogonalize_workspace(G)))


@pytest.mark.parametrize("steps", [1, 2, 5])
@pytest.mark.parametrize("shape", [(3, 15, 900), (9, 16, 129), (2, 17, 2048), (2, 32, 2048), (2, 2047, 31), (40, 32, 64), (1, 33, 1500), (2, 700, 48), (3, 64, 2048),
                                   (3, 65, 1536), (2, 112, 1300), (4, 1000, 10), (2, 300, 2500), (1, 2700, 520)])
def test_orthogonalize_forms_by_short_side_and_number_of_parts(b, shape, steps):
    """Short sides around 16, 32, 64 and 128 in clusters of 1 to 8, and chains whose X X^T is formed in parts; twice, the same bits."""
    G = matrices(23, *shape)
    for precision in (0, 1):
        got = b.prsgd_orthogonalize(G, steps=steps, precision=precision, workspace=(w := workspace(b, G, precision)))
        again = b.prsgd_orthogonalize(G, steps=steps, precision=precision, workspace=w)
        b.prsgd_work_status(w)
        assert torch.equal(got, again)
        assert rel(got, ref.orthogonalize(G, steps=steps)) <= TOL[precision]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("out_dtype", [F32, BF16, F16])
def test_orthogonalize_types(b, dtype, out_dtype):
    G = matrices(2, 2, 130, 190, dtype=dtype)
    out = torch.empty(2, 130, 190, dtype=out_dtype, device="cuda:0")
    b.prsgd_orthogonalize(G, out=out, scale=0.5)
    tol = TOL[0 if out_dtype == F32 else 1] + half_step(out_dtype)
    assert rel(out, 0.5 * ref.orthogonalize(G)) <= tol


@pytest.mark.parametrize("precision", [0, 1])
@pytest.mark.parametrize("rank,shape", [(1, (2, 96, 160)), (4, (1, 300, 520)), (8, (2, 520, 260)), (32, (1, 640, 640))])
def test_orthogonalize_of_low_rank(b, rank, shape, precision):
    """Directions that G does not contain grow 485-fold over five steps: what rounding leaves there must stay small.
    (Products in fp32, 2^-24 sqrt(K) of their size, and pairs of 2^-22 leave 485 2^-22 = 1.2e-4 of the result at
    rank 1; with 16-bit precision the last step rounds X alone, 3.44 2^-11 / sqrt(3) = 1e-3, inside its allowance.)"""
    G = matrices(3, *shape, rank=rank)
    got = b.prsgd_orthogonalize(G, precision=precision)
    assert rel(got, ref.orthogonalize(G)) <= (1.5e-4 if precision == 0 else TOL[1])


@pytest.mark.parametrize("steps,coefs", [(1, None), (2, None), (7, None), (16, (1.5, -0.5, 0.0)), (3, (2.0, -1.5, 0.5))])
def test_orthogonalize_steps_and_coefficients(b, steps, coefs):
    G = matrices(4, 2, 70, 300)
    got = b.prsgd_orthogonalize(G, steps=steps, coefs=coefs)
    assert rel(got, ref.orthogonalize(G, steps, coefs or ref.COEFS)) <= TOL[0]


@pytest.mark.parametrize("size", [1e-30, 1e-12, 1e30])
def test_orthogonalize_over_the_range_of_fp32(b, size):
    G = matrices(5, 2, 40, 150) * size
    got = b.prsgd_orthogonalize(G, eps=0.0)
    assert rel(got, ref.orthogonalize(G, eps=0.0)) <= TOL[0]


@pytest.mark.parametrize("shape", [(4, 60, 90), (4, 200, 300)])
def test_zero_and_non_finite_matrices_stay_by_themselves(b, shape):
    G = matrices(6, *shape)
    G[1] = 0
    G[2, 7, 5] = float("nan")
    G[3, 0, 0] = float("inf")
    for precision in (0, 1):
        got = b.prsgd_orthogonalize(G, precision=precision)
        assert rel(got[0], ref.orthogonalize(G[:1])[0]) <= TOL[precision]
        assert (got[1] == 0).all()
        assert got[2].isnan().all() and not got[3].isfinite().any()


@pytest.mark.parametrize("shape", [(3, 33, 70), (2, 150, 270), (2, 270, 150)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_orthogonalize_strides_alignment_and_aliasing(b, shape, dtype):
    B, R, Cn = shape
    G = matrices(7, *shape, dtype=dtype)
    want = ref.orthogonalize(G)
    tol = TOL[0 if dtype == F32 else 1] + half_step(dtype)
    wide = torch.full((B, R + 2, Cn + 3), float("nan"), dtype=dtype, device="cuda:0")
    wide[:, 1:R + 1, 1:Cn + 1] = G
    view = wide[:, 1:R + 1, 1:Cn + 1]
    out = torch.full((B, R + 1, Cn + 5), 7.0, dtype=dtype, device="cuda:0")
    b.prsgd_orthogonalize(view, out=out[:, :R, 1:Cn + 1])
    assert rel(out[:, :R, 1:Cn + 1], want) <= tol
    assert (out[:, R:] == 7).all() and (out[:, :, 0] == 7).all() and (out[:, :, Cn + 1:] == 7).all()   # nothing beside it is written
    assert wide[:, 0].isnan().all() and wide[:, R + 1].isnan().all()
    b.prsgd_orthogonalize(view, out=view)              # in place
    assert rel(view, want) <= tol
    one = G[:1].expand(B, R, Cn)                       # one matrix for all
    got = b.prsgd_orthogonalize(one)
    assert all(torch.equal(got[i], got[0]) for i in range(B)) and rel(got[0], want[0]) <= tol
    assert rel(b.prsgd_orthogonalize(G[0]), want[0]) <= tol


@pytest.mark.parametrize("shape", [(3, 48, 100), (3, 300, 200)])
def test_orthogonalize_is_deterministic_streams_and_workspaces(b, shape):
    G, H = matrices(8, *shape), matrices(9, *shape)
    first, other = b.prsgd_orthogonalize(G).clone(), b.prsgd_orthogonalize(H).clone()
    w = workspace(b, G, 0)
    for _ in range(3):                                 # one workspace, calls in turn, nothing carried over
        assert torch.equal(b.prsgd_orthogonalize(G, workspace=w), first)
        assert torch.equal(b.prsgd_orthogonalize(H, workspace=w), other)
    streams = [torch.cuda.Stream() for _ in range(2)]  # two at once, a workspace each: the caller's, then the binding's
    mine = [workspace(b, G, 0), workspace(b, H, 0)]
    torch.cuda.synchronize()
    outs = []
    for i in range(6):
        for s, x, w in zip(streams, (G, H), mine):
            outs.append((b.prsgd_orthogonalize(x, workspace=w if i < 3 else None, stream=s), x is G))
    torch.cuda.synchronize()
    for got, is_g in outs:
        assert torch.equal(got, first if is_g else other)


@pytest.mark.parametrize("shape", [(3, 48, 100), (2, 300, 400)])
def test_orthogonalize_captured_and_replayed(b, shape):
    G, H = matrices(10, *shape), matrices(11, *shape)
    want_g, want_h = b.prsgd_orthogonalize(G).clone(), b.prsgd_orthogonalize(H).clone()
    x, out, w = G.clone(), torch.empty_like(G), workspace(b, G, 0)
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        b.prsgd_orthogonalize(x, out=out, workspace=w)
    for src, want in ((G, want_g), (H, want_h), (G, want_g)):
        x.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_orthogonalize_of_nothing(b):
    for shape in ((0, 4, 4), (2, 0, 4), (2, 4, 0)):
        assert b.prsgd_orthogonalize(torch.zeros(*shape, device="cuda:0")).shape == shape


# ---- Muon step -----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("dtype,shape", [(F32, (2, 64, 200)), (BF16, (2, 64, 200)), (F32, (2, 300, 140)), (BF16, (3, 257, 400)), (F16, (1, 33, 17))])
def test_muon_steps(b, dtype, shape, nesterov):
    W, V = matrices(20, *shape, dtype=dtype) / math.sqrt(shape[2]), torch.zeros(shape, device="cuda:0")
    w, v = W.double(), V.double()
    lr, mu, wd, scale = 0.05, 0.9, 0.1, 0.7
    ws = workspace(b, W, b._precision_for(W))
    for step in range(3):
        G = matrices(21 + step, *shape, dtype=dtype)
        new_w, new_v = ref.muon(W, V, G, lr, mu, nesterov, wd, scale)    # from what the step is given
        moved = (new_w - (1 - lr * wd) * W.double()).norm().item()
        b.prsgd_muon_step(W, V, G, lr, mu=mu, nesterov=nesterov, weight_decay=wd, scale=scale, workspace=ws)
        assert rel(V, new_v) <= 2.0 ** -23             # one product and sum
        off = (W.double() - new_w).norm().item()
        assert off <= TOL[0 if dtype == F32 else 1] * moved + max(half_step(dtype), 2.0 ** -23) * new_w.norm().item()


def test_muon_leaves_the_rest_alone_and_takes_mixed_types(b):
    shape = (2, 70, 130)
    W = torch.full((2, 72, 140), 3.0, device="cuda:0")
    V = torch.full((2, 71, 133), 5.0, device="cuda:0")
    W[:, :70, :130], V[:, :70, :130] = matrices(30, *shape) * 0.1, matrices(31, *shape)
    w, v = W[:, :70, :130], V[:, :70, :130]
    G = matrices(32, *shape, dtype=BF16)
    want_w, want_v = ref.muon(w, v, G, 0.1, 0.95, True, 0.0, 1.0)
    b.prsgd_muon_step(w, v, G, 0.1)
    assert rel(w, want_w) <= TOL[0] and rel(v, want_v) <= 2.0 ** -23
    assert (W[:, 70:] == 3).all() and (W[:, :, 130:] == 3).all() and (V[:, 70:] == 5).all() and (V[:, :, 130:] == 5).all()


# ---- router --------------------------------------------------------------------------------------------------
def logits_of(seed, G, T, E, dtype=F32, grid=None):
    x = torch.randn(G, T, E, generator=gen(seed), device="cuda:0") * 2
    if grid:
        x = (x * grid).round() / grid                  # many ties
    return x.to(dtype)


def check_route(b, x, k, coef=0.01, normalize=False, live=None):
    got = b.prsgd_route(x, k, coef, normalize=normalize, live=live, workspace=poisoned(b.prsgd_route_workspace_bytes(*x.shape)))
    want = ref.route(x, k, coef, normalize, live)
    assert torch.equal(got[0].long(), want[0]) and torch.equal(got[2].long(), want[2])
    assert (got[1].double() - want[1]).abs().max() <= 5e-6 if got[1].numel() else True
    assert (got[3].double() - want[3]).abs().max() <= 1e-5 * max(want[3].max().item(), 1e-30)
    assert ((got[4].double() - want[4]).abs() <= 1e-5 * want[4].abs()).all()
    return got


@pytest.mark.parametrize("normalize", [False, True])
@pytest.mark.parametrize("T", [1, 2, 33, 700])
@pytest.mark.parametrize("E,k", [(1, 1), (2, 2), (5, 3), (8, 2), (31, 31), (32, 8), (33, 1), (64, 8), (65, 4), (100, 3), (128, 8), (200, 32), (257, 6), (512, 8), (1024, 4)])
def test_route_matches_the_formula(b, E, k, T, normalize):
    check_route(b, logits_of(40 + T, 3, T, E), k, normalize=normalize)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("E,k", [(8, 3), (64, 8), (96, 5), (300, 7)])
def test_route_types_and_ties_go_to_the_lowest_index(b, dtype, E, k):
    check_route(b, logits_of(41, 2, 300, E, dtype, grid=2), k, normalize=True)
    same = torch.zeros(1, 5, E, dtype=dtype, device="cuda:0")
    same[0, 1] = -0.0
    got = check_route(b, same, k)
    assert (got[0] == torch.arange(k, device="cuda:0")).all()


@pytest.mark.parametrize("E,k", [(6, 2), (64, 8), (130, 4)])
def test_route_masks(b, E, k):
    G, T = 4, 150
    x = logits_of(42, G, T, E)
    live = (torch.rand(G, T, generator=gen(43), device="cuda:0") < 0.6).to(torch.uint8)
    live[2] = 0                                        # a group without tokens
    x[live == 0] = float("nan")                        # whatever padding holds
    x[0, 0], live[0, 0] = float("-inf"), 1             # a live token without any expert
    x[1, 3, 1:] = float("-inf")                        # ... with one
    x[1, 4, : E - 1] = torch.finfo(F32).min            # ... with the type's lowest value
    live[1, 3] = live[1, 4] = 1
    x[1, 3, 0], x[1, 4, E - 1] = 0.5, 1.0
    got = check_route(b, x, k, live=live, normalize=False)
    assert (got[0][2] == -1).all() and (got[1][2] == 0).all() and (got[2][2] == 0).all() and got[4][2] == 0
    assert (got[0][0, 0] == -1).all() and got[0][1, 3, 0] == 0 and got[0][1, 4, 0] == E - 1
    check_route(b, x, k, live=live, normalize=True)


@pytest.mark.parametrize("E,k,G,T", [(64, 8, 5, 65), (64, 8, 36, 512), (64, 8, 37, 513), (64, 4, 3, 1024), (64, 4, 3, 1025), (1000, 2, 2, 128), (1000, 8, 2, 129), (128, 8, 140, 128),
                                     (7, 2, 2, 4096), (129, 3, 1, 513), (1024, 3, 2, 3000)])
def test_route_groups_of_one_cluster_and_of_many_blocks(b, E, k, G, T):
    """Both sides of where a group's blocks are a cluster; twice, the same bits; every third token off, one group all off."""
    x = logits_of(48, G, T, E)
    live = torch.ones(G, T, dtype=torch.uint8, device="cuda:0")
    live[:, ::3] = 0
    live[G - 1] = 0
    got = check_route(b, x, k, live=live, normalize=True)
    again = b.prsgd_route(x, k, 0.1, normalize=True, live=live)
    for p, q in zip(got[:4], again[:4]):
        assert torch.equal(p, q)


def test_route_with_nan_in_a_live_token(b):
    x = logits_of(44, 3, 40, 16)
    x[1, 5, 3] = float("nan")
    experts, weights, counts, mean, loss = b.prsgd_route(x, 2, 0.1)
    want = ref.route(x, 2, 0.1)
    assert experts[1, 5, 0] == 3 and weights[1, 5].isnan().all()
    assert mean[1].isnan().all() and loss[1].isnan() and counts[1].sum() == 80
    for g in (0, 2):
        assert torch.equal(experts[g].long(), want[0][g]) and abs(loss[g].item() - want[4][g].item()) <= 1e-5 * want[4][g].item()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_route_strides_and_alignment(b, dtype):
    for E, off in ((64, 1), (64, 4), (50, 3), (128, 8)):
        big = torch.full((2, 90, E + 9), float("nan"), dtype=dtype, device="cuda:0")
        big[:, :80, off:off + E] = logits_of(45, 2, 80, E, dtype)
        check_route(b, big[:, :80, off:off + E], 4)
    one = logits_of(46, 1, 30, 64, dtype).expand(3, 30, 64)
    got = check_route(b, one, 2)
    assert torch.equal(got[0][0], got[0][2])
    check_route(b, logits_of(47, 1, 30, 64, dtype), 2)


def test_route_of_nothing_and_many_groups(b):
    x = torch.zeros(2, 0, 8, device="cuda:0")
    experts, weights, counts, mean, loss = b.prsgd_route(x, 2, 0.1)
    assert experts.shape == (2, 0, 2) and (counts == 0).all() and (mean == 0).all() and (loss == 0).all()
    check_route(b, logits_of(48, 700, 3, 16), 2)
    check_route(b, logits_of(49, 1, 9001, 24), 2)


def test_route_is_deterministic_and_can_be_captured(b):
    x, y = logits_of(50, 4, 3000, 64), logits_of(51, 4, 3000, 64)
    want = [[t.clone() for t in b.prsgd_route(v, 6, 0.02, normalize=True)] for v in (x, y)]
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in zip(b.prsgd_route(x, 6, 0.02, normalize=True), want[0]))
    z, outs, w = x.clone(), b.route_outputs(x, 6), b.route_workspace(x)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        b.prsgd_route(z, 6, 0.02, normalize=True, out=outs, workspace=w)
    for i in (0, 1, 0):
        z.copy_((x, y)[i])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(outs, want[i]))


# ---- router gradient -----------------------------------------------------------------------------------------
def check_grad(b, x, k, normalize, live=None, use=("dw", "dl"), seed=60):
    G, T, E = x.shape
    chosen, _, counts, _, _ = ref.route(x, k, 0.05, normalize, live)
    dw = torch.randn(G, T, k, generator=gen(seed), device="cuda:0") if "dw" in use else None
    dl = (torch.rand(G, generator=gen(seed + 1), device="cuda:0") + 0.5) * T if "dl" in use else None
    got = b.prsgd_route_grad(x, chosen.int(), counts.int(), 0.05, normalize=normalize, live=live, dweights=dw, dloss=dl)
    want = ref.route_grad(x, chosen, counts, 0.05, normalize, live, dw, dl)
    size = want.abs().amax(-1, keepdim=True)
    # dlogit_te = p (h - sum p h): its error scales with p |h|, |h| up to the largest of the token's upstream gradients (and 1 / sum of the chosen p)
    if dw is not None:
        p = torch.softmax(torch.where(ref.alive(x, live)[..., None], x.double(), 0.0), -1)
        size = torch.maximum(size, p.amax(-1, keepdim=True) * dw.abs().amax(-1, keepdim=True).double())
    tiny = torch.finfo(x.dtype).smallest_normal * torch.finfo(x.dtype).eps      # a half-step of what is below the normal numbers
    assert ((got.double() - want).abs() <= 2e-5 * size + half_step(x.dtype) * want.abs() * 1.01 + tiny).all()
    return got


@pytest.mark.parametrize("normalize", [False, True])
@pytest.mark.parametrize("T", [1, 3, 257])
@pytest.mark.parametrize("E,k", [(1, 1), (2, 1), (5, 3), (31, 31), (32, 8), (64, 8), (65, 4), (100, 3), (128, 8), (257, 6), (1024, 32)])
def test_route_grad_matches_the_formula(b, E, k, T, normalize):
    check_grad(b, logits_of(61, 3, T, E), k, normalize)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("use", [("dw",), ("dl",), ("dw", "dl"), ()])
def test_route_grad_types_and_parts(b, dtype, use):
    got = check_grad(b, logits_of(62, 2, 100, 48, dtype), 4, True, use=use)
    if not use:
        assert (got == 0).all()


@pytest.mark.parametrize("E", [6, 64, 130])
@pytest.mark.parametrize("normalize", [False, True])
def test_route_grad_masks(b, E, normalize):
    x = logits_of(63, 3, 70, E)
    live = (torch.rand(3, 70, generator=gen(64), device="cuda:0") < 0.5).to(torch.uint8)
    live[1] = 0
    x[live == 0] = float("nan")
    x[0, 0], live[0, 0] = float("-inf"), 1
    x[0, 1, 2:], live[0, 1] = float("-inf"), 1
    x[0, 1, :2] = 0.25
    got = check_grad(b, x, 2, normalize, live)
    assert (got[live == 0] == 0).all() and (got[0, 0] == 0).all() and (got[1] == 0).all()


def test_route_grad_strides_and_in_place(b):
    big = torch.full((2, 60, 80), float("nan"), device="cuda:0")
    big[:, :50, 3:67] = logits_of(65, 2, 50, 64)
    x = big[:, :50, 3:67]
    want = check_grad(b, x, 4, True)
    chosen, _, counts, _, _ = ref.route(x, 4, 0.05, True)
    dw, dl = torch.randn(2, 50, 4, generator=gen(60), device="cuda:0"), (torch.rand(2, generator=gen(61), device="cuda:0") + 0.5) * 50
    out = torch.full((2, 51, 70), 9.0, device="cuda:0")
    b.prsgd_route_grad(x, chosen.int(), counts.int(), 0.05, normalize=True, dweights=dw, dloss=dl, out=out[:, :50, 2:66])
    assert torch.equal(out[:, :50, 2:66], want) and (out[:, 50:] == 9).all() and (out[:, :, :2] == 9).all() and (out[:, :, 66:] == 9).all()
    b.prsgd_route_grad(x, chosen.int(), counts.int(), 0.05, normalize=True, dweights=dw, dloss=dl, out=x)
    assert torch.equal(x, want)


def test_route_grad_against_differences_of_the_kernel_itself(b):
    """(loss(x + h) - loss(x - h)) / 2h of prsgd_route, where no choice changes: fp32 losses of about 1 differ by about
    2^-23 when rounded, over 2h = 0.02 that is 6e-6 (and h^2 / 6 times the third derivative, below 2e-5)."""
    x = logits_of(66, 1, 4, 5)
    chosen, _, counts, _, _ = b.prsgd_route(x, 2, 1.0)
    dl = torch.ones(1, device="cuda:0")
    grad = b.prsgd_route_grad(x, chosen, counts, 1.0, dloss=dl)
    for t in range(4):
        for e in range(5):
            f = []
            for s in (1e-2, -1e-2):
                y = x.clone()
                y[0, t, e] += s
                out = b.prsgd_route(y, 2, 1.0)
                assert torch.equal(out[2], counts)
                f.append(out[4].item())
            assert abs((f[0] - f[1]) / 2e-2 - grad[0, t, e].item()) <= 5e-5


# ---- beyond 32 bits, and a first call inside a capture ---------------------------------------------------------
def test_offsets_beyond_32_bits(b):
    """Groups and matrices more than 2^31 elements apart."""
    far = (1 << 31) + 4096
    buf = torch.zeros(far + 20000, dtype=BF16, device="cuda:0")
    x = buf.as_strided((2, 50, 64), (far, 64, 1))
    x.copy_(logits_of(90, 2, 50, 64, BF16))
    check_route(b, x, 4)
    chosen, _, counts, _, _ = ref.route(x, 4, 0.05)
    dl = torch.ones(2, device="cuda:0") * 50
    want = b.prsgd_route_grad(x.contiguous(), chosen.int(), counts.int(), 0.05, dloss=dl)
    assert torch.equal(b.prsgd_route_grad(x, chosen.int(), counts.int(), 0.05, dloss=dl, out=x), want) and torch.equal(x, want)
    for shape in ((2, 60, 80), (2, 140, 130)):         # both forms of the chain
        G = buf.as_strided(shape, (far, shape[2], 1))
        G.copy_(matrices(91, *shape, dtype=BF16))
        want = b.prsgd_orthogonalize(G.contiguous())
        assert torch.equal(b.prsgd_orthogonalize(G), want)
        assert torch.equal(b.prsgd_orthogonalize(G, out=G), want) and torch.equal(G, want)


def test_a_process_whose_first_call_is_captured(b):
    """The library finds out what it needs of the device on the first call, which may be inside a capture."""
    import subprocess
    import sys
    code = """
import torch
from paper_1807_06629_b200 import binding as b
G = [torch.randn(2, 40, 90, device="cuda:0"), torch.randn(2, 200, 300, device="cuda:0")]
x = torch.randn(2, 30, 16, device="cuda:0")
work = [b.orthogonalize_workspace(g) for g in G]
out, outs, w = [torch.empty_like(g) for g in G], b.route_outputs(x, 2), b.route_workspace(x)
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    for g, o, k in zip(G, out, work):
        b.prsgd_orthogonalize(g, out=o, workspace=k)
    b.prsgd_route(x, 2, 0.1, out=outs, workspace=w)
graph.replay()
torch.cuda.synchronize()
assert all(torch.equal(b.prsgd_orthogonalize(g), o) for g, o in zip(G, out))
assert all(torch.equal(p, q) for p, q in zip(b.prsgd_route(x, 2, 0.1), outs))
print("same")
"""
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    run = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "same" in run.stdout, run.stderr[-2000:]


# ---- together ------------------------------------------------------------------------------------------------
def test_a_period_of_router_training(b):
    """What the operators are for: N workers train a router's weights by local Muon steps on the balance loss and the
    gradient of the weights, then their models are averaged; against the same in 64 bits from the same choices."""
    N, T, D, E, k = 4, 96, 72, 16, 2
    W = matrices(70, 1, E, D).expand(N, E, D).contiguous() / math.sqrt(D)
    V = torch.zeros_like(W)
    w, v = W.double(), V.double()
    for step in range(3):
        X = matrices(71 + step, N, T, D)
        up = torch.randn(N, T, k, generator=gen(80 + step), device="cuda:0")
        logits = X @ W.mT
        experts, _, counts, _, _ = b.prsgd_route(logits, k, 0.1, normalize=True)
        ones = torch.ones(N, device="cuda:0") * T
        dlogits = b.prsgd_route_grad(logits, experts, counts, 0.1, normalize=True, dweights=up, dloss=ones)
        G = dlogits.mT @ X
        b.prsgd_muon_step(W, V, G, 0.02, mu=0.9)
        x64 = X.double()
        l64 = x64 @ w.mT
        d64 = ref.route_grad(l64, experts, counts, 0.1, True, None, up, ones)
        w, v = ref.muon(w, v, d64.mT @ x64, 0.02, 0.9, True, 0.0, 1.0)
    assert rel(W, w) <= 1e-4                           # three steps of 5e-5 of the step, which is smaller than W
    rows = W.reshape(N, E * D)
    b.prsgd_average_rows(rows, N, E * D)
    assert all(torch.equal(rows[i], rows[0]) for i in range(N)) and rel(rows[0], w.reshape(N, -1).mean(0)) <= 1e-4
