"""Embedding, dropout and vocabulary loss on the GPU against their formulas in 64 bits (tests/language_reference.py).

Tolerances, by element, with half = finfo(type).eps / 2 (one rounding of a result) and u = 2^-24:
 * embedding: one product and one rounding: (half + u) |want|.
 * its gradient: n terms added in fp32, then the scale: (n + 2) u sum|terms| + half |want|; added to what is there: half |sum|, u each.
 * dropout: the scale, the product and the sum round once each: 3 u (|x| / (1 - q) + |residual|) + half |want|.  What is kept is equal.
 * loss: a logit is a sum over D of products, exact for 16-bit types; a tensor core adds 16 at a time and cuts off what the sum does
   not hold: e_z = (D / 16 + 4) 2^-22 sum |h w| bounds it (fp32 operands as pairs: 2^-21 sum |h w| more, and three sums).  Maximum, logarithm
   and exponentials are good to 4 u of the numbers they take; a sum of V terms in parts of at most 2^10 in a row: 2^10 u at worst.
   loss and log sum: 2 max e_z + 2^-14 (relative to the sum, so absolute for its logarithm) + 8 u (|max| + |loss|); the maximum: e_z.
 * its gradient: G = (dloss + dlse) p - dloss onehot is held with one rounding `hold` (16-bit types their own, fp32 pairs 2^-21), p is off by
   2 e_z + 2^-20 relative, and the sums over V or T by (n / 16 + 4) 2^-22 of the sum of magnitudes M: (hold + 2 e_z + 2^-20 + (n / 16 + 4) 2^-22) M +
   half |want|.  fp16 and pairs hold nothing below 2^-38 of the group's (pairs: the token's) largest |dloss| + |dlse|: 2^-38 of it times sum |w| (or |h|).
"""
import math

import pytest
import torch

import language_reference as ref

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U = 2.0 ** -24


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


def randn(seed, *shape, dtype=F32):
    return torch.randn(*shape, generator=gen(seed), device="cuda:0").to(dtype)


def half(dtype):
    return torch.finfo(dtype).eps / 2


def tokens(seed, groups, count, vocab, padded=True):
    """Ids with repeats (rank-frequency), padding of several kinds among them."""
    u = torch.rand(groups, count, generator=gen(seed), device="cuda:0", dtype=torch.float64)
    ids = ((vocab + 1.0) ** u).floor().long().sub_(1).clamp_(0, vocab - 1)
    if padded:
        r = torch.rand(groups, count, generator=gen(seed + 1), device="cuda:0")
        ids[r < 0.1], ids[r < 0.06], ids[r < 0.03] = -1, vocab, -2 ** 31
    return ids.to(torch.int32)


def layout(t, kind):
    """t's values in another place: 'odd' rows and a base off 16 bytes, 'wide' rows that are multiples of 16 bytes, 'turn' the groups' rows in
    turn; (view, everything around it, which holds 7)."""
    G, R, D = t.shape
    v = 16 // t.element_size()
    if kind == "turn":
        big = torch.full((R, G, (D + v - 1) // v * v + v), 7.0, dtype=t.dtype, device=t.device)
        view = big.transpose(0, 1)[:, :, :D]
    elif kind == "wide":
        big = torch.full((G, R + 2, (D + v - 1) // v * v + 2 * v), 7.0, dtype=t.dtype, device=t.device)
        view = big[:, :R, :D]
    elif kind == "odd":
        big = torch.full((G * (R + 1) * (D + 3) + 1,), 7.0, dtype=t.dtype, device=t.device)
        view = big[1:].view(G, R + 1, D + 3)[:, :R, :D]
    else:
        return t.clone(), None
    view.copy_(t)
    return view, big


def untouched(view, big):
    if big is None:
        return True
    view.fill_(7.0)
    return bool((big == 7.0).all())


def check(got, want, tol):
    assert got.shape == want.shape
    far = (got.double() - want).abs() - tol
    assert torch.isfinite(got).all() and (far <= 0).all(), f"{(far > 0).sum().item()} of {far.numel()} off, worst {far.max().item():.3g} beyond"


LAYOUTS = ["dense", "odd", "wide", "turn"]


# ---- embedding ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", LAYOUTS)
@pytest.mark.parametrize("dtype,out", [(F32, F32), (BF16, BF16), (F16, F32), (F32, BF16), (BF16, F16)])
@pytest.mark.parametrize("G,T,V,D", [(1, 1, 1, 1), (3, 37, 50, 40), (2, 300, 1000, 333), (1, 5, 7, 4104)])
def test_embed(b, G, T, V, D, dtype, out, kind):
    table, _ = layout(randn(1, G, V, D, dtype=dtype), kind)
    ids = tokens(2, G, T, V)
    to, around = layout(torch.zeros(G, T, D, dtype=out, device="cuda:0"), kind)
    want = ref.embed(table, ids, 0.3)
    got = b.prsgd_embed(table, ids, scale=0.3, out=to)
    assert got is to
    check(got, want, (half(out) + 2 * U) * want.abs() + (2.0 ** -25 if out == F16 else 0.0))
    assert (got[~ref.live_tokens(ids, V)] == 0).all() and untouched(to, around)


def test_embed_shared_table_and_one_worker(b):
    table, ids = randn(3, 60, 48, dtype=BF16), tokens(4, 3, 20, 60)
    got = b.prsgd_embed(table.expand(3, 60, 48), ids)
    for g in range(3):
        assert torch.equal(got[g], b.prsgd_embed(table, ids[g]))
    assert b.prsgd_embed(table, ids[0, :0]).shape == (0, 48)


def test_embed_padding_reads_nothing(b):
    table = torch.full((1, 8, 24), float("nan"), device="cuda:0")
    table[0, 5] = 1.0
    got = b.prsgd_embed(table, torch.tensor([[5, -1, 8, 5]], dtype=torch.int32, device="cuda:0"), scale=2.0)
    assert got[0, :, 0].tolist() == [2.0, 0.0, 0.0, 2.0]


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("kind", LAYOUTS)
@pytest.mark.parametrize("dtype,out", [(F32, F32), (BF16, F32), (BF16, BF16), (F16, F16), (F32, BF16)])
@pytest.mark.parametrize("G,T,V,D", [(1, 1, 1, 1), (3, 37, 50, 40), (2, 700, 30, 333), (2, 2000, 5000, 96), (1, 70, 40, 4104)])
def test_embed_grad(b, G, T, V, D, dtype, out, kind, accumulate):
    dout, _ = layout(randn(5, G, T, D, dtype=dtype), kind)
    ids = tokens(6, G, T, V)
    before = randn(7, G, V, D, dtype=out) if accumulate else torch.full((G, V, D), float("nan"), dtype=out, device="cuda:0")
    to, around = layout(before, kind)
    sums, mags, many = ref.embed_grad(dout, ids, V, 0.7)
    want = sums + before.double() if accumulate else sums
    work = b.embed_grad_workspace(dout, to).fill_(0xFF)
    got = b.prsgd_embed_grad(dout, ids, to, scale=0.7, accumulate=accumulate, workspace=work)
    b.prsgd_work_status(work)
    check(got, want, (many[..., None] + 4) * U * (mags + (before.double().abs() if accumulate else 0.0)) + half(out) * want.abs() + (2.0 ** -25 if out == F16 else 0.0))
    if accumulate:
        idle = many == 0
        assert torch.equal(got[idle], before[idle])
    again = layout(before, kind)[0]
    assert torch.equal(b.prsgd_embed_grad(dout, ids, again, scale=0.7, accumulate=accumulate), got)
    assert untouched(to, around)


@pytest.mark.parametrize("T", [1, 31, 32, 33, 64, 1000, 5000, 20000])
@pytest.mark.parametrize("pattern", ["same", "none", "all different", "two"])
def test_embed_grad_runs(b, T, pattern):
    """Runs that fill every unit, none at all, runs of one."""
    V, D = 20011, 16
    ids = {"same": torch.full((1, T), 17), "none": torch.full((1, T), -1), "all different": torch.randperm(V, generator=torch.Generator().manual_seed(T))[None, :T],
           "two": (torch.arange(T) % 2)[None] * (V - 1)}[pattern].to(torch.int32).cuda()
    T = ids.shape[1]
    dout = randn(8, 1, T, D)
    got = b.prsgd_embed_grad(dout, ids, torch.full((1, V, D), float("nan"), device="cuda:0"))
    sums, mags, many = ref.embed_grad(dout, ids, V)
    check(got, sums, (many[..., None] + 2) * U * mags)


def test_embed_grad_three_digits(b):
    """A vocabulary whose ids take three digits of the sort."""
    V, D = 1 << 19, 8
    ids, dout = torch.randint(0, V, (2, 900), generator=gen(12), device="cuda:0").to(torch.int32), randn(13, 2, 900, D)
    ids[:, ::3] = ids[:, 1::3]
    sums, mags, many = ref.embed_grad(dout, ids, V)
    check(b.prsgd_embed_grad(dout, ids, torch.full((2, V, D), float("nan"), device="cuda:0")), sums, (many[..., None] + 2) * U * mags)


def test_embed_grad_masked_values_and_no_tokens(b):
    dout = randn(9, 2, 6, 8)
    ids = torch.tensor([[1, -1, 3, 9, 1, 4], [-1, -5, 4, 4, 0, -1]], dtype=torch.int32, device="cuda:0")
    dirty = dout.clone()
    dirty[~ref.live_tokens(ids, 4)] = float("nan")
    full = lambda: torch.full((2, 4, 8), 5.0, device="cuda:0")
    assert torch.equal(b.prsgd_embed_grad(dirty, ids, full()), b.prsgd_embed_grad(dout, ids, full()))
    assert (b.prsgd_embed_grad(dout[:, :0], ids[:, :0].contiguous(), full()) == 0).all()
    assert (b.prsgd_embed_grad(dout[:, :0], ids[:, :0].contiguous(), full(), accumulate=True) == 5).all()


# ---- dropout ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", LAYOUTS)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("with_residual", [False, True])
@pytest.mark.parametrize("G,R,D", [(1, 1, 1), (2, 5, 64), (3, 33, 1001), (1, 2000, 24), (1, 3, 9000)])
def test_dropout(b, G, R, D, with_residual, dtype, kind):
    x, _ = layout(randn(10, G, R, D, dtype=dtype), kind)
    r = layout(randn(11, G, R, D, dtype=dtype), kind)[0] if with_residual else None
    to, around = layout(torch.zeros_like(x), kind)
    p, seed, step = 0.3, 0xFEDCBA9876543210, 2 ** 32 + 11
    want = ref.dropout(x, p, seed, step, 5, r)
    got = b.prsgd_dropout(x, p, seed, step=step, first_group=5, residual=r, out=to)
    keep = torch.from_numpy(ref.dropout_keep(G, R, D, p, seed, step, 5)).cuda()
    mags = torch.where(keep, x.double().abs() / (1 - p), 0.0) + (r.double().abs() if with_residual else 0.0)
    check(got, want, 4 * U * mags + half(dtype) * want.abs() + (2.0 ** -25 if dtype == F16 else 0.0))
    if with_residual:
        assert torch.equal(got[~keep], r[~keep])
    else:
        assert (got[~keep] == 0).all()
    assert untouched(to, around)


def test_dropout_in_place_gradient_and_shards(b):
    x, dy = randn(12, 4, 50, 100, dtype=BF16), randn(13, 4, 50, 100, dtype=BF16)
    y = b.prsgd_dropout(x, 0.25, 77, step=3)
    assert torch.equal(b.prsgd_dropout(x.clone(), 0.25, 77, step=3, out=(z := x.clone())), y) and torch.equal(z, y)
    again = x.clone()
    assert torch.equal(b.prsgd_dropout(again, 0.25, 77, step=3, out=again), y)
    assert torch.equal(b.prsgd_dropout(again, 0.25, 77, step=3, residual=(res := dy.clone()), out=res), b.prsgd_dropout(y, 0.25, 77, step=3, residual=dy))
    for g in range(4):                                   # a shard's workers draw as they do in the whole job
        assert torch.equal(b.prsgd_dropout(x[g:g + 1], 0.25, 77, step=3, first_group=g), y[g:g + 1])
        assert torch.equal(b.prsgd_dropout(x[g], 0.25, 77, step=3, first_group=g), y[g])
    dx = b.prsgd_dropout(dy, 0.25, 77, step=3)           # the gradient keeps what the forward call kept
    assert torch.equal(dx != 0, (y != 0) & (dy != 0)) or ((dx != 0) == ((y != 0) | (x == 0)) & (dy != 0)).all()
    assert torch.equal(b.prsgd_dropout(x, 0.0, 77), x)
    assert torch.equal(y.float(), b.prsgd_dropout(x.float(), 0.25, 77, step=3).to(BF16).float())


def test_dropout_drops_nan(b):
    x = torch.full((1, 4, 64), float("nan"), device="cuda:0")
    keep = torch.from_numpy(ref.dropout_keep(1, 4, 64, 0.5, 1)).cuda()
    y = b.prsgd_dropout(x, 0.5, 1)
    assert (y[~keep] == 0).all() and torch.isnan(y[keep]).all()


def test_dropout_step_counter_in_a_graph(b):
    x, counter = randn(14, 2, 30, 40), torch.zeros(1, dtype=torch.int64, device="cuda:0")
    out = torch.empty_like(x)
    b.prsgd_dropout(x, 0.5, 9, step=100, step_counter=counter, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.prsgd_dropout(x, 0.5, 9, step=100, step_counter=counter, out=out)
        counter += 1
    for n in range(3):
        graph.replay()
        assert torch.equal(out, b.prsgd_dropout(x, 0.5, 9, step=100 + n)), n


# ---- vocabulary loss ----------------------------------------------------------------------------------------
def z_error(H, W, D):
    s = H.double().abs() @ W.double().abs().mT
    return (D / 16 + 4) * 2.0 ** -22 * s * (3 if H.dtype == F32 else 1) + (2.0 ** -21 * s if H.dtype == F32 else 0.0)


def case(seed, G, T, V, D, dtype, kind="dense", padded=True, spread=2.0):
    H, _ = layout(randn(seed, G, T, D, dtype=dtype), kind)
    W, _ = layout((randn(seed + 1, G, V, D) * (spread / math.sqrt(D))).to(dtype), kind)
    return H, W, tokens(seed + 2, G, T, V, padded)


def check_loss(got, H, W, y):
    loss, stats = got
    want, want_stats = ref.vocab_loss(H, W, y)
    on = ref.live_tokens(y, W.shape[1])
    ez = torch.where(on[..., None], z_error(torch.where(on[..., None], H, 0), W, H.shape[-1]), 0.0).amax(-1)
    tol = 2 * ez + (2.0 ** -14 + 8 * U * (want_stats[..., 0].abs() + want.abs())) * on
    check(loss, want, tol)
    check(stats[..., 0], want_stats[..., 0], ez + 2 * U * want_stats[..., 0].abs())
    check(stats[..., 1], want_stats[..., 1], tol)


SHAPES = [(1, 1, 1, 1), (2, 3, 5, 8), (1, 1, 1000, 64), (3, 40, 333, 72), (2, 130, 700, 500), (1, 300, 2500, 96), (1, 257, 257, 257)]


@pytest.mark.parametrize("kind", LAYOUTS)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("G,T,V,D", SHAPES)
def test_vocab_loss(b, G, T, V, D, dtype, kind):
    H, W, y = case(20, G, T, V, D, dtype, kind)
    work = b.vocab_loss_workspace(H, W).fill_(0xFF)
    got = b.prsgd_vocab_loss(H, W, y, workspace=work)
    b.prsgd_work_status(work)
    check_loss(got, H, W, y)
    assert all(torch.equal(p, q) for p, q in zip(got, b.prsgd_vocab_loss(H, W, y)))


def check_grad(got, H, W, y, dloss, dlse, before=None, stats=None):
    dH, dW = got
    (G, T, D), V = H.shape, W.shape[1]
    wH, wW, mH, mW, A = ref.vocab_grad(H, W, y, dloss, dlse)
    on = ref.live_tokens(y, V)
    ez = torch.where(on[..., None], z_error(torch.where(on[..., None], H, 0), W, D), 0.0).amax((1, 2))[:, None, None]
    hold = half(H.dtype) if H.dtype != F32 else 2.0 ** -21
    rel = hold + 2 * ez + 2.0 ** -20
    top = torch.where(on, sum(t.abs().double() for t in (dloss, dlse) if t is not None), 0.0).amax(-1)[:, None, None] if dloss is not None or dlse is not None else torch.zeros(G, 1, 1, device="cuda:0")
    least = top * 2.0 ** -38
    Hz = torch.where(on[..., None], H.double().abs(), 0.0)
    if dH is not None:
        pairs = 2.0 ** -20 * A.amax(-1, keepdim=True) * W.double().abs().sum(1, keepdim=True) * 2.0 ** -12 if H.dtype == F32 else 0.0
        check(dH, wH, (rel + (V / 16 + 4) * 2.0 ** -22) * mH + (least * W.double().abs().sum(1, keepdim=True) + pairs) * on[..., None] + half(dH.dtype) * wH.abs() + (2.0 ** -25 if dH.dtype == F16 else 0.0))
        assert (dH[~on] == 0).all()
    if dW is not None:
        if before is not None:
            wW = wW + before.double()
        pairs = 2.0 ** -32 * top * Hz.sum(1, keepdim=True) if H.dtype == F32 else 0.0
        check(dW, wW, (rel + (T / 16 + 4) * 2.0 ** -22) * mW + least * Hz.sum(1, keepdim=True) + pairs + (half(dW.dtype) + 2 * U) * wW.abs() + (2.0 ** -25 if dW.dtype == F16 else 0.0))


def exact_stats(H, W, y):
    return ref.vocab_loss(H, W, y)[1].float()


@pytest.mark.parametrize("kind", LAYOUTS)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("G,T,V,D", SHAPES)
def test_vocab_loss_grad(b, G, T, V, D, dtype, kind):
    H, W, y = case(30, G, T, V, D, dtype, kind)
    stats, dloss, dlse = exact_stats(H, W, y), randn(33, G, T), randn(34, G, T) * 0.1
    dH, aH = layout(torch.full_like(H, float("nan")), kind)
    dW, aW = layout(torch.full_like(W, float("nan")), kind)
    work = b.vocab_loss_grad_workspace(H, W).fill_(0xFF)
    got = b.prsgd_vocab_loss_grad(H, W, y, stats, dloss=dloss, dlse=dlse, dH=dH, dW=dW, workspace=work)
    b.prsgd_work_status(work)
    check_grad(got, H, W, y, dloss, dlse)
    again = b.prsgd_vocab_loss_grad(H, W, y, stats, dloss=dloss, dlse=dlse)
    assert torch.equal(again[0], dH) and torch.equal(again[1], dW)
    only_H = b.prsgd_vocab_loss_grad(H, W, y, stats, dloss=dloss, dlse=dlse, want_dW=False)
    only_W = b.prsgd_vocab_loss_grad(H, W, y, stats, dloss=dloss, dlse=dlse, want_dH=False)
    assert only_H[1] is None and only_W[0] is None and torch.equal(only_H[0], dH) and torch.equal(only_W[1], dW)
    assert untouched(dH, aH) and untouched(dW, aW)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("G,T,V,D", [(3, 2100, 17000, 40), (2, 9000, 9000, 72), (5, 300, 20000, 24), (40, 64, 1000, 128)])
def test_vocab_loss_pieces(b, G, T, V, D, dtype):
    """Several pieces of the vocabulary and groups whose G takes turns in its places; forty calls, each checked for an expired wait and for
    the same bits."""
    H, W, y = case(35, G, T, V, D, dtype)
    y[0, : T // 2] = -1
    got = b.prsgd_vocab_loss(H, W, y)
    check_loss(got, H, W, y)
    stats, dloss = exact_stats(H, W, y), randn(38, G, T)
    work = b.vocab_loss_grad_workspace(H, W)
    first = b.prsgd_vocab_loss_grad(H, W, y, stats, dloss=dloss, workspace=work)
    for g in range(G):
        one = slice(g, g + 1)
        check_grad((first[0][one], first[1][one]), H[one], W[one], y[one], dloss[one], None)
    dH, dW = torch.empty_like(H), torch.empty_like(W)
    for n in range(40):
        b.prsgd_vocab_loss_grad(H, W, y, stats, dloss=dloss, dH=dH, dW=dW, workspace=work)
        b.prsgd_work_status(work)
        assert torch.equal(dH, first[0]) and torch.equal(dW, first[1]), n


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("G,T,V,D", [(2, 130, 700, 500), (1, 20, 9000, 64)])
def test_vocab_loss_grad_into_fp32(b, G, T, V, D, dtype, accumulate):
    H, W, y = case(40, G, T, V, D, dtype)
    stats, dloss = exact_stats(H, W, y), randn(43, G, T)
    before = randn(44, G, V, D) if accumulate else None
    dW = before.clone() if accumulate else torch.full((G, V, D), float("nan"), device="cuda:0")
    check_grad(b.prsgd_vocab_loss_grad(H, W, y, stats, dloss=dloss, dW=dW, accumulate=accumulate), H, W, y, dloss, None, before)


@pytest.mark.parametrize("kind", LAYOUTS)
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_vocab_loss_grad_added_to_16_bits(b, dtype, kind):
    """One rounding of the sum: half of |before + sum|."""
    G, T, V, D = 2, 130, 300, 100
    H, W, y = case(45, G, T, V, D, dtype)
    stats, dloss, before = exact_stats(H, W, y), randn(48, G, T), randn(49, G, V, D, dtype=dtype)
    dW, around = layout(before, kind)
    check_grad(b.prsgd_vocab_loss_grad(H, W, y, stats, dloss=dloss, dW=dW, accumulate=True), H, W, y, dloss, None, before)
    assert untouched(dW, around)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [64, 65])
@pytest.mark.parametrize("T", [1, 70])
def test_vocab_loss_shared_weights(b, T, D, dtype):
    """All groups' W is one array (group stride 0); each group has its own dW."""
    H, W, y = case(46, 3, T, 400, D, dtype, padded=False)
    W = W[:1].expand(3, 400, D)
    got = b.prsgd_vocab_loss(H, W, y)
    check_loss(got, H, W, y)
    dloss = randn(47, 3, T)
    dW = torch.empty(3, 400, D, dtype=dtype, device="cuda:0")
    check_grad(b.prsgd_vocab_loss_grad(H, W, y, exact_stats(H, W, y), dloss=dloss, dW=dW), H, W, y, dloss, None)
    with pytest.raises(b.PRSGDError, match="overlap"):
        b.prsgd_vocab_loss_grad(H, W, y, got[1], dloss=dloss, dW=torch.empty(1, 400, D, dtype=dtype, device="cuda:0").expand(3, 400, D))


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_vocab_loss_masked_values(b, dtype):
    """What padding tokens hold reaches nothing, whole groups of padding among them."""
    H, W, y = case(50, 3, 70, 300, 48, dtype)
    y[1] = -1
    on = ref.live_tokens(y, 300)
    stats, dloss, dlse = exact_stats(H, W, y), randn(53, 3, 70), randn(54, 3, 70)
    want = b.prsgd_vocab_loss(H, W, y), b.prsgd_vocab_loss_grad(H, W, y, stats, dloss=dloss, dlse=dlse)
    check_grad(want[1], H, W, y, dloss, dlse)
    assert (want[1][1][1] == 0).all()
    for bad in (float("nan"), float("inf"), -torch.finfo(dtype).max):
        h, s, dl, ds = H.clone(), stats.clone(), dloss.clone(), dlse.clone()
        for t in (h, s, dl, ds):
            t[~on] = bad
        got = b.prsgd_vocab_loss(h, W, y), b.prsgd_vocab_loss_grad(h, W, y, s, dloss=dl, dlse=ds)
        for p, q in zip(got, want):
            assert torch.equal(p[0], q[0]) and torch.equal(p[1], q[1])


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("G,T,V,D", [(1, 1, 32000, 1024), (3, 2, 777, 1000), (2, 2, 500, 130), (5, 1, 33, 7), (1, 2, 900, 2048), (1, 2, 70, 2056), (300, 1, 50, 16), (2, 1, 1, 1)])
def test_vocab_loss_grad_few_tokens(b, G, T, V, D, dtype, wide):
    """One or two tokens a group, groups without any label among them; rows of any stride; added to fp32 and to W's type."""
    H, W, y = case(26, G, T, V, D, dtype, "wide" if wide else "dense")
    if G > 1:
        y[1] = -1
        H[1] = float("nan")
    stats, dloss, dlse = exact_stats(torch.where(ref.live_tokens(y, V)[..., None], H, 0), W, y), randn(27, G, T), randn(28, G, T) * 0.1
    Hz = torch.where(ref.live_tokens(y, V)[..., None], H, 0)
    work = b.vocab_loss_grad_workspace(H, W).fill_(0xFF)
    dH, dW = b.prsgd_vocab_loss_grad(H, W, y, stats, dloss=dloss, dlse=dlse, workspace=work)
    b.prsgd_work_status(work)
    check_grad((dH, dW), Hz, W, y, dloss, dlse)
    only = b.prsgd_vocab_loss_grad(H, W, y, stats, dloss=dloss, dlse=dlse, want_dW=False)[0], b.prsgd_vocab_loss_grad(H, W, y, stats, dloss=dloss, dlse=dlse, want_dH=False)[1]
    assert torch.equal(only[0], dH) and torch.equal(only[1], dW)
    for kind in {dtype, F32}:
        before = randn(29, G, V, D, dtype=kind)
        to, around = layout(before, "wide" if wide else "odd")
        check_grad(b.prsgd_vocab_loss_grad(H, W, y, stats, dloss=dloss, dlse=dlse, dW=to, accumulate=True), Hz, W, y, dloss, dlse, before)
        assert untouched(to, around)


@pytest.mark.parametrize("T", [1185, 9473, 11887])
def test_vocab_loss_tokens_that_leave_blocks_without_any(b, T):
    """Lengths whose equal shares of tokens end before the last of the blocks that move them together; the labels end where their memory does."""
    V, D = 50, 16
    room = torch.full((1 << 19,), 2, dtype=torch.int32, device="cuda:0")
    y = room[-T:].view(1, T)
    y.copy_(tokens(23, 1, T, V))
    H, W = randn(21, 1, T, D, dtype=BF16), randn(22, 1, V, D, dtype=BF16)
    got = b.prsgd_vocab_loss(H, W, y)
    check_loss(got, H, W, y)
    dloss = randn(24, 1, T)
    check_grad(b.prsgd_vocab_loss_grad(H, W, y, got[1], dloss=dloss), H, W, y, dloss, None)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("G,T,V,D", [(2, 5, 3001, 72), (1, 8, 500, 333), (40, 7, 100, 48), (1, 8, 20, 6144), (1, 8, 20, 6145), (3, 9, 300, 40), (1, 1, 32000, 1024), (3, 2, 777, 1000), (2, 3, 5000, 130), (5, 4, 33, 7), (1, 5, 900, 64), (1, 4, 40, 9000), (600, 1, 50, 16)])
def test_vocab_loss_few_tokens(b, G, T, V, D, dtype):
    """One to nine tokens a group, groups without any label among them."""
    H, W, y = case(25, G, T, V, D, dtype)
    if G > 1:
        y[1] = -1
        H[1] = float("nan")
    work = b.vocab_loss_workspace(H, W).fill_(0xFF)
    got = b.prsgd_vocab_loss(H, W, y, workspace=work)
    b.prsgd_work_status(work)
    check_loss(got, torch.where(ref.live_tokens(y, V)[..., None], H, 0), W, y)
    wide = torch.zeros(G, V + 3, D + 5, dtype=dtype, device="cuda:0")
    wide[:, :V, :D] = W
    check_loss(b.prsgd_vocab_loss(H, wide[:, :V, :D], y), torch.where(ref.live_tokens(y, V)[..., None], H, 0), W, y)


def test_vocab_loss_nan_stays_in_its_token(b):
    for dtype in (F32, BF16, F16):
        H, W, y = case(60, 2, 50, 300, 64, dtype, padded=False)
        want = b.prsgd_vocab_loss(H, W, y)
        H[0, 7, 3] = float("nan")
        loss, stats = b.prsgd_vocab_loss(H, W, y)
        assert torch.isnan(loss[0, 7]) and torch.isnan(loss).sum() == 1
        keep = torch.ones_like(loss, dtype=torch.bool)
        keep[0, 7] = False
        assert torch.equal(loss[keep], want[0][keep])
        dH, dW = b.prsgd_vocab_loss_grad(H, W, y, stats, dloss=torch.ones_like(loss))
        assert torch.isnan(dH[0, 7]).all() and torch.isnan(dH).sum() == 64 and not torch.isnan(dW[1]).any()


def test_vocab_loss_large_logits(b):
    """Logits of 1e3 to 1e4: the softmax comes from differences to the largest."""
    for dtype in (F32, BF16):
        H, W, y = case(70, 1, 40, 200, 32, dtype, padded=False, spread=1000.0)
        got = b.prsgd_vocab_loss(H, W, y)
        check_loss(got, H, W, y)
        dH, _ = b.prsgd_vocab_loss_grad(H, W, y, got[1], dloss=torch.ones(1, 40, device="cuda:0"))
        assert torch.isfinite(dH).all()


@pytest.mark.parametrize("scale", [1e-30, 1e-6, 1e4, 1e30])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_vocab_loss_grad_of_any_size(b, dtype, scale):
    """dloss of any magnitude: a 16-bit G is held relative to the group's largest.  Results into fp32, whose range holds them."""
    H, W, y = case(80, 2, 60, 200, 40, dtype)
    stats, dloss = exact_stats(H, W, y), randn(83, 2, 60) * scale
    dW = torch.empty(2, 200, 40, device="cuda:0")
    check_grad(b.prsgd_vocab_loss_grad(H, W, y, stats, dloss=dloss, dW=dW, want_dH=False), H, W, y, dloss, None)


@pytest.mark.parametrize("dtype", [F32, F16])
def test_vocab_loss_operands_of_any_size(b, dtype):
    """Pairs of fp16 values are scaled by powers of two: large and small fp32 operands; and a group of zeros."""
    H, W, y = case(90, 3, 30, 100, 64, dtype)
    if dtype == F32:
        H[0] *= 2.0 ** 60
        W[0] *= 2.0 ** -60
        H[1] *= 2.0 ** -70
        W[1] *= 2.0 ** 71
    H[2] = 0
    got = b.prsgd_vocab_loss(H, W, y)
    check_loss(got, H, W, y)
    dloss = randn(93, 3, 30)
    check_grad(b.prsgd_vocab_loss_grad(H, W, y, got[1], dloss=dloss), H, W, y, dloss, None)


@pytest.mark.parametrize("G,T,V,D", [(1, 40, 301, 64), (2, 300, 2500, 100), (1, 70, 400, 1100)])
def test_vocab_loss_rows_of_any_size(b, G, T, V, D):
    """fp32: tokens, their gradients and classes of very different sizes spoil nothing of the others: rows of H from 2^-30 to 2^60, dloss from
    2^-80 to 1, a class that a last column of ones and a weight of -1e9 mask (compared with the classes without it).

    A token's own e_z bounds its logits.  dH: the terms of check_grad with them; what a token's row of G does not hold is 2^-38 |dloss_t|, what W's columns do not is
    2^-38 of their largest.  dW: the same by columns of H times |dloss_t|, whose scale is known to a factor of two: 2^-37."""
    H, W, y = case(100, G, T, V - 1, D, F32)
    size = 2.0 ** (torch.arange(T, device="cuda:0") % 31 - 30.0)
    size[T // 2] = 2.0 ** 60
    H = H * size[:, None]
    H[..., -1] = 1.0
    W = torch.cat([W, torch.zeros(G, 1, D, device="cuda:0")], 1)
    W[:, -1, -1] = -1e9
    rest = W[:, :-1]
    loss, stats = b.prsgd_vocab_loss(H, W, y)
    masked = y == V - 1                       # (a label of that class: a loss of 1e9, or of what the token of 2^60 holds)
    assert (loss[masked] >= 0.99e9).all()
    y = torch.where(masked, -1, y)
    check_loss((torch.where(masked, 0.0, loss), torch.where(masked[..., None], 0.0, stats)), H, rest, y)
    dloss = randn(103, G, T) * 2.0 ** -(torch.arange(T, device="cuda:0") % 81).float()
    stats = exact_stats(H, rest, y)
    dH, dW = b.prsgd_vocab_loss_grad(H, W, y, stats, dloss=dloss)
    wH, wW, mH, mW, A = ref.vocab_grad(H, rest, y, dloss)
    on = ref.live_tokens(y, V)
    Hz, d = H.double().abs() * on[..., None], dloss.double().abs() * on
    ez = z_error(Hz, rest, D).amax(-1, keepdim=True)
    off = lambda n: 2.0 ** -21 + 2 * ez + 2.0 ** -20 + (n / 16 + 4) * 2.0 ** -22          # noqa: E731
    tol = off(V) * mH + 2.0 ** -38 * (d[..., None] * W.double().abs().sum(1, keepdim=True) + A.sum(-1, keepdim=True) * W.double().abs().amax(1, keepdim=True))
    check(dH, wH, tol + half(F32) * wH.abs())
    weight = (A / d.clamp(min=1e-300)[..., None]).sum(1)[..., None]
    tol = (A * off(T)).mT @ Hz + 2.0 ** -38 * (d[..., None] * Hz).sum(1, keepdim=True) + 2.0 ** -37 * weight * (Hz * d[..., None]).amax(1, keepdim=True)
    check(dW[:, :-1], wW, tol + 2 * half(F32) * wW.abs())
    assert (dW[:, -1] == 0).all()
    assert torch.equal(b.prsgd_vocab_loss_grad(H, W, y, stats, dloss=dloss, want_dW=False)[0], dH)
    assert torch.equal(b.prsgd_vocab_loss_grad(H, W, y, stats, dloss=dloss, want_dH=False)[1], dW)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("T", [1, 2, 5, 40, 300])
def test_vocab_loss_classes_of_minus_infinity(b, T, dtype):
    """Classes masked by a last column of ones and weights of -infinity, whole tiles of them: as without them.  (Their weights times a gradient of zero leave
    a NaN in that column of dH, as in the formula.)"""
    V, D, masked = 900, 72, slice(200, 700)
    H, W, y = case(120, 2, T, V, D, dtype, padded=False)
    H[..., -1] = 1.0
    W[:, masked, -1] = float("-inf")
    y = torch.where((y >= 200) & (y < 700), y % 200, y)
    rest, names = torch.cat([W[:, :200], W[:, 700:]], 1), torch.where(y >= 700, y - 500, y)
    loss, stats = b.prsgd_vocab_loss(H, W, y)
    check_loss((loss, stats), H, rest, names)
    dloss = randn(123, 2, T)
    dH, dW = b.prsgd_vocab_loss_grad(H, W, y, exact_stats(H, rest, names), dloss=dloss)
    assert (dW[:, masked] == 0).all()
    wH = ref.vocab_grad(H, rest, names, dloss)[0]
    check_grad((torch.cat([dH[..., :-1], wH[..., -1:].to(dtype)], -1), torch.cat([dW[:, :200], dW[:, 700:]], 1)), H, rest, names, dloss, None)
    y[0, 0] = 300
    assert b.prsgd_vocab_loss(H, W, y)[0][0, 0] == float("inf")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_vocab_loss_views_of_weights(b, dtype):
    """W's groups as overlapping windows of one table, and columns of a table side by side."""
    T, V, D = 70, 300, 64
    H, _, y = case(110, 3, T, V, D, dtype)
    table = randn(113, V + 40, 4 * D).to(dtype) * 0.25
    for W in (table[:, :D].as_strided((3, V, D), (20 * 4 * D, 4 * D, 1)), table.as_strided((3, V, D), (D, 4 * D, 1)), table.as_strided((3, V, D), (8, 4 * D, 1))):
        got = b.prsgd_vocab_loss(H, W, y)
        check_loss(got, H, W, y)
        dloss = randn(114, 3, T)
        check_grad(b.prsgd_vocab_loss_grad(H, W, y, exact_stats(H, W, y), dloss=dloss), H, W, y, dloss, None)


def test_vocab_loss_no_tokens(b):
    H, W = randn(100, 2, 0, 16), randn(101, 2, 30, 16)
    y = torch.zeros(2, 0, dtype=torch.int32, device="cuda:0")
    loss, stats = b.prsgd_vocab_loss(H, W, y)
    assert loss.shape == (2, 0)
    dW = torch.full_like(W, 3.0)
    assert (b.prsgd_vocab_loss_grad(H, W, y, stats, dW=dW, accumulate=True)[1] == 3).all()
    assert (b.prsgd_vocab_loss_grad(H, W, y, stats, dW=dW)[1] == 0).all()


def test_vocab_loss_gradient_by_differences(b):
    """The library's own loss along random directions, fp32: a difference quotient with h = 2^-6 is off by its third-order term, h^2 / 6
    times the third derivative (at most the cube of the largest |dz|, about 2^3), and by the loss's own rounding over h."""
    H, W, y = case(110, 1, 24, 60, 32, F32)
    stats = b.prsgd_vocab_loss(H, W, y)[1]
    dloss = torch.ones(1, 24, device="cuda:0")
    dH, dW = b.prsgd_vocab_loss_grad(H, W, y, stats, dloss=dloss)
    h = 2.0 ** -6
    for i in range(4):
        eH, eW = randn(111 + i, *H.shape) * 0.2, randn(121 + i, *W.shape) * 0.2
        f = lambda s: b.prsgd_vocab_loss(H + s * h * eH, W + s * h * eW, y)[0].double().sum().item()
        quotient, product = (f(1) - f(-1)) / (2 * h), ((dH.double() * eH).sum() + (dW.double() * eW).sum()).item()
        assert abs(quotient - product) < 24 * (h * h / 6 * 8 + 2.0 ** -20 / h)


# ---- streams, graphs, offsets -------------------------------------------------------------------------------
def step_inputs(seed, G=3, T=150, V=900, D=72, dtype=BF16):
    return randn(seed, G, V, D, dtype=dtype), tokens(seed + 1, G, T, V), tokens(seed + 2, G, T, V)


def language_step(b, table, ids, labels, dtable, p=0.2, seed=5, step=1, counter=None, works=None):
    """One step of workers' language models with tied embeddings: loss, and the table's gradient from both ends."""
    G, V, D = table.shape
    T = ids.shape[1]
    w = works or {}
    x = b.prsgd_embed(table, ids, scale=math.sqrt(D))
    h = b.prsgd_dropout(x, p, seed, step=step, step_counter=counter)
    loss, stats = b.prsgd_vocab_loss(h, table, labels, workspace=w.get("loss"))
    dloss = torch.full((G, T), 1.0 / T, device=table.device)
    dh, _ = b.prsgd_vocab_loss_grad(h, table, labels, stats, dloss=dloss, dW=dtable, workspace=w.get("grad"))
    dx = b.prsgd_dropout(dh, p, seed, step=step, step_counter=counter, out=dh)
    b.prsgd_embed_grad(dx, ids, dtable, scale=math.sqrt(D), accumulate=True, workspace=w.get("embed"))
    return loss


def reference_step(table, ids, labels, p=0.2, seed=5, step=1):
    """The same by automatic differentiation in 64 bits."""
    t = table.double().requires_grad_(True)
    G, V, D = table.shape
    keep = torch.from_numpy(ref.dropout_keep(G, ids.shape[1], D, p, seed, step)).to(table.device)
    on = ref.live_tokens(ids, V)
    x = torch.stack([t[g][ids[g].long().clamp(0, V - 1)] for g in range(G)]) * on[..., None] * math.sqrt(D)
    h = x * keep * (65536.0 / (65536.0 - round(p * 65536)))
    z = h @ t.mT
    live = ref.live_tokens(labels, V)
    loss = torch.where(live, torch.logsumexp(z, -1) - z.gather(-1, labels.long().clamp(0, V - 1)[..., None])[..., 0], 0.0)
    return loss.detach(), torch.autograd.grad(loss.sum() / ids.shape[1], t)[0]


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_step_of_language_models(b, dtype):
    """The operators as they are used together.  The loss of bf16 activations, rounded twice (2^-9 rms each relative to their size) beside
    logits that are sums of D of them; gradients are compared in norm: four roundings of their type, each at most `half`."""
    table, ids, labels = step_inputs(200, dtype=dtype)
    table *= 0.3
    dtable = torch.empty(table.shape, device="cuda:0")
    loss = language_step(b, table, ids, labels, dtable)
    want, grad = reference_step(table, ids, labels)
    e = half(dtype)
    on = ref.live_tokens(ids, table.shape[1])
    size = (table.double().abs().amax() ** 2 * math.sqrt(72) * 72).item()
    assert ((loss.double() - want).abs() <= 4 * e * size + 2.0 ** -14).all()
    assert (dtable.double() - grad).norm() <= (6 * max(e, 2.0 ** -20)) * grad.norm() * 3


def test_a_captured_step_replays(b):
    table, ids, labels = step_inputs(210)
    table *= 0.3
    counter = torch.zeros(1, dtype=torch.int64, device="cuda:0")
    dtable, static = torch.empty(table.shape, device="cuda:0"), ids.clone()
    language_step(b, table, static, labels, dtable, counter=counter)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = language_step(b, table, static, labels, dtable, counter=counter)
    for n in range(3):
        static.copy_(tokens(300 + n, *ids.shape, table.shape[1]))
        counter.fill_(n)
        dtable.fill_(float("nan"))
        graph.replay()
        other = torch.empty_like(dtable)
        want = language_step(b, table, static, labels, other, step=1 + n)
        assert torch.equal(loss, want) and torch.equal(dtable, other), n


def test_first_calls_inside_a_capture(b):
    """In a process of its own: no call before the capture."""
    import subprocess
    import sys
    code = """
import sys, torch
sys.path.insert(0, 'tests')
import test_gpu_language as t
from paper_1807_06629_b200 import binding as b
table, ids, labels = t.step_inputs(210)
dtable = torch.empty(table.shape, device='cuda:0')
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    loss = t.language_step(b, table, ids, labels, dtable)
g.replay()
other = torch.empty_like(dtable)
assert torch.equal(loss, t.language_step(b, table, ids, labels, other)) and torch.equal(dtable, other)
print('same')
"""
    out = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and "same" in out.stdout, out.stderr[-2000:]


def test_two_streams_at_once(b):
    jobs = [step_inputs(220 + 10 * i, G=2, T=200 + i, V=700 + 13 * i, D=64 + 8 * i) for i in range(2)]
    want = []
    for table, ids, labels in jobs:
        d = torch.empty(table.shape, device="cuda:0")
        want.append((language_step(b, table, ids, labels, d), d))
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in jobs], []
    for _ in range(5):
        got = []
        for s, (table, ids, labels) in zip(streams, jobs):
            with torch.cuda.stream(s):
                d = torch.empty(table.shape, device="cuda:0")
                got.append((language_step(b, table, ids, labels, d), d))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1])


def test_calls_given_a_stream(b):
    s = torch.cuda.Stream()
    table, ids, labels = step_inputs(240)
    h = randn(241, *ids.shape, table.shape[2], dtype=BF16)
    want = b.prsgd_vocab_loss(h, table, labels), b.prsgd_embed(table, ids), b.prsgd_dropout(h, 0.5, 3)
    torch.cuda.synchronize()
    got = b.prsgd_vocab_loss(h, table, labels, stream=s), b.prsgd_embed(table, ids, stream=s), b.prsgd_dropout(h, 0.5, 3, stream=s)
    s.synchronize()
    assert torch.equal(got[0][0], want[0][0]) and torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])


def test_offsets_beyond_32_bits(b):
    """Tables whose last rows lie beyond 2^32 bytes and 2^31 elements."""
    V, D = (1 << 21) + 77, 1032
    table = torch.zeros(1, V, D, dtype=BF16, device="cuda:0")
    ids = torch.tensor([[0, V - 1, V - 2, 1, V - 1, V]], dtype=torch.int32, device="cuda:0")
    rows = randn(250, 4, D, dtype=BF16)
    for i, v in enumerate((0, 1, V - 2, V - 1)):
        table[0, v] = rows[i]
    assert torch.equal(b.prsgd_embed(table, ids)[0, :5], rows[[0, 3, 2, 1, 3]])
    dout = randn(251, 1, 6, D, dtype=BF16)
    table.zero_()
    b.prsgd_embed_grad(dout, ids, table, accumulate=True)
    assert torch.equal(table[0, V - 1], (dout[0, 1].float() + dout[0, 4].float()).to(BF16)) and torch.equal(table[0, V - 2], dout[0, 2])
    y = b.prsgd_dropout(table, 0.5, 4, out=table)
    keep = torch.tensor([b.prsgd_dropout_keep(4, 0, V - 2, c, 0, 0.5) for c in range(D)], device="cuda:0")
    assert torch.equal(y[0, V - 2], torch.where(keep, dout[0, 2] * 2, 0))
