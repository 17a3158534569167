"""The context's own use of the training operators: the Muon local step (prsgd_enable_muon) and the balance loss over the
classes (prsgd_set_balance).

The Newton-Schulz step brings every singular value of a momentum buffer to about 1, the smallest included, so a run in
16 bits cannot be compared with one in 64 bits direction by direction.  Each step is therefore checked on what it was given:
the buffers read back after the step, W' = W - gamma scale NS64(v) for the Muon layers (bounds as in
test_gpu_operators.py: 5e-5 or 6e-3 of the step, plus the rounding of W, 2^-23 of it), x' = x - gamma v for the others, and
the buffers themselves against mu v + G of the oracle (1e-5 of their norm on the fp32 path, 2e-2 on the bf16 path, the bounds
of those paths)."""
import numpy as np
import pytest
import torch

import operator_reference as ref
from helpers import make_ctx, make_inputs, rel_l2
from oracle import prsgd_oracle as orc
from paper_1807_06629_b200 import synth

pytestmark = pytest.mark.gpu

F32 = synth.Workload("muon-f32", 3, (40, 70, 150, 10), 16, 0.05, 0, 2, 0, 64, mean_shift=0.5)
BF16 = synth.Workload("muon-bf16", 4, (128, 256, 320, 10), 32, 0.05, 0, 2, 1, 128, mean_shift=0.5)
NS_TOL, G_TOL = {0: 5e-5, 1: 6e-3}, {0: 1e-5, 1: 2e-2}


def segments(dims):
    off, out = 0, []
    for l in range(1, len(dims)):
        out.append((l, slice(off, off + dims[l] * dims[l - 1])))
        off += dims[l] * dims[l - 1]
        out.append((-l, slice(off, off + dims[l])))
        off += dims[l]
    return out


def scale_of(rule, o, i):
    return 0.2 * max(o, i) ** 0.5 if rule == 1 else max(1.0, o / i) ** 0.5


def expected(x, v, dims, gamma, layers, rule, steps=5):
    """One step from x with the new buffers v, per worker, in 64 bits; and the size of each row's Muon part."""
    y = x - gamma * v
    for l, seg in segments(dims):
        if l in layers:
            M = torch.from_numpy(v[:, seg].reshape(len(x), dims[l], dims[l - 1]))
            y[:, seg] = x[:, seg] - gamma * scale_of(rule, dims[l], dims[l - 1]) * ref.orthogonalize(M, steps).numpy().reshape(len(x), -1)
    return y


def check_step(p, w, before, v_before, mu, grads, layers, rule, active=None, averaged=False):
    after, v = p.get_params_stacked().astype(np.float64), p.get_velocity_stacked().astype(np.float64)
    on = [i for i in range(w.N) if active is None or active[i]]
    for i in range(w.N):
        if i not in on:
            assert np.array_equal(v[i], v_before[i])
    want_v = mu * v_before + grads
    assert rel_l2(v[on], want_v[on]) <= G_TOL[w.precision]
    want = expected(before, v, w.dims, w.gamma, layers, rule)
    for i in range(w.N):
        if i not in on:
            want[i] = before[i]
    if averaged:
        want[:] = want.mean(0)
    for l, seg in segments(w.dims):
        step = np.linalg.norm(want[:, seg] - before[:, seg])
        off = np.linalg.norm(after[:, seg] - want[:, seg])
        tol = NS_TOL[w.precision] if l in layers else 1e-5 if w.precision == 0 else 2e-2      # (bias steps are formed from dZ in either precision)
        assert off <= tol * step + 2.0 ** -22 * np.linalg.norm(want[:, seg]), (l, off / max(step, 1e-30))
    return after, v


def gradients(w, X, Y, x, t):
    fn = orc.mlp_grad_fn(w.dims, X.astype(np.float64), Y, w.B, w.seed)
    return np.stack([fn(i, t, x[i]) for i in range(w.N)])


@pytest.mark.parametrize("w", [F32, BF16], ids=lambda w: w.name)
@pytest.mark.parametrize("rule,layers", [(0, None), (1, (1,)), (0, (1, 2, 3))])
def test_muon_local_steps(w, rule, layers):
    X, Y, x0 = make_inputs(w)
    p = make_ctx(w, X, Y, x0)
    p.enable_momentum(0.9)
    p.enable_muon(layers, scale=rule)
    chosen = (1, 2) if layers is None else layers
    x, v = np.tile(x0.astype(np.float64), (w.N, 1)), np.zeros((w.N, x0.size))
    for t in (1, 2, 3):
        g = gradients(w, X, Y, x, t)
        p.local_steps(1)
        x, v = check_step(p, w, x, v, 0.9, g, chosen, rule)
    p.sync()
    p.close()


@pytest.mark.parametrize("w", [F32, BF16], ids=lambda w: w.name)
def test_muon_with_averages_masks_and_row_sums(w):
    X, Y, x0 = make_inputs(w)
    p = make_ctx(w, X, Y, x0, I=2)
    p.enable_momentum(0.9)
    p.enable_muon()
    x, v = np.tile(x0.astype(np.float64), (w.N, 1)), np.zeros((w.N, x0.size))
    for t in (1, 2):
        g = gradients(w, X, Y, x, t)
        p.local_steps(1)
        x, v = check_step(p, w, x, v, 0.9, g, (1, 2), 0, averaged=t == 2)
    assert all(np.array_equal(x[i], x[0]) for i in range(w.N))
    mask = np.array([1, 0] + [1] * (w.N - 2), dtype=np.uint8)      # an inactive worker keeps its point and its buffers
    p.set_interval(0)
    p.set_active(mask)
    g = gradients(w, X, Y, x, 3)
    p.local_steps(1)
    x, v = check_step(p, w, x, v, 0.9, g, (1, 2), 0, active=mask)
    p.set_active(None)
    q = make_ctx(w, X, Y, x0, I=0)                     # row sums instead of the average
    q.enable_momentum(0.9)
    q.enable_muon()
    r = make_ctx(w, X, Y, x0, I=0)
    r.enable_momentum(0.9)
    r.enable_muon()
    q.local_steps_sum(2)
    r.local_steps(2)
    rows = r.get_params_stacked()
    total = rows[0].copy()
    for i in range(1, w.N):
        total = total + rows[i]                        # fp32, in row order
    assert np.array_equal(q.get_params_stacked(), np.tile(total, (w.N, 1)))
    for c in (p, q, r):
        c.close()


@pytest.mark.parametrize("w", [F32, BF16], ids=lambda w: w.name)
def test_muon_replayed_direct_and_tile_major_give_the_same_bits(w):
    X, Y, x0 = make_inputs(w)
    out = []
    for graph, tiled in ((1, 1), (0, 1), (1, 0)):
        p = make_ctx(w, X, Y, x0, I=2)
        p.set_option(4, graph)                         # PRSGD_OPT_GRAPH
        p.set_option(19, tiled)                        # PRSGD_OPT_TILED_WEIGHTS
        p.enable_momentum(0.9)
        p.enable_muon()
        p.local_steps(6)
        out.append((p.get_params_stacked(), p.get_velocity_stacked(), p.get_losses()))
        p.sync()
        p.close()
    for other in out[1:]:
        assert all(np.array_equal(a, b) for a, b in zip(out[0], other))


def test_muon_switches_and_refusals():
    w = F32
    X, Y, x0 = make_inputs(w)
    p = make_ctx(w, X, Y, x0)
    from paper_1807_06629_b200 import binding as b
    lib = b.lib

    def rc(*a):
        return lib.prsgd_enable_muon(p.ctx, *a)

    assert rc(1, 0, 5, 65536, 1 << 30) == -4           # momentum first
    p.enable_momentum(0.9)
    p.enable_muon()
    work = p._muon_work
    assert rc(8, 0, 5, work.data_ptr(), work.numel()) == -1 and rc(1, 2, 5, work.data_ptr(), work.numel()) == -1
    assert rc(1, 0, 0, work.data_ptr(), work.numel()) == -1 and rc(1, 0, 17, work.data_ptr(), work.numel()) == -1
    assert rc(1, 0, 5, None, 0) == -3 and rc(1, 0, 5, work.data_ptr(), 256) == -3 and rc(1, 0, 5, work.data_ptr() + 16, work.numel()) == -2
    with pytest.raises(ValueError):
        p.enable_muon([4])
    # switched off again: the momentum step's bits
    p.enable_muon([])
    p.local_steps(2)
    q = make_ctx(w, X, Y, x0)
    q.enable_momentum(0.9)
    q.local_steps(2)
    assert np.array_equal(p.get_params_stacked(), q.get_params_stacked())
    # a standing device error keeps the parameters
    p.enable_muon()
    before = p.get_params_stacked()
    p.selftest_wait_expiry(1000)
    with pytest.raises(b.PRSGDError):
        p.sync()
    p.local_steps(1)
    with pytest.raises(b.PRSGDError):
        p.sync()
    p.clear_device_error()
    assert np.array_equal(p.get_params_stacked(), before)
    p.close()
    q.close()


# ---- balance loss ----------------------------------------------------------------------------------------------
def balanced_loss(x, dims, Xb, yb, coef, k, doubt=False):
    """(loss, gradient, doubt) of the cross-entropy plus the balance loss, in 64 bits by differentiation.

    `doubt`: how much of the gradient the choice of classes leaves open in bf16.  Weights and activations are rounded to
    2^-9 each, so a layer's z is off by at most 2^-8 |a| |W| plus |W| times what a is off by (the activations carry their
    own rounding, 2^-9 |a|, in that).  A class whose logit lies within twice that of a row's k-th largest may be chosen in
    its place; that moves 1 / (k B) of f from one class to the other, and the gradient, linear in f, by the gradient of
    coef C (P_other - P_kth) / (k B).  Summed over all such classes of all rows, by the triangle inequality."""
    x = torch.tensor(x, dtype=torch.float64, requires_grad=True)
    a, off = torch.from_numpy(np.asarray(Xb, dtype=np.float64)), 0
    da = torch.zeros_like(a)
    for l in range(1, len(dims)):
        W = x[off:off + dims[l] * dims[l - 1]].reshape(dims[l], dims[l - 1])
        off += dims[l] * dims[l - 1]
        z = a @ W.T + x[off:off + dims[l]]
        off += dims[l]
        dz = (2.0 ** -8 * a.abs() @ W.abs().T + da @ W.abs().T).detach()
        a = torch.relu(z)
        da = dz + 2.0 ** -9 * a.detach()
    y = torch.from_numpy(np.asarray(yb)).long()
    _, _, counts, _, loss = ref.route(z.detach()[None], k, coef)
    p = torch.softmax(z, -1)
    bal = coef * dims[-1] * (counts[0].double() / (k * len(y)) * p.mean(0)).sum()
    assert abs(bal.item() - loss[0].item()) < 1e-12
    f = torch.nn.functional.cross_entropy(z, y) + bal
    open_ = 0.0
    if doubt:
        order = torch.sort(z.detach(), dim=-1, descending=True).indices
        mean = p.mean(0)
        for b in range(len(y)):
            for j in range(k):                         # (any of the chosen may be the one that gives way)
                c = order[b, j]
                for o in order[b, k:]:
                    if (z[b, c] - z[b, o]).item() > (dz[b, c] + dz[b, o]).item():
                        break
                    g = torch.autograd.grad(coef * dims[-1] * (mean[o] - mean[c]) / (k * len(y)), x, retain_graph=True)[0]
                    open_ += g.norm().item()
    return f.item(), torch.autograd.grad(f, x)[0].numpy(), open_


@pytest.mark.parametrize("w", [F32, BF16, BF16.with_(dims=(128, 192, 200))], ids=["f32", "bf16", "bf16-200-classes"])
@pytest.mark.parametrize("coef,k", [(0.5, 1), (2.0, 3)])
def test_balance_loss_in_the_local_step(w, coef, k):
    X, Y, x0 = make_inputs(w)
    p = make_ctx(w, X, Y, x0)
    p.set_balance(coef, k)
    p.local_steps(1)
    got, losses, draws = p.get_params_stacked().astype(np.float64), p.get_losses(), p.get_draws()
    want = np.empty_like(got)
    for i in range(w.N):
        rows = slice(draws[i] * w.B, (draws[i] + 1) * w.B)
        loss, g, doubt = balanced_loss(x0, w.dims, X[i, rows], Y[i, rows], coef, k, doubt=w.precision == 1)
        want[i] = x0 - w.gamma * g
        assert losses[i] == pytest.approx(loss, rel=1e-5 if w.precision == 0 else 2e-2)
        tol = 2e-5 if w.precision == 0 else 2e-2
        assert np.linalg.norm(got[i] - want[i]) <= tol * w.gamma * np.linalg.norm(g) + w.gamma * doubt
    p.close()


@pytest.mark.parametrize("w", [F32, BF16], ids=lambda w: w.name)
def test_balance_loss_replayed_and_switched_off(w):
    X, Y, x0 = make_inputs(w)
    out = []
    for graph in (0, 1):
        p = make_ctx(w, X, Y, x0, I=2)
        p.set_option(4, graph)
        p.local_steps(2)
        p.set_balance(0.7, 2)
        p.local_steps(4)
        p.set_balance(0.0, 0)
        p.local_steps(2)
        out.append(p.get_params_stacked())
        p.close()
    assert np.array_equal(out[0], out[1])
    plain, off = make_ctx(w, X, Y, x0, I=2), make_ctx(w, X, Y, x0, I=2)
    off.set_balance(1.0, 1)
    off.set_balance(0.0, 0)
    for c in (plain, off):
        c.local_steps(4)
    assert np.array_equal(plain.get_params_stacked(), off.get_params_stacked())
    lib = __import__("paper_1807_06629_b200.binding", fromlist=["lib"]).lib
    assert lib.prsgd_set_balance(off.ctx, 0.1, -1) == -1 and lib.prsgd_set_balance(off.ctx, 0.1, w.dims[-1] + 1) == -1
    assert lib.prsgd_set_balance(off.ctx, float("nan"), 1) == -1
    plain.close()
    off.close()
