"""The balance loss over the classes in a run one of whose workers has diverged to NaN: every class can be among the chosen ones
(top_k = d_L), its counts stay within the classes, and the other workers' steps keep their bits."""
import numpy as np
import pytest

from helpers import make_ctx, make_inputs
from paper_1807_06629_b200 import synth

pytestmark = pytest.mark.gpu

F32 = synth.Workload("balance-f32", 3, (40, 70, 10), 16, 0.05, 0, 2, 0, 64, mean_shift=0.5)
BF16 = synth.Workload("balance-bf16", 3, (128, 256, 10), 32, 0.05, 0, 2, 1, 128, mean_shift=0.5)


@pytest.mark.parametrize("nan_class", [0, 1, 9])
@pytest.mark.parametrize("k", [1, 3, 10])
@pytest.mark.parametrize("w", [F32, BF16, BF16.with_(dims=(128, 192, 200)), F32.with_(dims=(40, 1))], ids=["f32", "bf16", "200-classes", "one-class"])
def test_a_diverged_worker_leaves_the_others_alone(w, k, nan_class):
    C = w.dims[-1]
    k, nan_class = min(k, C), min(nan_class, C - 1)
    X, Y, x0 = make_inputs(w)
    Y = Y % C
    out = []
    for bad in (False, True):
        x = np.tile(x0, (w.N, 1)).astype(np.float32)
        if bad:
            x[1, x.shape[1] - C + nan_class] = np.nan     # the bias of a class
        p = make_ctx(w, X, Y, x0, I=0)
        p.set_params_stacked(x)
        p.set_balance(0.5, k)
        p.local_steps(2)
        p.sync()
        out.append((p.get_params_stacked(), p.get_losses()))
        p.close()
    (x_ok, f_ok), (x_bad, f_bad) = out
    assert np.isfinite(x_ok).all() and np.isfinite(f_ok).all()
    for i in (0, 2):
        assert np.array_equal(x_ok[i], x_bad[i]) and f_ok[i] == f_bad[i]
    assert np.isnan(f_bad[1])


@pytest.mark.parametrize("w", [F32, BF16], ids=["f32", "bf16"])
def test_every_class_chosen_is_an_even_share(w):
    """top_k = d_L: f_c = 1 / C for every class, so the balance loss is the constant coef and its gradient is nothing but rounding.
    dot = sum_c p_c / C is within C 2^-24 of 1 / C, hence p (f - dot) C coef within C 2^-23 coef of 0 for each logit, over B; against the
    step without the loss, whose weights are sums of B such entries times an activation."""
    X, Y, x0 = make_inputs(w)
    C, coef = w.dims[-1], 0.5
    out = []
    for on in (False, True):
        p = make_ctx(w, X, Y, x0, I=0)
        p.set_option(5, 0)                             # PRSGD_OPT_FUSED_EPILOGUES: the softmax as a launch of its own in both runs
        if on:
            p.set_balance(coef, C)
        p.local_steps(1)
        out.append((p.get_params_stacked().astype(np.float64), p.get_losses()))
        p.close()
    assert np.allclose(out[1][1] - out[0][1], coef, rtol=0, atol=1e-5)
    step = np.linalg.norm(out[0][0] - x0)
    # deltas differ by C 2^-23 coef / B of at most 1 / B: relative to their norm far below 1e-4; on the bf16 path one in a few may round the other way
    assert np.linalg.norm(out[1][0] - out[0][0]) <= (1e-4 if w.precision == 0 else 2.0 ** -8) * step


@pytest.mark.parametrize("balance", [False, True])
@pytest.mark.parametrize("w", [F32, BF16, BF16.with_(dims=(128, 192, 200)), BF16.with_(dims=(64, 10))], ids=["f32", "bf16", "200-classes", "one-layer"])
def test_a_nan_in_the_outputs_reaches_the_weights(w, balance):
    """A diverged worker is seen in its parameters: NaN deltas do not become zeros when they are rounded to bf16, and the step of every
    class's weights and bias is NaN."""
    C = w.dims[-1]
    X, Y, x0 = make_inputs(w)
    x = np.tile(x0, (w.N, 1)).astype(np.float32)
    x[1, x.shape[1] - C] = np.nan
    p = make_ctx(w, X, Y, x0, I=0)
    p.set_params_stacked(x)
    if balance:
        p.set_balance(0.5, 2)
    else:
        p.set_option(5, 0)                             # PRSGD_OPT_FUSED_EPILOGUES
    p.local_steps(1)
    after = p.get_params_stacked()
    p.close()
    assert np.isnan(after[1, -C * (w.dims[-2] + 1):]).all() and np.isfinite(after[[0, 2]]).all()


@pytest.mark.parametrize("k", [1, 3])
@pytest.mark.parametrize("size", [1e3, 1e6, 1e10, -1e30])
@pytest.mark.parametrize("w", [F32.with_(dims=(40, 10)), BF16.with_(dims=(64, 10))], ids=["f32", "bf16"])
def test_large_logits_keep_their_softmax(w, size, k):
    """Equal logits of any size: p = 1 / C, the first k classes are chosen (f = 1 / k), and with weights of 0 the step of W is
    -gamma delta^T X.  p is off by the sum and the division (10 2^-24), delta by as much of (1 + coef C): below 1e-5 of its norm,
    sums over B rows included; deltas are rounded to bf16 on that path (2^-8)."""
    X, Y, x0 = make_inputs(w)
    C, D, coef = w.dims[-1], w.dims[0], 0.5
    x = np.zeros_like(x0)
    x[-C:] = size
    p = make_ctx(w, X, Y, x, I=0)
    p.set_balance(coef, k)
    p.local_steps(1)
    after, losses, draws = p.get_params_stacked().astype(np.float64), p.get_losses(), p.get_draws()
    p.close()
    f = np.where(np.arange(C) < k, 1.0 / k, 0.0)
    for i in range(w.N):
        rows = slice(draws[i] * w.B, (draws[i] + 1) * w.B)
        delta = (1 / C - np.eye(C)[Y[i, rows]] + coef * (f - 1 / C)) / w.B
        want = -w.gamma * delta.T @ X[i, rows].astype(np.float64)
        got = after[i, :C * D].reshape(C, D)
        assert abs(losses[i] - (np.log(C) + coef)) <= 1e-5 * (np.log(C) + coef)
        assert np.linalg.norm(got - want) <= (1e-5 if w.precision == 0 else 2.0 ** -8 + 1e-5) * np.linalg.norm(want)
