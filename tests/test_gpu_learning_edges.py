"""The gated scan's gates far from zero, AdamW's eps at both ends of fp32 and what the
operators that write in place tell autograd.  Tolerances are those of
test_gpu_learning.py where nothing else is said."""
import pytest
import torch

import learning_ref as ref
from test_gpu_learning import BF16, BWD, F32, FWD, check_step, close, ctx, g, gated_inputs, rand, tol_of, uniform  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("T", [7, 70, 600])
def test_gated_scan_gradients_of_saturated_gates(g, ctx, T, sign, dtype):  # noqa: F811
    """Gates of 8 to 20 on one side: what is left of a gate's slope is 3e-4 to 2e-9, and its gradient is right relative to
    that.  The slope is formed from exp(-|gate|), whose argument's rounding makes |gate| 2^-24 of it, 1.2e-6 at most, and
    three operations of 2^-23; the rest is the gradients' 1e-5."""
    args, reset, state, dy, dstate = gated_inputs(2, T, 12, dtype, seed=110)
    for k in (1, 2):
        args[k] = (sign * (8 + 12 * uniform(2, T, 12, seed=110 + k))).to(dtype)
    y, out, marks = g.gated_scan(ctx, *args, reset, state)
    wy, wh, _ = ref.gated(*args, reset, state)
    close(y, wy, tol_of(dtype, FWD), "y")
    close(out, wh, FWD, "state")
    got = g.gated_scan_backward(ctx, dy, *args, marks, reset, dstate)
    want = ref.gated_backward(dy, *args, reset, state, dstate)
    for k, name in ((0, "dx"), (3, "da_log"), (4, "dstate")):
        close(got[k], want[k], tol_of(got[k].dtype, BWD), name)
    for k, name in ((1, "dgate_a"), (2, "dgate_x")):
        slope = torch.sigmoid(-args[k].cpu().double().abs())
        close(got[k].cpu().double() / slope, want[k] / slope, tol_of(dtype, BWD), name)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [1e-45, 1e-40, 1e38, 3e38])
def test_adamw_eps_at_the_ends(g, ctx, bits, eps):  # noqa: F811
    """An eps below and far above the normal numbers, beside v of zero (no gradient at all, and squares that underflow) and not."""
    theta = rand(1024, seed=1, scale=0.05)
    theta[700:] = 0
    grad = rand(1024, seed=2)
    grad[:256], grad[256:512], grad[512:768] = 0, 1e-30, 1e18
    states, clock = g.adamw_state([theta], bits), g.adamw_clock()
    was = theta[:256].clone()
    for _ in range(2):
        check_step(g, ctx, [theta], [grad], states, clock, 0.0, seed=5, eps=eps)
    assert torch.equal(theta[:256], was)


def test_what_is_written_in_place_is_a_change_for_autograd(g, ctx):  # noqa: F811
    """States, clocks and pools count a new version with each call that writes them, as by any operation in place."""
    theta, grad = rand(300, seed=1), rand(300, seed=2)
    for bits in (32, 8):
        states, clock = g.adamw_state([theta], bits), g.adamw_clock()
        written = [theta, clock, *states[0]]
        before = [v._version for v in written]
        g.adamw(ctx, [theta], [grad], states, clock, 0.1)
        assert all(v._version > b for v, b in zip(written, before)) and grad._version == 0
    x, w = rand(2, 8, seed=3), rand(8, 4, seed=4)
    pool = torch.zeros(2, 8, device="cuda", requires_grad=True)
    kept = (pool * pool).sum()
    version = pool._version
    g.gated_scan_step(ctx, x, x, x, rand(8, seed=5), pool)
    assert pool._version > version
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        kept.backward()
    window = torch.zeros(2, 3, 8, device="cuda")
    version = window._version
    g.causal_conv_step(ctx, x, window, w)
    assert window._version > version
    pool = torch.zeros(2, 1, 8, 4, device="cuda")
    version = pool._version
    one = torch.ones(1, device="cuda")
    g.scan_step(ctx, x[:, None], rand(2, 1, seed=6), rand(2, 1, 4, seed=7), rand(2, 1, 4, seed=8), one, one, one, pool)
    assert pool._version > version
    with torch.inference_mode():  # such tensors have no versions
        pool = torch.zeros(2, 8, device="cuda")
        g.gated_scan_step(ctx, x, x, x, rand(8, seed=5), pool)
        assert bool(pool.any())
