"""The gated scan's gates far from zero.  Tolerances are those of test_gpu_learning.py
where nothing else is said."""
import pytest
import torch

import learning_ref as ref
from test_gpu_learning import BF16, BWD, F32, FWD, close, ctx, g, gated_inputs, tol_of, uniform  # noqa: F401

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
