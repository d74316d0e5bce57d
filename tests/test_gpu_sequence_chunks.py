"""The sequence operators where a workgroup goes round its outer loop: several chunks of
the scan in one segment, several rows or runs of a workgroup's sums, several batches and
passes of the 4-bit product.  Values against the definitions in 64 bits, with the
tolerances of test_gpu_sequence.py (their reasons do not depend on the length: errors of
32 bits that add as a random walk)."""
import pytest
import torch

import sequence_ref as ref
from test_gpu_sequence import BF16, BWD, EPS, F32, FWD, HALF, close, ctx, g, rand, resets, scan_inputs, spoil, tol_of  # noqa: F401

pytestmark = pytest.mark.gpu

# (sequences, steps, heads, channels, groups, states): chunks are 32 steps, and sequences are
# cut into segments where sequences x heads x 64-channel tiles are fewer than 512
WALKS = [(32, 100, 16, 4, 2, 20),   # one segment of 4 chunks
         (64, 70, 8, 6, 1, 16),     # one of 3, state tiles of one wave
         (32, 97, 16, 3, 1, 50),    # one of 4, the last of one step
         (64, 66, 8, 1, 1, 128),    # one of 3, 128 states
         (4, 300, 64, 2, 4, 24),    # 2 segments of 5 chunks
         (4, 2048, 16, 4, 1, 20),   # 8 of 8
         (2, 600, 32, 3, 2, 100),   # 7 of 3, the last of 1
         (1, 400, 32, 66, 1, 40)]   # 7 of 2, two tiles of channels


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T,H,P,G,N", WALKS)
def test_scan_walks_several_chunks(g, ctx, B, T, H, P, G, N, dtype):  # noqa: F811
    i = scan_inputs(B, T, H, P, G, N, dtype)
    i["dt_bias"] -= 2  # memory over several chunks
    reset, state = resets(B, T, "rare"), rand(B, H, P, N, seed=20)
    spoil(ctx)
    y, end = g.scan(ctx, **i, reset=reset, state=state)
    wy, wend = ref.scan(**i, reset=reset, state=state)
    close(y, wy, tol_of(dtype, FWD), "y")
    close(end, wend, FWD, "state")
    dy, ds = rand(B, T, H, P, dtype=dtype, seed=21), rand(B, H, P, N, seed=22)
    want = ref.scan_backward(dy, **i, reset=reset, state=state, dstate=ds)
    spoil(ctx)
    got = g.scan_backward(ctx, dy, **i, reset=reset, state=state, dstate_out=ds)
    again = g.scan_backward(ctx, dy, **i, reset=reset, state=state, dstate_out=ds)
    for k, (name, w) in enumerate(want.items()):
        close(got[k], w, tol_of(dtype, BWD) if k < 4 else BWD, name)
        assert torch.equal(got[k], again[k]), name


def same_finite(got, want, what):
    assert torch.equal(torch.isfinite(got.cpu()), torch.isfinite(want.cpu())), f"{what}: other values are finite"


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("name", ["x", "b", "c", "dt"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T,H,P,G,N", [(32, 150, 16, 3, 2, 20), (4, 300, 64, 2, 4, 24)])
def test_scan_middle_chunk_that_is_not_finite(g, ctx, B, T, H, P, G, N, dtype, name, value):  # noqa: F811
    """Whole chunks before and after it in the same segment, its episode's end two chunks on: finite where the
    definition is, and unmoved where nothing of it reaches."""
    i = scan_inputs(B, T, H, P, G, N, dtype)
    i["dt_bias"] -= 2
    reset = torch.zeros(B, T, dtype=torch.uint8, device="cuda")
    reset[0, 100], reset[1, 70] = 1, 1
    at = 40
    clean = {k: v.clone() for k, v in i.items()}
    i[name][0, at, 0] = value
    clean[name][0, at, 0] = 0.5
    y, end = g.scan(ctx, **i, reset=reset)
    wy, wend = ref.scan(**clean, reset=reset)
    exact = ref.scan(**i, reset=reset)
    same_finite(y, exact[0], "y")
    same_finite(end, exact[1], "state")
    close(y[0, 100:], wy[0, 100:], tol_of(dtype, FWD))
    close(y[1:], wy[1:], tol_of(dtype, FWD))
    close(end, wend, FWD)
    dy = rand(B, T, H, P, dtype=dtype, seed=21)
    got = g.scan_backward(ctx, dy, **i, reset=reset)
    want = ref.scan_backward(dy, **clean, reset=reset)
    exact = ref.scan_backward(dy, **i, reset=reset)
    for k, n in enumerate(("dx", "ddt", "db", "dc")):
        same_finite(got[k], exact[n], n)
        close(got[k][0, 100:], want[n][0, 100:], tol_of(dtype, BWD), n)
        close(got[k][1:], want[n][1:], tol_of(dtype, BWD), n)


# ---- the other operators' loops ----

@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,width", [(9001, 512), (1500, 3001), (700, 5000)])
def test_norm_backward_adds_rows(g, ctx, rows, width, dtype):  # noqa: F811
    """More rows than workgroups take at a time (8 x 512, or 512 of a wide row)."""
    x, w, dy = rand(rows, width, dtype=dtype, seed=1), 1 + rand(width, scale=0.1, seed=3), rand(rows, width, dtype=dtype, seed=4)
    rstd = g.add_rmsnorm(ctx, x, w, None, EPS)[2]
    spoil(ctx)
    dx, dw = g.add_rmsnorm_backward(ctx, dy, x, rstd, w)
    wdx, wdw = ref.norm_backward(dy, x, w, EPS)
    close(dx, wdx, tol_of(dtype, BWD), "dx")
    close(dw, wdw, BWD, "dweight")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T,C,taps", [(260, 33, 70, 4), (600, 5, 36, 3), (2, 40, 1152, 4), (2, 40, 1153, 2)])
def test_conv_backward_adds_runs(g, ctx, B, T, C, taps, dtype):  # noqa: F811
    """More runs than parts of the weights' gradients (512), with waves that are partly past the channels; several
    workgroups a run."""
    x, win = rand(B, T, C, dtype=dtype, seed=1), rand(B, taps - 1, C, dtype=dtype, seed=2)
    w, b, reset = rand(C, taps, scale=0.5, seed=3), rand(C, scale=0.5, seed=4), resets(B, T, "some")
    dy, dwo = rand(B, T, C, dtype=dtype, seed=5), rand(B, taps - 1, C, dtype=dtype, seed=6)
    y, out = g.causal_conv(ctx, x, w, b, reset, win)
    wy, _, wout, _ = ref.conv(x, w, b, reset, win)
    close(y, wy, tol_of(dtype, FWD), "y")
    assert torch.equal(out.cpu().double(), wout)
    spoil(ctx)
    got = g.causal_conv_backward(ctx, dy, x, w, b, reset, win, True, dwo)
    again = g.causal_conv_backward(ctx, dy, x, w, b, reset, win, True, dwo)
    for p, q, r, n in zip(got, ref.conv_backward(dy, x, w, b, reset, win, True, dwo), again, ("dx", "dweight", "dbias", "dwindow")):
        close(p, q, tol_of(dtype, BWD) if n in ("dx", "dwindow") else BWD, n)
        assert torch.equal(p, r), n


@pytest.mark.parametrize("rows,O,K,group", [(1, 8203, 8200, 128), (2, 8203, 8200, 64), (4, 8203, 8200, 64), (1, 50, 20001, 32),
                                            (2, 50, 20001, 128), (3, 33, 40004, 64), (20, 70, 20001, 64)])
def test_qmatvec_batches_and_passes(g, ctx, rows, O, K, group):  # noqa: F811
    """Outputs that a team takes in turns, and inputs that its lanes take in turns."""
    gen = torch.Generator().manual_seed(2)
    codes = torch.randint(0, 256, (O, 16 * -(-K // 32)), generator=gen, dtype=torch.uint8).cuda()
    scales = (0.5 + torch.rand((O, -(-K // group)), generator=gen)).cuda()
    full = ref.weights(codes, scales, K, group)
    for dtype in (F32, BF16):
        x = rand(rows, K, dtype=dtype, seed=3)
        want, size = x.cpu().double() @ full.t(), float((x.cpu().double().abs() @ full.abs().t()).norm())
        off = float((g.qmatvec(ctx, x, codes, scales, group).cpu().double() - want).norm())
        assert off <= FWD * size + (HALF * float(want.norm()) if dtype == BF16 else 0)
    x8 = torch.randint(-127, 128, (rows, K), generator=gen, dtype=torch.int8).cuda()
    xs = rand(rows, seed=5).abs()
    x = x8.cpu().double() * xs.cpu().double()[:, None]
    got = g.qmatvec(ctx, x8, codes, scales, group, x_scale=xs).cpu().double()
    assert float((got - x @ full.t()).norm()) <= FWD * float((x.abs() @ full.abs().t()).norm())
