"""The sequence operators on the GPU against their definitions in 64 bits
(sequence_ref.py), at the sizes, strides, resets and values where they can go wrong.

Tolerances.  fp32 results are sums of at most a few hundred rounded products (each
2^-24 relative, adding as a random walk) on both sides of one or two exponentials
(2 units of the last place): 2e-6 relative L2 forward; a gradient passes three such
stages and the sums over a chunk's steps: 1e-5.  bf16 results are those rounded once,
to 8 bits: at most 2^-8 relative L2.  Codes are whole numbers and equal.
"""
import math

import pytest
import torch

import sequence_ref as ref

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
FWD, BWD, HALF = 2e-6, 1e-5, 2.0 ** -8
EPS = 1e-6


@pytest.fixture(scope="module")
def g():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a ROCm device")
    import paper_1507_04296_amd as gmod
    gmod.lib()
    return gmod


@pytest.fixture(scope="module")
def ctx(g):
    c = g.Context(1, 1, min_bytes=1 << 30)
    yield c
    c.check()
    c.close()


def spoil(ctx):
    """What a call has not written itself is NaN."""
    ctx.workspace[8192:].fill_(255)


def rand(*shape, dtype=F32, scale=1.0, seed=0):
    gen = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(shape, generator=gen)).to(dtype).cuda()


def close(got, want, tol, what=""):
    got, want = got.detach().cpu().double(), want.cpu().double()
    assert got.shape == want.shape, what
    fine = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), fine), f"{what}: other values are finite"
    size = float(want[fine].norm())
    off = float((got[fine] - want[fine]).norm())
    assert off <= tol * size + 1e-30, f"{what}: {off / max(size, 1e-300):.2e} over {tol:.1e}"


def tol_of(dtype, exact):
    return exact if dtype == F32 else HALF


def strided(t, lead, extra=3, off=0):
    """The same values as a view into wider rows, `off` elements past their start."""
    inner = math.prod(t.shape[lead:])
    wide = torch.full((*t.shape[:lead], inner + extra + off), 7.0, dtype=t.dtype, device=t.device)
    wide[..., off:off + inner] = t.reshape(*t.shape[:lead], inner)
    return wide[..., off:off + inner].unflatten(-1, t.shape[lead:])


# ---- norm ----

@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,width", [(1, 1), (3, 5), (5, 64), (1, 512), (257, 512), (7, 1000), (2, 2047), (3, 3136),
                                        (2, 8190), (2, 16384), (1, 40003), (2500, 36)])
def test_norm(g, ctx, rows, width, dtype):
    x, r = rand(rows, width, dtype=dtype, seed=1), rand(rows, width, dtype=dtype, scale=2.0, seed=2)
    w, dy, dt = 1 + rand(width, scale=0.1, seed=3), rand(rows, width, dtype=dtype, seed=4), rand(rows, width, dtype=dtype, seed=5)
    y, total, rstd = g.add_rmsnorm(ctx, x, w, r, EPS)
    assert torch.equal(total, (x.float() + r.float()).to(dtype))
    want, rho = ref.norm(total, w, EPS)
    close(y, want, tol_of(dtype, FWD), "y")
    close(rstd, rho, FWD, "rstd")
    spoil(ctx)
    dx, dw = g.add_rmsnorm_backward(ctx, dy, total, rstd, w, dt)
    wdx, wdw = ref.norm_backward(dy, total, w, EPS, dt)
    close(dx, wdx, tol_of(dtype, BWD), "dx")
    # terms of dy * total * rho cancel: their size bounds the error
    size = float((dy.double().cpu() * total.double().cpu() * rho[:, None]).norm())
    assert float((dw.cpu().double() - wdw).norm()) <= BWD * size
    again, dw2 = g.add_rmsnorm_backward(ctx, dy, total, rstd, w, dt)
    assert torch.equal(dx, again) and torch.equal(dw, dw2)
    y2, t2, _ = g.add_rmsnorm(ctx, x, w)
    assert t2 is x
    close(y2, ref.norm(x, w, EPS)[0], tol_of(dtype, FWD), "no residual")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,width", [(1, 3), (5, 512), (33, 1000), (2, 9001)])
def test_norm_codes(g, ctx, rows, width, dtype):
    x, r, w = rand(rows, width, dtype=dtype, seed=1), rand(rows, width, dtype=dtype, seed=2), 1 + rand(width, scale=0.1, seed=3)
    codes, scale, total = g.add_rmsnorm_codes(ctx, x, w, r, EPS)
    u = total.float() * w
    m = u.abs().amax(1, keepdim=True)
    assert torch.equal(codes.float(), torch.round(u * (torch.full_like(m, 127) / m)))
    want, rho = ref.norm(total, w, EPS)
    close(scale, rho * m[:, 0].cpu().double() / 127, FWD, "scale")
    # half a step of the codes, and the roundings of both factors
    assert ((codes.cpu().double() * scale.cpu().double()[:, None] - want).abs() <= 0.501 * scale.cpu().double()[:, None] + 1e-5 * want.abs()).all()


def test_norm_odd_rows(g, ctx):
    """Strides, alignment of one element, rows of zeros, rows that are not finite."""
    for dtype in (F32, BF16):
        x, r = rand(9, 130, dtype=dtype, seed=1), rand(9, 130, dtype=dtype, seed=2)
        w = 1 + rand(130, scale=0.1, seed=3)
        want = g.add_rmsnorm(ctx, x, w, r, EPS)
        got = g.add_rmsnorm(ctx, strided(x, 1, 5, 1), w, strided(r, 1, 2, 3), EPS)
        close(got[0], want[0], tol_of(dtype, FWD))
        assert torch.equal(got[1], want[1])
        dy = rand(9, 130, dtype=dtype, seed=4)
        one = dy[:1].expand(9, 130)  # a broadcast gradient: stride 0
        close(g.add_rmsnorm_backward(ctx, one, want[1], want[2], w)[0],
              ref.norm_backward(one, want[1], w, EPS)[0], tol_of(dtype, BWD))
        x[2], x[3, 7], x[4, 0], r[2] = 0, float("inf"), float("nan"), 0
        y, total, rstd = g.add_rmsnorm(ctx, x, w, r, EPS)
        assert float(y[2].abs().max()) == 0
        rest = [0, 1, 5, 6, 7, 8]
        close(y[rest], ref.norm(total[rest], w, EPS)[0], tol_of(dtype, FWD))
        codes, scale, _ = g.add_rmsnorm_codes(ctx, x, w, r, EPS)
        assert int(codes[2:5].abs().max()) == 0 and float(scale[2]) == 0 and bool(scale[3:5].isnan().all())
        assert bool(torch.isfinite(scale[rest]).all()) and int(codes[rest].abs().amax(1).min()) == 127
    y, total, rstd = g.add_rmsnorm(ctx, x[:0], w, r[:0])
    dx, dw = g.add_rmsnorm_backward(ctx, y, total, rstd, w)
    assert dx.shape == (0, 130) and float(dw.abs().max()) == 0


# ---- short causal convolution ----

def resets(B, T, kind, seed=7):
    if kind == "none":
        return None
    r = torch.zeros(B, T, dtype=torch.uint8)
    if kind == "all":
        r[:] = 1
    elif kind == "first" and T:
        r[:, 0] = 1
    elif kind == "some":
        r[:] = torch.rand(B, T, generator=torch.Generator().manual_seed(seed)) < 0.15
    elif kind == "rare":
        r[:] = torch.rand(B, T, generator=torch.Generator().manual_seed(seed)) < 0.02
    return r.cuda()


@pytest.mark.parametrize("kind", ["none", "some", "all", "first"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T,C,taps", [(1, 1, 1, 4), (2, 2, 6, 4), (3, 17, 36, 4), (2, 33, 7, 3), (1, 50, 130, 2), (2, 0, 5, 4), (5, 3, 8, 2)])
def test_conv(g, ctx, B, T, C, taps, dtype, kind):
    x, win = rand(B, T, C, dtype=dtype, seed=1), rand(B, taps - 1, C, dtype=dtype, seed=2)
    w, b, reset = rand(C, taps, scale=0.5, seed=3), rand(C, scale=0.5, seed=4), resets(B, T, kind)
    dy, dwo = rand(B, T, C, dtype=dtype, seed=5), rand(B, taps - 1, C, dtype=dtype, seed=6)
    for bias, window, silu in ((b, win, True), (None, None, False)):
        y, out = g.causal_conv(ctx, x, w, bias, reset, window, silu)
        wy, _, wout, _ = ref.conv(x, w, bias, reset, window, silu)
        close(y, wy, tol_of(dtype, FWD), "y")
        assert torch.equal(out.cpu().double(), wout)
        spoil(ctx)
        dx, dw, db, dwin = g.causal_conv_backward(ctx, dy, x, w, bias, reset, window, silu, dwo if window is not None else None)
        rx, rw, rb, rwin = ref.conv_backward(dy, x, w, bias, reset, window, silu, dwo if window is not None else None)
        close(dx, rx, tol_of(dtype, BWD), "dx")
        close(dw, rw, BWD, "dweight")
        if bias is not None:
            close(db, rb, BWD, "dbias")
            close(dwin, rwin, tol_of(dtype, BWD), "dwindow")
        else:
            assert db is None and dwin is None


def test_conv_strides_and_values(g, ctx):
    """Views into wider rows, and values before an episode start that are not finite."""
    for dtype in (F32, BF16):
        B, T, C, K = 3, 40, 24, 4
        x, w, b, win = rand(B, T, C, dtype=dtype, seed=1), rand(C, K, seed=2), rand(C, seed=3), rand(B, K - 1, C, dtype=dtype, seed=4)
        dy, reset = rand(B, T, C, dtype=dtype, seed=5), resets(B, T, "none") or torch.zeros(B, T, dtype=torch.uint8, device="cuda")
        reset[0, 18], reset[1, 0] = 1, 1
        want, dwant = g.causal_conv(ctx, x, w, b, reset, win), g.causal_conv_backward(ctx, dy, x, w, b, reset, win)
        for off in (0, 1):
            xs, dys = strided(x, 2, 4 - off, off), strided(dy, 2, 8 - off, off)
            for p, q in zip(want, g.causal_conv(ctx, xs, w, b, reset, win)):
                close(q, p, tol_of(dtype, FWD))
            for p, q in zip(dwant, g.causal_conv_backward(ctx, dys, xs, w, b, reset, win)):
                close(q, p, tol_of(dtype, FWD))
        turned = x.transpose(0, 1).contiguous().transpose(0, 1)  # steps first in memory
        assert torch.equal(g.causal_conv(ctx, turned, w, b, reset, win)[0], want[0])
        x[0, 17], x[0, 12] = float("nan"), float("inf")
        win[1] = float("nan")
        y, out = g.causal_conv(ctx, x, w, b, reset, win)
        for rows in (y[0, 18:], y[0, :12], y[1], y[2], out):
            assert bool(torch.isfinite(rows).all())
        dx = g.causal_conv_backward(ctx, dy, x, w, b, reset, win)[0]
        assert bool(torch.isfinite(dx[0, 18:]).all()) and bool(torch.isfinite(dx[1:]).all())
        assert torch.equal(dx[0, 18:], dwant[0][0, 18:])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,C,taps", [(1, 1, 4), (1, 1152, 4), (33, 130, 3), (5, 7, 2)])
def test_conv_step(g, ctx, n, C, taps, dtype):
    x, pool, w, b = rand(n, C, dtype=dtype, seed=1), rand(n + 2, taps - 1, C, dtype=dtype, seed=2), rand(C, taps, seed=3), rand(C, seed=4)
    reset = (torch.arange(n) % 3 == 1).to(torch.uint8).cuda()
    slot = torch.randperm(n + 2, generator=torch.Generator().manual_seed(1))[:n].to(torch.int32).cuda()
    for sl, xx in ((slot, x), (None, strided(x, 1, 3, 1))):
        now = pool.clone()
        y = g.causal_conv_step(ctx, xx, now, w, b, sl, reset)
        at = torch.arange(n) if sl is None else sl.cpu().long()
        wy, _, wout, _ = ref.conv(x[:, None], w, b, reset[:, None], pool.cpu()[at])
        close(y, wy[:, 0], tol_of(dtype, FWD))
        expect = pool.cpu().double()
        expect[at] = wout
        assert torch.equal(now.cpu().double(), expect)


# ---- selective scan ----

def scan_inputs(B, T, H, P, G, N, dtype, seed=0):
    return dict(x=rand(B, T, H, P, dtype=dtype, seed=seed + 1), dt=rand(B, T, H, dtype=dtype, seed=seed + 2),
                b=rand(B, T, G, N, dtype=dtype, scale=0.7, seed=seed + 3), c=rand(B, T, G, N, dtype=dtype, scale=0.7, seed=seed + 4),
                a_log=rand(H, scale=0.7, seed=seed + 5) + 0.5, dt_bias=rand(H, seed=seed + 6) - 2, skip=rand(H, seed=seed + 7))


SCAN = [(1, 1, 1, 1, 1, 1), (2, 3, 2, 5, 1, 7), (1, 31, 2, 16, 2, 16), (2, 32, 1, 64, 1, 64), (1, 33, 4, 40, 2, 24), (2, 65, 2, 64, 1, 100),
        (1, 100, 2, 128, 1, 128), (3, 70, 6, 96, 3, 32), (1, 200, 1, 30, 1, 33), (2, 0, 2, 8, 1, 8)]


@pytest.mark.parametrize("kind", ["none", "some", "all"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T,H,P,G,N", SCAN)
def test_scan(g, ctx, B, T, H, P, G, N, dtype, kind):
    i = scan_inputs(B, T, H, P, G, N, dtype)
    reset, state = resets(B, T, kind), rand(B, H, P, N, seed=20)
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


@pytest.mark.parametrize("B,T,H,P,G,N", [(1, 1000, 2, 64, 1, 64), (2, 777, 3, 20, 1, 128)])
def test_scan_long(g, ctx, B, T, H, P, G, N):
    """Sequences cut into segments, without and with carried gradients, and zeros for an absent state."""
    i = scan_inputs(B, T, H, P, G, N, F32)
    i["dt_bias"] -= 3  # memory over hundreds of steps
    for kind in ("none", "rare"):
        reset = resets(B, T, kind)
        y, end = g.scan(ctx, **i, reset=reset)
        wy, wend = ref.scan(**i, reset=reset)
        close(y, wy, FWD, "y")
        close(end, wend, FWD, "state")
        dy = rand(B, T, H, P, seed=21)
        got = g.scan_backward(ctx, dy, **i, reset=reset)
        want = ref.scan_backward(dy, **i, reset=reset)
        assert got[7] is None
        for k, (name, w) in enumerate(want.items()):
            if k < 7:
                close(got[k], w, BWD, name)


def test_scan_in_parts_is_the_whole(g, ctx):
    """A sequence in two calls with the state carried, forward and backward."""
    B, T, H, P, G, N, cut = 2, 90, 2, 64, 1, 32, 41
    i = scan_inputs(B, T, H, P, G, N, F32)
    seq, par = ("x", "dt", "b", "c"), {k: i[k] for k in ("a_log", "dt_bias", "skip")}
    reset, dy = resets(B, T, "rare"), rand(B, T, H, P, seed=21)
    y, end = g.scan(ctx, **i, reset=reset)
    first = {k: i[k][:, :cut] for k in seq}
    last = {k: i[k][:, cut:] for k in seq}
    r1, r2 = reset[:, :cut].contiguous(), reset[:, cut:].contiguous()
    y1, mid = g.scan(ctx, **first, **par, reset=r1)
    y2, end2 = g.scan(ctx, **last, **par, reset=r2, state=mid)
    close(torch.cat([y1, y2], 1), y, FWD)
    close(end2, end, FWD)
    whole = g.scan_backward(ctx, dy, **i, reset=reset)
    b2 = g.scan_backward(ctx, dy[:, cut:], **last, **par, reset=r2, state=mid)
    b1 = g.scan_backward(ctx, dy[:, :cut], **first, **par, reset=r1, dstate_out=b2[7])
    for k in range(4):
        close(torch.cat([b1[k], b2[k]], 1), whole[k], BWD)
    for k in range(4, 7):
        close(b1[k] + b2[k], whole[k], BWD)


def test_scan_strides(g, ctx):
    """x, b and c as slices of one projection's rows, dt of another, steps before sequences in memory."""
    B, T, H, P, G, N = 2, 45, 2, 32, 1, 16
    for dtype in (F32, BF16):
        for extra in (0, 1):
            rows = rand(T, B, H * P + 2 * G * N + extra, dtype=dtype, seed=1).transpose(0, 1)
            dt = rand(B, T, H + 3, dtype=dtype, seed=2)[..., 1:1 + H]
            x, b, c = (rows[..., o:o + n] for o, n in ((0, H * P), (H * P, N), (H * P + N, N)))
            x, b, c = x.unflatten(-1, (H, P)), b.unflatten(-1, (G, N)), c.unflatten(-1, (G, N))
            par = {k: v for k, v in scan_inputs(1, 1, H, P, G, N, F32).items() if k in ("a_log", "dt_bias", "skip")}
            dy = rand(1, 1, H, P, dtype=dtype, seed=3).expand(B, T, H, P)
            whole = [t.contiguous() for t in (x, dt, b, c)]
            for p, q in zip(g.scan(ctx, x, dt, b, c, **par), g.scan(ctx, *whole, **par)):
                close(p, q, FWD if dtype == F32 else 1e-3)
            got = g.scan_backward(ctx, dy, x, dt, b, c, **par)
            want = g.scan_backward(ctx, dy.contiguous(), *whole, **par)
            for p, q in zip(got[:7], want[:7]):
                close(p, q, BWD if dtype == F32 else 1e-3)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("name", ["x", "b", "c", "dt"])
def test_scan_values_that_are_not_finite(g, ctx, name, value):
    """They reach later steps of their episode and nothing else: not the steps before, not the next episode, not
    another sequence, forward and backward."""
    B, T, H, P, G, N = 2, 75, 2, 24, 2, 20
    i = scan_inputs(B, T, H, P, G, N, F32)
    reset = torch.zeros(B, T, dtype=torch.uint8, device="cuda")
    reset[0, 50], reset[0, 3] = 1, 1
    at = 40  # the chunk of the next episode's start
    i[name][0, at, 0] = value
    clean = {k: v.clone() for k, v in i.items()}
    clean[name][0, at, 0] = 0.5
    y, end = g.scan(ctx, **i, reset=reset)
    wy, wend = ref.scan(**clean, reset=reset)
    close(y[0, :at], wy[0, :at], FWD)
    close(y[0, 50:], wy[0, 50:], FWD)
    close(y[1], wy[1], FWD)
    close(end, wend, FWD)
    close(y[0, :, 1], wy[0, :, 1], FWD)  # the other head (and group)
    exact = ref.scan(**i, reset=reset)[0]
    assert torch.equal(torch.isfinite(y).cpu(), torch.isfinite(exact))
    dy = rand(B, T, H, P, seed=21)
    got = g.scan_backward(ctx, dy, **i, reset=reset)
    want = ref.scan_backward(dy, **clean, reset=reset)
    for k, n in enumerate(("dx", "ddt", "db", "dc")):
        close(got[k][0, 50:], want[n][0, 50:], BWD, n)
        close(got[k][1], want[n][1], BWD, n)
    # and a gradient that is not finite stays out of the episode before
    dy[0, 52] = value
    got = g.scan_backward(ctx, dy, **clean, reset=reset)
    want = ref.scan_backward(torch.where(torch.isfinite(dy), dy, torch.zeros_like(dy)), **clean, reset=reset)
    for k, n in enumerate(("dx", "ddt", "db", "dc")):
        close(got[k][0, :50], want[n][0, :50], BWD, n)
        close(got[k][1], want[n][1], BWD, n)


def test_scan_extreme_step_sizes(g, ctx):
    """Steps that keep everything, and steps that forget everything."""
    B, T, H, P, G, N = 1, 80, 2, 16, 1, 16
    i = scan_inputs(B, T, H, P, G, N, F32)
    i["dt"][0, ::7] = 60.0
    i["dt"][0, 1::7] = -80.0
    i["a_log"][1] = 6.0
    y, end = g.scan(ctx, **i)
    wy, wend = ref.scan(**i)
    close(y, wy, FWD)
    close(end, wend, FWD)
    dy = rand(B, T, H, P, seed=21)
    got, want = g.scan_backward(ctx, dy, **i), ref.scan_backward(dy, **i)
    for k, n in enumerate(("dx", "ddt", "db", "dc", "da_log", "ddt_bias", "dskip")):
        close(got[k], want[n], BWD, n)


def test_scan_gradient_against_differences(g, ctx):
    """The library's gradient along random directions against differences of its own forward pass.  The sum that is
    differenced is about 1e3 in size with an error of 1e-6 of it on each side, over steps of 1e-2: 0.1; the
    difference's own error is of second order, h^2 times third derivatives of the gradient's size: 1e-3 of it."""
    B, T, H, P, G, N = 2, 70, 2, 16, 1, 16
    i = scan_inputs(B, T, H, P, G, N, F32)
    reset, state = resets(B, T, "rare"), rand(B, H, P, N, seed=20)
    dy = rand(B, T, H, P, seed=21)
    got = dict(zip((*i, "state"), g.scan_backward(ctx, dy, **i, reset=reset, state=state)))
    for k in got:
        direction = rand(*got[k].shape, seed=30)
        vals = []
        for s in (1e-2, -1e-2):
            moved = dict(i, state=state)
            moved[k] = moved[k] + s * direction
            vals.append(float((g.scan(ctx, **moved, reset=reset)[0].double() * dy.double()).sum()))
        want = float((got[k].double() * direction.double()).sum())
        size = float(got[k].double().norm() * direction.double().norm())
        assert abs((vals[0] - vals[1]) / 2e-2 - want) <= 0.1 + 1e-3 * size, k


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,H,P,G,N", [(1, 16, 64, 1, 64), (3, 2, 5, 1, 7), (70, 4, 40, 2, 24), (2, 1, 128, 1, 128), (5, 3, 1, 3, 1)])
def test_scan_step(g, ctx, n, H, P, G, N, dtype):
    i = scan_inputs(n, 1, H, P, G, N, dtype)
    pool, reset = rand(n + 2, H, P, N, seed=20), (torch.arange(n) % 3 == 1).to(torch.uint8).cuda()
    slot = torch.randperm(n + 2, generator=torch.Generator().manual_seed(1))[:n].to(torch.int32).cuda()
    one = {k: v[:, 0] if v.dim() > 2 else v for k, v in i.items()}
    for sl in (slot, None):
        now = pool.clone()
        y = g.scan_step(ctx, **one, state_pool=now, slot=sl, reset=reset)
        at = torch.arange(n) if sl is None else sl.cpu().long()
        wy, wend = ref.scan(**i, reset=reset[:, None], state=pool.cpu()[at])
        close(y, wy[:, 0], tol_of(dtype, FWD))
        expect = pool.cpu().double()
        expect[at] = wend
        close(now, expect, FWD)


def test_steps_are_the_sequence(g, ctx):
    """Prompt, then single steps: the same as one longer sequence; a reset empties states that are not finite."""
    B, T, H, P, G, N, C, K = 3, 40, 2, 32, 1, 16, 96, 4
    i = scan_inputs(B, T, H, P, G, N, F32)
    reset = resets(B, T, "some")
    y, end = g.scan(ctx, **i, reset=reset)
    par = {k: i[k] for k in ("a_log", "dt_bias", "skip")}
    half = {k: i[k][:, :20] for k in ("x", "dt", "b", "c")}
    _, pool = g.scan(ctx, **half, **par, reset=reset[:, :20].contiguous())
    xc, w, bias = rand(B, T, C, seed=40), rand(C, K, seed=41), rand(C, seed=42)
    yc, wend = g.causal_conv(ctx, xc, w, bias, reset)
    _, wpool = g.causal_conv(ctx, xc[:, :20], w, bias, reset[:, :20].contiguous())
    for t in range(20, T):
        r = reset[:, t].contiguous()
        one = {k: i[k][:, t] for k in ("x", "dt", "b", "c")}
        close(g.scan_step(ctx, **one, **par, state_pool=pool, reset=r), y[:, t], FWD)
        close(g.causal_conv_step(ctx, xc[:, t], wpool, w, bias, reset=r), yc[:, t], FWD)
    close(pool, end, FWD)
    assert torch.equal(wpool, wend)
    pool[1], wpool[1] = float("nan"), float("inf")
    r = torch.tensor([0, 1, 0], dtype=torch.uint8, device="cuda")
    one = {k: i[k][:, 0] for k in ("x", "dt", "b", "c")}
    assert bool(torch.isfinite(g.scan_step(ctx, **one, **par, state_pool=pool, reset=r)).all()) and bool(torch.isfinite(pool).all())
    assert bool(torch.isfinite(g.causal_conv_step(ctx, xc[:, 0], wpool, w, bias, reset=r)).all()) and bool(torch.isfinite(wpool).all())


def test_slots_out_of_range(g, ctx):
    """Seen on the device: nothing is written, the row counts as a new episode, the error is sticky."""
    i = {k: v[:, 0] if v.dim() > 2 else v for k, v in scan_inputs(4, 1, 2, 8, 1, 8, F32).items()}
    pool, win, xc, w = rand(4, 2, 8, 8, seed=20), rand(4, 3, 12, seed=21), rand(4, 12, seed=22), rand(12, 4, seed=23)
    for bad in (4, -1, 2 ** 31 - 1, -2 ** 31):
        slot = torch.tensor([0, bad, 2, 1], dtype=torch.int32, device="cuda")
        now, nwin = pool.clone(), win.clone()
        y = g.scan_step(ctx, **i, state_pool=now, slot=slot)
        with pytest.raises(g.GorilaError) as e:
            ctx.check()
        assert e.value.code == -2
        yc = g.causal_conv_step(ctx, xc, nwin, w, None, slot)
        with pytest.raises(g.GorilaError) as e:
            ctx.check()
        assert e.value.code == -2
        ctx.check()
        assert torch.equal(now[3], pool[3]) and torch.equal(nwin[3], win[3])
        fresh = g.scan_step(ctx, **i, state_pool=pool.clone(), reset=torch.ones(4, dtype=torch.uint8, device="cuda"))
        assert torch.equal(y[1], fresh[1])
        assert torch.equal(yc[1], g.causal_conv_step(ctx, xc, win.clone(), w, reset=torch.ones(4, dtype=torch.uint8, device="cuda"))[1])


# ---- 4-bit weights ----

@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,O,K", [(1, 1, 1), (1, 17, 40), (2, 64, 512), (3, 130, 1001), (1, 512, 3136), (16, 33, 96), (17, 40, 4097), (70, 100, 260)])
def test_qmatvec(g, ctx, rows, O, K, group):
    w = rand(O, K, seed=1)
    codes, scales = g.quantize_weights(ctx, w, group)
    m = torch.nn.functional.pad(w, (0, -K % group)).unflatten(1, (-1, group))
    top = m.abs().amax(2, keepdim=True)
    assert torch.equal(scales, (top / torch.full_like(top, 7))[..., 0])  # a tensor over a number would be a product
    q = torch.where(top > 0, torch.round(m * (torch.full_like(top, 7) / top)), 0.0).flatten(1)[:, :K]
    full = ref.weights(codes, scales, K, group)
    close(full, q.cpu().double() * scales.cpu().double()[:, torch.arange(K) // group], 1e-15)
    codes = torch.randint(0, 256, codes.shape, generator=torch.Generator().manual_seed(2), dtype=torch.uint8).cuda()
    full = ref.weights(codes, scales, K, group)
    for dtype in (F32, BF16):
        x = rand(rows, K, dtype=dtype, seed=3)
        want = x.cpu().double() @ full.t()
        # every product is exact or rounded once: the terms' size bounds the error
        size = float((x.cpu().double().abs() @ full.abs().t()).norm())
        for xx in (x, strided(x, 1, 3, 1)):
            got = g.qmatvec(ctx, xx, codes, scales, group)
            assert got.dtype == dtype
            off = float((got.cpu().double() - want).norm())
            assert off <= FWD * size + (HALF * float(want.norm()) if dtype == BF16 else 0)
    x8 = torch.randint(-127, 128, (rows, K), generator=torch.Generator().manual_seed(4), dtype=torch.int8).cuda()
    xs = rand(rows, seed=5).abs()
    want = (x8.cpu().double() * xs.cpu().double()[:, None]) @ full.t()
    size = float((x8.cpu().double().abs() * xs.cpu().double()[:, None] @ full.abs().t()).norm())
    for xx in (x8, strided(x8, 1, 3, 1)):
        assert float((g.qmatvec(ctx, xx, codes, scales, group, x_scale=xs).cpu().double() - want).norm()) <= FWD * size


def test_quantize_odd_weights(g, ctx):
    w = rand(6, 100, seed=1)
    w[0, :32], w[1, 3], w[2, 99] = 0, float("inf"), float("nan")
    codes, scales = g.quantize_weights(ctx, w, 32)
    assert float(scales[0, 0]) == 0 and set(codes[0, :16].tolist()) == {0x88}
    assert bool(scales[1, 0].isnan()) and bool(scales[2, 3].isnan()) and set(codes[1, :16].tolist()) == {0x88}
    assert bool(torch.isfinite(scales[3:]).all()) and set(codes[:, 50:].flatten().tolist()) == {0x88}  # past the inputs
    x = rand(2, 100, seed=2)
    y = g.qmatvec(ctx, x, codes, scales, 32)
    assert bool(y[:, 1:3].isnan().all()) and bool(torch.isfinite(y[:, [0, 3, 4, 5]]).all())
    half = g.quantize_weights(ctx, strided(w.to(BF16), 1, 3, 1), 32)
    whole = g.quantize_weights(ctx, w.to(BF16), 32)
    assert torch.equal(half[0], whole[0]) and torch.equal(half[1].nan_to_num(), whole[1].nan_to_num())
    assert g.qmatvec(ctx, x[:0], codes, scales, 32).shape == (0, 6)


# ---- what all of them share ----

def test_nothing_is_written_past_the_outputs(g, ctx):
    """Odd sizes into the middle of larger buffers, through the C entry points."""
    from paper_1507_04296_amd import sequence as sq
    L = g.lib()

    def room(n, dtype=F32):
        buf = torch.full((n + 128,), 7.0, dtype=dtype, device="cuda")
        return buf, buf[64:64 + n]

    def scan_struct(i, state):
        rows = [v for t in (i["x"], i["dt"], i["b"], i["c"]) for v in (t.data_ptr(), t.stride(0), t.stride(1))]
        return sq._ScanArgs(0 if i["x"].dtype == F32 else 1, B, T, H, P, G, N, 0, *rows, i["a_log"].data_ptr(), i["dt_bias"].data_ptr(),
                            i["skip"].data_ptr(), None, None if state is None else state.data_ptr())

    def check(bufs):
        for buf, mid in bufs:
            n = mid.numel()
            assert bool((buf[:64] == 7).all()) and bool((buf[64 + n:] == 7).all())
            assert not bool((mid == 7).all())

    B, T, H, P, G, N = 2, 37, 3, 13, 3, 9
    for dtype in (F32, BF16):
        i = scan_inputs(B, T, H, P, G, N, dtype)
        a = scan_struct(i, None)
        out = [room(B * T * H * P, dtype), room(B * H * P * N)]
        assert L.gorila_scan(a, *(m.data_ptr() for _, m in out), ctx.bind_stream()) == 0
        check(out)
        dy, st = rand(B, T, H, P, dtype=dtype, seed=9), rand(B, H, P, N, seed=8)
        a = scan_struct(i, st)
        out = [room(i[k].numel(), dtype if n < 4 else F32) for n, k in enumerate(i)] + [room(st.numel())]
        assert L.gorila_scan_backward(a, dy.data_ptr(), dy.stride(0), dy.stride(1), None, *(m.data_ptr() for _, m in out), ctx.bind_stream()) == 0
        check(out)
        x, w, b, win = rand(B, T, 11, dtype=dtype, seed=1), rand(11, 4, seed=2), rand(11, seed=3), rand(B, 3, 11, dtype=dtype, seed=4)
        a = sq._ConvArgs(0 if dtype == F32 else 1, B, T, 11, 4, 1, x.data_ptr(), *x.stride()[:2], w.data_ptr(), b.data_ptr(), None, win.data_ptr())
        out = [room(x.numel(), dtype), room(win.numel(), dtype)]
        assert L.gorila_causal_conv(a, *(m.data_ptr() for _, m in out), ctx.bind_stream()) == 0
        check(out)
        out = [room(x.numel(), dtype), room(w.numel()), room(b.numel()), room(win.numel(), dtype)]
        assert L.gorila_causal_conv_backward(a, x.data_ptr(), x.stride(0), x.stride(1), None, *(m.data_ptr() for _, m in out), ctx.bind_stream()) == 0
        check(out)


def test_other_streams(g, ctx):
    """Calls run on torch's current stream, in its order."""
    i = scan_inputs(2, 300, 4, 64, 1, 64, F32)
    want = g.scan(ctx, **i)[0]
    side = torch.cuda.Stream()
    x2 = torch.zeros_like(i["x"])
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        big = torch.randn(4096, 4096, device="cuda")
        for _ in range(4):
            big = big @ big * 1e-2  # work that the copy waits for
        x2.copy_(i["x"])
        got = g.scan(ctx, **dict(i, x=x2))[0]
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    torch.cuda.synchronize()
    assert torch.equal(g.scan(ctx, **i)[0], want)


def test_graph_replays(g, ctx):
    """Captured once, replayed with other work between, and with new inputs."""
    B, T, H, P, G, N = 2, 200, 4, 64, 1, 32
    i = scan_inputs(B, T, H, P, G, N, F32)
    dy, w, cw = rand(B, T, H, P, seed=9), 1 + rand(H * P, scale=0.1, seed=10), rand(H * P, 4, seed=11)
    q = g.quantize_weights(ctx, rand(96, H * P, seed=12), 64)
    slot = torch.arange(B, dtype=torch.int32, device="cuda")

    def work(x):
        flat = x.reshape(B * T, H * P)
        y, total, rstd = g.add_rmsnorm(ctx, flat, w, flat)
        out = [*g.add_rmsnorm_backward(ctx, y, total, rstd, w), *g.add_rmsnorm_codes(ctx, flat, w)[:2]]
        cx = y.view(B, T, H * P)
        out += [*g.causal_conv(ctx, cx, cw), *g.causal_conv_backward(ctx, cx, cx, cw)[:2]]
        out += [*g.scan(ctx, **dict(i, x=x)), *g.scan_backward(ctx, dy, **dict(i, x=x))[:7]]
        pool = torch.ones(B, H, P, N, device="cuda")
        out += [g.scan_step(ctx, x[:, 0], i["dt"][:, 0], i["b"][:, 0], i["c"][:, 0], i["a_log"], i["dt_bias"], i["skip"], pool, slot), pool]
        out += [g.qmatvec(ctx, flat[:2], *q), g.qmatvec(ctx, out[2][:2], *q, x_scale=out[3][:2])]
        return out

    x = i["x"].clone()
    other = rand(B, T, H, P, seed=50)
    want, want2 = [t.clone() for t in work(x)], [t.clone() for t in work(other)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = work(x)
    for k, (values, expect) in enumerate(((i["x"], want), (other, want2), (i["x"], want), (i["x"], want))):
        x.copy_(values)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q_) for p, q_ in zip(got, expect)), k
        assert all(torch.equal(p, q_) for p, q_ in zip(work(other), want2)), k


def test_offsets_past_32_bits(g, ctx):
    """A state pool and a batch stride beyond 2^31 elements."""
    H, P, N = 16, 64, 64
    slots = (1 << 31) // (H * P * N) + 3
    pool = torch.empty(slots, H, P, N, device="cuda")
    pool[0], pool[-1] = 5.0, 2.0
    i = {k: v[:, 0] if v.dim() > 2 else v for k, v in scan_inputs(1, 1, H, P, 1, N, F32).items()}
    small = torch.full((1, H, P, N), 2.0, device="cuda")
    y = g.scan_step(ctx, **i, state_pool=pool, slot=torch.tensor([slots - 1], dtype=torch.int32, device="cuda"))
    assert torch.equal(y, g.scan_step(ctx, **i, state_pool=small))
    assert torch.equal(pool[-1], small[0]) and bool((pool[0] == 5).all())
    far = pool.view(-1)[: (1 << 31) + (1 << 20)].view(BF16)  # 2^32 elements and more
    x = far.as_strided((2, 40, 4, 16), ((1 << 32) + 64, 64, 16, 1))
    x.copy_(rand(2, 40, 4, 16, dtype=BF16, seed=3))
    j = scan_inputs(2, 40, 4, 16, 1, 16, BF16)
    j["x"] = x
    near = dict(j, x=x.contiguous())
    assert torch.equal(g.scan(ctx, **j)[0], g.scan(ctx, **near)[0])
    xc = x.flatten(2)
    w = rand(64, 4, seed=4)
    assert torch.equal(g.causal_conv(ctx, xc, w)[0], g.causal_conv(ctx, xc.contiguous(), w)[0])
    rows = xc[:, 0]
    assert torch.equal(g.add_rmsnorm(ctx, rows, w[:, 0].contiguous())[0], g.add_rmsnorm(ctx, rows.contiguous(), w[:, 0].contiguous())[0])


def test_refusals(g, ctx):
    """Wrong shapes, types and places raise before anything runs; the library's own checks return their codes."""
    i = scan_inputs(2, 8, 2, 8, 1, 8, F32)
    bad = [dict(x=i["x"][..., :4]), dict(dt=i["dt"][:, :4]), dict(b=i["b"][:1]), dict(a_log=i["a_log"][:1]), dict(skip=i["skip"].cpu()),
           dict(x=i["x"].transpose(2, 3)), dict(reset=torch.zeros(2, 7, dtype=torch.uint8, device="cuda")), dict(state=i["x"])]
    for change in bad:
        with pytest.raises(ValueError):
            g.scan(ctx, **{**i, **change})
    for change in (dict(x=i["x"].half()), dict(dt=i["dt"].to(BF16)), dict(a_log=i["a_log"].double()), dict(reset=torch.zeros(2, 8, device="cuda"))):
        with pytest.raises(TypeError):
            g.scan(ctx, **{**i, **change})

    def code(f, *a, **k):
        with pytest.raises(g.GorilaError) as e:
            f(*a, **k)
        return e.value.code

    assert code(g.scan, ctx, **scan_inputs(1, 4, 3, 8, 2, 8, F32)) == -1  # groups do not divide heads
    assert code(g.scan, ctx, **scan_inputs(1, 4, 1, 129, 1, 8, F32)) == -5
    assert code(g.scan, ctx, **scan_inputs(1, 4, 1, 8, 1, 129, F32)) == -5
    none, tiny = g.Context(0, 1), g.Context(1, 1)
    long = scan_inputs(1, 64, 1, 8, 1, 8, F32)
    assert code(g.scan_backward, none, long["x"], **long) == -3
    assert code(g.scan, none, **scan_inputs(1, 4000, 1, 64, 1, 64, F32)) == -3
    big = scan_inputs(16, 512, 16, 64, 1, 64, F32)
    assert code(g.scan_backward, tiny, big["x"], **big) == -3
    x, w = rand(4, 8, seed=1), rand(8, 4, seed=2)
    one, sl = {k: v[:, 0] if v.dim() > 2 else v for k, v in scan_inputs(4, 1, 2, 8, 1, 8, F32).items()}, torch.zeros(4, dtype=torch.int32, device="cuda")
    pool = rand(4, 2, 8, 8, seed=3)
    assert code(g.scan_step, none, **one, state_pool=pool, slot=sl) == -3  # nowhere to report a slot
    g.scan_step(none, **one, state_pool=pool)  # and none needed without
    assert code(g.scan_step, ctx, **one, state_pool=pool[:3]) == -1
    assert code(g.causal_conv_step, none, x, rand(4, 3, 8, seed=4), w, slot=sl) == -3
    assert code(g.causal_conv_step, ctx, x, rand(3, 3, 8, seed=4), w) == -1
    for taps in (1, 5):
        with pytest.raises(g.GorilaError):
            g.causal_conv(ctx, x[None], rand(8, taps, seed=2))
    assert code(g.causal_conv_backward, none, x[None], x[None], w) == -3
    assert code(g.add_rmsnorm, ctx, x, w[:, 0].contiguous(), eps=-1.0) == -1
    assert code(g.add_rmsnorm, ctx, x, w[:, 0].contiguous(), eps=float("nan")) == -1
    assert code(g.add_rmsnorm, ctx, rand(1, 65537), rand(65537)) == -1
    y, total, rstd = g.add_rmsnorm(ctx, x, w[:, 0].contiguous())
    assert code(g.add_rmsnorm_backward, none, y, total, rstd, w[:, 0].contiguous()) == -3
    codes, scales = g.quantize_weights(ctx, rand(5, 8, seed=5), 32)
    for call in (lambda: g.quantize_weights(ctx, x, 48), lambda: g.qmatvec(ctx, x, codes, scales, 16), lambda: g.qmatvec(ctx, x, codes[:, :8], scales, 32),
                 lambda: g.qmatvec(ctx, x.to(torch.int8), codes, scales, 32), lambda: g.qmatvec(ctx, x, codes, scales, 32, x_scale=x[:, 0].contiguous())):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        g.qmatvec(ctx, x.half(), codes, scales, 32)
    ctx.check()
    none.close()
    tiny.close()
