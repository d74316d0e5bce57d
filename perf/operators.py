"""Performance cases of the sequence operators: the recurrent core that sits on
the Q-network's 512 features when a game has to be remembered.

Learners train it on replayed sequences (episodes start inside them), actors run
it one step at a time for their environments, on 4-bit replicas of its
projections.  Operators: the norm with the residual's addition (also with 8-bit
rows out), the short causal convolution, the selective scan, and products with
4-bit weights.

    own                 False: elementary torch in 32 bits; True: the library
    listed()            the cases that are always measured
    draw(rng)           one more case of the same ranges
    prepare(case, seed) what the program holds before the call, on the GPU
    run(state)          one pass; returns the outputs
    work(case)          bytes and operations that one pass cannot do without
    exact(case, seed)   the outputs from the definitions, in 64 bits
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
SIZE = {"f32": 4, "bf16": 2}
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # Norm and residual of a learner's 512 sequences of 32 features, forward
        # and backward (the width is FC-512's).
        dict(name="norm_train", kind="norm", rows=16384, width=512, type="f32"),
        # A bf16 learner's larger batch, at a width that fills no power of two.
        dict(name="norm_train_ragged", kind="norm", rows=40007, width=1000, type="bf16"),
        # 1024 environments' features as 8-bit rows.
        dict(name="norm_codes_1024", kind="codes", rows=1024, width=512, type="f32"),
        # The core's convolution over DQN's minibatch of 32 as sequences: 16
        # heads of 64 channels, and 64 + 64 for the two state projections.
        dict(name="conv_train", kind="conv", batch=32, length=128, channels=1152, taps=4, type="f32"),
        # The same, one step of 1024 environments.
        dict(name="conv_step_1024", kind="conv_step", rows=1024, channels=1152, taps=4, type="f32"),
        # The scan of that minibatch, forward and backward.
        dict(name="scan_train", kind="scan", batch=32, length=128, heads=16, width=64, groups=1, state=64, type="f32"),
        # Few long ragged sequences on a bf16 learner, with a larger state.
        dict(name="scan_train_long", kind="scan", batch=4, length=1999, heads=16, width=64, groups=2, state=128, type="bf16"),
        # One recorded episode through a bf16 replica, to rebuild its state.
        dict(name="scan_prompt", kind="prompt", batch=1, length=8192, heads=16, width=64, groups=1, state=64, type="bf16"),
        # One actor's next step: all latency.
        dict(name="scan_step_1", kind="step", rows=1, heads=16, width=64, groups=1, state=64, type="f32"),
        # All environments of one GPU stepping together.
        dict(name="scan_step_1024", kind="step", rows=1024, heads=16, width=64, groups=1, state=64, type="f32"),
        # One row through a large 4-bit matrix.
        dict(name="matvec_1", kind="matvec", rows=1, outputs=8192, inputs=8192, group=128, type="bf16"),
        # 16 environments' norm to 8-bit rows, and the core's input projection
        # (1024 + 128 channels and 16 step sizes) of them.
        dict(name="project_16", kind="project", rows=16, outputs=1168, inputs=512, group=64, type="f32"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi)))))))


def draw(rng):
    """Sizes over the whole range (uniform in the logarithm), odd ones among them."""
    kind = rng.choice(["norm", "codes", "conv", "conv_step", "scan", "scan", "prompt", "step", "matvec", "matvec", "project"])
    kw = dict(kind=kind, type=rng.choice(["f32", "bf16"]))
    if kind in ("norm", "codes"):
        width = _log_int(rng, 33, 8192)
        return dict(kw, width=width, rows=_log_int(rng, 1, 40_000_000 // width if width > 600 else 65536))
    if kind in ("conv", "conv_step"):
        channels, taps = _log_int(rng, 24, 2304), rng.randint(2, 4)
        if kind == "conv_step":
            return dict(kw, rows=_log_int(rng, 1, 2048), channels=channels, taps=taps)
        length = _log_int(rng, 1, 2048)
        return dict(kw, length=length, batch=_log_int(rng, 1, max(1, 8192 // length)), channels=channels, taps=taps)
    if kind in ("scan", "prompt", "step"):
        groups = rng.choice([1, 1, 2, 4])
        kw.update(groups=groups, heads=groups * rng.randint(1, 16 // groups),
                  width=rng.choice([16, 32, 40, 64, 64, 96, 128]), state=rng.choice([16, 24, 32, 64, 64, 100, 128]))
        if kind == "step":
            return dict(kw, rows=_log_int(rng, 1, 512))
        length = _log_int(rng, 1, 2000 if kind == "scan" else 8192)
        most = min(8192 // length, (250_000_000 if kind == "scan" else 1_000_000_000) // (kw["heads"] * length * length))
        return dict(kw, length=length, batch=_log_int(rng, 1, max(1, min(64, most))))
    return dict(kw, rows=_log_int(rng, 1, 64), outputs=_log_int(rng, 16, 8192), inputs=_log_int(rng, 40, 8192),
                group=rng.choice([32, 64, 128]))


# ---- inputs (from the seed alone) ----

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(1507 + 1000003 * int(seed))
    typ, kind = TYPE[case["type"]], case["kind"]

    def normal(*shape, scale=1.0, dtype=None):
        return (scale * torch.randn(shape, generator=gen, device="cuda")).to(dtype or typ)

    def uniform(*shape):
        return torch.rand(shape, generator=gen, device="cuda")

    s = {"case": case}
    if kind in ("norm", "codes", "project"):
        rows, width = case["rows"], case["inputs" if kind == "project" else "width"]
        s.update(x=normal(rows, width), residual=normal(rows, width, scale=2.0),
                 weight=1.0 + normal(width, scale=0.1, dtype=torch.float32))
    if kind == "norm":
        s.update(dy=normal(rows, width, scale=0.01), dtotal=normal(rows, width, scale=0.01))
    if kind in ("matvec", "project"):
        rows, out, k = case["rows"], case["outputs"], case["inputs"]
        packed = 16 * -(-k // 32)  # bytes a row: whole runs of 32 codes
        codes = torch.randint(0, 256, (out, packed), generator=gen, device="cuda", dtype=torch.uint8)
        s.update(codes=codes, scales=(0.5 + uniform(out, -(-k // case["group"]))) * (0.25 / math.sqrt(k)))
        if kind == "matvec":
            s.update(x=normal(rows, k))
    if kind in ("conv", "conv_step"):
        c, k = case["channels"], case["taps"]
        s.update(weight=(2.0 * uniform(c, k) - 1.0) / math.sqrt(k), bias=(2.0 * uniform(c) - 1.0) / math.sqrt(k))
    if kind == "conv":
        b, t = case["batch"], case["length"]
        s.update(x=normal(b, t, c), window=normal(b, k - 1, c), reset=(uniform(b, t) < 0.01).to(torch.uint8),
                 dy=normal(b, t, c, scale=0.01))
    if kind == "conv_step":
        n = case["rows"]
        s.update(x=normal(n, c), window=normal(n + 3, k - 1, c), reset=(uniform(n) < 0.01).to(torch.uint8),
                 slot=torch.randperm(n + 3, generator=gen, device="cuda")[:n].to(torch.int32))
    if kind in ("scan", "prompt", "step"):
        h, p, g, n = case["heads"], case["width"], case["groups"], case["state"]
        step = torch.exp(math.log(1e-3) + math.log(100.0) * uniform(h))  # step sizes at dt = 0: 0.001 .. 0.1
        s.update(a_log=torch.log(1.0 + 15.0 * uniform(h)), dt_bias=step + torch.log(-torch.expm1(-step)),
                 skip=1.0 + normal(h, scale=0.1, dtype=torch.float32))
        lead = (case["rows"],) if kind == "step" else (case["batch"], case["length"])
        s.update(x=normal(*lead, h, p, scale=0.7), dt=normal(*lead, h, scale=0.5), b=normal(*lead, g, n, scale=0.7),
                 c=normal(*lead, g, n, scale=0.7), reset=(uniform(*lead) < 0.01).to(torch.uint8))
        states = case["rows"] + 3 if kind == "step" else case["batch"]
        s.update(state=normal(states, h, p, n, scale=0.3, dtype=torch.float32))
        if kind == "step":
            s.update(slot=torch.randperm(states, generator=gen, device="cuda")[:lead[0]].to(torch.int32))
        if kind == "scan":
            s.update(dy=normal(*lead, h, p, scale=0.01))
    return s


# ---- one pass ----

def run(s):
    return (_own if own else _plain)(s, s["case"]["kind"])


def _own(s, kind):
    import paper_1507_04296_amd as g
    case = s["case"]
    if "ctx" not in s:  # the handle that such a program keeps
        need = 0
        if kind == "scan" or kind == "prompt":
            need = g.scan_workspace_bytes(case["batch"], case["length"], case["heads"], case["width"], case["groups"],
                                          case["state"], backward=kind == "scan")
        elif kind == "conv":
            need = g.causal_conv_workspace_bytes(case["channels"], case["taps"])
        elif kind == "norm":
            need = g.add_rmsnorm_workspace_bytes(case["width"])
        s["ctx"] = _context(g, need)
    ctx = s["ctx"]
    if kind == "norm":
        y, total, rstd = g.add_rmsnorm(ctx, s["x"], s["weight"], s["residual"], EPS)
        dx, dweight = g.add_rmsnorm_backward(ctx, s["dy"], total, rstd, s["weight"], s["dtotal"])
        return dict(y=y, total=total, dx=dx, dweight=dweight)
    if kind == "codes":
        codes, scale, total = g.add_rmsnorm_codes(ctx, s["x"], s["weight"], s["residual"], EPS)
        return dict(values=codes * scale[:, None], total=total)
    if kind == "project":
        codes, scale, total = g.add_rmsnorm_codes(ctx, s["x"], s["weight"], s["residual"], EPS)
        return dict(y=g.qmatvec(ctx, codes, s["codes"], s["scales"], case["group"], x_scale=scale), total=total)
    if kind == "matvec":
        return dict(y=g.qmatvec(ctx, s["x"], s["codes"], s["scales"], case["group"]))
    if kind == "conv":
        y, window = g.causal_conv(ctx, s["x"], s["weight"], s["bias"], s["reset"], s["window"])
        dx, dweight, dbias, _ = g.causal_conv_backward(ctx, s["dy"], s["x"], s["weight"], s["bias"], s["reset"], s["window"])
        return dict(y=y, window=window, dx=dx, dweight=dweight, dbias=dbias)
    if kind == "conv_step":
        y = g.causal_conv_step(ctx, s["x"], s["window"], s["weight"], s["bias"], s["slot"], s["reset"])
        return dict(y=y, window=s["window"])
    par = (s["a_log"], s["dt_bias"], s["skip"])
    if kind == "step":
        y = g.scan_step(ctx, s["x"], s["dt"], s["b"], s["c"], *par, s["state"], s["slot"], s["reset"])
        return dict(y=y, state=s["state"])
    y, state = g.scan(ctx, s["x"], s["dt"], s["b"], s["c"], *par, s["reset"], s["state"])
    out = dict(y=y, state=state)
    if kind == "scan":
        dx, ddt, db, dc, da_log, ddt_bias, dskip, _ = g.scan_backward(
            ctx, s["dy"], s["x"], s["dt"], s["b"], s["c"], *par, s["reset"], s["state"])
        out.update(dx=dx, ddt=ddt, db=db, dc=dc, da_log=da_log, ddt_bias=ddt_bias, dskip=dskip)
    return out


_held = {}


def _context(g, need):
    """One context, with the largest workspace asked for so far."""
    ctx = _held.get("ctx")
    if ctx is None or ctx.ws_bytes < need:
        _held["ctx"] = ctx = g.Context(1, 1, min_bytes=need)
    return ctx


def _plain(s, kind):
    typ = TYPE[s["case"]["type"]]
    f = {k: v.float() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in s.items()}
    if kind == "norm":
        w = f["weight"].detach().requires_grad_()
        total = (f["x"] + f["residual"]).to(typ)
        t = total.float().requires_grad_()
        y = t * torch.rsqrt(t.square().mean(1, keepdim=True) + EPS) * w
        dx, dweight = torch.autograd.grad([y, t], [t, w], [f["dy"], f["dtotal"]])
        return dict(y=y.detach().to(typ), total=total, dx=dx.to(typ), dweight=dweight)
    if kind == "codes":
        codes, scale, total = _plain_codes(f, typ)
        return dict(values=codes * scale, total=total)
    if kind == "project":
        codes, scale, total = _plain_codes(f, typ)
        return dict(y=(codes * scale) @ _plain_weights(f).t(), total=total)
    if kind == "matvec":
        return dict(y=(f["x"] @ _plain_weights(f).t()).to(typ))
    if kind == "conv":
        x, w, b = (f[k].detach().requires_grad_() for k in ("x", "weight", "bias"))
        y, window = _plain_conv(x, w, b, f["reset"], f["window"])
        dx, dweight, dbias = torch.autograd.grad(y, [x, w, b], f["dy"])
        return dict(y=y.detach().to(typ), window=window.to(typ), dx=dx.to(typ), dweight=dweight, dbias=dbias)
    if kind == "conv_step":
        at = s["slot"].long()
        y, window = _plain_conv(f["x"][:, None], f["weight"], f["bias"], f["reset"][:, None], f["window"][at])
        s["window"][at] = window.to(typ)
        return dict(y=y[:, 0].to(typ), window=s["window"])
    names = ("x", "dt", "b", "c", "a_log", "dt_bias", "skip")
    if kind == "step":
        at = s["slot"].long()
        rep = f["x"].shape[1] // f["b"].shape[1]
        d = torch.logaddexp(f["dt"] + f["dt_bias"], torch.zeros_like(f["dt"]))
        keep = torch.exp(-torch.exp(f["a_log"]) * d)[:, :, None, None]
        old = torch.where(f["reset"].bool()[:, None, None, None], torch.zeros_like(keep), keep * s["state"][at])
        new = old + (d[:, :, None] * f["x"])[..., None] * f["b"].repeat_interleave(rep, 1)[:, :, None]
        s["state"][at] = new
        y = (new * f["c"].repeat_interleave(rep, 1)[:, :, None]).sum(3) + f["skip"][:, None] * f["x"]
        return dict(y=y.to(typ), state=s["state"])
    leaves = [f[k].detach().requires_grad_(kind == "scan") for k in names]
    y, state = _plain_scan(*leaves, f["reset"], f["state"])
    out = dict(y=y.detach().to(typ), state=state.detach())
    if kind == "scan":
        grads = torch.autograd.grad(y, leaves, f["dy"])
        out.update(("d" + k, v.to(typ) if k in names[:4] else v) for k, v in zip(names, grads))
    return out


def _plain_codes(f, typ):
    """Codes of the row times the weight, relative to its largest; the norm's factor is in the scale alone."""
    total = (f["x"] + f["residual"]).to(typ)
    t = total.float()
    u = t * f["weight"]
    most = u.abs().amax(1, keepdim=True)
    codes = torch.round(u * (torch.full_like(most, 127.0) / most))
    return codes, torch.rsqrt(t.square().mean(1, keepdim=True) + EPS) * (most / 127.0), total


def _plain_weights(f):
    """The matrix that the codes and their groups' scales stand for."""
    k, group = f["case"]["inputs"], f["case"]["group"]
    codes = torch.stack((f["codes"] & 15, f["codes"] >> 4), 2).flatten(1)[:, :k].float() - 8.0
    return codes * f["scales"].repeat_interleave(group, 1)[:, :k]


def _plain_conv(x, w, bias, reset, window):
    taps = w.shape[1]
    e = torch.cat([window, x], 1)
    episode = torch.nn.functional.pad(reset.long().cumsum(1), (taps - 1, 0))
    same = episode.unfold(1, taps, 1) == episode[:, taps - 1:, None]  # [batch, length, taps]
    v = (torch.where(same[:, :, None], e.unfold(1, taps, 1), 0.0) * w).sum(3) + bias
    last = e[:, x.shape[1]:]
    live = (episode[:, x.shape[1]:] == episode[:, -1:])[..., None]
    return v * torch.sigmoid(v), torch.where(live, last, 0.0)


def _plain_scan(x, dt, b, c, a_log, dt_bias, skip, reset, state):
    """The scan as a masked product: y_t = sum over s <= t of (C_t . B_s) decay(s..t) d_s x_s."""
    rep = x.shape[2] // b.shape[2]
    d = torch.logaddexp(dt + dt_bias, torch.zeros_like(dt)).transpose(1, 2)  # [batch, heads, length]
    g = -torch.exp(a_log)[:, None] * d
    episode = reset.long().cumsum(1)
    length = x.shape[1]
    at = torch.arange(length, device=x.device)
    later = at[:, None] > at
    same = (at[:, None] >= at) & (episode[:, :, None] == episode[:, None])
    sums = torch.where(later, g[..., None], 0.0).cumsum(2)  # log-decays of s + 1 .. t
    decay = torch.where(same[:, None], torch.exp(sums), 0.0)
    bg, cg = b.transpose(1, 2), c.transpose(1, 2)
    both = (cg @ bg.transpose(2, 3)).repeat_interleave(rep, 1)
    v = d[..., None] * x.transpose(1, 2)  # [batch, heads, length, width]
    ch, bh = cg.repeat_interleave(rep, 1), bg.repeat_interleave(rep, 1)
    first = torch.where((episode == 0)[:, None], torch.exp(g.cumsum(2)), 0.0)  # decay of the state before
    y = (both * decay) @ v + first[..., None] * (ch @ state.transpose(2, 3)) + skip[:, None, None] * x.transpose(1, 2)
    end = (v * decay[:, :, -1, :, None]).transpose(2, 3) @ bh + first[:, :, -1, None, None] * state
    return y.transpose(1, 2), end


# ---- what one pass cannot do without ----

def work(case):
    kind, e = case["kind"], SIZE[case["type"]]
    if kind in ("norm", "codes"):
        n = case["rows"] * case["width"]
        if kind == "norm":  # x, residual, dy, dtotal in; y, total, dx out
            return dict(bytes=7 * e * n + 8 * case["width"], flops=14 * n)
        return dict(bytes=3 * e * n + 4 * n + 4 * case["width"], flops=8 * n)
    if kind in ("matvec", "project"):
        m, o, k = case["rows"], case["outputs"], case["inputs"]
        weights = o * k / 2 + 4 * o * -(-k // case["group"])
        if kind == "matvec":
            return dict(bytes=weights + e * m * (k + o), flops=2 * m * o * k)
        return dict(bytes=weights + 3 * e * m * k + 4 * m * o, flops=2 * m * o * k + 8 * m * k)
    if kind == "conv":
        n, c, k = case["batch"] * case["length"] * case["channels"], case["channels"], case["taps"]
        return dict(bytes=4 * e * n + 8 * c * (k + 1), flops=n * (6 * k + 20))
    if kind == "conv_step":
        n, k = case["rows"] * case["channels"], case["taps"]
        return dict(bytes=e * n * (2 + 2 * (k - 1)) + 4 * case["channels"] * (k + 1), flops=n * (2 * k + 6))
    h, p, g, n = case["heads"], case["width"], case["groups"], case["state"]
    t = case["rows"] if kind == "step" else case["batch"] * case["length"]
    states = 8 * h * p * n * (case["rows"] if kind == "step" else case["batch"])  # in and out
    row = e * (h * p + h + 2 * g * n)  # x, dt, b, c of one step
    if kind == "scan":  # y and the state; dy in, and a gradient of each input
        return dict(bytes=t * (2 * row + 2 * e * h * p) + states, flops=19 * t * h * p * n)
    return dict(bytes=t * (row + e * h * p) + states, flops=5 * t * h * p * n)


# ---- the definitions in 64 bits ----

def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    f = {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in s.items()}
    if kind in ("norm", "codes", "project"):
        total = f["x"] + f["residual"]
        t = total.to(TYPE[case["type"]]).double()  # the stream holds the rounded sum
        width = t.shape[1]
        rho = 1.0 / torch.sqrt((t * t).sum(1, keepdim=True) / width + EPS)
        if kind == "norm":
            wdy = f["dy"] * f["weight"]
            dx = f["dtotal"] + rho * wdy - t * rho ** 3 * ((wdy * t).sum(1, keepdim=True) / width)
            return dict(y=t * rho * f["weight"], total=total, dx=dx, dweight=(f["dy"] * t * rho).sum(0))
        # the codes' definition has its roundings to 32 bits: product, quotient, product
        u = (t * f["weight"]).float()
        most = u.abs().amax(1, keepdim=True)
        codes = torch.round((u.double() * (127.0 / most.double()).float().double()).float()).double()
        values = codes * rho * most.double() / 127.0
        if kind == "codes":
            return dict(values=values, total=total)
        return dict(y=values @ _exact_weights(f).t(), total=total)
    if kind == "matvec":
        return dict(y=f["x"] @ _exact_weights(f).t())
    if kind == "conv":
        return _exact_conv(f)
    if kind == "conv_step":
        at = s["slot"].long()
        got = _exact_conv(dict(f, x=f["x"][:, None], reset=s["reset"][:, None], window=f["window"][at], dy=None))
        f["window"][at] = got["window"]
        return dict(y=got["y"][:, 0], window=f["window"])
    if kind == "step":
        at = s["slot"].long()
        one = {k: f[k][:, None] for k in ("x", "dt", "b", "c")}
        got = _exact_scan(dict(f, **one, reset=s["reset"][:, None], state=f["state"][at], dy=None))
        f["state"][at] = got["state"]
        return dict(y=got["y"][:, 0], state=f["state"])
    return _exact_scan(dict(f, dy=f.get("dy")))


def _exact_weights(f):
    k, group, codes = f["case"]["inputs"], f["case"]["group"], f["codes"].long()
    w = torch.empty(codes.shape[0], 2 * codes.shape[1], dtype=torch.float64, device=codes.device)
    w[:, 0::2], w[:, 1::2] = (codes % 16 - 8).double(), (codes // 16 - 8).double()
    return w[:, :k] * f["scales"][:, torch.arange(k, device=codes.device) // group]


def _exact_conv(f):
    x, w, reset = f["x"], f["weight"], f["reset"]
    batch, length, taps = x.shape[0], x.shape[1], w.shape[1]
    e = torch.cat([f["window"], x], 1)
    v = f["bias"] + w[:, taps - 1] * x
    cut = torch.zeros(batch, length, 1, dtype=torch.bool, device=x.device)
    cuts = [cut]  # cuts[j]: an episode starts in the last j steps up to t
    for j in range(1, taps):
        moved = torch.zeros_like(cut)
        moved[:, j - 1:, 0] = reset[:, :length - j + 1].bool() if length >= j else False
        cut = cut | moved
        cuts.append(cut)
        v = v + w[:, taps - 1 - j] * torch.where(cut, 0.0, e[:, taps - 1 - j:taps - 1 - j + length])
    sig = 1.0 / (1.0 + torch.exp(-v))
    window = e[:, length:].clone()
    for i in range(taps - 1):  # step length - taps + 1 + i; a reset after it empties its place
        after = max(0, length - taps + 2 + i)
        window[:, i] *= 1.0 - reset[:, after:].bool().any(1).double()[:, None]
    out = dict(y=v * sig, window=window)
    if f["dy"] is None:
        return out
    dv = f["dy"] * sig * (1.0 + v * (1.0 - sig))
    de, dw = torch.zeros_like(e), torch.zeros_like(w)
    for j in range(taps):
        d = torch.where(cuts[j], 0.0, dv)
        at = slice(taps - 1 - j, taps - 1 - j + length)
        de[:, at] += w[:, taps - 1 - j] * d
        dw[:, taps - 1 - j] = (d * e[:, at]).sum((0, 1))
    return dict(out, dx=de[:, taps - 1:], dweight=dw, dbias=dv.sum((0, 1)))


def _exact_scan(f):
    x, b, c, dy = f["x"], f["b"], f["c"], f["dy"]
    length, heads, groups = x.shape[1], x.shape[2], b.shape[2]
    of = torch.arange(heads, device=x.device) // (heads // groups)  # the group of a head
    pre = f["dt"] + f["dt_bias"]
    d = torch.clamp(pre, min=0.0) + torch.log1p(torch.exp(-pre.abs()))
    rate = -torch.exp(f["a_log"])
    a = torch.exp(rate * d)
    a = torch.where(f["reset"].bool()[:, :, None], 0.0, a)
    state, y, before = f["state"], torch.empty_like(x), []
    for t in range(length):
        if dy is not None:
            before.append(state)
        state = a[:, t, :, None, None] * state + (d[:, t, :, None] * x[:, t])[..., None] * b[:, t, of, None]
        y[:, t] = (state * c[:, t, of, None]).sum(3) + f["skip"][:, None] * x[:, t]
    out = dict(y=y, state=state)
    if dy is None:
        return out
    dx, dd = torch.empty_like(x), torch.empty_like(d)
    dbh = torch.empty(*x.shape[:3], b.shape[3], dtype=x.dtype, device=x.device)
    dch = torch.empty_like(dbh)
    drate = torch.zeros_like(d[:, 0])
    r = torch.zeros_like(state)
    for t in range(length - 1, -1, -1):
        v = d[:, t, :, None] * x[:, t]
        bt, ct = b[:, t, of], c[:, t, of]
        r = r + dy[:, t, :, :, None] * ct[:, :, None]
        dv = (r * bt[:, :, None]).sum(3)
        dbh[:, t] = (r * v[..., None]).sum(2)
        now = a[:, t, :, None, None] * before[t]
        dch[:, t] = ((now + v[..., None] * bt[:, :, None]) * dy[:, t, :, :, None]).sum(2)
        dlog = (r * now).sum((2, 3))
        drate = drate + dlog * d[:, t]
        dx[:, t] = d[:, t, :, None] * dv + f["skip"][:, None] * dy[:, t]
        dd[:, t] = (dv * x[:, t]).sum(2) + dlog * rate
        r = a[:, t, :, None, None] * r
    ddt = dd / (1.0 + torch.exp(-pre))
    shape = (*x.shape[:2], groups, heads // groups, b.shape[3])
    return dict(out, dx=dx, ddt=ddt, db=dbh.view(shape).sum(3), dc=dch.view(shape).sum(3), da_log=(drate * rate).sum(0),
                ddt_bias=ddt.sum((0, 1)), dskip=(dy * x).sum((0, 1, 3)))
