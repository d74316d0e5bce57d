"""Performance cases of the operators with which a recurrent core learns and answers:
the layer norm with the residual's addition, the gated scan (a recurrence with a gate
for every channel), the AdamW step over many tensors, and sampled actions.

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

import numpy as np
import torch

own = False

EPS = 1e-5
BETA1, BETA2, RATE, ADAM_EPS, DECAY = 0.9, 0.999, 1e-3, 1e-8, 0.01
SIZE = {"f32": 4, "bf16": 2}
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
ONE = 1 << 40  # the weight of a row's largest value


def listed():
    return [
        # Norm and residual of DQN's minibatch of 32 as sequences of 128 steps,
        # forward and backward (the width is FC-512's).
        dict(name="layernorm_train", kind="norm", rows=4096, width=512, type="f32"),
        # A bf16 learner's larger batch, at a width that fills no power of two.
        dict(name="layernorm_ragged", kind="norm", rows=40007, width=1000, type="bf16"),
        # The recurrence of that minibatch, forward and backward: 1024 channels.
        dict(name="gated_train", kind="gated", batch=32, length=128, channels=1024, type="f32"),
        # Few long ragged sequences on a bf16 learner.
        dict(name="gated_train_long", kind="gated", batch=4, length=1999, channels=2000, type="bf16"),
        # One recorded episode through a bf16 replica, to rebuild its state.
        dict(name="gated_prompt", kind="prompt", batch=1, length=8192, channels=1024, type="bf16"),
        # One actor's next step: all latency.
        dict(name="gated_step_1", kind="step", rows=1, channels=1024, type="f32"),
        # All environments of one GPU stepping together.
        dict(name="gated_step_1024", kind="step", rows=1024, channels=1024, type="f32"),
        # One update of the Q-network's ten tensors (18 actions).
        dict(name="adamw_network", kind="adamw", bits=32, type="f32",
             sizes="8192,32,32768,64,36864,64,1605632,512,9216,18"),
        # A large model's tensors, states in 8 bits, gradients of a bf16 learner.
        dict(name="adamw_large_8bit", kind="adamw", bits=8, type="bf16",
             sizes="16777216,4099,1048577,33554432,1000001,1"),
        # 1024 environments' actions from 18 values each, with a temperature of
        # their own.
        dict(name="sample_1024", kind="sample", rows=1024, actions=18, filters="t", type="f32"),
        # Many actions, all filters.
        dict(name="sample_wide", kind="sample", rows=256, actions=32000, filters="tkpm", type="bf16"),
        # One row of very many.
        dict(name="sample_row", kind="sample", rows=1, actions=100003, filters="tp", type="f32"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi)))))))


def draw(rng):
    """Sizes over the whole range (uniform in the logarithm), odd ones among them."""
    kind = rng.choice(["norm", "norm", "gated", "gated", "prompt", "step", "adamw", "adamw", "sample", "sample"])
    kw = dict(kind=kind, type=rng.choice(["f32", "bf16"]))
    if kind == "norm":
        width = _log_int(rng, 33, 8192)
        return dict(kw, width=width, rows=_log_int(rng, 1, min(65536, 40_000_000 // width)))
    if kind == "step":
        return dict(kw, rows=_log_int(rng, 1, 2048), channels=_log_int(rng, 16, 4096))
    if kind in ("gated", "prompt"):
        channels, length = _log_int(rng, 16, 4096), _log_int(rng, 1, 2048 if kind == "gated" else 16384)
        return dict(kw, channels=channels, length=length, batch=_log_int(rng, 1, max(1, min(512, 16_000_000 // (channels * length)))))
    if kind == "adamw":
        sizes = [_log_int(rng, 1, 2_000_000) for _ in range(rng.randint(1, 20))]
        return dict(kw, bits=rng.choice([8, 32]), sizes=",".join(map(str, sizes)))
    actions = _log_int(rng, 2, 131072)
    return dict(kw, actions=actions, rows=_log_int(rng, 1, max(1, min(4096, 8_000_000 // actions))),
                filters=rng.choice(["", "t", "tk", "tp", "tm", "tkp", "tkpm", "p"]))


# ---- inputs (from the seed alone) ----

def _sizes(case):
    return [int(n) for n in case["sizes"].split(",")]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(4296 + 1000003 * int(seed))
    typ, kind = TYPE[case["type"]], case["kind"]

    def normal(*shape, scale=1.0, dtype=None):
        return (scale * torch.randn(shape, generator=gen, device="cuda")).to(dtype or typ)

    def uniform(*shape):
        return torch.rand(shape, generator=gen, device="cuda")

    s = {"case": case}
    if kind == "norm":
        rows, width = case["rows"], case["width"]
        s.update(x=normal(rows, width), residual=normal(rows, width, scale=2.0) + normal(rows, 1),
                 weight=1.0 + normal(width, scale=0.1, dtype=torch.float32), bias=normal(width, scale=0.1, dtype=torch.float32),
                 dy=normal(rows, width, scale=0.01), dtotal=normal(rows, width, scale=0.01))
    if kind in ("gated", "prompt", "step"):
        c = case["channels"]
        lead = (case["rows"],) if kind == "step" else (case["batch"], case["length"])
        # decays at an open gate: 0.5 .. 0.999 (uniform in the logarithm of -log)
        s.update(a_log=math.log(1e-3) + math.log(700.0) * uniform(c), x=normal(*lead, c), gate_a=normal(*lead, c),
                 gate_x=normal(*lead, c), reset=(uniform(*lead) < 0.01).to(torch.uint8))
        states = case["rows"] + 3 if kind == "step" else case["batch"]
        s.update(state=normal(states, c, dtype=torch.float32))
        if kind == "step":
            s.update(slot=torch.randperm(states, generator=gen, device="cuda")[:lead[0]].to(torch.int32))
        if kind == "gated":
            s.update(dy=normal(*lead, c, scale=0.01))
    if kind == "adamw":
        sizes = _sizes(case)
        s.update(thetas=[normal(n, scale=0.05, dtype=torch.float32) for n in sizes], grads=[normal(n, scale=1e-3) for n in sizes],
                 decay=[DECAY if n > 4096 else 0.0 for n in sizes],  # matrices, not biases
                 clock=torch.tensor([100.0, 1 - BETA1 ** 100, 1 - BETA2 ** 100], dtype=torch.float64, device="cuda"))
        if case["bits"] == 32:
            s.update(states=[(normal(n, scale=3e-4, dtype=torch.float32), (0.5 + uniform(n)) * 1e-6) for n in sizes])
        else:  # codes and a scale for every 256: the most frequent ones lie near the largest
            def codes(n, last):
                return (last - 1.0 - 40.0 * uniform(n).square()).to(torch.uint8)

            s.update(states=[(codes(n, 127) + 128 * (uniform(n) < 0.5).to(torch.uint8), codes(n, 255),
                              (0.5 + uniform(-(-n // 256))) * 1e-3, (0.5 + uniform(-(-n // 256))) * 4e-6) for n in sizes])
    if kind == "sample":
        rows, filters = case["rows"], case["filters"]
        s.update(values=normal(rows, case["actions"], scale=2.0), u=uniform(rows), temperature=None, top_k=None, top_p=None, min_p=None)
        if "t" in filters:  # a tenth of the rows are greedy
            t = 0.25 + 1.75 * uniform(rows)
            s.update(temperature=torch.where(uniform(rows) < 0.1, 0.0, t))
        if "k" in filters:
            s.update(top_k=torch.randint(1, max(2, min(2 * case["actions"], 200)), (rows,), generator=gen, device="cuda", dtype=torch.int32))
        if "p" in filters:
            s.update(top_p=0.3 + 0.7 * uniform(rows))
        if "m" in filters:
            s.update(min_p=0.1 * uniform(rows))
    return s


# ---- one pass ----

def run(s):
    return (_own if own else _plain)(s, s["case"]["kind"])


def _own(s, kind):
    import paper_1507_04296_amd as g
    case = s["case"]
    if "ctx" not in s:  # the handle that such a program keeps
        need = 0
        if kind == "norm":
            need = g.add_layernorm_workspace_bytes(case["width"])
        elif kind in ("gated", "prompt"):
            need = g.gated_scan_workspace_bytes(case["batch"], case["length"], case["channels"], backward=kind == "gated")
        s["ctx"] = _context(g, need)
    ctx = s["ctx"]
    if kind == "norm":
        y, total, mean, rstd = g.add_layernorm(ctx, s["x"], s["weight"], s["bias"], s["residual"], EPS)
        dx, dweight, dbias = g.add_layernorm_backward(ctx, s["dy"], total, mean, rstd, s["weight"], s["dtotal"])
        return dict(y=y, total=total, dx=dx, dweight=dweight, dbias=dbias)
    if kind == "adamw":
        g.adamw(ctx, s["thetas"], s["grads"], s["states"], s["clock"], RATE, BETA1, BETA2, ADAM_EPS, s["decay"], seed=7)
        values = s["states"] if case["bits"] == 32 else g.adamw_values(ctx, s["states"])
        return dict(theta=s["thetas"], m=[v[0] for v in values], v=[v[1] for v in values], clock=s["clock"])
    if kind == "sample":
        action, probability = g.sample_actions(ctx, s["values"], s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"])
        return dict(action=action, probability=probability)
    if kind == "step":
        y = g.gated_scan_step(ctx, s["x"], s["gate_a"], s["gate_x"], s["a_log"], s["state"], s["slot"], s["reset"])
        return dict(y=y, state=s["state"])
    y, state, marks = g.gated_scan(ctx, s["x"], s["gate_a"], s["gate_x"], s["a_log"], s["reset"], s["state"], marks=kind == "gated")
    if kind == "prompt":
        return dict(y=y, state=state)
    dx, dgate_a, dgate_x, da_log, dstate = g.gated_scan_backward(ctx, s["dy"], s["x"], s["gate_a"], s["gate_x"], s["a_log"], marks,
                                                                s["reset"])
    return dict(y=y, state=state, dx=dx, dgate_a=dgate_a, dgate_x=dgate_x, da_log=da_log, dstate=dstate)


_held = {}


def _context(g, need):
    """One context, with the largest workspace asked for so far."""
    ctx = _held.get("ctx")
    if ctx is None or ctx.ws_bytes < need:
        _held["ctx"] = ctx = g.Context(1, 1, min_bytes=need)
    return ctx


def _plain(s, kind):
    typ = TYPE[s["case"]["type"]]
    if kind == "adamw":
        return _plain_adamw(s)
    if kind == "sample":
        return _plain_sample(s)
    f = {k: v.float() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in s.items()}
    if kind == "norm":
        w, b = f["weight"].detach().requires_grad_(), f["bias"].detach().requires_grad_()
        total = (f["x"] + f["residual"]).to(typ)
        t = total.float().requires_grad_()
        d = t - t.mean(1, keepdim=True)
        y = d * torch.rsqrt(d.square().mean(1, keepdim=True) + EPS) * w + b
        dx, dweight, dbias = torch.autograd.grad([y, t], [t, w, b], [f["dy"], f["dtotal"]])
        return dict(y=y.detach().to(typ), total=total, dx=dx.to(typ), dweight=dweight, dbias=dbias)
    if kind == "step":
        at = s["slot"].long()
        h = _plain_gated(f["x"][:, None], f["gate_a"][:, None], f["gate_x"][:, None], f["a_log"], f["reset"][:, None], s["state"][at])
        s["state"][at] = h[:, 0]
        return dict(y=h[:, 0].to(typ), state=s["state"])
    names = ("x", "gate_a", "gate_x", "a_log", "state")
    leaves = [f[k].detach().requires_grad_(kind == "gated") for k in names]
    h = _plain_gated(*leaves[:4], f["reset"], leaves[4])
    out = dict(y=h.detach().to(typ), state=h[:, -1].detach().clone())
    if kind == "gated":
        grads = torch.autograd.grad(h, leaves, f["dy"])
        out.update(("d" + k, v.to(typ) if k in names[:3] else v) for k, v in zip(names, grads))
    return out


def _plain_gated(x, gate_a, gate_x, a_log, reset, state):
    """Every step's state: the recurrence of spans of 1, 2, 4, .. steps, joined in pairs."""
    log_a = -torch.exp(a_log) * torch.sigmoid(gate_a)
    start = reset.bool()[..., None]
    a = torch.where(start, 0.0, torch.exp(log_a))
    b = torch.where(start, 1.0, torch.sqrt(-torch.expm1(2.0 * log_a)))
    h = b * torch.sigmoid(gate_x) * x
    h = torch.cat([h[:, :1] + a[:, :1] * state[:, None], h[:, 1:]], 1)
    span = 1
    while span < x.shape[1]:  # log2(length) times
        before = (0, 0, span, 0)
        h = h + a * torch.nn.functional.pad(h[:, :-span], before)
        a = a * torch.nn.functional.pad(a[:, :-span], before)
        span *= 2
    return h


def _plain_adamw(s):
    case, clock = s["case"], s["clock"]
    t = clock[0] + 1.0
    clock.copy_(torch.stack([t, 1.0 - BETA1 ** t, 1.0 - BETA2 ** t]))
    c1, c2 = clock[1].float(), clock[2].float()
    sizes = _sizes(case)
    first = [sum(-(-n // 256) * 128 for n in sizes[:j]) for j in range(len(sizes))]
    new = [_plain_moments(case, g.float(), st, at, t) for g, st, at in zip(s["grads"], s["states"], first)]
    step = [m / c1 / (torch.sqrt(v / c2) + ADAM_EPS) for m, v, _ in new]
    [th.copy_(th - RATE * (k * th + d)) for th, k, d in zip(s["thetas"], s["decay"], step)]
    [old.copy_(now) for st, (_, _, held) in zip(s["states"], new) for old, now in zip(st, held)]
    values = [held if case["bits"] == 32 else (_plain_value(held[0] & 127, 889, held[2]) * (1.0 - 2.0 * (held[0] >> 7)), _plain_value(held[1], 761, held[3]))
              for _, _, held in new]
    return dict(theta=s["thetas"], m=[v[0] for v in values], v=[v[1] for v in values], clock=clock)


def _plain_moments(case, g, st, first, t):
    """Both averages after the step, and what is held of them."""
    m, v = st[:2] if case["bits"] == 32 else (_plain_value(st[0] & 127, 889, st[2]) * (1.0 - 2.0 * (st[0] >> 7)), _plain_value(st[1], 761, st[3]))
    m = BETA1 * m + (1.0 - BETA1) * g
    v = BETA2 * v + (1.0 - BETA2) * (g * g)
    if case["bits"] == 32:
        return m, v, (m, v)
    n = g.numel()
    bits = _plain_random(torch.arange(n, device=g.device) // 2 + first, t)
    odd = 32 * (torch.arange(n, device=g.device) % 2)
    cm, sm = _plain_codes(m.abs(), 889, (bits >> odd) & 0xffff)
    cv, sv = _plain_codes(v, 761, (bits >> (odd + 16)) & 0xffff)
    cv = torch.where(v > 0, cv.clamp(min=1), cv)  # never a division by eps alone
    return m, v, ((cm + 128 * (m < 0)).to(torch.uint8), cv.to(torch.uint8), sm, sv)


def _plain_value(code, least, scale):
    """3 bits of mantissa, the others the exponent; code 0 is zero."""
    n = code.numel()
    unit = ((code.to(torch.int32) + least) << 20).view(torch.float32)
    return torch.where(code > 0, unit, 0.0) * scale.repeat_interleave(256)[:n]


def _plain_codes(size, least, chance):
    """Codes of sizes relative to their block's largest, rounded up by chance."""
    n = size.numel()
    blocks = torch.nn.functional.pad(size, (0, -n % 256)).view(-1, 256)
    most = blocks.amax(1)
    unit = torch.where(most[:, None] > 0, blocks / most[:, None], 0.0).view(-1)[:n]
    code = ((unit.view(torch.int32) + (chance.to(torch.int32) << 4)) >> 20) - least
    return code.clamp(min=0), most


def _shift(z, n):
    """z >> n of 64 bits without a sign."""
    return (z >> n) & ((1 << (64 - n)) - 1)


def _mix(z):
    z = (z ^ _shift(z, 30)) * (0xBF58476D1CE4E5B9 - (1 << 64))
    z = (z ^ _shift(z, 27)) * (0x94D049BB133111EB - (1 << 64))
    return z ^ _shift(z, 31)


def _plain_random(place, t, seed=7):
    golden = 0x9E3779B97F4A7C15 - (1 << 64)
    return _mix(_mix(t.long() * golden + seed) + (place + 1) * golden)


def _plain_sample(s):
    v = s["values"].float()
    rows, actions = v.shape
    v = torch.where(torch.isnan(v), -math.inf, v)
    most = v.amax(1, keepdim=True)
    t = torch.ones_like(s["u"]) if s["temperature"] is None else s["temperature"]
    greedy = ~(t > 0)
    k = torch.full_like(s["u"], actions).long() if s["top_k"] is None else torch.where((s["top_k"] < 1) | (s["top_k"] > actions), actions, s["top_k"].long())
    k = torch.where(greedy, 1, k)
    z = (v.double() - most.double()) / torch.where(greedy, 1.0, t.double())[:, None]
    weight = torch.where(v == -math.inf, 0, torch.where(v == most, ONE, torch.round(torch.exp(z) * ONE).long()))
    order = torch.sort(v, dim=1, descending=True, stable=True).indices  # ties: the lowest index first
    sorted_weight = weight.gather(1, order)
    place = torch.arange(actions, device=v.device)
    sorted_weight = torch.where(place < k[:, None], sorted_weight, 0)
    before = sorted_weight.cumsum(1) - sorted_weight
    total = sorted_weight.sum(1)
    if s["top_p"] is not None:
        limit = torch.where(s["top_p"] < 1, torch.ceil(s["top_p"].double() * total.double()).long().clamp(min=1), total)
        sorted_weight = torch.where(before < limit[:, None], sorted_weight, 0)
    if s["min_p"] is not None:
        least = torch.ceil(s["min_p"].double().clamp(0, 1) * ONE).long()
        sorted_weight = torch.where(sorted_weight >= least[:, None], sorted_weight, 0)
    kept = torch.zeros_like(weight).scatter_(1, order, sorted_weight)
    total = kept.sum(1)
    at = torch.minimum((s["u"].double() * total.double()).long(), total - 1)
    action = (kept.cumsum(1) <= at[:, None]).sum(1)
    some = total > 0
    chosen = kept.gather(1, torch.where(some, action, 0)[:, None])[:, 0]
    return dict(action=torch.where(some, action, -1).to(torch.int32),
                probability=torch.where(some, chosen.double() / total.double(), 0.0).float())


# ---- what one pass cannot do without ----

def work(case):
    kind, e = case["kind"], SIZE[case["type"]]
    if kind == "norm":  # x, residual, dy, dtotal in; y, total, dx out
        n = case["rows"] * case["width"]
        return dict(bytes=7 * e * n + 16 * case["width"], flops=22 * n)
    if kind == "step":  # x, both gates in, y out; the states of the rows in and out
        n = case["rows"] * case["channels"]
        return dict(bytes=(4 * e + 8) * n + 4 * case["channels"], flops=40 * n)
    if kind in ("gated", "prompt"):  # x, both gates in, y out; dy in, three gradients out
        n = case["batch"] * case["length"] * case["channels"]
        states = case["batch"] * case["channels"] * (12 if kind == "gated" else 8)
        return dict(bytes=(8 if kind == "gated" else 4) * e * n + states + 8 * case["channels"], flops=(100 if kind == "gated" else 40) * n)
    if kind == "adamw":  # theta and both averages in and out, the gradient in; 8 bits: the values they stand for out
        n = sum(_sizes(case))
        return dict(bytes=n * (8 + e + (16 if case["bits"] == 32 else 4 + 8)), flops=n * (18 if case["bits"] == 32 else 60))
    n = case["rows"] * case["actions"]
    return dict(bytes=e * n + case["rows"] * (12 + 4 * len(case["filters"])), flops=30 * n)


# ---- the definitions in 64 bits ----

def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "adamw":
        return _exact_adamw(s)
    if kind == "sample":
        return _exact_sample(s)
    f = {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in s.items()}
    if kind == "norm":
        total = f["x"] + f["residual"]
        t = total.to(TYPE[case["type"]]).double()  # the stream holds the rounded sum
        width = t.shape[1]
        t = t - t.sum(1, keepdim=True) / width
        xh = t / torch.sqrt((t * t).sum(1, keepdim=True) / width + EPS)
        rho = 1.0 / torch.sqrt((t * t).sum(1, keepdim=True) / width + EPS)
        g = f["dy"] * f["weight"]
        dx = f["dtotal"] + rho * (g - g.sum(1, keepdim=True) / width - xh * ((g * xh).sum(1, keepdim=True) / width))
        return dict(y=xh * f["weight"] + f["bias"], total=total, dx=dx, dweight=(f["dy"] * xh).sum(0), dbias=f["dy"].sum(0))
    if kind == "step":
        at = s["slot"].long()
        got = _exact_gated(dict({k: f[k][:, None] for k in ("x", "gate_a", "gate_x")}, reset=s["reset"][:, None], a_log=f["a_log"],
                                state=f["state"][at]))
        f["state"][at] = got["state"]
        return dict(y=got["y"][:, 0], state=f["state"])
    return _exact_gated(f)


def _exact_gated(f):
    x, h = f["x"], f["state"]
    rate = torch.exp(f["a_log"])
    r, i = 1.0 / (1.0 + torch.exp(-f["gate_a"])), 1.0 / (1.0 + torch.exp(-f["gate_x"]))
    log_a = -rate * r
    go = 1.0 - f["reset"].double()[..., None]
    a = torch.exp(log_a) * go
    b = torch.sqrt(-torch.expm1(2.0 * log_a)) * go + (1.0 - go)
    y = torch.empty_like(x)
    before = torch.empty_like(x) if "dy" in f else None
    for t in range(x.shape[1]):
        if before is not None:
            before[:, t] = h
        h = a[:, t] * h + b[:, t] * (i[:, t] * x[:, t])
        y[:, t] = h
    out = dict(y=y, state=h)
    if before is None:
        return out
    back, back_all = torch.zeros_like(h), torch.empty_like(x)
    for t in range(x.shape[1] - 1, -1, -1):
        back = back + f["dy"][:, t]
        back_all[:, t] = back
        back = a[:, t] * back
    dlog = (back_all * a * before - back_all * i * x * a * a / b) * go  # at a start b is 1 whatever the gate
    da_log = dlog * log_a
    return dict(out, dx=back_all * b * i, dgate_a=da_log * (1.0 - r), dgate_x=back_all * b * x * i * (1.0 - i),
                da_log=da_log.sum((0, 1)), dstate=back)


def _exact_adamw(s):
    case, sizes = s["case"], _sizes(s["case"])
    t = int(s["clock"][0]) + 1
    c1, c2 = 1 - BETA1 ** t, 1 - BETA2 ** t
    out = dict(theta=[], m=[], v=[], clock=torch.tensor([t, c1, c2], dtype=torch.float64))
    place = 0
    for j, n in enumerate(sizes):
        g, theta, st = s["grads"][j].double(), s["thetas"][j].double(), s["states"][j]
        block = torch.arange(n, device=g.device) // 256
        if case["bits"] == 32:
            m, v = st[0].double(), st[1].double()
        else:  # held values are a code's times the scale, rounded to 32 bits
            low = (st[0] % 128).long()
            m = torch.where(low > 0, (8 + (low + 1) % 8).double() * 2.0 ** ((low + 889) // 8 - 130).double(), 0.0)
            high = st[1].long()
            v = torch.where(high > 0, (8 + (high + 1) % 8).double() * 2.0 ** ((high + 761) // 8 - 130).double(), 0.0)
            m = (m * st[2].double()[block]).float().double() * torch.where(st[0] >= 128, -1.0, 1.0)
            v = (v * st[3].double()[block]).float().double()
        m1, v1 = BETA1 * m + (1 - BETA1) * g, BETA2 * v + (1 - BETA2) * g * g
        out["theta"].append(theta - RATE * (s["decay"][j] * theta + m1 / c1 / (torch.sqrt(v1 / c2) + ADAM_EPS)))
        if case["bits"] == 8:  # the codes' definition has its roundings to 32 bits: each product, square and sum
            def r32(z):
                return z.float().double()

            b1, b2, o1, o2 = (float(np.float32(z)) for z in (BETA1, BETA2, 1 - BETA1, 1 - BETA2))
            m1 = r32(r32(b1 * m) + r32(o1 * g))
            v1 = r32(r32(b2 * v) + r32(o2 * r32(g * g)))
            e = np.arange(n, dtype=np.uint64)
            z = _exact_mix(e // np.uint64(2) + np.uint64(place), t)
            half = (z >> (np.uint64(32) * (e % np.uint64(2)))) & np.uint64(0xffffffff)
            chance = [torch.from_numpy(c.astype(np.int64)).to(g.device) for c in (half & np.uint64(0xffff), half >> np.uint64(16))]
            m1 = _exact_held(m1.abs(), block, chance[0], 127, False) * torch.sign(m1)
            v1 = _exact_held(v1, block, chance[1], 255, True)
        out["m"].append(m1)
        out["v"].append(v1)
        place += -(-n // 256) * 128
    return out


def _exact_mix(place, t, seed=7):
    with np.errstate(over="ignore"):
        def mix(z):
            z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
            z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
            return z ^ (z >> np.uint64(31))
        golden = np.uint64(0x9E3779B97F4A7C15)
        key = mix(np.array([t], dtype=np.uint64) * golden + np.uint64(seed))
        return mix(key + (place + np.uint64(1)) * golden)


def _exact_held(size, block, chance, last, floor):
    """What a size is held as: 8 values a power of two below the block's largest, `last` of them."""
    most = torch.zeros(int(block[-1]) + 1, dtype=torch.float64, device=size.device).scatter_reduce(0, block, size, "amax")[block]
    unit = torch.where(most > 0, (size / most).float().double(), 0.0)
    exponent = torch.floor(torch.log2(unit.clamp(min=2.0 ** -140)))
    exponent = torch.where(2.0 ** exponent > unit, exponent - 1, exponent)
    exponent = torch.where(2.0 ** (exponent + 1) <= unit, exponent + 1, exponent)
    eighths = unit / 2.0 ** (exponent - 3)  # 8 .. 16
    up = torch.floor((eighths - torch.floor(eighths)) * 2 ** 20 + chance.double() * 16 + 0.0) >= 2 ** 20
    code = last + 8 * exponent + torch.floor(eighths) - 8 + up
    code = torch.where(unit > 0, code, 0.0).clamp(min=0.0)
    if floor:
        code = torch.where(size > 0, code.clamp(min=1.0), code)
    whole = code - last + 8000  # 8000 stands for 1
    value = (8 + whole % 8) * 2.0 ** (torch.floor(whole / 8) - 1003)
    return torch.where(code > 0, value * most, 0.0)


def _exact_sample(s):
    v = s["values"].double().cpu().numpy()
    rows, actions = v.shape
    host = {k: None if s[k] is None else s[k].double().cpu().numpy() for k in ("u", "temperature", "top_k", "top_p", "min_p")}
    action, probability = np.full(rows, -1, dtype=np.int32), np.zeros(rows)
    for n in range(rows):
        get = lambda k, usual: usual if host[k] is None else float(host[k][n])
        t, best = get("temperature", 1.0), v[n].max()
        rank = np.lexsort((np.arange(actions), -v[n]))
        weights = np.rint(np.exp((v[n][rank] - best) / (t if t > 0 else 1.0)) * ONE).astype(np.int64)
        keep = weights.copy()
        k = 1 if t <= 0 else int(get("top_k", actions))
        keep[k if 1 <= k <= actions else actions:] = 0
        total = int(keep.sum())
        p = get("top_p", 1.0)
        if p < 1:
            before = np.concatenate([[0], np.cumsum(keep)[:-1]])
            keep[before >= max(1, math.ceil(p * float(total)))] = 0
        keep[keep < math.ceil(get("min_p", 0.0) * ONE)] = 0
        by_index = np.zeros(actions, dtype=np.int64)
        by_index[rank] = keep
        total = int(keep.sum())
        at = min(int(host["u"][n] * float(total)), total - 1)
        action[n] = int(np.searchsorted(np.cumsum(by_index), at, side="right"))
        probability[n] = by_index[action[n]] / total
    return dict(action=torch.from_numpy(action), probability=torch.from_numpy(probability))
