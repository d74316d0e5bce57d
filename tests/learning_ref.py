"""Definitions of the layer norm, the gated scan, AdamW and sampled actions in 64 bits on
the CPU, for the tests (no code of the library).  Gradients are those of automatic
differentiation of the same formulas in 64 bits."""
import math

import numpy as np
import torch

from sequence_ref import d64


def layernorm(total, weight, bias, eps):
    total, weight, bias = d64(total, weight, bias)
    mean = total.mean(1, keepdim=True)
    rho = ((total - mean).pow(2).mean(1, keepdim=True) + eps).rsqrt()
    y = (total - mean) * rho * weight
    return (y if bias is None else y + bias), mean[:, 0], rho[:, 0]


def layernorm_backward(dy, total, weight, eps, dtotal=None):
    dy, total, weight, dtotal = d64(dy, total, weight, dtotal)
    leaves = [v.clone().requires_grad_() for v in (total, weight, torch.zeros_like(weight))]
    y, _, _ = layernorm_leaves(*leaves, eps)
    dx, dw, db = torch.autograd.grad(y, leaves, dy)
    return (dx if dtotal is None else dx + dtotal), dw, db


def layernorm_leaves(total, weight, bias, eps):
    mean = total.mean(1, keepdim=True)
    rho = ((total - mean).pow(2).mean(1, keepdim=True) + eps).rsqrt()
    return (total - mean) * rho * weight + bias, mean, rho


def gated_leaves(x, gate_a, gate_x, a_log, reset, state):
    """y and every step's state before it, in the type of the arguments."""
    h, y, before = state, [], []
    log_a = -torch.exp(a_log).clamp(max=2.0 ** 127) * torch.sigmoid(gate_a)
    for t in range(x.shape[1]):
        before.append(h)
        u = torch.sigmoid(gate_x[:, t]) * x[:, t]
        now = torch.exp(log_a[:, t]) * h + torch.sqrt(-torch.expm1(2 * log_a[:, t])) * u
        h = now if reset is None else torch.where(reset[:, t].bool()[:, None], u, now)
        y.append(h)
    if not y:
        return torch.zeros_like(x), h, before
    return torch.stack(y, 1), h, before


def gated(x, gate_a, gate_x, a_log, reset=None, state=None):
    x, gate_a, gate_x, a_log, reset, state = d64(x, gate_a, gate_x, a_log, reset, state)
    if state is None:
        state = torch.zeros(x.shape[0], x.shape[2], dtype=torch.float64)
    return gated_leaves(x, gate_a, gate_x, a_log, reset, state)


def gated_backward(dy, x, gate_a, gate_x, a_log, reset=None, state=None, dstate=None):
    dy, x, gate_a, gate_x, a_log, reset, state, dstate = d64(dy, x, gate_a, gate_x, a_log, reset, state, dstate)
    if state is None:
        state = torch.zeros(x.shape[0], x.shape[2], dtype=torch.float64)
    leaves = [v.clone().requires_grad_() for v in (x, gate_a, gate_x, a_log, state)]
    y, h, _ = gated_leaves(*leaves[:4], reset, leaves[4])
    out = (y * dy).sum() + (0 if dstate is None else (h * dstate).sum())
    return torch.autograd.grad(out, leaves)


# ---- AdamW: numpy's float32 operations are rounded once each, as the definition's ----

LEAST = dict(m=889, v=761)


def held(code, least, scale):
    code = code.astype(np.int64)
    unit = ((code + least) << 20).astype(np.uint32).view(np.float32)
    return np.where(code > 0, unit, np.float32(0)) * scale


def mix(z):
    with np.errstate(over="ignore"):
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        return z ^ (z >> np.uint64(31))


def chances(n, place, seed, t):
    """The 16 bits of m and of v for every element."""
    with np.errstate(over="ignore"):
        golden, e = np.uint64(0x9E3779B97F4A7C15), np.arange(n, dtype=np.uint64)
        key = mix(np.array([seed], dtype=np.uint64) + np.array([t], dtype=np.uint64) * golden)
        z = mix(key + (np.uint64(place) + e // np.uint64(2) + np.uint64(1)) * golden)
    z = z >> (np.uint64(32) * (e % np.uint64(2)))
    return ((z & np.uint64(0xffff)).astype(np.int64), (z >> np.uint64(16) & np.uint64(0xffff)).astype(np.int64))


def hold(size, chance, least):
    """Codes and scales of sizes (float32, not negative)."""
    n, groups = size.size, -(-size.size // 256)
    code, scale = np.zeros(n, dtype=np.int64), np.zeros(groups, dtype=np.float32)
    for b in range(groups):
        at = slice(256 * b, min(n, 256 * b + 256))
        if not np.isfinite(size[at]).all():
            scale[b] = np.nan
            continue
        scale[b] = size[at].max()
        if scale[b] > 0:
            bits = (size[at] / scale[b]).astype(np.float32).view(np.uint32).astype(np.int64)
            code[at] = np.maximum((bits + 16 * chance[at] >> 20) - least, 0)
    return code, scale


def adamw(theta, grad, state, t, place, lr, beta1, beta2, eps, decay, seed):
    """theta' (float64) and the new state as numpy arrays; state: (m, v) or (m, v, m_scale, v_scale)."""
    f = np.float32
    theta, grad = theta.detach().cpu().double().numpy().reshape(-1), grad.detach().cpu().float().numpy().reshape(-1)
    s = [v.detach().cpu().numpy().reshape(-1) for v in state]
    n = grad.size
    with np.errstate(all="ignore"):
        if len(s) == 2:
            m, v = s
        else:
            m = held(s[0] & 127, LEAST["m"], s[2].repeat(256)[:n]) * np.where(s[0] >= 128, f(-1), f(1))
            v = held(s[1], LEAST["v"], s[3].repeat(256)[:n])
        m = f(beta1) * m + f(1 - beta1) * grad
        v = f(beta2) * v + f(1 - beta2) * (grad * grad)
        assert m.dtype == v.dtype == np.float32
        step = (m.astype(np.float64) / (1 - beta1 ** t)) / (np.sqrt(v.astype(np.float64) / (1 - beta2 ** t)) + eps)
        new = theta - lr * (decay * theta + step)
        if len(s) == 2:
            return new, (m, v)
        cm, cv = chances(n, place, seed, t)
        a, sa = hold(np.abs(m), cm, LEAST["m"])
        b, sb = hold(v, cv, LEAST["v"])
        b = np.where((v > 0) & np.isfinite(sb.repeat(256)[:n]), np.maximum(b, 1), b)
        a = np.where((m < 0) & np.isfinite(sa.repeat(256)[:n]), a + 128, a)
        return new, (a.astype(np.uint8), b.astype(np.uint8), sa, sb)


# ---- sampled actions ----

ONE = 1 << 40


def weights(v, temperature):
    """Whole weights of one row (float64, NaN already -inf), and the greedy flag."""
    greedy = not temperature > 0
    most = v.max()
    with np.errstate(all="ignore"):
        x = np.exp((v - most) / (1.0 if greedy else temperature)) * ONE
    x[v == -np.inf] = 0
    if most == np.inf:
        x[:] = 0
    x[v == most] = ONE
    return [int(w) for w in np.rint(x)], greedy


def sample(values, u, temperature=None, top_k=None, top_p=None, min_p=None):
    v = values.detach().cpu().double().numpy().copy()
    v[np.isnan(v)] = -np.inf
    rows, n = v.shape
    get = lambda t, i, usual: usual if t is None else float(t[i].cpu().double())
    action, probability = np.full(rows, -1, dtype=np.int32), np.zeros(rows)
    for i in range(rows):
        if v[i].max() == -np.inf:
            continue
        w, greedy = weights(v[i], get(temperature, i, 1.0))
        order = sorted(range(n), key=lambda j: (-v[i][j], j))
        k = n if top_k is None else int(top_k[i])
        k = 1 if greedy else k if 1 <= k <= n else n
        stay = order[:k]
        p = get(top_p, i, 1.0)
        if p < 1:
            sum_k = sum(w[j] for j in stay)
            limit = max(1, math.ceil(p * float(sum_k)) if p > 0 else 0)
            before, some = 0, []
            for j in stay:
                if before < limit:
                    some.append(j)
                before += w[j]
            stay = some
        m = get(min_p, i, 0.0)
        least = math.ceil(min(m, 1.0) * ONE) if m > 0 else 0
        kept = [0] * n
        for j in stay:
            kept[j] = w[j] if w[j] >= least else 0
        total = sum(kept)
        x = float(u[i])
        at = 0 if not x > 0 else total - 1 if x >= 1 else min(int(x * float(total)), total - 1)
        run = 0
        for j in range(n):
            run += kept[j]
            if run > at:
                action[i], probability[i] = j, kept[j] / total
                break
    return torch.from_numpy(action), torch.from_numpy(probability)
