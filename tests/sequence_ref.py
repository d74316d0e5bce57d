"""The sequence operators' definitions in 64 bits on the CPU, step by step, for the
tests (no code of the library).  Inputs are any float tensors; outputs float64."""
import torch


def d64(*ts):
    return tuple(None if t is None else t.detach().cpu().double() if t.is_floating_point() else t.detach().cpu() for t in ts)


def norm(total, weight, eps):
    total, weight = d64(total, weight)
    rho = (total.pow(2).mean(1) + eps).rsqrt()
    return total * rho[:, None] * weight, rho


def norm_backward(dy, total, weight, eps, dtotal=None):
    dy, total, weight, dtotal = d64(dy, total, weight, dtotal)
    rho = (total.pow(2).mean(1) + eps).rsqrt()[:, None]
    g = dy * weight
    dx = rho * g - total * rho ** 3 * (g * total).mean(1, keepdim=True)
    return dx if dtotal is None else dx + dtotal, (dy * total * rho).sum(0)


def conv(x, weight, bias=None, reset=None, window=None, silu=True):
    """y, v, the window behind, and used[b][t][j]: the value that tap j multiplied (0 where it is cut)."""
    x, weight, bias, reset, window = d64(x, weight, bias, reset, window)
    B, T, C = x.shape
    K = weight.shape[1]
    v, used = torch.zeros_like(x), torch.zeros(B, T, K, C, dtype=torch.float64)
    behind = torch.zeros(B, K - 1, C, dtype=torch.float64)
    for b in range(B):
        past = [torch.zeros(C, dtype=torch.float64) if window is None else window[b, j] for j in range(K - 1)]
        for t in range(T):
            if reset is not None and reset[b, t]:
                past = [torch.zeros(C, dtype=torch.float64)] * (K - 1)
            past = past[-(K - 1):] + [x[b, t]]
            for j in range(K):
                used[b, t, j] = past[j]
            v[b, t] = sum((weight[:, j] * past[j] for j in range(K)), torch.zeros(C, dtype=torch.float64))
            if bias is not None:
                v[b, t] += bias
        for j in range(K - 1):
            behind[b, j] = past[len(past) - (K - 1) + j]
    return (v * torch.sigmoid(v) if silu else v), v, behind, used


def conv_backward(dy, x, weight, bias=None, reset=None, window=None, silu=True, dbehind=None):
    dy, x, weight, bias, reset, window, dbehind = d64(dy, x, weight, bias, reset, window, dbehind)
    _, v, _, used = conv(x, weight, bias, reset, window, silu)
    B, T, C = x.shape
    K = weight.shape[1]
    s = torch.sigmoid(v)
    dv = dy * (s * (1 + v * (1 - s))) if silu else dy
    de = torch.zeros(B, T + K - 1, C, dtype=torch.float64)
    dw = torch.zeros_like(weight)
    for b in range(B):
        for t in range(T):
            for j in range(K):
                at = t - (K - 1) + j
                if reset is not None and reset[b, max(0, at + 1):t + 1].any():
                    continue
                de[b, at + K - 1] += weight[:, j] * dv[b, t]
                dw[:, j] += dv[b, t] * used[b, t, j]
        if dbehind is not None:
            for j in range(K - 1):
                at = T - (K - 1) + j
                if reset is None or not reset[b, max(0, at + 1):].any():
                    de[b, at + K - 1] += dbehind[b, j]
    return de[:, K - 1:], dw, dv.sum((0, 1)), de[:, :K - 1]


def steps(dt, a_log, dt_bias, reset):
    pre = dt + dt_bias
    d = torch.where(pre > 0, pre, torch.zeros_like(pre)) + torch.log1p(torch.exp(-pre.abs()))
    d = torch.where(pre.isnan(), pre, d)
    a = torch.exp(-torch.exp(a_log) * d)
    return pre, d, a


def scan(x, dt, b, c, a_log, dt_bias, skip, reset=None, state=None, keep=False):
    x, dt, b, c, a_log, dt_bias, skip, reset, state = d64(x, dt, b, c, a_log, dt_bias, skip, reset, state)
    B, T, H, P = x.shape
    G, N = b.shape[2:]
    of = [h * G // H for h in range(H)]
    _, d, a = steps(dt, a_log, dt_bias, reset)
    S = torch.zeros(B, H, P, N, dtype=torch.float64) if state is None else state.clone()
    y, before = torch.zeros_like(x), []
    for t in range(T):
        if reset is not None:
            S = torch.where(reset[:, t].bool()[:, None, None, None], torch.zeros_like(S), S)
        before.append(S)
        S = a[:, t, :, None, None] * S if reset is None else torch.where(
            reset[:, t].bool()[:, None, None, None], S, a[:, t, :, None, None] * S)
        S = S + (d[:, t, :, None] * x[:, t])[..., None] * b[:, t, of][:, :, None]
        y[:, t] = (S * c[:, t, of][:, :, None]).sum(-1) + skip[:, None] * x[:, t]
    return (y, S, before) if keep else (y, S)


def scan_backward(dy, x, dt, b, c, a_log, dt_bias, skip, reset=None, state=None, dstate=None):
    dy, x, dt, b, c, a_log, dt_bias, skip, reset, state, dstate = d64(dy, x, dt, b, c, a_log, dt_bias, skip, reset, state, dstate)
    _, _, before = scan(x, dt, b, c, a_log, dt_bias, skip, reset, state, keep=True)
    B, T, H, P = x.shape
    G, N = b.shape[2:]
    of = [h * G // H for h in range(H)]
    pre, d, a = steps(dt, a_log, dt_bias, reset)
    A = -torch.exp(a_log)
    R = torch.zeros(B, H, P, N, dtype=torch.float64) if dstate is None else dstate.clone()
    dx, dd, db, dc, dA = torch.zeros_like(x), torch.zeros_like(d), torch.zeros_like(b), torch.zeros_like(c), torch.zeros(H).double()
    for t in reversed(range(T)):
        bt, ct = b[:, t, of], c[:, t, of]
        start = torch.zeros(B, dtype=torch.bool) if reset is None else reset[:, t].bool()
        start = start[:, None, None, None]
        at = torch.where(start, torch.zeros_like(R), a[:, t, :, None, None] * before[t])  # what the step kept
        S = at + (d[:, t, :, None] * x[:, t])[..., None] * bt[:, :, None]
        R = R + dy[:, t][..., None] * ct[:, :, None]
        dch, dv = (S * dy[:, t][..., None]).sum(2), (R * bt[:, :, None]).sum(3)
        dbh = (R * (d[:, t, :, None] * x[:, t])[..., None]).sum(2)
        for h in range(H):
            dc[:, t, of[h]] += dch[:, h]
            db[:, t, of[h]] += dbh[:, h]
        dlog = torch.where(start, torch.zeros_like(R), R * at).sum((2, 3))
        dA += (dlog * torch.where(start[:, :, 0, 0], torch.zeros_like(d[:, t]), d[:, t])).sum(0)
        dd[:, t] = (dv * x[:, t]).sum(2) + torch.where(start[:, :, 0, 0], torch.zeros_like(dlog), dlog * A)
        dx[:, t] = d[:, t, :, None] * dv + skip[:, None] * dy[:, t]
        R = torch.where(start, torch.zeros_like(R), a[:, t, :, None, None] * R)
    ddt = dd * torch.sigmoid(pre)
    return dict(dx=dx, ddt=ddt, db=db, dc=dc, da_log=dA * A, ddt_bias=ddt.sum((0, 1)), dskip=(dy * x).sum((0, 1, 3)), dstate=R)


def weights(codes, scales, inputs, group):
    """[outputs, inputs] that 4-bit codes stand for."""
    codes, scales = codes.cpu().long(), scales.cpu().double()
    w = torch.stack((codes % 16, codes // 16), 2).flatten(1)[:, :inputs].double() - 8
    return w * scales[:, torch.arange(inputs) // group]
