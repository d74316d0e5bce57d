"""A recurrent Q-head on feature rows, made of the sequence operators: the learner's pass
over replayed sequences with its gradients, and the actors' single steps on a replica
with 4-bit weights.  The rows are the caller's, and so is what `backward` returns for
them: the library's forward calls give Q values and actions, not the network's features.

    y = norm(f);  (x, B, C, dt) = W_in y;  (x, B, C) = conv(x, B, C)
    s = scan(x, dt, B, C);  u = W_out s;  h = norm(f + u);  Q = W_q h

``python -m paper_1507_04296_amd.recurrent`` trains it on a game of memory (a cue is
seen in an episode's first step, the right action is the cue's in all of them), applies
the gradients as the parameter server does, and plays with a replica.
"""
from __future__ import annotations

import argparse
import math

import torch

from . import (Context, add_rmsnorm, add_rmsnorm_backward, add_rmsnorm_codes, add_rmsnorm_workspace_bytes, causal_conv,
               causal_conv_backward, causal_conv_step, causal_conv_workspace_bytes, gorila_ps_apply, qmatvec,
               quantize_weights, scan, scan_backward, scan_step, scan_workspace_bytes)


class RecurrentCore:
    """Sizes and parameters.  `theta` is one flat float32 vector (gradients are laid out
    the same, so that the parameter server's calls take both) and `params` its views."""

    def __init__(self, actions: int, features: int = 512, heads: int = 16, head_dim: int = 64, groups: int = 1,
                 state_dim: int = 64, taps: int = 4, device=None, seed: int = 0):
        self.actions, self.features, self.taps = actions, features, taps
        self.heads, self.head_dim, self.groups, self.state_dim = heads, head_dim, groups, state_dim
        self.inner = heads * head_dim
        self.channels = self.inner + 2 * groups * state_dim  # of the convolution: x, B and C
        self.shapes = dict(norm_in=(features,), w_in=(self.channels + heads, features), conv=(self.channels, taps),
                           conv_bias=(self.channels,), a_log=(heads,), dt_bias=(heads,), skip=(heads,),
                           w_out=(features, self.inner), norm_out=(features,), w_q=(actions, features))
        size = sum(-(-math.prod(s) // 4) * 4 for s in self.shapes.values())
        self.theta = torch.zeros(size, dtype=torch.float32, device=device if device is not None else "cuda")
        self.params = self.views(self.theta)
        gen = torch.Generator().manual_seed(seed)
        uniform = lambda *s: torch.rand(s, generator=gen)
        p = self.params
        for name in ("w_in", "conv", "w_out", "w_q"):
            p[name].copy_(torch.randn(self.shapes[name], generator=gen) / math.sqrt(self.shapes[name][1]))
        for name in ("norm_in", "norm_out", "skip"):
            p[name].fill_(1.0)
        step = torch.exp(math.log(1e-3) + math.log(100.0) * uniform(heads))  # softplus(dt_bias): 0.001 .. 0.1
        p["dt_bias"].copy_(step + torch.log(-torch.expm1(-step)))
        p["a_log"].copy_(torch.log(1.0 + 15.0 * uniform(heads)))

    def views(self, flat) -> dict:
        """The parameters' (or gradients') views of a flat vector, each on 16 bytes."""
        out, at = {}, 0
        for name, shape in self.shapes.items():
            n = math.prod(shape)
            out[name] = flat[at:at + n].view(shape)
            at += -(-n // 4) * 4
        return out

    def workspace_bytes(self, batch: int, length: int, backward: bool = True) -> int:
        """What a Context needs for forward (and backward) of up to [batch, length] steps."""
        return max(scan_workspace_bytes(batch, length, self.heads, self.head_dim, self.groups, self.state_dim, backward),
                   causal_conv_workspace_bytes(self.channels, self.taps), add_rmsnorm_workspace_bytes(self.features))

    def _split(self, v):
        """x, B and C of the convolution's channels, as the scan takes them."""
        n = self.groups * self.state_dim
        return (v[..., :self.inner].unflatten(-1, (self.heads, self.head_dim)),
                v[..., self.inner:self.inner + n].unflatten(-1, (self.groups, self.state_dim)),
                v[..., self.inner + n:self.channels].unflatten(-1, (self.groups, self.state_dim)))

    def forward(self, ctx, features, reset=None, carried=None):
        """Q [batch, length, actions] of features [batch, length, features], what the next
        steps need (window, state), and what the backward needs.  reset uint8
        [batch, length]: 1 where an episode starts."""
        p, (B, T, F) = self.params, features.shape
        window, state = carried if carried is not None else (None, None)
        f = features.reshape(B * T, F)
        y, _, rstd = add_rmsnorm(ctx, f, p["norm_in"])
        z = (y @ p["w_in"].T).view(B, T, -1)
        zc, dt = z[..., :self.channels], z[..., self.channels:]
        v, window_out = causal_conv(ctx, zc, p["conv"], p["conv_bias"], reset, window)
        x, b, c = self._split(v)
        s, state_out = scan(ctx, x, dt, b, c, p["a_log"], p["dt_bias"], p["skip"], reset, state)
        s = s.view(B * T, self.inner)
        h, total, rstd_out = add_rmsnorm(ctx, s @ p["w_out"].T, p["norm_out"], residual=f)
        q = (h @ p["w_q"].T).view(B, T, self.actions)
        return q, (window_out, state_out), (f, y, rstd, zc, dt, v, s, h, total, rstd_out, reset, window, state)

    def backward(self, ctx, dq, saved):
        """Gradients of every parameter, flat as theta is, and of the features.  What was
        carried into the sequence is taken as given (no gradient)."""
        f, y, rstd, zc, dt, v, s, h, total, rstd_out, reset, window, state = saved
        (B, T, _), p = dq.shape, self.params
        grad = torch.zeros_like(self.theta)
        g = self.views(grad)
        dq = dq.reshape(B * T, self.actions)
        torch.mm(dq.T, h, out=g["w_q"])
        df, dw = add_rmsnorm_backward(ctx, dq @ p["w_q"], total, rstd_out, p["norm_out"])
        g["norm_out"].copy_(dw)
        torch.mm(df.T, s, out=g["w_out"])
        ds = (df @ p["w_out"]).view(B, T, self.heads, self.head_dim)
        x, b, c = self._split(v)
        dx, ddt, db, dc, da_log, ddt_bias, dskip, _ = scan_backward(
            ctx, ds, x, dt, b, c, p["a_log"], p["dt_bias"], p["skip"], reset, state)
        dv = torch.cat([dx.flatten(2), db.flatten(2), dc.flatten(2)], dim=2)
        dzc, dconv, dbias, _ = causal_conv_backward(ctx, dv, zc, p["conv"], p["conv_bias"], reset, window)
        dz = torch.cat([dzc, ddt], dim=2).view(B * T, -1)
        for name, value in dict(a_log=da_log, dt_bias=ddt_bias, skip=dskip, conv=dconv, conv_bias=dbias).items():
            g[name].copy_(value)
        torch.mm(dz.T, y, out=g["w_in"])
        dfeatures, dw = add_rmsnorm_backward(ctx, dz @ p["w_in"], f, rstd, p["norm_in"], dtotal=df)
        g["norm_in"].copy_(dw)
        return grad, dfeatures.view(B, T, -1)


class Replica:
    """An actor's copy of a core: 4-bit matrices, and a window and a state for each of
    `slots` environments, held on the GPU and updated by every step."""

    GROUP = 64  # weights that share a scale

    def __init__(self, core: RecurrentCore, slots: int):
        self.core = core
        dev = core.theta.device
        self.windows = torch.zeros((slots, core.taps - 1, core.channels), dtype=torch.float32, device=dev)
        self.states = torch.zeros((slots, core.heads, core.head_dim, core.state_dim), dtype=torch.float32, device=dev)

    def pull(self, ctx) -> None:
        """Takes the core's present parameters."""
        c = self.core
        self.params = {n: c.params[n].clone() for n in ("norm_in", "norm_out", "conv", "conv_bias", "a_log", "dt_bias", "skip")}
        self.weights = {n: quantize_weights(ctx, c.params[n], self.GROUP) for n in ("w_in", "w_out", "w_q")}

    def step(self, ctx, features, slot=None, reset=None):
        """Q [rows, actions] of one step of every row of features [rows, features].  slot
        int32 [rows]: the rows' environments (None: row i's is i); reset uint8 [rows]: 1
        where the step starts an episode."""
        core, p, w = self.core, self.params, self.weights
        codes, scale, _ = add_rmsnorm_codes(ctx, features, p["norm_in"])
        z = qmatvec(ctx, codes, *w["w_in"], self.GROUP, scale)
        v = causal_conv_step(ctx, z[:, :core.channels], self.windows, p["conv"], p["conv_bias"], slot, reset)
        x, b, c = core._split(v)
        s = scan_step(ctx, x, z[:, core.channels:], b, c, p["a_log"], p["dt_bias"], p["skip"], self.states, slot, reset)
        u = qmatvec(ctx, s.flatten(1), *w["w_out"], self.GROUP)
        codes, scale, _ = add_rmsnorm_codes(ctx, u, p["norm_out"], residual=features)
        return qmatvec(ctx, codes, *w["w_q"], self.GROUP, scale)


def memory_game(core, gen, batch: int, length: int, episode: int):
    """features, reset and cue [batch, length] of episodes of `episode` steps each."""
    dev = core.theta.device
    starts = torch.arange(length, device=dev) % episode == 0
    cue = torch.randint(0, core.actions, (batch, -(-length // episode)), generator=gen, device=dev)
    cue = cue.repeat_interleave(episode, dim=1)[:, :length]
    features = torch.randn((batch, length, core.features), generator=gen, device=dev)
    marks = torch.zeros((core.actions, core.features), device=dev)
    marks[torch.arange(core.actions), torch.arange(core.actions)] = 0.3 * core.features ** 0.5
    features = features + marks[cue] * starts[None, :, None]
    return features, starts.to(torch.uint8).expand(batch, length).contiguous(), cue


def train(core, ctx, updates: int, batch: int = 32, length: int = 128, episode: int = 16, lr: float = 0.03, seed: int = 0):
    """Random actions; a step's reward is 1 for the cue's action.  The mean Huber loss of
    each update, and theta is updated in place by the parameter server's call."""
    dev = core.theta.device
    gen = torch.Generator(device=dev).manual_seed(seed)
    accum, applied = torch.zeros_like(core.theta), torch.zeros(1, dtype=torch.uint8, device=dev)
    version, now = torch.zeros(1, dtype=torch.int64, device=dev), torch.zeros(1, dtype=torch.int64, device=dev)
    losses = []
    for _ in range(updates):
        features, reset, cue = memory_game(core, gen, batch, length, episode)
        action = torch.randint(0, core.actions, cue.shape, generator=gen, device=dev)
        q, _, saved = core.forward(ctx, features, reset)
        delta = q.gather(2, action[..., None])[..., 0] - (action == cue).float()
        dq = torch.zeros_like(q).scatter_(2, action[..., None], (delta.clamp(-1, 1) / delta.numel())[..., None])
        grad, _ = core.backward(ctx, dq, saved)
        version.copy_(now)
        gorila_ps_apply(ctx, core.theta, accum, grad[None], version, now, 0, lr, 1e-8, applied)
        size = delta.abs()
        losses.append(torch.where(size <= 1, 0.5 * size * size, size - 0.5).mean())
    return torch.stack(losses).cpu()


def play(core, ctx, environments: int = 256, steps: int = 64, episode: int = 16, seed: int = 1) -> float:
    """The share of greedy actions that are right after an episode's first step."""
    gen = torch.Generator(device=core.theta.device).manual_seed(seed)
    replica = Replica(core, environments)
    replica.pull(ctx)
    features, reset, cue = memory_game(core, gen, environments, steps, episode)
    right = [replica.step(ctx, features[:, t].contiguous(), reset=reset[:, t].contiguous()).argmax(1) == cue[:, t]
             for t in range(steps)]
    return float(torch.stack([r for t, r in enumerate(right) if t % episode]).float().mean())


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--updates", type=int, default=600)
    ap.add_argument("--actions", type=int, default=6)
    args = ap.parse_args()
    core = RecurrentCore(args.actions)
    ctx = Context(1, 1, min_bytes=core.workspace_bytes(32, 128))
    before = play(core, ctx)
    losses = train(core, ctx, args.updates)
    print(f"loss {losses[:10].mean():.4f} -> {losses[-10:].mean():.4f} in {args.updates} updates; right actions of a "
          f"4-bit replica {before:.1%} -> {play(core, ctx):.1%} (by chance {1 / args.actions:.1%})")
    ctx.check()
    ctx.close()


if __name__ == "__main__":
    main()
