"""The recurrent core made of the sequence operators, against the same formulas in 64
bits with the gradients of automatic differentiation.

Tolerances.  Q passes two norms, three products of at most 512 terms, the convolution
and the scan, each 2e-6 relative L2 at most: 2e-5.  A gradient passes those and their
backwards, 1e-5 each at most: 1e-4.  A replica's rows of 8-bit codes are off by a
rounding of m / 127, m the row's largest value (about 3 times its root mean square): 0.7 %
of the row, for each of two norms; the scan multiplies three rows of the first: 3 % of Q
in all; twice that is allowed.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
Q_TOL, GRAD_TOL, REPLICA_TOL = 2e-5, 1e-4, 6e-2


@pytest.fixture(scope="module")
def rec():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a ROCm device")
    import paper_1507_04296_amd.recurrent as module
    return module


def off(got, want):
    got, want = got.detach().cpu().double(), want.detach().cpu().double()
    return float((got - want).norm() / want.norm())


def plain(core, p, features, reset, window, state):
    """Q in the type of its arguments, step by step; p as core.params."""
    B, T, _ = features.shape
    H, P, G, N, K = core.heads, core.head_dim, core.groups, core.state_dim, core.taps
    norm = lambda x, w: x * (x.pow(2).mean(-1, keepdim=True) + 1e-6).rsqrt() * w
    z = norm(features, p["norm_in"]) @ p["w_in"].T
    out = []
    for b in range(B):
        past, S = [window[b, j] for j in range(K - 1)], state[b]
        for t in range(T):
            if reset[b, t]:
                past, S = [torch.zeros_like(v) for v in past], torch.zeros_like(S)
            past = past[-(K - 1):] + [z[b, t, :core.channels]]
            v = p["conv_bias"] + sum(p["conv"][:, j] * past[j] for j in range(K))
            x, bb, cc = core._split(v * torch.sigmoid(v))
            bb, cc = (r.repeat_interleave(H // G, 0) for r in (bb, cc))
            d = torch.nn.functional.softplus(z[b, t, core.channels:] + p["dt_bias"])
            S = torch.exp(-torch.exp(p["a_log"]) * d)[:, None, None] * S + (d[:, None] * x)[:, :, None] * bb[:, None, :]
            out.append(((S * cc[:, None, :]).sum(-1) + p["skip"][:, None] * x).flatten())
    u = torch.stack(out).view(B, T, -1) @ p["w_out"].T
    return norm(features + u, p["norm_out"]) @ p["w_q"].T


def make(rec, B, T, seed, **sizes):
    core = rec.RecurrentCore(5, seed=seed, **sizes)
    gen = torch.Generator().manual_seed(seed)
    features = torch.randn((B, T, core.features), generator=gen).cuda()
    reset = (torch.rand((B, T), generator=gen) < 0.05).to(torch.uint8).cuda()
    window = torch.randn((B, core.taps - 1, core.channels), generator=gen).cuda()
    state = 0.3 * torch.randn((B, core.heads, core.head_dim, core.state_dim), generator=gen).cuda()
    from paper_1507_04296_amd import Context
    return core, Context(1, 1, min_bytes=core.workspace_bytes(B, T)), features, reset, window, state


SIZES = [dict(features=96, heads=4, head_dim=32, groups=2, state_dim=16, taps=4),
         dict(features=51, heads=3, head_dim=17, groups=1, state_dim=33, taps=3),
         dict(features=128, heads=2, head_dim=64, groups=1, state_dim=64, taps=2)]


@pytest.mark.parametrize("T", [1, 70])
@pytest.mark.parametrize("sizes", SIZES)
def test_core_values_and_gradients(rec, sizes, T):
    core, ctx, features, reset, window, state = make(rec, 2, T, 3, **sizes)
    q, _, saved = core.forward(ctx, features, reset, (window, state))
    gen = torch.Generator().manual_seed(9)
    dq = torch.randn(q.shape, generator=gen).cuda()
    grad, dfeatures = core.backward(ctx, dq, saved)
    p = {n: v.cpu().double().requires_grad_(True) for n, v in core.params.items()}
    f = features.cpu().double().requires_grad_(True)
    want = plain(core, p, f, reset.cpu(), window.cpu().double(), state.cpu().double())
    assert off(q, want) <= Q_TOL
    want.backward(dq.cpu().double())
    assert off(dfeatures, f.grad) <= GRAD_TOL
    for name, got in core.views(grad).items():
        assert off(got, p[name].grad) <= GRAD_TOL, name
    ctx.check()
    ctx.close()


def test_core_goes_on_from_what_it_carried(rec):
    core, ctx, features, reset, _, _ = make(rec, 3, 90, 4, **SIZES[0])
    whole, last, _ = core.forward(ctx, features, reset)
    first, carried, _ = core.forward(ctx, features[:, :37], reset[:, :37].contiguous())
    second, carried, _ = core.forward(ctx, features[:, 37:], reset[:, 37:].contiguous(), carried)
    assert off(torch.cat([first, second], 1), whole) <= Q_TOL
    for got, want in zip(carried, last):
        assert off(got, want) <= Q_TOL
    ctx.close()


def test_replica_steps_as_the_core_does(rec):
    """Matrices that 4 bits hold exactly: what is left is the rounding of the rows."""
    core, ctx, features, reset, _, _ = make(rec, 7, 40, 5, features=512)
    gen = torch.Generator().manual_seed(6)
    for name in ("w_in", "w_out", "w_q"):
        w = core.params[name]
        codes = torch.randint(-7, 8, w.shape, generator=gen)
        codes[:, ::32] = 7  # the largest of every group
        w.copy_(codes / 4.0 / math.sqrt(w.shape[1]))
    want, _, _ = core.forward(ctx, features, reset)
    replica = rec.Replica(core, 11)
    replica.pull(ctx)
    replica.windows.normal_()
    replica.states.normal_()
    slot = torch.tensor([3, 0, 10, 5, 1, 8, 6], dtype=torch.int32, device="cuda")
    reset[:, 0] = 1  # what the slots held before does not matter
    idle = replica.states[[2, 4, 7, 9]].clone()
    want, _, _ = core.forward(ctx, features, reset)
    got = torch.stack([replica.step(ctx, features[:, t].contiguous(), slot, reset[:, t].contiguous())
                       for t in range(features.shape[1])], 1)
    assert off(got, want) <= REPLICA_TOL
    assert torch.equal(replica.states[[2, 4, 7, 9]], idle)
    ctx.check()
    ctx.close()


def test_training_learns_to_remember(rec):
    core = rec.RecurrentCore(6)
    from paper_1507_04296_amd import Context
    ctx = Context(1, 1, min_bytes=core.workspace_bytes(32, 128))
    losses = rec.train(core, ctx, 600)
    assert torch.isfinite(losses).all() and losses[-20:].mean() < 0.5 * losses[20:40].mean()
    assert rec.play(core, ctx, environments=64, steps=32) > 2 / 3  # by chance 1 / 6
    ctx.check()
    ctx.close()
