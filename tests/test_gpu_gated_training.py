"""The training run's parts, each for itself: what `train` hands to its update, what the
AdamW update does with a loss that the filter refuses, and what `play` counts.
Tolerances are those of test_gpu_gated_core.py."""
import pytest
import torch

from test_gpu_gated_core import GRAD_TOL, Q_TOL, off, plain, rec  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,T,episode", [(2, 24, 8), (3, 7, 3)])
def test_train_hands_over_each_loss_and_its_gradient(rec, B, T, episode):  # noqa: F811
    """Of the mean Huber loss of Q at the actions taken, against automatic differentiation of it in 64 bits."""
    from paper_1507_04296_amd import Context
    core = rec.GatedCore(5, features=48, channels=64, seed=2)
    ctx = Context(1, 1, min_bytes=core.workspace_bytes(B, T))
    got = []
    losses = rec.train(core, ctx, 3, batch=B, length=T, episode=episode, seed=4, update=lambda c, grad, loss: got.append((c, grad, loss)))
    gen = torch.Generator(device="cuda").manual_seed(4)
    zero = torch.zeros(B, core.taps - 1, core.channels, dtype=torch.float64), torch.zeros(B, core.channels, dtype=torch.float64)
    for n in range(3):
        features, reset, cue = rec.memory_game(core, gen, B, T, episode)
        action = torch.randint(0, core.actions, cue.shape, generator=gen, device="cuda")
        p = {k: v.cpu().double().requires_grad_(True) for k, v in core.params.items()}
        q = plain(core, p, features.cpu().double(), reset.cpu(), *zero)
        loss = torch.nn.functional.huber_loss(q.gather(2, action.cpu()[..., None])[..., 0], (action == cue).cpu().double())
        loss.backward()
        c, grad, seen = got[n]
        assert c is ctx and off(seen, loss) <= Q_TOL and float(losses[n]) == float(seen)
        for name, v in core.views(grad).items():
            assert off(v, p[name].grad) <= GRAD_TOL, name
    ctx.check()
    ctx.close()


@pytest.mark.parametrize("bits", [8, 32])
def test_update_leaves_out_what_the_filter_refuses(rec, bits, oracle_mod):  # noqa: F811
    """Every loss's answer is the filter's own; a refused one leaves parameters, states and clock as they were."""
    from paper_1507_04296_amd import Context
    core = rec.GatedCore(5, features=16, channels=16, seed=3)
    ctx = Context(1, 1)
    update = rec.AdamW(core, bits=bits, k=2.0, warmup=3)
    grad = torch.ones_like(core.theta)
    stats, taken, answers = [[0.0, 0.0, 0.0]], 0, []
    for x in (1.0, 1.5, 0.5, 1.25, 1.0, 50.0, 1.25, 75.0, 0.75):
        before = [v.clone() for v in (core.theta, update.clock, *[v for s in update.states for v in s])]
        update(ctx, grad, torch.tensor(x, device="cuda"))
        keep, stats = oracle_mod.loss_filter(stats, [x], 0.05, 2.0, 3)
        answers.append(int(keep[0]))
        taken += answers[-1]
        after = [core.theta, update.clock, *[v for s in update.states for v in s]]
        assert int(update.keep[0]) == answers[-1] and int(update.clock[0]) == taken
        assert all(torch.equal(a, b) for a, b in zip(before, after)) == (not answers[-1])
    assert 0 in answers and answers.count(1) >= 5
    ctx.check()
    ctx.close()


@pytest.mark.parametrize("temperature", [0.0, 0.5])
def test_play_counts_right_actions(rec, temperature):  # noqa: F811
    """With Q of zeros everywhere a greedy action is the first, a drawn one floor(6 u)."""
    from paper_1507_04296_amd import Context
    core = rec.GatedCore(6, features=32, channels=64, seed=5)
    core.params["w_q"].zero_()
    ctx = Context(1, 1, min_bytes=core.workspace_bytes(1, 1))
    share = rec.play(core, ctx, environments=9, steps=12, episode=4, seed=6, temperature=temperature)
    gen = torch.Generator(device="cuda").manual_seed(6)
    _, _, cue = rec.memory_game(core, gen, 9, 12, 4)
    right = []
    for t in range(12):
        u = torch.rand(9, generator=gen, device="cuda").double()
        action = (6 * u).floor().long() if temperature > 0 else torch.zeros(9, dtype=torch.int64, device="cuda")
        if t % 4:
            right.append(action == cue[:, t])
    assert abs(share - float(torch.stack(right).double().mean())) <= 1e-6
    ctx.check()
    ctx.close()
