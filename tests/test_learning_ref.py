"""The reference formulas of learning_ref.py against differences and closed forms, and
what of the library's layer norm, gated scan, AdamW and sampling needs no device."""
import ctypes

import numpy as np
import pytest
import torch

import learning_ref as ref


def rand(*shape, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def difference(f, x, d, h=1e-6):
    return float((f(x + h * d) - f(x - h * d)) / (2 * h))


def test_gradients_of_the_formulas_against_differences():
    x, w, dy = rand(3, 7, seed=1), rand(7, seed=2), rand(3, 7, seed=3)
    dx, dw, db = ref.layernorm_backward(dy, x, w, 1e-5)
    for got, at, f in ((dx, x, lambda v: (ref.layernorm(v, w, None, 1e-5)[0] * dy).sum()),
                       (dw, w, lambda v: (ref.layernorm(x, v, None, 1e-5)[0] * dy).sum())):
        d = rand(*at.shape, seed=4)
        assert abs(float((got * d).sum()) - difference(f, at, d)) < 1e-7
    assert torch.allclose(db, dy.sum(0))
    a = [rand(2, 5, 3, seed=s) for s in (1, 2, 3)] + [rand(3, seed=4)]
    reset = torch.tensor([[0, 0, 1, 0, 0], [1, 0, 0, 0, 1]], dtype=torch.uint8)
    state, dy, ds = rand(2, 3, seed=5), rand(2, 5, 3, seed=6), rand(2, 3, seed=7)
    got = ref.gated_backward(dy, *a, reset, state, ds)

    def value(*args):
        y, h, _ = ref.gated(*args[:4], reset, args[4])
        return (y * dy).sum() + (h * ds).sum()

    args = [*a, state]
    for k, grad in enumerate(got):
        d = rand(*args[k].shape, seed=8 + k)
        want = difference(lambda v: value(*args[:k], v, *args[k + 1:]), args[k], d)
        assert abs(float((grad * d).sum()) - want) < 1e-7, k


def test_held_values():
    """The last code is 1, neighbours are an eighth of a power of two apart, and chance decides between them alone."""
    one = np.ones(1, dtype=np.float32)
    for name, last in (("m", 127), ("v", 255)):
        least = ref.LEAST[name]
        assert float(ref.held(np.array([last]), least, one)[0]) == 1.0
        assert float(ref.held(np.array([last - 1]), least, one)[0]) == 0.9375
        assert float(ref.held(np.array([last - 8]), least, one)[0]) == 0.5
        size = np.array([1.0, 0.9, 0.25, 0.0], dtype=np.float32)
        low, _ = ref.hold(size, np.zeros(4, dtype=np.int64), least)
        high, scale = ref.hold(size, np.full(4, 65535), least)
        assert scale[0] == 1.0 and list(low) == [last, last - 2, last - 16, 0] and list(high) == [last, last - 1, last - 16, 0]


def test_sample_closed_forms():
    v = torch.tensor([[0.0, 0.0, -float("inf")]]).repeat(4, 1)
    action, p = ref.sample(v, torch.tensor([0.0, 0.49, 0.5, 0.99]))
    assert action.tolist() == [0, 0, 1, 1] and p.tolist() == [0.5] * 4
    assert ref.sample(v, torch.tensor([0.99] * 4), top_p=torch.full((4,), 0.5))[0].tolist() == [0] * 4


def test_null_contexts_are_refused():
    import paper_1507_04296_amd as g
    L = g.lib()
    assert L.gorila_add_layernorm(*[None, 0, None, 0, None, None, 1, 8, 0, 1e-5, None, None, None, None, None]) == -1
    assert L.gorila_add_layernorm_backward(*[None, 0, None, 0, None, None, None, None, 1, 8, 0, None, None, None, None]) == -1
    assert L.gorila_gated_scan(None, None, None, None, None) == -1
    assert L.gorila_gated_scan_backward(None, None, None, 0, 0, *[None] * 7) == -1
    assert L.gorila_gated_scan_step(None, None, 0, None, None, None) == -1
    assert L.gorila_adamw(None, 0, 0, 32, None, None, 0.0, 0.9, 0.999, 1e-8, ctypes.c_uint64(0), None) == -1
    assert L.gorila_adamw_values(None, 0, None, None, None) == -1
    assert L.gorila_sample_actions(None, 0, 1, 2, 0, *[None] * 8) == -1


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("channels", [1, 63, 64, 65, 1000, 4096, 100000])
def test_gated_workspace_of_the_largest_is_enough_for_all_smaller(channels, backward):
    import paper_1507_04296_amd as g
    last = 0
    for length in (0, 1, 64, 255, 256, 257, 1000, 20000, 1 << 30):
        sizes = [g.gated_scan_workspace_bytes(b, length, channels, backward) for b in (0, 1, 2, 31, 600)]
        assert len(set(sizes)) == 1 and sizes[0] >= last  # of the length alone
        assert backward or length > 256 or sizes[0] == 0
        last = sizes[0]
    assert g.gated_scan_workspace_bytes(1, 1, 0) == 0 == g.add_layernorm_workspace_bytes(0) == g.add_layernorm_workspace_bytes(65537)


def test_adamw_states():
    import paper_1507_04296_amd as g
    thetas = [torch.zeros(3, 100), torch.zeros(0), torch.zeros(257)]
    assert [[tuple(v.shape) for v in s] for s in g.adamw_state(thetas, 8)] == [
        [(3, 100), (3, 100), (2,), (2,)], [(0,), (0,), (0,), (0,)], [(257,), (257,), (2,), (2,)]]
    assert [v.dtype for v in g.adamw_state(thetas)[0]] == [torch.float32] * 2
    assert g.adamw_clock("cpu").tolist() == [0.0] * 3
    with pytest.raises(ValueError, match="bits"):
        g.adamw_state(thetas, 4)
