"""The sequence operators on the CPU: the 64-bit definitions' gradients against
central differences, what the library refuses without a device, and its sizes."""
import ctypes

import pytest
import torch

import sequence_ref as ref


def _differences(f, leaves, weights, grads, h=1e-6, picks=6):
    """Each gradient against central differences of sum(outputs * weights) at a few elements (64 bits: the
    difference's own error is about h^2 + 1e-16 / h, so 1e-7 of the gradients' size is demanded)."""
    gen = torch.Generator().manual_seed(3)
    for name, leaf in leaves.items():
        flat, g = leaf.view(-1), grads[name].reshape(-1)
        size = float(g.abs().max()) + 1e-3
        for i in torch.randperm(flat.numel(), generator=gen)[:picks].tolist():
            keep = float(flat[i])
            vals = []
            for s in (h, -h):
                flat[i] = keep + s
                vals.append(sum(float((o * w).sum()) for o, w in zip(f(), weights)))
            flat[i] = keep
            assert abs((vals[0] - vals[1]) / (2 * h) - float(g[i])) < 1e-7 * size * 10, (name, i)


def _rand(*shape, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def test_norm_gradient_is_the_difference():
    x, w, dy, dt = _rand(3, 5, seed=1), _rand(5, seed=2), _rand(3, 5, seed=3), _rand(3, 5, seed=4)
    dx, dw = ref.norm_backward(dy, x, w, 1e-6, dt)
    _differences(lambda: (ref.norm(x, w, 1e-6)[0], x), dict(x=x, w=w), (dy, dt), dict(x=dx, w=dw))


@pytest.mark.parametrize("T,taps,silu", [(7, 4, True), (2, 4, True), (1, 3, False), (5, 2, True)])
def test_conv_gradient_is_the_difference(T, taps, silu):
    x, w, b, win = _rand(2, T, 3, seed=1), _rand(3, taps, seed=2), _rand(3, seed=3), _rand(2, taps - 1, 3, seed=4)
    reset = torch.zeros(2, T, dtype=torch.uint8)
    reset[0, T // 2] = 1
    dy, db = _rand(2, T, 3, seed=5), _rand(2, taps - 1, 3, seed=6)
    got = ref.conv_backward(dy, x, w, b, reset, win, silu, db)
    f = lambda: (lambda o: (o[0], o[2]))(ref.conv(x, w, b, reset, win, silu))  # noqa: E731
    _differences(f, dict(x=x, w=w, b=b, win=win), (dy, db), dict(zip(("x", "w", "b", "win"), got)))


def test_scan_gradient_is_the_difference():
    B, T, H, P, G, N = 2, 6, 4, 3, 2, 5
    leaves = dict(x=_rand(B, T, H, P, seed=1), dt=_rand(B, T, H, seed=2), b=_rand(B, T, G, N, seed=3), c=_rand(B, T, G, N, seed=4),
                  a_log=_rand(H, seed=5) * 0.3, dt_bias=_rand(H, seed=6), skip=_rand(H, seed=7))
    state, dy, ds = _rand(B, H, P, N, seed=8), _rand(B, T, H, P, seed=9), _rand(B, H, P, N, seed=10)
    reset = torch.zeros(B, T, dtype=torch.uint8)
    reset[1, 0] = reset[0, 3] = reset[0, 4] = 1
    got = ref.scan_backward(dy, *leaves.values(), reset, state, ds)
    grads = {k: got["d" + k] for k in (*leaves, "state")}
    _differences(lambda: ref.scan(*leaves.values(), reset, state), dict(leaves, state=state), (dy, ds), grads)


def test_calls_refuse_a_null_context():
    import paper_1507_04296_amd as g
    from paper_1507_04296_amd import sequence
    for name, (res, args) in sequence.SIGNATURES.items():
        if res is not ctypes.c_int32:
            continue
        call = [None if a in (ctypes.c_void_p, sequence._CA, sequence._SA) else 0 for a in args]
        assert getattr(g.lib(), name)(*call) == -1, name


def test_workspace_sizes():
    import paper_1507_04296_amd as g
    assert g.scan_workspace_bytes(64, 128, 16, 64, 1, 64) == 0  # enough sequences and heads: nothing is cut
    assert g.scan_workspace_bytes(1, 4096, 4, 64, 1, 64) > 8192
    for back in (False, True):
        sizes = [g.scan_workspace_bytes(2, t, 4, 64, 1, 64, back) for t in (64, 640, 6400)]
        assert sizes == sorted(sizes)
    assert g.scan_workspace_bytes(2, 8, 4, 129, 1, 64) == 0 and g.scan_workspace_bytes(2, 8, 4, 64, 1, 129) == 0
    assert g.scan_workspace_bytes(2, 8, 4, 64, 3, 64) == 0 and g.scan_workspace_bytes(-1, 8, 4, 64, 1, 64, True) == 0
    assert g.causal_conv_workspace_bytes(1152, 4) > g.causal_conv_workspace_bytes(64, 4) > 0
    assert g.causal_conv_workspace_bytes(64, 5) == 0 and g.causal_conv_workspace_bytes(0, 4) == 0
    assert g.add_rmsnorm_workspace_bytes(512) > 0
    assert g.add_rmsnorm_workspace_bytes(0) == 0 and g.add_rmsnorm_workspace_bytes(65537) == 0
