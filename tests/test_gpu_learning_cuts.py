"""The gated scan where a sequence is cut into segments and a segment's maps into parts,
where workgroups go round their loops, and sampled actions of rows past 65536 actions
without a workspace.  Values against the definitions in 64 bits, tolerances of
test_gpu_learning.py (their reasons do not depend on the length: errors of 32 bits
that add as a random walk)."""
import pytest
import torch

from test_gpu_learning import BF16, F32, check_gated, check_sample, ctx, g, gated_inputs, sample_inputs  # noqa: F401

# (sequences, steps, channels): sequences x 64-channel tiles are the workgroups at hand.  Forward fewer than 256
# are cut towards 256, backward towards 512, in segments of whole 256 steps; the forward maps of a segment go in parts
# of whole 256 steps while there are fewer than 512 workgroups for them.
CUTS = [(128, 520, 4),    # forward 2 segments of 512 whose maps are 2 parts of 256; backward 3 of 256
        (128, 1300, 5),   # forward 2 of 768, 3 parts; backward 3 of 512
        (60, 2000, 3),    # forward 4 of 512, 2 parts each; backward 8 of 256
        (100, 2500, 2),   # forward 2 of 1280, 5 parts; backward 5 of 512
        (20, 1600, 70),   # forward 4 of 512 in 2 tiles, 2 parts; backward 7 of 256
        (192, 1500, 8),   # forward uncut, 8 waves over 12 chunks; backward 3 of 512
        (150, 2100, 7),   # forward uncut; backward 3 of 768, the last of 564
        (1, 16700, 9),    # 33 of 512 both ways (64 at most), 2 parts
        (300, 150, 8),    # forward 4 waves over 3 chunks, backward too
        (130, 200, 129),  # the same in 3 tiles, the last of one channel
        (2100, 70, 4),    # backward workgroups with several sequences, 2 chunks each
        (2060, 150, 3),   # the same, 3 chunks
        (700, 40, 130)]   # the same in 3 tiles, one chunk


def cut(B, T, C, backward):
    """Segments, steps of one, parts of its map, by the rule in words above."""
    have = B * -(-C // 64)
    if have >= 256:
        return 1, T, 1
    k = min(-(-512 // have) if backward else 256 // have, -(-T // 256), 64)
    if k < 2:
        return 1, T, 1
    seg = -(-(-(-T // k)) // 256) * 256
    n = -(-T // seg)
    parts = 1 if backward or n < 2 else max(1, min(512 // (have * (n - 1)), seg // 256))
    while parts > 1 and seg % (parts * 256):
        parts -= 1
    return n, seg, parts


def test_the_cases_are_cut_in_every_way():
    forward, backward = [cut(*c, False) for c in CUTS], [cut(*c, True) for c in CUTS]
    assert {p for _, _, p in forward} >= {1, 2, 3, 5}
    assert {s for n, s, _ in backward if n > 1} >= {256, 512, 768}
    assert any(n > 2 and p > 1 for n, _, p in forward) and any(p > 1 and c[2] > 64 for c, (_, _, p) in zip(CUTS, forward))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T,C", CUTS)
def test_gated_scan_cuts(g, ctx, B, T, C, dtype):  # noqa: F811
    """Episodes of 1 / 0.002 steps, so that some pass whole segments and others begin in them."""
    args, reset, state, dy, dstate = gated_inputs(B, T, C, dtype, seed=120, resets=0.002)
    check_gated(g, ctx, args, reset, state, dy, dstate, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("filters", ["", "k", "p", "tkpm"])
def test_sample_of_very_long_rows_without_a_workspace(g, ctx, filters, dtype):  # noqa: F811
    """One workgroup a row: the definition's actions, and those of shared rows."""
    values, u, options = sample_inputs(3, 70001, filters, dtype, seed=130)
    if "k" in filters:
        options["top_k"][0] = 40
    bare = g.Context(0, 1)
    check_sample(g, bare, values, u, options)
    for a, b in zip(g.sample_actions(ctx, values, u, **options), g.sample_actions(bare, values, u, **options)):
        assert torch.equal(a, b)
    bare.close()
