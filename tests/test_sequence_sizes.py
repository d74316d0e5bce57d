"""Workspace sizes of the sequence operators (no device needed)."""
import pytest


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("heads,head_dim,state", [(16, 64, 64), (16, 64, 128), (3, 100, 20), (1, 1, 1)])
def test_scan_workspace_of_the_largest_is_enough_for_all_smaller(heads, head_dim, state, backward):
    """Whatever batch and length a context was made for, a smaller one asks for no more.  Forward calls of up to 128
    steps run without any workspace, so that what they ask for is only what makes them fast."""
    import paper_1507_04296_amd as g
    batches = [1, 2, 3, 7, 15, 16, 17, 31, 32, 33, 64, 171, 511, 512, 513, 2000]
    lengths = [1, 31, 32, 33, 64, 65, 128, 129, 160, 161, 300, 512, 1000, 1999, 8192]
    size = {(b, t): g.scan_workspace_bytes(b, t, heads, head_dim, 1, state, backward) for b in batches for t in lengths}
    for n, b in enumerate(batches):
        for m, t in enumerate(lengths):
            if not backward and t <= 128:
                continue
            for smaller in ((batches[n - 1], t), (b, lengths[m - 1])):
                if smaller[0] <= b and smaller[1] <= t and (backward or smaller[1] > 128):
                    assert size[smaller] <= size[b, t], (smaller, (b, t))
    assert all(size[b, t] > 0 for b, t in size if backward or t > 128)
