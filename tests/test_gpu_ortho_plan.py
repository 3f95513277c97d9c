"""Plans of the orthogonalised update that are too large to launch."""

import resource
import time

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tc():
    import paper_1801_03855_amd as tc
    tc.lib()
    return tc


@pytest.mark.parametrize("K,shapes", [
    (64, [(65536, 65536)]),                        # 2^24 tiles of P X, 2^23 of X X^T
    (64, [(65536, 32768), (32768, 32768)] * 2),    # the tiles of several matrices together
])
def test_lists_that_are_too_long_are_refused_before_they_are_built(tc, K, shapes):
    """Built, the lists would take 1 to 2 GB of host memory."""
    group = tc.Group([r * c for r, c in shapes])
    before, start = resource.getrusage(resource.RUSAGE_SELF).ru_maxrss, time.monotonic()
    with pytest.raises(tc.TCError):
        tc.OrthoPlan(group, K, shapes)
    took, grown = time.monotonic() - start, resource.getrusage(resource.RUSAGE_SELF).ru_maxrss - before
    assert grown < 400 << 10, f"{grown >> 10} MiB more"
    assert took < 1.0, f"{took:.1f} s"


def test_one_copy_of_such_a_matrix_has_a_plan(tc):
    """2^18 tiles, of which one launch takes 2^24 - 1."""
    shapes = [(65536, 65536)]
    plan = tc.OrthoPlan(tc.Group([1 << 32]), 1, shapes)
    assert tc.ortho_workspace(plan) >= 3 * 4 << 32
