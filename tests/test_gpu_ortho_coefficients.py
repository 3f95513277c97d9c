"""Which coefficients the orthogonalised update takes: those whose values fit,
and no others."""

import numpy as np
import pytest
import torch

from tests.test_gpu_ortho import CUBIC, DEV, QUINTIC, check, flat, plan_for

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tc():
    import paper_1801_03855_amd as tc
    tc.lib()
    return tc


def rounded(*triples):
    return [tuple(float(np.float32(v)) for v in t) for t in triples]


# the optimal quintic steps of Amsel et al. 2025, for singular values from 1e-3
OPTIMAL = rounded((8.28721201814563, -23.595886519098837, 17.300387312530933), (4.107059111542203, -2.9478499167379106, 0.5448431082926601),
                  (3.9486908534822946, -2.908902115962949, 0.5518191394370137), (3.3184196573706015, -2.488488024314874, 0.51004894012372),
                  (2.300652019954817, -1.6689039845747493, 0.4188073119525673), (1.891301407787398, -1.2679958271945868, 0.37680408948524835),
                  (1.875, -1.25, 0.375))
PAIRED = [(520, 1100), 5, (1030, 513)]
SINGLE = [(200, 390), 5, (300, 310), (20, 30)]


def call(tc, shapes, triples, kind="gauss"):
    gen = torch.Generator().manual_seed(len(triples))
    g = flat(gen, shapes, kind, torch.float32)
    out = torch.empty_like(g)
    tc.orthogonalize(plan_for(tc, 1, shapes), [g], [out], steps=len(triples), coefficients=triples)
    check(out, g, shapes, triples)


@pytest.mark.parametrize("shapes", [PAIRED, SINGLE, PAIRED + SINGLE])
@pytest.mark.parametrize("steps", [2, 3, 5, 7])
def test_optimal_quintic_steps(tc, shapes, steps):
    """The first two multiply small singular values by 8.3 and 4.1; what two of
    them at once store is up to 33.8 of 62.9."""
    call(tc, shapes, OPTIMAL[:steps], "directions")


@pytest.mark.parametrize("triples", [rounded((9.6, -30.9, 22.8), (6.5, -4.3, 0.7)), rounded((8.0, -24.8, 17.6), (7.7, -5.6, 1.0))])
def test_what_only_two_steps_at_once_cannot_hold(tc, triples):
    """|q1(x q^2) q - a1 a| reaches 66.3 and 65.8, which one step at a time
    never forms."""
    call(tc, SINGLE, triples)
    call(tc, PAIRED, triples[:1])
    call(tc, PAIRED, [CUBIC] + rounded((1.5, -0.5, 0.0), (1.0, 0.0, 0.0)))
    for shapes in (PAIRED, PAIRED + SINGLE):
        for more in ([], [CUBIC]):
            with pytest.raises(tc.TCError):
                call(tc, shapes, triples + more)
    # the pairs are the first and second, third and fourth steps
    with pytest.raises(tc.TCError):
        call(tc, PAIRED, rounded((1.0, 0.0, 0.0), (1.0, 0.0, 0.0)) + triples)
    call(tc, PAIRED, rounded((1.0, 0.0, 0.0)) + triples)


@pytest.mark.parametrize("triples", [
    rounded((4.1, 0.0, 0.0)), rounded((20.0, -19.5, 0.0)), rounded((3.9, 0.0, 0.0), (1.1, 0.0, 0.0)), [QUINTIC] * 3 + rounded((4.0, 0.0, 0.0)),
    rounded((0.5, 130.0, -130.0)), rounded((2.0, 0.0, -1.0), (0.0, 0.0, 1.0)) + [QUINTIC], rounded((60.0, -380.0, 325.0)),
])
def test_refused_for_every_plan(tc, triples):
    for shapes in (PAIRED, SINGLE, [(4, 5)]):
        with pytest.raises(tc.TCError):
            call(tc, shapes, triples)


@pytest.mark.parametrize("triples", [rounded((3.9, 0.0, 0.0)), rounded((-3.9, 0.0, 0.0)), rounded((0.0, -3.9, 0.0)), rounded((0.5, 8.0, -8.0)),
                                     rounded((1.0, 0.0, 0.0), (0.0, 0.0, 0.0), CUBIC)])
def test_taken_by_every_plan(tc, triples):
    for shapes in (PAIRED, SINGLE, [(4, 5)]):
        call(tc, shapes, triples)
