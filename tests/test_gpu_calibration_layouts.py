"""GPU tests of a calibration that prepares q and k itself: projections of any layout, and the caller's tensors as they were."""
import numpy as np
import pytest

from tests.test_gpu_layer_path import GEOMETRY, make, preparation

pytestmark = pytest.mark.gpu

H, D, N = 3, 64, int(np.prod(GEOMETRY))


def projections(rng, layout):
    fused = make(rng, (2, N, 3, H, D), gain=2.0)
    q, k = (fused[:, :, i].transpose(1, 2) for i in range(2))
    if layout == "packed":
        return q.contiguous(), k.contiguous()
    if layout == "bnhd":
        return tuple(t.transpose(1, 2).contiguous().transpose(1, 2) for t in (q, k))
    return q, k


def parts(prep, which):
    """The preparation without some of its steps."""
    import dataclasses

    return dataclasses.replace(prep, **{name: None for name in which})


@pytest.mark.parametrize("layout", ["packed", "bnhd", "fused"])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("without", [(), ("rope",), ("q_norm",), ("q_norm", "k_norm"), ("rope", "k_norm")])
def test_observe_leaves_what_it_is_given(lib, layout, in_place, without):
    import torch

    rng = np.random.default_rng(1)
    prep, _ = preparation(lib, rng, D, in_place=in_place)
    prep = parts(prep, without)
    q, k = projections(rng, layout)
    given = q.clone(), k.clone()
    a = lib.Calibrator(H, N, D, 64, 64, GEOMETRY, prepare=prep)
    for _ in range(2):  # twice the same votes
        a.observe("x", q, k, 0.8, 0.125)
    assert torch.equal(q, given[0]) and torch.equal(k, given[1])
    by_hand = parts(prep, ())
    by_hand.in_place = False
    b = lib.Calibrator(H, N, D, 64, 64, GEOMETRY)
    qp, kp = by_hand(q.contiguous(), k.contiguous(), GEOMETRY)
    for _ in range(2):
        b.observe("x", qp, kp, 0.8, 0.125)
    ra, rb = a.finalize()["x"], b.finalize()["x"]
    assert ra.n_prompts == rb.n_prompts == 4
    assert np.array_equal(ra.mask, rb.mask) and np.array_equal(ra.scores, rb.scores)


def test_a_refused_preparation_leaves_what_it_is_given(lib):
    import torch

    rng = np.random.default_rng(2)
    prep, _ = preparation(lib, rng, D, in_place=True)
    q, k = projections(rng, "fused")
    given = q.clone(), k.clone()
    with pytest.raises(ValueError):
        prep(q, k)  # no grid
    with pytest.raises(ValueError):
        lib.Calibrator(H, N, D, 64, 64, prepare=prep).observe("x", q, k, 0.8, 0.125)
    assert torch.equal(q, given[0]) and torch.equal(k, given[1])
