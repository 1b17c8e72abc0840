"""Routing from logits and its gradient, on the GPU: numbers of tokens beyond a launch, near ties in single places, logits and gradients at the
ends of their range."""
import numpy as np
import pytest
import torch

import paper_2503_00245_amd as pkg
from tests import operators_oracle as oo

pytestmark = pytest.mark.gpu


def dev():
    return torch.device("cuda:0")


# A dimension of a grid has less than 2^32 work items: 2^28 tokens of the picks' launch, 2^26 of the gradient's.
def test_more_tokens_than_a_launch_has_picks_for():
    T = (1 << 28) + 37
    l = torch.randn(T, 2, device=dev())
    idx, gate = torch.full((T, 1), -7, dtype=torch.int32, device=dev()), torch.full((T, 1), 7.0, device=dev())
    pkg.moe_route_scored(pkg.make_route_config(renormalize=False), l, None, idx, gate)
    right = bool((idx[:, 0] == (l[:, 1] > l[:, 0]).int()).all())  # (plain truth values: of tensors as long as these an assertion would make a text)
    assert right
    # the larger of two shares: 1 / (1 + e^-|l0 - l1|), from a difference rounded once
    right = bool(((gate[:, 0] - torch.sigmoid((l[:, 0] - l[:, 1]).abs())).abs() <= 2.0 ** -20).all())
    assert right


def test_more_tokens_than_32_bits_round_up():
    T = (1 << 31) - 1
    l = torch.zeros(T, 1, device=dev())
    idx, gate = torch.full((T, 1), -7, dtype=torch.int32, device=dev()), torch.full((T, 1), 7.0, device=dev())
    pkg.moe_route_scored(pkg.make_route_config(scale=2.5), l, None, idx, gate)
    ends = int(idx.min()), int(idx.max()), float(gate.min()), float(gate.max())
    assert ends == (0, 0, 2.5, 2.5)


def test_more_tokens_than_a_launch_has_gradients_for():
    T = (1 << 26) + 37
    l, dg = torch.randn(T, 2, device=dev()), torch.randn(T, 1, device=dev())
    idx = (torch.rand(T, 1, device=dev()) < 0.5).int()
    out = torch.full((T + 1, 2), 7.0, device=dev())
    pkg.moe_route_scored_backward(pkg.make_route_config(pkg.SCORE_SIGMOID, renormalize=False, scale=2.0), l, idx, dg, None, out[:T])
    right = bool((out[T] == 7).all())
    assert right
    s = torch.sigmoid(l.gather(1, idx.long()))
    right = bool(((out[:T].gather(1, idx.long()) - 2 * dg * s * (1 - s)).abs() <= 2.0 ** -18 * dg.abs()).all())
    assert right
    right = not bool(out[:T].gather(1, 1 - idx.long()).any())
    assert right


@pytest.mark.parametrize("E,groups", [(16, 4), (256, 8), (48, 4), (20, 4)])  # groups of whole lanes, and others
@pytest.mark.parametrize("sigmoid", [False, True])
def test_ranks_of_groups_beyond_the_range_of_fp32(E, groups, sigmoid):
    # finite biases whose sums of two are not: keys far apart, every group's rank above the largest fp32 number
    print("ranks", E, groups, sigmoid, flush=True)
    T, k = 37, 4
    rng = np.random.default_rng(E)
    l = rng.standard_normal((T, E)).astype(np.float32)
    for low, high in ((1.8e38, 3.3e38), (-3.3e38, -1.8e38)):
        bias = rng.permutation(np.linspace(low, high, E)).astype(np.float32)
        cfg = pkg.make_route_config(int(sigmoid), groups, 2, 2)
        idx, gate = torch.empty(T, k, dtype=torch.int32, device=dev()), torch.empty(T, k, device=dev())
        pkg.moe_route_scored(cfg, torch.from_numpy(l).to(dev()), torch.from_numpy(bias).to(dev()), idx, gate)
        ref, ref_gate, _ = oo.route(l, bias, k, sigmoid, groups, 2, 2, True, 1.0)
        assert np.array_equal(idx.cpu().numpy(), ref)
        assert (np.abs(gate.double().cpu().numpy() - ref_gate) <= 2.0 ** -18).all()


@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("E,k", [(8, 3), (60, 6), (256, 8), (512, 64)])
def test_gradients_of_experts_that_are_switched_off_play_no_part(E, k, sigmoid, renorm):
    # the gradient of s log s at s = 0 is minus infinity: at an expert whose score is a constant it is of nothing
    print("off", E, k, sigmoid, renorm, flush=True)
    T = 41
    rng = np.random.default_rng(E + k)
    l = rng.standard_normal((T, E)).astype(np.float32)
    dead = rng.random((T, E)) < 0.3
    dead[::7] = True          # rows of nothing else
    dead[1::7, : E - k + 1] = True  # ... and of fewer than k
    l[dead] = np.where(rng.random((T, E)) < 0.5, -np.inf, np.nan)[dead].astype(np.float32)
    idx, _, _ = oo.route(l, None, k, sigmoid, 1, 1, 1, renorm, 1.0)
    dg, ds = rng.standard_normal((T, k)).astype(np.float32), rng.standard_normal((T, E)).astype(np.float32)
    off_pick = np.take_along_axis(dead, idx.astype(np.int64), 1)
    assert off_pick.any() and not off_pick.all()
    out = []
    for fill in (0.0, -np.inf, np.nan):
        dg[off_pick], ds[dead] = fill, fill
        for aux in (True, False):
            g = torch.full((T, E), 7.0, device=dev())
            pkg.moe_route_scored_backward(pkg.make_route_config(int(sigmoid), renormalize=renorm), torch.from_numpy(l).to(dev()), torch.from_numpy(idx).to(dev()),
                                          torch.from_numpy(dg).to(dev()), torch.from_numpy(ds).to(dev()) if aux else None, g)
            out.append(g)
    for aux in (0, 1):
        assert torch.isfinite(out[aux]).all()
        assert not out[aux][torch.from_numpy(dead).to(dev())].any()
        assert torch.equal(out[aux], out[2 + aux]) and torch.equal(out[aux], out[4 + aux])
