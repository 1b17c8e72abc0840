"""The products of experts in microscaled 4-bit floating point and the sum of their rows, on the GPU, against plain implementations in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2503_00245_amd as pkg
from tests import operators_oracle as oo
from tests.mxfp4_cases import PATTERNS, TILED, picks
from tests.test_mxfp4_gpu import DTYPES, _layer, _run, dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1, 4, 5, 40, 300, 1500])
def test_the_gated_sum_is_of_rows_that_are_not_rounded(T):
    # Experts in pairs: the second one is the first with its down product's signs turned, but for one column in 64, so that a sum is an eighth to a
    # quarter of its two addends: what rounding those to bf16 would leave (2^-9 of them each) is above the result's own rounding
    # (2^-8 of an eighth).  The bound has no such rounding: sums in fp32 and steps of the hidden rows' 4 bits, then one rounding of y.
    print("sum", T, flush=True)
    E, d, F, k = 8, 128, 256, 2
    rng = np.random.default_rng(T)
    w, exact = _layer(rng, E, d, F)
    for n in ("gate", "up"):
        for part in ("_codes", "_scales"):
            w[n + part][1::2] = w[n + part][0::2]
    for m in (0, 1):
        exact[m][1::2] = exact[m][0::2]
    kept = np.arange(F) % 64 == 5
    turn = torch.from_numpy(np.where(kept[0::2], 0, 0x08) | np.where(kept[1::2], 0, 0x80)).to(torch.uint8).to(dev())
    w["down_codes"][1::2] = w["down_codes"][0::2] ^ turn
    w["down_scales"][1::2] = w["down_scales"][0::2]
    exact[2][1::2] = exact[2][0::2] * np.where(kept, 1.0, -1.0)
    first = rng.integers(0, E // 2, (T, 1)) * 2
    idx = np.concatenate([first, first + 1], 1).astype(np.int32)
    gate = np.ones((T, k), np.float32)
    x = torch.from_numpy(rng.standard_normal((T, d)).astype(np.float32)).bfloat16().to(dev())
    y = _run(x, w, torch.from_numpy(idx).to(dev()), torch.from_numpy(gate).to(dev()), E, k, d, F, "bf16", False)
    ref, tol = oo.experts(x.double().cpu().numpy(), exact, idx, gate.astype(np.float64), False, 2.0 ** -24)
    tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref)
    err = np.abs(y.double().cpu().numpy() - ref)
    assert np.isfinite(err).all()
    assert (err <= tol).all(), (err / np.maximum(tol, 1e-300)).max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,F,E,k,skew,hidden,down", TILED)
def test_tiled_products(T, d, F, E, k, skew, hidden, down, dtype):
    # (tests/test_mxfp4_plan_cpu.py holds the cases to the tiles that they name)
    print("tiled", T, d, F, E, k, skew, hidden, down, dtype, flush=True)
    rng = np.random.default_rng(T + d * 3 + F)
    w, exact = _layer(rng, E, d, F)
    idx, gate = picks(E, k, skew)
    x = torch.from_numpy(rng.standard_normal((PATTERNS, d)).astype(np.float32)).to(DTYPES[dtype]).to(dev())
    pattern = torch.arange(T, device=dev()) % PATTERNS
    residual = F % 3 == 0
    y = _run(x[pattern], w, torch.from_numpy(idx).to(dev())[pattern], torch.from_numpy(gate).to(dev())[pattern], E, k, d, F, dtype, residual)
    half_step = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    ref, tol = oo.experts(x.double().cpu().numpy(), exact, idx, gate.astype(np.float64), residual, 2.0 ** -24)
    tol = tol * (1 + half_step) + half_step * np.abs(ref)
    err = np.abs(y[:PATTERNS].double().cpu().numpy() - ref)
    assert np.isfinite(err).all()
    assert (err <= tol).all(), (err / np.maximum(tol, 1e-300)).max()
    # a row's sums are formed in the same order wherever it lies in a tile: copies of a token have its bits
    same = (y == y[:PATTERNS][pattern]).all(1)
    assert same.all(), same.logical_not().nonzero()[:8].flatten().tolist()


@pytest.mark.parametrize("T,d,F,E,k,skew,hidden,down", [c for c in TILED if c[-2:] in ((128, 64), (128, 256), (256, 128), (64, 128))][:6])
def test_a_token_of_nan_and_bad_picks_in_a_tile_leave_the_others_as_they_are(T, d, F, E, k, skew, hidden, down):
    print("alone", T, d, F, E, k, hidden, down, flush=True)
    rng = np.random.default_rng(T + F)
    w, _ = _layer(rng, E, d, F)
    weights = pkg.make_mxfp4_weights(w)
    idx, gate = picks(E, k, skew)
    pattern = torch.arange(T, device=dev()) % PATTERNS
    i, g = torch.from_numpy(idx).to(dev())[pattern], torch.from_numpy(gate).to(dev())[pattern]
    x = torch.from_numpy(rng.standard_normal((T, d)).astype(np.float32)).bfloat16().to(dev())
    want = _run(x, w, i, g, E, k, d, F, "bf16", False, weights).clone()
    odd = torch.tensor([0, 1, T // 3, T // 2, T - 1], device=dev())
    others = torch.ones(T, dtype=torch.bool, device=dev())
    others[odd] = False
    x2, i2 = x.clone(), i.clone()
    x2[odd, d - 1] = torch.tensor([float("nan"), float("inf"), -float("inf"), float("nan"), float("nan")], device=dev()).bfloat16()
    y = _run(x2, w, i, g, E, k, d, F, "bf16", False, weights)
    assert torch.equal(y[others], want[others])
    assert torch.isnan(y[odd]).all()
    i2[odd] = torch.tensor([-1, E, 1 << 30, -(1 << 31), E + 63], dtype=torch.int32, device=dev())[:, None]
    y = _run(x, w, i2, g, E, k, d, F, "bf16", False, weights)
    assert torch.equal(y[others], want[others])
