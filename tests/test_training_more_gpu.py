"""Layers whose experts have no gradient here, and forms of the kernels that ordinary sizes do not reach, against the plain implementations in 64 bits
(training_oracle)."""
import pytest
import torch

import paper_2503_00245_amd as pkg
from tests import test_block_gpu as block
from tests import test_training_gpu as base
from tests import training_oracle as to
from tests.block_cases import WIDE, WIDE_MANY
from tests.rows_cases import ROWS
from tests.test_training_gpu import dev, dispatched, gen, picks, rnd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("flags", [0, pkg.FLAG_SHARED_BASE])
def test_rows_of_a_weight_decomposed_layer(flags):
    # moe_dispatch takes layers that the experts' gradient refuses, and tells its workspace for them
    T, d, E, k = 5001, 40, 8, 2
    g = gen(8)
    shape = pkg.make_shape(T, d, 136, E, k, rank=64, act_dtype=pkg.MOE_F32, flags=flags)
    assert pkg.moe_training_workspace_bytes(shape) == 0
    ws = pkg.alloc_dispatch_workspace(shape, dev())
    idx, x, gate = picks(g, T, k, E, 0.2), rnd(g, T, d), rnd(g, T, k)
    off, perm, inv, rows = dispatched(shape, idx, None, x, ws)
    w_off, w_perm, w_inv = to.sort(idx, E)
    assert off.tolist() == w_off and perm.tolist() == w_perm and inv.tolist() == w_inv
    to.near(rows, to.dispatch(x, None, w_perm, k, torch.float32), "rows")
    y = torch.full((T, d), float("nan"), device=dev())
    pkg.moe_collect(shape, rows, inv, gate.to(dev()), None, y)
    to.near(y, to.gather_sum(rows.cpu(), inv.cpu().view(T, k), gate, None, torch.float32), "y")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,d,E,k", ROWS)
def test_forms_of_dispatch_and_its_gradient(T, d, E, k, dtype):
    base.test_dispatch_and_its_gradient(T, d, E, k, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,d,E,k", ROWS)
def test_forms_of_collect_and_its_gradient(T, d, E, k, dtype):
    base.test_collect_and_its_gradient(T, d, E, k, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("what", ["", "pgt"])
@pytest.mark.parametrize("T,d", WIDE)
def test_block_of_wide_rows(T, d, what, dtype):
    block.test_block(T, d, what, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,d", WIDE_MANY)
def test_wide_rows_do_not_depend_on_the_rows_around_them(T, d, dtype):
    block.test_rows_do_not_depend_on_the_rows_around_them(T, d, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,d,p", [(3, 10240, 0.1), (2, 20000, 0.3), (2, 32768, 0.5)])
def test_dropout_of_wide_rows(T, d, p, dtype):
    block.test_dropout(T, d, p, dtype)
