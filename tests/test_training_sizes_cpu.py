"""What a call around the experts needs is told for every shape that it accepts: sizes of workspaces, and which forms of the kernels the GPU tests reach."""
import ctypes as C
import os
import subprocess

import pytest
import torch

import paper_2503_00245_amd as pkg
from paper_2503_00245_amd import build as hip_build
from tests.block_cases import WIDE, WIDE_MANY
from tests.rows_cases import ROWS
from tests.test_block_gpu import SHAPES as BLOCKS
from tests.test_training_gpu import SIZES

WORKSPACE = -3
P = [C.c_void_p(i << 20) for i in range(1, 9)]  # addresses that no launch will see


def dispatch_on_the_host(shape, nbytes):
    """moe_dispatch's answer where its workspace has nbytes, but is misaligned: it is refused after its size has been looked at"""
    args = [C.byref(shape), P[0], None, P[1], P[2], P[3], P[4], P[5], C.c_void_p((7 << 20) + 2), nbytes, None]
    return pkg.lib().moe_dispatch(*args)


# weight-decomposed experts, experts with a shared base, experts wider than the gradient takes, more rows than it takes
LAYERS = [dict(rank=64), dict(rank=64, flags=pkg.FLAG_SHARED_BASE), dict(d_ff=(1 << 18) + 8), dict(d_model=(1 << 18) + 8), dict(n_tokens=1 << 20, d_model=1024, d_ff=28672),
          dict(n_tokens=(1 << 23) - 1), dict(n_experts=64, top_k=64), dict(n_experts=1, top_k=1, n_tokens=9000), dict(act_dtype=pkg.MOE_F32, rank=8)]


@pytest.mark.parametrize("kw", LAYERS)
def test_dispatch_tells_its_workspace_for_every_shape_it_takes(kw):
    shape = pkg.make_shape(**dict(dict(n_tokens=5000, d_model=64, d_ff=136, n_experts=8, top_k=2), **kw))
    need = pkg.moe_dispatch_workspace_bytes(shape)
    assert need > 0
    assert dispatch_on_the_host(shape, 4) == WORKSPACE
    assert dispatch_on_the_host(shape, need) == -1  # large enough; refused for its alignment
    assert pkg.alloc_dispatch_workspace(shape, "cpu").nbytes == need
    gradient = pkg.moe_training_workspace_bytes(shape)
    assert gradient == 0 or gradient >= need  # (where the gradient takes the shape, its workspace serves both)


def test_sizes_of_dispatch_refuse_and_do_not_fall():
    for kw in (dict(top_k=0), dict(n_tokens=-1), dict(d_model=60), dict(n_experts=65), dict(n_tokens=1 << 23), dict(flags=4)):
        shape = pkg.make_shape(**dict(dict(n_tokens=8, d_model=64, d_ff=136, n_experts=4, top_k=2), **kw))
        assert pkg.moe_dispatch_workspace_bytes(shape) == 0, kw
        with pytest.raises(pkg.MoeError):
            pkg.alloc_dispatch_workspace(shape, "cpu")
    for E, k in ((1, 1), (3, 2), (8, 2), (60, 6), (64, 64)):
        sizes = [pkg.moe_dispatch_workspace_bytes(pkg.make_shape(t, 64, 136, E, k, rank=64)) for t in [*range(3000), *range(3000, 200000, 97)]]
        assert sizes[0] > 0 and all(a <= b for a, b in zip(sizes, sizes[1:]))
    assert pkg.alloc_dispatch_workspace(pkg.make_shape(0, 64, 136, 4, 2), "cpu").dtype is torch.uint8


def _plans(tmp_path, source, cases):
    exe = str(tmp_path / "check")
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", hip_build.CSRC, os.path.join(os.path.dirname(__file__), source), "-o", exe], check=True)
    return {c: tuple(map(int, subprocess.run([exe, *map(str, c)], capture_output=True, text=True, check=True, timeout=60).stdout.split())) for c in cases}


def test_the_tested_rows_reach_every_form_of_their_kernels(tmp_path):
    plans = _plans(tmp_path, "rows_plan_check.cpp", ROWS + SIZES)
    assert {p[:2] for p in plans.values()} == {(w, n) for w in (1, 2, 4) for n in (0, 1, 2, 4, 8)}
    assert {p[2] for p in plans.values()} == {0, 1, 2}
    # by ballots, of every number of experts that is counted so: chunks that start within a wave's 64 keys, and keys for more than one wave
    for E in (1, 2, 3, 4):
        starts = [[chunk * i % 64 for i in range(chunks)] for c, (_, _, how, chunk, chunks) in plans.items() if how == 0 and c[2] == E and c[0] * c[3] > 64]
        assert any(any(at) for at in starts), E


def test_the_tested_blocks_reach_every_plan(tmp_path):
    plans = _plans(tmp_path, "block_plan_check.cpp", WIDE + WIDE_MANY + BLOCKS)
    every = {(w, 1) for w in (1, 2, 3, 4, 8)} | {(8, 2), (16, 2), (16, 3), (16, 4)}
    assert {p[:2] for p in plans.values()} == every
    wide = [p for p in plans.values() if p[0] == 16]
    for chunks in (2, 3, 4):  # workgroups that take several rows in turn: of a gradient with sums, and of the forward pass and a gradient without
        assert any(p[1] == chunks and p[2] > p[4] for p in wide)
        assert any(p[1] == chunks and p[2] > p[3] for p in wide)
