"""Refusals of the training step's entry points (found on the host, before any launch) and of their binding; the plain implementations
that the GPU tests compare with, against automatic differentiation and against differences."""
import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest
import torch

import paper_2503_00245_amd as pkg
from paper_2503_00245_amd import build as hip_build
from tests import training_oracle as to
from tests.training_cases import EXPERTS as LAYERS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3
P = [C.c_void_p(i << 20) for i in range(1, 20)]  # addresses that no launch will see
ODD = C.c_void_p((50 << 20) + 2)
HALF = C.c_void_p((51 << 20) + 8)
SHAPE = pkg.make_shape(8, 64, 136, 4, 2)
BIG = 1 << 40


def test_header_binding_and_library_agree():
    names = re.findall(r"MOE_API\s+[\w\s\*]+?\b(moe_\w+)\s*\(", open(os.path.join(ROOT, "include", "moe_training.h")).read())
    assert set(names) == set(pkg.TRAINING_EXPORTS)
    for n in names:
        assert getattr(pkg.lib(), n) is not None


def call(fn, defaults, **kw):
    args = dict(defaults, **kw)
    return getattr(pkg.lib(), fn)(*[C.byref(a) if isinstance(a, C.Structure) else a for a in args.values()])


DISPATCH = dict(shape=SHAPE, idx=P[0], weight=P[1], x=P[2], off=P[3], perm=P[4], inv=P[5], rows=P[6], ws=P[7], n=BIG, st=None)
DISPATCH_BACK = dict(shape=SHAPE, g=P[0], inv=P[1], x=P[2], w=P[3], gx=P[4], gw=P[5], st=None)
COLLECT = dict(shape=SHAPE, rows=P[0], inv=P[1], gate=P[2], res=P[3], y=P[4], st=None)
COLLECT_BACK = dict(shape=SHAPE, gy=P[0], rows=P[1], off=P[2], inv=P[3], gate=P[4], grad=P[5], gg=P[6], st=None)
LAYER = [("moe_dispatch", DISPATCH), ("moe_dispatch_backward", DISPATCH_BACK), ("moe_collect", COLLECT), ("moe_collect_backward", COLLECT_BACK)]


@pytest.mark.parametrize("fn,defaults", LAYER)
def test_rows_refuse_bad_shapes_and_pointers(fn, defaults):
    for bad, status in ((dict(top_k=0), INVALID), (dict(top_k=5), INVALID), (dict(n_tokens=-1), INVALID), (dict(d_model=60), UNSUPPORTED),
                        (dict(act_dtype=2), UNSUPPORTED), (dict(n_experts=65), UNSUPPORTED), (dict(n_tokens=1 << 23), UNSUPPORTED), (dict(flags=4), INVALID)):
        shape = pkg.make_shape(**dict(dict(n_tokens=8, d_model=64, d_ff=136, n_experts=4, top_k=2), **bad))
        assert call(fn, defaults, shape=shape) == status, bad
    needed = {"moe_dispatch": ("idx", "x", "off", "perm", "inv", "rows"), "moe_dispatch_backward": ("g", "inv", "gx", "x"),
              "moe_collect": ("rows", "inv", "gate", "y"), "moe_collect_backward": ("gy", "rows", "off", "inv", "gate")}[fn]
    for n in needed:
        assert call(fn, defaults, **{n: None}) == INVALID, n
    for n in defaults:
        if n not in ("shape", "ws", "n", "st"):
            assert call(fn, defaults, **{n: ODD}) == INVALID, n
            if n in ("x", "rows", "g", "gx", "res", "y", "gy", "grad"):
                assert call(fn, defaults, **{n: HALF}) == INVALID, n


def test_rows_refuse_overlap():
    assert call("moe_dispatch", DISPATCH, rows=P[2]) == INVALID
    assert call("moe_dispatch_backward", DISPATCH_BACK, gx=P[0]) == INVALID
    assert call("moe_dispatch_backward", DISPATCH_BACK, gx=P[2]) == INVALID
    assert call("moe_collect", COLLECT, y=P[0]) == INVALID
    assert call("moe_collect", COLLECT, y=P[3]) == INVALID
    assert call("moe_collect_backward", COLLECT_BACK, grad=P[0]) == INVALID


def test_rows_of_no_tokens_and_nothing_asked_for():
    none = pkg.make_shape(0, 64, 136, 4, 2)
    assert call("moe_dispatch_backward", DISPATCH_BACK, shape=none, g=None, inv=None, gx=None, x=None) == 0
    assert call("moe_collect", COLLECT, shape=none, rows=None, inv=None, gate=None, y=None) == 0
    assert call("moe_collect_backward", COLLECT_BACK, shape=none, gy=None) == 0
    assert call("moe_collect_backward", COLLECT_BACK, grad=None, gg=None) == 0
    assert call("moe_dispatch", DISPATCH, shape=none, off=None) == INVALID  # its bounds are an output all the same


def test_dispatch_of_many_pairs_needs_its_workspace():
    shape = pkg.make_shape(5000, 64, 136, 4, 2)
    need = 4 * 4 * 512  # counts of four experts in 500 chunks of ten tokens fit
    assert call("moe_dispatch", DISPATCH, shape=shape, n=16) == WORKSPACE
    assert call("moe_dispatch", DISPATCH, shape=shape, ws=None) == WORKSPACE
    assert call("moe_dispatch", DISPATCH, shape=shape, ws=ODD, n=need) == INVALID


def _weights(**kw):
    w = pkg.MoeWeights()
    for n in ("w_gate", "w_up", "w_down"):
        setattr(w, n, kw.get(n, 4096))
    return w


NEED = pkg.moe_training_workspace_bytes(SHAPE)
EXPERTS = dict(shape=SHAPE, w=_weights(), x=P[0], off=P[1], gy=P[2], gx=P[3], gg=P[4], gu=P[5], gd=P[6], ws=P[7], n=NEED, st=None)


def test_gradient_of_experts_refuses():
    fn = "moe_expert_ffn_backward"
    assert NEED > 0
    assert call(fn, EXPERTS, n=NEED - 1) == WORKSPACE
    assert call(fn, EXPERTS, ws=None) == WORKSPACE
    assert call(fn, EXPERTS, ws=HALF) == INVALID
    for n in ("x", "off", "gy"):
        assert call(fn, EXPERTS, **{n: None}) == INVALID
    for n in ("x", "gy", "gx", "gg", "gu", "gd"):
        assert call(fn, EXPERTS, **{n: HALF}) == INVALID
    assert call(fn, EXPERTS, off=ODD) == INVALID
    for n in ("w_gate", "w_up", "w_down"):
        assert call(fn, EXPERTS, w=_weights(**{n: 0})) == INVALID
        assert call(fn, EXPERTS, w=_weights(**{n: 4104})) == INVALID
        for out in ("gg", "gu", "gd"):
            assert call(fn, EXPERTS, w=_weights(**{n: EXPERTS[out].value})) == INVALID
    for n in ("gx", "gg", "gu", "gd"):
        assert call(fn, EXPERTS, **{n: P[0]}) == INVALID
        assert call(fn, EXPERTS, **{n: P[2]}) == INVALID
    assert call(fn, EXPERTS, gx=None, gg=None, gu=None, gd=None) == 0
    assert call(fn, EXPERTS, shape=pkg.make_shape(0, 64, 136, 4, 2), x=None, off=None, gy=None, gg=None, gu=None, gd=None) == 0
    for bad in (dict(rank=8), dict(d_ff=(1 << 18) + 8), dict(d_model=(1 << 18) + 8), dict(d_model=1 << 18, d_ff=1 << 18),
                dict(n_tokens=1 << 22, d_ff=1 << 14), dict(n_experts=64, d_model=1 << 16, d_ff=1 << 16)):
        shape = pkg.make_shape(**dict(dict(n_tokens=8, d_model=64, d_ff=136, n_experts=4, top_k=2), **bad))
        assert call(fn, EXPERTS, shape=shape) == UNSUPPORTED, bad
        assert pkg.moe_training_workspace_bytes(shape) == 0


@pytest.mark.parametrize("d,F,E,k,act", [(2048, 5632, 8, 2, 1), (64, 8, 64, 40, 1), (128, 256, 4, 2, 0), (8, 8, 1, 1, 0), (1440, 3840, 16, 4, 1)])
def test_a_workspace_for_more_tokens_holds_fewer(d, F, E, k, act):
    tokens = list(range(0, 1200)) + list(range(1200, 20000, 13))
    for size in (lambda t: pkg.moe_training_workspace_bytes(pkg.make_shape(t, d, F, E, k, act_dtype=act)), lambda t: pkg.moe_block_workspace_bytes(t, d),
                 lambda t: pkg.moe_block_stack_workspace_bytes(pkg.make_shape(t, d, F, E, k, act_dtype=act))):
        sizes = [size(t) for t in tokens]
        assert all(a <= b for a, b in zip(sizes, sizes[1:])) and sizes[1] > 0


def _block(**kw):
    b = pkg.binding.BlockStruct(1e-5, 1.0, 1.0, 0.0, None, None, None, None)
    for n, v in kw.items():
        setattr(b, n, v)
    return b


BLOCK = dict(block=_block(), T=4, d=64, dt=1, x=P[0], b=P[1], w=P[2], y=P[3], n=P[4], st=None)
BLOCK_NEED = pkg.moe_block_workspace_bytes(4, 64)
BACK = dict(block=_block(post_w=1 << 21), T=4, d=64, dt=1, gy=P[0], gn=P[1], y=P[2], b=P[3], w=P[4], gx=P[5], gb=P[6], gw=P[7], gp=P[8], gg=P[9], gt=P[10],
            ws=P[11], nb=BLOCK_NEED, st=None)


@pytest.mark.parametrize("fn,defaults", [("moe_block_norm", BLOCK), ("moe_block_norm_backward", BACK)])
def test_block_refuses_bad_numbers(fn, defaults):
    nan, inf = float("nan"), float("inf")
    for kw in (dict(eps=0.0), dict(eps=-1.0), dict(eps=nan), dict(eps=inf), dict(skip_scale=nan), dict(block_scale=inf), dict(dropout=-0.1), dict(dropout=1.0),
               dict(dropout=nan), dict(dropout=0.999999), dict(dropout=0.5), dict(dropout=0.5, rng=12), dict(post_w=8), dict(gate=8), dict(token_gate=2)):
        assert call(fn, defaults, block=_block(**kw)) == INVALID, kw
    for kw, status in ((dict(T=-1), INVALID), (dict(d=0), INVALID), (dict(d=60), UNSUPPORTED), (dict(d=32776), UNSUPPORTED), (dict(T=1 << 24), UNSUPPORTED),
                       (dict(dt=2), UNSUPPORTED)):
        assert call(fn, defaults, **kw) == status, kw
    for n in ("x", "b", "w", "y", "n", "gy", "gn", "gx", "gb"):
        if n in defaults:
            assert call(fn, defaults, **{n: HALF}) == INVALID, n
    assert getattr(pkg.lib(), fn)(None, *list(defaults.values())[1:]) == INVALID


def test_block_refuses_what_does_not_go_together():
    fn = "moe_block_norm"
    for kw in (dict(b=None), dict(y=None), dict(w=None), dict(n=None), dict(x=None), dict(b=None, y=None, w=None, n=None), dict(n=P[0]), dict(n=P[1]), dict(n=P[3]),
               dict(y=P[1])):
        assert call(fn, BLOCK, **kw) == INVALID, kw
    assert call(fn, BLOCK, T=0) == 0
    fn = "moe_block_norm_backward"
    for kw in (dict(gn=None), dict(w=None), dict(y=None), dict(b=None), dict(gb=None), dict(gy=None, gn=None, w=None, gw=None), dict(gx=None), dict(gx=P[1]),
               dict(gx=P[2]), dict(gx=P[3]), dict(gb=P[0]), dict(gb=P[5]), dict(gb=P[3]), dict(b=None, gb=None), dict(b=None, gb=None, gp=None, gt=None),
               dict(b=None, gb=None, gp=None, gg=None), dict(b=None, gb=None, gp=None, gg=None, gt=None, gn=None, w=None, gw=None),
               dict(gn=None, w=None), dict(gw=ODD), dict(gp=ODD), dict(gg=ODD), dict(gt=ODD), dict(ws=HALF)):
        assert call(fn, BACK, **kw) == INVALID, kw
    assert call(fn, BACK, block=_block()) == INVALID  # grad_post_w without post_w
    assert call(fn, BACK, nb=BLOCK_NEED - 1) == WORKSPACE
    assert call(fn, BACK, ws=None) == WORKSPACE
    assert call(fn, BACK, T=0, gw=None, gp=None, gg=None, ws=None) == 0
    for bad in ((-1, 64), (1 << 24, 64), (4, 0), (4, 12), (4, 32776)):
        assert pkg.moe_block_workspace_bytes(*bad) == 0


def test_stack_refuses():
    w = pkg.MoeWeights()
    for n in ("router_w", "w_gate", "w_up", "w_down"):
        setattr(w, n, 4096)
    need = pkg.moe_block_stack_workspace_bytes(SHAPE)
    layers, blocks, norms = (pkg.MoeWeights * 2)(w, w), (pkg.binding.BlockStruct * 2)(_block(), _block()), (C.c_void_p * 2)(4096, 4096)
    args = dict(shape=SHAPE, layers=layers, blocks=blocks, norms=norms, n=2, x=P[0], y=P[1], trace=None, ws=P[2], bytes=need, st=None)
    fn = "moe_block_stack_forward"
    assert need > pkg.moe_workspace_bytes(SHAPE)
    assert call(fn, args, n=0) == INVALID
    for n in ("layers", "blocks", "norms", "x", "y"):
        assert call(fn, args, **{n: None}) == INVALID, n
    assert call(fn, args, y=P[0]) == INVALID
    assert call(fn, args, bytes=need - 1) == WORKSPACE
    assert call(fn, args, ws=None) == WORKSPACE
    assert call(fn, args, norms=(C.c_void_p * 2)(4096, None)) == INVALID
    assert call(fn, args, norms=(C.c_void_p * 2)(4096, 4104)) == INVALID
    assert call(fn, args, blocks=(pkg.binding.BlockStruct * 2)(_block(), _block(eps=0.0))) == INVALID
    assert call(fn, args, layers=(pkg.MoeWeights * 2)(w, pkg.MoeWeights())) == INVALID
    assert call(fn, args, shape=pkg.make_shape(8, 64, 136, 4, 2, flags=pkg.FLAG_RESIDUAL)) == INVALID
    assert call(fn, args, shape=pkg.make_shape(0, 64, 136, 4, 2)) == 0
    assert pkg.moe_block_stack_workspace_bytes(pkg.make_shape(8, 32776, 136, 4, 2)) == 0


def test_binding_refuses():
    shape = pkg.make_shape(3, 16, 8, 4, 2, act_dtype=pkg.MOE_F32)
    t = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt)  # noqa: E731
    i32 = torch.int32
    with pytest.raises(TypeError):
        pkg.moe_dispatch(shape, t(3, 2, dt=torch.int64), None, t(3, 16), t(5, dt=i32), t(6, dt=i32), t(6, dt=i32), t(6, 16))
    with pytest.raises(ValueError):
        pkg.moe_dispatch(shape, t(3, 2, dt=i32), None, t(3, 16), t(4, dt=i32), t(6, dt=i32), t(6, dt=i32), t(6, 16))
    with pytest.raises(ValueError):
        pkg.moe_dispatch(shape, t(3, 2, dt=i32), None, t(16, 3).T, t(5, dt=i32), t(6, dt=i32), t(6, dt=i32), t(6, 16))
    with pytest.raises(TypeError):
        pkg.moe_collect(shape, t(6, 16, dt=torch.bfloat16), t(6, dt=i32), t(3, 2), None, t(3, 16))
    with pytest.raises(ValueError):
        pkg.moe_collect(shape, t(6, 16), t(5, dt=i32), t(3, 2), None, t(3, 16))
    with pytest.raises(ValueError):
        pkg.moe_expert_ffn_backward(shape, pkg.MoeWeights(), t(6, 16), t(5, dt=i32), t(6, 16), t(6, 16), t(4, 16, 8))
    with pytest.raises(ValueError):
        pkg.make_block(rng=t(3, dt=torch.int64))
    with pytest.raises(TypeError):
        pkg.make_block(post_w=t(16, dt=torch.bfloat16))
    with pytest.raises(ValueError):
        pkg.moe_block_norm(pkg.make_block(post_w=t(24)), t(3, 16), t(3, 16), None, t(3, 16), None)
    with pytest.raises(ValueError):
        pkg.make_block(post_w=t(16), gate=t(24))
    with pytest.raises(ValueError):
        pkg.moe_block_norm(pkg.make_block(token_gate=t(4)), t(3, 16), t(3, 16), None, t(3, 16), None)
    with pytest.raises(ValueError):
        pkg.moe_block_stack_forward(shape, [pkg.MoeWeights()], [], [], t(3, 16), t(3, 16))


def test_binding_refuses_host_tensors():
    # they have the right types and shapes, and nothing but the device tells them from what the library takes
    shape = pkg.make_shape(3, 16, 8, 4, 2, act_dtype=pkg.MOE_F32)
    x, rows, gate = torch.zeros(3, 16), torch.zeros(6, 16), torch.zeros(3, 2)
    idx, inv, off = (torch.zeros(*s, dtype=torch.int32) for s in ((3, 2), (6,), (5,)))
    w = torch.zeros(4, 8, 16)
    calls = [lambda: pkg.moe_dispatch(shape, idx, None, x, off, inv, inv.clone(), rows, torch.zeros(1 << 16)),
             lambda: pkg.moe_dispatch_backward(shape, rows, inv, None, gate, x), lambda: pkg.moe_collect(shape, rows, inv, gate, None, x),
             lambda: pkg.moe_collect_backward(shape, x, rows, off, inv, gate, rows.clone(), gate.clone()),
             lambda: pkg.moe_expert_ffn_backward(shape, pkg.MoeWeights(), rows, off, rows, rows.clone(), w, workspace=torch.zeros(1 << 16)),
             lambda: pkg.moe_block_norm(pkg.make_block(), x, x, None, x.clone(), None),
             lambda: pkg.moe_block_norm_backward(pkg.make_block(), x, None, None, x, None, x.clone(), x.clone()),
             lambda: pkg.moe_block_stack_forward(shape, [pkg.MoeWeights()], [pkg.make_block()], [torch.zeros(16)], x, x.clone())]
    for call_ in calls:
        with pytest.raises(ValueError, match="GPU"):
            call_()


def test_the_tested_layers_reach_every_tile_of_the_experts_gradient(tmp_path):
    exe = str(tmp_path / "check")
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", hip_build.CSRC, os.path.join(ROOT, "tests", "expert_grad_plan_check.cpp"), "-o", exe], check=True)
    plans = [tuple(map(int, subprocess.run([exe, str(T * k), str(E), str(d), str(F)], capture_output=True, text=True, check=True, timeout=60).stdout.split()))
             for T, d, F, E, k in LAYERS if d > 128 and F > 128]  # (narrower layers take the kernels for any size)
    assert {p[:2] for p in plans} == {(256, 96), (256, 128), (128, 128)}
    assert {p[2] for p in plans} == {1, 2, 3, 4}
    assert {p[3] for p in plans} == {0, 1}


# ---- the plain implementations themselves ---------------------------------------------------------------------------

def _f64(g, *shape):
    return torch.randn(*shape, generator=g, dtype=torch.float64)


def test_oracle_of_the_experts_gradient():
    g = torch.Generator().manual_seed(1)
    offsets, d, F = [0, 3, 3, 7], 8, 16
    x, gy = _f64(g, 7, d), _f64(g, 7, d)
    w = [_f64(g, 3, F, d), _f64(g, 3, F, d), _f64(g, 3, d, F)]

    def forward(x, wg, wu, wd):
        return torch.cat([(torch.nn.functional.silu(x[lo:hi] @ wg[e].T) * (x[lo:hi] @ wu[e].T)) @ wd[e].T
                          for e, (lo, hi) in enumerate(zip(offsets, offsets[1:]))])
    leaves = [t.clone().requires_grad_(True) for t in (x, *w)]
    want = torch.autograd.grad(forward(*leaves), leaves, gy)
    got = to.experts_grad(x, offsets, gy, *w, torch.float32)
    for a, b in zip(got, want):
        assert torch.allclose(a[0], b, rtol=1e-12, atol=1e-12)
    # against differences, in a direction of every input (error of the second order, 1e-10, over the step)
    step = 1e-5
    dirs = [_f64(g, *t.shape) for t in (x, *w)]
    up, down = (forward(*[t + s * step * v for t, v in zip((x, *w), dirs)]) for s in (1, -1))
    slope = ((up - down) * gy).sum() / (2 * step)
    assert abs(slope - sum((a[0] * v).sum() for a, v in zip(got, dirs))) < 1e-6 * abs(slope) + 1e-6


@pytest.mark.parametrize("what", ["", "p", "pgt"])
def test_oracle_of_the_blocks_gradient(what):
    g = torch.Generator().manual_seed(2)
    T, d = 5, 16
    p = {"x": _f64(g, T, d), "b": _f64(g, T, d), "open_w": _f64(g, d)}
    for letter, n, size in (("p", "post_w", d), ("g", "gate", d), ("t", "token_gate", T)):
        if letter in what:
            p[n] = _f64(g, size)
    cfg = {"eps": 1e-3, "skip_scale": 0.5, "block_scale": 2.0, "dropout": 0.25}
    mask = to.kept(T, d, 0.25, (3, 4))
    gy, gn = _f64(g, T, d), _f64(g, T, d)

    def loss(q):
        z = q["b"] if "post_w" not in q else q["b"] / torch.sqrt((q["b"] ** 2).mean(-1, keepdim=True) + 1e-3) * q["post_w"]
        z = z * mask * (4 / 3) * q.get("gate", torch.ones(d)) * q.get("token_gate", torch.ones(T))[:, None]
        y = 0.5 * q["x"] + 2.0 * z
        return (y * gy).sum() + (y / torch.sqrt((y ** 2).mean(-1, keepdim=True) + 1e-3) * q["open_w"] * gn).sum(), y.detach()
    leaves = {n: v.clone().requires_grad_(True) for n, v in p.items()}
    value, y = loss(leaves)
    want = dict(zip(leaves, torch.autograd.grad(value, list(leaves.values()))))
    got = to.block_grad({**cfg, **p}, gy, gn, y, p["b"], p["open_w"], mask, torch.float32)
    for n in p:
        assert torch.allclose(got[n][0], want[n], rtol=1e-10, atol=1e-10), n
    step = 1e-6
    dirs = {n: _f64(g, *v.shape) for n, v in p.items()}
    slope = (loss({n: v + step * dirs[n] for n, v in p.items()})[0] - loss({n: v - step * dirs[n] for n, v in p.items()})[0]) / (2 * step)
    assert abs(slope - sum((got[n][0] * dirs[n]).sum() for n in p)) < 1e-6 * abs(slope) + 1e-6


def test_philox_gives_the_published_vectors():
    # the published vectors of Philox4x32-10
    f = 0xFFFFFFFF
    assert to.philox((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert to.philox((f,) * 4, (f, f)) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert to.philox((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0)) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]
    assert np.isclose(to.kept(64, 256, 0.25, (5, 7)).double().mean(), 0.75, atol=5 * (0.75 * 0.25 / (64 * 256)) ** 0.5)
