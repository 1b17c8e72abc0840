"""Refusals of the routing-from-logits and 4-bit entry points (found on the host, before any launch), and of their
binding; the plain implementations that the GPU tests compare with, against each other."""
import ctypes as C
import os
import re

import numpy as np
import pytest
import torch

import paper_2503_00245_amd as pkg
from tests import operators_oracle as oo

OK, OK2, OK3 = C.c_void_p(1 << 20), C.c_void_p(1 << 21), C.c_void_p(3 << 20)
INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3


def _route(cfg=None, T=4, E=16, k=2, logits=OK, bias=None, idx=OK2, gate=OK2, scores=None, **kw):
    c = cfg or pkg.make_route_config(**kw)
    return pkg.lib().moe_route_scored(C.byref(c), T, E, k, logits, bias, idx, gate, scores, None)


def _grad(T=4, E=16, k=2, logits=OK, idx=OK2, dg=OK2, ds=None, out=OK3, **kw):
    return pkg.lib().moe_route_scored_backward(C.byref(pkg.make_route_config(**kw)), T, E, k, logits, idx, dg, ds, out, None)


@pytest.mark.parametrize("call", [_route, _grad])
def test_routing_refuses_bad_configurations(call):
    assert call(T=0) == 0  # no tokens: nothing to do
    assert call(T=-1) == INVALID
    assert call(E=0) == INVALID
    assert call(k=0) == INVALID
    assert call(k=17) == INVALID
    assert call(score=2) == INVALID
    assert call(n_groups=0) == INVALID
    assert call(n_groups=3) == INVALID                                   # 16 experts
    assert call(n_groups=4, groups_kept=0) == INVALID
    assert call(n_groups=4, groups_kept=5) == INVALID
    assert call(n_groups=4, groups_kept=1, group_top=3) == INVALID
    assert call(n_groups=16, groups_kept=8, group_top=2) == INVALID      # groups of one
    assert call(n_groups=4, groups_kept=1, k=5) == INVALID               # 4 eligible experts
    assert call(scale=float("nan")) == INVALID
    assert call(scale=float("inf")) == INVALID
    assert call(E=513) == UNSUPPORTED
    assert call(E=512, k=65) == UNSUPPORTED
    assert call(E=512, n_groups=128, groups_kept=8) == UNSUPPORTED
    assert call(logits=None) == INVALID
    assert call(logits=C.c_void_p(2)) == INVALID
    assert call(idx=None) == INVALID


def test_routing_refuses_bad_pointers():
    assert _route(gate=None) == INVALID
    assert _route(bias=C.c_void_p(6)) == INVALID
    assert _route(scores=OK) == INVALID     # in place of the logits
    assert _grad(dg=None) == INVALID
    assert _grad(out=None) == INVALID
    assert _grad(out=OK) == INVALID
    assert _grad(ds=OK3) == INVALID
    assert pkg.lib().moe_route_scored(None, 4, 16, 2, OK, None, OK2, OK2, None, None) == INVALID


def test_quantisation_refuses():
    L = pkg.lib()
    for fn in (lambda x, r, c, d, a, b: L.moe_mxfp4_quantize(x, r, c, d, a, b, None), lambda x, r, c, d, a, b: L.moe_mxfp4_dequantize(a, b, r, c, d, x, None)):
        assert fn(OK, 0, 32, 1, OK, OK) == 0
        assert fn(None, 0, 32, 1, None, None) == 0
        assert fn(OK, -1, 32, 1, OK, OK) == INVALID
        assert fn(OK, 1, 0, 1, OK, OK) == INVALID
        assert fn(OK, 1, 36, 1, OK, OK) == UNSUPPORTED
        assert fn(OK, 1, 32, 2, OK, OK) == UNSUPPORTED
        assert fn(OK, 1 << 40, 32, 1, OK, OK) == UNSUPPORTED
        assert fn(None, 1, 32, 1, OK, OK) == INVALID
        assert fn(OK, 1, 32, 1, None, OK) == INVALID
        assert fn(OK, 1, 32, 1, OK, None) == INVALID
        assert fn(C.c_void_p(8), 1, 32, 1, OK, OK) == INVALID
        assert fn(OK, 1, 32, 1, C.c_void_p(6), OK) == INVALID
    assert L.moe_mxfp4_packed_bytes(1, 8, 8) == 4096 + 256
    assert L.moe_mxfp4_packed_bytes(8, 40, 264) == 8 * 2 * 2 * 4352
    for bad in ((0, 8, 8), (1, 0, 8), (1, 8, 0), (1, 12, 8), (1, 8, 12), (-1, 8, 8)):
        assert L.moe_mxfp4_packed_bytes(*bad) == 0
    assert L.moe_mxfp4_pack(OK, OK, 1, 8, 12, OK, None) == UNSUPPORTED
    assert L.moe_mxfp4_pack(None, OK, 1, 8, 8, OK, None) == INVALID
    assert L.moe_mxfp4_pack(OK, OK, 1, 8, 8, C.c_void_p(8), None) == INVALID


def _weights(**kw):
    w = pkg.binding.Mxfp4WeightsStruct()
    for n in ("router_w", "gate", "up", "down"):
        setattr(w, n, kw.get(n, 4096))
    return w


def test_experts_refuse():
    L = pkg.lib()
    sh = pkg.make_shape(8, 256, 512, 4, 2)
    n = pkg.moe_mxfp4_workspace_bytes(sh)
    assert n > 0
    cfg = pkg.make_route_config()

    def experts(shape=sh, w=_weights(), x=OK, idx=OK2, gate=OK2, y=OK3, ws=OK, nbytes=n):
        return L.moe_mxfp4_experts(C.byref(shape), C.byref(w), x, idx, gate, y, ws, nbytes, None)

    def forward(shape=sh, w=_weights(), x=OK, idx=OK2, gate=OK2, y=OK3, ws=OK, nbytes=n):
        return L.moe_mxfp4_forward(C.byref(shape), C.byref(cfg), C.byref(w), x, y, idx, gate, None, ws, nbytes, None)

    for call in (experts, forward):
        assert call(shape=pkg.make_shape(0, 256, 512, 4, 2)) == 0
        assert call(nbytes=n - 1) == WORKSPACE
        assert call(x=None) == INVALID
        assert call(y=OK) == INVALID
        assert call(y=C.c_void_p(8)) == INVALID
        assert call(ws=None) == INVALID
        assert call(ws=C.c_void_p(24)) == INVALID
        assert call(idx=C.c_void_p(24)) == INVALID
        assert call(w=_weights(up=None)) == INVALID
        assert call(w=_weights(down=4100)) == INVALID
        for bad, status in ((pkg.make_shape(8, 252, 512, 4, 2), UNSUPPORTED), (pkg.make_shape(8, 256, 512, 65, 2), UNSUPPORTED),
                            (pkg.make_shape(8, 256, 512, 4, 5), INVALID), (pkg.make_shape(8, 256, 512, 4, 2, rank=64), UNSUPPORTED),
                            (pkg.make_shape(8, 256, 512, 4, 2, rank=64, flags=1), INVALID), (pkg.make_shape(8, 256, 512, 4, 2, act_dtype=3), UNSUPPORTED),
                            (pkg.make_shape(8, 256, (1 << 18) + 8, 4, 2), UNSUPPORTED), (pkg.make_shape(8, (1 << 18) + 8, 512, 4, 2), UNSUPPORTED)):
            assert call(shape=bad) == status
            assert pkg.moe_mxfp4_workspace_bytes(bad) == 0
    assert experts(idx=None) == INVALID
    assert experts(gate=None) == INVALID
    assert forward(w=_weights(router_w=None)) == INVALID


def test_a_workspace_of_the_largest_batch_serves_every_smaller_one():
    for d, F, E, k in ((256, 512, 4, 2), (1440, 3840, 8, 2), (64, 96, 64, 8), (8, 8, 1, 1)):
        sizes = [pkg.moe_mxfp4_workspace_bytes(pkg.make_shape(T, d, F, E, k)) for T in list(range(0, 600)) + list(range(600, 20000, 97))]
        assert all(a <= b for a, b in zip(sizes, sizes[1:]))


def test_the_binding_refuses_other_types_shapes_and_orders():
    cfg = pkg.make_route_config()
    l, idx, gate = torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    with pytest.raises(TypeError):
        pkg.moe_route_scored(cfg, l.double(), None, idx, gate)
    with pytest.raises(TypeError):
        pkg.moe_route_scored(cfg, l, None, idx.long(), gate)
    with pytest.raises(ValueError):
        pkg.moe_route_scored(cfg, l, None, idx, gate[:3])
    with pytest.raises(ValueError):
        pkg.moe_route_scored(cfg, l, torch.zeros(7), idx, gate)
    with pytest.raises(ValueError):
        pkg.moe_route_scored(cfg, torch.zeros(8, 4).T, None, idx, gate)
    with pytest.raises(ValueError):
        pkg.moe_route_scored_backward(cfg, l, idx, gate, torch.zeros(4, 7), torch.zeros(4, 8))
    with pytest.raises(ValueError):
        pkg.moe_mxfp4_quantize(torch.zeros(4, 64), torch.zeros(4, 31, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8))
    with pytest.raises(TypeError):
        pkg.moe_mxfp4_quantize(torch.zeros(4, 64), torch.zeros(4, 32, dtype=torch.int8), torch.zeros(4, 2, dtype=torch.uint8))
    with pytest.raises(TypeError):
        pkg.moe_mxfp4_quantize(torch.zeros(4, 64).half(), torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8))
    with pytest.raises(ValueError):
        pkg.moe_mxfp4_pack(torch.zeros(1, 8, 16, dtype=torch.uint8), torch.zeros(1, 8, 2, dtype=torch.uint8))


def test_library_exports_every_symbol_of_the_header():
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "moe_quantised.h")).read()
    names = re.findall(r"MOE_API\s+(?:int|size_t)\s+(moe_\w+)\(", text)
    assert sorted(names) == sorted(pkg.QUANTISED_EXPORTS)
    assert all(hasattr(pkg.lib(), n) for n in names)


def test_plain_quantisation_is_the_nearest_value():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((200, 72)) * np.exp(rng.standard_normal((200, 1)))
    c, b = oo.quantize(x)
    v = oo.values(c, b)
    grid = np.concatenate([oo.GRID, -oo.GRID])
    for r in range(0, 200, 7):
        for i in range(72):
            s = 2.0 ** (int(b[r, i // 32]) - 127)
            assert abs(v[r, i] - x[r, i]) == np.abs(grid * s - x[r, i]).min()
        for blk in range(3):
            big = np.abs(x[r, 32 * blk:32 * blk + 32]).max() / 2.0 ** (int(b[r, blk]) - 127)
            assert 4 <= big < 8


def test_plain_gradient_is_the_derivative():
    rng = np.random.default_rng(1)
    E, k, h = 12, 3, 1e-6
    for sigmoid in (False, True):
        for renorm in (False, True):
            l = rng.standard_normal((1, E))
            idx, _, _ = oo.route(l, None, k, sigmoid, 1, 1, 1, renorm, 2.5)
            dg, ds = rng.standard_normal((1, k)), rng.standard_normal((1, E))

            def f(z):
                s = oo.scores(z, sigmoid)
                w = s[0, idx[0]]
                return (2.5 * (w / w.sum() if renorm else w) * dg).sum() + (s * ds).sum()
            got, _ = oo.route_backward(l, idx, dg, ds, sigmoid, renorm, 2.5)
            for e in range(E):
                p, m = l.copy(), l.copy()
                p[0, e] += h
                m[0, e] -= h
                assert abs((f(p) - f(m)) / (2 * h) - got[0, e]) < 1e-8


def test_experts_refuse_more_tiles_than_a_launch_has():
    # 65536 groups of 256 rows by 128 tiles of 128 hidden, or of 256 output, columns: 2^23 workgroups of 512 threads
    T, L = (1 << 24) - 1, pkg.lib()
    for wide, d, F in ((True, 8, 1 << 14), (False, 8, (1 << 14) - 1024), (True, 1 << 15, 8), (False, (1 << 15) - 2048, 8)):
        shape = pkg.make_shape(T, d, F, 1, 1)
        n = pkg.moe_mxfp4_workspace_bytes(shape)
        assert (n == 0) == wide
        status = UNSUPPORTED if wide else WORKSPACE
        assert L.moe_mxfp4_experts(C.byref(shape), C.byref(_weights()), OK, OK2, OK2, OK3, OK, 1, None) == status
        cfg = pkg.make_route_config()
        assert L.moe_mxfp4_forward(C.byref(shape), C.byref(cfg), C.byref(_weights()), OK, OK3, OK2, OK2, None, OK, 1, None) == status


@pytest.mark.parametrize("name", ["router_b", "select_bias"])
def test_the_whole_layer_refuses_biases_between_values(name):
    sh, cfg, w = pkg.make_shape(8, 256, 512, 4, 2), pkg.make_route_config(), _weights()
    for at, status in ((4098, INVALID), (4100, WORKSPACE)):  # (4-byte alignment is enough: the workspace is what is wrong then)
        setattr(w, name, at)
        assert pkg.lib().moe_mxfp4_forward(C.byref(sh), C.byref(cfg), C.byref(w), OK, OK3, OK2, OK2, None, OK, 1, None) == status
