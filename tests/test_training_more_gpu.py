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
from tests.test_training_gpu import CODE, DTYPES, dev, dispatched, gen, picks, rnd

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


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 33])
def test_stack_of_blocks_with_dropout(T, dtype):
    # every block drops by its own numbers, in eager calls and in replays of a graph; blocks with the same numbers drop the same places
    dt, d, F, E, k, L, p = DTYPES[dtype], 128, 256, 8, 2, 3, 0.25
    g = gen(T + 40)
    shape = pkg.make_shape(T, d, F, E, k, act_dtype=CODE[dt])
    kept = [{n: rnd(g, *s, std=s[-1] ** -0.5, dtype=torch.float32 if n == "router_w" else dt).to(dev())
             for n, s in (("router_w", (E, d)), ("w_gate", (E, F, d)), ("w_up", (E, F, d)), ("w_down", (E, d, F)))} for _ in range(L)]
    layers = [pkg.make_weights(w) for w in kept]
    cfgs = [block.config(g, T, d, w, p) for w in ("pg", "pgt", "")]
    numbers = [torch.tensor([77, i], device=dev()) for i in range(L)]
    blocks = [pkg.make_block(**{n: block.on(v) if torch.is_tensor(v) else v for n, v in {**c, "rng": r}.items()}) for c, r in zip(cfgs, numbers)]
    open_w = [block.on(1 + rnd(g, d, std=0.2)) for _ in range(L)]
    x = block.on(rnd(g, T, d, dtype=dt))
    y, ws = torch.empty_like(x), pkg.alloc_block_stack_workspace(shape, dev())
    lws = pkg.alloc_workspace(shape, dev())

    def one_by_one():
        cur, masks = x.clone(), []
        for l in range(L):
            n, b, nxt = (torch.empty_like(x) for _ in range(3))
            pkg.moe_block_norm(blocks[max(l - 1, 0)], cur, None, open_w[l], None, n)
            pkg.moe_forward(shape, layers[l], n, b, None, None, lws)
            pkg.moe_block_norm(blocks[l], cur, b, None, nxt, None)
            masks.append(to.kept(T, d, p, numbers[l].tolist()))
            to.near(nxt, to.block(cfgs[l], cur.cpu(), b.cpu(), masks[-1], dt), "y")
            cur = nxt
        return cur, masks

    def run():
        pkg.moe_block_stack_forward(shape, layers, blocks, open_w, x, y, None, ws)
    run()
    want, masks = one_by_one()
    assert torch.equal(y, want)
    assert not any(torch.equal(masks[i], masks[j]) for i in range(L) for j in range(i))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for step in range(3):
        for r in numbers:
            r[1] += L
        if step == 2:  # the same numbers for every block
            for r in numbers:
                r.copy_(torch.tensor([5, 6]))
        graph.replay()
        torch.cuda.synchronize()
        replayed = y.clone()
        want, masks = one_by_one()
        assert torch.equal(replayed, want)
        assert torch.equal(masks[0], masks[1]) == (step == 2)


def _factored_forward(x, offsets, w, dtype):
    """y_perm of the rows that have a group, of experts M v = L (R v) (+ M0 v), with its bound: R v, h and y are rounded to the storage type"""
    u, live = to.HALF[dtype], offsets[-1]
    base = "w_gate" in w
    v, bound = (torch.zeros(live, x.shape[1], dtype=torch.float64, device=x.device) for _ in range(2))

    def product(A, eA, e, right, left, whole):
        R, L = w[right][e].double(), w[left][e].double()
        t = A @ R.T
        et = eA @ R.abs().T + (A.shape[1] + 2) * to.U32 * ((A.abs() + eA) @ R.abs().T)
        et = et + u * (t.abs() + et)
        out, size = t @ L.T, (t.abs() + et) @ L.abs().T
        off = et @ L.abs().T
        if base:
            M = w[whole][0].double()
            out, size, off = out + A @ M.T, size + (A.abs() + eA) @ M.abs().T, off + eA @ M.abs().T
        return out, off + (A.shape[1] + R.shape[0] + 4) * to.U32 * size
    for e, (lo, hi) in enumerate(zip(offsets, offsets[1:])):
        X = x[lo:hi].double()
        none = torch.zeros_like(X)
        a, ea = product(X, none, e, "rg", "lg", "w_gate")
        b, eb = product(X, none, e, "ru", "lu", "w_up")
        act = a * torch.sigmoid(a)
        h = act * b
        eact = 1.1 * ea + act.abs() * (1.5 * a.abs() + 8) * to.U32  # (|silu'| <= 1.1)
        eh = act.abs() * eb + (b.abs() + eb) * eact + 4 * to.U32 * h.abs()
        eh = eh + u * (h.abs() + eh)
        y, ey = product(h, eh, e, "rd", "ld", "w_down")
        v[lo:hi], bound[lo:hi] = y, ey + u * (y.abs() + ey)
    return v, bound


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("T,d,F,E,k,r", [(1, 128, 256, 8, 2, 64), (8, 256, 512, 4, 2, 128), (40, 432, 1152, 8, 2, 216), (300, 264, 520, 4, 2, 72), (2000, 136, 264, 8, 2, 40)])
def test_factored_experts_of_a_batch_with_padding(T, d, F, E, k, r, shared, dtype):
    # the forward pass of weight-decomposed experts, alone and beside a shared base, on groups that end before the last row
    dt, g = DTYPES[dtype], gen(T + r)
    shape = pkg.make_shape(T, d, F, E, k, rank=r, act_dtype=CODE[dt], flags=pkg.FLAG_SHARED_BASE if shared else 0)
    sizes = {"rg": (E, r, d), "ru": (E, r, d), "lg": (E, F, r), "lu": (E, F, r), "rd": (E, r, F), "ld": (E, d, r)}
    if shared:
        sizes.update(w_gate=(1, F, d), w_up=(1, F, d), w_down=(1, d, F))
    w = {n: rnd(g, *s, std=s[-1] ** -0.5, dtype=dt).to(dev()) for n, s in sizes.items()}
    for masked in (0.4, 1.0):
        idx = picks(g, T, k, E, masked)
        offsets = [0] + torch.bincount(idx[idx >= 0].flatten().long(), minlength=E).cumsum(0).tolist()
        live = offsets[-1]
        x = rnd(g, T * k, d, dtype=dt)
        x[live:] = float("nan")
        x, y = x.to(dev()), torch.full((T * k, d), -7.0, dtype=dt, device=dev())
        pkg.moe_expert_ffn(shape, pkg.make_weights(w), x, torch.tensor(offsets, dtype=torch.int32, device=dev()), y, pkg.alloc_workspace(shape, dev()))
        to.near(y[:live], _factored_forward(x, offsets, w, dt), "y_perm")
        assert (y[live:] == -7.0).all()


def _beyond_4_gb(d, F, row_bytes):
    """Layer of 2^21 pairs of one expert and of two, the data of a few thousand rows alone: those past 2^32 bytes of a tensor of row_bytes a row, and the
    128 before them.  The others are zeros, which add nothing to the gradients of weights, in any order."""
    T = 1 << 21
    first = (1 << 32) // row_bytes - 128
    assert 2000 < T - first < 40000
    g = torch.Generator(device=dev())
    g.manual_seed(d)
    x, gy = (torch.zeros(T, d, dtype=torch.bfloat16, device=dev()) for _ in range(2))
    for t in (x, gy):
        t[first:] = torch.randn(T - first, d, generator=g, device=dev()).bfloat16()
    w = [(torch.randn(2, *s, generator=g, device=dev()) * s[1] ** -0.5).bfloat16() for s in ((F, d), (F, d), (d, F))]
    return T, first, x, gy, w


@pytest.mark.parametrize("d,F", [(136, 1032), (1032, 136)])
def test_gradients_of_weights_from_rows_beyond_4_gb(d, F):
    # h, da and db are wide in the one layer, x and its gradient in the other; the rows that count lie behind 4 GB, in a group that starts there and in one
    # that starts at the first row
    T, first, x, gy, w = _beyond_4_gb(d, F, 2 * max(d, F))
    shape, ws = base.make(T, d, 2, 1, torch.bfloat16, F)
    weights = pkg.make_weights(dict(zip(("w_gate", "w_up", "w_down"), w)))
    for offsets in ([0, first, T], [0, T, T]):
        outs = [torch.full_like(t, float("nan")) for t in (x, *w)]
        pkg.moe_expert_ffn_backward(shape, weights, x, torch.tensor(offsets, dtype=torch.int32, device=dev()), gy, *outs, ws)
        e = 1 if offsets[1] == first else 0
        want = to.experts_grad(x[first:], [0, 0, T - first] if e else [0, T - first, T - first], gy[first:], *w, torch.bfloat16)
        to.near(outs[0][first:], want[0], "grad_x_perm")
        assert (outs[0][:first] == 0).all()
        for name, o, v in zip(("gate", "up", "down"), outs[1:], want[1:]):
            to.near(o, v, name)
        del outs
