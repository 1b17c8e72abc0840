"""Plain implementations in 64 bits of the operators of a training step, with bounds on what their kernels' roundings can do.

Every function returns pairs (value, bound): the bound adds up, element by element, half a step of each rounding on the way
(2^-24 of fp32, 2^-8 of bf16, relative to the value that is rounded), a sum of n terms in fp32 counted as n roundings of the sum of the
terms' magnitudes, whatever its order.
"""
import math

import numpy as np
import torch

U32 = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
TINY = 1e-30  # results this small may be flushed


def near(got, want, what=""):
    value, bound = want
    d = (got.detach().cpu().double() - value.cpu().double()).abs()
    b = bound.cpu().double() + TINY
    worst = (d / b).max().item() if d.numel() else 0.0
    assert worst <= 1.0, f"{what}: {worst:.3g} of the bound (difference {d.flatten()[(d / b).argmax()].item():.3g})"


# ---- tokens to rows and back --------------------------------------------------------------------------------

def sort(idx, E):
    """offsets, perm and inv_perm by their definition: experts in turn, pairs in turn"""
    flat = idx.flatten().tolist()
    perm = [p for e in range(E) for p, v in enumerate(flat) if v == e]
    inv = [-1] * len(flat)
    for s, p in enumerate(perm):
        inv[p] = s
    offsets = [sum(0 <= v < e for v in flat) for e in range(E + 1)]
    return offsets, perm + [-1] * (len(flat) - len(perm)), inv


def rows_of(rows, inv):
    """[T, k, d] in 64 bits, zero for pairs without a row"""
    on = (inv >= 0) & (inv < rows.shape[0])
    safe = torch.where(on, inv, 0).long()
    return torch.where(on[..., None], rows.double()[safe], 0.0)


def dispatch(x, weight, perm, k, dtype):
    p = torch.tensor(perm)
    rows = x.double()[(p.clamp(min=0) // k)]
    if weight is None:
        v = torch.where(p[:, None] >= 0, rows, 0.0)
        return v, torch.zeros_like(v)
    v = torch.where(p[:, None] >= 0, rows * weight.double().flatten()[p.clamp(min=0), None], 0.0)
    return v, v.abs() * (HALF[dtype] + 2 * U32)


def gather_sum(rows, inv, weight, residual, dtype):
    g = rows_of(rows, inv) * (1.0 if weight is None else weight.double()[..., None])
    g = torch.where((inv >= 0)[..., None], g, 0.0)  # (a gate of a pair without a row may be anything)
    v, size = g.sum(1), g.abs().sum(1)
    if residual is not None:
        v, size = v + residual.double(), size + residual.double().abs()
    return v, v.abs() * HALF[dtype] + size * (inv.shape[1] + 2) * U32 * 2


def dots(a, rows, inv):
    t = rows_of(rows, inv) * a.double()[:, None]
    return t.sum(-1), t.abs().sum(-1) * (a.shape[1] + 2) * U32


# ---- experts ---------------------------------------------------------------------------------------------------

def experts_grad(x, offsets, gy, wg, wu, wd, dtype):
    """gx, gwg, gwu, gwd with bounds; x, gy [P, d]; rows behind the last group: zero"""
    u, P = HALF[dtype], x.shape[0]
    outs = [torch.zeros_like(t, dtype=torch.float64) for t in (x, wg, wu, wd)]
    bounds = [torch.zeros_like(t) for t in outs]
    d, F = x.shape[1], wg.shape[1]
    for e in range(wg.shape[0]):
        lo, hi = offsets[e], offsets[e + 1]
        if lo == hi:
            continue
        X, G, Wg, Wu, Wd = (t.double() for t in (x[lo:hi], gy[lo:hi], wg[e], wu[e], wd[e]))
        a, b, dh = X @ Wg.T, X @ Wu.T, G @ Wd
        ea, eb, edh = ((d + 2) * U32 * t for t in (X.abs() @ Wg.abs().T, X.abs() @ Wu.abs().T, G.abs() @ Wd.abs()))
        s = torch.sigmoid(a)
        act, slope = a * s, s * (1 + a * (1 - s))
        h, da, db = act * b, dh * b * slope, dh * act
        # exp and the reciprocal: exp(-a) is off by the rounding of a log2(e), 2^-24 |a| 1.5, and a step or two of its own
        es = (1.5 * a.abs() + 8) * U32
        eh = act.abs() * eb + b.abs() * (1.1 * ea + act.abs() * es) + 4 * U32 * h.abs()
        edb = act.abs() * edh + dh.abs() * (1.1 * ea + act.abs() * es) + 4 * U32 * db.abs()
        # |slope'| <= 1/2; slope = s + act (1 - s)
        eslope = 0.5 * ea + (s + act.abs()) * (es + 4 * U32) * 2
        eda = (edh * b.abs() + dh.abs() * eb) * slope.abs() + (dh * b).abs() * eslope + 6 * U32 * da.abs()
        # rounding to the storage type, of what is off already
        eh, eda, edb = eh + u * (h.abs() + eh), eda + u * (da.abs() + eda), edb + u * (db.abs() + edb)
        n = hi - lo

        def product(A, eA, B, eB, length):
            v = A @ B
            off = eA @ B.abs() + (0 if eB is None else A.abs() @ eB + eA @ eB) + (length + 2) * U32 * ((A.abs() + eA) @ B.abs())
            return v, off
        g1, o1 = product(da, eda, Wg, None, 2 * F)
        g2, o2 = product(db, edb, Wu, None, 2 * F)
        o = o1 + o2
        outs[0][lo:hi], bounds[0][lo:hi] = g1 + g2, o + u * ((g1 + g2).abs() + o)
        for i, (A, eA, B) in enumerate(((da.T, eda.T, X), (db.T, edb.T, X)), 1):
            v, o = product(A, eA, B, None, n)
            outs[i][e], bounds[i][e] = v, o + u * (v.abs() + o)
        v, o = product(h.T, eh.T, G, None, n)
        outs[3][e], bounds[3][e] = v.T, (o + u * (v.abs() + o)).T
    return list(zip(outs, bounds))


def experts_forward(x, offsets, wg, wu, wd, dtype):
    """y_perm of the rows that have a group, with its bound: h and y are rounded, and a product's k-steps may be summed in two to four parts of
    the storage type"""
    u, live, d, F = HALF[dtype], offsets[-1], x.shape[1], wg.shape[1]
    v, bound = torch.zeros(live, d, dtype=torch.float64, device=x.device), torch.zeros(live, d, dtype=torch.float64, device=x.device)
    for e in range(wg.shape[0]):
        lo, hi = offsets[e], offsets[e + 1]
        X, Wg, Wu, Wd = (t.double() for t in (x[lo:hi], wg[e], wu[e], wd[e]))
        a, b = X @ Wg.T, X @ Wu.T
        ea, eb = (d + 2) * U32 * (X.abs() @ Wg.abs().T), (d + 2) * U32 * (X.abs() @ Wu.abs().T)
        act = a * torch.sigmoid(a)
        h = act * b
        eh = act.abs() * eb + b.abs() * (1.1 * ea + act.abs() * (1.5 * a.abs() + 8) * U32) + 4 * U32 * h.abs()
        eh = eh + u * (h.abs() + eh)
        size = (h.abs() + eh) @ Wd.abs().T
        v[lo:hi] = h @ Wd.T
        bound[lo:hi] = eh @ Wd.abs().T + (F + 2) * U32 * size + 2 * u * size
    return v, bound


# ---- block ------------------------------------------------------------------------------------------------------

def philox(counter, key):
    """Philox4x32-10 in Python's integers: counter of four words, key of two."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def kept(T, d, dropout, rng):
    """[T, d] truth values, from the definition"""
    seed, offset = (int(v) & (2 ** 64 - 1) for v in rng)
    drop = int(np.rint(np.float64(np.float32(dropout)) * 65536))
    m = np.empty(T * d, dtype=bool)
    for q in range(T * d // 8):
        w = philox((q & 0xFFFFFFFF, q >> 32, offset & 0xFFFFFFFF, offset >> 32), (seed & 0xFFFFFFFF, seed >> 32))
        for i in range(8):
            m[8 * q + i] = (w[i // 2] >> (16 * (i % 2)) & 0xFFFF) >= drop
    return torch.from_numpy(m.reshape(T, d))


def keep_scale(dropout):
    return 65536 / (65536 - int(np.rint(np.float64(np.float32(dropout)) * 65536)))


def _norm(v, eps):
    """1 / root mean square, and its relative error in fp32"""
    return 1 / torch.sqrt(v.square().mean(-1, keepdim=True) + eps), (v.shape[-1] / 2 + 8) * U32


def _factors(cfg, T, d, mask):
    one = torch.ones(1, 1, dtype=torch.float64)
    gate = one if cfg.get("gate") is None else cfg["gate"].double()[None]
    tg = one if cfg.get("token_gate") is None else cfg["token_gate"].double()[:, None]
    drop = one if mask is None else mask.double() * keep_scale(cfg["dropout"])
    return gate, tg, drop


def block(cfg, x, b, mask, dtype):
    """y with its bound"""
    x, b = x.double(), b.double()
    T, d = x.shape
    gate, tg, drop = _factors(cfg, T, d, mask)
    z, rel = b, 0.0
    if cfg.get("post_w") is not None:
        r, rel = _norm(b, cfg["eps"])
        z = b * r * cfg["post_w"].double()
    branch = cfg["block_scale"] * gate * tg * drop * z
    y = cfg["skip_scale"] * x + branch
    return y, branch.abs() * (rel + 8 * U32) + (cfg["skip_scale"] * x).abs() * 2 * U32 + y.abs() * (HALF[dtype] + U32)


def opened(y, w, eps, dtype):
    y = y.double()
    r, rel = _norm(y, eps)
    n = y * r * w.double()
    return n, n.abs() * (HALF[dtype] + rel + 4 * U32)


def block_grad(cfg, gy, gn, y, b, open_w, mask, dtype):
    """dict of (value, bound)"""
    shape = (gy if gy is not None else gn).shape
    T, d = shape
    out = {}
    G = torch.zeros(shape, dtype=torch.float64) if gy is None else gy.double()
    size = G.abs()  # of the terms of G
    if gn is not None:
        yy, n, w = y.double(), gn.double(), open_w.double()
        r, rel = _norm(yy, cfg["eps"])
        u = n * w
        G = G + r * (u - yy * r * r * (u * yy).mean(-1, keepdim=True))
        size = size + r * u.abs() + r ** 3 * yy.abs() * (u * yy).abs().mean(-1, keepdim=True)
        t = n * yy * r
        out["open_w"] = (t.sum(0), t.abs().sum(0) * (rel + (T + 4) * U32))
    eG = size * (3 * d + 40) * U32
    scale = 1.0 if b is None else cfg["skip_scale"]
    out["x"] = (scale * G, abs(scale) * (eG + HALF[dtype] * (G.abs() + eG)) + U32 * size)
    if b is None:
        return out
    bb = b.double()
    gate, tg, drop = _factors(cfg, T, d, mask)
    r, rel = (torch.ones(T, 1, dtype=torch.float64), 0.0) if cfg.get("post_w") is None else _norm(bb, cfg["eps"])
    w = torch.ones(1, d, dtype=torch.float64) if cfg.get("post_w") is None else cfg["post_w"].double()[None]
    up, eup = G * cfg["block_scale"] * drop, (eG + size * 4 * U32) * abs(cfg["block_scale"]) * drop
    bare = up * bb * r * w
    ebare = eup * (bb * r * w).abs() + bare.abs() * (rel + 6 * U32)
    out["gate"] = ((bare * tg).sum(0), ((ebare + bare.abs() * (T + 4) * U32) * tg.abs()).sum(0))
    out["token_gate"] = ((bare * gate).sum(1), ((ebare + bare.abs() * (d + 4) * U32) * gate.abs()).sum(1))
    f, z, ez = gate * tg, up * gate * tg, eup * (gate * tg).abs() + (up * gate * tg).abs() * 4 * U32
    v, ev = z * w, (ez + z.abs() * U32) * w.abs()
    if cfg.get("post_w") is None:
        out["b"] = (v, ev + HALF[dtype] * (v.abs() + ev))
        return out
    t = z * bb * r
    out["post_w"] = (t.sum(0), (ez * (bb * r).abs() + t.abs() * (rel + (T + 6) * U32)).sum(0))
    mean = (v * bb).mean(-1, keepdim=True)
    gb = r * (v - bb * r * r * mean)
    size_b = r * v.abs() + r ** 3 * bb.abs() * (v * bb).abs().mean(-1, keepdim=True)
    eb = r * ev + r ** 3 * bb.abs() * (ev * bb.abs()).mean(-1, keepdim=True) + size_b * (3 * d + 40) * U32
    out["b"] = (gb, eb + HALF[dtype] * (gb.abs() + eb))
    return out


def step(p, mask=None, dropout=0.0):
    """A block of norm, routing (softmax, top k, renormalised), experts, norm, gate, residual, in 64 bits, for automatic
    differentiation.  p: x, open_w, router_w, w_gate, w_up, w_down, post_w, gate, idx, eps, block_scale."""
    def rms(v, w):
        return v * w / torch.sqrt(v.square().mean(-1, keepdim=True) + p["eps"])
    n = rms(p["x"], p["open_w"])
    scores = torch.softmax(n @ p["router_w"].T, -1).gather(1, p["idx"])
    gates = scores / scores.sum(-1, keepdim=True)
    out = torch.zeros_like(n)
    for j in range(p["idx"].shape[1]):
        wg, wu, wd = (p[m][p["idx"][:, j]] for m in ("w_gate", "w_up", "w_down"))
        a, b = (wg @ n[..., None])[..., 0], (wu @ n[..., None])[..., 0]
        out = out + gates[:, j, None] * (wd @ (torch.nn.functional.silu(a) * b)[..., None])[..., 0]
    z = rms(out, p["post_w"]) * p["gate"]
    if mask is not None:
        z = z * mask * keep_scale(dropout)
    return p["x"] + p["block_scale"] * z


assert math.isclose(keep_scale(0.5), 2.0)
