"""Plain numpy implementations, in 64 bits, of routing from logits and of experts in microscaled 4-bit
floating point, with the bounds on what 32-bit sums and the stored types may differ by."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BORDERS = (GRID[:-1] + GRID[1:]) / 2


# ---- MXFP4 ------------------------------------------------------------------------------------------------

def quantize(x):
    """x [rows, cols] fp64 -> codes [rows, cols] uint8 (unpacked), scale bytes [rows, blocks] uint8."""
    rows, cols = x.shape
    blocks = -(-cols // 32)
    p = np.zeros((rows, blocks * 32))
    p[:, :cols] = x
    p = p.reshape(rows, blocks, 32)
    bad = ~np.isfinite(p).all(-1)
    big = np.abs(np.where(np.isfinite(p), p, 0.0)).max(-1)
    e = np.frexp(big)[1] - 1
    b = np.where(big == 0, 0, np.maximum(e - 2 + 127, 0))
    m = np.abs(p) / np.exp2(b - 127.0)[..., None]
    code = np.zeros(p.shape, np.uint8)
    for c, border in enumerate(BORDERS):  # a tie goes to the even code
        code += (m > border) if c % 2 == 0 else (m >= border)
    code = (code + 8 * np.signbit(p)).astype(np.uint8)
    code[bad] = 0
    return code.reshape(rows, -1)[:, :cols], np.where(bad, 255, b).astype(np.uint8)


def pack_nibbles(code):
    return (code[..., 0::2] | (code[..., 1::2] << 4)).astype(np.uint8)


def values(code, b):
    """Unpacked codes [..., cols] and scale bytes [..., blocks] -> fp64."""
    v = np.where(code >= 8, -1.0, 1.0) * GRID[code & 7]
    s = np.where(b == 255, np.nan, np.exp2(b.astype(np.float64) - 127))
    return v * np.repeat(s, 32, axis=-1)[..., :v.shape[-1]]


def rounded(x):
    return values(*quantize(x))


def experts(x, w, idx, gate, residual, half_step):
    """x [T,d], w = (gate [E,F,d], up [E,F,d], down [E,d,F]), all fp64 -> (y, bound on the error of y).

    half_step: of the stored type, 2^-8 (bf16) or 2^-24.  A sum of n products in fp32, in any order, is off by at most
    n 2^-24 of the sum of magnitudes; the hidden values' bound follows through silu (slope at most 1.1, its
    exponential (|a| + 8) 2^-22), and a hidden value that lies so near a border of the 4-bit grid, or its
    block's maximum so near a power of two, may fall to either side: what the two sides differ by is added."""
    T, d = x.shape
    E, F, _ = w[0].shape
    y = np.zeros((T, d))
    tol = np.zeros((T, d))
    xq = rounded(x)
    for e in range(E):
        t, j = np.nonzero(idx == e)
        if not t.size:
            continue
        a, b = xq[t] @ w[0][e].T, xq[t] @ w[1][e].T
        da = d * 2.0 ** -24 * (np.abs(xq[t]) @ np.abs(w[0][e]).T)
        db = d * 2.0 ** -24 * (np.abs(xq[t]) @ np.abs(w[1][e]).T)
        s = a / (1 + np.exp(-a))
        h = s * b
        dh = 1.1 * da * (np.abs(b) + db) + np.abs(s) * db + (np.abs(a) + 8) * 2.0 ** -22 * np.abs(h)
        hq = rounded(h)
        moved = np.zeros_like(h)
        lo, hi = np.maximum(np.abs(h) - dh, 0), np.abs(h) + dh
        # the block's scale may belong to either end as well: all four combinations
        for m in (lo, hi):
            for ref in (lo, hi):
                bb = quantize(ref)[1]
                sc = np.repeat(np.exp2(bb.astype(np.float64) - 127), 32, axis=-1)[:, :F]
                r = m / sc
                code = np.zeros(r.shape, np.int64)
                for c, border in enumerate(BORDERS):
                    code += (r > border) if c % 2 == 0 else (r >= border)
                moved = np.maximum(moved, np.abs(GRID[code] * sc - np.abs(hq)))
        # (a value whose sign is not certain moves through zero)
        moved = np.where(np.abs(h) <= dh, moved + np.abs(hq), moved)
        o = hq @ w[2][e].T
        do = moved @ np.abs(w[2][e]).T + F * 2.0 ** -24 * (np.abs(hq) @ np.abs(w[2][e]).T) + half_step * np.abs(o)
        g = gate[t, j][:, None]
        np.add.at(y, t, g * o)
        np.add.at(tol, t, np.abs(g) * (do + (idx.shape[1] + 2) * 2.0 ** -24 * np.abs(o)))
    if residual:
        y += x
        tol += 2.0 ** -23 * (np.abs(x) + np.abs(y))
    return y, tol * (1 + half_step) + half_step * np.abs(y) * 1.01


# ---- routing ------------------------------------------------------------------------------------------------

def off(logits):
    return np.isnan(logits) | (logits == -np.inf)


def scores(logits, sigmoid):
    l = np.where(off(logits), -np.inf, logits.astype(np.float64))
    if sigmoid:
        with np.errstate(over="ignore"):
            return 1 / (1 + np.exp(-l))
    top = l.max(-1, keepdims=True)
    p = np.exp(l - np.where(np.isinf(top), 0.0, top))
    den = p.sum(-1, keepdims=True)
    return np.divide(p, den, out=np.zeros_like(p), where=den > 0)


def route(logits, bias, k, sigmoid, n_groups, kept, group_top, renormalize, scale):
    """-> idx [T,k], gate [T,k], scores [T,E]; token by token, as the definition is read."""
    T, E = logits.shape
    s = scores(logits, sigmoid)
    dead = off(logits)
    idx = np.zeros((T, k), np.int32)
    gate = np.zeros((T, k))
    per = E // n_groups
    for t in range(T):
        key = s[t] + (0 if bias is None else bias.astype(np.float64))
        # (without a bias the order is the logits': scores of large ones are equal in 64 bits)
        order = logits[t].astype(np.float64) if bias is None else key
        ranks = []
        for g in range(n_groups):
            alive = [e for e in range(g * per, (g + 1) * per) if not dead[t, e]]
            if group_top == 1:
                ranks.append(max((order[e] for e in alive), default=-np.inf))
            else:
                ranks.append(sum(sorted((key[e] for e in alive), reverse=True)[:2]) if alive else -np.inf)
        groups = sorted(range(n_groups), key=lambda g: (-ranks[g], g))[:kept] if n_groups > 1 else [0]
        cand = [e for e in range(E) if e // per in groups]
        cand.sort(key=lambda e: (1, 0.0, e) if dead[t, e] else (0, -order[e], e))
        pick = cand[:k]
        idx[t] = pick
        alive = [j for j, e in enumerate(pick) if not dead[t, e]]
        l = logits[t, pick].astype(np.float64)
        if renormalize:
            if alive:
                # log score, against underflow
                ls = -np.logaddexp(0, -l[alive]) if sigmoid else l[alive]
                w = np.exp(ls - ls.max())
                gate[t, alive] = w / w.sum()
        else:
            gate[t] = s[t, pick]
    return idx, gate * scale, s


def route_backward(logits, idx, dg, ds_in, sigmoid, renormalize, scale):
    """-> (gradient [T,E], bound of its error but for a factor in units of the type)."""
    T, E = logits.shape
    s = scores(logits, sigmoid)
    out, mag = np.zeros((T, E)), np.zeros((T, E))
    for t in range(T):
        ok = [j for j in range(idx.shape[1]) if 0 <= idx[t, j] < E]
        ds = np.zeros(E) if ds_in is None else ds_in[t].astype(np.float64).copy()
        ms = np.abs(ds)
        p = idx[t, ok]
        w, d = s[t, p], dg[t, ok].astype(np.float64)
        if renormalize:
            l = np.where(off(logits[t, p]), -np.inf, logits[t, p].astype(np.float64))
            ls = -np.logaddexp(0, -l) if sigmoid else l
            if len(ok) and np.isfinite(ls).any():
                g = np.exp(ls - ls.max())
                g /= g.sum()
                v = scale * g * (d - (d * g).sum())
                m = abs(scale) * g * (np.abs(d) + (np.abs(d) * g).sum())
                slope = 1 / (1 + np.exp(l)) if sigmoid else np.ones_like(l)
                np.add.at(out[t], p, v * slope)
                np.add.at(mag[t], p, m * slope)
        else:
            np.add.at(ds, p, scale * d)
            np.add.at(ms, p, np.abs(scale * d))
        if sigmoid:
            out[t] += ds * s[t] * (1 - s[t])
            mag[t] += ms * s[t]
        else:
            out[t] += s[t] * (ds - (ds * s[t]).sum())
            mag[t] += s[t] * (ms + (ms * s[t]).sum())
    return out, mag
