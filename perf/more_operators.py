"""The operators of a training step around and through the experts, as a list of measurable cases.

Six kinds of pass:
  dispatch, dispatch_grad  tokens to rows sorted by expert, with weights; the gradient of tokens and weights
                           (moe_dispatch, moe_dispatch_backward)
  collect, collect_grad    rows back to tokens, summed by gates; the gradient of rows and gates
                           (moe_collect, moe_collect_backward)
  experts_grad             the gradient of the expert feed-forward with regard to its rows and weights
                           (moe_expert_ffn_backward)
  block, block_grad        what stands around such a layer: the norm after it, its gates, dropout, the scaled residual
                           and the norm before the next one; their gradient (moe_block_norm, moe_block_norm_backward)

listed() holds named cases over the real range, draw() gives further ones of the same ranges.  Where
`own` is false, run() computes the same in elementary torch operations.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
EPS = 1e-5


# ---- cases --------------------------------------------------------------------------------------

def _rows(kind, tokens, d, experts=8, top_k=2, dtype="bf16", weighted=True, masked=0.0, skew=1.1, residual=False):
    return {"kind": kind, "tokens": tokens, "d_model": d, "experts": experts, "top_k": top_k, "dtype": dtype, "weighted": weighted,
            "masked": masked, "skew": skew, "residual": residual}


def _experts(tokens, d, f, experts=8, top_k=2, dtype="bf16", skew=0.0):
    return {"kind": "experts_grad", "tokens": tokens, "d_model": d, "d_ff": f, "experts": experts, "top_k": top_k, "dtype": dtype, "skew": skew}


def _block(kind, tokens, d, dtype="bf16", post=True, gate=True, token_gate=False, opens=True, dropout=0.0):
    return {"kind": kind, "tokens": tokens, "d_model": d, "dtype": dtype, "post": post, "gate": gate, "token_gate": token_gate, "opens": opens,
            "dropout": dropout}


def listed():
    def named(name, c):
        return dict(name=name, **c)
    return [
        # a few sequences decoded together, more experts, weights put in before the experts
        named("dispatch_24", _rows("dispatch", 24, 1024, experts=16, top_k=4)),
        # a training batch in 32 bits, the gradient of tokens and of the weights
        named("dispatch_grad_2048", _rows("dispatch_grad", 2048, 1440, dtype="f32")),
        # an odd number of tokens at an odd width, some of them padding that no expert sees
        named("collect_777", _rows("collect", 777, 1600, masked=0.1, residual=True)),
        # the largest batch, loads skewed as trained routers' are
        named("collect_grad_16384", _rows("collect_grad", 16384, 2048)),
        # a small batch: the weights and their gradients are all there is to move
        named("experts_grad_24", _experts(24, 1024, 2816, experts=16, top_k=4)),
        # an odd number of tokens at widths that are no multiples of a tile
        named("experts_grad_777", _experts(777, 1440, 3840, skew=1.1)),
        # a training batch of the phone-sized layer
        named("experts_grad_2048", _experts(2048, 2048, 5632, skew=1.1)),
        # the largest batch
        named("experts_grad_16384", _experts(16384, 2048, 5632, skew=1.1)),
        # one generated token between two layers
        named("block_1", _block("block", 1, 2048)),
        # the largest batch in training, with dropout
        named("block_16384", _block("block", 16384, 2048, dropout=0.1)),
        # a training batch at a width that is no power of two, gated by token
        named("block_grad_2048", _block("block_grad", 2048, 1440, token_gate=True)),
        # the largest batch, dropout's mask made again
        named("block_grad_16384", _block("block_grad", 16384, 2048, dropout=0.1)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _mult8(v):
    return max(8, int(round(v / 8.0)) * 8)


def draw(rng):
    kind = rng.choice(["dispatch", "dispatch_grad", "collect", "collect_grad", "experts_grad", "experts_grad", "experts_grad", "block", "block_grad"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind in ("block", "block_grad"):
        return _block(kind, _log_int(rng, 1, 16384), _mult8(_log_int(rng, 400, 2048)), dtype, post=rng.random() < 0.8, gate=rng.random() < 0.6,
                      token_gate=rng.random() < 0.4, opens=rng.random() < 0.7, dropout=rng.choice([0.0, 0.0, 0.1, 0.25]))
    top_k = rng.choice([1, 2, 2, 4])
    skew = rng.choice([0.0, 1.1])
    if kind == "experts_grad":
        if dtype == "f32":  # layers in 32 bits are the small ones
            d, f, most = _mult8(_log_int(rng, 128, 432)), _mult8(_log_int(rng, 256, 1152)), 2048
        else:
            d, f, most = _mult8(_log_int(rng, 400, 2048)), _mult8(_log_int(rng, 1064, 5632)), 16384
        experts = rng.choice([4, 8, 8, 16, 32])
        while experts * d * f > 8 * 2048 * 5632:
            experts //= 2
        return _experts(min(_log_int(rng, 1, most), 16384 * 2 // top_k), d, f, experts, min(top_k, experts), dtype, skew)
    experts = rng.choice([4, 8, 8, 16, 32, 64])
    return _rows(kind, min(_log_int(rng, 1, 16384), 16384 * 2 // top_k), _mult8(_log_int(rng, 400, 2048)), experts, top_k, dtype, weighted=rng.random() < 0.6,
                 masked=rng.choice([0.0, 0.1, 0.5]), skew=skew, residual=rng.random() < 0.3)


def work(case):
    t, d, size = case["tokens"], case["d_model"], 4 if case["dtype"] == "f32" else 2
    row, kind = d * size, case["kind"]
    if kind == "block":
        return {"bytes": t * row * (3 + case["opens"]), "flops": t * d * 12}
    if kind == "block_grad":
        return {"bytes": t * row * (4 + 2 * case["opens"]), "flops": t * d * 24}
    pairs = t * case["top_k"]
    if kind == "experts_grad":
        f, e = case["d_ff"], case["experts"]
        return {"bytes": 3 * d * f * size * (min(e, pairs) + e) + 3 * pairs * row, "flops": 16 * pairs * d * f}
    live = pairs * (1 - case["masked"])
    if kind == "dispatch":
        return {"bytes": t * row + pairs * row + pairs * (12 + 4 * case["weighted"]), "flops": live * d}
    if kind == "dispatch_grad":
        return {"bytes": live * row + t * row * (1 + case["weighted"]) + pairs * (4 + 8 * case["weighted"]), "flops": live * d * (2 + 2 * case["weighted"])}
    if kind == "collect":
        return {"bytes": live * row + t * row * (1 + case["residual"]) + 8 * pairs, "flops": 2 * live * d}
    return {"bytes": live * row + t * row + pairs * row + 12 * pairs, "flops": 3 * live * d}


# ---- the plain forms -------------------------------------------------------------------------------

def _plain_sort(idx, experts):
    """Bounds of the groups, the pair of each sorted row and the row of each pair; switched-off pairs have no row (-1)."""
    key = idx.flatten().long()
    key = torch.where((key < 0) | (key >= experts), experts, key)
    order = torch.argsort(key, stable=True)
    at = torch.searchsorted(key[order].contiguous(), torch.arange(experts + 1, device=key.device))
    place = torch.empty_like(order).scatter_(0, order, torch.arange(order.numel(), device=key.device))
    on = key < experts
    return at.int(), torch.where(on[order], order, -1).int(), torch.where(on, place, -1).int()


def _plain_dispatch(s):
    offsets, perm, inv = _plain_sort(s["idx"], s["case"]["experts"])
    k, p = s["case"]["top_k"], perm.long().clamp(min=0)
    rows = s["x"].float()[p // k]
    if s["weight"] is not None:
        rows = rows * s["weight"].flatten()[p, None]
    return offsets, perm, inv, torch.where(perm[:, None] >= 0, rows, 0.0).to(s["x"].dtype)


def _plain_rows_of(rows, inv):
    """The rows of each token's pairs [T, k, d] in 32 bits, 0 where a pair has none."""
    return torch.where(inv[..., None] >= 0, rows.float()[inv.long().clamp(min=0)], 0.0)


def _plain_dispatch_grad(s):
    g = _plain_rows_of(s["grad_rows"], s["inv"])
    if s["weight"] is None:
        return g.sum(1).to(s["grad_rows"].dtype)
    return (g * s["weight"][..., None]).sum(1).to(s["grad_rows"].dtype), (g * s["x"].float()[:, None]).sum(-1)


def _plain_collect(s):
    y = (_plain_rows_of(s["rows"], s["inv"]) * s["weight"][..., None]).sum(1)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["rows"].dtype)


def _plain_collect_grad(s):
    gy, inv = s["grad_y"].float(), s["inv"].flatten().long()
    on = inv >= 0
    grad_gate = (_plain_rows_of(s["rows"], s["inv"]) * gy[:, None]).sum(-1)
    grad = torch.zeros_like(s["rows"])
    pair = torch.where(on)[0]
    grad[inv[pair]] = (gy[pair // s["case"]["top_k"]] * s["weight"].flatten()[pair, None]).to(grad.dtype)
    return grad, grad_gate


def _plain_experts_grad(s):
    x, gy, bounds = s["x"], s["grad_y"], s["bounds"]
    gx = torch.empty_like(x)
    gw = [torch.empty_like(w) for w in s["w"]]
    for e in range(s["case"]["experts"]):
        lo, hi = bounds[e], bounds[e + 1]
        wg, wu, wd = (w[e].float() for w in s["w"])
        xe, ge = x[lo:hi].float(), gy[lo:hi].float()
        a, b, dh = xe @ wg.T, xe @ wu.T, ge @ wd
        sig = 1 / (1 + torch.exp(-a))
        act = a * sig
        da, db = dh * b * (sig + act * (1 - sig)), dh * act
        gx[lo:hi] = (da @ wg + db @ wu).to(x.dtype)
        gw[0][e], gw[1][e], gw[2][e] = (m.to(x.dtype) for m in (da.T @ xe, db.T @ xe, ge.T @ (act * b)))
    return [gx] + gw


def _plain_kept(case, rng):
    """Dropout's mask: halves of 32-bit words of Philox 4x32-10, eight neighbours to a counter."""
    n, m32 = case["tokens"] * case["d_model"] // 8, 0xFFFFFFFF
    q = torch.arange(n, device=rng.device)
    seed, offset = rng[0], rng[1]
    c = [q & m32, q >> 32, (offset & m32).expand(n), (offset >> 32 & m32).expand(n)]
    k0, k1 = seed & m32, seed >> 32 & m32
    for _ in range(10):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [p1 >> 32 & m32 ^ c[1] ^ k0, p1 & m32, p0 >> 32 & m32 ^ c[3] ^ k1, p0 & m32]
        k0, k1 = k0 + 0x9E3779B9 & m32, k1 + 0xBB67AE85 & m32
    half = torch.stack([v for w in c for v in (w & 0xFFFF, w >> 16)], -1)
    return (half >= round(case["dropout"] * 65536)).view(case["tokens"], case["d_model"])


def _keep_scale(case):
    return 65536 / (65536 - round(case["dropout"] * 65536))


def _plain_norm(v):
    """1 / root mean square of rows in 32 bits"""
    return torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS)


def _plain_factor(s):
    """What the norm of the block's output is multiplied by: [T, d] or what broadcasts to it"""
    m = torch.full((1, 1), s["block_scale"], device=DEV)
    if s["gate"] is not None:
        m = m * s["gate"]
    if s["token_gate"] is not None:
        m = m * s["token_gate"][:, None]
    return m * torch.where(_plain_kept(s["case"], s["rng"]), _keep_scale(s["case"]), 0.0) if s["case"]["dropout"] else m


def _plain_block(s):
    x, b = s["x"].float(), s["b"].float()
    z = b * _plain_norm(b) * s["post_w"] if s["post_w"] is not None else b
    y = (s["skip_scale"] * x + _plain_factor(s) * z).to(s["x"].dtype)
    if s["open_w"] is None:
        return [y]
    return [y, (y.float() * _plain_norm(y.float()) * s["open_w"]).to(y.dtype)]


def _plain_block_grad(s):
    out, g = {}, s["grad_y"].float()
    if s["open_w"] is not None:
        y, gn = s["y"].float(), s["grad_n"].float()
        r = _plain_norm(y)
        out["open_w"] = (gn * y * r).sum(0)
        u = gn * s["open_w"]
        g = g + r * (u - y * r * r * (u * y).mean(-1, keepdim=True))
    b, factor = s["b"].float(), _plain_factor(s)
    r = _plain_norm(b) if s["post_w"] is not None else torch.ones_like(b[:, :1])
    z = b * r * s["post_w"] if s["post_w"] is not None else b
    out["x"] = (g * s["skip_scale"]).to(s["b"].dtype)
    dz = g * factor
    if s["gate"] is not None or s["token_gate"] is not None:
        bare = g * z * s["block_scale"]
        if s["case"]["dropout"]:
            bare = bare * torch.where(_plain_kept(s["case"], s["rng"]), _keep_scale(s["case"]), 0.0)
        if s["gate"] is not None:
            out["gate"] = (bare * s["token_gate"][:, None] if s["token_gate"] is not None else bare).sum(0)
        if s["token_gate"] is not None:
            out["token_gate"] = (bare * s["gate"] if s["gate"] is not None else bare).sum(-1)
    if s["post_w"] is not None:
        out["post_w"] = (dz * b * r).sum(0)
        u = dz * s["post_w"]
        dz = r * (u - b * r * r * (u * b).mean(-1, keepdim=True))
    out["b"] = dz.to(s["b"].dtype)
    return out


# ---- inputs and passes ---------------------------------------------------------------------------------

def _picks(g, case):
    """Experts by a Zipf law of exponent `skew`, without replacement; padding tokens have none (-1)."""
    t, e, k = case["tokens"], case["experts"], case["top_k"]
    pull = -case["skew"] * torch.log(torch.arange(1, e + 1, device=DEV).float())
    noise = -torch.log(-torch.log(torch.rand(t, e, generator=g, device=DEV).clamp(1e-7, 1 - 1e-7)))
    idx = (pull + noise).topk(k, -1).indices.int().contiguous()
    if case.get("masked"):
        idx.masked_fill_(torch.rand(t, 1, generator=g, device=DEV) < case["masked"], -1)
    return idx


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    t, d = case["tokens"], case["d_model"]
    dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16

    def normal(*shape, std=1.0, to=dtype):
        return (torch.randn(*shape, generator=g, device=DEV) * std).to(to)

    s = {"case": case}
    if case["kind"] in ("block", "block_grad"):
        s["skip_scale"], s["block_scale"] = 1.0, 0.5
        s["x"], s["b"] = normal(t, d), normal(t, d, std=0.3)
        s["post_w"] = 1 + normal(d, std=0.1, to=torch.float32) if case["post"] else None
        s["open_w"] = 1 + normal(d, std=0.1, to=torch.float32) if case["opens"] else None
        s["gate"] = normal(d, std=0.5, to=torch.float32) if case["gate"] else None
        s["token_gate"] = torch.rand(t, generator=g, device=DEV) if case["token_gate"] else None
        s["rng"] = torch.tensor([0x243F6A8885A308D3 ^ seed, 1 << 33 | seed], device=DEV)
        if case["kind"] == "block_grad":
            s["y"] = _plain_block(s)[0]
            s["grad_y"] = normal(t, d)
            s["grad_n"] = normal(t, d) if case["opens"] else None
        if own:
            import paper_2503_00245_amd as moe
            s["block"] = moe.make_block(eps=EPS, skip_scale=s["skip_scale"], block_scale=s["block_scale"], dropout=case["dropout"], post_w=s["post_w"],
                                        gate=s["gate"], token_gate=s["token_gate"], rng=s["rng"] if case["dropout"] else None)
            s["workspace"] = moe.alloc_block_workspace(t, d, s["x"].device)
        return s
    k, e = case["top_k"], case["experts"]
    idx = _picks(g, case)
    offsets, _, inv = _plain_sort(idx, e)
    if case["kind"] == "experts_grad":
        f = case["d_ff"]
        s["offsets"], s["bounds"] = offsets, offsets.tolist()
        s["x"] = normal(t, d)[torch.argsort(idx.flatten(), stable=True) // k].contiguous()
        s["grad_y"] = normal(t * k, d)
        s["w"] = [normal(e, *shape, std=0.02) for shape in ((f, d), (f, d), (d, f))]
    else:
        s["idx"], s["offsets"], s["inv"] = idx, offsets, inv.view(t, k)
        s["x"] = normal(t, d)
        s["weight"] = torch.softmax(normal(t, k, to=torch.float32), -1) if case["weighted"] or case["kind"].startswith("collect") else None
        s["residual"] = normal(t, d) if case["residual"] else None
        if case["kind"] == "dispatch_grad":
            s["grad_rows"] = normal(t * k, d)
        elif case["kind"].startswith("collect"):
            s["rows"], s["grad_y"] = normal(t * k, d), normal(t, d)
    if own:
        import paper_2503_00245_amd as moe
        s["shape"] = moe.make_shape(t, d, case.get("d_ff", 8), e, k, act_dtype=moe.MOE_F32 if dtype is torch.float32 else moe.MOE_BF16)
        if case["kind"] == "experts_grad":
            s["weights"] = moe.make_weights(dict(zip(("w_gate", "w_up", "w_down"), s["w"])))
        s["workspace"] = moe.alloc_training_workspace(s["shape"], s["x"].device)
    return s


def run(state):
    s, kind = state, state["case"]["kind"]
    if not own:
        return {"dispatch": _plain_dispatch, "dispatch_grad": _plain_dispatch_grad, "collect": _plain_collect, "collect_grad": _plain_collect_grad,
                "experts_grad": _plain_experts_grad, "block": _plain_block, "block_grad": _plain_block_grad}[kind](s)
    import paper_2503_00245_amd as moe
    c = s["case"]
    dev = s["x"].device
    if kind == "block":
        y, n = torch.empty_like(s["x"]), None if s["open_w"] is None else torch.empty_like(s["x"])
        moe.moe_block_norm(s["block"], s["x"], s["b"], s["open_w"], y, n)
        return [y] if n is None else [y, n]
    if kind == "block_grad":
        out = {"x": torch.empty_like(s["b"]), "b": torch.empty_like(s["b"])}
        for name in ("open_w", "post_w", "gate", "token_gate"):
            if s[name] is not None:
                out[name] = torch.empty_like(s[name])
        moe.moe_block_norm_backward(s["block"], s["grad_y"], s["grad_n"], s["y"], s["b"], s["open_w"], out["x"], out["b"], out.get("open_w"),
                                    out.get("post_w"), out.get("gate"), out.get("token_gate"), s["workspace"])
        return out
    pairs = c["tokens"] * c["top_k"]
    if kind == "experts_grad":
        gx, gw = torch.empty_like(s["x"]), [torch.empty_like(w) for w in s["w"]]
        moe.moe_expert_ffn_backward(s["shape"], s["weights"], s["x"], s["offsets"], s["grad_y"], gx, *gw, s["workspace"])
        return [gx] + gw
    if kind == "dispatch":
        offsets = torch.empty(c["experts"] + 1, dtype=torch.int32, device=dev)
        perm, inv = (torch.empty(pairs, dtype=torch.int32, device=dev) for _ in range(2))
        rows = torch.empty(pairs, c["d_model"], dtype=s["x"].dtype, device=dev)
        moe.moe_dispatch(s["shape"], s["idx"], s["weight"], s["x"], offsets, perm, inv, rows, s["workspace"])
        return offsets, perm, inv, rows
    if kind == "dispatch_grad":
        gx = torch.empty_like(s["x"])
        gw = None if s["weight"] is None else torch.empty_like(s["weight"])
        moe.moe_dispatch_backward(s["shape"], s["grad_rows"], s["inv"], s["x"] if gw is not None else None, s["weight"], gx, gw)
        return gx if gw is None else (gx, gw)
    if kind == "collect":
        y = torch.empty_like(s["x"])
        moe.moe_collect(s["shape"], s["rows"], s["inv"], s["weight"], s["residual"], y)
        return y
    grad, grad_gate = torch.empty_like(s["rows"]), torch.empty_like(s["weight"])
    moe.moe_collect_backward(s["shape"], s["grad_y"], s["rows"], s["offsets"], s["inv"], s["weight"], grad, grad_gate)
    return grad, grad_gate


# ---- from the definitions, in 64 bits -----------------------------------------------------------------------

def _exact_kept(case, rng):
    """Philox 4x32-10 in unsigned 64-bit integers on the host."""
    seed, offset = (int(v) & 0xFFFFFFFFFFFFFFFF for v in rng.tolist())
    n, low, u = case["tokens"] * case["d_model"] // 8, np.uint64(0xFFFFFFFF), np.uint64
    q = np.arange(n, dtype=np.uint64)
    x0, x1 = q & low, q >> u(32)
    x2, x3 = np.full(n, offset & 0xFFFFFFFF, dtype=np.uint64), np.full(n, offset >> 32, dtype=np.uint64)
    for r in range(10):
        ka, kb = u((seed + r * 0x9E3779B9) & 0xFFFFFFFF), u(((seed >> 32) + r * 0xBB67AE85) & 0xFFFFFFFF)
        a, b = x0 * u(0xD2511F53), x2 * u(0xCD9E8D57)
        x0, x1, x2, x3 = (b >> u(32)) ^ x1 ^ ka, b & low, (a >> u(32)) ^ x3 ^ kb, a & low
    words = np.stack([x0, x1, x2, x3], 1).astype("<u4")
    kept = words.view("<u2").astype(np.int64) >= round(case["dropout"] * 65536)
    return torch.from_numpy(kept.reshape(case["tokens"], case["d_model"])).to(rng.device)


def _exact_rms(v, w):
    return v / torch.sqrt(v.square().sum(-1, keepdim=True) / v.shape[-1] + EPS) * w


def _exact_y(s, x, b, post_w, gate, token_gate):
    z = b if post_w is None else _exact_rms(b, post_w)
    if s["case"]["dropout"]:
        z = z * _exact_kept(s["case"], s["rng"]) * _keep_scale(s["case"])
    z = z if gate is None else z * gate
    z = z if token_gate is None else z * token_gate.unsqueeze(-1)
    return s["skip_scale"] * x + s["block_scale"] * z


def _leaf(v):
    return None if v is None else v.double().requires_grad_(True)


def _exact_block_grad(s):
    leaves = {n: _leaf(s[n]) for n in ("x", "b", "post_w", "gate", "token_gate")}
    with torch.enable_grad():
        up = s["grad_y"].double()
        out = {}
        if s["open_w"] is not None:
            y, w = _leaf(s["y"]), _leaf(s["open_w"])
            gy, out["open_w"] = torch.autograd.grad(_exact_rms(y, w), (y, w), s["grad_n"].double())
            up = up + gy
        used = {n: v for n, v in leaves.items() if v is not None}
        grads = torch.autograd.grad(_exact_y(s, *leaves.values()), list(used.values()), up)
    out.update(zip(used, grads))
    return out


def _exact_experts_grad(s):
    gx, gw = torch.zeros_like(s["x"], dtype=torch.float64), [torch.zeros_like(w, dtype=torch.float64) for w in s["w"]]
    for e, (lo, hi) in enumerate(zip(s["bounds"], s["bounds"][1:])):
        if lo == hi:
            continue
        x, w = _leaf(s["x"][lo:hi]), [_leaf(v[e]) for v in s["w"]]
        with torch.enable_grad():
            y = (torch.nn.functional.silu(x @ w[0].t()) * (x @ w[1].t())) @ w[2].t()
            grads = torch.autograd.grad(y, [x, *w], s["grad_y"][lo:hi].double())
        gx[lo:hi] = grads[0]
        for m, v in zip(gw, grads[1:]):
            m[e] = v
    return [gx] + gw


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "block":
        y = _exact_y(s, *(None if s[n] is None else s[n].double() for n in ("x", "b", "post_w", "gate", "token_gate")))
        return [y] if s["open_w"] is None else [y, _exact_rms(y.to(s["x"].dtype).double(), s["open_w"].double())]
    if kind == "block_grad":
        return _exact_block_grad(s)
    if kind == "experts_grad":
        return _exact_experts_grad(s)
    k, pairs = case["top_k"], case["tokens"] * case["top_k"]
    inv = s["inv"].flatten().long()
    live = inv[inv >= 0]
    # rows from tokens as a matrix of weights: a pair's row is its weight times its token
    token = torch.arange(pairs, device=inv.device)[inv >= 0] // k
    weight = torch.ones(pairs, dtype=torch.float64, device=inv.device) if s["weight"] is None else s["weight"].double().flatten()
    weight = weight[inv >= 0, None]
    if kind == "dispatch":
        rows = torch.zeros(pairs, case["d_model"], dtype=torch.float64, device=inv.device)
        rows[live] = s["x"].double()[token] * weight
        return None, None, None, rows
    if kind == "dispatch_grad":
        g = s["grad_rows"].double()[live]
        gx = torch.zeros(s["x"].shape, dtype=torch.float64, device=inv.device).index_add_(0, token, g * weight)
        if s["weight"] is None:
            return gx
        gw = torch.zeros(pairs, dtype=torch.float64, device=inv.device)
        gw[inv >= 0] = torch.linalg.vecdot(g, s["x"].double()[token])
        return gx, gw.view(-1, k)
    rows = s["rows"].double()[live]
    if kind == "collect":
        y = torch.zeros(s["x"].shape, dtype=torch.float64, device=inv.device).index_add_(0, token, rows * weight)
        return y if s["residual"] is None else y + s["residual"].double()
    gy = s["grad_y"].double()[token]
    grad = torch.zeros(pairs, case["d_model"], dtype=torch.float64, device=inv.device)
    grad[live] = gy * weight
    grad_gate = torch.zeros(pairs, dtype=torch.float64, device=inv.device)
    grad_gate[inv >= 0] = torch.linalg.vecdot(gy, rows)
    return grad, grad_gate.view(-1, k)
