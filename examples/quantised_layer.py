"""A layer of experts in 4 bits, from a bf16 checkpoint's matrices to a prompt and generated tokens.

    python examples/quantised_layer.py [--tokens 300] [--experts 32]

Quantises the three matrices of every expert (moe_mxfp4_quantize), lays them out (make_mxfp4_weights), runs a prompt
and a few single tokens through router, picks and experts in one call (moe_mxfp4_forward), compares with the same layer
on the unquantised weights (moe_forward's experts on the same picks), and takes the gradient of the gates with
regard to the router's logits, as a training step of the router alone would (moe_route_scored_backward).
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2503_00245_amd as moe  # noqa: E402


def quantise(w):
    """[E, R, C] -> codes, scales"""
    codes = torch.empty(*w.shape[:-1], w.shape[-1] // 2, dtype=torch.uint8, device=w.device)
    scales = torch.empty(*w.shape[:-1], (w.shape[-1] + 31) // 32, dtype=torch.uint8, device=w.device)
    moe.moe_mxfp4_quantize(w, codes, scales)
    return codes, scales


def main(tokens=300, experts=32, d=1024, f=2816, top_k=4):
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev)
    g.manual_seed(1)
    normal = lambda *shape, std=1.0: torch.randn(*shape, generator=g, device=dev) * std  # noqa: E731
    dense = {"gate": normal(experts, f, d, std=0.02).bfloat16(), "up": normal(experts, f, d, std=0.02).bfloat16(),
             "down": normal(experts, d, f, std=0.02).bfloat16()}
    router = {"router_w": normal(experts, d, std=0.02), "router_b": None, "select_bias": normal(experts, std=0.01)}
    quantised = dict(router)
    for name, w in dense.items():
        quantised[name + "_codes"], quantised[name + "_scales"] = quantise(w)
    weights = moe.make_mxfp4_weights(quantised)
    # scores by sigmoid, the best half of four groups of experts, gates that sum to 1
    config = moe.make_route_config(moe.SCORE_SIGMOID, n_groups=4, groups_kept=2, group_top=2)

    errors = []
    for t in (tokens, 1, 1, 1):  # the prompt, then generated tokens
        x = normal(t, d).bfloat16()
        shape = moe.make_shape(t, d, f, experts, top_k)
        workspace = moe.alloc_mxfp4_workspace(shape, dev)
        y, logits = torch.empty_like(x), torch.empty(t, experts, device=dev)
        idx, gate = torch.empty(t, top_k, dtype=torch.int32, device=dev), torch.empty(t, top_k, device=dev)
        moe.moe_mxfp4_forward(shape, config, weights, x, y, idx, gate, logits, workspace)

        # the unquantised experts on the same picks, stage by stage
        pairs = t * top_k
        offsets = torch.empty(experts + 1, dtype=torch.int32, device=dev)
        perm, inv = torch.empty(pairs, dtype=torch.int32, device=dev), torch.empty(pairs, dtype=torch.int32, device=dev)
        rows, out, ref = x.new_empty(pairs, d), x.new_empty(pairs, d), torch.empty_like(x)
        ws = moe.alloc_workspace(shape, dev)
        moe.moe_permute(shape, idx, offsets, perm, inv, x, rows, ws)
        dense_weights = moe.make_weights({"router_w": router["router_w"], "w_gate": dense["gate"], "w_up": dense["up"], "w_down": dense["down"]})
        moe.moe_expert_ffn(shape, dense_weights, rows, offsets, out, ws)
        moe.moe_combine(shape, out, inv, gate, None, ref)
        err = float((y.float() - ref.float()).norm() / ref.float().norm())
        errors.append(err)
        print(f"{t:5d} tokens: 4-bit experts differ from the bf16 ones by {err:.3f} of the output's norm")

        # what a loss on the gates says about the logits
        grad = torch.empty_like(logits)
        moe.moe_route_scored_backward(config, logits, idx, torch.ones_like(gate), None, grad)
        print(f"              gradient of the sum of the gates, which is 1: at most {float(grad.abs().max()):.1e}")
        assert float(grad.abs().max()) < 1e-5
    held = sum(t.numel() for n, t in weights.tensors.items() if n in ("gate", "up", "down"))
    whole = sum(w.numel() * 2 for w in dense.values())
    print(f"weights: {held / 1e6:.0f} MB in place of {whole / 1e6:.0f}")
    return errors


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--tokens", type=int, default=300)
    ap.add_argument("--experts", type=int, default=32)
    a = ap.parse_args()
    main(a.tokens, a.experts)
