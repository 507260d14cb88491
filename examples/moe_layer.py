"""Loads one mixture-of-experts layer and runs its products on the parameters as loaded.

    python examples/moe_layer.py [--tokens 64] [--hidden 1024] [--inter 3584] [--experts 8]

The checkpoint (seeded random weights in Mixtral's layout) lies in page-locked host memory.  A plan
fuses q/k/v and stacks the experts' w1/w3 and w2; the layer's readiness group gates the stream that
the operators run on, so the host never waits between the load and the result:

    load_async -> wait_layer(1, stream) -> linear (qkv)
                                        -> linear (router logits) -> route -> experts (+ residual)
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2607_18957_gb300 as cfa  # noqa: E402
from workloads import moe_config  # noqa: E402
from workloads.harness import entries_for  # noqa: E402

LAYER = "model.layers.0."
TOP_K = 2


def checkpoint(m, seed):
    """The blob of manifest m with seeded normal weights, scaled by their row length."""
    g = torch.Generator().manual_seed(seed)
    blob = torch.zeros(m.blob_bytes, dtype=torch.uint8).pin_memory()
    tensors = {}
    for i, name in enumerate(m.e_name):
        shape, at = m.e_shape_tuple(i), int(m.e_offset[i])
        t = (torch.randn(shape, generator=g) * shape[-1] ** -0.5).to(torch.bfloat16)
        blob[at:at + t.numel() * 2].view(torch.bfloat16).copy_(t.view(-1))
        tensors[name] = t
    return blob, tensors


def run(tokens=64, hidden=1024, inter=3584, experts=8, seed=0):
    """(results of the operators, the same in 64 bits on the checkpoint's own tensors)."""
    m = moe_config("moe_layer", seed, layers=1, hidden=hidden, n_q=hidden // 64,
                   n_kv=max(1, hidden // 256), head_dim=64, inter=inter, n_experts=experts,
                   vocab=256)
    blob, tensors = checkpoint(m, seed)
    params = {m.d_name[j]: torch.empty(m.d_shape_tuple(j), dtype=torch.bfloat16, device="cuda")
              for j in range(m.n_dsts)}
    dsts = [(p.data_ptr(), "bf16", tuple(p.shape)) for p in params.values()]
    x = torch.randn(tokens, hidden, generator=torch.Generator().manual_seed(seed + 1))
    x = x.to(torch.bfloat16).cuda()

    moe = LAYER + "block_sparse_moe."
    stream = torch.cuda.current_stream()
    with cfa.Plan(entries_for(m), dsts, m.blob_bytes, chunk_bytes=1 << 20) as plan:
        plan.load_async(cfa.Source.pinned(blob.data_ptr()), stream)
        plan.wait_layer(1, stream=stream)  # the stream waits, the host does not
        qkv = cfa.linear(x, params[LAYER + "self_attn.qkv_proj.weight"])
        logits = cfa.linear(x, params[moe + "gate.weight"], out_dtype="f32")
        weights, ids = cfa.route(logits, TOP_K)
        y = cfa.experts(x, ids, weights, params[moe + "experts.w13_weight"],
                        params[moe + "experts.w2_weight"], residual=x)
        plan.wait_layer()

    x64 = x.double().cpu()
    w = {n: t.double() for n, t in tensors.items()}
    p = LAYER + "self_attn."
    want = {"qkv": torch.cat([x64 @ w[p + n + "_proj.weight"].t() for n in "qkv"], dim=1),
            "logits": x64 @ w[moe + "gate.weight"].t(), "y": x64.clone()}
    for t in range(tokens):
        for j in range(TOP_K):
            q = moe + f"experts.{ids[t, j].item()}."
            a = w[q + "w1.weight"] @ x64[t]
            h = a * torch.sigmoid(a) * (w[q + "w3.weight"] @ x64[t])
            want["y"][t] += weights[t, j].item() * (w[q + "w2.weight"] @ h)
    got = {"qkv": qkv.cpu(), "logits": logits.cpu(), "y": y.cpu()}
    return got, want


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    for name, default in (("tokens", 64), ("hidden", 1024), ("inter", 3584), ("experts", 8)):
        ap.add_argument("--" + name, type=int, default=default)
    results, expected = run(**vars(ap.parse_args()))
    for key, v in results.items():
        off = ((v.double() - expected[key]).norm() / expected[key].norm()).item()
        print(f"{key:7s} {tuple(v.shape)}  {v.dtype}  relative difference from 64 bits {off:.2e}")
