"""Loads a decoder of one layer and runs prompts and decoding steps on the parameters as loaded.

    python examples/decode_step.py [--sequences 5] [--hidden 512] [--steps 2]

The checkpoint (seeded random weights) lies in page-locked host memory.  A plan fuses q/k/v and gate/up;
each readiness group gates the stream that the operators run on.  The prompts' keys and values go into
the paged cache in one call; then every step takes one token of each sequence through

    norm -> linear (qkv) -> append -> attend -> linear (o, + residual) -> norm -> linear (gate/up)
         -> linear (down, + residual) -> norm -> linear (vocabulary) -> logprobs

and goes on with the likeliest token.  Of several sequences the one in the middle is a padded row: its
length is 0 and its slots are -1.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2607_18957_gb300 as cfa  # noqa: E402
from examples.moe_layer import checkpoint  # noqa: E402
from workloads import dense_config  # noqa: E402
from workloads.harness import entries_for  # noqa: E402

LAYER = "model.layers.0."
PAGE, TOP = 16, 5


class Step:
    """One decoding step over buffers that stay where they are, so that it can be captured as a graph."""

    def __init__(self, params, heads, kv_heads, dim, lengths, pages, caches):
        self.p, self.heads, self.kv_heads, self.dim = params, heads, kv_heads, dim
        self.lengths, self.pages, (self.k, self.v) = lengths, pages, caches
        f, self.magnitude = cfa.rotary_frequencies(dim, 500000.0, scaling="bands", factor=8.0, length=8192)
        self.frequencies = torch.tensor(f, dtype=torch.float64, device="cuda")
        self.tokens = torch.zeros(lengths.shape, dtype=torch.int32, device="cuda")
        self.none = torch.full_like(self.tokens, -1)

    def rotary(self, positions):
        return dict(positions=positions, frequencies=self.frequencies, magnitude=self.magnitude)

    def prompt(self, tokens, positions, slots):
        """Appends the prompts' keys and values: with one layer they need nothing but the embeddings."""
        x = self.p["model.embed_tokens.weight"][tokens]
        h = cfa.norm(x, self.p[LAYER + "input_layernorm.weight"])
        qkv = cfa.linear(h, self.p[LAYER + "self_attn.qkv_proj.weight"])
        cfa.append(qkv, self.k, self.v, slots, heads=self.heads, **self.rotary(positions))

    def __call__(self, slots):
        """(logits, log probabilities of the tokens chosen, entropy, the best, their ids)

        The tokens chosen, which the next step takes in, are the best ones: none are given beforehand."""
        p, mlp, attn = self.p, LAYER + "mlp.", LAYER + "self_attn."
        x = p["model.embed_tokens.weight"][self.tokens]
        h = cfa.norm(x, p[LAYER + "input_layernorm.weight"])
        qkv = cfa.linear(h, p[attn + "qkv_proj.weight"])
        q = cfa.append(qkv, self.k, self.v, slots, heads=self.heads, **self.rotary(self.lengths - 1))
        a = cfa.attend(q, self.k, self.v, self.pages, self.lengths)
        a = cfa.linear(a.flatten(1), p[attn + "o_proj.weight"])
        h, x = cfa.norm(a, p[LAYER + "post_attention_layernorm.weight"], residual=x)
        m = cfa.linear(h, p[mlp + "gate_up_proj.weight"], activation="silu", gated=True)
        m = cfa.linear(m, p[mlp + "down_proj.weight"])
        h, _ = cfa.norm(m, p["model.norm.weight"], residual=x)
        logits = cfa.linear(h, p["lm_head.weight"], out_dtype="f32")
        _, entropy, best, ids = cfa.logprobs(logits, self.none, top=TOP)
        return logits, best[:, 0], entropy, best, ids


def reference(w, tokens, heads, kv_heads, dim, frequencies):
    """Logits of the last position of one sequence in 64 bits, from the checkpoint's own tensors."""
    def norm(v, name):
        return v / torch.sqrt((v * v).mean(-1, keepdim=True) + 1e-6) * w[name]

    def turn(v):
        angle = torch.arange(len(tokens), dtype=torch.float64)[:, None, None] * frequencies
        a, b = v.chunk(2, -1)
        return torch.cat((a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()), -1)

    x = w["model.embed_tokens.weight"][tokens]
    h = norm(x, LAYER + "input_layernorm.weight")
    q, k, v = ((h @ w[LAYER + f"self_attn.{n}_proj.weight"].t()).unflatten(1, (-1, dim)) for n in "qkv")
    q, k = turn(q)[-1].view(kv_heads, -1, dim), turn(k)
    p = torch.softmax(torch.einsum("hgd,nhd->hgn", q, k) * dim ** -0.5, 2)
    x = x[-1] + torch.einsum("hgn,nhd->hgd", p, v).flatten() @ w[LAYER + "self_attn.o_proj.weight"].t()
    h = norm(x, LAYER + "post_attention_layernorm.weight")
    gate = h @ w[LAYER + "mlp.gate_proj.weight"].t()
    x = x + (gate * torch.sigmoid(gate) * (h @ w[LAYER + "mlp.up_proj.weight"].t())) @ \
        w[LAYER + "mlp.down_proj.weight"].t()
    return norm(x, "model.norm.weight") @ w["lm_head.weight"].t()


def run(sequences=5, hidden=512, steps=2, seed=0, graph=True):
    """For each step the operators' results, the logits in 64 bits and the tokens chosen."""
    dim, vocab = 64, 1000
    heads, kv_heads = hidden // dim, max(1, hidden // dim // 4)
    m = dense_config("decode_step", seed, layers=1, hidden=hidden, n_q=heads, n_kv=kv_heads, head_dim=dim,
                     inter=2 * hidden, vocab=vocab)
    blob, tensors = checkpoint(m, seed)
    params = {m.d_name[j]: torch.empty(m.d_shape_tuple(j), dtype=torch.bfloat16, device="cuda")
              for j in range(m.n_dsts)}
    dsts = [(p.data_ptr(), "bf16", tuple(p.shape)) for p in params.values()]

    g = torch.Generator().manual_seed(seed + 1)
    padded = sequences // 2 if sequences > 1 else None
    lens = [0 if s == padded else 1 + (37 * s + 11) % 90 for s in range(sequences)]
    told = [torch.randint(0, vocab, (n + 1,), generator=g) for n in lens]  # a prompt and a token more
    per = (max(lens) + steps) // PAGE + 1
    order = torch.randperm(sequences * per, generator=g).view(sequences, per)
    caches = torch.zeros(2, sequences * per, PAGE, kv_heads, dim, dtype=torch.bfloat16, device="cuda")

    def slots_of(s, positions):
        return (order[s, positions // PAGE] * PAGE + positions % PAGE).tolist()

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    prompts = [(s, torch.arange(n)) for s, n in enumerate(lens)]
    step = Step(params, heads, kv_heads, dim, ints(lens), order.to(torch.int32).cuda(), caches)
    slots = torch.full((sequences,), -1, dtype=torch.int32, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    found = []
    with torch.cuda.stream(stream), cfa.Plan(entries_for(m), dsts, m.blob_bytes,
                                             chunk_bytes=1 << 20) as plan:
        plan.load_async(cfa.Source.pinned(blob.data_ptr()), stream)
        plan.wait_layer(stream=stream)  # the stream waits, the host does not
        step.prompt(torch.cat([told[s][:-1] for s, _ in prompts]).cuda(),
                    ints(torch.cat([p for _, p in prompts]).tolist()),
                    ints([x for s, p in prompts for x in slots_of(s, p)]))
        step.tokens.copy_(ints([t[-1].item() for t in told]))
        captured = None
        for _ in range(steps):
            lens = [0 if s == padded else n + 1 for s, n in enumerate(lens)]
            step.lengths.copy_(ints(lens))
            slots.copy_(ints([slots_of(s, torch.tensor([n - 1]))[0] if n else -1
                              for s, n in enumerate(lens)]))
            if not graph:
                results = step(slots)
            elif captured is None:
                step(slots)  # the same keys and values again: what a capture must not set up, set up
                captured = torch.cuda.CUDAGraph()
                with torch.cuda.graph(captured, stream=stream):
                    results = step(slots)
                captured.replay()
            else:
                captured.replay()
            stream.synchronize()
            found.append([r.cpu().clone() for r in results])
            step.tokens.copy_(results[4][:, 0])
            chosen = results[4][:, 0].tolist()
            told = [torch.cat((t, torch.tensor([c]))) for t, c in zip(told, chosen)]
        plan.wait_layer()

    w = {n: t.double() for n, t in tensors.items()}
    f = step.frequencies.cpu()
    wanted = [[None if s == padded else reference(w, told[s][:len(told[s]) - steps + i], heads, kv_heads, dim,
                                                  f) for s in range(sequences)] for i in range(steps)]
    chosen = [[t[len(t) - steps + i].item() for t in told] for i in range(steps)]
    return found, wanted, chosen


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    for name, default in (("sequences", 5), ("hidden", 512), ("steps", 2)):
        ap.add_argument("--" + name, type=int, default=default)
    for n, (r, e, tokens) in enumerate(zip(*run(**vars(ap.parse_args())))):
        for s, z in enumerate(e):
            if z is not None:
                off = ((r[0][s].double() - z).norm() / z.norm()).item()
                print(f"step {n} sequence {s}: token {tokens[s]}, log probability {r[1][s].item():.4f}, "
                      f"relative difference of the logits from 64 bits {off:.2e}")
