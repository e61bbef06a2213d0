#!/usr/bin/env python3
"""A small language model with layers of 4 bits, judged and tuned against the dense one.

    python examples/tuned_model.py [--width 256] [--hidden 512] [--vocab 4000] [--tokens 512] [--top 32] [--steps 30]

The model is  logits = head(norm2(down(up(norm1(x))) + x)),  x = scale table[ids],  with random weights.  The example

1. rounds its linear layers to 4 bits on group grids and packs them;
2. judges both models' answers: log probabilities of the next tokens, entropies;
3. takes the dense model's top logits and tunes what stays uncompressed against them -- the embedding table (16 bits with an
   fp32 copy, 8-bit moments), the norms' gains and biases (fp32) -- with gradients through the 4-bit products and AdamW
   steps, one training step being captured into a graph and replayed.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2208_11580_amd as obc  # noqa: E402


def forward(ctx, p, layers, ids, scale):
    """Logits of the compressed model, and what its backward pass needs.  p: table, gain1, bias1, gain2, bias2."""
    x = ctx.obc_embed(p["table"], ids, scale=scale)
    n1 = ctx.obc_layernorm(x, p["gain1"], p["bias1"], want_stats=True)
    u = ctx.obc_product4(layers["down"], ctx.obc_product4(layers["up"], n1["y"]))
    n2 = ctx.obc_layernorm(u, p["gain2"], p["bias2"], residual=x, want_stats=True)
    return ctx.obc_product4(layers["head"], n2["y"]), n1, n2


def backward(ctx, p, layers, ids, scale, n1, n2, dz):
    """Gradients of the parameters from those of the logits."""
    g2 = ctx.obc_layernorm_grad(n2["h"], p["gain2"], n2["mean"], n2["rstd"], ctx.obc_product4_grad(layers["head"], dz))
    dy = ctx.obc_product4_grad(layers["up"], ctx.obc_product4_grad(layers["down"], g2["dx"]))
    # the residual path's gradient is added on the way
    g1 = ctx.obc_layernorm_grad(n1["h"], p["gain1"], n1["mean"], n1["rstd"], dy, dh=g2["dx"])
    return dict(table=ctx.obc_embed_grad(ids, g1["dx"], p["table"].shape[0], scale=scale), gain1=g1["dgain"], bias1=g1["dbias"],
                gain2=g2["dgain"], bias2=g2["dbias"])


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--hidden", type=int, default=512)
    ap.add_argument("--vocab", type=int, default=4000)
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--group", type=int, default=64)
    ap.add_argument("--top", type=int, default=32)
    ap.add_argument("--steps", type=int, default=30)
    a = ap.parse_args(argv)
    dev, bf16 = "cuda:0", torch.bfloat16
    gen = torch.Generator(device=dev)
    gen.manual_seed(1)

    def rand(*shape, scale=1.0):
        return torch.randn(*shape, generator=gen, device=dev) * scale

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ctx = obc.Context(side)
        scale = float(a.width) ** 0.5
        p = {"table": rand(a.vocab, a.width, scale=1.0 / scale).to(bf16)}
        for n in ("1", "2"):
            p["gain" + n], p["bias" + n] = 1.0 + 0.2 * rand(a.width), 0.1 * rand(a.width)
        dense = {"up": rand(a.hidden, a.width, scale=a.width ** -0.5), "down": rand(a.width, a.hidden, scale=a.hidden ** -0.5),
                 "head": rand(a.vocab, a.width, scale=4.0 * a.width ** -0.5)}
        ids = (torch.rand(a.tokens, generator=gen, device=dev).pow(3) * a.vocab).to(torch.int32)
        follow = torch.cat([ids[1:], ids.new_full((1,), -1)])

        # the dense model, in fp32
        x = p["table"].float()[ids.long()] * scale
        h = torch.nn.functional.layer_norm(x, (a.width,), p["gain1"], p["bias1"]) @ dense["up"].T @ dense["down"].T + x
        logits = torch.nn.functional.layer_norm(h, (a.width,), p["gain2"], p["bias2"]) @ dense["head"].T

        # 1. four bits
        layers = {}
        for name, W in dense.items():
            delta, offset, maxq = ctx.obc_group_grid(W, 4, a.group)
            g = torch.arange(W.shape[1], device=dev) // a.group
            codes = torch.round((W - offset[:, g]) / delta[:, g]).clamp(0, maxq).to(torch.int32)
            layers[name] = ctx.obc_pack4(codes, delta, offset, group=a.group)

        # 2. judged, and the dense model's top logits
        teacher = ctx.obc_score(logits, follow, top=a.top)

        def judge():
            s = ctx.obc_score(forward(ctx, p, layers, ids, scale)[0], teacher["top_index"][:, 0].contiguous())
            return float(s["logp"].mean()), float(s["entropy"].mean())

        report = {"dense_logp": float(teacher["logp"][:-1].mean()), "dense_entropy": float(teacher["entropy"].mean())}
        report["agreement_before"], report["entropy_before"] = judge()

        # 3. tuned
        small = ["gain1", "bias1", "gain2", "bias2"]
        grads = {n: torch.zeros_like(t) for n, t in p.items()}
        table = ctx.obc_adamw_plan([p["table"]], [grads["table"]], [ctx.obc_adamw_state(p["table"], bits=8, master=True)], decay=0.0)
        norms = ctx.obc_adamw_plan([p[n] for n in small], [grads[n] for n in small], [ctx.obc_adamw_state(p[n]) for n in small], decay=0.0)
        step = torch.ones(1, dtype=torch.int64, device=dev)
        weight = torch.full((a.tokens,), 1.0 / a.tokens, device=dev)
        loss = torch.empty(a.tokens, device=dev)

        def train():
            z, n1, n2 = forward(ctx, p, layers, ids, scale)
            r = ctx.obc_distill(z, teacher["top_index"], teacher["top_logit"], weight=weight, want_grad=True, out={"dz": z, "loss": loss})
            for n, g in backward(ctx, p, layers, ids, scale, n1, n2, r["dz"]).items():
                grads[n].copy_(g)
            ctx.obc_adamw(table, step, 1e-3)
            ctx.obc_adamw(norms, step, 1e-2)
            step.add_(1)

        train()
        losses = [float(loss.sum())]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            train()
        for _ in range(a.steps):
            graph.replay()
            losses.append(float(loss.sum()))
        report["loss_before"], report["loss_after"] = losses[0], losses[-1]
        report["agreement_after"], report["entropy_after"] = judge()
        report["steps"] = int(step) - 1
        ctx.obc_check()
        side.synchronize()
        del graph
        ctx.close()
    for k, v in report.items():
        print("%-20s %.5f" % (k, v))
    return report


if __name__ == "__main__":
    main()
