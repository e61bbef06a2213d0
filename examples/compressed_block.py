#!/usr/bin/env python3
"""A gated feed-forward block of a language model, compressed to 4 bits, served and tuned.

    python examples/compressed_block.py [--width 512] [--hidden 1024] [--vocab 4096] [--group 128] [--steps 40]

The dense block is  logits = head(down(up(norm(x + r)))), with random weights and correlated inputs.  The example

1. calibrates each linear layer on its inputs and quantizes it with OBQ on group grids: a group of columns at a time,
   the columns behind it moved to make up for what the group lost, as Sec. 4 does for single weights;
2. packs the codes and runs the block: norm with 8-bit outputs into a 4-bit product for serving, 16-bit throughout for
   tuning;
3. tunes what stays uncompressed -- the norm's gain -- against the dense block's top logits, through the frozen codes:
   distillation loss, gradients through the 4-bit products, the norm's backward pass.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2208_11580_amd as obc  # noqa: E402


def quantize(ctx, W, X, group):
    """OBQ of W (rows x cols) for inputs X (cols x samples) on 4-bit grids of `group` columns: codes, steps, offsets."""
    R, d = W.shape
    codes = torch.empty(R, d, dtype=torch.int32, device=W.device)
    steps, offsets = [], []
    W = W.double()
    Hinv = ctx.obc_invert(ctx.obc_hessian(X, damp_rel=0.01)).double()
    for a in range(0, d, group):
        b = min(a + group, d)
        own = W[:, a:b].float().contiguous()
        delta, offset, maxq = ctx.obc_group_grid(own, 4)
        # the group's own columns, the others being free to follow: their inverse Hessian is this block of the whole one
        block = Hinv[a:b, a:b]
        q = ctx.obc_quant_rows(own, block.float().contiguous(), delta[:, 0].contiguous(), offset[:, 0].contiguous(), maxq)
        codes[:, a:b] = q["codes"]
        steps.append(delta)
        offsets.append(offset)
        # eq. (5) for the group as a whole, then Lemma 1: the columns behind it, and their inverse Hessian without it
        solved = torch.linalg.solve(block, Hinv[a:b, b:])
        W[:, b:] -= (W[:, a:b] - q["W"].double()) @ solved
        Hinv[b:, b:] -= Hinv[b:, a:b] @ solved
    ctx.obc_check()
    return codes, torch.cat(steps, 1).contiguous(), torch.cat(offsets, 1).contiguous()


def nearest(ctx, W, group):
    """The same grids without the Hessian: every weight to the nearest value."""
    d = W.shape[1]
    delta, offset, maxq = ctx.obc_group_grid(W, 4, group)
    g = torch.arange(d, device=W.device) // group
    return torch.round((W - offset[:, g]) / delta[:, g]).clamp(0, maxq).to(torch.int32), delta, offset


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--vocab", type=int, default=4096)
    ap.add_argument("--group", type=int, default=128)
    ap.add_argument("--tokens", type=int, default=768)
    ap.add_argument("--top", type=int, default=32)
    ap.add_argument("--steps", type=int, default=40)
    a = ap.parse_args(argv)
    dev = "cuda:0"
    gen = torch.Generator(device=dev)
    gen.manual_seed(1)

    def rand(*shape, scale=1.0):
        return torch.randn(*shape, generator=gen, device=dev) * scale

    ctx = obc.Context()
    bf16 = torch.bfloat16
    mix = rand(a.width, a.width, scale=a.width ** -0.5)
    x = (rand(a.tokens, a.width) @ mix).to(bf16)
    residual = (2.0 * rand(a.tokens, a.width) @ mix).to(bf16)
    gain = 1.0 + 0.2 * rand(a.width)
    dense = [rand(a.hidden, a.width, scale=a.width ** -0.5), rand(a.width, a.hidden, scale=a.hidden ** -0.5),
             rand(a.vocab, a.width, scale=4.0 * a.width ** -0.5)]

    # the dense block, in fp32
    h = ctx.obc_rmsnorm(x, gain, residual=residual)["h"]
    inputs = [h.float() * (h.float().square().mean(1, keepdim=True) + 1e-6).rsqrt() * gain]
    for W in dense[:2]:
        inputs.append(inputs[-1] @ W.T)
    logits = inputs[-1] @ dense[2].T
    top = logits.topk(a.top, dim=1)
    top_index, top_logit = top.indices.to(torch.int32).contiguous(), top.values.contiguous()

    # 1. quantize: each layer on its dense inputs
    report = {}
    packed = []
    for i, W in enumerate(dense):
        X = inputs[i].t().contiguous()
        want = inputs[i] @ W.T
        for name, q in (("nearest", nearest(ctx, W, a.group)), ("obq", quantize(ctx, W, X, a.group))):
            P = ctx.obc_pack4(*q, group=a.group)
            err = ctx.obc_product4(P, inputs[i]) - want
            report["layer%d_%s" % (i, name)] = float(err.norm() / want.norm())
        packed.append(P)
    ctx.obc_check()

    # 2. serve: one token after the other and the whole prompt, the norm's output in 8 bits
    def serve(x, residual):
        n = ctx.obc_rmsnorm(x, gain, residual=residual, quant8=True)
        y = ctx.obc_product4(packed[0], n["y"], x_scale=n["scale"], out_dtype=bf16)
        return ctx.obc_product4(packed[2], ctx.obc_product4(packed[1], y), out_dtype=torch.float32)

    prompt = serve(x, residual)
    single = torch.cat([serve(x[t:t + 1], residual[t:t + 1]) for t in range(8)])
    report["served_logits"] = float((prompt - logits).norm() / logits.norm())
    report["single_against_prompt"] = float((single - prompt[:8]).norm() / prompt[:8].norm())

    # 3. tune the gain against the dense block's top logits
    weight = torch.full((a.tokens,), 1.0 / a.tokens, device=dev)
    tuned = gain.clone()
    losses = []
    for _ in range(a.steps):
        n = ctx.obc_rmsnorm(x, tuned, residual=residual, want_rstd=True)
        y1 = ctx.obc_product4(packed[0], n["y"])
        y2 = ctx.obc_product4(packed[1], y1)
        z = ctx.obc_product4(packed[2], y2)
        loss = ctx.obc_distill(z, top_index, top_logit, temperature=1.0, weight=weight, want_grad=True, out={"dz": z})
        losses.append(float(loss["loss"].sum()))
        g = ctx.obc_product4_grad(packed[2], loss["dz"])
        g = ctx.obc_product4_grad(packed[0], ctx.obc_product4_grad(packed[1], g))
        dgain = ctx.obc_rmsnorm_grad(n["h"], tuned, n["rstd"], g)["dgain"]
        tuned -= 0.02 * dgain / (dgain.square().mean().sqrt() + 1e-12)
    ctx.obc_check()
    report["loss_before"], report["loss_after"] = losses[0], min(losses)
    for k, v in report.items():
        print("%-24s %.5f" % (k, v))
    ctx.close()
    return report


if __name__ == "__main__":
    main()
