"""Captured graphs of the operators around compressed layers beside later work on the same context."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _layer(ctx, R, d, g):
    codes = torch.randint(0, 16, (R, d), generator=g, device="cuda", dtype=torch.int32)
    delta = (torch.rand(R, -(-d // 64), generator=g, device="cuda") * 0.02 + 0.001).half().float()
    return ctx.obc_pack4(codes, delta, -7.0 * delta, group=64)


@pytest.mark.parametrize("own_stream", [True, False])
def test_a_graph_keeps_its_workspace(own_stream):
    """Small products and gradients are captured; then longer eager ones on the same context need a larger workspace, it is released,
    and its memory goes to other tensors.  Replays give what eager calls give and write nothing of those tensors."""
    import paper_2208_11580_amd as pkg

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ctx = pkg.Context(side)
        g = torch.Generator(device="cuda")
        g.manual_seed(7)
        R, d = 600, 520
        P = _layer(ctx, R, d, g)
        gain = torch.rand(d, generator=g, device="cuda") + 0.5
        x = torch.randn(40, d, generator=g, device="cuda").bfloat16()
        long = torch.randn(3000, d, generator=g, device="cuda")

        def work(x):
            n = ctx.obc_rmsnorm(x, gain, want_rstd=True)
            y = ctx.obc_product4(P, n["y"])
            dy = ctx.obc_product4_grad(P, y)
            r = ctx.obc_rmsnorm_grad(x, gain, n["rstd"], dy)
            return [y, dy, r["dx"], r["dgain"]]

        work(x)
        side.synchronize()
        graphs = []
        for _ in range(2):                      # two graphs of one context
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                graphs.append((graph, work(x)))
        want = [t.clone() for t in work(x)]
        held = ctx._ws.numel()
        others = []
        for turn in range(4):
            if turn == 1:
                work(long)
                assert ctx._ws.numel() > held
            if turn == 2:
                ctx.release_workspace()
            side.synchronize()
            # what was freed: tensors of all sizes up to the workspaces', which the replays must not touch
            others += [torch.full((n,), 0x5a, dtype=torch.uint8, device="cuda") for n in (1 << 14, 1 << 17, 1 << 20, 1 << 22, held) for _ in range(4)]
            for graph, got in graphs:
                for t in got:
                    t.zero_()
                if own_stream:
                    graph.replay()
                else:                            # another stream than the context's, eager work on the context's beside it
                    side.synchronize()
                    with torch.cuda.stream(torch.cuda.default_stream()):
                        graph.replay()
                    eager = work(x)
                torch.cuda.synchronize()
                for a, b in zip(got, want):
                    assert torch.equal(a, b), turn
                if not own_stream:
                    for a, b in zip(eager, want):
                        assert torch.equal(a, b), turn
            for t in others:
                assert (t == 0x5a).all(), turn
        ctx.obc_check()
        ctx.close()


def test_a_context_whose_stream_joins_a_capture():
    """The capture begins on one stream and the context works on another that waits for it."""
    import paper_2208_11580_amd as pkg

    first, side = torch.cuda.Stream(), torch.cuda.Stream()
    ctx = pkg.Context(side)
    g = torch.Generator(device="cuda")
    g.manual_seed(8)
    P = _layer(ctx, 300, 260, g)
    x = torch.randn(50, 260, generator=g, device="cuda")
    doubled = 2.0 * x
    torch.cuda.synchronize()
    want = ctx.obc_product4(P, doubled)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=first):
        twice = 2.0 * x
        side.wait_stream(first)
        y = ctx.obc_product4(P, twice)
        first.wait_stream(side)
        z = y + 0.0
    big = torch.randn(2000, 260, generator=g, device="cuda")
    torch.cuda.synchronize()
    for _ in range(3):
        ctx.obc_product4(P, big)
        side.synchronize()
        z.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(z, want)
    ctx.obc_check()
    ctx.close()
