"""The operators by which compressed models are judged and tuned as they are used together: a model's gradients and step against
autograd in 64 bits, captured in a graph, on other streams, two graphs at once; the example."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("tuned_model", os.path.join(ROOT, "examples", "tuned_model.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_example_model():
    r = _example().main(["--width", "128", "--hidden", "192", "--vocab", "500", "--tokens", "200", "--top", "8", "--steps", "5"])
    assert r["steps"] == 6
    assert all(v == v and abs(v) < 1e6 for v in r.values())


def _model(ctx, kind, g, V=300, d=96, hidden=130, T=150):
    def rand(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * scale

    p = {"table": rand(V, d, scale=d ** -0.5).to(kind), "gain1": 1 + 0.2 * rand(d), "bias1": 0.1 * rand(d), "gain2": 1 + 0.2 * rand(d),
         "bias2": 0.1 * rand(d)}
    layers, weights = {}, {}
    for name, R, c in (("up", hidden, d), ("down", d, hidden), ("head", V, d)):
        codes = torch.randint(0, 16, (R, c), generator=g, device="cuda", dtype=torch.int32)
        delta = (torch.rand(R, -(-c // 32), generator=g, device="cuda") * 0.5 * c ** -0.5 + 0.1 * c ** -0.5).half().float()
        offset = (-7.5 * delta).half().float()
        layers[name] = ctx.obc_pack4(codes, delta, offset, group=32)
        at = torch.arange(c, device="cuda") // 32
        weights[name] = offset.double()[:, at] + delta.double()[:, at] * codes.double()
    ids = torch.randint(-1, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    teacher = ctx.obc_score(2.0 * rand(T, V), top=9)
    return p, layers, weights, ids, teacher


def _autograd(p, weights, ids, scale, teacher):
    q = {n: t.double().requires_grad_() for n, t in p.items()}
    d = q["table"].shape[1]
    x = torch.where(ids[:, None] >= 0, q["table"][ids.clamp_min(0).long()] * scale, 0.0)
    norm = lambda h, n: torch.nn.functional.layer_norm(h, (d,), q["gain" + n], q["bias" + n], 1e-5)  # noqa: E731
    h = norm(x, "1") @ weights["up"].T @ weights["down"].T + x
    z = norm(h, "2") @ weights["head"].T
    logq = torch.log_softmax(z, 1)
    prob = torch.softmax(teacher["top_logit"].double(), 1)
    loss = (prob * (prob.log() - logq.gather(1, teacher["top_index"].long()))).sum()
    loss.backward()
    return z.detach(), {n: t.grad for n, t in q.items()}


def test_gradients_of_a_model():
    """Each of a dozen operators is within 300 2^-24 of its terms' magnitudes; the layers' products and the norms' differences pass
    errors on up to ten times larger: 12 x 10 x 300 x 2^-24 = 2e-3 of a gradient's norm.  A wrong term would be of its own size."""
    import paper_2208_11580_amd as pkg

    ctx, ex = pkg.Context(), _example()
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    p, layers, weights, ids, teacher = _model(ctx, torch.float32, g)
    z, n1, n2 = ex.forward(ctx, p, layers, ids, 9.0)
    want_z, want = _autograd(p, weights, ids, 9.0, teacher)
    assert float((z - want_z).norm() / want_z.norm()) < 2e-3
    r = ctx.obc_distill(z, teacher["top_index"], teacher["top_logit"], want_grad=True)
    got = ex.backward(ctx, p, layers, ids, 9.0, n1, n2, r["dz"])
    for n in p:
        assert float((got[n] - want[n]).norm() / want[n].norm()) < 2e-3, n
    # a step from these gradients: at t = 1 every element moves by lr times its gradient's sign, but for eps
    before = {n: t.clone() for n, t in p.items()}
    names = list(p)
    ctx.obc_adamw(ctx.obc_adamw_plan([p[n] for n in names], [got[n] for n in names], [ctx.obc_adamw_state(p[n]) for n in names], decay=0.0), 1, 0.5)
    for n in names:
        want_step = 0.5 * got[n].double() / (got[n].double().abs() + 1e-8)
        assert float((before[n].double() - p[n].double() - want_step).abs().max()) < 0.5 * 32 * 2.0 ** -24 + 4 * 2.0 ** -24 * float(before[n].abs().max() + 1)
    ctx.obc_check()
    ctx.close()


@pytest.mark.parametrize("bits", [8, 32])
def test_a_training_step_in_a_graph(bits):
    """Forward, loss, backward and AdamW captured on a side stream, the step's number on the device: replays move the parameters as
    eager steps do, bit for bit, with other work between them."""
    import paper_2208_11580_amd as pkg

    ex = _example()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ctx = pkg.Context(side)
        g = torch.Generator(device="cuda")
        g.manual_seed(4)
        p0, layers, _, ids, teacher = _model(ctx, torch.bfloat16, g, T=700)
        runs = []
        for captured in (False, True):
            p = {n: t.clone() for n, t in p0.items()}
            small = ["gain1", "bias1", "gain2", "bias2"]
            grads = {n: torch.zeros_like(t) for n, t in p.items()}
            states = {n: ctx.obc_adamw_state(t, bits=bits, master=n == "table") for n, t in p.items()}
            plans = [ctx.obc_adamw_plan([p["table"]], [grads["table"]], [states["table"]]),
                     ctx.obc_adamw_plan([p[n] for n in small], [grads[n] for n in small], [states[n] for n in small], decay=[0.0, 0.1, 0.0, 0.1])]
            step = torch.ones(1, dtype=torch.int64, device="cuda")
            rate = torch.full((1,), 1e-3, device="cuda")
            seen = []

            def train():
                z, n1, n2 = ex.forward(ctx, p, layers, ids, 9.0)
                s = ctx.obc_score(z, ids, top=3)
                r = ctx.obc_distill(z, teacher["top_index"], teacher["top_logit"], want_grad=True)
                for n, t in ex.backward(ctx, p, layers, ids, 9.0, n1, n2, r["dz"]).items():
                    grads[n].copy_(t)
                for plan in plans:
                    ctx.obc_adamw(plan, step, rate, seed=5)
                step.add_(1)
                return [s["logp"], s["entropy"], s["top_index"], s["top_logit"], r["loss"]]

            if captured:
                state = [t.clone() for t in (*p.values(), step, *[t for st in states.values() for t in st if t is not None])]
                train()      # (workspaces)
                for t, old in zip((*p.values(), step, *[t for st in states.values() for t in st if t is not None]), state):
                    t.view(torch.uint8).copy_(old.view(torch.uint8))
                side.synchronize()
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=side):
                    out = train()
            for turn in range(5):
                if captured:
                    graph.replay()
                    seen.append([t.clone() for t in out])
                    torch.empty(1 << 20, device="cuda").fill_(float("nan"))
                    ctx.obc_embed_grad(ids[:50], torch.ones(50, 70, device="cuda"), 4000)
                    side.synchronize()
                else:
                    seen.append([t.clone() for t in train()])
                rate.mul_(0.9)
            runs.append((seen, p, states, int(step)))
        (seen_a, pa, sa, ta), (seen_b, pb, sb, tb) = runs
        assert ta == tb == 6
        for a, b in zip(seen_a, seen_b):
            assert all(torch.equal(x, y) for x, y in zip(a, b))
        for n in pa:
            assert torch.equal(pa[n], pb[n]), n
            assert all(x is None or torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(sa[n], sb[n]))
            assert not torch.equal(pa[n], p0[n])
        ctx.obc_check()
        del graph
        ctx.close()


def test_two_graphs_of_one_context():
    """Their workspaces are their own: replayed one after the other, and beside larger eager calls, both give what they gave."""
    import paper_2208_11580_amd as pkg

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ctx = pkg.Context(side)
        g = torch.Generator(device="cuda")
        g.manual_seed(6)
        z = torch.randn(3, 70000, generator=g, device="cuda")
        ids = torch.randint(-1, 900, (400,), generator=g, device="cuda", dtype=torch.int32)
        dy = torch.randn(400, 130, generator=g, device="cuda")
        h, gain = torch.randn(60, 300, generator=g, device="cuda"), torch.ones(300, device="cuda")
        stats = ctx.obc_layernorm(h, gain, want_stats=True)

        def work(k):
            s = ctx.obc_score(z, top=k)
            r = ctx.obc_layernorm_grad(h, gain, stats["mean"], stats["rstd"], h)
            return [s["lse"], s["top_index"], s["top_logit"], ctx.obc_embed_grad(ids, dy, 900), r["dx"], r["dgain"], r["dbias"]]

        want = [[t.clone() for t in work(k)] for k in (5, 40)]
        side.synchronize()
        graphs = []
        for k in (5, 40):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                graphs.append((graph, work(k)))
        for turn in range(4):
            for (graph, got), w in zip(graphs, want):
                for t in got:
                    t.zero_()
                graph.replay()
                side.synchronize()
                assert all(torch.equal(a, b) for a, b in zip(got, w)), turn
            ctx.obc_embed_grad(ids, torch.randn(400, 3000, generator=g, device="cuda"), 5000)
            if turn == 2:
                ctx.release_workspace()
                torch.empty(1 << 22, device="cuda").fill_(float("nan"))
        ctx.obc_check()
        del graphs, graph
        ctx.close()


def test_another_stream_than_the_current_one():
    """Calls queue on the context's stream: results are there once that has passed, and memory that the current stream still uses is
    not taken for outputs or workspaces."""
    import paper_2208_11580_amd as pkg

    side = torch.cuda.Stream()
    ctx = pkg.Context(side)
    g = torch.Generator(device="cuda")
    g.manual_seed(7)
    table = torch.randn(500, 64, generator=g, device="cuda")
    ids = torch.randint(-1, 500, (900,), generator=g, device="cuda", dtype=torch.int32)
    z = torch.randn(40, 9000, generator=g, device="cuda")
    p = torch.randn(3000, generator=g, device="cuda")
    torch.cuda.synchronize()
    main = pkg.Context()
    n = main.obc_layernorm(table, torch.ones(64, device="cuda"), want_stats=True)
    want = [main.obc_embed(table, ids), main.obc_embed_grad(ids, main.obc_embed(table, ids), 500), main.obc_score(z, top=7)["top_logit"], n["y"]]
    q = p.clone()
    main.obc_adamw(main.obc_adamw_plan([q], [p], [main.obc_adamw_state(q, bits=8)]), 1, 0.1)
    torch.cuda.synchronize()
    for _ in range(3):
        busy = torch.randn(4000, 4000, device="cuda")
        busy = busy @ busy
        del busy
        y = ctx.obc_embed(table, ids)
        r = p.clone()
        torch.cuda.synchronize()
        got = [y, ctx.obc_embed_grad(ids, y, 500), ctx.obc_score(z, top=7)["top_logit"], ctx.obc_layernorm(table, torch.ones(64, device="cuda"))["y"]]
        ctx.obc_adamw(ctx.obc_adamw_plan([r], [p], [ctx.obc_adamw_state(r, bits=8)]), 1, 0.1)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(q, r)
    ctx.obc_check()
    ctx.close()
    main.close()
