"""Scores, layer norm and AdamW at the ends of what their arguments may be, against plain implementations in 64 bits."""
import pytest
import torch

from .test_gpu_lm_tuning import B1, B2, INF, LR, NAN, ROUND, TINY, TYPES, U32, _blocks, _check_score, _gen, _norm_reference, _values, _within, ctx  # noqa: F401

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ scores
@pytest.mark.parametrize("V", [300, 9000, 40000, 70000])
@pytest.mark.parametrize("kind,top,tau", [
    ("f32", 22.499048, 1e-8), ("f32", 14.95, 1e-8), ("f32", 15.4825, 1e-8), ("f32", 15.5675, 1e-8), ("f32", 4757779968.0, 1.0),
    ("f16", 14.9921875, 1e-8), ("f16", 17.234375, 4.196192726624304e-09), ("bf16", 20.125, 1.2176419872389488e-08)])
def test_score_of_one_logit_at_a_small_temperature(ctx, kind, top, tau, V):
    """The largest logit over the temperature is about 2^31, so that its product with the reciprocal is rounded by 2^7: by more than
    the exponents of fp32 hold."""
    g = _gen(V)
    tau = float(torch.tensor(tau))
    z = (torch.randn(3, V, generator=g, device="cuda") + 0.3 * top).clamp_max(0.9 * top).to(TYPES[kind])
    for row, at in enumerate((0, V // 2, V - 1)):
        z[row, at] = top
    target = torch.tensor([0, 1, -1], dtype=torch.int32, device="cuda")
    for k in (0, 3):
        _check_score(ctx.obc_score(z, target, top=k, temperature=tau), z, target, k, tau)
    ctx.obc_check()


@pytest.mark.parametrize("T,V", [(700, 300), (60, 40000)])
@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("power", range(18, 46, 3))
def test_score_at_small_temperatures(ctx, power, kind, T, V):
    """Largest logits of about 2^power temperatures."""
    g = _gen(power)
    z = (10.0 + 10.0 * torch.rand(T, V, generator=g, device="cuda")).to(TYPES[kind])
    target = torch.randint(-1, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    tau = float(torch.tensor(15.0 * 2.0 ** -power))
    _check_score(ctx.obc_score(z, target, top=2, temperature=tau), z, target, 2, tau)
    ctx.obc_check()


@pytest.mark.parametrize("low", [-1e37, -2e37, -1e38, -3e38])
@pytest.mark.parametrize("T,V,k", [(3, 700, 7), (2, 9000, 20), (600, 40000, 64), (3, 40000, 0)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_score_of_masks_far_below(ctx, kind, T, V, k, low):
    """Every other logit masked with a large negative number, at random places."""
    g = _gen(V)
    z = 3.0 * torch.randn(T, V, generator=g, device="cuda")
    z = torch.where(torch.rand(T, V, generator=g, device="cuda") < 0.5, low, z).to(TYPES[kind])
    target = torch.randint(-1, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    _check_score(ctx.obc_score(z, target, top=k), z, target, k, 1.0)
    ctx.obc_check()


@pytest.mark.parametrize("V", [8, 700, 40000])
@pytest.mark.parametrize("k", [0, 4])
@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
def test_score_of_rows_of_low_numbers_alone(ctx, kind, k, V):
    """Rows of large negative numbers, which are no rows of -inf: all equal, one of them above the others, and one alone in each of a
    piece's places."""
    for low in (torch.finfo(TYPES[kind]).min, -INF if kind == "f16" else -1e37, -1.0):
        z = torch.full((10, V), low, device="cuda").to(TYPES[kind])
        z[1, 1] = low / 2
        z[2:] = -INF
        for place in range(8):
            z[2 + place, place] = low
        target = torch.tensor([V - 1, 1, 0, 1, 2, 3, 4, 5, -1, 0], dtype=torch.int32, device="cuda")
        _check_score(ctx.obc_score(z, target, top=k), z, target, k, 1.0)
    ctx.obc_check()


# ------------------------------------------------------------------------------------------------ layer norm
@pytest.mark.parametrize("mean", [3000.0, -30000.0])
@pytest.mark.parametrize("kind", ["f32", "f16"])
@pytest.mark.parametrize("T,d", [(4, 1000), (3, 4099), (520, 8192), (2, 16384), (2, 40001)])
def test_layernorm_of_a_large_mean(ctx, T, d, kind, mean):
    """Values a few units about a mean of thousands of them.  With n = 90 roundings in a sum the first mean is off by
    D = n 2^-24 |mean| at most, and its correction by n roundings of the deviations' size; nothing else depends on the mean."""
    g = _gen(d)
    x = (mean + 30.0 * torch.randn(T, d, generator=g, device="cuda")).to(TYPES[kind])
    gain, bias = 1.0 + 0.3 * torch.randn(d, generator=g, device="cuda"), 0.5 * torch.randn(d, generator=g, device="cuda")
    got = ctx.obc_layernorm(x, gain, bias, want_stats=True)
    _, m, rstd, y, dm, _, _ = _norm_reference(x, None, gain, bias, 1e-5)
    n, c = 90, (x.double() - m[:, None]).abs()
    D = dm[:, None]
    size = c.mean(1, keepdim=True) + D                                          # of c as the kernel has it
    e = (n + 3) * U32 * size                                                    # the correction: n roundings, each term's, the quotient's
    _within(got["mean"], m, U32 * m.abs() + e[:, 0])
    # c - e: a rounding of c, one of the difference, and e's; the variance's relative error, half of it rstd's: n roundings of its terms, 4 of the
    # terms' factors and the quotient, over a sum that is larger by D^2
    r = 0.5 * (n + 6) * U32 * (1 + (D * rstd[:, None]) ** 2) + 3 * U32
    _within(got["rstd"], rstd, (r[:, 0] + U32) * rstd)
    bound = gain.double().abs() * rstd[:, None] * (2 * U32 * (c + D) + e + c * (r + 2 * U32)) + U32 * (y.abs() + bias.double().abs())
    _within(got["y"], y, bound + ROUND[kind] * 1.01 * y.abs() + TINY[kind])
    ctx.obc_check()


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
def test_layernorm_of_constant_rows(ctx, kind):
    """The variance is zero, not a little less: y is the bias, and no number is lost at an eps of nearly nothing either."""
    g = _gen(5)
    for d in (3, 1000, 4097, 20000):
        x = (torch.rand(50, 1, generator=g, device="cuda") * 1000).to(TYPES[kind]).expand(50, d).contiguous()
        gain, bias = torch.rand(d, generator=g, device="cuda"), torch.rand(d, generator=g, device="cuda")
        got = ctx.obc_layernorm(x, gain, bias, eps=1e-30, want_stats=True)
        assert torch.isfinite(got["rstd"]).all() and torch.isfinite(got["y"]).all()
        got = ctx.obc_layernorm(x, gain, bias, eps=1e-5, want_stats=True)
        # c is one number for all, within 90 roundings of x; its mean is off by as many of it
        rest = (90 * U32) ** 2 * 1.1 * x.double().abs() * 1e5 ** 0.5
        _within(got["y"], bias.double().expand(50, d), gain.double() * rest + 2 * U32 + ROUND[kind] * 1.01 * (bias.double() + rest) + TINY[kind])
        _within(got["mean"], x[:, 0].double(), (U32 + 1.1 * (90 * U32) ** 2) * x[:, 0].double())
    ctx.obc_check()


# ------------------------------------------------------------------------------------------------ AdamW
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("master", [True, False])
def test_adamw_outputs_in_the_place_of_inputs(ctx, bits, master):
    """Results in the place of the tensor's gradient or of another of its inputs, a gradient that two tensors share: as apart.  What
    another tensor's step reads is refused."""
    import paper_2208_11580_amd as pkg

    g = _gen(bits)
    n = 5000

    def copied(st):
        return pkg.AdamState(*[None if t is None else t.clone() for t in st])

    p = torch.randn(n, generator=g, device="cuda")
    grad = torch.randn(n, generator=g, device="cuda")
    st = ctx.obc_adamw_state(p, bits=bits, master=master)
    for step in (1, 2):
        ctx.obc_adamw(ctx.obc_adamw_plan([p], [grad], [st]), step, 1e-2, seed=3)
    if master:
        st.master.add_(1e-3)      # (not the parameters' own values)
    for scale in (0.5, INF):      # (inf: all stays as it was)
        gs = torch.full((1,), scale, device="cuda")
        want_p, want = ctx.obc_adamw(ctx.obc_adamw_plan([p], [grad], [st], out=([torch.zeros_like(p)], [pkg.AdamState(
            *[None if t is None else torch.zeros_like(t) for t in st])])), 3, 1e-2, grad_scale=gs, seed=3)
        q, gr, su = p.clone(), grad.clone(), copied(st)
        ctx.obc_adamw(ctx.obc_adamw_plan([q], [gr], [su], out=([gr], [su])), 3, 1e-2, grad_scale=gs, seed=3)
        assert torch.equal(gr, want_p[0]) and torch.equal(q, p)
        assert all(a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(su, want[0]))
        if master:      # copies and parameters change places
            q, su = p.clone(), copied(st)
            new = su._replace(master=q)
            ctx.obc_adamw(ctx.obc_adamw_plan([q], [grad], [su], out=([su.master], [new])), 3, 1e-2, grad_scale=gs, seed=3)
            assert torch.equal(su.master, want_p[0]) and torch.equal(q, want[0].master)
    q, su = p.clone(), copied(st)
    with pytest.raises(pkg.ObcError):
        ctx.obc_adamw_plan([p, q], [grad, grad], [st, su], out=([q, p], [st, su]))
    with pytest.raises(pkg.ObcError):
        ctx.obc_adamw_plan([p, q], [q, grad], [st, su])
    with pytest.raises(pkg.ObcError):
        ctx.obc_adamw_plan([p[:n - 1]], [p[1:]], [ctx.obc_adamw_state(p[1:], bits=bits)])
    ctx.obc_check()


@pytest.mark.parametrize("n", [300, 5000])
def test_adamw_of_small_gradients(ctx, n):
    """Moments in 32 bits whose v is below fp32's smallest normal number, and an eps below their roots."""
    g, eps = _gen(n), 2.0 ** -110
    grad = 10.0 ** (-21.0 + 4.0 * torch.rand(n, generator=g, device="cuda"))
    grad = torch.where(torch.rand(n, generator=g, device="cuda") < 0.5, grad, -grad)
    grad[::9] = 0.0
    p = torch.zeros(n, device="cuda")
    st = ctx.obc_adamw_state(p)
    m, v = (torch.zeros(n, dtype=torch.float64, device="cuda") for _ in range(2))
    for step in (1, 2, 3):
        p.zero_()
        old_m, old_v = st.m.double(), st.v.double()
        ctx.obc_adamw(ctx.obc_adamw_plan([p], [grad], [st], decay=0.0), step, LR, B1, B2, eps)
        m, v = B1 * old_m + (1 - B1) * grad.double(), B2 * old_v + (1 - B2) * grad.double() ** 2
        _within(st.m, m, 6 * U32 * m.abs())
        # v: its terms' roundings, and those of the square and of the sum among numbers that lie 2^-149 apart
        dv = 8 * U32 * v + 2.0 ** -149
        _within(st.v, v, dv)
        c1, c2 = 1 / (1 - B1 ** step), (1 - B2 ** step) ** -0.5
        most, least = (LR * c1 * m.abs() / ((w.clamp_min(0.0)).sqrt() * c2 + eps) for w in (v - dv, v + dv))
        assert (p.double().abs() <= most * (1 + 24 * U32)).all() and (p.double().abs() >= least * (1 - 24 * U32)).all()
        assert (torch.sign(p) == -torch.sign(grad)).all()
    ctx.obc_check()


@pytest.mark.parametrize("size", [1e-17, 1e-19, 1e-20, 1e-22, 1e-25, 1e-28])
@pytest.mark.parametrize("n", [300, 5000])
def test_adamw_of_8_bit_moments_of_small_gradients(ctx, n, size):
    """Roots of v down to the smallest that a block may have, and an eps below them, among blocks of ordinary ones: m over the root is what
    a step moves by, and a root that is not zero does not become zero."""
    g, eps = _gen(n), 2.0 ** -115
    grad = size * torch.randn(n, generator=g, device="cuda") * torch.randn(n, generator=g, device="cuda").exp()
    grad[100:200] = 0.0
    grad[256:290] = torch.randn(34, generator=g, device="cuda")
    p = torch.zeros(n, device="cuda")
    st = ctx.obc_adamw_state(p, bits=8)
    for step in (1, 2, 3):
        p.zero_()
        m, v = _values(st.m, st.m_scale), _values(st.v, st.v_scale) ** 2
        ctx.obc_adamw(ctx.obc_adamw_plan([p], [grad], [st], decay=0.0), step, LR, B1, B2, eps, seed=2)
        em = 6 * U32 * (B1 * m.abs() + (1 - B1) * grad.double().abs())
        m, v = B1 * m + (1 - B1) * grad.double(), B2 * v + (1 - B2) * grad.double() ** 2
        c1, c2 = 1 / (1 - B1 ** step), (1 - B2 ** step) ** -0.5
        want = LR * c1 * m / (v.sqrt() * c2 + eps)
        _within(p, -want, 32 * U32 * want.abs() + LR * c1 * em / (v.sqrt() * c2 + eps))
        for got, scale, x, e in ((st.m, st.m_scale, m, em), (st.v, st.v_scale, v.sqrt(), 8 * U32 * v.sqrt())):
            top = _blocks(x.abs()).amax(1)
            _within(scale, top / 448, _blocks(e).amax(1) / 448 + 2 * U32 * top / 448)
            s = scale.double().repeat_interleave(256)[:n]
            # up or down: less than a step, an eighth or 2^-9 of the scale
            assert ((_values(got, scale) - x).abs() <= torch.maximum(x.abs() / 8, 2.0 ** -9 * s) * (1 + 1e-5) + e).all()
        assert ((st.v.float() > 0) == (v > 0)).all()
    ctx.obc_check()


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_with_other_gradients(ctx, bits):
    """Steps of one plan with gradients that change place from step to step, more tensors than one launch lays out: as plans of their
    own."""
    g = _gen(bits)
    sizes = [700, 1, 2048, 5000, 33] * 7
    params = [torch.randn(n, generator=g, device="cuda") for n in sizes]
    grads = [[torch.randn(n, generator=g, device="cuda") for n in sizes] for _ in range(3)]
    both = []
    for kept in (True, False):
        ps = [p.clone() for p in params]
        states = [ctx.obc_adamw_state(p, bits=bits) for p in ps]
        plan = ctx.obc_adamw_plan(ps, grads[0], states)
        for step in (1, 2, 3):
            if kept and step > 1:
                plan.use(grads[step - 1])
            if not kept:
                plan = ctx.obc_adamw_plan(ps, grads[step - 1], states)
            ctx.obc_adamw(plan, step, LR, seed=4)
        both.append((ps, states))
    for p, q, st, su in zip(both[0][0], both[1][0], both[0][1], both[1][1]):
        assert torch.equal(p, q)
        assert all(a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(st, su))
    ctx.obc_check()


def test_tensors_that_go_while_a_step_is_queued():
    """A plan's gradients are replaced, and then the plan goes, while its steps wait on the context's stream: their memory is not handed out
    on the stream that they were allocated on before that."""
    import paper_2208_11580_amd as pkg

    side = torch.cuda.Stream()
    ctx = pkg.Context(side)
    g = _gen(3)
    n = 3000000
    p = torch.randn(n, generator=g, device="cuda")
    start = [torch.randn(n, generator=g, device="cuda") for _ in range(2)]
    busy = torch.randn(6000, 6000, device="cuda")
    main = pkg.Context()
    want, state = p.clone(), main.obc_adamw_state(p)
    for step in (1, 2):
        main.obc_adamw(main.obc_adamw_plan([want], [start[step - 1]], [state]), step, LR)
    for _ in range(3):
        q = p.clone()
        grads = [t.clone() for t in start]
        st = pkg.AdamState(torch.zeros_like(p), torch.zeros_like(p))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(10):
                busy @ busy
        plan = ctx.obc_adamw_plan([q], [grads.pop(0)], [st])
        ctx.obc_adamw(plan, 1, LR)
        plan.use([grads.pop(0)])
        late = [torch.full((n,), NAN, device="cuda") for _ in range(3)]
        ctx.obc_adamw(plan, 2, LR)
        del plan, st
        late += [torch.full((n,), NAN, device="cuda") for _ in range(5)]
        torch.cuda.synchronize()
        assert torch.equal(q, want)
        del late
    ctx.obc_check()
    ctx.close()
    main.close()
