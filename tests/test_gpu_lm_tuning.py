"""What compressed models are judged by and tuned with (scores of logits, layer norm, embeddings, AdamW) against plain
implementations in 64 bits.  Bounds are worst-case ones of the arithmetic that the header states: a sum of n fp32 terms
is off by at most n 2^-24 of the sum of their magnitudes, a result is rounded once to its type."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ROUND = {k: torch.finfo(t).eps / 2 for k, t in TYPES.items()}      # half a unit in the last place, relative
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}      # the smallest numbers
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def ctx():
    import paper_2208_11580_amd as pkg

    c = pkg.Context()
    yield c
    c.close()


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _within(got, want, bound):
    err = (got.double() - want).abs()
    bad = ~(err <= bound)
    assert not bad.any(), "%d of %d outside, worst %.3g of its bound" % (
        int(bad.sum()), bad.numel(), float((err / bound.clamp_min(1e-300)).nan_to_num(INF).max()))


def _unaligned(t):
    """The same values at an address that is a multiple of nothing but an element."""
    flat = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)
    flat[1:] = t.reshape(-1)
    return flat[1:].view(t.shape)


# ------------------------------------------------------------------------------------------------ scores
def _check_score(r, z, target, k, tau):
    z64 = z.double()
    T, V = z.shape
    best, order = torch.sort(z64 + 0.0, dim=1, descending=True, stable=True)
    if k:
        n = min(k, V)
        index = torch.full((T, k), -1, dtype=torch.int32, device="cuda")
        logit = torch.full((T, k), -INF, dtype=torch.float32, device="cuda")
        real = best[:, :n] > -INF
        index[:, :n] = torch.where(real, order[:, :n], -1).to(torch.int32)
        logit[:, :n] = best[:, :n].float()
        assert torch.equal(r["top_logit"], logit)
        assert torch.equal(r["top_index"], index)
    else:
        assert r["top_index"] is None and r["top_logit"] is None
    top = best[:, :1]
    live = top[:, 0] > -INF
    d = torch.where(top > -INF, (z64 - top) / tau, -INF)
    e = torch.exp(d)
    S = e.sum(1)
    dd = d.clamp_min(-1e30)
    D, Q = -(e * dd).sum(1), (e * dd * dd).sum(1)
    lnS = S.clamp_min(1.0).log()
    D, Q = D / S.clamp_min(1.0), Q / S.clamp_min(1.0)
    # per thread at most 17 pieces of 8, then waves, workgroups and parts: 200 roundings; (z - top) c, with c's two
    # roundings, is off by 4 of them, and so are e's relative errors
    n = 200 + V // 8192
    dS = (n + 4 * D) * U32
    lse = top[:, 0] / tau + lnS
    _within(torch.where(live, r["lse"].double(), 0.0), torch.where(live, lse, 0.0),
            (dS + 3 * U32 * (lnS + (top[:, 0] / tau).abs() + lse.abs())).nan_to_num(0.0, 0.0))
    assert (r["lse"][~live] == -INF).all() and (r["entropy"][~live] == 0).all()
    _within(torch.where(live, r["entropy"].double(), 0.0), torch.where(live, lnS + D, 0.0), 2 * dS + ((n + 8) * D + 4 * Q + 4 * lnS) * U32)
    if target is None:
        assert r["logp"] is None
        return
    t = target.long()
    dt = torch.gather(d, 1, t.clamp_min(0)[:, None])[:, 0]
    want = torch.where(t >= 0, dt - lnS, 0.0)
    finite = want > -INF
    assert torch.equal(r["logp"] == -INF, ~finite)
    _within(torch.where(finite, r["logp"].double(), 0.0), torch.where(finite, want, 0.0),
            torch.where(finite & (t >= 0), dS + U32 * (4 * dt.abs() + 3 * lnS + want.abs()), 0.0))


SCORES = [  # T, V, k
    (1, 1, 0), (1, 1, 1), (2, 2, 4), (3, 7, 10), (2, 255, 3), (5, 1000, 183), (1, 1024, 1024), (1, 32000, 20), (4, 8192, 64), (3, 8193, 65),
    (2, 16384, 129), (2, 32768, 256), (1, 32769, 1024), (700, 1000, 5), (520, 4097, 0), (600, 33000, 64), (1, 131072, 1000), (2, 300001, 40),
]


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,V,k", SCORES)
def test_score(ctx, T, V, k, kind):
    g = _gen(T + V + k)
    z = (3.0 * torch.randn(T, V, generator=g, device="cuda")).to(TYPES[kind])
    target = torch.randint(-1, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    for tau in (1.0, 0.37):
        r = ctx.obc_score(z, target, top=k, temperature=tau)
        ctx.obc_check()
        _check_score(r, z, target, k, tau)
    again = ctx.obc_score(z, target, top=k, temperature=tau)
    assert all(r[n] is None or torch.equal(r[n], again[n]) for n in r)


VALUES = ["equal", "two", "zeros", "ascending", "descending", "one_lane", "masked", "mostly_masked", "one_left", "negative", "lowest"]


@pytest.mark.parametrize("values", VALUES)
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V,k", [(2, 5000, 7), (2, 20000, 100), (1, 70000, 64), (520, 9000, 20), (1, 40000, 1024)])
def test_score_of_ties_and_masks(ctx, T, V, k, kind, values):
    """Rows whose largest logits are equal, in order, in one thread's hands, or few."""
    g = _gen(V + k)
    z = torch.randn(T, V, generator=g, device="cuda")
    at = torch.arange(V, device="cuda").float()
    if values == "equal":
        z = torch.full_like(z, -1.25)
    elif values == "two":
        z = (z > 0.5).float()
    elif values == "zeros":
        z = torch.where(z > 0, 0.0, -0.0)
    elif values == "ascending":
        z = (at / V * 20 - 10).expand(T, V).clone()
    elif values == "descending":
        z = (10 - at / V * 20).expand(T, V).clone()
    elif values == "one_lane":      # eight neighbours in every 2048 hold all the large ones
        z = z + 50.0 * ((at.long() % 2048) < 8)
    elif values == "masked":
        z[:, V // 3:] = -INF
    elif values == "mostly_masked":
        z[:, :] = torch.where(torch.rand(T, V, generator=g, device="cuda") < 20.0 / V, z, -INF)
    elif values == "one_left":
        z[:, 1:] = -INF
    elif values == "negative":
        z = -100.0 - z.abs()
    elif values == "lowest":
        z[:, ::3] = torch.finfo(TYPES[kind]).min
    z = z.to(TYPES[kind])
    target = torch.randint(-1, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    r = ctx.obc_score(z, target, top=k)
    _check_score(r, z, target, k, 1.0)
    ctx.obc_check()


@pytest.mark.parametrize("V", [3, 900, 40000])
def test_score_of_lost_rows(ctx, V):
    """Rows of -inf alone; rows with a NaN or +inf somewhere, beside whole ones."""
    g = _gen(V)
    for kind in TYPES.values():
        z = torch.randn(7, V, generator=g, device="cuda").to(kind)
        z[1] = -INF
        z[2, V // 2] = NAN
        z[3, V - 1] = INF
        z[4, 0] = -NAN
        z[5] = NAN
        target = torch.tensor([V - 1, 0, 0, V - 1, -1, 1, 0], dtype=torch.int32, device="cuda")
        r = ctx.obc_score(z, target, top=5)
        whole = [0, 1, 6]
        _check_score({n: t[whole] for n, t in r.items()}, z[whole], target[whole], 5, 1.0)
        assert r["logp"][1] == -INF and (r["top_index"][1] == -1).all()
        for i in (2, 3, 4, 5):
            assert r["lse"][i].isnan() and r["entropy"][i].isnan() and (r["top_index"][i] == -1).all() and r["top_logit"][i].isnan().all()
            assert r["logp"][i].isnan() or i == 4
        assert r["logp"][4] == 0
    ctx.obc_check()


def test_score_layouts_and_outputs(ctx):
    g = _gen(3)
    for kind in TYPES.values():
        big = torch.randn(9, 3001, generator=g, device="cuda").to(kind)
        z = big[1:8, 3:2500]
        target = torch.randint(0, 2497, (7,), generator=g, device="cuda", dtype=torch.int32)
        want = ctx.obc_score(z.contiguous(), target, top=9)
        out = {n: torch.full_like(t, 3) for n, t in want.items()}
        r = ctx.obc_score(z, target, top=9, out=out)
        assert all(r[n] is out[n] and torch.equal(r[n], want[n]) for n in want)
        none = ctx.obc_score(z)
        assert none["logp"] is None and none["top_index"] is None and torch.equal(none["lse"], want["lse"])
    assert ctx.obc_score(z[:0], target[:0], top=3)["top_index"].shape == (0, 3)
    with pytest.raises(Exception):
        target[2] = 2497
        ctx.obc_score(z, target)
        ctx.obc_check()
    target[2] = -1
    r = ctx.obc_score(z, target)
    assert r["logp"][2] == 0
    ctx.obc_check()


# ------------------------------------------------------------------------------------------------ layer norm
NORMS = [(1, 1), (3, 2), (1, 768), (5, 7), (2, 2048), (7, 2049), (600, 500), (530, 4096), (3, 4099), (520, 8192), (2, 8191), (2, 16384), (513, 9000),
         (2, 16385), (1, 65536), (2, 40001)]


def _norm_inputs(T, d, kind, g, residual=True):
    x = (torch.randn(T, d, generator=g, device="cuda") + 3.0).to(TYPES[kind])
    r = (2.0 * torch.randn(T, d, generator=g, device="cuda")).to(TYPES[kind]) if residual else None
    gain = 1.0 + 0.3 * torch.randn(d, generator=g, device="cuda")
    bias = 0.5 * torch.randn(d, generator=g, device="cuda")
    return x, r, gain, bias


def _norm_reference(x, r, gain, bias, eps):
    h = x.double() + (0 if r is None else r.double())
    d = h.shape[1]
    mean = h.mean(1, keepdim=True)
    c = h - mean
    rstd = (c.square().mean(1, keepdim=True) + eps).rsqrt()
    y = c * rstd * gain.double() + (0 if bias is None else bias.double())
    # sums of 64 terms in a thread, 6 steps in a wave, 16 waves; the sum h itself is rounded once
    n = 90
    dm = n * U32 * h.abs().mean(1, keepdim=True) + U32 * mean.abs()
    # the squares: a sum, each off by twice c's error
    dr = (n + 6) * U32 + 2 * (dm * c.abs().mean(1, keepdim=True) + U32 * (c * h).abs().mean(1, keepdim=True)) * rstd.square()
    dy = gain.double().abs() * rstd * (dm + 2 * U32 * (c.abs() + h.abs()) + c.abs() * (dr + 4 * U32)) + 2 * U32 * y.abs()
    if bias is not None:
        dy = dy + U32 * bias.double().abs()
    return h, mean[:, 0], rstd[:, 0], y, dm[:, 0], dr[:, 0] * rstd[:, 0], dy


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,d", NORMS)
def test_layernorm(ctx, T, d, kind):
    g = _gen(T * 3 + d)
    x, r, gain, bias = _norm_inputs(T, d, kind, g)
    for res, b in ((r, bias), (None, None)):
        got = ctx.obc_layernorm(x, gain, b, eps=1e-5, residual=res, want_stats=True)
        h, mean, rstd, y, dm, dr, dy = _norm_reference(x, res, gain, b, 1e-5)
        if res is not None:
            _within(got["h"], h, (ROUND[kind] + U32) * h.abs())
        else:
            assert got["h"] is x
        _within(got["mean"], mean, dm)
        _within(got["rstd"], rstd, dr + 2 * U32 * rstd)
        _within(got["y"], y, dy + ROUND[kind] * 1.01 * y.abs() + TINY[kind])
        assert torch.equal(got["y"], ctx.obc_layernorm(x, gain, b, eps=1e-5, residual=res)["y"])
        q = ctx.obc_layernorm(x, gain, b, eps=1e-5, residual=res, quant8=True)
        top, dtop = y.abs().amax(1), dy.amax(1)
        live = top > 4 * dtop
        _within(q["scale"][live], top[live] / 127, dtop[live] / 127 + 2 * U32 * top[live])
        # half a step of rounding, and where y's error takes it over the edge
        v = q["y"].double() * q["scale"].double()[:, None]
        _within(v[live], y[live], (0.5 * q["scale"].double()[:, None] * (1 + 1e-5) + dy + 127 * (dtop / 127)[:, None])[live])
        assert (q["y"].abs().amax(1)[live] == 127).all()
    ctx.obc_check()


def test_layernorm_in_place_and_unaligned(ctx):
    g = _gen(8)
    for kind in TYPES:
        for d in (31, 1283):
            x, r, gain, bias = _norm_inputs(6, d, kind, g)
            want = ctx.obc_layernorm(x, gain, bias, residual=r, want_stats=True)
            xu, ru, yu = _unaligned(x), _unaligned(r), _unaligned(torch.zeros_like(x))
            got = ctx.obc_layernorm(xu, _unaligned(gain), _unaligned(bias), residual=ru, want_stats=True, out={"h": ru, "y": yu})
            assert got["h"] is ru and all(torch.equal(want[n], got[n]) for n in ("h", "y", "mean", "rstd"))
            want8 = ctx.obc_layernorm(x, gain, bias, residual=r, quant8=True)
            got8 = ctx.obc_layernorm(xu, gain, bias, residual=r, quant8=True, out={"h": xu, "y": _unaligned(torch.zeros(6, d, dtype=torch.int8, device="cuda"))})
            assert all(torch.equal(want8[n], got8[n]) for n in ("h", "y", "scale"))
    ctx.obc_check()


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
def test_layernorm_of_lost_rows(ctx, kind):
    """Constant rows, a NaN, an infinity, a gain that is not finite: the others stay as they are."""
    g = _gen(4)
    x, _, gain, bias = _norm_inputs(6, 300, kind, g)
    x[1] = 5.0
    x[2, 7] = NAN
    x[3, 299] = INF
    got = ctx.obc_layernorm(x, gain, bias)["y"]
    q = ctx.obc_layernorm(x, gain, bias, quant8=True)
    clean = x.clone()
    clean[2:4] = 0.0
    want, want8 = ctx.obc_layernorm(clean, gain, bias)["y"], ctx.obc_layernorm(clean, gain, bias, quant8=True)
    for i in (0, 1, 4, 5):
        assert torch.equal(got[i], want[i]) and torch.equal(q["y"][i], want8["y"][i]) and q["scale"][i] == want8["scale"][i]
    _within(got[1], bias.double(), ROUND[kind] * bias.double().abs() + TINY[kind])
    for i in (2, 3):
        assert got[i].isnan().all() and q["scale"][i].isnan() and (q["y"][i] == 0).all()
    zero = ctx.obc_layernorm(x[1:2], gain, quant8=True)
    assert zero["scale"][0] == 1 and (zero["y"] == 0).all()
    gain[5] = NAN
    q = ctx.obc_layernorm(x, gain, bias, quant8=True)
    assert q["scale"].isnan().all() and (q["y"] == 0).all()
    ctx.obc_check()


def test_layernorm_keeps_the_variance_of_a_large_mean(ctx):
    x = 3000.0 + torch.randn(4, 1000, generator=_gen(1), device="cuda")
    y = ctx.obc_layernorm(x, torch.ones(1000, device="cuda"))["y"].double()
    want = _norm_reference(x, None, torch.ones(1000, device="cuda"), None, 1e-5)[3]
    # the mean's rounding moves all values alike, by 3000 x 90 x 2^-24 at most; it takes none of the variance's digits
    assert float((y - want).abs().max()) < 3000 * 92 * U32


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,d", NORMS + [(1500, 300), (1025, 2048)])
def test_layernorm_grad(ctx, T, d, kind):
    g = _gen(T * 5 + d)
    h = (torch.randn(T, d, generator=g, device="cuda") + 1.0).to(TYPES[kind])
    dy, dh = (torch.randn(T, d, generator=g, device="cuda").to(TYPES[kind]) for _ in range(2))
    gain = 1.0 + 0.3 * torch.randn(d, generator=g, device="cuda")
    h64 = h.double()
    mean = h64.mean(1).float()
    rstd = (h64.var(1, correction=0) + 1e-5).rsqrt().float()
    r64 = rstd.double()[:, None]
    xhat = (h64 - mean.double()[:, None]) * r64
    w = gain.double() * dy.double()
    aw, ax = w.abs(), xhat.abs()
    n = 64 + 6 + 16 + 4
    for extra in (dh, None):
        got = ctx.obc_layernorm_grad(h, gain, mean, rstd, dy, dh=extra)
        m0, m1 = w.mean(1, keepdim=True), (w * xhat).mean(1, keepdim=True)
        inner = w - m0 - xhat * m1
        want = r64 * inner + (0 if extra is None else extra.double())
        e = r64 * U32 * (4 * (aw + m0.abs()) + n * aw.mean(1, keepdim=True) + ax * (n + 8) * (aw * ax).mean(1, keepdim=True)) + 2 * U32 * want.abs()
        if extra is not None:
            e = e + U32 * extra.double().abs()
        _within(got["dx"], want, e + ROUND[kind] * 1.01 * want.abs() + TINY[kind])
        rows = -(-T // 512) + 64
        _within(got["dgain"], (dy.double() * xhat).sum(0), (rows + 4) * U32 * (dy.double() * xhat).abs().sum(0))
        _within(got["dbias"], dy.double().sum(0), rows * U32 * dy.double().abs().sum(0))
    again = ctx.obc_layernorm_grad(h, gain, mean, rstd, dy, out={"dx": dy})
    assert again["dx"] is dy and all(torch.equal(got[n], again[n]) for n in got)
    ctx.obc_check()


def test_layernorm_grad_against_differences(ctx):
    """The gradients of sum(y c) by central differences of the formula in 64 bits."""
    g = _gen(12)
    T, d = 3, 40
    h, gain, bias = torch.randn(T, d, generator=g, device="cuda"), torch.rand(d, generator=g, device="cuda") + 0.5, torch.zeros(d, device="cuda")
    c = torch.randn(T, d, generator=g, device="cuda")
    f = ctx.obc_layernorm(h, gain, bias, want_stats=True)
    got = ctx.obc_layernorm_grad(h, gain, f["mean"], f["rstd"], c)

    def value(h, gain, bias):
        return float((_norm_reference(h, None, gain, bias, 1e-5)[3] * c.double()).sum())

    step = 2.0 ** -17
    for name, x in (("dx", h), ("dgain", gain), ("dbias", bias)):
        for i in range(0, x.numel(), 7):
            up, down = x.double(), x.double()
            up.view(-1)[i] += step
            down.view(-1)[i] -= step
            args = {"dx": h, "dgain": gain, "dbias": bias}
            hi, lo = dict(args), dict(args)
            hi[name], lo[name] = up, down
            diff = (value(hi["dx"], hi["dgain"], hi["dbias"]) - value(lo["dx"], lo["dgain"], lo["dbias"])) / (2 * step)
            # third derivatives of about a hundred times step^2, sums of 1e2 to 52 bits over the step, and fp32's part
            assert abs(float(got[name].view(-1)[i]) - diff) < 1e-6 + 100 * 2.0 ** -34 + 1e2 * 2.0 ** -50 / step + 200 * U32 * (1 + abs(diff))


def test_layernorm_of_no_rows(ctx):
    e = torch.empty(0, 64, device="cuda")
    gain = torch.ones(64, device="cuda")
    assert ctx.obc_layernorm(e, gain)["y"].shape == (0, 64)
    r = ctx.obc_layernorm_grad(e, gain, torch.empty(0, device="cuda"), torch.empty(0, device="cuda"), e)
    assert (r["dgain"] == 0).all() and (r["dbias"] == 0).all()


# ------------------------------------------------------------------------------------------------ embeddings
@pytest.mark.parametrize("kind,out", [(a, b) for a in TYPES for b in TYPES])
@pytest.mark.parametrize("T,V,d", [(1, 1, 1), (3, 10, 7), (100, 50, 64), (33, 1000, 1283), (5, 300, 2048), (7, 100, 2049), (2, 9, 10000)])
def test_embed(ctx, T, V, d, kind, out):
    g = _gen(T + V + d)
    table = torch.randn(V, d, generator=g, device="cuda").to(TYPES[kind])
    ids = torch.randint(-2, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    y = ctx.obc_embed(table, ids, scale=1.7, out_dtype=TYPES[out])
    s = float(torch.tensor(1.7, dtype=torch.float32))
    want = torch.where(ids[:, None] >= 0, table.double()[ids.clamp_min(0).long()] * s, 0.0)
    _within(y, want, (ROUND[out] + U32) * 1.01 * want.abs() + TINY[out])
    assert (y[ids < 0] == 0).all()
    ctx.obc_check()


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
def test_embed_layouts(ctx, kind):
    """Rows with gaps, at odd addresses; what lies between them stays; what no id names may be NaN; ids out of range."""
    g = _gen(2)
    table = torch.randn(40, 105, generator=g, device="cuda").to(TYPES[kind])
    table[20:] = NAN
    part = table[:, 1:98]
    ids = torch.randint(-1, 20, (12,), generator=g, device="cuda", dtype=torch.int32)
    out = torch.full((12, 120), 9.0, device="cuda", dtype=TYPES[kind])
    ctx.obc_embed(part, ids, scale=0.5, out=out[:, 3:100])
    assert torch.equal(out[:, 3:100], ctx.obc_embed(part.contiguous(), ids, scale=0.5))
    assert (out[:, :3] == 9).all() and (out[:, 100:] == 9).all() and not out.isnan().any()
    ctx.obc_check()
    ids[3] = 40
    y = ctx.obc_embed(part, ids)
    assert (y[3] == 0).all()
    with pytest.raises(Exception):
        ctx.obc_check()
    assert ctx.obc_embed(part, ids[:0]).shape == (0, 97)


def _embed_grad_reference(ids, dy, V, scale):
    d = dy.shape[1]
    real = ids >= 0
    total, mag = (torch.zeros(V, d, dtype=torch.float64, device="cuda") for _ in range(2))
    at = ids[real].long()
    total.index_add_(0, at, dy[real].double())
    mag.index_add_(0, at, dy[real].double().abs())
    count = torch.bincount(at, minlength=V).double()[:, None]
    return total * scale, mag * abs(scale) * (count + 2) * U32


EMBED_GRADS = [  # T, V, d, ids
    (0, 5, 8, "even"), (1, 1, 1, "even"), (5, 3, 7, "even"), (64, 1000, 96, "even"), (100, 70, 300, "even"), (33, 4, 2049, "even"),
    (3000, 500, 64, "even"), (5000, 40000, 33, "zipf"), (2000, 131, 513, "zipf"), (1500, 7, 100, "one"), (4097, 3000, 64, "one"), (20000, 100, 40, "zipf"),
    (70000, 33, 16, "zipf"), (777, 20000, 65, "none"), (3100, 300000, 8, "zipf"), (2500, 65, 2600, "blocks"),
]


def _some_ids(T, V, how, g):
    if how == "zipf":
        u = torch.rand(T, generator=g, device="cuda", dtype=torch.float64)
        ids = (torch.exp(u * math.log(V + 1.0)).floor() - 1).clamp(0, V - 1).to(torch.int32)
        return torch.where(torch.rand(T, generator=g, device="cuda") < 0.1, -1, ids)
    if how == "one":
        return torch.full((T,), V - 1, dtype=torch.int32, device="cuda")
    if how == "none":
        return torch.full((T,), -3, dtype=torch.int32, device="cuda")
    if how == "blocks":      # ids' tokens next to one another: 32, 33, 64, ... of them, ends on stretches' ends and not
        lengths = [32, 33, 31, 64, 1, 96, 200, 32, 500]
        ids = torch.cat([torch.full((n,), 3 * i, dtype=torch.int32) for i, n in enumerate(lengths)])
        return torch.cat([ids, torch.full((T - ids.numel(),), 60, dtype=torch.int32)])[:T].to("cuda")
    return torch.randint(-1, V, (T,), generator=g, device="cuda", dtype=torch.int32)


@pytest.mark.parametrize("kind,out", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16")])
@pytest.mark.parametrize("T,V,d,how", EMBED_GRADS)
def test_embed_grad(ctx, T, V, d, how, kind, out):
    g = _gen(T + V + d)
    ids = _some_ids(T, V, how, g)
    dy = torch.randn(T, d, generator=g, device="cuda").to(TYPES[kind])
    got = ctx.obc_embed_grad(ids, dy, V, scale=3.0, out_dtype=TYPES[out])
    want, bound = _embed_grad_reference(ids, dy, V, 3.0)
    _within(got, want, bound + ROUND[out] * 1.01 * want.abs() + TINY[out])
    assert torch.equal(got, ctx.obc_embed_grad(ids, dy, V, scale=3.0, out=torch.full_like(got, NAN)))
    # added to what is there; rows without a token keep their bits
    old = torch.randn(V, d, generator=g, device="cuda").to(TYPES[out])
    total = ctx.obc_embed_grad(ids, dy, V, scale=3.0, out=old.clone(), accumulate=True)
    sum_ = want + old.double()
    _within(total, sum_, bound + (ROUND[out] + U32) * 1.01 * sum_.abs() + TINY[out])
    empty = torch.ones(V, dtype=torch.bool, device="cuda")
    empty[ids[ids >= 0].long()] = False
    assert torch.equal(total[empty], old[empty])
    ctx.obc_check()


def test_embed_grad_layouts(ctx):
    """Gradients with gaps and at odd addresses; NaN and scales that no row with tokens shares; ids out of range."""
    g = _gen(6)
    ids = _some_ids(500, 90, "zipf", g)
    ids[7] = -1
    big = torch.randn(500, 70, generator=g, device="cuda").bfloat16()
    big[7] = NAN
    out = torch.full((90, 80), 4.0, device="cuda")
    ctx.obc_embed_grad(ids, big[:, 1:62], 90, out=out[:, 5:66])
    assert torch.equal(out[:, 5:66], ctx.obc_embed_grad(ids, big[:, 1:62].contiguous(), 90, out_dtype=torch.float32))
    assert (out[:, :5] == 4).all() and (out[:, 66:] == 4).all() and not out.isnan().any()
    empty = torch.ones(90, dtype=torch.bool, device="cuda")
    empty[ids[ids >= 0].long()] = False
    assert (ctx.obc_embed_grad(ids, big, 90, scale=INF)[empty] == 0).all()
    ctx.obc_check()
    want = ctx.obc_embed_grad(torch.where(ids == 89, -1, ids), big, 90)
    bad = torch.where(ids == 89, 90, ids)
    assert torch.equal(ctx.obc_embed_grad(bad, big, 90), want) or not (ids == 89).any()
    bad[9] = 2 ** 31 - 1
    ctx.obc_embed_grad(bad, big, 90)
    with pytest.raises(Exception):
        ctx.obc_check()
    ctx.obc_check()


def test_embed_grad_against_the_lookup(ctx):
    """<embed(table + e), c> - <embed(table), c> = <e, gradient of c>: the lookup is linear."""
    g = _gen(9)
    V, d, T = 50, 33, 200
    ids = torch.randint(-1, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    c = torch.randn(T, d, generator=g, device="cuda")
    grad = ctx.obc_embed_grad(ids, c, V, scale=2.0).double()
    e = torch.randn(V, d, generator=g, device="cuda")
    lhs = float((ctx.obc_embed(e, ids, scale=2.0).double() * c.double()).sum())
    rhs = float((grad * e.double()).sum())
    mag = float((_embed_grad_reference(ids, c.abs(), V, 2.0)[0] * e.abs().double()).sum())
    assert abs(lhs - rhs) < (T + 4) * U32 * mag


# ------------------------------------------------------------------------------------------------ AdamW
B1, B2, EPS, LR, DECAY = 0.9, 0.99, 1e-8, 1e-2, 0.1
MIX = (0x9E3779B1, 0x6A09E667, 0xBB67AE85, 0x3C6EF373, 0x243F6A89)


def _dither(n, seed, step, ordinal):
    low = 0xffffffff
    h = torch.arange(n, device="cuda") ^ ((seed * MIX[1] + step * MIX[2] + ordinal * MIX[3]) & low)
    for mul, shift in ((MIX[0], 15), (MIX[1], 14), (MIX[4], 16)):
        h = (h * mul) & low
        h = h ^ (h >> shift)
    return h & 0xffff, h >> 16


def _blocks(x):
    n = x.numel()
    return torch.nn.functional.pad(x.reshape(-1), (0, -n % 256)).view(-1, 256)


def _values(q, scale):
    flat = q.reshape(-1).float().double()
    return flat * scale.double().repeat_interleave(256)[:flat.numel()]


def _adam_reference(p, g, m, v, step, gs=1.0, lr=LR, decay=DECAY):
    """In 64 bits; the new values and how far fp32 may be off them."""
    b1, b2 = (torch.tensor(b).double() for b in (B1, B2))
    g = g.double().reshape(-1) * gs
    p, m, v = (t.double().reshape(-1) for t in (p, m, v))
    em = 6 * U32 * (B1 * m.abs() + (1 - B1) * g.abs())
    m, v = B1 * m + (1 - B1) * g, B2 * v + (1 - B2) * g * g
    ev = 8 * U32 * v
    c1, c2 = 1 / (1 - B1 ** step), (1 - B2 ** step) ** -0.5
    denom = v.sqrt() * c2 + EPS
    upd = lr * c1 * m / denom
    new = p * (1 - lr * decay) - upd
    return new, m, v, 4 * U32 * p.abs() + abs(lr) * c1 * em / denom + 16 * U32 * upd.abs() + 2.0 ** -140, em + 2.0 ** -140, ev + 2.0 ** -140


def _adam_inputs(n, kind, g, master):
    p32 = torch.randn(n, generator=g, device="cuda")
    grad = (torch.randn(n, generator=g, device="cuda") * torch.randn(n, generator=g, device="cuda").exp()).to(TYPES[kind])
    return p32.to(TYPES[kind]), grad, (p32 if master else None)


@pytest.mark.parametrize("kind,master", [("f32", False), ("bf16", False), ("bf16", True), ("f16", True), ("f16", False)])
@pytest.mark.parametrize("n", [1, 7, 8, 255, 256, 257, 2048, 2049, 5000, 70001])
def test_adamw(ctx, n, kind, master):
    import paper_2208_11580_amd as pkg

    g = _gen(n)
    p, grad, copy = _adam_inputs(n, kind, g, master)
    m, v = torch.randn(n, generator=g, device="cuda"), torch.rand(n, generator=g, device="cuda")
    st = pkg.AdamState(m, v, None, None, copy)
    want = _adam_reference(p if copy is None else copy, grad, m, v, 3, gs=0.25)
    gs = torch.full((1,), 0.25, device="cuda")
    out = [torch.full_like(p, NAN)], [pkg.AdamState(*[None if t is None else torch.full_like(t, NAN) for t in st])]
    plan = ctx.obc_adamw_plan([p], [grad], [st], decay=DECAY, out=out)
    held = [t.clone() for t in (p, grad, m, v)]
    new_p, new = ctx.obc_adamw(plan, 3, LR, B1, B2, EPS, grad_scale=gs)
    assert all(torch.equal(a, b) for a, b in zip(held, (p, grad, m, v)))
    _within(new_p[0], want[0], want[3] + ROUND[kind] * 1.01 * want[0].abs() + TINY[kind])
    _within(new[0].m, want[1], want[4])
    _within(new[0].v, want[2], want[5])
    if master:
        _within(new[0].master, want[0], want[3])
        assert torch.equal(new_p[0], new[0].master.to(TYPES[kind]))
    # in place, the step and the rate on the device: the same bits
    at, rate = torch.tensor([3], device="cuda"), torch.full((1,), LR, device="cuda")
    ctx.obc_adamw(ctx.obc_adamw_plan([p], [grad], [st], decay=[DECAY]), at, rate, B1, B2, EPS, grad_scale=gs)
    assert torch.equal(p, new_p[0]) and all(a is None or torch.equal(a, b) for a, b in zip(st, new[0]))
    ctx.obc_check()


@pytest.mark.parametrize("kind,master", [("f32", False), ("bf16", True), ("f16", False)])
@pytest.mark.parametrize("n", [1, 9, 256, 300, 2047, 2049, 70001])
def test_adamw_of_8_bit_moments(ctx, n, kind, master):
    import paper_2208_11580_amd as pkg

    g = _gen(n + 1)
    p, grad, copy = _adam_inputs(n, kind, g, master)
    st = ctx.obc_adamw_state(p, bits=8, master=master)
    assert (copy is None) == (st.master is None)
    if copy is not None:
        st.master.copy_(copy)
    blocks = -(-n // 256)
    st.m.copy_((torch.randn(n, generator=g, device="cuda") * 60).clamp(-448, 448).to(torch.float8_e4m3fn))
    st.v.copy_((torch.rand(n, generator=g, device="cuda") * 448).to(torch.float8_e4m3fn))
    st.m_scale.copy_(torch.rand(blocks, generator=g, device="cuda") * 1e-2)
    st.v_scale.copy_(torch.rand(blocks, generator=g, device="cuda") * 1e-3)
    m0, r0 = _values(st.m, st.m_scale), _values(st.v, st.v_scale)
    want = _adam_reference(p if copy is None else copy, grad, m0, r0 * r0, 5)
    out = [torch.empty_like(p)], [pkg.AdamState(*[None if t is None else torch.empty_like(t) for t in st])]
    (new_p,), (new,) = ctx.obc_adamw(ctx.obc_adamw_plan([p], [grad], [st], decay=DECAY, out=out), 5, LR, B1, B2, EPS, seed=11)
    # (the stored root and its square are rounded on the way in)
    _within(new_p, want[0], want[3] + 8 * U32 * (want[0] - p.double() * (1 - LR * DECAY)).abs() + 8 * U32 * want[0].abs()
            + ROUND[kind] * 1.01 * want[0].abs() + TINY[kind])
    um, uv = _dither(n, 11, 5, 0)
    for got, scale, x, err, u in ((new.m, new.m_scale, want[1], want[4] + 2 * U32 * want[1].abs(), um),
                                  (new.v, new.v_scale, want[2].sqrt(), 8 * U32 * want[2].sqrt(), uv)):
        top = _blocks(x.abs()).amax(1)
        _within(scale, top / 448, _blocks(err).amax(1) / 448 + 2 * U32 * top / 448)
        a = (x.abs() / (top / 448).repeat_interleave(256)[:n]).clamp_max(448.0)
        q = torch.exp2(torch.log2(a.clamp_min(2.0 ** -6)).floor() - 3)
        # the number below or above that the dither says; near the edge, or near the next octave, either
        slack = (err / (top / 448).repeat_interleave(256)[:n] + 8 * U32 * a) / q + 2.0 ** -23
        place = a / q + u.double() / 65536
        lo, hi = (place - slack).floor() * q, (place + slack).floor() * q
        c = got.reshape(-1).float().double()
        octave = torch.log2(a.clamp_min(2.0 ** -20))
        edge = (octave - octave.round()).abs() < 1e-5
        least = 2.0 ** -9 if got is new.v else 0.0
        ok = ((c.abs() >= lo) & (c.abs() <= hi.clamp_min(least))) | (edge & ((c.abs() - a).abs() <= q))
        assert ok.all(), int((~ok).sum())
        assert ((c == 0) | (torch.sign(c) == torch.sign(x))).all()
        if got is new.v:
            assert (c[x > 0] > 0).all()
    # in place, the step on the device: the same bits
    ctx.obc_adamw(ctx.obc_adamw_plan([p], [grad], [st], decay=DECAY), torch.tensor([5], device="cuda"), LR, B1, B2, EPS, seed=11)
    assert torch.equal(p, new_p) and all(a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(st, new))
    ctx.obc_check()


def test_adamw_of_many_tensors(ctx):
    """More tensors than a launch takes, empty ones among them, at odd addresses: what each alone gives; neighbours stay."""
    import paper_2208_11580_amd as pkg

    g = _gen(17)
    sizes = [0, 5, 4096, 0, 1, 257, 10000] * 15 + [0]
    params, grads, states, wants, fences = [], [], [], [], []
    for i, n in enumerate(sizes):
        p = torch.randn(n, generator=g, device="cuda").bfloat16()
        grad = torch.randn(n, generator=g, device="cuda").bfloat16()
        m, v = torch.randn(n, generator=g, device="cuda"), torch.rand(n, generator=g, device="cuda")
        alone = p.clone(), pkg.AdamState(m.clone(), v.clone())
        ctx.obc_adamw(ctx.obc_adamw_plan([alone[0]], [grad], [alone[1]], decay=0.01 * i), 2, LR)
        wants.append(alone)
        held = torch.full((n + 4,), 7.0, device="cuda", dtype=torch.bfloat16)
        held[1:n + 1] = p
        fences.append(held)
        params.append(held[1:n + 1])
        grads.append(grad)
        states.append(pkg.AdamState(_unaligned(m), _unaligned(v)))
    ctx.obc_adamw(ctx.obc_adamw_plan(params, grads, states, decay=[0.01 * i for i in range(len(sizes))]), 2, LR)
    for p, st, held, (want_p, want) in zip(params, states, fences, wants):
        assert torch.equal(p, want_p) and torch.equal(st.m, want.m) and torch.equal(st.v, want.v)
        assert held[0] == 7 and (held[p.numel() + 1:] == 7).all()
    ctx.obc_adamw(ctx.obc_adamw_plan([], [], []), 1, LR)
    ctx.obc_check()


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw_that_is_skipped(ctx, bits):
    """A gradient scale that is not finite, or a step on the device that is none, leaves every bit as it is."""
    import paper_2208_11580_amd as pkg

    g = _gen(bits)
    for master in (True, False):
        p, grad, _ = _adam_inputs(3000, "bf16", g, False)
        st = ctx.obc_adamw_state(p, bits=bits, master=master)
        plan = ctx.obc_adamw_plan([p], [grad], [st])
        ctx.obc_adamw(plan, 1, LR)
        if master:
            st.master.add_(1e-5)      # (p need not be its rounded copy)
        held = [t.clone() for t in (p, *st) if t is not None]
        out = [torch.zeros_like(p)], [pkg.AdamState(*[None if t is None else torch.zeros_like(t) for t in st])]
        away = ctx.obc_adamw_plan([p], [grad], [st], out=out)
        for scale in (NAN, INF, -INF):
            gs = torch.full((1,), scale, device="cuda")
            ctx.obc_adamw(plan, 2, LR, grad_scale=gs)
            ctx.obc_adamw(away, 2, LR, grad_scale=gs)
            for a, b, c in zip(held, [t for t in (p, *st) if t is not None], [t for t in (out[0][0], *out[1][0]) if t is not None]):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)) and torch.equal(a.view(torch.uint8), c.view(torch.uint8))
        ctx.obc_check()
        ctx.obc_adamw(plan, torch.tensor([0], device="cuda"), LR)
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(held, [t for t in (p, *st) if t is not None]))
        with pytest.raises(Exception):
            ctx.obc_check()


def test_adamw_of_values_that_are_not_finite(ctx):
    """A NaN stays in its element (32 bits) or its block (8), an infinity too; blocks of zeros stay zeros."""
    import paper_2208_11580_amd as pkg

    p = torch.zeros(1024, device="cuda")
    grad = torch.ones(1024, device="cuda")
    grad[5], grad[300] = NAN, INF
    grad[512:768] = 0.0
    st = ctx.obc_adamw_state(p, bits=32)
    ctx.obc_adamw(ctx.obc_adamw_plan([p], [grad], [st], decay=0.0), 1, LR)
    assert p.isnan().sum() == 2 and p[5].isnan() and p[300].isnan() and st.m.isnan().sum() == 1 and (p[512:768] == 0).all()
    p.zero_()
    st = ctx.obc_adamw_state(p, bits=8)
    ctx.obc_adamw(ctx.obc_adamw_plan([p], [grad], [st], decay=0.0), 1, LR)
    assert p.isnan().sum() == 2
    assert st.m_scale.isnan().tolist() == [True, True, False, False] and st.v_scale.isnan().tolist() == [True, True, False, False]
    assert st.m_scale[2] == 0 and (st.m.float()[512:768] == 0).all() and (p[512:768] == 0).all()
    assert torch.isfinite(p[768:]).all() and (st.m.float()[768:] == 448).all()
    # a block below the smallest scale becomes zeros, and the step divides by no zero
    tiny = ctx.obc_adamw_state(p[:256], bits=8)
    q = torch.zeros(256, device="cuda")
    ctx.obc_adamw(ctx.obc_adamw_plan([q], [torch.full((256,), 1e-35, device="cuda")], [tiny], decay=0.0), 1, LR)
    assert torch.isfinite(q).all() and tiny.m_scale[0] == 0
    ctx.obc_check()
    assert isinstance(tiny, pkg.AdamState)


@pytest.mark.parametrize("together", [True, False])
def test_8_bit_moments_follow_on_average(ctx, together):
    """After steps with small changes the 8-bit moments' means are the exact ones': a step changes v by a hundredth and the 8-bit
    numbers' distance is an eighth, so that rounding to nearest would leave every one of them where it was."""
    n, steps = 1 << 18, 60
    p = torch.zeros(n, device="cuda")
    st = ctx.obc_adamw_state(p, bits=8)
    grad = torch.full((n,), 1.0, device="cuda")
    grad[::256] = 8.0      # the blocks' largest, whose codes stay 448
    small = torch.ones(n, dtype=torch.bool, device="cuda")
    small[::256] = False
    plan = ctx.obc_adamw_plan([p], [grad], [st], decay=0.0)
    for t in range(1, steps + 1):
        if t == 31:      # the largest with the others (which then stay an eighth of them: 56 of 448, exactly), or not
            grad[small] *= 0.5
            if together:
                grad[::256] *= 0.5
        ctx.obc_adamw(plan, t, 0.0, B1, B2, EPS)
    v = 0.0
    for t in range(1, steps + 1):
        v = B2 * v + (1 - B2) * (0.25 if t > 30 else 1.0)
    r = _values(st.v, st.v_scale)[small]
    # r is rounded with error at most an eighth each step, zero on average; its square's mean gains the variance: a grid step q is
    # at most r / 8, the variance of one rounding at most q^2 / 4, and each step keeps B2 of it: below (1 / 8)^2 / 4 / (1 - B2)
    # of v in all steps, 39 % -- but r follows v as v = B2 r^2 + ..., whose mean is exact but for that gain per step
    mean = float((r * r).mean())
    assert mean > v * 0.97
    assert mean < v * (1 + (1 / 8) ** 2 / 4) ** steps
    m = 0.0
    for t in range(1, steps + 1):
        m = B1 * m + (1 - B1) * (0.5 if t > 30 else 1.0)
    got = float(_values(st.m, st.m_scale)[small].mean())
    # m is linear: no gain.  An element's deviation is at most a sixteenth of it each step, a tenth of which goes: sqrt(1 / 0.19) of
    # that, and the mean of n has a deviation of 1 / 512 of it; five of those
    assert abs(got - m) < 5 * m / 16 * (1 / 0.19) ** 0.5 / 512
    # every step's dither is another, every tensor's too, and the seed's
    p2 = torch.zeros(4096, device="cuda")
    codes = []
    for step, seed, place in ((1, 0, 0), (2, 0, 0), (1, 1, 0), (1, 0, 1)):
        pair = [ctx.obc_adamw_state(p2, bits=8) for _ in range(2)]
        gr = torch.rand(4096, generator=_gen(1), device="cuda")
        ctx.obc_adamw(ctx.obc_adamw_plan([p2, p2.clone()], [gr, gr], pair), step, 0.0, seed=seed)
        codes.append(pair[place].m.view(torch.uint8).clone())
    for i in range(4):
        for j in range(i):
            assert 0.05 < float((codes[i] != codes[j]).float().mean())


# ------------------------------------------------------------------------------------------------ refusals
def test_refusals(ctx):
    import paper_2208_11580_amd as pkg

    z = torch.randn(3, 50, device="cuda")
    i3 = torch.zeros(3, dtype=torch.int32, device="cuda")
    gain = torch.ones(50, device="cuda")
    p = torch.randn(20, device="cuda")
    st = ctx.obc_adamw_state(p)
    st8 = ctx.obc_adamw_state(p, bits=8)
    plan = ctx.obc_adamw_plan([p], [p], [st])
    refused = [
        lambda: ctx.obc_score(z, top=-1), lambda: ctx.obc_score(z, top=1025), lambda: ctx.obc_score(z, temperature=0.0),
        lambda: ctx.obc_score(z, temperature=INF), lambda: ctx.obc_score(z, temperature=NAN), lambda: ctx.obc_score(z, temperature=1e-39),
        lambda: ctx.obc_score(z.to(torch.int8)), lambda: ctx.obc_score(z.double()), lambda: ctx.obc_score(z.t()), lambda: ctx.obc_score(z, i3.long()),
        lambda: ctx.obc_score(z, i3[:2]), lambda: ctx.obc_score(z.cpu()), lambda: ctx.obc_score(z, top=4, out={"top_index": i3}),
        lambda: ctx.obc_score(z, out={"lse": p}), lambda: ctx.obc_score(z[0]),
        lambda: ctx.obc_layernorm(z, gain[:49]), lambda: ctx.obc_layernorm(z, gain, p), lambda: ctx.obc_layernorm(z, gain, eps=-1.0),
        lambda: ctx.obc_layernorm(z, gain, eps=NAN), lambda: ctx.obc_layernorm(z, gain, residual=z[:2]),
        lambda: ctx.obc_layernorm(z, gain, residual=z.half()), lambda: ctx.obc_layernorm(z.t(), gain[:3]),
        lambda: ctx.obc_layernorm(torch.zeros(1, 65537, device="cuda"), torch.zeros(65537, device="cuda")),
        lambda: ctx.obc_layernorm_grad(z, gain, gain[:3], gain[:2], z), lambda: ctx.obc_layernorm_grad(z, gain, gain[:3], gain[:3], z.half()),
        lambda: ctx.obc_layernorm_grad(z, gain, gain[:3], gain[:3], z[:2]),
        lambda: ctx.obc_embed(z, i3.long()), lambda: ctx.obc_embed(z.t(), i3), lambda: ctx.obc_embed(z.double(), i3),
        lambda: ctx.obc_embed(z, i3, out=torch.empty(2, 50, device="cuda")), lambda: ctx.obc_embed(z, i3, out_dtype=torch.int8),
        lambda: ctx.obc_embed_grad(i3[:2], z, 9), lambda: ctx.obc_embed_grad(i3, z, 9, accumulate=True),
        lambda: ctx.obc_embed_grad(i3, z, 9, out=torch.empty(8, 50, device="cuda")), lambda: ctx.obc_embed_grad(i3, z, 0),
        lambda: ctx.obc_adamw(plan, 0, LR), lambda: ctx.obc_adamw(plan, 1, NAN), lambda: ctx.obc_adamw(plan, 1, LR, beta1=1.0),
        lambda: ctx.obc_adamw(plan, 1, LR, beta2=-0.1), lambda: ctx.obc_adamw(plan, 1, LR, eps=0.0),
        lambda: ctx.obc_adamw(plan, i3[:1], LR), lambda: ctx.obc_adamw(plan, 1, LR, grad_scale=gain),
        lambda: ctx.obc_adamw_plan([p], [p.half()], [st]), lambda: ctx.obc_adamw_plan([p], [p[:19]], [st]), lambda: ctx.obc_adamw_plan([p], [p], []),
        lambda: ctx.obc_adamw_plan([p, p], [p, p], [st, st8]), lambda: ctx.obc_adamw_plan([p], [p], [st], decay=[0.1, 0.2]),
        lambda: ctx.obc_adamw_plan([p], [p], [pkg.AdamState(st8.m, st8.v)]), lambda: ctx.obc_adamw_plan([p], [p], [st], out=([p], [st8])),
        lambda: ctx.obc_adamw_plan([p], [p], [st], decay=NAN) and ctx.obc_adamw(ctx.obc_adamw_plan([p], [p], [st], decay=NAN), 1, LR),
        lambda: ctx.obc_adamw_state(p, bits=16), lambda: plan.use([p[:3]]), lambda: plan.use([]),
    ]
    for i, call in enumerate(refused):
        with pytest.raises((ValueError, pkg.ObcError)):
            call()
            pytest.fail("call %d was not refused" % i)
    for call in (lambda f: ctx.obc_score(f(z)), lambda f: ctx.obc_layernorm(f(z), gain), lambda f: ctx.obc_layernorm(z, gain, f(gain)),
                 lambda f: ctx.obc_layernorm_grad(z, gain, gain[:3], gain[:3], f(z)), lambda f: ctx.obc_embed(f(z), i3),
                 lambda f: ctx.obc_embed_grad(i3, f(z), 5), lambda f: ctx.obc_adamw_plan([f(p)], [p], [st]), lambda f: plan.use([f(p)])):
        with pytest.raises(ValueError):
            call(lambda t: t.clone().requires_grad_())
        with torch.no_grad():
            call(lambda t: t.clone().requires_grad_())
    ctx.obc_check()


@pytest.mark.parametrize("kind,factor", [("f32", 1e35), ("bf16", 1e35), ("f16", 2e3), ("f32", 1e-30), ("bf16", 1e-38)])
def test_score_of_huge_and_tiny_logits(ctx, kind, factor):
    """Differences that no exponential survives, maxima that a product with 1 / temperature brings near fp32's end, and logits that
    are all but equal."""
    g = _gen(1)
    for V in (300, 9000, 40000):
        z = (torch.randn(3, V, generator=g, device="cuda") * factor).to(TYPES[kind])
        z[1, ::7] = -INF
        z[2, ::3] = torch.finfo(TYPES[kind]).min
        target = torch.randint(0, V, (3,), generator=g, device="cuda", dtype=torch.int32)
        r = ctx.obc_score(z, target, top=12, temperature=0.5)
        _check_score(r, z, target, 12, 0.5)
    ctx.obc_check()


@pytest.mark.parametrize("allowed", [1, 5, 63, 64, 65, 2000])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_score_of_constrained_answers(ctx, kind, allowed):
    """Few tokens are allowed, fewer than are asked for and more: the rest is masked with -inf or with the type's lowest value."""
    g = _gen(allowed)
    V = 50000
    z = torch.full((4, V), -INF, device="cuda")
    for row in range(4):
        at = torch.randperm(V, generator=g, device="cuda")[:allowed]
        z[row, at] = torch.randn(allowed, generator=g, device="cuda")
    z[2:] = z[2:].clamp_min(torch.finfo(TYPES[kind]).min)
    z = z.to(TYPES[kind])
    r = ctx.obc_score(z, None, top=64)
    _check_score(r, z, None, 64, 1.0)
    ctx.obc_check()


def test_offsets_beyond_32_bits(ctx):
    """Rows that begin beyond 2^31 and 2^32 elements."""
    g = _gen(1)
    big = torch.empty(3 * 1600000000 + 6000, dtype=torch.bfloat16, device="cuda")
    z = big.as_strided((4, 5000), (1600000000, 1))
    z.copy_(torch.randn(4, 5000, generator=g, device="cuda"))
    target = torch.randint(0, 5000, (4,), generator=g, device="cuda", dtype=torch.int32)
    want = ctx.obc_score(z.contiguous(), target, top=20)
    got = ctx.obc_score(z, target, top=20)
    assert all(torch.equal(want[n], got[n]) for n in want)
    ids = torch.tensor([3, 1, -1, 2, 0, 3], dtype=torch.int32, device="cuda")
    y = ctx.obc_embed(z, ids, scale=2.0)
    assert torch.equal(y, ctx.obc_embed(z.contiguous(), ids, scale=2.0))
    dt = ctx.obc_embed_grad(ids, y, 4)
    z.zero_()
    ctx.obc_embed_grad(ids, y, 4, out=z)
    assert torch.equal(z, dt)
    del big, z
    T, d = 33000, 65536
    x = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    x.normal_(generator=g)
    gain, bias = torch.rand(d, generator=g, device="cuda"), torch.rand(d, generator=g, device="cuda")
    n = ctx.obc_layernorm(x, gain, bias, want_stats=True)
    last = ctx.obc_layernorm(x[-5:].contiguous(), gain, bias, want_stats=True)
    assert all(torch.equal(n[k][-5:], last[k]) for k in ("y", "mean", "rstd"))
    dy = n["y"]
    r = ctx.obc_layernorm_grad(x, gain, n["mean"], n["rstd"], dy)
    tail = ctx.obc_layernorm_grad(x[-5:].contiguous(), gain, n["mean"][-5:].contiguous(), n["rstd"][-5:].contiguous(), dy[-5:].contiguous())
    assert torch.equal(r["dx"][-5:], tail["dx"])
    ctx.obc_check()


def test_adamw_beyond_32_bits(ctx):
    """A tensor of more than 2^32 elements: its last ones as a short tensor's, but for the dither, which their places give."""
    import paper_2208_11580_amd as pkg

    n, m = 2 ** 32 + 5000, 5000 - 5000 % 256
    p = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    grad = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g = _gen(2)
    tail = slice(2 ** 32, 2 ** 32 + m)
    grad[tail] = torch.randn(m, generator=g, device="cuda").to(torch.bfloat16)
    st = ctx.obc_adamw_state(p, bits=8)
    ctx.obc_adamw(ctx.obc_adamw_plan([p], [grad], [st], decay=0.0), 1, LR, B1, B2, EPS)
    want = _adam_reference(p[tail] * 0, grad[tail], torch.zeros(m, device="cuda"), torch.zeros(m, device="cuda"), 1, decay=0.0)
    _within(p[tail], want[0], want[3] + ROUND["bf16"] * 1.01 * want[0].abs() + TINY["bf16"])
    assert (p[:2 ** 32].view(torch.int64) == 0).all()
    scale = st.m_scale[2 ** 32 // 256:][:m // 256].double()
    _within(scale, _blocks(want[1].abs()).amax(1) / 448, 8 * U32 * scale + 1e-30)
    got = _values(st.m[tail], scale)
    # up or down: within a step of an eighth, and of 2^-9 of the scale
    assert ((got - want[1]).abs() <= want[1].abs() / 8 + 2.0 ** -9 * scale.repeat_interleave(256)).all()
    assert isinstance(st, pkg.AdamState)


def test_refusals_of_plans_and_devices(ctx):
    import paper_2208_11580_amd as pkg

    p, q = torch.zeros(600, device="cuda"), torch.zeros(600, device="cuda")
    st, su = ctx.obc_adamw_state(p), ctx.obc_adamw_state(q)
    both = pkg.AdamState(st.m, st.v)
    big = torch.zeros(1000, device="cuda")
    for args, out in ((([p, p], [p, p], [st, su]), None), (([p, q], [p, p], [st, both]), None), (([p], [q], [st]), ([st.m], [su])),
                      (([big[:600]], [q], [st]), ([big[8:608]], [su])), (([p], [q], [pkg.AdamState(big[:600], big[400:])]), None),
                      (([p, q], [p, p], [st, su]), ([big[:600], big[400:]], [ctx.obc_adamw_state(p), ctx.obc_adamw_state(p)]))):
        if out is not None and out[0][0] is st.m:
            out = ([su.m], [su])
        with pytest.raises(pkg.ObcError):
            ctx.obc_adamw_plan(*args, out=out)
    ctx.obc_adamw_plan([big[:600], big[600:]], [p, p[:400]], [st, ctx.obc_adamw_state(big[600:])])      # neighbours are apart
    plan = ctx.obc_adamw_plan([p], [q], [st])
    other = pkg.Context()
    with pytest.raises(ValueError):
        other.obc_adamw(plan, 1, LR)
    other._device = 1      # as if it were another device's
    i3 = torch.zeros(3, dtype=torch.int32, device="cuda")
    z = torch.zeros(3, 600, device="cuda")
    for call in (lambda c: c.obc_score(z), lambda c: c.obc_layernorm(z, p), lambda c: c.obc_layernorm_grad(z, p, p[:3], p[:3], z),
                 lambda c: c.obc_embed(z, i3), lambda c: c.obc_embed_grad(i3, z, 4), lambda c: c.obc_adamw_plan([p], [q], [st])):
        with pytest.raises(ValueError):
            call(other)
    other._device = 0
    other.close()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c = pkg.Context(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            y = c.obc_embed(z, i3)
            with pytest.raises(ValueError):
                c.obc_adamw_plan([p], [q], [st])
        graph.replay()
        side.synchronize()
        assert (y == 0).all()
        del graph
        c.close()
    ctx.obc_check()


@pytest.mark.parametrize("V", [300, 9000, 40000])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("power", [90, 105, 115, 120, 125])
def test_score_at_temperatures_as_large_as_the_logits(ctx, power, kind, V):
    """Logits up to the ends of their types at temperatures that bring them back to a few units: differences of two logits are beyond
    fp32's end, and every logit counts."""
    g = _gen(power)
    end = torch.finfo(TYPES[kind]).max
    z = (torch.randn(4, V, generator=g, device="cuda") * 2.0 ** min(power, 125)).clamp(-end, end).to(TYPES[kind])
    z[1, 1::5] = -end
    z[1, 3] = end
    z[2, V // 2:] = -INF
    z[3] = z[3].abs().neg()
    target = torch.tensor([0, 1, V - 1, 2], dtype=torch.int32, device="cuda")
    for k in (0, 12, 300):
        _check_score(ctx.obc_score(z, target, top=k, temperature=2.0 ** power), z, target, k, 2.0 ** power)
    ctx.obc_check()
