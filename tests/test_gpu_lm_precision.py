"""What the operators around compressed layers hold in how many bits: gradients of 16-bit products against their weights in
full, fp32 results over long sums, grids and norms at the ends of their ranges."""
import pytest
import torch

from .test_gpu_lm import ROUND, TINY, TYPES, U32, _gen, _layer, _product_bound, _within, ctx  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("T,R,d,group", [(7, 300, 257, 32), (50, 512, 640, 128), (64, 100, 1000, 0), (300, 512, 384, 64), (2000, 260, 3100, 128)])
def test_gradients_of_16_bits_are_rounded_once(ctx, T, R, d, group, kind):
    """A sum of R products of two terms each, partial sums cut off at 2^-23, is off by 2^-23 sqrt(R / 3) of its size in the mean
    square.  That takes a value to its neighbour if it lies that near to the middle of two, which is 2 / eps of that share
    of the values, and more of those that came out small by cancellation: 8 / eps in all.  A weight rounded to half precision,
    2^-13 off in the mean, would move tens of per cent."""
    g = _gen(T + R)
    codes, delta, offset, W, _ = _layer(R, d, group, g)
    dy = torch.randn(T, R, generator=g, device="cuda").to(TYPES[kind])
    dx = ctx.obc_product4_grad(ctx.obc_pack4(codes, delta, offset, group), dy)
    ctx.obc_check()
    want = (dy.double() @ W).to(TYPES[kind])
    moved = float((dx != want).double().mean())
    assert moved <= 8 * 2.0 ** -23 * (R / 3) ** 0.5 / torch.finfo(TYPES[kind]).eps, moved


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,R,d,group", [(3, 40, 300, 128), (50, 300, 300, 32), (100, 700, 129, 0), (2000, 300, 3100, 64)])
def test_weights_beyond_half_precision(ctx, T, R, d, group, kind):
    """Steps and offsets are numbers of half precision; the weights they stand for reach 2^20.  Some groups of some rows go
    there, the others stay as they are."""
    g = _gen(T + R + d)
    codes, delta, offset, _, _ = _layer(R, d, group, g)
    n = delta.shape[1]
    delta[R // 2, n - 1], offset[R // 2, n - 1] = 65504.0, 65504.0
    delta[1, 0], offset[1, 0] = 8368.0, -60000.0                  # -60000 .. 65520
    G = d if group <= 0 or group >= d else group
    col = torch.arange(d, device="cuda") // G
    W = offset.double()[:, col] + delta.double()[:, col] * codes.double()
    P = ctx.obc_pack4(codes, delta, offset, group)
    dy = (torch.randn(T, R, generator=g, device="cuda") * 1e-3).to(TYPES[kind])
    dx = ctx.obc_product4_grad(P, dy)
    ctx.obc_check()
    want = dy.double() @ W
    total = dy.double().abs() @ W.abs()
    assert torch.isfinite(dx[torch.isfinite(want.to(TYPES[kind]))].float()).all()
    # sums as in the gradients' other tests, weights to 2^-22 and, a 32nd of them being held, 2^-20 of the columns that go there
    far = (W.abs().amax(0) > 65504.0).double()
    tiny = 2.0 ** -20 * far * dy.double().abs().sum(1, keepdim=True)
    bound = (2.0 ** -22 * 1.01 + (6 * R + 64) * U32) * total + tiny + ROUND[kind] * 1.01 * want.abs() + TINY[kind]
    _within(torch.where(torch.isfinite(dx), dx.double(), want), want, bound)


@pytest.mark.parametrize("T,R,d", [(40, 4096, 300), (500, 4096, 2048), (600, 4096, 4096), (1000, 16384, 1024), (64, 16384, 384)])
def test_fp32_gradients_are_as_exact_as_sums_of_sums_of_128_rows(ctx, T, R, d):
    """Sums of 128 rows, then the sum of those, each addition rounded to nearest: off by 2^-24 sqrt(128 / 6) and by 2^-24 sqrt(R / 128 / 6)
    in the mean square."""
    g = _gen(T + R)
    for group in (0, 128):
        codes, delta, offset, W, _ = _layer(R, d, group, g)
        dy = torch.randn(T, R, generator=g, device="cuda")
        want = dy.double() @ W
        err = float((ctx.obc_product4_grad(ctx.obc_pack4(codes, delta, offset, group), dy).double() - want).norm() / want.norm())
        assert err <= U32 * ((128 / 6) ** 0.5 + (R / 128 / 6) ** 0.5), (group, err)


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("T,d", [(1, 128), (3, 8192), (16, 1000), (40, 300), (40, 8192), (100, 128), (100, 2000)])
def test_16_bit_inputs_with_fp32_outputs_are_as_exact_as_fp32(ctx, T, d, kind):
    """Sums of 128 columns, then the sum of those, each addition rounded to nearest: off by 2^-24 sqrt(128 / 6) and by
    2^-24 sqrt(d / 128 / 6) in the mean square."""
    g = _gen(T + d)
    for R, group in ((300, 0), (300, 32), (300, 64), (4500, 128)):
        codes, delta, offset, W, mag = _layer(R, d, group, g)
        x = torch.randn(T, d, generator=g, device="cuda").to(TYPES[kind])
        want = x.double() @ W.T
        y = ctx.obc_product4(ctx.obc_pack4(codes, delta, offset, group), x, out_dtype=torch.float32)
        err = float((y.double() - want).norm() / want.norm())
        assert err <= U32 * ((128 / 6) ** 0.5 + (d / 128 / 6) ** 0.5), (R, group, err)
        _within(y, want, _product_bound(x, mag, want, "f32", d))
    ctx.obc_check()


def test_8_bit_norm_of_a_gain_that_is_not_finite(ctx):
    """A NaN in the gain (or an infinite gain, also where h is zero) leaves no 8-bit values: scale NaN, codes 0."""
    for kind in TYPES:
        for d in (8, 500, 5000, 20000):
            for value in (float("nan"), float("inf")):
                g = _gen(d)
                x = torch.randn(4, d, generator=g, device="cuda").to(TYPES[kind])
                x[2, d - 3] = 0
                gain = torch.ones(d, device="cuda")
                gain[d - 3] = value
                q = ctx.obc_rmsnorm(x, gain, quant8=True)
                assert torch.isnan(q["scale"]).all() and not q["y"].any(), (kind, d, value)


def test_grids_cover_weights_whose_range_rounds_down(ctx):
    """The range of these groups is rounded down in fp32, to fifteen times a number of half precision."""
    W = torch.tensor([[-1.0, 0.875 + 2.0 ** -24], [-1.0, 0.875 - 2.0 ** -24], [-2.0, 1.75 + 2.0 ** -23], [0.0, 1.875 + 2.0 ** -23]],
                     device="cuda")
    for group in (0, 32):
        delta, offset, maxq = ctx.obc_group_grid(W, 4, group)
        ctx.obc_check()
        top = offset.double() + maxq * delta.double()
        assert (offset.double() <= W.double()).all() and (W.double() <= top).all(), (W.double() - top)
        assert (delta <= 0.1252 * torch.tensor([[1.0], [1.0], [2.0], [1.0]], device="cuda")).all()
