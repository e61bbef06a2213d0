"""Products with 4-bit weights, norms and distillation at the sizes where the larger tiles, the wider workgroups and the loops over rows
take over, each with something ragged at its end; rows too long for a kernel's arithmetic."""
import ctypes

import pytest
import torch

from . import test_gpu_lm as lm
from .test_gpu_lm import ROUND, TINY, TYPES, U32, _gen, _layer, _logits, _product_bound, _within, ctx  # noqa: F401

pytestmark = pytest.mark.gpu


def test_rows_of_more_than_eight_million_columns(ctx):
    """One group: every tile of columns belongs to it, also where the number of tiles squared passes 2^32."""
    R, d = 16, 128 * 65600 + 5
    g = _gen(3)
    codes = torch.randint(0, 16, (R, d), generator=g, device="cuda", dtype=torch.int32)
    delta = (torch.rand(R, 1, generator=g, device="cuda") * 0.02 + 0.001).half().float()
    offset = (-7.5 * delta).half().float()
    P = ctx.obc_pack4(codes, delta, offset)
    W = offset.double() + delta.double() * codes.double()
    del codes
    x = torch.randn(3, d, generator=g, device="cuda").half()
    y = ctx.obc_product4(P, x, out_dtype=torch.float32)
    ctx.obc_check()
    want = x.double() @ W.T
    err = float((y.double() - want).norm() / want.norm())
    # sums of 128 columns, and the sum of those
    assert err <= U32 * ((128 / 6) ** 0.5 + (d / 128 / 6) ** 0.5), err


def test_groups_too_long_for_their_rows_are_refused(ctx):
    """Checked before anything is launched: the addresses are none."""
    import paper_2208_11580_amd as pkg

    p = ctypes.c_void_p(256)
    for d, group in ((128 * 65600, 128 * 65599), (2 ** 31 - 1, 2 ** 30), (2 ** 31 - 1, 128 * 256)):
        for T in (1, 3, 100):
            rc = ctx.lib.obc_product4(ctx.h, p, 16, d, group, p, pkg.binding.F16, None, T, d, p, pkg.binding.F16, 16, p, 1 << 60)
            assert rc == pkg.OBC_ERR_BAD_SHAPE, (d, group, T)


# -------------------------------------------------------- tiles of 128 x 256, 32 rows to a workgroup, chunks of columns
@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d,group", [(1283, 0), (1283, 32), (1290, 64), (1283, 128), (1280, 128), (1283, 384)])
def test_products_of_prompts(ctx, d, group, kind):
    """16 x 13 tiles of 128 x 256 (fp32: 64 x 128), ragged at every end; 1280 columns are multiplied as they lie."""
    lm.test_product(ctx, 2000, 3300, d, group, kind)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("d,group", [(1283, 0), (1283, 32), (1290, 64), (1280, 128)])
def test_products_of_8_bit_prompts(ctx, d, group, out):
    lm.test_product_of_8_bit_inputs(ctx, 2000, 3300, d, group, out)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16", "i8"])
@pytest.mark.parametrize("T,R,d,group", [(1, 4200, 1283, 128), (5, 4200, 1283, 64), (16, 5000, 1283, 32), (7, 5000, 640, 0), (3, 4100, 2049, 256),
                                         (16, 6500, 1283, 128), (16, 6500, 8192, 32), (13, 6500, 5000, 64), (16, 6500, 9300, 64)])
def test_few_tokens_through_many_rows(ctx, T, R, d, group, kind):
    """32 rows of weights to a workgroup; the last four also with tokens that do not fit in LDS at once (the last in any type)."""
    if kind == "i8":
        lm.test_product_of_8_bit_inputs(ctx, T, R, d, group, "f32")
    else:
        lm.test_product(ctx, T, R, d, group, kind)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16", "i8"])
@pytest.mark.parametrize("T,R,d,group", [(30, 500, 1283, 32), (18, 333, 1290, 64), (31, 200, 2049, 128)])
def test_up_to_32_tokens(ctx, T, R, d, group, kind):
    if kind == "i8":
        lm.test_product_of_8_bit_inputs(ctx, T, R, d, group, "f16")
    else:
        lm.test_product(ctx, T, R, d, group, kind)


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("T,R,d,group", [(2000, 3300, 1283, 0), (2000, 3300, 1283, 32), (2000, 3300, 1290, 64), (2000, 3300, 1280, 128),
                                         (100, 500, 1283, 32), (100, 500, 1283, 64), (30, 500, 1283, 32), (30, 500, 1283, 64),
                                         (16, 6500, 8192, 32), (5, 4200, 1283, 64), (7, 5000, 640, 0), (3, 300, 1283, 64), (3, 300, 1283, 32)])
def test_16_bit_inputs_into_fp32(ctx, T, R, d, group, kind):
    g = _gen(T + R + d)
    codes, delta, offset, W, mag = _layer(R, d, group, g)
    x = torch.randn(T, d, generator=g, device="cuda").to(TYPES[kind])
    y = ctx.obc_product4(ctx.obc_pack4(codes, delta, offset, group), x, out_dtype=torch.float32)
    ctx.obc_check()
    want = x.double() @ W.T
    _within(y, want, _product_bound(x, mag, want, "f32", d))
    # sums of 128 columns, and the sum of those, each addition rounded to nearest
    err = float((y.double() - want).norm() / want.norm())
    assert err <= U32 * ((128 / 6) ** 0.5 + (d / 128 / 6) ** 0.5), err


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("group", [0, 32, 64, 128, 256])
def test_gradients_of_prompts(ctx, group, kind):
    """16 x 13 tiles of 128 x 256, the last of 28 columns' tile alone (fp32: 32 x 25 of 64 x 128)."""
    lm.test_product_grad(ctx, 2000, 700, 3100, group, kind)


# ------------------------------------------------------------------------------------------------------- norms
@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,d", [(600, 2049), (600, 4096), (600, 4097), (520, 8191), (520, 16384), (513, 16391)])
def test_norms_of_many_rows(ctx, T, d, kind):
    lm.test_rmsnorm(ctx, T, d, kind)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,d", [(600, 2049), (600, 4097), (1100, 8192), (600, 9000), (520, 16384), (530, 16391)])
def test_norm_gradients_of_several_rows_to_a_workgroup(ctx, T, d, kind):
    lm.test_rmsnorm_grad(ctx, T, d, kind)


# ------------------------------------------------------------------------------------------------ distillation
def _distill(z, index, logit, tau, weight):
    """The plain form in 64 bits, with the bounds of the other tests, all rows at a time."""
    valid, at = index >= 0, index.clamp_min(0).long()
    x, t, w = z.double() / tau, logit.double() / tau, weight.double()
    lq = torch.log_softmax(x, 1)
    lp = torch.log_softmax(torch.where(valid, t, float("-inf")), 1)
    p = torch.where(valid, lp.exp(), 0.0)
    l1, l2 = torch.where(valid, lp, 0.0), lq.gather(1, at)
    loss = w * tau * tau * (p * (l1 - l2)).sum(1)
    lb = w * tau * tau * (200 * U32 + 20 * U32 * (p * (l1.abs() + l2.abs())).sum(1))
    q, full = lq.exp(), torch.zeros_like(x).scatter_add_(1, at, p)
    spread = torch.where(valid, t, float("-inf")).amax(1) - torch.where(valid, t, float("inf")).amin(1)
    db = ((200 + 16 * (x - x.amax(1, keepdim=True)).abs()) * q + (200 + 16 * spread[:, None]) * full) * (w * tau * U32)[:, None]
    return loss, (q - full) * (w * tau)[:, None], lb, db


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,V,k,tau", [(2100, 777, 5, 1.0), (1100, 15001, 20, 2.0), (1100, 30001, 20, 0.7), (1100, 40001, 33, 1.0),
                                       (600, 70001, 64, 1.5), (520, 131072, 100, 1.0)])
def test_distillation_of_more_rows_than_workgroups(ctx, T, V, k, tau, kind):
    """A workgroup takes several rows, the next one's logits on their way as a row's gradient goes out: beside the logits, in
    their place, and between rows that lie apart."""
    z, index, logit, weight, g = _logits(T, V, k, kind, T + V)
    count = torch.randint(1, k + 1, (T, 1), generator=g, device="cuda")
    index = torch.where(torch.arange(k, device="cuda") < count, index, -1).to(torch.int32)
    weight[::7] = 0.0
    out = ctx.obc_distill(z, index, logit, temperature=tau, weight=weight, want_grad=True)
    ctx.obc_check()
    for a in range(0, T, 256):
        rows = slice(a, a + 256)
        loss, dz, lb, db = _distill(z[rows], index[rows], logit[rows], tau, weight[rows])
        _within(out["loss"][rows], loss, lb + 2 * U32 * loss.abs())
        _within(out["dz"][rows], dz, db + ROUND[kind] * 1.01 * dz.abs() + max(TINY[kind], 1e-38))
    assert not out["dz"][::7].any() and not out["loss"][::7].any()
    assert torch.equal(ctx.obc_distill(z, index, logit, temperature=tau, weight=weight)["loss"], out["loss"])
    apart = torch.full((T, V + 3), float("nan"), device="cuda", dtype=z.dtype)
    apart[:, 1:1 + V] = z
    into = torch.full((T, V + 5), 7.0, device="cuda", dtype=z.dtype)
    r = ctx.obc_distill(apart[:, 1:1 + V], index, logit, temperature=tau, weight=weight, want_grad=True, out={"dz": into[:, 2:2 + V]})
    assert torch.equal(into[:, 2:2 + V], out["dz"]) and torch.equal(r["loss"], out["loss"])
    assert (into[:, :2] == 7.0).all() and (into[:, 2 + V:] == 7.0).all()
    over = ctx.obc_distill(z, index, logit, temperature=tau, weight=weight, want_grad=True, out={"dz": z})
    assert over["dz"] is z and torch.equal(z, out["dz"]) and torch.equal(over["loss"], out["loss"])
