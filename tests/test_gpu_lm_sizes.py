"""Products with 4-bit weights, norms and distillation at the sizes where the larger tiles, the wider workgroups and the loops over rows
take over, each with something ragged at its end; rows too long for a kernel's arithmetic."""
import ctypes

import pytest
import torch

from .test_gpu_lm import U32, _gen, _layer, _product_bound, _within, ctx  # noqa: F401

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
