"""Scales at the ends of fp32 in the products of codes, in each of the kernels."""
import numpy as np
import pytest
import torch

from fp8_testlib import codes, product, product_tolerance, scales, up

pytestmark = pytest.mark.gpu

# few rows (16, 32, 64 at a time; the reduction axis cut and not), single SMs, pairs of SMs
SHAPES = [(3, 200, 600), (3, 9600, 600), (30, 200, 600), (100, 200, 1200), (600, 300, 600), (2700, 2800, 300)]


@pytest.fixture(scope="module")
def ctx():
    import paper_1904_02205_b200 as psb

    c = psb.Context(0)
    yield c
    c.check_device()
    c.close()


def _operands(m, n, k):
    rng = np.random.default_rng(m + n + k)
    return codes(rng, m, k), scales(rng, m, up(k, 128)), codes(rng, n, k), scales(rng, up(n, 128), up(k, 128))


def _check(ctx, a, sa, b, sb):
    got = ctx.gemm_fp8(a, sa, b, sb, out_dtype=torch.float32)
    ctx.check_device()
    k = a.shape[1]
    want, size = product(a, sa, b, sb)
    # a product of two scales below 2^-126 is off by 2^-150 at most, which counts as often as its block's sum; and each of the additions of
    # scaled sums by 2^-150
    sums = a.double().abs() @ b.double().abs().t()
    tol = product_tolerance(want, size, k, torch.float32) + sums * 2.0 ** -150 + (up(k, 128) + 18) * 2.0 ** -150
    off = (got.double() - want).abs()
    assert not torch.isnan(off).any() and (off <= tol).all()
    return got


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_products_of_scales_below_the_normal_numbers(ctx, m, n, k):
    a, sa, b, sb = _operands(m, n, k)
    got = _check(ctx, a, sa * 2.0 ** -90, b, sb * 2.0 ** -40)
    assert (got != 0).any()
    _check(ctx, a, sa * 2.0 ** -110, b, sb * 2.0 ** -110)


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_very_large_scales_that_meet_very_small_ones(ctx, m, n, k):
    a, sa, b, sb = _operands(m, n, k)
    _check(ctx, a, sa * 2.0 ** 100, b, sb * 2.0 ** -100)
    _check(ctx, a, sa * 2.0 ** -60, b, sb * 2.0 ** 110)


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_blocks_of_zeros_as_they_are_quantised(ctx, m, n, k):
    """A block of zeros has the scale 2^-126, and adds nothing whatever it meets."""
    rng = np.random.default_rng(m)
    x = torch.from_numpy(rng.normal(size=(m, k)).astype(np.float32)).cuda()
    x[::2, 128:256] = 0.0
    _, _, b, sb = _operands(m, n, k)
    a, sa = ctx.quantize_fp8(x)
    got = _check(ctx, a, sa, b, sb)
    keep = torch.ones(k, device="cuda")
    keep[128:256] = 0.0
    # (the other blocks alone, in the same order of additions)
    alone = ctx.gemm_fp8((a.float() * keep).to(a.dtype), sa, b, sb, out_dtype=torch.float32) if k % 16 == 0 else None
    if alone is not None:
        assert torch.equal(got[::2], alone[::2])


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_products_of_scales_beyond_the_largest_number_are_reported(ctx, m, n, k):
    import paper_1904_02205_b200 as psb

    a, sa, b, sb = _operands(m, n, k)
    want = _check(ctx, a, sa, b, sb)
    for row, block in ((0, 0), (m - 1, up(k, 128) - 1), (m // 2, 1)):
        big, wide = sa.clone(), sb.clone()
        big[row, block], wide[-1, block] = 2.0 ** 100, 2.0 ** 40
        got = ctx.gemm_fp8(a, big, b, wide, out_dtype=torch.float32)
        assert ctx.device_status() == psb.PSB_ERR_RANGE
        rest = torch.arange(m, device="cuda") != row
        cols = torch.arange(n, device="cuda") < (up(n, 128) - 1) * 128
        assert torch.equal(got[rest][:, cols], want[rest][:, cols])
    assert ctx.device_status() == psb.PSB_OK


@pytest.mark.parametrize("gather", [True, False])
@pytest.mark.parametrize("rows", [40, 600])
def test_scales_of_experts_rows_are_reported_where_they_meet(ctx, rows, gather):
    """Row 1 of `a` has a scale that only the last expert's filter makes too large; rows behind the last run are not looked at."""
    import paper_1904_02205_b200 as psb

    rng = np.random.default_rng(rows)
    E, n, k = 3, 260, 400
    a, sa = codes(rng, rows, k), scales(rng, rows, up(k, 128))
    b, sb = codes(rng, n, k, batch=E), scales(rng, E, up(n, 128), up(k, 128))
    sa[1], sb[E - 1] = 2.0 ** 100, 2.0 ** 40
    used = rows - 5
    sa[used:] = 2.0 ** 100
    order = torch.arange(rows, dtype=torch.int32, device="cuda") if gather else None

    def call(*ends):
        ctx.gemm_fp8_experts(a, sa, b, sb, torch.tensor([0, *ends], dtype=torch.int32, device="cuda"), order=order)
        return ctx.device_status()
    assert call(7, used, used) == psb.PSB_OK and call(0, used, used) == psb.PSB_OK
    assert call(2, 7, used) == psb.PSB_OK       # (rows 7 and on meet the last filter, row 1 does not)
    assert call(0, 1, used) == psb.PSB_ERR_RANGE
