"""Quantisation to 8-bit floating point and the product of codes, against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

from fp8_testlib import E4, E5, TOP, check_product, codes, product, scales, up

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def ctx():
    import paper_1904_02205_b200 as psb

    c = psb.Context(0)
    yield c
    c.check_device()
    c.close()


# -- quantisation -----------------------------------------------------------------------------------------------------------

def quantise(x, block_rows, dtype):
    """By the definition; every step is one correctly rounded fp32 operation, so that equality is wanted."""
    x = x.float().cpu()
    R, C = x.shape
    wide = torch.nn.functional.pad(x, (0, -C % 128, 0, -R % block_rows)).reshape(up(R, block_rows), block_rows, up(C, 128), 128)
    amax = torch.where(torch.isfinite(wide), wide.abs(), torch.zeros_like(wide)).amax(dim=(1, 3))
    scale = torch.clamp(amax / TOP[dtype], min=2.0 ** -126)
    v = wide * (1.0 / scale)[:, None, :, None]
    v = torch.where(torch.isfinite(wide), v.clamp(-TOP[dtype], TOP[dtype]), torch.full_like(v, float("nan")))
    return v.reshape(up(R, block_rows) * block_rows, -1)[:R, :C].to(dtype), scale


def same_codes(got, want):
    g, w = got.float().cpu(), want.float()
    assert torch.equal(torch.isnan(g), torch.isnan(w)) and torch.equal(torch.nan_to_num(g), torch.nan_to_num(w))


@pytest.mark.parametrize("in_dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,cols,code", [(1, 1, E4), (1, 128, E4), (3, 127, E5), (129, 129, E4), (128, 4096, E4), (300, 1000, E5), (37, 2040, E4)])
def test_codes_and_scales(ctx, rows, cols, code, block_rows, in_dtype):
    rng = np.random.default_rng(rows * cols + block_rows)
    x = torch.from_numpy((rng.normal(size=(rows, cols)) * np.exp(rng.normal(0, 2, size=(1, cols)))).astype(np.float32)).to(DT[in_dtype])
    got, scale = ctx.quantize_fp8(x.cuda(), block_rows=block_rows, code_dtype=code)
    want, want_scale = quantise(x, block_rows, code)
    assert torch.equal(scale.cpu(), want_scale)
    same_codes(got, want)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_blocks_of_zeros_infinities_and_extremes(ctx, block_rows):
    x = torch.zeros(300, 640)
    x[0, 3], x[1, 130], x[2, 300], x[3, 301] = float("inf"), float("-inf"), float("nan"), 5.0
    x[130, 0], x[131, 1], x[132, 520], x[260, 639] = 3.4e38, -1e-45, 1e-38, -2.5e-39
    got, scale = ctx.quantize_fp8(x.cuda(), block_rows=block_rows)
    want, want_scale = quantise(x, block_rows, E4)
    assert torch.equal(scale.cpu(), want_scale)
    same_codes(got, want)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_strided_input_and_outputs_leave_what_lies_between(ctx, block_rows):
    rng = np.random.default_rng(5)
    big = torch.from_numpy(rng.normal(size=(140, 333)).astype(np.float32)).cuda().bfloat16()
    x = big[:, 5:265]                                       # rows start at odd addresses
    store = torch.full((140, 277), 7.0, device="cuda").to(E4)
    sstore = torch.full((140, 9), -3.0, device="cuda")
    want, want_scale = quantise(x, block_rows, E4)
    ctx.quantize_fp8(x, block_rows=block_rows, out=(store[:, 3:263], sstore[:want_scale.shape[0], 2:5]))
    same_codes(store[:, 3:263], want)
    assert torch.equal(sstore[:want_scale.shape[0], 2:5].cpu(), want_scale)
    left = torch.cat([store[:, :3], store[:, 263:]], 1).float()
    assert (left == 7.0).all() and (sstore[:, :2] == -3.0).all() and (sstore[:, 5:] == -3.0).all()


# -- product ----------------------------------------------------------------------------------------------------------------

SHAPES = [(1, 1, 1), (1, 128, 128), (3, 5, 17), (2, 1000, 2048), (15, 300, 129), (17, 130, 1000), (64, 127, 256), (65, 129, 640), (127, 64, 384),
          (128, 128, 128), (129, 257, 130), (200, 1000, 2048), (257, 384, 1152), (300, 520, 4096), (513, 260, 72), (1030, 777, 400), (2, 4096, 4096),
          (145, 554, 2774), (3000, 2500, 1000), (2999, 2507, 900)]


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_product(ctx, m, n, k, out):
    rng = np.random.default_rng(m * 7 + n * 3 + k)
    a, b = codes(rng, m, k), codes(rng, n, k)
    sa, sb = scales(rng, m, up(k, 128)), scales(rng, up(n, 128), up(k, 128))
    got = ctx.gemm_fp8(a, sa, b, sb, out_dtype=DT[out])
    ctx.check_device()
    check_product(got, *product(a, sa, b, sb), k)


@pytest.mark.parametrize("m,n,k", [(5, 70, 300), (150, 200, 300), (700, 600, 300), (2700, 2800, 300)])
@pytest.mark.parametrize("ta,tb", [(E4, E5), (E5, E4), (E5, E5)])
def test_formats_bias_relu_and_half(ctx, m, n, k, ta, tb):
    rng = np.random.default_rng(m)
    a, b = codes(rng, m, k, ta), codes(rng, n, k, tb)
    sa, sb = scales(rng, m, 3), scales(rng, up(n, 128), 3)
    bias = torch.from_numpy(rng.normal(0, 30, size=n).astype(np.float32)).cuda()
    got = ctx.gemm_fp8(a, sa, b, sb, bias=bias, relu=True, out_dtype=torch.float16)
    want, size = product(a, sa, b, sb, bias, True)
    assert float(want.max()) < 6e4 and (want == 0).any()
    check_product(got, want, size, k)


@pytest.mark.parametrize("m", [3, 60, 140, 600])
@pytest.mark.parametrize("out,offset", [("f32", 1), ("bf16", 3), ("bf16", 8)])
def test_strides_of_everything(ctx, m, out, offset):
    rng = np.random.default_rng(m)
    n, k = 270, 500
    a, b = codes(rng, m, k, pitch=560), codes(rng, n, k, pitch=512)
    sa, sb = scales(rng, m, 7)[:, 1:5], scales(rng, 3, 9)[:, 3:7]
    store = torch.full((m, n + 50), -77.0, dtype=DT[out], device="cuda")
    view = store[:, offset:offset + n]
    ctx.gemm_fp8(a, sa, b, sb, out=view)
    ctx.check_device()
    check_product(view, *product(a, sa, b, sb), k)
    assert (store[:, :offset] == -77.0).all() and (store[:, offset + n:] == -77.0).all()


@pytest.mark.parametrize("m", [2, 100, 520])
def test_nan_codes_reach_their_rows_and_columns_only(ctx, m):
    rng = np.random.default_rng(1)
    n, k = 300, 260
    a, b = codes(rng, m, k).clone(), codes(rng, n, k).clone()
    a = torch.nn.functional.pad(a.view(torch.uint8), (0, 12)).view(E4)[:, :k]
    b = torch.nn.functional.pad(b.view(torch.uint8), (0, 12)).view(E4)[:, :k]
    a[m - 1, 259] = float("nan")
    b[150, 3] = float("nan")
    sa, sb = scales(rng, m, 3), scales(rng, 3, 3)
    got = ctx.gemm_fp8(a, sa, b, sb, relu=True)
    bad = torch.isnan(got)
    assert bad[m - 1].all() and bad[:, 150].all() and int(bad.sum()) == n + m - 1


def test_zero_scales_and_zero_codes(ctx):
    rng = np.random.default_rng(2)
    a, b = codes(rng, 130, 256), codes(rng, 200, 256)
    sa, sb = scales(rng, 130, 2), scales(rng, 2, 2)
    sa[5], sb[1] = 0.0, 0.0
    got = ctx.gemm_fp8(a, sa, b, sb, out_dtype=torch.float32)
    check_product(got, *product(a, sa, b, sb), 256)
    assert (got[5] == 0).all() and (got[:, 128:] == 0).all()


@pytest.mark.parametrize("m", [1, 70, 600, 5000])
def test_the_same_call_gives_the_same_bits(ctx, m):
    rng = np.random.default_rng(3)
    a, b = codes(rng, m, 2048), codes(rng, 1000, 2048)
    sa, sb = scales(rng, m, 16), scales(rng, 8, 16)
    first = ctx.gemm_fp8(a, sa, b, sb, out_dtype=torch.float32)
    for _ in range(5):
        assert torch.equal(first, ctx.gemm_fp8(a, sa, b, sb, out_dtype=torch.float32))


def test_captured_and_replayed_on_other_streams(ctx):
    rng = np.random.default_rng(4)
    x = torch.from_numpy(rng.normal(size=(96, 600)).astype(np.float32)).cuda()
    w = torch.from_numpy(rng.normal(size=(300, 600)).astype(np.float32)).cuda()
    b, sb = ctx.quantize_fp8(w, block_rows=128)

    def layer(stream=None):
        return ctx.gemm_fp8(*ctx.quantize_fp8(x, stream=stream), b, sb, relu=True, stream=stream)

    want = layer()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        got = layer()
    for i in range(3):
        x.mul_(1.5)
        graph.replay()
        assert torch.equal(got, layer())
    with torch.cuda.stream(side):
        side.wait_stream(torch.cuda.default_stream())
        other = layer(side)
    side.synchronize()
    assert torch.equal(other, got) and not torch.equal(want, got)


def test_outputs_beyond_32_bits(ctx):
    """Byte offsets of more than 32 bits in the values, the codes and the product."""
    m, n, k = 66000, 33100, 72
    rng = np.random.default_rng(7)
    a, b = codes(rng, m, k), codes(rng, n, k)
    sa, sb = scales(rng, m, 1), scales(rng, up(n, 128), 1)
    y = ctx.gemm_fp8(a, sa, b, sb)
    ctx.check_device()
    assert y.numel() * 2 > 1 << 32
    for rows in (slice(0, 40), slice(32700, 32800), slice(m - 50, m)):
        check_product(y[rows], *product(a[rows], sa[rows], b, sb), k)
    got, scale = ctx.quantize_fp8(y)
    for rows in (slice(0, 3), slice(m - 3, m)):
        want, want_scale = quantise(y[rows], 1, E4)
        assert torch.equal(scale[rows].cpu(), want_scale)
        same_codes(got[rows], want)
    del got, scale
    w = torch.full((2, 2), 0.5, device="cuda")
    out = ctx.combine_experts(y, w, torch.tensor([[0, m - 1], [m - 1, m - 2]], dtype=torch.int32, device="cuda"), out_dtype=torch.float32)
    assert torch.equal(out[0], 0.5 * y[0].float() + 0.5 * y[m - 1].float()) and torch.equal(out[1], 0.5 * y[m - 1].float() + 0.5 * y[m - 2].float())


@pytest.mark.parametrize("m", [40, 500])
def test_two_streams_at_once(ctx, m):
    rng = np.random.default_rng(m)
    a, b = codes(rng, m, 1024), codes(rng, 600, 1024)
    sa, sb = scales(rng, m, 8), scales(rng, 5, 8)
    want = ctx.gemm_fp8(a, sa, b, sb)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        got = []
        for s in streams:
            with torch.cuda.stream(s):
                got.append(ctx.gemm_fp8(a, sa, b, sb))
        torch.cuda.synchronize()
        assert all(torch.equal(g, want) for g in got)
