"""Products over long reduction axes: more blocks than are handed over together within one tile, in each of the kernels."""
import numpy as np
import pytest
import torch

from fp8_testlib import check_product, codes, product, scales, up

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ctx():
    import paper_1904_02205_b200 as psb

    c = psb.Context(0)
    yield c
    c.check_device()
    c.close()


# pairs of SMs, single SMs, and few rows with and without a cut reduction axis
@pytest.mark.parametrize("m,n,k", [(2999, 2507, 2100), (600, 700, 2100), (9, 9600, 2100), (30, 9600, 2100), (100, 9601, 2100), (30, 520, 9000), (3, 260, 16500)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_product(ctx, m, n, k, out):
    rng = np.random.default_rng(m + n + k)
    a, b = codes(rng, m, k), codes(rng, n, k)
    sa, sb = scales(rng, m, up(k, 128)), scales(rng, up(n, 128), up(k, 128))
    got = ctx.gemm_fp8(a, sa, b, sb, out_dtype=DT[out])
    ctx.check_device()
    check_product(got, *product(a, sa, b, sb), k)


@pytest.mark.parametrize("experts,rows,n,k", [(2, 6000, 2600, 2100), (64, 256, 384, 2048), (64, 1024, 300, 2100), (5, 900, 270, 2100)])
@pytest.mark.parametrize("gather", [True, False])
def test_products_of_experts(ctx, experts, rows, n, k, gather):
    rng = np.random.default_rng(rows + k)
    share = rng.dirichlet(np.ones(experts))
    offsets = np.concatenate([[0], np.cumsum(rng.multinomial(rows, share))]).astype(np.int32)
    a, b = codes(rng, rows, k), codes(rng, n, k, batch=experts)
    sa, sb = scales(rng, rows, up(k, 128)), scales(rng, experts, up(n, 128), up(k, 128))
    bias = torch.from_numpy(rng.normal(0, 30, size=(experts, n)).astype(np.float32)).cuda()
    order = rng.permutation(rows).astype(np.int32) if gather else np.arange(rows, dtype=np.int32)
    got = ctx.gemm_fp8_experts(a, sa, b, sb, torch.from_numpy(offsets).cuda(), order=torch.from_numpy(order).cuda() if gather else None, bias=bias,
                               relu=True, out_dtype=torch.float32)
    ctx.check_device()
    for e in range(experts):
        lo, hi = int(offsets[e]), int(offsets[e + 1])
        if hi > lo:
            at = torch.from_numpy(order[lo:hi].astype(np.int64)).cuda()
            x = a.view(torch.uint8)[at].view(a.dtype)
            check_product(got[lo:hi], *product(x, sa[at], b[e], sb[e], bias[e], True), k)


@pytest.mark.parametrize("m,n", [(3000, 2500), (30, 9600), (700, 800)])
def test_the_same_bits_on_every_call_and_on_two_streams(ctx, m, n):
    rng = np.random.default_rng(m)
    a, b = codes(rng, m, 2048), codes(rng, n, 2048)
    sa, sb = scales(rng, m, 16), scales(rng, up(n, 128), 16)
    want = ctx.gemm_fp8(a, sa, b, sb, out_dtype=torch.float32)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for s in streams:
            with torch.cuda.stream(s):
                got.append(ctx.gemm_fp8(a, sa, b, sb, out_dtype=torch.float32))
        torch.cuda.synchronize()
        assert all(torch.equal(g, want) for g in got)
