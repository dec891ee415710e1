"""Routing, the experts' products and their weighted sum, each against its definition, and all of them as one layer."""
import math

import numpy as np
import pytest
import torch

from fp8_testlib import E4, check_product, codes, product, scales, sort_choices, up

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def ctx():
    import paper_1904_02205_b200 as psb

    c = psb.Context(0)
    yield c
    c.check_device()
    c.close()


# -- routing ----------------------------------------------------------------------------------------------------------------

def route(x, top_k, score, bias, groups, top_groups, group_best, renormalise, scaling, mask):
    """Row by row in 64 bits."""
    x = np.minimum(x.astype(np.float64), float(np.finfo(np.float32).max))
    T, E = x.shape
    ids, w = np.full((T, top_k), -1, np.int32), np.zeros((T, top_k))
    size = E // groups
    for t in range(T):
        if mask is not None and not mask[t]:
            continue
        on = ~np.isnan(x[t]) & (x[t] != -np.inf)
        with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
            if score == "softmax":
                p = np.where(on, np.exp(x[t] - (x[t][on].max() if on.any() else 0.0)), 0.0)
                p = p / p.sum() if on.any() else p
            else:
                p = np.where(on, 1.0 / (1.0 + np.exp(-x[t])), 0.0)
        select = (x[t] if groups == 1 else p) if bias is None else p + bias.astype(np.float64)
        left = [e for e in range(E) if on[e] and not np.isnan(select[e])]
        if groups > 1:
            strength = []
            for g in range(groups):
                best = sorted((select[e] for e in left if e // size == g), reverse=True)[:group_best]
                strength.append(sum(best) if best else -math.inf)
            empty = [not any(e // size == g for e in left) for g in range(groups)]
            stay = sorted(range(groups), key=lambda g: (empty[g], -strength[g], g))[:top_groups]
            left = [e for e in left if e // size in stay]
        best = sorted(left, key=lambda e: (-select[e], e))[:top_k]
        if not best:
            continue
        ids[t, :len(best)] = best
        if renormalise:
            top = x[t][best].max()
            if score == "softmax":
                s = np.exp(x[t][best] - top)
            else:       # ratios of sigmoids without underflow
                s = np.exp(np.minimum(x[t][best], 0) - min(top, 0)) / (1 + np.exp(-np.abs(x[t][best])))
            s = s / s.sum()
        else:
            s = p[best]
        w[t, :len(best)] = s * scaling
    return ids, w


def check_route(ctx, x, top_k, score="softmax", bias=None, groups=1, top_groups=1, group_best=1, renormalise=True, scaling=1.0, mask=None,
                dtype="f32"):
    t = torch.from_numpy(x).cuda().to(DT[dtype])
    got = ctx.route_experts(t, top_k, score=score, bias=None if bias is None else torch.from_numpy(bias).cuda(), groups=groups, top_groups=top_groups,
                            group_best=group_best, renormalise=renormalise, scaling=scaling,
                            token_mask=None if mask is None else torch.from_numpy(mask).cuda())
    ctx.check_device()
    ids, w = route(t.float().cpu().numpy(), top_k, score, bias, groups, top_groups, group_best, renormalise, scaling, mask)
    assert np.array_equal(got["ids"].cpu().numpy(), ids)
    # weights: exp is good to 2 ulp, its argument to half a one (2^-24 times at most 104), sums of up to 1024 terms to 10 + 32
    # roundings, quotient and product to one each: below 128 ulp of 2^-24; below the normal range, steps of 2^-149
    assert np.allclose(got["weights"].cpu().numpy(), w, rtol=128 * 2.0 ** -24, atol=2.0 ** -126 * abs(scaling))
    offsets, order, slot = sort_choices(ids, x.shape[1])
    assert np.array_equal(got["offsets"].cpu().numpy(), offsets)
    assert np.array_equal(got["order"].cpu().numpy(), order)
    assert np.array_equal(got["slot"].cpu().numpy(), slot)
    return got


@pytest.mark.parametrize("tokens,experts,top_k", [(1, 1, 1), (1, 8, 2), (3, 7, 7), (16, 64, 6), (33, 60, 4), (100, 256, 8), (300, 100, 3), (40, 512, 10),
                                                  (9, 1000, 32), (5, 1024, 16), (2, 33, 32)])
@pytest.mark.parametrize("score,with_bias", [("softmax", False), ("sigmoid", False), ("softmax", True), ("sigmoid", True)])
def test_choices_weights_and_order(ctx, tokens, experts, top_k, score, with_bias):
    rng = np.random.default_rng(tokens + experts)
    x = rng.normal(0, 2, size=(tokens, experts)).astype(np.float32)
    bias = rng.normal(0, 0.2, size=experts).astype(np.float32) if with_bias else None
    check_route(ctx, x, top_k, score, bias, renormalise=experts % 2 == 0, scaling=2.5)


@pytest.mark.parametrize("experts,groups,top_groups,group_best,top_k", [(256, 8, 4, 2, 8), (64, 4, 1, 1, 6), (60, 5, 3, 2, 7), (96, 96, 9, 2, 9),
                                                                        (1024, 64, 40, 2, 8), (40, 2, 1, 2, 20), (128, 32, 31, 1, 5), (8, 8, 2, 2, 1)])
@pytest.mark.parametrize("score,with_bias", [("softmax", False), ("sigmoid", True)])
def test_groups(ctx, experts, groups, top_groups, group_best, top_k, score, with_bias):
    rng = np.random.default_rng(experts + groups)
    x = rng.normal(0, 1.5, size=(50, experts)).astype(np.float32)
    bias = rng.normal(0, 0.1, size=experts).astype(np.float32) if with_bias else None
    check_route(ctx, x, top_k, score, bias, groups, top_groups, group_best)


@pytest.mark.parametrize("experts", [256, 512, 1024])
@pytest.mark.parametrize("tokens", [3, 400])
def test_every_expert_a_group_of_its_own(ctx, experts, tokens):
    """The largest scratch of a block; rows of coarse logits, most of which are settled in 64 bits."""
    rng = np.random.default_rng(experts + tokens)
    x = (np.round(rng.normal(0, 1, size=(tokens, experts)) * 8) / 8).astype(np.float32)
    check_route(ctx, x, 8, "softmax", None, experts, 20, 2)
    check_route(ctx, x, 8, "sigmoid", (rng.integers(0, 3, size=experts) / 8).astype(np.float32), experts, 20, 1)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("groups", [1, 4])
def test_ties_go_to_the_lower_index(ctx, dtype, groups):
    rng = np.random.default_rng(8)
    x = np.round(rng.normal(0, 1, size=(200, 64)) * 4).astype(np.float32) / 4
    x[:3] = 0.0
    x[3, ::2] = -0.0
    check_route(ctx, x, 6, "softmax", None, groups, 2 if groups > 1 else 1, 2, dtype=dtype)
    check_route(ctx, x, 6, "sigmoid", np.zeros(64, np.float32), groups, 2 if groups > 1 else 1, 2, dtype=dtype)
    check_route(ctx, x, 6, "sigmoid", (rng.integers(0, 3, size=64) / 8).astype(np.float32), groups, 2 if groups > 1 else 1, 1, dtype=dtype)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups", [1, 4])
def test_select_values_that_fp32_cannot_tell_apart(ctx, score, groups):
    """The bias makes up for the score, so that all select values of a row are alike up to the rounding of the bias."""
    rng = np.random.default_rng(9)
    x = np.tile(rng.normal(0, 1, size=(1, 48)).astype(np.float32), (20, 1))
    x64 = x[0].astype(np.float64)
    p = np.exp(x64) / np.exp(x64).sum() if score == "softmax" else 1 / (1 + np.exp(-x64))
    bias = (0.5 - p).astype(np.float32)
    x[1:] += (rng.integers(-2, 3, size=(19, 48)) * 2.0 ** -24).astype(np.float32)
    check_route(ctx, x, 8, score, bias, groups, 2 if groups > 1 else 1, 2)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("groups", [1, 4])
def test_rows_whose_mask_leaves_little_or_nothing(ctx, score, with_bias, groups):
    rng = np.random.default_rng(10)
    low, inf, nan = float(np.finfo(np.float32).min), np.inf, np.nan
    x = rng.normal(0, 1, size=(12, 24)).astype(np.float32)
    x[0] = -inf
    x[1] = nan
    x[2] = low
    x[3, 1:] = -inf
    x[4, :20] = -inf
    x[5, 3], x[5, 9] = inf, inf
    x[6, 2], x[6, 3] = nan, low
    x[7] = -200.0 - np.arange(24)
    x[8] = 200.0 + np.arange(24)
    x[9, :] = low
    x[9, 7] = 1.0
    x[10, 12:] = nan
    bias = rng.normal(0, 0.3, size=24).astype(np.float32) if with_bias else None
    for renormalise in (True, False):
        check_route(ctx, x, 5, score, bias, groups, 2 if groups > 1 else 1, 2, renormalise)
    mask = np.array([1, 0, 1, 1, 1, 0, 1, 0, 1, 1, 1, 0], np.uint8)
    x[11] = nan
    check_route(ctx, x, 5, score, bias, groups, 2 if groups > 1 else 1, 2, mask=mask)
    check_route(ctx, x, 5, score, bias, groups, 2 if groups > 1 else 1, 2, mask=np.zeros(12, np.uint8))


@pytest.mark.parametrize("tokens", [1, 31, 32, 33, 64, 65, 149, 4736, 4737, 9000])
def test_order_over_many_blocks(ctx, tokens):
    rng = np.random.default_rng(tokens)
    x = rng.normal(0, 1, size=(tokens, 16)).astype(np.float32)
    x[:, 3] += 3.0
    check_route(ctx, x, 2, mask=(rng.random(tokens) < 0.8).astype(np.uint8))


def test_order_of_very_many_rows(ctx):
    """Blocks of the largest size; the order against a stable sort."""
    T, E, k = 160000, 12, 2
    x = torch.randn(T, E, device="cuda")
    got = ctx.route_experts(x, k)
    ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k]
    assert torch.equal(got["ids"].long(), ids)
    by = torch.sort(ids.reshape(-1), stable=True).indices
    assert torch.equal(got["order"].long(), by // k)
    assert torch.equal(got["slot"].reshape(-1).long()[by], torch.arange(T * k, device="cuda"))
    assert torch.equal(got["offsets"][1:].long(), torch.bincount(ids.reshape(-1), minlength=E).cumsum(0))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,top_k,groups,group_best", [(48, 3, 1, 1), (64, 30, 1, 1), (64, 31, 1, 1), (256, 8, 8, 2), (64, 8, 4, 1), (512, 7, 1, 1)])
def test_rows_of_pairs_that_are_nearly_equal(ctx, score, experts, top_k, groups, group_best):
    """Rows that differ from one another by less than fp32 resolves, under a bias that makes them flat; and without one."""
    rng = np.random.default_rng(experts + top_k)
    x0 = rng.normal(0, 1, size=experts)
    p = np.exp(x0.astype(np.float32).astype(np.float64))
    p = p / p.sum() if score == "softmax" else p / (1 + p)
    bias = (0.5 - p).astype(np.float32)
    for step in (1e-7, 1e-6, 1e-4):
        x = (x0[None] + step * rng.normal(size=(64, experts))).astype(np.float32)
        check_route(ctx, x, top_k, score, bias, groups, max(1, groups // 2), group_best)
        y = np.sort(x, axis=1)
        y[:, 1::2] = np.nextafter(y[:, ::2], np.inf)
        check_route(ctx, y, top_k, score, None, groups, max(1, groups // 2), group_best)


def test_strided_logits_and_no_order(ctx):
    rng = np.random.default_rng(11)
    x = torch.from_numpy(rng.normal(size=(50, 70)).astype(np.float32)).cuda()
    a, b = ctx.route_experts(x[:, 3:67], 4), ctx.route_experts(x[:, 3:67].contiguous(), 4, sort=False)
    assert sorted(b) == ["ids", "weights"] and torch.equal(a["ids"], b["ids"]) and torch.equal(a["weights"], b["weights"])


# -- experts' products ----------------------------------------------------------------------------------------------------

def runs(rng, experts, rows, skew=1.0):
    """offsets of `rows` rows dealt out unevenly, some experts without any."""
    share = rng.exponential(size=experts) ** skew
    share[rng.random(experts) < 0.3] = 0.0
    if share.sum() == 0:
        share[experts // 2] = 1.0
    cut = np.floor(np.cumsum(share / share.sum()) * rows + 0.5).astype(np.int32)
    return np.concatenate([[0], cut]).astype(np.int32)


def check_experts(ctx, a, sa, b, sb, offsets, order, k, out, fill, **how):
    got = ctx.gemm_fp8_experts(a, sa, b, sb, torch.from_numpy(offsets).cuda(), order=None if order is None else torch.from_numpy(order).cuda(),
                               out=out, **how)
    ctx.check_device()
    bias = how.get("bias")
    for e in range(b.shape[0]):
        lo, hi = int(offsets[e]), int(offsets[e + 1])
        if hi > lo:
            rows = torch.arange(lo, hi) if order is None else torch.from_numpy(order[lo:hi].astype(np.int64))
            pick = a.view(torch.uint8)[rows.cuda()].view(a.dtype)
            want, size = product(pick, sa[rows.cuda()], b[e], sb[e], None if bias is None else bias[e], how.get("relu", False))
            check_product(got[lo:hi], want, size, k)
    assert (out[int(offsets[-1]):] == fill).all()
    return got


@pytest.mark.parametrize("experts,rows,n,k", [(1, 1, 1, 1), (4, 3, 128, 128), (8, 40, 200, 300), (3, 300, 130, 256), (16, 100, 256, 1000), (64, 256, 384, 512),
                                              (5, 1500, 520, 640), (2, 700, 1000, 130), (1024, 500, 64, 128), (7, 2000, 256, 2048), (20, 800, 2000, 300), (2, 6000, 2600, 400)])
@pytest.mark.parametrize("gather", [True, False])
def test_products_of_experts(ctx, experts, rows, n, k, gather):
    rng = np.random.default_rng(experts + rows)
    tokens = max(1, rows // 2) if gather else rows + 3
    a, b = codes(rng, tokens, k), codes(rng, n, k, batch=experts)
    sa, sb = scales(rng, tokens, up(k, 128)), scales(rng, experts, up(n, 128), up(k, 128))
    offsets = runs(rng, experts, rows)
    order = rng.integers(0, tokens, size=rows + 5).astype(np.int32) if gather else None
    if gather:
        order[rows:] = -1
    out = torch.full((rows + 5 if gather else tokens, n), -7.0, dtype=torch.bfloat16, device="cuda")
    check_experts(ctx, a, sa, b, sb, offsets, order, k, out, -7.0)


@pytest.mark.parametrize("rows", [6, 200, 900])
def test_products_of_experts_bias_relu_strides(ctx, rows):
    rng = np.random.default_rng(rows)
    experts, n, k, tokens = 6, 270, 400, 50
    a, sa = codes(rng, tokens, k, pitch=448), scales(rng, tokens, 6)[:, 1:5]
    store = codes(rng, 300, k, pitch=432, batch=experts)
    b, sb = store[:, 10:10 + n], scales(rng, experts, 5, 4)[:, 1:4]
    bias = torch.from_numpy(rng.normal(0, 30, size=(experts, n)).astype(np.float32)).cuda()
    wide = torch.full((rows, n + 30), -7.0, device="cuda")
    check_experts(ctx, a, sa, b, sb, runs(rng, experts, rows), rng.integers(0, tokens, size=rows).astype(np.int32), k, wide[:, 9:9 + n], -7.0,
                  bias=bias, relu=True)
    assert (wide[:, :9] == -7.0).all() and (wide[:, 9 + n:] == -7.0).all()


@pytest.mark.parametrize("rows", [20, 400])
def test_no_rows_at_all_and_all_rows_of_one_expert(ctx, rows):
    rng = np.random.default_rng(rows)
    experts, n, k = 5, 140, 200
    a, b = codes(rng, rows, k), codes(rng, n, k, batch=experts)
    sa, sb = scales(rng, rows, 2), scales(rng, experts, 2, 2)
    for offsets in ([0] * 6, [0, 0, 0, rows, rows, rows], [0, 0, 0, 0, 0, rows], [0, rows, rows, rows, rows, rows], [0, 0, 1, 2, 3, 4]):
        out = torch.full((rows, n), -7.0, dtype=torch.float16, device="cuda")
        check_experts(ctx, a, sa, b, sb, np.array(offsets, np.int32), None, k, out, -7.0)


@pytest.mark.parametrize("rows", [12, 300])
def test_bad_offsets_and_bad_rows_are_reported(ctx, rows):
    """The kernels clamp what they read, so that nothing outside the tensors is touched."""
    import paper_1904_02205_b200 as psb

    rng = np.random.default_rng(rows)
    experts, n, k = 4, 130, 256
    a, b = codes(rng, rows, k), codes(rng, n, k, batch=experts)
    sa, sb = scales(rng, rows, 2), scales(rng, experts, 2, 2)
    t = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    good = t([0, 2, 2, rows // 2, rows])
    guard = torch.full((rows + 64, n), -7.0, device="cuda")
    out = guard[32:32 + rows]
    for offsets in (t([0, 2, 2, rows // 2, rows + 1]), t([-1, 2, 2, rows // 2, rows]), t([0, 6, 2, rows // 2, rows]), t([0, 2 ** 31 - 1, 2, 5, 6])):
        ctx.gemm_fp8_experts(a, sa, b, sb, offsets, out=out)
        assert ctx.device_status() == psb.PSB_ERR_RANGE
    for bad in (rows, -1, 2 ** 31 - 1, -2 ** 31):
        order = torch.arange(rows, dtype=torch.int32, device="cuda")
        order[rows - 1] = bad
        ctx.gemm_fp8_experts(a, sa, b, sb, good, order=order, out=out)
        assert ctx.device_status() == psb.PSB_ERR_RANGE
    assert (guard[:32] == -7.0).all() and (guard[32 + rows:] == -7.0).all()


# -- weighted sum ---------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("tokens,top_k,n", [(1, 1, 1), (1, 8, 4096), (7, 3, 130), (50, 9, 1000), (33, 32, 72), (600, 2, 264)])
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f32", "f16"), ("f16", "f32")])
def test_weighted_sum(ctx, tokens, top_k, n, dtype, out):
    rng = np.random.default_rng(tokens + n)
    rows = tokens * top_k
    y = torch.from_numpy(rng.normal(size=(rows, n + 8)).astype(np.float32)).cuda().to(DT[dtype])[:, :n]
    slot = rng.permutation(rows).reshape(tokens, top_k).astype(np.int32)
    slot[rng.random(slot.shape) < 0.2] = -1
    if tokens > 3:
        slot[2] = -1
    w = rng.random((tokens, top_k)).astype(np.float32)
    got = ctx.combine_experts(y, torch.from_numpy(w).cuda(), torch.from_numpy(slot).cuda(), out_dtype=DT[out])
    ctx.check_device()
    full = np.where(slot[:, :, None] >= 0, y.double().cpu().numpy()[np.maximum(slot, 0)], 0.0) * w[:, :, None].astype(np.float64)
    want, size = full.sum(1), np.abs(full).sum(1)
    half = torch.finfo(DT[out]).eps / 2
    # an fma a choice, each off by at most half a step of fp32 of the sum of magnitudes; then half a step of the output (subnormals: its least step)
    tol = size * (top_k + 1) * 2.0 ** -24 + np.abs(want) * half * (1 + 2.0 ** -10) + torch.finfo(DT[out]).smallest_normal * torch.finfo(DT[out]).eps
    assert (np.abs(got.double().cpu().numpy() - want) <= tol).all()


def test_weighted_sum_strides_and_bad_slots(ctx):
    import paper_1904_02205_b200 as psb

    y = torch.arange(40.0, device="cuda").reshape(4, 10)[:, 1:8]
    store = torch.full((2, 12), -7.0, device="cuda")
    w = torch.ones(2, 3, device="cuda")
    ctx.combine_experts(y, w, torch.tensor([[0, 3, -1], [1, -5, 2]], dtype=torch.int32, device="cuda"), out=store[:, 2:9])
    assert torch.equal(store[:, 2:9], torch.stack([y[0] + y[3], y[1] + y[2]])) and (store[:, :2] == -7).all() and (store[:, 9:] == -7).all()
    assert ctx.device_status() == 0
    got = ctx.combine_experts(y, w, torch.tensor([[0, 4, -1], [2 ** 31 - 1, 1, 2]], dtype=torch.int32, device="cuda"))
    assert ctx.device_status() == psb.PSB_ERR_RANGE
    assert torch.equal(got, torch.stack([y[0], y[1] + y[2]]))


# -- the layer ------------------------------------------------------------------------------------------------------------

def _layer(ctx, x, gate, w1, w2, top_k, mask, stream=None):
    """x [T, K] -> router -> relu(x w1) w2 of each chosen expert -> weighted sum."""
    r = ctx.route_experts(x.float() @ gate, top_k, score="sigmoid", token_mask=mask, stream=stream)
    h = ctx.gemm_fp8_experts(*ctx.quantize_fp8(x, stream=stream), *w1, r["offsets"], order=r["order"], relu=True, stream=stream)
    y = ctx.gemm_fp8_experts(*ctx.quantize_fp8(h, stream=stream), *w2, r["offsets"], stream=stream)
    return r, ctx.combine_experts(y, r["weights"], r["slot"], stream=stream)


def _parts(ctx, rng, T, E, K, H):
    t = lambda *s: torch.from_numpy(rng.normal(size=s).astype(np.float32)).cuda()
    x, gate = t(T, K).bfloat16(), t(K, E) / math.sqrt(K)
    f1, f2 = t(E, H, K) / math.sqrt(K), t(E, K, H) / math.sqrt(H)
    q = lambda f: tuple(torch.stack(v) for v in zip(*[tuple(p.view(torch.uint8) if p.dtype == E4 else p for p in ctx.quantize_fp8(w, block_rows=128)) for w in f]))
    w1, w2 = ((c.view(E4), s) for c, s in (q(f1), q(f2)))
    return x, gate, f1, f2, w1, w2


@pytest.mark.parametrize("T,E,top_k", [(1, 8, 2), (40, 8, 2), (300, 6, 3)])
def test_a_whole_layer_of_experts(ctx, T, E, top_k):
    rng = np.random.default_rng(T)
    K, H = 256, 384
    x, gate, f1, f2, w1, w2 = _parts(ctx, rng, T, E, K, H)
    mask = torch.ones(T, dtype=torch.uint8, device="cuda")
    if T > 1:
        mask[T - T // 5:] = 0
    r, got = _layer(ctx, x, gate, w1, w2, top_k, mask)
    ctx.check_device()
    p = torch.sigmoid((x.float() @ gate).double())
    ids = p.topk(top_k, dim=1).indices
    want = torch.zeros(T, K, dtype=torch.float64, device="cuda")
    for t in range(T):
        if mask[t]:
            w = p[t, ids[t]] / p[t, ids[t]].sum()
            for j in range(top_k):
                e = int(ids[t, j])
                want[t] += w[j] * (f2[e].double() @ torch.relu(f1[e].double() @ x[t].double()))
    assert (got[mask == 0] == 0).all()
    # four roundings to e4m3 (half a step 2^-4 each) of independent values: errors add like a random walk, so the 2-norm is off by
    # well below 4 * 2^-4; a row sent to a wrong expert or weighed wrongly is off by about its whole norm
    rel = (got.double() - want).norm(dim=1)[mask != 0] / want.norm(dim=1)[mask != 0]
    assert float(rel.max()) < 0.25


def test_a_captured_layer_follows_its_inputs(ctx):
    rng = np.random.default_rng(12)
    T, E, K, H, top_k = 50, 8, 256, 128, 2
    x, gate, _, _, w1, w2 = _parts(ctx, rng, T, E, K, H)
    mask = torch.ones(T, dtype=torch.uint8, device="cuda")
    _layer(ctx, x, gate, w1, w2, top_k, mask)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        x.float() @ gate                                    # (the library behind it sets itself up outside the capture)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        r, got = _layer(ctx, x, gate, w1, w2, top_k, mask)
    for i in range(4):
        x.copy_(torch.from_numpy(rng.normal(size=(T, K)).astype(np.float32)))
        mask.copy_(torch.from_numpy((rng.random(T) < 0.7).astype(np.uint8)))
        graph.replay()
        eager_r, eager = _layer(ctx, x, gate, w1, w2, top_k, mask)
        assert torch.equal(got, eager)
        for key in eager_r:
            assert torch.equal(r[key], eager_r[key])
    ctx.check_device()


def test_two_streams_route_at_once(ctx):
    x = [torch.randn(5000, 64, device="cuda") for _ in range(2)]
    want = [ctx.route_experts(v, 4) for v in x]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        got = []
        for v, s in zip(x, streams):
            with torch.cuda.stream(s):
                got.append(ctx.route_experts(v, 4))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            for key in w:
                assert torch.equal(g[key], w[key])


def test_two_captured_graphs_and_eager_calls_keep_their_scratch_apart(ctx):
    """Graphs captured on different streams, replayed at once beside eager calls: gathered rows and counts are their own."""
    rng = np.random.default_rng(13)
    E, K, H, top_k = 6, 256, 128, 2
    layers = []
    for T in (300, 700, 500):
        x, gate, _, _, w1, w2 = _parts(ctx, rng, T, E, K, H)
        mask = torch.ones(T, dtype=torch.uint8, device="cuda")
        layers.append((x, gate, w1, w2, top_k, mask))
    want = [_layer(ctx, *l)[1].clone() for l in layers]
    streams, graphs, got = [torch.cuda.Stream() for _ in range(2)], [], []
    for s, l in zip(streams, layers):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            l[0].float() @ l[1]
    torch.cuda.synchronize()
    for s, l in zip(streams, layers):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            got.append(_layer(ctx, *l)[1])
        graphs.append(g)
    for _ in range(10):
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        eager = _layer(ctx, *layers[2])[1]
        torch.cuda.synchronize()
        assert torch.equal(eager, want[2])
        for y, w in zip(got, want):
            assert torch.equal(y, w)
    ctx.check_device()


@pytest.mark.parametrize("experts,groups", [(64, 4), (60, 3), (512, 8)])
@pytest.mark.parametrize("top_k", [2, 3, 4])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_scores_that_are_equal_in_64_bits_go_by_the_index(ctx, experts, groups, top_k, score):
    """In groups the scores count, not the logits: those that 64 bits hold as 0 or as the same number are ties, whichever way a row's
    comparisons take."""
    rows = [{10: 0.0, 3: -900.0, 5: -800.0}, {10: 0.0, 3: -1e9, 5: -800.0, 30: -3.0}, {10: 0.0, 3: -720.0, 5: -710.0}, {10: 4.0, 3: 0.0, 5: 1e-20},
            {40: 2.0, 3: 1e-25, 5: -1e-25, 9: 1.0}, {10: 0.0, 41: -800.0, 5: -900.0}, {10: 0.0, 3: -3.4e38, 5: -1e30}, {3: -50.0, 5: -60.0, 7: -20.0},
            {10: 0.0, 3: -900.0, 5: -800.0, 44: -1000.0, 45: -1e5}, {10: 0.0, 3: 2.0 ** -24, 5: 2.0 ** -23},
            {10: 50.0, 3: 40.0, 5: 60.0, 41: 45.0}, {3: -1e-20, 5: 1e-20, 10: -1e-30, 41: 1e-19}]
    x = np.full((len(rows), experts), -np.inf, np.float32)
    for t, row in enumerate(rows):
        for e, v in row.items():
            x[t, e] = v
    for top_groups in (groups, groups - 1):
        check_route(ctx, x, top_k, score, None, groups, top_groups, 2)


@pytest.mark.parametrize("rows", [12, 64, 300, 4000])
@pytest.mark.parametrize("gather", [True, False])
def test_offsets_that_decrease_are_no_runs_at_all(ctx, rows, gather):
    """Runs that share rows could be more tiles than 32 bits count."""
    import paper_1904_02205_b200 as psb

    rng = np.random.default_rng(rows)
    experts, n, k = 40, 300, 1200
    a, b = codes(rng, rows, k), codes(rng, n, k, batch=experts)
    sa, sb = scales(rng, rows, up(k, 128)), scales(rng, experts, up(n, 128), up(k, 128))
    order = torch.arange(rows, dtype=torch.int32, device="cuda") if gather else None
    for late in (False, True):
        offsets = torch.full((experts + 1,), rows, dtype=torch.int32)
        offsets[0] = 0
        if late:
            offsets[-2] = 0
        else:
            offsets[2::2] = 0
            offsets[-1] = rows
        out = torch.full((rows, n), -5.0, device="cuda")
        ctx.gemm_fp8_experts(a, sa, b, sb, offsets.cuda(), order=order, out=out)
        assert ctx.device_status() == psb.PSB_ERR_RANGE
        assert (out == -5.0).all()
    assert ctx.device_status() == psb.PSB_OK


@pytest.mark.parametrize("experts,below", [(1024, 5.2), (1000, 7.0), (256, 4.0), (64, 2.6), (32, 2.4), (31, 9.0)])
@pytest.mark.parametrize("groups", [1, "all"])
def test_near_ties_beside_many_middling_scores(ctx, experts, below, groups):
    """Scores whose sum is far from the largest of them, which is where the sum's error is largest; the bias brings half of the row's
    select values within a few units of fp32 of one another."""
    rng = np.random.default_rng(experts)
    groups = 1 if groups == 1 else next(g for g in (8, 4, 2, 1) if experts % g == 0)
    x = np.full((60, experts), -below, np.float32) + rng.normal(0, 0.3, size=(60, experts)).astype(np.float32)
    x[np.arange(60), rng.integers(0, experts, size=60)] = 0.0
    x[1:] = x[0] + (rng.integers(-3, 4, size=(59, experts)) * 2.0 ** -22).astype(np.float32)
    x64 = x[0].astype(np.float64)
    p = np.exp(x64) / np.exp(x64).sum()
    bias = np.where(rng.random(experts) < 0.5, 0.75 - p, -0.5).astype(np.float32)
    check_route(ctx, x, min(8, experts), "softmax", bias, groups, max(1, groups // 2), 2)
