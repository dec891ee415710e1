"""What the calls of the 8-bit and experts' layers refuse, and what the binding does not pass on (no GPU needed: nothing is
launched by a call that returns an error, and the arguments are looked at before the context is)."""
import ctypes as C

import pytest
import torch

import paper_1904_02205_b200.binding as B

P = 1 << 20      # an address that nothing reads


def _ctx():
    return C.cast(C.create_string_buffer(1 << 16), C.c_void_p)


def _quantize(x=P, codes=P, scales=P, **f):
    d = dict(in_dtype=B.PSB_DT_BF16, code_dtype=B.PSB_DT_E4M3, rows=4, cols=300, block_rows=1)
    d.update(f)
    return B.load_library().psb_quantize_fp8(_ctx(), x, C.byref(B.psb_quantize_desc(**d)), codes, scales, None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(codes=None), dict(scales=None), dict(x=P + 1), dict(scales=P + 2), dict(rows=0), dict(cols=0),
                                 dict(block_rows=0), dict(block_rows=64), dict(in_dtype=B.PSB_DT_U8), dict(in_dtype=B.PSB_DT_E4M3),
                                 dict(code_dtype=B.PSB_DT_BF16), dict(reserved=1), dict(x_stride=299), dict(code_stride=299),
                                 dict(scale_stride=2), dict(x_stride=1 << 40)])
def test_quantize_refuses(bad):
    assert _quantize(**bad) == B.PSB_ERR_INVALID_ARG


def test_quantize_too_large():
    assert _quantize(rows=1 << 31) == B.PSB_ERR_UNSUPPORTED


_GEMM = dict(a_dtype=B.PSB_DT_E4M3, b_dtype=B.PSB_DT_E5M2, out_dtype=B.PSB_DT_F32, m=5, n=7, k=160)


def _gemm(a=P, sa=P, b=P, sb=P, out=P, **f):
    return B.load_library().psb_gemm_fp8(_ctx(), a, sa, b, sb, out, C.byref(B.psb_gemm_fp8_desc(**dict(_GEMM, **f))), None)


_BAD_GEMM = [dict(a=None), dict(sa=None), dict(b=None), dict(sb=None), dict(out=None), dict(a=P + 8), dict(b=P + 4), dict(sa=P + 2), dict(out=P + 2),
             dict(m=0), dict(n=0), dict(k=0), dict(a_dtype=B.PSB_DT_U8), dict(b_dtype=B.PSB_DT_F32), dict(out_dtype=B.PSB_DT_E4M3), dict(relu=2),
             dict(reserved=1), dict(a_stride=152), dict(b_stride=168), dict(k=161), dict(a_scale_stride=1), dict(b_scale_stride=1),
             dict(out_stride=6), dict(bias_dev=P + 1)]


@pytest.mark.parametrize("bad", _BAD_GEMM)
def test_gemm_refuses(bad):
    assert _gemm(**bad) == B.PSB_ERR_INVALID_ARG


def test_gemm_too_large():
    assert _gemm(m=1 << 31) == B.PSB_ERR_UNSUPPORTED


def _experts(a=P, sa=P, b=P, sb=P, out=P, offsets=P, order=P, experts=3, rows=9, bes=0, bses=0, **f):
    d = B.psb_gemm_fp8_experts_desc(B.psb_gemm_fp8_desc(**dict(_GEMM, **f)), experts, rows, bes, bses)
    return B.load_library().psb_gemm_fp8_experts(_ctx(), a, sa, b, sb, offsets, order, out, C.byref(d), None)


@pytest.mark.parametrize("bad", _BAD_GEMM + [dict(offsets=None), dict(offsets=P + 2), dict(order=P + 1), dict(experts=0), dict(rows=0),
                                             dict(order=None), dict(bes=160 * 7 + 8), dict(bes=160 * 6), dict(bses=1)])
def test_experts_refuse(bad):
    assert _experts(**bad) == B.PSB_ERR_INVALID_ARG


def test_too_many_experts():
    assert _experts(experts=1025) == B.PSB_ERR_UNSUPPORTED


def _route(logits=P, bias=P, mask=P, ids=P, weights=P, offsets=P, order=P, slot=P, **f):
    d = dict(in_dtype=B.PSB_DT_F32, score=B.PSB_SCORE_SOFTMAX, tokens=4, experts=24, top_k=3, groups=4, top_groups=2, group_best=2, renormalise=1,
             scaling=1.0)
    d.update(f)
    return B.load_library().psb_route_experts(_ctx(), logits, bias, mask, C.byref(B.psb_route_desc(**d)), ids, weights, offsets, order, slot, None)


@pytest.mark.parametrize("bad", [dict(logits=None), dict(ids=None), dict(weights=None), dict(order=None), dict(slot=None), dict(offsets=None),
                                 dict(logits=P + 2), dict(bias=P + 1), dict(ids=P + 1), dict(slot=P + 2), dict(tokens=0), dict(experts=0), dict(top_k=0),
                                 dict(groups=0), dict(groups=5), dict(top_groups=0), dict(top_groups=5), dict(group_best=0), dict(group_best=3),
                                 dict(top_k=13), dict(score=2), dict(renormalise=2), dict(in_dtype=B.PSB_DT_S8), dict(logit_stride=23)])
def test_route_refuses(bad):
    assert _route(**bad) == B.PSB_ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [dict(experts=1025, groups=1, top_groups=1), dict(experts=64, top_k=33, groups=1, top_groups=1),
                                 dict(tokens=1 << 30)])
def test_route_too_large(bad):
    assert _route(**bad) == B.PSB_ERR_UNSUPPORTED


def _combine(y=P, weights=P, slot=P, out=P, **f):
    d = dict(in_dtype=B.PSB_DT_F16, out_dtype=B.PSB_DT_F32, tokens=4, top_k=2, n=70, rows=8)
    d.update(f)
    return B.load_library().psb_combine_experts(_ctx(), y, weights, slot, C.byref(B.psb_combine_desc(**d)), out, None)


@pytest.mark.parametrize("bad", [dict(y=None), dict(weights=None), dict(slot=None), dict(out=None), dict(y=P + 1), dict(out=P + 2), dict(weights=P + 2),
                                 dict(slot=P + 1), dict(tokens=0), dict(top_k=0), dict(n=0), dict(rows=0), dict(in_dtype=B.PSB_DT_U8),
                                 dict(out_dtype=B.PSB_DT_E4M3), dict(y_stride=69), dict(out_stride=1)])
def test_combine_refuses(bad):
    assert _combine(**bad) == B.PSB_ERR_INVALID_ARG


def test_combine_too_many_choices():
    assert _combine(top_k=33) == B.PSB_ERR_UNSUPPORTED


class _Ctx:
    device, handle, lib = torch.device("cpu"), None, None


@pytest.mark.parametrize("shape_a,shape_sa,shape_b,shape_sb", [((4, 160), (4, 2), (8, 128), (1, 1)), ((4, 160), (4, 1), (8, 160), (1, 2)),
                                                               ((4, 160), (4, 2), (130, 160), (1, 2))])
def test_the_binding_compares_codes_and_scales(shape_a, shape_sa, shape_b, shape_sb):
    e4 = torch.float8_e4m3fn
    with pytest.raises(ValueError):
        B.Context.gemm_fp8(type("X", (_Ctx,), dict(_gemm_fp8_head=B.Context._gemm_fp8_head))(), torch.zeros(shape_a).to(e4), torch.ones(shape_sa),
                           torch.zeros(shape_b).to(e4), torch.ones(shape_sb))


def test_the_binding_wants_rows_in_one_piece():
    with pytest.raises(ValueError):
        B._rows(torch.zeros(4, 6).t())
    assert B._rows(torch.zeros(1, 100).expand(1, 100), 16) == 112 and B._rows(torch.zeros(3, 32)[:, :20]) == 32


def test_the_binding_refuses_tensors_of_another_device():
    with pytest.raises(ValueError):
        B.Context.quantize_fp8(type("X", (), dict(device=torch.device("cuda", 0)))(), torch.zeros(2, 2))


def test_the_binding_refuses_rows_on_top_of_one_another():
    """A stride of 0 means rows that follow one another to the library: an expanded tensor would be read beyond its end."""
    for t in (torch.zeros(1, 32).expand(4, 32), torch.zeros(1, 1).expand(4, 1), torch.zeros(2, 1, 16).expand(2, 3, 16)):
        with pytest.raises(ValueError):
            B._rows(t)


@pytest.mark.parametrize("which", ["b", "b_scale"])
def test_the_binding_refuses_one_filter_for_all_experts(which):
    e4 = torch.float8_e4m3fn
    b, sb = torch.zeros(3, 8, 160).to(e4), torch.ones(3, 1, 2)
    if which == "b":
        b = b[:1].expand(3, 8, 160)
    else:
        sb = sb[:1].expand(3, 1, 2)
    with pytest.raises(ValueError):
        B.Context.gemm_fp8_experts(type("X", (_Ctx,), dict(_gemm_fp8_head=B.Context._gemm_fp8_head))(), torch.zeros(4, 160).to(e4), torch.ones(4, 2),
                                   b, sb, torch.zeros(4, dtype=torch.int32))


@pytest.mark.parametrize("block_rows", [0, 64])
def test_the_library_sees_other_blocks_than_it_has(block_rows):
    class Seen(Exception):
        pass

    def call(*args):
        raise Seen(B.psb_quantize_desc.from_buffer_copy(args[2]).block_rows)
    lib = type("L", (), dict(packed_quantize_fp8=staticmethod(call)))
    with pytest.raises(Seen) as e:
        B.Context.quantize_fp8(type("X", (_Ctx,), dict(lib=lib))(), torch.zeros(2, 200), block_rows=block_rows, stream=type("S", (), dict(cuda_stream=0)))
    assert e.value.args[0] == block_rows


class _Passed(Exception):
    """The binding handed its arguments on."""


def _stand_in(device="cpu"):
    """A context whose library only says that it was called, with the arguments."""
    def call(*args):
        raise _Passed(*args)
    names = ("quantize_fp8", "gemm_fp8", "gemm_fp8_experts", "route_experts", "combine_experts")
    ctx = type("X", (), dict(_gemm_fp8_head=B.Context._gemm_fp8_head))()
    ctx.device, ctx.handle = torch.device(device), None
    ctx.lib = type("L", (), {"packed_" + n: staticmethod(call) for n in names})
    return ctx


_STREAM = type("S", (), dict(cuda_stream=0))


def _product_of_experts(bias, experts=3, n=8, k=160, **how):
    e4 = torch.float8_e4m3fn
    return B.Context.gemm_fp8_experts(_stand_in(), torch.zeros(4, k).to(e4), torch.ones(4, 2), torch.zeros(experts, n, k).to(e4),
                                      torch.ones(experts, 1, 2), torch.zeros(experts + 1, dtype=torch.int32), bias=bias, stream=_STREAM, **how)


@pytest.mark.parametrize("shape", [(1, 8), (2, 8), (0, 8), (4, 8), (3, 1), (8,), (1, 3, 8)])
def test_the_binding_refuses_biases_of_other_experts(shape):
    """The kernels read the bias of expert e at e * n: fewer rows than experts would be read past their end."""
    with pytest.raises(ValueError):
        _product_of_experts(torch.zeros(shape))


def test_the_binding_passes_a_bias_for_each_expert():
    with pytest.raises(_Passed):
        _product_of_experts(torch.zeros(3, 8))


@pytest.mark.parametrize("shape", [(1, 8), (7,), (9,), (1,), (0,)])
def test_the_binding_refuses_other_biases_of_one_filter(shape):
    e4 = torch.float8_e4m3fn
    with pytest.raises(ValueError):
        B.Context.gemm_fp8(_stand_in(), torch.zeros(4, 160).to(e4), torch.ones(4, 2), torch.zeros(8, 160).to(e4), torch.ones(1, 2),
                           bias=torch.zeros(shape), stream=_STREAM)


def _meta(*shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="meta")


_MANY = (1 << 32) + 5


@pytest.mark.parametrize("call", [
    lambda c: B.Context.quantize_fp8(c, _meta(_MANY, 1), stream=_STREAM),
    lambda c: B.Context.quantize_fp8(c, _meta(1, _MANY), stream=_STREAM),
    lambda c: B.Context.quantize_fp8(c, _meta(4, 4), block_rows=_MANY, stream=_STREAM),
    lambda c: B.Context.gemm_fp8(c, _meta(_MANY, 16, dtype=torch.float8_e4m3fn), _meta(_MANY, 1), _meta(4, 16, dtype=torch.float8_e4m3fn), _meta(1, 1),
                                 stream=_STREAM),
    lambda c: B.Context.gemm_fp8_experts(c, _meta(4, 16, dtype=torch.float8_e4m3fn), _meta(4, 1), _meta(2, 4, 16, dtype=torch.float8_e4m3fn),
                                         _meta(2, 1, 1), _meta(3, dtype=torch.int32), order=_meta(_MANY, dtype=torch.int32), stream=_STREAM),
    lambda c: B.Context.route_experts(c, _meta(_MANY, 4), 1, stream=_STREAM),
    lambda c: B.Context.route_experts(c, _meta(4, 4), 1, groups=(1 << 32) + 1, stream=_STREAM),
    lambda c: B.Context.route_experts(c, _meta(4, 4), 1, top_groups=1 - (1 << 32), stream=_STREAM),
    lambda c: B.Context.combine_experts(c, _meta(_MANY, 4), _meta(4, 2), _meta(4, 2, dtype=torch.int32), stream=_STREAM),
    lambda c: B.Context.combine_experts(c, _meta(8, 1), _meta(_MANY, 1), _meta(_MANY, 1, dtype=torch.int32), stream=_STREAM)])
def test_the_binding_refuses_sizes_that_do_not_fit_their_field(call):
    """2^32 + 5 rows are not five."""
    with pytest.raises(ValueError):
        call(_stand_in("meta"))


def test_factors_beyond_fp32_become_infinities():
    seen = []
    ctx = _stand_in()
    ctx.lib.packed_route_experts = staticmethod(lambda *a: seen.append(B.psb_route_desc.from_buffer_copy(a[4]).scaling) or 0)
    B.Context.route_experts(ctx, torch.zeros(2, 4), 1, scaling=1e39, stream=_STREAM)
    assert seen == [float("inf")]


@pytest.mark.parametrize("shape", [(3, 1, 2), (1, 1, 2), (0, 1, 2), (2,)])
def test_the_binding_refuses_scales_of_other_filters(shape):
    """One filter has one matrix of scales: of several, the first alone would count."""
    e4 = torch.float8_e4m3fn
    with pytest.raises(ValueError):
        B.Context.gemm_fp8(_stand_in(), torch.zeros(4, 160).to(e4), torch.ones(4, 2), torch.zeros(8, 160).to(e4), torch.ones(shape), stream=_STREAM)


@pytest.mark.parametrize("shape", [(2, 1, 2), (0, 1, 2), (4, 1, 2), (3, 2, 2)])
def test_the_binding_refuses_scales_of_other_experts(shape):
    e4 = torch.float8_e4m3fn
    with pytest.raises(ValueError):
        B.Context.gemm_fp8_experts(_stand_in(), torch.zeros(4, 160).to(e4), torch.ones(4, 2), torch.zeros(3, 8, 160).to(e4), torch.ones(shape),
                                   torch.zeros(4, dtype=torch.int32), stream=_STREAM)
