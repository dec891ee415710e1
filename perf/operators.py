"""Operators of language models next to the sampled layers: 8-bit floating point and experts.

Five kinds of case, each one call:

  quantize  ``Context.quantize_fp8``: codes in e4m3 with an fp32 scale for each block, 1 x 128 (activations) or
            128 x 128 (weights).  scale = max(largest magnitude / 448, 2^-126), code = round(x * (1 / scale)).
  gemm      ``Context.gemm_fp8``: y = act(sum over blocks of sa * sb * (a . b) + bias), rows of ``a`` against filters
            ``b`` stored [out][in]
  route     ``Context.route_experts``: scores of all experts, top-k of each row, and the rows sorted by expert
  experts   ``Context.gemm_fp8_experts``: rows sorted by expert, each run against the filter of its expert
  combine   ``Context.combine_experts``: the weighted sum of the chosen experts' rows for each row

Everything random is made on the GPU from the seed.
"""
import math

import torch

own = False

_QUANT = dict(kind="quantize", dtype="bf16", block_rows=1)
_GEMM = dict(kind="gemm", out="bf16", bias=False, relu=False)
_ROUTE = dict(kind="route", dtype="f32", score="softmax", bias=False, groups=1, top_groups=1, group_best=1, renormalise=True, scaling=1.0,
              padded=False)
_EXPERTS = dict(kind="experts", out="bf16", gather=True, relu=False, bias=False, padded=False)
_COMBINE = dict(kind="combine", dtype="bf16", padded=False)

_DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_TOP, _TINY = 448.0, 2.0 ** -126


def listed():
    return [
        # the hidden state of one new token on its way into an 8-bit layer: the smallest call, all latency
        dict(_QUANT, name="quantize_1x4096", rows=1, cols=4096),
        # a trained filter of odd size brought to 8 bits, one scale for each 128 x 128
        dict(_QUANT, name="quantize_1000x2040_filter", rows=1000, cols=2040, dtype="f32", block_rows=128),
        # the hidden states of long prompts
        dict(_QUANT, name="quantize_16384x4096", rows=16384, cols=4096),
        # one new token through a square layer: the filter is read once, nothing else counts
        dict(_GEMM, name="gemm_1x4096x4096", m=1, n=4096, k=4096),
        # the 1000-class head of the networks on a batch that fills no tile, real-valued logits
        dict(_GEMM, name="gemm_1500x1000x2048_logits", m=1500, n=1000, k=2048, out="f32", bias=True),
        # a wide layer over long prompts: bound by the tensor cores
        dict(_GEMM, name="gemm_8192x8192x8192_relu", m=8192, n=8192, k=8192, relu=True),
        # a few requests' tokens choose among 64 experts
        dict(_ROUTE, name="route_16_64_top6", tokens=16, experts=64, top_k=6, dtype="bf16"),
        # prompts over 256 experts: sigmoid scores, a bias that balances the load, four of eight groups, padded rows
        dict(_ROUTE, name="route_16384_256_top8_groups", tokens=16384, experts=256, top_k=8, score="sigmoid", bias=True, groups=8,
             top_groups=4, group_best=2, scaling=2.5, padded=True),
        # 32 requests, one token each, eight of 64 experts: about four rows an expert, every filter is read
        dict(_EXPERTS, name="experts_32_top8_of_64_2048x2048", tokens=32, top_k=8, experts=64, n=2048, k=2048, relu=True),
        # prompts, two of eight experts
        dict(_EXPERTS, name="experts_8192_top2_of_8_4096x4096", tokens=8192, top_k=2, experts=8, n=4096, k=4096, relu=True),
        # the chosen experts' rows of a few tokens
        dict(_COMBINE, name="combine_16_top6_2048", tokens=16, top_k=6, n=2048),
        # the same for prompts
        dict(_COMBINE, name="combine_8192_top8_4096", tokens=8192, top_k=8, n=4096),
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["quantize", "gemm", "gemm", "route", "experts", "experts", "combine"])
    if kind == "quantize":
        cols = _log(rng, 64, 8192)
        return dict(_QUANT, rows=_log(rng, 1, min(16384, 16384 * 4096 // cols)), cols=cols, dtype=rng.choice(["bf16", "f16", "f32"]),
                    block_rows=rng.choice([1, 1, 128]))
    if kind == "gemm":
        n, k = _log(rng, 64, 8192), _log(rng, 64, 8192)
        return dict(_GEMM, m=_log(rng, 1, 8192), n=n, k=k, out=rng.choice(["bf16", "bf16", "f16", "f32"]), bias=rng.random() < 0.3,
                    relu=rng.random() < 0.3)
    if kind == "route":
        groups = rng.choice([1, 1, 2, 4, 8])
        experts = groups * _log(rng, 8, 256 // groups)
        top_groups = rng.randint(1, groups)
        most = min(16, top_groups * (experts // groups))
        return dict(_ROUTE, tokens=_log(rng, 1, 16384), experts=experts, top_k=rng.randint(1, most), dtype=rng.choice(["f32", "bf16", "f16"]),
                    score=rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.5, groups=groups, top_groups=top_groups,
                    group_best=rng.choice([1, 2]), renormalise=rng.random() < 0.7, scaling=rng.choice([1.0, 2.5]), padded=rng.random() < 0.4)
    if kind == "experts":
        experts, top_k = rng.randint(2, 64), rng.choice([1, 2, 4, 6, 8])
        n, k = _log(rng, 128, 4096), _log(rng, 128, 4096)
        return dict(_EXPERTS, tokens=_log(rng, 1, 16384 // top_k), top_k=min(top_k, experts), experts=experts, n=n, k=k,
                    out=rng.choice(["bf16", "bf16", "f16", "f32"]), gather=rng.random() < 0.6, relu=rng.random() < 0.3,
                    bias=rng.random() < 0.3, padded=rng.random() < 0.3)
    top_k, n = rng.randint(1, 8), _log(rng, 64, 8192)
    return dict(_COMBINE, tokens=_log(rng, 1, min(8192, 8192 * 8 * 4096 // (top_k * n))), top_k=top_k, n=n,
                dtype=rng.choice(["bf16", "f16", "f32"]), padded=rng.random() < 0.4)


# -- inputs ------------------------------------------------------------------------------------------------------------------
def _rand(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _codes(gen, rows, cols, block_rows, count=None):
    """Codes and scales of normal values whose blocks differ in size; rows start every 16 bytes, as the copy engine wants them."""
    batch = () if count is None else (count,)
    pitch = -(-cols // 16) * 16
    blocks = batch + (-(-rows // block_rows), -(-cols // 128))
    scales = torch.exp(0.3 * _rand(gen, *blocks)) / (100.0 * (1.0 if block_rows == 1 else math.sqrt(cols)))
    store = torch.empty(batch + (rows, pitch), dtype=torch.float8_e4m3fn, device="cuda")
    x = torch.empty(rows, pitch, device="cuda")
    for part in (store if batch else [store]):
        part.copy_((x.normal_(generator=gen) * 100.0).clamp_(-_TOP, _TOP))
    return store[..., :cols], scales


def _real_tokens(case):
    """Rows in use of a padded batch."""
    return case["tokens"] - case["tokens"] // 5 if case["padded"] else case["tokens"]


def _choices(gen, case):
    """Experts chosen by uneven popularity, and the rows sorted by them: ids, offsets, order, slot (see route_experts)."""
    T, E, k = case["tokens"], case.get("experts", 64), case["top_k"]
    taste = _rand(gen, T, E) + 0.7 * _rand(gen, E)
    ids = taste.topk(k, dim=1).indices.to(torch.int32)
    ids[_real_tokens(case):] = -1
    return (ids,) + _sorted_rows(ids, E)


def _sorted_rows(ids, E):
    """offsets [E + 1], order [T * k] (the row behind each sorted place, -1 behind the last), slot [T, k] (the place of each choice)."""
    T, k = ids.shape
    flat = ids.reshape(-1).long()
    key = torch.where(flat < 0, torch.full_like(flat, E), flat)
    by = torch.sort(key, stable=True).indices
    counts = torch.zeros(E + 1, dtype=torch.int64, device=ids.device).scatter_add_(0, key, torch.ones_like(key))
    offsets = torch.cat([counts.new_zeros(1), counts[:E].cumsum(0)])
    place = torch.arange(T * k, device=ids.device)
    order = torch.where(place < offsets[E], by // k, -torch.ones_like(by))
    slot = torch.empty_like(by).scatter_(0, by, place)
    slot = torch.where(flat < 0, -torch.ones_like(slot), slot)
    return offsets.to(torch.int32), order.to(torch.int32), slot.reshape(T, k).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 1000003 + 17)
    s = dict(case=case)
    if case["kind"] == "quantize":
        # hidden states have a few channels that are many times larger than the rest
        size = torch.exp(0.6 * _rand(gen, case["cols"])) if case["block_rows"] == 1 else 0.02
        s["x"] = (_rand(gen, case["rows"], case["cols"]) * size).to(_DT[case["dtype"]])
    elif case["kind"] == "gemm":
        s["a"], s["a_scale"] = _codes(gen, case["m"], case["k"], 1)
        s["b"], s["b_scale"] = _codes(gen, case["n"], case["k"], 128)
        s["bias"] = _rand(gen, case["n"]) if case["bias"] else None
    elif case["kind"] == "route":
        T, E = case["tokens"], case["experts"]
        s["logits"] = (1.5 * _rand(gen, T, E) + 0.5 * _rand(gen, E)).to(_DT[case["dtype"]])
        s["bias"] = 0.1 * _rand(gen, E) if case["bias"] else None
        s["mask"] = (torch.arange(T, device="cuda") < _real_tokens(case)).to(torch.uint8) if case["padded"] else None
    elif case["kind"] == "experts":
        _, s["offsets"], s["order"], _ = _choices(gen, case)
        rows = case["tokens"] * case["top_k"]
        s["a"], s["a_scale"] = _codes(gen, case["tokens"] if case["gather"] else rows, case["k"], 1)
        s["b"], s["b_scale"] = _codes(gen, case["n"], case["k"], 128, count=case["experts"])
        s["bias"] = _rand(gen, case["experts"], case["n"]) if case["bias"] else None
        s["out"] = torch.zeros(rows, case["n"], dtype=_DT[case["out"]], device="cuda")
        s["most"] = int((s["offsets"][1:] - s["offsets"][:-1]).max().item())
    else:
        ids, _, _, s["slot"] = _choices(gen, case)
        w = torch.rand(case["tokens"], case["top_k"], generator=gen, device="cuda")
        s["weights"] = torch.where(ids < 0, torch.zeros_like(w), w / w.sum(1, keepdim=True))
        s["y"] = _rand(gen, case["tokens"] * case["top_k"], case["n"]).to(_DT[case["dtype"]])
    return s


# -- one pass ----------------------------------------------------------------------------------------------------------------
_state = {}


def _context():
    import paper_1904_02205_b200 as psb

    if "ctx" not in _state:
        _state["ctx"] = psb.Context(torch.cuda.current_device())
    return _state["ctx"]


def run(state):
    case = state["case"]
    return (_OWN if own else _PLAIN)[case["kind"]](case, state)


def _own_quantize(case, s):
    return _context().quantize_fp8(s["x"], block_rows=case["block_rows"])


def _own_gemm(case, s):
    return _context().gemm_fp8(s["a"], s["a_scale"], s["b"], s["b_scale"], bias=s["bias"], relu=case["relu"], out_dtype=_DT[case["out"]])


def _own_route(case, s):
    return _context().route_experts(s["logits"], case["top_k"], score=case["score"], bias=s["bias"], groups=case["groups"],
                                    top_groups=case["top_groups"], group_best=case["group_best"], renormalise=case["renormalise"],
                                    scaling=case["scaling"], token_mask=s["mask"])


def _own_experts(case, s):
    return _context().gemm_fp8_experts(s["a"], s["a_scale"], s["b"], s["b_scale"], s["offsets"], order=s["order"] if case["gather"] else None,
                                       bias=s["bias"], relu=case["relu"], out=s["out"])


def _own_combine(case, s):
    return _context().combine_experts(s["y"], s["weights"], s["slot"])


def _blocks(x, block_rows):
    """[R][C] as [R / block_rows][block_rows][C / 128][128], zeros behind the ends."""
    R, C = x.shape
    x = torch.nn.functional.pad(x, (0, -C % 128, 0, -R % block_rows))
    return x.reshape(x.shape[0] // block_rows, block_rows, x.shape[1] // 128, 128)


def _plain_quantize(case, s):
    R, C = s["x"].shape
    x = _blocks(s["x"].float(), case["block_rows"])
    scale = (x.abs().amax(dim=(1, 3)) / _TOP).clamp(min=_TINY)
    codes = (x * (1.0 / scale)[:, None, :, None]).clamp(-_TOP, _TOP).reshape(-1, x.shape[2] * 128)[:R, :C]
    return codes.to(torch.float8_e4m3fn), scale


def _real(codes, scales, block_rows):
    """The values that codes and scales stand for, in fp32."""
    wide = scales.repeat_interleave(128, dim=-1)[..., :codes.shape[-1]]
    if block_rows > 1:
        wide = wide.repeat_interleave(block_rows, dim=-2)[..., :codes.shape[-2], :]
    return codes.float() * wide


def _finish(y, bias, case):
    if bias is not None:
        y = y + bias
    return (y.clamp(min=0) if case["relu"] else y).to(_DT[case["out"]])


def _plain_gemm(case, s):
    y = _real(s["a"], s["a_scale"], 1) @ _real(s["b"], s["b_scale"], 128).t()
    return _finish(y, s["bias"], case)


def _plain_route(case, s):
    T, E, G = case["tokens"], case["experts"], case["groups"]
    x = s["logits"].double()
    score = torch.exp(x - x.amax(1, keepdim=True)) if case["score"] == "softmax" else 1.0 / (1.0 + torch.exp(-x))
    if case["score"] == "softmax":
        score = score / score.sum(1, keepdim=True)
    pick = score if s["bias"] is None else score + s["bias"].double()
    if G > 1:
        best = torch.sort(pick.reshape(T, G, E // G), dim=2, descending=True).values[:, :, :case["group_best"]].sum(2)
        kept = torch.sort(best, dim=1, descending=True, stable=True).indices[:, :case["top_groups"]]
        inside = torch.zeros(T, G, dtype=torch.bool, device=x.device).scatter_(1, kept, True).repeat_interleave(E // G, dim=1)
        pick = torch.where(inside, pick, torch.full_like(pick, -math.inf))
    ids = torch.sort(pick, dim=1, descending=True, stable=True).indices[:, :case["top_k"]]
    w = score.gather(1, ids)
    if case["renormalise"]:
        w = w / w.sum(1, keepdim=True)
    w, ids = (w * case["scaling"]).float(), ids.to(torch.int32)
    if s["mask"] is not None:
        off = s["mask"][:, None] == 0
        w, ids = torch.where(off, torch.zeros_like(w), w), torch.where(off, -torch.ones_like(ids), ids)
    offsets, order, slot = _sorted_rows(ids, E)
    return dict(ids=ids, weights=w, offsets=offsets, order=order, slot=slot)


def _by_expert(case, s):
    """Of each sorted row: is it in use, its expert, its place in the expert's run, its row of ``a``."""
    place = torch.arange(s["out"].shape[0], device="cuda")
    used = place < s["offsets"][-1]
    expert = torch.searchsorted(s["offsets"][1:].long(), place, right=True).clamp(max=case["experts"] - 1)
    return used, expert, (place - s["offsets"][expert]).clamp(0, s["most"] - 1), s["order"].clamp(min=0).long() if case["gather"] else place


def _plain_experts(case, s):
    used, expert, place, row = _by_expert(case, s)
    a = _real(s["a"], s["a_scale"], 1)[row]
    runs = torch.zeros(case["experts"], s["most"], case["k"], device="cuda")
    runs.index_put_((expert, place), torch.where(used[:, None], a, torch.zeros_like(a)), accumulate=True)
    y = torch.bmm(runs, _real(s["b"], s["b_scale"], 128).transpose(1, 2))[expert, place]
    y = _finish(y, None if s["bias"] is None else s["bias"][expert], case)
    return torch.where(used[:, None], y, torch.zeros_like(y))


def _plain_combine(case, s):
    rows = s["y"][s["slot"].clamp(min=0).long()].float()
    w = torch.where(s["slot"] < 0, torch.zeros_like(s["weights"]), s["weights"])
    return (rows * w[:, :, None]).sum(1).to(s["y"].dtype)


_PLAIN = dict(quantize=_plain_quantize, gemm=_plain_gemm, route=_plain_route, experts=_plain_experts, combine=_plain_combine)
_OWN = dict(quantize=_own_quantize, gemm=_own_gemm, route=_own_route, experts=_own_experts, combine=_own_combine)


# -- what a pass cannot do without ---------------------------------------------------------------------------------------------
def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2}
    if case["kind"] == "quantize":
        n, blocks = case["rows"] * case["cols"], -(-case["rows"] // case["block_rows"]) * -(-case["cols"] // 128)
        return dict(bytes=n * (size[case["dtype"]] + 1) + 4 * blocks, flops=4 * n)
    if case["kind"] == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        kb = -(-k // 128)
        return dict(bytes=m * k + n * k + 4 * kb * (m + -(-n // 128)) + m * n * size[case["out"]] + (4 * n if case["bias"] else 0),
                    flops=2 * m * n * k)
    if case["kind"] == "route":
        T, E, k = case["tokens"], case["experts"], case["top_k"]
        return dict(bytes=T * E * size[case["dtype"]] + 16 * T * k + 4 * (E + 1) + (4 * E if case["bias"] else 0) + (T if case["padded"] else 0),
                    flops=8 * T * E)
    rows = _real_tokens(case) * case["top_k"]
    if case["kind"] == "experts":
        n, k = case["n"], case["k"]
        kb = -(-k // 128)
        active = case["experts"] * (1.0 - (1.0 - 1.0 / case["experts"]) ** rows)   # of evenly popular experts
        a = (_real_tokens(case) if case["gather"] else rows) * (k + 4 * kb)
        return dict(bytes=a + active * (n * k + 4 * kb * -(-n // 128)) + rows * n * size[case["out"]] + 4 * rows, flops=2 * rows * n * k)
    return dict(bytes=(rows + case["tokens"]) * case["n"] * size[case["dtype"]] + 8 * case["tokens"] * case["top_k"], flops=2 * rows * case["n"])


# -- the definition in 64 bits -------------------------------------------------------------------------------------------------
def _to_e4m3(v):
    """The nearest value of the format (ties to even), |v| <= 448: 4 significant bits down to 2^-6, steps of 2^-9 below."""
    _, e = torch.frexp(v.abs().clamp(min=2.0 ** -6))
    step = torch.exp2((e - 4).double())
    return torch.round(v / step) * step


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "quantize":
        x, br = s["x"].double(), case["block_rows"]
        codes, scales = torch.empty_like(x), torch.empty(-(-x.shape[0] // br), -(-x.shape[1] // 128), dtype=torch.float64, device="cuda")
        for j in range(scales.shape[1]):
            part = x[:, 128 * j:128 * j + 128]
            most = part.abs().amax(1)
            most = torch.stack([most[i:i + br].amax() for i in range(0, len(most), br)]) if br > 1 else most
            scales[:, j] = torch.clamp(most / 448, min=2.0 ** -126)
            codes[:, 128 * j:128 * j + 128] = _to_e4m3((part / scales[:, j].repeat_interleave(br)[:len(part), None]).clamp(-448, 448))
        return codes, scales
    if case["kind"] == "gemm":
        return _exact_product(s["a"], s["a_scale"], s["b"], s["b_scale"], s["bias"], case["relu"])
    if case["kind"] == "experts":
        y = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
        ends = s["offsets"].tolist()
        for e in range(case["experts"]):
            lo, hi = ends[e], ends[e + 1]
            if hi > lo:
                rows = s["order"][lo:hi].long() if case["gather"] else torch.arange(lo, hi, device="cuda")
                y[lo:hi] = _exact_product(s["a"].view(torch.uint8)[rows].view(torch.float8_e4m3fn), s["a_scale"][rows], s["b"][e], s["b_scale"][e],
                                          None if s["bias"] is None else s["bias"][e], case["relu"])
        return y
    if case["kind"] == "combine":
        y = torch.zeros(case["tokens"], case["n"], dtype=torch.float64, device="cuda")
        for j in range(case["top_k"]):
            on = s["slot"][:, j] >= 0
            y[on] += s["weights"][on, j].double()[:, None] * s["y"][s["slot"][on, j].long()].double()
        return y
    x = s["logits"].double()
    p = torch.softmax(x, 1) if case["score"] == "softmax" else torch.special.expit(x)
    left = p.clone() if s["bias"] is None else p + s["bias"].double()
    if case["groups"] > 1:
        by_group = left.view(x.shape[0], case["groups"], -1)
        strength = by_group.topk(min(case["group_best"], by_group.shape[2]), dim=2).values.sum(2)
        rank = (strength[:, None, :] > strength[:, :, None]).sum(2)
        left = torch.where((rank < case["top_groups"]).repeat_interleave(by_group.shape[2], 1), left, torch.full_like(left, -math.inf))
    w = torch.empty(x.shape[0], case["top_k"], dtype=torch.float64, device="cuda")
    for j in range(case["top_k"]):
        at = left.argmax(1, keepdim=True)
        w[:, j:j + 1] = p.gather(1, at)
        left.scatter_(1, at, -math.inf)
    if case["renormalise"]:
        w = w / w.sum(1, keepdim=True)
    w = w * case["scaling"]
    if s["mask"] is not None:
        w[s["mask"] == 0] = 0
    return dict(ids=None, weights=w, offsets=None, order=None, slot=None)


def _exact_product(a, sa, b, sb, bias, relu):
    y = torch.zeros(a.shape[0], b.shape[0], dtype=torch.float64, device="cuda")
    a, b = a.double(), b.double()
    for j in range(sa.shape[1]):
        cut = slice(128 * j, 128 * j + 128)
        y += (a[:, cut] @ b[:, cut].t()) * sa[:, j].double()[:, None] * sb[:, j].double().repeat_interleave(128)[:b.shape[0]]
    if bias is not None:
        y += bias.double()
    return y.clamp(min=0) if relu else y
