"""Layers of experts beside an encoder slice, and their update, as cases to time and to check.

A user who puts experts in the place of a layer's feed-forward block runs

- ``route_fwd`` / ``route_bwd``: the top k experts of every token by its logits, their
  weights, and the plan that sorts the tokens' rows by expert; the logits' gradient;
- ``dispatch_fwd`` / ``dispatch_bwd`` / ``combine_fwd`` / ``combine_bwd``: rows to the
  experts' order, and the weighted sum of what the experts made of them, with gradients;
- ``product``: the experts' products over ragged groups of rows, in the three forms of a
  layer (``xwt`` forward, ``xw`` data gradient, ``xtw`` weight gradient) with the epilogues
  of a feed-forward block; ``column_sum``: their bias gradients;
- ``adamw``: one AdamW step over all of the layer's tensors, with moments in 32 bits or in 8.

Widths are those of the library's own workloads (width 128 in fp32, 768 and 1024 in bf16, four
times that inside) and values around them; batches of 16 new tokens to 8192.  Logits are N(0, 1)
beside an expert's own N(0, 0.5), padded tokens have no finite logit, activations N(0, 1), weights
N(0, 0.02), upstream gradients N(0, 1e-2).  Group sizes follow from the case; the seed orders them.
"""
import math

import numpy as np
import torch

own = False

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
BLOCK = 256  # moments that share a scale in 8 bits
BETA1, BETA2, EPS, LR, DECAY, STEP = 0.9, 0.999, 1e-8, 2e-4, 0.01, 1000
ALIGN = 64  # values: where a tensor starts in the buffers


# ------------------------------------------------------------------- the cases
def _route(op, name, tokens, experts, top_k, dtype, over, padded):
    return dict(name=name, op=op, tokens=tokens, experts=experts, top_k=top_k, dtype=dtype, over=over, padded=padded)


def _rows(op, name, tokens, top_k, width, dtype, padded):
    return dict(name=name, op=op, tokens=tokens, top_k=top_k, width=width, dtype=dtype, padded=padded)


def _product(name, form, rows, groups, d_out, d_in, dtype, epilogue, skew, empty, behind):
    return dict(name=name, op="product", form=form, rows=rows, groups=groups, d_out=d_out, d_in=d_in, dtype=dtype,
                epilogue=epilogue, skew=skew, empty=empty, behind=behind)


def _adamw(name, layers, width, ffn, experts, states, grads):
    return dict(name=name, op="adamw", layers=layers, width=width, ffn=ffn, experts=experts, states=states, grads=grads)


def listed():
    return [
        # One new token of each of 16 requests: the smallest call.
        _route("route_fwd", "route_tokens", 16, 8, 2, "fp32", "chosen", 0),
        # The benchmark workload's tokens over many experts, some of them padding; and a
        # training step's gradient on an odd batch, weights by the softmax over all experts.
        _route("route_fwd", "route_large", 8192, 64, 4, "fp32", "chosen", 800),
        _route("route_bwd", "route_bwd_odd", 4999, 128, 6, "bf16", "all", 99),
        # What the experts made of the benchmark workload's tokens, added up; the gradient of
        # that sum on an odd batch of base width.
        _rows("combine_fwd", "combine_fwd_large", 8192, 2, 1024, "bf16", 0),
        _rows("combine_bwd", "combine_bwd_odd", 3001, 4, 768, "bf16", 101),
        # The first product of a feed-forward block of experts, large width, with bias and GELU.
        _product("up_large", "xwt", 16384, 8, 4096, 1024, "bf16", "gelu", 1.0, 0, 0),
        # The data gradient through GELU at base width, many small ragged groups, one empty.
        _product("dgrad_ragged", "xw", 5003, 16, 768, 2048, "bf16", "gelu_bwd", 2.0, 1, 13),
        # Weight gradients of the large width, ragged, one expert without a token.
        _product("wgrad_ragged", "xtw", 9001, 8, 4096, 1024, "bf16", "store", 1.5, 1, 7),
        # Four new tokens, two experts each: the weights are read for a row or two.
        _product("product_tokens", "xwt", 8, 8, 4096, 1024, "bf16", "gelu", 1.0, 3, 0),
        # The width of the fp32 workload, full precision, odd rows.
        _product("product_f32", "xwt", 257, 4, 512, 128, "fp32", "gelu", 1.0, 0, 0),
        # The update of a base-width layer's tensors; of a layer of eight large experts, moments in 8 bits.
        _adamw("adamw_layer", 1, 768, 2048, 0, "fp32", "fp32"),
        _adamw("adamw_experts8", 1, 1024, 4096, 8, "8bit", "fp32"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


MOST_FLOP = 16384 * 4096 * 1024  # multiply-adds of a drawn bf16 product
MOST_WEIGHTS = 8 * 4096 * 1024


def draw(rng):
    op = rng.choice(["route_fwd", "route_fwd", "route_bwd", "dispatch_fwd", "dispatch_bwd", "combine_fwd", "combine_bwd",
                     "product", "product", "product", "product", "tokens", "column_sum", "adamw", "adamw"])
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    if op.startswith("route"):
        experts = _log_int(rng, 2, 256)
        tokens = _log_int(rng, 1, 16384 * 64 // max(64, experts))
        return dict(op=op, tokens=tokens, experts=experts, top_k=rng.randint(1, min(8, experts)),
                    dtype=rng.choice(["fp32", "bf16"]), over=rng.choice(["chosen", "all"]), padded=rng.randint(0, tokens // 8))
    if op.startswith("dispatch") or op.startswith("combine"):
        top_k, width = rng.choice([1, 2, 2, 3, 4, 6, 8]), 8 * _log_int(rng, 8, 256)
        tokens = _log_int(rng, 1, min(16384, 8192 * 3 * 1024 // ((top_k + 1) * width)))
        return dict(op=op, tokens=tokens, top_k=top_k, width=width, dtype=dtype, padded=rng.randint(0, tokens // 8))
    if op == "adamw":
        experts = rng.choice([0, 2, 4, 8])
        return dict(op=op, layers=1 if experts else rng.randint(1, 4), width=4 * _log_int(rng, 16, 256),
                    ffn=4 * _log_int(rng, 32, 512), experts=experts, states=rng.choice(["8bit", "8bit", "fp32"]),
                    grads=rng.choice(["fp32", "fp32", "bf16"]))
    groups = _log_int(rng, 1, 64)
    step = 8 if dtype == "bf16" else 1
    if dtype == "fp32":
        d_out, d_in = _log_int(rng, 16, 1024), _log_int(rng, 16, 768)
    else:
        d_out, d_in = step * _log_int(rng, 8, 512), step * _log_int(rng, 8, 256)
    while groups * d_out * d_in > MOST_WEIGHTS:
        groups = (groups + 1) // 2
    most = MOST_FLOP // (d_out * d_in) if dtype == "bf16" else 1024 * 768 * 768 // (d_out * d_in)
    skew, empty, behind = round(rng.uniform(0.0, 3.0), 2), rng.randint(0, groups // 2), rng.randint(0, 40)
    if op == "column_sum":
        return dict(op=op, rows=_log_int(rng, 1, 16384 if dtype == "bf16" else 4096), groups=groups, d_out=d_out, dtype=dtype,
                    skew=skew, empty=empty, behind=behind)
    form = "xwt" if op == "tokens" else rng.choice(["xwt", "xw", "xtw"])
    rows = _log_int(rng, 1, 96) if op == "tokens" else _log_int(rng, 16, max(16, min(16384, most)))
    epilogue = {"xwt": ["store", "gelu"], "xw": ["store", "gelu_bwd"], "xtw": ["store"]}[form]
    return dict(op="product", form=form, rows=rows, groups=groups, d_out=d_out, d_in=d_in, dtype=dtype,
                epilogue=rng.choice(epilogue), skew=skew, empty=empty, behind=behind)


def _sizes(case):
    """Rows of every group, largest first, the empty ones last; the seed only orders them."""
    full = max(1, case["groups"] - case["empty"])
    share = [math.exp(-case["skew"] * i / full) for i in range(full)]
    ends = [round(case["rows"] * sum(share[:i + 1]) / sum(share)) for i in range(full)]
    return [b - a for a, b in zip([0] + ends, ends)] + [0] * (case["groups"] - full)


def _tensors(case):
    """(values, weight decay) of every tensor: an attention block, and its feed-forward block or experts."""
    h, f = case["width"], case["ffn"]
    block = [(f * h, True), (f, False), (h * f, True), (h, False)]
    attention = [] if case["experts"] else [(3 * h * h, True), (3 * h, False), (h * h, True), (h, False)] + [(h, False)] * 4
    router = [(case["experts"] * h, True)] if case["experts"] else []
    return (attention + router + block * max(1, case["experts"])) * case["layers"]


def _places(case):
    """Where each tensor starts in the buffers, and their length."""
    at, starts = 0, []
    for n, _ in _tensors(case):
        starts.append(at)
        at += -(-n // BLOCK) * BLOCK if case["states"] == "8bit" else -(-n // ALIGN) * ALIGN
    return starts, at


# ------------------------------------------------------------- their arithmetic
def _chosen(case, logits):
    """(experts, their logits), best first, lower index first among equals; -1 where no finite logit is left."""
    value, index = torch.sort(logits, dim=-1, descending=True, stable=True)
    value, index = value[:, :case["top_k"]], index[:, :case["top_k"]]
    return torch.where(value == -math.inf, -1, index), value


def _exp_from(x, top):
    return torch.where(x == -math.inf, 0.0, (x - top).exp())


def _route_forward(case, logits, to):
    logits = logits.to(to)
    expert, value = _chosen(case, logits)
    top = value[:, :1].clamp_min(torch.finfo(to).min)
    e = _exp_from(value, top)
    total = (e if case["over"] == "chosen" else _exp_from(logits, top)).sum(-1, keepdim=True)
    weight = torch.where(total > 0, e / total, 0.0)
    # the plan: choices sorted by expert, earlier tokens first
    key = torch.where(expert < 0, case["experts"], expert).flatten()
    order = torch.sort(key, stable=True).indices
    place = torch.empty_like(order)
    place[order] = torch.arange(order.numel(), device=order.device)
    row = torch.where(expert < 0, -1, place.view_as(expert))
    count = (key[:, None] == torch.arange(case["experts"], device=key.device)).sum(0)
    offset = torch.cat((torch.zeros_like(count[:1]), count.cumsum(0)))
    return expert.int(), weight, row.int(), offset.int()


def _route_backward(case, logits, expert, dweight, to):
    """Through the softmax over the chosen experts or over all."""
    logits, dweight = logits.to(to), dweight.to(to)
    live = expert >= 0
    at = expert.clamp_min(0).long()
    chosen = torch.zeros_like(logits).scatter_add_(1, at, live.to(to)) > 0
    dw = torch.zeros_like(logits).scatter_add_(1, at, torch.where(live, dweight, 0.0))
    over = logits if case["over"] == "all" else torch.where(chosen, logits, -math.inf)
    top = over.amax(-1, keepdim=True).clamp_min(torch.finfo(to).min)
    e = _exp_from(over, top)
    total = e.sum(-1, keepdim=True)
    p = torch.where(total > 0, e / total, 0.0)
    return p * (dw - (p * dw).sum(-1, keepdim=True))


def _pick(rows, row, to):
    """rows[row] as [tokens, top_k, width], zeros where a choice has no row."""
    return torch.where((row >= 0)[..., None], rows[row.clamp_min(0).long()].to(to), 0.0)


def _gelu(z):
    return z * 0.5 * (1.0 + torch.erf(z / math.sqrt(2.0)))


def _gelu_slope(z):
    return 0.5 * (1.0 + torch.erf(z / math.sqrt(2.0))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)


def _by_group(st, to):
    """The product of every group, in `to`."""
    case, n = st["case"], sum(st["sizes"])
    a = st["a"][:n].to(to).split(st["sizes"])
    if case["form"] == "xtw":
        b = st["b"][:n].to(to).split(st["sizes"])
        return torch.stack([x.t() @ y for x, y in zip(a, b)])
    w = st["w"].to(to)
    return torch.cat([x @ (v.t() if case["form"] == "xwt" else v) for x, v in zip(a, w)])


def _f32(x):
    return float(np.float32(x))


def _decode_m(codes, scale, to):
    return (codes.view(torch.float8_e4m3fn).to(to).view(-1, BLOCK) * scale.to(to)[:, None]).flatten()


def _decode_r(codes, scale, to):
    """Code c > 0 stands for (1 + (c % 16) / 16) 2^(c / 16 - 16), code 0 for 0."""
    c = codes.int()
    x = torch.where(c > 0, (1.0 + (c % 16).to(to) / 16.0) * torch.exp2((c // 16).to(to) - 16.0), 0.0)
    return (x.view(-1, BLOCK) * scale.to(to)[:, None]).flatten()


def _scales(x, unit):
    """A block's scale, and what its values are multiplied by: largest to `1 / unit`."""
    top = x.view(-1, BLOCK).abs().amax(-1)
    scale = torch.where(top < 1e-30, 0.0, top * unit)
    return scale, torch.where(top < 1e-30, 0.0, scale.reciprocal())


def _encode_m(x):
    scale, inv = _scales(x, _f32(1.0 / 448.0))
    return (x.view(-1, BLOCK) * inv[:, None]).flatten().to(torch.float8_e4m3fn).view(torch.uint8), scale


def _encode_r(x):
    """To the nearest code, ties to even; what is not 0 stays above 0."""
    scale, inv = _scales(x, _f32(1.0 / 0.96875))
    y = (x.view(-1, BLOCK) * inv[:, None]).flatten()
    bits = y.view(torch.int32)
    code = ((bits + 0x3ffff + ((bits >> 19) & 1)) >> 19) - (111 << 4)
    return torch.where(y > 0, code.clamp(1, 255), 0).to(torch.uint8), scale


def _update(case, w, g, m, r2, decay):
    """(w, m, v) after a step; products and sums rounded one by one."""
    b1, b2 = _f32(BETA1), _f32(BETA2)
    m = m * b1 + g * _f32(np.float32(1) - np.float32(BETA1))
    v = r2 * b2 + (g * g) * _f32(np.float32(1) - np.float32(BETA2))
    w = w - w * (decay * _f32(LR * DECAY))
    step = (m * _f32(1.0 / (1.0 - BETA1 ** STEP))) / ((v * _f32(1.0 / (1.0 - BETA2 ** STEP))).sqrt() + _f32(EPS))
    return w - step * _f32(LR), m, v


# ------------------------------------------------------------------ the passes
def _plan(case, g):
    """A plan as routing makes it: every token's choices are different experts."""
    experts = 4 * case["top_k"]
    logits = torch.randn(case["tokens"], experts, device="cuda", generator=g)
    logits[torch.randperm(case["tokens"], device="cuda", generator=g)[:case["padded"]]] = -math.inf
    expert, weight, row, offset = _route_forward(dict(case, experts=experts, over="chosen"), logits, torch.float32)
    return weight, row, int(offset[-1])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, dt = case["op"], DT[case.get("dtype", "fp32")]

    def normal(*shape, std=1.0, dtype=None):
        return (torch.randn(*shape, device="cuda", generator=g) * std).to(dtype or dt)

    st = dict(case=case)
    if op.startswith("route"):
        t, e, k = case["tokens"], case["experts"], case["top_k"]
        logits = torch.randn(t, e, device="cuda", generator=g) + 0.5 * torch.randn(e, device="cuda", generator=g)
        logits[torch.randperm(t, device="cuda", generator=g)[:case["padded"]]] = -math.inf
        st["logits"] = logits.to(dt)
        st["expert"], st["row"] = (torch.empty(t, k, device="cuda", dtype=torch.int32) for _ in range(2))
        st["weight"] = torch.empty(t, k, device="cuda")
        st["offset"] = torch.empty(e + 1, device="cuda", dtype=torch.int32)
        if op == "route_bwd":
            st["expert"] = _route_forward(case, st["logits"], torch.float32)[0]
            st["dweight"] = normal(t, k, std=1e-2, dtype=torch.float32)
            st["dlogits"] = torch.empty_like(st["logits"])
        return st
    if op.startswith("dispatch") or op.startswith("combine"):
        t, k, h = case["tokens"], case["top_k"], case["width"]
        st["weight"], st["row"], used = _plan(case, g)
        st["rows"], st["x"] = normal(t * k, h), normal(t, h)
        st["rows"][used:] = 0
        if op == "combine_bwd":
            st["x"] = normal(t, h, std=1e-2)  # the upstream gradient
        st["out"] = torch.zeros(t * k if op in ("dispatch_fwd", "combine_bwd") else t, h, device="cuda", dtype=dt)
        st["dweight"] = torch.empty(t, k, device="cuda")
        return st
    if op == "adamw":
        starts, n = _places(case)
        mask = torch.zeros(n, device="cuda")
        st["decay"] = torch.zeros(n, device="cuda")
        for (size, decay), at in zip(_tensors(case), starts):
            mask[at:at + size] = 1
            st["decay"][at:at + size] = float(decay)
        st["w"] = normal(n, std=0.02, dtype=torch.float32) * mask
        st["g"] = (normal(n, std=1e-3, dtype=torch.float32) * mask).to(DT[case["grads"]])
        st["p"] = st["w"].to(torch.bfloat16)
        m = normal(n, std=3e-4, dtype=torch.float32) * mask
        r = (normal(n, std=3e-4, dtype=torch.float32).abs() + 5e-4) * mask
        if case["states"] == "fp32":
            st["m"], st["v"] = m, r * r
        else:
            st["m"], st["m_scale"] = _encode_m(m)
            st["r"], st["r_scale"] = _encode_r(r)
        return st
    rows, e = case["rows"] + case["behind"], case["groups"]
    sizes = _sizes(case)
    st["sizes"] = [sizes[i] for i in torch.randperm(e, device="cuda", generator=g).tolist()]
    ends = np.cumsum([0] + st["sizes"])
    st["offset"] = torch.tensor(ends, dtype=torch.int32, device="cuda")
    if op == "column_sum":
        st["a"] = normal(rows, case["d_out"], std=1e-2)
        st["c"] = torch.empty(e, case["d_out"], device="cuda")
        return st
    o, i, form = case["d_out"], case["d_in"], case["form"]
    if form == "xwt":
        st["a"], st["c"] = normal(rows, i), torch.zeros(rows, o, device="cuda", dtype=dt)
        st["bias"] = normal(e, o, std=0.02)
    elif form == "xw":
        st["a"], st["c"] = normal(rows, o, std=1e-2), torch.zeros(rows, i, device="cuda", dtype=dt)
    else:
        st["a"], st["b"] = normal(rows, o, std=1e-2), normal(rows, i)
        st["c"] = torch.empty(e, o, i, device="cuda")
    if form != "xtw":
        st["w"] = normal(e, o, i, std=0.02)
    slope = torch.float16 if case["dtype"] == "bf16" else torch.float32
    if case["epilogue"] == "gelu":
        st["slope"] = torch.zeros(rows, o, device="cuda", dtype=slope)
    if case["epilogue"] == "gelu_bwd":
        st["slope"] = _gelu_slope(normal(rows, i, dtype=torch.float32)).to(slope)
    return st


def _run_own(st):
    from paper_2202_11836_gb300 import _lib as L
    case, op = st["case"], st["case"]["op"]
    code = {"bf16": L.SKY_DTYPE_BF16, "fp32": L.SKY_DTYPE_FP32}
    stream = torch.cuda.current_stream().cuda_stream
    if op.startswith("route"):
        if "shape" not in st:  # kept beside the model, with the workspace
            st["shape"] = L.SkyRouteShape(case["tokens"], case["experts"], case["top_k"], code[case["dtype"]],
                                          L.SKY_ROUTE_OVER_CHOSEN if case["over"] == "chosen" else L.SKY_ROUTE_OVER_ALL)
            st["ws"] = torch.empty(L.lib().sky_route_workspace_bytes(st["shape"]), dtype=torch.uint8, device="cuda")
        if op == "route_fwd":
            L.call("sky_route_fwd", st["shape"], st["logits"].data_ptr(), st["expert"].data_ptr(),
                   st["weight"].data_ptr(), st["row"].data_ptr(), st["offset"].data_ptr(), st["ws"].data_ptr(),
                   st["ws"].numel(), None, stream)
            return st["expert"], st["weight"], st["row"], st["offset"]
        L.call("sky_route_bwd", st["shape"], st["logits"].data_ptr(), st["expert"].data_ptr(),
               st["dweight"].data_ptr(), st["dlogits"].data_ptr(), stream)
        return st["dlogits"]
    if op.startswith("dispatch") or op.startswith("combine"):
        if "shape" not in st:
            st["shape"] = L.SkyRowsShape(case["tokens"], case["top_k"], case["width"], code[case["dtype"]])
        x, rows, out, row = (st[n].data_ptr() for n in ("x", "rows", "out", "row"))
        if op == "dispatch_fwd":
            L.call("sky_dispatch_fwd", st["shape"], x, row, out, stream)
        elif op == "dispatch_bwd":
            L.call("sky_dispatch_bwd", st["shape"], rows, row, out, stream)
        elif op == "combine_fwd":
            L.call("sky_combine_fwd", st["shape"], rows, row, st["weight"].data_ptr(), out, stream)
        else:
            L.call("sky_combine_bwd", st["shape"], rows, x, row, st["weight"].data_ptr(), out,
                   st["dweight"].data_ptr(), stream)
            return st["out"], st["dweight"]
        return st["out"]
    if op == "adamw":
        if "table" not in st:
            starts, _ = _places(case)
            small = case["states"] == "8bit"
            moments = (("m", 1), ("r", 1)) if small else (("m", 4), ("v", 4))
            table = []
            for (n, decay), at in zip(_tensors(case), starts):
                m, v = (st[x].data_ptr() + size * at for x, size in moments)
                ms, vs = (st[x].data_ptr() + 4 * (at // BLOCK) if small else None for x in ("m_scale", "r_scale"))
                table.append(L.SkyAdamwTensor(st["w"].data_ptr() + 4 * at,
                                              st["g"].data_ptr() + st["g"].element_size() * at, m, v, ms, vs,
                                              st["p"].data_ptr() + 2 * at, n, int(decay)))
            st["table"] = (L.SkyAdamwTensor * len(table))(*table)
            st["config"] = L.SkyAdamwConfig(LR, BETA1, BETA2, EPS, DECAY, STEP, code[case["grads"]],
                                            L.SKY_STATE_8BIT if small else L.SKY_STATE_FP32)
        L.call("sky_adamw_step", st["config"], st["table"], len(st["table"]), None, stream)
        return _moments(st)
    if "shape" not in st:
        rows = case["rows"] + case["behind"]
        st["shape"] = L.SkyGroupedShape(case["groups"], rows, case["d_out"], case.get("d_in", 0), code[case["dtype"]])
    offset, a, c = st["offset"].data_ptr(), st["a"].data_ptr(), st["c"].data_ptr()
    if op == "column_sum":
        L.call("sky_grouped_column_sum", st["shape"], offset, a, c, None, stream)
        return st["c"]
    form = {"xwt": L.SKY_GEMM_XWT, "xw": L.SKY_GEMM_XW, "xtw": L.SKY_GEMM_XTW}[case["form"]]
    out = L.SKY_DTYPE_FP32 if case["form"] == "xtw" else code[case["dtype"]]
    if "ws" not in st:
        n = L.lib().sky_grouped_gemm_workspace_bytes(form, st["shape"], out)
        st["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    b = st["b" if case["form"] == "xtw" else "w"].data_ptr()
    bias = st["bias"].data_ptr() if case["form"] == "xwt" else None
    epilogue = {"store": L.SKY_EPI_STORE, "gelu": L.SKY_EPI_BIAS_GELU, "gelu_bwd": L.SKY_EPI_GELU_BWD}[case["epilogue"]]
    slope = st["slope"].data_ptr() if "slope" in st else None
    L.call("sky_grouped_gemm", form, st["shape"], offset, a, b, c, out, epilogue, bias,
           slope if case["epilogue"] == "gelu_bwd" else None, slope if case["epilogue"] == "gelu" else None,
           st["ws"].data_ptr(), st["ws"].numel(), None, stream)
    return (st["c"], st["slope"]) if case["epilogue"] == "gelu" else st["c"]


def _moments(st):
    """Weights, their copy, and the moments as the values that they stand for."""
    if st["case"]["states"] == "fp32":
        return st["w"], st["p"], st["m"], st["v"]
    return (st["w"], st["p"], _decode_m(st["m"], st["m_scale"], torch.float32),
            _decode_r(st["r"], st["r_scale"], torch.float32))


def run(st):
    if own:
        return _run_own(st)
    case, op, to = st["case"], st["case"]["op"], torch.float32
    dt = DT[case.get("dtype", "fp32")]
    if op == "route_fwd":
        return _route_forward(case, st["logits"], to)
    if op == "route_bwd":
        return _route_backward(case, st["logits"], st["expert"], st["dweight"], to).to(dt)
    if op == "dispatch_fwd":
        live = st["row"] >= 0  # rows of no choice stay as they were: all of them go to one row behind
        out = torch.cat((st["out"], st["out"][:1]))
        at = torch.where(live, st["row"], st["out"].shape[0]).flatten().long()
        out[at] = st["x"].repeat_interleave(case["top_k"], 0)
        return out[:-1]
    if op == "dispatch_bwd":
        return _pick(st["rows"], st["row"], to).sum(1).to(dt)
    if op == "combine_fwd":
        return (_pick(st["rows"], st["row"], to) * st["weight"][..., None]).sum(1).to(dt)
    if op == "combine_bwd":
        dy = st["x"].to(to)[:, None]
        out = torch.cat((st["out"], st["out"][:1]))
        at = torch.where(st["row"] >= 0, st["row"], st["out"].shape[0]).flatten().long()
        out[at] = (dy * st["weight"][..., None]).to(dt).flatten(0, 1)
        return out[:-1], (_pick(st["rows"], st["row"], to) * dy).sum(-1)
    if op == "adamw":
        small = case["states"] == "8bit"
        m = _decode_m(st["m"], st["m_scale"], to) if small else st["m"]
        v = _decode_r(st["r"], st["r_scale"], to).square() if small else st["v"]
        st["w"], m, v = _update(case, st["w"], st["g"].to(to), m, v, st["decay"])
        st["p"] = st["w"].to(torch.bfloat16)
        if small:
            st["m"], st["m_scale"] = _encode_m(m)
            st["r"], st["r_scale"] = _encode_r(v.sqrt())
        else:
            st["m"], st["v"] = m, v
        return _moments(st)
    if op == "column_sum":
        return torch.stack([x.sum(0) for x in st["a"][:case["rows"]].to(to).split(st["sizes"])])
    z = _by_group(st, to)
    if case["form"] == "xtw":
        return z
    n = z.shape[0]
    if case["form"] == "xwt":
        group = torch.bucketize(torch.arange(n, device=z.device), st["offset"][1:], right=True)
        z = z + st["bias"].to(to)[group]
    out = st["c"].clone()
    if case["epilogue"] == "gelu":
        slope = st["slope"].clone()
        out[:n], slope[:n] = _gelu(z).to(dt), _gelu_slope(z).to(slope.dtype)
        return out, slope
    out[:n] = (z * st["slope"][:n].to(to) if case["epilogue"] == "gelu_bwd" else z).to(dt)
    return out


# ---------------------------------------------------------------- in 64 bits
def _exact_route(case, st):
    """Best expert first, one after the other, each then taken out of the running."""
    x = st["logits"].double()
    t, k = case["tokens"], case["top_k"]
    if case["op"] == "route_fwd":
        left, values = x.clone(), []
        for _ in range(k):
            v, i = left.max(-1)
            first = (left == v[:, None]).int().argmax(-1)  # the lowest index among equals
            values.append(v)
            left[torch.arange(t, device=x.device), first] = -math.inf
        values = torch.stack(values, -1)
        total = torch.logsumexp(values if case["over"] == "chosen" else x, -1, keepdim=True)
        weight = torch.exp(values - total)
        return None, torch.where(values == -math.inf, 0.0, weight), None, None
    dx = torch.zeros_like(x)
    p_all = torch.softmax(x, -1)
    t_of = torch.arange(t, device=x.device)
    dw, at, live = st["dweight"].double(), st["expert"].clamp_min(0).long(), st["expert"] >= 0
    values = torch.where(live, x.gather(1, at), -math.inf)
    p = torch.softmax(values, -1) if case["over"] == "chosen" else p_all.gather(1, at)
    p = torch.where(live, p, 0.0)
    mean = (p * dw).sum(-1)
    for c in range(k):
        dx[t_of, at[:, c]] += torch.where(live[:, c], p[:, c] * (dw[:, c] - (mean if case["over"] == "chosen" else 0.0)), 0.0)
    if case["over"] == "all":
        dx -= torch.where(live[:, :1], p_all * mean[:, None], 0.0)
    return dx


def _exact_rows(case, st):
    """Choice by choice."""
    op, row = case["op"], st["row"].long()
    x, rows, w = st["x"].double(), st["rows"].double(), st["weight"].double()
    out = st["out"].double()
    dweight = torch.zeros_like(w)
    for c in range(case["top_k"]):
        t = torch.nonzero(row[:, c] >= 0).flatten()
        r = row[t, c]
        if op == "dispatch_fwd":
            out[r] = x[t]
        elif op == "dispatch_bwd":
            out[t] += rows[r]
        elif op == "combine_fwd":
            out[t] += w[t, c, None] * rows[r]
        else:
            out[r] = w[t, c, None] * x[t]
            dweight[t, c] = torch.linalg.vecdot(x[t], rows[r])
    return (out, dweight) if op == "combine_bwd" else out


def _exact_product(case, st):
    n, ends = sum(st["sizes"]), st["offset"].tolist()
    out = st["c"].double()
    slope = st["slope"].double() if "slope" in st else None
    for e, (lo, hi) in enumerate(zip(ends, ends[1:])):
        a = st["a"][lo:hi].double()
        if case["op"] == "column_sum":
            out[e] = torch.ones(1, hi - lo, dtype=torch.float64, device=a.device).mm(a)[0]
        elif case["form"] == "xtw":
            out[e] = a.T.mm(st["b"][lo:hi].double())
        elif case["form"] == "xw":
            z = a.mm(st["w"][e].double())
            out[lo:hi] = z * slope[lo:hi] if case["epilogue"] == "gelu_bwd" else z
        else:
            z = torch.addmm(st["bias"][e].double(), a, st["w"][e].double().T)
            if case["epilogue"] == "gelu":
                phi = torch.special.ndtr(z)
                out[lo:hi] = z * phi
                slope[lo:hi] = phi + z * (-z * z / 2).exp() * (2 * math.pi) ** -0.5
            else:
                out[lo:hi] = z
    return (out, slope) if case.get("epilogue") == "gelu" else out


def _exact_adamw(case, st):
    """The step by its formulas.  Of moments in 8 bits the first has no value here: 64 bits put
    some that lie next to a border between two codes on its other side.  (The second, a root, moves
    by a fraction of a code in a step.)"""
    g, w = st["g"].double(), st["w"].double()
    small = case["states"] == "8bit"
    if small:
        every = torch.arange(256, device=g.device, dtype=torch.uint8)
        e4m3 = every.view(torch.float8_e4m3fn).double()
        steps = torch.cat((torch.zeros(1, dtype=torch.float64, device=g.device),
                           torch.tensor([(16 + c % 16) * 2.0 ** (c // 16 - 20) for c in range(1, 256)],
                                        dtype=torch.float64, device=g.device)))
        m = (e4m3[st["m"].long()].view(-1, BLOCK) * st["m_scale"].double()[:, None]).flatten()
        v = (steps[st["r"].long()].view(-1, BLOCK) * st["r_scale"].double()[:, None]).flatten() ** 2
    else:
        m, v = st["m"].double(), st["v"].double()
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g ** 2
    m_hat, v_hat = m / (1 - BETA1 ** STEP), v / (1 - BETA2 ** STEP)
    w = w * (1 - LR * DECAY * st["decay"].double()) - LR * m_hat / (torch.sqrt(v_hat) + EPS)
    if not small:
        return w, w, m, v
    # to the nearest of all codes' values, never from above 0 to 0
    r = torch.sqrt(v).view(-1, BLOCK)
    unit = r.amax(-1, keepdim=True) / 0.96875
    y = torch.where(unit > 0, r / unit, 0.0).flatten()
    hi = torch.searchsorted(steps, y).clamp(1, 255)
    pick = torch.where((y - steps[hi - 1] > steps[hi] - y) | (hi == 1), steps[hi], steps[hi - 1])
    return w, w, None, (torch.where(y > 0, pick, 0.0).view(-1, BLOCK) * unit).flatten()


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op.startswith("route"):
        return _exact_route(case, st)
    if op.startswith("dispatch") or op.startswith("combine"):
        return _exact_rows(case, st)
    return _exact_adamw(case, st) if op == "adamw" else _exact_product(case, st)


def work(case):
    op = case["op"]
    if op == "adamw":
        n = sum(size for size, _ in _tensors(case))
        state = 2 * 2 * (4 if case["states"] == "fp32" else 1 + 4 / BLOCK)  # both moments, read and written
        return {"bytes": n * (state + 8 + 2 + DT[case["grads"]].itemsize), "flops": 16 * n}
    size = DT[case["dtype"]].itemsize
    if op.startswith("route"):
        t, e, k = case["tokens"], case["experts"], case["top_k"]
        if op == "route_fwd":
            return {"bytes": t * e * size + 12 * t * k + 4 * (e + 1), "flops": t * (e * k + 8 * k)}
        return {"bytes": 2 * t * e * size + 8 * t * k, "flops": 6 * t * e}
    if op.startswith("dispatch") or op.startswith("combine"):
        t, k, h = case["tokens"] - case["padded"], case["top_k"], case["width"]
        rows = {"dispatch_fwd": 1, "dispatch_bwd": 1, "combine_fwd": 1, "combine_bwd": 2}[op]
        index = 4 * k * (1 if op.startswith("dispatch") else 2 if op == "combine_fwd" else 3)
        return {"bytes": t * ((1 + rows * k) * h * size + index) + (case["padded"] * h * size if rows == 1 and op != "dispatch_fwd" else 0),
                "flops": t * k * h * (0 if op == "dispatch_fwd" else 3 if op == "combine_bwd" else 2)}
    groups, rows = sum(n > 0 for n in _sizes(case)), case["rows"]
    if op == "column_sum":
        return {"bytes": rows * case["d_out"] * size + 4 * case["groups"] * case["d_out"], "flops": rows * case["d_out"]}
    o, i = case["d_out"], case["d_in"]
    if case["form"] == "xtw":
        return {"bytes": rows * (o + i) * size + 4 * case["groups"] * o * i, "flops": 2 * rows * o * i}
    out = o if case["form"] == "xwt" else i
    extra = rows * out * size if case["epilogue"] in ("gelu", "gelu_bwd") else 0
    bias = case["groups"] * o * size if case["form"] == "xwt" else 0
    return {"bytes": rows * (o + i) * size + groups * o * i * size + extra + bias, "flops": 2 * rows * o * i}
