"""Attention over an encoder's states, and the head norms and rotation before it, as
cases to time and to check.

A slice's output is what a decoder attends to.  What it runs there, and what a
slice's own queries and keys go through where a model norms them, are:

- ``qk_norm_fwd`` / ``qk_norm_bwd``: every query and key head of a token divided by
  its root mean square, scaled by a gain and turned by the token's position, and the
  gradients of the heads and of both gains;
- ``cross_fwd`` / ``cross_bwd``: queries of one length over keys and values of another,
  with ragged valid lengths, heads that share keys and values, sequences without any
  key; the forward also for one new token.

Widths, heads and lengths are those of the library's own workloads (width 128 in fp32,
768 x 12 heads, 1024 x 16 heads; 32 to 2048 tokens) and values around them; encoder
states of a served request are longer.  Queries and keys are N(0, 1) before the norm and
N(0, 1.5) at the attention, values N(0, 1), gains around 1, upstream gradients N(0, 1e-2),
positions anywhere below 2^20, valid lengths spread evenly over [len_lo, kv_len] in an
order that the seed gives.
"""
import math

import torch

own = False

EPS = 1e-6
THETA = 10000.0
LOG2E = math.log2(math.e)
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ------------------------------------------------------------------- the cases
def _norm(op, name, rows, heads, kv_heads, dim, dtype, rotation):
    return dict(name=name, op=op, rows=rows, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype,
                rotation=rotation)


def _cross(op, name, batch, q_len, kv_len, heads, kv_heads, dim, dtype, len_lo):
    return dict(name=name, op=op, batch=batch, q_len=q_len, kv_len=kv_len, heads=heads, kv_heads=kv_heads,
                dim=dim, dtype=dtype, len_lo=len_lo)


def listed():
    return [
        # One new token of each of 16 requests, base width: the smallest call.
        _norm("qk_norm_fwd", "norm_fwd_tokens", 16, 12, 12, 64, "bf16", "halves"),
        # The benchmark workload's tokens, large width, forward and backward.
        _norm("qk_norm_fwd", "norm_fwd_large", 8192, 16, 16, 64, "bf16", "halves"),
        _norm("qk_norm_bwd", "norm_bwd_large", 8192, 16, 16, 64, "bf16", "halves"),
        # Neighbouring dims turned together, few key heads, odd rows: a checked run in
        # full precision, and a training step on an odd batch with wider heads.
        _norm("qk_norm_fwd", "norm_fwd_f32", 1213, 12, 4, 128, "fp32", "pairs"),
        _norm("qk_norm_bwd", "norm_bwd_ragged", 1999, 12, 4, 96, "bf16", "pairs"),
        # A decoder's training step over the benchmark workload's encoder states.
        _cross("cross_fwd", "cross_fwd_large", 16, 512, 512, 16, 16, 64, "bf16", 256),
        _cross("cross_bwd", "cross_bwd_large", 16, 512, 512, 16, 16, 64, "bf16", 256),
        # Odd targets over long sources, four query heads to a key head.
        _cross("cross_fwd", "cross_fwd_long", 4, 333, 2048, 16, 4, 64, "bf16", 512),
        # Backward at odd lengths, three query heads to a key head, one source empty.
        _cross("cross_bwd", "cross_bwd_grouped", 6, 197, 777, 12, 4, 64, "bf16", 0),
        # The same in full precision at the width of the fp32 workload.
        _cross("cross_bwd", "cross_bwd_f32", 4, 45, 32, 2, 2, 64, "fp32", 16),
        # One new token of each request: short sources, many requests; long sources, few.
        _cross("cross_fwd", "cross_token", 32, 1, 512, 16, 16, 64, "bf16", 256),
        _cross("cross_fwd", "cross_token_long", 4, 1, 20000, 16, 4, 64, "bf16", 5000),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


MOST_SCORES = {"bf16": 16 * 16 * 512 * 384, "fp32": 1 << 22}  # of a drawn batch, and values of its widest tensor
MOST_VALUES = {"bf16": 16 * 512 * 1024, "fp32": 16 * 512 * 256}


def draw(rng):
    op = rng.choice(["qk_norm_fwd", "qk_norm_bwd", "cross_fwd", "cross_fwd", "cross_token", "cross_bwd", "cross_bwd"])
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    if op.startswith("qk_norm"):
        dim = rng.choice([32, 64, 64, 96, 128])
        kv_heads = rng.randint(1, 8)
        heads = kv_heads * rng.choice([1, 2, 3, 4])
        most = 8192 * 32 * 64 // ((heads + kv_heads) * dim) // (2 if dtype == "fp32" else 1)
        return dict(op=op, rows=_log_int(rng, 1, min(most, 16384)), heads=heads, kv_heads=kv_heads, dim=dim,
                    dtype=dtype, rotation=rng.choice(["halves", "pairs"]))
    kv_heads = rng.randint(1, 8)
    heads = kv_heads * rng.choice([1, 1, 2, 3, 4])
    dim = 64 if dtype == "bf16" else rng.choice([32, 64, 128])
    if op == "cross_token":
        q_len = rng.choice([1, 1, 1, 2, 4])
        kv_len = _log_int(rng, 1, 20000)
        most = max(1, min(64, 4 * 4 * 20000 * 128 // (kv_len * kv_heads * dim * DT[dtype].itemsize)))
        batch = _log_int(rng, 1, most)
        return dict(op="cross_fwd", batch=batch, q_len=q_len, kv_len=kv_len, heads=heads, kv_heads=kv_heads, dim=dim,
                    dtype=dtype, len_lo=rng.randint(0, kv_len))
    q_len = _log_int(rng, 5, 1024)
    kv_len = _log_int(rng, 5, 2048)
    most = MOST_SCORES[dtype] // (q_len * kv_len * heads)
    while most < 1:
        q_len, kv_len = max(5, q_len // 2), max(5, kv_len // 2)
        most = MOST_SCORES[dtype] // (q_len * kv_len * heads)
    most = min(most, MOST_VALUES[dtype] // (max(q_len * heads, kv_len * kv_heads) * dim), 32)
    return dict(op=op, batch=_log_int(rng, 1, max(1, most)), q_len=q_len, kv_len=kv_len, heads=heads,
                kv_heads=kv_heads, dim=dim, dtype=dtype, len_lo=rng.randint(kv_len // 4, kv_len))


def _lengths(case):
    """The valid lengths, evenly over [len_lo, kv_len]; the seed only orders them."""
    b, lo, hi = case["batch"], case["len_lo"], case["kv_len"]
    return [hi if b == 1 else lo + (hi - lo) * i // (b - 1) for i in range(b)]


# ------------------------------------------------------------- their arithmetic
def _rotate(x, cos, sin, rotation):
    """Turns x [rows, heads, dim] by the angles of cos, sin [rows, 1, dim / 2]."""
    if rotation == "halves":
        a, b = x.chunk(2, -1)
        return torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)


def _turns(pos, dim):
    freq = THETA ** (-torch.arange(0, dim, 2, dtype=torch.float64, device=pos.device) / dim)
    angle = pos.double()[:, None] * freq
    return angle.cos()[:, None], angle.sin()[:, None]


def _gains(case, q_gain, k_gain, to):
    return torch.cat((q_gain.to(to).expand(case["heads"], -1), k_gain.to(to).expand(case["kv_heads"], -1)))


def _norm_forward(case, x, q_gain, k_gain, pos, to):
    cos, sin = (t.to(to) for t in _turns(pos, case["dim"]))
    x = x.to(to)
    r = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
    return _rotate(x * r * _gains(case, q_gain, k_gain, to), cos, sin, case["rotation"])


def _norm_backward(case, x, dy, q_gain, k_gain, pos, to):
    cos, sin = (t.to(to) for t in _turns(pos, case["dim"]))
    x = x.to(to)
    r = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
    xhat = x * r
    dz = _rotate(dy.to(to), cos, -sin, case["rotation"])
    dgain = dz * xhat
    h = dz * _gains(case, q_gain, k_gain, to)
    dx = r * (h - xhat * (h * xhat).mean(-1, keepdim=True))
    return dx, dgain[:, :case["heads"]].sum((0, 1)), dgain[:, case["heads"]:].sum((0, 1))


def _split(case, q, k, v, to):
    """q [B, Akv, G, Sq, D], k and v [B, Akv, 1, Skv, D]."""
    b, a, kv, d = case["batch"], case["heads"], case["kv_heads"], case["dim"]
    q = q.to(to).view(b, case["q_len"], kv, a // kv, d).permute(0, 2, 3, 1, 4)
    k, v = (t.to(to).reshape(b, case["kv_len"], kv, 1, d).permute(0, 2, 3, 1, 4) for t in (k, v))
    return q, k, v


def _probabilities(case, q, k, lens):
    """(P, log2 of the sum of exp2 of the scaled scores): zeros and -inf without keys."""
    s = (q @ k.transpose(-1, -2)) * (1.0 / math.sqrt(case["dim"]))
    dead = torch.arange(case["kv_len"], device=q.device)[None, :] >= lens[:, None]
    s = s.masked_fill(dead[:, None, None, None, :], -math.inf)
    m = s.amax(-1, keepdim=True).clamp_min(torch.finfo(s.dtype).min)
    e = (s - m).exp()
    l = e.sum(-1, keepdim=True)
    lse = m * LOG2E + l.log2()
    return torch.where(l > 0, e / l, 0.0), lse.squeeze(-1).flatten(1, 2)


def _joined(x):
    """[B, heads, G, S, D] as [B, S, heads * G * D]."""
    return x.permute(0, 3, 1, 2, 4).flatten(2)


def _cross_forward(case, q, k, v, lens, to):
    q, k, v = _split(case, q, k, v, to)
    p, lse = _probabilities(case, q, k, lens)
    return _joined(p @ v), lse


def _cross_backward(case, q, k, v, dctx, lens, to):
    c = 1.0 / math.sqrt(case["dim"])
    q, k, v = _split(case, q, k, v, to)
    p, _ = _probabilities(case, q, k, lens)
    do = dctx.to(to).view(q.shape[0], q.shape[3], q.shape[1], q.shape[2], q.shape[4]).permute(0, 2, 3, 1, 4)
    dp = do @ v.transpose(-1, -2)
    ds = p * (dp - (p * dp).sum(-1, keepdim=True))
    dq, dk, dv = (ds @ k) * c, (ds.transpose(-1, -2) @ q) * c, p.transpose(-1, -2) @ do
    return _joined(dq), _joined(dk.sum(2, keepdim=True)), _joined(dv.sum(2, keepdim=True))


# ------------------------------------------------------------------ the passes
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, d, a, kv = DT[case["dtype"]], case["dim"], case["heads"], case["kv_heads"]

    def normal(*shape, std=1.0, mean=0.0):
        return (torch.randn(*shape, device="cuda", generator=g) * std + mean).to(dt)

    st = dict(case=case)
    if case["op"].startswith("qk_norm"):
        rows = case["rows"]
        st["qkv"] = normal(rows, (a + 2 * kv) * d)  # a projection's output: Q | K | V
        st["q_gain"], st["k_gain"] = normal(d, std=0.1, mean=1.0), normal(d, std=0.1, mean=1.0)
        st["pos"] = torch.randint(0, 1 << 20, (rows,), device="cuda", generator=g, dtype=torch.int32)
        if case["op"] == "qk_norm_fwd":
            st["y"] = torch.empty(rows, (a + kv) * d, device="cuda", dtype=dt)
        else:
            st["dy"] = normal(rows, (a + kv) * d, std=1e-2)
            st["dqkv"] = torch.zeros_like(st["qkv"])
            st["dq_gain"], st["dk_gain"] = (torch.empty(d, device="cuda") for _ in range(2))
        return st
    b, sq, skv = case["batch"], case["q_len"], case["kv_len"]
    st["q"] = normal(b, sq, a * d, std=1.5)
    st["kv"] = torch.cat((normal(b, skv, kv * d, std=1.5), normal(b, skv, kv * d)), -1)  # a projection's output: K | V
    order = torch.randperm(b, device="cuda", generator=g)
    st["lens"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")[order]
    st["ctx"] = torch.empty(b, sq, a * d, device="cuda", dtype=dt)
    st["lse"] = torch.empty(b, a, sq, device="cuda")
    if case["op"] == "cross_bwd":
        k, v = st["kv"].chunk(2, -1)
        ctx, lse = _cross_forward(case, st["q"], k, v, st["lens"], torch.float32)  # what the forward left
        st["ctx"].copy_(ctx)
        st["lse"].copy_(lse)
        st["dctx"] = normal(b, sq, a * d, std=1e-2)
        st["dq"], st["dkv"] = torch.empty_like(st["q"]), torch.empty_like(st["kv"])
    return st


def _run_own(st):
    from paper_2202_11836_gb300 import _lib as L
    case = st["case"]
    dt = L.SKY_DTYPE_BF16 if case["dtype"] == "bf16" else L.SKY_DTYPE_FP32
    stream = torch.cuda.current_stream().cuda_stream
    d, a, kv = case["dim"], case["heads"], case["kv_heads"]
    op = case["op"]
    if op.startswith("qk_norm"):
        nd = (a + kv) * d
        if "shape" not in st:  # kept beside the model, with the workspace
            rot = L.SKY_ROTATE_HALVES if case["rotation"] == "halves" else L.SKY_ROTATE_PAIRS
            st["shape"] = L.SkyQkNormShape(case["rows"], a, kv, d, dt, nd + kv * d, nd, EPS, rot, THETA)
            n = 0 if op == "qk_norm_fwd" else L.lib().sky_qk_norm_bwd_workspace_bytes(st["shape"])
            st["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
        if op == "qk_norm_fwd":
            L.call("sky_qk_norm_fwd", st["shape"], st["qkv"].data_ptr(), st["q_gain"].data_ptr(),
                   st["k_gain"].data_ptr(), st["pos"].data_ptr(), st["y"].data_ptr(), stream)
            return st["y"]
        L.call("sky_qk_norm_bwd", st["shape"], st["qkv"].data_ptr(), st["dy"].data_ptr(), st["q_gain"].data_ptr(),
               st["k_gain"].data_ptr(), st["pos"].data_ptr(), st["dqkv"].data_ptr(), st["dq_gain"].data_ptr(),
               st["dk_gain"].data_ptr(), st["ws"].data_ptr(), st["ws"].numel(), stream)
        return st["dqkv"][:, :nd], st["dq_gain"], st["dk_gain"]
    if "shape" not in st:
        st["shape"] = L.SkyCrossShape(case["batch"], case["q_len"], case["kv_len"], a, kv, d, dt, a * d, 2 * kv * d,
                                      2 * kv * d, a * d)
        n = L.lib().sky_cross_attention_bwd_workspace_bytes(st["shape"]) if op == "cross_bwd" else 0
        st["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    k = st["kv"].data_ptr()
    v = k + kv * d * st["kv"].element_size()
    if op == "cross_fwd":
        L.call("sky_cross_attention_fwd", st["shape"], st["q"].data_ptr(), k, v, st["lens"].data_ptr(),
               st["ctx"].data_ptr(), st["lse"].data_ptr(), None, stream)
        return st["ctx"], st["lse"]
    dk = st["dkv"].data_ptr()
    dv = dk + kv * d * st["kv"].element_size()
    L.call("sky_cross_attention_bwd", st["shape"], st["q"].data_ptr(), k, v, st["ctx"].data_ptr(),
           st["dctx"].data_ptr(), st["lse"].data_ptr(), st["lens"].data_ptr(), st["dq"].data_ptr(), dk, dv,
           st["ws"].data_ptr(), st["ws"].numel(), None, stream)
    return st["dq"], st["dkv"]


def _run(st, to):
    """The plain form in the type `to`, not rounded."""
    case = st["case"]
    d, a, kv = case["dim"], case["heads"], case["kv_heads"]
    if case["op"].startswith("qk_norm"):
        x = st["qkv"][:, :(a + kv) * d].view(case["rows"], a + kv, d)
        if case["op"] == "qk_norm_fwd":
            return [_norm_forward(case, x, st["q_gain"], st["k_gain"], st["pos"], to).flatten(1)]
        dx, dq, dk = _norm_backward(case, x, st["dy"].view_as(x), st["q_gain"], st["k_gain"], st["pos"], to)
        return [dx.flatten(1), dq, dk]
    k, v = st["kv"].chunk(2, -1)
    if case["op"] == "cross_fwd":
        return list(_cross_forward(case, st["q"], k, v, st["lens"], to))
    dq, dk, dv = _cross_backward(case, st["q"], k, v, st["dctx"], st["lens"], to)
    return [dq, torch.cat((dk, dv), -1)]


def run(st):
    if own:
        return _run_own(st)
    case, dt = st["case"], DT[st["case"]["dtype"]]
    out = _run(st, torch.float32)
    # heads and their gradients in the storage type; statistics and gain gradients stay fp32
    if case["op"] == "qk_norm_fwd":
        return out[0].to(dt)
    if case["op"] == "qk_norm_bwd":
        return out[0].to(dt), out[1], out[2]
    if case["op"] == "cross_fwd":
        return out[0].to(dt), out[1]
    return out[0].to(dt), out[1].to(dt)


def _exact_norm(st):
    """Head by head as a sum over complex planes: a pair of dims is one complex number."""
    case = st["case"]
    d, a, kv, rows = case["dim"], case["heads"], case["kv_heads"], case["rows"]
    halves = case["rotation"] == "halves"

    def planes(x):
        x = x.double()
        return torch.complex(x[..., :d // 2], x[..., d // 2:]) if halves else torch.complex(x[..., ::2], x[..., 1::2])

    def dims(z):
        return torch.cat((z.real, z.imag), -1) if halves else torch.view_as_real(z).flatten(-2)

    x = st["qkv"][:, :(a + kv) * d].double().view(rows, a + kv, d)
    rms = torch.sqrt((x * x).sum(-1, keepdim=True) / d + EPS)
    gain = torch.empty(a + kv, d, dtype=torch.float64, device=x.device)
    gain[:a], gain[a:] = st["q_gain"].double(), st["k_gain"].double()
    exponent = torch.arange(d // 2, dtype=torch.float64, device=x.device) * (-2.0 * math.log(THETA) / d)
    turn = torch.polar(torch.ones(1, dtype=torch.float64, device=x.device),
                       torch.exp(exponent) * st["pos"].double()[:, None])[:, None]
    if case["op"] == "qk_norm_fwd":
        return dims(planes(x / rms * gain) * turn).reshape(rows, -1)
    dz = dims(planes(st["dy"].view_as(x)) * turn.conj())
    unit = x / rms
    h = dz * gain
    dx = h / rms - x * (h * x).sum(-1, keepdim=True) / (d * rms ** 3)
    by_head = (dz * unit).sum(0)
    return dx.reshape(rows, -1), by_head[:a].sum(0), by_head[a:].sum(0)


def _exact_cross(st):
    """Sequence by sequence over the valid keys alone."""
    case = st["case"]
    b, sq, a, kv, d = case["batch"], case["q_len"], case["heads"], case["kv_heads"], case["dim"]
    bwd = case["op"] == "cross_bwd"
    ctx = torch.zeros(b, sq, a, d, dtype=torch.float64, device="cuda")
    lse = torch.full((b, a, sq), -math.inf, dtype=torch.float64, device="cuda")
    dq, dkv = torch.zeros_like(ctx), torch.zeros(b, case["kv_len"], 2, kv, d, dtype=torch.float64, device="cuda")
    for i, n in enumerate(st["lens"].tolist()):
        if n == 0:
            continue
        q = st["q"][i].double().view(sq, a, d).transpose(0, 1)
        k, v = (t.repeat_interleave(a // kv, 0) for t in st["kv"][i, :n].double().view(n, 2, kv, d).permute(1, 2, 0, 3))
        s = torch.bmm(q, k.transpose(1, 2)) / d ** 0.5
        lse[i] = torch.logsumexp(s, -1) / math.log(2.0)
        p = torch.softmax(s, -1)
        if not bwd:
            ctx[i] = torch.bmm(p, v).transpose(0, 1)
            continue
        do = st["dctx"][i].double().view(sq, a, d).transpose(0, 1)
        dp = torch.bmm(do, v.transpose(1, 2))
        ds = p * dp - p * (p * dp).sum(-1, keepdim=True)
        dq[i] = torch.bmm(ds, k).transpose(0, 1) / d ** 0.5
        dkv[i, :n, 0] = (torch.bmm(ds.transpose(1, 2), q) / d ** 0.5).view(kv, a // kv, n, d).sum(1).transpose(0, 1)
        dkv[i, :n, 1] = torch.bmm(p.transpose(1, 2), do).view(kv, a // kv, n, d).sum(1).transpose(0, 1)
    if bwd:
        return dq.flatten(2), dkv.flatten(2)
    return ctx.flatten(2), lse


def exact(case, seed):
    st = prepare(case, seed)
    return _exact_norm(st) if case["op"].startswith("qk_norm") else _exact_cross(st)


def work(case):
    """Valid keys only; a backward's scores, formed again, are not counted."""
    size = 2 if case["dtype"] == "bf16" else 4
    d, a, kv = case["dim"], case["heads"], case["kv_heads"]
    if case["op"].startswith("qk_norm"):
        n = case["rows"] * (a + kv) * d
        tensors, flops = (2, 8) if case["op"] == "qk_norm_fwd" else (3, 16)
        return {"bytes": tensors * n * size + 4 * case["rows"] + 2 * d * size, "flops": flops * n}
    keys = sum(_lengths(case))
    queries = case["batch"] * case["q_len"]
    pairs = case["q_len"] * keys * a * d
    if case["op"] == "cross_fwd":
        return {"bytes": (2 * queries * a + 2 * keys * kv) * d * size + 4 * queries * a, "flops": 4 * pairs}
    rows = case["batch"] * case["kv_len"]  # the gradients of padded keys are zeros that are written
    return {"bytes": (4 * queries * a + (2 * keys + 2 * rows) * kv) * d * size + 4 * queries * a, "flops": 8 * pairs}
