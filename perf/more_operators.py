"""Operators between a served model's products, and the product of its INT8 container: what they are timed on.

A weight that is decoded to INT8 is multiplied by activations that are rounded to INT8 row by row (``quantize_rows``,
``int8_matmul``).  Between two products stand the norm of the block that ended and of the one that begins, with gate and
residual (``norm``), and the rotation of queries and keys by their tokens' positions (``rotary``).

Formulas.
  quantize_rows  m[t] = max(max_j |x[t, j]|, 2^-119) over a row; s[t] = m[t] / 127, q[t, j] = round(x[t, j] * (127 / m[t])), ties to
                 even, each operation in float32; a row of zeros has s = 1, one with a value that is not finite s = NaN and q = 0
  int8_matmul    y[t, r] = a[r] (s[t] sum_k xq[t, k] wq[r, k]) + bias[r], the sum over whole numbers
  norm           b = norm(x) (o + p) if there is a post weight p, else x;  r = c h + g b with a residual h, else b;
                 z = norm(r) (o + w) + d;  norm(v) = (v - mean) / sqrt(mean((v - mean)^2) + eps), mean 0 unless centred.  Vectors p, g,
                 w, d belong to all rows or to groups of rows that follow one another; z goes to E4M3 or INT8 as above
  rotary         pairs (u, v) of a head's first `rot` values, i and i + rot / 2 or 2 i and 2 i + 1, become
                 f (u cos a - v sin a, v cos a + u sin a), a = position * frequency[i]; the other values stay

A case: ``kind`` rows | product | norm | rotary, ``type`` of the values, and for
  rows     ``T`` rows, ``C`` columns
  product  ``T`` tokens, ``R`` rows of the weight, ``C`` columns, ``type`` of the result, ``a``: with row scales, ``bias``
  norm     ``T`` rows, ``C`` columns, ``out`` same | e4m3 | int8, ``res``: with a residual, of 32 bits if ``wide``, ``post``: with a norm before it,
           ``gate`` and ``mod``: groups of rows that share a gate, weight and bias (0: none; weight alone), ``center``
  rotary   ``T`` tokens, ``H`` heads of ``D`` values, ``more`` heads beside them that stay, ``rot`` values that turn, ``pairs`` half |
           next, ``far``: positions up to that, of tokens ``apart`` or in a row, ``stretch``: the factor of a longer context
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
BLOCK = 128
EPS = 1e-6


def listed():
    return [
        # activations of a few requests before a projection: latency of one call
        {"name": "rows, 16 tokens", "kind": "rows", "T": 16, "C": 5120, "type": "bf16"},
        # a weight brought into the container, one scale for each of its rows
        {"name": "rows, a weight", "kind": "rows", "T": 5120, "C": 17408, "type": "fp32"},
        # token generation for one request on the paper's reference layer
        {"name": "product, 1 token", "kind": "product", "T": 1, "R": 10240, "C": 3840, "type": "bf16", "a": True, "bias": False},
        # token generation for a batch of requests, the last projection of a block
        {"name": "product, 48 tokens", "kind": "product", "T": 48, "R": 5120, "C": 17408, "type": "fp16", "a": True, "bias": True},
        # a ragged middle-sized product
        {"name": "product, ragged", "kind": "product", "T": 777, "R": 3000, "C": 1744, "type": "fp32", "a": True, "bias": False},
        # prompts of a batch times a large square weight
        {"name": "product, prompts", "kind": "product", "T": 8192, "R": 8192, "C": 8192, "type": "bf16", "a": True, "bias": False},
        # one step of a few requests: the residual added, the next block's norm rounded for its products
        {"name": "norm, 16 tokens", "kind": "norm", "T": 16, "C": 5120, "type": "bf16", "out": "e4m3", "res": True, "wide": False, "post": False,
         "gate": 0, "mod": 1, "center": False},
        # prompts between two blocks, norms on both sides of the residual
        {"name": "norm, prompts", "kind": "norm", "T": 8192, "C": 5120, "type": "bf16", "out": "same", "res": True, "wide": False, "post": True,
         "gate": 0, "mod": 1, "center": False},
        # a batch of two images in a diffusion transformer: gates, scales and shifts of each image, a residual of 32 bits, INT8 for the next product
        {"name": "norm, gated", "kind": "norm", "T": 2050, "C": 3840, "type": "fp16", "out": "int8", "res": True, "wide": True, "post": True,
         "gate": 2, "mod": 2, "center": True},
        # queries and keys of one step of a few requests, far into their documents
        {"name": "rotary, 16 tokens", "kind": "rotary", "T": 16, "H": 48, "D": 128, "more": 8, "rot": 128, "pairs": "half", "type": "bf16", "far": 200000,
         "apart": True, "stretch": 8.0},
        # queries and keys of a prompt
        {"name": "rotary, a prompt", "kind": "rotary", "T": 8192, "H": 48, "D": 128, "more": 8, "rot": 128, "pairs": "half", "type": "bf16", "far": 0,
         "apart": False, "stretch": 1.0},
        # pairs side by side in a part of the head, in 32 bits, far out
        {"name": "rotary, a part", "kind": "rotary", "T": 1001, "H": 12, "D": 80, "more": 0, "rot": 32, "pairs": "next", "type": "fp32", "far": 1000000,
         "apart": False, "stretch": 1.0},
    ]


def _log_size(rng, lo, hi, step=1):
    """A multiple of `step` in [lo, hi], spread evenly over the logarithm."""
    return max(lo, min(hi, step * round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)))


def draw(rng):
    kind = rng.choice(["rows", "product", "product", "norm", "norm", "rotary"])
    c = {"kind": kind, "type": rng.choice(["bf16", "bf16", "fp16", "fp32"])}
    if kind == "rows":
        c.update(T=_log_size(rng, 1, 8192), C=_log_size(rng, 64, 17408, rng.choice([1, 16, 16])))
    elif kind == "product":
        c.update(T=_log_size(rng, 1, 8192), R=_log_size(rng, 64, 8192), C=_log_size(rng, 128, 8192, 16), a=rng.random() < 0.7, bias=rng.random() < 0.3)
    elif kind == "norm":
        c.update(T=_log_size(rng, 1, 8192), C=_log_size(rng, 64, 17408, rng.choice([1, 16, 16])), out=rng.choice(["same", "same", "e4m3", "int8"]),
                 res=rng.random() < 0.75, wide=rng.random() < 0.3, post=rng.random() < 0.4, gate=rng.choice([0, 0, 1, 2, 5]), mod=rng.choice([0, 1, 1, 2, 5]),
                 center=rng.random() < 0.3)
        while c["T"] * c["C"] > 8192 * 5120 // (2 if c["type"] == "fp32" else 1):
            c["T"] = c["T"] * 2 // 3
        groups = math.lcm(c["gate"] or 1, c["mod"] or 1)
        c["T"] = max(1, c["T"] // groups) * groups
    else:
        D = rng.choice([64, 80, 96, 128, 128, 256])
        c.update(T=_log_size(rng, 1, 8192), H=rng.choice([1, 5, 12, 16, 40, 48]), D=D, more=rng.choice([0, 2, 8]), rot=rng.choice([D, D, D // 2, D // 4]),
                 pairs=rng.choice(["half", "half", "next"]), far=rng.choice([0, 4096, 200000, 1 << 24]), apart=rng.random() < 0.5, stretch=rng.choice([1.0, 1.0, 4.0, 32.0]))
        while c["T"] * c["H"] * D > 8192 * 48 * 128 // (2 if c["type"] == "fp32" else 1):
            c["T"] = c["T"] * 2 // 3
    return c


def _activations(T, C, g, like=1.5):
    """Rows of different sizes with some channels much larger than the others."""
    x = torch.randn(T, C, generator=g, device="cuda")
    x *= torch.exp(like * torch.rand(T, 1, generator=g, device="cuda"))
    x *= torch.where(torch.rand(1, C, generator=g, device="cuda") < 0.01, 20.0, 1.0)
    return x


def _vectors(groups, C, g, at, spread, dtype):
    shape = (C,) if groups == 1 else (groups, C)
    return (at + spread * torch.randn(shape, generator=g, device="cuda")).to(dtype)


def _frequencies(rot, base, stretch, original=8192.0, fast=32.0, slow=1.0):
    """base^(-2 i / rot) in radians a token; in a context `stretch` times as long as the `original` one, those that turn less than `slow` times
    in it are divided by `stretch`, those that turn more than `fast` times stay, and between them it is shared out linearly."""
    f = torch.pow(torch.tensor(base, dtype=torch.float64), -torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    if stretch == 1.0:
        return f
    stay = ((original * f / (2 * math.pi) - slow) / (fast - slow)).clamp(0.0, 1.0)
    return f * (stay + (1.0 - stay) / stretch)


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(1000003 * seed + 29)
    kind, dtype = case["kind"], TYPES[case["type"]]
    s = {"kind": kind, "type": dtype}
    if kind == "rows":
        T, C = case["T"], case["C"]
        s["x"] = _activations(T, C, g).to(dtype)
        s["out"] = (torch.empty(T, C, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda"))
        return s
    if kind == "product":
        T, R, C = case["T"], case["R"], case["C"]
        s["x"], s["xs"] = _rows(_activations(T, C, g, 0.5))
        w = torch.randn(R, C, generator=g, device="cuda") * torch.exp(torch.rand(R, 1, generator=g, device="cuda")) * 0.02
        s["w"], a = _rows(w)
        s["a"] = a if case["a"] else None
        s["bias"] = torch.randn(R, generator=g, device="cuda") if case["bias"] else None
        s["y"] = torch.empty(T, R, dtype=dtype, device="cuda")
        return s
    if kind == "norm":
        T, C = case["T"], case["C"]
        s["x"] = _activations(T, C, g, 0.5).to(dtype)
        wide = torch.float32 if case["wide"] else dtype
        s["h"] = (_activations(T, C, g, 0.5) * 3.0).to(wide) if case["res"] else None
        s["r"] = torch.empty(T, C, dtype=wide, device="cuda") if case["res"] else None
        s["post"] = _vectors(1, C, g, 0.3, 0.1, dtype) if case["post"] else None
        s["gate"] = torch.tanh(_vectors(case["gate"], C, g, 0.0, 1.0, torch.float32)).to(dtype) if case["gate"] and case["res"] else None
        s["w"] = _vectors(max(case["mod"], 1), C, g, 0.0 if case["mod"] > 1 else 1.0, 0.2, dtype)
        s["d"] = _vectors(case["mod"], C, g, 0.0, 0.3, dtype) if case["mod"] > 1 else None
        s.update(offset=1.0 if case["mod"] > 1 else 0.0, c=0.7 if case["post"] else 1.0, center=case["center"], out=case["out"])
        if case["out"] == "same":
            s["z"] = torch.empty(T, C, dtype=dtype, device="cuda")
        elif case["out"] == "e4m3":
            s["z"] = (torch.empty(T, C, dtype=E4M3, device="cuda"), torch.empty(T, -(-C // BLOCK), dtype=E8M0, device="cuda"))
        else:
            s["z"] = (torch.empty(T, C, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda"))
            s["value"] = torch.empty(T, C, dtype=torch.bfloat16, device="cuda")
        return s
    T, H, D = case["T"], case["H"], case["D"]
    qkv = torch.randn(T, (H + case["more"]) * D, generator=g, device="cuda").to(dtype)
    s["x"] = qkv.view(T, H + case["more"], D)[:, :H]                             # the heads that turn, in the row of a product
    if case["apart"]:
        s["at"] = torch.randint(0, case["far"] + T, (T,), generator=g, device="cuda", dtype=torch.int32)
    else:
        s["at"] = torch.arange(case["far"], case["far"] + T, device="cuda", dtype=torch.int32)
    s["f"] = _frequencies(case["rot"], 1e6 if case["far"] > 4096 else 1e4, case["stretch"]).cuda()
    s["factor"] = 0.1 * math.log(case["stretch"]) + 1.0
    s["next"] = case["pairs"] == "next"
    s["o"] = torch.empty(T, H, D, dtype=dtype, device="cuda")
    return s


def _rows(x):
    """INT8 values and a scale for each row."""
    x = x.float()
    fine = (x.abs() < math.inf).all(1, keepdim=True)
    m = torch.where(fine, x.abs(), 0.0).amax(1, keepdim=True)
    some = m > 0
    m = m.clamp(min=2.0 ** -119)
    q = torch.where(fine, torch.round(x * (torch.full_like(m, 127.0) / m)), 0.0).to(torch.int8)
    scale = torch.where(some, m / torch.full_like(m, 127.0), 1.0)
    return q, torch.where(fine, scale, math.nan)[:, 0]


def _blocks(x):
    """E4M3 values and E8M0 scales of 128 columns of a row: the smallest power of two s with |x| <= 448 s (448 = 0.875 * 2^9)."""
    T, C = x.shape
    n = -(-C // BLOCK)
    x = torch.nn.functional.pad(x, (0, n * BLOCK - C)).view(T, n, BLOCK)
    fine = x.abs() < math.inf
    top = torch.where(fine, x.abs(), 0.0).amax(2, keepdim=True)
    m, e = torch.frexp(top)
    e = torch.where(top > 0, e - 9 + (m > 0.875).to(e.dtype), 0).clamp(min=-126).to(torch.int32)
    power = lambda e: (e + 127 << 23).view(torch.float32)  # noqa: E731
    q = torch.where(fine, x * power(-e), math.nan).view(T, n * BLOCK)[:, :C].contiguous().to(E4M3)
    return q, power(e).view(T, n).to(E8M0)


def _product(s):
    y = (s["x"].float() @ s["w"].float().t()) * s["xs"][:, None]
    if s["a"] is not None:
        y = y * s["a"]
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(s["type"])


def _unit(v, center):
    if center:
        v = v - v.mean(1, keepdim=True)
    return v * torch.rsqrt(v.square().mean(1, keepdim=True) + EPS)


def _spread(v, T):
    """A vector, or a row for each of the groups that T rows fall into, as 32-bit rows."""
    v = v.float()
    return v if v.dim() == 1 else v.repeat_interleave(T // v.shape[0], 0)


def _norm(s):
    T = s["x"].shape[0]
    r = s["x"].float()
    if s["post"] is not None:
        r = _unit(r, s["center"]) * (s["offset"] + s["post"].float())
    if s["gate"] is not None:
        r = r * _spread(s["gate"], T)
    if s["h"] is not None:
        r = s["c"] * s["h"].float() + r
    z = _unit(r, s["center"]) * (s["offset"] + _spread(s["w"], T))
    if s["d"] is not None:
        z = z + _spread(s["d"], T)
    if s["out"] == "same":
        z = z.to(s["type"])
    elif s["out"] == "e4m3":
        z = _blocks(z)
    else:
        q, scale = _rows(z)
        z = torch.mul(q, scale[:, None], out=s["value"])                         # what the eight bits stand for
    return z if s["h"] is None else (z, r.to(s["h"].dtype))


def _rotary(s):
    x, half = s["x"].float(), s["f"].numel()
    a = s["at"].double()[:, None] * s["f"]
    cos, sin = (s["factor"] * torch.cos(a)).float()[:, None], (s["factor"] * torch.sin(a)).float()[:, None]
    o = x.clone()
    u, v = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if s["next"] else (x[..., :half], x[..., half:2 * half])
    first, second = u * cos - v * sin, v * cos + u * sin
    if s["next"]:
        o[..., 0:2 * half:2], o[..., 1:2 * half:2] = first, second
    else:
        o[..., :half], o[..., half:2 * half] = first, second
    return o.to(s["type"])


def run(state):
    s = state
    kind = s["kind"]
    if own:
        import paper_2609_34185_b200 as ep
        if kind == "rows":
            return ep.quantize_rows(s["x"], out=s["out"])
        if kind == "product":
            return ep.int8_matmul(s["x"], s["xs"], s["w"], row_scale=s["a"], bias=s["bias"], out=s["y"])
        if kind == "norm":
            z = ep.norm(s["x"], s["w"], s["d"], residual=s["h"], residual_scale=s["c"], gate=s["gate"], post_weight=s["post"], weight_offset=s["offset"],
                        eps=EPS, center=s["center"], out=s["z"], residual_out=s["r"])
            z, r = z if s["h"] is not None else (z, None)
            if s["out"] == "int8":
                z = torch.mul(z[0], z[1][:, None], out=s["value"])
            return z if r is None else (z, r)
        return ep.rotary(s["x"], s["at"], s["f"], interleaved=s["next"], factor=s["factor"], out=s["o"])
    if kind == "rows":
        return _rows(s["x"])
    if kind == "product":
        return _product(s)
    return _norm(s) if kind == "norm" else _rotary(s)


def work(case):
    """Each input read once, each output written once; 2 operations for a multiply and add of the product, one for each value that is
    rounded, four for each that is normed, three for each that turns."""
    size = 4 if case["type"] == "fp32" else 2
    if case["kind"] == "rows":
        n = case["T"] * case["C"]
        return {"bytes": n * (size + 1) + 4 * case["T"], "flops": n}
    if case["kind"] == "product":
        T, R, C = case["T"], case["R"], case["C"]
        return {"bytes": T * C + R * C + 4 * T + 4 * R * (case["a"] + case["bias"]) + size * T * R, "flops": 2.0 * T * R * C}
    if case["kind"] == "norm":
        T, C = case["T"], case["C"]
        wide = 4 if case["wide"] else size
        vectors = case["post"] + (case["gate"] if case["res"] else 0) + max(case["mod"], 1) + (case["mod"] if case["mod"] > 1 else 0)
        out = size if case["out"] == "same" else 1 + 1 / BLOCK if case["out"] == "e4m3" else 1 + 1 + 2          # INT8: read back and spelt out
        return {"bytes": T * C * (size + out + (2 * wide if case["res"] else 0)) + vectors * C * size, "flops": 4.0 * T * C * (1 + case["post"])}
    n = case["T"] * case["H"] * case["D"]
    return {"bytes": 2 * n * size + 4 * case["T"] + 4 * case["rot"], "flops": 3.0 * case["T"] * case["H"] * case["rot"]}


# ---- the operators' definitions in 64 bits, apart from the plain forms ------------------------------------------------

def _normed(v, weight, centre):
    """Rows of v with mean square 1 (variance 1), in 64 bits, times weight."""
    if centre:
        v = v - v.sum(1, keepdim=True) / v.shape[1]
    return v / torch.sqrt((v * v).sum(1, keepdim=True) / v.shape[1] + EPS) * weight


def _per_row(v, T):
    v = v.double()
    return v[None] if v.dim() == 1 else v[torch.arange(T, device="cuda") * v.shape[0] // T]


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "rows":
        top = s["x"].double().abs().amax(1)
        return None, torch.where(top > 0, top / 127, 1.0)
    if kind == "product":
        y = torch.empty(case["T"], case["R"], dtype=torch.float64, device="cuda")
        w = s["w"].double().t().contiguous()
        for lo in range(0, case["T"], 1024):
            y[lo:lo + 1024] = s["x"][lo:lo + 1024].double() @ w
        y *= s["xs"].double()[:, None]
        if s["a"] is not None:
            y *= s["a"].double()
        return y if s["bias"] is None else y.add_(s["bias"].double())
    if kind == "norm":
        T, C = case["T"], case["C"]
        b = s["x"].double()
        if s["post"] is not None:
            b = _normed(b, s["offset"] + s["post"].double(), case["center"])
        if s["gate"] is not None:
            b = b * _per_row(s["gate"], T)
        r = b if s["h"] is None else b.add_(s["h"].double(), alpha=s["c"])
        z = _normed(r, s["offset"] + _per_row(s["w"], T), case["center"])
        if s["d"] is not None:
            z += _per_row(s["d"], T)
        if case["out"] == "e4m3":
            scale = torch.empty(T, -(-C // BLOCK), dtype=torch.float64, device="cuda")
            for j in range(scale.shape[1]):
                part = z[:, j * BLOCK:(j + 1) * BLOCK]
                top = part.abs().amax(1)
                e = torch.ceil(torch.log2(top.clamp(min=1e-30) / 448))
                e = torch.where(top <= 448 * torch.exp2(e - 1), e - 1, torch.where(top > 448 * torch.exp2(e), e + 1, e))
                scale[:, j] = torch.exp2(torch.where(top > 0, e, 0.0))
                y = part / scale[:, j, None]
                # steps of 2^-9 below 2^-6, then an eighth of the power of two below
                step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))).clamp(max=8) - 3)
                step = torch.where(y.abs() >= 16 * step, 2 * step, torch.where((y.abs() < 8 * step) & (step > 2.0 ** -9), step / 2, step))
                part.copy_(torch.round(y / step) * step)
            z = (z, scale)
        elif case["out"] == "int8":
            top = z.abs().amax(1, keepdim=True)
            z = torch.where(top > 0, torch.round(z * (127 / top.clamp(min=1e-30))) * (top / 127), 0.0)
        return z if s["h"] is None else (z, r)
    T, D, rot = case["T"], case["D"], case["rot"]
    o = s["x"].double()
    turns = s["at"].double()[:, None] * (s["f"] / (2 * math.pi))
    wave = torch.polar(torch.full_like(turns, s["factor"]), 2 * math.pi * (turns - torch.round(turns)))[:, None]
    if s["next"]:
        pair = torch.view_as_complex(o[..., :rot].reshape(T, -1, rot // 2, 2).contiguous())
        o[..., :rot] = torch.view_as_real(pair * wave).reshape(T, -1, rot)
    else:
        pair = torch.complex(o[..., :rot // 2].contiguous(), o[..., rot // 2:rot].contiguous()) * wave
        o[..., :rot // 2], o[..., rot // 2:rot] = pair.real, pair.imag
    return o
