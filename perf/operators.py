"""Workloads of the operators around the attention: the norm in front of it and the 8-bit projections of a sampler.

A transformer block adds what the block before it computed to the residual stream and normalises the sum (RMSNorm, with
or without a learnable scale).  In training the tangent runs along, and the backward goes through both outputs; a
sampler needs neither, and takes the normalised rows in 8 bits, with a scale for each token, into products with weights
that have a scale for each channel.  Widths: 1152 = 16 x 72 (DiT-XL/2), 1024 = 16 x 64 and 768 = 12 x 64 (the other head
layouts of the workloads), 3456 = 3 x 1152 and 4608 = 4 x 1152 (fused QKV projection, MLP), generic wide ones beyond.

A case: op    "norm"      h = x + res, y = RMSNorm(h) g, and with tan the tangents th, ty
              | "norm_bwd"  the cotangents of y, h (and ty, th) back to x (and tx) and g
              | "norm8"     h = x + res, RMSNorm(h) g in 8 bits with a scale for each token
              | "linear8"   product of 8-bit rows with 8-bit weights, scales and bias
              | "proj8"     norm8, then linear8: a block's input, normalised and projected
              | "out8"      rows to 8 bits, then linear8: the attention's output, projected
        rows, D   tokens, and their width;  N  output channels of a product
        dtype     "bf16" | "fp32" of the rows (for linear8: of its output)
        tan, res, scale, bias   whether there are tangents, a residual, a learnable scale g, a bias
"""
import math

import torch

own = False

OPS = ("norm", "norm_bwd", "norm8", "linear8", "proj8", "out8")
EPS = 1e-6
_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _norm(name, op, rows, D, dtype="bf16", tan=True, res=True, scale=True):
    return {"name": name, "op": op, "rows": rows, "D": D, "dtype": dtype, "tan": tan, "res": res, "scale": scale}


def _product(name, op, rows, D, N, dtype="bf16", bias=True, res=True, scale=True):
    return {"name": name, "op": op, "rows": rows, "D": D, "N": N, "dtype": dtype, "bias": bias, "res": res, "scale": scale}


def listed():
    return [
        # one DiT-XL/2 layer on 512-pixel latents in training: the residual sum, its norm, and their tangents; no learnable
        # scale, since the block's modulation has its own
        _norm("dit512_norm", "norm", 16 * 1024, 1152, scale=False),
        # odd rows and an odd width, in the checking precision, primal only
        _norm("odd_norm_fp32", "norm", 5003, 1151, "fp32", tan=False),
        # the backward of the first one, with a scale to be learned; and that of a small batch without tangents
        _norm("dit512_norm_bwd", "norm_bwd", 16 * 1024, 1152),
        _norm("cross_norm_bwd", "norm_bwd", 8 * 333, 768, tan=False),
        # the same norm in a sampler, its result in 8 bits; and one token of a wide model, where latency counts
        _norm("dit512_norm8", "norm8", 16 * 1024, 1152, tan=False, scale=False),
        _norm("token_norm8", "norm8", 1, 8192, tan=False),
        # fused QKV projection of DiT-XL/2, 512-pixel latents; the first layer of its MLP over a larger batch
        _product("dit512_qkv8", "linear8", 16 * 1024, 1152, 3456),
        _product("dit256_mlp8", "linear8", 256 * 256, 1152, 4608, bias=False),
        # one token against a wide layer: the weights' bytes are all there is; and a ragged handful, results in fp32
        _product("token_linear8", "linear8", 1, 4096, 14336, bias=False),
        _product("ragged_linear8", "linear8", 77, 1000, 2303, "fp32"),
        # a block's input in a sampler (residual, norm, 8 bits, QKV), and the attention's output back into the stream
        _product("dit256_proj8", "proj8", 64 * 256, 1152, 3456),
        _product("cross_out8", "out8", 8 * 1000, 768, 768),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


#: The most one drawn case may have: elements of one tensor of rows, and multiply-adds of a product.
_MOST_ELEMENTS, _MOST_MACS = 2.0e7, 3.0e11


def draw(rng):
    while True:
        op = rng.choice(OPS)
        rows = _log(rng, 1, 65536)
        D = rng.choice((512, 768, 1024, 1152, 1152, 2048, 4096, 8192)) if rng.random() < 0.6 else _log(rng, 32, 8192)
        if rows * D > _MOST_ELEMENTS:
            continue
        flip = lambda: rng.random() < 0.5  # noqa: E731
        if op in ("norm", "norm_bwd", "norm8"):
            tan = op != "norm8" and flip()
            return {"op": op, "rows": rows, "D": D, "dtype": rng.choice(("bf16", "bf16", "fp32")), "tan": tan, "res": flip(), "scale": flip()}
        N = rng.choice((768, 1024, 1152, 3456, 4608, 8192)) if rng.random() < 0.6 else _log(rng, 32, 16384)
        if rows * N <= 16 * _MOST_ELEMENTS and 1.0 * rows * N * D <= _MOST_MACS:
            # rounding an activation to 8 bits makes near ties of it, whose two sides an fp32 result would tell apart
            dtype = rng.choice(("bf16", "bf16", "fp32")) if op == "linear8" else "bf16"
            return {"op": op, "rows": rows, "D": D, "N": N, "dtype": dtype, "bias": flip(), "res": flip(), "scale": flip()}


def _rows8(x):
    """8-bit rows and their scales, in the precision of x: what a user has in hand of weights that were quantised once."""
    s = x.abs().amax(dim=-1) / 127.0
    q = torch.round(x / torch.where(s > 0, s, torch.ones_like(s)).unsqueeze(-1))
    return q.clamp_(-127, 127).to(torch.int8), s


def _pitched(q):
    """The same values with rows that begin on 16 bytes, as an 8-bit matrix is stored for the products."""
    pitch = (q.shape[-1] + 15) // 16 * 16
    if pitch == q.shape[-1]:
        return q
    to = torch.zeros(q.shape[:-1] + (pitch,), dtype=q.dtype, device=q.device)[..., : q.shape[-1]]
    return to.copy_(q)


def prepare(case, seed):
    op, rows, D, dtype = case["op"], case["rows"], case["D"], _TYPES[case["dtype"]]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(9000 + int(seed))

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=gen, device="cuda").mul_(std)

    # the residual stream of a transformer has a few channels much larger than the others
    stream = torch.where(torch.rand(D, generator=gen, device="cuda") < 0.01, 6.0, 1.0)
    s = {"op": op, "x": None, "res": None, "tx": None, "tres": None, "g": None, "bias": None, "dtype": dtype}
    if op in ("norm", "norm8", "proj8"):
        s["x"] = normal(rows, D, std=0.5).to(dtype) if case["res"] else (normal(rows, D) * stream).to(dtype)
        s["res"] = (normal(rows, D) * stream).to(dtype) if case["res"] else None
    if op == "norm" and case["tan"]:
        s["tx"] = normal(rows, D, std=0.5).to(dtype)
        s["tres"] = normal(rows, D, std=0.5).to(dtype) if case["res"] else None
    if op == "norm_bwd":
        s["h"], s["dy"] = (normal(rows, D) * stream).to(dtype), normal(rows, D).to(dtype)
        s["dh"] = normal(rows, D).to(dtype) if case["res"] else None
        s["th"], s["dty"], s["dth"] = None, None, None
        if case["tan"]:
            s["th"], s["dty"] = normal(rows, D, std=0.5).to(dtype), normal(rows, D).to(dtype)
            s["dth"] = normal(rows, D).to(dtype) if case["res"] else None
    if op == "out8":
        s["x"] = normal(rows, D, std=0.3).to(dtype)
    if op in ("norm", "norm_bwd", "norm8", "proj8") and case["scale"]:
        s["g"] = 1.0 + normal(D, std=0.3)
    if op in ("linear8", "proj8", "out8"):
        N = case["N"]
        wq, s["ws"] = _rows8(normal(N, D, std=D ** -0.5))
        s["wq"] = _pitched(wq)
        s["bias"] = normal(N, std=0.1) if case["bias"] else None
        if op == "linear8":
            q, s["s"] = _rows8(normal(rows, D) * stream)
            s["q"] = _pitched(q)
    return s


def _own_run(s):
    from paper_2511_19797_b200 import binding

    op = s["op"]
    if op == "norm":
        return binding.tvm_attn_rmsnorm_jvp_fwd(s["x"], s["res"], s["tx"], s["tres"], s["g"], eps=EPS)
    if op == "norm_bwd":
        return binding.tvm_attn_rmsnorm_jvp_bwd(s["h"], s["dy"], s["th"], s["dty"], s["dh"], s["dth"], s["g"], eps=EPS)
    if op == "linear8":
        return binding.tvm_attn_linear_s8(s["q"], s["s"], s["wq"], s["ws"], s["bias"], dtype=s["dtype"])
    if op == "out8":
        q, sx = binding.tvm_attn_quantize_s8(s["x"])
        return binding.tvm_attn_linear_s8(q, sx, s["wq"], s["ws"], s["bias"])
    q, sx, h = binding.tvm_attn_rmsnorm_s8(s["x"], s["res"], s["g"], eps=EPS)
    if op == "proj8":
        return h, binding.tvm_attn_linear_s8(q, sx, s["wq"], s["ws"], s["bias"])
    # the values that the 8 bits stand for
    return h, torch.mul(q, sx.unsqueeze(-1), out=torch.empty(q.shape, dtype=torch.bfloat16, device=q.device)), sx


def _plain_norm(s):
    """h and the norm's output in 32 bits, with 1 / r."""
    h = s["x"].float()
    if s["res"] is not None:
        h = h + s["res"].float()
    inv = torch.rsqrt(h.square().mean(dim=-1, keepdim=True) + EPS)
    y = h * inv
    return h, y if s["g"] is None else y * s["g"], inv


def _plain_product(q, sx, s):
    y = (q.float() @ s["wq"].float().t()) * sx.unsqueeze(-1) * s["ws"]
    return (y if s["bias"] is None else y + s["bias"]).to(s["dtype"])


def _plain_bwd(s):
    h, dy, D = s["h"].float(), s["dy"].float(), s["h"].shape[-1]
    inv = torch.rsqrt(h.square().mean(dim=-1, keepdim=True) + EPS)
    u = h * inv

    def scaled(v):
        return v if s["g"] is None else v * s["g"]

    def through(v):  # the Jacobian of u, which is symmetric
        return (v - u * (u * v).mean(dim=-1, keepdim=True)) * inv

    dx, dg, dtx = through(scaled(dy)), dy * u, None
    if s["th"] is not None:
        th, dty = s["th"].float(), s["dty"].float()
        b = scaled(dty)
        dtx, jt = through(b), through(th)
        # b . J(h) th differentiated with respect to h
        hb, ht, bt = (h * b).mean(dim=-1, keepdim=True), (h * th).mean(dim=-1, keepdim=True), (b * th).mean(dim=-1, keepdim=True)
        dx = dx + inv ** 3 * (3.0 * hb * ht * inv.square() * h - bt * h - ht * b - hb * th)
        dg = dg + dty * jt
        if s["dth"] is not None:
            dtx = dtx + s["dth"].float()
        dtx = dtx.to(s["dtype"])
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    return dx.to(s["dtype"]), dtx, None if s["g"] is None else dg.sum(dim=0)


def run(s):
    if own:
        return _own_run(s)
    op, dtype = s["op"], s["dtype"]
    if op == "norm_bwd":
        return _plain_bwd(s)
    if op == "linear8":
        return _plain_product(s["q"], s["s"], s)
    if op == "out8":
        q, sx = _rows8(s["x"].float())
        return _plain_product(q, sx, s)
    h, y, inv = _plain_norm(s)
    sum_ = s["x"] if s["res"] is None else h.to(dtype)
    if op == "norm":
        if s["tx"] is None:
            return y.to(dtype), sum_, None, None
        th = s["tx"].float()
        if s["tres"] is not None:
            th = th + s["tres"].float()
        u = h * inv
        ty = (th - u * (u * th).mean(dim=-1, keepdim=True)) * inv
        ty = ty if s["g"] is None else ty * s["g"]
        return y.to(dtype), sum_, ty.to(dtype), s["tx"] if s["tres"] is None else th.to(dtype)
    q, sx = _rows8(y)
    if op == "proj8":
        return sum_, _plain_product(q, sx, s)
    return sum_, (q * sx.unsqueeze(-1)).to(torch.bfloat16), sx


def exact(case, seed):
    """The definitions in 64 bits: norms by division by the root, the backward from sums over the row (not by the Jacobian's
    product form), products of whole numbers, which 64-bit floats hold exactly."""
    s = {k: v.double() if isinstance(v, torch.Tensor) else v for k, v in prepare(case, seed).items()}
    op, D = s["op"], case["D"]

    def dot(a, b):
        return (a * b).sum(dim=-1, keepdim=True)

    def eight(v):
        top = v.abs().amax(dim=-1, keepdim=True)
        step = top / 127
        return torch.where(top > 0, torch.round(v / step), torch.zeros_like(v)), step

    def product(q, step):
        y = torch.mm(q, s["wq"].t()).mul_(step).mul_(s["ws"])
        return y if s["bias"] is None else y.add_(s["bias"])

    if op == "linear8":
        return product(s["q"], s["s"].unsqueeze(-1))
    if op == "out8":
        return product(*eight(s["x"]))
    g = 1.0 if s["g"] is None else s["g"]
    if op == "norm_bwd":
        h, a = s["h"], s["dy"] * g
        r = (dot(h, h) / D + EPS).sqrt()
        dx = a / r - h * dot(a, h) / (D * r ** 3)
        terms, dtx = s["dy"] * h / r, None
        if s["th"] is not None:
            t, b = s["th"], s["dty"] * g
            bh, ht, bt = dot(b, h), dot(h, t), dot(b, t)
            dtx = b / r - h * bh / (D * r ** 3)
            dx = dx - (bt * h + ht * b + bh * t) / (D * r ** 3) + 3 * bh * ht * h / (D * D * r ** 5)
            terms = terms + s["dty"] * (t / r - h * ht / (D * r ** 3))
            dtx = dtx if s["dth"] is None else dtx + s["dth"]
        return dx if s["dh"] is None else dx + s["dh"], dtx, None if s["g"] is None else terms.sum(dim=0)
    h = s["x"] if s["res"] is None else s["x"] + s["res"]
    r = (dot(h, h) / D + EPS).sqrt()
    y = h / r * g
    if op == "norm":
        if s["tx"] is None:
            return y, h, None, None
        t = s["tx"] if s["tres"] is None else s["tx"] + s["tres"]
        return y, h, (t / r - h * dot(h, t) / (D * r ** 3)) * g, t
    q, step = eight(y)
    if op == "proj8":
        return h, product(q, step)
    return h, q * step, step.squeeze(-1)


def work(case):
    """Every input read once and every output written once."""
    op, rows, D = case["op"], case["rows"], case["D"]
    size = 2 if case["dtype"] == "bf16" else 4
    t, n, r = size * rows * D, 2 if case.get("tan") else 1, 1 if case["res"] else 0
    g = 4 * D if case["scale"] else 0
    if op == "norm":       # in x (res), out y (h); the same for the tangents
        return {"bytes": n * (2 + 2 * r) * t + g, "flops": (10 if n == 2 else 5) * rows * D}
    if op == "norm_bwd":   # in h dy (dh), out dx; the same for the tangents; the scale and its gradient
        return {"bytes": n * (3 + r) * t + 2 * g, "flops": (36 if n == 2 else 12) * rows * D}
    if op == "norm8":      # in x (res), out (h), the 8-bit rows and their scales
        return {"bytes": (1 + 2 * r) * t + rows * D + 4 * rows + g, "flops": 8 * rows * D}
    N = case["N"]
    weights, flops = N * D + 4 * N + (4 * N if case["bias"] else 0), 2 * rows * N * D
    if op == "linear8":    # in the 8-bit rows, the weights and the scales, out the product
        return {"bytes": rows * D + 4 * rows + weights + size * rows * N, "flops": flops}
    if op == "out8":       # in the rows and the weights, out the product
        return {"bytes": t + weights + size * rows * N, "flops": flops + 3 * rows * D}
    # in x (res) and the weights, out (h) and the product
    return {"bytes": (1 + 2 * r) * t + g + weights + size * rows * N, "flops": flops + 8 * rows * D}
