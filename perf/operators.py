"""Performance cases of the operators around the quantized linear layer: what a transformer block runs between its products.

Kinds of a case
  gemm      MXFP4 product with its epilogue: z = A B^T + bias, d = act(z) * multiplier + residual, z kept for a backward pass
  act_bwd   backward of that epilogue: dz = dy * multiplier * act'(z), the multiplier's gradient, the bias's gradient
  norm      root-mean-square norm of x or of the residual stream with x added, result as bf16, MXFP8 or MXFP4 operand
  norm_bwd  its backward: gradients of the stream and of the weight
  clip      global norm of many gradient tensors and their copies scaled to a largest norm (fp32 main gradients)

Where `own` is false the operators run in their plain form: elementary torch operations in 32 bits, sums over many rows in 64.
Codes are returned as the values they stand for: E4M3 bytes and E8M0 scale bytes under torch's types of those formats, E2M1 codes one by
one as E4M3 values (every E2M1 value is one).
"""
import math

import torch

own = False

DEVICE = "cuda:0"
MAX_PRODUCT = 16384 * 4096 * 11008      # m * n * k of the largest listed product
MAX_VALUES = 16384 * 11008              # rows * columns of the largest elementwise case
GELU_C, GELU_A = math.sqrt(2.0 / math.pi), 0.044715


def listed():
    return [
        # A decode batch's gate projection of a 7B-shaped MLP: silu of the product times the up projection; reads the 4-bit weights once.
        dict(name="gemm_24x4096x11008_gate", kind="gemm", m=24, n=11008, k=4096, act="silu", bias="", mul=True, res="", pre=False, out="bf16"),
        # Training forward of a GELU MLP with bias on a ragged number of tokens, z kept for the backward pass.
        dict(name="gemm_1003x2048x5632_gelu", kind="gemm", m=1003, n=5632, k=2048, act="gelu", bias="bf16", mul=False, res="", pre=True, out="bf16"),
        # Attention output projection of a 2048-wide model added to an fp32 residual stream.
        dict(name="gemm_4096x2048x2048_res32", kind="gemm", m=4096, n=2048, k=2048, act="none", bias="", mul=False, res="f32", pre=False, out="f32"),
        # Down projection of a 7B-shaped MLP over a full training batch, added to the bf16 residual stream.
        dict(name="gemm_16384x11008x4096_res", kind="gemm", m=16384, n=4096, k=11008, act="none", bias="", mul=False, res="bf16", pre=False, out="bf16"),
        # Backward of the gated MLP of that batch: both branches' gradients.
        dict(name="act_bwd_16384x11008_gate", kind="act_bwd", m=16384, n=11008, act="silu", mul=True, dbias=False),
        # Backward of the ragged GELU MLP: column sums for the bias beside the elementwise part.
        dict(name="act_bwd_1003x5632_gelu", kind="act_bwd", m=1003, n=5632, act="gelu", mul=False, dbias=True),
        # One decoded token: a single row, latency decides.
        dict(name="norm_1x4096_mxfp8", kind="norm", rows=1, n=4096, x="bf16", res="bf16", w="bf16", out="mxfp8", rstd=False),
        # A small layer's tokens (no power of two) on an fp32 stream into the MXFP4 operand.
        dict(name="norm_2336x1376_mxfp4", kind="norm", rows=2336, n=1376, x="bf16", res="f32", w="f32", out="mxfp4", rstd=True),
        # Prefill or a training batch at 7B width, 8-bit operand with scales.
        dict(name="norm_16384x4096_mxfp8", kind="norm", rows=16384, n=4096, x="bf16", res="bf16", w="bf16", out="mxfp8", rstd=False),
        # Backward of the norm of a 2048-wide model on an fp32 stream, with the gradient that arrives along the stream.
        dict(name="norm_bwd_8192x2048", kind="norm_bwd", rows=8192, n=2048, h="f32", w="bf16", dh=True),
        # Gradients of a small model's layers (the 288 x 320 x 352 layer's size and vectors beside it): launches decide.
        dict(name="clip_small", kind="clip", sizes="112640,101376,92160,352,320,288,320,1,0,1003", g="f32", out="f32", max_norm=1.0),
        # One layer of a 7B-shaped model: bf16 weight gradients of its seven products into fp32 main gradients.
        dict(name="clip_layer_7b", kind="clip", sizes="16777216,16777216,16777216,16777216,45088768,45088768,45088768,4096,4096", g="bf16", out="f32", max_norm=1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["gemm", "gemm", "act_bwd", "norm", "norm", "norm_bwd", "clip"])
    if kind == "gemm":
        while True:
            m, n, k = _log(rng, 1, 16384), _log(rng, 8, 11008), 32 * _log(rng, 1, 344)
            if rng.random() < 0.6:
                n = max(8, n // 8 * 8)
            if m * n * k <= MAX_PRODUCT:
                break
        return dict(kind=kind, m=m, n=n, k=k, act=rng.choice(["none", "relu", "gelu", "silu"]), bias=rng.choice(["", "bf16", "f32"]),
                    mul=rng.random() < 0.3, res=rng.choice(["", "bf16", "f32"]), pre=rng.random() < 0.3, out=rng.choice(["bf16", "bf16", "f32"]))
    if kind == "act_bwd":
        while True:
            m, n = _log(rng, 1, 16384), _log(rng, 8, 11008)
            if m * n <= MAX_VALUES:
                break
        return dict(kind=kind, m=m, n=n, act=rng.choice(["none", "relu", "gelu", "silu"]), mul=rng.random() < 0.5, dbias=rng.random() < 0.6)
    if kind == "norm":
        out = rng.choice(["bf16", "mxfp8", "mxfp8", "mxfp4"])
        rows, n = _log(rng, 1, 16384), _log(rng, 32, 8192)
        if out != "bf16":
            n = max(32, n // 32 * 32)
        return dict(kind=kind, rows=rows, n=n, x=rng.choice(["bf16", "f32"]), res=rng.choice(["", "bf16", "f32"]), w=rng.choice(["bf16", "f32"]),
                    out=out, rstd=rng.random() < 0.5)
    if kind == "norm_bwd":
        return dict(kind=kind, rows=_log(rng, 1, 16384), n=_log(rng, 32, 8192), h=rng.choice(["bf16", "f32"]), w=rng.choice(["bf16", "f32"]),
                    dh=rng.random() < 0.7)
    sizes = [_log(rng, 1, 1 << 23) for _ in range(_log(rng, 1, 200))]
    while sum(sizes) > MAX_VALUES:
        sizes.pop()
    return dict(kind=kind, sizes=",".join(map(str, sizes)), g=rng.choice(["bf16", "f32"]), out=rng.choice(["f32", "f32", "bf16"]),
                max_norm=rng.choice([1.0, 1e9]))


# ---------------------------------------------------------------------------------------------- formats, plain

def _dtype(name):
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def _up(v, to):
    return (v + to - 1) // to * to


def _tile_scales(e):
    """E8M0 bytes [rows, groups] in the tiled layout of include/quartet.h; bytes that stand for nothing are 0."""
    rows, groups = e.shape
    t = torch.zeros((_up(rows, 32), _up(groups, 8)), dtype=torch.uint8, device=e.device)
    t[:rows, :groups] = e
    return t.view(_up(rows, 32) // 32, 32, _up(groups, 8) // 8, 4, 2).permute(0, 2, 4, 1, 3).contiguous().view(-1)


def _untile_scales(t, rows, groups):
    t = t.view(_up(rows, 32) // 32, _up(groups, 8) // 8, 2, 32, 4).permute(0, 3, 1, 4, 2)
    return t.reshape(_up(rows, 32), _up(groups, 8))[:rows, :groups]


def _exp2(e):
    """2^e of integers in -126 .. 127, exactly"""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _exponent(v):
    """biased exponents of fp32 values"""
    return (v.view(torch.int32) >> 23) & 255


def _mxfp8(y):
    """E4M3 values [rows, n] and E8M0 bytes [rows, n / 32] of fp32 values"""
    rows, n = y.shape
    g = y.view(rows, n // 32, 32)
    b = (_exponent(g.abs().amax(2)) - 8).clamp_min(0)
    v = (g * _exp2(127 - b)[..., None]).clamp(-448.0, 448.0)
    return v.view(rows, n).to(torch.float8_e4m3fn), b.to(torch.uint8)


def _hadamard32(device, dtype):
    i = torch.arange(32, device=device)
    bits = i[:, None] & i[None, :]
    parity = (bits ^ (bits >> 1) ^ (bits >> 2) ^ (bits >> 3) ^ (bits >> 4)) & 1
    return 1.0 - 2.0 * parity.to(dtype)


def _mxfp4(y):
    """E2M1 values [rows, n] (fp32) and E8M0 bytes of the forward quantizer's rule: rotate, scale by the root mean square, round"""
    rows, n = y.shape
    h = (y.view(-1, 32) @ _hadamard32(y.device, torch.float32)) * (1.0 / math.sqrt(32.0))
    ss = (h * h).sum(1)
    e = torch.where(_exponent(ss) > 0, torch.div(_exponent(ss) - 127 - 6, 2, rounding_mode="floor"), torch.zeros_like(_exponent(ss)))
    v = h * _exp2(-e)[:, None]
    a = v.abs()
    step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
    v = torch.copysign((torch.round(a / step) * step).clamp_max(6.0), v)
    return v.view(rows, n), (e + 127).to(torch.uint8).view(rows, n // 32)


def _pack_e2m1(v):
    a = v.abs()
    code = (a >= 0.5).to(torch.uint8) + (a >= 1.0) + (a >= 1.5) + (a >= 2.0) + (a >= 3.0) + (a >= 4.0) + (a >= 6.0)
    code = code + 8 * torch.signbit(v).to(torch.uint8)
    return (code[:, 0::2] | (code[:, 1::2] << 4)).to(torch.uint8)


def _decode_mxfp4(codes, scales, rows, k):
    """fp32 values of an MXFP4 operand"""
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    both = torch.stack((codes & 15, codes >> 4), 2).view(rows, k).int()
    s = _exp2(_untile_scales(scales, rows, k // 32).int() - 127)
    return (table[both].view(rows, k // 32, 32) * s[..., None]).view(rows, k)


def _sigmoid(v):
    return 1.0 / (1.0 + torch.exp(-v))


def _act(z, act):
    if act == "relu":
        return torch.maximum(z, torch.zeros_like(z))
    if act == "gelu":
        return z * _sigmoid(2.0 * GELU_C * (z + GELU_A * z * z * z))
    return z * _sigmoid(z) if act == "silu" else z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        s = _sigmoid(2.0 * GELU_C * (z + GELU_A * z * z * z))
        return s + z * s * (1.0 - s) * 2.0 * GELU_C * (1.0 + 3.0 * GELU_A * z * z)
    if act == "silu":
        s = _sigmoid(z)
        return s + z * s * (1.0 - s)
    return torch.ones_like(z)


# ---------------------------------------------------------------------------------------------- inputs

def _buffer(rows, n, dtype):
    """rows of n values, leading dimension a multiple of 8"""
    return torch.zeros((rows, _up(n, 8)), dtype=dtype, device=DEVICE)


def _values(gen, rows, n, dtype, scale=1.0, outliers=False):
    v = torch.randn((rows, _up(n, 8)), generator=gen, device=DEVICE) * scale
    if outliers:      # a few wide columns, as activations have them
        v = v * torch.exp(torch.randn((1, v.shape[1]), generator=gen, device=DEVICE))
    return v.to(dtype)


def prepare(case, seed):
    c, gen = case, torch.Generator(device=DEVICE).manual_seed(seed)
    s = {"case": c}
    bf16, f32 = torch.bfloat16, torch.float32
    if c["kind"] == "gemm":
        m, n, k = c["m"], c["n"], c["k"]
        for name, rows, scale in (("a", m, 1.0), ("b", n, k ** -0.5)):
            v, e = _mxfp4(torch.randn((rows, k), generator=gen, device=DEVICE) * scale)
            s[name], s[name + "s"] = _pack_e2m1(v), _tile_scales(e)
        s["bias"] = torch.randn(n, generator=gen, device=DEVICE).to(_dtype(c["bias"])) if c["bias"] else None
        s["mul"] = _values(gen, m, n, bf16) if c["mul"] else None
        s["res"] = _values(gen, m, n, _dtype(c["res"])) if c["res"] else None
        s["d"] = _buffer(m, n, _dtype(c["out"]))
        s["pre"] = _buffer(m, n, bf16) if c["pre"] else None
    elif c["kind"] == "act_bwd":
        m, n = c["m"], c["n"]
        s["dy"], s["pre"] = _values(gen, m, n, bf16, 1e-3), _values(gen, m, n, bf16)
        s["mul"] = _values(gen, m, n, bf16) if c["mul"] else None
        s["dz"] = _buffer(m, n, bf16)
        s["dmul"] = _buffer(m, n, bf16) if c["mul"] else None
        s["dbias"] = torch.zeros(n, device=DEVICE) if c["dbias"] else None
    elif c["kind"] == "norm":
        rows, n = c["rows"], c["n"]
        s["x"] = _values(gen, rows, n, _dtype(c["x"]), 1.0, True)
        s["res"] = _values(gen, rows, n, _dtype(c["res"]), 3.0, True) if c["res"] else None
        s["w"] = (1.0 + 0.1 * torch.randn(n, generator=gen, device=DEVICE)).to(_dtype(c["w"]))
        s["h"] = _buffer(rows, n, _dtype(c["res"])) if c["res"] else None
        s["rstd"] = torch.zeros(rows, device=DEVICE) if c["rstd"] else None
        s["y"] = _buffer(rows, n, bf16) if c["out"] == "bf16" else None
        if c["out"] != "bf16":
            s["codes"] = torch.zeros((rows, n if c["out"] == "mxfp8" else n // 2), dtype=torch.uint8, device=DEVICE)
            s["scales"] = torch.zeros(_up(rows, 32) // 32 * (_up(n, 256) // 256) * 256, dtype=torch.uint8, device=DEVICE)
            values = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=DEVICE).to(torch.float8_e4m3fn).view(torch.uint8).int()
            pair = torch.arange(256, device=DEVICE)
            s["pairs"] = (values[pair & 15] | (values[pair >> 4] << 8)).to(torch.int16)     # the two E4M3 values of a byte of E2M1 codes
    elif c["kind"] == "norm_bwd":
        rows, n, h = c["rows"], c["n"], _dtype(c["h"])
        s["dy"], s["h"] = _values(gen, rows, n, bf16, 1e-2), _values(gen, rows, n, h, 3.0, True)
        s["w"] = (1.0 + 0.1 * torch.randn(n, generator=gen, device=DEVICE)).to(_dtype(c["w"]))
        s["rstd"] = (s["h"][:, :n].double().square().mean(1) + 1e-5).rsqrt().float()
        s["dh"] = _values(gen, rows, n, h, 1e-2) if c["dh"] else None
        s["dx"], s["dw"] = _buffer(rows, n, h), torch.zeros(n, device=DEVICE)
        s["dx16"] = _buffer(rows, n, bf16) if c["h"] == "f32" else None
    else:
        sizes = [int(v) for v in c["sizes"].split(",")]
        s["g"] = [(torch.randn(v, generator=gen, device=DEVICE) * 1e-2).to(_dtype(c["g"])) for v in sizes]
        # the copies lie in one buffer, as main gradients do; each starts at a multiple of eight values
        s["flat"] = torch.zeros(sum(_up(v, 8) for v in sizes), dtype=_dtype(c["out"]), device=DEVICE)
        s["out"] = [piece[:v] for piece, v in zip(s["flat"].split([_up(v, 8) for v in sizes]), sizes)]
        s["norm"] = torch.zeros(1, device=DEVICE)
    return s


# ---------------------------------------------------------------------------------------------- one pass

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _workspace(s, size):
    """kept with the state, as a program keeps it between its steps"""
    if "ws" not in s:
        s["ws"] = torch.empty(max(16, size), dtype=torch.uint8, device=DEVICE)
    return s["ws"], s["ws"].numel()


def _run_own(s):
    from paper_2505_14669_amd import block as q
    c = s["case"]
    code = lambda t: q.QUARTET_DTYPE_F32 if t is None or t.dtype == torch.float32 else q.QUARTET_DTYPE_BF16
    ld = lambda t: 0 if t is None else t.shape[1]
    if c["kind"] == "gemm":
        n = c["n"]
        q.check(q.quartet_mxfp4_gemm_act(s["a"], s["as"], s["b"], s["bs"], c["m"], n, c["k"], 1.0, s["bias"], code(s["bias"]), q.ACTIVATIONS[c["act"]],
                                         s["mul"], ld(s["mul"]), s["res"], code(s["res"]), ld(s["res"]), s["pre"], ld(s["pre"]), s["d"],
                                         code(s["d"]), ld(s["d"])))
        return {"d": s["d"][:, :n], "pre": None if s["pre"] is None else s["pre"][:, :n]}
    if c["kind"] == "act_bwd":
        n = c["n"]
        q.check(q.quartet_act_bwd(s["dy"], ld(s["dy"]), s["pre"], ld(s["pre"]), s["mul"], ld(s["mul"]), c["m"], n, q.ACTIVATIONS[c["act"]], s["dz"],
                                  ld(s["dz"]), s["dmul"], ld(s["dmul"]), s["dbias"], *_workspace(s, q.quartet_act_bwd_workspace_bytes(c["m"], n))))
        return {"dz": s["dz"][:, :n], "dmul": None if s["dmul"] is None else s["dmul"][:, :n], "dbias": s["dbias"]}
    if c["kind"] == "norm":
        n, four = c["n"], c["out"] == "mxfp4"
        codes, scales = s.get("codes"), s.get("scales")
        fmt = q.QUARTET_FORMAT_NONE if c["out"] == "bf16" else q.QUARTET_FORMAT_MXFP4 if four else q.QUARTET_FORMAT_MXFP8
        q.check(q.quartet_rmsnorm_fwd(s["x"], code(s["x"]), ld(s["x"]), s["res"], ld(s["res"]), c["rows"], n, s["w"], code(s["w"]), 1e-5, s["h"],
                                      code(s["h"]), ld(s["h"]), s["y"], ld(s["y"]), fmt, codes, scales, None, s["rstd"]))
        if four:
            codes = s["pairs"][codes.int()].view(torch.uint8)
        return {"h": None if s["h"] is None else s["h"][:, :n], "y": None if s["y"] is None else s["y"][:, :n], "rstd": s["rstd"],
                "codes": None if codes is None else codes.view(torch.float8_e4m3fn), "scales": None if scales is None else scales.view(torch.float8_e8m0fnu)}
    if c["kind"] == "norm_bwd":
        n = c["n"]
        q.check(q.quartet_rmsnorm_bwd(s["dy"], ld(s["dy"]), s["h"], code(s["h"]), ld(s["h"]), c["rows"], n, s["w"], code(s["w"]), s["rstd"], s["dh"],
                                      ld(s["dh"]), s["dx"], ld(s["dx"]), s["dx16"], ld(s["dx16"]), s["dw"],
                                      *_workspace(s, q.quartet_rmsnorm_bwd_workspace_bytes(c["rows"], n))))
        return {"dx": s["dx"][:, :n], "dx16": None if s["dx16"] is None else s["dx16"][:, :n], "dw": s["dw"]}
    if "list" not in s:
        s["list"] = q.grad_tensors(s["g"], s["out"])
    q.check(q.quartet_grad_clip(s["list"], len(s["list"]), c["max_norm"], s["norm"], *_workspace(s, q.quartet_grad_clip_workspace_bytes())))
    return {"norm": s["norm"], "out": s["flat"]}


def _run_plain(s):
    c = s["case"]
    if c["kind"] == "gemm":
        m, n, k = c["m"], c["n"], c["k"]
        z = _decode_mxfp4(s["a"], s["as"], m, k) @ _decode_mxfp4(s["b"], s["bs"], n, k).t()
        if s["bias"] is not None:
            z = z + s["bias"].float()
        d = _act(z, c["act"])
        if s["mul"] is not None:
            d = d * s["mul"][:, :n].float()
        if s["res"] is not None:
            d = d + s["res"][:, :n].float()
        return {"d": d.to(_dtype(c["out"])), "pre": z.to(torch.bfloat16) if c["pre"] else None}
    if c["kind"] == "act_bwd":
        n = c["n"]
        dy, z = s["dy"][:, :n].float(), s["pre"][:, :n].float()
        da = dy if s["mul"] is None else dy * s["mul"][:, :n].float()
        dz = da * _act_slope(z, c["act"])
        return {"dz": dz.to(torch.bfloat16), "dmul": None if s["mul"] is None else (dy * _act(z, c["act"])).to(torch.bfloat16),
                "dbias": dz.double().sum(0).float() if c["dbias"] else None}
    if c["kind"] == "norm":
        rows, n = c["rows"], c["n"]
        h = s["x"][:, :n].float()
        if s["res"] is not None:
            h = (h + s["res"][:, :n].float()).to(s["res"].dtype)      # the stream's own type: what the norm reads is what the stream holds
        hf = h.float()
        rstd = 1.0 / torch.sqrt((hf * hf).sum(1) / n + 1e-5)
        y = hf * rstd[:, None] * s["w"].float()
        codes = scales = None
        if c["out"] == "mxfp8":
            codes, e = _mxfp8(y)
            scales = _tile_scales(e).view(torch.float8_e8m0fnu)
        elif c["out"] == "mxfp4":
            v, e = _mxfp4(y)
            codes, scales = v.to(torch.float8_e4m3fn), _tile_scales(e).view(torch.float8_e8m0fnu)
        return {"h": None if s["res"] is None else h, "y": y.to(torch.bfloat16) if c["out"] == "bf16" else None, "rstd": rstd if c["rstd"] else None,
                "codes": codes, "scales": scales}
    if c["kind"] == "norm_bwd":
        n = c["n"]
        dy, h, r = s["dy"][:, :n].float(), s["h"][:, :n].float(), s["rstd"][:, None]
        g = dy * s["w"].float()
        dx = r * (g - h * (r * r) * ((g * h).sum(1, keepdim=True) / n))
        if s["dh"] is not None:
            dx = dx + s["dh"][:, :n].float()
        return {"dx": dx.to(s["h"].dtype), "dx16": dx.to(torch.bfloat16) if s["dx16"] is not None else None,
                "dw": (dy * h * r).double().sum(0).float()}
    total = torch.stack([g.double().square().sum() for g in s["g"]]).sum().sqrt().float()
    scale = (c["max_norm"] / (total + 1e-6)).clamp_max(1.0)
    flat = torch.cat([torch.nn.functional.pad(g, (0, -g.numel() % 8)) for g in s["g"]])
    return {"norm": total.view(1), "out": (flat.float() * scale).to(_dtype(c["out"]))}


# ---------------------------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    c = case
    size = lambda name: {"": 0, "bf16": 2, "f32": 4}[name]
    if c["kind"] == "gemm":
        m, n, k = c["m"], c["n"], c["k"]
        per = 2 * c["mul"] + size(c["res"]) + 2 * c["pre"] + size(c["out"])
        return {"bytes": (m + n) * k * (0.5 + 1 / 32) + m * n * per + n * size(c["bias"]), "flops": 2.0 * m * n * k}
    if c["kind"] == "act_bwd":
        return {"bytes": c["m"] * c["n"] * (6 + 4 * c["mul"]) + 4 * c["n"] * c["dbias"], "flops": 20.0 * c["m"] * c["n"]}
    if c["kind"] == "norm":
        out = {"bf16": 2.0, "mxfp8": 1 + 1 / 32, "mxfp4": 0.5 + 1 / 32}[c["out"]]
        return {"bytes": c["rows"] * c["n"] * (size(c["x"]) + 2 * size(c["res"]) + out) + 4 * c["rows"] * c["rstd"] + c["n"] * size(c["w"]),
                "flops": 6.0 * c["rows"] * c["n"]}
    if c["kind"] == "norm_bwd":
        per = 2 + size(c["h"]) * (2 + c["dh"]) + 2 * (c["h"] == "f32")
        return {"bytes": c["rows"] * c["n"] * per + 4 * c["rows"] + c["n"] * (4 + size(c["w"])), "flops": 12.0 * c["rows"] * c["n"]}
    values = sum(int(v) for v in c["sizes"].split(","))
    return {"bytes": values * (size(c["g"]) + size(c["out"])), "flops": 3.0 * values}


# ---------------------------------------------------------------------------------------------- from the definitions, in 64 bits

def _exact_operand(codes, scales, rows, k):
    """code s e1 e0 m: (-1)^s m / 2 for e = 0, else (-1)^s (1 + m / 2) 2^(e - 1); scale 2^(b - 127) of row r and group g at its tiled place"""
    c = torch.empty((rows, k), dtype=torch.int64, device=codes.device)
    c[:, 0::2], c[:, 1::2] = (codes % 16).long(), (codes // 16).long()
    sign, e, man = 1.0 - 2.0 * (c // 8), (c // 2) % 4, (c % 2).double()
    v = sign * torch.where(e == 0, man / 2, torch.ldexp(1 + man / 2, e - 1))
    r, g, kq = torch.arange(rows, device=codes.device)[:, None], torch.arange(k // 32, device=codes.device)[None, :], (k + 255) // 256
    at = ((r // 32) * kq + g // 8) * 256 + ((g % 2) * 32 + r % 32) * 4 + (g % 8) // 2
    b = scales.long()[at]
    return v * torch.ldexp(torch.ones_like(b, dtype=torch.float64), b - 127).repeat_interleave(32, 1)


def _exact_act(z, act):
    """value and slope"""
    if act == "relu":
        return torch.where(z > 0, z, 0.0), torch.where(z > 0, 1.0, 0.0).double()
    if act == "gelu":
        t = torch.tanh(GELU_C * (z + GELU_A * z ** 3))
        return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * GELU_C * (1 + 3 * GELU_A * z ** 2)
    if act == "silu":
        t = torch.sigmoid(z)
        return z * t, t * (1 + z * (1 - t))
    return z, torch.ones_like(z)


def _exact_tiles(b, rows, groups):
    kq = (groups + 7) // 8
    out = torch.zeros(((rows + 31) // 32) * kq * 256, dtype=torch.float64, device=b.device) + 2.0 ** -127
    r, g = torch.arange(rows, device=b.device)[:, None], torch.arange(groups, device=b.device)[None, :]
    out[(((r // 32) * kq + g // 8) * 256 + ((g % 2) * 32 + r % 32) * 4 + (g % 8) // 2).reshape(-1)] = torch.ldexp(torch.ones_like(b), (b - 127).long()).reshape(-1)
    return out


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "gemm":
        m, n, k = c["m"], c["n"], c["k"]
        z = _exact_operand(s["a"], s["as"], m, k) @ _exact_operand(s["b"], s["bs"], n, k).t()
        z = z if s["bias"] is None else z + s["bias"].double()
        d = _exact_act(z, c["act"])[0]
        d = d if s["mul"] is None else d * s["mul"][:, :n].double()
        return {"d": d if s["res"] is None else d + s["res"][:, :n].double(), "pre": z if c["pre"] else None}
    if c["kind"] == "act_bwd":
        n = c["n"]
        dy = s["dy"][:, :n].double()
        value, slope = _exact_act(s["pre"][:, :n].double(), c["act"])
        dz = slope * dy if s["mul"] is None else slope * dy * s["mul"][:, :n].double()
        return {"dz": dz, "dmul": None if s["mul"] is None else dy * value, "dbias": dz.sum(0) if c["dbias"] else None}
    if c["kind"] == "norm":
        rows, n = c["rows"], c["n"]
        h = s["x"][:, :n].double()
        if s["res"] is not None:
            h = (h + s["res"][:, :n].double()).to(s["res"].dtype).double()
        rstd = ((h ** 2).mean(1) + 1e-5) ** -0.5
        y = h * rstd[:, None] * s["w"].double()
        codes = scales = None
        if c["out"] != "bf16":
            g = y.reshape(rows, n // 32, 32)
            if c["out"] == "mxfp8":
                top = g.abs().amax(2)
                e = torch.frexp(top).exponent.double() - 1 - 8                        # the largest magnitude in [2^8, 2^9)
                v = torch.ldexp(g, -e[..., None]).clamp(-448, 448)
                fine = torch.ldexp(torch.ones_like(v), (torch.frexp(v).exponent - 1).clamp_min(-6) - 3)
                codes = torch.round(v / fine) * fine
            else:
                for d in (1, 2, 4, 8, 16):
                    p = g.reshape(rows, n // 32, 16 // d, 2, d)
                    g = torch.stack((p[..., 0, :] + p[..., 1, :], p[..., 0, :] - p[..., 1, :]), 3).reshape(rows, n // 32, 32)
                g = g / math.sqrt(32)
                ss = (g ** 2).sum(2)
                e = torch.where(ss > 0, torch.floor((torch.frexp(ss).exponent.double() - 1 - 6) / 2), 0.0)
                v = torch.ldexp(g, -e[..., None])
                grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=v.device)
                at = torch.bucketize(v.abs().contiguous(), (grid[1:] + grid[:-1]) / 2)
                codes = grid[at] * torch.sign(v)
            codes, scales = codes.reshape(rows, n), _exact_tiles(e + 127, rows, n // 32)
        return {"h": None if s["res"] is None else h, "y": y if c["out"] == "bf16" else None, "rstd": rstd if c["rstd"] else None,
                "codes": codes, "scales": scales}
    if c["kind"] == "norm_bwd":
        n = c["n"]
        dy, h, r, w = s["dy"][:, :n].double(), s["h"][:, :n].double(), s["rstd"].double()[:, None], s["w"].double()
        dx = r * dy * w - r ** 3 * h * (dy * w * h).mean(1, keepdim=True)
        dx = dx if s["dh"] is None else dx + s["dh"][:, :n].double()
        return {"dx": dx, "dx16": dx if s["dx16"] is not None else None, "dw": (dy * h * r).sum(0)}
    total = sum(float((g.double() ** 2).sum()) for g in s["g"]) ** 0.5
    scale = min(1.0, c["max_norm"] / (total + 1e-6))
    out = torch.zeros(s["flat"].numel(), dtype=torch.float64, device=DEVICE)
    at = 0
    for g in s["g"]:
        out[at:at + g.numel()] = g.double() * scale
        at += (g.numel() + 7) // 8 * 8
    return {"norm": torch.tensor([total], dtype=torch.float64), "out": out}
