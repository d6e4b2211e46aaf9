"""Drop-in linear layer over the C ABI: forward and backward of Algorithm 1 as one autograd function.

Argument marshalling only, and that in native code: every arithmetic step runs in the library's kernels
(quartet_linear_fwd / quartet_linear_bwd).  torch provides device memory, streams and the autograd
graph.  There is no fallback: without a GPU or without the built library these calls raise.

Shapes: the flattened token count, in_features and out_features must be multiples of the Hadamard
block (32, the MXFP4 group, unless a layer asks for 64, 128 or 256).

Around the layer, over include/quartet_block.h: an activation, a gate and a residual in the product's epilogue
(QuartetLinear(activation=...), multiplier=, residual=), the norm of the residual stream (QuartetRMSNorm) and the
clipping of a step's gradients (clip_grad_norm_).
"""
import torch
from torch.autograd.function import once_differentiable

from . import binding as q
from . import block
from . import _nn_native as _native          # fails loudly if it has not been built (python -m paper_2505_14669_amd.build)

_native.set_error(q.QuartetError)


class _PythonFunction(torch.autograd.Function):
    """The node's twin in Python over the same two native halves, for the calls that the native node does not serve (it says which):
    what torch does with an autograd function there, or the reason why it cannot, comes from torch itself."""

    @staticmethod
    def forward(ctx, x, weight, seed, rounding, hadamard_block):
        y, context = _native.forward(x, weight, hadamard_block)
        ctx.save_for_backward(context)
        ctx.call = (tuple(x.shape), weight.shape[0], seed, rounding, hadamard_block)
        return y

    @staticmethod
    def backward(ctx, dy):
        return (*_native.backward(*ctx.saved_tensors, dy, *ctx.call), None, None, None)


class QuartetLinearFunction:
    """y = x W^T with MXFP4 operands (Algorithm 1 Forward); the backward pass returns the gradients of
    Algorithm 1 Backward.  x: [..., in] bf16, weight: [out, in] bf16, seed: python int naming the
    stochastic-rounding draws of this call's backward pass, rounding: 0 stochastic / 1 nearest,
    hadamard_block: 32 (the method), 64, 128 or 256.  The autograd node is native code (csrc/nn_autograd.cpp)."""

    @staticmethod
    def apply(x, weight, seed, rounding, hadamard_block=32):
        call = (x, weight, int(seed), int(rounding), int(hadamard_block))
        y = _native.linear(*call)
        return _PythonFunction.apply(*call) if y is None else y


def _dtype_code(t):
    return q.QUARTET_DTYPE_F32 if t is None or t.dtype == torch.float32 else q.QUARTET_DTYPE_BF16


def _new_rows(shape, dtype, device):
    """A new tensor [..., n] whose rows lie n, rounded up to a multiple of 8, values apart (the kernels' 16-byte accesses).  It has no wider base: torch
    refuses changes in place of a function's results that are views."""
    n = shape[-1]
    if n % 8 == 0:
        return torch.empty(shape, dtype=dtype, device=device)
    strides, step = [1], n + -n % 8
    for size in reversed(shape[:-1]):
        strides.insert(0, step)
        step *= size
    return torch.empty_strided(shape, strides, dtype=dtype, device=device)


def _distance(t):
    """the distance of the rows of a tensor [..., n] if the kernels take it as it lies, else None"""
    n = t.shape[-1]
    if t.data_ptr() % 16:
        return None
    if t.is_contiguous() and n % 8 == 0:
        return n
    if n > 1 and t.stride(-1) != 1:
        return None
    distance = step = None
    for size, stride in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:
            continue
        if distance is None:
            distance = step = stride
        if stride != step:
            return None
        step *= size
    if distance is None:
        return n + -n % 8
    return distance if distance >= n and distance % 8 == 0 else None


def _rows(t):
    """a tensor [..., n] as rows that the kernels take, copied if it is not, and their distance"""
    distance = _distance(t)
    if distance is None:
        t = _new_rows(t.shape, t.dtype, t.device).copy_(t)
        distance = _distance(t)
    return t, distance


def _dense(t):
    """a tensor (or None) with its values side by side from a multiple of 16 bytes on, copied if it is not: a piece of a program's buffer may start anywhere"""
    if t is None:
        return None
    t = t.contiguous()
    return t.clone(memory_format=torch.contiguous_format) if t.data_ptr() % 16 else t


def _address(t):
    """(the binding takes a tensor only where its values lie side by side)"""
    return None if t is None else t.data_ptr()


def _check_tensor(t, name, dtypes, device):
    if not t.is_cuda or t.device != device:
        raise RuntimeError(f"{name} must be on {device}: there is no CPU path")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} must be {' or '.join(str(d) for d in dtypes)}, not {t.dtype}")


_ANY = (torch.bfloat16, torch.float32)


class _EpilogueFunction(torch.autograd.Function):
    """a(x W^T + bias) * multiplier + residual: the layer's operands, its product with the epilogue, and both backward passes.  The gradient of an fp32
    result is rounded to bf16 before the gate, the slope, dmul and dbias (quartet_act_bwd and the layer's backward pass take bf16, and so does the gradient
    that reaches a layer with a bf16 result); the residual's gradient stays as it came."""

    @staticmethod
    def forward(ctx, x, weight, bias, multiplier, residual, seed, rounding, hadamard_block, activation, graph):
        device = x.device
        _check_tensor(x, "x", (torch.bfloat16,), device)
        _check_tensor(weight, "weight", (torch.bfloat16,), device)
        if weight.dim() != 2 or x.dim() < 1 or x.shape[-1] != weight.shape[1]:
            raise ValueError("x [..., in_features] and weight [out_features, in_features] do not fit together")
        out, inf = weight.shape
        if hadamard_block not in (32, 64, 128, 256):
            raise ValueError("hadamard_block must be 32, 64, 128 or 256")
        tokens = x.numel() // inf if inf else 0
        if tokens % hadamard_block or inf % hadamard_block or out % hadamard_block:
            raise ValueError(f"tokens, in_features and out_features must be multiples of {hadamard_block}")
        shape = (*x.shape[:-1], out)
        for name, t, dtypes in (("multiplier", multiplier, (torch.bfloat16,)), ("residual", residual, _ANY)):
            if t is not None:
                _check_tensor(t, name, dtypes, device)
                if tuple(t.shape) != shape:
                    raise ValueError(f"{name} must have the result's shape {tuple(shape)}")
        if bias is not None:
            _check_tensor(bias, "bias", _ANY, device)
            if tuple(bias.shape) != (out,):
                raise ValueError(f"bias must have {out} values")
        ctx.call = (tokens, inf, out, seed, rounding, hadamard_block, activation)
        ctx.like = (x.shape, None if bias is None else bias.dtype, None if residual is None else residual.dtype)
        if inf and not tokens * out:                # no tokens or no features: nothing to multiply, and the library takes no address of nothing
            return torch.empty(shape, dtype=torch.bfloat16 if residual is None else residual.dtype, device=device)
        with torch.cuda.device(device):
            x2, w2, bias2, mul2, res2 = _dense(x), _dense(weight), _dense(bias), _dense(multiplier), _dense(residual)
            byte = dict(dtype=torch.uint8, device=device)
            operands = []
            for t, rows in ((x2, tokens), (w2, out)):
                operands += [torch.empty(max(16, rows * inf // 2), **byte), torch.empty(max(16, q.quartet_scale_bytes(rows, inf)), **byte),
                             torch.empty(max(16, rows * inf // 8), **byte)]
            if hadamard_block == 32:
                q.check(q.quartet_fwd_operands(x2, w2, tokens, inf, out, *operands))
            else:
                q.check(q.quartet_quant_fwd_block(x2, tokens, inf, inf, 0, hadamard_block, *operands[:3]))
                q.check(q.quartet_quant_fwd_block(w2, out, inf, inf, 0, hadamard_block, *operands[3:]))
            # z is kept for a backward pass only (needs_input_grad is true of a weight under no_grad too; in here no_grad always holds, so the caller says)
            track = graph and any(ctx.needs_input_grad[:4])            # (the residual's gradient is the result's)
            pre = torch.empty((tokens, out), dtype=torch.bfloat16, device=device) if track and (activation or mul2 is not None) else None
            y = torch.empty(shape, dtype=torch.bfloat16 if residual is None else residual.dtype, device=device)
            q.check(block.quartet_mxfp4_gemm_act(operands[0], operands[1], operands[3], operands[4], tokens, out, inf, 1.0, bias2, _dtype_code(bias2),
                                                 activation, mul2, out, res2, _dtype_code(res2), out, pre, out, y, _dtype_code(y), out))
        ctx.save_for_backward(pre, mul2, *operands)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        tokens, inf, out, seed, rounding, hadamard_block, activation = ctx.call
        x_shape, bias_dtype, residual_dtype = ctx.like
        device, need = dy.device, ctx.needs_input_grad
        if not tokens * out:
            zeros = [torch.zeros(s, dtype=t, device=device) if n else None
                     for s, t, n in zip((x_shape, (out, inf), (out,), dy.shape), (torch.bfloat16, torch.bfloat16, bias_dtype, torch.bfloat16), need)]
            return (*zeros, dy.to(residual_dtype) if need[4] else None, None, None, None, None, None)
        pre, mul, *operands = ctx.saved_tensors
        dx = dw = dbias = dmul = None
        with torch.cuda.device(device):
            dz = dy2 = _dense(dy.reshape(tokens, out).to(torch.bfloat16))
            if pre is not None or need[2]:
                plain = activation == 0 and mul is None
                dz = dy2 if plain else torch.empty_like(dy2)
                dmul = torch.empty(dy.shape, dtype=torch.bfloat16, device=device) if need[3] else None
                dbias = torch.empty(out, dtype=torch.float32, device=device) if need[2] else None
                size = block.quartet_act_bwd_workspace_bytes(tokens, out) if need[2] else 0
                ws = torch.empty(size, dtype=torch.uint8, device=device) if size else None
                if dbias is not None or dmul is not None or not plain:
                    q.check(block.quartet_act_bwd(dy2, out, pre, out, mul, out, tokens, out, activation, None if plain else dz, out, dmul, out, dbias,
                                                  ws, size))
            if need[0] or need[1]:
                dx = torch.empty(x_shape, dtype=torch.bfloat16, device=device)
                dw = torch.empty((out, inf), dtype=torch.bfloat16, device=device)
                size = q.quartet_linear_workspace_bytes_block(tokens, inf, out, hadamard_block)
                ws = torch.empty(max(256, size), dtype=torch.uint8, device=device)
                q.check(q.quartet_linear_bwd_block(dz, tokens, inf, out, hadamard_block, *operands, seed, rounding, dx, dw, q.QUARTET_DTYPE_BF16, ws, size))
        return (dx, dw, None if dbias is None else dbias.to(bias_dtype), dmul, dy.to(residual_dtype) if need[4] else None, None, None, None, None, None)


class QuartetLinear(torch.nn.Module):
    """nn.Linear replacement: weight [out, in] (bf16, or fp32 master weights cast to bf16 on the way
    in), optional bf16 bias.  activation ("none", "relu", "gelu" in its tanh form: torch's approximate="tanh", "silu"), multiplier (bf16, the other branch
    of a gated layer) and residual (bf16 or fp32, whose type the result then has) join the product's epilogue: a(x W^T + bias) * multiplier + residual; a
    bias alone is added by torch to the product's bf16 result.  Every backward pass uses a fresh stochastic-rounding seed: base seed, layer id and a
    per-layer call counter packed into 64 bits, so runs are reproducible and no two calls share draws."""
    _next_id = 0

    def __init__(self, in_features, out_features, bias=False, seed=0, rounding=0, device="cuda",
                 weight_dtype=torch.bfloat16, hadamard_block=32, activation="none"):
        super().__init__()
        if activation not in block.ACTIVATIONS:
            raise ValueError(f"activation must be one of {', '.join(block.ACTIVATIONS)}")
        self.activation = activation
        self.hadamard_block = hadamard_block
        self.in_features, self.out_features = in_features, out_features
        w = torch.randn(out_features, in_features, device=device) * (in_features ** -0.5)
        # weight_dtype=torch.float32 keeps fp32 master weights; the kernels always see a bf16 copy
        self.weight = torch.nn.Parameter(w.to(weight_dtype))
        self.bias = torch.nn.Parameter(torch.zeros(out_features, dtype=torch.bfloat16, device=device)) if bias else None
        self.rounding = rounding
        self.base_seed = int(seed) & 0xFFFF
        self.layer_id = QuartetLinear._next_id & 0xFFFF
        QuartetLinear._next_id += 1
        self.calls = 0

    def forward(self, x, multiplier=None, residual=None):
        seed = (self.base_seed << 48) | (self.layer_id << 32) | (self.calls & 0xFFFFFFFF)
        self.calls += 1
        weight = self.weight.to(torch.bfloat16)
        if self.activation != "none" or multiplier is not None or residual is not None:
            return _EpilogueFunction.apply(x, weight, self.bias, multiplier, residual, seed, self.rounding, self.hadamard_block,
                                           block.ACTIVATIONS[self.activation], torch.is_grad_enabled())
        y = QuartetLinearFunction.apply(x, weight, seed, self.rounding, self.hadamard_block)
        return y if self.bias is None else y + self.bias


class _RMSNormFunction(torch.autograd.Function):
    """(y, h) of the norm over x, or over h = residual + x"""

    @staticmethod
    def forward(ctx, x, residual, weight, eps):
        device = x.device
        n = weight.numel()
        _check_tensor(x, "x", _ANY, device)
        _check_tensor(weight, "weight", _ANY, device)
        if weight.dim() != 1 or n < 1 or x.dim() < 1 or x.shape[-1] != n:
            raise ValueError("x [..., n] and weight [n] do not fit together")
        if residual is not None:
            _check_tensor(residual, "residual", _ANY, device)
            if residual.shape != x.shape:
                raise ValueError("residual must have the shape of x")
        rows = x.numel() // n
        with torch.cuda.device(device):
            x2, ldx = _rows(x)
            res2, ldres = (None, 0) if residual is None else _rows(residual)
            w2 = _dense(weight)
            h = None if residual is None else _new_rows(x.shape, residual.dtype, device)
            y, rstd, ld = _new_rows(x.shape, torch.bfloat16, device), torch.empty(rows, dtype=torch.float32, device=device), n + -n % 8
            if rows:
                q.check(block.quartet_rmsnorm_fwd(_address(x2), _dtype_code(x2), ldx, _address(res2), ldres, rows, n, w2, _dtype_code(w2), float(eps), _address(h),
                                                  _dtype_code(h), ld, _address(y), ld, block.QUARTET_FORMAT_NONE, None, None, None, rstd))
        ctx.save_for_backward(x2 if h is None else h, w2, rstd)
        ctx.like = (x.dtype, rows, n)
        ctx.set_materialize_grads(False)
        return y, h

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dh):
        h, w, rstd = ctx.saved_tensors
        x_dtype, rows, n = ctx.like
        if dy is None:
            return (None if dh is None else dh.to(x_dtype)), dh, None, None
        need, device = ctx.needs_input_grad, h.device
        with torch.cuda.device(device):
            h, ldh = _rows(h)                   # (what a hook on saved tensors gives back may be laid out otherwise)
            dy2, lddy = _rows(dy.to(torch.bfloat16))
            dh2, lddh = (None, 0) if dh is None else _rows(dh.to(h.dtype))
            wants_x, ld = need[0] or need[1], n + -n % 8
            dx = _new_rows(h.shape, h.dtype, device) if wants_x else None
            dx16 = _new_rows(h.shape, torch.bfloat16, device) if wants_x and h.dtype == torch.float32 and x_dtype == torch.bfloat16 else None
            dw = (torch.empty if rows else torch.zeros)(n, dtype=torch.float32, device=device) if need[2] else None
            size = block.quartet_rmsnorm_bwd_workspace_bytes(rows, n) if need[2] else 0
            ws = torch.empty(size, dtype=torch.uint8, device=device) if size else None
            if rows and (wants_x or need[2]):
                q.check(block.quartet_rmsnorm_bwd(_address(dy2), lddy, _address(h), _dtype_code(h), ldh, rows, n, w, _dtype_code(w), rstd, _address(dh2), lddh,
                                                  _address(dx), ld, _address(dx16), ld, dw, ws, size))
        # one tensor object for both where they are the same values: autograd then knows that it is shared and copies it for one of two leaves
        # (two tensors over one memory it would hand out as two gradients)
        gx = dx if dx16 is None else dx16
        return (gx.to(x_dtype) if need[0] else None, dx if need[1] else None, None if dw is None else dw.to(w.dtype), None)


class QuartetRMSNorm(torch.nn.Module):
    """y = h / sqrt(mean(h^2) + eps) * weight as bf16, what QuartetLinear takes.  forward(x): h = x.  forward(x, residual): h = residual + x in
    residual's type, and the result is (y, h): the norm and the stream it leaves for the next layer.  x, residual [..., n] bf16 or fp32.  The backward pass
    needs h as it is.  (block.quartet_rmsnorm_fwd also writes MXFP4 and MXFP8 operands; QuartetLinear makes its operand from y itself.)"""

    def __init__(self, n, eps=1e-5, device="cuda", weight_dtype=torch.float32):
        super().__init__()
        self.weight = torch.nn.Parameter(torch.ones(n, dtype=weight_dtype, device=device))
        self.eps = eps

    def forward(self, x, residual=None):
        y, h = _RMSNormFunction.apply(x, residual, self.weight, self.eps)
        return y if residual is None else (y, h)


def _in_storage_order(g):
    """a dense gradient as it lies in memory"""
    v = g.permute(sorted(range(g.dim()), key=lambda d: (-g.stride(d), d))) if g.dim() > 1 and not g.is_contiguous() else g
    if not v.is_contiguous():
        raise q.QuartetError("gradients must be dense")
    return v


@torch.no_grad()
def clip_grad_norm_(parameters, max_norm):
    """Scales the gradients of `parameters` (bf16 or fp32, on one GPU) in place so that their common norm is at most max_norm, and returns
    the norm they had, on the device.  Two launches for 80 tensors, no synchronization.  A norm that is not finite leaves the gradients as they are."""
    parameters = [parameters] if isinstance(parameters, torch.Tensor) else list(parameters)
    grads = [_in_storage_order(p.grad) for p in {id(p): p for p in parameters}.values() if p.grad is not None]
    if not grads:
        return torch.zeros((), device=parameters[0].device if parameters else None)
    device = grads[0].device
    if device.type != "cuda" or any(g.device != device for g in grads):
        raise q.QuartetError("all gradients must be on one GPU: there is no CPU path")
    with torch.cuda.device(device):
        norm = torch.empty((), dtype=torch.float32, device=device)
        size = block.quartet_grad_clip_workspace_bytes()
        tensors = block.grad_tensors(grads)
        q.check(block.quartet_grad_clip(tensors, len(tensors), float(max_norm), norm, torch.empty(size, dtype=torch.uint8, device=device), size))
    return norm
