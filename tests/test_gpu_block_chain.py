"""The operators of include/quartet_block.h as they are used together: a gated block forward, backward and clipped through the C ABI,
eager, on a side stream and captured into a HIP graph; and the torch layer over them."""
import pytest
import torch

from block_util import BF16, DEV, F32, U16, act, assert_within, b, code, q, rng

pytestmark = pytest.mark.gpu
T, D, H = 96, 256, 416


class Block:
    """h = res + x; v = norm(h); y = h + W2 (silu(Wg v) * (Wu v)) through MXFP4 operands, its backward pass and the clipping of the weights' gradients"""

    def __init__(self, seed):
        g = rng(seed)
        new = lambda *s, dtype=BF16, scale=1.0: (torch.randn(s, generator=g, device=DEV) * scale).to(dtype)
        empty = lambda *s, dtype=BF16: torch.zeros(s, dtype=dtype, device=DEV)
        byte = lambda n: torch.zeros(max(16, n), dtype=torch.uint8, device=DEV)
        self.x, self.res, self.dy = new(T, D), new(T, D, dtype=F32), new(T, D, scale=0.01)
        self.w = new(D, dtype=F32, scale=0.1) + 1
        self.weights = {"g": new(H, D, scale=D ** -0.5), "u": new(H, D, scale=D ** -0.5), "d": new(D, H, scale=H ** -0.5)}
        operand = lambda r, k: (byte(r * k // 2), byte(q.quartet_scale_bytes(r, k)), byte(r * k // 8))
        self.op = {"v": operand(T, D), "a": operand(T, H), "g": operand(H, D), "u": operand(H, D), "d": operand(D, H)}
        self.h, self.rstd, self.up, self.gate_pre, self.inner = empty(T, D, dtype=F32), empty(T, dtype=F32), empty(T, H), empty(T, H), empty(T, H)
        self.y = empty(T, D, dtype=F32)
        self.d_inner, self.dz, self.dup, self.dv, self.dv2 = empty(T, H), empty(T, H), empty(T, H), empty(T, D), empty(T, D)
        self.dx, self.dx16, self.dw = empty(T, D, dtype=F32), empty(T, D), empty(D, dtype=F32)
        self.grads = {k: empty(*v.shape) for k, v in self.weights.items()}
        self.main = {k: empty(*v.shape, dtype=F32) for k, v in self.weights.items()}
        self.list = b.grad_tensors([*self.grads.values(), self.dw], [*self.main.values(), self.dw])
        self.norm = empty(1, dtype=F32)
        sizes = [q.quartet_linear_workspace_bytes(T, D, H), q.quartet_linear_workspace_bytes(T, H, D), b.quartet_act_bwd_workspace_bytes(T, H),
                 b.quartet_rmsnorm_bwd_workspace_bytes(T, D), b.quartet_grad_clip_workspace_bytes()]
        self.ws = byte(max(sizes))

    def step(self, stream=None):
        p = lambda *args: q.check(args[0](*args[1:], stream))
        for k, w in self.weights.items():
            p(q.quartet_quant_fwd, w, w.shape[0], w.shape[1], w.shape[1], 0, *self.op[k])
        p(b.quartet_rmsnorm_fwd, self.x, 1, D, self.res, D, T, D, self.w, 0, 1e-5, self.h, 0, D, None, 0, b.QUARTET_FORMAT_MXFP4, *self.op["v"], self.rstd)
        v, u, g, d, a = (self.op[k] for k in "vugda")
        p(b.quartet_mxfp4_gemm_act, v[0], v[1], u[0], u[1], T, H, D, 1.0, None, 0, 0, None, 0, None, 0, 0, None, 0, self.up, 1, H)
        p(b.quartet_mxfp4_gemm_act, v[0], v[1], g[0], g[1], T, H, D, 1.0, None, 0, 3, self.up, H, None, 0, 0, self.gate_pre, H, self.inner, 1, H)
        p(q.quartet_quant_fwd, self.inner, T, H, H, 0, *a)
        p(b.quartet_mxfp4_gemm_act, a[0], a[1], d[0], d[1], T, D, H, 1.0, None, 0, 0, None, 0, self.h, 0, D, None, 0, self.y, 0, D)
        n = self.ws.numel()
        p(q.quartet_linear_bwd, self.dy, T, H, D, *a, *d, 1, 1, self.d_inner, self.grads["d"], 1, self.ws, n)
        p(b.quartet_act_bwd, self.d_inner, H, self.gate_pre, H, self.up, H, T, H, 3, self.dz, H, self.dup, H, None, None, 0)
        p(q.quartet_linear_bwd, self.dz, T, D, H, *v, *g, 2, 1, self.dv, self.grads["g"], 1, self.ws, n)
        p(q.quartet_linear_bwd, self.dup, T, D, H, *v, *u, 3, 1, self.dv2, self.grads["u"], 1, self.ws, n)
        total = self.dv + self.dv2
        dh = self.dy.float()
        p(b.quartet_rmsnorm_bwd, total, D, self.h, 0, D, T, D, self.w, 0, self.rstd, dh, D, self.dx, D, self.dx16, D, self.dw, self.ws, n)
        p(b.quartet_grad_clip, self.list, len(self.list), 0.05, self.norm, self.ws, n)

    def results(self):
        return [self.h, self.rstd, *self.op["v"], self.up, self.gate_pre, self.inner, self.y, self.d_inner, self.dz, self.dup, self.dx, self.dx16, self.dw, self.norm,
                *self.grads.values(), *self.main.values()]


def snapshot(block):
    torch.cuda.synchronize()
    return [t.clone() for t in block.results()]


def test_block_forward_is_near_the_unquantized_one():
    # five MXFP4 operands, each off by about 0.11 of its norm (relative squared error 0.0127): a product's two operands make 0.16 of a product; the
    # result is the stream plus such a product of such products.  A wrong gate, residual or norm is off by the size of the block itself.
    k = Block(1)
    k.step()
    h = (k.res + k.x.float()).double()
    v = h * (h.square().mean(1, keepdim=True) + 1e-5).rsqrt() * k.w.double()
    w = {n: t.double() for n, t in k.weights.items()}
    inner = act(v @ w["g"].t(), "silu")[0] * (v @ w["u"].t())
    want = h + inner @ w["d"].t()
    assert torch.equal(k.h.double(), h.float().double())
    rel = lambda x, y: float((x.double() - y).norm() / y.norm())
    assert rel(k.up, v @ w["u"].t()) < 0.25 and rel(k.inner, inner) < 0.4 and rel(k.y - k.h, want - h) < 0.5
    grads = torch.cat([t.flatten().double() for t in k.grads.values()])
    assert float(k.norm) > 0.05 and float(torch.cat([*(t.flatten() for t in k.main.values()), k.dw]).double().norm()) == pytest.approx(0.05, rel=1e-4)
    assert float(k.norm) >= float(grads.norm()) * (1 - 1e-6)


def test_on_another_stream_than_the_current_one():
    want = Block(2)
    want.step()
    want = snapshot(want)
    k, side = Block(2), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        k.step()
    assert all(torch.equal(x, y) for x, y in zip(snapshot(k), want))


def test_captured_and_replayed_between_eager_work():
    k, other = Block(3), Block(4)
    eager = {}
    for seed in (3, 4):
        e = Block(seed)
        e.step()
        eager[seed] = snapshot(e)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        k.step()                                       # once outside the capture: allocations of the sums between the calls
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        k.step()
    for turn in range(4):
        for t in (k.x, k.res, k.dy, k.w, *k.weights.values()):
            t.copy_(t)
        source = Block(3 + turn % 2)
        for name in ("x", "res", "dy", "w"):
            getattr(k, name).copy_(getattr(source, name))
        for n, t in source.weights.items():
            k.weights[n].copy_(t)
        other.step()                                   # eager work of another block between the replays
        graph.replay()
        assert all(torch.equal(x, y) for x, y in zip(snapshot(k), eager[3 + turn % 2])), turn


def test_two_captured_graphs_with_a_workspace_each():
    ks, graphs = [Block(5), Block(6)], []
    want = []
    for k in ks:
        k.step()
        want.append(snapshot(k))
    for k in ks:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            k.step()
        graphs.append(graph)
    for _ in range(3):
        for graph in graphs:
            graph.replay()
        for k, w in zip(ks, want):
            assert all(torch.equal(x, y) for x, y in zip(snapshot(k), w))


# ---------------------------------------------------------------------------------------------- the torch layer

@pytest.fixture(scope="module")
def nn():
    from paper_2505_14669_amd import nn
    return nn


def test_layer_with_epilogue_is_the_layer_and_the_plain_steps(nn):
    # the product's operands and gradients are those of the plain layer with the same seed, so the epilogue's autograd must agree with torch's own over it
    t, i, o = 64, 128, 96
    for kind in ("none", "relu", "gelu", "silu"):
        g = rng(7)
        x, up, res = (torch.randn(s, generator=g, device=DEV).to(BF16) for s in ((2, t // 2, i), (2, t // 2, o), (2, t // 2, o)))
        lin = nn.QuartetLinear(i, o, bias=True, seed=5, rounding=1, activation=kind)
        with torch.no_grad():
            lin.bias.copy_(torch.randn(o, generator=g, device=DEV))
        leaves = [x.clone().requires_grad_(), up.clone().requires_grad_(), res.float().requires_grad_()]
        y = lin(leaves[0], multiplier=leaves[1], residual=leaves[2])
        assert y.dtype == F32 and y.shape == (2, t // 2, o)
        dy = (torch.randn(y.shape, generator=g, device=DEV) * 0.1).to(BF16).float()
        y.backward(dy)
        # plain: z from the same function, the rest in fp64
        x2 = x.clone().requires_grad_()
        seed = (lin.base_seed << 48) | (lin.layer_id << 32)
        z0 = nn.QuartetLinearFunction.apply(x2, lin.weight, seed, 1)
        z = z0.double() + lin.bias.double()
        value, slope = act(z.detach(), kind)
        want = value * up.double() + res.double()
        assert_within(y, want, (z.detach().abs() * 2 * U16 + 2 * U16) * 1.2 * up.double().abs() + 1e-5)       # z0 was rounded to bf16
        dz = dy.double() * up.double() * slope
        slack = (dy.double() * up.double()).abs() * (4 * U16 * (1 + z.detach().abs()))
        assert_within(leaves[1].grad, dy.double() * value, dy.double().abs() * 4 * U16 * (1 + z.detach().abs()))
        assert torch.equal(leaves[2].grad, dy)
        inside = torch.ones_like(z, dtype=torch.bool) if kind != "relu" else z.detach().abs() > 0.05            # next to 0 the step may fall either way
        bound = torch.where(inside, slack, slack + (dy.double() * up.double()).abs())
        assert_within(lin.bias.grad, dz.sum((0, 1)), bound.sum((0, 1)) + dz.sum((0, 1)).abs() * U16)
        # the product's gradients: those of the plain layer for a gradient near dz (nearest rounding of nearby values: some codes differ)
        z0.backward(dz.to(BF16))
        rel = lambda a, c: float((a.double() - c.double()).norm() / c.double().norm())
        assert rel(leaves[0].grad, x2.grad) < 0.1
        assert bool(torch.isfinite(lin.weight.grad).all()) and bool((lin.weight.grad != 0).any())


def test_layer_without_epilogue_is_what_it_was(nn):
    x = torch.randn((64, 128), generator=rng(8), device=DEV).to(BF16)
    lin = nn.QuartetLinear(128, 96, bias=True, seed=5)
    seed = (lin.base_seed << 48) | (lin.layer_id << 32)
    y = lin(x)
    assert torch.equal(y, nn.QuartetLinearFunction.apply(x, lin.weight, seed, 0) + lin.bias)


def test_bias_alone_with_a_residual(nn):
    # no activation, no gate: z is not kept, the bias's gradient is the column sum of dy
    lin = nn.QuartetLinear(64, 32, bias=True, seed=5, hadamard_block=32)
    x, res = torch.randn((32, 64), device=DEV).to(BF16), torch.randn((32, 32), device=DEV).to(BF16).requires_grad_()
    y = lin(x, residual=res)
    dy = torch.randn((32, 32), generator=rng(9), device=DEV).to(BF16)
    y.backward(dy)
    d = dy.double()
    assert y.dtype == BF16 and torch.equal(res.grad, dy)
    assert_within(lin.bias.grad, d.sum(0), d.sum(0).abs() * U16 + d.abs().sum(0) * 1e-5)


@pytest.mark.parametrize("hadamard_block", [32, 64, 128])
def test_wide_blocks(nn, hadamard_block):
    lin = nn.QuartetLinear(256, 128, seed=5, hadamard_block=hadamard_block, activation="relu")
    x = torch.randn((128, 256), generator=rng(10), device=DEV).to(BF16).requires_grad_()
    y = lin(x)
    plain = nn.QuartetLinearFunction.apply(x, lin.weight, 0, 0, hadamard_block)
    assert_within(y, plain.double().clamp_min(0), plain.double().abs() * 2 * U16 + 1e-6)
    y.sum().backward()
    assert bool(torch.isfinite(x.grad).all()) and bool(torch.isfinite(lin.weight.grad).all())


@pytest.mark.parametrize("shape,n", [((3, 5), 96), ((7,), 100), ((0,), 40)])
@pytest.mark.parametrize("x_dtype,res_dtype", [(BF16, F32), (BF16, BF16), (F32, F32)])
def test_norm_module(nn, shape, n, x_dtype, res_dtype):
    g = rng(11)
    norm = nn.QuartetRMSNorm(n)
    with torch.no_grad():
        norm.weight.add_(0.1 * torch.randn(n, generator=g, device=DEV))
    x = torch.randn((*shape, n), generator=g, device=DEV).to(x_dtype).requires_grad_()
    res = torch.randn((*shape, n), generator=g, device=DEV).to(res_dtype).requires_grad_()
    y, h = norm(x, res)
    assert y.dtype == BF16 and h.dtype == res_dtype and y.shape == h.shape == x.shape
    dy, dh = (torch.randn(x.shape, generator=g, device=DEV) for _ in range(2))
    ((y.float() * dy).sum() + (h.float() * dh).sum()).backward()
    hs = h.detach().double().requires_grad_()
    wd = norm.weight.detach().double().requires_grad_()
    v = hs * (hs.square().mean(-1, keepdim=True) + norm.eps).rsqrt() * wd
    v.backward(dy.to(BF16).double())
    want = hs.grad + dh.to(res_dtype).double()
    scale = want.abs() * 2 * U16 + (hs.grad.abs() + dh.double().abs()) * U16 + 1e-6
    assert_within(x.grad, want, scale)
    assert_within(res.grad, want, scale)
    assert_within(norm.weight.grad, wd.grad, wd.grad.abs() * 1e-5 + 1e-4)
    y1 = norm(x)
    if x.numel():
        xs = x.detach().double()
        w1 = xs * (xs.square().mean(-1, keepdim=True) + norm.eps).rsqrt() * norm.weight.detach().double()
        assert_within(y1, w1, w1.abs() * 1.01 * U16)
    y1.float().sum().backward()


def test_layer_refuses(nn):
    lin = nn.QuartetLinear(64, 32, activation="relu")
    x = torch.zeros((32, 64), dtype=BF16, device=DEV)
    with pytest.raises(ValueError):
        nn.QuartetLinear(64, 32, activation="tanh")
    with pytest.raises(TypeError):
        lin(x.float())
    with pytest.raises(ValueError):
        lin(x[:31])
    with pytest.raises(ValueError):
        lin(x, residual=x)
    with pytest.raises(TypeError):
        lin(x, multiplier=torch.zeros((32, 32), device=DEV))
    with pytest.raises(RuntimeError):
        lin(x, residual=torch.zeros((32, 32)))
    norm = nn.QuartetRMSNorm(64)
    with pytest.raises(ValueError):
        norm(x[:, :32])
    with pytest.raises(TypeError):
        norm(x.half())
    with pytest.raises(ValueError):
        norm(x, x[:31])
    y = lin(x.requires_grad_())
    with pytest.raises(RuntimeError):
        torch.autograd.grad(torch.autograd.grad(y.float().sum(), x, create_graph=True)[0].float().sum(), x)


def test_clip_module(nn):
    g = rng(12)
    params = [torch.nn.Parameter(torch.zeros(s, device=DEV, dtype=d)) for s, d in (((5, 7), F32), ((11,), BF16), ((4, 6), F32), ((3,), F32))]
    for p in params[:3]:
        p.grad = torch.randn(p.shape, generator=g, device=DEV).to(p.dtype)
    params[2].grad = params[2].grad.t().contiguous().t()              # dense, not row-major
    before = [p.grad.double().clone() for p in params[:3]]
    want = sum(float(t.square().sum()) for t in before) ** 0.5
    norm = nn.clip_grad_norm_([*params, params[0]], 0.5)               # a parameter named twice counts once
    assert float(norm) == pytest.approx(want, rel=1e-6)
    for p, t in zip(params, before):
        assert_within(p.grad, t * 0.5 / (want + 1e-6), t.abs() * (U16 if p.dtype == BF16 else 1e-6))
    assert float(nn.clip_grad_norm_(params, 1e9)) == pytest.approx(0.5, rel=1e-2)
    assert float(nn.clip_grad_norm_([params[3]], 1.0)) == 0.0
    params[3].grad = torch.zeros(6, device=DEV)[::2]
    with pytest.raises(nn.q.QuartetError):
        nn.clip_grad_norm_(params, 1.0)


def test_training_step_of_a_block(nn):
    # runs, gives every parameter a finite gradient and clips them
    d, h = 128, 256
    norm, gate, up, down = nn.QuartetRMSNorm(d), nn.QuartetLinear(d, h, activation="silu"), nn.QuartetLinear(d, h), nn.QuartetLinear(h, d)
    params = [p for m in (norm, gate, up, down) for p in m.parameters()]
    x, stream = torch.randn((64, d), generator=rng(13), device=DEV).to(BF16), torch.randn((64, d), generator=rng(14), device=DEV)
    y, s = norm(x, stream)
    out = down(gate(y, multiplier=up(y)), residual=s)
    out.square().mean().backward()
    assert out.dtype == F32 and all(p.grad is not None and bool(torch.isfinite(p.grad).all()) and bool((p.grad != 0).any()) for p in params)
    total = nn.clip_grad_norm_(params, 1e-3)
    assert float(total) > 1e-3
    assert float(torch.cat([p.grad.flatten().double() for p in params]).norm()) == pytest.approx(1e-3, rel=1e-2)
