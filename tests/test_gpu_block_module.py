"""The torch layer over include/quartet_block.h as a program meets it: gradients that accumulate, results changed in place, tensors anywhere in a
buffer, inference without a graph."""
import pytest
import torch
import torch.utils.checkpoint

from block_util import BF16, DEV, F32, rng

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nn():
    from paper_2505_14669_amd import nn
    return nn


def new(g, *shape, dtype=BF16, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [96, 100])
@pytest.mark.parametrize("through", ["y", "h", "both"])
def test_gradients_of_x_and_of_the_stream_accumulate_apart(nn, dtype, n, through):
    g = rng(1)
    norm = nn.QuartetRMSNorm(n)
    x, res = (new(g, 3, 5, n, dtype=dtype).requires_grad_() for _ in range(2))
    dy, dh = new(g, 3, 5, n), new(g, 3, 5, n, dtype=dtype)

    def step():
        y, h = norm(x, res)
        torch.autograd.backward([t for t in (y, h) if through in (("y" if t is y else "h"), "both")],
                                [d for d, name in ((dy, "y"), (dh, "h")) if through in (name, "both")])

    step()
    assert x.grad.data_ptr() != res.grad.data_ptr() and torch.equal(x.grad, res.grad)
    once = x.grad.clone()
    step()
    assert torch.equal(x.grad, 2 * once) and torch.equal(res.grad, 2 * once)      # doubling is exact
    assert float(nn.clip_grad_norm_([x, res], 1e30)) > 0
    x.grad.zero_()
    assert torch.equal(res.grad, 2 * once)


@pytest.mark.parametrize("n", [96, 100])
def test_results_can_be_changed_in_place(nn, n):
    g = rng(2)
    norm = nn.QuartetRMSNorm(n)
    x, res, dy = new(g, 3, 5, n).requires_grad_(), new(g, 3, 5, n, dtype=F32).requires_grad_(), new(g, 3, 5, n)
    y, h = norm(x, res)
    assert y._base is None and h._base is None
    y.backward(2 * dy)                                     # halving and doubling are exact
    want = x.grad.clone(), res.grad.clone(), norm.weight.grad.clone()
    x.grad = res.grad = norm.weight.grad = None
    y2, h2 = norm(x, res)
    y2.mul_(2)
    assert torch.equal(y2, 2 * y)
    y2.backward(dy)
    assert all(torch.equal(a, c) for a, c in zip((x.grad, res.grad, norm.weight.grad), want))
    with torch.no_grad():
        h3 = norm(x, res)[1]
        h3 += 1
        assert torch.equal(h3, h + 1)
    y4, h4 = norm(x, res)                                  # the backward pass needs h: a changed one is refused there, not used
    h4.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        (y4.float().sum() + h4.sum()).backward()


@pytest.mark.parametrize("n", [96, 100])
def test_saved_tensors_that_come_back_laid_out_otherwise(nn, n):
    g = rng(3)
    norm = nn.QuartetRMSNorm(n)
    x, res, dy = new(g, 3, 5, n).requires_grad_(), new(g, 3, 5, n).requires_grad_(), new(g, 3, 5, n)
    found = []
    for hooks in (torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: t), torch.autograd.graph.save_on_cpu(),
                  torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: t.t().contiguous().t() if t.dim() == 2 else t.transpose(0, -1).contiguous().transpose(0, -1))):
        x.grad = res.grad = norm.weight.grad = None
        with hooks:
            y = norm(x, res)[0]
            y1 = norm(x)
        torch.autograd.backward([y, y1], [dy, dy])
        found.append((x.grad, res.grad, norm.weight.grad))
    assert all(torch.equal(a, c) for other in found[1:] for a, c in zip(other, found[0]))


def test_rows_of_a_wider_tensor(nn):
    # columns of a wider matrix, one row used many times, a transposed one, a single row: the same bits as their copies
    g = rng(4)
    for n in (64, 100, 1):
        norm = nn.QuartetRMSNorm(n)
        wide, column = new(g, 6, 4, n + 28), new(g, n, 6, 4)
        for x in (wide[..., :n], wide[..., 8:8 + n], wide[..., 4:4 + n], wide[:, :1, :n], wide[0, 0, :n], wide[:1, :1, :n].expand(6, 4, n), column.permute(1, 2, 0), wide[::2, 1:, :n]):
            res = new(g, *x.shape, dtype=F32)
            want = norm(x.clone(memory_format=torch.contiguous_format), res)
            assert all(torch.equal(a, c) for a, c in zip(norm(x, res), want))
            want = norm(x.clone(memory_format=torch.contiguous_format), x.clone(memory_format=torch.contiguous_format))
            assert all(torch.equal(a, c) for a, c in zip(norm(x, x), want))


def calls(monkeypatch, nn, name):
    """the argument lists of the binding's call `name` from now on"""
    seen, real = [], getattr(nn.block, name)
    monkeypatch.setattr(nn.block, name, lambda *args: (seen.append(args), real(*args))[1])
    return seen


def test_inference_keeps_nothing_for_a_backward_pass(nn, monkeypatch):
    g = rng(5)
    lin, x, up = nn.QuartetLinear(64, 96, activation="silu"), new(g, 32, 64), new(g, 32, 96)
    seen = calls(monkeypatch, nn, "quartet_mxfp4_gemm_act")
    pre = 16                                              # z's place among the arguments
    y = lin(x, multiplier=up)
    with torch.no_grad():
        y_no_grad = lin(x, multiplier=up)
    with torch.inference_mode():
        y_inference = lin(x, multiplier=up)
    assert [args[pre] is not None for args in seen] == [True, False, False]
    assert torch.equal(y, y_no_grad) and torch.equal(y, y_inference)
    y = torch.utils.checkpoint.checkpoint(lambda t: lin(t, multiplier=up), x.requires_grad_(), use_reentrant=True)      # first without a graph, then with one
    assert [args[pre] is not None for args in seen[3:]] == [False]
    y.float().sum().backward()
    assert [args[pre] is not None for args in seen[3:]] == [False, True] and bool(torch.isfinite(x.grad).all())
    # a frozen layer: what goes along the residual needs no z
    lin.requires_grad_(False)
    res = new(g, 32, 96, dtype=F32).requires_grad_()
    lin(x.detach(), multiplier=up, residual=res).backward(new(g, 32, 96, dtype=F32))
    assert seen[-1][pre] is None and res.grad is not None


def test_workspaces_only_for_sums_over_the_rows(nn, monkeypatch):
    g = rng(6)
    x, up, dy = new(g, 64, 128).requires_grad_(), new(g, 64, 96).requires_grad_(), new(g, 64, 96)
    for bias in (False, True):
        lin, seen = nn.QuartetLinear(128, 96, bias=bias, activation="gelu"), calls(monkeypatch, nn, "quartet_act_bwd")
        lin(x, multiplier=up).backward(dy)
        size = nn.block.quartet_act_bwd_workspace_bytes(64, 96)
        assert size > 0 and (seen[-1][14] is not None, seen[-1][15]) == ((True, size) if bias else (False, 0))
    for weight in (True, False):
        norm, seen = nn.QuartetRMSNorm(128).requires_grad_(weight), calls(monkeypatch, nn, "quartet_rmsnorm_bwd")
        norm(x).backward(new(g, 64, 128))
        size = nn.block.quartet_rmsnorm_bwd_workspace_bytes(64, 128)
        assert size > 0 and (seen[-1][17] is not None, seen[-1][18]) == ((True, size) if weight else (False, 0))
    assert bool(torch.isfinite(x.grad).all()) and bool(torch.isfinite(up.grad).all())


def anywhere(t, leaf=True):
    """a copy of t in the middle of a buffer, at an odd element"""
    buffer = torch.zeros(t.numel() + 16, dtype=t.dtype, device=DEV)
    view = buffer[3:3 + t.numel()].view(t.shape).copy_(t)
    assert view.data_ptr() % 16
    return view.detach().requires_grad_() if leaf else view


def test_layer_takes_tensors_that_start_anywhere(nn):
    # pieces of flat buffers (sharded parameters, packed activations): the same bits as tensors of their own
    g = rng(7)
    x, up, res, dy = new(g, 32, 64), new(g, 32, 96), new(g, 32, 96, dtype=F32), new(g, 32, 96, dtype=F32)
    lin = nn.QuartetLinear(64, 96, bias=True, rounding=1, activation="silu")
    with torch.no_grad():
        lin.bias.copy_(new(g, 96))
    found = []
    for place in (lambda t: t.clone().requires_grad_(), anywhere):
        leaves = [place(t) for t in (x, up, res)]
        lin.weight.data, lin.bias.data = place(lin.weight.data).detach(), place(lin.bias.data).detach()
        lin.weight.grad = lin.bias.grad = None
        lin.calls = 0                                          # (a call's number is part of the backward pass's random signs)
        y = lin(leaves[0], multiplier=leaves[1], residual=leaves[2])
        y.backward(place(dy).detach())
        y16 = lin(leaves[0])
        y16.backward(place(up).detach())
        found.append([y, y16, *(t.grad for t in leaves), lin.weight.grad, lin.bias.grad])
    assert all(torch.equal(a, c) for a, c in zip(*found))


@pytest.mark.parametrize("n", [64, 101])
def test_norm_takes_tensors_that_start_anywhere(nn, n):
    g = rng(8)
    x, res, dy, dh = new(g, 3, 5, n), new(g, 3, 5, n, dtype=F32), new(g, 3, 5, n), new(g, 3, 5, n, dtype=F32)
    norm, found = nn.QuartetRMSNorm(n), []
    with torch.no_grad():
        norm.weight.copy_(new(g, n, dtype=F32))
    for place in (lambda t: t.clone().requires_grad_(), anywhere):
        leaves = [place(t) for t in (x, res)]
        norm.weight.data, norm.weight.grad = place(norm.weight.data).detach(), None
        y, h = norm(*leaves)
        torch.autograd.backward([y, h], [place(dy).detach(), place(dh).detach()])
        found.append([y, h, *(t.grad for t in leaves), norm.weight.grad])
    assert all(torch.equal(a, c) for a, c in zip(*found))


@pytest.mark.parametrize("hadamard_block,t,i,o", [(32, 96, 160, 64), (64, 128, 192, 64), (128, 128, 256, 384), (256, 256, 512, 256)])
@pytest.mark.parametrize("kind", ["none", "relu", "gelu", "silu"])
def test_gradients_are_the_plain_layers_for_the_epilogues_gradient(nn, kind, hadamard_block, t, i, o):
    # dz from the operator's own call on the plain product's result; with it the plain layer's backward pass must give the same bits for x and for the weight
    g = rng(9)
    x, up, res, dy = new(g, t, i), new(g, t, o), new(g, t, o), new(g, t, o, scale=0.1)
    lin = nn.QuartetLinear(i, o, seed=5, rounding=0, hadamard_block=hadamard_block, activation=kind)
    x1, x2, up1 = x.clone().requires_grad_(), x.clone().requires_grad_(), up.clone().requires_grad_()
    y = lin(x1, multiplier=up1, residual=res)
    y.backward(dy)
    got, lin.weight.grad = lin.weight.grad, None
    z = nn.QuartetLinearFunction.apply(x2, lin.weight, (lin.base_seed << 48) | (lin.layer_id << 32), 0, hadamard_block)
    dz, dup = torch.empty_like(dy), torch.empty_like(dy)
    nn.q.check(nn.block.quartet_act_bwd(dy, o, z.detach(), o, up, o, t, o, nn.block.ACTIVATIONS[kind], dz, o, dup, o, None, None, 0))
    z.backward(dz)
    assert torch.equal(x1.grad, x2.grad) and torch.equal(got, lin.weight.grad) and torch.equal(up1.grad, dup)
    assert bool((got != 0).any()) and bool((x2.grad != 0).any())


@pytest.mark.parametrize("shape", [(0, 64), (3, 0, 64)])
def test_layer_with_an_epilogue_over_no_tokens(nn, shape):
    # a batch without tokens (an expert that got none): an empty result, gradients of zeros
    lin = nn.QuartetLinear(64, 96, bias=True, activation="silu")
    x, res = torch.empty(shape, dtype=BF16, device=DEV).requires_grad_(), torch.empty((*shape[:-1], 96), device=DEV).requires_grad_()
    up = torch.empty((*shape[:-1], 96), dtype=BF16, device=DEV).requires_grad_()
    y = lin(x, multiplier=up, residual=res)
    assert y.shape == (*shape[:-1], 96) and y.dtype == F32
    y.sum().backward()
    assert x.grad.shape == x.shape and up.grad.shape == up.shape and res.grad.dtype == F32
    assert lin.weight.grad.shape == (96, 64) and bool((lin.weight.grad == 0).all()) and lin.bias.grad.shape == (96,) and bool((lin.bias.grad == 0).all())
    with torch.no_grad():
        assert lin(x).shape == y.shape


class GatedBlock(torch.nn.Module):
    """norm, gated projections with bias and down projection onto the stream"""

    def __init__(self, nn, d, h):
        super().__init__()
        self.norm, self.gate, self.up = nn.QuartetRMSNorm(d), nn.QuartetLinear(d, h, bias=True, activation="silu"), nn.QuartetLinear(d, h)
        self.down = nn.QuartetLinear(h, d, bias=True)

    def forward(self, x, stream):
        for lin in (self.gate, self.up, self.down):
            lin.calls = 0                                      # the same draws in every pass: a graph replays those of its capture
        y, stream = self.norm(x, stream)
        return self.down(self.gate(y, multiplier=self.up(y)), residual=stream)


def test_block_captured_forward_and_backward(nn):
    g = rng(10)
    captured, eager = (GatedBlock(nn, 128, 256) for _ in range(2))
    eager.load_state_dict(captured.state_dict())
    for a, c in zip(captured.children(), eager.children()):
        if a is not captured.norm:
            c.layer_id = a.layer_id
    inputs = [(new(g, 64, 128), new(g, 64, 128, dtype=F32), new(g, 64, 128, dtype=F32, scale=0.1)) for _ in range(3)]
    x, stream, dy = (t.clone() for t in inputs[0])
    x.requires_grad_()
    stream.requires_grad_()
    leaves = [x, stream, *captured.parameters()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        captured(x, stream).backward(dy)
    torch.cuda.current_stream().wait_stream(side)
    for t in leaves:
        t.grad = None
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = captured(x, stream)
        out.backward(dy)
        norm = nn.clip_grad_norm_(captured.parameters(), 0.01)
    for turn in range(5):
        with torch.no_grad():
            for t, source in zip((x, stream, dy), inputs[turn % 3]):
                t.copy_(source)
        xe, se = (t.clone().requires_grad_() for t in inputs[turn % 3][:2])      # eager work between the replays, on leaves of its own
        eager.zero_grad(set_to_none=True)
        want = eager(xe, se)
        want.backward(inputs[turn % 3][2])
        want_norm = nn.clip_grad_norm_(eager.parameters(), 0.01)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(norm, want_norm) and float(norm) > 0.01, turn
        assert all(torch.equal(a.grad, c.grad) for a, c in zip(leaves, [xe, se, *eager.parameters()])), turn
