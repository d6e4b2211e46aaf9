"""The torch layer over include/quartet_block.h as a program meets it: gradients that accumulate, results changed in place, tensors anywhere in a
buffer, inference without a graph."""
import pytest
import torch

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
