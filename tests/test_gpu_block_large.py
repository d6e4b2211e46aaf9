"""The operators of include/quartet_block.h where sizes make them take another path: accesses past the memory-side cache, longer chunks, blocks handed
out by scale tile.  The plain versions and bounds are those of the operators' own tests."""
import pytest
import torch

import test_gpu_block_act as A
from block_util import BF16, DEV, F32, GUARD, rng

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("g_dtype,o_dtype", [(F32, F32), (BF16, F32), (F32, BF16)])
def test_clip_copies_that_the_cache_cannot_hold(g_dtype, o_dtype):
    # gradients and copies of 270 MB together and more
    sizes = [34000003, 11000001, 5, 8191]
    g = rng(1)
    grads = [torch.randn(s, generator=g, device=DEV).to(g_dtype) for s in sizes]
    guard = [torch.full((s + 16,), GUARD, dtype=o_dtype, device=DEV) for s in sizes]
    outs = [t[8:8 + s] for t, s in zip(guard, sizes)]
    A.check_clip(grads, outs, 0.5)
    assert all(bool((t[:8] == GUARD).all() and (t[8 + s:] == GUARD).all()) for t, s in zip(guard, sizes))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_clip_of_more_chunks_than_the_workspace_has_sums_for(dtype):
    # 140 M values: chunks of 8192, the last one of each tensor cut short in its first or second half
    sizes = [100000001, 34000003, 6004099, 5, 0, 8193, 4097]
    assert sum((s + 4095) // 4096 for s in sizes) > 32768
    g = rng(2)
    flat = torch.randn(sum(sizes) + 16, generator=g, device=DEV).to(dtype)
    views, at = [], 3
    for s in sizes:
        views.append(flat[at:at + s])
        at += s
    ends = flat[:3].clone(), flat[at:].clone()
    before = [v.double() for v in views]
    A.check_clip(views, views, 1.0, before)                        # in place, at odd elements
    assert torch.equal(flat[:3], ends[0]) and torch.equal(flat[at:], ends[1])
    copies = [torch.empty(s, dtype=F32, device=DEV) for s in sizes]
    A.check_clip(views, copies, 0.5)
