"""The operators of include/quartet_block.h where sizes make them take another path: accesses past the memory-side cache, longer chunks, blocks handed
out by scale tile.  The plain versions and bounds are those of the operators' own tests."""
import pytest
import torch

import test_gpu_block_act as A
import test_gpu_block_norm as N
from block_util import BF16, DEV, F32, GUARD, HALF, U32, assert_within, b, code, matrix, q, quantized, rng

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


# 1024 rows and more: blocks go by the tiles of 32 rows of the scales, 4, 2 or 1 rows a block
TILED = [(1024, 480), (1100, 1376), (1057, 992), (1030, 4096), (1025, 8224), (2050, 512)]


@pytest.mark.parametrize("rows,n", TILED)
@pytest.mark.parametrize("res_dtype", [None, F32])
def test_norm_operands_by_scale_tile(rows, n, res_dtype):
    N.test_mxfp8_operand(rows, n, res_dtype)
    N.test_mxfp4_operand(rows, n, res_dtype, True)


def test_norm_results_that_the_cache_cannot_hold():
    # codes of 64 MiB and more, bf16 results of 256 MiB and more; rows of sixteen waves and of one
    for rows, n in ((32900, 4128), (1050000, 128)):
        N.test_mxfp4_operand(rows, n, None, False)
        torch.cuda.empty_cache()
        N.test_forward(rows, n, BF16, BF16, F32)
        torch.cuda.empty_cache()
    N.test_mxfp8_operand(16500, 4128, BF16)
    torch.cuda.empty_cache()


# one, two, four and sixteen waves a row, sixteen with two and four chunks a lane; widths with and without an incomplete chunk
@pytest.mark.parametrize("rows,n,h_dtype,dh", [(270001, 100, F32, True), (130003, 520, BF16, True), (27001, 1003, F32, True), (6601, 4100, F32, True),
                                               (16500, 4096, BF16, False), (3301, 8203, F32, True), (1650, 16392, F32, True)])
def test_norm_backward_of_what_the_cache_cannot_hold(rows, n, h_dtype, dh):
    assert rows * n * (2 + (4 if h_dtype == F32 else 2) * (2 if dh else 1)) >= 256 << 20
    N.test_backward(rows, n, h_dtype, F32, dh)
    torch.cuda.empty_cache()


# the in-block split's kernels, tiles of every size, ragged ones, results of 256 MiB and more
@pytest.mark.parametrize("m,n,k", [(1, 8, 64), (24, 11008, 512), (96, 416, 256), (600, 768, 1024), (1003, 5632, 2048), (2100, 4448, 320), (4096, 2048, 2048),
                                   (8192, 4096, 512), (16500, 8200, 288)])
@pytest.mark.parametrize("out", [BF16, F32])
def test_without_an_epilogue_it_is_the_plain_product_to_the_bit(m, n, k, out):
    # same sizes, same kernel, same order of sums, without a forced plan too
    a, a_scales, _ = quantized(rng(3), m, k)
    w, w_scales, _ = quantized(rng(4), n, k)
    d, want = torch.empty((m, n), dtype=out, device=DEV), torch.empty((m, n), dtype=out, device=DEV)
    q.check(q.quartet_mxfp4_gemm(a, a_scales, w, w_scales, m, n, k, 0.75, want, code(want), n))
    q.check(b.quartet_mxfp4_gemm_act(a, a_scales, w, w_scales, m, n, k, 0.75, None, 0, 0, None, 0, None, 0, 0, None, 0, d, code(d), n))
    assert torch.equal(d, want)


# What the norm's rounding adds up to, in half steps u of fp32: squares, sum, quotient and root are in 64 bits and rounded to fp32 once: rstd within u, v, two
# products more, within 3 u (and what is smaller by 2^-24 and more).
@pytest.mark.parametrize("rows,n", [(3, 8), (33, 1376), (130, 1003), (2, 8192), (2, 32768), (700, 4096)])
def test_norm_statistic_in_64_bits(monkeypatch, rows, n):
    monkeypatch.setattr(N, "RSTD", 1.01 * U32)
    monkeypatch.setattr(N, "V", 3.02 * U32)
    for types in ((BF16, None, F32), (F32, F32, F32), (BF16, F32, BF16)):
        N.test_forward(rows, n, *types)
    if n % 32 == 0:
        N.test_mxfp8_operand(rows, n, F32)
        N.test_mxfp4_operand(rows, n, F32, True)


@pytest.mark.parametrize("scale,eps", [(1e20, 1e-5), (1e30, 1e-5), (1e-25, 0.0), (1e-30, 0.0)])
@pytest.mark.parametrize("rows,n", [(3, 100), (5, 4096), (2, 16392)])
def test_norm_of_values_whose_squares_fp32_cannot_hold(rows, n, scale, eps):
    # the mean is finite and not 0, so is everything behind it
    for dtype in (BF16, F32):
        o = N.forward(rng(5), rows, n, dtype, None, F32, eps=eps, scale=scale)
        assert_within(o["rstd"][:rows], o["want_rstd"], o["want_rstd"] * N.RSTD, "rstd")
        assert_within(o["y"], o["want_v"], o["want_v"].abs() * (HALF[BF16] + 2 * N.V), "y")
        # the backward pass from that statistic: bounds as in the norm's own test
        dy, h, w, rstd, ld = matrix(rng(6), rows, n, BF16, 0.01), o["x"], o["w"], o["rstd"][:rows], o["x"].shape[1]
        dx, dw, size = torch.empty_like(h), torch.empty(n, device=DEV), b.quartet_rmsnorm_bwd_workspace_bytes(rows, n)
        q.check(b.quartet_rmsnorm_bwd(dy, ld, h, code(h), ld, rows, n, w, 0, rstd, None, 0, dx, ld, None, 0, dw, torch.empty(size, dtype=torch.uint8, device=DEV), size))
        gd, hd, r = dy[:, :n].double() * w.double(), h[:, :n].double(), rstd.double()[:, None]
        gh = gd * hd
        want = r * (gd - hd * r * r * gh.mean(1, keepdim=True))
        assert_within(dx[:, :n], want, 36 * U32 * hd.abs() * r ** 3 * gh.abs().mean(1, keepdim=True) + 6 * U32 * r * gd.abs() + want.abs() * HALF[dtype], "dx")
        terms = dy[:, :n].double() * hd * r
        assert_within(dw, terms.sum(0), (rows / 64 + 200) * U32 * terms.abs().sum(0), "dw")


@pytest.mark.parametrize("variant", [-1, 0, 1, 2, 22])
@pytest.mark.parametrize("m,n", [(1, 8), (5, 256), (40, 4096), (129, 300), (200, 512), (257, 1001)])
def test_product_leaves_the_rows_behind_the_last_one(variant, m, n):
    # a tile has up to 256 rows; every row that it could reach lies in the buffer
    k = 96
    a, a_scales, _ = quantized(rng(7), m, k)
    w, w_scales, _ = quantized(rng(8), n, k)
    ld = (n + 7) // 8 * 8 + 8
    try:
        q.check(q.quartet_debug_set_gemm_plan(variant, 0))
        for out in (BF16, F32):
            d, pre = (torch.full((m + 520, ld), GUARD, dtype=t, device=DEV) for t in (out, BF16))
            res, up = (torch.ones((m + 520, ld), dtype=t, device=DEV) for t in (F32, BF16))
            q.check(b.quartet_mxfp4_gemm_act(a, a_scales, w, w_scales, m, n, k, 1.0, None, 0, 3, up, ld, res, 0, ld, pre, ld, d, code(d), ld))
            for t in (d, pre):
                assert bool((t[m:] == GUARD).all()) and bool((t[:m, n:] == GUARD).all()) and not bool((t[:m, :n] == GUARD).any())
    finally:
        q.quartet_debug_set_gemm_plan(-1, 0)
