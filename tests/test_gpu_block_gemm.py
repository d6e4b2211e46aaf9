"""quartet_mxfp4_gemm_act against the product and its epilogue in 64 bits.

Tolerances: the products are exact and summed in fp32 on the matrix cores: off by (k / 64 + 3) 2^-23 of the sum of their magnitudes at most (the bound
of the plain product's tests); scale, bias: a rounding each.  The activation's slope is below 1.13 and its own arithmetic is good to (|t| + 8) 2^-24 of
|z| (test_gpu_block_act.py); gate and residual add a rounding each, the result's type the last."""
import pytest
import torch

from block_util import BF16, DEV, F32, GUARD, HALF, U16, U32, act, assert_within, b, code, guarded, matrix, output, q, quantized, rng

pytestmark = pytest.mark.gpu


def product(g, m, n, k, kind="none", bias=None, mul=False, res=None, pre=False, out=BF16, alpha=1.0, extra=0, odd_ld=False, in_place=None):
    A, As, a = quantized(g, m, k)
    B, Bs, w = quantized(g, n, k, max(k, 1) ** -0.5)
    bias_t = None if bias is None else torch.randn(n, generator=g, device=DEV).to(bias)
    shape = lambda t: t if t is None or not odd_ld else torch.as_strided(torch.cat([t.reshape(-1), t.new_zeros(8)]).clone(), (t.shape[0], t.shape[1]), (t.shape[1], 1))
    gate, stream = matrix(g, m, n, BF16, 1.0, extra) if mul else None, matrix(g, m, n, res, 1.0, extra) if res else None
    whole, d = output(m, n, out, extra)
    whole_pre, z_out = output(m, n, BF16, extra)
    if odd_ld:       # rows n apart: any column may start a row
        pack = lambda t: None if t is None else t[:, :n].contiguous()
        gate, stream = pack(gate), pack(stream)
        d, z_out = torch.full((m, n), GUARD, dtype=out, device=DEV), torch.full((m, n), GUARD, dtype=BF16, device=DEV)
    before = {"mul": gate, "res": stream}
    gate_v, stream_v = (None if t is None else t[:, :n].double() for t in (gate, stream))
    if in_place:
        d = before[in_place]
    ld = lambda t: 0 if t is None else t.shape[1]
    q.check(b.quartet_mxfp4_gemm_act(A, As, B, Bs, m, n, k, alpha, bias_t, code(bias_t), b.ACTIVATIONS[kind], gate, ld(gate), stream, code(stream), ld(stream),
                                     z_out if pre else None, ld(z_out), d, code(d), ld(d)))
    torch.cuda.synchronize()
    z = alpha * (a @ w.t()) + (0 if bias_t is None else bias_t.double())
    off_z = abs(alpha) * (k / 64 + 3) * 2.0 ** -23 * (a.abs() @ w.abs().t()) + 4 * U32 * (z.abs() + (0 if bias_t is None else bias_t.double().abs()))
    value, _ = act(z, kind)
    t = (z.abs() * 2.5 + z.abs() ** 3 * 0.1).clamp_max(104) + 12
    off = 1.13 * off_z + (0 if kind in ("none", "relu") else z.abs() * t * 2 * U32)
    want = value
    if gate_v is not None:
        want, off = want * gate_v, off * gate_v.abs() + 2 * U32 * (value * gate_v).abs()
    if stream_v is not None:
        off = off + 2 * U32 * (want.abs() + stream_v.abs())
        want = want + stream_v
    assert_within(d[:, :n], want, off * (1 + U16) + want.abs() * HALF[out], "d")
    if pre:
        assert_within(z_out[:, :n], z, off_z * (1 + U16) + z.abs() * U16, "pre")
    if not in_place and not odd_ld:
        assert guarded(whole, n) and (not pre or guarded(whole_pre, n))
    return d[:, :n].clone()


FULL = dict(kind="gelu", bias=F32, mul=True, res=F32, pre=True)


@pytest.mark.parametrize("m,n,k", [(1, 1, 32), (1, 8, 0), (3, 5, 64), (24, 1000, 4096), (33, 65, 96), (64, 64, 256), (100, 257, 2848), (129, 300, 512), (1003, 520, 1376),
                                   (512, 512, 512), (300, 2048, 288), (2000, 1003, 320)])
@pytest.mark.parametrize("out", [BF16, F32])
def test_everything_at_once(m, n, k, out):
    product(rng(m + n + k), m, n, k, out=out, extra=8 * (m % 2), **FULL)


@pytest.mark.parametrize("kind", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("m,n,k", [(24, 512, 512), (700, 640, 512)])
def test_activations(kind, m, n, k):
    product(rng(1), m, n, k, kind, out=F32)
    product(rng(2), m, n, k, kind, bias=BF16, out=BF16, alpha=-0.5)


@pytest.mark.parametrize("bias", [None, BF16, F32])
@pytest.mark.parametrize("res", [None, BF16, F32])
@pytest.mark.parametrize("mul", [False, True])
@pytest.mark.parametrize("m,n,k", [(40, 256, 512), (900, 1000, 512)])
def test_operands_of_the_epilogue(bias, res, mul, m, n, k):
    product(rng(3), m, n, k, "silu", bias, mul, res, pre=mul, out=F32 if res == F32 else BF16)


@pytest.mark.parametrize("m,n,k", [(20, 33, 64), (300, 1001, 512), (517, 258, 1024)])
def test_rows_at_any_distance(m, n, k):
    product(rng(4), m, n, k, odd_ld=True, out=BF16, **FULL)
    product(rng(5), m, n, k, odd_ld=True, out=F32, **FULL)


@pytest.mark.parametrize("m,n,k", [(24, 512, 512), (2048, 1024, 512), (1003, 500, 320)])
def test_in_place(m, n, k):
    want = product(rng(6), m, n, k, "silu", res=F32, out=F32)
    assert torch.equal(product(rng(6), m, n, k, "silu", res=F32, out=F32, in_place="res"), want)
    want = product(rng(7), m, n, k, "gelu", mul=True, res=F32, out=BF16)
    assert torch.equal(product(rng(7), m, n, k, "gelu", mul=True, res=F32, out=BF16, in_place="mul"), want)
    want = product(rng(8), m, n, k, res=BF16, out=BF16)
    assert torch.equal(product(rng(8), m, n, k, res=BF16, out=BF16, in_place="res"), want)


def test_rows_far_apart():
    # rows of 2^21 elements: the last ones lie past 2^32 bytes, in the split kernels and in the streaming ones
    m, n, k, ld = 1100, 64, 64, 2 ** 21
    A, As, a = quantized(rng(17), m, k)
    B, Bs, w = quantized(rng(18), n, k, 0.1)
    res, d = torch.empty((m, ld), device=DEV), torch.empty((m, ld), dtype=BF16, device=DEV)
    res[:, :n] = torch.randn((m, n), generator=rng(19), device=DEV)
    want = a @ w.t() + res[:, :n].double()
    off = 5 * 2.0 ** -23 * (a.abs() @ w.abs().t() + res[:, :n].double().abs()) + want.abs() * U16 * 1.01
    try:
        for variant in (-1, 0, 1, 2, 22):
            q.check(q.quartet_debug_set_gemm_plan(variant, 0))
            d[:, :n] = GUARD
            q.check(b.quartet_mxfp4_gemm_act(A, As, B, Bs, m, n, k, 1.0, None, 0, 0, None, 0, res, 0, ld, None, 0, d, 1, ld))
            assert_within(d[:, :n], want, off, variant)
    finally:
        q.quartet_debug_set_gemm_plan(-1, 0)


# every kernel that the sizes pick: block tiles of 256 x 256, 128 x 256, 128 x 128 (one block and two per compute unit) and the in-block split's
@pytest.mark.parametrize("m,n,k", [(4096, 4096, 1024), (2100, 4448, 320), (4096, 2048, 2048), (2048, 2048, 4096), (10327, 992, 800), (1003, 5632, 2048), (16640, 1280, 256)])
@pytest.mark.parametrize("epilogue", [dict(kind="gelu", bias=BF16, pre=True), dict(kind="silu", mul=True), dict(res=F32, out=F32), dict(res=BF16), FULL], ids=str)
def test_large(m, n, k, epilogue):
    product(rng(9), m, n, k, **epilogue)


@pytest.fixture()
def plan():
    yield lambda variant: q.check(q.quartet_debug_set_gemm_plan(variant, 0))
    q.quartet_debug_set_gemm_plan(-1, 0)


@pytest.mark.parametrize("variant", [0, 1, 2, 22])
@pytest.mark.parametrize("m,n,k", [(256, 256, 256), (512, 1024, 96), (300, 520, 544), (1, 8, 32), (700, 1001, 320), (40, 4096, 2048)])
def test_every_streaming_kernel(plan, variant, m, n, k):
    plan(variant)
    for epilogue in (FULL, dict(kind="silu", mul=True), dict(res=BF16, bias=F32), dict(res=F32, out=F32, pre=True), dict(kind="relu"), dict()):
        product(rng(10), m, n, k, **epilogue)


@pytest.mark.parametrize("variant", [-1, 0, 1, 2, 22])
def test_without_an_epilogue_it_is_the_plain_product(plan, variant):
    plan(variant)
    m, n, k = 600, 768, 1024
    A, As, _ = quantized(rng(11), m, k)
    B, Bs, _ = quantized(rng(12), n, k)
    for out in (BF16, F32):
        d, want = torch.empty((m, n), dtype=out, device=DEV), torch.empty((m, n), dtype=out, device=DEV)
        q.check(q.quartet_mxfp4_gemm(A, As, B, Bs, m, n, k, 0.75, want, code(want), n))
        q.check(b.quartet_mxfp4_gemm_act(A, As, B, Bs, m, n, k, 0.75, None, 0, 0, None, 0, None, 0, 0, None, 0, d, code(d), n))
        # the same kernel sums in the same order; without a forced plan the two calls may take kernels that sum in another
        bound = 0 if variant >= 0 else want.double().abs() * HALF[out] * 2 + 1e-4
        assert_within(d, want, bound)


def test_values_that_are_not_finite_stay_in_their_place():
    m, n, k = 300, 512, 512
    A, As, _ = quantized(rng(13), m, k)
    B, Bs, _ = quantized(rng(14), n, k)
    res, gate = matrix(rng(15), m, n, F32), matrix(rng(16), m, n, BF16)
    run = lambda: (d := torch.empty((m, n), device=DEV), q.check(b.quartet_mxfp4_gemm_act(A, As, B, Bs, m, n, k, 1.0, None, 0, 3, gate, n, res, 0, n, None, 0, d, 0, n)))[0]
    want = run()
    res[7, 9], gate[200, 300], res[299, 511] = float("inf"), float("nan"), float("-inf")
    got = run()
    changed = [(7, 9), (200, 300), (299, 511)]
    assert got[7, 9] == float("inf") and bool(torch.isnan(got[200, 300])) and got[299, 511] == float("-inf")
    for r, c in changed:
        got[r, c] = want[r, c]
    assert torch.equal(got, want)
