"""Host-side checks of include/quartet_block.h that need no GPU: exports, the binding, workspace sizes and every refusal."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "quartet_block.h")
LIB = os.path.join(ROOT, "paper_2505_14669_amd", "libquartet.so")

pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="HIP library not built (run __graft_entry__.build())")
P = 0x10000       # fake, aligned, never dereferenced: every call here is refused or empty


def declared_symbols():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return sorted(set(re.findall(r"\b(quartet_[a-z0-9_]+)\s*\(", text)))


@pytest.fixture(scope="module")
def b():
    from paper_2505_14669_amd import block
    return block


def launches(b):
    """kernel launches so far in the host-only build with counting stand-ins for the launchers; None in the library itself"""
    try:
        return b._lib.quartet_hostcheck_block_launches()
    except AttributeError:
        return None


def test_library_and_binding_have_every_declared_symbol(b):
    lib = ctypes.CDLL(LIB)
    assert sorted(b.EXPORTS) == declared_symbols()
    for name in declared_symbols():
        assert hasattr(lib, name) and callable(getattr(b, name)), name


GEMM = dict(a_codes=P, a_scales=P, b_codes=P, b_scales=P, m=4, n=24, k=64, alpha=1.0, bias=P, bias_dtype=0, activation=1, multiplier_bf16=P, ldmul=24,
            residual=P, residual_dtype=0, ldres=24, pre_bf16=2 * P, ldpre=24, d=3 * P, d_dtype=0, ldd=24, stream=0)


@pytest.mark.parametrize("change", [
    dict(a_codes=None), dict(d=None), dict(b_codes=P + 8), dict(b_scales=P + 2), dict(m=-1), dict(k=48), dict(ldd=23), dict(d_dtype=2), dict(activation=4),
    dict(activation=-1), dict(bias_dtype=3), dict(bias=P + 4), dict(residual=P + 8), dict(residual_dtype=5), dict(ldres=20), dict(multiplier_bf16=P + 2),
    dict(ldmul=8), dict(pre_bf16=P + 8), dict(ldpre=16), dict(pre_bf16=3 * P), dict(pre_bf16=P), dict(residual=3 * P, residual_dtype=1),
    dict(residual=3 * P, ldres=32), dict(multiplier_bf16=3 * P)])
def test_gemm_act_refuses(b, change):
    before = launches(b)
    assert b.quartet_mxfp4_gemm_act(**{**GEMM, **change}) == b.QUARTET_EINVAL
    assert launches(b) == before


@pytest.mark.parametrize("change", [dict(ldres=2 ** 21 + 1), dict(ldmul=2 ** 22), dict(ldpre=2 ** 30), dict(ldd=2 ** 22), dict(k=2 ** 24), dict(m=2 ** 31)])
def test_gemm_act_does_not_support(b, change):
    assert b.quartet_mxfp4_gemm_act(**{**GEMM, **change}) == b.QUARTET_ENOTSUP


def test_gemm_act_looks_at_nothing_that_is_not_given(b):
    args = {**GEMM, **dict(m=0, bias=None, bias_dtype=9, multiplier_bf16=None, ldmul=-3, residual=None, residual_dtype=9, ldres=2 ** 40, pre_bf16=None, ldpre=0)}
    assert b.quartet_mxfp4_gemm_act(**args) == b.QUARTET_OK


ACT = dict(dy_bf16=P, lddy=24, pre_bf16=2 * P, ldpre=24, multiplier_bf16=3 * P, ldmul=24, m=4, n=20, activation=3, dz_bf16=4 * P, lddz=24, dmul_bf16=5 * P,
           lddmul=24, dbias=6 * P, workspace=7 * P, workspace_bytes=1 << 30, stream=0)


@pytest.mark.parametrize("change", [
    dict(dy_bf16=None), dict(dy_bf16=P + 8), dict(lddy=16), dict(lddy=20), dict(pre_bf16=None), dict(pre_bf16=None, activation=0), dict(m=-1), dict(n=-1),
    dict(activation=4), dict(multiplier_bf16=P + 2), dict(ldmul=21), dict(dz_bf16=4 * P + 8), dict(lddz=12), dict(lddmul=8), dict(dbias=P + 4),
    dict(dz_bf16=None, dmul_bf16=None, dbias=None), dict(workspace=None), dict(workspace=P + 8), dict(workspace_bytes=95), dict(dz_bf16=P, lddz=32),
    dict(dz_bf16=5 * P), dict(dz_bf16=2 * P), dict(dz_bf16=3 * P), dict(dmul_bf16=P), dict(dmul_bf16=2 * P, lddmul=32), dict(dmul_bf16=3 * P, lddmul=32)])
def test_act_bwd_refuses(b, change):
    before = launches(b)
    assert b.quartet_act_bwd(**{**ACT, **change}) == b.QUARTET_EINVAL
    assert launches(b) == before


def test_act_bwd_sizes(b):
    assert b.quartet_act_bwd(**{**ACT, "m": 2 ** 31}) == b.QUARTET_ENOTSUP
    assert b.quartet_act_bwd(**{**ACT, "n": 2 ** 26 + 8, **{k: 2 ** 26 + 8 for k in ACT if k.startswith("ld")}}) == b.QUARTET_ENOTSUP
    assert b.quartet_act_bwd(**{**ACT, "m": 0, "dbias": None, "workspace": None, "workspace_bytes": 0}) == b.QUARTET_OK
    assert b.quartet_act_bwd(**{**ACT, "n": 0, "workspace": None}) == b.QUARTET_OK
    assert b.quartet_act_bwd_workspace_bytes(4, 20) == 96 and b.quartet_act_bwd_workspace_bytes(0, 20) == 0
    assert b.quartet_act_bwd_workspace_bytes(-1, 20) == 0 and b.quartet_act_bwd_workspace_bytes(2 ** 31, 20) == 0
    for m in (1, 15, 16, 17, 1003, 16384, 2 ** 22, 2 ** 31 - 1):
        for n in (1, 511, 512, 513, 11008, 2 ** 20):
            assert 0 < b.quartet_act_bwd_workspace_bytes(m, n) <= (m + 15) // 16 * (n + 7) * 4


NORM = dict(x=P, x_dtype=1, ldx=64, residual=2 * P, ldres=64, rows=4, n=64, weight=3 * P, weight_dtype=0, eps=1e-5, h=4 * P, h_dtype=0, ldh=64, y_bf16=5 * P,
            ldy=64, format=1, codes=6 * P, scales=7 * P, mask=8 * P, rstd=9 * P, stream=0)


@pytest.mark.parametrize("change", [
    dict(x=None), dict(x=P + 8), dict(ldx=56), dict(ldx=68), dict(x_dtype=2), dict(residual=P + 4), dict(ldres=60), dict(rows=-1), dict(n=0), dict(weight=None),
    dict(weight=P + 8), dict(weight_dtype=-1), dict(eps=-1e-9), dict(eps=float("nan")), dict(eps=float("inf")), dict(residual=None), dict(h_dtype=2),
    dict(ldh=8), dict(ldy=65), dict(format=3), dict(format=0), dict(format=2), dict(codes=None), dict(scales=None), dict(codes=P + 8), dict(scales=P + 2),
    dict(mask=P + 4), dict(n=60), dict(rstd=P + 2), dict(h=2 * P, ldh=72), dict(h=P), dict(h=5 * P), dict(y_bf16=P), dict(y_bf16=2 * P),
    dict(h=None, y_bf16=None, format=0, codes=None, scales=None, mask=None, rstd=None)])
def test_rmsnorm_fwd_refuses(b, change):
    before = launches(b)
    assert b.quartet_rmsnorm_fwd(**{**NORM, **change}) == b.QUARTET_EINVAL
    assert launches(b) == before


def test_rmsnorm_sizes(b):
    assert b.quartet_rmsnorm_fwd(**{**NORM, "n": 32800, "ldx": 32800, "ldres": 32800, "ldh": 32800, "ldy": 32800}) == b.QUARTET_ENOTSUP
    assert b.quartet_rmsnorm_fwd(**{**NORM, "rows": 2 ** 30}) == b.QUARTET_ENOTSUP
    assert b.quartet_rmsnorm_fwd(**{**NORM, "rows": 0}) == b.QUARTET_OK
    assert b.quartet_rmsnorm_bwd_workspace_bytes(0, 64) == 0 and b.quartet_rmsnorm_bwd_workspace_bytes(4, 0) == 0
    assert b.quartet_rmsnorm_bwd_workspace_bytes(4, 32769) == 0
    for rows in (1, 3, 1000, 10 ** 6):
        for n in (1, 7, 8, 2048, 32768):
            size = b.quartet_rmsnorm_bwd_workspace_bytes(rows, n)
            assert size % (4 * ((n + 7) // 8 * 8)) == 0 and 0 < size <= 1024 * 4 * (n + 7)


NORM_BWD = dict(dy_bf16=P, lddy=64, h=2 * P, h_dtype=0, ldh=64, rows=4, n=61, weight=3 * P, weight_dtype=1, rstd=4 * P, dh=5 * P, lddh=64, dx=6 * P, lddx=64,
                dx16=7 * P, lddx16=64, dweight=8 * P, workspace=9 * P, workspace_bytes=1 << 20, stream=0)


@pytest.mark.parametrize("change", [
    dict(dy_bf16=None), dict(lddy=60), dict(h=None), dict(h=P + 8), dict(h_dtype=2), dict(ldh=56), dict(weight=None), dict(weight_dtype=2), dict(rstd=None),
    dict(rstd=P + 2), dict(dh=P + 4), dict(lddh=61), dict(lddx=62), dict(lddx16=1), dict(dx=None), dict(h_dtype=1), dict(dweight=P + 4),
    dict(dx=None, dx16=None, dweight=None), dict(workspace=None), dict(workspace=P + 4), dict(workspace_bytes=100), dict(dx=5 * P, lddx=72),
    dict(dx=2 * P, lddx=72), dict(dx=7 * P), dict(dx=P), dict(dx16=P, lddx16=72), dict(dx16=2 * P), dict(dx16=5 * P), dict(rows=-1), dict(n=0)])
def test_rmsnorm_bwd_refuses(b, change):
    before = launches(b)
    assert b.quartet_rmsnorm_bwd(**{**NORM_BWD, **change}) == b.QUARTET_EINVAL
    assert launches(b) == before


def clip(b, entries, max_norm=1.0, norm=P, workspace=P, size=None, count=None):
    array = (b.GradTensor * max(1, len(entries)))(*[b.GradTensor(*e) for e in entries])
    size = b.quartet_grad_clip_workspace_bytes() if size is None else size
    return b.quartet_grad_clip(ctypes.addressof(array), len(entries) if count is None else count, max_norm, norm, workspace, size, 0)


@pytest.mark.parametrize("entries", [
    [(None, P, 4, 0, 0)], [(P, None, 4, 0, 0)], [(P, 2 * P, -1, 0, 0)], [(P, 2 * P, 4, 2, 0)], [(P, 2 * P, 4, 0, 7)], [(P + 2, 2 * P, 4, 0, 0)], [(P, 2 * P + 1, 4, 0, 1)],
    [(P, P, 4, 0, 1)], [(P, P + 8, 4, 0, 0)], [(P + 8, P, 4, 0, 0)], [(P, P, 8, 0, 0), (P, P, 8, 0, 0)], [(P, P, 8, 0, 0), (P + 28, P + 28, 8, 0, 0)],
    [(P, 2 * P, 8, 0, 0), (P, 2 * P, 8, 0, 0)], [(P, 2 * P, 8, 0, 0), (2 * P + 16, 3 * P, 8, 0, 0)], [(P, 2 * P, 64, 0, 0), (3 * P, P + 128, 8, 0, 0)],
    [(P, 4 * P, 64, 0, 0), (2 * P, 2 * P, 16, 1, 1), (3 * P, 2 * P + 30, 8, 0, 1)]])
def test_grad_clip_refuses_lists(b, entries):
    before = launches(b)
    assert clip(b, entries) == b.QUARTET_EINVAL
    assert launches(b) == before


def test_grad_clip_refuses(b):
    good = [(P, 2 * P, 4, 0, 0)]
    for kw in (dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(norm=None), dict(norm=P + 2), dict(workspace=None), dict(workspace=P + 8), dict(size=8), dict(count=-1)):
        assert clip(b, good, **kw) == b.QUARTET_EINVAL
    assert b.quartet_grad_clip(None, 1, 1.0, P, P, 1 << 20, 0) == b.QUARTET_EINVAL
    assert clip(b, [(P, 2 * P, 2 ** 43, 0, 0)]) == b.QUARTET_ENOTSUP
    assert clip(b, [(P, 2 ** 50, 2 ** 42, 0, 0), (2 ** 51, 2 ** 52, 2 ** 42, 0, 0)]) == b.QUARTET_ENOTSUP
    assert b.quartet_grad_clip(P, 2 ** 21, 1.0, P, P, 1 << 20, 0) == b.QUARTET_ENOTSUP
    many = [(P * (i + 1), P * (i + 1), P // 4, 0, 0) for i in range(700)]          # side by side: not an overlap
    many[699] = (P * 300 + 4, P * 300 + 4, 1, 0, 0)                                # inside another
    assert clip(b, many) == b.QUARTET_EINVAL
