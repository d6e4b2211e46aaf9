"""quartet_act_bwd against plain versions in 64 bits, and quartet_grad_clip.

Tolerances: with u = 2^-24 the gate s(t) is off by at most (|t| + 8) u relative to itself or to 1 (2^x, sum and reciprocal to an ulp each, the argument's two
roundings times |t|), |t| <= 2.5 |z| + 0.1 |z|^3 wherever s(t) is not 0 or 1 to fp32; value and slope are sums of products of it with factors
no larger than 2 + |z|."""
import pytest
import torch

from block_util import BF16, DEV, F32, GUARD, HALF, U16, U32, act, assert_within, b, code, guarded, ld_of, matrix, output, q, rng

pytestmark = pytest.mark.gpu


def backward(g, m, n, kind, mul=True, dbias=True, dmul=True, extra=0, scale=2.0):
    dy, pre = matrix(g, m, n, BF16, 0.01, extra), matrix(g, m, n, BF16, scale, extra)
    gate = matrix(g, m, n, BF16, 1.0, extra) if mul else None
    wz, dz = output(m, n, BF16, extra)
    wm, dm = output(m, n, BF16, extra)
    db = torch.full((n + 1,), GUARD, device=DEV) if dbias else None
    size = b.quartet_act_bwd_workspace_bytes(m, n)
    ws = torch.full((size + 64,), 0xEE, dtype=torch.uint8, device=DEV)
    ld = dy.shape[1]
    q.check(b.quartet_act_bwd(dy, ld, pre, ld, gate, ld, m, n, b.ACTIVATIONS[kind], dz, ld, dm if dmul else None, ld, db, ws, size))
    torch.cuda.synchronize()
    assert bool((ws[size:] == 0xEE).all()) and guarded(wz, n) and guarded(wm, n)
    z, d = pre[:, :n].double(), dy[:, :n].double()
    value, slope = act(z, kind)
    dgate = d if gate is None else d * gate[:, :n].double()
    off = (z.abs() * 2.5 + z.abs() ** 3 * 0.1).clamp_max(104) + 12      # beyond |t| = 104 the gate is 0 or 1
    assert_within(dz[:, :n], dgate * slope, dgate.abs() * (slope.abs() * U16 + 2 * (2 + z.abs()) * off * U32), "dz")
    if dmul:
        assert_within(dm[:, :n], d * value, d.abs() * (value.abs() * U16 + z.abs() * off * 2 * U32), "dmul")
    if dbias:
        terms = dgate * slope
        assert_within(db[:n], terms.sum(0), (m / 16 + 300) * U32 * terms.abs().sum(0) + (dgate.abs() * 2 * (2 + z.abs()) * off * U32).sum(0), "dbias")
        assert float(db[n]) == GUARD
    return dict(dy=dy, pre=pre, gate=gate, dz=dz[:, :n].clone(), dm=dm[:, :n].clone(), db=None if db is None else db[:n].clone(), ld=ld)


@pytest.mark.parametrize("kind", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("mul", [False, True])
@pytest.mark.parametrize("m,n", [(1, 1), (1, 4096), (3, 9), (17, 512), (5, 513), (1003, 200), (64, 11008), (300, 1003), (5000, 96)])
def test_backward(m, n, kind, mul):
    backward(rng(m + n), m, n, kind, mul, extra=8 * (m % 2), dmul=True)


@pytest.mark.parametrize("dbias", [False, True])
def test_more_rows_than_blocks_of_the_usual_size(dbias):
    m, n = 2 ** 25 + 5, 8
    dy, pre = torch.empty((m, n), dtype=BF16, device=DEV).normal_(generator=rng(5)), torch.empty((m, n), dtype=BF16, device=DEV).normal_(generator=rng(6))
    dz, db = torch.full((m + 1, n), GUARD, dtype=BF16, device=DEV), torch.empty(n, device=DEV) if dbias else None
    size = b.quartet_act_bwd_workspace_bytes(m, n)
    q.check(b.quartet_act_bwd(dy, n, pre, n, None, 0, m, n, 1, dz, n, None, 0, db, torch.empty(size, dtype=torch.uint8, device=DEV), size))
    want = torch.where(pre > 0, dy, torch.zeros_like(dy))
    assert torch.equal(dz[:m], want) and bool((dz[m] == GUARD).all())
    if dbias:      # partial sums of 16 rows and their sums over 2^21 / 32 of them in a thread
        assert_within(db, want.double().sum(0), (2 ** 16 + 64) * U32 * want.double().abs().sum(0))


def test_far_values():
    # gates that are 0 or 1 in every type, squares that overflow
    for kind in ("gelu", "silu", "relu", "none"):
        g = rng(2)
        n = 64
        dy, z = torch.ones((1, n), dtype=BF16, device=DEV), torch.zeros((1, n), dtype=BF16, device=DEV)
        z[0, :8] = torch.tensor([0.0, -0.0, 100.0, -100.0, 1e30, -1e30, 3e38, -3e38])
        dz, dm = torch.empty_like(z), torch.empty_like(z)
        q.check(b.quartet_act_bwd(dy, n, z, n, dy, n, 1, n, b.ACTIVATIONS[kind], dz, n, dm, n, None, None, 0))
        half = {"gelu": 0.5, "silu": 0.5, "relu": 0.0, "none": 1.0}[kind]
        low = 1.0 if kind == "none" else 0.0
        assert dz[0, :8].tolist() == [half, half, 1.0, low, 1.0, low, 1.0, low]
        want = z[0, :8].clone()
        if kind != "none":
            want[want < 0] = 0
        assert torch.equal(dm[0, :8].abs(), want.abs())


def test_in_place_and_parts():
    m, n = 70, 1003
    o = backward(rng(3), m, n, "silu")
    ld = o["ld"]
    dy, gate, pre = o["dy"].clone(), o["gate"].clone(), o["pre"].clone()
    q.check(b.quartet_act_bwd(dy, ld, pre, ld, gate, ld, m, n, 3, dy, ld, gate, ld, None, None, 0))
    assert torch.equal(dy[:, :n], o["dz"]) and torch.equal(gate[:, :n], o["dm"])
    q.check(b.quartet_act_bwd(o["dy"], ld, pre, ld, o["gate"], ld, m, n, 3, None, 0, pre, ld, None, None, 0))
    assert torch.equal(pre[:, :n], o["dm"])
    # the bias of a plain product: column sums of dy alone
    db, size = torch.empty(n, device=DEV), b.quartet_act_bwd_workspace_bytes(m, n)
    q.check(b.quartet_act_bwd(o["dy"], ld, None, 0, None, 0, m, n, 0, None, 0, None, 0, db, torch.empty(size, dtype=torch.uint8, device=DEV), size))
    d = o["dy"][:, :n].double()
    assert_within(db, d.sum(0), 100 * U32 * d.abs().sum(0))
    empty = torch.full((n,), GUARD, device=DEV)
    q.check(b.quartet_act_bwd(o["dy"], ld, None, 0, None, 0, 0, n, 0, None, 0, None, 0, empty, None, 0))
    assert bool((empty == 0).all())


def test_values_that_are_not_finite_stay_where_they_are():
    m, n = 20, 40
    o = backward(rng(4), m, n, "gelu", dbias=False)
    dy = o["dy"].clone()
    dy[3, 4], dy[5, 6] = float("nan"), float("inf")
    dz, dm, db = torch.empty_like(dy), torch.empty_like(dy), torch.empty(n, device=DEV)
    size = b.quartet_act_bwd_workspace_bytes(m, n)
    q.check(b.quartet_act_bwd(dy, o["ld"], o["pre"], o["ld"], o["gate"], o["ld"], m, n, 2, dz, o["ld"], dm, o["ld"], db, torch.empty(size, dtype=torch.uint8, device=DEV), size))
    same = torch.ones((m, n), dtype=torch.bool, device=DEV)
    same[3, 4] = same[5, 6] = False
    assert torch.equal(dz[:, :n][same], o["dz"][same]) and bool(torch.isnan(dz[3, 4])) and not bool(torch.isfinite(dz[5, 6]))
    assert torch.isfinite(db).tolist() == [c not in (4, 6) for c in range(n)]


def test_slopes_against_differences():
    z = torch.linspace(-12, 12, 4096, device=DEV).to(BF16)
    one = torch.ones_like(z)
    for kind in ("gelu", "silu"):
        dz = torch.empty_like(z)
        q.check(b.quartet_act_bwd(one, 4096, z, 4096, None, 0, 1, 4096, b.ACTIVATIONS[kind], dz, 4096, None, 0, None, None, 0))
        d = 1e-6
        want = (act(z.double() + d, kind)[0] - act(z.double() - d, kind)[0]) / (2 * d)
        assert_within(dz, want, want.abs() * U16 + 1e-5)


# ---------------------------------------------------------------------------------------------- gradient norm and clipping

def clip(grads, outs, max_norm):
    size = b.quartet_grad_clip_workspace_bytes()
    ws = torch.full((size + 64,), 0xEE, dtype=torch.uint8, device=DEV)
    norm = torch.full((3,), GUARD, device=DEV)
    tensors = b.grad_tensors(grads, outs)
    q.check(b.quartet_grad_clip(tensors, len(tensors), max_norm, norm[1:2], ws, size))
    torch.cuda.synchronize()
    assert bool((ws[size:] == 0xEE).all()) and norm[[0, 2]].tolist() == [GUARD, GUARD]
    return float(norm[1])


def check_clip(grads, outs, max_norm, before=None):
    before = [t.double() for t in grads] if before is None else before
    norm = clip(grads, outs, max_norm)
    want = sum(float(t.square().sum()) for t in before) ** 0.5
    assert norm == pytest.approx(want, rel=2 * U32, abs=1e-45)           # fp64 sums, one rounding
    factor = min(1.0, max_norm / (want + 1e-6))
    for t, o in zip(before, outs):
        assert_within(o, t * factor, (t * factor).abs() * (HALF[o.dtype] + 5 * U32))      # sum, quotient, product: a rounding each, and the norm's
    return norm


SIZES = [[1], [7, 0, 8, 1], [8192], [8193, 8191, 1], [100000, 3, 77777], [5] * 79, [5] * 80, [33] * 81, [17] * 500, [3000000, 11],
         [4096 * 1024], [4096 * 1024, 1], [9000000, 5, 4097], [34000000, 9]]


@pytest.mark.parametrize("g_dtype,o_dtype", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
def test_clip_into_copies(sizes, g_dtype, o_dtype):
    g = rng(len(sizes) + sum(sizes))
    grads = [torch.randn(s, generator=g, device=DEV).to(g_dtype) for s in sizes]
    guard = [torch.full((s + 16,), GUARD, dtype=o_dtype, device=DEV) for s in sizes]
    outs = [t[8:8 + s] for t, s in zip(guard, sizes)]
    for max_norm in (0.5, 1e9, 0.0, float("inf")):
        check_clip(grads, outs, max_norm)
        assert all(bool((t[:8] == GUARD).all() and (t[8 + s:] == GUARD).all()) for t, s in zip(guard, sizes))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("offset", [0, 1, 3, 5])
def test_clip_in_place_at_any_alignment(dtype, offset):
    g = rng(offset)
    flat = torch.randn(50000, generator=g, device=DEV).to(dtype)
    cuts = [offset, offset + 1, offset + 8200, offset + 8203, offset + 40000]
    views = [flat[a:e] for a, e in zip(cuts, cuts[1:])]
    before, rest = [v.double() for v in views], flat.clone()
    check_clip(views, views, 1.0, before)
    assert torch.equal(flat[:cuts[0]], rest[:cuts[0]]) and torch.equal(flat[cuts[-1]:], rest[cuts[-1]:])
    kept = flat.clone()
    assert clip(views, views, 10.0) == pytest.approx(1.0, rel=2 * U16) and torch.equal(flat, kept)      # below the largest norm: untouched


def test_clip_range_of_values():
    for scale in (1e-30, 1e-12, 1e25):                         # squares that fp32 cannot hold
        grads = [torch.randn(1000, generator=rng(1), device=DEV) * scale]
        check_clip(grads, [torch.empty_like(grads[0])], 1.0)
    zero = [torch.zeros(9, device=DEV)]
    assert clip(zero, zero, 1.0) == 0.0 and bool((zero[0] == 0).all())
    assert clip([], [], 1.0) == 0.0


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_clip_leaves_a_step_that_is_not_finite(bad):
    g = torch.randn(20000, generator=rng(2), device=DEV)
    g[12345] = bad
    kept, copy = g.clone(), torch.zeros(20000, dtype=BF16, device=DEV)
    norm = clip([g], [g], 1.0)
    assert norm != norm or norm == float("inf")
    assert torch.equal(g.view(torch.int32), kept.view(torch.int32))
    clip([g], [copy], 1.0)
    assert torch.equal(copy.nan_to_num(7.0), kept.to(BF16).nan_to_num(7.0))


def test_clip_same_bits_every_time():
    grads = [torch.randn(s, generator=rng(s), device=DEV).to(BF16) for s in (1 << 20, 12345, 777777)]
    outs = [torch.empty(t.numel(), device=DEV) for t in grads]
    first = clip(grads, outs, 0.1)
    kept = [o.clone() for o in outs]
    assert clip(grads, outs, 0.1) == first and all(torch.equal(a, c) for a, c in zip(kept, outs))
