"""quartet_rmsnorm_fwd and quartet_rmsnorm_bwd against plain versions in 64 bits.

Tolerances, counted in half steps u = 2^-24 of fp32: a row's sum of squares is a tree of at most 3 + 2 additions in a lane (four
chunks of eight), 6 across the wave and 16 across a row's waves, every term positive: 1 + 27 u with the square's own rounding, halved by the root;
quotient by n, eps, root and reciprocal add 2.5 u: rstd is within 17 u of the exact one.  v = h rstd w rounds twice more."""
import math

import pytest
import torch

from block_util import BF16, DEV, F32, GUARD, HALF, U16, U32, assert_within, b, code, guarded, ld_of, matrix, output, q, rng, scale_bytes_of

pytestmark = pytest.mark.gpu
RSTD, V = 17 * U32, 20 * U32


def forward(g, rows, n, x_dtype, res_dtype, w_dtype, fmt=0, extra=0, eps=1e-5, scale=1.0, want_y=True, mask=False, x=None):
    x = matrix(g, rows, n, x_dtype, scale, extra) if x is None else x
    res = None if res_dtype is None else matrix(g, rows, n, res_dtype, 2.0, extra)
    w = (1 + 0.2 * torch.randn(n, generator=g, device=DEV)).to(w_dtype)
    out = {"x": x, "res": res, "w": w, "rstd": torch.full((rows + 1,), GUARD, device=DEV)}
    out["h_all"], h = output(rows, n, res_dtype or F32, extra)
    out["y_all"], y = output(rows, n, BF16, extra)
    codes = scales = bits = None
    if fmt:
        per = n if fmt == b.QUARTET_FORMAT_MXFP8 else n // 2
        codes = torch.full((rows + 1, per), 0xEE, dtype=torch.uint8, device=DEV)
        scales = torch.full((q.quartet_scale_bytes(rows, n) + 64,), 0xEE, dtype=torch.uint8, device=DEV)
        bits = torch.full((rows + 1, n // 32), 0x5A5A5A5A, dtype=torch.int32, device=DEV) if mask else None
    ld = x.shape[1]
    q.check(b.quartet_rmsnorm_fwd(x, code(x), ld, res, ld, rows, n, w, code(w), eps, h if res is not None else None, code(h), ld, y if want_y else None, ld,
                                  fmt, codes, scales, bits, out["rstd"]))
    torch.cuda.synchronize()
    out |= {"h": h[:, :n], "y": y[:, :n], "codes": codes, "scales": scales, "mask": bits}
    # plain
    hs = x[:, :n] if res is None else (x[:, :n].float() + res[:, :n].float()).to(res_dtype)
    h64 = hs.double()
    out["want_h"] = hs
    out["want_rstd"] = (h64.square().mean(1) + eps).rsqrt()
    out["want_v"] = h64 * out["want_rstd"][:, None] * w.double()
    return out


CASES = [(1, 1), (1, 7), (3, 8), (5, 33), (1, 4096), (2, 512), (7, 520), (33, 1376), (64, 2048), (9, 2056), (130, 1003), (3, 4100), (2, 8192), (5, 11008), (1, 16385),
         (2, 32768), (700, 4096), (2100, 640)]


@pytest.mark.parametrize("x_dtype,res_dtype,w_dtype", [(BF16, None, F32), (BF16, BF16, BF16), (BF16, F32, F32), (F32, None, BF16), (F32, F32, F32), (F32, BF16, F32)])
@pytest.mark.parametrize("rows,n", CASES)
def test_forward(rows, n, x_dtype, res_dtype, w_dtype):
    o = forward(rng(rows * 31 + n), rows, n, x_dtype, res_dtype, w_dtype, extra=8 * (n % 3))
    if res_dtype is not None:
        assert torch.equal(o["h"], o["want_h"]) and guarded(o["h_all"], n)      # one addition, one rounding: the same bits
    assert guarded(o["y_all"], n) and float(o["rstd"][rows]) == GUARD
    assert_within(o["rstd"][:rows], o["want_rstd"], o["want_rstd"] * RSTD, "rstd")
    assert_within(o["y"], o["want_v"], o["want_v"].abs() * (U16 + 2 * V), "y")


def rest_untouched(o, rows, n):
    """the bytes of the scale buffer that stand for no group"""
    left = o["scales"].clone()
    r, g = torch.arange(rows, device=DEV)[:, None], torch.arange(n // 32, device=DEV)[None, :]
    left[((r // 32) * ((n // 32 + 7) // 8) + g // 8) * 256 + ((g % 2) * 32 + r % 32) * 4 + (g % 8) // 2] = 0xEE
    return bool((left == 0xEE).all())


@pytest.mark.parametrize("rows,n", [(1, 32), (1, 4096), (3, 96), (33, 1376), (40, 2048), (7, 4128), (130, 544), (2, 11008), (1, 32768), (2500, 256)])
@pytest.mark.parametrize("res_dtype", [None, BF16, F32])
def test_mxfp8_operand(rows, n, res_dtype):
    o = forward(rng(rows + n), rows, n, BF16, res_dtype, F32, b.QUARTET_FORMAT_MXFP8, scale=3.0, want_y=res_dtype is None)
    v = o["want_v"].view(rows, n // 32, 32)
    e = scale_bytes_of(o["scales"], rows, n // 32).double() - 127
    assert bool((o["codes"][rows] == 0xEE).all()) and rest_untouched(o, rows, n)
    top = v.abs().amax(2)
    # the largest magnitude lies in [2^8, 2^9) scales; next to a power of two the fp32 value may lie on its other side
    assert bool(((torch.ldexp(top, -e) >= 256 * (1 - 2 * V)) & (torch.ldexp(top, -e) < 512 * (1 + 2 * V))).all())
    got = o["codes"][:rows].view(torch.float8_e4m3fn).double().view(rows, n // 32, 32)
    s = torch.ldexp(v, -e[..., None])
    step = torch.ldexp(torch.ones_like(s), (torch.frexp(s.clamp(-448, 448)).exponent - 1).clamp_min(-6) - 3)
    assert_within(got, s.clamp(-448, 448), step / 2 + s.abs() * 2 * V, "codes")


@pytest.mark.parametrize("rows,n", [(1, 32), (1, 4096), (3, 96), (33, 1376), (40, 2048), (7, 4128), (130, 544), (2, 11008), (1, 32768), (2500, 256)])
@pytest.mark.parametrize("res_dtype,mask", [(None, True), (BF16, False), (F32, True)])
def test_mxfp4_operand(rows, n, res_dtype, mask):
    o = forward(rng(rows + n + 1), rows, n, BF16, res_dtype, F32, b.QUARTET_FORMAT_MXFP4, scale=3.0, mask=mask)
    v = o["want_v"].view(rows, n // 32, 32)
    i = torch.arange(32, device=DEV)
    x = i[:, None] & i[None, :]
    sign = 1.0 - 2.0 * ((x ^ (x >> 1) ^ (x >> 2) ^ (x >> 3) ^ (x >> 4)) & 1).double()
    h = (v.reshape(-1, 32) @ sign / math.sqrt(32)).view_as(v)
    # five butterflies and the factor, each rounding something no larger than the sum of magnitudes
    off = (2 * V + 7 * U32) * v.abs().sum(2, keepdim=True) / math.sqrt(32)
    e = scale_bytes_of(o["scales"], rows, n // 32).double() - 127
    ss = h.square().sum(2)
    slack = 2 * (off.squeeze(2) * h.abs().sum(2)) + 64 * U32 * ss
    lo, hi = torch.exp2(2 * e + 6), torch.exp2(2 * e + 8)                     # 2 e + 6 <= log2 ss < 2 e + 8
    assert bool(((ss + slack >= lo) & (ss - slack < hi)).all())
    raw = o["codes"][:rows].long()
    both = torch.stack((raw & 15, raw >> 4), 2).view(rows, n // 32, 32)
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64, device=DEV)
    s, off = torch.ldexp(h, -e[..., None]), torch.ldexp(off, -e[..., None])
    half = torch.where(s.abs() + off < 2, 0.25, torch.where(s.abs() + off < 4, 0.5, 1.0))
    assert_within(table[both], s.clamp(-6, 6), half + off, "codes")
    assert bool((o["codes"][rows] == 0xEE).all()) and rest_untouched(o, rows, n)
    if mask:
        kept = ((o["mask"][:rows].long()[..., None] >> i) & 1).bool()
        sure = (s.abs() - 6).abs() > off
        assert torch.equal(kept[sure], (s.abs() <= 6)[sure]) and bool((o["mask"][rows] == 0x5A5A5A5A).all())


@pytest.mark.parametrize("fmt", [b.QUARTET_FORMAT_MXFP4, b.QUARTET_FORMAT_MXFP8])
def test_operands_are_the_quantizers_own(fmt):
    # x holds +1 and -1 only, eps = 0: rstd = 1, v = w in bf16 exactly, so the operand must be the quantizer's of that matrix, bit for bit
    rows, n = 96, 1376
    g = rng(5)
    x = (torch.randint(0, 2, (rows, n), generator=g, device=DEV) * 2 - 1).to(BF16)
    w = torch.randn(n, generator=g, device=DEV).to(BF16)
    per = n if fmt == b.QUARTET_FORMAT_MXFP8 else n // 2
    new = lambda: (torch.zeros((rows, per), dtype=torch.uint8, device=DEV), torch.zeros(q.quartet_scale_bytes(rows, n), dtype=torch.uint8, device=DEV),
                   torch.zeros((rows, n // 32), dtype=torch.int32, device=DEV) if fmt == b.QUARTET_FORMAT_MXFP4 else None)
    got, want = new(), new()
    q.check(b.quartet_rmsnorm_fwd(x, 1, n, None, 0, rows, n, w, 1, 0.0, None, 0, 0, None, 0, fmt, *got, None))
    v = x * w
    if fmt == b.QUARTET_FORMAT_MXFP4:
        q.check(q.quartet_quant_fwd(v, rows, n, n, 0, *want))
    else:
        q.check(q.quartet_mxfp8_quant(v, rows, n, n, *want[:2]))
    for a, c in zip(got, want):
        assert a is None or torch.equal(a, c)


def test_rows_of_zeros_and_values_that_are_not_finite():
    n = 96
    x = matrix(rng(1), 5, n, BF16)
    x[1, :n] = 0
    x[2, 5], x[3, 7] = float("inf"), float("nan")
    for fmt in (b.QUARTET_FORMAT_NONE, b.QUARTET_FORMAT_MXFP8, b.QUARTET_FORMAT_MXFP4):
        o = forward(rng(2), 5, n, BF16, None, F32, fmt, x=x)
        assert bool((o["y"][1] == 0).all()) and float(o["rstd"][1]) == pytest.approx(1e-5 ** -0.5, rel=RSTD)
        assert float(o["rstd"][2]) == 0.0 and bool(torch.isnan(o["y"][2, 5])) and bool((o["y"][2, 6:] == 0).all()) and bool(torch.isnan(o["y"][3]).all())
        if fmt:
            assert bool((o["codes"][1] == 0).all())
            assert bool((scale_bytes_of(o["scales"], 5, n // 32)[1] == (0 if fmt == b.QUARTET_FORMAT_MXFP8 else 127)).all())
        for r in (0, 4):      # the other rows know nothing of it
            assert_within(o["y"][r], o["want_v"][r], o["want_v"][r].abs() * (U16 + 2 * V))


def test_in_place_and_optional_results():
    rows, n = 37, 1003
    o = forward(rng(3), rows, n, BF16, BF16, F32)
    ld = ld_of(n)
    for target in ("res", "x"):
        t = {"x": o["x"].clone(), "res": o["res"].clone()}
        q.check(b.quartet_rmsnorm_fwd(t["x"], 1, ld, t["res"], ld, rows, n, o["w"], 0, 1e-5, t[target], 1, ld, None, 0, 0, None, None, None, None))
        assert torch.equal(t[target][:, :n], o["h"])
    y = torch.empty((rows, ld), dtype=BF16, device=DEV)
    q.check(b.quartet_rmsnorm_fwd(o["x"], 1, ld, o["res"], ld, rows, n, o["w"], 0, 1e-5, None, 1, 0, y, ld, 0, None, None, None, None))      # h not stored
    assert torch.equal(y[:, :n], o["y"])


def test_rows_far_apart():
    # the second row's values lie past 2^32 bytes
    n, ld = 96, 2 ** 31 + 8
    x = torch.empty((2, ld), dtype=BF16, device=DEV)
    y = torch.empty((2, ld), dtype=BF16, device=DEV)
    x[:, :n] = torch.randn((2, n), generator=rng(4), device=DEV).to(BF16)
    w = torch.ones(n, device=DEV)
    q.check(b.quartet_rmsnorm_fwd(x, 1, ld, None, 0, 2, n, w, 0, 1e-5, None, 0, 0, y, ld, 0, None, None, None, None))
    h = x[:, :n].double()
    want = h * (h.square().mean(1, keepdim=True) + 1e-5).rsqrt()
    assert_within(y[:, :n], want, want.abs() * (U16 + 2 * V))


@pytest.mark.parametrize("rows,n,fmt", [(4300001, 8, 0), (4200001, 32, 2)])
def test_more_rows_than_one_dimension_of_blocks(rows, n, fmt):
    o = forward(rng(6), rows, n, BF16, None, F32, fmt)
    assert_within(o["y"], o["want_v"], o["want_v"].abs() * (U16 + 2 * V), "y")
    if fmt:
        e = scale_bytes_of(o["scales"], rows, 1).double()[:, 0] - 127
        assert_within(torch.ldexp(o["codes"][:rows].view(torch.float8_e4m3fn).double(), e[:, None]), o["want_v"], o["want_v"].abs() * 2.0 ** -4 * 1.01 + torch.ldexp(torch.ones_like(e), e - 10)[:, None] + o["want_v"].abs().amax(1, keepdim=True) * 0.125 * (o["want_v"].abs() > torch.ldexp(torch.ones_like(e), e)[:, None] * 448))


def backward(g, rows, n, h_dtype, w_dtype, dh=True, dx16=False, want_dw=True, extra=0):
    dy, h = matrix(g, rows, n, BF16, 0.01, extra), matrix(g, rows, n, h_dtype, 2.0, extra)
    w = (1 + 0.2 * torch.randn(n, generator=g, device=DEV)).to(w_dtype)
    rstd = (h[:, :n].double().square().mean(1) + 1e-5).rsqrt().float() if rows else torch.empty(1, device=DEV)
    add = matrix(g, rows, n, h_dtype, 0.02, extra) if dh else None
    whole, dx = output(rows, n, h_dtype, extra)
    whole16, d16 = output(rows, n, BF16, extra)
    dw = torch.full((n + 1,), GUARD, device=DEV)
    size = b.quartet_rmsnorm_bwd_workspace_bytes(rows, n)
    ws = torch.full((size + 64,), 0xEE, dtype=torch.uint8, device=DEV)
    ld = dy.shape[1]
    some = lambda t: t if rows else torch.empty(64, device=DEV)      # (torch gives a tensor without elements no address)
    q.check(b.quartet_rmsnorm_bwd(some(dy), ld, some(h), code(h), ld, rows, n, w, code(w), rstd, add if rows else None, ld, some(dx), ld, d16 if dx16 else None, ld,
                                  dw if want_dw else None, ws, size))
    torch.cuda.synchronize()
    assert bool((ws[size:] == 0xEE).all()) and float(dw[n]) == GUARD and guarded(whole, n)
    gd, hd, r = dy[:, :n].double() * w.double(), h[:, :n].double(), rstd[:rows].double()[:, None]
    gh = gd * hd
    want = r * (gd - hd * r * r * gh.mean(1, keepdim=True)) + (0 if add is None else add[:, :n].double())
    # the row's sum: 30 roundings of the magnitudes' sum at most; c = sum / n r r 4 more; the element's own arithmetic 6 of its terms
    bound = 36 * U32 * hd.abs() * r ** 3 * gh.abs().mean(1, keepdim=True) + 6 * U32 * (r * gd.abs() + (0 if add is None else add[:, :n].double().abs())) + want.abs() * HALF[h_dtype]
    terms = dy[:, :n].double() * hd * r
    return dict(dx=dx[:, :n], d16=d16[:, :n], whole16=whole16, dw=dw[:n], want=want, bound=bound, want_dw=terms.sum(0), dw_bound=(rows / 64 + 200) * U32 * terms.abs().sum(0),
                args=(dy, h, w, rstd, add, ld))


@pytest.mark.parametrize("h_dtype,w_dtype,dh", [(BF16, F32, True), (F32, BF16, True), (F32, F32, False), (BF16, BF16, False)])
@pytest.mark.parametrize("rows,n", CASES)
def test_backward(rows, n, h_dtype, w_dtype, dh):
    o = backward(rng(rows * 7 + n), rows, n, h_dtype, w_dtype, dh, dx16=h_dtype == F32, extra=8 * (n % 2))
    assert_within(o["dx"], o["want"], o["bound"], "dx")
    assert_within(o["dw"], o["want_dw"], o["dw_bound"], "dw")
    if h_dtype == F32:
        assert torch.equal(o["d16"], o["dx"].to(BF16)) and guarded(o["whole16"], n)


def test_backward_of_nothing_and_of_parts():
    o = backward(rng(8), 0, 40, F32, F32)
    assert bool((o["dw"] == 0).all())
    whole = backward(rng(9), 50, 1003, F32, F32)
    dy, h, w, rstd, add, ld = whole["args"]
    dx, dw = torch.empty_like(h), torch.empty(1003, device=DEV)
    size = b.quartet_rmsnorm_bwd_workspace_bytes(50, 1003)
    q.check(b.quartet_rmsnorm_bwd(dy, ld, h, 0, ld, 50, 1003, w, 0, rstd, add, ld, dx, ld, None, 0, None, None, 0))
    assert torch.equal(dx[:, :1003], whole["dx"])
    q.check(b.quartet_rmsnorm_bwd(dy, ld, h, 0, ld, 50, 1003, w, 0, rstd, None, 0, None, 0, None, 0, dw, torch.empty(size, dtype=torch.uint8, device=DEV), size))
    assert torch.equal(dw, whole["dw"])
    for target in (add.clone(), h.clone()):                       # in place
        use_add = torch.equal(target[:, :1003], add[:, :1003])
        q.check(b.quartet_rmsnorm_bwd(dy, ld, h if use_add else target, 0, ld, 50, 1003, w, 0, rstd, target if use_add else add, ld, target, ld, None, 0, None, None, 0))
        assert torch.equal(target[:, :1003], whole["dx"])


def test_gradients_against_differences():
    # (f(h + d e) - f(h - d e)) / 2 d of the plain forward pass in 64 bits, along random directions
    g = rng(10)
    rows, n = 6, 200
    o = backward(g, rows, n, F32, F32, dh=False)
    dy, h, w, *_ = o["args"]
    f = lambda hh, ww: float((hh * (hh.square().mean(1, keepdim=True) + 1e-5).rsqrt() * ww * dy[:, :n].double()).sum())
    hd, wd = h[:, :n].double(), w.double()
    for _ in range(5):
        eh, ew = torch.randn((rows, n), generator=g, device=DEV).double(), torch.randn(n, generator=g, device=DEV).double()
        d = 1e-5
        assert float((o["dx"].double() * eh).sum()) == pytest.approx((f(hd + d * eh, wd) - f(hd - d * eh, wd)) / (2 * d), rel=1e-4, abs=1e-6)
        assert float((o["dw"].double() * ew).sum()) == pytest.approx((f(hd, wd + d * ew) - f(hd, wd - d * ew)) / (2 * d), rel=1e-4, abs=1e-6)


def test_same_bits_every_time():
    first = backward(rng(11), 3000, 1376, BF16, F32)
    again = backward(rng(11), 3000, 1376, BF16, F32)
    assert torch.equal(first["dw"], again["dw"]) and torch.equal(first["dx"], again["dx"])
