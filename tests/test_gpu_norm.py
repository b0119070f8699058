"""Root-mean-square norm on the GPU against the formula in 64 bits, its quantized forms bit for bit, and its gradient."""
import numpy as np
import pytest
import torch

import paper_2409_12517_amd as ssg
from gpu_util import DEV, f32, u8
from oracle import fp8, i8, mx4, norm

pytestmark = pytest.mark.gpu
SSG = {torch.bfloat16: ssg.SSG_BF16, torch.float32: ssg.SSG_F32}
BF, F = torch.bfloat16, torch.float32
EPS = 1e-5
# A row's squares: a thread adds at most 32 of its own, then come six steps over the lanes and at most 16 over the waves; every addition is off by at
# most 2^-24 of a partial sum.  The square root halves that; division by d, eps's addition, the root and the reciprocal add 4 roundings at most.
RSTD = (54 / 2 + 4) * 2.0 ** -24
Y = RSTD + 2 * 2.0 ** -24                                    # two products more
STEP = {BF: 2.0 ** -8, F: 2.0 ** -24}

SHAPES = [(1, 16), (3, 64), (70, 64), (5, 80), (33, 128), (130, 128), (9, 256), (7, 512), (6, 528), (3, 1376), (2, 2048), (5, 2736), (1, 4096), (18, 4096), (2, 8192), (3, 11008), (2, 32768)]


def rows(T, d, dtype, seed, gap=0):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(T, d, generator=gen) * torch.exp(torch.randn(T, 1, generator=gen))
    x[:, 3] *= 16
    out = torch.full((T, d + gap), 9.0, dtype=dtype)
    out[:, :d] = x.to(dtype)
    return out


def weights(d, dtype, offset=0.0):
    w = (1 - offset + 0.2 * torch.randn(d, generator=torch.Generator().manual_seed(d))).to(dtype)
    g = np.float32(offset) + f32(w)                          # one binary32 addition
    return w, g.astype(np.float32)


def forward(T, d, x_dtype=BF, r_dtype=None, w_dtype=BF, form=ssg.SSG_NORM_F32, offset=0.0, rule=0, gap=0, scale=None, x=None):
    x = rows(T, d, x_dtype, T + d, gap) if x is None else x
    r = rows(T, d, r_dtype, T + d + 1) if r_dtype else None
    w, g = weights(d, w_dtype, offset)
    desc = ssg.make_rmsnorm_desc(T, d, EPS, x_dtype=SSG[x_dtype], residual=int(r is not None), r_dtype=SSG[r_dtype or BF], w_dtype=SSG[w_dtype], w_offset=offset,
                                 y_format=form, ldx=d + gap, rule=rule)
    kept = torch.empty_like(r, device=DEV) if r is not None else None
    if form == ssg.SSG_NORM_I8:
        y = torch.full((ssg.ssg_i8_bytes(T, d),), 0xA5, dtype=torch.uint8, device=DEV)
    elif form == ssg.SSG_NORM_MX4:
        y = torch.full((ssg.ssg_mx4_bytes(T, d),), 0xA5, dtype=torch.uint8, device=DEV)
    else:
        y = torch.empty(T, d, dtype={ssg.SSG_NORM_BF16: BF, ssg.SSG_NORM_F32: F, ssg.SSG_NORM_E4M3: torch.uint8}[form], device=DEV)
    rstd, amax = torch.empty(T, device=DEV), torch.empty(T, device=DEV) if scale is not None else None
    ssg.ssg_rmsnorm_fwd(desc, x.to(DEV), None if r is None else r.to(DEV), w.to(DEV), kept, y, None if scale is None else torch.tensor([scale], device=DEV), amax, rstd)
    s = f32(x[:, :d])
    if r is not None:
        want = (s + f32(r)).astype(np.float32)
        s = f32(torch.from_numpy(want).to(r_dtype))
        assert np.array_equal(f32(kept), s), "the residual"
    return y, s, g, rstd.cpu().numpy(), amax


@pytest.mark.parametrize("T,d", SHAPES)
@pytest.mark.parametrize("x_dtype,r_dtype,w_dtype,form,offset,gap", [
    (BF, None, BF, ssg.SSG_NORM_BF16, 0.0, 0), (F, None, F, ssg.SSG_NORM_F32, 1.0, 16), (BF, BF, F, ssg.SSG_NORM_F32, 0.0, 8), (BF, F, BF, ssg.SSG_NORM_BF16, 1.0, 0),
    (F, BF, BF, ssg.SSG_NORM_F32, 0.0, 0), (F, F, F, ssg.SSG_NORM_BF16, 0.0, 4)])
def test_forward(T, d, x_dtype, r_dtype, w_dtype, form, offset, gap):
    y, s, g, rstd, _ = forward(T, d, x_dtype, r_dtype, w_dtype, form, offset, gap=gap)
    want, want_rstd = norm.forward(s, g, EPS)
    assert (np.abs(rstd - want_rstd) <= RSTD * want_rstd).all()
    step = STEP[BF] if form == ssg.SSG_NORM_BF16 else 0.0
    assert (np.abs(f32(y) - want) <= (Y + step * (1 + Y)) * np.abs(want)).all()


@pytest.mark.parametrize("T,d", SHAPES)
@pytest.mark.parametrize("x_dtype,r_dtype", [(BF, None), (BF, F), (F, BF)])
def test_i8_rows(T, d, x_dtype, r_dtype):
    q, s, g, rstd, _ = forward(T, d, x_dtype, r_dtype, form=ssg.SSG_NORM_I8)
    codes, scales = i8.quantize(norm.quantized_rows(s, rstd, g))
    up, wide = -(-T // 16) * 16, -(-d // 128) * 128
    raw = u8(q)
    at = -(-up * wide // 256) * 256
    assert np.array_equal(raw[:up * wide], i8.layout(codes))
    got = raw[at:at + 4 * up].view(np.float32)
    assert np.array_equal(got[:T], scales) and not got[T:].any()


@pytest.mark.parametrize("rule", [ssg.SSG_MX_FLOOR, ssg.SSG_MX_CEIL])
@pytest.mark.parametrize("T,d", SHAPES)
@pytest.mark.parametrize("x_dtype,r_dtype", [(BF, None), (BF, F), (F, BF)])
def test_mx4_rows(T, d, x_dtype, r_dtype, rule):
    q, s, g, rstd, _ = forward(T, d, x_dtype, r_dtype, form=ssg.SSG_NORM_MX4, rule=rule)
    code_bytes, scale_bytes = mx4.layout(*mx4.quantize(norm.quantized_rows(s, rstd, g), rule == ssg.SSG_MX_CEIL))
    raw = u8(q)
    assert np.array_equal(raw[:code_bytes.size], code_bytes)
    assert np.array_equal(raw[code_bytes.size:code_bytes.size + scale_bytes.size], scale_bytes)


@pytest.mark.parametrize("T,d", SHAPES)
def test_e4m3_rows(T, d):
    for scale in (40.0, 4000.0):                             # the larger one saturates
        y, s, g, rstd, amax = forward(T, d, BF, F, form=ssg.SSG_NORM_E4M3, scale=scale)
        v = norm.quantized_rows(s, rstd, g)
        assert np.array_equal(u8(y), fp8.satcast((v * np.float32(scale)).astype(np.float32), fp8.by_name("e4m3")))
        assert np.array_equal(amax.cpu().numpy(), np.abs(v).max(-1))


@pytest.mark.parametrize("d", [64, 528, 4096, 11008])
def test_rows_out_of_the_range_of_their_squares(d):
    x = rows(4, d, F, d)
    x[0] *= 1e30
    x[1] *= 1e-30
    x[2] = 0
    x[3] = 3e38
    for form in (ssg.SSG_NORM_F32, ssg.SSG_NORM_MX4):
        y, s, g, rstd, _ = forward(4, d, F, form=form, x=x)
        want, want_rstd = norm.forward(s, g, EPS)
        # (a reciprocal root below 2^-126 is a subnormal number: half of 2^-149 beside the rest)
        assert (np.abs(rstd - want_rstd) <= RSTD * want_rstd + 2.0 ** -150).all()
        if form == ssg.SSG_NORM_F32:
            assert (np.abs(f32(y) - want) <= (Y + 2.0 ** -150 / want_rstd[:, None]) * np.abs(want) + 2.0 ** -149).all()


@pytest.mark.parametrize("d", [64, 4096])
def test_rows_with_no_number(d):
    """One row's NaN or infinity is its own."""
    x = rows(40, d, BF, d)
    x[7, 5], x[20, 40] = torch.nan, torch.inf
    y, s, g, rstd, _ = forward(40, d, BF, form=ssg.SSG_NORM_F32, x=x)
    got = f32(y)
    assert np.isnan(got[7]).all() and np.isnan(got[20, 40]) and (np.delete(got[20], 40) == 0).all() and rstd[20] == 0
    keep = np.delete(np.arange(40), [7, 20])
    assert np.isfinite(got[keep]).all()
    q, *_ = forward(40, d, BF, form=ssg.SSG_NORM_MX4, x=x)
    v = torch.empty(40, d, device=DEV)
    ssg.ssg_mx4_dequantize(q, 40, d, v, ssg.SSG_F32, d)
    v = f32(v)
    assert np.isnan(v[7]).all() and np.isnan(v[20, 32:64]).all() and np.isfinite(v[keep]).all() and not v[20, :32].any()
    q, *_ = forward(40, d, BF, form=ssg.SSG_NORM_I8, x=x)
    codes, scales = torch.empty(40, d, dtype=torch.int8, device=DEV), torch.empty(40, device=DEV)
    ssg.ssg_i8_unpack(q, 40, d, codes, scales)
    assert torch.isnan(scales).cpu().nonzero().flatten().tolist() == [7, 20]


def test_in_place_and_without_weights():
    T, d = 33, 528
    x, r = rows(T, d, BF, 1).to(DEV), rows(T, d, F, 2).to(DEV)
    desc = ssg.make_rmsnorm_desc(T, d, EPS, residual=1, r_dtype=ssg.SSG_F32, y_format=ssg.SSG_NORM_F32, ldy=d + 4)
    apart, y, y2 = torch.empty_like(r), torch.full((T, d + 4), 5.0, device=DEV), torch.full((T, d + 4), 5.0, device=DEV)
    ssg.ssg_rmsnorm_fwd(desc, x, r, None, apart, y, None, None, None)
    ssg.ssg_rmsnorm_fwd(desc, x, r, None, r, y2, None, None, None)
    assert torch.equal(apart, r) and torch.equal(y, y2) and (y[:, d:] == 5).all()
    want, _ = norm.forward(f32(apart), np.ones(d), EPS)
    assert (np.abs(f32(y[:, :d]) - want) <= Y * np.abs(want)).all()


def backward_bounds(dy, s, rstd, g):
    """How far ds and dw may be off: n and a = dy g are products rounded once each; mean(a n) is a sum of d terms of which a thread adds at most 32, then
    6 + 16, each term off by 3 half-steps, with a division: 58 half-steps of the sum of magnitudes; a - n mean and the product with rstd, fused with ds's
    addition, 2 more of what they join.  dw: T terms off by one half-step each, added in some order."""
    u = 2.0 ** -24
    n = s.astype(np.float64) * rstd.astype(np.float64)[:, None]
    a = dy.astype(np.float64) * g
    mean = np.abs(a * n).mean(-1, keepdims=True)
    ds = rstd.astype(np.float64)[:, None] * (3 * np.abs(a) + 64 * np.abs(n) * mean) * u
    return ds, (dy.shape[0] + 2) * np.abs(dy.astype(np.float64) * n).sum(0) * u


@pytest.mark.parametrize("T,d", SHAPES + [(1500, 64), (3000, 128), (1100, 512), (1030, 2736), (600, 4096), (530, 11008)])
@pytest.mark.parametrize("dy_dtype,x_dtype,r_dtype,w_dtype,offset,gap", [
    (BF, BF, None, BF, 0.0, 0), (F, F, None, F, 1.0, 8), (BF, BF, BF, F, 0.0, 0), (BF, BF, F, BF, 1.0, 8), (F, F, BF, BF, 0.0, 0), (F, BF, F, F, 0.0, 0)])
def test_backward(T, d, dy_dtype, x_dtype, r_dtype, w_dtype, offset, gap):
    s_dtype = r_dtype or x_dtype
    s, dy = rows(T, d, s_dtype, 1), rows(T, d, dy_dtype, 2, gap)
    ds_in = rows(T, d, s_dtype, 3) if r_dtype else None
    w, g = weights(d, w_dtype, offset)
    rstd = torch.from_numpy(norm.forward(f32(s), g, EPS)[1].astype(np.float32))
    desc = ssg.make_rmsnorm_desc(T, d, EPS, x_dtype=SSG[x_dtype], residual=int(bool(r_dtype)), r_dtype=SSG[r_dtype or BF], w_dtype=SSG[w_dtype], w_offset=offset)
    dx, dw = torch.empty(T, d, dtype=x_dtype, device=DEV), torch.empty(d, device=DEV)
    dr = torch.empty(T, d, dtype=r_dtype, device=DEV) if r_dtype else None
    work = torch.full((ssg.ssg_rmsnorm_bwd_workspace_bytes(desc),), 0xA5, dtype=torch.uint8, device=DEV)
    args = (desc, dy.to(DEV), SSG[dy_dtype], d + gap, s.to(DEV), rstd.to(DEV), w.to(DEV))
    ds_dev = ds_in.to(DEV) if r_dtype else None
    ssg.ssg_rmsnorm_bwd(*args, ds_dev, dx, dr, dw, work)
    want, want_dw = norm.backward(f32(dy[:, :d]), f32(s), rstd.numpy(), g)
    off, off_dw = backward_bounds(f32(dy[:, :d]), f32(s), rstd.numpy(), g)
    if r_dtype:
        want = want + f32(ds_in)
    for out, t in ((dx, x_dtype), (dr, r_dtype)):
        if out is not None:
            assert (np.abs(f32(out) - want) <= off + STEP[t] * (np.abs(want) + off)).all()
    assert (np.abs(f32(dw) - want_dw) <= off_dw).all()
    # each output alone, the residual's gradient in place: the same bits
    dw2, dx2 = torch.empty_like(dw), torch.empty_like(dx)
    ssg.ssg_rmsnorm_bwd(*args, ds_dev, None, None, dw2, work)
    ssg.ssg_rmsnorm_bwd(*args, ds_dev, dx2, None, None, None)
    assert torch.equal(dw, dw2) and torch.equal(dx, dx2)
    if r_dtype:
        ssg.ssg_rmsnorm_bwd(*args, ds_dev, None, ds_dev, None, None)
        assert torch.equal(ds_dev, dr)


def test_backward_of_no_rows():
    desc = ssg.make_rmsnorm_desc(0, 80, EPS)
    dw = torch.full((80,), 3.0, device=DEV)
    ssg.ssg_rmsnorm_bwd(desc, None, ssg.SSG_BF16, 80, None, None, torch.ones(80, dtype=BF, device=DEV), None, None, None, dw,
                        torch.empty(ssg.ssg_rmsnorm_bwd_workspace_bytes(desc), dtype=torch.uint8, device=DEV))
    assert not dw.any()


@pytest.mark.parametrize("T,d", [(1, 64), (37, 80), (19, 528), (5, 4096), (3, 11008)])
@pytest.mark.parametrize("form", [ssg.SSG_NORM_BF16, ssg.SSG_NORM_F32, ssg.SSG_NORM_E4M3])
def test_strides(T, d, form):
    """Rows inside wider matrices: the same results, and what lies between and behind them stays."""
    dtype = {ssg.SSG_NORM_BF16: BF, ssg.SSG_NORM_F32: F, ssg.SSG_NORM_E4M3: torch.uint8}[form]
    x, r, w = rows(T, d, BF, 1), rows(T, d, F, 2), weights(d, BF)[0].to(DEV)
    scale = torch.tensor([30.0], device=DEV) if form == ssg.SSG_NORM_E4M3 else None

    def run(gx, gr, gy):
        xs, rs = torch.full((T + 1, d + gx), 7.0, dtype=BF, device=DEV), torch.full((T + 1, d + gr), 7.0, device=DEV)
        xs[:T, :d], rs[:T, :d] = x.to(DEV), r.to(DEV)
        kept, y, rstd = torch.full_like(rs, 5.0), torch.full((T + 1, d + gy), 5, dtype=dtype, device=DEV), torch.full((T + 1,), 5.0, device=DEV)
        desc = ssg.make_rmsnorm_desc(T, d, EPS, residual=1, r_dtype=ssg.SSG_F32, y_format=form, ldx=d + gx, ldr=d + gr, ldy=d + gy)
        ssg.ssg_rmsnorm_fwd(desc, xs, rs, w, kept, y, scale, None, rstd)
        for t in (kept, y):
            assert bool((t[T] == 5).all()) and bool((t[:, d:] == 5).all())
        assert float(rstd[T]) == 5
        # the gradient with the same strides
        dy, ds = rows(T, d, BF, 3, 8).to(DEV), torch.full_like(rs, 7.0)
        ds[:T, :d] = rows(T, d, F, 4).to(DEV)
        dx, dr, dw = torch.full_like(xs, 5.0), torch.full_like(rs, 5.0), torch.empty(d, device=DEV)
        work = torch.empty(ssg.ssg_rmsnorm_bwd_workspace_bytes(desc), dtype=torch.uint8, device=DEV)
        ssg.ssg_rmsnorm_bwd(desc, dy, ssg.SSG_BF16, d + 8, kept, rstd, w, ds, dx, dr, dw, work)
        for t in (dx, dr):
            assert bool((t[T] == 5).all()) and bool((t[:, d:] == 5).all())
        return [kept[:T, :d], y[:T, :d], rstd[:T], dx[:T, :d], dr[:T, :d], dw]

    assert all(torch.equal(a, b) for a, b in zip(run(0, 0, 0), run(8, 4, 16)))


def test_gradient_without_weights():
    T, d = 40, 528
    s, dy = rows(T, d, F, 1), rows(T, d, F, 2)
    rstd = torch.from_numpy(norm.forward(f32(s), np.ones(d), EPS)[1].astype(np.float32))
    dx = torch.empty(T, d, device=DEV)
    ssg.ssg_rmsnorm_bwd(ssg.make_rmsnorm_desc(T, d, EPS, x_dtype=ssg.SSG_F32), dy.to(DEV), ssg.SSG_F32, d, s.to(DEV), rstd.to(DEV), None, None, dx, None, None, None)
    want, _ = norm.backward(f32(dy), f32(s), rstd.numpy(), np.ones(d))
    off, _ = backward_bounds(f32(dy), f32(s), rstd.numpy(), np.ones(d, np.float32))
    assert (np.abs(f32(dx) - want) <= off + STEP[F] * (np.abs(want) + off)).all()


@pytest.mark.parametrize("d", [64, 528, 4096])
def test_gradient_against_differences(d):
    """sum(y dy) along a direction v: a central difference is off by h^2 / 6 of the third derivative between its ends, and by the forward
    pass's rounding over h.  With m = mean(s^2) + eps, r = m^-1/2 and V^2 = mean(v^2): the first derivative of m is at most 2 V / r (Cauchy and
    Schwarz), its second is 2 V^2, so the second of m^-1/2 is at most 4 V^2 r^3, the third at most 24 V^3 r^4, and that of y = g s m^-1/2 at most
    |g| (24 |s| V^3 r^4 + 12 |v| V^2 r^3).  Up to h away r is at most r / (1 - h V r) and |s| grows by h |v|."""
    T, h = 3, 2.0 ** -5
    s, dy, v = rows(T, d, F, 1), rows(T, d, F, 2), torch.randn(T, d, generator=torch.Generator().manual_seed(3))
    w, g = weights(d, F)
    desc = ssg.make_rmsnorm_desc(T, d, EPS, x_dtype=ssg.SSG_F32, w_dtype=ssg.SSG_F32, y_format=ssg.SSG_NORM_F32)

    def total(x):
        y, rstd = torch.empty(T, d, device=DEV), torch.empty(T, device=DEV)
        ssg.ssg_rmsnorm_fwd(desc, x.to(DEV), None, w.to(DEV), None, y, None, None, rstd)
        return (f32(y).astype(np.float64) * f32(dy)).sum(-1), f32(y), rstd

    rstd = total(s)[2]
    ds = torch.empty(T, d, device=DEV)
    ssg.ssg_rmsnorm_bwd(desc, dy.to(DEV), ssg.SSG_F32, d, s.to(DEV), rstd, w.to(DEV), None, ds, None, None, None)
    got = (f32(ds).astype(np.float64) * f32(v)).sum(-1)
    up, y1, _ = total(s + h * v)
    down, y2, _ = total(s - h * v)
    a = np.abs(f32(dy).astype(np.float64))
    r = rstd.cpu().numpy().astype(np.float64)[:, None]
    V = np.sqrt((f32(v).astype(np.float64) ** 2).mean(-1, keepdims=True))
    assert (h * V * r < 0.9).all()
    r = r / (1 - h * V * r)
    third = (np.abs(g) * a * (24 * (np.abs(f32(s)) + h * np.abs(f32(v))) * V ** 3 * r ** 4 + 12 * np.abs(f32(v)) * V ** 2 * r ** 3)).sum(-1)
    rounding = (2.0 ** -24 + Y) * (a * (np.abs(y1) + np.abs(y2))).sum(-1) / (2 * h)
    off, _ = backward_bounds(f32(dy), f32(s), rstd.cpu().numpy(), g)
    assert (np.abs((up - down) / (2 * h) - got) <= h * h / 6 * third + rounding + (off * np.abs(f32(v))).sum(-1)).all()
