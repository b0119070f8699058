"""The norm and its gradient in each way of sharing a row out: widths and numbers of rows that lie between those of the other tests."""
import numpy as np
import pytest
import torch

import paper_2409_12517_amd as ssg
import test_gpu_norm as tn
from gpu_util import DEV, f32
from oracle import norm

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32

# runs of eight columns: 513 to 768, 769 to 1024, 1025 to 1536 and 1537 to 2048, first and last of a range and between
WIDTHS = [(5, 4112), (5, 5120), (18, 6144), (3, 7168), (3, 12288), (3, 12304), (3, 14336), (2, 16384)]


@pytest.mark.parametrize("T,d", WIDTHS)
@pytest.mark.parametrize("x_dtype,r_dtype,w_dtype,form,offset,gap", [
    (BF, None, BF, ssg.SSG_NORM_BF16, 0.0, 0), (F, BF, BF, ssg.SSG_NORM_F32, 0.0, 0), (BF, F, F, ssg.SSG_NORM_F32, 1.0, 8), (F, F, F, ssg.SSG_NORM_BF16, 0.0, 4)])
def test_rows(T, d, x_dtype, r_dtype, w_dtype, form, offset, gap):
    tn.test_forward(T, d, x_dtype, r_dtype, w_dtype, form, offset, gap)


@pytest.mark.parametrize("T,d", WIDTHS)
def test_e4m3_rows(T, d):
    tn.test_e4m3_rows(T, d)


# more than 512 rows: four to a block of 1024 threads
@pytest.mark.parametrize("T,d", WIDTHS + [(530, 2736), (513, 2064), (600, 4096), (512, 4096)])
@pytest.mark.parametrize("x_dtype,r_dtype", [(BF, None), (BF, F), (F, BF), (F, F)])
def test_quantized_rows(T, d, x_dtype, r_dtype):
    tn.test_i8_rows(T, d, x_dtype, r_dtype)
    tn.test_mx4_rows(T, d, x_dtype, r_dtype, ssg.SSG_MX_CEIL)


@pytest.mark.parametrize("T,d", WIDTHS + [(600, 5120), (530, 6144), (300, 7168), (270, 12304), (300, 14336), (600, 8192)])
@pytest.mark.parametrize("dy_dtype,x_dtype,r_dtype,w_dtype,offset,gap", [
    (BF, BF, None, BF, 0.0, 0), (F, F, None, F, 1.0, 8), (BF, BF, F, BF, 1.0, 8), (F, F, BF, BF, 0.0, 0)])
def test_backward(T, d, dy_dtype, x_dtype, r_dtype, w_dtype, offset, gap):
    tn.test_backward(T, d, dy_dtype, x_dtype, r_dtype, w_dtype, offset, gap)


@pytest.mark.parametrize("T,d", [(5, 80), (70, 528), (600, 4096), (3, 5120)])
@pytest.mark.parametrize("x_dtype,r_dtype", [(BF, BF), (BF, F), (F, BF)])
def test_last_layers_residual(T, d, x_dtype, r_dtype):
    """A residual that nothing behind the norm reads: no gradient comes down it."""
    s, dy = tn.rows(T, d, r_dtype, 1), tn.rows(T, d, BF, 2)
    w, g = tn.weights(d, BF)
    rstd = torch.from_numpy(norm.forward(f32(s), g, tn.EPS)[1].astype(np.float32))
    desc = ssg.make_rmsnorm_desc(T, d, tn.EPS, x_dtype=tn.SSG[x_dtype], residual=1, r_dtype=tn.SSG[r_dtype])
    dx, dr, dw = torch.empty(T, d, dtype=x_dtype, device=DEV), torch.empty(T, d, dtype=r_dtype, device=DEV), torch.empty(d, device=DEV)
    work = torch.empty(ssg.ssg_rmsnorm_bwd_workspace_bytes(desc), dtype=torch.uint8, device=DEV)
    ssg.ssg_rmsnorm_bwd(desc, dy.to(DEV), ssg.SSG_BF16, d, s.to(DEV), rstd.to(DEV), w.to(DEV), None, dx, dr, dw, work)
    want, want_dw = norm.backward(f32(dy), f32(s), rstd.numpy(), g)
    off, off_dw = tn.backward_bounds(f32(dy), f32(s), rstd.numpy(), g)
    for out, t in ((dx, x_dtype), (dr, r_dtype)):
        assert (np.abs(f32(out) - want) <= off + tn.STEP[t] * (np.abs(want) + off)).all()
    assert (np.abs(f32(dw) - want_dw) <= off_dw).all()


def test_rows_beyond_4_gib():
    """Rows that repeat after 4096, from the first to the last, against the formula; dw over all of them.  The 512 blocks add up at most 2049 rows each, whose terms are
    off by two half-steps, the second launch 16 of their sums in each of 32 shares, then those: 2049 + 2 + 16 + 32 half-steps of the sum of magnitudes."""
    T, d, period, u = (1 << 20) + 16, 4112, 1 << 12, 2.0 ** -24
    base, dy_base = (tn.rows(period, d, BF, seed) for seed in (1, 2))
    w, g = tn.weights(d, BF)
    x, dy = (torch.empty(T, d, dtype=BF, device=DEV) for _ in range(2))
    for big, small in ((x, base.to(DEV)), (dy, dy_base.to(DEV))):
        for i in range(0, T, period):
            big[i:i + period] = small[:min(period, T - i)]
    desc = ssg.make_rmsnorm_desc(T, d, tn.EPS)
    y, rstd = torch.empty_like(x), torch.empty(T, device=DEV)
    ssg.ssg_rmsnorm_fwd(desc, x, None, w.to(DEV), None, y, None, None, rstd)
    for out in (y, rstd):
        assert all(torch.equal(out[i:i + period], out[:min(period, T - i)]) for i in range(period, T, period))
    want, want_rstd = norm.forward(f32(base), g, tn.EPS)
    first = rstd[:period].cpu().numpy()
    assert (np.abs(first - want_rstd) <= tn.RSTD * want_rstd).all()
    assert (np.abs(f32(y[:period]) - want) <= (tn.Y + tn.STEP[BF] * (1 + tn.Y)) * np.abs(want)).all()
    dw, work = torch.empty(d, device=DEV), torch.empty(ssg.ssg_rmsnorm_bwd_workspace_bytes(desc), dtype=torch.uint8, device=DEV)
    ssg.ssg_rmsnorm_bwd(desc, dy, ssg.SSG_BF16, d, x, rstd, w.to(DEV), None, y, None, dw, work)          # (y's rows are free: dx)
    assert all(torch.equal(y[i:i + period], y[:min(period, T - i)]) for i in range(period, T, period))
    want, _ = norm.backward(f32(dy_base), f32(base), first, g)
    off, _ = tn.backward_bounds(f32(dy_base), f32(base), first, g)
    assert (np.abs(f32(y[:period]) - want) <= off + tn.STEP[BF] * (np.abs(want) + off)).all()
    term = f32(dy_base).astype(np.float64) * f32(base) * first.astype(np.float64)[:, None]
    times = T // period
    total, size = (times * t.sum(0) + t[:T - times * period].sum(0) for t in (term, np.abs(term)))
    assert (np.abs(f32(dw) - total) <= (2049 + 2 + 16 + 32) * u * size).all()
