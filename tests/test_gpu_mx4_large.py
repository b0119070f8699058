"""Operands, results and rows beyond 4 GiB: what the end holds is what the same rows hold at the start."""
import pytest
import torch

import paper_2409_12517_amd as ssg
from gpu_util import DEV

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def repeated(rows, cols, period, seed):
    """[rows, cols] bf16 whose rows repeat after `period`."""
    base = torch.randn(period, cols, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(BF)
    x = torch.empty(rows, cols, dtype=BF, device=DEV)
    for i in range(0, rows, period):
        x[i:i + period] = base[:min(period, rows - i)]
    return x, base


def test_rows_and_products():
    """2^20 + 48 rows of 8208: codes beyond 4 GiB."""
    rows, K, N, period = (1 << 20) + 48, 8208, 48, 1 << 14
    x, base = repeated(rows, K, period, 1)
    q = torch.empty(ssg.ssg_mx4_bytes(rows, K), dtype=torch.uint8, device=DEV)
    ssg.ssg_mx4_quantize(x, ssg.SSG_BF16, rows, K, K, 0, 0, q)
    small = torch.empty(ssg.ssg_mx4_bytes(period, K), dtype=torch.uint8, device=DEV)
    ssg.ssg_mx4_quantize(base, ssg.SSG_BF16, period, K, K, 0, 0, small)
    wide = -(-K // 256) * 256
    at = (rows - 48) * wide // 2
    assert at > 1 << 32 and torch.equal(q[at:at + 48 * wide // 2], small[:48 * wide // 2])
    w = torch.randn(N, K, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV).to(BF)
    qw = torch.empty(ssg.ssg_mx4_bytes(N, K), dtype=torch.uint8, device=DEV)
    ssg.ssg_mx4_quantize(w, ssg.SSG_BF16, N, K, K, 0, 0, qw)
    y = torch.empty(rows, N, device=DEV)
    ssg.ssg_mx4_gemm(q, rows, qw, N, K, y, ssg.SSG_F32, N)
    assert torch.equal(y[rows - 48:], y[:48]) and torch.equal(y[rows - 48 - period:rows - period], y[:48])
    ssg.ssg_mx4_dequantize(q, rows, K, x, ssg.SSG_BF16, K)
    assert torch.equal(x[rows - 48:], x[:48])


def test_columns():
    """The transpose of 2^20 + 256 tokens of 8208 columns."""
    K, rows, period = (1 << 20) + 256, 8208, 1 << 14
    x, base = repeated(K, rows, period, 3)
    q = torch.empty(ssg.ssg_mx4_bytes(rows, K), dtype=torch.uint8, device=DEV)
    ssg.ssg_mx4_quantize(x, ssg.SSG_BF16, rows, K, rows, 1, 0, q)
    del x
    small = torch.empty(ssg.ssg_mx4_bytes(rows, 256), dtype=torch.uint8, device=DEV)
    ssg.ssg_mx4_quantize(base, ssg.SSG_BF16, rows, 256, rows, 1, 0, small)       # the first 256 tokens
    blocks = K // 128                                        # of a row of blocks; the last 16 columns, their last two blocks
    end = (rows // 16 - 1) * blocks * 1024 + (blocks - 2) * 1024
    mine = (rows // 16 - 1) * 2048
    assert end > 1 << 32 and torch.equal(q[end:end + 2048], small[mine:mine + 2048])


def test_results():
    """A result of 2^20 + 16 rows of 4112 in bf16 and its rows' norm and gradient, each beyond 4 GiB."""
    M, N, K, period = (1 << 20) + 16, 4112, 48, 1 << 12
    x, _ = repeated(M, K, period, 4)
    q, qw = (torch.empty(ssg.ssg_mx4_bytes(r, K), dtype=torch.uint8, device=DEV) for r in (M, N))
    ssg.ssg_mx4_quantize(x, ssg.SSG_BF16, M, K, K, 0, 0, q)
    w = torch.randn(N, K, generator=torch.Generator(device=DEV).manual_seed(5), device=DEV).to(BF)
    ssg.ssg_mx4_quantize(w, ssg.SSG_BF16, N, K, K, 0, 0, qw)
    y = torch.empty(M, N, dtype=BF, device=DEV)
    ssg.ssg_mx4_gemm(q, M, qw, N, K, y, ssg.SSG_BF16, N)
    assert y.numel() * 2 > 1 << 33 and torch.equal(y[M - 16:], y[:16])
    desc = ssg.make_rmsnorm_desc(M, N, 1e-5)
    h, rstd, g = torch.empty_like(y), torch.empty(M, device=DEV), torch.ones(N, dtype=BF, device=DEV)
    ssg.ssg_rmsnorm_fwd(desc, y, None, g, None, h, None, None, rstd)
    assert torch.equal(h[M - 16:], h[:16]) and torch.equal(rstd[M - 16:], rstd[:16])
    dx, dw = torch.empty_like(y), torch.empty(N, device=DEV)
    work = torch.empty(ssg.ssg_rmsnorm_bwd_workspace_bytes(desc), dtype=torch.uint8, device=DEV)
    ssg.ssg_rmsnorm_bwd(desc, h, ssg.SSG_BF16, N, y, rstd, g, None, dx, None, dw, work)
    assert torch.equal(dx[M - 16:], dx[:16])
    for form, size in ((ssg.SSG_NORM_MX4, ssg.ssg_mx4_bytes), (ssg.SSG_NORM_I8, ssg.ssg_i8_bytes)):
        out = torch.empty(size(M, N), dtype=torch.uint8, device=DEV)
        ssg.ssg_rmsnorm_fwd(ssg.make_rmsnorm_desc(M, N, 1e-5, y_format=form), y, None, g, None, out, None, None, None)
        per = (-(-N // 256) * 256 // 2 if form == ssg.SSG_NORM_MX4 else -(-N // 128) * 128) * 16
        at = (M // 16 - 1) * per
        assert torch.equal(out[at:at + per], out[:per])
        del out
