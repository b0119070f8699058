"""What the entry points of 4-bit floating point and of the norm refuse: host checks alone, nothing is launched."""
import pytest

import paper_2409_12517_amd as ssg

BIG = 1 << 40


def refused(status, word, call, *args, **more):
    with pytest.raises(ssg.SsgError) as e:
        call(*args, stream=0, **more)
    assert e.value.status == status and word in str(e.value), str(e.value)


def test_sizes():
    assert ssg.ssg_mx4_bytes(0, 16) == 256 and ssg.ssg_mx4_bytes(1, 1) == 16 * 128 + 16 * 8 + 128
    assert ssg.ssg_mx4_bytes(17, 257) == 32 * 256 + 32 * 16
    for rows, K in ((-1, 16), (16, 0), (16, (1 << 24) + 1), ((1 << 26) + 1, 16)):
        assert ssg.ssg_mx4_bytes(rows, K) == 0
    last = 0
    for M in range(0, 300):
        n = ssg.ssg_mx4_linear_workspace_bytes(M, 80)
        assert n >= last and n % 256 == 0
        last = n
    last = 0
    for M in range(0, 600, 7):
        n = ssg.ssg_mx4_linear_bwd_workspace_bytes(M, 48, 80)
        assert n >= last and n % 256 == 0
        last = n
    assert ssg.ssg_mx4_linear_bwd_workspace_bytes(16, 40, 80) == 0 and "N = 40" in ssg.ssg_last_error()


def test_quantize_refusals():
    q = ssg.ssg_mx4_quantize
    refused(ssg.SSG_ERR_SHAPE, "K = 20", q, 4096, ssg.SSG_BF16, 4, 20, 24, 0, 0, 4096, q_bytes=BIG)
    refused(ssg.SSG_ERR_SHAPE, "rows = 20", q, 4096, ssg.SSG_BF16, 20, 7, 24, 1, 0, 4096, q_bytes=BIG)
    refused(ssg.SSG_ERR_SHAPE, "rows of src", q, 4096, ssg.SSG_BF16, 4, 32, 24, 0, 0, 4096, q_bytes=BIG)
    refused(ssg.SSG_ERR_SHAPE, "rows of src", q, 4096, ssg.SSG_BF16, 32, 4, 24, 1, 0, 4096, q_bytes=BIG)
    refused(ssg.SSG_ERR_SHAPE, "rows of src", q, 4096, ssg.SSG_F32, 4, 32, 34, 0, 0, 4096, q_bytes=BIG)
    refused(ssg.SSG_ERR_ARG, "transposed", q, 4096, ssg.SSG_F32, 4, 32, 32, 2, 0, 4096, q_bytes=BIG)
    refused(ssg.SSG_ERR_ARG, "rule", q, 4096, ssg.SSG_F32, 4, 32, 32, 0, 2, 4096, q_bytes=BIG)
    refused(ssg.SSG_ERR_ARG, "data type", q, 4096, 2, 4, 32, 32, 0, 0, 4096, q_bytes=BIG)
    refused(ssg.SSG_ERR_ARG, "src", q, 4104, ssg.SSG_F32, 4, 32, 32, 0, 0, 4096, q_bytes=BIG)
    refused(ssg.SSG_ERR_ARG, "src is NULL", q, None, ssg.SSG_F32, 4, 32, 32, 0, 0, 4096, q_bytes=BIG)
    refused(ssg.SSG_ERR_ARG, "256-byte", q, 4096, ssg.SSG_F32, 4, 32, 32, 0, 0, 4112, q_bytes=BIG)
    refused(ssg.SSG_ERR_WORKSPACE, "q holds", q, 4096, ssg.SSG_F32, 4, 32, 32, 0, 0, 4096, q_bytes=ssg.ssg_mx4_bytes(4, 32) - 1)
    ssg.ssg_mx4_quantize(None, ssg.SSG_F32, 0, 32, 32, 0, 0, None, stream=0)          # no rows: nothing to do
    refused(ssg.SSG_ERR_SHAPE, "rows of dst", ssg.ssg_mx4_dequantize, 4096, 4, 33, 4096, ssg.SSG_BF16, 36, q_bytes=BIG)
    refused(ssg.SSG_ERR_WORKSPACE, "q holds", ssg.ssg_mx4_dequantize, 4096, 4, 33, 4096, ssg.SSG_BF16, 40, q_bytes=16)
    refused(ssg.SSG_ERR_SHAPE, "K = 33", ssg.ssg_mx4_pack, 4096, 4096, 4, 33, 4096, q_bytes=BIG)
    refused(ssg.SSG_ERR_ARG, "codes", ssg.ssg_mx4_pack, 4100, 4096, 4, 32, 4096, q_bytes=BIG)
    refused(ssg.SSG_ERR_ARG, "scales", ssg.ssg_mx4_unpack, 4096, 4, 32, 4096, None, q_bytes=BIG)


def test_product_refusals():
    g, need = ssg.ssg_mx4_gemm, ssg.ssg_mx4_bytes(16, 64)
    refused(ssg.SSG_ERR_SHAPE, "N = 20", g, 4096, 16, 4096, 20, 64, 4096, ssg.SSG_F32, 20, A_bytes=need, B_bytes=BIG)
    refused(ssg.SSG_ERR_SHAPE, "K = 0", g, 4096, 16, 4096, 16, 0, 4096, ssg.SSG_F32, 16, A_bytes=need, B_bytes=BIG)
    refused(ssg.SSG_ERR_WORKSPACE, "A holds", g, 4096, 17, 4096, 16, 64, 4096, ssg.SSG_F32, 16, A_bytes=need, B_bytes=need)
    refused(ssg.SSG_ERR_WORKSPACE, "B holds", g, 4096, 16, 4096, 32, 64, 4096, ssg.SSG_F32, 32, A_bytes=need, B_bytes=need)
    refused(ssg.SSG_ERR_SHAPE, "rows of C", g, 4096, 16, 4096, 16, 64, 4096, ssg.SSG_BF16, 8, A_bytes=need, B_bytes=need)
    refused(ssg.SSG_ERR_SHAPE, "too many", g, 4096, 1 << 26, 4096, 1 << 26, 64, 4096, ssg.SSG_F32, 1 << 26, A_bytes=BIG, B_bytes=BIG)
    refused(ssg.SSG_ERR_ARG, "C is NULL", g, 4096, 16, 4096, 16, 64, None, ssg.SSG_F32, 16, A_bytes=need, B_bytes=need)
    lin = ssg.ssg_mx4_linear
    refused(ssg.SSG_ERR_WORKSPACE, "workspace", lin, 4096, ssg.SSG_BF16, 4, 64, 64, 0, 4096, 16, 4096, ssg.SSG_F32, 16, 4096, W_bytes=need, workspace_bytes=0)
    refused(ssg.SSG_ERR_SHAPE, "K = 72", lin, 4096, ssg.SSG_BF16, 4, 72, 72, 0, 4096, 16, 4096, ssg.SSG_F32, 16, 4096, W_bytes=BIG, workspace_bytes=BIG)
    refused(ssg.SSG_ERR_ARG, "rule", lin, 4096, ssg.SSG_BF16, 4, 64, 64, 3, 4096, 16, 4096, ssg.SSG_F32, 16, 4096, W_bytes=need, workspace_bytes=BIG)
    refused(ssg.SSG_ERR_SHAPE, "rows of y", lin, 4096, ssg.SSG_BF16, 4, 64, 64, 0, 4096, 16, 4096, ssg.SSG_F32, 12, 4096, W_bytes=need, workspace_bytes=BIG)
    for args in ((0, 16, 16), (16, 20, 16), (16, 16, 0)):
        with pytest.raises(ssg.SsgError):
            ssg.ssg_mx4_gemm_plan(*args)


def bwd(dy=4096, lddy=48, x=4096, ldx=64, M=5, N=48, K=64, rule=0, Wt=4096, dx=4096, lddx=64, dW=4096, lddw=64, work=4096, dt=1, Wt_bytes=BIG, workspace_bytes=BIG):
    return (dy, dt, lddy, x, dt, ldx, M, N, K, rule, Wt, dx, dt, lddx, dW, dt, lddw, work), {"Wt_bytes": Wt_bytes, "workspace_bytes": workspace_bytes}


@pytest.mark.parametrize("status,word,change", [
    (ssg.SSG_ERR_SHAPE, "M = -1", dict(M=-1)), (ssg.SSG_ERR_SHAPE, "N = 40", dict(N=40)), (ssg.SSG_ERR_SHAPE, "K = 0", dict(K=0)), (ssg.SSG_ERR_ARG, "rule", dict(rule=2)),
    (ssg.SSG_ERR_SHAPE, "rows of dy", dict(lddy=47)), (ssg.SSG_ERR_SHAPE, "rows of x", dict(ldx=60)), (ssg.SSG_ERR_SHAPE, "rows of dx", dict(lddx=60)),
    (ssg.SSG_ERR_SHAPE, "rows of dW", dict(lddw=60)), (ssg.SSG_ERR_ARG, "both NULL", dict(dx=None, dW=None)), (ssg.SSG_ERR_ARG, "dy", dict(dy=None)),
    (ssg.SSG_ERR_ARG, "x is NULL", dict(x=None)), (ssg.SSG_ERR_ARG, "Wt is NULL", dict(Wt=None)), (ssg.SSG_ERR_WORKSPACE, "Wt holds", dict(Wt_bytes=ssg.ssg_mx4_bytes(64, 48) - 1)),
    (ssg.SSG_ERR_ARG, "data type", dict(dt=2)),
    (ssg.SSG_ERR_WORKSPACE, "workspace holds", dict(workspace_bytes=ssg.ssg_mx4_linear_bwd_workspace_bytes(5, 48, 64) - 1)), (ssg.SSG_ERR_ARG, "workspace", dict(work=None))])
def test_linear_bwd_refusals(status, word, change):
    args, more = bwd(**change)
    refused(status, word, ssg.ssg_mx4_linear_bwd, *args, **more)


def test_nothing_to_compute_is_refused_without_rows_too():
    args, more = bwd(M=0, dx=None, dW=None)
    refused(ssg.SSG_ERR_ARG, "both NULL", ssg.ssg_mx4_linear_bwd, *args, **more)


def test_plan():
    """Host logic only: which kernel a product runs in."""
    def plan(*args):
        p = ssg.ssg_mx4_gemm_plan(*args)
        return p.tile or (p.rows, p.cols)

    assert [plan(M, 4096, 4096) for M in (1, 16, 17, 32, 33, 64, 128, 256)] == [(16, 16)] * 2 + [(32, 16)] * 2 + [(32, 32)] * 2 + [(64, 32), (64, 64)]
    # more workgroups than compute units in any block: by rows
    assert [plan(M, 11008, 4096) for M in (1, 16, 32, 64, 65, 512)] == [(16, 16), (16, 16), (32, 16), (64, 64), 128, 128]
    assert plan(64, 16400, 4096) == (32, 32)
    # few columns: the smallest blocks whose workgroups the chip holds at once
    assert [plan(M, 1040, 2736) for M in (32, 64, 128, 256)] == [(16, 16), (32, 16), (32, 32), (64, 32)]
    # 64 x 64 for long sums only
    assert plan(512, 1376, 2560) == (64, 64) and plan(512, 1376, 2304) == 128
    assert plan(4096, 4096, 11008) == 256 == plan(4096, 11008, 4096) and plan(2048, 4096, 11008) == 128 and plan(8192, 8192, 512) == 128


def fwd(desc, x=4096, residual=None, w=4096, residual_out=None, y=4096, y_scale=None, y_amax=None, rstd=4096, y_bytes=BIG):
    return (desc, x, residual, w, residual_out, y, y_scale, y_amax, rstd), {"y_bytes": y_bytes}


@pytest.mark.parametrize("status,word,change", [
    (ssg.SSG_ERR_SHAPE, "T = -1", dict(T=-1)), (ssg.SSG_ERR_SHAPE, "d = 24", dict(d=24)), (ssg.SSG_ERR_SHAPE, "d = 32784", dict(d=32784)), (ssg.SSG_ERR_ARG, "eps", dict(eps=0.0)),
    (ssg.SSG_ERR_ARG, "eps", dict(eps=float("nan"))), (ssg.SSG_ERR_ARG, "eps", dict(eps=2.0)), (ssg.SSG_ERR_ARG, "data types", dict(x_dtype=2)),
    (ssg.SSG_ERR_ARG, "residual 2", dict(residual=2)), (ssg.SSG_ERR_ARG, "y_format", dict(y_format=5)), (ssg.SSG_ERR_ARG, "rule", dict(rule=2)),
    (ssg.SSG_ERR_ARG, "w_offset", dict(w_offset=float("inf"))), (ssg.SSG_ERR_SHAPE, "rows (0 to 67108864)", dict(T=(1 << 26) + 1, y_format=ssg.SSG_NORM_I8))])
def test_norm_descriptors(status, word, change):
    desc = ssg.make_rmsnorm_desc(**{**dict(T=4, d=64, eps=1e-5), **change})
    args, more = fwd(desc)
    refused(status, word, ssg.ssg_rmsnorm_fwd, *args, **more)
    refused(status, word, ssg.ssg_rmsnorm_bwd, desc, 4096, 0, 64, 4096, 4096, 4096, None, 4096, None, 4096, 4096, workspace_bytes=BIG)
    assert ssg.ssg_rmsnorm_bwd_workspace_bytes(desc) == 0


def test_norm_buffers():
    plain, res = ssg.make_rmsnorm_desc(4, 64, 1e-5), ssg.make_rmsnorm_desc(4, 64, 1e-5, residual=1)

    def no(status, word, desc, **change):
        args, more = fwd(desc, **change)
        refused(status, word, ssg.ssg_rmsnorm_fwd, *args, **more)

    no(ssg.SSG_ERR_ARG, "x is NULL", plain, x=None)
    no(ssg.SSG_ERR_ARG, "w is not", plain, w=4100)
    no(ssg.SSG_ERR_ARG, "rstd is not", plain, rstd=4097)
    no(ssg.SSG_ERR_ARG, "desc.residual is 0", plain, residual=4096)
    no(ssg.SSG_ERR_ARG, "residual is NULL", res, residual_out=4096)
    no(ssg.SSG_ERR_ARG, "residual_out is NULL", res, residual=4096)
    no(ssg.SSG_ERR_ARG, "y is NULL", plain, y=None)
    no(ssg.SSG_ERR_ARG, "y_scale", plain, y_scale=4096)
    no(ssg.SSG_ERR_ARG, "y_scale is NULL", ssg.make_rmsnorm_desc(4, 64, 1e-5, y_format=ssg.SSG_NORM_E4M3))
    for ld, form in ((68, ssg.SSG_NORM_BF16), (66, ssg.SSG_NORM_F32), (72, ssg.SSG_NORM_E4M3), (48, ssg.SSG_NORM_BF16)):
        no(ssg.SSG_ERR_SHAPE, "rows of y", ssg.make_rmsnorm_desc(4, 64, 1e-5, y_format=form, ldy=ld), y_scale=4096 if form == ssg.SSG_NORM_E4M3 else None)
    no(ssg.SSG_ERR_WORKSPACE, "y holds", ssg.make_rmsnorm_desc(4, 64, 1e-5, y_format=ssg.SSG_NORM_I8), y_bytes=ssg.ssg_i8_bytes(4, 64) - 1)
    no(ssg.SSG_ERR_WORKSPACE, "y holds", ssg.make_rmsnorm_desc(4, 64, 1e-5, y_format=ssg.SSG_NORM_MX4), y_bytes=ssg.ssg_mx4_bytes(4, 64) - 1)
    no(ssg.SSG_ERR_ARG, "256-byte", ssg.make_rmsnorm_desc(4, 64, 1e-5, y_format=ssg.SSG_NORM_MX4), y=4112)
    bad = ssg.make_rmsnorm_desc(4, 64, 1e-5)
    bad.reserved[1] = 1
    no(ssg.SSG_ERR_ARG, "reserved", bad)

    def no_bwd(status, word, desc, dy=4096, s=4096, rstd=4096, w=4096, ds=None, dx=4096, dr=None, dw=4096, work=4096, nbytes=BIG, lddy=64):
        refused(status, word, ssg.ssg_rmsnorm_bwd, desc, dy, 0, lddy, s, rstd, w, ds, dx, dr, dw, work, workspace_bytes=nbytes)

    no_bwd(ssg.SSG_ERR_ARG, "dy is NULL", plain, dy=None)
    no_bwd(ssg.SSG_ERR_SHAPE, "rows of dy", plain, lddy=60)
    no_bwd(ssg.SSG_ERR_ARG, "s is NULL", plain, s=None)
    no_bwd(ssg.SSG_ERR_ARG, "rstd is NULL", plain, rstd=None)
    no_bwd(ssg.SSG_ERR_ARG, "desc.residual is 0", plain, ds=4096)
    no_bwd(ssg.SSG_ERR_ARG, "desc.residual is 0", plain, dr=4096)
    no_bwd(ssg.SSG_ERR_ARG, "all NULL", plain, dx=None, dw=None)
    no_bwd(ssg.SSG_ERR_ARG, "w is NULL", plain, w=None)
    no_bwd(ssg.SSG_ERR_ARG, "ds is not", res, ds=4104)
    no_bwd(ssg.SSG_ERR_ARG, "dw is not", plain, dw=4100)
    no_bwd(ssg.SSG_ERR_ARG, "workspace is NULL", plain, work=None)
    no_bwd(ssg.SSG_ERR_WORKSPACE, "workspace holds", plain, nbytes=ssg.ssg_rmsnorm_bwd_workspace_bytes(plain) - 1)
    ssg.ssg_rmsnorm_fwd(ssg.make_rmsnorm_desc(0, 64, 1e-5), None, None, 4096, None, None, None, None, None, stream=0)     # no rows: nothing to do
