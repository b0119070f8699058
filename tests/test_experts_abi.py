"""What the entry points of routing, of 8-bit products and of the mixture refuse: host checks alone, nothing is launched."""
import pytest

import paper_2409_12517_amd as ssg


def refused(status, word, call, *args, **more):
    with pytest.raises(ssg.SsgError) as e:
        call(*args, stream=0, **more)
    assert e.value.status == status and word in str(e.value)


def route_with(desc, logits=4096, bias=None, ids=4096, weights=4096, counts=4096, offsets=4096, place=4096, source=4096, work=4096, nbytes=1 << 30):
    return (desc, logits, bias, ids, weights, counts, offsets, place, source, work), {"workspace_bytes": nbytes}


@pytest.mark.parametrize("status,word,change", [
    (ssg.SSG_ERR_SHAPE, "E = 0", dict(E=0)), (ssg.SSG_ERR_SHAPE, "E = 1025", dict(E=1025)), (ssg.SSG_ERR_SHAPE, "k = 0", dict(k=0)),
    (ssg.SSG_ERR_SHAPE, "k = 33", dict(E=64, k=33)), (ssg.SSG_ERR_SHAPE, "k = 17", dict(k=17)), (ssg.SSG_ERR_SHAPE, "T = -1", dict(T=-1)),
    (ssg.SSG_ERR_SHAPE, "T = ", dict(T=1 << 40)), (ssg.SSG_ERR_SHAPE, "ld = 15", dict(ld=15)), (ssg.SSG_ERR_ARG, "logits_dtype", dict(logits_dtype=2)),
    (ssg.SSG_ERR_ARG, "score", dict(score=2)), (ssg.SSG_ERR_SHAPE, "groups = 3", dict(groups=3)), (ssg.SSG_ERR_SHAPE, "groups = 0", dict(groups=0)),
    (ssg.SSG_ERR_SHAPE, "top_groups", dict(groups=4, top_groups=5)), (ssg.SSG_ERR_SHAPE, "top_groups", dict(groups=8, top_groups=1, k=3)),
    (ssg.SSG_ERR_ARG, "group_top", dict(group_top=3)), (ssg.SSG_ERR_ARG, "renorm", dict(renorm=2)), (ssg.SSG_ERR_ARG, "scale", dict(scale=float("nan"))),
    (ssg.SSG_ERR_ARG, "row_align", dict(row_align=3)), (ssg.SSG_ERR_ARG, "row_align", dict(row_align=512))])
def test_route_descriptors(status, word, change):
    desc = ssg.make_route_desc(**{**dict(T=4, E=16, k=2), **change})
    args, more = route_with(desc)
    refused(status, word, ssg.ssg_route, *args, **more)
    refused(status, word, ssg.ssg_route_bwd, desc, 4096, 4096, 4096, 4096, 4096)
    assert ssg.ssg_route_workspace_bytes(desc) == 0
    with pytest.raises(ssg.SsgError):
        ssg.ssg_route_rows(desc)
    assert ssg.ssg_moe_workspace_bytes(ssg.make_moe_desc(desc, 64, 64)) == 0


def test_route_buffers():
    desc = ssg.make_route_desc(4, 16, 2)
    for name in ("logits", "ids", "weights", "counts", "offsets", "place", "source"):
        args, more = route_with(desc, **{name: None})
        refused(ssg.SSG_ERR_ARG, name, ssg.ssg_route, *args, **more)
        args, more = route_with(desc, **{name: 4097})
        refused(ssg.SSG_ERR_ARG, name, ssg.ssg_route, *args, **more)
    long = ssg.make_route_desc(5000, 16, 2)
    need = ssg.ssg_route_workspace_bytes(long)
    args, more = route_with(long, nbytes=0)
    refused(ssg.SSG_ERR_WORKSPACE, "workspace", ssg.ssg_route, *args, **more)
    args, more = route_with(long, work=None)
    refused(ssg.SSG_ERR_ARG, "workspace", ssg.ssg_route, *args, **more)
    assert need % 256 == 0 and need > 0
    refused(ssg.SSG_ERR_ARG, "dlogits", ssg.ssg_route_bwd, desc, 4096, 4096, 4096, 4096, 4100)


def test_rows_bound():
    assert ssg.ssg_route_rows(ssg.make_route_desc(0, 16, 2)) == 0
    assert ssg.ssg_route_rows(ssg.make_route_desc(1, 64, 8)) == 128
    assert ssg.ssg_route_rows(ssg.make_route_desc(100, 4, 1, row_align=1)) == 100
    assert ssg.ssg_route_rows(ssg.make_route_desc(100, 4, 1)) == 160


def test_i8_refusals():
    assert ssg.ssg_i8_bytes(5, 24) == 0 and "multiple of 16" in ssg.ssg_last_error()
    assert ssg.ssg_i8_bytes(-1, 64) == 0 and ssg.ssg_i8_bytes(1, 131072) == 0 and ssg.ssg_i8_bytes(0, 64) == 256
    assert ssg.ssg_i8_bytes(17, 80) == 32 * 128 + 256
    q = ssg.ssg_i8_quantize
    refused(ssg.SSG_ERR_SHAPE, "K = 20", q, 4096, ssg.SSG_BF16, 4, 20, 20, 4096, q_bytes=1 << 20)
    refused(ssg.SSG_ERR_SHAPE, "rows of src", q, 4096, ssg.SSG_BF16, 4, 64, 60, 4096, q_bytes=1 << 20)
    refused(ssg.SSG_ERR_SHAPE, "rows of src", q, 4096, ssg.SSG_BF16, 4, 64, 68, 4096, q_bytes=1 << 20)
    refused(ssg.SSG_ERR_ARG, "data type", q, 4096, 2, 4, 64, 64, 4096, q_bytes=1 << 20)
    refused(ssg.SSG_ERR_ARG, "src", q, 4100, ssg.SSG_F32, 4, 64, 64, 4096, q_bytes=1 << 20)
    refused(ssg.SSG_ERR_ARG, "256-byte", q, 4096, ssg.SSG_F32, 4, 64, 64, 4112, q_bytes=1 << 20)
    refused(ssg.SSG_ERR_WORKSPACE, "q holds", q, 4096, ssg.SSG_F32, 4, 64, 64, 4096, q_bytes=ssg.ssg_i8_bytes(4, 64) - 1)
    refused(ssg.SSG_ERR_ARG, "codes", ssg.ssg_i8_pack, None, 4096, 4, 64, 4096, q_bytes=1 << 20)
    refused(ssg.SSG_ERR_ARG, "scales", ssg.ssg_i8_unpack, 4096, 4, 64, 4096, None, q_bytes=1 << 20)
    g = ssg.ssg_i8_gemm
    need = ssg.ssg_i8_bytes(16, 64)
    refused(ssg.SSG_ERR_SHAPE, "N = 20", g, 4096, 16, 4096, 20, 64, 4096, ssg.SSG_F32, 20, A_bytes=need, B_bytes=1 << 20)
    refused(ssg.SSG_ERR_WORKSPACE, "A holds", g, 4096, 17, 4096, 16, 64, 4096, ssg.SSG_F32, 16, A_bytes=need, B_bytes=need)
    refused(ssg.SSG_ERR_WORKSPACE, "B holds", g, 4096, 16, 4096, 32, 64, 4096, ssg.SSG_F32, 32, A_bytes=need, B_bytes=need)
    refused(ssg.SSG_ERR_SHAPE, "rows of C", g, 4096, 16, 4096, 16, 64, 4096, ssg.SSG_BF16, 8, A_bytes=need, B_bytes=need)
    refused(ssg.SSG_ERR_SHAPE, "too many", g, 4096, 1 << 26, 4096, 1 << 26, 64, 4096, ssg.SSG_F32, 1 << 26, A_bytes=1 << 40, B_bytes=1 << 40)
    refused(ssg.SSG_ERR_WORKSPACE, "workspace", ssg.ssg_i8_linear, 4096, ssg.SSG_BF16, 4, 64, 64, 4096, 16, 4096, ssg.SSG_F32, 16, 4096, W_bytes=need,
            workspace_bytes=0)


def test_moe_refusals():
    route = ssg.make_route_desc(4, 8, 2)
    desc = ssg.make_moe_desc(route, 64, 48)
    assert ssg.ssg_moe_workspace_bytes(desc) % 256 == 0
    sizes = dict(W1_bytes=ssg.ssg_i8_bytes(8 * 48, 64), W2_bytes=ssg.ssg_i8_bytes(8 * 48, 64), W3_bytes=ssg.ssg_i8_bytes(8 * 64, 48),
                 workspace_bytes=ssg.ssg_moe_workspace_bytes(desc))
    for name in sizes:
        refused(ssg.SSG_ERR_WORKSPACE, name.replace("_bytes", ""), ssg.ssg_moe_fwd, desc, *[4096] * 8, **{**sizes, name: sizes[name] - 1})
    for bad, status in ((ssg.make_moe_desc(ssg.make_route_desc(4, 8, 2, row_align=32), 64, 48), ssg.SSG_ERR_ARG), (ssg.make_moe_desc(route, 60, 48), ssg.SSG_ERR_SHAPE),
                        (ssg.make_moe_desc(route, 64, 0), ssg.SSG_ERR_SHAPE), (ssg.make_moe_desc(route, 64, 48, y_dtype=7), ssg.SSG_ERR_ARG)):
        refused(status, "ssg_moe_fwd", ssg.ssg_moe_fwd, bad, *[4096] * 8, **sizes)
        assert ssg.ssg_moe_workspace_bytes(bad) == 0
    desc.reserved[1] = 1
    refused(ssg.SSG_ERR_ARG, "reserved", ssg.ssg_moe_fwd, desc, *[4096] * 8, **sizes)


def test_plan():
    """Host logic only: which kernel a product runs in."""
    def plan(*args):
        p = ssg.ssg_i8_gemm_plan(*args)
        return (p.tile, p.rows, p.cols)

    assert [plan(M, 4096, 4096) for M in (1, 16, 17, 32, 33, 64)] == [(0, 16, 16)] * 2 + [(0, 32, 16)] * 2 + [(0, 64, 32)] * 2
    # few columns: the smallest blocks whose workgroups the chip holds at once
    assert plan(128, 512, 11008) == (0, 16, 16) and plan(129, 512, 11008) == (0, 32, 16) and plan(257, 512, 11008) == (0, 64, 32)
    assert plan(256, 4096, 4096) == (0, 64, 32) and plan(257, 4096, 4096) == (128, 0, 0)          # 64 and 96 tiles of 128
    assert plan(4096, 4096, 11008) == (256, 0, 0) and plan(2048, 4096, 11008) == (128, 0, 0)
    # experts: 12 rows each on average, and one more
    assert plan(64 * 12, 1376, 2048, 64, 1) == (0, 16, 16) and plan(64 * 12 + 64, 1376, 2048, 64, 1) == (128, 0, 0)
    assert plan(4096 * 8, 1376, 2048, 64, 1) == (256, 0, 0) == plan(4096 * 8, 2048, 1376, 64, 0)
    for args in ((0, 16, 16), (16, 20, 16), (16, 16, 16, -1), (16, 16, 16, 2000), (16, 16, 16, 4, 2), (16, 16, 16, 0, 1)):
        with pytest.raises(ssg.SsgError):
            ssg.ssg_i8_gemm_plan(*args)


def test_workspaces_do_not_shrink_with_more_tokens():
    last = 0
    for T in list(range(0, 300)) + [1000, 1 << 14]:
        n = ssg.ssg_moe_workspace_bytes(ssg.make_moe_desc(ssg.make_route_desc(T, 8, 2), 64, 48))
        assert n >= last
        last = n
