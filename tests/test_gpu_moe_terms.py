"""The mixture with bf16 results from fp32 terms: one rounding to bf16, that of the sum."""
import pytest
import torch

import paper_2409_12517_amd as ssg
from gpu_util import DEV


def test_refused():
    desc = ssg.make_moe_desc(ssg.make_route_desc(4, 8, 2), 64, 48, ssg.SSG_BF16, f32_terms=2)
    with pytest.raises(ssg.SsgError, match="f32_terms 2"):
        ssg.ssg_moe_fwd(desc, *[4096] * 8, stream=0, W1_bytes=1 << 20, W2_bytes=1 << 20, W3_bytes=1 << 20, workspace_bytes=1 << 20)
    assert ssg.ssg_moe_workspace_bytes(desc) == 0


def test_workspace():
    def size(y_dtype, terms):
        return ssg.ssg_moe_workspace_bytes(ssg.make_moe_desc(ssg.make_route_desc(100, 8, 2), 64, 48, y_dtype, terms))

    assert size(ssg.SSG_BF16, 1) == size(ssg.SSG_F32, 0) == size(ssg.SSG_F32, 1) > size(ssg.SSG_BF16, 0)


def test_what_a_caller_gets_who_names_nothing():
    route = ssg.make_route_desc(4, 8, 2)
    kinds = [(d.y_dtype, d.f32_terms) for d in (ssg.make_moe_desc(route, 64, 48), ssg.make_moe_desc(route, 64, 48, ssg.SSG_BF16),
                                                ssg.make_moe_desc(route, 64, 48, ssg.SSG_F32), ssg.make_moe_desc(route, 64, 48, f32_terms=0))]
    assert kinds == [(ssg.SSG_BF16, 1), (ssg.SSG_BF16, 0), (ssg.SSG_F32, 0), (ssg.SSG_BF16, 0)]


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 4, 5, 40, 700])
@pytest.mark.parametrize("E,k,d,f", [(3, 1, 272, 80), (8, 2, 528, 400), (12, 5, 96, 208), (24, 8, 256, 336), (40, 20, 80, 64)])
def test_one_rounding(T, E, k, d, f):
    """The bits of the fp32 result, which holds the same terms and sums them in the same order, rounded to bf16."""
    gen = torch.Generator(device=DEV).manual_seed(T + E)
    x = torch.randn(T, d, generator=gen, device=DEV).bfloat16()
    logits = torch.randn(T, E, generator=gen, device=DEV)
    logits[T // 2, : E // 2] = -torch.inf

    def quantized(rows, K):
        q = torch.empty(ssg.ssg_i8_bytes(rows, K), dtype=torch.uint8, device=DEV)
        ssg.ssg_i8_quantize(torch.randn(rows, K, generator=gen, device=DEV) * K ** -0.5, ssg.SSG_F32, rows, K, K, q)
        return q

    W = quantized(E * f, d), quantized(E * f, d), quantized(E * d, f)

    def mixture(y_dtype, terms):
        desc = ssg.make_moe_desc(ssg.make_route_desc(T, E, k), d, f, ssg.SSG_F32 if y_dtype == torch.float32 else ssg.SSG_BF16, terms)
        y = torch.full((T, d), 9.0, dtype=y_dtype, device=DEV)
        work = torch.full((ssg.ssg_moe_workspace_bytes(desc),), 0xC3, dtype=torch.uint8, device=DEV)
        ssg.ssg_moe_fwd(desc, x, logits, None, *W, y, work)
        return y, desc, work

    y32, desc32, work32 = mixture(torch.float32, 0)
    y16, desc16, work16 = mixture(torch.bfloat16, 1)
    assert torch.equal(y16, y32.bfloat16())
    if T > 4:                                                   # (up to four tokens keep no results of experts)
        def results(desc, work):
            view = ssg.ssg_moe_view_workspace(desc, work)
            rows = int(ssg.view_tensor(work, work.data_ptr(), view.offsets, (E + 1,), torch.int32)[-1])
            return ssg.view_tensor(work, work.data_ptr(), view.o, (rows, d), torch.float32)

        assert torch.equal(results(desc16, work16), results(desc32, work32))
