"""Routing of long batches: above 4096 tokens a wave chooses for four at once, and a block may order several thousand assignments."""
import numpy as np
import pytest
import torch

import paper_2409_12517_amd as ssg
from gpu_util import DEV, f32
from test_gpu_route import W_TOL, call, check, desc_of, logits_of

pytestmark = pytest.mark.gpu
SOFTMAX, SIGMOID = ssg.SSG_ROUTE_SOFTMAX, ssg.SSG_ROUTE_SIGMOID
NAMES = ("ids", "weights", "counts", "offsets", "place", "source")


def bias_of(E):
    return (torch.randint(-50, 51, (E,), generator=torch.Generator().manual_seed(5)) * 1e-3).to(DEV)


def compare_with_a_short_batch(z, bias, got, first, rows, sums, **more):
    """The same tokens in a call whose waves choose for one: the same choice and the same bits of the weights, but for the softmax's
    sum, whose terms are added in another order (and a choice that hangs on it)."""
    part = z[first:first + rows].contiguous()
    short = call(desc_of(rows, z.shape[1], got["ids"].shape[1], z.dtype, **more), part, bias, sort=False)
    ids, w = (got[n][first:first + rows] for n in ("ids", "weights"))
    if not sums:
        assert torch.equal(ids, short["ids"]) and torch.equal(w, short["weights"])
    else:
        same = (ids == short["ids"]).all(-1)
        assert same.float().mean() > 0.9
        assert ((w - short["weights"]).abs() <= 2 * W_TOL * w.abs())[same].all()


@pytest.mark.parametrize("T,E,k,dtype", [(4099, 3, 2, torch.float32), (5003, 16, 1, torch.bfloat16), (4097, 17, 16, torch.float32), (4110, 33, 5, torch.bfloat16),
                                         (4099, 64, 8, torch.float32), (4098, 160, 6, torch.bfloat16), (4101, 256, 16, torch.float32)])
@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
@pytest.mark.parametrize("biased", [False, True])
def test_choice(T, E, k, dtype, score, biased):
    more = dict(score=score, renorm=T % 2, scale=2.5)
    d = desc_of(T, E, k, dtype, **more)
    z = logits_of(T, E, dtype, T + E, closed=0.3 if E > 30 else 0.0).to(DEV)
    bias = bias_of(E) if biased else None
    got = call(d, z, bias)
    check(d, z, bias, got)
    compare_with_a_short_batch(z, bias, got, 1000, 70, score == SOFTMAX and (biased or not more["renorm"]), **more)


@pytest.mark.parametrize("E,k,groups,top", [(64, 8, 8, 3), (250, 7, 10, 4), (256, 16, 16, 5), (48, 3, 16, 1), (30, 16, 2, 2), (12, 2, 4, 2)])
@pytest.mark.parametrize("by", [1, 2])
@pytest.mark.parametrize("score,biased", [(SOFTMAX, False), (SIGMOID, False), (SIGMOID, True)])
def test_groups(E, k, groups, top, by, score, biased):
    T = 4099
    more = dict(score=score, groups=groups, top_groups=top, group_top=by)
    d = desc_of(T, E, k, torch.float32, **more)
    z = logits_of(T, E, torch.float32, E + k, closed=0.2).to(DEV)
    bias = bias_of(E) if biased else None
    got = call(d, z, bias)
    check(d, z, bias, got)
    compare_with_a_short_batch(z, bias, got, 4000, 99, score == SOFTMAX and by == 2, **more)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strided_logits(dtype):
    T, E = 4103, 40
    wide = logits_of(T, 50, dtype, 3).to(DEV)
    d = desc_of(T, E, 4, dtype, ld=50)
    part = wide[:, 7:7 + E]
    check(d, part, None, call(d, part))


@pytest.mark.parametrize("T,E,k", [(9001, 1024, 32), (70001, 64, 8), (70001, 8, 3), (33000, 300, 20)])
def test_order_where_a_block_has_several_sets_of_assignments(T, E, k):
    """More than 1024 assignments to a block, the last set partly filled: the order is that of a stable sort."""
    d = desc_of(T, E, k, torch.float32)
    gen = torch.Generator(device=DEV).manual_seed(T + E)
    z = torch.randn(T, E, generator=gen, device=DEV)
    z[:, E // 2] += 3.0                                         # one expert with most of the rows
    z[torch.rand(T, generator=gen, device=DEV) < 0.1] = -torch.inf
    got = {n: v.cpu().numpy() for n, v in call(d, z).items()}
    flat = got["ids"].reshape(-1)
    live = np.nonzero(flat >= 0)[0]
    order = live[np.argsort(flat[live], kind="stable")]
    counts = np.bincount(flat[live], minlength=E)
    offsets = np.concatenate([[0], np.cumsum(-(-counts // 16) * 16)])
    place, source = np.full(flat.size, -1), np.full(ssg.ssg_route_rows(d), -1)
    place[order] = np.arange(order.size) - (np.cumsum(counts) - counts)[flat[order]] + offsets[flat[order]]
    source[place[order]] = order
    for name, ref in (("counts", counts), ("offsets", offsets), ("place", place), ("source", source)):
        assert np.array_equal(got[name], ref), name
