"""Routing where scores are next to 0 or 1: weights and gradients with errors relative to themselves, from references without differences of
nearly equal numbers."""
import numpy as np
import pytest
import torch

import paper_2409_12517_amd as ssg
from gpu_util import DEV, f32

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
SOFTMAX, SIGMOID = ssg.SSG_ROUTE_SOFTMAX, ssg.SSG_ROUTE_SIGMOID


def desc_of(z, k, **more):
    return ssg.make_route_desc(z.shape[0], z.shape[1], k, logits_dtype=ssg.SSG_BF16 if z.dtype == torch.bfloat16 else ssg.SSG_F32, **more)


def route(desc, z, bias=None):
    ids, w = torch.full((desc.T, desc.k), -77, dtype=torch.int32, device=DEV), torch.full((desc.T, desc.k), -77.0, device=DEV)
    ssg.ssg_route(desc, z.to(DEV), bias, ids, w, None, None, None, None, None)
    return ids, w


def gradient(desc, z, ids, w, dw):
    dz = torch.full((desc.T, desc.E), -5.0, dtype=z.dtype, device=DEV)
    ssg.ssg_route_bwd(desc, z.to(DEV), ids, w, dw, dz)
    return f32(dz).astype(np.float64)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sigmoid_gradient_of_confident_choices(dtype):
    """s (1 - s) of logits from 0 to 80, on both sides: two sigmoids good to 6 ulp, three products, one rounding to the logits' type."""
    at = torch.arange(0, 80, 0.375)
    z = torch.cat([at, -at])[:, None].to(dtype)
    desc = desc_of(z, 1, score=SIGMOID, renorm=0, scale=2.5)
    ids, w = route(desc, z)
    dw = torch.randn(z.shape[0], 1, generator=torch.Generator().manual_seed(1)).to(DEV)
    zz = f32(z).astype(np.float64)
    ref = 2.5 * f32(dw).astype(np.float64) / (1 + np.exp(-zz)) / (1 + np.exp(zz))
    tol = (2 * 12 + 4) * EPS + (2.0 ** -8 if dtype == torch.bfloat16 else 0.0)
    assert (np.abs(gradient(desc, z, ids, w, dw) - ref) <= tol * np.abs(ref)).all()


# relative error of a weight: the argument of the exponential rounded once where it is below 32, expf and the sigmoid good to 6 ulp, a sum of 16
# terms in sequence and 6 in a tree, two divisions and a product
W_TOL = (32 + 2 * 6 + 22 + 3) * 2 * EPS


def test_sigmoid_scores_of_low_logits():
    """As they are: e^z down to the smallest number, in steps of it."""
    z = -torch.arange(75, 110, 0.25)[:, None]
    desc = desc_of(z, 1, score=SIGMOID, renorm=0)
    ids, w = route(desc, z)
    ref = np.exp(f32(z).astype(np.float64))
    assert (np.abs(f32(w) - ref) <= W_TOL * ref + 2 * 2.0 ** -149).all()
    dz = gradient(desc, z, ids, w, torch.ones(z.shape[0], 1, device=DEV))
    assert (np.abs(dz - ref) <= W_TOL * ref + 4 * 2.0 ** -149).all()
    dz = gradient(desc_of(z, 1, score=SIGMOID, renorm=0), -z, ids, w, torch.ones(z.shape[0], 1, device=DEV))
    assert (np.abs(dz - ref) <= W_TOL * ref + 4 * 2.0 ** -149).all()


def test_the_order_of_the_lowest_scores():
    z = torch.tensor([[-100.0, -89.0, -95.0, -92.0, -101.0]])
    for bias in (None, torch.zeros(5, device=DEV)):
        assert route(desc_of(z, 5, score=SIGMOID), z, bias)[0].tolist() == [[1, 3, 2, 0, 4]]


def shares(z):
    """Sigmoids of each row of z, divided by their sum."""
    log = -np.logaddexp(0.0, -z)
    e = np.exp(log - log.max(-1, keepdims=True))
    return e / e.sum(-1, keepdims=True)


def low_logits(T, E):
    """Rows whose largest logit is between -10 and -3e38, the others up to 30 below it."""
    gen = np.random.default_rng(3)
    base = np.array([-10, -15, -21, -60, -79.5, -86, -88.5, -90, -104, -120, -500, -3e38])[np.arange(T) % 12]
    return torch.from_numpy((base[:, None] - gen.permuted(np.linspace(0, 30, E), axis=None) * gen.random((T, 1)))).float()


@pytest.mark.parametrize("E,k", [(5, 1), (16, 4), (40, 20)])
def test_renormalised_sigmoid_weights_of_low_logits(E, k):
    z = low_logits(48, E)
    desc = desc_of(z, k, score=SIGMOID, scale=2.5)
    ids, w = route(desc, z)
    ids = ids.cpu().numpy()
    ref = 2.5 * shares(np.take_along_axis(f32(z).astype(np.float64), ids, 1))
    assert (np.abs(f32(w) - ref) <= W_TOL * ref).all()
    # the gradient: r_j (1 - s_j) sum_i r_i (dw_j - dw_i) scale, where 1 - s_j is 1 to 5e-5
    dw = torch.randn(48, k, generator=torch.Generator().manual_seed(1)).to(DEV)
    got = np.take_along_axis(gradient(desc, z, torch.from_numpy(ids).to(DEV), w, dw), ids, 1)
    chosen, d = np.take_along_axis(f32(z).astype(np.float64), ids, 1), f32(dw).astype(np.float64)
    r = shares(chosen)
    want = 2.5 * r / (1 + np.exp(chosen)) * (r[:, None, :] * (d[:, :, None] - d[:, None, :])).sum(-1)
    assert (np.abs(got - want) <= 4 * W_TOL * 2.5 * r * np.abs(d).max(-1, keepdims=True)).all()


def test_renormalised_softmax_weights_far_below_the_largest():
    """A bias sends tokens past their best expert; the chosen ones' scores, e^-60 to e^-130, still have their ratios."""
    z = torch.tensor([[t, 0.0, -1.0, -2.5, 1.5] for t in (0.0, 60.0, 85.0, 95.0, 130.0)])
    bias = torch.tensor([-1e3, 4.0, 3.0, 2.0, 1.0], device=DEV)
    desc = desc_of(z, 3, scale=2.5)
    ids, w = route(desc, z, bias)
    assert ids.tolist() == [[1, 2, 3]] * 5
    e = np.exp(np.array([0.0, -1.0, -2.5]))
    ref = 2.5 * e / e.sum()
    assert (np.abs(f32(w) - ref) <= W_TOL * ref).all()


@pytest.mark.parametrize("renorm", [0, 1])
@pytest.mark.parametrize("k", [1, 3, 20])
@pytest.mark.parametrize("E", [23, 160])
def test_softmax_gradient_of_confident_choices(renorm, k, E):
    """dz_e = s_e sum_i s_i (q_e - q_i): over the pairs with the expert that has nearly all of the softmax, and every other.  An error is
    relative to the terms of the sum, each a product of two scores (of shares, where they are renormalised)."""
    gen = torch.Generator().manual_seed(E + k)
    z = torch.randn(64, E, generator=gen)
    z[torch.arange(64), torch.randint(0, E, (64,), generator=gen)] += torch.linspace(0, 20, 64)
    desc = desc_of(z, k, renorm=renorm, scale=2.5)
    ids, w = route(desc, z)
    dw = torch.randn(64, k, generator=gen).to(DEV)
    got = gradient(desc, z, ids, w, dw)
    rows, host = np.arange(64)[:, None], ids.cpu().numpy()
    zz, q = f32(z).astype(np.longdouble), np.zeros((64, E), np.longdouble)
    q[rows, host] = 2.5 * f32(dw)
    s = np.exp(zz - zz.max(-1, keepdims=True))
    if renorm:
        chosen = np.zeros((64, E), bool)
        chosen[rows, host] = True
        s = np.where(chosen, s, 0)
    s /= s.sum(-1, keepdims=True)
    apart = q[:, :, None] - q[:, None, :]
    ref = s * (s[:, None, :] * apart).sum(-1)
    size = s * (s[:, None, :] * (np.abs(q)[:, :, None] + np.abs(q)[:, None, :]) * ~np.eye(E, dtype=bool)).sum(-1)
    assert (np.abs(got - ref) <= 4 * W_TOL * size).all()


@pytest.mark.parametrize("shut", [-torch.inf, torch.nan])
def test_a_bias_that_shuts_an_expert_changes_no_score(shut):
    z = torch.tensor([[3.0, 2.0, 1.0, 0.0], [-torch.inf, 0.5, 0.25, torch.nan]])
    bias = torch.tensor([shut, 0.0, 0.0, 0.0], device=DEV)
    desc = desc_of(z, 3, renorm=0)
    ids, w = route(desc, z, bias)
    assert ids.tolist() == [[1, 2, 3], [1, 2, -1]]
    e = np.exp(np.array([[3.0, 2.0, 1.0, 0.0], [-np.inf, 0.5, 0.25, -np.inf]]))
    s = e / e.sum(-1, keepdims=True)
    ref = np.stack([s[0, 1:], [s[1, 1], s[1, 2], 0.0]])
    assert (np.abs(f32(w) - ref) <= W_TOL * ref).all()
    # its logit moves the others' scores: dz_0 = -s_0 sum_j s_j dw_j
    got = gradient(desc, z, ids, w, torch.ones(2, 3, device=DEV))
    assert abs(got[0, 0] + s[0, 0] * s[0, 1:].sum()) <= 4 * W_TOL and got[1, 0] == 0.0
