"""Up to four tokens: a wave's share of K from one step to the most that there can be, and the sizes from which such calls run like longer ones."""
import pytest
import torch

import paper_2409_12517_amd as ssg
from gpu_util import DEV
from test_gpu_moe import Layer


def few(T, k, d, f):
    """Whether a call keeps an order of dispatch (host logic)."""
    return ssg.ssg_moe_view_workspace(ssg.make_moe_desc(ssg.make_route_desc(T, 32, k), d, f), 1 << 20).offsets is None


@pytest.mark.parametrize("k", range(1, 33))
def test_which_calls_keep_an_order(k):
    waves = max(w for w in (1, 2, 4, 8, 16) if w * k <= 16 or w == 1)
    most = min(8192 * waves, 131056)
    assert few(4, k, 64, most) and few(1, k, 65536, 16) and not few(5, k, 64, 64) and not few(1, k, 65552, 16)
    if most < 131056:
        assert not few(1, k, 64, most + 16)


@pytest.mark.gpu
@pytest.mark.parametrize("E,k,d,f", [(3, 2, 64, 11008), (9, 8, 64, 4112), (12, 11, 48, 1376), (5, 5, 32, 1040), (10, 9, 64, 8192), (3, 1, 32, 28672)])
def test_shares(E, k, d, f):
    """Several sets of weights to a wave, more codes than lanes, 128 KB of LDS."""
    assert few(2, k, d, f)
    for y_dtype in (torch.bfloat16, torch.float32):
        layer = Layer(2, E, k, d, f, y_dtype=y_dtype)
        layer.check(layer.run())


@pytest.mark.gpu
def test_beyond_the_limit():
    """One block of 16 channels more than LDS takes: the other path, whose bits at the limit are the same."""
    layer = Layer(2, 10, 9, 64, 8208)
    assert not few(2, 9, 64, 8208)
    layer.check(layer.run())
    layer = Layer(6, 10, 9, 64, 8192)
    whole, x, z = layer.run(), layer.x, layer.logits
    part = Layer(4, 10, 9, 64, 8192)
    part.x, part.logits = x[:4].contiguous(), z[:4].contiguous()
    assert torch.equal(part.run(), whole[:4])


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 3])
@pytest.mark.parametrize("K", [2048, 5120, 8192, 14336, 16384])
def test_linear_shares(M, K):
    """The same of one matrix, against rows that other kernels take (a token's bits do not depend on its batch)."""
    N = 48
    gen = torch.Generator(device=DEV).manual_seed(K)
    x = torch.randn(40, K, generator=gen, device=DEV).bfloat16()
    W = torch.empty(ssg.ssg_i8_bytes(N, K), dtype=torch.uint8, device=DEV)
    ssg.ssg_i8_quantize(torch.randn(N, K, generator=gen, device=DEV), ssg.SSG_F32, N, K, K, W)

    def linear(rows):
        y = torch.empty(rows.shape[0], N, device=DEV)
        work = torch.empty(ssg.ssg_i8_linear_workspace_bytes(rows.shape[0], K), dtype=torch.uint8, device=DEV)
        ssg.ssg_i8_linear(rows, ssg.SSG_BF16, rows.shape[0], K, K, W, N, y, ssg.SSG_F32, N, work)
        return y

    assert torch.equal(linear(x[:M]), linear(x)[:M])
