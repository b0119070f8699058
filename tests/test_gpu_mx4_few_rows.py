"""Which linear layers of few rows quantize them in the product's own launch: by the launches that a call records."""
import pytest
import torch

import paper_2409_12517_amd as ssg
from gpu_util import DEV

pytestmark = pytest.mark.gpu
SSG = {torch.bfloat16: ssg.SSG_BF16, torch.float32: ssg.SSG_F32}
BF, F = torch.bfloat16, torch.float32
ROWS, PRODUCT = 55, 56                                       # tags of the launches


def launches(M, N, K, dtype):
    x = torch.ones(M, K, dtype=dtype, device=DEV)
    W = torch.zeros(ssg.ssg_mx4_bytes(N, K), dtype=torch.uint8, device=DEV)
    y = torch.full((M, N), 3.0, device=DEV)
    work = torch.empty(ssg.ssg_mx4_linear_workspace_bytes(M, K), dtype=torch.uint8, device=DEV)
    ssg.ssg_profile_select(-1)
    ssg.ssg_profile_enable(4)
    try:
        ssg.ssg_mx4_linear(x, SSG[dtype], M, K, K, ssg.SSG_MX_FLOOR, W, N, y, ssg.SSG_F32, N, work)
        _, tags = ssg.ssg_profile_read(4)
    finally:
        ssg.ssg_profile_enable(0)
    assert not y.any()                                       # (weights of zeros)
    return tags


@pytest.mark.parametrize("M,N,K,one", [(1, 32, 92416, True), (1, 32, 92432, False), (2, 32, 46080, True), (3, 32, 4096, True), (17, 32, 256, False), (16, 32, 256, True)])
def test_room_for_the_rows(M, N, K, one):
    """48 KiB for their codes and scales, 17 bytes to a block of 32 of K filled up to 256."""
    assert launches(M, N, K, BF) == ([PRODUCT] if one else [ROWS, PRODUCT])


@pytest.mark.parametrize("dtype,M,N,K,one", [
    # one row in one launch, unless short weights of many columns leave its quantization bare
    (BF, 1, 11008, 4096, True), (F, 1, 11008, 4096, True), (BF, 1, 28672, 8192, True), (BF, 1, 28672, 1024, False), (F, 1, 28672, 1024, False), (F, 1, 28672, 4096, False),
    # two to four: fp32 rows sooner in a launch of their own
    (BF, 2, 11008, 4096, True), (F, 2, 11008, 4096, False), (F, 2, 4096, 8192, True), (F, 2, 8192, 8192, False), (BF, 4, 4096, 4096, True), (F, 4, 4096, 4096, True),
    (F, 4, 4096, 4112, False), (F, 4, 11008, 4096, False), (BF, 4, 11008, 4096, True), (BF, 4, 11008, 11008, False), (F, 4, 16, 4112, False),
    # more
    (BF, 5, 4096, 4096, True), (F, 5, 4096, 4096, False), (BF, 8, 4096, 5728, True), (BF, 8, 4096, 5744, False), (F, 8, 1040, 1680, True), (F, 8, 1040, 1696, False),
    (BF, 16, 4096, 2192, True), (BF, 16, 4096, 2208, False), (F, 16, 16, 768, True), (F, 16, 16, 784, False)])
def test_cost_of_the_rows(dtype, M, N, K, one):
    assert launches(M, N, K, dtype) == ([PRODUCT] if one else [ROWS, PRODUCT])
