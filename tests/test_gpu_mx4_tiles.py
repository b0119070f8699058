"""4-bit products in the tiles: one and several tiles to a workgroup, halves of tiles, ragged edges, K of one step to many."""
import pytest
import torch

import paper_2409_12517_amd as ssg
from gpu_util import DEV

pytestmark = pytest.mark.gpu
LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def operand(rows, K, seed):
    """Codes of every value with scales of 1 and 2, packed by the library; their values."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    codes = torch.randint(0, 16, (rows, K), generator=gen, device=DEV)
    scales = torch.randint(0, 2, (rows, -(-K // 32)), generator=gen, device=DEV)
    q = torch.full((ssg.ssg_mx4_bytes(rows, K),), 0xA5, dtype=torch.uint8, device=DEV)
    ssg.ssg_mx4_pack((codes[:, ::2] + 16 * codes[:, 1::2]).to(torch.uint8), (scales + 127).to(torch.uint8), rows, K, q)
    level = torch.tensor(LEVELS + [-v for v in LEVELS], dtype=torch.float64, device=DEV)
    return q, level[codes] * (2.0 ** scales.double()).repeat_interleave(32, 1)[:, :K]


# Sums of up to 11008 terms, multiples of 1/4 up to 144, are exact in fp32 in any order (their partial sums are below 2^23 quarters): the
# result is the exact sum rounded once.
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,N,K", [
    (1000, 2064, 208), (1000, 2064, 528), (2500, 2064, 1200), (1090, 1040, 640), (1040, 16400, 304), (4420, 4112, 1040), (4096, 4096, 512), (4100, 4096, 208), (4100, 4096, 272),
    (8300, 4112, 1296), (4100, 8208, 2736), (4096, 4096, 11008), (4096, 11008, 4096), (20000, 4096, 784), (3900, 4080, 1040), (4000, 4096, 800)])
def test_tiles(dtype, M, N, K):
    (qa, a), (qb, b) = operand(M, K, 1), operand(N, K, 2)
    out = torch.full((M + 1, N + 16), 3.0, dtype=dtype, device=DEV)
    ssg.ssg_mx4_gemm(qa, M, qb, N, K, out, ssg.SSG_BF16 if dtype == torch.bfloat16 else ssg.SSG_F32, N + 16)
    assert torch.equal(out[:M, :N], (a @ b.t()).to(dtype))
    assert bool((out[:, N:] == 3).all()) and bool((out[M] == 3).all()), "written outside the result"
