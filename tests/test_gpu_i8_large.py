"""Codes of more than 64 GB: a thread for every 16 bytes is more threads than a launch takes along one axis."""
import pytest
import torch

import paper_2409_12517_amd as ssg
from gpu_util import DEV

pytestmark = pytest.mark.gpu


def test_pack_and_unpack():
    rows, K = (1 << 19) + 37, 131056
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 160 << 30:
        pytest.skip("needs 160 GB of free device memory")
    codes = torch.empty(rows, K, dtype=torch.int8, device=DEV)
    scales = torch.rand(rows, device=DEV)
    q = torch.empty(ssg.ssg_i8_bytes(rows, K), dtype=torch.uint8, device=DEV)
    parts = [(0, 32), (1 << 18, 48), ((1 << 19) - 16, 53)]        # (from a multiple of 16; the last two lie on both sides of 2^32 runs of 16)
    for first, n in parts:
        codes[first:first + n].random_(-128, 128)
    held = [codes[first:first + n].clone() for first, n in parts]
    ssg.ssg_i8_pack(codes, scales, rows, K, q)
    for (first, n), part in zip(parts, held):
        alone = torch.empty(ssg.ssg_i8_bytes(n, K), dtype=torch.uint8, device=DEV)
        ssg.ssg_i8_pack(part, scales[first:first + n], n, K, alone)
        size = -(-n // 16) * 16 * 131072
        assert torch.equal(q[first * 131072:first * 131072 + size], alone[:size]), first
        codes[first:first + n] = 0
    back = torch.empty(rows, device=DEV)
    ssg.ssg_i8_unpack(q, rows, K, codes, back)
    assert torch.equal(back, scales)
    for (first, n), part in zip(parts, held):
        assert torch.equal(codes[first:first + n], part), first
    del codes, q
    torch.cuda.empty_cache()
