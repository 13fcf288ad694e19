"""Decode over 8 bits: sums over thousands of rows of one warp do not drift.

All values are one number, so the output is that number times sum_j p'_j / sum_j p_j with p' what the products take of the
weights p: whatever the logits are, what remains are the roundings of the two sums.  Rounded to the nearest they have no mean:
after N additions of a sum that grows evenly their deviation is sqrt(N / 3) * 2^-24 / sqrt(3).  A warp adds rows / 16 / SUBS
sums of the tensor core (of 16 rows, from zero: two products that each cut off at most 2^-23 of the sum, towards zero, in all
a mean of at most 2^-22) and every one of its eight lanes rows / 8 / SUBS weights (of an own part of the sum: a deviation of
1 / sqrt(8) of the whole).  So the mean error over all regions and heads stays within 2^-22 (and what is left of the
deviation), and no output is off by more than six deviations beside it.  Sums that the tensor core carries on from row to row lose 2^-24
on average with every product: a mean that grows with the rows."""
import math

import pytest
import torch

import paper_2503_23956_b200 as ac

DEV = "cuda:0"


@pytest.mark.gpu
@pytest.mark.parametrize("H,G,d", [(1, 16, 128), (2, 9, 128), (4, 12, 128), (8, 9, 128), (8, 16, 128),
                                   (8, 8, 128), (2, 16, 64), (8, 12, 64)])
@pytest.mark.parametrize("n", [500, 4000])
def test_the_mean_error_does_not_grow(n, H, G, d):
    R = 150   # more regions than SMs: a region is whole in a block, with a warp for every SUBS-th tile of a head
    sh = ac.shape(R, 1, H * G, H, d, 3, 1, 1, 0)
    rows, subs = R * n, 8 // H
    gen = torch.Generator(device=DEV).manual_seed(n + H)
    offsets = torch.arange(R + 1, device=DEV) * n
    lens = torch.full((R,), n, dtype=torch.int32, device=DEV)
    k8 = torch.randint(0, 0x48, (rows, H, d), generator=gen, dtype=torch.uint8, device=DEV)   # up to 4
    k8 |= torch.randint(0, 2, (rows, H, d), generator=gen, dtype=torch.uint8, device=DEV) << 7
    v8 = torch.full((rows, H, d), 0x3b, dtype=torch.uint8, device=DEV)   # 1.375
    blocks = ac.aircache_scale_blocks(sh, rows)
    k_scale, v_scale = torch.ones((blocks, H), device=DEV), torch.full((blocks, H), 0.25, device=DEV)
    q = torch.randn((R, H * G, d), generator=gen, device=DEV).mul_(0.5).bfloat16()
    out = torch.empty((R, H * G, d), device=DEV)
    ws = torch.zeros(ac.aircache_workspace_bytes(sh), dtype=torch.uint8, device=DEV)
    ac.aircache_decode_attn_quantized(sh, ac.quantized_view(k8, v8, k_scale, v_scale, offsets, lens, rows), q, out, ws)
    error = out.double() / (1.375 * 0.25) - 1
    deviation = (math.sqrt(n / 16 / subs / 3) + math.sqrt(n / 8 / subs / 3 / 8)) * 2.0 ** -24 / math.sqrt(3)
    # (channels of a head are alike; the heads and regions are independent)
    assert abs(error.mean().item()) <= 2.0 ** -22 + 6 * deviation / math.sqrt(R * H * G)
    assert error.abs().max().item() <= 2.0 ** -22 + 6 * deviation
