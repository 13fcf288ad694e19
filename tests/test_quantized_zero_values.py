"""Decode over 8 bits where whole blocks of the cache are zero or tiny: their scale is 2^-126, the smallest that there is.

Tolerance: that of test_quantized_cache, where the largest V scale S counts as 2^-116 at least, and for values near the smallest fp32 numbers what the steps between those cost: a
sum in them is off by at most 2^-150 for each of its roundings (the posting of up to 8 warps' sums, their merge, that of up
to 256 parts, the division by a sum of weights of at least one): below 2^-140."""
import numpy as np
import pytest
import torch

import paper_2503_23956_b200 as ac
from test_quantized_cache import BLOCK, DEV, TABLE, Cache, attention, queries

LENGTHS = {
    "whole": [130, 64, 1, 70, 33],
    "cut": [5000, 200],
    "list": [(7 * i) % 150 + 1 for i in range(200)],   # more regions than there are SMs
}
HEADS = [(H, G, d) for d in (64, 128) for H, G in ((1, 7), (2, 4), (4, 7), (8, 8), (1, 16), (2, 9), (4, 12), (8, 9))]


def blocks_of(c, pattern):
    """The rows of the blocks that a pattern names, over all regions."""
    rows = []
    for r, n in enumerate(c.lens0):
        o, blocks = int(c.offs[r]), -(-n // BLOCK)
        take = {"all": range(blocks), "first": [0], "last": [blocks - 1], "even": range(0, blocks, 2),
                "odd": range(1, blocks, 2)}[pattern]
        for b in take:
            rows.extend(range(o + b * BLOCK, o + min(n, (b + 1) * BLOCK)))
    return torch.tensor(rows, dtype=torch.int64, device=DEV)


def held_by(c):
    return {x: getattr(c, x).cpu().numpy() for x in ("k8", "v8", "k_scale", "v_scale")}


def check(c, G, lens, seed=1):
    q = queries(c, G, seed)
    out = torch.full((c.R, c.H * G, c.d), float("nan"), device=DEV)
    ac.aircache_decode_attn_quantized(c.sh, c.cache8, q, out, c.ws)
    q, got = q.double().cpu().numpy(), out.double().cpu().numpy()
    now = held_by(c)
    for r, (k, v, _) in enumerate(c.values(now, lens)):
        o, n = int(c.offs[r]), lens[r]
        largest = now["v_scale"][o // BLOCK + r + np.arange(n) // BLOCK].max(axis=0, initial=2.0 ** -116)
        held = 2.0 ** -36 * largest.astype(np.float64)[:, None] * np.abs(TABLE[now["v8"][o:o + n]]).sum(axis=0)
        for h in range(c.H):
            heads = slice(h * G, (h + 1) * G)
            want, tol = attention(q[r, heads], k[:, h], v[:, h], c.sh.scale, held[h])
            assert (np.abs(got[r, heads] - want) <= tol + 2.0 ** -140).all(), (r, h, lens[r])
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("H,G,d", HEADS)
@pytest.mark.parametrize("lens", list(LENGTHS))
def test_blocks_of_zeros(lens, H, G, d):
    lens = LENGTHS[lens]
    c = Cache(lens, H, d, Hq=H * G, seed=H)
    k, v = c.k.clone(), c.v.clone()
    for pattern, what in (("all", "v"), ("first", "v"), ("last", "v"), ("even", "kv"), ("odd", "v"), ("first", "k")):
        c.k.copy_(k)
        c.v.copy_(v)
        rows = blocks_of(c, pattern)
        for x in what:
            getattr(c, x)[rows] = 0
        ac.aircache_quantize(c.sh, c.ragged, c.cache8)
        out = check(c, G, lens)
        if pattern == "all":
            assert (out == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("H,G,d", [(1, 7, 128), (2, 4, 64), (8, 9, 128), (4, 12, 64)])
@pytest.mark.parametrize("lens", list(LENGTHS))
@pytest.mark.parametrize("size", [2.0 ** -110, 2.0 ** -117, 2.0 ** -120, 2.0 ** -133])
def test_tiny_values(size, lens, H, G, d):
    """Scales of 2^-117 and below, where 2^11 over the scale is no fp32 number; alone and in front of ordinary blocks."""
    lens = LENGTHS[lens]
    c = Cache(lens, H, d, Hq=H * G, seed=H)
    v = c.v.clone()
    for pattern in ("all", "first"):
        c.v.copy_(v)
        rows = blocks_of(c, pattern)
        c.v[rows] = (c.v[rows].double() * size).bfloat16()
        ac.aircache_quantize(c.sh, c.ragged, c.cache8)
        check(c, G, lens)


@pytest.mark.gpu
@pytest.mark.parametrize("H,G,d", [(1, 7, 128), (4, 7, 64), (2, 16, 128)])
def test_appended_rows_of_zeros(H, G, d):
    """Into an empty region, into a new block and into one that is there; then an ordinary row behind them."""
    lens = [0, 64, 128, 65, 40, 0]
    c = Cache(lens, H, d, Hq=H * G, slack=3, seed=2)
    ac.aircache_quantize(c.sh, c.ragged, c.cache8)
    gen = torch.Generator().manual_seed(5)
    for i in range(3):
        new = torch.randn((2, c.R, H, d), generator=gen).bfloat16().to(DEV) * (i == 2)
        ac.aircache_append_quantized(c.sh, c.cache8, new[0], new[1], i)
        out = check(c, G, [n + i + 1 for n in lens], seed=i)
        if i < 2:
            assert (out[0] == 0).all() and (out[5] == 0).all()


def test_the_smallest_scale_under_the_lift():
    """2^11 / 2^-126 is no fp32 number; 2^11 / 2^-116 is."""
    with np.errstate(over="ignore"):
        assert np.isinf(np.float32(2048) / np.float32(2.0 ** -126))
    assert np.float32(2048) / np.float32(2.0 ** -116) == 2.0 ** 127
