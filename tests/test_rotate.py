"""aircache_rotate against its formula in 64 bits.

The kernel works in fp32 and rounds to bf16 once: half a step, 2^-8 of the value, and for the fp32 part some 32 roundings
(norm, angle, two products) of 2^-24 of the two numbers that turn."""
import numpy as np
import pytest
import torch

import paper_2503_23956_b200 as ac

DEV = "cuda:0"


def formula(x, weight, positions, inv_freq, sections, interleaved, eps, factor):
    """x [L, T, H, d]: result and what it may be off by."""
    x = x.double().cpu().numpy()
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight.double().cpu().numpy()[:, None, None]
    y, tol = x.copy(), np.abs(x)
    axis = [a for a, s in enumerate(sections) for _ in range(s)]
    n = len(axis)
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        angle = positions[axis[i]].double().cpu().numpy() * float(inv_freq[i])
        c, s = factor * np.cos(angle)[None, :, None], factor * np.sin(angle)[None, :, None]
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
        tol[..., a] = tol[..., b] = abs(factor) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return y, 2.0 ** -8 * np.abs(y) + 32 * 2.0 ** -24 * tol + 1e-38


def case(L, T, Hq, Hkv, d, R, sections, norm, seed=0, far=1 << 20):
    gen = torch.Generator().manual_seed(seed)
    qkv = torch.randn((L, T, Hq + 2 * Hkv, d), generator=gen).bfloat16().to(DEV)
    pos = torch.randint(-5, far, (len(sections), T), generator=gen, dtype=torch.int32).to(DEV)
    inv = (1e4 ** (-torch.arange(R // 2, dtype=torch.float64) / max(R // 2, 1))).float().to(DEV)
    w = [(1 + torch.randn((L, d), generator=gen)).bfloat16().to(DEV) if norm else None for _ in range(2)]
    return qkv, pos, inv, w


@pytest.mark.gpu
@pytest.mark.parametrize("L,T,Hq,Hkv,d,R,sections,interleaved,norm", [
    (1, 1, 1, 1, 64, 64, [32], 0, True),
    (2, 5, 7, 1, 128, 128, [16, 24, 24], 0, True),
    (3, 9, 8, 2, 64, 32, [16], 1, False),
    (1, 17, 28, 4, 128, 64, [8, 12, 12], 1, True),
    (1, 6000, 28, 4, 128, 128, [16, 24, 24], 0, True),   # a warp takes all heads of a token
    (2, 33, 3, 3, 64, 16, [0, 8, 0], 0, False),
    (1, 40, 0, 2, 128, 128, [64], 0, True),
    (1, 40, 5, 0, 128, 48, [24], 0, True),
    (1, 8, 4, 2, 64, 0, [], 0, True),                    # norms alone
])
def test_against_the_formula(L, T, Hq, Hkv, d, R, sections, interleaved, norm):
    qkv, pos, inv, (wq, wk) = case(L, T, Hq, Hkv, d, R, sections or [0], norm)
    q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
    n_rows = T + 5
    perm = torch.randperm(n_rows, generator=torch.Generator().manual_seed(4))[:T].to(DEV)
    cache = torch.full((2, L, n_rows, Hkv, d), 7.0, dtype=torch.bfloat16, device=DEV)
    out = torch.full((L, T, Hq, d), 7.0, dtype=torch.bfloat16, device=DEV)
    spec = ac.rotary(L, T, Hq, Hkv, d, R, interleaved, sections, eps=1e-5, factor=1.25)
    view = ac.tokens_view
    ac.aircache_rotate(spec, view(q) if Hq else None, view(k) if Hkv else None, view(v) if Hkv else None, pos if R else None,
                       inv if R else None, wq, wk, view(out) if Hq else None, view(cache[0]) if Hkv else None,
                       view(cache[1]) if Hkv else None, perm, n_rows)
    for x, w, got in ((q, wq, out), (k, wk, cache[0][:, perm])):
        want, tol = formula(x, w, pos, inv, sections, interleaved, 1e-5, 1.25)
        assert (np.abs(got.double().cpu().numpy() - want) <= tol).all()
    if Hkv:
        assert torch.equal(cache[1][:, perm], v)
        left = torch.ones(n_rows, dtype=torch.bool, device=DEV)
        left[perm] = False
        assert (cache[:, :, left] == 7).all()


@pytest.mark.gpu
def test_padding_rows_strides_and_in_place():
    """Rows of -1 and beyond the cache are left out; a head-major cache; queries in place."""
    L, T, Hq, Hkv, d = 1, 6, 4, 2, 64
    qkv, pos, inv, (wq, wk) = case(L, T, Hq, Hkv, d, d, [32], True)
    before = qkv.clone()
    q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
    k_c, v_c = (torch.full((L, Hkv, 9, d), 3.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    rows = torch.tensor([4, -1, 0, 9, 8, 1 << 40], device=DEV)
    spec = ac.rotary(L, T, Hq, Hkv, d, eps=1e-5)
    heads_last = lambda t: ac.tokens_view(t.transpose(1, 2))   # noqa: E731
    ac.aircache_rotate(spec, ac.tokens_view(q), ac.tokens_view(k), ac.tokens_view(v), pos, inv, wq, wk, ac.tokens_view(q),
                       heads_last(k_c), heads_last(v_c), rows, 9)
    want, tol = formula(before[:, :, :Hq], wq, pos, inv, [32], 0, 1e-5, 1.0)
    assert (np.abs(q.double().cpu().numpy() - want) <= tol).all()
    want, tol = formula(k, wk, pos, inv, [32], 0, 1e-5, 1.0)
    for t, row in ((0, 4), (2, 0), (4, 8)):
        assert (np.abs(k_c[0, :, row].double().cpu().numpy() - want[0, t]) <= tol[0, t]).all()
        assert torch.equal(v_c[0, :, row], v[0, t])
    for row in (1, 2, 3, 5, 6, 7):
        assert (k_c[0, :, row] == 3).all() and (v_c[0, :, row] == 3).all()
    assert torch.equal(k, before[:, :, Hq:Hq + Hkv])


@pytest.mark.gpu
def test_far_positions():
    """The largest 32-bit positions, where an angle in fp32 is off by whole turns."""
    T, d = 64, 128
    qkv, _, inv, _ = case(1, T, 2, 1, d, d, [64], False)
    pos = (torch.arange(T, dtype=torch.int64) * 33333333 + (1 << 30)).clamp_(max=(1 << 31) - 1).to(torch.int32)[None].to(DEV)
    out = torch.empty((1, T, 2, d), dtype=torch.bfloat16, device=DEV)
    ac.aircache_rotate(ac.rotary(1, T, 2, 0, d), ac.tokens_view(qkv[:, :, :2]), None, None, pos, inv, None, None,
                       ac.tokens_view(out), None, None, None, 0)
    want, tol = formula(qkv[:, :, :2], None, pos, inv, [64], 0, 1e-6, 1.0)
    assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()


def test_refusals():
    P = 0x10000000
    good = dict(n_layers=1, n_tokens=4, n_q_heads=4, n_kv_heads=2, head_dim=64)

    def call(over=None, q=None, k=None, v=None, q_out=None, k_out=None, pos=P, inv=P, wq=0, rows=0, n_rows=4):
        spec = ac.rotary(**{**good, **(over or {})})
        t = ac.Tokens(P, 0, 4 * 64, 64)
        c = ac.Tokens(P, 0, 2 * 64, 64)
        other = ac.Tokens(2 * P, 0, 4 * 64, 64)
        return ac.aircache_rotate(spec, q or t, k or c, v or c, pos, inv, wq or None, None, q_out or other, k_out or c, c,
                                  rows or None, n_rows, stream=1, check=False)

    bad = [
        (dict(over=dict(n_layers=0)), ac.ERR_INVALID_ARG), (dict(over=dict(n_tokens=-1)), ac.ERR_INVALID_ARG),
        (dict(over=dict(n_q_heads=0, n_kv_heads=0)), ac.ERR_INVALID_ARG), (dict(over=dict(head_dim=96)), ac.ERR_UNSUPPORTED),
        (dict(over=dict(rotary_dim=72)), ac.ERR_INVALID_ARG), (dict(over=dict(rotary_dim=24)), ac.ERR_UNSUPPORTED),
        (dict(over=dict(interleaved=2)), ac.ERR_INVALID_ARG), (dict(over=dict(sections=[16, 15])), ac.ERR_INVALID_ARG),
        (dict(over=dict(sections=[33, -1])), ac.ERR_INVALID_ARG), (dict(over=dict(eps=-1.0)), ac.ERR_INVALID_ARG),
        (dict(over=dict(eps=float("nan"))), ac.ERR_INVALID_ARG), (dict(over=dict(factor=float("inf"))), ac.ERR_INVALID_ARG),
        (dict(pos=None), ac.ERR_INVALID_ARG), (dict(inv=None), ac.ERR_INVALID_ARG), (dict(pos=P + 1), ac.ERR_ALIGNMENT),
        (dict(wq=P + 8), ac.ERR_ALIGNMENT), (dict(rows=P + 4), ac.ERR_ALIGNMENT), (dict(n_rows=-1), ac.ERR_INVALID_ARG),
        (dict(q=ac.Tokens(P + 8, 0, 256, 64)), ac.ERR_ALIGNMENT), (dict(k=ac.Tokens(P, 0, 132, 64)), ac.ERR_ALIGNMENT),
        (dict(v=ac.Tokens(P, 0, -128, 64)), ac.ERR_INVALID_ARG), (dict(q=ac.Tokens(0, 0, 256, 64)), ac.ERR_INVALID_ARG),
        (dict(q_out=ac.Tokens(2 * P, 0, 128, 64)), ac.ERR_INVALID_ARG),       # tokens over one another
        (dict(k_out=ac.Tokens(2 * P, 0, 64, 64)), ac.ERR_INVALID_ARG),
        (dict(q_out=ac.Tokens(P, 0, 512, 64)), ac.ERR_INVALID_ARG),           # in place with other strides
    ]
    for kw, code in bad:
        assert call(**kw) == code, kw
    assert call(over=dict(n_tokens=0)) == ac.OK   # nothing to do, nothing launched
