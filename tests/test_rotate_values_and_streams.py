"""aircache_rotate: infinities and NaN stay where the formula has them, and the call in a capture and on two streams."""
import numpy as np
import pytest
import torch

import paper_2503_23956_b200 as ac
from test_rotate import DEV, case, formula


def rotate(spec, q, k, v, pos, inv, w, q_out, k_out, v_out, n_rows, stream=None):
    view = ac.tokens_view
    ac.aircache_rotate(spec, view(q), view(k), view(v), pos, inv, w[0], w[1], view(q_out), view(k_out), view(v_out), None, n_rows,
                       stream)


def buffers(L, T, Hq, Hkv, d):
    return [torch.full((L, T, H, d), 7.0, dtype=torch.bfloat16, device=DEV) for H in (Hq, Hkv, Hkv)]


def agree(got, want, tol):
    got = got.double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        near = np.abs(got - want) <= tol
    return (near | (got == want) | (np.isnan(got) & np.isnan(want))).all()


@pytest.mark.gpu
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("d,R,interleaved", [(64, 64, 0), (128, 64, 0), (128, 64, 1), (64, 32, 1)])
def test_infinities_and_nan(d, R, interleaved, norm):
    """A head's own, with norm (all of its channels) and without (the pair); other heads and tokens, and values, as they are."""
    L, T, Hq, Hkv = 1, 9, 6, 2
    qkv, pos, inv, w = case(L, T, Hq, Hkv, d, R, [R // 2], norm, seed=3)
    pos[0, 4] = 0   # sine of zero: infinity times it is NaN
    for t, h, c, x in ((0, 0, 0, "inf"), (1, 1, R - 1, "-inf"), (2, 2, 5, "nan"), (3, Hq, d - 1, "inf"), (4, Hq + 1, 1, "inf"),
                       (5, 3, d - 1, "nan"), (6, Hq + Hkv, 2, "nan"), (7, Hq + Hkv + 1, 3, "-inf")):
        qkv[0, t, h, c] = float(x)
    q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
    q_out, k_out, v_out = buffers(L, T, Hq, Hkv, d)
    rotate(ac.rotary(L, T, Hq, Hkv, d, R, interleaved, eps=1e-5), q, k, v, pos, inv, w, q_out, k_out, v_out, T)
    with np.errstate(invalid="ignore"):
        for x, weight, got in ((q, w[0], q_out), (k, w[1], k_out)):
            want, tol = formula(x, weight, pos, inv, [R // 2], interleaved, 1e-5, 1.0)
            assert agree(got, want, tol)
            assert np.isnan(want).any() and not np.isnan(want).all()
    assert torch.equal(v_out.view(torch.int16), v.contiguous().view(torch.int16))


@pytest.mark.gpu
def test_captured_and_on_two_streams():
    L, T, Hq, Hkv, d = 2, 33, 8, 2, 64
    a, b = (case(L, T, Hq, Hkv, d, d, [32], True, seed=s) for s in (1, 2))
    spec = ac.rotary(L, T, Hq, Hkv, d, eps=1e-5)
    parts = [(x[0][:, :, :Hq], x[0][:, :, Hq:Hq + Hkv], x[0][:, :, Hq + Hkv:]) for x in (a, b)]
    outs = [buffers(L, T, Hq, Hkv, d) for _ in (a, b)]
    want = []
    for x, part, out in zip((a, b), parts, outs):
        rotate(spec, *part, x[1], x[2], x[3], *out, T)
        want.append([o.clone() for o in out])
        for o in out:
            o.fill_(7)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rotate(spec, *parts[0], a[1], a[2], a[3], *outs[0], T)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(streams[0]):
            graph.replay()
        rotate(spec, *parts[1], b[1], b[2], b[3], *outs[1], T, stream=streams[1])
    torch.cuda.synchronize()
    for got, expected in zip(outs, want):
        assert all(torch.equal(x, y) for x, y in zip(got, expected))
    # new inputs in the same places
    a[0].copy_(b[0]), a[1].copy_(b[1]), a[3][0].copy_(b[3][0]), a[3][1].copy_(b[3][1])
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(outs[0], want[1]))
