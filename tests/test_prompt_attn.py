"""aircache_prompt_attn against its formula in 64 bits.

Off by at most: half a step of bf16 in the output, 2^-8 of it; half a step of bf16 in every weight and 2^-18 for the
exponential and the sums, (2^-8 + 2^-18) sum_j p_j |v_j|; and what fp32 sums of exact products cost a logit, at most
128 * 2^-24 * scale * sum |q k|, twice.  Which keys a token sees is tested exactly (test_which_keys_a_token_sees)."""
import numpy as np
import pytest
import torch

import paper_2503_23956_b200 as ac
from paper_2503_23956_b200.session import Session

DEV = "cuda:0"


def formula(q, k, v, n_q, n_k, causal, scale):
    """Packed [T, H, d] on any device: output and what it may be off by, fp64."""
    out, tol = torch.zeros(q.shape, dtype=torch.float64, device=q.device), torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    G = q.shape[1] // k.shape[1]
    a = b = 0
    for nq, nk in zip(n_q, n_k):
        if nq and nk:
            kk, vv = (x[b:b + nk].double().repeat_interleave(G, dim=1).transpose(0, 1) for x in (k, v))   # [Hq, nk, d]
            qq = q[a:a + nq].double().transpose(0, 1)
            seen = torch.full((nq, 1), nk, device=q.device)
            if causal:
                seen = nk - nq + 1 + torch.arange(nq, device=q.device)[:, None]
            hidden = torch.arange(nk, device=q.device)[None] >= seen
            x = (scale * qq @ kk.transpose(1, 2)).masked_fill(hidden, -torch.inf)
            wide = (scale * qq.abs() @ kk.abs().transpose(1, 2)).masked_fill(hidden, 0).amax(-1, keepdim=True)
            p = torch.exp(x - x.amax(-1, keepdim=True).clamp_min(-1e300))
            p = p / p.sum(-1, keepdim=True).clamp_min(1e-300)
            o = p @ vv
            t = 2.0 ** -8 * o.abs() + (2.0 ** -8 + 2.0 ** -18 + 2 * 128 * 2.0 ** -24 * wide) * (p @ vv.abs())
            out[a:a + nq], tol[a:a + nq] = o.transpose(0, 1), t.transpose(0, 1)
        a, b = a + nq, b + nk
    return out, tol


def offsets(n):
    return torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=torch.int32, device=DEV)


def attend(q, k, v, n_q, n_k, causal=1, out=None, scale=None):
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV) if out is None else out
    spec = ac.prompt(len(n_q), q.shape[0], k.shape[0], q.shape[1], k.shape[1], q.shape[2], scale, causal)
    ac.aircache_prompt_attn(spec, ac.tokens_view(q), ac.tokens_view(k), ac.tokens_view(v), offsets(n_q), offsets(n_k),
                            ac.tokens_view(out))
    assert ac.aircache_prompt_check_status() == 0
    return out


def inputs(Tq, Tk, Hq, Hkv, d, seed=0, size=1.0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return [(size * torch.randn(s, generator=gen, device=DEV)).bfloat16() for s in ((Tq, Hq, d), (Tk, Hkv, d), (Tk, Hkv, d))]


def check(q, k, v, n_q, n_k, causal=1, out=None, scale=None):
    got = attend(q, k, v, n_q, n_k, causal, out, scale)
    want, tol = formula(q, k, v, n_q, n_k, causal, scale or 1 / np.sqrt(q.shape[2]))
    bad = ~((got.double() - want).abs() <= tol)
    bad[sum(n_q):] = False
    assert not bad.any(), (bad.nonzero()[:4].tolist(), (got.double() - want).abs().max().item())
    assert (got[sum(n_q):] == 7).all()   # rows behind the last sequence
    return got


HEADS = [(1, 1, 64), (2, 1, 128), (3, 1, 64), (8, 2, 64), (5, 1, 128), (6, 1, 64), (28, 4, 128), (16, 2, 128), (9, 1, 64),
         (20, 2, 64), (11, 1, 128), (13, 1, 64), (30, 2, 128), (16, 1, 64), (32, 8, 64)]


@pytest.mark.gpu
@pytest.mark.parametrize("Hq,Hkv,d", HEADS)
@pytest.mark.parametrize("causal", [1, 0])
def test_lengths(Hq, Hkv, d, causal):
    n_q = [1, 17, 0, 128, 129, 300, 36, 255]
    n_k = [1, 17, 5, 128, 129, 300, 500, 256]
    q, k, v = inputs(sum(n_q) + 3, sum(n_k) + 2, Hq, Hkv, d, seed=Hq)
    check(q, k, v, n_q, n_k, causal)


@pytest.mark.gpu
@pytest.mark.parametrize("Hq,Hkv,d", [(7, 1, 128), (8, 2, 64), (1, 1, 128)])
def test_long_and_sharp(Hq, Hkv, d):
    """Long enough for the ring to go round often; logits hundreds apart, growing and falling along the keys."""
    n = [2500, 700]
    q, k, v = inputs(sum(n), sum(n), Hq, Hkv, d, seed=3)
    check(q, k, v, n, n)
    ramp = torch.linspace(-1, 1, 2500, device=DEV)[:, None, None]
    k[:2500] += (6 * ramp * torch.ones(d, device=DEV) / np.sqrt(d)).bfloat16()
    q[:2500] += 20
    check(q, k, v, n, n)
    k[:2500] -= (12 * ramp * torch.ones(d, device=DEV) / np.sqrt(d)).bfloat16()
    check(q, k, v, n, n)


@pytest.mark.gpu
@pytest.mark.parametrize("Hq,Hkv,d", [(1, 1, 64), (7, 1, 128), (12, 2, 64), (16, 1, 128)])
@pytest.mark.parametrize("n_q,n_k,causal", [([400, 333], [400, 333], 1), ([1, 40, 7], [700, 1000, 7], 1),
                                            ([200, 50], [120, 1], 1), ([37, 130], [129, 600], 0)])
def test_which_keys_a_token_sees(Hq, Hkv, d, n_q, n_k, causal):
    """Queries of zero weigh all visible keys alike; value row j is one in channel j mod d: a channel counts its keys."""
    q = torch.zeros((sum(n_q), Hq, d), dtype=torch.bfloat16, device=DEV)
    k = inputs(1, sum(n_k), Hq, Hkv, d)[1]
    within = torch.cat([torch.arange(n) for n in n_k]).to(DEV)
    v = torch.nn.functional.one_hot(within % d, d).bfloat16()[:, None].expand(-1, Hkv, -1).contiguous()
    got = attend(q, k, v, n_q, n_k, causal).double()
    at = 0
    for a, b in zip(n_q, n_k):
        seen = (b - a + 1 + torch.arange(a, device=DEV)).clamp(min=0) if causal else torch.full((a,), b, device=DEV)
        want = (seen[:, None] - torch.arange(d, device=DEV)[None] + d - 1).div(d, rounding_mode="floor")   # keys of channel c
        count = got[at:at + a] * seen[:, None, None]
        assert torch.equal(count.round(), want[:, None].expand(-1, Hq, -1).double())
        assert (count - count.round()).abs().max() < 0.25
        at += a


@pytest.mark.gpu
@pytest.mark.parametrize("Hq,Hkv,d", [(32, 32, 64), (64, 32, 128)])
@pytest.mark.parametrize("causal", [1, 0])
def test_calls_of_many_blocks(Hq, Hkv, d, causal):
    """So many that a block takes two row tiles, not one whose keys its halves share."""
    n_q, n_k = [700, 1, 129, 300, 257, 640, 33, 128, 450, 90], [700, 900, 129, 500, 257, 640, 33, 60, 450, 1000]
    check(*inputs(sum(n_q) + 3, sum(n_k), Hq, Hkv, d, seed=6), n_q, n_k, causal)
    test_which_keys_a_token_sees(Hq, Hkv, d, n_q, n_k, causal)


@pytest.mark.gpu
def test_tokens_that_see_nothing():
    q, k, v = inputs(100, 40, 7, 1, 128)
    out = attend(q, k, v, [100], [40])
    assert (out[:60] == 0).all() and (out[60:] != 0).any()
    out = attend(q, k[:0], v[:0], [100], [0])
    assert (out == 0).all()
    out = attend(q, k, v, [60, 40], [0, 40])
    assert (out[:60] == 0).all()


@pytest.mark.gpu
def test_nan_elsewhere_reaches_nothing():
    n = [70, 130, 65]
    q, k, v = inputs(sum(n) + 200, sum(n) + 200, 8, 2, 64, seed=5)
    nan = float("nan")
    k[sum(n):], v[sum(n):], q[sum(n):] = nan, nan, nan
    check(q, k, v, n, n)
    clean = attend(q, k, v, n, n)
    q[70:200], k[70:200], v[70:200] = nan, nan, float("inf")   # the second sequence
    got = attend(q, k, v, n, n)
    assert torch.equal(got[:70], clean[:70]) and torch.equal(got[200:265], clean[200:265])
    assert got[70:200].isnan().all()
    assert (got[265:] == 7).all()


@pytest.mark.gpu
def test_strides():
    """Parts of a fused projection, a layer of a cache, head-major buffers, heads of the output apart."""
    n = [50, 200, 33]
    T, Hq, Hkv, d = sum(n), 14, 2, 128
    gen = torch.Generator(device=DEV).manual_seed(8)
    qkv = torch.randn((T, Hq + 2 * Hkv, d), generator=gen, device=DEV).bfloat16()
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    plain = check(q, k, v, n, n)
    major = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v)]
    assert torch.equal(attend(*major, n, n), plain)
    wide = torch.full((T, Hq, 2 * d), 3.0, dtype=torch.bfloat16, device=DEV)
    attend(q, k, v, n, n, out=wide[:, :, d:])
    assert torch.equal(wide[:, :, d:], plain) and (wide[:, :, :d] == 3).all()
    one = [k[:, :1].expand(-1, Hkv, -1), v[:, :1].expand(-1, Hkv, -1)]   # heads that are one and the same
    assert torch.equal(attend(q, *one, n, n), attend(q, one[0].contiguous(), one[1].contiguous(), n, n))


@pytest.mark.gpu
def test_many_sequences_and_single_tokens():
    n_k = [(7 * i) % 90 + 1 for i in range(1024)]
    q, k, v = inputs(1024, sum(n_k), 14, 2, 64, seed=2)
    check(q, k, v, [1] * 1024, n_k)


@pytest.mark.gpu
def test_offsets_outside_the_buffers_are_clamped():
    q, k, v = inputs(64, 64, 4, 1, 64)
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    spec = ac.prompt(3, 64, 64, 4, 1, 64)
    for off in ([-5, 20, 10, 1 << 30], [100, -3, 50, 64], [0, 1 << 31 - 1, 5, 3]):
        o = torch.tensor(off, dtype=torch.int64, device=DEV).to(torch.int32)
        ac.aircache_prompt_attn(spec, ac.tokens_view(q), ac.tokens_view(k), ac.tokens_view(v), o, None, ac.tokens_view(out))
        assert ac.aircache_prompt_check_status() == 0


@pytest.mark.gpu
def test_captured_two_streams_and_same_bits():
    n = [300, 45]
    a, b = inputs(345, 345, 28, 4, 128, seed=1), inputs(345, 345, 28, 4, 128, seed=2)
    want = [attend(*x, n, n) for x in (a, b)]
    assert torch.equal(attend(*a, n, n), want[0])
    off, outs = offsets(n), [torch.zeros_like(x[0]) for x in (a, b)]
    spec = ac.prompt(2, 345, 345, 28, 4, 128)
    views = [[ac.tokens_view(t) for t in x] + [off, None, ac.tokens_view(o)] for x, o in zip((a, b), outs)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ac.aircache_prompt_attn(spec, *views[0])
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        with torch.cuda.stream(streams[0]):
            graph.replay()
        ac.aircache_prompt_attn(spec, *views[1], stream=streams[1])
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])


@pytest.mark.gpu
def test_beside_the_scores_of_another_stream():
    """The scoring kernel has tensor memory and clusters of its own; calls of both on two streams leave each other alone."""
    L, B, Hq, Hkv, d, Nv, Nt = 4, 2, 28, 4, 128, 2000, 64
    gen = torch.Generator(device=DEV).manual_seed(3)
    s = Session(ac.shape(L, B, Hq, Hkv, d, Nv, Nt, 16), 0.2, device=DEV)
    k = torch.randn((L, B, Nv + Nt, Hkv, d), generator=gen, device=DEV).bfloat16()
    s.set_full(k.permute(0, 1, 3, 2, 4), k.permute(0, 1, 3, 2, 4))
    qw = torch.randn((L, B, 16, Hq, d), generator=gen, device=DEV).bfloat16()
    s.score(qw)
    scores = s.scores.clone()
    n = [900, 300, 41]
    x = inputs(sum(n), sum(n), Hq, Hkv, d, seed=4)
    want = attend(*x, n, n)
    out, off = torch.zeros_like(want), offsets(n)
    spec, views = ac.prompt(3, sum(n), sum(n), Hq, Hkv, d), [ac.tokens_view(t) for t in x]
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(30):
        ac.aircache_prompt_attn(spec, *views, off, None, ac.tokens_view(out), stream=a)
        s.score(qw, stream=b)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(s.scores, scores)
    assert s.status() == 0 and ac.aircache_prompt_check_status() == 0


@pytest.mark.gpu
def test_from_the_projection_to_decoding():
    """A layer after the other as an engine runs them: rotation into the cache, attention over it, scores, then the
    compression, 8 bits, and a token.  Two sequences of 300 visual and 20 text tokens."""
    L, B, Hq, Hkv, d, Nv, Nt, W = 2, 2, 14, 2, 128, 300, 20, 8
    N = Nv + Nt
    gen = torch.Generator(device=DEV).manual_seed(1)
    s = Session(ac.shape(L, B, Hq, Hkv, d, Nv, Nt, W, 3), 0.2, device=DEV)
    k, v = (torch.zeros((L, B, N, Hkv, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    s.set_full(k.permute(0, 1, 3, 2, 4), v.permute(0, 1, 3, 2, 4))
    inv = (1e4 ** (-torch.arange(d // 2, dtype=torch.float64) / (d // 2))).float().to(DEV)
    pos = torch.arange(N, dtype=torch.int32, device=DEV).repeat(B)[None]
    off = offsets([N] * B)
    w = torch.ones((1, d), dtype=torch.bfloat16, device=DEV)
    qw = torch.empty((L, B, W, Hq, d), dtype=torch.bfloat16, device=DEV)
    for l in range(L):
        qkv = torch.randn((B * N, Hq + 2 * Hkv, d), generator=gen, device=DEV).bfloat16()
        q, out = (torch.empty((B * N, Hq, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        kc, vc = k[l].view(B * N, Hkv, d), v[l].view(B * N, Hkv, d)
        view = ac.tokens_view
        ac.aircache_rotate(ac.rotary(1, B * N, Hq, Hkv, d), view(qkv[:, :Hq]), view(qkv[:, Hq:Hq + Hkv]),
                           view(qkv[:, Hq + Hkv:]), pos, inv, w, w, view(q), view(kc), view(vc), None, B * N)
        ac.aircache_prompt_attn(ac.prompt(B, B * N, B * N, Hq, Hkv, d), view(q), view(kc), view(vc), off, None, view(out))
        want, tol = formula(q, kc, vc, [N] * B, [N] * B, 1, 1 / np.sqrt(d))
        assert ((out.double() - want).abs() <= tol).all()
        qw[l] = q.view(B, N, Hq, d)[:, -W:]
    s.score(qw)
    s.budget()
    s.compact()
    s.quantize()
    new = torch.randn((L, B, Hkv, d), generator=gen, device=DEV).bfloat16()
    s.append_quantized(new, new, 0)
    qn = torch.randn((L, B, Hq, d), generator=gen, device=DEV).bfloat16()
    s.decode_quantized(qn)
    assert s.status() == 0 and ac.aircache_prompt_check_status() == 0
    # the last row of every region is the new token: with its own scale it is held to 2^-4
    for r in range(L * B):
        o, n = int(s.offsets[r]), int(s.lens[r])
        b = o // 64 + r
        codes = s.k8[o:o + n].view(torch.float8_e4m3fn).double()
        scale = s.k_scale[b + torch.arange(n, device=DEV) // 64].double()[..., None]
        vals = s.v8[o:o + n].view(torch.float8_e4m3fn).double() * s.v_scale[b + torch.arange(n, device=DEV) // 64].double()[..., None]
        want, _ = formula(qn[r // B, r % B][None], (codes * scale), vals, [1], [n], 1, 1 / np.sqrt(d))
        assert ((s.out[r // B, r % B].double() - want[0]).norm() / want.norm()).item() < 1e-5
        assert (((codes * scale)[-1] - new[r // B, r % B].double()).norm() / new[r // B, r % B].double().norm()).item() < 2.0 ** -4


def test_refusals():
    P = 0x10000000
    good = dict(n_seqs=2, q_tokens=50, k_tokens=50, n_q_heads=8, n_kv_heads=2, head_dim=64)

    def call(over=None, q=None, k=None, out=None, qo=P, ko=P):
        t, o = ac.Tokens(P, 0, 8 * 64, 64), ac.Tokens(2 * P, 0, 8 * 64, 64)
        return ac.aircache_prompt_attn(ac.prompt(**{**good, **(over or {})}), q or t, k or t, t, qo, ko, out or o, stream=1,
                                       check=False)

    bad = [
        (dict(over=dict(n_seqs=-1)), ac.ERR_INVALID_ARG), (dict(over=dict(n_seqs=1025)), ac.ERR_UNSUPPORTED),
        (dict(over=dict(q_tokens=-1)), ac.ERR_INVALID_ARG), (dict(over=dict(head_dim=96)), ac.ERR_UNSUPPORTED),
        (dict(over=dict(n_q_heads=7)), ac.ERR_INVALID_ARG), (dict(over=dict(n_q_heads=34)), ac.ERR_UNSUPPORTED),
        (dict(over=dict(n_kv_heads=0)), ac.ERR_INVALID_ARG), (dict(over=dict(causal=2)), ac.ERR_INVALID_ARG),
        (dict(over=dict(scale=0.0)), ac.ERR_INVALID_ARG), (dict(over=dict(scale=float("nan"))), ac.ERR_INVALID_ARG),
        (dict(qo=None), ac.ERR_INVALID_ARG), (dict(qo=P + 2), ac.ERR_ALIGNMENT), (dict(ko=P + 1), ac.ERR_ALIGNMENT),
        (dict(ko=None, over=dict(k_tokens=60)), ac.ERR_INVALID_ARG),
        (dict(q=ac.Tokens(P + 8, 0, 512, 64)), ac.ERR_ALIGNMENT), (dict(k=ac.Tokens(P, 0, 512, 68)), ac.ERR_ALIGNMENT),
        (dict(k=ac.Tokens(0, 0, 512, 64)), ac.ERR_INVALID_ARG), (dict(out=ac.Tokens(P, 0, 256, 64)), ac.ERR_INVALID_ARG),
        (dict(out=ac.Tokens(P, 0, 512, -64)), ac.ERR_INVALID_ARG),
    ]
    for kw, code in bad:
        assert call(**kw) == code, kw
    assert call(over=dict(n_seqs=0)) == ac.OK and call(over=dict(q_tokens=0)) == ac.OK
