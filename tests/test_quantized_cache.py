"""The ragged cache of 8 bits: aircache_quantize, aircache_append_quantized, aircache_decode_attn_quantized against their
definitions in 64 bits.

Scales and codes are compared with `==`: a power-of-two scale makes x / s exact, so the nearest e4m3 number is decided by
the definition alone.  Attention: the products of fp16 numbers are exact in fp32 and are summed there, which costs a
logit at most n * 2^-24 * sum |q k| with n = 128 terms and half as much in practice; one ex2.approx and one sum of weights
2^-22 and n * 2^-24.  So a value of the output is off by at most (2 * dlogit + 2^-18) * sum_j p_j |v_j|, and by what the
16-bit weights cannot hold: weight times 2^11 times its block's V scale s_j over the largest, S, is a sum of two fp16 numbers, the
second to within half of the smallest one, 2^-25.  That is 2^-36 S / s_j of a weight, for a value of |code_j| s_j:
2^-36 S sum_j |code_j| (it shows where the key that has nearly all of the weight holds a zero)."""
import numpy as np
import pytest
import torch

import paper_2503_23956_b200 as ac
from paper_2503_23956_b200.session import Session

DEV = "cuda:0"
BLOCK = 64


# ---------------------------------------------------------------------------------------------
# the definitions, on the CPU in 64 bits
# ---------------------------------------------------------------------------------------------
def e4m3_table():
    codes = np.arange(256)
    sign, e, m = codes >> 7, codes >> 3 & 15, codes & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v = np.where(sign == 1, -v, v)
    v[[0x7f, 0xff]] = np.nan
    return v


TABLE = e4m3_table()
POSITIVE = TABLE[:0x7f]   # ascending


def codes_of(y):
    """Nearest e4m3 code (ties to the even one), saturated; NaN is 0x7f."""
    y = np.asarray(y, dtype=np.float64)
    a = np.minimum(np.abs(y), 448.0)
    a = np.where(np.isnan(y), 0.0, a)
    hi = np.searchsorted(POSITIVE, a).clip(1, len(POSITIVE) - 1)
    lo = hi - 1
    d_lo, d_hi = a - POSITIVE[lo], POSITIVE[hi] - a
    c = np.where(d_lo < d_hi, lo, np.where(d_hi < d_lo, hi, np.where(lo % 2 == 0, lo, hi)))
    c = c | np.where(np.signbit(y), 0x80, 0)
    return np.where(np.isnan(y), 0x7f, c).astype(np.uint8)


def scale_of(x):
    x = np.abs(np.asarray(x, dtype=np.float64))
    top = x[np.isfinite(x)].max(initial=0.0)
    e = -126
    while top > 448 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def quantized(x, offsets, lens, blocks, codes, scale, first_region=0):
    """x [rows, H, d] -> codes and scales, in place."""
    for r, n in enumerate(lens):
        o = int(offsets[r])
        for j in range(0, int(n), BLOCK):
            rows = slice(o + j, o + min(int(n), j + BLOCK))
            for h in range(x.shape[1]):
                s = scale_of(x[rows, h])
                scale[o // BLOCK + first_region + r + j // BLOCK, h] = s
                codes[rows, h] = codes_of(x[rows, h] / s)


def appended(new, offsets, lens, codes, scale, first_region=0):
    """new [regions, H, d] into the first free rows; lens is not changed."""
    for r, n in enumerate(lens):
        o, n = int(offsets[r]), int(n)
        b, first = o // BLOCK + first_region + r + n // BLOCK, o + n - n % BLOCK
        for h in range(new.shape[1]):
            s = scale_of(new[r, h])
            if n % BLOCK:
                held = TABLE[codes[first:o + n, h]] * float(scale[b, h])
                s = max(s, float(scale[b, h]))
                codes[first:o + n, h] = codes_of(held / s)
            scale[b, h] = s
            codes[o + n, h] = codes_of(new[r, h] / s)


def attention(q, k, v, sm_scale, held):
    """q [G, d], k and v [n, d]: output, and what it may be off by.  held [d]: 2^-36 S sum_j |code_j|."""
    if len(k) == 0:
        return np.zeros_like(q), np.zeros_like(q)
    x = sm_scale * (q @ k.T)
    d_logit = (sm_scale * (np.abs(q) @ np.abs(k).T)).max() * 128 * 2.0 ** -24
    p = np.exp(x - x.max(axis=1, keepdims=True))
    p /= p.sum(axis=1, keepdims=True)
    return p @ v, (2 * d_logit + 2.0 ** -18) * (p @ np.abs(v)) + held


# ---------------------------------------------------------------------------------------------
# a cache with regions of given lengths
# ---------------------------------------------------------------------------------------------
class Cache:
    """Regions of given lengths, `slack` free rows behind each; guard rows and blocks behind the buffers."""

    def __init__(self, lens, H, d, Hq=None, slack=0, per_kv_head=0, Hkv=None, seed=0, first_region=0, first_row=0):
        self.lens0, self.H, self.d = list(lens), H, d
        Hkv = H if Hkv is None else Hkv
        cells = Hkv if per_kv_head else 1
        assert len(lens) % cells == 0
        self.R = len(lens)
        self.sh = ac.shape(len(lens) // cells, 1, Hq or Hkv, Hkv, d, 3, 1, 1, slack, per_kv_head=per_kv_head)
        offs = first_row + np.concatenate([[0], np.cumsum([n + slack for n in lens])])
        self.rows = int(offs[-1]) + 1
        self.first_region = first_region
        self.blocks = ac.aircache_scale_blocks(self.sh, self.rows, first_region)
        self.offs = offs
        self.offsets = torch.tensor(offs, dtype=torch.int64, device=DEV)
        self.lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
        gen = torch.Generator().manual_seed(seed)
        shape = (self.rows, H, d)
        self.k = (torch.randn(shape, generator=gen) * torch.exp(torch.randn((H, d), generator=gen))).bfloat16().to(DEV)
        self.v = torch.randn(shape, generator=gen).bfloat16().to(DEV)
        self.k8 = torch.full(shape, 0x55, dtype=torch.uint8, device=DEV)
        self.v8 = torch.full(shape, 0x2a, dtype=torch.uint8, device=DEV)
        self.k_scale = torch.full((self.blocks, H), 7.0, device=DEV)
        self.v_scale = torch.full((self.blocks, H), 5.0, device=DEV)
        self.ragged = ac.ragged_view(self.k, self.v, self.offsets, self.lens, self.rows)
        self.cache8 = ac.quantized_view(self.k8, self.v8, self.k_scale, self.v_scale, self.offsets, self.lens, self.rows,
                                        first_region)
        self.ws = torch.empty(ac.aircache_workspace_bytes(self.sh), dtype=torch.uint8, device=DEV)
        ac.aircache_reset_status(self.ws)

    def expected(self):
        out = {}
        for x, c, s in (("k", "k8", "k_scale"), ("v", "v8", "v_scale")):
            codes, scale = getattr(self, c).cpu().numpy().copy(), getattr(self, s).cpu().numpy().copy()
            quantized(getattr(self, x).double().cpu().numpy(), self.offs, self.lens0, self.blocks, codes, scale,
                      self.first_region)
            out[c], out[s] = codes, scale
        return out

    def check(self, want):
        for name, w in want.items():
            assert np.array_equal(getattr(self, name).cpu().numpy(), w), name

    def values(self, want, lens):
        """[region][K or V] of the elements' values, and what the weights cannot hold of V."""
        got = []
        for r, n in enumerate(lens):
            o, n = int(self.offs[r]), int(n)
            b = o // BLOCK + self.first_region + r + np.arange(n) // BLOCK
            got.append([TABLE[want[c][o:o + n]] * want[s][b][..., None].astype(np.float64)
                        for c, s in (("k8", "k_scale"), ("v8", "v_scale"))])
            largest = want["v_scale"][b].max(axis=0, initial=0).astype(np.float64)   # of every head
            got[-1].append(2.0 ** -36 * largest[:, None] * np.abs(TABLE[want["v8"][o:o + n]]).sum(axis=0))
        return got

    def check_attention(self, q, out, want, lens):
        """q and out [regions, H * G, d]."""
        q, out = q.double().cpu().numpy(), out.double().cpu().numpy()
        G = q.shape[1] // self.H
        for r, (k, v, held) in enumerate(self.values(want, lens)):
            for h in range(self.H):
                ref, tol = attention(q[r, h * G:(h + 1) * G], k[:, h], v[:, h], self.sh.scale, held[h])
                assert (np.abs(out[r, h * G:(h + 1) * G] - ref) <= tol).all(), (r, h, np.abs(out[r, h * G:(h + 1) * G] - ref).max())


def queries(c, G, seed=1):
    gen = torch.Generator().manual_seed(seed)
    return torch.randn((c.R, c.H * G, c.d), generator=gen).bfloat16().to(DEV)


# ---------------------------------------------------------------------------------------------
# the definitions themselves, and refusals (no GPU)
# ---------------------------------------------------------------------------------------------
def test_the_table_is_the_type():
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(codes, TABLE, equal_nan=True)
    x = torch.randn(20000, dtype=torch.float64) * 100
    x = torch.cat([x, x / 4096, torch.tensor(POSITIVE), torch.tensor((POSITIVE[1:] + POSITIVE[:-1]) / 2)])
    x = x.clamp(-448, 448)
    assert np.array_equal(codes_of(x.numpy()), x.float().to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_scale_is_the_smallest_power_of_two():
    assert scale_of([448.0]) == 1 and scale_of([449.0]) == 2 and scale_of([224.0]) == 0.5 and scale_of([0.0]) == 2.0 ** -126
    assert scale_of([np.inf, 3.5, np.nan]) == 2.0 ** -7


def _fake(total=1000, blocks=None, first_region=0, **kw):
    P = 0x10000000
    f = dict(k=P, v=P, k_scale=P, v_scale=P, offsets=P, lens=P)
    f.update(kw)
    blocks = total // 64 + first_region + 2 if blocks is None else blocks
    return ac.quantized_view(f["k"], f["v"], f["k_scale"], f["v_scale"], f["offsets"], f["lens"], total, first_region, blocks)


def test_refusals():
    sh = ac.shape(2, 1, 8, 2, 64, 10, 4, 4, 3)
    P = 0x10000000
    rag = ac.ragged_view(P, P, P, P, 1000)
    assert ac.aircache_scale_blocks(sh, 1000) == 1000 // 64 + 2
    assert ac.aircache_scale_blocks(sh, 64, 5) == 1 + 5 + 2
    assert ac.aircache_scale_blocks(sh, -1) == ac.ERR_INVALID_ARG
    assert ac.aircache_scale_blocks(sh, 1 << 31) == ac.ERR_CAPACITY
    assert ac.aircache_scale_blocks(ac.shape(2, 1, 8, 2, 96, 10, 4, 4), 10) == ac.ERR_UNSUPPORTED
    bad = [(_fake(k=0), ac.ERR_INVALID_ARG), (_fake(v_scale=0), ac.ERR_INVALID_ARG), (_fake(lens=0), ac.ERR_INVALID_ARG),
           (_fake(k=P + 8), ac.ERR_ALIGNMENT), (_fake(k_scale=P + 2), ac.ERR_ALIGNMENT), (_fake(offsets=P + 4), ac.ERR_ALIGNMENT),
           (_fake(total=0, blocks=99), ac.ERR_CAPACITY), (_fake(total=1 << 31, blocks=1 << 40), ac.ERR_CAPACITY),
           (_fake(blocks=16), ac.ERR_CAPACITY), (_fake(first_region=-1), ac.ERR_INVALID_ARG)]
    need = ac.aircache_workspace_bytes(sh)
    lib = ac.lib()
    import ctypes as C
    for c, code in bad:
        assert ac.aircache_quantize(sh, rag, c, stream=1, check=False) == code
        assert ac.aircache_append_quantized(sh, c, P, P, 0, stream=1, check=False) == code
        assert lib.aircache_decode_attn_quantized(C.byref(sh), C.byref(c), P, P, P, need, 1) == code
    good = _fake()
    assert ac.aircache_quantize(sh, rag, _fake(offsets=P + 64), stream=1, check=False) == ac.ERR_INVALID_ARG
    assert ac.aircache_quantize(sh, rag, _fake(lens=P + 64), stream=1, check=False) == ac.ERR_INVALID_ARG
    assert ac.aircache_quantize(sh, ac.ragged_view(P + 64, P, P, P, 1000), good, stream=1, check=False) == ac.ERR_ALIGNMENT
    assert ac.aircache_append_quantized(sh, good, P, 0, 0, stream=1, check=False) == ac.ERR_INVALID_ARG
    assert ac.aircache_append_quantized(sh, good, P, P, -1, stream=1, check=False) == ac.ERR_INVALID_ARG
    assert ac.aircache_append_quantized(sh, good, P, P, 3, stream=1, check=False) == ac.ERR_CAPACITY
    assert ac.aircache_append_quantized(sh, good, P + 2, P, 0, stream=1, check=False) == ac.ERR_ALIGNMENT
    assert lib.aircache_decode_attn_quantized(C.byref(sh), C.byref(good), 0, P, P, need, 1) == ac.ERR_INVALID_ARG
    assert lib.aircache_decode_attn_quantized(C.byref(sh), C.byref(good), P, P + 4, P, need, 1) == ac.ERR_ALIGNMENT
    assert lib.aircache_decode_attn_quantized(C.byref(sh), C.byref(good), P, P, P, need - 1, 1) == ac.ERR_WORKSPACE_TOO_SMALL
    assert lib.aircache_decode_attn_quantized(C.byref(sh), C.byref(good), P, P, P + 16, need, 1) == ac.ERR_ALIGNMENT
    with pytest.raises(ac.AirCacheError):
        ac.aircache_append_quantized(sh, good, P, P, 3, stream=1)


# ---------------------------------------------------------------------------------------------
# on the GPU
# ---------------------------------------------------------------------------------------------
LENGTHS = {
    "one": [1],
    "edges": [0, 1, 15, 16, 17, 63, 64, 65, 0, 127, 128, 129, 300],
    "long": [5000, 3],
    "many": [(7 * i) % 50 for i in range(200)],
    "lanes": [(37 * i) % 90 + (4000 if i == 41 else 0) for i in range(100)],   # more than a warp's lanes, one far longer
    "most": [(5 * i) % 40 for i in range(1792)],   # as many regions as a shape may have
}


@pytest.mark.gpu
@pytest.mark.parametrize("H,d", [(1, 64), (1, 128), (2, 128), (4, 64), (8, 128)])
@pytest.mark.parametrize("lens", ["one", "edges", "many", "most"])
def test_quantize(lens, H, d):
    c = Cache(LENGTHS[lens], H, d, slack=2, seed=H)
    want = c.expected()
    ac.aircache_quantize(c.sh, c.ragged, c.cache8)
    c.check(want)   # slack rows, guard rows and the scales of blocks without rows among them


@pytest.mark.gpu
def test_quantize_values_at_the_edges_of_the_type():
    c = Cache([64, 64, 130, 5], 2, 64)
    c.k[:64] = 0                                     # a block of zeros
    c.k[64:128, 0] = 448 * 2.0 ** 100
    c.k[70, 0, 3] = 1e-30                            # far below the block's scale
    c.k[128:192, 1] = float("inf")                   # nothing finite
    c.k[200, 0, 5], c.k[201, 0, 6], c.k[202, 0, 7] = float("nan"), float("-inf"), float("inf")
    c.v[:] = torch.tensor(POSITIVE, dtype=torch.float32)[torch.randint(0, 127, c.v.shape)].bfloat16().to(DEV)   # and ties between
    c.v[::3] *= 1.0625
    c.v[64:128] = 2.0 ** -133                        # subnormal bf16
    want = c.expected()
    ac.aircache_quantize(c.sh, c.ragged, c.cache8)
    c.check(want)


@pytest.mark.gpu
def test_quantize_leaves_out_regions_that_do_not_fit():
    c = Cache([40, 40, 40], 2, 64, slack=8)
    c.lens[1] = 49                                   # more than the region has
    c.offsets[3] += 100                              # behind the buffer
    before = {x: getattr(c, x).clone() for x in ("k8", "v8", "k_scale", "v_scale")}
    ac.aircache_quantize(c.sh, c.ragged, c.cache8)
    torch.cuda.synchronize()
    assert not torch.equal(c.k8[:40], before["k8"][:40])
    assert torch.equal(c.k8[40:], before["k8"][40:]) and torch.equal(c.v_scale[1:], before["v_scale"][1:])
    q, out = queries(c, 2), torch.full((3, 4, 64), 9.0, device=DEV)
    sh = ac.shape(3, 1, 4, 2, 64, 3, 1, 1, 8)
    ws = torch.zeros(ac.aircache_workspace_bytes(sh), dtype=torch.uint8, device=DEV)
    ac.aircache_decode_attn_quantized(sh, c.cache8, q, out, ws)
    assert (out[0] != 0).any() and (out[1:] == 0).all()
    ac.aircache_append_quantized(sh, c.cache8, q[:, :2].contiguous(), q[:, 2:].contiguous(), 0)
    assert c.lens.tolist()[:2] == [41, 49]


@pytest.mark.gpu
@pytest.mark.parametrize("H,G,d", [(1, 7, 128), (2, 4, 64), (4, 7, 128), (4, 16, 64), (8, 8, 128), (2, 16, 128), (8, 9, 128),
                                   (1, 1, 64), (8, 2, 64), (1, 12, 64)])
@pytest.mark.parametrize("lens", ["one", "edges", "long", "many", "lanes"])
def test_decode(lens, H, G, d):
    c = Cache(LENGTHS[lens], H, d, Hq=H * G, slack=1, seed=G)
    want = c.expected()
    ac.aircache_quantize(c.sh, c.ragged, c.cache8)
    q = queries(c, G)
    out = torch.full((c.R, H * G, d), float("nan"), device=DEV)
    ac.aircache_decode_attn_quantized(c.sh, c.cache8, q, out, c.ws)
    c.check_attention(q, out, want, c.lens0)
    again = torch.full_like(out, float("nan"))
    ac.aircache_decode_attn_quantized(c.sh, c.cache8, q, again, c.ws)
    assert torch.equal(out, again)


@pytest.mark.gpu
@pytest.mark.parametrize("H,G,d", [(1, 7, 64), (2, 9, 64), (4, 2, 128)])
def test_decode_of_as_many_regions_as_there_may_be(H, G, d):
    test_decode("most", H, G, d)


@pytest.mark.gpu
def test_decode_per_kv_head():
    c = Cache([33, 64, 0, 700, 1, 90, 12, 65], 1, 128, Hq=14, per_kv_head=1, Hkv=2, seed=3)
    want = c.expected()
    ac.aircache_quantize(c.sh, c.ragged, c.cache8)
    q = queries(c, 7)   # [cells, G, d] is [L, B, Hq, d]
    out = torch.full((c.R, 7, 128), float("nan"), device=DEV)
    ac.aircache_decode_attn_quantized(c.sh, c.cache8, q, out, c.ws)
    c.check_attention(q, out, want, c.lens0)


@pytest.mark.gpu
def test_decode_sharp_and_wide_values():
    """Logits hundreds apart in both orders, queries of very different sizes, blocks whose scales differ by 2^12."""
    c = Cache([400, 400], 2, 128, Hq=16, seed=5)
    ramp = torch.linspace(-1, 1, 400, device=DEV)[:, None, None]
    c.k[:400] = (c.k[:400].float() * 0.1 + 40 * ramp).bfloat16()
    c.k[400:800] = (c.k[400:800].float() * 0.1 - 40 * ramp).bfloat16()
    c.v[100:200] *= 4096
    c.v[500:520] /= 4096
    want = c.expected()
    ac.aircache_quantize(c.sh, c.ragged, c.cache8)
    q = (queries(c, 8).float() * torch.tensor([1.0, 1e-6, 30.0, 1e-30, 0.0, 3.0, 0.1, 1.0] * 2, device=DEV)[:, None]).bfloat16()
    out = torch.full(q.shape, float("nan"), device=DEV)
    ac.aircache_decode_attn_quantized(c.sh, c.cache8, q, out, c.ws)
    c.check_attention(q, out, want, c.lens0)


@pytest.mark.gpu
def test_decode_keys_without_a_finite_logit_first():
    """The first rows of a region have logits of minus infinity (their scale times the query leaves fp32); what follows counts."""
    c = Cache([300, 40], 2, 64, Hq=8, seed=8)
    ac.aircache_quantize(c.sh, c.ragged, c.cache8)
    q = queries(c, 4)
    q[0, :4] = q[0, :4].abs() + 1
    c.k8[:64, 0] = 0xfe                                # -448
    c.k_scale[0, 0] = 2.0 ** 120
    want = {x: getattr(c, x).cpu().numpy() for x in ("k8", "v8", "k_scale", "v_scale")}
    out = torch.full((2, 8, 64), float("nan"), device=DEV)
    ac.aircache_decode_attn_quantized(c.sh, c.cache8, q, out, c.ws)
    k, v, held = c.values(want, [300, 40])[0]
    for h in range(4):   # without the first block
        ref, tol = attention(q[0, h:h + 1].double().cpu().numpy(), k[64:, 0], v[64:, 0], c.sh.scale, held[0])
        assert (np.abs(out[0, h:h + 1].double().cpu().numpy() - ref) <= tol).all()


@pytest.mark.gpu
def test_garbage_behind_the_rows_in_use_reaches_nothing():
    c = Cache([17, 70], 2, 64, Hq=8, slack=40)
    want = c.expected()
    ac.aircache_quantize(c.sh, c.ragged, c.cache8)
    for x in (c.k8, c.v8):
        x[17:57] = 0x7f   # NaN
        x[57 + 70:] = 0xff
    q = queries(c, 4)
    out = torch.full((2, 8, 64), float("nan"), device=DEV)
    ac.aircache_decode_attn_quantized(c.sh, c.cache8, q, out, c.ws)
    c.check_attention(q, out, want, c.lens0)


@pytest.mark.gpu
@pytest.mark.parametrize("H,G,d,per", [(4, 7, 128, 0), (2, 4, 64, 0), (1, 7, 128, 1), (8, 8, 128, 0), (1, 2, 64, 1)])
def test_append_and_decode_step_by_step(H, G, d, per):
    Hkv = 2 if per else H
    lens = [0, 1, 62, 63, 64, 126, 200, 130]
    c = Cache(lens, H, d, Hq=Hkv * G, slack=6, per_kv_head=per, Hkv=Hkv, seed=7)
    want = c.expected()
    ac.aircache_quantize(c.sh, c.ragged, c.cache8)
    gen = torch.Generator().manual_seed(9)
    for i in range(6):
        new = [(torch.randn((c.R, H, d), generator=gen) * (4.0 ** (i - 2) if x else 30.0 * (i % 2) + 0.01)).bfloat16() for x in (0, 1)]
        for x, cc, s in zip(new, ("k8", "v8"), ("k_scale", "v_scale")):
            appended(x.double().numpy(), c.offs, [n + i for n in lens], want[cc], want[s])
        ac.aircache_append_quantized(c.sh, c.cache8, new[0].to(DEV), new[1].to(DEV), i)
        c.check(want)
        assert c.lens.tolist() == [n + i + 1 for n in lens]
        q = queries(c, G, seed=20 + i)
        out = torch.full((c.R, H * G, d), float("nan"), device=DEV)
        ac.aircache_decode_attn_quantized(c.sh, c.cache8, q, out, c.ws)
        c.check_attention(q, out, want, [n + i + 1 for n in lens])


@pytest.mark.gpu
def test_two_caches_share_buffers():
    """Two requests of their own shapes in one pair of buffers, one attention call over both."""
    d, H = 64, 2
    a = Cache([70, 5], H, d, Hq=8, slack=1)
    rows_a = int(a.offs[-1])
    lens = [70, 5, 130]
    both = Cache(lens, H, d, Hq=8, slack=1, seed=4)
    want = both.expected()
    sh_a, sh_b = ac.shape(2, 1, 8, H, d, 3, 1, 1, 1), ac.shape(1, 1, 8, H, d, 3, 1, 1, 1)
    size = both.offsets.element_size()
    for sh, first, n in ((sh_a, 0, 2), (sh_b, 2, 1)):
        o, l = both.offsets.data_ptr() + first * size, both.lens.data_ptr() + first * 4
        view = ac.quantized_view(both.k8, both.v8, both.k_scale, both.v_scale, o, l, both.rows, first)
        ac.aircache_quantize(sh, ac.ragged_view(both.k, both.v, o, l, both.rows, rows_a if first else 0), view)
    both.check(want)
    q, out = queries(both, 4), torch.empty((3, 8, d), device=DEV)
    ac.aircache_decode_attn_quantized(both.sh, both.cache8, q, out, both.ws)
    both.check_attention(q, out, want, lens)


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    """Rows whose elements lie more than 2^32 bytes into the buffers (8 heads of 128: 1 KB a row)."""
    H, d, rows = 8, 128, (1 << 22) + 4096
    lens = torch.tensor([100, 90], dtype=torch.int32, device=DEV)
    offsets = torch.tensor([0, rows - 100, rows], dtype=torch.int64, device=DEV)
    sh = ac.shape(2, 1, 64, H, d, 3, 1, 1, 10)
    blocks = ac.aircache_scale_blocks(sh, rows)
    k8, v8 = (torch.zeros((rows, H, d), dtype=torch.uint8, device=DEV) for _ in range(2))
    ks, vs = (torch.ones((blocks, H), device=DEV) for _ in range(2))
    gen = torch.Generator().manual_seed(2)
    c = Cache([100, 90], H, d, Hq=64, slack=10, seed=6)
    want = c.expected()
    ac.aircache_quantize(c.sh, c.ragged, c.cache8)
    at = [(0, 0), (rows - 100, 110)]
    for r, (to, fro) in enumerate(at):
        n = [100, 90][r]
        k8[to:to + n], v8[to:to + n] = c.k8[fro:fro + n], c.v8[fro:fro + n]
        b, f = to // 64 + r, fro // 64 + r
        ks[b:b + 2], vs[b:b + 2] = c.k_scale[f:f + 2], c.v_scale[f:f + 2]
    view = ac.quantized_view(k8, v8, ks, vs, offsets, lens, rows)
    q, out = queries(c, 8), torch.empty((2, 64, d), device=DEV)
    ws = torch.zeros(ac.aircache_workspace_bytes(sh), dtype=torch.uint8, device=DEV)
    ac.aircache_decode_attn_quantized(sh, view, q, out, ws)
    c.check_attention(q, out, want, [100, 90])
    new = torch.randn((2, 1, H, d), generator=gen).bfloat16().to(DEV)
    ac.aircache_append_quantized(sh, view, new, new, 0)
    assert (k8[rows - 10] != 0).any() and (k8[100] != 0).any() and lens.tolist() == [101, 91]


@pytest.mark.gpu
def test_captured_and_replayed_on_another_stream():
    lens = [40, 64, 90]
    c = Cache(lens, 2, 64, Hq=8, slack=4, seed=11)
    want = c.expected()
    ac.aircache_quantize(c.sh, c.ragged, c.cache8)
    gen = torch.Generator().manual_seed(3)
    k_new, v_new = ((torch.randn((3, 2, 64), generator=gen) * 50).bfloat16().to(DEV) for _ in range(2))
    q, out = queries(c, 4), torch.empty((3, 8, 64), device=DEV)
    ac.aircache_decode_attn_quantized(c.sh, c.cache8, q, out, c.ws)   # (sets the kernel's limits before the capture)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        ac.aircache_append_quantized(c.sh, c.cache8, k_new, v_new, 0)
        ac.aircache_decode_attn_quantized(c.sh, c.cache8, q, out, c.ws)
    for i in range(3):
        for x, cc, s in ((k_new, "k8", "k_scale"), (v_new, "v8", "v_scale")):
            appended(x.double().cpu().numpy(), c.offs, [n + i for n in lens], want[cc], want[s])
        graph.replay()
        torch.cuda.synchronize()
        c.check(want)
        c.check_attention(q, out, want, [n + i + 1 for n in lens])


@pytest.mark.gpu
def test_from_compaction():
    """The compressed cache as the library makes it, then in 8 bits through the session."""
    L, B, Hq, Hkv, d, Nv, Nt = 3, 2, 8, 2, 64, 300, 20
    s = Session(ac.shape(L, B, Hq, Hkv, d, Nv, Nt, 8, 5), 0.2, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(1)
    k, v = (torch.randn((L, B, Hkv, Nv + Nt, d), generator=gen, device=DEV).bfloat16() for _ in range(2))
    s.set_full(k, v)
    s.score(torch.randn((L, B, 8, Hq, d), generator=gen, device=DEV).bfloat16())
    s.budget()
    s.compact()
    s.quantize()
    q = torch.randn((L, B, Hq, d), generator=gen, device=DEV).bfloat16()
    s.decode(q)
    wide = s.out.clone()
    s.decode_quantized(q)
    # 3 bits behind the point: an element is off by at most 2^-4 of itself
    assert ((s.out - wide).norm() / wide.norm()).item() < 2.0 ** -4
    new = torch.randn((L, B, Hkv, d), generator=gen, device=DEV).bfloat16()
    before = s.lens.clone()
    s.append_quantized(new, new, 0)
    assert torch.equal(s.lens, before + 1)
