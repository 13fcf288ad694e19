"""The operators around the compressed cache: the prompt's keys and attention in front of it, a cache of 8 bits behind it.

A vision-language serving engine runs a layer of the prompt as aircache_rotate (norms of queries and keys, rotary
positions, keys and values into the rows of the full cache) and aircache_prompt_attn (packed sequences), scores and
compresses the cache, may then hold it in 8 bits (aircache_quantize) and decodes over that: aircache_append_quantized for
a token's keys and values, aircache_decode_attn_quantized for its attention.  The kinds of case:

  rotate    norms, rotation and the store into the cache, of one layer's or all layers' new tokens
  prompt    attention of one layer over packed sequences, with or without keys of earlier turns
  quantize  a compressed bf16 cache into 8 bits
  steps     `rounds` tokens of a request batch over the cache of 8 bits: append, then attention
  attn      one attention call over the cache of 8 bits

Definitions.  rotate: y = x * rsqrt(mean(x^2) + eps) * w over a head's channels (where there are weights), then pairs of
the first `rotary` channels turned by position * inv_freq.  prompt: row i of a sequence's new tokens sees its first
n_k - n_q + i + 1 keys.  quantize: 64 rows of a region and KV head share a scale, the smallest power of two s with
max|x| <= 448 s; a value is held as e4m3(x / s).  append: the block's scale becomes the larger of its own and the new
row's, what the block holds is rounded again if it grew.
"""
import math
import random

import torch

own = False

_DEV = "cuda:0"
_BLOCK = 64

# layers, query heads, KV heads, head_dim: the tiny cache, the Qwen2-7B-shaped decoder and the Qwen2-72B-shaped stack
# of this repository's configurations, and two generic decoders (two KV heads; eight KV heads of 64 channels)
_MODELS = {
    "tiny": (4, 8, 2, 64),
    "7b": (28, 28, 4, 128),
    "72b": (80, 64, 8, 128),
    "two_kv": (24, 32, 2, 128),
    "small_heads": (24, 32, 8, 64),
}


def listed():
    return [
        # the new tokens of four requests in one layer: launch latency
        dict(name="rotate_token", kind="rotate", model="7b", layers=1, tokens=4, axes=3, norm=True, pairs="half",
             part=1.0),
        # one layer of the prompts of four video requests, three position axes (time, height, width)
        dict(name="rotate_video", kind="rotate", model="7b", layers=1, tokens=27136, axes=3, norm=True, pairs="half",
             part=1.0),
        # one layer of the smallest prompt: one image and some text
        dict(name="prompt_tiny", kind="prompt", model="tiny", seqs=1, least=640, most=640, before=0, causal=True),
        # one layer of a follow-up turn of sixteen users: some new tokens each over the keys of earlier turns
        dict(name="prompt_turns", kind="prompt", model="7b", seqs=16, least=1, most=300, before=3172, causal=True),
        # one layer of eight prompts of different lengths, packed
        dict(name="prompt_packed", kind="prompt", model="7b", seqs=8, least=300, most=3172, before=0, causal=True),
        # one layer of a long prompt to a large model
        dict(name="prompt_long", kind="prompt", model="72b", seqs=1, least=9338, most=9338, before=0, causal=True),
        # the compressed cache of one image
        dict(name="quantize_image", kind="quantize", model="7b", batch=1, visual=7290, text=128, ratio=0.10,
             heads=False),
        # the compressed cache of a full serving batch
        dict(name="quantize_batch", kind="quantize", model="7b", batch=64, visual=2916, text=256, ratio=0.10,
             heads=False),
        # interactive use: one high-resolution image, one user, 32 tokens generated
        dict(name="steps_image", kind="steps", model="7b", batch=1, visual=7290, text=128, ratio=0.10, heads=False,
             rounds=32),
        # four video requests, 8 tokens generated
        dict(name="steps_video", kind="steps", model="7b", batch=4, visual=6272, text=512, ratio=0.10, heads=False,
             rounds=8),
        # one token of a full serving batch
        dict(name="attn_batch", kind="attn", model="7b", batch=64, visual=2916, text=256, ratio=0.10, heads=False),
        # one token of a long-context request to a large model whose budgets differ by KV head
        dict(name="attn_heads", kind="attn", model="72b", batch=1, visual=7290, text=2048, ratio=0.05, heads=True),
    ]


# A drawn case stays below the largest listed ones: bytes and operations of a pass, and the logits of a prompt.
_MOST_BYTES = 2.0e9
_MOST_FLOPS = 1.3e12
_MOST_LOGITS = 5.5e9


def draw(rng):
    def log_uniform(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["rotate", "prompt", "prompt", "quantize", "steps", "attn"])
    model = rng.choice(["tiny", "7b", "7b", "7b", "72b", "two_kv", "small_heads"])
    L, _, Hkv, _ = _MODELS[model]
    case = dict(kind=kind, model=model)
    if kind == "rotate":
        case.update(layers=rng.choice([1, 1, L]), tokens=log_uniform(1, 28000), axes=rng.choice([1, 3]),
                    norm=rng.random() < 0.5, pairs=rng.choice(["half", "half", "interleaved"]),
                    part=rng.choice([1.0, 1.0, 0.5, 0.25]))
        if case["layers"] > 1:
            case["tokens"] = max(1, case["tokens"] // L)
        return case
    if kind == "prompt":
        case.update(seqs=log_uniform(1, 32), least=log_uniform(1, 600), before=rng.choice([0, 0, log_uniform(1, 6000)]),
                    causal=rng.random() < 0.85)
        case["most"] = case["least"] + log_uniform(1, 8000)
        while True:
            n_q, n_k = _lengths(case)
            logits = case["seqs"] * max(n_q) * max(n_k) * _MODELS[model][1]
            if work(case)["flops"] <= _MOST_FLOPS and logits <= _MOST_LOGITS:
                return case
            if case["seqs"] > 1:
                case["seqs"] = case["seqs"] * 3 // 4
            else:
                case["most"] = max(case["least"], case["most"] * 3 // 4)
                case["before"] = case["before"] * 3 // 4
    case.update(visual=log_uniform(400, 9000), text=log_uniform(24, 2048), ratio=rng.choice([0.05, 0.10, 0.25, 0.50]),
                heads=rng.random() < 0.2)
    # the library takes at most 1792 regions (cells, with budgets per KV head)
    case["batch"] = min(log_uniform(1, 64), 1792 // (L * (Hkv if case["heads"] else 1)))
    if kind == "steps":
        case["rounds"] = log_uniform(2, 32)
    while work(case)["bytes"] > _MOST_BYTES:
        if case["batch"] > 1:
            case["batch"] = case["batch"] * 3 // 4
        elif case.get("rounds", 1) > 2:
            case["rounds"] = case["rounds"] * 3 // 4
        else:
            case["visual"] = case["visual"] * 3 // 4
            case["text"] = max(24, case["text"] * 3 // 4)
    return case


def _lengths(case):
    """New tokens and keys of every packed sequence, between `least` and `most`, evenly over the logarithm."""
    rng = random.Random("%(seqs)d %(least)d %(most)d %(before)d" % case)
    n_q = [int(round(math.exp(rng.uniform(math.log(case["least"]), math.log(case["most"])))))
           for _ in range(case["seqs"])]
    n_k = [n + (rng.randint(case["before"] // 4, case["before"]) if case["before"] else 0) for n in n_q]
    return n_q, n_k


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
def _normal(shape, gen):
    return torch.empty(shape, dtype=torch.bfloat16, device=_DEV).normal_(generator=gen)


def _rotary_channels(case):
    return int(_MODELS[case["model"]][3] * case["part"])


def _sections(case):
    """Frequencies that follow each position axis: a quarter the first, the rest in equal parts."""
    n = _rotary_channels(case) // 2
    if case["axes"] == 1:
        return [n]
    rest = (n - n // 4) // 2
    return [n - 2 * rest, rest, rest]


def _prepare_rotate(case, gen):
    _, Hq, Hkv, d = _MODELS[case["model"]]
    L, T = case["layers"], case["tokens"]
    qkv = _normal((L, T, Hq + 2 * Hkv, d), gen)     # a layer's projection gives all three
    st = dict(q=qkv[:, :, :Hq], k=qkv[:, :, Hq:Hq + Hkv], v=qkv[:, :, Hq + Hkv:])
    # positions of a long context; the rows that the tokens take in the cache, in no order
    st["positions"] = torch.randint(0, 1 << 17, (case["axes"], T), generator=gen, device=_DEV, dtype=torch.int32)
    n_rows = T + T // 8 + 3
    st["rows"] = torch.randperm(n_rows, generator=gen, device=_DEV)[:T].contiguous()
    n = _rotary_channels(case) // 2
    st["inv_freq"] = (1e6 ** (-torch.arange(n, dtype=torch.float64) / n)).float().to(_DEV)
    st["axis"] = torch.tensor(sum(([a] * s for a, s in enumerate(_sections(case))), []), device=_DEV)
    st["q_weight"] = st["k_weight"] = None
    if case["norm"]:
        st["q_weight"] = (1 + 0.2 * _normal((L, d), gen).float()).bfloat16()
        st["k_weight"] = (1 + 0.2 * _normal((L, d), gen).float()).bfloat16()
    st["q_out"] = torch.empty((L, T, Hq, d), dtype=torch.bfloat16, device=_DEV)
    st["k_cache"] = torch.zeros((L, n_rows, Hkv, d), dtype=torch.bfloat16, device=_DEV)
    st["v_cache"] = torch.zeros_like(st["k_cache"])
    return st


def _prepare_prompt(case, gen):
    _, Hq, Hkv, d = _MODELS[case["model"]]
    n_q, n_k = _lengths(case)
    offsets = lambda n: torch.tensor([0] + n, device=_DEV).cumsum(0).to(torch.int32)  # noqa: E731
    st = dict(q_offsets=offsets(n_q), k_offsets=offsets(n_k), n_q=n_q, n_k=n_k)
    st["q"] = _normal((sum(n_q), Hq, d), gen)
    st["k"] = _normal((sum(n_k), Hkv, d), gen)
    st["v"] = _normal((sum(n_k), Hkv, d), gen)
    # some keys that the queries agree on, as in a trained model: rows of the softmax differ in how sharp they are
    u = torch.randn((Hkv, d), generator=gen, device=_DEV)
    u = u / u.norm(dim=-1, keepdim=True) * math.sqrt(math.sqrt(d))
    strong = 2.5 * (torch.rand((sum(n_k), 1, 1), generator=gen, device=_DEV) < 0.05)
    st["k"] += (strong * u).bfloat16()
    st["q"] += u.repeat_interleave(Hq // Hkv, dim=0).bfloat16()
    st["out"] = torch.empty_like(st["q"])
    return st


def _ragged(case, gen):
    """Offsets, rows in use and the 8-bit buffers of a compressed cache whose regions differ in length."""
    L, Hq, Hkv, d = _MODELS[case["model"]]
    B, slack = case["batch"], case.get("rounds", 0)
    cells, row_heads = (Hkv, 1) if case["heads"] else (1, Hkv)
    total = math.floor(case["ratio"] * case["visual"] * L * cells + 0.5)
    share = 0.5 + torch.rand((B, L * cells), generator=gen, device=_DEV, dtype=torch.float64)
    ends = (share.cumsum(1) / share.sum(1, keepdim=True) * total).round().to(torch.int64)
    kept = torch.diff(ends, dim=1, prepend=torch.zeros_like(ends[:, :1]))
    kept = kept.view(B, L, cells).transpose(0, 1).reshape(-1)
    R = L * B * cells
    st = dict(offsets=torch.zeros(R + 1, dtype=torch.int64, device=_DEV), lens=(kept + case["text"]).to(torch.int32))
    st["offsets"][1:] = (kept + case["text"] + slack).cumsum(0)
    rows = B * (total + L * cells * (case["text"] + slack))
    st["rows"], st["R"], st["H"] = rows, R, row_heads
    st["most"] = int(st["lens"].max()) + slack
    st["k8"] = torch.zeros((rows, row_heads, d), dtype=torch.uint8, device=_DEV).view(torch.float8_e4m3fn)
    st["v8"] = torch.zeros((rows, row_heads, d), dtype=torch.uint8, device=_DEV).view(torch.float8_e4m3fn)
    blocks = rows // _BLOCK + R
    st["k_scale"] = torch.ones((blocks, row_heads), device=_DEV)
    st["v_scale"] = torch.ones((blocks, row_heads), device=_DEV)
    st["shape"] = (L, B, Hq, Hkv, d, case["visual"], case["text"], 1, slack, None, int(case["heads"]))
    return st


def _prepare_quantize(case, gen):
    st = _ragged(case, gen)
    d = _MODELS[case["model"]][3]
    for x in ("k", "v"):
        t = _normal((st["rows"], st["H"], d), gen)
        if x == "k":   # a few channels of the keys are much larger than the rest
            t *= torch.exp(0.7 * torch.randn((st["H"], d), generator=gen, device=_DEV)).bfloat16()
        st[x] = t
    return st


def _fill(st, gen):
    for c, s in (("k8", "k_scale"), ("v8", "v_scale")):
        flat = st[c].view(-1)
        for at in range(0, flat.numel(), 1 << 28):
            part = flat[at:at + (1 << 28)]
            part.copy_(torch.randn(part.shape, generator=gen, device=_DEV).mul_(100).clamp_(-448, 448))
        power = torch.randint(-8, -5, st[s].shape, generator=gen, device=_DEV)
        st[s].copy_(torch.ldexp(torch.ones_like(st[s]), power))


def _prepare_attn(case, gen):
    st = _ragged(case, gen)
    _fill(st, gen)
    L, Hq, _, d = _MODELS[case["model"]]
    st["q"] = _normal((L, case["batch"], Hq, d), gen)
    st["out"] = torch.empty(st["q"].shape, device=_DEV)
    return st


def _prepare_steps(case, gen):
    st = _ragged(case, gen)
    _fill(st, gen)
    L, Hq, Hkv, d = _MODELS[case["model"]]
    B, n = case["batch"], case["rounds"]
    st["start"] = st["lens"].clone()
    st["q"] = _normal((n, L, B, Hq, d), gen)
    st["out"] = torch.empty(st["q"].shape, device=_DEV)
    for x in ("k_new", "v_new"):   # now and then a token that is larger than its block
        wide = 1 + 3 * (torch.rand((n, L, B, 1, 1), generator=gen, device=_DEV) < 0.1)
        st[x] = (_normal((n, L, B, Hkv, d), gen).float() * wide).bfloat16()
    return st


_PREPARE = dict(rotate=_prepare_rotate, prompt=_prepare_prompt, quantize=_prepare_quantize, steps=_prepare_steps,
                attn=_prepare_attn)


def prepare(case, seed):
    gen = torch.Generator(device=_DEV)
    gen.manual_seed(seed)
    st = _PREPARE[case["kind"]](case, gen)
    st["case"] = case
    return st


# ---------------------------------------------------------------------------------------------
# one pass through the library
# ---------------------------------------------------------------------------------------------
def _kept(st, make):
    """What a program builds once for its buffers: shapes, views of them, the workspace.  No data."""
    if "kept" not in st:
        import paper_2503_23956_b200 as ac
        st["kept"] = (ac,) + make(ac, st)
    return st["kept"]


def _views_rotate(ac, st):
    case = st["case"]
    L, T, Hq, d = st["q_out"].shape
    spec = ac.rotary(L, T, Hq, st["k_cache"].shape[2], d, rotary_dim=_rotary_channels(case),
                     interleaved=int(case["pairs"] == "interleaved"), sections=_sections(case), eps=1e-6)
    return spec, [ac.tokens_view(st[x]) for x in ("q", "k", "v")], [ac.tokens_view(st[x]) for x in
                                                                   ("q_out", "k_cache", "v_cache")]


def _own_rotate(st):
    ac, spec, new, to = _kept(st, _views_rotate)
    ac.aircache_rotate(spec, *new, st["positions"], st["inv_freq"], st["q_weight"], st["k_weight"], *to, st["rows"],
                       st["k_cache"].shape[1])


def _views_prompt(ac, st):
    T, Hq, d = st["q"].shape
    spec = ac.prompt(len(st["n_q"]), T, st["k"].shape[0], Hq, st["k"].shape[1], d, causal=int(st["case"]["causal"]))
    return spec, [ac.tokens_view(st[x]) for x in ("q", "k", "v")], ac.tokens_view(st["out"])


def _own_prompt(st):
    ac, spec, qkv, out = _kept(st, _views_prompt)
    ac.aircache_prompt_attn(spec, *qkv, st["q_offsets"], st["k_offsets"], out)


def _views_cache(ac, st):
    sh = ac.shape(*st["shape"])
    ws = torch.empty(ac.aircache_workspace_bytes(sh), dtype=torch.uint8, device=_DEV)
    ac.aircache_reset_status(ws)
    return sh, ws, ac.quantized_view(st["k8"], st["v8"], st["k_scale"], st["v_scale"], st["offsets"], st["lens"],
                                     st["rows"])


def _own_quantize(st):
    ac, sh, _, cache8 = _kept(st, _views_cache)
    ac.aircache_quantize(sh, ac.ragged_view(st["k"], st["v"], st["offsets"], st["lens"], st["rows"]), cache8)


def _own_attn(st):
    ac, sh, ws, cache8 = _kept(st, _views_cache)
    ac.aircache_decode_attn_quantized(sh, cache8, st["q"], st["out"], ws)


def _own_steps(st):
    ac, sh, ws, cache8 = _kept(st, _views_cache)
    for i in range(st["case"]["rounds"]):
        ac.aircache_append_quantized(sh, cache8, st["k_new"][i], st["v_new"][i], i)
        ac.aircache_decode_attn_quantized(sh, cache8, st["q"][i], st["out"][i], ws)


# ---------------------------------------------------------------------------------------------
# one pass in plain form
# ---------------------------------------------------------------------------------------------
def _plain_turn(x, w, st):
    """Norm and rotation of [L, T, H, d] in 32 bits, the angles in 64."""
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w.float()[:, None, None]
    n = st["inv_freq"].numel()
    angle = st["positions"].t()[:, st["axis"]].double() * st["inv_freq"].double()
    c, s = angle.cos().float()[:, None], angle.sin().float()[:, None]
    turned, rest = x[..., :2 * n], x[..., 2 * n:]
    if st["case"]["pairs"] == "interleaved":
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack((a * c - b * s, b * c + a * s), dim=-1).flatten(-2)
    else:
        a, b = turned[..., :n], turned[..., n:]
        turned = torch.cat((a * c - b * s, b * c + a * s), dim=-1)
    return torch.cat((turned, rest), dim=-1).bfloat16()


def _plain_rotate(st):
    st["q_out"].copy_(_plain_turn(st["q"], st["q_weight"], st))
    st["k_cache"][:, st["rows"]] = _plain_turn(st["k"], st["k_weight"], st)
    st["v_cache"][:, st["rows"]] = st["v"]


def _softmax_(s):
    """exp(s - max) in place over the last axis, and its sums; a row without a finite value sums to zero."""
    top = s.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    s.sub_(top).exp_()
    return s, s.sum(-1, keepdim=True)


def _plain_prompt(st):
    """All sequences padded to the longest one."""
    case = st["case"]
    (Tq, Hq, d), (Tk, Hkv, _) = st["q"].shape, st["k"].shape
    S, mq, mk, G = len(st["n_q"]), max(st["n_q"]), max(st["n_k"]), Hq // Hkv
    q_at, k_at = st["q_offsets"].long(), st["k_offsets"].long()
    i, j = torch.arange(mq, device=_DEV), torch.arange(mk, device=_DEV)
    qp = st["q"][(q_at[:-1, None] + i).clamp_(max=Tq - 1)].float()          # [S, mq, Hq, d]
    rows = (k_at[:-1, None] + j).clamp_(max=Tk - 1)
    kp, vp = st["k"][rows].float(), st["v"][rows].float()                   # [S, mk, Hkv, d]
    n_q, n_k = torch.diff(q_at), torch.diff(k_at)
    seen = n_k[:, None, None].expand(S, mq, 1)
    if case["causal"]:
        seen = torch.minimum(seen, (n_k - n_q)[:, None, None] + i[:, None] + 1)
    hidden = j >= seen                                                      # [S, mq, mk]
    qg = qp.view(S, mq, Hkv, G, d).permute(0, 2, 3, 1, 4).reshape(S, Hkv, G * mq, d)
    s = torch.matmul(qg, kp.permute(0, 2, 3, 1)).mul_(1 / math.sqrt(d)).view(S, Hkv, G, mq, mk)
    s.masked_fill_(hidden[:, None, None], -math.inf)
    p, total = _softmax_(s)
    o = torch.matmul(p.view(S, Hkv, G * mq, mk), vp.permute(0, 2, 1, 3)).view(S, Hkv, G, mq, d)
    o = (o / torch.where(total == 0, torch.ones_like(total), total)).permute(0, 3, 1, 2, 4).reshape(S, mq, Hq, d)
    t = torch.arange(Tq, device=_DEV)
    seq = torch.searchsorted(q_at[1:], t, right=True)
    st["out"].copy_(o[seq, t - q_at[seq]])


def _places(st):
    """Region, place in the region and block of every row of a ragged cache."""
    t = torch.arange(st["rows"], device=_DEV)
    r = torch.searchsorted(st["offsets"][1:], t, right=True)
    j = t - st["offsets"][r]
    return r, j, st["offsets"][r] // _BLOCK + r + j // _BLOCK


def _scale_of(top):
    """The smallest power of two s with top <= 448 s, but at least 2^-126."""
    m, e = torch.frexp(top)
    e = torch.where(m > 0.875, e - 8, e - 9).clamp_(min=-126)
    e = torch.where(top == 0, torch.full_like(e, -126), e)
    return torch.ldexp(torch.ones_like(top), e)


def _plain_quantize(st):
    r, j, block = _places(st)
    used = (j < st["lens"][r])
    for x, c, s in (("k", "k8", "k_scale"), ("v", "v8", "v_scale")):
        t = st[x].float()
        top = t.abs().amax(-1) * used[:, None]
        most = torch.zeros_like(st[s]).scatter_reduce_(0, block[:, None].expand_as(top), top, "amax")
        touched = torch.zeros(len(most), dtype=torch.int32, device=_DEV).scatter_reduce_(0, block, used.int(), "amax")
        st[s].copy_(torch.where((touched > 0)[:, None], _scale_of(most), st[s]))
        codes = (t / st[s][block][..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
        st[c].view(torch.uint8).copy_(torch.where(used[:, None, None], codes, st[c].view(torch.uint8)))


def _cells(t, st):
    """New rows [L, B, Hkv, d] as [regions, heads of a row, d]."""
    return t.reshape(st["R"], st["H"], t.shape[-1])


def _plain_append(st, k_new, v_new):
    lens = st["lens"].long()
    at = st["offsets"][:-1] + lens
    place = lens % _BLOCK
    block = st["offsets"][:-1] // _BLOCK + torch.arange(st["R"], device=_DEV) + lens // _BLOCK
    i = torch.arange(_BLOCK, device=_DEV)
    rows = (at - place)[:, None] + i                                        # the block's rows, [R, 64]
    before = (i < place[:, None])
    rows = torch.where(before, rows, at[:, None])
    for new, c, s in ((k_new, "k8", "k_scale"), (v_new, "v8", "v_scale")):
        new = _cells(new, st).float()
        fresh = _scale_of(new.abs().amax(-1))                               # [R, H]
        old = st[s][block]
        scale = torch.where((place == 0)[:, None], fresh, torch.maximum(old, fresh))
        held = st[c].view(torch.uint8)[rows].view(torch.float8_e4m3fn).float() * old[:, None, :, None]
        values = torch.where(before[:, :, None, None], held, new[:, None])
        codes = (values / scale[:, None, :, None]).to(torch.float8_e4m3fn)
        st[c].view(torch.uint8)[rows] = codes.view(torch.uint8)
        st[s][block] = scale
    st["lens"].add_(1)


def _plain_attend(st, q, out):
    """All regions padded to the longest one."""
    R, H, rows = st["R"], st["H"], st["rows"]
    j = torch.arange(st["most"], device=_DEV)
    at = (st["offsets"][:-1, None] + j).clamp_(max=rows - 1)                # [R, most]
    block = st["offsets"][:-1, None] // _BLOCK + torch.arange(R, device=_DEV)[:, None] + j // _BLOCK
    block.clamp_(max=len(st["k_scale"]) - 1)
    hidden = j >= st["lens"][:, None]

    def values(c, s):
        x = st[c].view(torch.uint8)[at].view(torch.float8_e4m3fn).float()
        return x.mul_(st[s][block][..., None]).masked_fill_(hidden[:, :, None, None], 0.0).permute(0, 2, 1, 3)

    qg = q.reshape(R, H, -1, q.shape[-1]).float()                           # [R, H, G, d]
    s = torch.matmul(qg, values("k8", "k_scale").transpose(2, 3)).mul_(1 / math.sqrt(q.shape[-1]))
    s.masked_fill_(hidden[:, None, None], -math.inf)
    p, total = _softmax_(s)
    o = torch.matmul(p, values("v8", "v_scale")) / torch.where(total == 0, torch.ones_like(total), total)
    out.copy_(o.view(out.shape))


def _plain_steps(st):
    for i in range(st["case"]["rounds"]):
        _plain_append(st, st["k_new"][i], st["v_new"][i])
        _plain_attend(st, st["q"][i], st["out"][i])


_RUN = dict(rotate=(_plain_rotate, _own_rotate), prompt=(_plain_prompt, _own_prompt),
            quantize=(_plain_quantize, _own_quantize), steps=(_plain_steps, _own_steps),
            attn=(lambda st: _plain_attend(st, st["q"], st["out"]), _own_attn))
_OUTPUTS = dict(rotate=("q_out", "k_cache", "v_cache"), prompt=("out",), quantize=("k8", "v8", "k_scale", "v_scale"),
                steps=("out", "k8", "v8", "k_scale", "v_scale", "lens"), attn=("out",))


def run(state):
    kind = state["case"]["kind"]
    if kind == "steps":
        state["lens"].copy_(state["start"])   # the request starts again behind its compressed prompt
    if own:
        _RUN[kind][1](state)
    else:
        _RUN[kind][0](state)
    return {x: state[x] for x in _OUTPUTS[kind]}


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------
def work(case):
    L, Hq, Hkv, d = _MODELS[case["model"]]
    kind = case["kind"]
    if kind == "rotate":
        rows = case["layers"] * case["tokens"]
        return {"bytes": 2 * 2.0 * rows * (Hq + 2 * Hkv) * d + case["tokens"] * (4.0 * case["axes"] + 8), "flops": 0.0}
    if kind == "prompt":
        n_q, n_k = _lengths(case)
        seen = sum(a * (b - a) + a * (a + 1) / 2 if case["causal"] else a * b for a, b in zip(n_q, n_k))
        return {"bytes": 2.0 * d * (2 * sum(n_q) * Hq + 2 * sum(n_k) * Hkv), "flops": 4.0 * d * Hq * seen}
    LB, rounds = L * case["batch"], case.get("rounds", 0)
    # rows (of all KV heads) of the compressed cache, and the bytes of one in 8 bits, keys and values
    rows = case["batch"] * math.floor(case["ratio"] * case["visual"] * L + 0.5) + LB * case["text"]
    row = 2 * Hkv * d + 2 * Hkv * 4 / _BLOCK
    if kind == "quantize":
        return {"bytes": (row + 4.0 * Hkv * d) * rows, "flops": 0.0}
    if kind == "attn":
        return {"bytes": row * rows + 6.0 * Hq * d * LB, "flops": 4.0 * Hq * d * rows}
    grown = LB * rounds * (rounds + 1) / 2   # rows that earlier and this round appended
    return {"bytes": row * (rounds * rows + grown) + rounds * LB * (6.0 * Hq * d + 3 * 2 * Hkv * d),
            "flops": 4.0 * Hq * d * (rounds * rows + grown)}


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------
def _exact_rotate(st):
    case = st["case"]
    n = _rotary_channels(case) // 2
    first = lambda i: i if case["pairs"] == "half" else 2 * i        # noqa: E731
    second = lambda i: i + n if case["pairs"] == "half" else 2 * i + 1  # noqa: E731
    axis = [a for a, s in enumerate(_sections(case)) for _ in range(s)]

    def turn(x, w):
        x = x.double()
        if w is not None:
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + 1e-6) * w.double().view(len(w), 1, 1, -1)
        y = x.clone()
        for i in range(n):
            angle = st["positions"][axis[i]].double() * float(st["inv_freq"][i])
            c, s = torch.cos(angle)[None, :, None], torch.sin(angle)[None, :, None]
            a, b = x[..., first(i)], x[..., second(i)]
            y[..., first(i)] = a * c - b * s
            y[..., second(i)] = a * s + b * c
        return y

    k, v = torch.zeros_like(st["k_cache"]).double(), torch.zeros_like(st["v_cache"]).double()
    k.index_copy_(1, st["rows"], turn(st["k"], st["k_weight"]))
    v.index_copy_(1, st["rows"], st["v"].double())
    return dict(q_out=turn(st["q"], st["q_weight"]), k_cache=k, v_cache=v)


def _exact_prompt(st):
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=_DEV)
    Hq, Hkv, d = st["q"].shape[1], st["k"].shape[1], st["q"].shape[2]
    a = b = 0
    for n_q, n_k in zip(st["n_q"], st["n_k"]):
        last = torch.arange(n_k - n_q, n_k, device=_DEV) if st["case"]["causal"] else torch.full((n_q,), n_k, device=_DEV)
        visible = torch.arange(n_k, device=_DEV)[None] <= last[:, None]
        for h in range(Hq):
            g = h * Hkv // Hq
            x = st["q"][a:a + n_q, h].double() @ st["k"][b:b + n_k, g].double().T / math.sqrt(d)
            out[a:a + n_q, h] = torch.softmax(x.masked_fill(~visible, -math.inf), dim=1) @ st["v"][b:b + n_k, g].double()
        a, b = a + n_q, b + n_k
    return dict(out=out)


def _e4m3(y):
    """The nearest number of four significant bits (ties to even), of three bits behind the point below 2^-6."""
    e = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -20))).clamp(min=-6)
    step = torch.exp2(e - 3)
    return torch.round(y / step) * step


def _power(top):
    """Smallest power of two with top <= 448 times it, by stepping from the logarithm's neighbourhood."""
    top = top.double()
    e = torch.floor(torch.log2(top.clamp(min=1e-300) / 448)) - 1
    for _ in range(3):
        e = torch.where(448 * torch.exp2(e) < top, e + 1, e)
    return torch.exp2(e.clamp(min=-126))


def _exact_quantize(st):
    offs, lens = st["offsets"].tolist(), st["lens"].tolist()
    got = {}
    for x, c, s in (("k", "k8", "k_scale"), ("v", "v8", "v_scale")):
        codes = torch.zeros(st[c].shape, dtype=torch.float32, device=_DEV)
        scale = st[s].double()
        for r, n in enumerate(lens):
            o, b = offs[r], offs[r] // _BLOCK + r
            t = torch.zeros((-(-n // _BLOCK) * _BLOCK,) + codes.shape[1:], dtype=torch.float64, device=_DEV)
            t[:n] = st[x][o:o + n]
            t = t.view(-1, _BLOCK, *codes.shape[1:])
            p = _power(t.abs().amax(dim=(1, 3)))
            scale[b:b + len(p)] = p
            codes[o:o + n] = _e4m3(t / p[:, None, :, None]).flatten(0, 1)[:n]
        got[c], got[s] = codes, scale
    return got


def _exact_attend(st, q, k, v, k_scale, v_scale, lens, offs):
    R, H = st["R"], st["H"]
    q = q.reshape(R, H, -1, q.shape[-1]).double()
    out = torch.zeros_like(q)
    for r in range(R):
        o, n = offs[r], lens[r]
        if n == 0:
            continue
        b = torch.arange(n, device=_DEV) // _BLOCK + o // _BLOCK + r
        keys = (k[o:o + n].double() * k_scale[b][..., None].double()).transpose(0, 1)
        vals = (v[o:o + n].double() * v_scale[b][..., None].double()).transpose(0, 1)
        out[r] = torch.softmax(q[r] @ keys.transpose(1, 2) / math.sqrt(q.shape[-1]), dim=-1) @ vals
    return out


def _exact_attn(st):
    o = _exact_attend(st, st["q"], st["k8"], st["v8"], st["k_scale"], st["v_scale"], st["lens"].tolist(),
                      st["offsets"].tolist())
    return dict(out=o.view(st["out"].shape))


def _exact_steps(st):
    if st["R"] * st["case"]["rounds"] > 6000:
        return None   # too many small pieces
    offs, lens = st["offsets"].tolist(), st["start"].tolist()
    held = {c: st[c].float() for c in ("k8", "v8")}
    scale = {s: st[s].double() for s in ("k_scale", "v_scale")}
    outs = []
    for i in range(st["case"]["rounds"]):
        for x, c, s in (("k_new", "k8", "k_scale"), ("v_new", "v8", "v_scale")):
            new = st[x][i].reshape(st["R"], st["H"], -1).double()
            want = _power(new.abs().amax(-1))
            for r in range(st["R"]):
                n, place, b = lens[r], lens[r] % _BLOCK, offs[r] // _BLOCK + r + lens[r] // _BLOCK
                p = torch.maximum(want[r], scale[s][b]) if place else want[r]
                o = offs[r] + n
                part = held[c][o - place:o]
                part.copy_(_e4m3(part.double() * (scale[s][b] / p)[None, :, None]))
                held[c][o] = _e4m3(new[r] / p[:, None])
                scale[s][b] = p
        lens = [n + 1 for n in lens]
        outs.append(_exact_attend(st, st["q"][i], held["k8"], held["v8"], scale["k_scale"], scale["v_scale"], lens, offs))
    got = dict(out=torch.stack(outs).view(st["out"].shape), lens=None)
    got.update(held)
    got.update(scale)
    return got


_EXACT = dict(rotate=_exact_rotate, prompt=_exact_prompt, quantize=_exact_quantize, steps=_exact_steps, attn=_exact_attn)


def exact(case, seed):
    return _EXACT[case["kind"]](prepare(case, seed))
