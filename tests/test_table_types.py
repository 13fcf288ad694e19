"""Tables whose type matters (positions, frequencies, weights, rows, offsets, scales) are refused where a tensor has another type
or gaps: torch makes 64-bit integers and 32-bit floats where it is not told otherwise, and a kernel would read something else
from them, or past their end.  Natively and through ctypes; no GPU."""
import ctypes as C

import pytest
import torch

import paper_2503_23956_b200 as ac

P = 0x10000000   # never followed: the calls have no tokens
T = 6


@pytest.fixture(params=["ctypes", "native"])
def path(request, monkeypatch):
    if request.param == "ctypes":
        monkeypatch.setattr(ac, "_native", False)
        return
    from paper_2503_23956_b200 import _binding
    _binding.setup(ac.Shape, ac.Ragged, lambda: 0, lambda dev: 0, ac.Tokens, ac.Rotary, ac.Prompt, ac.Quantized, torch.int32,
                   torch.int64, torch.float32, torch.bfloat16)
    fns = [C.cast(getattr(ac.lib(), "aircache_" + n), C.c_void_p).value
           for n in ("decode_attn", "decode_step", "decode_attn_quantized", "append_quantized", "rotate", "prompt_attn")]
    monkeypatch.setattr(ac, "_native", (_binding, *fns))


def rotate(**over):
    a = dict(positions=torch.zeros((3, T), dtype=torch.int32), inv_freq=torch.ones(32), q_weight=torch.ones((2, 64)).bfloat16(),
             k_weight=torch.ones((2, 64)).bfloat16(), rows=torch.arange(T))
    a.update(over)
    t, o = ac.Tokens(P, 4096, 256, 64), ac.Tokens(2 * P, 4096, 256, 64)
    spec = ac.rotary(2, 0, 4, 2, 64, sections=[8, 12, 12])   # no tokens: checked, nothing launched
    return ac.aircache_rotate(spec, t, t, t, a["positions"], a["inv_freq"], a["q_weight"], a["k_weight"], o, o, o, a["rows"], T,
                              stream=1, check=False)


def prompt(q_offsets, k_offsets):
    t = ac.Tokens(P, 0, 256, 64)
    return ac.aircache_prompt_attn(ac.prompt(0, T, T, 4, 2, 64), t, t, t, q_offsets, k_offsets, t, stream=1, check=False)


def test_rotate(path):
    assert rotate() == ac.OK
    assert rotate(positions=P, inv_freq=P, q_weight=None, k_weight=P, rows=None) == ac.OK   # addresses, and none
    assert rotate(q_weight=torch.nn.Parameter(torch.ones((2, 64)).bfloat16())) == ac.OK
    for name, wrong in (("positions", torch.zeros((3, T), dtype=torch.int64)), ("positions", torch.zeros((3, T))),
                        ("positions", torch.zeros((T, 3), dtype=torch.int32).t()),
                        ("inv_freq", torch.ones(32, dtype=torch.float64)), ("inv_freq", torch.ones(32).bfloat16()),
                        ("q_weight", torch.ones((2, 64))), ("k_weight", torch.ones((2, 64)).half()),
                        ("rows", torch.arange(T, dtype=torch.int32)), ("rows", torch.arange(2 * T)[::2])):
        with pytest.raises(TypeError, match=name):
            rotate(**{name: wrong})


def test_prompt(path):
    good = torch.tensor([0, T], dtype=torch.int32)
    assert prompt(good, good) == ac.OK and prompt(good, None) == ac.OK and prompt(P, P) == ac.OK
    for wrong in (torch.tensor([0, T]), torch.tensor([0, 1, T, 1], dtype=torch.int32)[::2]):
        with pytest.raises(TypeError, match="q_offsets"):
            prompt(wrong, good)
        with pytest.raises(TypeError, match="k_offsets"):
            prompt(good, wrong)


def test_the_cache_of_8_bits():
    codes, scale = torch.zeros((64, 2, 64), dtype=torch.uint8), torch.ones((3, 2))
    good = dict(k=codes, v=codes.view(torch.float8_e4m3fn), k_scale=scale, v_scale=scale,
                offsets=torch.tensor([0, 32, 64]), lens=torch.tensor([30, 30], dtype=torch.int32))
    view = ac.quantized_view(**good, total_rows=64)
    assert view.k == codes.data_ptr() and view.scale_blocks == 3
    assert ac.quantized_view(P, P, P, P, P, P, 64, 0, 3).lens == P
    for name, wrong in (("k", codes.bfloat16()), ("v", codes.transpose(0, 1)), ("k_scale", scale.bfloat16()),
                        ("v_scale", scale.double()), ("k_scale", torch.ones((2, 3)).t()),
                        ("offsets", torch.tensor([0, 32, 64], dtype=torch.int32)), ("lens", torch.tensor([30, 30]))):
        with pytest.raises(TypeError, match=name):
            ac.quantized_view(**{**good, name: wrong}, total_rows=64)
