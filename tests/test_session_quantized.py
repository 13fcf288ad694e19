"""The session's two caches share rows and lengths: calls that would read rows that one of them does not have are refused."""
import pytest
import torch

import paper_2503_23956_b200 as ac
from paper_2503_23956_b200.session import Session

DEV = "cuda:0"
L, B, HQ, HKV, D, NV, NT = 2, 1, 4, 2, 64, 200, 16


def session():
    gen = torch.Generator(device=DEV).manual_seed(1)
    s = Session(ac.shape(L, B, HQ, HKV, D, NV, NT, 8, 4), 0.2, device=DEV)
    k, v = (torch.randn((L, B, HKV, NV + NT, D), generator=gen, device=DEV).bfloat16() for _ in range(2))
    s.set_full(k, v)
    s.score(torch.randn((L, B, 8, HQ, D), generator=gen, device=DEV).bfloat16())
    s.budget()
    s.compact()
    q = torch.randn((L, B, HQ, D), generator=gen, device=DEV).bfloat16()
    new = torch.randn((L, B, HKV, D), generator=gen, device=DEV).bfloat16()
    return s, q, new


@pytest.mark.gpu
def test_nothing_in_8_bits_yet():
    s, q, new = session()
    for call in (lambda: s.decode_quantized(q), lambda: s.append_quantized(new, new, 0)):
        with pytest.raises(RuntimeError, match="quantize"):
            call()
    s.quantize()
    s.decode_quantized(q)
    s.decode(q)   # both hold the same rows
    assert s.status() == 0


@pytest.mark.gpu
def test_rows_appended_in_8_bits():
    s, q, new = session()
    s.quantize()
    s.append_quantized(new, new, 0)
    s.decode_quantized(q)
    with_row = s.out.clone()
    lens = s.lens.clone()
    for call in (lambda: s.decode(q), s.quantize):
        with pytest.raises(RuntimeError, match="appended"):
            call()
    s.decode_quantized(q)   # as it was
    assert torch.equal(s.out, with_row) and torch.equal(s.lens, lens)
    s.compact()   # does not set the lengths
    for call in (lambda: s.decode(q), s.quantize):
        with pytest.raises(RuntimeError, match="appended"):
            call()
    s.budget()
    s.compact()
    s.decode(q)
    with pytest.raises(RuntimeError, match="quantize"):   # of the cache before this compression
        s.decode_quantized(q)
    s.quantize()
    s.append_quantized(new, new, 0)
    s.decode_quantized(q)
    assert torch.equal(s.out, with_row) and torch.equal(s.lens, lens)


@pytest.mark.gpu
def test_the_16_bit_cache_dropped():
    s, q, new = session()
    s.quantize()
    s.decode_quantized(q)
    want = s.out.clone()
    s.k_c = s.v_c = None
    torch.cuda.empty_cache()
    for call in (lambda: s.decode(q), s.quantize, s.compact):
        with pytest.raises(RuntimeError, match="dropped"):
            call()
    s.decode_quantized(q)
    assert torch.equal(s.out, want)
    s.append_quantized(new, new, 0)
    s.decode_quantized(q)
    assert s.status() == 0
