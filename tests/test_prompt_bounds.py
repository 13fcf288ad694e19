"""aircache_prompt_attn inside larger buffers: offsets that point outside the rows declared are clamped to them, nothing else is
read (guard rows of NaN around queries, keys and values) or written (guard rows around the output); keys in a strided cache."""
import numpy as np
import pytest
import torch

import paper_2503_23956_b200 as ac
from test_prompt_attn import DEV, attend, formula, inputs

LOW, HIGH, GUARD = -(1 << 31), (1 << 31) - 1, 40


def inside(t):
    """The same rows in the middle of a buffer of NaN."""
    big = torch.full((t.shape[0] + 2 * GUARD,) + t.shape[1:], float("nan"), dtype=t.dtype, device=DEV)
    big[GUARD:GUARD + t.shape[0]] = t
    return big[GUARD:GUARD + t.shape[0]]


def run(q, k, v, q_off, k_off, causal):
    big = torch.full((q.shape[0] + 2 * GUARD,) + q.shape[1:], 7.0, dtype=torch.bfloat16, device=DEV)
    out = big[GUARD:GUARD + q.shape[0]]
    tensor = lambda o: None if o is None else torch.tensor(o, dtype=torch.int64).to(torch.int32).to(DEV)   # noqa: E731
    spec = ac.prompt(len(q_off) - 1, q.shape[0], k.shape[0], q.shape[1], k.shape[1], q.shape[2], None, causal)
    held = [inside(x) for x in (q, k, v)]   # (a view keeps no memory)
    ac.aircache_prompt_attn(spec, *[ac.tokens_view(x) for x in held], tensor(q_off), tensor(k_off), ac.tokens_view(out))
    assert ac.aircache_prompt_check_status() == 0
    assert (big[:GUARD] == 7).all() and (big[GUARD + q.shape[0]:] == 7).all()
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 1, 64), (14, 2, 128), (32, 32, 64)])
@pytest.mark.parametrize("causal", [1, 0])
@pytest.mark.parametrize("T,q_off,k_off", [
    (64, [LOW, 20, 40, HIGH], None),
    (300, [-5, 130, 1 << 30], None),
    (300, [0, 300, HIGH, HIGH], None),                    # sequences behind the buffer: none
    (300, [LOW, LOW, 150, 301], None),
    (200, [0, 64, HIGH], [LOW, 100, HIGH]),
    (200, [100, 150, 200], [-1, 1 << 30, HIGH]),           # rows in front of the first sequence; a second one without keys
])
def test_offsets_outside_the_buffers(T, q_off, k_off, causal, Hq, Hkv, d):
    Tk = T if k_off is None else T + 77
    q, k, v = inputs(T, Tk, Hq, Hkv, d, seed=T)
    got = run(q, k, v, q_off, k_off, causal).double()
    q_at, k_at = np.clip(q_off, 0, T), np.clip(q_off if k_off is None else k_off, 0, Tk)
    n_q, n_k = np.diff(q_at), np.diff(k_at)
    first, last, first_k = int(q_at[0]), int(q_at[-1]), int(k_at[0])
    want, tol = formula(q[first:], k[first_k:], v[first_k:], n_q.tolist(), n_k.tolist(), causal, 1 / np.sqrt(d))
    n = last - first
    assert ((got[first:last] - want[:n]).abs() <= tol[:n]).all()
    assert (got[:first] == 7).all() and (got[last:] == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("q_off,k_off", [([0, 150, 20, HIGH], None), ([150, 0, LOW, 200], [HIGH, 3, LOW, 100]),
                                         ([HIGH, LOW, HIGH, LOW], None)])
def test_offsets_in_no_order(q_off, k_off):
    """No meaning, and still nothing outside is read or written: what is written is finite."""
    got = run(*inputs(200, 260 if k_off else 200, 4, 1, 64), q_off, k_off, 1)
    assert got.isfinite().all()


@pytest.mark.gpu
@pytest.mark.parametrize("Hq,Hkv,d", [(28, 4, 128), (8, 2, 64), (64, 32, 128)])
def test_keys_in_a_strided_cache(Hq, Hkv, d):
    """A layer of [rows, K | V, heads, d] and of a head-major cache with room behind the rows, keys of many tiles."""
    n_q, n_k = [5, 300, 1], [700, 1290, 131]
    q, k, v = inputs(sum(n_q), sum(n_k), Hq, Hkv, d, seed=9)
    plain = attend(q, k, v, n_q, n_k)
    want, tol = formula(q, k, v, n_q, n_k, 1, 1 / np.sqrt(d))
    assert ((plain.double() - want).abs() <= tol).all()
    both = torch.full((sum(n_k), 2, Hkv, d), float("nan"), dtype=torch.bfloat16, device=DEV)
    both[:, 0], both[:, 1] = k, v
    assert torch.equal(attend(q, both[:, 0], both[:, 1], n_q, n_k), plain)
    major = torch.full((2, Hkv, sum(n_k) + 500, d + 8), float("nan"), dtype=torch.bfloat16, device=DEV)
    km, vm = (major[i, :, :sum(n_k), :d].transpose(0, 1) for i in range(2))
    km.copy_(k), vm.copy_(v)
    assert torch.equal(attend(q, km, vm, n_q, n_k), plain)
