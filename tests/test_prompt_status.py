"""A wait of the prompt attention that gave up is reported to every stream that is checked: one check takes nothing from
another, whichever comes first and whichever stream the call was on."""
import ctypes as C
import glob
import os
import threading

import pytest
import torch

import paper_2503_23956_b200 as ac
from test_prompt_attn import check, inputs


def runtime():
    found = glob.glob(os.path.join(os.path.dirname(torch.__file__), "..", "nvidia", "cuda_runtime", "lib", "libcudart.so*"))
    return C.CDLL(sorted(found)[-1] if found else "/usr/local/cuda/lib64/libcudart.so")


def status(stream=None):
    return ac.aircache_prompt_check_status(stream, check=False)


@pytest.mark.gpu
def test_each_stream_is_told_once():
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for s in (a, b, None):
        status(s)   # (whatever was before)
    for s in (a, b, None):
        assert status(s) == ac.OK
    for first, then in ((a, b), (b, a)):
        ac.aircache_selftest_prompt_timeout(a)
        torch.cuda.synchronize()
        assert status(first) == ac.ERR_TIMEOUT   # (of b's check in front of a's: not b's call, but told all the same)
        assert status(then) == ac.ERR_TIMEOUT
        assert status(first) == ac.OK and status(then) == ac.OK
    assert status() == ac.ERR_TIMEOUT and status() == ac.OK
    with pytest.raises(ac.AirCacheError):
        ac.aircache_selftest_prompt_timeout(b)
        ac.aircache_prompt_check_status(b)
    assert status() == ac.ERR_TIMEOUT
    check(*inputs(300, 300, 8, 2, 64), [300], [300])   # goes on as before


@pytest.mark.gpu
def test_checks_of_several_threads():
    streams = [torch.cuda.Stream() for _ in range(4)]
    for s in streams + [None]:
        status(s)
    ac.aircache_selftest_prompt_timeout(streams[0])
    torch.cuda.synchronize()
    got = [None] * 4

    def run(i):
        got[i] = [status(streams[i].cuda_stream) for _ in range(20)]

    threads = [threading.Thread(target=run, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert got == [[ac.ERR_TIMEOUT] + [ac.OK] * 19] * 4
    assert status() == ac.ERR_TIMEOUT and status() == ac.OK


@pytest.mark.gpu
def test_more_streams_than_are_remembered():
    """Those forgotten are told again, none is left out."""
    status()
    ac.aircache_selftest_prompt_timeout()
    torch.cuda.synchronize()
    made = [C.c_void_p() for _ in range(300)]
    rt = runtime()
    for s in made:
        assert rt.cudaStreamCreateWithFlags(C.byref(s), 1) == 0
    assert all(status(s.value) == ac.ERR_TIMEOUT for s in made)
    assert status(made[-1].value) == ac.OK
    status()
    assert status() == ac.OK
    for s in made:
        assert rt.cudaStreamDestroy(s) == 0
