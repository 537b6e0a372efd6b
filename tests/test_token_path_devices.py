"""Tensors, caches and frequencies that are not all on one GPU are refused before the library sees a pointer; no GPU is needed: the GPU
tensors here are fake ones, which have a device and no memory."""
import numpy as np
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2511_10645_amd as paro
from paper_2511_10645_amd import binding as B


@pytest.fixture(params=["native", "ctypes"])
def host(request):
    native = B._native()
    B._host = native if request.param == "native" else B._CtypesCalls
    yield
    B._host = native


def gpu(*shape, dtype=torch.float16, at=0):
    with FakeTensorMode():
        return torch.empty(shape, dtype=dtype, device=f"cuda:{at}")


def rows(at=0):
    return gpu(3, 128, at=at)


def ints(at=0):
    return gpu(3, dtype=torch.int32, at=at)


def longs(at=0):
    return gpu(3, dtype=torch.int64, at=at)


def table(at=0):
    return gpu(3, 2, dtype=torch.int32, at=at)


def workspace(buf):
    ws = paro.Workspace(1 << 12, device="cpu")
    ws.buf = buf
    return ws


def refused(call, *why):
    with pytest.raises(AssertionError, match="|".join(why) if why else None):
        call()


def test_cache_and_frequencies_in_host_memory(host):
    cache, rope = paro.KVCache(2, 2, 64, 16, "e4m3", device="cpu"), paro.Rope(np.ones(32, np.float32), 64, device="cpu")
    ws = workspace(gpu(1 << 12, dtype=torch.uint8))
    refused(lambda: paro.paro_rope(rope, rows(), ints()), "one GPU")
    refused(lambda: paro.paro_kv_append(cache, rows(), rows(), longs()), "one GPU")
    refused(lambda: paro.paro_paged_attention(cache, rows(), table(), ints(), ws), "one GPU")
    cache.c.device = 0                                                  # the frequencies alone
    refused(lambda: paro.paro_kv_append(cache, rows(), rows(), longs(), rope, ints(), rows()), "one GPU")


def test_tensors_of_two_gpus(host):
    cache, rope = paro.KVCache(2, 2, 64, 16, device="cpu"), paro.Rope(np.ones(32, np.float32), 64, device="cpu")
    cache.c.device = rope.c.device = 0
    w, buf = gpu(128), gpu(1 << 12, dtype=torch.uint8)
    norm, quantised, append, attend = paro.paro_rms_norm, paro.paro_rms_norm_quantize_e4m3, paro.paro_kv_append, paro.paro_paged_attention
    for call in (lambda: norm(rows(), gpu(128, at=1), 1e-5), lambda: norm(rows(), w, 1e-5, residual=rows(1)), lambda: quantised(rows(), gpu(128, at=1), 1e-5),
                 lambda: quantised(rows(), w, 1e-5, residual=rows(1)),
                 lambda: paro.paro_rope(rope, rows(), ints(1)), lambda: paro.paro_rope(rope, rows(1), ints(1)),
                 lambda: append(cache, rows(), rows(1), longs()), lambda: append(cache, rows(), rows(), longs(1)), lambda: append(cache, rows(1), rows(1), longs(1)),
                 lambda: append(cache, rows(), rows(), longs(), rope, ints(1)), lambda: append(cache, rows(), rows(), longs(), rope, ints(), rows(1)),
                 lambda: attend(cache, rows(), table(1), ints(), workspace(buf)), lambda: attend(cache, rows(), table(), ints(1), workspace(buf)),
                 lambda: attend(cache, rows(), table(), ints(), workspace(gpu(1 << 12, dtype=torch.uint8, at=1))),
                 lambda: attend(cache, rows(1), table(1), ints(1), workspace(gpu(1 << 12, dtype=torch.uint8, at=1)))):
        refused(call, "one GPU")


def test_caches_and_frequencies_take_one_device():
    k, v, s = torch.zeros((2, 2, 4, 16, 16), dtype=torch.uint8), torch.zeros((2, 2, 16, 64), dtype=torch.uint8), torch.zeros((2, 2, 16), dtype=torch.uint8)
    assert paro.KVCache.from_device(k, v, s, s.clone()).c.device == -1
    for i in range(4):
        parts = [k, v, s, s.clone()]
        parts[i] = parts[i].to("meta")
        refused(lambda: paro.KVCache.from_device(*parts))
    refused(lambda: paro.KVCache.from_device(k, v, s))                 # scales of both or of neither
    refused(lambda: paro.KVCache.from_device(k.half(), v.half(), None, s))
    assert paro.Rope(torch.ones(32), 64, device="meta").inv_freq.device.type == "meta"      # a tensor goes where an array goes
    assert paro.Rope(torch.ones(32), 64, device="cpu").c.device == -1
