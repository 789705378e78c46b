"""The calls over a cache of 8 bits and the log-probabilities, as far as they go without a GPU: what they refuse before they reach one."""
import ctypes

import pytest
import torch

from paper_1712_02912_amd import binding

NULL, NO = ctypes.c_void_p(), ctypes.c_float(0)
WIDE = ctypes.c_int64(1)


def test_calls_without_a_context_are_rejected():
    lib = ctypes.CDLL(binding.LIB_PATH)
    assert lib.pq_kv_append8(NULL, NULL, 0, NULL, 0, NULL, NULL, WIDE, NULL, NULL, NULL, NULL, WIDE, 0, 0, 0, NULL, NULL, NO, NULL) == -1
    assert lib.pq_kv_attention8(NULL, NULL, 0, NULL, 1, WIDE, NULL, NULL, 1, NULL, 1, 1, NO, 0, NULL, NULL) == -1
    assert lib.pq_token_logprobs(NULL, NULL, 0, WIDE, 1, 1, NULL, 0, NULL, NULL, NULL, NULL, NULL) == -1


def test_tensors_of_the_host_are_refused():
    ctx = binding.Context.__new__(binding.Context)
    ctx.lib, ctx.handle, ctx._address = binding.load(), ctypes.c_void_p(), None
    x, one = torch.zeros((1, 1, 64)), torch.ones(1, dtype=torch.int32)
    cache, scales = torch.zeros((1, 16, 1, 64)).to(torch.float8_e4m3fn), torch.ones((1, 1))
    for call in (lambda: ctx.pq_kv_append8(x, x, x, one, one.long(), cache, cache, scales, scales),
                 lambda: ctx.pq_kv_attention8(x, cache, cache, scales, scales, one.view(1, 1), one, one, 1), lambda: ctx.pq_token_logprobs(x[0])):
        with pytest.raises(TypeError, match="must be a GPU tensor"):
            call()


def test_wrong_numbers_of_arguments_are_refused():
    for f in (binding._views.append8, binding._views.attention8, binding._views.logprobs):
        with pytest.raises(TypeError, match="takes .* arguments"):
            f(1, 2, 3)
