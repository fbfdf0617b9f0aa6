"""Host side of the 4-bit generation calls that needs no GPU: refusals without a context, argument checks of the binding, and
the plain forms that the GPU tests compare with."""
import ctypes as C

import numpy as np
import pytest
import torch

import generate4_ref as R


@pytest.fixture(scope="module")
def lib():
    from paper_2601_13155_b200 import binding, build
    build.build()
    return binding.load_library()


def test_calls_without_a_context_are_refused(lib):
    from paper_2601_13155_b200 import binding
    w, c, r = binding.W4C(), binding.Kv4CacheC(), binding.LogitsRulesC()
    assert lib.spts_w4_quantize(None, None, 1, 32, 32, None, None) == 1
    assert lib.spts_w4_gemv(None, C.byref(w), None, None, 0, 1, None, 0, 0, None, 0) == 1
    assert lib.spts_kv4_append(None, C.byref(c), None, 0, None, 0, None, None, None, 1, None, None) == 1
    assert lib.spts_kv4_attention(None, C.byref(c), None, 0, None, 0) == 1
    assert lib.spts_process_logits(None, None, 0, 1, 1, C.byref(r), None, 0, None) == 1


def test_host_tensors_and_wrong_forms_are_refused():
    from paper_2601_13155_b200 import binding, synth
    with pytest.raises(ValueError):
        binding.W4Weight(torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(4, 1, 2, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        binding.W4Weight(torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(4, 1, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        binding.Kv4Cache(synth.TINY, 2, 32, group=128, device="cpu")
    with pytest.raises(ValueError):
        binding.LogitsRules(history=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError):
        binding.LogitsRules(mask=torch.zeros(3, dtype=torch.int32))


def test_storage_orders_hold_every_dim_once():
    for d in (64, 128):
        for dims in (R.key_dims(d), R.value_dims(d)):
            assert sorted(dims) == list(range(d))
    assert list(R.key_dims(64)[:18]) == [0, 1, 2, 3, 4, 5, 6, 7, 32, 33, 34, 35, 36, 37, 38, 39, 8, 9]
    assert list(R.value_dims(64)[:10]) == [0, 1, 2, 3, 32, 33, 34, 35, 4, 5]


def test_quantiser_stays_within_half_a_step():
    rng = np.random.default_rng(1)
    x = R.bf16(rng.normal(size=(50, 128)))
    codes, scale, mid, vals = R.quantise(x, 32)
    s = np.repeat(scale, 32, -1)
    # half a step; the scale rounded down by up to half a bf16 step shortens the range of 15 steps by 15 * 2^-8 / 2 at
    # either end, and the rounded mid shifts it by up to 2^-8 |mid|
    slack = 0.5 * s + 7.5 * 2.0 ** -8 * s + 2.0 ** -8 * np.abs(np.repeat(mid, 32, -1))
    assert (np.abs(vals - x) <= slack + 1e-12).all()
    assert codes.min() == 0 and codes.max() == 15
