"""Host side of the paged-cache calls that needs no GPU: refusals without a context, the binding's checks, and the plain forms that the
GPU tests compare with."""
import ctypes as C
import math
from types import SimpleNamespace

import pytest
import torch

import paged_ref as R
from paper_2601_13155_b200 import binding, synth


@pytest.fixture(scope="module")
def lib():
    from paper_2601_13155_b200 import build
    build.build()
    return binding.load_library()


def test_calls_without_a_context_are_refused(lib):
    c = C.byref(binding.PagedKvC())
    assert lib.spts_paged_append(None, c, None, 0, None, 0, None, None, None, 1) == 1
    assert lib.spts_paged_attention(None, c, None, 0, None, 1, None, 0, None) == 1
    assert lib.spts_paged_weights(None, c, None, 0, None, 1, None, 1.0) == 1
    assert lib.spts_paged_evict(None, c, None, 0, 0) == 1
    assert lib.spts_token_logprobs(None, None, 0, 1, 1, None, 0, None, None, None, None, None) == 1


def test_host_tensors_and_wrong_forms_are_refused():
    table = torch.zeros(2, 4, dtype=torch.int32)
    with pytest.raises(ValueError):
        binding.PagedKv(synth.TINY, table, page_size=64, n_pages=8)          # a host tensor
    with pytest.raises(ValueError):
        binding.PagedKv(synth.TINY, table, page_size=48, n_pages=8)          # no such page


def context():
    """A context whose library records the calls that reach it."""
    lib = binding.Spts.__new__(binding.Spts)
    called = []
    take = lambda *a: called.append(a) or 0
    lib.lib = SimpleNamespace(spts_paged_append=take, spts_paged_attention=take, spts_paged_weights=take, spts_paged_evict=take,
                              spts_token_logprobs=take, spts_destroy=lambda h: None)
    lib.h, lib.shape, lib.dev, lib.dtype, lib.device = 1, synth.TINY, 0, binding.torch_dtype(synth.TINY.dtype), "cpu"
    return lib, called


def tensor(*size, dtype=None, device=0):
    dtype = dtype or binding.torch_dtype(synth.TINY.dtype)
    strides = [math.prod(size[i + 1:]) for i in range(len(size))]
    return SimpleNamespace(shape=size, dtype=dtype, get_device=lambda: device, is_cuda=True, is_contiguous=lambda: True, dim=lambda: len(size),
                           numel=lambda: math.prod(size), data_ptr=lambda: 256, device=f"cuda:{device}",
                           stride=lambda i=None: strides if i is None else strides[i])


def cache(**kw):
    s = synth.TINY
    full = dict(heads=(s.n_kv_heads, s.head_dim), dtype=binding.torch_dtype(s.dtype), device_index=0, n_seq=2, c=None, weight=1, pos=1)
    return SimpleNamespace(**{**full, **kw})


@pytest.mark.parametrize("kw", [dict(heads=(1, 64)), dict(dtype=torch.float16), dict(device_index=1)], ids=["heads", "type", "device"])
def test_caches_of_another_kind_are_refused(kw):
    lib, called = context()
    s, i32 = synth.TINY, torch.int32
    kv, q = tensor(2, s.n_kv_heads, s.head_dim), tensor(2, s.n_q_heads, s.head_dim)
    with pytest.raises(ValueError):
        lib.paged_append(cache(**kw), kv, kv)
    with pytest.raises(ValueError):
        lib.paged_attention(cache(**kw), q, O_out=tensor(2, s.n_q_heads * s.head_dim))
    with pytest.raises(ValueError):
        lib.paged_weights(cache(**kw), q, tensor(2, s.n_q_heads, dtype=torch.float32))
    with pytest.raises(ValueError):
        lib.paged_evict(cache(**kw), tensor(2, dtype=i32))
    assert not called


def test_tensors_of_other_sizes_types_and_devices_are_refused():
    lib, called = context()
    s, i32, f32 = synth.TINY, torch.int32, torch.float32
    kv, q, o = tensor(2, s.n_kv_heads, s.head_dim), tensor(2, s.n_q_heads, s.head_dim), tensor(2, s.n_q_heads * s.head_dim)
    lse = tensor(2, s.n_q_heads, dtype=f32)
    bad = [lambda: lib.paged_append(cache(), kv, tensor(3, s.n_kv_heads, s.head_dim)),
           lambda: lib.paged_append(cache(), kv, kv, row_start=tensor(2, dtype=i32)),
           lambda: lib.paged_append(cache(), kv, kv, at=tensor(2, dtype=torch.int64)),
           lambda: lib.paged_append(cache(), kv, kv, pos=tensor(3, dtype=i32)),
           lambda: lib.paged_append(cache(), tensor(2, s.n_kv_heads, s.head_dim, device=1), kv),
           lambda: lib.paged_attention(cache(), q, O_out=tensor(3, s.n_q_heads * s.head_dim)),
           lambda: lib.paged_attention(cache(), q, O_out=o, lse_out=tensor(3, s.n_q_heads, dtype=f32)),
           lambda: lib.paged_attention(cache(), kv, O_out=o),
           lambda: lib.paged_weights(cache(), q, tensor(1, s.n_q_heads, dtype=f32)),
           lambda: lib.paged_weights(cache(weight=None), q, lse),
           lambda: lib.paged_evict(cache(), tensor(3, dtype=i32)),
           lambda: lib.paged_evict(cache(weight=None), tensor(2, dtype=i32)),
           lambda: lib.paged_evict(cache(pos=None), tensor(2, dtype=i32), n_recent=1),
           lambda: lib.token_logprobs(tensor(2, 50, dtype=f32), n_top=33),
           lambda: lib.token_logprobs(tensor(2, 50, dtype=torch.bfloat16)),
           lambda: lib.token_logprobs(tensor(2, 50, dtype=f32), tensor(3, dtype=i32))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    assert not called
    lib.paged_append(cache(), kv, kv, row_start=tensor(3, dtype=i32), at=tensor(2, dtype=i32), pos=tensor(2, dtype=i32))
    lib.paged_attention(cache(), q, O_out=o, lse_out=lse)
    lib.paged_weights(cache(), q, lse)
    lib.paged_evict(cache(pos=None), tensor(2, dtype=i32))
    assert len(called) == 4


def test_plain_attention_is_its_formula():
    g = torch.Generator().manual_seed(0)
    q, k, v = torch.randn(5, 4, 8, generator=g), torch.randn(7, 2, 8, generator=g), torch.randn(7, 2, 8, generator=g)
    o, _, lse, _ = R.attention(q, k, v, 1, torch.float32)
    for i in range(5):
        for h in range(4):
            s = [float(q[i, h].double() @ k[j, h // 2].double()) / math.sqrt(8) for j in range(1 + i + 1)]
            z = sum(math.exp(x) for x in s)
            assert abs(float(lse[i, h]) - math.log(z)) < 1e-12
            want = sum(math.exp(x) / z * v[j, h // 2].double() for j, x in enumerate(s))
            assert bool((o[i, h] - want).abs().max() < 1e-12)
    w, _ = R.weights(q, k, lse, 1)
    assert abs(float(w.sum()) - 5) < 1e-9                     # every query gives one, the mean over the heads


def test_plain_eviction_keeps_what_it_says():
    k = torch.arange(8.0)[:, None, None]
    pos, w = torch.tensor([0, 1, 2, 3, 5, 8, 9, 12]), torch.tensor([0.0, 0.1, 0.9, 0.1, 0.9, 0.1, 0.0, 0.0])
    kk, _, p, ww = R.evict(k, k, pos, w, 5, 1, 1)
    # row 0 (sink) and row 7 (newest) first, then rows 2 and 4, then the first of the three with 0.1; row 7 takes the hole of row 3
    assert kk.flatten().tolist() == [0, 1, 2, 7, 4] and p.tolist() == [0, 1, 2, 12, 5]
    assert R.evict(k, k, pos, w, 8, 1, 1)[2] is pos and R.evict(k, k, pos, w, -1, 1, 1)[2] is pos


def test_plain_log_probabilities_are_their_formula():
    x = torch.tensor([0.5, 2.0, 2.0, float("-inf"), -1.0])
    z = sum(math.exp(float(v)) for v in x)
    lp, rank, ent, top, tok, _, _ = R.logprobs(x, 2, 5)
    assert abs(lp - (2 - math.log(z))) < 1e-12 and rank == 1 and tok == [1, 2, 0, 4, -1] and top[4] == float("-inf")
    assert abs(ent + sum(math.exp(v) / z * (v - math.log(z)) for v in (0.5, 2.0, 2.0, -1.0))) < 1e-12
