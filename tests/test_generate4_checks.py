"""Checks of the binding before a 4-bit decode step that need no GPU: the embedding table and the devices of the weights.  The
objects stand in for device tensors; a step whose checks pass would reach the library, which here records the call."""
from types import SimpleNamespace

import pytest
import torch

from paper_2601_13155_b200 import binding, synth

SHAPE = synth.TINY
L, V, D = SHAPE.n_layers, SHAPE.vocab, SHAPE.hidden


def table(rows=V, width=D, dtype=torch.float32, device=0):
    return SimpleNamespace(shape=(rows, width), dtype=dtype, get_device=lambda: device, is_cuda=True, is_contiguous=lambda: True,
                           dim=lambda: 2, numel=lambda: rows * width, data_ptr=lambda: 256, device=f"cuda:{device}")


def weight(device=0):
    return SimpleNamespace(c=binding.W4C(), device_index=device)


def model(embed=None, layer_device=0, head_device=0):
    layers = [{n: weight(layer_device if n == "w_down" else 0) for n in ("wqkv", "wo", "w_gate", "w_up", "w_down")} for _ in range(L)]
    return binding.Model4(layers, weight(head_device), embed)


def step(m, **kw):
    """The calls that reached the library (0 or 1)."""
    called = []
    lib = binding.Spts.__new__(binding.Spts)
    lib.lib = SimpleNamespace(spts_decode_step4=lambda *a: called.append(a) or 0, spts_destroy=lambda h: None)
    lib.h, lib.shape, lib.dev, lib.dtype = 1, SHAPE, 0, torch.float32
    cache = SimpleNamespace(heads=(SHAPE.n_kv_heads, SHAPE.head_dim), device_index=0)
    caches = SimpleNamespace(n_seq=2, layers=[cache] * L, c=None)
    ints = SimpleNamespace(is_cuda=True, is_contiguous=lambda: True, dtype=torch.int32, numel=lambda: 2, get_device=lambda: 0, data_ptr=lambda: 512)
    lib.decode_step4(m, caches, ints, token_in=ints, **kw)
    return len(called)


def test_a_table_of_the_vocabulary_reaches_the_library():
    assert step(model(table())) == 1
    assert step(model(table(rows=V + 3))) == 1


@pytest.mark.parametrize("embed", [table(rows=V - 1), table(width=D - 8), table(dtype=torch.bfloat16), table(device=1)],
                         ids=["short", "narrow", "type", "device"])
def test_a_table_that_would_be_read_wrongly_is_refused(embed):
    with pytest.raises(ValueError):
        step(model(embed))


def test_a_table_that_the_step_does_not_read_is_not_looked_at():
    rows = SimpleNamespace(is_cuda=True, is_contiguous=lambda: True, dtype=torch.float32, numel=lambda: 2 * D, get_device=lambda: 0, data_ptr=lambda: 1024)
    assert step(model(table(rows=1)), x_in=rows) == 1
    assert step(model(), x_in=rows) == 1


def test_host_and_strided_tables_are_refused():
    with pytest.raises(ValueError):
        model(torch.zeros(V, D))
    flat = table()
    flat.dim = lambda: 1
    strided = table()
    strided.is_contiguous = lambda: False
    for t in (flat, strided):
        with pytest.raises(ValueError):
            model(t)


@pytest.mark.parametrize("where", [dict(layer_device=1), dict(head_device=1)])
def test_weights_of_another_device_are_refused(where):
    with pytest.raises(ValueError):
        step(model(table(), **where))
