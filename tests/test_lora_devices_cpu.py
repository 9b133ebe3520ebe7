"""Calls with adapters refuse what lies on another device than they run on, before the library sees an address (CPU; the other device is torch's meta)."""
import types

import pytest
import torch


class Called(Exception):
    pass


@pytest.fixture
def qt(monkeypatch):
    import paper_2602_10431_amd as pkg
    from paper_2602_10431_amd import binding

    def load():
        raise Called
    monkeypatch.setattr(binding, "load_library", load)
    return pkg


N, K = 16, 64


def _lora(qt, device, rank_on=None):
    half = dict(dtype=torch.float16, device=device)
    rank = None if rank_on is None else torch.full((2,), 8, dtype=torch.int32, device=rank_on)
    return qt.Lora(torch.zeros(2, 8, K, **half), torch.zeros(2, N, 8, **half), rank)


def _linear(qt, device):
    return qt.QuantLinear(N, K, 4, 64, None, None, None, torch.zeros(256, dtype=torch.uint8, device=device))


def test_linears(qt):
    A, ids = torch.zeros(3, K, dtype=torch.float16), torch.zeros(3, dtype=torch.int32)
    here, there = _lora(qt, "cpu"), _lora(qt, "meta")
    with pytest.raises(Called):
        qt.qtale_linear_lora_w4a16(_linear(qt, "cpu"), here, A, ids)
    for linear, lora, x, i in ((_linear(qt, "meta"), here, A, ids), (_linear(qt, "cpu"), there, A, ids), (_linear(qt, "cpu"), here, A.to("meta"), ids),
                               (_linear(qt, "cpu"), here, A, ids.to("meta"))):
        with pytest.raises(AssertionError):
            qt.qtale_linear_lora_w4a16(linear, lora, x, i)
    good = _linear(qt, "cpu")
    with pytest.raises(Called):
        qt.qtale_swiglu_lora_w4a16(good, good, here, here, A, ids)
    for gate, up, lg, lu in ((good, good, here, there), (good, good, there, here), (good, _linear(qt, "meta"), here, None), (_linear(qt, "meta"), good, None, here)):
        with pytest.raises(AssertionError):
            qt.qtale_swiglu_lora_w4a16(gate, up, lg, lu, A, ids)
    with pytest.raises(AssertionError):
        _lora(qt, "cpu", "meta")


def test_layers(qt):
    ints = lambda *n: torch.zeros(n, dtype=torch.int32)
    pages = torch.zeros(4, 1, 16, 64, dtype=torch.float16)
    kv = qt.PagedKV(pages, pages.clone(), ints(4), ints(1), ints(1, 2, 2), ints(1, 2), ints(1, 2))
    stack = types.SimpleNamespace(n=1, kvs=None, cfg=qt.make_cfg(64, 1, 1, 64, 64))
    rope = types.SimpleNamespace(freqs=torch.zeros(32, dtype=torch.float64))
    x = torch.zeros(3, 64, dtype=torch.float16)
    call = lambda loras, ids=ints(1): qt.qtale_paged_stack_forward(None, stack, x, ints(2), ints(3), kv, rope, loras=loras, adapter=ids)
    with pytest.raises(Called):
        call(qt.StackLora([{"q": _lora(qt, "cpu")}]))
    with pytest.raises(AssertionError):
        call(qt.StackLora([{"q": _lora(qt, "meta")}]))
    with pytest.raises(AssertionError):                           # one of several, of any layer
        call(qt.StackLora([{"q": _lora(qt, "cpu"), "gate": _lora(qt, "meta")}]))
    with pytest.raises(AssertionError):
        call(qt.StackLora([{"q": _lora(qt, "cpu")}]), ints(1).to("meta"))
