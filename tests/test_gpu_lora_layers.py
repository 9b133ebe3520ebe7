"""Layers with adapters on the GPU (run with -m gpu) at their ends: calls of many tokens none of which executes a layer, layers without adapters among others."""
import pytest
import torch

import synth_inputs as si
from tests.paged_helpers import ints
from tests.test_gpu_serving_stack import NAMES, _context, _loras, _stack

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qt():
    import paper_2602_10431_amd as pkg
    pkg.load_library()
    return pkg


@pytest.mark.parametrize("T", [1, 3, 40, 257, 700, 2100])
@pytest.mark.parametrize("bits", [4, 16])
def test_no_token_executes(qt, T, bits):
    # the count of executed rows is 0 on the device alone; what lies in the scratch names sequences and adapters that there are not
    shape, L = si.LayerShape(256, 4, 2, 64, 512, 4, 32, "fp16"), 2
    stack, ctx, rope = _stack(qt, shape, L), _context(qt, "threshold", 1.0), qt.Rope(64)
    loras = qt.StackLora([_loras(qt, shape, NAMES, 4, 16, l)[0] for l in range(L)])
    kv = qt.PagedKV.empty(T // 16 + 4, 16, 2, 64, 2, T // 16 + 2, L, bits=bits)
    lens = [T - T // 3, T // 3]
    offs, pos = (t.cuda() for t in si.ragged_sequences(lens, [0, 0]))
    ws = qt.alloc_paged_stack_workspace(stack.cfg, kv, T, 2, loras)
    x = si.hidden_states(shape, T, 3).cuda()
    before = x.clone()
    for fill in (0, 1, 127, 255):
        ws.fill_(fill)
        count = ints([-1] * L)
        qt.qtale_paged_stack_forward(ctx, stack, x, offs, pos, kv, rope, max_new=max(lens), sel_count=count, loras=loras, adapter=ints([1, 3]), workspace=ws)
        assert count.tolist() == [0] * L
        assert torch.equal(x, before) and int(kv.kv_len.sum()) == 0
    # and the same scratch serves a call whose tokens all execute
    y = x.clone()
    qt.qtale_paged_stack_forward(_context(qt, "ratio", 1.0), stack, x, offs, pos, kv, rope, max_new=max(lens), loras=loras, adapter=ints([1, 3]), workspace=ws)
    qt.qtale_pages_release(kv)
    qt.qtale_paged_stack_forward(_context(qt, "ratio", 1.0), stack, y, offs, pos, kv, rope, max_new=max(lens), loras=loras, adapter=ints([1, 3]))
    assert torch.equal(x, y) and not torch.equal(x, before)


@pytest.mark.parametrize("T", [1, 2, 4, 5, 60])
def test_layers_without_adapters_run_as_in_a_plain_stack(qt, T):
    # the same launches, and the same bits: a handful of tokens have their decision and norms inside the products' launches
    shape, L = si.LayerShape(256, 4, 2, 64, 512, 4, 32, "bf16"), 4
    stack, ctx, rope = _stack(qt, shape, L), _context(qt, "ratio", 1.0), qt.Rope(64)
    some = _loras(qt, shape, NAMES, 4, 16, 1)[0]
    mixed = qt.StackLora([some, {}, {}, {}])
    offs, pos = (t.cuda() for t in si.ragged_sequences([T], [0]))
    outs, launches = [], []
    for first in (qt.StackLora([some]), mixed):                    # the first layer, then the others as a plain stack; all four in one call
        kv = qt.PagedKV.empty(4 * (T // 16 + 2), 16, 2, 64, 1, T // 16 + 2, L)
        x = si.hidden_states(shape, T, 3).cuda()
        qt.qtale_paged_stack_forward(ctx, qt.Stack(stack.cfg, stack.layers[: first.n]), x, offs, pos, kv, rope, loras=first, adapter=ints([2]))
        if first.n == 1:
            qt.qtale_paged_stack_forward(ctx, qt.Stack(stack.cfg, stack.layers[1:]), x, offs, pos, kv, rope, first_layer=1)
        outs.append(x)
    assert torch.equal(outs[0], outs[1])
    for n, loras in ((3, None), (4, mixed), (1, qt.StackLora([some]))):
        kv = qt.PagedKV.empty(4 * (T // 16 + 2), 16, 2, 64, 1, T // 16 + 2, L)
        qt.qtale_profile_enable(ctx, True)
        qt.qtale_paged_stack_forward(ctx, qt.Stack(stack.cfg, stack.layers[4 - n if loras is None else 0:][:n]), si.hidden_states(shape, T, 3).cuda(), offs, pos, kv, rope,
                                     loras=loras, adapter=None if loras is None else ints([2]))
        launches.append({k: v[1] for k, v in qt.qtale_profile_read(ctx).items()})
        qt.qtale_profile_enable(ctx, False)
    plain, all_four, adapted = launches
    for k in ("select", "norm1", "norm2", "qkv_gemm"):            # (scores of a layer are part of the one before it in a stack)
        assert all_four[k] == plain[k] + adapted[k], (k, launches)
