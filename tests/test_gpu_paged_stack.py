"""Layers on a paged cache on the GPU (run with -m gpu): against the CPU oracle in both control modes, against the layers on a contiguous cache, pages
taken for executed tokens only, forks, a window, an empty pool, graphs.  References and tolerances are those of the other layer tests."""
import numpy as np
import pytest
import torch

import synth_inputs as si
from oracle import qtale_oracle as orc
from tests.helpers import cfg_dict, check_parity, oracle_layer, to_f64
from tests.paged_helpers import ints

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qt():
    import paper_2602_10431_amd as pkg
    pkg.load_library()
    return pkg


def _context(qt, mode, value):
    ctx = qt.Context()
    (qt.qtale_set_exec_ratio if mode == "ratio" else qt.qtale_set_threshold)(ctx, value)
    return ctx


def _entries(kv, layer, slot, n):
    """The first n entries of a slot, token-major float64 [n, kv heads * head size]."""
    row, P = kv.table[layer, slot].tolist(), kv.page_size
    pick = lambda pool: np.stack([to_f64(pool[row[j // P], :, j % P]).reshape(-1) for j in range(n)]) if n else np.zeros((0, 1))
    return pick(kv.k), pick(kv.v)


def _oracle_case(qt, shape, lens, old, page, mode, value, seed, layer=1):
    T, B = sum(lens), len(lens)
    tensors = si.layer_tensors(shape, 0, seed, unit_gains=False, std=1.28 / shape.hidden ** 0.5)
    x = si.hidden_states(shape, T, seed)
    offs, pos = si.ragged_sequences(lens, old)
    cap = max(o + n for o, n in zip(old, lens)) + 1
    kc, vc = si.kv_cache(shape, B, cap, 0, seed)
    kv = qt.PagedKV.empty(sum(-(-(o + n) // page) for o, n in zip(old, lens)) + 5, page, shape.n_kv_heads, shape.head_dim, B + 2, -(-cap // page) + 1, 3)
    kv.k.fill_(float("nan"))
    kv.v.fill_(float("nan"))
    slots = np.random.default_rng(seed).permutation(B + 2)[:B].tolist()
    # the cached tokens: room by the library, contents as given
    qt.qtale_pages_reserve(kv, ints([0] + np.cumsum(old).tolist()), slots=ints(slots), layer=layer, first=ints([0] * B))
    for b in range(B):
        row = kv.table[layer, slots[b]].tolist()
        for j in range(old[b]):
            kv.k[row[j // page], :, j % page] = kc[b, j].view(shape.n_kv_heads, -1).cuda()
            kv.v[row[j // page], :, j % page] = vc[b, j].view(shape.n_kv_heads, -1).cuda()
    stack = qt.Stack(qt.cfg_from_shape(shape), [qt.quantize_layer(tensors, shape.bits, shape.group)])
    xg, idx, cnt, missing = x.cuda(), ints([-1] * T), ints([-1]), ints([-1])
    qt.qtale_paged_stack_forward(_context(qt, mode, value), stack, xg, offs.cuda(), pos.cuda(), kv, qt.Rope(shape.head_dim, shape.rope_base), slots=ints(slots),
                                 first_layer=layer, max_new=max(lens), missing=missing, sel_idx=idx, sel_count=cnt)
    got, k = xg.cpu(), int(cnt.item())
    p, _ = oracle_layer(shape, 0, seed, tensors=tensors)
    okv = orc.KVCache(to_f64(kc), to_f64(vc), old)
    want, widx, _ = orc.layer_forward(to_f64(x), p, cfg_dict(shape), offs.numpy(), pos.numpy(), mode, value, okv)
    assert missing.item() == (0 if len(widx) or mode == "threshold" else -1)
    assert np.array_equal(idx[:k].cpu().numpy(), widx)
    skipped = np.setdiff1d(np.arange(T), widx)
    assert torch.equal(got[skipped], x[skipped])
    if len(widx):
        check_parity(orc.parity_error(to_f64(got)[widx], want[widx]), shape.act_dtype, ("paged", shape.hidden, shape.bits, T), hidden=shape.hidden)
    for b in range(B):
        n0, n1 = old[b], int(okv.kv_len[b])
        assert int(kv.kv_len[layer, slots[b]]) == n1 and int(kv.kv_cap[layer, slots[b]]) == -(-n1 // page) * page   # pages for executed tokens only
        gk, gv = _entries(kv, layer, slots[b], n1)
        assert np.array_equal(gk[:n0], okv.k[b, :n0]) if n0 else True
        if n1 > n0:
            check_parity(orc.parity_error(gk[n0:], okv.k[b, n0:n1]), "fp16", "appended keys")
            check_parity(orc.parity_error(gv[n0:], okv.v[b, n0:n1]), "fp16", "appended values")
    assert int(kv.kv_len.sum()) == int(sum(okv.kv_len)) and int(kv.page_refs.sum()) == sum(-(-int(n) // page) for n in okv.kv_len)


@pytest.mark.parametrize("mode,value", [("ratio", 0.6), ("ratio", 1.0), ("ratio", 0.0), ("threshold", 0.5), ("threshold", 0.99)])
@pytest.mark.parametrize("nh,nkv,d", [(4, 4, 64), (8, 2, 128), (6, 2, 64)])
def test_layer_against_the_oracle(qt, mode, value, nh, nkv, d):
    shape = si.LayerShape(256, nh, nkv, d, 512, 4, 32, "fp16" if nkv == 4 else "bf16")
    _oracle_case(qt, shape, [1] * 8, [37, 5, 100, 64, 1, 99, 0, 63], 16, mode, value, 31)            # decode, selection with the first norm
    _oracle_case(qt, shape, [1, 1], [130, 1500], 64, mode, value, 32)                                # in the GEMM's prologue
    _oracle_case(qt, shape, [90, 0, 33, 150, 1], [0, 7, 64, 31, 500], 32, mode, value, 33)           # chunks beside single tokens
    _oracle_case(qt, shape, [300, 201], [0, 70], 128, mode, value, 34)                               # selection of its own


@pytest.mark.parametrize("bits", [2, 3])
def test_layer_with_other_code_widths(qt, bits):
    _oracle_case(qt, si.LayerShape(256, 8, 4, 64, 512, bits, 64, "bf16"), [5, 1, 40], [20, 64, 0], 16, "ratio", 0.7, 40 + bits)


def _stack(qt, shape, L, seed=3):
    return qt.Stack(qt.cfg_from_shape(shape), [qt.quantize_layer(si.layer_tensors(shape, l, seed, unit_gains=False, std=1.28 / shape.hidden ** 0.5), shape.bits, shape.group)
                                               for l in range(L)])


@pytest.mark.parametrize("mode,value", [("ratio", 1.0), ("ratio", 0.5), ("threshold", 0.5)])
def test_stack_beside_the_contiguous_cache(qt, mode, value):
    # a prompt and ten decode steps, each layer of the paged stack fed the contiguous stack's own layer inputs; lengths agree exactly
    shape, L, B, page = si.LayerShape(256, 8, 2, 64, 512, 4, 32, "fp16"), 3, 3, 16
    stack = _stack(qt, shape, L)
    ctx, rope = _context(qt, mode, value), qt.Rope(64, shape.rope_base)
    kv = qt.PagedKV.empty(80, page, 2, 64, B, 10, L)
    flat = [qt.KVCache(*(torch.zeros(B, 2, 128, 64, dtype=torch.float16, device="cuda") for _ in range(2)), ints([0] * B)) for _ in range(L)]
    with_cache = qt.Stack(stack.cfg, stack.layers, flat)
    singles = [qt.Stack(stack.cfg, [w]) for w in stack.layers]
    lens, done = [40, 17, 1], [0] * B
    for step in range(11):
        offs, pos = si.ragged_sequences(lens, done)
        T = sum(lens)
        x = si.hidden_states(shape, T, 50 + step).cuda()
        dbg = torch.empty(L, T, shape.hidden, dtype=x.dtype, device="cuda")
        idx, idx2 = ints([-1] * (L * T)).view(L, T), ints([-1] * (L * T)).view(L, T)
        qt.qtale_stack_forward(ctx, with_cache, x, offs.cuda(), pos.cuda(), sel_idx=idx, dbg_hidden=dbg)
        for l in range(L):
            y = dbg[l].clone()
            qt.qtale_paged_stack_forward(ctx, singles[l], y, offs.cuda(), pos.cuda(), kv, rope, first_layer=l, max_new=max(lens), sel_idx=idx2[l])
            want = dbg[l + 1] if l + 1 < L else x
            check_parity(orc.parity_error(to_f64(y), to_f64(want)), "fp16", "paged beside contiguous", hidden=shape.hidden)
            assert kv.kv_len[l].tolist() == flat[l].kv_len.tolist()
        assert torch.equal(idx, idx2)
        done, lens = [a + n for a, n in zip(done, lens)], [1] * B
    for l in range(L):
        for b in range(B):
            n = int(kv.kv_len[l, b])
            k, v = _entries(kv, l, b, n)
            check_parity(orc.parity_error(k, to_f64(flat[l].k_token_major()[b, :n])), "fp16", "keys")
            check_parity(orc.parity_error(v, to_f64(flat[l].v_token_major()[b, :n])), "fp16", "values")


def test_whole_stack_is_its_layers(qt):
    shape, L, B = si.LayerShape(256, 4, 4, 64, 512, 4, 32, "bf16"), 4, 5
    stack, ctx, rope = _stack(qt, shape, L), _context(qt, "ratio", 0.7), qt.Rope(64)
    a, b = (qt.PagedKV.empty(200, 16, 4, 64, B, 10, L) for _ in range(2))
    for step, lens in enumerate([[30, 3, 1, 50, 12], [1] * 5, [1] * 5]):
        offs, pos = si.ragged_sequences(lens, [step * 50] * B)
        x = si.hidden_states(shape, sum(lens), step).cuda()
        y, missing = x.clone(), ints([-1] * L)
        qt.qtale_paged_stack_forward(ctx, stack, x, offs.cuda(), pos.cuda(), a, rope, missing=missing)
        for l in range(L):
            qt.qtale_paged_stack_forward(ctx, qt.Stack(stack.cfg, [stack.layers[l]]), y, offs.cuda(), pos.cuda(), b, rope, first_layer=l)
        # (the stack links a layer's last kernel to the next one's scores: the same sums)
        assert torch.equal(x, y) and missing.tolist() == [0] * L
        for s, t in ((a.table, b.table), (a.kv_len, b.kv_len), (a.page_refs, b.page_refs)):
            assert torch.equal(s, t)


def test_forked_answers_are_those_of_separate_prompts(qt):
    shape, L = si.LayerShape(256, 4, 2, 64, 512, 4, 32, "fp16"), 2
    stack, ctx, rope = _stack(qt, shape, L), _context(qt, "ratio", 1.0), qt.Rope(64)
    forked, apart = (qt.PagedKV.empty(100, 16, 2, 64, 4, 10, L) for _ in range(2))
    prompt = si.hidden_states(shape, 43, 1).cuda()
    offs, pos = si.ragged_sequences([43], [0])
    qt.qtale_paged_stack_forward(ctx, stack, prompt.clone(), offs.cuda(), pos.cuda(), forked, rope)
    qt.qtale_pages_fork(forked, ints([0, 0]), ints([2, 3]))
    for s in (0, 2, 3):
        qt.qtale_paged_stack_forward(ctx, stack, prompt.clone(), offs.cuda(), pos.cuda(), apart, rope, slots=ints([s]))
    assert int((forked.page_refs > 0).sum()) == L * 3 and int((apart.page_refs > 0).sum()) == L * 9
    for step in range(8):
        offs, pos = si.ragged_sequences([1, 1, 1], [43 + step] * 3)
        x = si.hidden_states(shape, 3, 10 + step).cuda()
        y = x.clone()
        qt.qtale_paged_stack_forward(ctx, stack, x, offs.cuda(), pos.cuda(), forked, rope, slots=ints([0, 2, 3]), max_new=1)
        qt.qtale_paged_stack_forward(ctx, stack, y, offs.cuda(), pos.cuda(), apart, rope, slots=ints([0, 2, 3]), max_new=1)
        assert torch.equal(x, y)                                 # the same numbers on other pages
    assert int((forked.page_refs > 0).sum()) == L * (2 + 3 * 2)  # two full pages shared, the third and fourth of each its own


def test_a_window_with_trimmed_pages_and_a_compaction(qt):
    shape, L, W, S = si.LayerShape(256, 4, 2, 64, 512, 4, 32, "fp16"), 2, 40, 5
    stack, ctx, rope = _stack(qt, shape, L), _context(qt, "ratio", 1.0), qt.Rope(64)
    kept, trimmed = (qt.PagedKV.empty(60, 16, 2, 64, 2, 20, L) for _ in range(2))
    lens, done = [100, 30], [0, 0]
    for step in range(60):
        offs, pos = si.ragged_sequences(lens, done)
        x = si.hidden_states(shape, sum(lens), 10 + step).cuda()
        y = x.clone()
        qt.qtale_paged_stack_forward(ctx, stack, x, offs.cuda(), pos.cuda(), kept, rope, window=W, sinks=S, max_new=max(lens))
        qt.qtale_paged_stack_forward(ctx, stack, y, offs.cuda(), pos.cuda(), trimmed, rope, window=W, sinks=S, max_new=max(lens))
        assert torch.equal(x, y), step
        qt.qtale_pages_trim(trimmed, W, S)
        if step % 7 == 3:
            qt.qtale_pages_compact(trimmed)
        free = trimmed.page_refs == 0                            # what nobody holds is anything
        trimmed.k[free], trimmed.v[free] = float("nan"), float("nan")
        done, lens = [a + n for a, n in zip(done, lens)], [1, 1]
    assert int((trimmed.page_refs > 0).sum()) <= L * 2 * 5 < int((kept.page_refs > 0).sum())


def test_an_empty_pool_drops_the_newest_tokens(qt):
    # as a full contiguous cache does: the entries that are there are seen, lengths stop at the room
    shape = si.LayerShape(256, 4, 2, 64, 512, 4, 32, "fp16")
    stack, ctx, rope = _stack(qt, shape, 1), _context(qt, "ratio", 1.0), qt.Rope(64, shape.rope_base)
    kv = qt.PagedKV.empty(4, 16, 2, 64, 2, 10, 1)
    flat = qt.KVCache(*(torch.zeros(2, 2, 48, 64, dtype=torch.float16, device="cuda") for _ in range(2)), ints([0, 0]))
    with_cache = qt.Stack(stack.cfg, stack.layers, [flat])
    offs, pos = si.ragged_sequences([60, 5], [0, 0])
    x = si.hidden_states(shape, 65, 3).cuda()
    y, missing = x.clone(), ints([0])
    qt.qtale_pages_reserve(kv, ints([0, 0, 1]))                  # a page for the second sequence first: three are left for the first, which wants four
    qt.qtale_stack_forward(ctx, with_cache, y, offs.cuda(), pos.cuda())
    qt.qtale_paged_stack_forward(ctx, stack, x, offs.cuda(), pos.cuda(), kv, rope, missing=missing)
    assert missing.item() == 1 and kv.kv_len[0].tolist() == [48, 5] == flat.kv_len.tolist()
    check_parity(orc.parity_error(to_f64(x), to_f64(y)), "fp16", "full cache", hidden=shape.hidden)


def test_captured_decode_steps(qt):
    shape, L, B = si.LayerShape(256, 8, 2, 64, 512, 4, 32, "fp16"), 2, 6
    stack, ctx, rope = _stack(qt, shape, L), _context(qt, "threshold", 0.45), qt.Rope(64)
    a, b = (qt.PagedKV.empty(100, 16, 2, 64, B, 10, L) for _ in range(2))
    offs, pos = (t.cuda() for t in si.ragged_sequences([1] * B, [0] * B))
    x = si.hidden_states(shape, B, 0).cuda()
    ws = qt.alloc_paged_stack_workspace(stack.cfg, a, B, B)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qt.qtale_paged_stack_forward(ctx, stack, x, offs, pos, a, rope, max_new=1, workspace=ws)
    for step in range(40):
        x.copy_(si.hidden_states(shape, B, step))
        pos.fill_(step)
        y = x.clone()
        qt.qtale_paged_stack_forward(ctx, stack, y, offs, pos, b, rope, max_new=1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(x, y), step
        for s, t in ((a.table, b.table), (a.kv_len, b.kv_len), (a.free_bits, b.free_bits)):
            assert torch.equal(s, t)


def test_profile_classes_count_the_paged_launches(qt):
    shape = si.LayerShape(256, 4, 2, 64, 512, 4, 32, "fp16")
    stack, ctx = _stack(qt, shape, 2), _context(qt, "ratio", 1.0)
    kv = qt.PagedKV.empty(20, 16, 2, 64, 3, 5, 2)
    offs, pos = si.ragged_sequences([5, 6, 7], [0, 0, 0])
    qt.qtale_profile_enable(ctx, True)
    qt.qtale_paged_stack_forward(ctx, stack, si.hidden_states(shape, 18, 0).cuda(), offs.cuda(), pos.cuda(), kv, qt.Rope(64))
    prof = qt.qtale_profile_read(ctx)
    assert prof["rope_append"][1] == 2 and prof["attention"][1] == 2 and prof["attention"][0] > 0
