"""Layers on a cache in 4 bits, with adapters, and with both, on the GPU (run with -m gpu): against a 64-bit layer built from the oracle's pieces, requests
that come, fork and go over many steps, a stack against its layers, graphs, refusals.

The cache's codes hang on roundings of keys that the layer computes itself, so the 64-bit layer attends to the entries that the cache then holds (read back),
and those are held against the keys and values of the 64-bit layer: half a step, plus what the layer's own arithmetic is off (TOL of the row's
largest value, as everywhere in these tests) once for the value and, through the range, for up to 16 codes of a 15th of it."""
import ctypes as C

import numpy as np
import pytest
import torch

import synth_inputs as si
from oracle import qtale_oracle as orc
from tests.helpers import TOL, check_parity, oracle_layer, to_f64
from tests.paged_helpers import ints

pytestmark = pytest.mark.gpu
NAMES = ["q", "k", "v", "o", "gate", "up", "down"]


@pytest.fixture(scope="module")
def qt():
    import paper_2602_10431_amd as pkg
    pkg.load_library()
    return pkg


def _context(qt, mode, value):
    ctx = qt.Context()
    (qt.qtale_set_exec_ratio if mode == "ratio" else qt.qtale_set_threshold)(ctx, value)
    return ctx


def _tensors(shape, layer, seed):
    return si.layer_tensors(shape, layer, seed, unit_gains=False, std=1.28 / shape.hidden ** 0.5)


def _loras(qt, shape, names, n, r, seed, std=0.5):
    """One layer's adapters: {name: Lora}, and {name: [n matrices of the weights' change, float64]}."""
    g = torch.Generator().manual_seed(seed)
    out, change = {}, {}
    for name, N, K in shape.linear_shapes():
        if name not in names:
            continue
        down, up = (torch.randn(n, r, K, generator=g) / K ** 0.5).half(), (std * torch.randn(n, N, r, generator=g) / r ** 0.5).half()
        rank = torch.randint(1, r + 1, (n,), generator=g).int()
        scale = 0.5 + torch.rand(n, generator=g)
        out[name] = qt.Lora(down.cuda(), up.cuda(), rank.cuda(), scale.cuda())
        change[name] = [float(scale[a]) * to_f64(up[a, :, : rank[a]]) @ to_f64(down[a, : rank[a]]) for a in range(n)]
    return out, change


def _weights(p, change, a):
    """name -> weights of a sequence with adapter a."""
    base = dict(q=p.Wq, k=p.Wk, v=p.Wv, o=p.Wo, gate=p.Wg, up=p.Wu, down=p.Wd)
    return {n: base[n] + change[n][a] if change and n in change and 0 <= a < len(change[n]) else base[n] for n in NAMES}


def _layer64(x, p, change, adapters, shape, offs, positions, idx, cached, old):
    """Executed rows' outputs, keys and values [rows, nkv, d] in float64; cached[b]: keys and values that sequence b's slot holds after the call."""
    nh, nkv, d = shape.n_heads, shape.n_kv_heads, shape.head_dim
    xc = x[idx]
    out, keys, values = np.empty_like(xc), np.empty((len(idx), nkv, d)), np.empty((len(idx), nkv, d))
    for b in range(len(offs) - 1):
        rows = [i for i, t in enumerate(idx) if offs[b] <= t < offs[b + 1]]
        if not rows:
            continue
        w = _weights(p, change, int(adapters[b]) if adapters is not None else -1)
        n1 = orc.rmsnorm(xc[rows], p.g1, shape.rms_eps)
        q, k, v = (n1 @ w[n].T for n in "qkv")
        for j, i in enumerate(rows):
            q[j], k[j] = (orc.rope(m[j], positions[idx[i]], d, shape.rope_base) for m in (q, k))
        keys[rows], values[rows] = k.reshape(-1, nkv, d), v.reshape(-1, nkv, d)
        kb, vb = cached[b] if cached is not None else (keys[rows], values[rows])
        attn = np.zeros((len(rows), nh * d))
        for h in range(nh):
            s = q[:, h * d:(h + 1) * d] @ kb[:, h * nkv // nh].T / d ** 0.5
            for j in range(len(rows)):
                s[j, old[b] + j + 1:] = -np.inf
            e = np.exp(s - s.max(axis=1, keepdims=True))
            attn[:, h * d:(h + 1) * d] = e / e.sum(axis=1, keepdims=True) @ vb[:, h * nkv // nh]
        h1 = xc[rows] + attn @ w["o"].T
        n2 = orc.rmsnorm(h1, p.g2, shape.rms_eps)
        out[rows] = h1 + (orc.silu(n2 @ w["gate"].T) * (n2 @ w["up"].T)) @ w["down"].T
    return out, keys, values


def _read(qt, kv, layer, slot):
    n = int(kv.kv_len[layer, slot])
    k, v = qt.qtale_paged_read(kv, layer, ints([0, n]), ints([0]), slots=ints([slot]), T=n)
    return to_f64(k), to_f64(v)


def _run(qt, shape, bits, names, steps, mode, value, seed, first_layer=1, page=16, n_adapters=5, r=12):
    """steps: lists of new tokens per sequence."""
    B = len(steps[0])
    tensors = _tensors(shape, 0, seed)
    p, _ = oracle_layer(shape, 0, seed, tensors=tensors)
    stack = qt.Stack(qt.cfg_from_shape(shape), [qt.quantize_layer(tensors, shape.bits, shape.group)])
    lora, change = _loras(qt, shape, names, n_adapters, r, seed + 1) if names else (None, None)
    loras = qt.StackLora([lora]) if names else None
    ctx = _context(qt, mode, value)
    kv = qt.PagedKV.empty(sum(-(-sum(s[b] for s in steps) // page) for b in range(B)) + 4, page, shape.n_kv_heads, shape.head_dim, B + 2, 40, 3, bits=bits)
    kv.k.fill_(255 if bits == 4 else float("nan"))
    kv.v.fill_(255 if bits == 4 else float("nan"))
    slots = np.random.default_rng(seed).permutation(B + 2)[:B].tolist()
    adapters = ints([(3 * b) % (n_adapters + 2) - 1 for b in range(B)]) if names else None   # one each, none, and numbers past the last
    done = [0] * B
    for i, lens in enumerate(steps):
        T = sum(lens)
        x = si.hidden_states(shape, T, seed + 10 * i)
        offs, pos = si.ragged_sequences(lens, done)
        old = [int(kv.kv_len[first_layer, s]) for s in slots]
        xg, idx, cnt = x.cuda(), ints([-1] * T), ints([-1])
        qt.qtale_paged_stack_forward(ctx, stack, xg, offs.cuda(), pos.cuda(), kv, qt.Rope(shape.head_dim, shape.rope_base), slots=ints(slots),
                                     first_layer=first_layer, max_new=max(lens), sel_idx=idx, sel_count=cnt, loras=loras, adapter=adapters)
        got, widx = xg.cpu(), orc.decide(to_f64(x), p, mode, value)[1]
        assert np.array_equal(idx[: int(cnt.item())].cpu().numpy(), widx)
        skipped = np.setdiff1d(np.arange(T), widx)
        assert torch.equal(got[skipped], x[skipped])
        cached = [_read(qt, kv, first_layer, s) for s in slots]
        want, k, v = _layer64(to_f64(x), p, change, adapters.tolist() if names else None, shape, offs.numpy(), pos.numpy(), widx, cached, old)
        check_parity(orc.parity_error(to_f64(got)[widx], want), shape.act_dtype, ("serving", bits, bool(names), T), hidden=shape.hidden)
        for b in range(B):
            rows = [j for j, t in enumerate(widx) if offs[b] <= t < offs[b + 1]]
            assert len(cached[b][0]) == old[b] + len(rows)
            for held, mine in zip(cached[b], (k[rows], v[rows])):
                if not rows:
                    continue
                top = np.abs(mine).max(axis=2, keepdims=True)
                span = np.maximum(mine.max(axis=2, keepdims=True), 0) - np.minimum(mine.min(axis=2, keepdims=True), 0)
                step = span / 15 if bits == 4 else 0.0
                assert (np.abs(held[old[b]:] - mine) <= 0.5 * step + TOL * top * (1 + 16 / 7.5)).all()
        done = [a + n for a, n in zip(done, lens)]


SHAPES = [si.LayerShape(256, 4, 4, 64, 512, 4, 32, "fp16"), si.LayerShape(256, 8, 2, 128, 512, 4, 32, "bf16")]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("mode,value", [("ratio", 0.6), ("ratio", 1.0), ("threshold", 0.5)])
@pytest.mark.parametrize("bits,names", [(4, []), (16, NAMES), (4, NAMES), (4, ["q", "v"]), (4, ["up", "o"])])
def test_layer_in_64_bits(qt, shape, bits, names, mode, value):
    _run(qt, shape, bits, names, [[30, 0, 17, 1], [1, 1, 1, 1], [1, 90, 2, 150], [1] * 4], mode, value, 31)
    _run(qt, shape, bits, names, [[3, 1], [1, 0], [1, 1]], mode, value, 32)                          # at most four tokens
    _run(qt, shape, bits, names, [[2] * 9, [40, 1, 300, 1, 1, 1, 1, 1, 80]], mode, value, 33)


@pytest.mark.parametrize("bits", [2, 3])
def test_layer_with_other_weights(qt, bits):
    _run(qt, si.LayerShape(256, 8, 4, 64, 512, bits, 64, "bf16"), 4, NAMES, [[5, 1, 40], [1, 1, 1]], "ratio", 0.7, 40 + bits)


def _stack(qt, shape, L, seed=3):
    return qt.Stack(qt.cfg_from_shape(shape), [qt.quantize_layer(_tensors(shape, l, seed), shape.bits, shape.group) for l in range(L)])


def test_whole_stack_is_its_layers(qt):
    # requests that come, share a prompt, fork, and go, each with its adapter; some layers have adapters on some linears, one on none
    shape, L, S = si.LayerShape(256, 4, 2, 64, 512, 4, 32, "fp16"), 4, 8
    stack, ctx, rope = _stack(qt, shape, L), _context(qt, "ratio", 0.7), qt.Rope(64)
    layers = [_loras(qt, shape, names, 6, 16, 5 + l)[0] for l, names in enumerate([NAMES, ["q", "k", "v"], [], ["down", "gate"]])]
    loras, single = qt.StackLora(layers), [qt.StackLora([l]) for l in layers]
    a, b = (qt.PagedKV.empty(300, 16, 2, 64, S, 20, L, bits=4) for _ in range(2))

    def step(slots, lens, seed, adapters):
        offs, pos = si.ragged_sequences(lens, [7 * s for s in slots])
        x = si.hidden_states(shape, sum(lens), seed).cuda()
        y = x.clone()
        how = dict(slots=ints(slots), max_new=max(lens), adapter=ints(adapters))
        qt.qtale_paged_stack_forward(ctx, stack, x, offs.cuda(), pos.cuda(), a, rope, loras=loras, **how)
        for l in range(L):
            qt.qtale_paged_stack_forward(ctx, qt.Stack(stack.cfg, [stack.layers[l]]), y, offs.cuda(), pos.cuda(), b, rope, first_layer=l, loras=single[l], **how)
        assert torch.equal(x, y) and bool(x.isfinite().all())
        for s, t in ((a.table, b.table), (a.kv_len, b.kv_len), (a.page_refs, b.page_refs)):
            assert torch.equal(s, t)
        return x

    step([0, 5, 2], [50, 33, 1], 1, [0, 3, -1])
    for kv in (a, b):
        qt.qtale_pages_fork(kv, ints([0, 0, 5]), ints([1, 3, 7]))
    for i in range(6):
        step([0, 1, 3, 5, 7, 2], [1] * 6, 10 + i, [0, 1, 2, 3, 99, -1])
    for kv in (a, b):
        qt.qtale_pages_release(kv, ints([0, 5]))
        qt.qtale_pages_compact(kv)
    step([1, 4, 3, 5, 7], [1, 60, 1, 20, 3], 30, [1, 5, 2, 4, 0])
    # a sequence's result does not hang on who else is in the call, nor on the others' adapters
    for kv in (a, b):
        qt.qtale_pages_release(kv)
    ctx2 = _context(qt, "threshold", 0.3)
    x = si.hidden_states(shape, 40, 50).cuda()
    outs = []
    for slots, adapters in (([0, 1], [2, 4]), ([0, 1], [2, 1])):
        y = x.clone()
        offs, pos = si.ragged_sequences([25, 15], [0, 0])
        qt.qtale_paged_stack_forward(ctx2, stack, y, offs.cuda(), pos.cuda(), a, rope, slots=ints(slots), loras=loras, adapter=ints(adapters))
        qt.qtale_pages_release(a)
        outs.append(y)
    assert torch.equal(outs[0][:25], outs[1][:25]) and not torch.equal(outs[0][25:], outs[1][25:])


def test_without_adapters_it_is_the_plain_stack(qt):
    shape, L = si.LayerShape(256, 4, 2, 64, 512, 4, 32, "bf16"), 2
    stack, ctx, rope = _stack(qt, shape, L), _context(qt, "ratio", 1.0), qt.Rope(64)
    none = qt.StackLora([{}, {}])
    some = qt.StackLora([_loras(qt, shape, NAMES, 2, 8, 1)[0], {}])
    offs, pos = si.ragged_sequences([20, 9], [0, 0])
    outs = []
    caches = []
    for loras, ids in ((None, None), (none, [0, 1]), (some, [-1, 2])):
        kv = qt.PagedKV.empty(40, 16, 2, 64, 2, 10, L, bits=4)
        x = si.hidden_states(shape, 29, 1).cuda()
        if loras is not some:
            qt.qtale_paged_stack_forward(ctx, stack, x, offs.cuda(), pos.cuda(), kv, rope, loras=loras, adapter=None if ids is None else ints(ids))
            outs.append(x)
        # The first layer alone.  (Rows of a call with adapters that have none: the same bits up to gate and up, which are rounded to fp16 before their
        # product then.  That can move the layer's output by a bf16 step, 2^-8 of a value; the next layer's keys move with it, and where x / s lies
        # within 7.5 * 2^-8 of a half, for 3 to 6 codes of a hundred, a code moves by a whole step, a 15th of its row's range, so that a second layer on
        # a cache in 4 bits has no such bound.)
        kv = qt.PagedKV.empty(40, 16, 2, 64, 2, 10, L, bits=4)
        y = si.hidden_states(shape, 29, 1).cuda()
        one = qt.StackLora(loras.layers[:1]) if loras else None
        qt.qtale_paged_stack_forward(ctx, qt.Stack(stack.cfg, stack.layers[:1]), y, offs.cuda(), pos.cuda(), kv, rope, loras=one,
                                     adapter=None if ids is None else ints(ids))
        caches.append((y, [t for s in (0, 1) for t in qt.qtale_paged_read(kv, 0, ints([0, 20 - 11 * s]), slots=ints([s]), T=20 - 11 * s)]))
    assert torch.equal(outs[0], outs[1]) and torch.equal(caches[0][0], caches[1][0])
    assert all(torch.equal(a, b) for c in caches[1:] for a, b in zip(c[1], caches[0][1]))
    check_parity(orc.parity_error(to_f64(caches[2][0]), to_f64(caches[0][0])), "bf16", "no adapter", hidden=256)


@pytest.mark.parametrize("names", [[], NAMES])
def test_captured_decode_steps(qt, names):
    shape, L, B = si.LayerShape(256, 8, 2, 64, 512, 4, 32, "fp16"), 2, 6
    stack, ctx, rope = _stack(qt, shape, L), _context(qt, "threshold", 0.45), qt.Rope(64)
    loras = qt.StackLora([_loras(qt, shape, names, 4, 16, l)[0] for l in range(L)]) if names else None
    ids = ints([0, 1, 2, 3, -1, 0]) if names else None
    a, b = (qt.PagedKV.empty(100, 16, 2, 64, B, 10, L, bits=4) for _ in range(2))
    offs, pos = (t.cuda() for t in si.ragged_sequences([1] * B, [0] * B))
    x = si.hidden_states(shape, B, 0).cuda()
    ws = qt.alloc_paged_stack_workspace(stack.cfg, a, B, B, loras)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qt.qtale_paged_stack_forward(ctx, stack, x, offs, pos, a, rope, max_new=1, workspace=ws, loras=loras, adapter=ids)
    for step in range(40):
        x.copy_(si.hidden_states(shape, B, step))
        pos.fill_(step)
        if names and step == 20:
            ids.copy_(ints([3, 3, -1, 0, 1, 2]))                  # other requests in the same places
        y = x.clone()
        qt.qtale_paged_stack_forward(ctx, stack, y, offs, pos, b, rope, max_new=1, loras=loras, adapter=ids)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(x, y), step
        for s, t in ((a.table, b.table), (a.kv_len, b.kv_len), (a.free_bits, b.free_bits)):
            assert torch.equal(s, t)


def test_refusals_before_any_work(qt):
    shape, L = si.LayerShape(256, 4, 2, 64, 512, 4, 32, "fp16"), 2
    stack, ctx, rope = _stack(qt, shape, L), _context(qt, "ratio", 1.0), qt.Rope(64)
    good, _ = _loras(qt, shape, NAMES, 3, 8, 1)
    kv = qt.PagedKV.empty(40, 16, 2, 64, 2, 10, L, bits=4)
    offs, pos = (t.cuda() for t in si.ragged_sequences([4, 5], [0, 0]))
    x = si.hidden_states(shape, 9, 1).cuda()
    before = x.clone()
    call = lambda loras, **how: qt.qtale_paged_stack_forward(ctx, stack, x, offs, pos, kv, rope, loras=loras, adapter=ints([0, 1]), **how)
    wrong = dict(good, o=good["gate"])                            # another linear's sizes
    with pytest.raises(qt.QtaleError) as e:
        call(qt.StackLora([good, wrong]))
    assert e.value.code == -2
    loras = qt.StackLora([good, good])
    with pytest.raises(qt.QtaleError) as e:
        call(loras, workspace=qt.alloc_paged_stack_workspace(stack.cfg, kv, 9, 2))
    assert e.value.code == -4
    with pytest.raises(AssertionError):
        call(qt.StackLora([good]))
    with pytest.raises(AssertionError):
        qt.qtale_paged_stack_forward(ctx, stack, x, offs, pos, kv, rope, loras=loras)
    lib = qt.load_library()
    attn = qt.qtale_paged_attn(4, 0, 0, 0.125, 0, 0)
    ws = qt.alloc_paged_stack_workspace(stack.cfg, kv, 9, 2, loras)
    raw = lambda l, ids: lib.qtale_paged_stack_lora_forward(ctx._h, C.byref(stack.cfg), stack._w, l, L, 0, x.data_ptr(), 9, offs.data_ptr(), 2, pos.data_ptr(), kv._ref,
                                                            None, ids, rope._ref, C.byref(attn), None, None, None, None, ws.data_ptr(), ws.numel(), None)
    assert raw(None, 256) == -1 and raw(loras._c, None) == -1
    assert lib.qtale_paged_stack_lora_workspace_bytes(C.byref(stack.cfg), kv._ref, 12, 9, 2) == 0
    bf16 = qt.PagedKV.empty(40, 16, 2, 64, 2, 10, L, dtype=torch.bfloat16, bits=4)                    # the layers' keys and values are fp16
    with pytest.raises(qt.QtaleError) as e:
        qt.qtale_paged_stack_forward(ctx, stack, x, offs, pos, bf16, rope)
    assert e.value.code == -3
    torch.cuda.synchronize()
    assert torch.equal(x, before) and int(kv.kv_len.sum()) == 0
