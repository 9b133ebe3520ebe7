"""Attention over pages in 4 bits on the GPU (run with -m gpu) against 64 bits: head layouts, lengths around tile and page edges, few and many tokens, key
ranges, windows with first tokens, missing pages, rows that see nothing, scales of all sizes, NaN in places that a row does not see."""
import math
import random

import pytest
import torch

from tests.kv4_helpers import attention_bound4, pack, random_cache4, shadow, unpack, values64
from tests.paged_helpers import attend64, ints, offsets

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qt():
    import paper_2602_10431_amd as pkg
    pkg.load_library()
    return pkg


def _largest_scale(dense, kv, d):
    """The largest scale in use (a row's range is at most 15.5 steps)."""
    return max(float(torch.nan_to_num(x).abs().max()) for x in (dense.k, dense.v)) / 4


def _compare(dense, layer, q, out, new, first, slots, window, sinks, scale, clean=False):
    want, size = attend64(dense, layer, q, new, first, slots, window, sinks, scale, clean)
    bound = attention_bound4(want, size, q, q.dtype, scale, _largest_scale(dense, None, q.shape[2]))
    wrong = ~((out.double() - want).abs() <= bound)
    assert not bool(wrong.any()), (wrong.nonzero()[:4].tolist(), float((out.double() - want).abs().max()), float(bound.min()))


def _case(qt, dtype, rep, nkv, d, page, new, old, window=0, sinks=0, gone=(), seed=0, hints=True, scale=None, max_len=0, given_first=True):
    nh = rep * nkv
    lens = [o + n for o, n in zip(old, new)]
    kv, slots, dense = random_cache4(qt, lens, page, nkv, d, dtype, seed, n_layers=2, layer=1, gone=gone)
    T = sum(new)
    q = torch.randn(T, nh * d + 16, generator=torch.Generator().manual_seed(seed + 1)).to(dtype).cuda()[:, : nh * d].unflatten(1, (nh, d))
    out = torch.full((T, nh * d + 4), 7.0, dtype=dtype, device="cuda")
    view = out[:, : nh * d].unflatten(1, (nh, d))
    how = dict(max_new=max(new), max_len=max_len or max(lens + [1])) if hints else {}
    got = qt.qtale_paged_attention(kv, 1, q, offsets(new), first=ints(old) if given_first else None, slots=ints(slots), out=view, window=window, sinks=sinks,
                                   scale=scale, **how)
    assert got is view and bool((out[:, nh * d:] == 7.0).all())
    _compare(dense, 1, q, view, new, old, slots, window, sinks, scale or d ** -0.5)
    return kv, slots, dense, q, view


EDGES = [0, 1, 2, 14, 15, 16, 17, 30, 31, 32, 33, 47, 62, 63, 64, 65, 127, 128, 129, 191, 255, 256, 257, 600]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rep,nkv", [(1, 3), (3, 2), (4, 8), (16, 1)])
def test_one_token_per_sequence(qt, dtype, d, rep, nkv):
    for page in (16, 64):
        _case(qt, dtype, rep, nkv, d, page, [1] * len(EDGES), EDGES, seed=rep)


@pytest.mark.parametrize("d", [64, 128])
def test_one_token_of_many_sequences(qt, d):
    old = [(37 * i) % 300 for i in range(150)]
    _case(qt, torch.float16, 4, 4, d, 32, [1] * 150, old)
    _case(qt, torch.bfloat16, 2, 1, d, 32, [1] * 150, old)
    _case(qt, torch.float16, 1, 16, d, 16, [1] * 150, old)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
def test_one_token_on_long_caches(qt, dtype, d):
    _case(qt, dtype, 4, 2, d, 64, [1, 1], [5000, 900])
    _case(qt, dtype, 1, 2, d, 1024, [1], [3001])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rep", [1, 2, 5, 8, 24])
def test_a_few_tokens(qt, dtype, d, rep):
    _case(qt, dtype, rep, 2, d, 16, [2, 3, 0, 1, 9, 4], [0, 61, 5, 16, 300, 31], seed=rep)
    _case(qt, dtype, rep, 2, d, 32, [7, 8], [1000, 24], seed=rep + 1, hints=False)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rep,nkv", [(1, 2), (4, 1), (3, 3)])
def test_chunks(qt, dtype, d, rep, nkv):
    _case(qt, dtype, rep, nkv, d, 16, [65, 130, 1, 200, 0, 63], [0, 31, 77, 64, 9, 500], seed=rep)
    _case(qt, dtype, rep, nkv, d, 64, [300], [0], seed=rep, hints=False)
    _case(qt, dtype, rep, nkv, d, 128, [257, 96], [1000, 130], seed=rep, given_first=False)


@pytest.mark.parametrize("d", [64, 128])
def test_chunks_with_key_ranges_and_many_tiles(qt, d):
    _case(qt, torch.float16, 4, 2, d, 64, [150], [9000])
    _case(qt, torch.bfloat16, 4, 8, d, 64, [700, 900], [0, 250])
    _case(qt, torch.float16, 2, 8, d, 32, [2300], [0])
    _case(qt, torch.bfloat16, 1, 2, d, 32, [40, 1, 90, 1], [4000, 30, 6000, 5000])                    # single tokens beside


@pytest.mark.parametrize("window,sinks", [(1, 0), (7, 0), (33, 3), (64, 64), (100, 17), (500, 1)])
@pytest.mark.parametrize("new", [[1] * 6, [3] * 6, [40, 1, 90, 2, 70, 130]])
def test_windows(qt, window, sinks, new):
    for d in (64, 128):
        _case(qt, torch.float16, 4, 2, d, 16, new, [0, 40, 200, 3, 99, 700], window, sinks)
        _case(qt, torch.bfloat16, 1, 2, d, 64, new, [1000, 64, 128, 5, 90, 333], window, sinks)


@pytest.mark.parametrize("new", [[1, 1, 1], [5, 5, 5], [100, 80, 20]])
def test_missing_pages(qt, new):
    for d, page in ((64, 16), (128, 32), (128, 64)):
        old = [10 * page, 3 * page, 2 * page]
        gone = [(0, 0), (0, 3), (0, 4), (1, 1)] + [(2, j) for j in range(10)]                        # the third sees nothing: zeros
        _, _, _, _, out = _case(qt, torch.float16, 4, 2, d, page, new, old, gone=gone)
        assert bool((out[new[0] + new[1]:] == 0).all())


def test_rows_that_see_nothing(qt):
    # rows before their slot's begin, an empty slot, a slot that does not exist, rows past the last sequence
    kv, slots, dense = random_cache4(qt, [4, 0, 30], 16, 2, 64, torch.float16, 3)
    for n in (2, 40):
        q = torch.randn(4 * n + 3, 4, 64, generator=torch.Generator().manual_seed(1)).half().cuda()
        out = torch.full_like(q, 7.0)
        qt.qtale_paged_attention(kv, 0, q, offsets([n] * 4), first=ints([-n, 0, 20, 0]), slots=ints(slots + [99]), out=out)
        assert bool((out[: 2 * n] == 0).all()) and bool((out[3 * n: 4 * n] == 0).all()) and bool((out[4 * n:] == 7.0).all())
        _compare(dense, 0, q[2 * n: 3 * n], out[2 * n: 3 * n], [n], [20], slots[2:], 0, 0, 64 ** -0.5)


def test_max_len_hides_entries(qt):
    for new in ([1, 1], [30, 50]):
        kv, slots, dense = random_cache4(qt, [200, 90], 16, 2, 128, torch.float16, 5)
        q = torch.randn(sum(new), 2, 128, generator=torch.Generator().manual_seed(2)).half().cuda()
        first = [200 - new[0], 90 - new[1]]
        out = qt.qtale_paged_attention(kv, 0, q, offsets(new), first=ints(first), slots=ints(slots), max_len=100, max_new=max(new))
        dense.kv_len = kv.kv_len.clamp(max=100)
        _compare(dense, 0, q, out, new, first, slots, 0, 0, 128 ** -0.5)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("new", [[1, 1], [6, 3], [70, 130]])
@pytest.mark.parametrize("size", [2.0 ** -14, 2.0 ** -7, 200.0, 4000.0])
def test_scales_of_all_sizes(qt, dtype, new, size):
    # values of all sizes (their scale may be far from one, and differ by 2^10 from token to token)
    kv, slots, dense = random_cache4(qt, [300, 201], 32, 2, 64, dtype, 11)
    codes, scale, zero = unpack(kv.v, 64, False, dtype)
    g = torch.Generator().manual_seed(4)
    factor = size * torch.exp2(torch.randint(-9, 1, scale.shape, generator=g).float())
    scale = (scale.float() * factor).to(dtype)
    kv.v.copy_(pack(codes, scale, zero, False))
    dense.v = values64(codes, scale, zero).cuda()
    q = torch.randn(sum(new), 4, 64, generator=g).to(dtype).cuda()
    first = [300 - new[0], 201 - new[1]]
    out = qt.qtale_paged_attention(kv, 0, q, offsets(new), first=ints(first), slots=ints(slots), max_new=max(new))
    want, total = attend64(dense, 0, q, new, first, slots, 0, 0, 0.125)
    bound = attention_bound4(want, total, q, dtype, 0.125, float(torch.nan_to_num(dense.k).abs().max()) / 4) - 0.0
    bound = bound + 30 * float(torch.nan_to_num(scale.float()).max()) * 64 * 2.0 ** -24
    assert bool(((out.double() - want).abs() <= bound).all())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("new", [[1], [9], [150]])
def test_scores_of_any_size(qt, dtype, new):
    # one key per row is far ahead of all others: the output is its value
    kv, slots, dense = random_cache4(qt, [256], 16, 1, 64, dtype, 13)
    q = (30 * torch.randn(new[0], 1, 64, generator=torch.Generator().manual_seed(6))).to(dtype).cuda()
    for scale in (1.0, 1e6, 1e20):
        out = qt.qtale_paged_attention(kv, 0, q, offsets(new), slots=ints(slots), scale=scale)
        assert bool(out.isfinite().all())
        first = 256 - new[0]
        row = kv.table[0, slots[0]].tolist()
        k, v = (torch.stack([x[row[j // 16], 0, j % 16] for j in range(256)]) for x in (dense.k, dense.v))
        z = q[:, 0].double() @ k.t()
        z = z.masked_fill(torch.arange(256, device="cuda")[None] > first + torch.arange(new[0], device="cuda")[:, None], -math.inf)
        best, at = z.topk(2, 1)
        clear = (best[:, 0] - best[:, 1]) * scale > 100
        clear &= (best[:, 0] - best[:, 1]) > 1e-3 * best[:, 0].abs()   # (and further apart than 32-bit sums are off)
        assert bool(clear.any())
        want = v[at[:, 0]][clear]
        assert bool(((out[:, 0].double()[clear] - want).abs() <= 2 * (2.0 ** -11 if dtype == torch.float16 else 2.0 ** -8) * want.abs() + 1e-4).all())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new,old", [([1], [90]), ([7], [50]), ([150], [40]), ([90, 300], [0, 33])])
def test_rows_that_are_not_finite_reach_only_who_sees_them(qt, dtype, d, new, old):
    lens = [o + n for o, n in zip(old, new)]
    kv, slots, dense = random_cache4(qt, lens, 16, 2, d, dtype, 17)
    where = [(0, lens[0] - 1 - new[0] // 2, True, 0), (0, lens[0] - 1 - new[0] // 3, False, 1)]       # (sequence, token, keys, head)
    for b, t, keys, head in where:
        pool = kv.k if keys else kv.v
        codes, scale, zero = unpack(pool, d, keys, dtype)
        scale = scale.clone()
        scale[int(kv.table[0, slots[b], t // 16]), head, t % 16] = math.nan
        pool.copy_(pack(codes, scale, zero, keys))
    q = torch.randn(sum(new), 6, d, generator=torch.Generator().manual_seed(8)).to(dtype).cuda()
    out = qt.qtale_paged_attention(kv, 0, q, offsets(new), first=ints(old), slots=ints(slots), max_new=max(new))
    for b, t, keys, head in where:
        rows = torch.arange(new[b], device="cuda") + old[b] >= t
        assert bool(out[: new[b]][rows][:, 3 * head: 3 * head + 3].isnan().all())
        for x in (dense.k, dense.v):                              # who does not see it: as without it
            pass
        out[: new[b], 3 * head: 3 * head + 3] = torch.where(rows[:, None, None], torch.zeros_like(out[: new[b], :3]), out[: new[b], 3 * head: 3 * head + 3])
    want, size = attend64(dense, 0, q, new, old, slots, 0, 0, d ** -0.5)
    for b, t, keys, head in where:
        rows = torch.arange(new[b], device="cuda") + old[b] >= t
        want[: new[b], 3 * head: 3 * head + 3] = torch.where(rows[:, None, None], torch.zeros_like(want[: new[b], :3]), want[: new[b], 3 * head: 3 * head + 3])
    bound = attention_bound4(want, size, q, dtype, d ** -0.5, _largest_scale(dense, None, d))
    assert bool(((out.double() - want).abs() <= bound).all())


def test_random_calls(qt):
    rng = random.Random(5)
    for i in range(40):
        d, dtype, page = rng.choice([64, 128]), rng.choice([torch.float16, torch.bfloat16]), rng.choice([16, 32, 64, 256])
        nkv, rep = rng.randint(1, 5), rng.choice([1, 2, 3, 4, 7, 8])
        most = rng.choice([1, 1, 4, 40, 300])
        B = rng.randint(1, 9)
        new, old = [rng.randint(0, most) for _ in range(B)], [rng.choice([0, rng.randint(0, 50), rng.randint(0, 1200)]) for _ in range(B)]
        if sum(new) == 0:
            new[0] = 1
        window, sinks = rng.choice([(0, 0), (rng.randint(1, 300), rng.choice([0, rng.randint(1, 70)]))])
        gone = [(b, rng.randrange(max(1, (o + n) // page))) for b, (n, o) in enumerate(zip(new, old)) if rng.random() < 0.3]
        _case(qt, dtype, rep, nkv, d, page, new, old, window, sinks, gone, seed=100 + i, hints=rng.random() < 0.7)


@pytest.mark.parametrize("new,old", [([1] * 5, [700, 30, 5, 2000, 64]), ([5] * 5, [700, 30, 5, 2000, 64]), ([150, 90, 1, 60, 40], [0, 1500, 300, 20, 2])])
def test_repeated_calls_give_the_same_bits(qt, new, old):
    kv, slots, dense, q, out = _case(qt, torch.float16, 4, 2, 128, 32, new, old)
    first = out.clone()
    for _ in range(20):
        again = qt.qtale_paged_attention(kv, 1, q, offsets(new), first=ints(old), slots=ints(slots), max_new=max(new), max_len=max(o + n for o, n in zip(old, new)))
        assert torch.equal(again.view(torch.int16), first.view(torch.int16))


@pytest.mark.parametrize("new,old", [([1] * 4, [700, 30, 5, 2000]), ([150, 90, 1], [0, 1500, 300])])
def test_graph_and_side_stream(qt, new, old):
    kv, slots, dense, q, out = _case(qt, torch.bfloat16, 4, 2, 128, 32, new, old)
    eager = out.clone()
    T = sum(new)
    lens = max(o + n for o, n in zip(old, new))
    ws = qt.alloc_paged_workspace(kv, 8, T, len(new), max(new), lens)
    offs, first, sl = offsets(new), ints(old), ints(slots)
    static = torch.zeros(T, 8, 128, dtype=torch.bfloat16, device="cuda")
    call = lambda: qt.qtale_paged_attention(kv, 1, q, offs, first=first, slots=sl, out=static, max_new=max(new), max_len=lens, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(static, eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(4):
        static.zero_()
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(static, eager)
