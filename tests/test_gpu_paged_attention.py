"""Attention over pages on the GPU (run with -m gpu) against 64 bits: head layouts, lengths around every tile and page edge, key ranges, windows with
first tokens, missing pages, rows that see nothing, memory that holds NaN, large pools, graphs.  The bound on the error is derived in paged_helpers."""
import random

import pytest
import torch

from tests.paged_helpers import attend64, attention_bound, ints, offsets, random_cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qt():
    import paper_2602_10431_amd as pkg
    pkg.load_library()
    return pkg


def _compare(kv, layer, q, out, new, first, slots, window, sinks, scale, few):
    want, size = attend64(kv, layer, q, new, first, slots, window, sinks, scale)
    bound = attention_bound(want, size, q.dtype, few)
    wrong = ~((out.double() - want).abs() <= bound)
    assert not bool(wrong.any()), (wrong.nonzero()[:4].tolist(), float((out.double() - want).abs().max()))


def _case(qt, dtype, rep, nkv, d, page, new, old, window=0, sinks=0, gone=(), seed=0, hints=True, scale=None, max_len=0, given_first=True):
    nh = rep * nkv
    lens = [o + n for o, n in zip(old, new)]
    kv, slots = random_cache(qt, lens, page, nkv, d, dtype, seed, n_layers=2, layer=1, gone=gone)
    T = sum(new)
    q = (2 * torch.randn(T, nh * d + 16, generator=torch.Generator().manual_seed(seed + 1))).to(dtype).cuda()[:, : nh * d].unflatten(1, (nh, d))
    out = torch.full((T, nh * d + 4), 7.0, dtype=dtype, device="cuda")
    view = out[:, : nh * d].unflatten(1, (nh, d))
    how = dict(max_new=max(new), max_len=max_len or max(lens + [1])) if hints else {}
    got = qt.qtale_paged_attention(kv, 1, q, offsets(new), first=ints(old) if given_first else None, slots=ints(slots), out=view, window=window, sinks=sinks,
                                   scale=scale, **how)
    assert got is view and bool((out[:, nh * d:] == 7.0).all())
    few = max(new) * rep <= 16 if hints else False
    _compare(kv, 1, q, view, new, old, slots, window, sinks, scale or d ** -0.5, few)
    return kv, slots, q, view


EDGES = [0, 1, 2, 14, 15, 16, 17, 30, 31, 32, 33, 47, 62, 63, 64, 65, 127, 128, 129, 191, 255, 256, 257, 600]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rep,nkv", [(1, 3), (3, 2), (4, 8), (16, 1)])
def test_one_token_per_sequence(qt, dtype, d, rep, nkv):
    for page in (16, 64):
        _case(qt, dtype, rep, nkv, d, page, [1] * len(EDGES), EDGES, seed=rep)                       # few workgroups: keys may be cut


@pytest.mark.parametrize("d", [64, 128])
def test_one_token_of_many_sequences(qt, d):
    old = [(37 * i) % 300 for i in range(150)]
    _case(qt, torch.float16, 4, 4, d, 32, [1] * 150, old)                                            # keys not cut, several waves of sequences
    _case(qt, torch.bfloat16, 2, 1, d, 32, [1] * 150, old)                                           # cut


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rep", [1, 4, 5])
def test_a_few_tokens_per_sequence(qt, d, rep):
    new = [1, 3, 2, 0, 3, 1, 3]
    _case(qt, torch.float16, rep, 2, d, 16, new, [0, 0, 14, 9, 61, 700, 255], seed=rep)
    _case(qt, torch.bfloat16, rep, 2, d, 128, new, [0, 127, 126, 9, 61, 700, 255], seed=rep)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rep,nkv", [(1, 8), (4, 2), (8, 1), (6, 3)])
def test_chunks_around_the_tiles(qt, dtype, d, rep, nkv):
    n = 128 // rep
    new = [n - 1, n, n + 1, 2 * n + 1, 17, 70]
    _case(qt, dtype, rep, nkv, d, 64, new, [0, 1, 63, 64, 65, 130], seed=rep)
    _case(qt, dtype, rep, nkv, d, 16, new, [500, 0, 15, 17, 300, 31], seed=rep)


# Calls that the kernel for chunks gets: its keys cut into ranges (a bound on long caches), many column tiles on short keys, and the same on longer
# ones, which two groups of waves share.  (Few column tiles on short keys are the other kernel's, sixteen columns at a time.)
FORMS = {"ranges": ([31, 33, 1, 65, 17], [0, 500, 64, 1, 300], 60000), "tiles": ([31, 33, 32, 65, 1, 64, 17, 40] * 3, [0, 1, 64, 63, 300, 128, 30, 200] * 3, 400),
         "groups": ([31, 33, 32, 65, 1, 64, 17, 40] * 3, [0, 600, 64, 63, 900, 128, 30, 500] * 3, 1000)}


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d,rep", [(64, 4), (128, 1), (128, 4), (64, 17)])
@pytest.mark.parametrize("form", sorted(FORMS))
def test_forms_of_the_kernel_for_chunks(qt, form, d, rep, dtype):
    new, old, bound = FORMS[form]
    nkv = 8 if rep < 17 else 2
    _case(qt, dtype, rep, nkv, d, 64, new, old, max_len=bound, seed=rep)
    _case(qt, dtype, rep, nkv, d, 16, new, old, window=70, sinks=20, max_len=bound, seed=rep, gone={(0, 0), (1, 2), (3, 1)})


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("form", sorted(FORMS))
def test_values_that_are_not_finite_in_every_form(qt, form, d, dtype):
    new, old, bound = FORMS[form]
    nkv, rep, page = 8, 1, 32
    kv, slots = random_cache(qt, [o + n for o, n in zip(old, new)], page, nkv, d, dtype, 12)
    for b, h, e, pool, value in ((0, 0, 5, kv.v, "nan"), (1, 3, 9, kv.k, "inf"), (3, 7, 63, kv.v, "-inf")):
        at = old[b] + new[b] // 2
        pool[int(kv.table[0, slots[b], at // page]), h, at % page, e] = float(value)
    q = torch.randn(sum(new), rep * nkv, d, generator=torch.Generator().manual_seed(5)).to(dtype).cuda()
    got = qt.qtale_paged_attention(kv, 0, q, offsets(new), first=ints(old), slots=ints(slots), max_new=max(new), max_len=bound)
    few = [0, 1, 3]                                              # the sequences that hold such values row by row, the others as ever
    want, size = attend64(kv, 0, q, new, old, slots, 0, 0, d ** -0.5)
    begin = offsets(new).tolist()
    for b in few:
        rows = slice(begin[b], begin[b + 1])
        want[rows], size[rows] = attend64(kv, 0, q[rows], new[b: b + 1], old[b: b + 1], slots[b: b + 1], 0, 0, d ** -0.5, clean=True)
    whole = torch.isfinite(want) & torch.isfinite(size)
    assert not bool(whole.all()) and bool(whole.any())
    assert bool(((got.double() - want).abs() <= attention_bound(want, size, dtype, False))[whole].all())
    assert not bool(torch.isfinite(got[~whole]).any())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rep,d,tokens", [(1, 128, 17), (3, 64, 11), (4, 128, 8), (16, 64, 3), (5, 64, 13), (24, 128, 2)])
def test_columns_by_sixteen(qt, rep, d, tokens, dtype):
    new = [tokens, 1, tokens - 1, 0, tokens]
    _case(qt, dtype, rep, 2, d, 32, new, [0, 40, 33, 7, 300], seed=rep)
    _case(qt, dtype, rep, 2, d, 16, new, [90, 40, 333, 7, 300], window=33, sinks=5, seed=rep, gone={(0, 1), (2, 3)})


@pytest.mark.parametrize("rep", [17, 32, 40])
def test_more_heads_per_kv_head_than_columns_of_the_decode_kernel(qt, rep):
    _case(qt, torch.float16, rep, 1, 64, 32, [1, 1, 4, 0, 9], [0, 100, 33, 5, 600])


@pytest.mark.parametrize("rep,d", [(1, 128), (4, 128), (2, 64)])
@pytest.mark.parametrize("hints", [True, False])
def test_single_tokens_beside_chunks(qt, rep, d, hints):
    # both kernels run, with and without cut keys
    _case(qt, torch.float16, rep, 2, d, 32, [1, 300, 1, 2, 0, 45, 1], [900, 10, 0, 31, 5, 700, 64], hints=hints, seed=rep)
    _case(qt, torch.bfloat16, rep, 8, d, 32, [1, 300] + [1] * 70, [90, 10] + [(11 * i) % 200 for i in range(70)], hints=hints, seed=rep)


@pytest.mark.parametrize("left", [0.0, 2.0, 1e30, float("nan")])
@pytest.mark.parametrize("d", [64, 128])
def test_what_a_workspace_held_does_not_show(qt, d, left):
    # single tokens beside a chunk whose keys are cut: a workspace that other calls have used
    rep, nkv, new, old = 4, 2, [1, 300, 1, 2, 0, 45] + [1] * 12, [900, 10, 0, 31, 5, 2600] + [70] * 12
    nh, lens, T, B = rep * nkv, [o + n for o, n in zip(old, new)], sum(new), len(new)
    kv, slots = random_cache(qt, lens, 64, nkv, d, torch.float16, 3)
    q = torch.randn(T, nh, d, generator=torch.Generator().manual_seed(4)).half().cuda()
    workspace = qt.alloc_paged_workspace(kv, nh, T, B, max(new))
    workspace.view(torch.float32).fill_(left)
    out = qt.qtale_paged_attention(kv, 0, q, offsets(new), first=ints(old), slots=ints(slots), max_new=max(new), max_len=4096, workspace=workspace)
    _compare(kv, 0, q, out, new, old, slots, 0, 0, d ** -0.5, False)


@pytest.mark.parametrize("dtype,d,rep,nkv", [(torch.float16, 64, 1, 1), (torch.bfloat16, 128, 4, 2), (torch.float16, 128, 2, 8), (torch.bfloat16, 64, 8, 3)])
@pytest.mark.parametrize("B", [2, 7, 40, 170])
def test_spans_that_end_one_sequence_and_begin_the_next(qt, dtype, d, rep, nkv, B):
    # lengths of nothing, of a few keys and of thousands beside each other: pieces of every kind
    if B * nkv >= 512:
        pytest.skip("not cut")
    old = [(0, 2500, 3, 130, 1, 900, 127, 64, 1400, 300)[i % 10] + i for i in range(B)]
    new = [0 if i % 9 == 4 else 1 for i in range(B)]
    _case(qt, dtype, rep, nkv, d, 64, new, old, seed=B)
    if 2 * rep <= 16:
        _case(qt, dtype, rep, nkv, d, 16, [min(2 * n, 1 + i % 2) for i, n in enumerate(new)], old, seed=B)
    _case(qt, dtype, rep, nkv, d, 32, new, old, window=1500, sinks=20, seed=B, gone={(1, 0), (1, 3), (B - 1, 0)})


@pytest.mark.parametrize("new,old", [(1, 5000), (2, 9000), (40, 6000), (300, 3000)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_one_long_sequence_is_cut(qt, new, old, dtype):
    _case(qt, dtype, 4, 2, 128, 64, [new], [old])
    _case(qt, dtype, 1, 1, 64, 128, [new], [old], hints=False)


@pytest.mark.parametrize("window", [1, 2, 16, 33, 100, 128, 1000])
@pytest.mark.parametrize("sinks", [0, 1, 4, 32, 70])
def test_windows_and_first_tokens(qt, window, sinks):
    _case(qt, torch.float16, 4, 2, 64, 16, [1] * 8, [0, 1, 30, 99, 128, 200, 500, 1400], window, sinks, seed=window)
    _case(qt, torch.bfloat16, 2, 2, 128, 32, [3, 1, 2, 5], [0, 31, 400, 77], window, sinks, seed=window)
    _case(qt, torch.float16, 2, 3, 128, 32, [200, 33, 70], [0, 400, 129], window, sinks, seed=window)


@pytest.mark.parametrize("sinks", [0, 5, 20])
def test_pages_behind_the_window_are_gone_or_hold_nan(qt, sinks):
    page, window = 16, 40
    for new, old in (([1, 2], [200, 411]), ([90, 60], [200, 411])):
        reach = [[j for j in range(o // page) if (j + 1) * page <= o + 1 - window and j * page >= sinks] for o in old]
        gone = {(b, j) for b, pages in enumerate(reach) for j in pages}
        kv, slots, q, out = _case(qt, torch.float16, 2, 2, 64, page, new, old, window, sinks, gone=gone)
        # the same with the pages there, full of NaN, and NaN between the window and its page's begin
        whole, slots2 = random_cache(qt, [o + n for o, n in zip(old, new)], page, 2, 64, torch.float16, 0, n_layers=2, layer=1)
        first_seen = [o + 1 - window for o in old]
        for b, lo in enumerate(first_seen):
            for j in range(sinks, lo):
                p = int(whole.table[1, slots2[b], j // page])
                whole.k[p, :, j % page], whole.v[p, :, j % page] = float("nan"), float("nan")
        got = qt.qtale_paged_attention(whole, 1, q, offsets(new), first=ints(old), slots=ints(slots2), window=window, sinks=sinks, max_new=max(new), max_len=600)
        _compare(whole, 1, q, got, new, old, slots2, window, sinks, 64 ** -0.5, False)


@pytest.mark.parametrize("new", [[1, 1, 1], [30, 50, 1]])
def test_missing_pages_anywhere(qt, new):
    gone = {(0, 0), (0, 3), (1, 5), (1, 6), (1, 7), (2, 0)}
    _case(qt, torch.float16, 4, 2, 128, 32, new, [300, 250, 20], gone=gone)
    _case(qt, torch.bfloat16, 1, 2, 64, 16, new, [300, 250, 20], gone=gone)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_long_chunks(qt, dtype):
    # enough column tiles and keys for the workgroups whose halves take turns: even and odd numbers of tiles, a last tile with few columns, missing
    # pages, a window, a page per tile and several
    _case(qt, dtype, 16, 8, 128, 64, [1400, 907, 300], [1000, 1201, 64], gone={(0, 5), (1, 30)}, seed=1)
    _case(qt, dtype, 4, 8, 128, 16, [2048, 2048], [0, 0], seed=2)
    _case(qt, dtype, 16, 8, 128, 128, [1333, 1300], [2100, 900], window=2300, sinks=5, seed=3)


def test_a_long_chunk_with_a_value_that_is_not_finite(qt):
    nkv, rep, d, page, new, old = 8, 16, 128, 64, [1400, 1200], [900, 10]
    kv, slots = random_cache(qt, [o + n for o, n in zip(old, new)], page, nkv, d, torch.float16, 12)
    q = torch.randn(sum(new), rep * nkv, d, device="cuda").half()
    kw = dict(first=ints(old), slots=ints(slots), max_new=1400, max_len=2300)
    clean = qt.qtale_paged_attention(kv, 0, q, offsets(new), **kw)
    at = old[0] + 700                                            # a new token's value: rows before it do not see it
    kv.v[int(kv.table[0, slots[0], at // page]), 2, at % page, 7] = float("nan")
    got = qt.qtale_paged_attention(kv, 0, q, offsets(new), **kw)
    hit = torch.zeros_like(got, dtype=torch.bool)
    hit[700:1400, 2 * rep: 3 * rep, 7] = True
    assert bool(torch.isnan(got[hit]).all())
    # rows in a tile with it are done again key by key: equal within what two such results may differ
    size = torch.ones_like(clean).double()
    assert bool(((got.double() - clean.double()).abs() <= 2 * attention_bound(clean.double(), size, torch.float16, False))[~hit].all())
    assert torch.equal(got[1400:], clean[1400:])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("new,old", [([3, 4, 2], [60, 5, 700]), ([60, 33, 40], [70, 0, 700]), ([3, 4, 2], [60, 5, 9000])])
def test_values_that_are_not_finite_reach_only_the_rows_that_see_them(qt, dtype, value, new, old):
    # in keys and values of new tokens, which earlier rows of the same tile do not see, and in cached ones that leave the window of later rows
    nkv, rep, d, page = 2, 2, 64, 16
    for window in (0, 21):
        kv, slots = random_cache(qt, [o + n for o, n in zip(old, new)], page, nkv, d, dtype, 11)
        def put(pool, b, at, h, e):
            pool[int(kv.table[0, slots[b], at // page]), h, at % page, e] = value
        put(kv.v, 0, old[0] + 1, 0, 5)
        put(kv.k, 0, old[0] + 2, 1, 9)
        put(kv.v, 1, old[1] + new[1] // 2, 1, 63)
        put(kv.v, 2, old[2] - 20, 0, 0)                          # out of the window of the second new token
        q = torch.randn(sum(new), rep * nkv, d, device="cuda").to(dtype)
        got = qt.qtale_paged_attention(kv, 0, q, offsets(new), first=ints(old), slots=ints(slots), window=window, max_new=max(new), max_len=10000)
        want, size = attend64(kv, 0, q, new, old, slots, window, 0, d ** -0.5, clean=True)
        whole = torch.isfinite(want) & torch.isfinite(size)
        assert not bool(whole.all()) and bool(whole.any())
        bound = attention_bound(want, size, dtype, False)
        assert bool(((got.double() - want).abs() <= bound)[whole].all())
        assert not bool(torch.isfinite(got[~whole]).any())


@pytest.mark.parametrize("new", [[3, 5, 2, 1], [40, 33, 20, 1]])
def test_rows_that_see_nothing_are_zero(qt, new):
    d, nkv, nh = 64, 2, 4
    # an empty slot, a slot shorter than its new tokens (the first rows lie before its begin), and a slot that does not exist
    kv, slots = random_cache(qt, [0, 3, 50], 16, nkv, d, torch.float16, 3)
    q = torch.randn(sum(new), nh, d, device="cuda").half()
    use = [slots[0], slots[1], slots[2], 77]
    out = torch.full_like(q, 9.0)
    qt.qtale_paged_attention(kv, 0, q, offsets(new), slots=ints(use), out=out, max_new=max(new), max_len=50)
    first = [0 - new[0], 3 - new[1], 50 - new[2]]
    t = sum(new[:3])
    _compare(kv, 0, q[:t], out[:t], new[:3], first, slots, 0, 0, d ** -0.5, False)
    assert bool((out[: new[0]] == 0).all()) and bool((out[new[0]: new[0] + new[1] - 3] == 0).all()) and bool((out[t:] == 0).all())


def test_entries_past_the_bound_are_not_seen(qt):
    for new in ([1, 1], [40, 30]):
        kv, slots, q, _ = _case(qt, torch.float16, 2, 1, 64, 16, new, [200, 90])
        got = qt.qtale_paged_attention(kv, 1, q, offsets(new), first=ints([200, 90]), slots=ints(slots), max_new=max(new), max_len=100)
        kv.kv_len[1].clamp_(max=100)
        _compare(kv, 1, q, got, new, [200, 90], slots, 0, 0, 64 ** -0.5, False)


def test_strides_of_a_single_token_or_head(qt):
    # [heads, 1, d] and [1, T, d] seen from the other side: contiguous, whatever the strides say
    d = 64
    for T, rep, nkv in ((1, 4, 2), (5, 1, 1)):
        kv, slots = random_cache(qt, [70], 16, nkv, d, torch.float16, 2, max_extra=4)
        q = torch.randn(rep * nkv, T, d, generator=torch.Generator().manual_seed(3)).half().cuda().transpose(0, 1)
        assert q.is_contiguous() and q.stride() != (rep * nkv * d, d, 1)
        kv_len = kv.kv_len.clone()
        out = qt.qtale_paged_attention(kv, 0, q, offsets([T]), slots=ints(slots), max_new=T, out=torch.empty_like(q))
        _compare(kv, 0, q, out, [T], [70 - T], slots, 0, 0, d ** -0.5, True)
        k, v = (torch.randn(nkv, T, d, generator=torch.Generator().manual_seed(i)).half().cuda().transpose(0, 1) for i in (4, 5))
        rope, pos = qt.Rope(d), ints(list(range(70 - T, 70)))
        a = qt.qtale_paged_rope_append(kv, 0, rope, q, k, v, offsets([T]), pos, slots=ints(slots))
        kept = kv.k.clone(), kv.v.clone()
        b = qt.qtale_paged_rope_append(kv, 0, rope, *(t.clone(memory_format=torch.contiguous_format) for t in (q, k, v)), offsets([T]), pos, slots=ints(slots))
        assert torch.equal(a, b) and torch.equal(kept[0].nan_to_num(), kv.k.nan_to_num()) and torch.equal(kept[1].nan_to_num(), kv.v.nan_to_num())
        assert torch.equal(kv_len, kv.kv_len)


def test_no_slots_no_first(qt):
    # sequence b is slot b, its tokens are the slot's last ones
    kv, slots = random_cache(qt, [70, 33, 5], 16, 2, 64, torch.float16, 8, extra_slots=0)
    lens = kv.kv_len[0].tolist()
    for new in ([1, 1, 1], [20, 5, 5]):
        q = torch.randn(sum(new), 4, 64, device="cuda").half()
        got = qt.qtale_paged_attention(kv, 0, q, offsets(new))
        _compare(kv, 0, q, got, new, [l - n for l, n in zip(lens, new)], [0, 1, 2], 0, 0, 64 ** -0.5, False)


@pytest.mark.parametrize("new", [[1], [60]])
def test_scores_of_any_size(qt, new):
    # the reference point of the exponentials has to follow: scores of a thousand, growing along the keys, and all far below zero
    kv, slots = random_cache(qt, [400], 16, 1, 64, torch.bfloat16, 4)
    q = torch.ones(new[0], 2, 64, device="cuda", dtype=torch.bfloat16)
    row = kv.table[0, slots[0]].tolist()
    for sign in (1.0, -1.0):
        for j in range(400):
            kv.k[row[j // 16], 0, j % 16] = sign * (j // 40) * 2.0
        for scale in (0.125, 8.0):
            got = qt.qtale_paged_attention(kv, 0, q, offsets(new), slots=ints(slots), scale=scale)
            _compare(kv, 0, q, got, new, [400 - new[0]], slots, 0, 0, scale, False)


@pytest.mark.parametrize("new,old", [([1], [300]), ([60], [300]), ([1], [9000])])
def test_scores_far_below_zero(qt, new, old):
    # bf16 queries and keys of 10^17: every score is about -10^34, and what counts is how far they are from each other
    nkv, rep, d = 2, 2, 64
    kv, slots = random_cache(qt, [o + n for o, n in zip(old, new)], 32, nkv, d, torch.bfloat16, 8)
    kv.k.fill_(-1e17)
    kv.k[..., 1::2] = 0.0                                        # half of the columns: the scores are the same number
    kv.v.copy_(torch.randn(kv.v.shape, generator=torch.Generator().manual_seed(9)))
    q = torch.full((sum(new), nkv * rep, d), 1e17, dtype=torch.bfloat16, device="cuda")
    out = qt.qtale_paged_attention(kv, 0, q, offsets(new), first=ints(old), slots=ints(slots), max_new=max(new), max_len=max(old) + max(new))
    _compare(kv, 0, q, out, new, old, slots, 0, 0, d ** -0.5, max(new) == 1)


@pytest.mark.parametrize("new,old", [([1], [300]), ([60], [300]), ([2, 60], [9000, 40]), ([400], [4000])])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_the_largest_scores_of_fp16(qt, new, old, sign):
    # queries and keys of 60000: scores of 10^10, equal for every other key, half of that for the rest
    nkv, rep, d = 2, 2, 64
    kv, slots = random_cache(qt, [o + n for o, n in zip(old, new)], 32, nkv, d, torch.float16, 8)
    kv.k.fill_(sign * 60000.0)
    kv.k[:, :, 1::2] = sign * 30000.0
    kv.v.copy_(torch.randn(kv.v.shape, generator=torch.Generator().manual_seed(9)))
    q = torch.full((sum(new), nkv * rep, d), 60000.0, dtype=torch.float16, device="cuda")
    out = qt.qtale_paged_attention(kv, 0, q, offsets(new), first=ints(old), slots=ints(slots), max_new=max(new), max_len=max(o + n for o, n in zip(old, new)))
    _compare(kv, 0, q, out, new, old, slots, 0, 0, d ** -0.5, max(new) * rep <= 16)


@pytest.mark.parametrize("seed", range(24))
def test_calls_of_any_kind(qt, seed):
    rng = random.Random(seed)
    d, dtype, page = rng.choice([64, 128]), rng.choice([torch.float16, torch.bfloat16]), rng.choice([16, 32, 64, 128, 256, 1024])
    nkv, rep = rng.choice([1, 2, 3, 4, 8, 16]), rng.choice([1, 2, 3, 4, 5, 8, 12, 16, 17])
    B = rng.choice([2, 5, 30])
    longest = rng.choice([5, 50, 300, 1500] if B == 30 else [50, 1500, 6000])
    most = rng.choice([1, 4, 100, 400])
    new = [most] + [rng.choice([0, 1, 1, 2, rng.randint(1, most)]) if most > 1 else rng.choice([0, 1, 1]) for _ in range(B - 1)]
    old = [rng.choice([0, longest, rng.randint(0, longest)]) for _ in range(B)]
    lens = [o + n for o, n in zip(old, new)]
    gone = {(b, rng.randrange(max(-(-lens[b] // page), 1))) for b in range(B) if rng.random() < 0.1}
    window, sinks, hints = rng.choice([0, 0, 1, 17, 100, 700]), rng.choice([0, 4, 33]), rng.random() < 0.7
    kv, slots = random_cache(qt, lens, page, nkv, d, dtype, seed, gone=gone)
    q = torch.randn(sum(new), rep * nkv, d, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()
    how = dict(max_new=most, max_len=max(lens) + rng.choice([0, 4000])) if hints else {}
    workspace = qt.alloc_paged_workspace(kv, rep * nkv, sum(new), B, how.get("max_new", 0))
    workspace.view(torch.float32).fill_(rng.choice([0.0, 2.0, 1e30, float("nan")]))
    out = qt.qtale_paged_attention(kv, 0, q, offsets(new), first=ints(old), slots=ints(slots), window=window, sinks=sinks, workspace=workspace, **how)
    _compare(kv, 0, q, out, new, old, slots, window, sinks, d ** -0.5, hints and most * rep <= 16)


@pytest.mark.parametrize("new", [1, 50])
def test_a_pool_beyond_32_bit_offsets(qt, new):
    # 2.1e9 elements of keys: the pages in use lie at the end
    page, nkv, d = 128, 8, 128
    n_pages = (1 << 31) // (page * nkv * d) + 60
    kv = qt.PagedKV.empty(n_pages, page, nkv, d, 1, 20)
    kv.k[-40:].normal_()
    kv.v[-40:].normal_()
    kv.table[0, 0, :8] = torch.arange(n_pages - 1, n_pages - 33, -4, dtype=torch.int32, device="cuda")
    kv.kv_len[0, 0] = 1000
    qkv = torch.randn(new, 32 + 16, d, device="cuda").half()
    q, k, v = qkv.split((32, 8, 8), 1)
    q = qt.qtale_paged_rope_append(kv, 0, qt.Rope(d), q, k, v, offsets([new]), ints(list(range(1000 - new, 1000))))
    assert torch.equal(kv.v[int(kv.table[0, 0, 7]), :, 999 - 7 * 128], v[-1])
    got = qt.qtale_paged_attention(kv, 0, q, offsets([new]))
    _compare(kv, 0, q, got, [new], [1000 - new], [0], 0, 0, d ** -0.5, False)


def test_the_same_bits_every_time(qt):
    for new in ([1, 1, 1], [70, 1, 200]):
        kv, slots, q, out = _case(qt, torch.bfloat16, 4, 2, 128, 32, new, [3000, 50, 700])
        for _ in range(3):
            again = qt.qtale_paged_attention(kv, 1, q, offsets(new), first=ints([3000, 50, 700]), slots=ints(slots), max_new=max(new), max_len=max(3001, 900, 3070))
            assert torch.equal(again, qt.qtale_paged_attention(kv, 1, q, offsets(new), first=ints([3000, 50, 700]), slots=ints(slots), max_new=max(new), max_len=max(3001, 900, 3070)))


def test_no_tokens_and_a_step_of_several_streams(qt):
    kv, slots, q, out = _case(qt, torch.float16, 2, 2, 64, 16, [1, 1], [100, 30])
    empty = torch.empty(0, 4, 64, device="cuda", dtype=torch.float16)
    assert qt.qtale_paged_attention(kv, 1, empty, offsets([0, 0]), slots=ints(slots)).shape == (0, 4, 64)
    args = (offsets([1, 1]), ints([100, 30]), ints(slots))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = []
    for s in streams:                                            # a workspace each
        with torch.cuda.stream(s):
            outs.append(qt.qtale_paged_attention(kv, 1, q, args[0], first=args[1], slots=args[2], max_new=1, max_len=101))
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o, out)


@pytest.mark.parametrize("rep,page", [(4, 16), (1, 64)])
def test_a_captured_decode_step(qt, rep, page):
    # room, rotary append and attention of a step in one graph; every replay against the eager calls on a copy
    nkv, d, B = 2, 64, 5
    nh = rep * nkv
    lens = [14, 0, 63, 200, 31]
    kv, slots = random_cache(qt, lens, page, nkv, d, torch.float16, 6, spare=40, max_extra=4)
    twin = qt.PagedKV(*(t.clone() for t in (kv.k, kv.v, kv.page_refs, kv.free_bits, kv.table, kv.kv_len, kv.kv_cap)))
    rope, offs, slot = qt.Rope(d), offsets([1] * B), ints(slots)
    qkv, pos = torch.zeros(B, nh + 2 * nkv, d, device="cuda", dtype=torch.float16), ints([0] * B)
    ws_p, ws_a = qt.alloc_pages_workspace(kv, B), qt.alloc_paged_workspace(kv, nh, B, B, 1)
    turned, out = (torch.empty(B, nh, d, device="cuda", dtype=torch.float16) for _ in range(2))

    def step(cache, first, missing, turned, out):
        qt.qtale_pages_reserve(cache, offs, slots=slot, first=first, missing=missing, workspace=ws_p)
        q, k, v = qkv.split((nh, nkv, nkv), 1)
        qt.qtale_paged_rope_append(cache, 0, rope, q, k, v, offs, pos, first=first, slots=slot, q_out=turned)
        qt.qtale_paged_attention(cache, 0, turned, offs, first=first, slots=slot, out=out, max_new=1, workspace=ws_a)

    first, missing = ints([0] * B), ints([0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(kv, first, missing, turned, out)
    for i in range(20):
        qkv.normal_()
        pos.copy_(torch.tensor(lens, dtype=torch.int32) + i)
        first2, missing2 = ints([0] * B), ints([0])
        turned2, out2 = torch.empty_like(turned), torch.empty_like(out)
        step(twin, first2, missing2, turned2, out2)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, out2) and torch.equal(first, first2) and missing.item() == missing2.item() == 0
        for a, b in ((kv.table, twin.table), (kv.kv_len, twin.kv_len), (kv.page_refs, twin.page_refs), (kv.free_bits, twin.free_bits)):
            assert torch.equal(a, b)
        _compare(kv, 0, turned, out, [1] * B, [n + i for n in lens], slots, 0, 0, d ** -0.5, True)
