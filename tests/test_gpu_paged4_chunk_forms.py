"""The chunk kernel over pages in 4 bits where small calls would take the form of few columns: with key ranges, as a program gets them that passes its cache's
capacity as the bound on the keys and whose slots have room for many more tokens than they hold; without, in calls that fill the chip, with windows, missing
pages and rows that are not finite."""
import math

import pytest
import torch

import tests.test_gpu_paged4_attention as small
from tests.kv4_helpers import pack, random_cache4, unpack
from tests.paged_helpers import attend64, ints, offsets
from tests.test_gpu_paged4_attention import (test_chunks, test_missing_pages, test_random_calls, test_repeated_calls_give_the_same_bits,  # noqa: F401
                                       test_graph_and_side_stream, test_rows_that_are_not_finite_reach_only_who_sees_them, test_rows_that_see_nothing,
                                       test_scales_of_all_sizes, test_scores_of_any_size)
from tests.test_gpu_paged4_chunk import _Loose

pytestmark = pytest.mark.gpu
ROOM = 1 << 18                                                   # tokens that a slot has room for, and the bound on its keys


@pytest.fixture(scope="module")
def qt():
    import paper_2602_10431_amd
    return _Loose(paper_2602_10431_amd)


@pytest.fixture(autouse=True)
def _slots_with_room(monkeypatch):
    monkeypatch.setattr(small, "random_cache4", lambda qt, lens, page, *a, **kw: random_cache4(qt, lens, page, *a, **dict(kw, max_extra=ROOM // page)))


@pytest.fixture
def tight(monkeypatch):
    import paper_2602_10431_amd
    monkeypatch.setattr(small, "random_cache4", random_cache4)
    return paper_2602_10431_amd


NEW, OLD = [600, 500, 700, 590, 3], [0, 37, 64, 1000, 5]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("window,sinks", [(1, 0), (50, 3), (64, 64), (300, 100), (333, 0)])
def test_windows_of_calls_that_fill_the_chip(tight, dtype, window, sinks):
    for d, page in ((64, 16), (128, 64)):
        small._case(tight, dtype, 4, 8, d, page, NEW, OLD, window, sinks)


@pytest.mark.parametrize("page", [16, 32, 64, 256])
def test_missing_pages_of_calls_that_fill_the_chip(tight, page):
    gone = [(0, 0), (0, 1), (1, 100 // page), (2, 64 // page), (3, 1000 // page), (3, 3)] + [(4, j) for j in range(16)]
    for d in (64, 128):
        out = small._case(tight, torch.float16, 4, 8, d, page, NEW, OLD, gone=gone)[-1]
        assert bool((out[-3:] == 0).all())
        small._case(tight, torch.bfloat16, 4, 8, d, page, NEW, OLD, 130, 20, gone=gone)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_that_are_not_finite_of_calls_that_fill_the_chip(tight, dtype, d):
    lens = [o + n for o, n in zip(OLD, NEW)]
    kv, slots, dense = random_cache4(tight, lens, 32, 8, d, dtype, 17)
    where = [(0, 599, True, 0), (0, 300, False, 1), (2, 64 + 699, False, 2), (3, 1003, True, 3), (1, 400, False, 3)]   # (sequence, token, keys, head)
    for b, t, keys, head in where:
        pool = kv.k if keys else kv.v
        codes, scale, zero = unpack(pool, d, keys, dtype)
        scale = scale.clone()
        scale[int(kv.table[0, slots[b], t // 32]), head, t % 32] = math.nan
        pool.copy_(pack(codes, scale, zero, keys))
    q = torch.randn(sum(NEW), 32, d, generator=torch.Generator().manual_seed(8)).to(dtype).cuda()
    for window in (0, 200):
        out = tight.qtale_paged_attention(kv, 0, q, offsets(NEW), first=ints(OLD), slots=ints(slots), max_new=max(NEW), max_len=max(lens), window=window)
        hit = torch.zeros(sum(NEW), 32, dtype=torch.bool, device="cuda")
        for b, t, _, head in where:
            place = torch.arange(NEW[b], device="cuda") + OLD[b]
            hit[sum(NEW[:b]): sum(NEW[:b + 1]), 4 * head: 4 * head + 4] |= ((place >= t) & ((place < t + window) | (window == 0)))[:, None]
        assert torch.equal(out.isnan().all(2), hit) and torch.equal(out.isnan().any(2), hit)
        want, size = attend64(dense, 0, q, NEW, OLD, slots, window, 0, d ** -0.5)                    # (the values beside the pages are without NaN)
        bound = small.attention_bound4(want, size, q, dtype, d ** -0.5, small._largest_scale(dense, None, d))
        assert bool((((out.double() - want).abs() <= bound) | hit[..., None]).all())
