"""Attention over pages at the ends of its arguments' ranges (run with -m gpu): windows up to the largest 32-bit number, with queries whose places lie
before their slot's begin; the same call again and again."""
import pytest
import torch

from tests.paged_helpers import attend64, attention_bound, ints, offsets, random_cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qt():
    import paper_2602_10431_amd as pkg
    pkg.load_library()
    return pkg


@pytest.mark.parametrize("window", [(1 << 31) - 1, (1 << 31) - 3, 1 << 30])
@pytest.mark.parametrize("sinks", [0, 2, (1 << 31) - 1])
@pytest.mark.parametrize("new,d,nkv,rep,max_len", [([5, 6, 1], 64, 2, 2, 0), ([16, 9, 2], 128, 1, 1, 0), ([40, 70, 33] * 2, 64, 2, 4, 9000),
                                                   ([40, 70, 33] * 40, 128, 2, 4, 0)])
def test_a_window_without_end(qt, new, d, nkv, rep, max_len, window, sinks):
    # slots with fewer entries than new tokens, which are their last ones: the first queries' places are negative and see nothing, the others see all
    # before them, as without a window
    lens = [(2, 5, 50)[b % 3] for b in range(len(new))]
    kv, slots = random_cache(qt, lens, 16, nkv, d, torch.float16, 3, max_extra=12)
    q = torch.randn(sum(new), rep * nkv, d, generator=torch.Generator().manual_seed(1)).half().cuda()
    first = [a - n for a, n in zip(lens, new)]
    got = qt.qtale_paged_attention(kv, 0, q, offsets(new), slots=ints(slots), window=window, sinks=sinks, max_new=max(new), max_len=max_len)
    plain = qt.qtale_paged_attention(kv, 0, q, offsets(new), slots=ints(slots), max_new=max(new), max_len=max_len)
    want, size = attend64(kv, 0, q, new, first, slots, window, sinks, d ** -0.5)
    assert bool(((got.double() - want).abs() <= attention_bound(want, size, q.dtype, False)).all())
    assert bool(((plain.double() - want).abs() <= attention_bound(want, size, q.dtype, False)).all())
    assert bool((want.abs().amax((1, 2)) > 0).any())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("new,old,rep,nkv,d,bound", [([1, 1, 1], [3000, 50, 700], 4, 2, 128, 0), ([1] * 5, [30, 900, 0, 64, 500], 1, 60, 64, 0),
                                                     ([70, 1, 200], [3000, 50, 700], 4, 2, 128, 30000), ([64] * 16, [1000] * 16, 4, 8, 64, 0),
                                                     ([1400, 1300], [2000, 900], 16, 8, 128, 0)])
def test_repeated_calls_give_the_bits_of_the_first(qt, new, old, rep, nkv, d, bound, dtype):
    lens = [o + n for o, n in zip(old, new)]
    kv, slots = random_cache(qt, lens, 32, nkv, d, dtype, 5)
    q = torch.randn(sum(new), rep * nkv, d, generator=torch.Generator().manual_seed(6)).to(dtype).cuda()
    call = lambda: qt.qtale_paged_attention(kv, 0, q, offsets(new), first=ints(old), slots=ints(slots), max_new=max(new), max_len=bound or max(lens))
    one = call()
    assert bool(torch.isfinite(one).all())
    for _ in range(4):
        assert torch.equal(one, call())
