"""The chunk kernels over pages in 4 bits.  Small calls take the form of few columns, whose workgroups walk all keys; with a loose bound on the keys, as a
program passes that always gives its cache's capacity, the calls of the other module's tests take the chunk kernels with key ranges instead.  Calls that fill
the chip take them without ranges."""
import pytest
import torch

from tests.test_gpu_paged4_attention import (_case, test_chunks, test_chunks_with_key_ranges_and_many_tiles, test_graph_and_side_stream,  # noqa: F401
                                       test_missing_pages, test_random_calls, test_repeated_calls_give_the_same_bits, test_rows_that_are_not_finite_reach_only_who_sees_them,
                                       test_rows_that_see_nothing, test_scales_of_all_sizes, test_scores_of_any_size, test_windows)

pytestmark = pytest.mark.gpu
LOOSE = 1 << 20


class _Loose:
    """The package, with LOOSE in place of attention's max_len."""

    def __init__(self, package):
        self._package = package

    def __getattr__(self, name):
        return getattr(self._package, name)

    def qtale_paged_attention(self, *args, max_len=0, **kw):
        return self._package.qtale_paged_attention(*args, max_len=LOOSE, **kw)

    def alloc_paged_workspace(self, kv, n_heads, T, B, max_new=0, max_len=0):
        return self._package.alloc_paged_workspace(kv, n_heads, T, B, max_new, LOOSE)


@pytest.fixture(scope="module")
def qt():
    import paper_2602_10431_amd
    return _Loose(paper_2602_10431_amd)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new,old", [([1000, 900, 700, 1100], [0, 0, 130, 7]), ([32] * 63 + [3], list(range(900, 1540, 10)))])
def test_calls_that_fill_the_chip(dtype, d, new, old):
    import paper_2602_10431_amd
    _case(paper_2602_10431_amd, dtype, 4, 8, d, 64, new, old)
