"""Attention over pages in 4 bits as a whole against 64 bits on the GPU (run with -m gpu): every kernel form, ordinary values."""
import pytest
import torch

from tests.kv4_precision import beside, norm_error, precise
from tests.paged_helpers import attend64
from tests.test_gpu_paged4_sizes import FORMS, _call

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qt():
    import paper_2602_10431_amd as pkg
    pkg.load_library()
    return pkg


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("window,sinks", [(0, 0), (200, 5)])
def test_precision(qt, form, dtype, d, window, sinks):
    for q_size in (1.0, 3.0):
        kv, slots, dense, q, new, old, attend = _call(qt, form, dtype, d, 43, q_size=q_size)
        out = attend(window=window, sinks=sinks)
        want, _ = attend64(dense, 0, q, new, old, slots, window, sinks, d ** -0.5)
        assert precise(out, want), (q_size, norm_error(out, want), beside(out, want))
