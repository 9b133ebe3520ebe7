"""Attention over pages in 4 bits as a whole against 64 bits on the GPU (run with -m gpu): every kernel form, ordinary values."""
import math

import pytest
import torch

from tests.kv4_precision import beside, norm_error, precise
from tests.paged_helpers import TINY, U, attend64
from tests.test_gpu_paged4_sizes import FORMS, _best, _call

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


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("form", list(FORMS))
def test_one_key_that_takes_all_is_its_value(qt, form, dtype, d):
    # rows whose other keys weigh less than 2^-16 together, and rows that see one key: a probability of a power of two times a scale of 11 bits is not rounded, so
    # that the output's own rounding is left, 2^-15 for exponentials, the division and sums in 32 bits, and 2^-11 of what the other keys add
    kv, slots, dense, q, new, old, attend = _call(qt, form, dtype, d, 47)
    top = float(torch.nan_to_num(dense.v).abs().max())
    for how in (dict(window=1), dict(scale=5.0), dict(scale=40.0)):
        out = attend(**how)
        want, _ = attend64(dense, 0, q, new, old, slots, how.get("window", 0), 0, how.get("scale", d ** -0.5))
        clear = torch.ones(out.shape[:2], dtype=torch.bool, device="cuda")
        if "scale" in how:
            clear = _best(kv, dense, q, new, old, slots)[1] * how["scale"] > 16 * math.log(2) + math.log(max(map(sum, zip(old, new))))
            assert int(clear.sum()) > clear.numel() // 8
        wrong = ((out.double() - want).abs() > (U[dtype] + 2.0 ** -15) * want.abs() + 2.0 ** -26 * top + TINY[dtype]) & clear[..., None]
        assert not bool(wrong.any()), (how, wrong.nonzero()[:3].tolist(), out[wrong][:3].tolist(), want[wrong][:3].tolist())
