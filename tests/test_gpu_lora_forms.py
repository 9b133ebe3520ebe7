"""Low-rank adapters on the GPU (run with -m gpu) in every form of their kernels: ranks on both sides of 16, 32 and 64, alike and apart in a gated pair, for
few rows, more than 256 and more than 2048, with NaN past each adapter's rank; and the sums into the layers' residual."""
import pytest
import torch

import synth_inputs as si
from tests.kv4_precision import ADAPTERS16, GATED16, norm_error
from tests.test_gpu_lora import _adapters, _base, _expect, _ids
from tests.test_gpu_serving_stack import NAMES, _run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qt():
    import paper_2602_10431_amd as pkg
    pkg.load_library()
    return pkg


@pytest.mark.parametrize("r", [7, 16, 33, 61, 64, 65, 100, 128])
@pytest.mark.parametrize("M", [257, 300, 2100])
@pytest.mark.parametrize("pattern", ["mixed", "runs"])
def test_ranks_of_many_rows(qt, r, M, pattern):
    N, K = 328, 200
    q, base = _base(qt, N, K, 4, 64, r)
    ranks = [0, r, max(r // 2, 1), min(r, 9)]
    lora, down, up = _adapters(qt, 4, r, N, K, r, ranks, fill=float("nan"))
    x = torch.randn(M, K, generator=torch.Generator().manual_seed(r)).half().cuda()
    ids = _ids(pattern, M, 4, r)
    y, bound = _expect(base, lora, down, up, x, ids)
    assert bool(((qt.qtale_linear_lora_w4a16(q, lora, x, ids).double() - y).abs() <= bound).all())


def _gated(qt, rg, ru, M, N, K, ranks=None, pattern="mixed"):
    pairs = [_base(qt, N, K, 4, 64, s) for s in (1, 2)]
    of = lambda r, n: [r if a == 1 else (a * 5) % (r + 1) for a in range(n)]
    lg, dg, ug = _adapters(qt, 5, rg, N, K, 3, of(rg, 5), fill=float("nan"))
    lu, du, uu = _adapters(qt, 9, ru, N, K, 4, of(ru, 9), fill=float("nan"))
    x = torch.randn(M, K, generator=torch.Generator().manual_seed(M)).half().cuda()
    ids = _ids(pattern, M, 9, M)
    only = torch.full_like(ids, -1)
    for a, b in ((lg, lu), (lg, None), (None, lu)):
        g, bg = _expect(pairs[0][1], lg, dg, ug, x, ids if a else only, False)
        u, bu = _expect(pairs[1][1], lu, du, uu, x, ids if b else only, False)
        got = qt.qtale_swiglu_lora_w4a16(pairs[0][0], pairs[1][0], a, b, x, ids)
        s = torch.sigmoid(g)
        # silu's slope is at most 1.1; the product's rounding, and silu in 32 bits
        bound = 1.1 * bg * (u.abs() + bu) + (g * s).abs() * bu + (2.0 ** -11 + 2.0 ** -20) * (g * s * u).abs() + 2.0 ** -24
        assert bool(((got.double() - g * s * u).abs() <= bound).all()), (a is None, b is None)


@pytest.mark.parametrize("rg,ru", [(16, 24), (40, 64), (8, 128), (100, 33), (128, 128), (61, 61)])
@pytest.mark.parametrize("M", [6, 200, 256, 257, 513, 2100])
def test_gated_pairs_of_ranks(qt, rg, ru, M):
    _gated(qt, rg, ru, M, 456, 264)
    _gated(qt, rg, ru, M, 1032, 512, pattern="runs")


@pytest.mark.parametrize("r", [40, 100, 128])
def test_requests_of_many_rows(qt, r):
    N, K, M = 1032, 2048, 3000
    q, base = _base(qt, N, K, 4, 128, 9)
    lora, down, up = _adapters(qt, 3, r, N, K, 9, [r, 5, r // 2], fill=float("nan"))
    x = torch.randn(M, K, generator=torch.Generator().manual_seed(1)).half().cuda()
    ids = torch.tensor([0] * 1000 + [1] * 3 + [-1] * 497 + [2] * 1500, dtype=torch.int32).cuda()
    y, bound = _expect(base, lora, down, up, x, ids)
    assert bool(((qt.qtale_linear_lora_w4a16(q, lora, x, ids).double() - y).abs() <= bound).all())


@pytest.mark.parametrize("r", [24, 40, 64, 104, 128])
@pytest.mark.parametrize("names", [NAMES, ["o", "down"], ["k", "gate"]])
def test_layers(qt, r, names):
    shape = si.LayerShape(256, 4, 2, 64, 512, 4, 32, "fp16")
    _run(qt, shape, 4, names, [[30, 0, 17, 1], [1, 1, 1, 1], [1, 90, 2, 250]], "ratio", 0.7, 60 + r, r=r)
    _run(qt, shape, 16, names, [[3, 1], [1, 0], [500, 2]], "threshold", 0.5, 61 + r, r=r)


def test_layers_of_more_rows_than_a_small_tile_is_for(qt):
    shape = si.LayerShape(256, 4, 2, 64, 512, 4, 32, "fp16")
    _run(qt, shape, 4, NAMES, [[600, 300, 640, 620]], "ratio", 1.0, 71, r=72, page=64)


@pytest.mark.parametrize("M", [1, 3, 16, 64, 200, 300, 2100])
@pytest.mark.parametrize("r", [16, 60, 128])
def test_precision(qt, M, r):
    N, K = 1032, 1024
    (qg, g64), (qu, u64) = _base(qt, N, K, 4, 128, 5), _base(qt, N, K, 4, 128, 6)
    (lg, dg, ug), (lu, du, uu) = _adapters(qt, 4, r, N, K, 7), _adapters(qt, 4, r, N, K, 8)
    x = torch.randn(M, K, generator=torch.Generator().manual_seed(M)).half().cuda()
    ids = torch.arange(M, dtype=torch.int32).cuda() % 4
    (g, _), (u, _) = _expect(g64, lg, dg, ug, x, ids), _expect(u64, lu, du, uu, x, ids)
    assert norm_error(qt.qtale_linear_lora_w4a16(qg, lg, x, ids), g) <= ADAPTERS16
    assert norm_error(qt.qtale_swiglu_lora_w4a16(qg, qu, lg, lu, x, ids), g * torch.sigmoid(g) * u) <= GATED16


@pytest.mark.parametrize("M", [1, 5, 40, 200, 300, 2100])
def test_gated_rows_without_an_adapter_are_those_of_the_plain_pair(qt, M):
    # the same sums in 32 bits, or in another order, and silu in 32 bits: 2^-19 of the value, so that one in a hundred rounds to the neighbouring fp16 number
    N, K = 1032, 1024
    (qg, _), (qu, _) = _base(qt, N, K, 4, 128, 5), _base(qt, N, K, 4, 128, 6)
    lora, _, _ = _adapters(qt, 4, 16, N, K, 7)
    x = torch.randn(M, K, generator=torch.Generator().manual_seed(M)).half().cuda()
    ids = torch.where(torch.arange(M) % 3 == 0, -1, 7).int().cuda()
    got, want = qt.qtale_swiglu_lora_w4a16(qg, qu, lora, lora, x, ids), qt.qtale_swiglu_w4a16(qg, qu, x)
    assert bool(((got.double() - want.double()).abs() <= 2.0 ** -10 * want.double().abs() + 2.0 ** -22).all())
    assert float((got != want).double().mean()) <= 0.02
