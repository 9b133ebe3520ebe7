"""What the precision asked of attention over pages in 4 bits and of adapters can tell apart: models of the kernels with a rounding too many, on the CPU."""
import pytest
import torch

from tests.kv4_helpers import quantize64, values64
from tests.kv4_precision import ADAPTERS16, norm_error, precise


def _round(x, bits):
    """To `bits` bits of mantissa, half to even."""
    m, e = torch.frexp(x)
    return torch.ldexp(torch.round(m * 2.0 ** bits) / 2.0 ** bits, e)


def _model(dtype, d, n, keys, seed, probabilities=11, queries=None, scales=None):
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(n, d, generator=g).to(dtype).double()
    k, v = (values64(*quantize64(torch.randn(keys, d, generator=g).to(dtype))) for _ in range(2))
    codes, scale, zero = quantize64(torch.randn(keys, d, generator=g).to(dtype))
    v = values64(codes, scale, zero)
    want = torch.softmax(q @ k.T * d ** -0.5, 1) @ v
    p = torch.softmax((q if queries is None else _round(q, queries)) @ k.T * d ** -0.5, 1)
    t = scale.double() if scales is None else _round(scale.double(), scales)
    out = _round(p * t, probabilities) @ (codes - zero[:, None]).double()
    return out.to(dtype), want


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d,n,keys", [(64, 64, 300), (128, 64, 300), (128, 32, 1000), (64, 32, 5000)])
def test_roundings_that_are_told_apart(dtype, d, n, keys):
    for seed in range(3):
        assert precise(*_model(dtype, d, n, keys, seed))
        assert not precise(*_model(dtype, d, n, keys, seed, probabilities=8))         # bf16
        assert not precise(*_model(dtype, d, n, keys, seed, probabilities=7))
        if dtype == torch.float16:                                # (bf16's own scales and queries have 8 bits)
            assert not precise(*_model(dtype, d, n, keys, seed, scales=8))
            assert not precise(*_model(dtype, d, n, keys, seed, queries=8))


@pytest.mark.parametrize("K,N,r", [(512, 256, 16), (1024, 512, 64)])
def test_roundings_of_adapters_that_are_told_apart(K, N, r):
    for seed in range(3):
        g = torch.Generator().manual_seed(seed)
        x, w = torch.randn(64, K, generator=g).half().double(), torch.randn(N, K, generator=g).double() / K ** 0.5
        down, up = (torch.randn(r, K, generator=g) / K ** 0.5).half().double(), (torch.randn(N, r, generator=g) / r ** 0.5).half().double()
        want = x @ w.T + x @ down.T @ up.T
        model = lambda inner, base: (base(x @ _round(w, 11).T) + inner(x @ down.T) @ up.T).half()
        assert norm_error(model(lambda y: _round(y, 11), lambda y: y), want) <= ADAPTERS16
        assert norm_error(model(lambda y: _round(y, 8), lambda y: y), want) > ADAPTERS16              # bf16 inner values
        assert norm_error(model(lambda y: _round(y, 11), lambda y: _round(y, 8)), want) > ADAPTERS16  # or a shared product rounded to bf16
