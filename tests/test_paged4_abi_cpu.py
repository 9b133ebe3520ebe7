"""CPU-only checks of pages in 4 bits and of reading entries: types, shapes and pointers that are refused before any GPU work, and sizes."""
import ctypes as C
import os

import pytest
import torch

from tests.kv4_helpers import pack, quantize64, unpack, values64

FAKE = C.c_void_p(256)
ODD = C.c_void_p(258)


@pytest.fixture(scope="module")
def qt():
    import paper_2602_10431_amd as pkg
    if not os.path.exists(pkg.LIB_PATH):
        from paper_2602_10431_amd import build
        build.build(verbose=False)
    pkg.load_library()
    return pkg


def _kv(qt, **how):
    a = dict(k_pages=256, v_pages=256, page_refs=256, free_bits=256, table=256, kv_len=256, kv_cap=256, n_pages=100, page_size=32,
             n_kv_heads=4, head_dim=128, n_layers=3, n_slots=6, max_pages=20, dtype=qt.QTALE_KV_INT4)
    a.update(how)
    return C.byref(qt.qtale_paged_kv(**a))


def test_types(qt):
    lib = qt.load_library()
    for dtype, code in ((0, True), (1, True), (4, True), (5, True), (2, False), (3, False), (6, False), (7, False), (8, False), (12, False), (-1, False)):
        assert (lib.qtale_pages_workspace_bytes(_kv(qt, dtype=dtype), 2) > 0) == code, dtype
        if not code:
            assert lib.qtale_pages_init(_kv(qt, dtype=dtype), None) == -3
    for how, code in ((dict(head_dim=96), -3), (dict(page_size=8), -3), (dict(k_pages=264), -1), (dict(v_pages=None), -1)):
        assert lib.qtale_pages_init(_kv(qt, **how), None) == code
    for dtype in (0, 1, 5):                                       # pages of another form are not copied
        assert lib.qtale_pages_copy(_kv(qt), _kv(qt, dtype=dtype), FAKE, FAKE, 1, None) == -2


def test_read_refuses(qt):
    lib = qt.load_library()
    for kv in (_kv(qt), _kv(qt, dtype=1)):
        def call(layer=0, k=FAKE, ks=512, v=FAKE, vs=512, T=4, offs=FAKE, slots=FAKE, B=2):
            return lib.qtale_paged_read(kv, layer, k, ks, v, vs, T, offs, slots, None, B, None)

        assert call(layer=3) == -1 and call(layer=-1) == -1 and call(T=-1) == -1 and call(B=-1) == -1 and call(B=0) == -1
        for missing in ("k", "v", "offs"):
            assert call(**{missing: None}) == -1
        assert call(k=ODD) == -1 and call(v=ODD) == -1
        assert call(ks=504) == -2 and call(vs=516) == -2 and call(slots=None, B=7) == -2
        assert call(T=0) == 0
    assert lib.qtale_paged_read(None, 0, FAKE, 512, FAKE, 512, 4, FAKE, FAKE, None, 2, None) == -1


def test_python_cache_checks(qt):
    ints = lambda *n: torch.zeros(*n, dtype=torch.int32)
    k = torch.zeros(5, 2, 16 * 36, dtype=torch.uint8)
    rest = (ints(5), ints(1), ints(1, 2, 3), ints(1, 2), ints(1, 2))
    kv = qt.PagedKV(k, k.clone(), *rest, dtype=torch.bfloat16, head_dim=64)
    assert (kv.bits, kv.page_size, kv.head_dim, kv.dtype, kv.c_struct().dtype) == (4, 16, 64, torch.bfloat16, 5)
    for bad in (dict(dtype=torch.bfloat16), dict(head_dim=64), dict(dtype=torch.float32, head_dim=64), dict(dtype=torch.float16, head_dim=128)):
        with pytest.raises(AssertionError):
            qt.PagedKV(k, k.clone(), *rest, **bad)
    x = torch.zeros(5, 2, 16, 64, dtype=torch.float16)
    assert qt.PagedKV(x, x.clone(), *rest).c_struct().dtype == 0
    with pytest.raises(AssertionError):
        qt.PagedKV(x, x.clone(), *rest, dtype=torch.bfloat16)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
def test_the_model_packs_and_holds_values(dtype, d):
    # the tests' own model: packing and its inverse, and that a value is off by half a step (of the rounded scale) at most
    x = torch.randn(3, 2, 16, d, generator=torch.Generator().manual_seed(1)).to(dtype)
    codes, scale, zero = quantize64(x)
    for keys in (True, False):
        block = pack(codes, scale, zero, keys)
        assert block.shape == (3, 2, 16 * (d // 2 + 4))
        back = unpack(block, d, keys, dtype)
        assert torch.equal(back[0], codes) and torch.equal(back[1], scale) and torch.equal(back[2], zero)
    # the scale is off by half a unit, so an end of the range by up to 15 of those on top of half a step
    u = 2.0 ** -11 if dtype == torch.float16 else 2.0 ** -8
    assert bool(((values64(codes, scale, zero) - x.double()).abs() <= scale.double()[..., None] * (0.5 + 16 * u + 0.5)).all())
    assert bool(((values64(codes, scale, zero) - x.double()).abs() <= scale.double()[..., None] * (0.5 + 16 * u)).double().mean() > 0.97)
