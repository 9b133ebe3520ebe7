"""CPU-only checks of the paged cache's calls: refusals before any GPU work, sizes, and the rotary frequencies against their formulas."""
import ctypes as C
import math
import os

import pytest

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
             n_kv_heads=4, head_dim=128, n_layers=3, n_slots=6, max_pages=20, dtype=0)
    a.update(how)
    return C.byref(qt.qtale_paged_kv(**a))


BAD_CACHES = [(dict(n_pages=0), -1), (dict(n_layers=-1), -1), (dict(n_slots=0), -1), (dict(max_pages=0), -1), (dict(n_kv_heads=0), -1),
              (dict(page_size=0), -1), (dict(page_size=8), -3), (dict(page_size=48), -3), (dict(page_size=2048), -3), (dict(head_dim=96), -3),
              (dict(dtype=2), -3), (dict(n_layers=65536), -3), (dict(max_pages=1 << 26, page_size=32), -3), (dict(n_pages=(1 << 30) + 1), -3)]
NO_BUFFER = [(dict(k_pages=None), -1), (dict(v_pages=None), -1), (dict(page_refs=None), -1), (dict(free_bits=None), -1), (dict(table=None), -1),
             (dict(kv_len=None), -1), (dict(kv_cap=None), -1), (dict(k_pages=264), -1)]


@pytest.mark.parametrize("how,code", BAD_CACHES + NO_BUFFER)
def test_every_call_refuses_a_bad_cache(qt, how, code):
    lib = qt.load_library()
    kv, attn, rope = _kv(qt, **how), qt.qtale_paged_attn(8, 0, 0, 0.1, 1, 0), qt.qtale_rope(0, 64, 256, 1.0)
    assert lib.qtale_pages_init(kv, None) == code
    assert lib.qtale_pages_init(None, None) == -1
    assert lib.qtale_pages_fork(kv, FAKE, FAKE, 2, None) == code
    assert lib.qtale_pages_release(kv, FAKE, 2, None) == code
    assert lib.qtale_pages_trim(kv, FAKE, 2, 4, 0, None) == code
    assert lib.qtale_pages_reserve(kv, -1, FAKE, FAKE, 2, None, None, FAKE, 1 << 20, None) == code
    assert lib.qtale_pages_compact(kv, None, FAKE, 1 << 20, None) == code
    assert lib.qtale_pages_copy(kv, _kv(qt), FAKE, FAKE, 1, None) == code
    assert lib.qtale_pages_copy(_kv(qt), kv, FAKE, FAKE, 1, None) == code
    assert lib.qtale_paged_rope_append(kv, 0, C.byref(rope), FAKE, 1024, FAKE, 512, FAKE, 512, FAKE, 1024, 8, 4, FAKE, FAKE, FAKE, 2, FAKE, None) == code
    assert lib.qtale_paged_attention(kv, 0, C.byref(attn), FAKE, 1024, FAKE, 1024, 4, FAKE, FAKE, FAKE, 2, FAKE, 1 << 30, None) == code
    if (how, code) in BAD_CACHES:                                # sizes do not look at the buffers
        assert lib.qtale_pages_workspace_bytes(kv, 2) == 0
        assert lib.qtale_paged_attention_workspace_bytes(kv, C.byref(attn), 4, 2) == 0
    else:
        assert lib.qtale_pages_workspace_bytes(kv, 2) > 0


def test_page_calls_refuse(qt):
    lib, kv = qt.load_library(), _kv(qt)
    ws = lib.qtale_pages_workspace_bytes(kv, 4)
    assert ws >= 256 + 3 * 4 * 16 and lib.qtale_pages_workspace_bytes(kv, 0) >= 256 + 100 * 12
    assert lib.qtale_pages_workspace_bytes(kv, -1) == 0 and lib.qtale_pages_workspace_bytes(kv, 2049) == 0
    reserve = lambda layer=-1, offs=FAKE, slots=FAKE, B=4, work=FAKE, size=ws: lib.qtale_pages_reserve(kv, layer, offs, slots, B, None, None, work, size, None)
    assert reserve(layer=3) == -1 and reserve(layer=-2) == -1 and reserve(B=-1) == -1 and reserve(offs=None) == -1
    assert reserve(B=2049) == -3 and reserve(slots=None, B=7) == -2
    assert reserve(work=None) == -1 and reserve(work=ODD) == -1 and reserve(size=ws - 1) == -4
    assert reserve(B=0) == 0
    assert lib.qtale_pages_fork(kv, None, FAKE, 1, None) == -1 and lib.qtale_pages_fork(kv, FAKE, FAKE, -1, None) == -1
    assert lib.qtale_pages_fork(kv, None, None, 0, None) == 0
    assert lib.qtale_pages_release(kv, FAKE, -1, None) == -1 and lib.qtale_pages_release(kv, None, 7, None) == -2 and lib.qtale_pages_release(kv, FAKE, 0, None) == 0
    assert lib.qtale_pages_trim(kv, FAKE, 1, 0, 0, None) == -1 and lib.qtale_pages_trim(kv, FAKE, 1, 1, -1, None) == -1
    assert lib.qtale_pages_trim(kv, None, 7, 1, 0, None) == -2 and lib.qtale_pages_trim(kv, None, 0, 1, 0, None) == 0
    assert lib.qtale_pages_compact(kv, None, FAKE, 256, None) == -4 and lib.qtale_pages_compact(kv, None, ODD, 1 << 20, None) == -1
    for other in (dict(page_size=64), dict(n_kv_heads=8), dict(head_dim=64), dict(dtype=1)):
        assert lib.qtale_pages_copy(kv, _kv(qt, **other), FAKE, FAKE, 1, None) == -2
    assert lib.qtale_pages_copy(kv, kv, None, FAKE, 1, None) == -1 and lib.qtale_pages_copy(kv, kv, FAKE, FAKE, 0, None) == 0


def test_rope_append_refuses(qt):
    lib, kv = qt.load_library(), _kv(qt)

    def call(rope=(0, 64, 256, 1.0), layer=0, q=FAKE, qs=1024, k=FAKE, ks=512, v=FAKE, vs=512, out=FAKE, os_=1024, nh=8, T=4, offs=FAKE, slots=FAKE,
             B=2, pos=FAKE):
        r = None if rope is None else C.byref(qt.qtale_rope(*rope))
        return lib.qtale_paged_rope_append(kv, layer, r, q, qs, k, ks, v, vs, out, os_, nh, T, offs, slots, None, B, pos, None)

    assert call(rope=None) == -1 and call(rope=(0, 64, None, 1.0)) == -1 and call(rope=(0, 64, 256, math.inf)) == -1
    assert call(rope=(2, 64, 256, 1.0)) == -3
    for rd in (0, 63, 130, -2):
        assert call(rope=(0, rd, 256, 1.0)) == -2
    assert call(layer=3) == -1 and call(layer=-1) == -1 and call(T=-1) == -1 and call(B=-1) == -1 and call(B=0) == -1 and call(nh=0) == -1
    for missing in ("q", "k", "v", "out", "offs", "pos"):
        assert call(**{missing: None}) == -1
    for odd in ("q", "k", "v", "out"):
        assert call(**{odd: ODD}) == -1
    assert call(qs=1016) == -2 and call(qs=1028) == -2 and call(ks=504) == -2 and call(vs=513) == -2 and call(os_=1020) == -2
    assert call(slots=None, B=7) == -2
    assert call(T=0) == 0


def test_attention_refuses(qt):
    lib, kv = qt.load_library(), _kv(qt)

    def call(attn=(8, 0, 0, 0.1, 1, 0), layer=0, q=FAKE, qs=1024, out=FAKE, os_=1024, T=4, offs=FAKE, slots=FAKE, B=4, work=FAKE, size=1 << 30):
        a = None if attn is None else C.byref(qt.qtale_paged_attn(*attn))
        return lib.qtale_paged_attention(kv, layer, a, q, qs, out, os_, T, offs, slots, None, B, work, size, None)

    assert call(attn=None) == -1 and call(attn=(0, 0, 0, 0.1, 1, 0)) == -1 and call(attn=(6, 0, 0, 0.1, 1, 0)) == -2
    for scale in (0.0, -1.0, math.nan, math.inf):
        assert call(attn=(8, 0, 0, scale, 1, 0)) == -1
    for attn in ((8, -1, 0, 0.1, 1, 0), (8, 5, -1, 0.1, 1, 0), (8, 0, 0, 0.1, -1, 0), (8, 0, 0, 0.1, 1, -1)):
        assert call(attn=attn) == -1
    assert call(layer=3) == -1 and call(layer=-1) == -1 and call(T=-1) == -1 and call(B=0) == -1 and call(B=62000) == -3 and call(slots=None, B=7) == -2
    for missing in ("q", "out", "offs", "work"):
        assert call(**{missing: None}) == -1
    assert call(q=C.c_void_p(264)) == -1 and call(out=C.c_void_p(260)) == -1 and call(work=ODD) == -1
    assert call(qs=1020) == -2 and call(qs=1000) == -2 and call(os_=1022) == -2
    assert call(size=16) == -4
    assert call(T=0) == 0
    size = lambda *attn: lib.qtale_paged_attention_workspace_bytes(kv, C.byref(qt.qtale_paged_attn(*attn)), 4, 4)
    assert size(8, 0, 0, 0.1, 1, 0) % 256 == 0 and size(8, 0, 0, -0.1, 1, 0) == 0


def _formula(rd, base, scaling, factor, length, low, high):
    """Written from the definitions in the header, pair by pair."""
    if scaling == "base":
        base = base * factor ** (rd / (rd - 2))
    w = [base ** (-2.0 * i / rd) for i in range(rd // 2)]
    if scaling == "linear":
        return [x / factor for x in w], 1.0
    if scaling == "bands":
        out = []
        for x in w:
            turns = length * x / (2 * math.pi)
            if turns >= high:
                out.append(x)
            elif turns <= low:
                out.append(x / factor)
            else:
                t = (turns - low) / (high - low)
                out.append(t * x + (1 - t) * x / factor)
        return out, 1.0
    if scaling == "parts":
        at = lambda turns: rd * math.log(length / (turns * 2 * math.pi)) / (2 * math.log(base))
        lo, hi = max(math.floor(at(high)), 0), min(math.ceil(at(low)), rd - 1)
        ramp = [min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0) for i in range(rd // 2)]
        return [x / factor * r + x * (1 - r) for x, r in zip(w, ramp)], 0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0
    return w, 1.0


@pytest.mark.parametrize("rd", [4, 16, 48, 64, 128])
@pytest.mark.parametrize("scaling,factor,length,low,high", [("none", 1.0, 0, 0.0, 0.0), ("linear", 4.0, 0, 0.0, 0.0), ("base", 8.0, 0, 0.0, 0.0),
                                                            ("bands", 8.0, 8192, 1.0, 4.0), ("bands", 2.5, 1000, 0.5, 32.0),
                                                            ("parts", 16.0, 4096, 1.0, 32.0), ("parts", 0.5, 2048, 1.0, 8.0)])
@pytest.mark.parametrize("base", [10000.0, 500000.0])
def test_frequencies(qt, rd, scaling, factor, length, low, high, base):
    got, magnitude = qt.qtale_rope_frequencies(rd, base, scaling, factor, length, low, high)
    want, want_magnitude = _formula(rd, base, scaling, factor, length, low, high)
    assert got.tolist() == pytest.approx(want, rel=1e-12) and magnitude == pytest.approx(want_magnitude, rel=1e-7)


def test_frequencies_keep_their_ends(qt):
    # stretched by `factor` at the slow end, untouched at the fast end, in between at most the plain frequency
    plain, _ = qt.qtale_rope_frequencies(128, 10000.0)
    for scaling, how in (("bands", dict(factor=8.0, original_len=8192, low=1.0, high=4.0)), ("parts", dict(factor=8.0, original_len=8192, low=1.0, high=32.0)),
                         ("base", dict(factor=8.0))):
        f, _ = qt.qtale_rope_frequencies(128, 10000.0, scaling, **how)
        assert f[0] == plain[0] and float(plain[-1] / f[-1]) == pytest.approx(8.0, rel=1e-6)
        assert bool((f <= plain * (1 + 1e-15)).all())


def test_frequencies_refuse(qt):
    lib = qt.load_library()
    f, m = (C.c_double * 64)(), C.c_float()
    call = lambda rd=128, base=1e4, how=0, factor=1.0, n=0, low=0.0, high=0.0, out=f, mag=C.byref(m): lib.qtale_rope_frequencies(rd, base, how, factor, n, low, high, out, mag)
    assert call() == 0
    assert call(rd=0) == -1 and call(rd=7) == -1 and call(base=0.0) == -1 and call(base=math.nan) == -1 and call(base=math.inf) == -1
    assert call(out=None) == -1 and call(mag=None) == -1 and call(how=5) == -3 and call(how=-1) == -3
    assert call(how=1, factor=0.0) == -1 and call(how=1, factor=math.nan) == -1 and call(how=2, rd=2, factor=2.0) == -3
    for how in (3, 4):
        assert call(how=how, factor=2.0, n=0, low=1.0, high=4.0) == -1
        assert call(how=how, factor=2.0, n=10, low=0.0, high=4.0) == -1
        assert call(how=how, factor=2.0, n=10, low=4.0, high=4.0) == -1
    assert call(how=4, base=1.0, factor=2.0, n=10, low=1.0, high=4.0) == -1


def test_paged_stack_refuses(qt):
    lib = qt.load_library()
    ctx = qt.Context()
    cfg = qt.make_cfg(256, 8, 4, 128, 512, group=32, act_dtype="fp16")
    w = qt.qtale_layer_weights()
    size = lib.qtale_paged_stack_workspace_bytes(C.byref(cfg), _kv(qt), 4, 2)
    assert size > qt.qtale_workspace_bytes(cfg, 4, 2)
    assert lib.qtale_paged_stack_workspace_bytes(C.byref(cfg), _kv(qt, page_size=8), 4, 2) == 0
    assert lib.qtale_paged_stack_workspace_bytes(C.byref(cfg), _kv(qt), 4, 2049) == 0

    def call(cfg_=cfg, kv=None, layers=True, n=1, first=0, x=FAKE, T=4, offs=FAKE, B=2, pos=FAKE, slots=FAKE, rope=(0, 64, 256, 1.0),
             attn=(8, 0, 0, 0.1, 1, 0), work=FAKE, room=size):
        return lib.qtale_paged_stack_forward(ctx._h, C.byref(cfg_), C.byref(w) if layers else None, n, first, x, T, offs, B, pos, kv or _kv(qt), slots,
                                             None if rope is None else C.byref(qt.qtale_rope(*rope)), None if attn is None else C.byref(qt.qtale_paged_attn(*attn)),
                                             None, None, None, None, work, room, None)

    assert call() == -1                                          # weights without prepacked buffers
    assert call(n=0) == 0 and call(T=0) == -1 and call(T=0, n=0) == 0
    assert call(layers=False) == -1 and call(n=-1) == -1 and call(first=-1) == -1 and call(first=3) == -2 and call(first=2, n=2) == -2
    for missing in ("x", "offs", "pos", "work"):
        assert call(**{missing: None}) == -1
    assert call(rope=None) == -1 and call(rope=(0, 200, 256, 1.0)) == -2 and call(attn=None) == -1 and call(attn=(8, 0, 0, 0.0, 1, 0)) == -1
    assert call(attn=(4, 0, 0, 0.1, 1, 0)) == -2 and call(kv=_kv(qt, n_kv_heads=8)) == -2 and call(kv=_kv(qt, head_dim=64)) == -2
    assert call(kv=_kv(qt, dtype=1)) == -3 and call(kv=_kv(qt, table=None)) == -1 and call(B=0) == -1 and call(slots=None, B=7, room=1 << 40) == -2
    assert call(B=3000, room=1 << 40) == -3 and call(room=16) == -4
