"""Rotary embedding with the append on the GPU (run with -m gpu) against 64 bits: layouts, parts of the head, scalings, late positions, strides, in
place, dropped entries."""
import pytest
import torch

from tests.paged_helpers import TINY, U, ints, offsets, random_cache, turn64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qt():
    import paper_2602_10431_amd as pkg
    pkg.load_library()
    return pkg


def _check(got, want, size, dtype, what):
    # one rounding to the type; cosine, sine, two products and a sum in 32 bits: less than 6 * 2^-24 of the products
    bound = U[dtype] * want.abs() + 6 * 2.0 ** -24 * size + TINY[dtype]
    assert bool(((got.double() - want).abs() <= bound).all()), what


def _case(qt, dtype, nh, nkv, d, page, new, old, layout="half", rd=None, scaling="none", late=0, in_place=False, given_first=True, seed=0, how=None):
    rd = d if rd is None else rd
    lens = [o + n for o, n in zip(old, new)]
    kv, slots = random_cache(qt, lens, page, nkv, d, dtype, seed, n_layers=2, layer=1)
    T = sum(new)
    g = torch.Generator().manual_seed(seed + 1)
    qkv = torch.randn(T, (nh + 2 * nkv) * d + 8, generator=g).to(dtype).cuda()[:, : (nh + 2 * nkv) * d].unflatten(1, (nh + 2 * nkv, d))
    q, k, v = qkv.split((nh, nkv, nkv), 1)
    positions = torch.randint(0, 5, (T,), generator=g).cumsum(0).int().cuda() + late
    rope = qt.Rope(rd, 10000.0, layout, scaling, **(how or {}))
    src, pools = qkv.double(), [kv.k.clone(), kv.v.clone()]
    out = qt.qtale_paged_rope_append(kv, 1, rope, q, k, v, offsets(new), positions, first=ints(old) if given_first else None, slots=ints(slots),
                                     q_out=q if in_place else None)
    freqs, magnitude = qt.qtale_rope_frequencies(rd, 10000.0, scaling, **(how or {}))
    want, size = turn64(src[:, : nh + nkv], positions.double()[:, None] * freqs.cuda(), magnitude, layout, rd)
    _check(out, want[:, :nh], size[:, :nh], dtype, "q")
    if not in_place:
        assert torch.equal(qkv.double(), src)                    # the inputs stay
    t = 0
    for b, (n, o) in enumerate(zip(new, old)):
        for i in range(n):
            p, at = int(kv.table[1, slots[b], (o + i) // page]), (o + i) % page
            _check(kv.k[p, :, at], want[t + i, nh:], size[t + i, nh:], dtype, ("k", b, i))
            assert torch.equal(kv.v[p, :, at].double(), src[t + i, nh + nkv:])
            pools[0][p, :, at], pools[1][p, :, at] = kv.k[p, :, at], kv.v[p, :, at]
        t += n
    for a, b in zip(pools, (kv.k, kv.v)):                        # nothing else was written (NaN stays NaN)
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d,rd", [(64, 64), (64, 16), (64, 2), (64, 50), (128, 128), (128, 96), (128, 32), (128, 20), (128, 126)])
def test_layouts_and_parts(qt, dtype, layout, d, rd):
    _case(qt, dtype, 6, 2, d, 16, [3, 0, 1, 18], [5, 2, 0, 30], layout, rd, seed=rd)
    _case(qt, dtype, 3, 3, d, 64, [2], [63], layout, rd, in_place=True, seed=rd)


@pytest.mark.parametrize("scaling,how", [("linear", dict(factor=4.0)), ("base", dict(factor=4.0)), ("bands", dict(factor=8.0, original_len=8192, low=1.0, high=4.0)),
                                         ("parts", dict(factor=16.0, original_len=4096, low=1.0, high=32.0))])
@pytest.mark.parametrize("late", [0, 131000, 2000000000])
def test_scalings_and_late_positions(qt, scaling, how, late):
    _case(qt, torch.float16, 4, 2, 128, 32, [9, 4], [0, 31], "half", 64, scaling, late, how=how, seed=late % 97)


@pytest.mark.parametrize("nh,nkv", [(1, 1), (32, 8), (40, 40), (7, 1)])
@pytest.mark.parametrize("T", [1, 2, 600])
def test_heads_and_lengths(qt, nh, nkv, T):
    _case(qt, torch.bfloat16, nh, nkv, 128, 64, [T], [100], seed=T + nh)
    _case(qt, torch.float16, nh, nkv, 64, 16, [T], [0], "interleaved", given_first=False, seed=T + nh)


def test_many_sequences(qt):
    new = [(i * 7) % 3 for i in range(200)]
    _case(qt, torch.float16, 4, 2, 64, 16, new, [(i * 5) % 40 for i in range(200)])
    _case(qt, torch.float16, 4, 2, 64, 16, [0] * 70 + [1] + [0] * 70, [3] * 141, in_place=True)


def test_entries_past_the_length_or_without_a_page_are_not_stored(qt):
    dtype, page, nh, nkv, d = torch.float16, 16, 2, 1, 64
    kv, slots = random_cache(qt, [40, 20], page, nkv, d, dtype, 5, gone={(0, 1)}, fill=0.5)
    before = [kv.k.clone(), kv.v.clone()]
    new, first = [45, 4, 3], [0, 18, 0]                          # rows 40 .. 44 and 20, 21 lie past the lengths, 16 .. 31 have no page
    qkv = torch.randn(52, nh + 2 * nkv, d, device="cuda").to(dtype)
    q, k, v = qkv.split((nh, nkv, nkv), 1)
    out = qt.qtale_paged_rope_append(kv, 0, qt.Rope(d), q, k, v, offsets(new), ints(list(range(52))), first=ints(first),
                                     slots=ints([slots[0], slots[1], 99]))   # (no such slot: its queries are turned, nothing is stored)
    angle = torch.arange(52, dtype=torch.float64, device="cuda")[:, None] * qt.qtale_rope_frequencies(d)[0].cuda()
    want, size = turn64(qkv.double()[:, : nh + nkv], angle, 1.0, "half", d)
    _check(out, want[:, :nh], size[:, :nh], dtype, "q")
    stored = [(b, f + i, t0 + i) for b, f, t0, m in ((0, 0, 0, 45), (1, 18, 45, 4)) for i in range(m)
              if f + i < (40, 20)[b] and not (b == 0 and 16 <= f + i < 32)]
    for b, at, t in stored:
        p = int(kv.table[0, slots[b], at // page])
        assert torch.equal(kv.v[p, :, at % page], v[t])
        _check(kv.k[p, :, at % page], want[t, nh:], size[t, nh:], dtype, (b, at))
        before[0][p, :, at % page], before[1][p, :, at % page] = kv.k[p, :, at % page], kv.v[p, :, at % page]
    assert torch.equal(before[0], kv.k) and torch.equal(before[1], kv.v)


def test_infinities_and_nan_stay_in_their_pairs(qt):
    kv, slots = random_cache(qt, [2], 16, 1, 64, torch.float16, 1)
    qkv = torch.ones(2, 3, 64, device="cuda", dtype=torch.float16)
    qkv[0, 0, 3], qkv[1, 0, 60] = float("nan"), float("inf")
    out = qt.qtale_paged_rope_append(kv, 0, qt.Rope(48), *qkv.split((1, 1, 1), 1), offsets([2]), ints([7, 8]), slots=ints(slots))
    bad = ~torch.isfinite(out[:, 0])
    assert bad[0].nonzero().flatten().tolist() == [3, 27] and bad[1].nonzero().flatten().tolist() == [60]


def test_no_tokens(qt):
    kv, slots = random_cache(qt, [2], 16, 1, 64, torch.float16, 1)
    e = torch.empty(0, 1, 64, device="cuda", dtype=torch.float16)
    assert qt.qtale_paged_rope_append(kv, 0, qt.Rope(64), e, e, e, offsets([0]), ints([]), slots=ints(slots)).shape == (0, 1, 64)
