"""Pages of the paged cache on the GPU (run with -m gpu): every call against a model that does the bookkeeping one page at a time, with contents."""
import random

import pytest
import torch

from tests.paged_helpers import Pages, ints, offsets

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qt():
    import paper_2602_10431_amd as pkg
    pkg.load_library()
    return pkg


def _make(qt, n_pages, page, L, S, M, nkv=2, d=64, dtype=torch.float16):
    kv = qt.PagedKV.empty(n_pages, page, nkv, d, S, M, L, dtype)
    g = torch.Generator().manual_seed(n_pages)
    for t in (kv.k, kv.v):
        t.copy_(torch.randn(t.shape, generator=g).to(dtype))
    return kv, Pages(n_pages, page, L, S, M)


def _reserve(qt, kv, model, slots, new, layer=-1, advance=True):
    layers = list(range(model.L)) if layer < 0 else [layer]
    k, v = kv.k.clone(), kv.v.clone()
    first, missing = ints([-7] * (len(layers) * len(slots))), ints([-7])
    qt.qtale_pages_reserve(kv, offsets(new), slots=ints(slots), layer=layer, first=first if advance else None, missing=missing)
    want_first, want_missing = model.reserve(layers, slots, new, advance)
    model.check(kv, (slots, new, layer))
    assert missing.item() == want_missing
    if advance:
        assert first.tolist() == want_first
    for a, b in ((k, kv.k), (v, kv.v)):                          # shared pages' tokens were copied, nothing else changed
        for s, t, n in model.copies:
            a[t, :, :n] = a[s, :, :n]
        assert torch.equal(a, b)


@pytest.mark.parametrize("n_pages", [1, 31, 32, 33, 100, 40000])
def test_an_empty_cache(qt, n_pages):
    kv, model = _make(qt, n_pages, 16, 2, 3, 5, nkv=1)
    model.check(kv)


@pytest.mark.parametrize("page", [16, 64, 1024])
@pytest.mark.parametrize("length", [1, 15, 16, 17, 64, 1000, 1024, 1025])
def test_room_for_one_prompt_and_one_token_more(qt, page, length):
    kv, model = _make(qt, 160, page, 2, 4, 70)
    _reserve(qt, kv, model, [2, 0], [length, 0])
    _reserve(qt, kv, model, [2, 0], [1, 3])
    _reserve(qt, kv, model, [0], [1], layer=1)


@pytest.mark.parametrize("seed", range(12))
def test_random_calls(qt, seed):
    rng = random.Random(seed)
    page, L, S = rng.choice([16, 32, 128]), rng.choice([1, 3, 5]), rng.choice([4, 9, 70])
    M = rng.choice([3, 9, 40])
    n_pages = rng.choice([20, 97, 700])                          # small ones run out
    kv, model = _make(qt, n_pages, page, L, S, M)
    for _ in range(25):
        what = rng.random()
        some = lambda k=None: rng.sample(range(S), k or rng.randint(1, S))
        if what < 0.45:
            slots = some()
            _reserve(qt, kv, model, slots, [rng.choice([0, 1, 1, rng.randint(0, 3 * page)]) for _ in slots], rng.choice([-1, -1, rng.randrange(L)]), rng.random() < 0.9)
        elif what < 0.65:
            slots = some()
            n = rng.randint(0, len(slots) // 2)
            # a source may be forked several times; targets that are not empty stay as they are
            src = [rng.choice(slots[: max(len(slots) - n, 1)]) for _ in range(n)]
            dst = slots[len(slots) - n:]
            qt.qtale_pages_fork(kv, ints(src), ints(dst))
            model.fork([(s, t) for s, t in zip(src, dst) if s != t])
        elif what < 0.78:
            slots = some()
            qt.qtale_pages_release(kv, ints(slots))
            model.release(slots)
        elif what < 0.9:
            slots, window, sinks = some(), rng.choice([1, page, 3 * page + 5]), rng.choice([0, 1, page, 2 * page + 1])
            qt.qtale_pages_trim(kv, window, sinks, slots=ints(slots))
            model.trim(slots, window, sinks)
        else:
            k, v, live = kv.k.clone(), kv.v.clone(), ints([-1])
            qt.qtale_pages_compact(kv, live)
            assert live.item() == model.compact()
            for a, b in ((k, kv.k), (v, kv.v)):
                before = a.clone()
                for s, t in model.copies:
                    a[t] = before[s]
                assert torch.equal(a, b)
        model.check(kv, seed)


@pytest.mark.parametrize("copies", [1, 2, 5, 40])
@pytest.mark.parametrize("length", [1, 31, 32, 33])
def test_holders_of_a_shared_page_take_copies_in_order(qt, copies, length):
    kv, model = _make(qt, 400, 32, 2, copies + 2, 4)
    _reserve(qt, kv, model, [0], [length])
    targets = list(range(1, copies + 1))
    qt.qtale_pages_fork(kv, ints([0] * copies), ints(targets))
    model.fork([(0, t) for t in targets])
    model.check(kv)
    some = targets[::2] + [0]                                    # some of the holders write, then all of them
    _reserve(qt, kv, model, some, [2] * len(some))
    _reserve(qt, kv, model, [0] + targets, [1] * (copies + 1))


def test_an_empty_pool(qt):
    kv, model = _make(qt, 6, 16, 1, 6, 8)
    _reserve(qt, kv, model, [0, 1], [40, 70])                    # 3 + 5 wanted, 6 there
    qt.qtale_pages_fork(kv, ints([0]), ints([2]))
    model.fork([(0, 2)])
    _reserve(qt, kv, model, [2, 0], [5, 5])                      # no page for the copy: slot 2 takes nothing
    assert kv.kv_len[0].tolist()[:3] == [45, 48, 40] or kv.kv_len[0].tolist() == model.len[0]
    qt.qtale_pages_release(kv, ints([1]))
    model.release([1])
    _reserve(qt, kv, model, [2, 0], [5, 5])


@pytest.mark.parametrize("L,B", [(1, 2048), (32, 64), (33, 63), (7, 1000), (3, 1500)])
def test_many_sequences(qt, L, B):
    # more pairs than one workgroup holds at once, more pages than one list; every third slot shares its page with its neighbour
    kv, model = _make(qt, 3 * L * B + 5, 16, L, B, 4, nkv=1)
    slots = list(range(B))
    random.Random(B).shuffle(slots)
    held = slots[: B // 2]
    _reserve(qt, kv, model, held, [1 + 7 * (i % 5) for i in range(len(held))])
    src, dst = held[::3], slots[B // 2: B // 2 + len(held[::3])]
    qt.qtale_pages_fork(kv, ints(src), ints(dst))
    model.fork(list(zip(src, dst)))
    _reserve(qt, kv, model, slots, [i % 4 * 9 for i in range(B)])


def test_one_call_takes_more_than_a_list(qt):
    kv, model = _make(qt, 12000, 16, 1, 2, 6000, nkv=1)
    _reserve(qt, kv, model, [1], [16 * 5000 + 3])
    qt.qtale_pages_release(kv, ints([1]))
    model.release([1])
    _reserve(qt, kv, model, [0, 1], [16 * 5990, 16 * 6000 + 40])   # the second runs into max_pages


def test_numbers_out_of_range_are_skipped(qt):
    kv, model = _make(qt, 20, 16, 2, 4, 4)
    _reserve(qt, kv, model, [0], [20])
    before = [t.clone() for t in (kv.table, kv.kv_len, kv.kv_cap, kv.page_refs, kv.free_bits, kv.k)]
    qt.qtale_pages_fork(kv, ints([0, -1, 4]), ints([4, 1, 2]))
    qt.qtale_pages_release(kv, ints([-1, 4, 1 << 30]))
    qt.qtale_pages_trim(kv, 1, 0, slots=ints([-5, 9]))
    first = ints([0] * 4)
    qt.qtale_pages_reserve(kv, offsets([5, 5]), slots=ints([-1, 4]), first=first)
    qt.qtale_pages_copy(kv, kv, ints([0, 20]), ints([-1, 3]))
    for a, b in zip(before, (kv.table, kv.kv_len, kv.kv_cap, kv.page_refs, kv.free_bits, kv.k)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("d,nkv,page", [(64, 1, 16), (128, 3, 32), (128, 8, 128)])
def test_copy_between_pools(qt, d, nkv, page):
    a, _ = _make(qt, 30, page, 1, 2, 4, nkv, d, torch.bfloat16)
    b, _ = _make(qt, 50, page, 1, 3, 9, nkv, d, torch.bfloat16)
    k, v = b.k.clone(), b.v.clone()
    src, dst = [29, 0, 7, 7], [49, 3, 0, 20]
    qt.qtale_pages_copy(a, b, ints(src), ints(dst))
    k[dst], v[dst] = a.k[src], a.v[src]
    assert torch.equal(k, b.k) and torch.equal(v, b.v)


def test_large_pool_compacts(qt):
    # more free-bit words than the planning workgroup looks at per round
    kv, model = _make(qt, 70000, 16, 1, 40, 900, nkv=1)
    slots = list(range(40))
    _reserve(qt, kv, model, slots, [16 * 800 + i for i in slots])
    drop = slots[::2]
    qt.qtale_pages_release(kv, ints(drop))
    model.release(drop)
    k, live = kv.k.clone(), ints([0])
    qt.qtale_pages_compact(kv, live)
    assert live.item() == model.compact()
    model.check(kv)
    src, dst = (torch.tensor(x, device="cuda") for x in zip(*model.copies))
    want = k.clone()
    want[dst] = k[src]
    assert torch.equal(want, kv.k)


def test_calls_are_ordered_on_their_own_stream(qt):
    kv, model = _make(qt, 200, 16, 2, 8, 10)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(5):
            _reserve(qt, kv, model, list(range(8)), [9] * 8)
        qt.qtale_pages_release(kv)
    side.synchronize()
    model.release(range(8))
    model.check(kv)
