"""Pools that run dry: what a slot holds is followed entry by entry through forks, copies that were not granted and calls in other orders.  A model on
the CPU; the page calls with the append, and the layers (whose copies run beside the append), on the GPU (run with -m gpu)."""
import random

import pytest
import torch

import synth_inputs as si
from tests.paged_helpers import Pages, ints, offsets


class LongestKeeps(Pages):
    """Of a page's holders, all in the call, the one with the most tokens (the last of several) keeps the page; `Pages` takes the last in any case, which
    is the same as long as every holder has as many tokens."""

    def reserve(self, layers, slots, new, advance):
        P, first, missing, self.copies = self.page, [], 0, []
        plans = []
        for l in layers:
            pages = [self.table[l][s][self.len[l][s] // P] if new[b] > 0 and self.len[l][s] % P and self.len[l][s] // P < self.M else -1
                     for b, s in enumerate(slots)]
            for b, s in enumerate(slots):
                holders = [(self.len[l][t], e) for e, t in enumerate(slots) if pages[e] == pages[b]]
                keeps = pages[b] < 0 or (len(holders) >= self.refs[pages[b]] and max(holders)[1] == b)
                plans.append((l, b, s, -1 if keeps else pages[b]))
        for l, b, s, shared in plans:
            n, room = self.len[l][s], True
            first.append(n)
            if shared >= 0:
                p = self.take()
                if p < 0:
                    missing, room = missing + 1, False
                else:
                    self.copies.append((shared, p, n % P))
                    self.refs[shared] -= 1
                    self.table[l][s][n // P] = p
            want = min(-(-(n + new[b]) // P), self.M) if new[b] > 0 else 0
            for j in range(self.cap[l][s] // P, want):
                p = self.take()
                if p < 0:
                    missing += 1
                    continue
                self.table[l][s][j] = p
                self.cap[l][s] = (j + 1) * P
            if advance and room:
                self.len[l][s] = max(n, min(n + new[b], self.cap[l][s]))
        return first, missing


def _calls(seed, n_slots, steps, most=(0, 1, 1, 2, 5)):
    """Random calls, the same for the model and the library: ("new", slots, tokens), ("fork", from, to), ("release", slot), ("compact",)."""
    rng = random.Random(seed)
    for _ in range(steps):
        what = rng.random()
        if what < 0.6:
            slots = rng.sample(range(n_slots), rng.randint(1, n_slots))
            yield "new", slots, [rng.choice(most) for _ in slots]
        elif what < 0.85:
            yield ("fork", *rng.sample(range(n_slots), 2))
        elif what < 0.93:
            yield "release", rng.randrange(n_slots)
        else:
            yield ("compact",)


def test_the_rule_keeps_what_a_slot_has_written():
    # the model alone, many runs: entries of a slot never change, and no place that a call copies from is stored into by the same call
    for seed in range(1500):
        n_slots, m, memory, stamp = 3 + seed % 5, LongestKeeps((2, 4, 7, 12)[seed % 4], 4, 1, 3 + seed % 5, 6), {}, 0
        want = [[] for _ in range(n_slots)]
        for call, *args in _calls(seed, n_slots, 40):
            if call == "new":
                slots, new = args
                first, _ = m.reserve([0], slots, new, True)
                read = {(s, i) for s, _, n in m.copies for i in range(n)}
                for s, t, n in m.copies:
                    memory.update({(t, i): memory[s, i] for i in range(n)})
                for b, s in enumerate(slots):
                    for at in range(first[b], m.len[0][s]):
                        place = (m.table[0][s][at // 4], at % 4)
                        assert place not in read
                        stamp += 1
                        memory[place] = stamp
                        want[s].append(stamp)
            elif call == "fork":
                if m.cap[0][args[1]] == 0:
                    want[args[1]] = list(want[args[0]])
                m.fork([tuple(args)])
            elif call == "release":
                m.release(args)
                want[args[0]] = []
            else:
                m.compact()
                memory.update({(t, i): memory.get((s, i)) for s, t in m.copies for i in range(4)})
            assert [[memory[m.table[0][s][j // 4], j % 4] for j in range(m.len[0][s])] for s in range(n_slots)] == want, seed


@pytest.fixture(scope="module")
def qt():
    import paper_2602_10431_amd as pkg
    pkg.load_library()
    return pkg


class Follow:
    """A cache and what each of its slots has to hold, token by token."""

    def __init__(self, qt, n_pages, page, n_slots, max_pages, nkv, d):
        self.qt, self.page, self.nkv, self.d = qt, page, nkv, d
        self.kv, self.model = qt.PagedKV.empty(n_pages, page, nkv, d, n_slots, max_pages), LongestKeeps(n_pages, page, 1, n_slots, max_pages)
        self.kv.k.fill_(float("nan"))
        self.kv.v.fill_(float("nan"))
        self.want = [[] for _ in range(n_slots)]                 # (key, value), [nkv, d] each
        self.rope = qt.Rope(d)

    def store(self, slots, new, k, v):
        """Room and append of a call; keys at position 0, which no rotation changes."""
        T, first, missing = sum(new), ints([-7] * len(slots)), ints([-7])
        self.qt.qtale_pages_reserve(self.kv, offsets(new), slots=ints(slots), first=first, missing=missing)
        if T:
            self.qt.qtale_paged_rope_append(self.kv, 0, self.rope, torch.zeros_like(k), k, v, offsets(new), ints([0] * T), first=first, slots=ints(slots))
        self.took(slots, new, k, v)
        return missing.item()

    def took(self, slots, new, k, v, missing=None):
        first, wanted = self.model.reserve([0], slots, new, True)
        assert missing is None or missing == wanted
        at = 0
        for b, s in enumerate(slots):
            for i in range(self.model.len[0][s] - first[b]):
                self.want[s].append((k[at + i].cpu(), v[at + i].cpu()))
            at += new[b]

    def other(self, call, *args):
        if call == "fork":
            src, dst = args
            self.qt.qtale_pages_fork(self.kv, ints([src]), ints([dst]))
            if self.model.cap[0][dst] == 0:
                self.want[dst] = list(self.want[src])
            self.model.fork([(src, dst)])
        elif call == "release":
            self.qt.qtale_pages_release(self.kv, ints(list(args)))
            self.model.release(args)
            self.want[args[0]] = []
        else:
            self.qt.qtale_pages_compact(self.kv)
            self.model.compact()

    def check(self, what=None):
        self.model.check(self.kv, what)
        k, v, table = self.kv.k.cpu(), self.kv.v.cpu(), self.kv.table[0].tolist()
        for s, entries in enumerate(self.want):
            assert self.model.len[0][s] == len(entries)
            for j, (a, b) in enumerate(entries):
                p, i = table[s][j // self.page], j % self.page
                assert torch.equal(k[p, :, i], a) and torch.equal(v[p, :, i], b), (what, s, j)

    def rows(self, n, seed):
        g = torch.Generator().manual_seed(seed)
        return (torch.randn(n, self.nkv, self.d, generator=g).half().cuda() for _ in range(2))


@pytest.mark.gpu
def test_a_copy_that_was_not_granted(qt):
    f = Follow(qt, 1, 16, 4, 3, 2, 64)
    f.store([0], [5], *f.rows(5, 0))
    f.other("fork", 0, 1)
    lens = lambda: f.kv.kv_len[0].tolist()[:3]
    # no page for a copy: the last holder goes on in the page, the other one stays where it is, whatever the order of the next calls
    for step, (slots, want) in enumerate([([0, 1], [5, 6, 0]), ([1, 0], [5, 7, 0]), ([0, 1], [5, 8, 0])]):
        assert f.store(slots, [1, 1], *f.rows(2, 1 + step)) == 1
        assert lens() == want
        f.check(step)
    f.other("fork", 0, 2)                                        # a third holder, of five tokens
    for step, (slots, want) in enumerate([([1, 0, 2], [5, 9, 5]), ([2, 1, 0], [5, 10, 5])]):
        assert f.store(slots, [1, 1, 1], *f.rows(3, 10 + step)) == 2
        assert lens() == want
        f.check(step)
    assert f.store([0, 2], [1, 1], *f.rows(2, 20)) == 2 and lens() == [5, 10, 5]   # not all holders: nobody keeps the page
    f.check("some")
    f.other("release", 1)
    assert f.store([2, 0], [1, 1], *f.rows(2, 21)) == 1 and lens() == [6, 0, 5]
    f.check("released")


@pytest.mark.gpu
@pytest.mark.parametrize("order", [[0, 1], [1, 0]])
def test_a_copy_that_is_granted_later(qt, order):
    f = Follow(qt, 2, 16, 4, 3, 2, 64)
    f.store([0, 3], [5, 1], *f.rows(6, 0))
    f.other("fork", 0, 1)
    assert f.store([0, 1], [1, 1], *f.rows(2, 1)) == 1 and f.kv.kv_len[0].tolist() == [5, 6, 0, 1]
    f.other("release", 3)
    assert f.store(order, [3, 3], *f.rows(6, 2)) == 0 and f.kv.kv_len[0].tolist() == [8, 9, 0, 0]
    f.check()


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(16))
def test_random_calls_on_a_dry_pool(qt, seed):
    n_slots, page = 3 + seed % 6, (16, 32)[seed % 2]
    f = Follow(qt, (2, 4, 7, 12)[seed % 4], page, n_slots, 6, 1 + seed % 2, 64)
    for step, (call, *args) in enumerate(_calls(seed, n_slots, 40, (0, 1, 1, 3, page + 5))):
        if call == "new":
            f.store(*args, *f.rows(sum(args[1]), 100 * seed + step))
        else:
            f.other(call, *args)
        f.check((seed, step, call))


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(6))
def test_layers_on_a_dry_pool(qt, seed):
    # one layer that every token executes: what its tokens append is what the same call appends to an empty cache, positions as given
    shape = si.LayerShape(256, 4, 2, 64, 512, 4, 32, "fp16")
    stack = qt.Stack(qt.cfg_from_shape(shape), [qt.quantize_layer(si.layer_tensors(shape, 0, 3, unit_gains=False, std=1.28 / shape.hidden ** 0.5), 4, 32)])
    ctx, rope = qt.Context(), qt.Rope(64, shape.rope_base)
    qt.qtale_set_exec_ratio(ctx, 1.0)
    n_slots, page = 4 + seed % 4, 16
    f = Follow(qt, (3, 5, 8)[seed % 3], page, n_slots, 6, 2, 64)
    for step, (call, *args) in enumerate(_calls(seed + 50, n_slots, 40, (0, 1, 1, 2, page + 3))):
        if call == "new":
            slots, new = args
            T = sum(new)
            if T == 0:
                continue
            x = si.hidden_states(shape, T, 100 * seed + step).cuda()
            pos = torch.randint(0, 500, (T,), generator=torch.Generator().manual_seed(step)).int().cuda()
            empty, missing = qt.PagedKV.empty(64, 64, 2, 64, len(slots), 2), ints([-7])
            qt.qtale_paged_stack_forward(ctx, stack, x.clone(), offsets(new), pos, empty, rope)
            qt.qtale_paged_stack_forward(ctx, stack, x, offsets(new), pos, f.kv, rope, slots=ints(slots), missing=missing)
            k, v = ([pool[int(empty.table[0, b, i // 64]), :, i % 64] for b, n in enumerate(new) for i in range(n)] for pool in (empty.k, empty.v))
            f.took(slots, new, k, v, missing.item())
        else:
            f.other(call, *args)
        f.check((seed, step, call))
