"""Plain models of the paged cache for its tests: the bookkeeping as Python lists, rotary embedding and attention in float64."""
import math

import torch

U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}       # half a unit in the last place, relative
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}  # the same below the normal numbers


class Pages:
    """The bookkeeping of include/qtale.h, one page and one entry at a time."""

    def __init__(self, n_pages, page, n_layers, n_slots, max_pages):
        self.n_pages, self.page, self.L, self.S, self.M = n_pages, page, n_layers, n_slots, max_pages
        self.refs = [0] * n_pages
        self.table = [[[-1] * max_pages for _ in range(n_slots)] for _ in range(n_layers)]
        self.len = [[0] * n_slots for _ in range(n_layers)]
        self.cap = [[0] * n_slots for _ in range(n_layers)]
        self.copies = []                                         # (from, to, tokens) of the last reserve, (from, to) of the last compaction

    def take(self):
        for p, r in enumerate(self.refs):
            if r == 0:
                self.refs[p] = 1
                return p
        return -1

    def fork(self, pairs):
        for l in range(self.L):
            for s, t in pairs:
                if self.cap[l][t]:
                    continue
                n = -(-self.len[l][s] // self.page)
                for j in range(n):
                    self.table[l][t][j] = self.table[l][s][j]
                    if self.table[l][s][j] >= 0:
                        self.refs[self.table[l][s][j]] += 1
                self.len[l][t], self.cap[l][t] = self.len[l][s], n * self.page

    def reserve(self, layers, slots, new, advance):
        P, first, missing, self.copies = self.page, [], 0, []
        plans = []
        for l in layers:                                         # who copies is decided by the counts before the call
            seen = {}
            for b, s in enumerate(slots):
                n, j = self.len[l][s], self.len[l][s] // P
                page = self.table[l][s][j] if new[b] > 0 and n % P and j < self.M else -1
                copy = False
                if page >= 0:
                    copy = self.refs[page] - seen.get(page, 0) > 1
                    seen[page] = seen.get(page, 0) + 1
                plans.append((l, b, s, page if copy else -1))
        for l, b, s, shared in plans:
            n = self.len[l][s]
            first.append(n)
            room = True
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

    def drop(self, l, s, j):
        p = self.table[l][s][j]
        if p >= 0:
            self.refs[p] -= 1
            self.table[l][s][j] = -1

    def release(self, slots):
        for l in range(self.L):
            for s in slots:
                for j in range(self.M):
                    self.drop(l, s, j)
                self.len[l][s] = self.cap[l][s] = 0

    def trim(self, slots, window, sinks):
        for l in range(self.L):
            for s in slots:
                for j in range(self.M):
                    if (j + 1) * self.page <= self.len[l][s] + 1 - window and j * self.page >= sinks:
                        self.drop(l, s, j)

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        src = [p for p in range(live, self.n_pages) if self.refs[p] > 0]
        dst = [p for p in range(live) if self.refs[p] == 0]
        to = dict(zip(src, dst))
        self.copies = list(to.items())
        for s, t in to.items():
            self.refs[t], self.refs[s] = self.refs[s], 0
        self.table = [[[to.get(p, p) for p in row] for row in layer] for layer in self.table]
        return live

    def bits(self):
        words = [0] * ((self.n_pages + 31) // 32)
        for p, r in enumerate(self.refs):
            if r == 0:
                words[p // 32] |= 1 << (p % 32)
        return [w - (1 << 32) if w >> 31 else w for w in words]

    def check(self, kv, what=""):
        assert kv.table.tolist() == self.table, what
        assert kv.kv_len.tolist() == self.len and kv.kv_cap.tolist() == self.cap, what
        assert kv.page_refs.tolist() == self.refs and kv.free_bits.tolist() == self.bits(), what


def turn64(x, angle, magnitude, layout, rd):
    """Rotates [T, heads, d] (float64) by angle [T, rd / 2]; also the sum of the products' magnitudes, for the error bound."""
    c, s = (magnitude * angle.cos())[:, None], (magnitude * angle.sin())[:, None]
    a, b = (x[..., : rd // 2], x[..., rd // 2: rd]) if layout == "half" else (x[..., 0:rd:2], x[..., 1:rd:2])
    out, size = x.clone(), torch.zeros_like(x)
    first, second = a * c - b * s, b * c + a * s
    big = (a.abs() + b.abs()) * abs(magnitude)
    if layout == "half":
        out[..., : rd // 2], out[..., rd // 2: rd] = first, second
        size[..., : rd // 2], size[..., rd // 2: rd] = big, big
    else:
        out[..., 0:rd:2], out[..., 1:rd:2] = first, second
        size[..., 0:rd:2], size[..., 1:rd:2] = big, big
    return out, size


def attend64(kv, layer, q, new, first, slots, window, sinks, scale, clean=False):
    """(outputs, sum of probability times |value|) in float64, row by row of sequences; keys and values that no row of the sequence sees are never
    touched.  clean: nor those that a single row does not see (row by row, for values that are not finite)."""
    T, nh, d = q.shape
    nkv, P = kv.n_kv_heads, kv.page_size
    out, size = (torch.zeros(T, nh, d, dtype=torch.float64, device=q.device) for _ in range(2))
    t = 0
    for b, n in enumerate(new):
        length = int(kv.kv_len[layer, slots[b]])
        row = kv.table[layer, slots[b]].tolist()
        keys = [j for j in range(length) if row[j // P] >= 0]
        if n and keys:
            where = torch.tensor(keys, device=q.device)
            page = torch.tensor([row[j // P] for j in keys], device=q.device)
            place = first[b] + torch.arange(n, device=q.device)
            seen = where[None] <= place[:, None]
            if window:
                seen &= (where[None] > place[:, None] - window) | (where[None] < sinks)
            any_row = seen.any(0)
            where, page, seen = where[any_row], page[any_row], seen[:, any_row]
            if where.numel():
                for h in range(nkv):
                    k, v = (x[page, h, where % P].double() for x in (kv.k, kv.v))
                    for i in range(h * (nh // nkv), (h + 1) * (nh // nkv)):
                        z = (q[t: t + n, i].double() @ k.t().contiguous()) * scale
                        z = z.masked_fill(~seen, -math.inf)
                        p = torch.exp(z - z.amax(1, keepdim=True).clamp(min=-1e300))
                        p = p / p.sum(1, keepdim=True).clamp(min=1e-300)
                        if clean:
                            for r in range(n):
                                out[t + r, i], size[t + r, i] = p[r][seen[r]] @ v[seen[r]], p[r][seen[r]] @ v[seen[r]].abs()
                        else:
                            out[t: t + n, i], size[t: t + n, i] = p @ v, p @ v.abs()
        t += n
    return out, size


# Bound on |attention output - 64-bit reference|: the output's own rounding; probabilities as operands, rounded to 16 bits (chunks) or to two
# 16-bit terms (few queries): u or 2^-15 of sum p |v|; scores, exponentials and sums in 32 bits: a score is a sum of up to 128 products whose
# magnitudes add up to less than 200 with the inputs here, so it is off by less than 200 * 2^-24 * 3 = 4e-5, and so is p in relation.
def attention_bound(want, size, dtype, split_terms):
    u = U[dtype]
    return u * want.abs() + ((2.0 ** -15 if split_terms else u) + 4e-5 + 2e-5) * size + TINY[dtype]


def random_cache(qt, lens, page, nkv, d, dtype, seed, spare=3, n_layers=1, layer=0, gone=(), fill=float("nan"), extra_slots=2, max_extra=1):
    """A cache whose slots of `layer` hold `lens` random tokens on shuffled pages, and the slots; all other memory is `fill`.
    gone: (sequence, page of it) whose table entry is -1."""
    g = torch.Generator().manual_seed(seed)
    held = [-(-n // page) for n in lens]
    n_pages, n_slots = sum(held) + spare, len(lens) + extra_slots
    kv = qt.PagedKV.empty(n_pages, page, nkv, d, n_slots, max(held + [1]) + max_extra, n_layers, dtype)
    slots = torch.randperm(n_slots, generator=g)[: len(lens)].tolist()
    order = torch.randperm(n_pages, generator=g).tolist()
    table, length, cap, refs = kv.table.cpu(), kv.kv_len.cpu(), kv.kv_cap.cpu(), kv.page_refs.cpu()
    k, v = (torch.full(kv.k.shape, fill, dtype=dtype) for _ in range(2))
    for b, n in enumerate(lens):
        length[layer, slots[b]], cap[layer, slots[b]] = n, held[b] * page
        for j in range(held[b]):
            p = order.pop()
            m = min(page, n - j * page)
            if (b, j) in gone:
                continue
            table[layer, slots[b], j], refs[p] = p, 1
            k[p, :, :m], v[p, :, :m] = (torch.randn(nkv, m, d, generator=g).to(dtype) for _ in range(2))
    free = [int(r == 0) for r in refs.tolist()] + [0] * (-n_pages % 32)
    words = [sum(bit << i for i, bit in enumerate(free[w: w + 32])) for w in range(0, len(free), 32)]
    kv.free_bits.copy_(torch.tensor([w - (1 << 32) if w >> 31 else w for w in words], dtype=torch.int32))
    for dst, src in ((kv.table, table), (kv.kv_len, length), (kv.kv_cap, cap), (kv.page_refs, refs), (kv.k, k), (kv.v, v)):
        dst.copy_(src)
    return kv, slots


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def offsets(new):
    return ints([0] + torch.tensor(new, dtype=torch.int64).cumsum(0).tolist())
