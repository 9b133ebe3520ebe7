"""Plain models of pages in 4 bits for their tests: the quantizer in float64, packing by the layout of include/qtale.h code by code, random caches with the
values that they stand for beside them."""
import types

import torch

from tests.paged_helpers import TINY, U


def quantize64(x):
    """Rows of 16-bit values (any device) -> codes (int64), scale (of x's type), zero (int64), as the header defines them."""
    w = x.double()
    bad = ~torch.isfinite(w).all(-1, keepdim=True)
    w = torch.where(bad, torch.zeros_like(w), w)
    lo, hi = w.amin(-1, keepdim=True).clamp(max=0), w.amax(-1, keepdim=True).clamp(min=0)
    scale = ((hi - lo) / 15).to(x.dtype)
    scale = torch.where(scale == 0, torch.ones_like(scale), scale)
    s = scale.double()
    zero = torch.round(-lo / s).clamp(max=15)
    codes = (torch.round(w / s) + zero).clamp(0, 15)
    codes, zero = torch.where(bad, torch.zeros_like(codes), codes), torch.where(bad, torch.zeros_like(zero), zero)
    scale = torch.where(bad, torch.full_like(scale, float("nan")), scale)
    return codes.long(), scale[..., 0], zero[..., 0].long()


def values64(codes, scale, zero):
    return (codes - zero[..., None]).double() * scale.double()[..., None]


def _places(d, page, keys):
    """(word of the block, shift) of code [token, column]."""
    t, c = torch.arange(page)[:, None], torch.arange(d)[None]
    if keys:
        return t * (d // 8) + c // 8, 4 * ((c % 8) // 2) + 16 * (c % 2)
    return (t // 4) * (d // 2) + 2 * (c // 4) + (t % 4) // 2, 4 * (c % 4) + 16 * (t % 2)


def pack(codes, scale, zero, keys):
    """codes [n_pages, nkv, page, d], scale (16-bit floats) and zero [n_pages, nkv, page] (CPU) -> bytes [n_pages, nkv, page * (d / 2 + 4)]."""
    n, h, page, d = codes.shape
    word, shift = (x.expand(page, d).reshape(-1) for x in _places(d, page, keys))
    words = torch.zeros(n, h, page * d // 8, dtype=torch.int64).index_add_(2, word, codes.reshape(n, h, -1) << shift)
    params = (scale.contiguous().view(torch.int16).long() & 0xffff) | zero << 16
    words = torch.cat([words, params], 2)
    return (words[..., None] >> torch.tensor([0, 8, 16, 24]) & 255).to(torch.uint8).reshape(n, h, -1)


def unpack(block, d, keys, dtype):
    """The inverse: codes, scale, zero."""
    block = block.cpu()
    n, h, size = block.shape
    page = size // (d // 2 + 4)
    words = (block.view(n, h, -1, 4).long() << torch.tensor([0, 8, 16, 24])).sum(3)
    word, shift = (x.expand(page, d) for x in _places(d, page, keys))
    params = words[:, :, page * d // 8:]
    scale = (((params & 0xffff) + 0x8000) % 0x10000 - 0x8000).to(torch.int16).view(dtype)
    return words[:, :, : page * d // 8][:, :, word] >> shift & 15, scale, params >> 16


def shadow(kv, k, v):
    """What attend64 reads: dense values beside the cache's own bookkeeping."""
    return types.SimpleNamespace(k=k.cuda(), v=v.cuda(), table=kv.table, kv_len=kv.kv_len, n_kv_heads=kv.n_kv_heads, page_size=kv.page_size)


def random_cache4(qt, lens, page, nkv, d, dtype, seed, spare=3, n_layers=1, layer=0, gone=(), extra_slots=2, max_extra=1, std=1.0):
    """(cache, slots, shadow): slots of `layer` hold `lens` random tokens on shuffled pages; every other place has a NaN for its scale and
    zero point, and codes of 15."""
    g = torch.Generator().manual_seed(seed)
    held = [-(-n // page) for n in lens]
    n_pages, n_slots = sum(held) + spare, len(lens) + extra_slots
    kv = qt.PagedKV.empty(n_pages, page, nkv, d, n_slots, max(held + [1]) + max_extra, n_layers, dtype, bits=4)
    slots = torch.randperm(n_slots, generator=g)[: len(lens)].tolist()
    order = torch.randperm(n_pages, generator=g).tolist()
    table, length, cap, refs = kv.table.cpu(), kv.kv_len.cpu(), kv.kv_cap.cpu(), kv.page_refs.cpu()
    used = torch.zeros(n_pages, page, dtype=torch.bool)
    for b, n in enumerate(lens):
        length[layer, slots[b]], cap[layer, slots[b]] = n, held[b] * page
        for j in range(held[b]):
            p = order.pop()
            if (b, j) in gone:
                continue
            table[layer, slots[b], j], refs[p] = p, 1
            used[p, : min(page, n - j * page)] = True
    dense = []
    for keys in (True, False):
        x = (std * torch.randn(n_pages, nkv, page, d, generator=g)).to(dtype)
        codes, scale, zero = quantize64(x)
        hole = ~used[:, None].expand(n_pages, nkv, page)
        codes = torch.where(hole[..., None], torch.full_like(codes, 15), codes)
        scale = torch.where(hole, torch.full_like(scale, float("nan")), scale)
        (kv.k if keys else kv.v).copy_(pack(codes, scale, torch.where(hole, torch.full_like(zero, 0x7e01), zero), keys))
        dense.append(values64(codes, scale, zero))
    free = [int(r == 0) for r in refs.tolist()] + [0] * (-n_pages % 32)
    words = [sum(bit << i for i, bit in enumerate(free[w: w + 32])) for w in range(0, len(free), 32)]
    kv.free_bits.copy_(torch.tensor([w - (1 << 32) if w >> 31 else w for w in words], dtype=torch.int32))
    for dst, src in ((kv.table, table), (kv.kv_len, length), (kv.kv_cap, cap), (kv.page_refs, refs)):
        dst.copy_(src)
    return kv, slots, shadow(kv, *dense)


# Bound on |attention output - 64-bit reference|: the output's own rounding; probabilities (with the value's scale) as operands of 16 bits, 2^-11 of
# sum p |code - zero| s at most twice (the codes and the zero points may be summed apart: up to 15 + 15 where the difference is 1, but both with the
# same rounded probability, so that the rounding itself counts once); scores: d products of a query and a code up to 15, and the zero point times
# the queries' sum, each off by 2^-24 of the magnitudes' sum per addition, times the scales; exponentials and sums in 32 bits 2e-5; the sums of up
# to n products with codes and zero points apart 2^-24 * 30 / 1 per step of the scale, `step` of the largest one.
def attention_bound4(want, size, q, dtype, scale, kv_scale, steps=64):
    d = q.shape[2]
    score = float(q.double().abs().sum(2).max()) * 30 * kv_scale * scale * (d + 4) * 2.0 ** -24
    return U[dtype] * want.abs() + (2.0 ** -11 + 2 * score + 2e-5) * size + 30 * kv_scale * steps * 2.0 ** -24 + TINY[dtype]
