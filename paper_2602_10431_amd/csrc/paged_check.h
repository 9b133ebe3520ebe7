// Checks of the paged cache's arguments and their device views, for the entry points that take one.
#pragma once
#include <algorithm>
#include <cmath>

#include "../../include/qtale.h"
#include "paged.h"

namespace qtale {

// buffers: also the pointers (size queries do not need them)
inline int check_paged(const qtale_paged_kv* kv, bool buffers) {
    if (!kv) return QTALE_ERR_INVALID_ARG;
    if (kv->n_pages <= 0 || kv->n_kv_heads <= 0 || kv->n_layers <= 0 || kv->n_slots <= 0 || kv->max_pages <= 0 || kv->page_size <= 0 || kv->head_dim <= 0)
        return QTALE_ERR_INVALID_ARG;
    if (kv->head_dim != 64 && kv->head_dim != 128) return QTALE_ERR_UNSUPPORTED;
    if (kv->page_size < 16 || kv->page_size > 1024 || (kv->page_size & (kv->page_size - 1)) != 0) return QTALE_ERR_UNSUPPORTED;
    if ((kv->dtype & ~QTALE_KV_INT4) != QTALE_ACT_FP16 && (kv->dtype & ~QTALE_KV_INT4) != QTALE_ACT_BF16) return QTALE_ERR_UNSUPPORTED;
    if (kv->n_layers > 65535) return QTALE_ERR_UNSUPPORTED;
    // places in a slot and slots of all layers are counted in 32 bits
    if (static_cast<int64_t>(kv->max_pages) * kv->page_size > (int64_t{1} << 30)) return QTALE_ERR_UNSUPPORTED;
    if (static_cast<int64_t>(kv->n_layers) * kv->n_slots > (int64_t{1} << 30)) return QTALE_ERR_UNSUPPORTED;
    if (kv->n_pages > (1 << 30)) return QTALE_ERR_UNSUPPORTED;
    if (!buffers) return QTALE_OK;
    if (!kv->k_pages || !kv->v_pages || !kv->page_refs || !kv->free_bits || !kv->table || !kv->kv_len || !kv->kv_cap) return QTALE_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(kv->k_pages) | reinterpret_cast<uintptr_t>(kv->v_pages)) % 16 != 0) return QTALE_ERR_INVALID_ARG;
    return QTALE_OK;
}

// The cache on the device; layer >= 0: table, lengths and room begin at that layer.
inline PagedDev paged_device(const qtale_paged_kv* kv, int layer) {
    PagedDev p{};
    const size_t skip = layer > 0 ? static_cast<size_t>(layer) * kv->n_slots : 0;
    p.k = static_cast<uint16_t*>(kv->k_pages); p.v = static_cast<uint16_t*>(kv->v_pages);
    p.refs = kv->page_refs; p.bits = kv->free_bits;
    p.table = kv->table ? kv->table + skip * kv->max_pages : nullptr;
    p.len = kv->kv_len ? kv->kv_len + skip : nullptr;
    p.cap = kv->kv_cap ? kv->kv_cap + skip : nullptr;
    p.n_pages = kv->n_pages; p.nkv = kv->n_kv_heads; p.d = kv->head_dim; p.n_layers = kv->n_layers; p.n_slots = kv->n_slots;
    p.max_pages = kv->max_pages; p.bf16 = (kv->dtype & ~QTALE_KV_INT4) == QTALE_ACT_BF16; p.q4 = (kv->dtype & QTALE_KV_INT4) != 0;
    while ((1 << p.shift) < kv->page_size) ++p.shift;
    return p;
}

inline int check_rope(const qtale_rope* rope, int head_dim) {
    if (!rope || !rope->freqs) return QTALE_ERR_INVALID_ARG;
    if (rope->layout != QTALE_ROPE_HALF && rope->layout != QTALE_ROPE_INTERLEAVED) return QTALE_ERR_UNSUPPORTED;
    if (rope->rotary_dim < 2 || rope->rotary_dim % 2 != 0 || rope->rotary_dim > head_dim) return QTALE_ERR_SHAPE;
    return std::isfinite(rope->magnitude) ? QTALE_OK : QTALE_ERR_INVALID_ARG;
}

// Rows of 16-bit values that are read or written in pieces of `unit` values.
inline int check_rows(const void* p, int64_t stride, int64_t row, int unit) {
    if (stride < row || stride % unit != 0) return QTALE_ERR_SHAPE;
    return reinterpret_cast<uintptr_t>(p) % (2 * unit) != 0 ? QTALE_ERR_INVALID_ARG : QTALE_OK;
}

inline int check_paged_attn(const qtale_paged_attn* a, const qtale_paged_kv* kv) {
    if (!a) return QTALE_ERR_INVALID_ARG;
    if (a->n_heads <= 0 || a->window < 0 || a->sinks < 0 || a->max_new < 0 || a->max_len < 0) return QTALE_ERR_INVALID_ARG;
    if (a->n_heads % kv->n_kv_heads != 0) return QTALE_ERR_SHAPE;
    return a->scale > 0.0f && std::isfinite(a->scale) ? QTALE_OK : QTALE_ERR_INVALID_ARG;
}

struct PagedAttnBounds { int max_new, max_len; };
inline PagedAttnBounds attn_bounds(const qtale_paged_attn* a, const qtale_paged_kv* kv, int T) {
    const int most = kv->max_pages * kv->page_size;
    return {a->max_new > 0 ? std::min(a->max_new, T) : T, a->max_len > 0 ? std::min(a->max_len, most) : most};
}

inline PagedAttnDev attn_device(const qtale_paged_kv* kv, int layer, const qtale_paged_attn* attn, const PagedAttnBounds& m, int T) {
    const PagedDev p = paged_device(kv, layer);
    PagedAttnDev a{};
    a.k = p.k; a.v = p.v; a.table = p.table; a.len = p.len; a.bf16 = p.bf16; a.q4 = p.q4;
    a.nh = attn->n_heads; a.nkv = p.nkv; a.rep = attn->n_heads / p.nkv; a.shift = p.shift; a.max_pages = p.max_pages; a.n_slots = p.n_slots;
    a.n_pages = p.n_pages; a.sinks = attn->window > 0 ? attn->sinks : 0; a.max_len = m.max_len;
    // places begin at -T (rows before their slot's begin), so that place - window stays in 32 bits; windows beyond the cache are all the same
    a.window = std::min(attn->window, INT32_MAX - T);
    a.scale_log2 = 1.4426950408889634f * attn->scale;
    return a;
}

}  // namespace qtale
