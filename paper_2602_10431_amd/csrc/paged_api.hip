// Host side of the paged K/V cache's C ABI (include/qtale.h): argument validation before any HIP call, then the launches.
#include <cmath>

#include "../../include/qtale.h"
#include "paged_check.h"

using namespace qtale;

namespace {

#define HIP_TRY(expr)                                   \
    do {                                                \
        hipError_t e__ = (expr);                        \
        if (e__ != hipSuccess) return QTALE_ERR_HIP;    \
    } while (0)

inline hipStream_t stream_of(void* s) { return reinterpret_cast<hipStream_t>(s); }

int check_workspace(const void* ws, size_t have, size_t need) {
    if (!ws || reinterpret_cast<uintptr_t>(ws) % 256 != 0) return QTALE_ERR_INVALID_ARG;
    return have < need ? QTALE_ERR_WORKSPACE_TOO_SMALL : QTALE_OK;
}

}  // namespace

extern "C" {

int qtale_pages_init(const qtale_paged_kv* kv, void* stream) {
    int e = check_paged(kv, true);
    if (e) return e;
    HIP_TRY(launch_pages_init(paged_device(kv, -1), stream_of(stream)));
    return QTALE_OK;
}

size_t qtale_pages_workspace_bytes(const qtale_paged_kv* kv, int max_seqs) {
    if (check_paged(kv, false) || max_seqs < 0 || max_seqs > kReserveItems) return 0;
    return pages_workspace_bytes(paged_device(kv, -1), max_seqs);
}

int qtale_pages_fork(const qtale_paged_kv* kv, const int32_t* src, const int32_t* dst, int n, void* stream) {
    int e = check_paged(kv, true);
    if (e) return e;
    if (n < 0 || (n > 0 && (!src || !dst))) return QTALE_ERR_INVALID_ARG;
    if (n == 0) return QTALE_OK;
    HIP_TRY(launch_pages_fork(paged_device(kv, -1), src, dst, n, stream_of(stream)));
    return QTALE_OK;
}

int qtale_pages_release(const qtale_paged_kv* kv, const int32_t* slots, int n, void* stream) {
    int e = check_paged(kv, true);
    if (e) return e;
    if (n < 0) return QTALE_ERR_INVALID_ARG;
    if (!slots && n > kv->n_slots) return QTALE_ERR_SHAPE;
    if (n == 0) return QTALE_OK;
    HIP_TRY(launch_pages_drop(paged_device(kv, -1), slots, n, true, 0, 0, stream_of(stream)));
    return QTALE_OK;
}

int qtale_pages_trim(const qtale_paged_kv* kv, const int32_t* slots, int n, int window, int sinks, void* stream) {
    int e = check_paged(kv, true);
    if (e) return e;
    if (n < 0 || window < 1 || sinks < 0) return QTALE_ERR_INVALID_ARG;
    if (!slots && n > kv->n_slots) return QTALE_ERR_SHAPE;
    if (n == 0) return QTALE_OK;
    HIP_TRY(launch_pages_drop(paged_device(kv, -1), slots, n, false, window, sinks, stream_of(stream)));
    return QTALE_OK;
}

int qtale_pages_reserve(const qtale_paged_kv* kv, int layer, const int32_t* seq_offsets, const int32_t* slots, int B, int32_t* first,
                        int32_t* missing, void* workspace, size_t workspace_bytes, void* stream) {
    int e = check_paged(kv, true);
    if (e) return e;
    if (B < 0 || layer < -1 || layer >= kv->n_layers) return QTALE_ERR_INVALID_ARG;
    if (B > kReserveItems) return QTALE_ERR_UNSUPPORTED;
    if (!slots && B > kv->n_slots) return QTALE_ERR_SHAPE;
    if (B == 0) return QTALE_OK;
    if (!seq_offsets) return QTALE_ERR_INVALID_ARG;
    const PagedDev p = paged_device(kv, -1);
    if ((e = check_workspace(workspace, workspace_bytes, pages_workspace_bytes(p, B)))) return e;
    HIP_TRY(launch_pages_reserve(p, layer, seq_offsets, slots, B, first, missing, true, workspace, stream_of(stream)));
    return QTALE_OK;
}

int qtale_pages_compact(const qtale_paged_kv* kv, int32_t* n_live, void* workspace, size_t workspace_bytes, void* stream) {
    int e = check_paged(kv, true);
    if (e) return e;
    const PagedDev p = paged_device(kv, -1);
    if ((e = check_workspace(workspace, workspace_bytes, pages_workspace_bytes(p, 0)))) return e;
    HIP_TRY(launch_pages_compact(p, n_live, workspace, stream_of(stream)));
    return QTALE_OK;
}

int qtale_pages_copy(const qtale_paged_kv* from, const qtale_paged_kv* to, const int32_t* src, const int32_t* dst, int n, void* stream) {
    int e = check_paged(from, true);
    if (e || (e = check_paged(to, true))) return e;
    if (from->page_size != to->page_size || from->n_kv_heads != to->n_kv_heads || from->head_dim != to->head_dim || from->dtype != to->dtype)
        return QTALE_ERR_SHAPE;
    if (n < 0 || (n > 0 && (!src || !dst))) return QTALE_ERR_INVALID_ARG;
    if (n == 0) return QTALE_OK;
    HIP_TRY(launch_pages_copy(paged_device(from, -1), paged_device(to, -1), src, dst, n, stream_of(stream)));
    return QTALE_OK;
}

int qtale_rope_frequencies(int rotary_dim, float base, int scaling, float factor, int original_len, float low, float high, double* freqs,
                           float* magnitude) {
    if (rotary_dim < 2 || rotary_dim % 2 != 0 || !(base > 0.0f) || !std::isfinite(base) || !freqs || !magnitude) return QTALE_ERR_INVALID_ARG;
    if (scaling < QTALE_ROPE_PLAIN || scaling > QTALE_ROPE_PARTS) return QTALE_ERR_UNSUPPORTED;
    if (scaling != QTALE_ROPE_PLAIN && (!(factor > 0.0f) || !std::isfinite(factor))) return QTALE_ERR_INVALID_ARG;
    const bool by_length = scaling == QTALE_ROPE_BANDS || scaling == QTALE_ROPE_PARTS;
    if (by_length && (original_len <= 0 || !(low > 0.0f) || !(high > low) || !std::isfinite(high))) return QTALE_ERR_INVALID_ARG;
    if (scaling == QTALE_ROPE_BASE && rotary_dim == 2) return QTALE_ERR_UNSUPPORTED;
    if (scaling == QTALE_ROPE_PARTS && !(base > 1.0f)) return QTALE_ERR_INVALID_ARG;
    const double r = rotary_dim, two_pi = 6.283185307179586477, f = factor;
    const double theta = scaling == QTALE_ROPE_BASE ? base * std::pow(f, r / (r - 2.0)) : static_cast<double>(base);
    *magnitude = 1.0f;
    double ramp_lo = 0.0, ramp_hi = 0.0;
    if (scaling == QTALE_ROPE_PARTS) {
        // the pair that makes `turns` turns over the original length
        auto pair_of = [&](double turns) { return r * std::log(original_len / (turns * two_pi)) / (2.0 * std::log(theta)); };
        ramp_lo = std::max(std::floor(pair_of(high)), 0.0);
        ramp_hi = std::min(std::ceil(pair_of(low)), r - 1.0);
        *magnitude = f > 1.0 ? static_cast<float>(0.1 * std::log(f) + 1.0) : 1.0f;
    }
    for (int i = 0; i < rotary_dim / 2; ++i) {
        const double w = std::pow(theta, -2.0 * i / r);
        double keep = 1.0;                                       // share of the unscaled frequency
        if (scaling == QTALE_ROPE_LINEAR) keep = 0.0;
        else if (scaling == QTALE_ROPE_BANDS) keep = (original_len * w / two_pi - low) / (static_cast<double>(high) - low);
        else if (scaling == QTALE_ROPE_PARTS) keep = 1.0 - (i - ramp_lo) / std::max(ramp_hi - ramp_lo, 0.001);
        keep = std::min(std::max(keep, 0.0), 1.0);
        freqs[i] = scaling == QTALE_ROPE_PLAIN || scaling == QTALE_ROPE_BASE ? w : w * keep + w / f * (1.0 - keep);
    }
    return QTALE_OK;
}

int qtale_paged_rope_append(const qtale_paged_kv* kv, int layer, const qtale_rope* rope, const void* q, int64_t q_stride, const void* k,
                            int64_t k_stride, const void* v, int64_t v_stride, void* q_out, int64_t q_out_stride, int n_heads, int T,
                            const int32_t* seq_offsets, const int32_t* slots, const int32_t* first, int B, const int32_t* positions, void* stream) {
    int e = check_paged(kv, true);
    if (e) return e;
    if ((e = check_rope(rope, kv->head_dim))) return e;
    if (layer < 0 || layer >= kv->n_layers || n_heads <= 0 || T < 0 || B < 0) return QTALE_ERR_INVALID_ARG;
    if (!slots && B > kv->n_slots) return QTALE_ERR_SHAPE;
    if (T == 0) return QTALE_OK;
    if (B == 0 || !q || !k || !v || !q_out || !seq_offsets || !positions) return QTALE_ERR_INVALID_ARG;
    const int d = kv->head_dim;
    const int64_t q_row = static_cast<int64_t>(n_heads) * d, kv_row = static_cast<int64_t>(kv->n_kv_heads) * d;
    if ((e = check_rows(q, q_stride, q_row, 8)) || (e = check_rows(k, k_stride, kv_row, 8)) || (e = check_rows(v, v_stride, kv_row, 8)) ||
        (e = check_rows(q_out, q_out_stride, q_row, 8)))
        return e;
    PagedRopeArgs a{};
    a.kv = paged_device(kv, layer);
    a.layout = rope->layout; a.rotary_dim = rope->rotary_dim; a.freqs = rope->freqs; a.magnitude = rope->magnitude;
    a.q = static_cast<const uint16_t*>(q); a.k = static_cast<const uint16_t*>(k); a.v = static_cast<const uint16_t*>(v);
    a.q_out = static_cast<uint16_t*>(q_out);
    a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.q_out_stride = q_out_stride;
    a.nh = n_heads; a.T = T; a.B = B; a.seq_offsets = seq_offsets; a.slots = slots; a.first = first; a.positions = positions;
    HIP_TRY(launch_paged_rope(a, stream_of(stream)));
    return QTALE_OK;
}

int qtale_paged_read(const qtale_paged_kv* kv, int layer, void* k, int64_t k_stride, void* v, int64_t v_stride, int T, const int32_t* seq_offsets,
                     const int32_t* slots, const int32_t* first, int B, void* stream) {
    int e = check_paged(kv, true);
    if (e) return e;
    if (layer < 0 || layer >= kv->n_layers || T < 0 || B < 0) return QTALE_ERR_INVALID_ARG;
    if (!slots && B > kv->n_slots) return QTALE_ERR_SHAPE;
    if (T == 0) return QTALE_OK;
    if (B == 0 || !k || !v || !seq_offsets) return QTALE_ERR_INVALID_ARG;
    const int64_t row = static_cast<int64_t>(kv->n_kv_heads) * kv->head_dim;
    if ((e = check_rows(k, k_stride, row, 8)) || (e = check_rows(v, v_stride, row, 8))) return e;
    PagedReadArgs a{};
    a.kv = paged_device(kv, layer);
    a.k = static_cast<uint16_t*>(k); a.v = static_cast<uint16_t*>(v); a.k_stride = k_stride; a.v_stride = v_stride;
    a.T = T; a.B = B; a.seq_offsets = seq_offsets; a.slots = slots; a.first = first;
    HIP_TRY(launch_paged_read(a, stream_of(stream)));
    return QTALE_OK;
}

size_t qtale_paged_attention_workspace_bytes(const qtale_paged_kv* kv, const qtale_paged_attn* attn, int T, int B) {
    if (check_paged(kv, false) || check_paged_attn(attn, kv) || T < 0 || B < 0) return 0;
    return T == 0 || B == 0 ? 256 : paged_attention_bytes(attn->n_heads, kv->n_kv_heads, kv->head_dim, T, B);
}

int qtale_paged_attention(const qtale_paged_kv* kv, int layer, const qtale_paged_attn* attn, const void* q, int64_t q_stride, void* out,
                          int64_t out_stride, int T, const int32_t* seq_offsets, const int32_t* slots, const int32_t* first, int B,
                          void* workspace, size_t workspace_bytes, void* stream) {
    int e = check_paged(kv, true);
    if (e) return e;
    if ((e = check_paged_attn(attn, kv))) return e;
    if (layer < 0 || layer >= kv->n_layers || T < 0 || B < 0) return QTALE_ERR_INVALID_ARG;
    if (B > 65535 - 4096) return QTALE_ERR_UNSUPPORTED;
    if (!slots && B > kv->n_slots) return QTALE_ERR_SHAPE;
    if (T == 0) return QTALE_OK;
    if (B == 0 || !q || !out || !seq_offsets) return QTALE_ERR_INVALID_ARG;
    const int64_t row = static_cast<int64_t>(attn->n_heads) * kv->head_dim;
    if ((e = check_rows(q, q_stride, row, 8)) || (e = check_rows(out, out_stride, row, 4))) return e;
    const PagedAttnBounds m = attn_bounds(attn, kv, T);
    const PagedAttnPlan plan = plan_paged_attention((kv->dtype & QTALE_KV_INT4) != 0, attn->n_heads, kv->n_kv_heads, kv->head_dim, T, B, m.max_new, m.max_len, attn->window, attn->sinks);
    if (plan.too_large) return QTALE_ERR_UNSUPPORTED;
    if ((e = check_workspace(workspace, workspace_bytes, plan.bytes))) return e;
    PagedAttnDev a = attn_device(kv, layer, attn, m, T);
    a.q = static_cast<const uint16_t*>(q); a.out = static_cast<uint16_t*>(out); a.q_stride = q_stride; a.out_stride = out_stride;
    a.offs = seq_offsets; a.slots = slots; a.first = first; a.B = B;
    HIP_TRY(launch_paged_attention(a, plan, kv->head_dim, T, static_cast<float*>(workspace), stream_of(stream)));
    return QTALE_OK;
}

}  // extern "C"
