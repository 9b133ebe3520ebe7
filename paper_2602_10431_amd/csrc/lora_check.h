// Checks of the adapters' arguments and their device views, for the entry points that take them.
#pragma once
#include "../../include/qtale.h"
#include "lora.h"

namespace qtale {

// buffers: also the pointers (size queries do not need them)
inline int check_lora(const qtale_lora* l, int N, int K, bool buffers) {
    if (!l || l->n_adapters <= 0 || l->max_rank <= 0) return QTALE_ERR_INVALID_ARG;
    if (l->max_rank > 128 || l->n_adapters > (1 << 20)) return QTALE_ERR_UNSUPPORTED;
    if (l->max_rank % 8 != 0 || l->N != N || l->K != K) return QTALE_ERR_SHAPE;
    if (!buffers) return QTALE_OK;
    if (!l->down || !l->up) return QTALE_ERR_INVALID_ARG;
    return (reinterpret_cast<uintptr_t>(l->down) | reinterpret_cast<uintptr_t>(l->up)) % 16 != 0 ? QTALE_ERR_INVALID_ARG : QTALE_OK;
}

inline LoraDev lora_device(const qtale_lora* l) {
    LoraDev x{};
    if (!l || l->n_adapters <= 0) return x;
    x.down = static_cast<const uint16_t*>(l->down); x.up = static_cast<const uint16_t*>(l->up); x.rank = l->rank; x.scale = l->scale;
    x.n = l->n_adapters; x.R = l->max_rank; x.N = l->N; x.K = l->K;
    return x;
}

}  // namespace qtale
