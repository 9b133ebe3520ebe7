// Copies of shared, partly filled pages, by the launch after the one that lists them (pages.hip): a launch of its own, or beside the rotation and
// the append of the same tokens, which writes other places of these pages: nobody stores below the length of a holder (pages_reserve_kernel).
#pragma once
#include "paged.h"
#include "qtale_dev.h"

namespace qtale {

// The `tokens` first places of every head.  A workgroup of 256 threads per (entry, head) at a time; this one takes units first, first + step, ...
__device__ __forceinline__ void split_pages(const PagedDev& p, const SplitList& l, int first, int step) {
    const int units = *l.n * p.nkv;
    const int row_chunks = p.d >> 3;                             // 16-byte chunks of a token's head
    for (int u = first; u < units; u += step) {
        const int4 e = l.entries[u / p.nkv];
        const int chunks = e.z * row_chunks;
        const size_t head = static_cast<size_t>(u % p.nkv) * row_chunks << p.shift, page = static_cast<size_t>(p.nkv) * row_chunks << p.shift;
        const size_t from = e.x * page + head, to = e.y * page + head;
        const u32x4_t *k0 = reinterpret_cast<const u32x4_t*>(p.k) + from, *v0 = reinterpret_cast<const u32x4_t*>(p.v) + from;
        u32x4_t *k1 = reinterpret_cast<u32x4_t*>(p.k) + to, *v1 = reinterpret_cast<u32x4_t*>(p.v) + to;
        // (chunks of keys, then of values: four of them in flight per thread)
        for (int c = threadIdx.x; c < 2 * chunks; c += 4 * 256) {
            u32x4_t x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at = min(c + i * 256, 2 * chunks - 1);
                x[i] = at < chunks ? k0[at] : v0[at - chunks];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at = c + i * 256;
                if (at < chunks) k1[at] = x[i];
                else if (at < 2 * chunks) v1[at - chunks] = x[i];
            }
        }
    }
}

}  // namespace qtale
