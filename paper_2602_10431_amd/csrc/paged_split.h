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

// The same for pages in 4 bits: keys' codes and scales are contiguous by tokens, values' codes by fours; of a last four that is only partly held the
// 16-bit pieces of the held tokens alone (the others' are somebody's to write).
__device__ __forceinline__ void split_pages4(const PagedDev& p, const SplitList& l, int first, int step) {
    const int units = *l.n * p.nkv;
    const size_t block = head_bytes(p), codes = static_cast<size_t>(p.d / 2) << p.shift;
    for (int u = first; u < units; u += step) {
        const int4 e = l.entries[u / p.nkv];
        const size_t from = (static_cast<size_t>(e.x) * p.nkv + u % p.nkv) * block, to = (static_cast<size_t>(e.y) * p.nkv + u % p.nkv) * block;
        const char *k0 = reinterpret_cast<const char*>(p.k) + from, *v0 = reinterpret_cast<const char*>(p.v) + from;
        char *k1 = reinterpret_cast<char*>(p.k) + to, *v1 = reinterpret_cast<char*>(p.v) + to;
        const int nk = e.z * (p.d / 32), nv = e.z / 4 * (p.d / 8);   // 16-byte chunks
        for (int c = threadIdx.x; c < nk + nv; c += 256) {
            const size_t at = 16 * static_cast<size_t>(c < nk ? c : c - nk);
            *reinterpret_cast<u32x4_t*>((c < nk ? k1 : v1) + at) = *reinterpret_cast<const u32x4_t*>((c < nk ? k0 : v0) + at);
        }
        for (int t = threadIdx.x; t < 2 * e.z; t += 256) {           // scales and zero points
            const size_t at = codes + 4 * static_cast<size_t>(t < e.z ? t : t - e.z);
            *reinterpret_cast<uint32_t*>((t < e.z ? k1 : v1) + at) = *reinterpret_cast<const uint32_t*>((t < e.z ? k0 : v0) + at);
        }
        const int rest = e.z & 3;
        for (int x = threadIdx.x; x < rest * (p.d / 4); x += 256) {
            const int t = x / (p.d / 4), q = x - t * (p.d / 4);
            const size_t at = 16 * static_cast<size_t>(nv) + 8 * q + 2 * t;   // (word 2 q + t / 2, half t % 2)
            *reinterpret_cast<uint16_t*>(v1 + at) = *reinterpret_cast<const uint16_t*>(v0 + at);
        }
    }
}

}  // namespace qtale
