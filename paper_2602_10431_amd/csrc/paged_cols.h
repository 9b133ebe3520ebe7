// What the chunk kernels of both page forms share: which columns a workgroup has, and the pages of a tile of keys.
#pragma once
#include "paged_attn.h"

namespace qtale {

constexpr int kTileKeys = kChunkTileKeys;

// Work of a call, in tiles per kv head: the column tiles of a sequence see a number of key tiles that grows evenly from the first to the last.
__device__ __forceinline__ int chunk_work(const PagedAttnDev& p, int b) {
    const SeqView s(p, b);
    const int cols = s.n * p.rep;
    if (cols == 0 || (p.take != 0 && cols <= kDecodeCols)) return 0;
    const int nt = (cols + kChunkCols - 1) / kChunkCols;
    const int least = KeySteps<kTileKeys>(s.first, s.first + (min(kChunkCols, cols) - 1) / p.rep, s.len, p.window, p.sinks).steps;
    const int most = KeySteps<kTileKeys>(s.first + (nt - 1) * kChunkCols / p.rep, s.first + s.n - 1, s.len, p.window, p.sinks).steps;
    return nt * (least + most) / 2;
}

// Column tile `item` of the call, tiles of PER columns walked by their distance from their sequence's end, the longest first; false: there is
// none.  The same in every lane.
template <int PER>
__device__ __forceinline__ bool find_columns(const PagedAttnDev& p, int item, int* b_out, int* tile_out) {
    const int lane = threadIdx.x & 63;
    auto tiles_of = [&](int i) {                                 // column tiles of sequence i
        if (i >= p.B) return 0;
        const int cols = max(p.offs[i + 1] - p.offs[i], 0) * p.rep;
        return p.take != 0 && cols <= kDecodeCols ? 0 : (cols + PER - 1) / PER;
    };
    int b = 0, tile;
    if (p.B == 1) {
        tile = tiles_of(0) - 1 - item;
        if (tile < 0) return false;
    } else {
        // level j holds the j-th tile from the end of every sequence that has one: the largest j with fewer tiles before it than `item` + 1
        auto before = [&](int j) {
            int sum = 0;
            for (int b0 = 0; b0 < p.B; b0 += 64) sum += min(tiles_of(b0 + lane), j);
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
            return sum;
        };
        int j0 = 0, j1 = p.items;                                // before(j0) <= item; no level from j1 on
        if (before(j1) <= item) return false;
        while (j1 - j0 > 1) {
            const int mid = (j0 + j1) >> 1;
            if (before(mid) <= item) j0 = mid;
            else j1 = mid;
        }
        int rank = item - before(j0);
        b = -1;
        for (int b0 = 0; b0 < p.B && b < 0; b0 += 64) {
            const int nt = tiles_of(b0 + lane);
            const uint64_t here = __ballot(nt > j0);
            const int n = __popcll(here);
            if (rank < n) {
                // the lane whose bit has `rank` bits below it
                const bool me = ((here >> lane) & 1u) != 0 && __popcll(here & ((1ull << lane) - 1ull)) == rank;
                const int at = __ffsll(static_cast<long long>(__ballot(me))) - 1;
                b = b0 + at;
                tile = __shfl(nt, at, 64) - 1 - j0;
            } else {
                rank -= n;
            }
        }
        if (b < 0) return false;
    }
    *b_out = __builtin_amdgcn_readfirstlane(b);
    *tile_out = __builtin_amdgcn_readfirstlane(tile);
    return true;
}

// Workgroup -> (kv head, item).  Ids go round-robin to the 8 XCDs: with a multiple of 8 kv heads each XCD has its own, whose keys its L2 holds.
__device__ __forceinline__ void find_head(const PagedAttnDev& p, int* hk, int* item) {
    if ((p.nkv & 7) == 0) {
        const int hx = p.nkv >> 3, local = blockIdx.x >> 3;
        *item = __builtin_amdgcn_readfirstlane(local / hx);
        *hk = (blockIdx.x & 7) * hx + (local - *item * hx);
    } else {
        *item = __builtin_amdgcn_readfirstlane(static_cast<int>(blockIdx.x) / p.nkv);
        *hk = blockIdx.x - *item * p.nkv;
    }
}

// Pages of a tile: the one of a wave's keys, and which of the tile's four groups of 16 keys have none.
struct TilePages { int page, gone; };
__device__ __forceinline__ TilePages tile_pages(const PageRow& pages, int key0, int group) {
    const int p0 = pages.at(key0);
    if (pages.shift >= 6) return TilePages{p0, p0 < 0 ? 15 : 0};  // (tiles begin at multiples of 64)
    const int p1 = pages.at(key0 + 16), p2 = pages.at(key0 + 32), p3 = pages.at(key0 + 48);
    return TilePages{group == 0 ? p0 : group == 1 ? p1 : group == 2 ? p2 : p3, (p0 < 0) | (p1 < 0) << 1 | (p2 < 0) << 2 | (p3 < 0) << 3};
}

}  // namespace qtale
