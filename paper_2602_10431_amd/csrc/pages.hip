// Pages of the paged K/V cache: who holds them, and moving their contents.
//
// Everything is decided on the device, because what a layer's cache needs is known there only: a layer holds the tokens that executed it.
// What bounds these kernels is latency, chains of dependent loads, except where contents move.  us: room in one layer for a token of 1 / 64 / 256
// sequences 5.8 / 7.4 / 8.3 (with the launch that copies); in 32 layers for 32 sequences, 24 of them with a page to copy, 12.8, and 34.6 for the copies
// (190 MB read and written, 5.6 TB/s); fork, release, trim 4.6 to 7.4; compaction 6.8 to plan, 230 to move pages at 5.2 TB/s.
// Every result is a function of the state before the call alone: pages are taken lowest free index first, in the order of layers, then of
// the call's sequences, then of the pages' places; the counts are integers, so the order of their atomic updates does not show.
#include <algorithm>

#include "paged.h"
#include "paged_split.h"
#include "qtale_dev.h"

namespace qtale {

__device__ __forceinline__ bool page_ok(const PagedDev& p, int page) { return static_cast<uint32_t>(page) < static_cast<uint32_t>(p.n_pages); }
__device__ __forceinline__ bool slot_ok(const PagedDev& p, int slot) { return static_cast<uint32_t>(slot) < static_cast<uint32_t>(p.n_slots); }

__device__ __forceinline__ void drop_page(const PagedDev& p, int page) {
    if (atomicSub(&p.refs[page], 1) == 1) atomicOr(&p.bits[page >> 5], 1u << (page & 31));
}

__global__ void __launch_bounds__(256)
pages_init_kernel(PagedDev p) {
    const size_t step = static_cast<size_t>(gridDim.x) * 256, i0 = static_cast<size_t>(blockIdx.x) * 256 + threadIdx.x;
    const size_t slots = static_cast<size_t>(p.n_layers) * p.n_slots, entries = slots * p.max_pages;
    const size_t words = (static_cast<size_t>(p.n_pages) + 31) / 32;
    for (size_t i = i0; i < entries; i += step) p.table[i] = -1;
    for (size_t i = i0; i < slots; i += step) p.len[i] = p.cap[i] = 0;
    for (size_t i = i0; i < static_cast<size_t>(p.n_pages); i += step) p.refs[i] = 0;
    for (size_t i = i0; i < words; i += step) {
        const int left = p.n_pages - static_cast<int>(i * 32);
        p.bits[i] = left >= 32 ? 0xffffffffu : (1u << left) - 1u;
    }
}

hipError_t launch_pages_init(const PagedDev& p, hipStream_t stream) {
    const size_t entries = static_cast<size_t>(p.n_layers) * p.n_slots * p.max_pages;
    const int grid = static_cast<int>(std::min<size_t>((std::max<size_t>(entries, p.n_pages) + 255) / 256, 2048));
    hipLaunchKernelGGL(pages_init_kernel, dim3(grid), dim3(256), 0, stream, p);
    return hipGetLastError();
}

// One workgroup per (fork, layer): the copy shares the pages that hold tokens of its source; pages that the source only keeps room in stay
// its own.  A target that already has pages is left alone.
__global__ void __launch_bounds__(256)
pages_fork_kernel(PagedDev p, const int32_t* __restrict__ src, const int32_t* __restrict__ dst) {
    const int s = src[blockIdx.x], t = dst[blockIdx.x];
    if (!slot_ok(p, s) || !slot_ok(p, t) || s == t) return;
    const size_t at = static_cast<size_t>(blockIdx.y) * p.n_slots;
    __shared__ int taken;
    if (threadIdx.x == 0) taken = p.cap[at + t];
    const int len = p.len[at + s];
    __syncthreads();
    if (taken != 0) return;
    const int written = (len + (1 << p.shift) - 1) >> p.shift;
    const int32_t* from = p.table + (at + s) * p.max_pages;
    int32_t* to = p.table + (at + t) * p.max_pages;
    for (int j = threadIdx.x; j < p.max_pages; j += 256) {
        const int page = j < written ? from[j] : -1;
        to[j] = page;
        if (page_ok(p, page)) atomicAdd(&p.refs[page], 1);
    }
    if (threadIdx.x == 0) {
        p.len[at + t] = len;
        p.cap[at + t] = written << p.shift;
    }
}

hipError_t launch_pages_fork(const PagedDev& p, const int32_t* src, const int32_t* dst, int n, hipStream_t stream) {
    hipLaunchKernelGGL(pages_fork_kernel, dim3(n, p.n_layers), dim3(256), 0, stream, p, src, dst);
    return hipGetLastError();
}

// One workgroup per (slot, layer): RELEASE lets go of every page and empties the slot; otherwise of the pages that neither the first `sinks`
// tokens nor the window of the slot's next token reach.
template <bool RELEASE>
__global__ void __launch_bounds__(256)
pages_drop_kernel(PagedDev p, const int32_t* __restrict__ slots, int window, int sinks) {
    const int s = slots ? slots[blockIdx.x] : static_cast<int>(blockIdx.x);
    if (!slot_ok(p, s)) return;
    const size_t at = static_cast<size_t>(blockIdx.y) * p.n_slots + s;
    int32_t* row = p.table + at * p.max_pages;
    const int cap = p.cap[at], len = p.len[at];
    const int held = min(RELEASE ? (cap + (1 << p.shift) - 1) >> p.shift : max(len + 1 - window, 0) >> p.shift, p.max_pages);
    for (int j = threadIdx.x; j < held; j += 256) {
        if (!RELEASE && (static_cast<int64_t>(j) << p.shift) < sinks) continue;
        const int page = row[j];
        if (page < 0) continue;
        row[j] = -1;
        if (page_ok(p, page)) drop_page(p, page);
    }
    if (RELEASE) {
        __syncthreads();                                         // every thread has read the room
        if (threadIdx.x == 0) p.len[at] = p.cap[at] = 0;
    }
}

hipError_t launch_pages_drop(const PagedDev& p, const int32_t* slots, int n, bool release, int window, int sinks, hipStream_t stream) {
    const dim3 grid(n, p.n_layers), block(256);
    if (release) hipLaunchKernelGGL(pages_drop_kernel<true>, grid, block, 0, stream, p, slots, 0, 0);
    else hipLaunchKernelGGL(pages_drop_kernel<false>, grid, block, 0, stream, p, slots, window, sinks);
    return hipGetLastError();
}

// ---- moving pages ----------------------------------------------------------------------------------------
// Work lists in the workspace: [0] number of entries, then (from, to) or (from, to, tokens, -) per entry from byte 256 on.
constexpr int kMoveUnit = 16384;                 // bytes that a workgroup moves at a time: 256 threads x 4 x 16 bytes

__global__ void __launch_bounds__(256)
pages_split_kernel(PagedDev p, SplitList list) {
    split_pages(p, list, blockIdx.x, gridDim.x);
}

// Whole pages, keys and values; workgroups past `movers` rewrite the page table instead (remap of the pages from n_live on).
struct MoveArgs {
    const uint16_t *k0, *v0;
    uint16_t *k1, *v1;
    const int32_t* n_list;       // nullable: n
    int n, n_from, n_to;
    const int32_t *src, *dst;
    size_t page_bytes;
    int movers;
    int32_t* table;
    size_t entries;
    const int32_t* remap;
    const int32_t* n_live;
};
__global__ void __launch_bounds__(256)
pages_move_kernel(MoveArgs a) {
    if (static_cast<int>(blockIdx.x) >= a.movers) {
        const int live = *a.n_live;
        const size_t step = static_cast<size_t>(gridDim.x - a.movers) * 256;
        for (size_t i = static_cast<size_t>(blockIdx.x - a.movers) * 256 + threadIdx.x; i < a.entries; i += step) {
            const int page = a.table[i];
            if (page >= live && page < a.n_from) a.table[i] = a.remap[page];
        }
        return;
    }
    const int n = a.n_list ? *a.n_list : a.n;
    const int per = static_cast<int>((a.page_bytes + kMoveUnit - 1) / kMoveUnit);   // units of a page's keys, and of its values
    const int64_t units = static_cast<int64_t>(n) * 2 * per;
    const uint32_t chunks = static_cast<uint32_t>(a.page_bytes / 16);
    for (int64_t u = blockIdx.x; u < units; u += a.movers) {
        const int64_t e = u / (2 * per);
        const int part = static_cast<int>(u - e * (2 * per));
        const int s = a.src[e], t = a.dst[e];
        if (static_cast<uint32_t>(s) >= static_cast<uint32_t>(a.n_from) || static_cast<uint32_t>(t) >= static_cast<uint32_t>(a.n_to)) continue;
        const bool v = part >= per;
        const u32x4_t* from = reinterpret_cast<const u32x4_t*>((v ? a.v0 : a.k0) + s * (a.page_bytes / 2));
        u32x4_t* to = reinterpret_cast<u32x4_t*>((v ? a.v1 : a.k1) + t * (a.page_bytes / 2));
        const uint32_t c0 = static_cast<uint32_t>(v ? part - per : part) * (kMoveUnit / 16) + threadIdx.x;
        u32x4_t x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __builtin_nontemporal_load(from + min(c0 + i * 256, chunks - 1));
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c0 + i * 256 < chunks) __builtin_nontemporal_store(x[i], to + c0 + i * 256);
    }
}

constexpr int kMovers = 2048;                    // workgroups: eight per CU

hipError_t launch_pages_copy(const PagedDev& from, const PagedDev& to, const int32_t* src, const int32_t* dst, int n, hipStream_t stream) {
    MoveArgs a{};
    a.k0 = from.k; a.v0 = from.v; a.k1 = to.k; a.v1 = to.v;
    a.n = n; a.n_from = from.n_pages; a.n_to = to.n_pages; a.src = src; a.dst = dst;
    a.page_bytes = (static_cast<size_t>(from.nkv) * from.d * 2) << from.shift;
    const size_t units = static_cast<size_t>(n) * 2 * ((a.page_bytes + kMoveUnit - 1) / kMoveUnit);
    a.movers = static_cast<int>(std::min<size_t>(units, kMovers));
    hipLaunchKernelGGL(pages_move_kernel, dim3(a.movers), dim3(256), 0, stream, a);
    return hipGetLastError();
}

// ---- one workgroup of 1024 threads: sums over the workgroup ----------------------------------------------
constexpr int kPlan = 1024;

// Exclusive prefix sum of v over the workgroup; *total gets the sum.  Two barriers.
__device__ __forceinline__ int block_prefix(int v, int* sums, int* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o, 64);
        if (lane >= o) x += y;
    }
    __syncthreads();                                             // the sums of an earlier call have been read
    if (lane == 63) sums[wave] = x;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kPlan / 64; ++w) {
        const int s = sums[w];
        all += s;
        if (w < wave) before += s;
    }
    *total = all;
    return before + x - v;
}

// ---- room for new tokens ---------------------------------------------------------------------------------
// Per (layer, sequence): a page for the copy of a shared, partly filled last page, and the pages of tokens beyond its room.  Where all holders of such
// a page are in the call, the one with the most tokens (of several the last in order) writes into it and only the others take copies.  The
// most tokens, because holders need not have equally many: one whose copy the pool could not give stays behind with the page, and its next token
// would lie where the others have one already.  So no call writes below the length of any holder, nor where a copy of the same call reads.
// Thread t owns items 2 t and 2 t + 1 of a chunk of whole layers.
//   1. what each item needs, and its place in the order (prefix sum);
//   2. the free pages in ascending order, up to kFreeList at a time, into LDS; 32768 pages are looked at per round;
//   3. list entry k goes to the item whose span of the order holds it (binary search in LDS);
//   4. room and lengths, and the list of page contents to copy, which the next launch does.
constexpr int kFreeList = 4096;

__global__ void __launch_bounds__(kPlan)
pages_reserve_kernel(PagedDev p, int layer, const int32_t* __restrict__ offs, const int32_t* __restrict__ slots, int B, int32_t* __restrict__ first,
                     int32_t* __restrict__ missing, int32_t* __restrict__ n_copies, int4* __restrict__ copies) {
    __shared__ int start[kReserveItems + 1], row[kReserveItems], place[kReserveItems];
    __shared__ __attribute__((aligned(16))) int list[kFreeList];
    // until the list is made: the page that an item would go on in (-1: none), and its next place there with its place in the order, which decide
    int2* writers = reinterpret_cast<int2*>(list);
    static_assert(kFreeList >= 2 * kReserveItems, "the items fit the list");
    __shared__ int sums[kPlan / 64], s_copies;
    const int tid = threadIdx.x;
    const int l_begin = layer < 0 ? 0 : layer, l_end = layer < 0 ? p.n_layers : layer + 1;
    const int per = kReserveItems / B;                           // layers per chunk
    const int words = (p.n_pages + 31) >> 5;
    if (tid == 0) s_copies = 0;
    int w0 = 0, short_by = 0;                                    // free pages lie from word w0 on
    uint32_t ahead = tid < words ? p.bits[tid] : 0u;             // the first words, on their way beside the chain of loads below
    bool have_ahead = true;
    for (int l0 = l_begin; l0 < l_end; l0 += per) {
        const int items = min(per, l_end - l0) * B;
        int len[2], cap[2], n[2], at[2], need[2], shared[2], extra[2], old[2];
        bool copied[2];
        __syncthreads();                                         // the chunk before is done with LDS
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int i = 2 * tid + u;
            n[u] = len[u] = cap[u] = need[u] = extra[u] = shared[u] = 0;
            at[u] = old[u] = -1;
            copied[u] = false;
            if (i >= items) continue;
            const int b = i % B, l = l0 + i / B;
            const int slot = slots ? slots[b] : b;
            n[u] = max(offs[b + 1] - offs[b], 0);
            if (slot_ok(p, slot)) {
                at[u] = l * p.n_slots + slot;
                len[u] = p.len[at[u]];
                cap[u] = p.cap[at[u]];
                const int j = len[u] >> p.shift;
                if (n[u] > 0 && (len[u] & ((1 << p.shift) - 1)) != 0 && j < p.max_pages) {
                    const int page = p.table[static_cast<size_t>(at[u]) * p.max_pages + j];
                    if (page_ok(p, page)) { old[u] = page; shared[u] = p.refs[page]; }
                }
                const int64_t want = min((static_cast<int64_t>(len[u]) + n[u] + (1 << p.shift) - 1) >> p.shift, static_cast<int64_t>(p.max_pages));
                if (n[u] > 0) extra[u] = max(static_cast<int>(want) - (cap[u] >> p.shift), 0);
            }
            writers[i] = int2{old[u], (len[u] & ((1 << p.shift) - 1)) * kReserveItems + i % B};
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int i = 2 * tid + u;
            if (i < items && shared[u] > 1) {
                int holders = 0, keeps = -1;
                const int e0 = i - i % B;
#pragma unroll 8
                for (int e = e0; e < e0 + B; ++e) {
                    const int2 w = writers[e];
                    holders += w.x == old[u];
                    keeps = max(keeps, w.x == old[u] ? w.y : -1);
                }
                copied[u] = holders < shared[u] || keeps != writers[i].y;
            }
            need[u] = extra[u] + copied[u];
        }
        int total;
        const int before = block_prefix(need[0] + need[1], sums, &total);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int i = 2 * tid + u;
            if (i < items) {
                start[i] = before + (u ? need[0] : 0);
                row[i] = at[u];
                place[i] = copied[u] ? -1 - ((cap[u] >> p.shift) - 1) : (cap[u] >> p.shift);   // of order entry start[i]; negative: the copy, then from cap / P on
            }
        }
        int got = 0;                                             // pages handed out in this chunk
        while (got < total && w0 < words) {
            const int w = w0 + tid;
            const uint32_t bits = have_ahead ? ahead : w < words ? p.bits[w] : 0u;
            have_ahead = false;
            int found;
            const int rank = block_prefix(__popc(bits), sums, &found);
            const int room = min(total - got, kFreeList);
            uint32_t rest = bits;
            for (int r = rank; rest != 0u && r < room; ++r) {
                list[r] = w * 32 + __ffs(static_cast<int>(rest)) - 1;
                rest &= rest - 1u;
            }
            if (rest != bits) p.bits[w] = rest;
            const int taken = min(found, room);
            __syncthreads();
            for (int k = tid; k < taken; k += kPlan) {
                const int order = got + k;
                int lo = 0, hi = items;                          // the last item with start <= order (items without needs share their start)
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (start[mid] <= order) lo = mid;
                    else hi = mid;
                }
                const int page = list[k];
                p.refs[page] = 1;
                const int rel = order - start[lo], pl = place[lo];
                if (pl < 0 && rel == 0) continue;                // the copy's page: its owner takes it below
                const int j = pl < 0 ? -1 - pl + rel : pl + rel;
                p.table[static_cast<size_t>(row[lo]) * p.max_pages + j] = page;
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int i = 2 * tid + u;
                if (i >= items || !copied[u]) continue;
                const int k = start[i] - got;
                if (k < 0 || k >= taken) continue;
                p.table[static_cast<size_t>(at[u]) * p.max_pages + (len[u] >> p.shift)] = list[k];
                atomicSub(&p.refs[old[u]], 1);                   // (at least one holder is left: no page becomes free here)
                copies[atomicAdd(&s_copies, 1)] = int4{old[u], list[k], len[u] & ((1 << p.shift) - 1), 0};
            }
            got += taken;
            if (found <= room) w0 += kPlan;                      // else the same words again, less what was taken
            __syncthreads();                                     // the list has been read; the words are written
        }
        short_by += total - got;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int i = 2 * tid + u;
            if (i >= items) continue;
            const int b = i % B, l = l0 + i / B;
            int now = len[u];
            if (at[u] >= 0) {
                const int have = min(max(got - start[i], 0), need[u]) - copied[u];   // -1: not even the page of the copy
                if (have > 0) p.cap[at[u]] = cap[u] + (have << p.shift);
                if (have >= 0) now = static_cast<int>(min(static_cast<int64_t>(len[u]) + n[u], static_cast<int64_t>(max(cap[u] + (have << p.shift), len[u]))));
                if (first) p.len[at[u]] = now;
            }
            if (first) first[(l - l_begin) * B + b] = len[u];
        }
    }
    __syncthreads();
    if (tid == 0) {
        *n_copies = s_copies;
        if (missing) *missing = short_by;
    }
}

size_t pages_workspace_bytes(const PagedDev& p, int B) {
    const size_t reserve = static_cast<size_t>(p.n_layers) * B * sizeof(int4);
    const size_t compact = static_cast<size_t>(p.n_pages) * 12;  // sources, targets, remap
    return 256 + (std::max(reserve, compact) + 255) / 256 * 256;
}

SplitList pages_split_list(void* workspace) {
    return SplitList{reinterpret_cast<int32_t*>(workspace), reinterpret_cast<const int4*>(reinterpret_cast<char*>(workspace) + 256)};
}

hipError_t launch_pages_reserve(const PagedDev& p, int layer, const int32_t* seq_offsets, const int32_t* slots, int B, int32_t* first,
                                int32_t* missing, bool split, void* workspace, hipStream_t stream) {
    const SplitList list = pages_split_list(workspace);
    hipLaunchKernelGGL(pages_reserve_kernel, dim3(1), dim3(kPlan), 0, stream, p, layer, seq_offsets, slots, B, first, missing, const_cast<int32_t*>(list.n),
                       const_cast<int4*>(list.entries));
    if (!split) return hipGetLastError();
    const int64_t units = static_cast<int64_t>(layer < 0 ? p.n_layers : 1) * B * p.nkv;
    hipLaunchKernelGGL(pages_split_kernel, dim3(static_cast<int>(std::min<int64_t>(units, kMovers))), dim3(256), 0, stream, p, list);
    return hipGetLastError();
}

// ---- compaction ------------------------------------------------------------------------------------------
// The k-th page in use at or past n_live (the number of pages in use) moves to the k-th free page below it.  One workgroup lists both from
// the free bits and rewrites counts and bits; the next launch moves the contents and rewrites the table.
__global__ void __launch_bounds__(kPlan)
pages_compact_plan_kernel(PagedDev p, int32_t* __restrict__ n_live, int32_t* __restrict__ n_moves, int32_t* __restrict__ src, int32_t* __restrict__ dst,
                          int32_t* __restrict__ remap) {
    __shared__ int sums[kPlan / 64];
    const int tid = threadIdx.x, words = (p.n_pages + 31) >> 5;
    auto used = [&](int w) {                                     // pages of word w that are in use
        if (w >= words) return 0u;
        const int left = p.n_pages - w * 32;
        return ~p.bits[w] & (left >= 32 ? 0xffffffffu : (1u << left) - 1u);
    };
    int mine = 0, live;
    for (int w = tid; w < words; w += kPlan) mine += __popc(used(w));
    block_prefix(mine, sums, &live);
    auto below = [&](int w) {                                    // bits of word w that lie below n_live
        const int n = live - w * 32;
        return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u;
    };
    int n_src = 0, n_dst = 0;
    for (int w0 = 0; w0 < words; w0 += kPlan) {
        const int w = w0 + tid;
        const uint32_t in_use = used(w), low = below(w);
        const int left = w < words ? p.n_pages - w * 32 : 0;
        const uint32_t valid = left >= 32 ? 0xffffffffu : left <= 0 ? 0u : (1u << left) - 1u;
        uint32_t from = in_use & ~low, to = ~in_use & low & valid;
        int found;
        int at = n_src + block_prefix(__popc(from), sums, &found);
        n_src += found;
        for (; from != 0u; from &= from - 1u) src[at++] = w * 32 + __ffs(static_cast<int>(from)) - 1;
        at = n_dst + block_prefix(__popc(to), sums, &found);
        n_dst += found;
        for (; to != 0u; to &= to - 1u) dst[at++] = w * 32 + __ffs(static_cast<int>(to)) - 1;
        if (w < words) p.bits[w] = valid & ~low;
    }
    __syncthreads();
    const int moves = min(n_src, n_dst);                         // (equal)
    for (int k = tid; k < moves; k += kPlan) {
        const int s = src[k], t = dst[k];
        remap[s] = t;
        p.refs[t] = p.refs[s];
        p.refs[s] = 0;
    }
    if (tid == 0) {
        n_moves[0] = moves;
        n_moves[1] = live;
        if (n_live) *n_live = live;
    }
}

hipError_t launch_pages_compact(const PagedDev& p, int32_t* n_live, void* workspace, hipStream_t stream) {
    int32_t* n_moves = reinterpret_cast<int32_t*>(workspace);
    int32_t* src = reinterpret_cast<int32_t*>(reinterpret_cast<char*>(workspace) + 256);
    int32_t *dst = src + p.n_pages, *remap = dst + p.n_pages;
    hipLaunchKernelGGL(pages_compact_plan_kernel, dim3(1), dim3(kPlan), 0, stream, p, n_live, n_moves, src, dst, remap);
    MoveArgs a{};
    a.k0 = a.k1 = p.k; a.v0 = a.v1 = p.v;
    a.n_list = n_moves; a.n_from = a.n_to = p.n_pages; a.src = src; a.dst = dst;
    a.page_bytes = (static_cast<size_t>(p.nkv) * p.d * 2) << p.shift;
    a.movers = kMovers;
    a.table = p.table; a.entries = static_cast<size_t>(p.n_layers) * p.n_slots * p.max_pages; a.remap = remap; a.n_live = n_moves + 1;
    const int writers = static_cast<int>(std::min<size_t>((a.entries + 1023) / 1024, 256));
    hipLaunchKernelGGL(pages_move_kernel, dim3(a.movers + writers), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace qtale
