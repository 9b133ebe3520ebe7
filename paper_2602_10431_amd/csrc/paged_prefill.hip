// Attention of a chunk of new tokens over pages.
//
// One workgroup of four waves per (sequence, kv head, 128 columns[, key range]); a column is a (query, head) pair of the kv head, queries
// slowest, so the query heads that share keys share their tiles and a chunk's diagonal is short.  Keys and values come in tiles of 64 from the
// pages straight into LDS (no registers between), each wave fetches 16 keys: they lie in one page whatever its size, so a tile costs a wave
// one table entry and two buffer descriptors.  The descriptors end at the last key: what lies past it, or in pages that are gone, arrives as
// zeros.  S^T = K Q^T, so a lane owns one column (softmax statistics per lane); the probabilities, in the accumulator's layout, are the B
// operand of O^T = V^T P^T, and V^T comes from LDS by transposing reads (4 keys x 16 columns per 16 lanes).
//
// LDS tiles are [key][d] without padding (the fetch writes 16 bytes per lane in lane order); bank conflicts are avoided by where a lane
// fetches from: 16-byte chunk c of key k lies at chunk c ^ swizzle(k), for keys such that 16 rows of one chunk (what a K read touches at a
// time) and 4 rows of 4 chunks (a V read) cover all banks.
// Tile t + 1 is fetched while tile t is computed, one barrier per tile, two workgroups per CU.
#include <algorithm>
#include <type_traits>

#include "paged_attn.h"

namespace qtale {

constexpr int kTileKeys = kChunkTileKeys;

typedef __fp16 fp16x4_t __attribute__((ext_vector_type(4)));

// (The host pass does not know these instructions' forms and would drop the kernels that name them.)
__device__ __forceinline__ u32x2_t read_transposed(const uint16_t* at) {
#ifdef __HIP_DEVICE_COMPILE__
    return __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4f16((__attribute__((address_space(3))) fp16x4_t*)(at)));
#else
    return u32x2_t{0u, 0u};
#endif
}
// 16 bytes per lane from `offset` of the buffer to LDS, in lane order from `to` on
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t from, uint32_t offset, uint16_t* to) {
#ifdef __HIP_DEVICE_COMPILE__
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)(to), 16, offset, 0, 0, 0);
#endif
}

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

template <int D, bool BF16, bool SPLIT, int KG>
__global__ void __launch_bounds__(256 * KG, 2)
paged_chunk_kernel(PagedAttnDev p) {
    using A = Act16<BF16>;
    constexpr int KS = D / 16;                   // k-steps of the scores
    constexpr int DF = D / 32;                   // output fragments
    constexpr int CPR = D / 8;                   // 16-byte chunks of a row
    constexpr int RPF = 64 / CPR;                // rows per fetch instruction (1 KB)
    constexpr int NF = 16 / RPF;                 // fetch instructions per wave for 16 keys
    constexpr int TILE = kTileKeys * D;
    __shared__ __attribute__((aligned(1024))) uint16_t K0s[KG * TILE], K1s[KG * TILE], V0s[KG * TILE], V1s[KG * TILE];

    const int tid = threadIdx.x, lane = tid & 63;
    const int group = KG > 1 ? __builtin_amdgcn_readfirstlane(tid >> 8) : 0;
    const int wave = __builtin_amdgcn_readfirstlane((tid >> 6) & 3);   // of its group
    const int l32 = lane & 31, lhi = lane >> 5;

    // Workgroup -> (range, column tile, kv head).  Ids go round-robin to the 8 XCDs: with a multiple of 8 kv heads each XCD has its own, whose
    // keys its L2 then holds.  Column tiles are walked by their distance from their sequence's end, the longest first.
    int hk, item;
    if ((p.nkv & 7) == 0) {
        const int hx = p.nkv >> 3, local = blockIdx.x >> 3;
        item = __builtin_amdgcn_readfirstlane(local / hx);
        hk = (blockIdx.x & 7) * hx + (local - item * hx);
    } else {
        item = __builtin_amdgcn_readfirstlane(static_cast<int>(blockIdx.x) / p.nkv);
        hk = blockIdx.x - item * p.nkv;
    }
    int z = 0;
    if (SPLIT) {
        z = __builtin_amdgcn_readfirstlane(item / p.items);
        item -= z * p.items;
    }
    int b, qt;
    auto tiles_of = [&](int i) {                                 // column tiles of sequence i
        if (i >= p.B) return 0;
        const int cols = max(p.offs[i + 1] - p.offs[i], 0) * p.rep;
        return p.take != 0 && cols <= kDecodeCols ? 0 : (cols + kChunkCols - 1) / kChunkCols;
    };
    if (p.B == 1) {
        b = 0;
        qt = tiles_of(0) - 1 - item;
        if (qt < 0) return;
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
        if (before(j1) <= item) return;
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
                qt = __shfl(nt, at, 64) - 1 - j0;
            } else {
                rank -= n;
            }
        }
        if (b < 0) return;
    }
    b = __builtin_amdgcn_readfirstlane(b);
    qt = __builtin_amdgcn_readfirstlane(qt);
    SeqView s(p, b);
    s.uniform();
    const int cols = s.n * p.rep;
    const int c_lo = qt * kChunkCols, c_hi = min(c_lo + kChunkCols, cols) - 1;   // this workgroup's columns

    // this lane's column, clamped to a live one
    const int col = min(c_lo + wave * 32 + l32, c_hi);
    const int qi = col / p.rep, head = hk * p.rep + col - qi * p.rep;
    const int place = s.first + qi;
    const int reach = p.window > 0 ? place - p.window : INT32_MIN;   // keys after it are in its window
    const bool wave_live = c_lo + wave * 32 <= c_hi;
    auto place_of = [&](int column) { return s.first + __builtin_amdgcn_readfirstlane(column / p.rep); };   // (divisions run on the vector ALUs)
    const int w_first = place_of(min(c_lo + wave * 32, c_hi)), w_last = place_of(min(c_lo + wave * 32 + 31, c_hi));   // the wave's queries
    const KeySteps<kTileKeys> walk(place_of(c_lo), place_of(c_hi), s.len, p.window, p.sinks);
    int t0 = 0, t1 = walk.steps, ranges = 1;
    if (SPLIT) {
        // ranges of about equal length over the whole call, as many as are to run at once; no item is cut into more than p.ranges
        int work = 0;
        for (int b0 = 0; b0 < p.B; b0 += 64) work += b0 + lane < p.B ? chunk_work(p, b0 + lane) : 0;
#pragma unroll
        for (int x = 32; x > 0; x >>= 1) work += __shfl_xor(work, x, 64);
        const int wanted = max(p.target / p.nkv, 1);
        const int per = __builtin_amdgcn_readfirstlane(max(max((work + wanted - 1) / wanted, (walk.steps + p.ranges - 1) / p.ranges), 4 * KG));
        ranges = __builtin_amdgcn_readfirstlane(max((walk.steps + per - 1) / per, 1));
        if (z >= ranges) return;
        t0 = z * per;
        t1 = min(t0 + per, walk.steps);
    }

    u32x4_t qf[KS];
    const uint16_t* qrow = p.q + (s.row0 + qi) * p.q_stride + head * D + 8 * lhi;
#pragma unroll
    for (int k = 0; k < KS; ++k) qf[k] = *reinterpret_cast<const u32x4_t*>(qrow + 16 * k);

    const PageRow pages(p, s.slot);
    const size_t head_elems = static_cast<size_t>(D) << p.shift;
    const int page_mask = (1 << p.shift) - 1, hi = walk.hi;

    // this lane's source offsets: LDS place (row r of the wave's 16, chunk c) holds chunk c ^ swizzle
    uint32_t k_src[NF], v_src[NF];
#pragma unroll
    for (int i = 0; i < NF; ++i) {
        const int r = i * RPF + lane / CPR, c = lane % CPR;
        const int ks = D == 128 ? r & 15 : (r >> 1) & 7, vs = D == 128 ? 4 * (r & 3) : 4 * ((r >> 1) & 1);
        k_src[i] = r * (2 * D) + (c ^ ks) * 16;
        v_src[i] = r * (2 * D) + (c ^ vs) * 16;
    }
    auto fetch = [&](int tile, int page, uint16_t* K, uint16_t* V) {   // page: of this wave's keys of the tile
        const int key = walk.key(tile) + 16 * wave;
        const int rows = page < 0 ? 0 : min(max(hi - key, 0), 16);
        const size_t at = (static_cast<size_t>(max(page, 0)) * p.nkv + hk) * head_elems + static_cast<size_t>(key & page_mask) * D;
        const auto kb = buffer_of(p.k + at, rows * (2 * D)), vb = buffer_of(p.v + at, rows * (2 * D));
#pragma unroll
        for (int i = 0; i < NF; ++i)
            load_to_lds(kb, k_src[i], K + 16 * D * wave + 512 * i);
#pragma unroll
        for (int i = 0; i < NF; ++i)
            load_to_lds(vb, v_src[i], V + 16 * D * wave + 512 * i);
    };
    struct Ids { int page, gone; };                              // page of this wave's keys; which of the tile's four groups have none
    auto ids_of = [&](int tile) {
        const int key0 = walk.key(min(tile, walk.steps - 1));
        const int p0 = pages.at(key0), p1 = pages.at(key0 + 16), p2 = pages.at(key0 + 32), p3 = pages.at(key0 + 48);
        return Ids{wave == 0 ? p0 : wave == 1 ? p1 : wave == 2 ? p2 : p3, (p0 < 0) | (p1 < 0) << 1 | (p2 < 0) << 2 | (p3 < 0) << 3};
    };

    // LDS reads: element offsets of this lane
    const int k_row = l32 * D, k_sw = D == 128 ? l32 & 15 : (l32 >> 1) & 7;
    int k_at[KS];                                                // chunk 2 k + lhi of key l32 (the tile's second half: 32 rows further)
#pragma unroll
    for (int k = 0; k < KS; ++k) k_at[k] = k_row + (((2 * k + lhi) ^ k_sw) * 8);
    const int v_key = 4 * lhi + ((lane & 15) >> 2);              // the transposing read's row of this lane, of 8
    const int v_sw = D == 128 ? 4 * (v_key & 3) : 4 * ((v_key >> 1) & 1);
    int v_at[DF];
#pragma unroll
    for (int f = 0; f < DF; ++f) v_at[f] = v_key * D + (((4 * f + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1)) ^ v_sw) * 8) + 4 * (lane & 1);

    const float sc = p.scale_log2;
    float16_t o[DF];
#pragma unroll
    for (int f = 0; f < DF; ++f)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[f][r] = 0.0f;
    float m_run = kPagedNone, l_run = 0.0f;

    auto compute = [&](int tile, int gone, const uint16_t* K, const uint16_t* V) {   // gone: bit per 16 keys without a page
        const int key0 = walk.key(tile);
        // S^T: rows are keys (two fragments of 32), the column this lane's query
        float16_t st[2];
#pragma unroll
        for (int kf = 0; kf < 2; ++kf) {
#pragma unroll
            for (int r = 0; r < 16; ++r) st[kf][r] = 0.0f;
#pragma unroll
            for (int k = 0; k < KS; ++k)
                st[kf] = A::mfma32(*reinterpret_cast<const u32x4_t*>(&K[kf * 32 * D + k_at[k]]), qf[k], st[kf]);
        }
        // a tile that every query of the wave sees whole needs no mask
        if (!(gone == 0 && key0 + kTileKeys <= min(w_first + 1, hi) && (p.window == 0 || key0 > w_last - p.window || key0 + kTileKeys <= p.sinks))) {
#pragma unroll
            for (int kf = 0; kf < 2; ++kf)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int key = key0 + kf * 32 + 8 * (r >> 2) + 4 * lhi + (r & 3);
                    const bool seen = (key <= place) & (key < hi) & ((gone >> (kf * 2 + (r >> 3)) & 1) == 0) & ((key > reach) | (key < p.sinks));
                    st[kf][r] = seen ? st[kf][r] : -INFINITY;
                }
        }
        float mx = -INFINITY;
#pragma unroll
        for (int kf = 0; kf < 2; ++kf)
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, st[kf][r]);
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        // Reference point of the exponentials: it follows the running maximum only when some column's has grown by more than kLazy
        // (probabilities stay below 2^kLazy), since moving it rescales all output accumulators.
        constexpr float kLazy = 4.0f;
        const float m_cand = fmaxf(m_run, mx * sc);
        if (__any(m_cand > m_run + kLazy)) {
            const float alpha = __builtin_amdgcn_exp2f(m_run - m_cand);
            l_run *= alpha;
#pragma unroll
            for (int f = 0; f < DF; ++f)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[f][r] *= alpha;
            m_run = m_cand;
        }
        float psum = 0.0f;
        u32x4_t pf[4];
#pragma unroll
        for (int kf = 0; kf < 2; ++kf)
#pragma unroll
            for (int r = 0; r < 16; r += 2) {
                const float p0 = __builtin_amdgcn_exp2f(fmaf(st[kf][r], sc, -m_run)), p1 = __builtin_amdgcn_exp2f(fmaf(st[kf][r + 1], sc, -m_run));
                psum += p0 + p1;                                 // in 32 bits
                pf[kf * 2 + (r >> 3)][(r & 7) >> 1] = A::pack(p0, p1);
            }
        l_run += psum;
        // O^T: k-step s2 covers keys 16 s2 .. + 15; operand element e of a lane is key 16 s2 + 8 (e / 4) + 4 lhi + e % 4
#pragma unroll
        for (int s2 = 0; s2 < 4; ++s2)
#pragma unroll
            for (int f = 0; f < DF; ++f) {
                const u32x2_t a = read_transposed(&V[16 * s2 * D + v_at[f]]), c = read_transposed(&V[(16 * s2 + 8) * D + v_at[f]]);
                o[f] = A::mfma32(u32x4_t{a[0], a[1], c[0], c[1]}, pf[s2], o[f]);
            }
    };

    if (t0 < t1) {
        // page ids are read a tile before the fetch that uses them; the groups of waves take every KG-th tile
        uint16_t *K0 = K0s + group * TILE, *K1 = K1s + group * TILE, *V0 = V0s + group * TILE, *V1 = V1s + group * TILE;
        const int own = t0 + group;
        Ids now = ids_of(own), next = ids_of(own + KG);
        if (own < t1) fetch(own, now.page, K0, V0);
        auto turn = [&](int t, uint16_t* K, uint16_t* V, uint16_t* K_next, uint16_t* V_next) {
            __builtin_amdgcn_s_waitcnt(0x0f70);                  // vmcnt(0): this wave's part of the tile is in LDS
            __syncthreads();                                     // everybody's is, and the other buffers have been read
            if (t + KG < t1) fetch(t + KG, next.page, K_next, V_next);
            const int gone = now.gone;
            now = next;
            next = ids_of(t + 2 * KG);
            if (wave_live && t < t1 && walk.key(t) <= w_last) compute(t, gone, K, V);
        };
        for (int t = t0; t < t1; t += 2 * KG) {
            turn(t + group, K0, V0, K1, V1);
            if (t + KG < t1) turn(t + KG + group, K1, V1, K0, V0);
        }
    }

    float l_tot = l_run + __shfl_xor(l_run, 32, 64);
    if constexpr (KG > 1) {
        // the second group's sums go through LDS, in the tiles' buffers, to the first
        static_assert(KG == 2, "two groups");
        float4_t* sums = reinterpret_cast<float4_t*>((wave < 2 ? K0s : K1s) + (wave & 1) * TILE) + lane;   // [DF * 4][64 lanes] per wave
        float2_t* stats = reinterpret_cast<float2_t*>(V0s) + wave * 64 + lane;
        __syncthreads();
        if (group == 1) {
#pragma unroll
            for (int f = 0; f < DF; ++f)
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) sums[(4 * f + q4) * 64] = float4_t{o[f][4 * q4], o[f][4 * q4 + 1], o[f][4 * q4 + 2], o[f][4 * q4 + 3]};
            *stats = float2_t{m_run, l_tot};
        }
        __syncthreads();
        if (group == 1) return;
        const float2_t other = *stats;
        const float m = fmaxf(m_run, other[0]), a0 = __builtin_amdgcn_exp2f(m_run - m), a1 = __builtin_amdgcn_exp2f(other[0] - m);
        m_run = m;
        l_tot = l_tot * a0 + other[1] * a1;
#pragma unroll
        for (int f = 0; f < DF; ++f)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                const float4_t x = sums[(4 * f + q4) * 64];
#pragma unroll
                for (int e = 0; e < 4; ++e) o[f][4 * q4 + e] = o[f][4 * q4 + e] * a0 + x[e] * a1;
            }
    }
    // columns whose sum is not finite (redo_column): both lanes of a column are left out below
    float zero = l_tot * 0.0f;
#pragma unroll
    for (int f = 0; f < DF; ++f)
#pragma unroll
        for (int r = 0; r < 16; ++r) zero = fmaf(o[f][r], 0.0f, zero);
    uint64_t redo = __ballot(zero != 0.0f && c_lo + wave * 32 + l32 <= c_hi);
    redo = (redo | redo >> 32) & 0xffffffffull;
#pragma unroll 1
    for (uint64_t left = redo; left != 0; left &= left - 1) {
        const int j = __ffsll(static_cast<long long>(left)) - 1;
        const int qj = __shfl(qi, j, 64), hj = __shfl(head, j, 64);
        float num[D / 64], m, l;
        redo_column<D, BF16>(p, walk, s.slot, hk, p.q + (s.row0 + qj) * p.q_stride + hj * D, s.first + qj, t0, t1, num, &m, &l);
        const size_t row = s.row0 + qj;
        put_column<D, BF16>(num, m, l, ranges > 1 ? p.part + ((row * p.nh + hj) * p.ranges + z) * part_stride(D) : nullptr, p.out + row * p.out_stride + hj * D);
    }
    if (c_lo + wave * 32 + l32 > c_hi) return;
    const bool done = (redo >> l32 & 1) != 0;
    const size_t pair = static_cast<size_t>(s.row0 + qi) * p.nh + head;
    if (SPLIT && ranges > 1) {
        float* dst = p.part + (pair * p.ranges + z) * part_stride(D);
        if (lhi == 0) dst[D + 2] = static_cast<float>(ranges);
        if (done) return;
#pragma unroll
        for (int f = 0; f < DF; ++f)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4)
                *reinterpret_cast<float4_t*>(dst + f * 32 + 8 * q4 + 4 * lhi) = float4_t{o[f][4 * q4], o[f][4 * q4 + 1], o[f][4 * q4 + 2], o[f][4 * q4 + 3]};
        if (lhi == 0) *reinterpret_cast<float2_t*>(dst + D) = float2_t{m_run, l_tot};
        return;
    }
    if (SPLIT && lhi == 0) p.part[pair * p.ranges * part_stride(D) + D + 2] = 1.0f;
    if (done) return;
    const float inv = l_tot != 0.0f ? 1.0f / l_tot : 0.0f;       // a row that sees no key is zero
    uint16_t* orow = p.out + (s.row0 + qi) * p.out_stride + head * D;
#pragma unroll
    for (int f = 0; f < DF; ++f)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
            u32x2_t w;
            w[0] = A::pack(o[f][4 * q4] * inv, o[f][4 * q4 + 1] * inv);
            w[1] = A::pack(o[f][4 * q4 + 2] * inv, o[f][4 * q4 + 3] * inv);
            *reinterpret_cast<u32x2_t*>(orow + f * 32 + 8 * q4 + 4 * lhi) = w;
        }
}

// Adds the key ranges of a (row, head) where there are several: D / 4 lanes each.
template <int D, bool BF16>
__global__ void __launch_bounds__(256)
chunk_combine_kernel(PagedAttnDev p, int T) {
    constexpr int W = part_stride(D), LANES = D / 4;
    const int pair = blockIdx.x * (256 / LANES) + threadIdx.x / LANES, row = pair / p.nh;
    if (row >= min(T, p.offs[p.B])) return;
    const float* src = p.part + static_cast<size_t>(pair) * p.ranges * W;
    const int ranges = min(static_cast<int>(src[D + 2]), p.ranges);
    if (ranges <= 1) return;
    RangeSum sum;
    sum.add_all<D>(0, 1, ranges, threadIdx.x % LANES, [&](int z) { return src + static_cast<size_t>(z) * W; });
    sum.put<BF16>(p.out + row * p.out_stride + (pair - row * p.nh) * D, threadIdx.x % LANES);
}

template <int D, bool BF16, int KG>
static hipError_t chunk_form(const PagedAttnDev& a, hipStream_t stream) {
    const bool split = a.ranges > 1;
    const int64_t items = static_cast<int64_t>(a.items) * a.ranges;
    const dim3 grid(static_cast<uint32_t>(items * a.nkv)), block(256 * KG);
    if (split) hipLaunchKernelGGL((paged_chunk_kernel<D, BF16, true, KG>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((paged_chunk_kernel<D, BF16, false, KG>), grid, block, 0, stream, a);
    return hipGetLastError();
}

template <int D, bool BF16>
static hipError_t chunk_groups(const PagedAttnDev& a, int groups, hipStream_t stream) {
    return groups == 2 ? chunk_form<D, BF16, 2>(a, stream) : chunk_form<D, BF16, 1>(a, stream);
}

hipError_t launch_paged_chunk(const PagedAttnDev& a, int groups, int d, int bf16, hipStream_t stream) {
    if (d == 128) return bf16 ? chunk_groups<128, true>(a, groups, stream) : chunk_groups<128, false>(a, groups, stream);
    return bf16 ? chunk_groups<64, true>(a, groups, stream) : chunk_groups<64, false>(a, groups, stream);
}

hipError_t launch_chunk_combine(const PagedAttnDev& a, int d, int bf16, int T, hipStream_t stream) {
    const int per = 1024 / d;                                    // (row, head) pairs per workgroup
    const dim3 grid(static_cast<uint32_t>((static_cast<int64_t>(T) * a.nh + per - 1) / per)), block(256);
    if (d == 128) {
        if (bf16) hipLaunchKernelGGL((chunk_combine_kernel<128, true>), grid, block, 0, stream, a, T);
        else hipLaunchKernelGGL((chunk_combine_kernel<128, false>), grid, block, 0, stream, a, T);
    } else {
        if (bf16) hipLaunchKernelGGL((chunk_combine_kernel<64, true>), grid, block, 0, stream, a, T);
        else hipLaunchKernelGGL((chunk_combine_kernel<64, false>), grid, block, 0, stream, a, T);
    }
    return hipGetLastError();
}

}  // namespace qtale
