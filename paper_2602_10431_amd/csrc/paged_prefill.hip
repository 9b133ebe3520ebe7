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
// Tile t + 1 is fetched while tile t is computed, one barrier per tile, two workgroups per CU (heads of 64: four).
//
// Probabilities go into the second product rounded to 16 bits, which adds about as much error as the output's own rounding (fp16 2.7e-4 where the
// output's alone is 2.1e-4, bf16 2.3e-3 / 1.7e-3); the second term that the kernel for few columns spends on it would be half as many products again.
//
// What bounds it is the chip's power: the same call on zeros, at the clock that those leave, takes 457 us where random data takes 570 to 597, card by card
// (4 x 4096 tokens, 32 heads on 8 kv heads of 128, the wide form: 920 to 960 TFLOP/s; a library product of 8192^3 reaches 1150).  500 tokens on 24000 take
// 204 to 214 us, 930 to 970 TFLOP/s.  Heads of 64, where a score costs half the products and as much softmax: 4 x 4096 325 us, 850 TFLOP/s; 350 and 1050
// tokens on 700 and 2100 44 us, 390 TFLOP/s, with the long prompt on the long cache 58 us, 440: one uneven round of workgroups.
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

// Where chunk c (16 bytes) of the tile's key r lies in LDS: at chunk c ^ swizzle of its row.
template <int D> __device__ __forceinline__ int k_swizzle(int r) { return D == 128 ? r & 15 : (r >> 1) & 7; }
template <int D> __device__ __forceinline__ int v_swizzle(int r) { return D == 128 ? 4 * (r & 3) : 4 * ((r >> 1) & 1); }

// Pages of a tile: the one of a wave's keys, and which of the tile's four groups of 16 keys have none.
struct TilePages { int page, gone; };
__device__ __forceinline__ TilePages tile_pages(const PageRow& pages, int key0, int group) {
    const int p0 = pages.at(key0);
    if (pages.shift >= 6) return TilePages{p0, p0 < 0 ? 15 : 0};  // (tiles begin at multiples of 64)
    const int p1 = pages.at(key0 + 16), p2 = pages.at(key0 + 32), p3 = pages.at(key0 + 48);
    return TilePages{group == 0 ? p0 : group == 1 ? p1 : group == 2 ? p2 : p3, (p0 < 0) | (p1 < 0) << 1 | (p2 < 0) << 2 | (p3 < 0) << 3};
}

// The buffer of up to 16 keys from `key` on in a page: it ends at the last key of the call's range.
template <int D>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t key_buffer(const PagedAttnDev& p, const uint16_t* pool, int hk, int page, int key, int hi) {
    const int rows = page < 0 ? 0 : min(max(hi - key, 0), 16);
    const size_t at = (static_cast<size_t>(max(page, 0)) * p.nkv + hk) * (static_cast<size_t>(D) << p.shift) + static_cast<size_t>(key & ((1 << p.shift) - 1)) * D;
    return buffer_of(pool + at, rows * (2 * D));
}

// One wave's 32 columns: their queries, scores of a tile, probabilities and sums.
template <int D, bool BF16>
struct ColumnWave {
    using A = Act16<BF16>;
    static constexpr int KS = D / 16;            // k-steps of the scores
    static constexpr int DF = D / 32;            // output fragments
    int qi, head, place, reach;                  // this lane's column (clamped to a live one): query, head, its place, keys after `reach` are in its window
    bool mine;                                   // the lane's column exists
    int w_first, w_last;                         // places of the wave's queries
    u32x4_t qf[KS];
    int k_at[KS], v_at[DF];                      // LDS elements that this lane reads: chunk 2 k + lhi of key l32; rows of the transposing reads
    float16_t st[2], o[DF];
    u32x4_t pf[4];
    float m_run, l_run;

    // columns c_lo .. c_hi; c0: the wave's first
    __device__ __forceinline__ ColumnWave(const PagedAttnDev& p, const SeqView& s, int hk, int c0, int c_hi) {
        const int lane = threadIdx.x & 63, l32 = lane & 31, lhi = lane >> 5;
        const int col = min(c0 + l32, c_hi);
        qi = col / p.rep;
        head = hk * p.rep + col - qi * p.rep;
        place = s.first + qi;
        reach = p.window > 0 ? place - p.window : INT32_MIN;
        mine = c0 + l32 <= c_hi;
        w_first = s.first + __builtin_amdgcn_readfirstlane(min(c0, c_hi) / p.rep);   // (divisions run on the vector ALUs)
        w_last = s.first + __builtin_amdgcn_readfirstlane(min(c0 + 31, c_hi) / p.rep);
        const uint16_t* qrow = p.q + (s.row0 + qi) * p.q_stride + head * D + 8 * lhi;
#pragma unroll
        for (int k = 0; k < KS; ++k) qf[k] = *reinterpret_cast<const u32x4_t*>(qrow + 16 * k);
#pragma unroll
        for (int k = 0; k < KS; ++k) k_at[k] = l32 * D + (((2 * k + lhi) ^ k_swizzle<D>(l32)) * 8);
        const int row = 4 * lhi + ((lane & 15) >> 2);            // of 8
#pragma unroll
        for (int f = 0; f < DF; ++f) v_at[f] = row * D + (((4 * f + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1)) ^ v_swizzle<D>(row)) * 8) + 4 * (lane & 1);
#pragma unroll
        for (int f = 0; f < DF; ++f)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[f][r] = 0.0f;
        m_run = kPagedNone;
        l_run = 0.0f;
    }

    // S^T: rows are keys (two fragments of 32), the column this lane's query.  between(i) is called after product i of 2 KS.
    template <class Between>
    __device__ __forceinline__ void scores(const uint16_t* K, Between between) {
#pragma unroll
        for (int kf = 0; kf < 2; ++kf)
#pragma unroll
            for (int r = 0; r < 16; ++r) st[kf][r] = 0.0f;
#pragma unroll
        for (int i = 0; i < 2 * KS; ++i) {
            const int kf = i / KS, k = i % KS;
            st[kf] = A::mfma32(*reinterpret_cast<const u32x4_t*>(&K[kf * 32 * D + k_at[k]]), qf[k], st[kf]);
            between(i);
        }
    }

    // Scores of keys key0 .. key0 + 63 -> probabilities; gone: bit per 16 keys without a page.
    __device__ __forceinline__ void softmax(const PagedAttnDev& p, int key0, int gone, int hi) {
        const int lhi = (threadIdx.x & 63) >> 5;
        const float sc = p.scale_log2;
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
        // Probabilities are 2^(score sc - scaled(m_run) + lift), one fused operation each; where scores are so large that the rounding of scaled(m_run)
        // shows, put() finds a sum that is not finite or too small for its own largest term.  The reference point m_run need not be the maximum,
        // only near it: it stays as long as the lane's probabilities of the tile add up to no more than kMost (for fp16 its largest number, so each
        // fits), which is seen from the sum that is needed anyway.  Finding the maximum, meeting the other half of the column and rescaling the
        // sums are left to the tiles that break it: the first, and few after it.
        constexpr float kMost = BF16 ? 16384.0f : 65504.0f;
        float sum = weigh(sc);
        if (__any(!(sum <= kMost))) {
            float mx = -INFINITY;
#pragma unroll
            for (int kf = 0; kf < 2; ++kf)
#pragma unroll
                for (int r = 0; r < 16; ++r) mx = fmaxf(mx, st[kf][r]);
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            const float m_new = fmaxf(m_run, mx), alpha = __builtin_amdgcn_exp2f(scaled(m_run, sc) - scaled(m_new, sc));
            l_run *= alpha;
#pragma unroll
            for (int f = 0; f < DF; ++f)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[f][r] *= alpha;
            m_run = m_new;
            sum = weigh(sc);
        }
        l_run += sum;
    }

    static __device__ __forceinline__ float scaled(float m, float sc) { return fmaxf(m * sc, -3.0e38f); }   // (finite also for a row that has seen no key)

    // Scores -> probabilities as operands; their sum, in 32 bits.
    __device__ __forceinline__ float weigh(float sc) {
        const float ms = scaled(m_run, sc) - kChunkLift<BF16>;
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int kf = 0; kf < 2; ++kf)
#pragma unroll
            for (int r = 0; r < 16; r += 2) {
                const float p0 = __builtin_amdgcn_exp2f(fmaf(st[kf][r], sc, -ms)), p1 = __builtin_amdgcn_exp2f(fmaf(st[kf][r + 1], sc, -ms));
                sum[(r >> 1) & 3] += p0 + p1;
                uint32_t w = A::pack(p0, p1);
                asm("" : "+v"(w));                               // (packed here: carried past the caller's branch, 32 values would take 16 registers more)
                pf[kf * 2 + (r >> 3)][(r & 7) >> 1] = w;
            }
        return (sum[0] + sum[1]) + (sum[2] + sum[3]);
    }

    // O^T: k-step s2 covers keys 16 s2 .. + 15; operand element e of a lane is key 16 s2 + 8 (e / 4) + 4 lhi + e % 4
    __device__ __forceinline__ void products(const uint16_t* V) {
#pragma unroll
        for (int s2 = 0; s2 < 4; ++s2)
#pragma unroll
            for (int f = 0; f < DF; ++f) {
                const u32x2_t a = read_transposed(&V[16 * s2 * D + v_at[f]]), c = read_transposed(&V[(16 * s2 + 8) * D + v_at[f]]);
                o[f] = A::mfma32(u32x4_t{a[0], a[1], c[0], c[1]}, pf[s2], o[f]);
            }
    }

    // products(V) and scores(K) of the next tile in one go, operands read AHEAD products before their use; between(i): as above, of ALL.
    static constexpr int PV = 4 * DF, ALL = PV + 2 * KS;
    template <class Between>
    __device__ __forceinline__ void products_scores(const uint16_t* V, const uint16_t* K, Between between) {
        constexpr int AHEAD = 6;
        u32x4_t x[AHEAD];
        auto read = [&](int i) __attribute__((always_inline)) {
            if (i < PV) {
                const int s2 = i / DF, f = i % DF;
                const u32x2_t a = read_transposed(&V[16 * s2 * D + v_at[f]]), c = read_transposed(&V[(16 * s2 + 8) * D + v_at[f]]);
                return u32x4_t{a[0], a[1], c[0], c[1]};
            }
            return *reinterpret_cast<const u32x4_t*>(&K[((i - PV) & 1) * 32 * D + k_at[(i - PV) >> 1]]);
        };
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) x[i] = read(i);
#pragma unroll
        for (int kf = 0; kf < 2; ++kf)
#pragma unroll
            for (int r = 0; r < 16; ++r) st[kf][r] = 0.0f;
#pragma unroll
        for (int i = 0; i < ALL; ++i) {
            const u32x4_t now = x[i % AHEAD];
            if (i < PV) o[i % DF] = A::mfma32(now, pf[i / DF], o[i % DF]);
            else st[(i - PV) & 1] = A::mfma32(now, qf[(i - PV) >> 1], st[(i - PV) & 1]);
            if (i + AHEAD < ALL) x[i % AHEAD] = read(i + AHEAD);
            between(i);
            __builtin_amdgcn_sched_barrier(0);
        }
    }

    // Results of steps t0 .. t1 - 1: to the output, or (SPLIT, several ranges) among the sums of range z.
    template <bool SPLIT>
    __device__ __forceinline__ void put(const PagedAttnDev& p, const SeqView& s, const KeySteps<kTileKeys>& walk, int hk, int t0, int t1, int z, int ranges, float l_tot) {
        const int lane = threadIdx.x & 63, l32 = lane & 31, lhi = lane >> 5;
        // columns whose sum is not finite, or below the one that the largest term is (redo_column): both lanes of a column are left out below
        constexpr float LEAST = BF16 ? 0.25f : 128.0f;           // a quarter of 2^lift
        float zero = m_run > kPagedNone && l_tot < LEAST ? 1.0f : l_tot * 0.0f;
#pragma unroll
        for (int f = 0; f < DF; ++f)
#pragma unroll
            for (int r = 0; r < 16; ++r) zero = fmaf(o[f][r], 0.0f, zero);
        uint64_t redo = __ballot(zero != 0.0f && mine);
        redo = (redo | redo >> 32) & 0xffffffffull;
#pragma unroll 1
        for (uint64_t left = redo; left != 0; left &= left - 1) {
            const int j = __ffsll(static_cast<long long>(left)) - 1;
            const int qj = __shfl(qi, j, 64), hj = __shfl(head, j, 64);
            const size_t row = s.row0 + qj;
            float num[D / 64], m, l;
            redo_column<D, BF16>(p, walk, s.slot, hk, p.q + row * p.q_stride + hj * D, s.first + qj, t0, t1, kChunkLift<BF16>, num, &m, &l);
            put_column<D, BF16>(num, m, l, SPLIT && ranges > 1 ? p.part + ((row * p.nh + hj) * p.ranges + z) * part_stride(D) : nullptr, p.out + row * p.out_stride + hj * D);
        }
        if (!mine) return;
        const bool done = (redo >> l32 & 1) != 0;
        if (SPLIT) {
            float* dst = p.part + ((static_cast<size_t>(s.row0 + qi) * p.nh + head) * p.ranges + z) * part_stride(D);
            if (lhi == 0) dst[D + 2] = static_cast<float>(ranges);
            if (done) return;
            if (ranges > 1) {
                // sums relative to scaled(m_run) -> to m_run times the scale: what the rounding left
                const float to = m_run > kPagedNone ? __builtin_amdgcn_exp2f(-fmaf(m_run, p.scale_log2, -scaled(m_run, p.scale_log2))) : 1.0f;
#pragma unroll
                for (int f = 0; f < DF; ++f)
#pragma unroll
                    for (int q4 = 0; q4 < 4; ++q4)
                        *reinterpret_cast<float4_t*>(dst + f * 32 + 8 * q4 + 4 * lhi) = float4_t{o[f][4 * q4], o[f][4 * q4 + 1], o[f][4 * q4 + 2], o[f][4 * q4 + 3]} * to;
                if (lhi == 0) *reinterpret_cast<float2_t*>(dst + D) = float2_t{m_run, l_tot * to};
                return;
            }
        }
        if (done) return;
        const float inv = l_tot != 0.0f ? 1.0f / l_tot : 0.0f;   // a row that sees no key is zero
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
};

// SPLIT: key ranges.  KG: groups of four waves that share the keys.  Waves per SIMD: two; for heads of 64 without ranges four, although a few
// registers go to memory then (4 x 4096 tokens 324 us, with three 334), with ranges, which are two workgroups per CU, two (3 x 440 tokens on 12728
// keys 199 us, with four 208).
template <int D, bool BF16, bool SPLIT, int KG>
__global__ void __launch_bounds__(256 * KG, D == 64 && !SPLIT ? 4 : 2)
paged_chunk_kernel(PagedAttnDev p) {
    static_assert(KG == 1 || !SPLIT, "ranges have one group");
    constexpr int DF = D / 32;                   // output fragments
    constexpr int CPR = D / 8;                   // 16-byte chunks of a row
    constexpr int RPF = 64 / CPR;                // rows per fetch instruction (1 KB)
    constexpr int NF = 16 / RPF;                 // fetch instructions per wave for 16 keys
    constexpr int TILE = kTileKeys * D;
    __shared__ __attribute__((aligned(1024))) uint16_t K0s[KG * TILE], K1s[KG * TILE], V0s[KG * TILE], V1s[KG * TILE];

    const int tid = threadIdx.x, lane = tid & 63;
    const int group = KG > 1 ? __builtin_amdgcn_readfirstlane(tid >> 8) : 0;
    const int wave = __builtin_amdgcn_readfirstlane((tid >> 6) & 3);   // of its group

    int hk, item, z = 0, b, qt;
    find_head(p, &hk, &item);
    if (SPLIT) {
        z = __builtin_amdgcn_readfirstlane(item / p.items);
        item -= z * p.items;
    }
    if (!find_columns<kChunkCols>(p, item, &b, &qt)) return;
    SeqView s(p, b);
    s.uniform();
    const int c_lo = qt * kChunkCols, c_hi = min(c_lo + kChunkCols, s.n * p.rep) - 1;   // this workgroup's columns
    const KeySteps<kTileKeys> walk(s.first + __builtin_amdgcn_readfirstlane(c_lo / p.rep), s.first + __builtin_amdgcn_readfirstlane(c_hi / p.rep), s.len, p.window, p.sinks);
    int t0 = 0, t1 = walk.steps, ranges = 1;
    if (SPLIT) {
        // ranges of about equal length over the whole call, as many as are to run at once; no item is cut into more than p.ranges
        int work = 0;
        for (int b0 = 0; b0 < p.B; b0 += 64) work += b0 + lane < p.B ? chunk_work(p, b0 + lane) : 0;
#pragma unroll
        for (int x = 32; x > 0; x >>= 1) work += __shfl_xor(work, x, 64);
        const int wanted = max(p.target / p.nkv, 1);
        const int per = __builtin_amdgcn_readfirstlane(max(max((work + wanted - 1) / wanted, (walk.steps + p.ranges - 1) / p.ranges), 4));
        ranges = __builtin_amdgcn_readfirstlane(max((walk.steps + per - 1) / per, 1));
        if (z >= ranges) return;
        t0 = z * per;
        t1 = min(t0 + per, walk.steps);
    }
    ColumnWave<D, BF16> cw(p, s, hk, c_lo + wave * 32, c_hi);

    const PageRow pages(p, s.slot);
    // this lane's source offsets among its wave's 16 keys
    uint32_t k_src[NF], v_src[NF];
#pragma unroll
    for (int i = 0; i < NF; ++i) {
        const int r = i * RPF + lane / CPR, c = lane % CPR;
        k_src[i] = r * (2 * D) + (c ^ k_swizzle<D>(r)) * 16;
        v_src[i] = r * (2 * D) + (c ^ v_swizzle<D>(r)) * 16;
    }
    // this wave's keys of a tile: the buffers (past the last tile empty: requests from them write zeros that nobody reads), and request i of 2 NF
    struct Source { __amdgpu_buffer_rsrc_t k, v; };
    auto source = [&](int tile, int page) __attribute__((always_inline)) {
        const int key = walk.key(tile) + 16 * wave, there = tile < t1 ? page : -1;
        return Source{key_buffer<D>(p, p.k, hk, there, key, walk.hi), key_buffer<D>(p, p.v, hk, there, key, walk.hi)};
    };
    auto request = [&](const Source& from, int i, uint16_t* K, uint16_t* V) __attribute__((always_inline)) {
        if (i < NF) load_to_lds(from.k, k_src[i], K + 16 * D * wave + 512 * i);
        else load_to_lds(from.v, v_src[i - NF], V + 16 * D * wave + 512 * (i - NF));
    };
    auto ids_of = [&](int tile) { return tile_pages(pages, walk.key(min(tile, walk.steps - 1)), wave); };

    if (t0 < t1) {
        // page ids are read a tile before the fetch that uses them; the groups of waves take every KG-th tile
        uint16_t *K0 = K0s + group * TILE, *K1 = K1s + group * TILE, *V0 = V0s + group * TILE, *V1 = V1s + group * TILE;
        const int own = t0 + group;
        TilePages now = ids_of(own), next = ids_of(own + KG);
        Source from = source(own, now.page);
#pragma unroll
        for (int i = 0; i < 2 * NF; ++i) request(from, i, K0, V0);
        from = source(own + KG, next.page);
        auto turn = [&](int t, uint16_t* K, uint16_t* V, uint16_t* K_next, uint16_t* V_next) __attribute__((always_inline)) {
            __builtin_amdgcn_s_waitcnt(0x0f70);                  // vmcnt(0): this wave's part of the tile is in LDS
            __syncthreads();                                     // everybody's is, and the other buffers have been read
            // (No branch around the tile: past the range, and for columns that see nothing of it, the mask leaves nothing.  The next tile's
            // requests go out among the products; sent at once they hold the wave up.)
            const int gone = t < t1 ? now.gone : 15, key0 = walk.key(t);
            cw.scores(K, [&](int i) __attribute__((always_inline)) {
                constexpr int EVERY = 2 * ColumnWave<D, BF16>::KS / (2 * NF);
                if (i % EVERY == 0) request(from, i / EVERY, K_next, V_next);
            });
            now = next;
            next = ids_of(t + 2 * KG);
            from = source(t + 2 * KG, next.page);
            cw.softmax(p, key0, gone, walk.hi);
            cw.products(V);
        };
        for (int t = t0; t < t1; t += 2 * KG) {
            turn(t + group, K0, V0, K1, V1);
            if (t + KG < t1) turn(t + KG + group, K1, V1, K0, V0);
        }
        // the last turn's requests are past the range and bring zeros; they have to be in LDS before a sum takes their place or the
        // workgroup's LDS goes to another
        __builtin_amdgcn_s_waitcnt(0x0f70);
    }

    float l_tot = cw.l_run + __shfl_xor(cw.l_run, 32, 64);
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
                for (int q4 = 0; q4 < 4; ++q4) sums[(4 * f + q4) * 64] = float4_t{cw.o[f][4 * q4], cw.o[f][4 * q4 + 1], cw.o[f][4 * q4 + 2], cw.o[f][4 * q4 + 3]};
            *stats = float2_t{cw.m_run, l_tot};
        }
        __syncthreads();
        if (group == 1) return;
        const float2_t other = *stats;
        const float m = fmaxf(cw.m_run, other[0]), ms = cw.scaled(m, p.scale_log2);
        const float a0 = __builtin_amdgcn_exp2f(cw.scaled(cw.m_run, p.scale_log2) - ms), a1 = __builtin_amdgcn_exp2f(cw.scaled(other[0], p.scale_log2) - ms);
        cw.m_run = m;
        l_tot = l_tot * a0 + other[1] * a1;
#pragma unroll
        for (int f = 0; f < DF; ++f)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                const float4_t x = sums[(4 * f + q4) * 64];
#pragma unroll
                for (int e = 0; e < 4; ++e) cw.o[f][4 * q4 + e] = cw.o[f][4 * q4 + e] * a0 + x[e] * a1;
            }
    }
    cw.template put<SPLIT>(p, s, walk, hk, t0, t1, z, ranges, l_tot);
}

// The same for calls of many column tiles: one workgroup of eight waves per 256 columns and CU, two waves per SIMD that take turns.  While the
// first half of the waves runs its products (matrix cores, LDS), the second half, which shares their SIMDs, runs its softmax (vector ALUs), then
// they change places; a barrier separates the phases.  Products of a turn: O^T of tile t and the scores of tile t + 1.
//   phase      0         1          2          3          4
//   half 0     S0, P0    O0, S1     P1         O1, S2     P2
//   half 1     S0        P0         O0, S1     P1         O1, S2
// In phase 2 t + 1 the first half requests keys t + 2 and values t + 1, into the buffers that phase 2 t was the last to read; it waits for them
// before phase 2 t + 3.
template <int D, bool BF16>
__global__ void __launch_bounds__(512, 2)
paged_wide_kernel(PagedAttnDev p) {
    constexpr int CPR = D / 8, RPF = 64 / CPR;
    constexpr int NF = 16 / RPF;                 // fetch instructions per wave for 16 keys
    constexpr int TILE = kTileKeys * D;
    __shared__ __attribute__((aligned(1024))) uint16_t K0[TILE], K1[TILE], V0[TILE], V1[TILE];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int hk, item, b, qt;
    find_head(p, &hk, &item);
    if (!find_columns<kWideCols>(p, item, &b, &qt)) return;
    SeqView s(p, b);
    s.uniform();
    const int c_lo = qt * kWideCols, c_hi = min(c_lo + kWideCols, s.n * p.rep) - 1;
    const KeySteps<kTileKeys> walk(s.first + __builtin_amdgcn_readfirstlane(c_lo / p.rep), s.first + __builtin_amdgcn_readfirstlane(c_hi / p.rep), s.len, p.window, p.sinks);
    ColumnWave<D, BF16> cw(p, s, hk, c_lo + wave * 32, c_hi);
    const int n = walk.steps;

    const PageRow pages(p, s.slot);
    uint32_t k_src[NF], v_src[NF];               // this lane's source offsets among the 16 keys that a wave of the first half fetches
#pragma unroll
    for (int i = 0; i < NF; ++i) {
        const int r = i * RPF + lane / CPR, c = lane % CPR;
        k_src[i] = r * (2 * D) + (c ^ k_swizzle<D>(r)) * 16;
        v_src[i] = r * (2 * D) + (c ^ v_swizzle<D>(r)) * 16;
    }
    // the buffer of this wave's keys of a tile (past the last one: empty, requests from it write zeros that nobody reads)
    auto buffer_at = [&](const uint16_t* pool, int tile, int page) __attribute__((always_inline)) {
        return key_buffer<D>(p, pool, hk, tile < n ? page : -1, walk.key(tile) + 16 * (wave & 3), walk.hi);
    };
    auto request = [&](__amdgpu_buffer_rsrc_t from, const uint32_t* src, int i, uint16_t* to) __attribute__((always_inline)) {
        load_to_lds(from, src[i], to + 16 * D * (wave & 3) + 512 * i);
    };
    auto ids_of = [&](int tile) __attribute__((always_inline)) { return tile_pages(pages, walk.key(min(tile, n - 1)), wave & 3); };
    // A phase's LDS reads have been consumed by its products, so nothing of a wave's own is outstanding but requests, which are to stay so:
    // a bare barrier that no access and no instruction is moved across.
    auto phase_end = [&]() __attribute__((always_inline)) {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
    };

    if (n > 0) {
        TilePages i0 = ids_of(0), i1 = ids_of(1), i2 = ids_of(2);
        if (wave < 4) {
            const auto k0 = buffer_at(p.k, 0, i0.page), v0 = buffer_at(p.v, 0, i0.page), k1 = buffer_at(p.k, 1, i1.page);
#pragma unroll
            for (int i = 0; i < NF; ++i) {
                request(k0, k_src, i, K0);
                request(v0, v_src, i, V0);
                request(k1, k_src, i, K1);
            }
            __builtin_amdgcn_s_waitcnt(0x0f70);
        }
        phase_end();
        auto weigh = [&](int t, int gone) __attribute__((always_inline)) { cw.softmax(p, walk.key(t), t < n ? gone : 15, walk.hi); };
        cw.scores(K0, [](int) {});
        // (both halves walk the same barriers)
        if (wave < 4) {
            // The requests go out among the products, two fetch instructions' time apart: sent at once, they held the wave up for 680 cycles of
            // the tile's 3600.  (Past the last tile the scores are of whatever lies there, and not used.)
            weigh(0, i0.gone);
            auto kb = buffer_at(p.k, 2, i2.page), vb = buffer_at(p.v, 1, i1.page);
            phase_end();
            auto turn = [&](int t, uint16_t* Kt, uint16_t* Vt, uint16_t* Kn, uint16_t* Vn) __attribute__((always_inline)) {
                constexpr int EVERY = ColumnWave<D, BF16>::ALL / (2 * NF);
                auto piece = [&](int i) __attribute__((always_inline)) {
                    if (i % EVERY != 0) return;
                    if (i / EVERY < NF) request(vb, v_src, i / EVERY, Vn);
                    else request(kb, k_src, i / EVERY - NF, Kt);
                };
                __builtin_amdgcn_s_setprio(1);
                cw.products_scores(Vt, Kn, piece);
                __builtin_amdgcn_s_setprio(0);
                phase_end();
                weigh(t + 1, i1.gone);
                i1 = i2;
                i2 = ids_of(t + 3);
                vb = buffer_at(p.v, t + 2, i1.page);
                kb = buffer_at(p.k, t + 3, i2.page);
                __builtin_amdgcn_s_waitcnt(0x0f70);
                phase_end();
            };
            for (int t = 0; t < n; t += 2) {
                turn(t, K0, V0, K1, V1);
                if (t + 1 < n) turn(t + 1, K1, V1, K0, V0);
            }
        } else {
            phase_end();
            auto turn = [&](int t, uint16_t* Vt, uint16_t* Kn) __attribute__((always_inline)) {
                weigh(t, i0.gone);
                i0 = i1;
                i1 = ids_of(t + 2);
                phase_end();
                __builtin_amdgcn_s_setprio(1);
                cw.products_scores(Vt, Kn, [](int) {});
                __builtin_amdgcn_s_setprio(0);
                phase_end();
            };
            for (int t = 0; t < n; t += 2) {
                turn(t, V0, K1);
                if (t + 1 < n) turn(t + 1, V1, K0);
            }
        }
    }
    cw.template put<false>(p, s, walk, hk, 0, n, 0, 1, cw.l_run + __shfl_xor(cw.l_run, 32, 64));
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
    RangeSum sum{p.scale_log2};
    sum.add_all<D>(0, 1, ranges, threadIdx.x % LANES, [&](int z) { return src + static_cast<size_t>(z) * W; });
    sum.put<BF16>(p.out + row * p.out_stride + (pair - row * p.nh) * D, threadIdx.x % LANES);
}

template <int D, bool BF16>
static hipError_t chunk_form(const PagedAttnDev& a, int groups, hipStream_t stream) {
    const dim3 grid(static_cast<uint32_t>(static_cast<int64_t>(a.items) * a.ranges * a.nkv));
    if constexpr (D == 128) {                                    // (heads of 64 have no wide form: plan_paged_attention)
        if (groups == 0) {
            hipLaunchKernelGGL((paged_wide_kernel<D, BF16>), grid, dim3(512), 0, stream, a);
            return hipGetLastError();
        }
    }
    if (groups == 2) hipLaunchKernelGGL((paged_chunk_kernel<D, BF16, false, 2>), grid, dim3(512), 0, stream, a);
    else if (a.ranges > 1) hipLaunchKernelGGL((paged_chunk_kernel<D, BF16, true, 1>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((paged_chunk_kernel<D, BF16, false, 1>), grid, dim3(256), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_paged_chunk(const PagedAttnDev& a, int groups, int d, int bf16, hipStream_t stream) {
    if (d == 128) return bf16 ? chunk_form<128, true>(a, groups, stream) : chunk_form<128, false>(a, groups, stream);
    return bf16 ? chunk_form<64, true>(a, groups, stream) : chunk_form<64, false>(a, groups, stream);
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
