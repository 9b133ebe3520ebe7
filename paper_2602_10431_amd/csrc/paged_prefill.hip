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

constexpr int kTileKeys = 64;

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

template <int D, bool BF16, bool SPLIT>
__global__ void __launch_bounds__(256, 2)
paged_chunk_kernel(PagedAttnDev p) {
    using A = Act16<BF16>;
    constexpr int KS = D / 16;                   // k-steps of the scores
    constexpr int DF = D / 32;                   // output fragments
    constexpr int CPR = D / 8;                   // 16-byte chunks of a row
    constexpr int RPF = 64 / CPR;                // rows per fetch instruction (1 KB)
    constexpr int NF = 16 / RPF;                 // fetch instructions per wave for 16 keys
    __shared__ __attribute__((aligned(1024))) uint16_t K0[kTileKeys * D], K1[kTileKeys * D], V0[kTileKeys * D], V1[kTileKeys * D];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
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
        const int per = __builtin_amdgcn_readfirstlane(max((walk.steps + p.ranges - 1) / p.ranges, 4));
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
        // page ids are read a tile before the fetch that uses them
        Ids now = ids_of(t0), next = ids_of(t0 + 1);
        fetch(t0, now.page, K0, V0);
        auto turn = [&](int t, uint16_t* K, uint16_t* V, uint16_t* K_next, uint16_t* V_next) {
            __builtin_amdgcn_s_waitcnt(0x0f70);                  // vmcnt(0): this wave's part of the tile is in LDS
            __syncthreads();                                     // everybody's is, and the other buffers have been read
            if (t + 1 < t1) fetch(t + 1, next.page, K_next, V_next);
            const int gone = now.gone;
            now = next;
            next = ids_of(t + 2);
            if (wave_live && walk.key(t) <= w_last) compute(t, gone, K, V);
        };
        for (int t = t0; t < t1; t += 2) {
            turn(t, K0, V0, K1, V1);
            if (t + 1 < t1) turn(t + 1, K1, V1, K0, V0);
        }
    }

    const float l_tot = l_run + __shfl_xor(l_run, 32, 64);
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
        put_column<D, BF16>(p, s.row0 + qj, hj, z, ranges, num, m, l);
    }
    if (c_lo + wave * 32 + l32 > c_hi) return;
    const bool done = (redo >> l32 & 1) != 0;
    const size_t pair = static_cast<size_t>(s.row0 + qi) * p.nh + head;
    if (SPLIT && ranges > 1) {
        float* dst = p.part + (pair * p.n_split + z) * part_stride(D);
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
    if (SPLIT && lhi == 0) p.part[pair * p.n_split * part_stride(D) + D + 2] = 1.0f;
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

// CUs of the current device (queried once per device).
static int device_cus() {
    static int cus[64] = {0};
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
    if (cus[dev] == 0) {
        int n = 0;
        if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) n = 256;
        cus[dev] = n;
    }
    return cus[dev];
}

PagedAttnPlan plan_paged_attention(int nh, int nkv, int d, int T, int B, int max_new, int max_len) {
    PagedAttnPlan l{};
    const int rep = nh / nkv, cus = device_cus();
    const int64_t most = static_cast<int64_t>(max_new) * rep;
    // a sequence of few columns has a kernel of its own; both run where the call may hold sequences of either kind
    l.chunk = most > kDecodeCols;
    l.decode = !l.chunk || (static_cast<int64_t>(T) < static_cast<int64_t>(B) * max_new && rep <= kDecodeCols);
    const int live = std::min(B, T);
    l.items = static_cast<int>((static_cast<int64_t>(T) * rep + static_cast<int64_t>(kChunkCols - 1) * live) / kChunkCols);
    l.decode_split = l.chunk_split = 1;
    if (l.decode) {
        l.target = 3 * cus;
        if (static_cast<int64_t>(B) * nkv < 2 * cus) {
            const int ranges = (max_len + kDecodeRangeKeys - 1) / kDecodeRangeKeys;
            l.decode_split = std::max(std::min({ranges, (l.target + nkv - 1) / nkv, 64}), 1);
        }
    }
    if (l.chunk) {
        const int64_t wgs = std::max<int64_t>(static_cast<int64_t>(l.items) * nkv, 1);
        const int tiles = (max_len + kTileKeys - 1) / kTileKeys;
        if (wgs < 2 * cus) l.chunk_split = static_cast<int>(std::max<int64_t>(std::min<int64_t>({(2 * cus + wgs - 1) / wgs, tiles / 8, 32}), 1));
    }
    const int split = std::max(l.decode_split, l.chunk_split);
    l.too_large = (static_cast<int64_t>(T) * rep + static_cast<int64_t>(kChunkCols - 1) * live) / kChunkCols * nkv * l.chunk_split > INT32_MAX ||
                  static_cast<int64_t>(T) * nh > INT32_MAX;
    l.bytes = 256 + (split > 1 ? static_cast<size_t>(T) * nh * split * part_stride(d) * 4 : 0);
    return l;
}

template <int D, bool BF16>
static hipError_t chunk_form(const PagedAttnDev& a, hipStream_t stream) {
    const bool split = a.n_split > 1;
    const int64_t items = static_cast<int64_t>(a.items) * a.ranges;
    const dim3 grid(static_cast<uint32_t>(items * a.nkv)), block(256);
    if (split) hipLaunchKernelGGL((paged_chunk_kernel<D, BF16, true>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((paged_chunk_kernel<D, BF16, false>), grid, block, 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_paged_chunk(const PagedAttnDev& a, int d, int bf16, hipStream_t stream) {
    if (d == 128) return bf16 ? chunk_form<128, true>(a, stream) : chunk_form<128, false>(a, stream);
    return bf16 ? chunk_form<64, true>(a, stream) : chunk_form<64, false>(a, stream);
}

hipError_t launch_paged_attention(PagedAttnDev a, const PagedAttnPlan& plan, int d, int bf16, int T, float* workspace, hipStream_t stream) {
    // both kernels number their ranges in the same partial sums
    a.n_split = std::max(plan.decode_split, plan.chunk_split);
    a.items = plan.items;
    a.take = plan.decode && plan.chunk;
    a.part = workspace;
    hipError_t e = hipSuccess;
    a.ranges = plan.decode_split;
    a.target = plan.decode_split > 1 ? plan.target : 0;
    if (plan.decode && (e = launch_paged_decode(a, d, bf16, stream)) != hipSuccess) return e;
    a.ranges = plan.chunk_split;
    if (plan.chunk && (e = launch_paged_chunk(a, d, bf16, stream)) != hipSuccess) return e;
    return a.n_split > 1 ? launch_paged_combine(a, d, bf16, T, stream) : e;
}

}  // namespace qtale
