// Attention of a chunk of new tokens over pages in 4 bits: columns, tiles of 64 keys and key ranges as in paged_prefill.hip, the products on codes.
//
// The waves of a workgroup unpack a tile together: codes less their zero point as fp16 multiples of 2^-24 (code bits 4 - 7: of 2^-20, with the 16 in the
// queries' elements or taken from the result), exact, into LDS, K as [key][d], V transposed as [column][key] in the order of the second product's
// operand, which the layout of a value page gives without permutations.  Scales stay outside the products:
//   score = s_j (q . (c_j - z_j)),   out = sum_j (p_j t_j) (c'_j - z'_j) / sum_j p_j.
// Queries are fp16; a row that is too large for it, or small, comes relative to its power of two.  Probabilities are 2^(score - m_ref + off): m_ref is a score
// (below 128: to a multiple of 2^-16), off = kChunkLift4 - log2 t_ref with a power of two t_ref above all t that the row has seen, so that p t fits fp16 whatever the values'
// size, for one multiplication; it is off by 2^-11 of itself or 2^-31 of the largest p times the largest t (but not where p is a power of two, as that of the
// score at m_ref is).  Mostly 32 bits hold m_ref - off exactly, and it goes in as one number; else, as for scores whose spacing is that of whole numbers, off
// goes in apart, an addition per score more.
//
// What bounds it: a wave has 449 vector instructions and 123 scalar ones per tile beside 32 MFMAs (counted, 4 x 4096 tokens; 16-bit pages: 163): nine for each of the
// eight words that it takes apart, 64 multiplications by scales, and their loads, exchanges and addresses.  4 x 4096 tokens, 32 heads on 8 of 128, 0.73 to 0.75 ms, 730
// to 755 TFLOP/s, after some 100 calls in a row (the first ones after a pause take up to 1.0: clocks; 16-bit pages 0.59 ms); 500 tokens on 24000 keys 273 us and 8 for
// the ranges' sums.  Unpacking the next tile behind the scores' products, which run on, instead of before them: 0.78 -> 0.72 ms.
// Eight waves on 256 columns whose halves take turns with the matrix cores and the vector ALUs, the best form for 16-bit pages, lose here, since the vector half
// takes more than twice the other's time: 0.83 ms, 2 x 300 tokens on 6000 keys 139 us instead of 117, heads of 64 4 x 4096 700 instead of 548.
#include <algorithm>

#include "paged4.h"
#include "paged_cols.h"

namespace qtale {

constexpr float kChunkLift4 = 9.0f;

__device__ __forceinline__ uint32_t less(uint32_t a, uint32_t b) {       // two fp16 numbers at once (exact here)
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2_t, a) - __builtin_bit_cast(half2_t, b));
}
// Eight codes less their zero points (z: two, as they lie in the operand): elements 2 i, 2 i + 1 are codes at bits 4 i and 16 + 4 i, those of odd i times 16.
__device__ __forceinline__ u32x4_t codes_less4(uint32_t w, uint32_t z) {
    const uint32_t y = w >> 8, z16 = z << 4;
    return u32x4_t{less(w & 0x000f000fu, z), less(w & 0x00f000f0u, z16), less(y & 0x000f000fu, z), less(y & 0x00f000f0u, z16)};
}
// A value that is to be made where it is used: what is derived from it is not kept in registers across the loop.
__device__ __forceinline__ int here(int x) {
    asm volatile("" : "+v"(x));
    return x;
}
// Where 16-byte chunk c of a row lies: at chunk c ^ swizzle, such that what a read or a write touches at a time spreads over the banks.
template <int D> __device__ __forceinline__ int k4_swizzle(int key) { return D == 128 ? key & 15 : (key >> 1) & 7; }
__device__ __forceinline__ int v4_swizzle(int col) { return ((col >> 1) ^ (col >> 4)) & 7; }

// A tile in LDS.
template <int D>
struct Tile4 {
    uint16_t* K;                 // [64 keys][D]
    uint16_t* V;                 // [D columns][64 keys]
    float *ks, *ts;              // scales of keys (with the softmax scale) and values
    uint32_t* tmax;              // the largest of 16 values each, as bits; their sign: some are no numbers
};

// Pages of tiles one after the other: a lane per 16 keys holds the page of sixteen tiles, the next sixteen's are on their way.
template <class Walk>
struct TileWalk {
    const PageRow& row;
    const Walk& walk;
    int t0, part, ids, later;
    uint64_t bad;
    __device__ __forceinline__ TileWalk(const PageRow& row, const Walk& walk, int t0, int part) : row(row), walk(walk), t0(t0), part(part), ids(0), later(read(0)), bad(0) {}
    __device__ __forceinline__ int read(int t) const {
        const int lane = threadIdx.x & 63;
        return row.row[min((walk.key(min(t0 + t + (lane >> 2), walk.steps - 1)) + 16 * (lane & 3)) >> row.shift, row.last)];
    }
    // the tile after the last call's
    __device__ __forceinline__ TilePages next(int t) {
        if ((t & 15) == 0) {
            ids = later;
            bad = __ballot(static_cast<uint32_t>(ids) >= static_cast<uint32_t>(row.n_pages));
            later = read(t + 16);
        }
        const int at = 4 * (t & 15), gone = __builtin_amdgcn_readfirstlane(static_cast<int>(bad >> at) & 15), page = __builtin_amdgcn_readlane(ids, at + part);
        return TilePages{gone >> part & 1 ? -1 : page, gone};
    }
};

// One wave's part of unpacking tiles: 16 keys, or 16 values, or both.
template <int D, bool BF16>
struct Unpack4 {
    static constexpr int S = D / 32;             // words of codes per lane
    typedef uint32_t Words __attribute__((ext_vector_type(S)));
    const PagedAttnDev& p;
    int hk, part, hi;
    uint32_t params_at, block;
    float unit;
    Words kw, vw;
    uint32_t kp;
    u32x4_t vp;

    __device__ __forceinline__ Unpack4(const PagedAttnDev& p, int hk, int part, int hi)
        : p(p), hk(hk), part(part), hi(hi), params_at(static_cast<uint32_t>(D / 2) << p.shift), block(params_at + (4u << p.shift)), unit(p.scale_log2 * 0x1p12f) {}
    static __device__ __forceinline__ Words load(__amdgpu_buffer_rsrc_t buf, uint32_t off, uint32_t base) {
        if constexpr (S == 4) return __builtin_amdgcn_raw_buffer_load_b128(buf, off, base, 0);
        else return __builtin_amdgcn_raw_buffer_load_b64(buf, off, base, 0);
    }
    // the head's block of a page; of one that is gone: an empty buffer, zeros
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const uint16_t* pool, int page) const {
        page = __builtin_amdgcn_readfirstlane(page);
        return buffer_of(reinterpret_cast<const char*>(pool) + (static_cast<size_t>(max(page, 0)) * p.nkv + hk) * block, page < 0 ? 0 : static_cast<int>(block));
    }
    // key0: the tile's first
    __device__ __forceinline__ void request_keys(int key0, int page) {
        const int lane = threadIdx.x & 63;
        const uint32_t t = __builtin_amdgcn_readfirstlane((key0 + 16 * part) & ((1 << p.shift) - 1));
        const auto buf = buffer(p.k, page);
        kw = load(buf, (lane >> 2) * (D / 2) + (lane & 3) * (D / 8), t * (D / 2));
        kp = __builtin_amdgcn_raw_buffer_load_b32(buf, 4 * (lane >> 2), params_at + 4 * t, 0);
    }
    __device__ __forceinline__ void request_values(int key0, int page) {
        const int lane = threadIdx.x & 63;
        const uint32_t t = __builtin_amdgcn_readfirstlane((key0 + 16 * part) & ((1 << p.shift) - 1));
        const auto buf = buffer(p.v, page);
        vw = load(buf, (lane >> 4) * (2 * D) + (lane & 15) * (D / 8), t * (D / 2));
        vp = __builtin_amdgcn_raw_buffer_load_b128(buf, 16 * (lane >> 4), params_at + 4 * t, 0);
    }
    // Places from `hi` on get scales of zero (what lies in unused places may be anything, zero points too).
    __device__ __forceinline__ void put_keys(int key0, const Tile4<D>& to) const {
        const int lane = threadIdx.x & 63, key = 16 * part + (lane >> 2);
        const uint32_t zz = __builtin_amdgcn_perm(kp, kp, 0x07060706u) & 0x000f000fu;
        const int at = here(key * D + ((S * (lane & 3)) ^ k4_swizzle<D>(key)) * 8);   // of the lane's first chunk; chunk w: w flipped in
#pragma unroll
        for (int w = 0; w < S; ++w) *reinterpret_cast<u32x4_t*>(&to.K[at ^ (8 * w)]) = codes_less4(kw[w], zz);
        if ((lane & 3) == 0) to.ks[key] = key0 + key < hi ? act_to_float<BF16>(static_cast<uint16_t>(kp & 0xffffu)) * unit : 0.0f;
    }
    __device__ __forceinline__ void put_values(int key0, const Tile4<D>& to) const {
        const int lane = threadIdx.x & 63, four = lane >> 4, c = lane & 15;
        float4_t t4;
        uint32_t big = 0;                                        // (numbers without their sign compare as their bits do)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            t4[r] = key0 + 16 * part + 4 * four + r < hi ? act_to_float<BF16>(static_cast<uint16_t>(vp[r] & 0xffffu)) : 0.0f;
            const uint32_t u = __float_as_uint(t4[r]) & 0x7fffffffu;
            big = max(big, u);
        }
        if (c == 0) *reinterpret_cast<float4_t*>(&to.ts[16 * part + 4 * four]) = t4;
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) most = max(most, static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(big), 16 * i)));
        if (most >= 0x7f800000u) {                               // some are no numbers: the largest of the others, and a mark
            big = 0;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const uint32_t u = __float_as_uint(t4[r]) & 0x7fffffffu;
                big = max(big, u < 0x7f800000u ? u : 0u);
            }
            most = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) most = max(most, static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(big), 16 * i)));
            most |= 0x80000000u;
        }
        if (lane == 0) to.tmax[part] = most;
        const uint32_t z01 = __builtin_amdgcn_perm(vp[1], vp[0], 0x07060302u) & 0x000f000fu, z23 = __builtin_amdgcn_perm(vp[3], vp[2], 0x07060302u) & 0x000f000fu;
        // tokens 4 four .. + 3 of 16: chunk 2 part + (four & 1) of a column's row, its half four >> 1 (of the lane's columns, D / 16 from a multiple of that on,
        // the swizzle is the first one's with half of what is added flipped in)
        const int first = (D / 16) * c;
        const int at = here(first * kTileKeys + (((2 * part + (four & 1)) ^ v4_swizzle(first)) * 8) + 4 * (four >> 1));
#pragma unroll
        for (int h = 0; h < S / 2; ++h) {
            const u32x4_t a = codes_less4(vw[2 * h], z01), b = codes_less4(vw[2 * h + 1], z23);
#pragma unroll
            for (int i = 0; i < 4; ++i) *reinterpret_cast<u32x2_t*>(&to.V[(at ^ (8 * (2 * h + (i >> 1)))) + (4 * h + i) * kTileKeys]) = u32x2_t{a[i], b[i]};
        }
    }
};

// One wave's 32 columns: their queries, scores of a tile, probabilities and sums.
template <int D, bool BF16>
struct Columns4 {
    using H = Act16<false>;
    static constexpr int KS = D / 16;            // k-steps of the scores
    static constexpr int DF = D / 32;            // output fragments
    static constexpr int PV = 4 * DF, ALL = PV + 2 * KS;
    int qi, head, place, reach;                  // this lane's column (clamped to a live one): query, head, its place, keys after `reach` are in its window
    bool mine;                                   // the lane's column exists
    int whole_from, whole_to, first_to;          // a tile that every query of the wave sees whole begins in whole_from .. whole_to, or not after first_to
    u32x4_t qf[KS], pf[4];
    float up;                                    // the power of two that a score's unit stands for, with half of the codes' 2^24 (keys' scales have the other)
    int k_at[KS], v_at[4];                       // LDS elements that this lane reads
    float16_t st[2], o[DF];
    float m_ref, l_run, off;
    bool far;                                    // some row's m_ref - off is not exact (the same in all lanes)

    // columns .. c_hi; c0: the wave's first
    __device__ __forceinline__ Columns4(const PagedAttnDev& p, const SeqView& s, int hk, int c0, int c_hi, int hi) {
        const int lane = threadIdx.x & 63, l32 = lane & 31, lhi = lane >> 5;
        const int col = min(c0 + l32, c_hi);
        qi = col / p.rep;
        head = hk * p.rep + col - qi * p.rep;
        place = s.first + qi;
        reach = p.window > 0 ? place - p.window : INT32_MIN;
        mine = c0 + l32 <= c_hi;
        // (divisions run on the vector ALUs)
        whole_to = min(s.first + __builtin_amdgcn_readfirstlane(min(c0, c_hi) / p.rep) + 1, hi) - kTileKeys;
        whole_from = p.window > 0 ? s.first + __builtin_amdgcn_readfirstlane(min(c0 + 31, c_hi) / p.rep) - p.window + 1 : 0;
        first_to = p.sinks - kTileKeys;
        const uint16_t* qrow = p.q + (s.row0 + qi) * p.q_stride + head * D + 8 * lhi;
        float big = 0.0f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            qf[k] = *reinterpret_cast<const u32x4_t*>(qrow + 16 * k);
#pragma unroll
            for (int w = 0; w < 4; ++w) big = fmaxf(big, fmaxf(fabsf(Act16<BF16>::low(qf[k][w])), fabsf(Act16<BF16>::high(qf[k][w]))));
        }
        big = fmaxf(big, __shfl_xor(big, 32, 64));
        // (elements of a row between 2^-4 and 2^15 at its largest: a sixteenth of one that is 2^-6 of the largest still has all its bits)
        const int e = static_cast<int>(__float_as_uint(big) >> 23) - 127, move = e >= 15 || e < -4 ? 13 - min(max(e, -100), 127) : 0;
        const float f = ldexpf(1.0f, move), f16 = f * 0.0625f;
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int w = 0; w < 4; ++w) qf[k][w] = H::pack(Act16<BF16>::low(qf[k][w]) * (w & 1 ? f16 : f), Act16<BF16>::high(qf[k][w]) * (w & 1 ? f16 : f));
        up = ldexpf(1.0f, 12 - move);
        // chunk 2 k + lhi of key l32; chunk 2 s2 + lhi of column 32 f + l32: v_at[(f ^ s2) & 3] + 32 f rows (the swizzle of that column is l32's with 2 f
        // flipped in)
#pragma unroll
        for (int k = 0; k < KS; ++k) k_at[k] = l32 * D + (((2 * k + lhi) ^ k4_swizzle<D>(l32)) * 8);
#pragma unroll
        for (int x = 0; x < 4; ++x) v_at[x] = l32 * kTileKeys + (((2 * x + lhi) ^ v4_swizzle(l32)) * 8);
#pragma unroll
        for (int f = 0; f < DF; ++f)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[f][r] = 0.0f;
        m_ref = kPagedNone;
        l_run = 0.0f;
        off = kChunkLift4 + 60.0f;
        far = false;
    }

    // m_ref - off is exact: what its subtraction lost (|off| <= 120; below 128 nothing is lost) is zero.
    __device__ __forceinline__ bool near() const { return (m_ref - (m_ref - off)) - off == 0.0f; }

    __device__ __forceinline__ u32x4_t operand(const uint16_t* V, const uint16_t* K, int i) const {
        if (i < PV) {
            const int s2 = i / DF, f = i % DF;
            return *reinterpret_cast<const u32x4_t*>(&V[32 * f * kTileKeys + v_at[(f ^ s2) & 3]]);
        }
        return *reinterpret_cast<const u32x4_t*>(&K[((i - PV) & 1) * 32 * D + k_at[(i - PV) >> 1]]);
    }
    // Products FROM .. ALL - 1 of O^T += V^T P^T of one tile, then S^T = K Q^T of the next; operands read AHEAD products before their use.
    template <int FROM, int TO>
    __device__ __forceinline__ void products(const uint16_t* V, const uint16_t* K) {
        constexpr int AHEAD = 6;
        u32x4_t x[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) x[i] = operand(V, K, FROM + i);
        if (TO > PV) {
#pragma unroll
            for (int kf = 0; kf < 2; ++kf)
#pragma unroll
                for (int r = 0; r < 16; ++r) st[kf][r] = 0.0f;
        }
#pragma unroll
        for (int i = FROM; i < TO; ++i) {
            const u32x4_t now = x[(i - FROM) % AHEAD];
            if (i < PV) o[i % DF] = H::mfma32(now, pf[i / DF], o[i % DF]);
            else st[(i - PV) & 1] = H::mfma32(now, qf[(i - PV) >> 1], st[(i - PV) & 1]);
            if (i + AHEAD < TO) x[(i - FROM) % AHEAD] = operand(V, K, i + AHEAD);
            __builtin_amdgcn_sched_barrier(0);
        }
    }

    // Keys' scales of the first half of a tile and the largest of the values': asked for together; the others follow as these are used.
    struct Scales { float4_t k[4]; u32x4_t most; };
    __device__ __forceinline__ Scales scales(const Tile4<D>& tile) const {
        const int quad = here(4 * ((threadIdx.x & 63) >> 5));
        Scales x;
        x.most = *reinterpret_cast<const u32x4_t*>(tile.tmax);
#pragma unroll
        for (int i = 0; i < 4; ++i) x.k[i] = *reinterpret_cast<const float4_t*>(&tile.ks[quad + 8 * i]);
        __builtin_amdgcn_sched_barrier(0);
        return x;
    }
    // Probabilities of keys key0 .. key0 + 63, times their values' scales, as operands; gone: bit per 16 keys without a page.
    __device__ __forceinline__ void softmax(const PagedAttnDev& p, const Tile4<D>& tile, Scales& x, int key0, int gone, int hi) {
        key0 = __builtin_amdgcn_readfirstlane(key0);
        gone = __builtin_amdgcn_readfirstlane(gone);
        const int quad = here(4 * ((threadIdx.x & 63) >> 5));
        const float* ks = tile.ks + quad;
        const float* ts = tile.ts + quad;
        uint32_t most = 0, odds = 0;                             // the largest scale of a value; the sign's bit: some are no numbers
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t u = __builtin_amdgcn_readfirstlane(x.most[i]);
            most = max(most, u & 0x7fffffffu);
            odds |= u;
        }
        const bool odd = (odds >> 31) != 0;
        // products -> scores (in units of `up`)
#pragma unroll
        for (int g = 0; g < 8; ++g) {
            const float4_t k4 = x.k[g & 3];
            x.k[g & 3] = *reinterpret_cast<const float4_t*>(g < 4 ? ks + 8 * (g + 4) : ts + 8 * (g - 4));
#pragma unroll
            for (int r = 0; r < 4; ++r) st[g >> 2][4 * (g & 3) + r] *= k4[r];
            __builtin_amdgcn_sched_barrier(0);
        }
        // A tile that every query of the wave sees whole needs no mask.
        const bool all = (gone == 0) & (key0 <= whole_to) & ((key0 >= whole_from) | (key0 <= first_to));
        if (!all) {
            // of the lane's keys, key0 + quad + a constant each: constants up to `last` that are after `before`, or below `stay`
            const int last = min(place, hi - 1) - key0 - quad, before = max(reach, -1) - key0 - quad, stay = p.sinks - key0 - quad;
#pragma unroll
            for (int kf = 0; kf < 2; ++kf)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int at = kf * 32 + 8 * (r >> 2) + (r & 3);
                    const bool seen = (at <= last) & ((gone >> (kf * 2 + (r >> 3)) & 1) == 0) & ((at > before) | (at < stay));
                    st[kf][r] = seen ? st[kf][r] : -INFINITY;
                    if (r & 1) __builtin_amdgcn_sched_barrier(0);   // (few masks at a time)
                }
        }
        float mx = -INFINITY;
#pragma unroll
        for (int kf = 0; kf < 2; ++kf)
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, st[kf][r]);
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * up;
        // The reference point stays as long as no probability passes 2^15 t_ref^-1 and no value's scale t_ref.  It moves so that the largest probability is about
        // 2^kChunkLift4 t_ref^-1, and t_ref to the next power of two but one.
        auto room = [](uint32_t t) { return kChunkLift4 + 127.0f - static_cast<float>(t >> 23); };   // of `off`: with less than 1 left such a scale may pass t_ref
        if (__any((mx - m_ref > 15.0f - kChunkLift4) | (room(most) < off + 1.0f))) {
            if (!all && __any(room(most) < off + 1.0f)) {        // the largest scale that the row sees (others may be anything)
                most = 0;
#pragma unroll
                for (int kf = 0; kf < 2; ++kf)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const uint32_t t = __float_as_uint(ts[kf * 32 + 8 * (r >> 2) + (r & 3)]) & 0x7fffffffu;
                        most = max(most, ((st[kf][r] > -INFINITY) & (t < 0x7f800000u)) ? t : 0u);
                    }
                most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), 32, 64)));
            }
            const float m_new = fmaxf(m_ref, fabsf(mx) < 128.0f ? rintf(mx * 0x1p16f) * 0x1p-16f : mx), off_new = room(most) < off + 1.0f ? room(most) - 2.0f : off;
            rescale(__builtin_amdgcn_exp2f((m_ref - m_new) + (off_new - off)));
            off = off_new;
            m_ref = m_new;
            far = __any(!near() & (m_ref > kPagedNone));
        }
        if (odd | far) weigh<true>(x, ts);
        else weigh<false>(x, ts);
    }
    // Scores -> probabilities, times their values' scales, as operands; the probabilities' sum.  ODD: m_ref and off apart, and a scale may be no number: a key
    // that is not seen then takes no part.
    template <bool ODD>
    __device__ __forceinline__ void weigh(Scales& x, const float* ts) {
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        const float m = ODD ? m_ref : m_ref - off;
#pragma unroll
        for (int g = 0; g < 8; ++g) {
            const float4_t t4 = x.k[g & 3];
            if (g < 4) x.k[g] = *reinterpret_cast<const float4_t*>(ts + 8 * (g + 4));
            const int kf = g >> 2, q4 = g & 3;
#pragma unroll
            for (int r = 0; r < 4; r += 2) {
                float w[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float at = fmaf(st[kf][4 * q4 + r + i], up, -m), e = __builtin_amdgcn_exp2f(ODD ? at + off : at);
                    sum[q4] += e;
                    w[i] = ODD && at == -INFINITY ? 0.0f : e * t4[r + i];
                }
                pf[kf * 2 + (q4 >> 1)][2 * (q4 & 1) + (r >> 1)] = H::pack(w[0], w[1]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        l_run += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    }
    __device__ __forceinline__ void rescale(float by) {
        l_run *= by;
#pragma unroll
        for (int f = 0; f < DF; ++f)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[f][r] *= by;
    }

    // Results: to the output, or (SPLIT, several ranges) among the sums of range z.  (Odd columns' codes were times 16.)
    template <bool SPLIT>
    __device__ __forceinline__ void put(const PagedAttnDev& p, const SeqView& s, int z, int ranges) {
        const int lhi = (threadIdx.x & 63) >> 5;
        const float l_tot = l_run + __shfl_xor(l_run, 32, 64);
        if (!mine) return;
        if (SPLIT) {
            float* dst = p.part + ((static_cast<size_t>(s.row0 + qi) * p.nh + head) * p.ranges + z) * part_stride(D);
            if (lhi == 0) dst[D + 2] = static_cast<float>(ranges);
            if (ranges > 1) {
                // `off` goes into the reference point, or (not exact there) into the sums
                const bool whole = near();
                const float by = whole ? 1.0f : __builtin_amdgcn_exp2f(-off);
#pragma unroll
                for (int f = 0; f < DF; ++f)
#pragma unroll
                    for (int q4 = 0; q4 < 4; ++q4)
                        *reinterpret_cast<float4_t*>(dst + f * 32 + 8 * q4 + 4 * lhi) =
                            float4_t{o[f][4 * q4] * 0x1p24f * by, o[f][4 * q4 + 1] * 0x1p20f * by, o[f][4 * q4 + 2] * 0x1p24f * by, o[f][4 * q4 + 3] * 0x1p20f * by};
                if (lhi == 0) *reinterpret_cast<float2_t*>(dst + D) = float2_t{whole ? m_ref - off : m_ref, l_tot * by};
                return;
            }
        }
        const float inv = l_tot != 0.0f ? 1.0f / l_tot : 0.0f;   // (l_tot may be 2^-120); a row that sees no key is zero
        uint16_t* orow = p.out + (s.row0 + qi) * p.out_stride + head * D;
#pragma unroll
        for (int f = 0; f < DF; ++f)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                u32x2_t w;
                w[0] = Act16<BF16>::pack(o[f][4 * q4] * inv * 0x1p24f, o[f][4 * q4 + 1] * inv * 0x1p20f);
                w[1] = Act16<BF16>::pack(o[f][4 * q4 + 2] * inv * 0x1p24f, o[f][4 * q4 + 3] * inv * 0x1p20f);
                *reinterpret_cast<u32x2_t*>(orow + f * 32 + 8 * q4 + 4 * lhi) = w;
            }
    }
};

// The tiles of an item that this workgroup walks, and how many ranges the item has.
struct Range4 { int t0, t1, ranges; };
__device__ __forceinline__ Range4 range_of(const PagedAttnDev& p, int steps, int z) {
    // ranges of about equal length over the whole call, as many as are to run at once; no item is cut into more than p.ranges
    const int lane = threadIdx.x & 63;
    int work = 0;
    for (int b0 = 0; b0 < p.B; b0 += 64) work += b0 + lane < p.B ? chunk_work(p, b0 + lane) : 0;
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) work += __shfl_xor(work, x, 64);
    const int wanted = max(p.target / p.nkv, 1);
    const int per = __builtin_amdgcn_readfirstlane(max(max((work + wanted - 1) / wanted, (steps + p.ranges - 1) / p.ranges), 4));
    const int ranges = __builtin_amdgcn_readfirstlane(max((steps + per - 1) / per, 1));
    return Range4{z * per, min(z * per + per, steps), ranges};
}

// Four waves, 128 columns.  Tile t + 1 is unpacked and tile t + 2 requested while tile t is computed; one barrier per tile, two workgroups per CU.
template <int D, bool BF16, bool SPLIT>
__global__ void __launch_bounds__(256, 2)
paged4_chunk_kernel(PagedAttnDev p) {
    using Cols = Columns4<D, BF16>;
    constexpr int TILE = kTileKeys * D;
    __shared__ __attribute__((aligned(1024))) uint16_t Ks[2][TILE], Vs[2][TILE];
    __shared__ __attribute__((aligned(16))) float ks[2][kTileKeys], ts[2][kTileKeys];
    __shared__ __attribute__((aligned(16))) uint32_t tmax[2][4];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

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
    Range4 range{0, walk.steps, 1};
    if (SPLIT) range = range_of(p, walk.steps, z);
    if (SPLIT && z >= range.ranges) return;
    Cols cw(p, s, hk, c_lo + 32 * wave, c_hi, walk.hi);
    const PageRow pages(p, s.slot);
    Unpack4<D, BF16> un(p, hk, wave, walk.hi);
    const int t0 = range.t0, t1 = range.t1;
    auto tile = [&](int t) __attribute__((always_inline)) {
        const int i = (t - t0) & 1;
        return Tile4<D>{Ks[i], Vs[i], ks[i], ts[i], tmax[i]};
    };
    auto request = [&](int t, int page) __attribute__((always_inline)) {
        if (t >= t1) page = -1;
        un.request_keys(walk.key(t), page);
        un.request_values(walk.key(t), page);
    };
    auto unpack = [&](int t) __attribute__((always_inline)) {
        un.put_keys(walk.key(t), tile(t));
        un.put_values(walk.key(t), tile(t));
    };
    if (t0 < t1) {
        TileWalk ids(pages, walk, t0, wave);
        TilePages i0 = ids.next(0), i1 = ids.next(1), i2 = ids.next(2);
        request(t0, i0.page);
        unpack(t0);
        request(t0 + 1, i1.page);
        for (int t = t0; t < t1; ++t) {
            __syncthreads();                                     // tile t is in LDS, and the other buffers have been read
            const Tile4<D> now = tile(t);
            cw.template products<Cols::PV, Cols::ALL>(now.V, now.K);
            if (t + 1 < t1) unpack(t + 1);
            request(t + 2, i2.page);
            typename Cols::Scales sc = cw.scales(now);
            cw.softmax(p, now, sc, walk.key(t), i0.gone, walk.hi);
            cw.template products<0, Cols::PV>(now.V, now.K);
            i0 = i1;
            i1 = i2;
            i2 = ids.next(t + 3 - t0);
        }
    }
    cw.template put<SPLIT>(p, s, z, range.ranges);
}

template <int D, bool BF16>
static hipError_t chunk4_form(const PagedAttnDev& a, hipStream_t stream) {
    const dim3 grid(static_cast<uint32_t>(static_cast<int64_t>(a.items) * a.ranges * a.nkv));
    if (a.ranges > 1) hipLaunchKernelGGL((paged4_chunk_kernel<D, BF16, true>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((paged4_chunk_kernel<D, BF16, false>), grid, dim3(256), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_paged4_chunk(const PagedAttnDev& a, int d, hipStream_t stream) {
    if (d == 128) return a.bf16 ? chunk4_form<128, true>(a, stream) : chunk4_form<128, false>(a, stream);
    return a.bf16 ? chunk4_form<64, true>(a, stream) : chunk4_form<64, false>(a, stream);
}

}  // namespace qtale
