// What the two paged attention kernels share: 16-bit types on the matrix cores, page loads that return zeros outside the keys, partial sums.
#pragma once
#include "paged.h"
#include "qtale_dev.h"

namespace qtale {

// Reference points of softmax sums are scores before their scale, so that the largest score less itself is zero whatever its size (scaled scores
// would be rounded first, and at 10^10 by more than an exponent has room for).  This one is a row's that has seen no key.
constexpr float kPagedNone = -3.0e38f;

// Probabilities are 2^(score - reference point + lift).  fp16 ends at 2^16 and has all its bits down to 2^-14 only: with the largest probability at 2^0
// those 15 nats below it, all of the output where its value is about zero, would keep a few bits or none, while the 32-bit denominator has them.
// So the largest is 2^lift when the reference point moves.  In the kernel for few columns that is free, and a score passes the reference point by
// kDecodeHead at most.  In chunks, where the sum of a lane's 32 probabilities has to stay below fp16's end, each power of two is room less for later
// scores, and more tiles move the reference point: us at lift 0 / 8 / 9 / 10 / 11, 4 x 4096 tokens, heads of 128, 576 / 585 / 582 / 591 / 606; 2 x 700 on
// 1400, heads of 64, 44.4 / 44.7 / 45.1 / 46.8 / 48.1.  A probability is then off by 2^-11 of itself (two terms: 2^-22), or by 2^-34 (2^-37) of the
// largest one if that is more.  bf16 has the exponents of 32 bits and no use for it.
template <bool BF16> constexpr float kDecodeLift = BF16 ? 0.0f : 12.0f;
template <bool BF16> constexpr float kChunkLift = BF16 ? 0.0f : 9.0f;
constexpr float kDecodeHead = 3.5f;

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

// Operands travel as 16-byte words whatever their type.
template <bool BF16>
struct Act16 {
    static __device__ __forceinline__ float16_t mfma32(const u32x4_t& a, const u32x4_t& b, const float16_t& c) {
        if constexpr (BF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
        else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ float4_t mfma16(const u32x4_t& a, const u32x4_t& b, const float4_t& c) {
        if constexpr (BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
        else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float x, float y) {      // nearest even, one instruction
        const float2_t v = {x, y};
        if constexpr (BF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
        else return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, half2_t));
    }
    static __device__ __forceinline__ float low(uint32_t w) { return act_to_float<BF16>(static_cast<uint16_t>(w & 0xffffu)); }
    static __device__ __forceinline__ float high(uint32_t w) {
        if constexpr (BF16) return __uint_as_float(w & 0xffff0000u);
        else return act_to_float<false>(static_cast<uint16_t>(w >> 16));
    }
};

// A buffer of `bytes` bytes from `base` on, both the same in every lane: loads past them return zeros and touch no memory.  (Named lane by
// lane, because what the compiler cannot see to be uniform it would load in a loop over the lanes' descriptors.)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void* base, int bytes) {
    const uint64_t a = reinterpret_cast<uint64_t>(base);
    const uint64_t lo = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(a))), hi = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(a >> 32)));
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(lo | hi << 32), 0, __builtin_amdgcn_readfirstlane(bytes), 0x00027000);
}

// Table row of a slot, read through the scalar cache (no kernel that reads it writes it).
struct PageRow {
    const QT_CONST_AS int32_t* row;
    int shift, last, n_pages;
    __device__ __forceinline__ PageRow(const PagedAttnDev& p, int slot)
        : row((const QT_CONST_AS int32_t*)(p.table + static_cast<size_t>(slot) * p.max_pages)), shift(p.shift), last(p.max_pages - 1), n_pages(p.n_pages) {}
    // page of a key (the same in every lane), -1 if there is none
    __device__ __forceinline__ int at(int key) const {
        const int page = row[__builtin_amdgcn_readfirstlane(min(key >> shift, last))];
        return page < n_pages ? page : -1;
    }
};

// What a launch has to know of a sequence: its rows, its slot's tokens, the place of its first row in the slot.
struct SeqView {
    int row0, n, slot, len, first;
    __device__ __forceinline__ SeqView(const PagedAttnDev& p, int b) {
        row0 = p.offs[b];
        n = max(p.offs[b + 1] - row0, 0);
        slot = p.slots ? p.slots[b] : b;
        const bool ok = static_cast<uint32_t>(slot) < static_cast<uint32_t>(p.n_slots);
        if (!ok) slot = 0;
        len = ok ? min(p.len[slot], p.max_len) : 0;
        first = p.first ? p.first[b] : (ok ? p.len[slot] : 0) - n;
    }
    // for a sequence that the whole wave works on: into scalar registers
    __device__ __forceinline__ void uniform() {
        row0 = __builtin_amdgcn_readfirstlane(row0);
        n = __builtin_amdgcn_readfirstlane(n);
        slot = __builtin_amdgcn_readfirstlane(slot);
        len = __builtin_amdgcn_readfirstlane(len);
        first = __builtin_amdgcn_readfirstlane(first);
    }
};

// One column by one wave on the vector ALUs, keys [key(s0), ...) of steps s0 .. s1 - 1, touching only keys that the column sees; lane l gets the
// numerators of columns (D / 64) l ..  For the rare column whose sum is not finite: the matrix products serve columns that see a key and columns
// that do not, and a masked key's probability of zero times an infinity or a NaN is NaN.  A finite sum has met neither, so it stands; one that
// is not is done again here.  (A load at a time for each key of each column, column after column: 4 x 4096 tokens, 32 heads of 128, take 0.59 ms, and 200 ms
// when every head holds a NaN that all rows see, some 900 cycles per key and column with eight waves on a CU.)
template <int D, bool BF16, int G>
__device__ void redo_column(const PagedAttnDev& p, const KeySteps<G>& walk, int slot, int hk, const uint16_t* q, int place, int s0, int s1, float lift,
                            float* num, float* m_out, float* l_out) {
    constexpr int E = D / 64;
    const int lane = threadIdx.x & 63;
    const int32_t* row = p.table + static_cast<size_t>(slot) * p.max_pages;
    auto at = [&](int page, int key) { return (((static_cast<size_t>(page) * p.nkv + hk) << p.shift) + (key & ((1 << p.shift) - 1))) * D; };
    float m = kPagedNone, l = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) num[e] = 0.0f;
#pragma unroll 1
    for (int st = s0; st < s1; ++st) {
        const int key = walk.key(st) + lane;
        int page = -1;
        if (lane < G && key <= place && key < walk.hi && (p.window == 0 || key > place - p.window || key < p.sinks)) page = row[min(key >> p.shift, p.max_pages - 1)];
        const bool seen = static_cast<uint32_t>(page) < static_cast<uint32_t>(p.n_pages);
        uint64_t who = __ballot(seen);
        if (who == 0) continue;
        float score = -INFINITY;
        if (seen) {
            const uint16_t* k = p.k + at(page, key);
            float sum = 0.0f;
#pragma unroll 1
            for (int e = 0; e < D; e += 2) {
                const uint32_t a = *reinterpret_cast<const uint32_t*>(k + e), b = *reinterpret_cast<const uint32_t*>(q + e);
                sum = fmaf(Act16<BF16>::low(a), Act16<BF16>::low(b), sum);
                sum = fmaf(Act16<BF16>::high(a), Act16<BF16>::high(b), sum);
            }
            score = sum;
        }
        const float m_new = fmaxf(m, wave_max(score)), alpha = __builtin_amdgcn_exp2f((m - m_new) * p.scale_log2);
        const float w = seen ? __builtin_amdgcn_exp2f(fmaf(score - m_new, p.scale_log2, lift)) : 0.0f;
        m = m_new;
        l = l * alpha + wave_sum(w);
#pragma unroll
        for (int e = 0; e < E; ++e) num[e] *= alpha;
#pragma unroll 1
        for (; who != 0; who &= who - 1) {
            const int j = __ffsll(static_cast<long long>(who)) - 1;
            const float wj = __shfl(w, j, 64);
            const uint16_t* v = p.v + at(__shfl(page, j, 64), walk.key(st) + j) + E * lane;
#pragma unroll
            for (int e = 0; e < E; ++e) num[e] = fmaf(wj, act_to_float<BF16>(v[e]), num[e]);
        }
    }
    *m_out = m;
    *l_out = l;
}

// A column's result, by one wave, lane l with columns (D / 64) l ..: to its place among the partial sums, or (none) to the output.
template <int D, bool BF16>
__device__ void put_column(const float* num, float m, float l, float* part, uint16_t* out) {
    constexpr int E = D / 64;
    const int lane = threadIdx.x & 63;
    if (part) {
#pragma unroll
        for (int e = 0; e < E; ++e) part[E * lane + e] = num[e];
        if (lane == 0) { part[D] = m; part[D + 1] = l; }
        return;
    }
    const float inv = l != 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) out[E * lane + e] = static_cast<uint16_t>(Act16<BF16>::pack(num[e] * inv, 0.0f) & 0xffffu);
}

// Sums of key ranges, 16 bytes per lane: lane l of D / 4 has columns 4 l .. 4 l + 3.
struct RangeSum {
    float sc, m = kPagedNone, den = 0.0f;        // sc: of scores, with log2(e)
    float4_t num = {0.f, 0.f, 0.f, 0.f};
    // adds N ranges at once (those with on[u]); the reference point of a range without keys lets it drop out
    template <int N>
    __device__ __forceinline__ void add(const float4_t* x, const float2_t* s, const bool* on) {
        float m_new = m;
#pragma unroll
        for (int u = 0; u < N; ++u) m_new = on[u] ? fmaxf(m_new, s[u][0]) : m_new;
        const float a = __builtin_amdgcn_exp2f((m - m_new) * sc);
        m = m_new;
        den *= a;
#pragma unroll
        for (int e = 0; e < 4; ++e) num[e] *= a;
#pragma unroll
        for (int u = 0; u < N; ++u) {
            if (!on[u]) continue;                                // (what was loaded in its place may be anything)
            const float f = __builtin_amdgcn_exp2f((s[u][0] - m) * sc);
            den += s[u][1] * f;
#pragma unroll
            for (int e = 0; e < 4; ++e) num[e] += x[u][e] * f;
        }
    }
    // ranges z0, z0 + step, ... < ranges; row_of(z): the sums of range z
    template <int D, class RowOf>
    __device__ __forceinline__ void add_all(int z0, int step, int ranges, int lane, RowOf row_of) {
        constexpr int N = 4;                                     // ranges whose loads are in flight together
        for (int z = z0; z < ranges; z += N * step) {
            float4_t x[N];
            float2_t s[N];
            bool on[N];
#pragma unroll
            for (int u = 0; u < N; ++u) {
                on[u] = z + u * step < ranges;
                const float* row = row_of(on[u] ? z + u * step : z);
                s[u] = *reinterpret_cast<const float2_t*>(row + D);
                x[u] = *reinterpret_cast<const float4_t*>(row + 4 * lane);
            }
            add<N>(x, s, on);
        }
    }
    template <bool BF16>
    __device__ __forceinline__ void put(uint16_t* out, int lane) const {
        const float inv = den != 0.0f ? 1.0f / den : 0.0f;       // a row that sees no key is zero
        u32x2_t w;
        w[0] = Act16<BF16>::pack(num[0] * inv, num[1] * inv);
        w[1] = Act16<BF16>::pack(num[2] * inv, num[3] * inv);
        *reinterpret_cast<u32x2_t*>(out + 4 * lane) = w;
    }
};

}  // namespace qtale
