// Attention of a chunk of new tokens over pages in 4 bits: columns, tiles of 64 keys and key ranges as in paged_prefill.hip, the products on codes.
//
// The waves of a workgroup unpack a tile together: codes less their zero point as fp16 multiples of 2^-24 (code bits 4 - 7: of 2^-20, with the 16 in the
// queries' elements or taken from the result), exact, into LDS, K as [key][d], V transposed as [column][key] in the order of the second product's
// operand, which the layout of a value page gives without permutations.  Tile t + 1 is unpacked and tile t + 2 requested while tile t is
// computed; one barrier per tile.  Scales stay outside the products:
//   score = s_j (q . (c_j - z_j)),   out = sum_j (p_j t_j) (c'_j - z'_j) / sum_j p_j.
// Queries are fp16 relative to their row's power of two.  Probabilities are 2^(score - m_run), where m_run holds the reference point, the lift
// (kChunkLift) and log2 of t_ref, a power of two above all t so far: so p t fits fp16 whatever the values' size, for one multiplication.
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
template <int D> __device__ __forceinline__ int k4_swizzle(int key) { return D == 128 ? key & 15 : (key >> 1) & 7; }
__device__ __forceinline__ int v4_swizzle(int col) { return ((col >> 1) ^ (col >> 4)) & 7; }

// NW waves of 32 columns.  SPLIT: key ranges.
template <int D, bool BF16, bool SPLIT, int NW>
__global__ void __launch_bounds__(64 * NW, 2)
paged4_chunk_kernel(PagedAttnDev p) {
    using H = Act16<false>;
    constexpr int KS = D / 16;                   // k-steps of the scores
    constexpr int DF = D / 32;                   // output fragments
    constexpr int S = D / 32;                    // words of codes per lane
    constexpr int COLS = 32 * NW, TILE = kTileKeys * D;
    typedef uint32_t Words __attribute__((ext_vector_type(S)));
    __shared__ __attribute__((aligned(1024))) uint16_t Ks[2][TILE], Vs[2][TILE];
    __shared__ __attribute__((aligned(16))) float ks[2][kTileKeys], ts[2][kTileKeys], tmax[2][4];   // scales of keys and values, largest of 16 values each

    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, lhi = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), part = wave & 3;   // part: which 16 keys of a tile this wave unpacks

    int hk, item, z = 0, b, qt;
    find_head(p, &hk, &item);
    if (SPLIT) {
        z = __builtin_amdgcn_readfirstlane(item / p.items);
        item -= z * p.items;
    }
    if (!find_columns<COLS>(p, item, &b, &qt)) return;
    SeqView s(p, b);
    s.uniform();
    const int c_lo = qt * COLS, c_hi = min(c_lo + COLS, s.n * p.rep) - 1;   // this workgroup's columns
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
    // this lane's column (clamped to a live one): query, head, its place, keys after `reach` are in its window
    const int col = min(c_lo + 32 * wave + l32, c_hi), qi = col / p.rep, head = hk * p.rep + col - qi * p.rep;
    const int place = s.first + qi, reach = p.window > 0 ? place - p.window : INT32_MIN;
    const bool mine = c_lo + 32 * wave + l32 <= c_hi;
    const int w_first = s.first + __builtin_amdgcn_readfirstlane(min(c_lo + 32 * wave, c_hi) / p.rep);   // places of the wave's queries
    const int w_last = s.first + __builtin_amdgcn_readfirstlane(min(c_lo + 32 * wave + 31, c_hi) / p.rep);

    // queries as fp16, the row's largest at 2^13; up: the power of two that a score's unit stands for
    u32x4_t qf[KS];
    float up;
    {
        const uint16_t* qrow = p.q + (s.row0 + qi) * p.q_stride + head * D + 8 * lhi;
        float big = 0.0f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            qf[k] = *reinterpret_cast<const u32x4_t*>(qrow + 16 * k);
#pragma unroll
            for (int w = 0; w < 4; ++w) big = fmaxf(big, fmaxf(fabsf(Act16<BF16>::low(qf[k][w])), fabsf(Act16<BF16>::high(qf[k][w]))));
        }
        big = fmaxf(big, __shfl_xor(big, 32, 64));
        const int e = min(max(static_cast<int>(__float_as_uint(big) >> 23) - 127, -100), 127);
        const float f = ldexpf(1.0f, 13 - e), f16 = f * 0.0625f;
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int w = 0; w < 4; ++w) qf[k][w] = H::pack(Act16<BF16>::low(qf[k][w]) * (w & 1 ? f16 : f), Act16<BF16>::high(qf[k][w]) * (w & 1 ? f16 : f));
        up = ldexpf(1.0f, e - 13);
    }
    const float unit = p.scale_log2 * 0x1p24f;

    // LDS elements that this lane reads: chunk 2 k + lhi of key l32; chunk 2 s2 + lhi of column l32 of a fragment
    int k_at[KS];
#pragma unroll
    for (int k = 0; k < KS; ++k) k_at[k] = l32 * D + (((2 * k + lhi) ^ k4_swizzle<D>(l32)) * 8);
    auto v_chunk = [&](int f, int s2) { return (32 * f + l32) * kTileKeys + (((2 * s2 + lhi) ^ v4_swizzle(32 * f + l32)) * 8); };

    // what a wave requests of a tile: its 16 keys' codes and words s | z << 16 (NW 8: waves 0 - 3 keys, waves 4 - 7 values)
    const bool keys = NW == 4 || wave < 4, values = NW == 4 || wave >= 4;
    const PageRow pages(p, s.slot);
    const uint32_t params_at = static_cast<uint32_t>(D / 2) << p.shift, block = params_at + (4u << p.shift);
    const int my_key = lane >> 2, my_part = lane & 3, my_four = lane >> 4, my_c = lane & 15;
    Words kw, vw;
    uint32_t kp = 0;
    u32x4_t vp;
    auto load = [](__amdgpu_buffer_rsrc_t buf, uint32_t off, uint32_t base) __attribute__((always_inline)) {
        if constexpr (S == 4) return __builtin_amdgcn_raw_buffer_load_b128(buf, off, base, 0);
        else return __builtin_amdgcn_raw_buffer_load_b64(buf, off, base, 0);
    };
    auto request = [&](int tile, int page) __attribute__((always_inline)) {
        const uint32_t t = (walk.key(tile) + 16 * part) & ((1 << p.shift) - 1);
        const size_t at = (static_cast<size_t>(max(page, 0)) * p.nkv + hk) * block;
        const int size = page < 0 || tile >= t1 ? 0 : static_cast<int>(block);   // (of a page that is gone: an empty buffer, zeros)
        if (keys) {
            const auto buf = buffer_of(reinterpret_cast<const char*>(p.k) + at, size);
            kw = load(buf, my_key * (D / 2) + my_part * (D / 8), t * (D / 2));
            kp = __builtin_amdgcn_raw_buffer_load_b32(buf, 4 * my_key, params_at + 4 * t, 0);
        }
        if (values) {
            const auto buf = buffer_of(reinterpret_cast<const char*>(p.v) + at, size);
            vw = load(buf, my_four * (2 * D) + my_c * (D / 8), t * (D / 2));
            vp = __builtin_amdgcn_raw_buffer_load_b128(buf, 16 * my_four, params_at + 4 * t, 0);
        }
    };
    // the requested tile -> LDS; places from `hi` on get scales of zero (what lies there may be anything)
    auto unpack = [&](int tile, int buf) __attribute__((always_inline)) {
        const int key0 = walk.key(tile) + 16 * part;
        if (keys) {
            const int key = 16 * part + my_key;
            const uint32_t zz = __builtin_amdgcn_perm(kp, kp, 0x07060706u) & 0x000f000fu;   // (in unused places it may be anything)
#pragma unroll
            for (int w = 0; w < S; ++w)
                *reinterpret_cast<u32x4_t*>(&Ks[buf][key * D + (((S * my_part + w) ^ k4_swizzle<D>(key)) * 8)]) = codes_less4(kw[w], zz);
            if (my_part == 0) ks[buf][key] = key0 + my_key < walk.hi ? act_to_float<BF16>(static_cast<uint16_t>(kp & 0xffffu)) * unit : 0.0f;
        }
        if (values) {
            float t4[4], big = 0.0f;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                t4[r] = key0 + 4 * my_four + r < walk.hi ? act_to_float<BF16>(static_cast<uint16_t>(vp[r] & 0xffffu)) : 0.0f;
                big = fmaxf(big, t4[r]);
            }
            if (my_c == 0) *reinterpret_cast<float4_t*>(&ts[buf][16 * part + 4 * my_four]) = float4_t{t4[0], t4[1], t4[2], t4[3]};
            big = fmaxf(big, __shfl_xor(big, 16, 64));
            big = fmaxf(big, __shfl_xor(big, 32, 64));
            if (lane == 0) tmax[buf][part] = big;
            const uint32_t z01 = __builtin_amdgcn_perm(vp[1], vp[0], 0x07060302u) & 0x000f000fu, z23 = __builtin_amdgcn_perm(vp[3], vp[2], 0x07060302u) & 0x000f000fu;
            // tokens 4 my_four .. + 3 of 16: chunk 2 part + (my_four & 1) of a column's row, its half my_four >> 1
#pragma unroll
            for (int h = 0; h < S / 2; ++h) {
                const u32x4_t a = codes_less4(vw[2 * h], z01), c = codes_less4(vw[2 * h + 1], z23);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int column = (D / 16) * my_c + 4 * h + i;
                    *reinterpret_cast<u32x2_t*>(&Vs[buf][column * kTileKeys + (((2 * part + (my_four & 1)) ^ v4_swizzle(column)) * 8) + 4 * (my_four >> 1)]) = u32x2_t{a[i], c[i]};
                }
            }
        }
    };
    auto ids_of = [&](int tile) __attribute__((always_inline)) { return tile_pages(pages, walk.key(min(tile, walk.steps - 1)), part); };

    float16_t o[DF];
#pragma unroll
    for (int f = 0; f < DF; ++f)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[f][r] = 0.0f;
    float m_run = kPagedNone, l_run = 0.0f;
    int t_exp = -60;                             // log2 of t_ref
    auto turn = [&](int t, int gone, int buf) __attribute__((always_inline)) {
        const int key0 = walk.key(t);
        float16_t st[2];
#pragma unroll
        for (int kf = 0; kf < 2; ++kf)
#pragma unroll
            for (int r = 0; r < 16; ++r) st[kf][r] = 0.0f;
#pragma unroll
        for (int i = 0; i < 2 * KS; ++i) {
            const int kf = i / KS, k = i % KS;
            st[kf] = H::mfma32(*reinterpret_cast<const u32x4_t*>(&Ks[buf][kf * 32 * D + k_at[k]]), qf[k], st[kf]);
        }
#pragma unroll
        for (int kf = 0; kf < 2; ++kf)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                const float4_t x = *reinterpret_cast<const float4_t*>(&ks[buf][32 * kf + 8 * q4 + 4 * lhi]);
#pragma unroll
                for (int r = 0; r < 4; ++r) st[kf][4 * q4 + r] *= x[r];
            }
        // a tile that every query of the wave sees whole needs no mask
        uint32_t hidden = 0;
        const bool all = gone == 0 && key0 + kTileKeys <= min(w_first + 1, walk.hi) && (p.window == 0 || key0 > w_last - p.window || key0 + kTileKeys <= p.sinks);
        if (!all) {
#pragma unroll
            for (int kf = 0; kf < 2; ++kf)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int key = key0 + kf * 32 + 8 * (r >> 2) + 4 * lhi + (r & 3);
                    const bool seen = (key <= place) & (key < walk.hi) & ((gone >> (kf * 2 + (r >> 3)) & 1) == 0) & ((key > reach) | (key < p.sinks));
                    st[kf][r] = seen ? st[kf][r] : -INFINITY;
                    hidden |= seen ? 0u : 1u << (16 * kf + r);
                }
        }
        // values' scales above the reference so far: the next power of two but one
        const float4_t tm = *reinterpret_cast<const float4_t*>(tmax[buf]);
        const float tx = fmaxf(fmaxf(tm[0], tm[1]), fmaxf(tm[2], tm[3]));
        if (tx > ldexpf(1.0f, t_exp)) {
            const int e = min(static_cast<int>(__float_as_uint(tx) >> 23) - 127 + 2, 126);
            const float beta = ldexpf(1.0f, t_exp - e);
            m_run = m_run > kPagedNone ? m_run + static_cast<float>(e - t_exp) : m_run;
            l_run *= beta;
#pragma unroll
            for (int f = 0; f < DF; ++f)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[f][r] *= beta;
            t_exp = e;
        }
        // Probabilities; the reference point stays as long as their sum over the lane's keys does not pass fp16's largest number, so each fits.
        u32x4_t pf[4];
        auto weigh = [&](float16_t* st) __attribute__((always_inline)) {
            float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int kf = 0; kf < 2; ++kf)
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) {
                    const float4_t t4 = *reinterpret_cast<const float4_t*>(&ts[buf][32 * kf + 8 * q4 + 4 * lhi]);
#pragma unroll
                    for (int r = 0; r < 4; r += 2) {
                        const float p0 = __builtin_amdgcn_exp2f(fmaf(st[kf][4 * q4 + r], up, -m_run)), p1 = __builtin_amdgcn_exp2f(fmaf(st[kf][4 * q4 + r + 1], up, -m_run));
                        sum[q4] += p0 + p1;
                        float w0 = p0 * t4[r], w1 = p1 * t4[r + 1];
                        if (!all) {                              // (a scale that the column does not see may be NaN)
                            w0 = hidden >> (16 * kf + 4 * q4 + r) & 1 ? 0.0f : w0;
                            w1 = hidden >> (16 * kf + 4 * q4 + r + 1) & 1 ? 0.0f : w1;
                        }
                        uint32_t w = H::pack(w0, w1);
                        asm("" : "+v"(w));
                        pf[kf * 2 + (q4 >> 1)][2 * (q4 & 1) + (r >> 1)] = w;
                    }
                }
            return (sum[0] + sum[1]) + (sum[2] + sum[3]);
        };
        float sum = weigh(st);
        if (__any(!(sum <= ldexpf(65504.0f, -t_exp)))) {
            float mx = -INFINITY;
#pragma unroll
            for (int kf = 0; kf < 2; ++kf)
#pragma unroll
                for (int r = 0; r < 16; ++r) mx = fmaxf(mx, st[kf][r]);
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * up;
            const float m_new = fmaxf(m_run, mx - (kChunkLift4 - static_cast<float>(t_exp))), alpha = __builtin_amdgcn_exp2f(m_run - m_new);
            l_run *= alpha;
#pragma unroll
            for (int f = 0; f < DF; ++f)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[f][r] *= alpha;
            m_run = m_new;
            sum = weigh(st);
        }
        l_run += sum;
#pragma unroll
        for (int s2 = 0; s2 < 4; ++s2)
#pragma unroll
            for (int f = 0; f < DF; ++f) o[f] = H::mfma32(*reinterpret_cast<const u32x4_t*>(&Vs[buf][v_chunk(f, s2)]), pf[s2], o[f]);
    };
    if (t0 < t1) {
        // page ids are read a tile before the request that uses them
        TilePages i0 = ids_of(t0), i1 = ids_of(t0 + 1), i2 = ids_of(t0 + 2);
        request(t0, i0.page);
        unpack(t0, 0);
        request(t0 + 1, i1.page);
        for (int t = t0; t < t1; ++t) {
            const int buf = (t - t0) & 1;
            __syncthreads();                                     // tile t is in LDS, and the other buffers have been read
            if (t + 1 < t1) unpack(t + 1, buf ^ 1);
            request(t + 2, i2.page);
            turn(t, i0.gone, buf);
            i0 = i1;
            i1 = i2;
            i2 = ids_of(t + 3);
        }
    }

    const float l_tot = l_run + __shfl_xor(l_run, 32, 64);
    if (!mine) return;
    // (odd columns' codes were times 16)
    if (SPLIT) {
        float* dst = p.part + ((static_cast<size_t>(s.row0 + qi) * p.nh + head) * p.ranges + z) * part_stride(D);
        if (lhi == 0) dst[D + 2] = static_cast<float>(ranges);
        if (ranges > 1) {
#pragma unroll
            for (int f = 0; f < DF; ++f)
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4)
                    *reinterpret_cast<float4_t*>(dst + f * 32 + 8 * q4 + 4 * lhi) = float4_t{o[f][4 * q4] * 0x1p24f, o[f][4 * q4 + 1] * 0x1p20f, o[f][4 * q4 + 2] * 0x1p24f, o[f][4 * q4 + 3] * 0x1p20f};
            if (lhi == 0) *reinterpret_cast<float2_t*>(dst + D) = float2_t{m_run, l_tot};
            return;
        }
    }
    const float inv = l_tot != 0.0f ? 0x1p20f / l_tot : 0.0f;    // a row that sees no key is zero
    uint16_t* orow = p.out + (s.row0 + qi) * p.out_stride + head * D;
#pragma unroll
    for (int f = 0; f < DF; ++f)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
            u32x2_t w;
            w[0] = Act16<BF16>::pack(o[f][4 * q4] * 16.0f * inv, o[f][4 * q4 + 1] * inv);
            w[1] = Act16<BF16>::pack(o[f][4 * q4 + 2] * 16.0f * inv, o[f][4 * q4 + 3] * inv);
            *reinterpret_cast<u32x2_t*>(orow + f * 32 + 8 * q4 + 4 * lhi) = w;
        }
}

template <int D, bool BF16>
static hipError_t chunk4_form(const PagedAttnDev& a, int groups, hipStream_t stream) {
    const dim3 grid(static_cast<uint32_t>(static_cast<int64_t>(a.items) * a.ranges * a.nkv));
    if (groups == 0) hipLaunchKernelGGL((paged4_chunk_kernel<D, BF16, false, 8>), grid, dim3(512), 0, stream, a);
    else if (a.ranges > 1) hipLaunchKernelGGL((paged4_chunk_kernel<D, BF16, true, 4>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((paged4_chunk_kernel<D, BF16, false, 4>), grid, dim3(256), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_paged4_chunk(const PagedAttnDev& a, int groups, int d, hipStream_t stream) {
    if (d == 128) return a.bf16 ? chunk4_form<128, true>(a, groups, stream) : chunk4_form<128, false>(a, groups, stream);
    return a.bf16 ? chunk4_form<64, true>(a, groups, stream) : chunk4_form<64, false>(a, groups, stream);
}

}  // namespace qtale
