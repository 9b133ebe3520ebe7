// Rotary embedding of queries and new keys and the append of keys and values to pages in 4 bits; entries of pages as the values they stand for.
//
// Pairs, layouts and the angle in turns are those of paged_rope.hip.  Queries turn in 32 bits.  Keys turn in 64 and are rounded to 32 and then to the
// cache's type: a code is a rounding of a rounding, and with keys that are a bit of 32 off some would land a whole step away from what their
// definition says.  d / 8 lanes hold a (token, head) row, eight columns each; they find its ends by d / 8-wide exchanges.  The quotient of
// the scale is taken in 64 bits and the codes' in 32, which decides them exactly: x and s are 16-bit numbers, and x / s that is not
// a half itself is further from one than 2^-17 of it, where the division errs by 2^-24.
#include <algorithm>

#include "paged4.h"
#include "paged_split.h"

namespace qtale {

constexpr double kTurnsPerRadian = 0.15915494309189533577;

template <bool BF16>
__device__ __forceinline__ uint16_t round_act(float f) {         // no saturation: an infinity stays one
    return BF16 ? __builtin_bit_cast(uint16_t, static_cast<__bf16>(f)) : __builtin_bit_cast(uint16_t, static_cast<half_t>(f));
}

// 64 bits to 32, to be rounded again: two roundings, also where the compiler could make them one.
__device__ __forceinline__ float narrow(double x) {
    float f = static_cast<float>(x);
    asm("" : "+v"(f));
    return f;
}

// Codes of this lane's eight values of a row that `lanes` (8 or 16) neighbouring lanes hold, one per nibble in the columns' order, and the row's word
// s | z << 16.
template <bool BF16>
__device__ __forceinline__ uint32_t quantize_row(const float* x, int lanes, uint32_t* param) {
    float lo = 0.0f, hi = 0.0f;
    int bad = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        lo = fminf(lo, x[e]);
        hi = fmaxf(hi, x[e]);
        bad |= !(fabsf(x[e]) < INFINITY);
    }
    for (int o = lanes >> 1; o > 0; o >>= 1) {
        lo = fminf(lo, __shfl_xor(lo, o, 64));
        hi = fmaxf(hi, __shfl_xor(hi, o, 64));
        bad |= __shfl_xor(bad, o, 64);
    }
    if (bad) {
        *param = BF16 ? 0x7fc0u : 0x7e00u;
        return 0;
    }
    const uint16_t bits = round_act<BF16>(narrow((static_cast<double>(hi) - static_cast<double>(lo)) / 15.0));
    float s = act_to_float<BF16>(bits);
    const uint16_t stored = s == 0.0f ? round_act<BF16>(1.0f) : bits;
    if (s == 0.0f) s = 1.0f;
    const float z = fminf(rintf(-lo / s), 15.0f);
    *param = stored | static_cast<uint32_t>(z) << 16;
    uint32_t codes = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) codes |= static_cast<uint32_t>(fminf(fmaxf(rintf(x[e] / s) + z, 0.0f), 15.0f)) << (4 * e);
    return codes;
}

// Nibbles in the order of columns -> the order of a key's word: even columns in the low half, odd ones in the high half.
__device__ __forceinline__ uint32_t key_order(uint32_t c) {
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) w |= (c >> (4 * e) & 15u) << (4 * (e >> 1) + 16 * (e & 1));
    return w;
}

// A workgroup per token (few tokens: per 256 units), so that cosines and sines, in 64 bits, are made once for all its heads.  Bound by HBM for many tokens, a
// launch for few: 5100 tokens of 48 heads of 128 in bf16 30.5 us, 3.6 TB/s read and written (the rotation into 16-bit pages 28 us, 4.6 TB/s, twice the
// writes for keys and values, and no exchanges); 64 tokens of 96 heads 5.4 us.
// PAIRS: 0 half with r a multiple of 16 (a lane's partners are one chunk), 1 interleaved, 2 half with any r.  COPIES as in paged_rope_kernel.
template <bool BF16, int PAIRS, bool COPIES>
__global__ void __launch_bounds__(256)
paged4_rope_kernel(PagedRopeArgs a) {
    __shared__ double cs[64], sn[64];                            // head_dim <= 128
    const int i = blockIdx.x;
    if (COPIES && i >= a.T) {
        if (blockIdx.y == 0) split_pages4(a.kv, a.copies, i - a.T, gridDim.x - a.T);
        return;
    }
    if (a.count && i >= *a.count) return;
    const int tid = threadIdx.x;
    const int d = a.kv.d, r = a.rotary_dim, half = r >> 1, cpr = d >> 3;
    const int t = a.rows ? a.rows[i] : i;
    const int position = a.positions[t];
    // units of eight columns: keys, values, queries.  A row's lanes are neighbours in one wave (their number divides 64, and units of all
    // rows before them are a multiple of it)
    const int n_kv = a.kv.nkv * cpr, units = 2 * n_kv + a.nh * cpr;
    if (tid < half) {
        const double turns = static_cast<double>(position) * (a.freqs[tid] * kTurnsPerRadian);
        double s, c;
        sincospi(2.0 * (turns - rint(turns)), &s, &c);
        cs[tid] = c * static_cast<double>(a.magnitude);
        sn[tid] = s * static_cast<double>(a.magnitude);
    }
    const RowEntry to = entry_of_row(a.kv, a.seq_offsets, a.slots, a.first, a.B, i);
    const Block4 block{d, a.kv.shift};
    __syncthreads();
    for (int u = blockIdx.y * 256 + tid; u < units; u += gridDim.y * 256) {
        const int kind = u < n_kv ? 0 : u < 2 * n_kv ? 1 : 2;     // key, value, query
        const int w = kind == 0 ? u : kind == 1 ? u - n_kv : u - 2 * n_kv;
        const int head = w / cpr, chunk = w - head * cpr, col = 8 * chunk;
        const uint16_t* src = (kind == 0 ? a.k + i * a.k_stride : kind == 1 ? a.v + i * a.v_stride : a.q + i * a.q_stride) + head * d;
        const u32x4_t own = *reinterpret_cast<const u32x4_t*>(src + col);
        uint16_t x[8], y[8];                                     // this lane's columns, and their partners
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = static_cast<uint16_t>(own[e >> 1] >> (16 * (e & 1)) & 0xffffu);
        const bool turns = kind != 1 && col < r;
        if (PAIRS == 0) {
            const u32x4_t other = *reinterpret_cast<const u32x4_t*>(src + (turns ? (col < half ? col + half : col - half) : col));
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = static_cast<uint16_t>(other[e >> 1] >> (16 * (e & 1)) & 0xffffu);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                y[e] = PAIRS == 1 ? x[e ^ 1] : turns && col + e < r ? src[col + e < half ? col + e + half : col + e - half] : 0;
        }
        __builtin_amdgcn_wave_barrier();                         // q may be turned in place: a head's loads come before its stores
        auto first_of = [&](int e) { return PAIRS == 1 ? (e & 1) == 0 : col + e < half; };
        auto pair_of = [&](int e) { return PAIRS == 1 ? (col + e) >> 1 : first_of(e) ? col + e : col + e - half; };
        if (kind == 2) {
            u32x4_t out;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                uint16_t v = x[e];
                if (col + e < r) {
                    const float c = static_cast<float>(cs[pair_of(e)]), s = static_cast<float>(sn[pair_of(e)]);
                    const float p = act_to_float<BF16>(x[e]), q = act_to_float<BF16>(y[e]);
                    v = round_act<BF16>(fmaf(p, c, first_of(e) ? -(q * s) : q * s));
                }
                if (e & 1) out[e >> 1] |= static_cast<uint32_t>(v) << 16;
                else out[e >> 1] = v;
            }
            *reinterpret_cast<u32x4_t*>(a.q_out + i * a.q_out_stride + head * d + col) = out;
            continue;
        }
        if (to.page < 0) continue;                               // (the same in all lanes of the row)
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            f[e] = act_to_float<BF16>(x[e]);
            if (kind == 0 && col + e < r) {
                const double c = cs[pair_of(e)], s = sn[pair_of(e)], p = act_to_float<BF16>(x[e]), q = act_to_float<BF16>(y[e]);
                f[e] = act_to_float<BF16>(round_act<BF16>(narrow(fma(p, c, first_of(e) ? -(q * s) : q * s))));
            }
        }
        uint32_t param;
        const uint32_t codes = quantize_row<BF16>(f, cpr, &param);
        char* base = reinterpret_cast<char*>(kind == 0 ? a.kv.k : a.kv.v) + (static_cast<size_t>(to.page) * a.kv.nkv + head) * block.bytes();
        if (chunk == 0) *reinterpret_cast<uint32_t*>(base + block.param(to.place)) = param;
        if (kind == 0) {
            *reinterpret_cast<uint32_t*>(base + block.key(to.place) + 4 * chunk) = key_order(codes);
        } else {
            *reinterpret_cast<uint16_t*>(base + block.value(to.place, col)) = static_cast<uint16_t>(codes & 0xffffu);
            *reinterpret_cast<uint16_t*>(base + block.value(to.place, col + 4)) = static_cast<uint16_t>(codes >> 16);
        }
    }
}

template <bool BF16, bool COPIES>
static void rope4_form(const PagedRopeArgs& a, dim3 grid, hipStream_t stream) {
    if (a.layout == 1) hipLaunchKernelGGL((paged4_rope_kernel<BF16, 1, COPIES>), grid, dim3(256), 0, stream, a);
    else if (a.rotary_dim % 16 == 0) hipLaunchKernelGGL((paged4_rope_kernel<BF16, 0, COPIES>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((paged4_rope_kernel<BF16, 2, COPIES>), grid, dim3(256), 0, stream, a);
}

hipError_t launch_paged4_rope(const PagedRopeArgs& a, hipStream_t stream) {
    // few tokens: a row's units go to several workgroups, about one unit per thread
    const int units = (a.nh + 2 * a.kv.nkv) * (a.kv.d >> 3);
    const int parts = a.T >= 512 ? 1 : std::min((units + 255) / 256, 16);
    const dim3 grid(a.T + (a.copies.n ? std::min(a.B * a.kv.nkv, 256) : 0), parts);
    if (a.copies.n) rope4_form<false, true>(a, grid, stream);    // (inside the layers, whose cache is fp16)
    else if (a.kv.bf16) rope4_form<true, false>(a, grid, stream);
    else rope4_form<false, false>(a, grid, stream);
    return hipGetLastError();
}

// A workgroup per row: eight columns per thread.  (5100 rows of 8 + 8 heads of 128: 11.2 us, 2.4 TB/s: a chain of table, word and code for so little.)
__global__ void __launch_bounds__(256)
paged_read_kernel(PagedReadArgs a) {
    const int i = blockIdx.x, d = a.kv.d, cpr = d >> 3;
    if (i >= a.seq_offsets[a.B]) return;
    const RowEntry at = entry_of_row(a.kv, a.seq_offsets, a.slots, a.first, a.B, i);
    const Block4 block{d, a.kv.shift};
    for (int u = threadIdx.x; u < 2 * a.kv.nkv * cpr; u += 256) {
        const bool value = u >= a.kv.nkv * cpr;
        const int w = value ? u - a.kv.nkv * cpr : u, head = w / cpr, col = 8 * (w - head * cpr);
        u32x4_t out = {0u, 0u, 0u, 0u};
        if (at.page >= 0) {
            const char* base = reinterpret_cast<const char*>(value ? a.kv.v : a.kv.k) + (static_cast<size_t>(at.page) * a.kv.nkv + head) * head_bytes(a.kv);
            if (!a.kv.q4) {
                out = *reinterpret_cast<const u32x4_t*>(base + (static_cast<size_t>(at.place) * d + col) * 2);
            } else {
                const uint32_t param = *reinterpret_cast<const uint32_t*>(base + block.param(at.place));
                const float s = scale4(param, a.kv.bf16);
                const int z = static_cast<int>(param >> 16);
                uint32_t lo, hi;                                 // codes of columns 0 .. 3 and 4 .. 7, a nibble each
                uint32_t word = 0;
                if (value) {
                    lo = *reinterpret_cast<const uint16_t*>(base + block.value(at.place, col));
                    hi = *reinterpret_cast<const uint16_t*>(base + block.value(at.place, col + 4));
                } else {
                    word = *reinterpret_cast<const uint32_t*>(base + block.key(at.place) + col / 2);
                    lo = hi = 0;
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t code = value ? (e < 4 ? lo : hi) >> (4 * (e & 3)) & 15u : word >> (4 * (e >> 1) + 16 * (e & 1)) & 15u;
                    const float x = static_cast<float>(static_cast<int>(code) - z) * s;
                    const uint32_t bits = a.kv.bf16 ? round_act<true>(x) : round_act<false>(x);
                    out[e >> 1] |= bits << (16 * (e & 1));
                }
            }
        }
        *reinterpret_cast<u32x4_t*>((value ? a.v + i * a.v_stride : a.k + i * a.k_stride) + head * d + col) = out;
    }
}

hipError_t launch_paged_read(const PagedReadArgs& a, hipStream_t stream) {
    hipLaunchKernelGGL(paged_read_kernel, dim3(a.T), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace qtale
