// Rotary embedding of queries and new keys, and the append of keys and values to the pages of their slots.
//
// A pair (a, b) of a head turns by angle = position * freq[pair]: (a cos - b sin, b cos + a sin) * magnitude.  Pairs are (i, i + r/2) or
// (2i, 2i + 1) for i < r/2; columns from r on stay as they are.  The angle is reduced in 64 bits, in turns (a late position times a frequency
// has lost its fraction in 32), the sine and cosine and the products are in 32, and there is one rounding, to the cache's type.
// Bytes bound it for many tokens: 5100 tokens of 32 + 2 x 8 heads of 128 take 27.6 us, 4.6 TB/s read and written (a copy reaches 5.1).  For few the
// chain offsets -> slot -> length, page does, which runs beside the loads of the row: 64 tokens of 3 x 32 heads 4.4 us, most of it the launch's own.
#include <algorithm>

#include "paged.h"
#include "paged_split.h"
#include "qtale_dev.h"

namespace qtale {

constexpr double kTurnsPerRadian = 0.15915494309189533577;

template <bool BF16>
__device__ __forceinline__ uint16_t round_act(float f) {         // no saturation: an infinity stays one
    return BF16 ? __builtin_bit_cast(uint16_t, static_cast<__bf16>(f)) : __builtin_bit_cast(uint16_t, static_cast<half_t>(f));
}

// PAIRS: 0 half (r a multiple of 16: a thread turns 8 columns and their 8 partners), 1 interleaved, 2 half with any r.
// COPIES: workgroups past the rows copy shared pages, the tokens before those that the rows append (a launch less, 2.5 us; 5100 rows without
// copies 27.6 us, with this branch 29.5).
template <bool BF16, int PAIRS, bool COPIES>
__global__ void __launch_bounds__(256)
paged_rope_kernel(PagedRopeArgs a) {
    __shared__ float cs[64], sn[64];                             // head_dim <= 128
    const int i = blockIdx.x;
    if (COPIES && i >= a.T) {
        if (blockIdx.y == 0) split_pages(a.kv, a.copies, i - a.T, gridDim.x - a.T);
        return;
    }
    if (a.count && i >= *a.count) return;
    const int tid = threadIdx.x, lane = tid & 63;
    const int d = a.kv.d, r = a.rotary_dim, half = r >> 1;
    const int t = a.rows ? a.rows[i] : i;
    const int position = a.positions[t];
    // columns of a head that a thread takes together; units per turned head and per value head
    const int turned = PAIRS == 0 ? (r >> 4) : 0;                // units of 16 columns (two chunks of 8)
    const int per = PAIRS == 0 ? turned + ((d - r) >> 3) : d >> 3;
    const int cpr = d >> 3;
    const int n_turn = (a.nh + a.kv.nkv) * per, units = n_turn + a.kv.nkv * cpr;
    const int u0 = blockIdx.y * 256 + tid, step = gridDim.y * 256;
    // where unit u reads: chunk (8 columns) of a head of q, k or v, and for PAIRS 0 its partner
    struct Unit { const uint16_t* src; int head, chunk; bool value; };
    auto find = [&](int u) {
        Unit x;
        x.value = u >= n_turn;
        const int w = x.value ? u - n_turn : u;
        const int p = x.value ? cpr : per;
        x.head = w / p;
        const int c = w - x.head * p;
        x.chunk = x.value || PAIRS != 0 || c < turned ? c : c + turned;
        x.src = x.value ? a.v + i * a.v_stride + x.head * d
                        : x.head < a.nh ? a.q + i * a.q_stride + x.head * d : a.k + i * a.k_stride + (x.head - a.nh) * d;
        return x;
    };
    constexpr int KEEP = 3;                                      // units whose loads are on their way before anything else is known
    u32x4_t lo[KEEP], hi[KEEP];
#pragma unroll
    for (int k = 0; k < KEEP; ++k) {
        const Unit x = find(min(u0 + k * step, units - 1));
        lo[k] = *reinterpret_cast<const u32x4_t*>(x.src + 8 * x.chunk);
        if (PAIRS == 0) hi[k] = *reinterpret_cast<const u32x4_t*>(x.src + 8 * x.chunk + (!x.value && x.chunk < turned ? half : 0));
    }
    if (tid < half) {
        const double turns = static_cast<double>(position) * (a.freqs[tid] * kTurnsPerRadian);
        float s, c;
        sincospif(2.0f * static_cast<float>(turns - rint(turns)), &s, &c);
        cs[tid] = c * a.magnitude;
        sn[tid] = s * a.magnitude;
    }
    // the row's sequence: the number of sequences that end at or before it
    int b = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) b += __popcll(__ballot(b0 + lane < a.B && a.seq_offsets[min(b0 + lane, a.B - 1) + 1] <= i));
    int64_t dst = -1;                                            // element of (page, head 0, place) in the pool
    if (b < a.B) {
        const int slot = a.slots ? a.slots[b] : b;
        if (static_cast<uint32_t>(slot) < static_cast<uint32_t>(a.kv.n_slots)) {
            const int begin = a.seq_offsets[b], len = a.kv.len[slot];
            const int at = (a.first ? a.first[b] : len - (a.seq_offsets[b + 1] - begin)) + (i - begin);
            if (at >= 0 && at < len && (at >> a.kv.shift) < a.kv.max_pages) {
                const int page = a.kv.table[static_cast<size_t>(slot) * a.kv.max_pages + (at >> a.kv.shift)];
                if (static_cast<uint32_t>(page) < static_cast<uint32_t>(a.kv.n_pages))
                    dst = ((static_cast<int64_t>(page) * a.kv.nkv << a.kv.shift) + (at & ((1 << a.kv.shift) - 1))) * d;
            }
        }
    }
    const int64_t head_step = static_cast<int64_t>(d) << a.kv.shift;
    __syncthreads();

    // q goes to q_out, k to its page; a value chunk only moves
    auto target = [&](const Unit& x) -> uint16_t* {
        if (x.value) return dst >= 0 ? a.kv.v + dst + x.head * head_step : nullptr;
        if (x.head < a.nh) return a.q_out + i * a.q_out_stride + x.head * d;
        return dst >= 0 ? a.kv.k + dst + (x.head - a.nh) * head_step : nullptr;
    };
    auto turn = [&](float x, float y, int pair, uint16_t* first, uint16_t* second) {
        const float c = cs[pair], s = sn[pair];
        *first = round_act<BF16>(fmaf(x, c, -(y * s)));
        *second = round_act<BF16>(fmaf(y, c, x * s));
    };
    auto low = [](uint32_t w) { return static_cast<uint16_t>(w & 0xffffu); };
    auto high = [](uint32_t w) { return static_cast<uint16_t>(w >> 16); };
    auto finish = [&](const Unit& x, u32x4_t p, u32x4_t q) {
        uint16_t* to = target(x);
        if (x.value) {
            if (to) *reinterpret_cast<u32x4_t*>(to + 8 * x.chunk) = p;
            return;
        }
        if (PAIRS == 0) {
            if (x.chunk < turned) {
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint16_t f0, s0, f1, s1;
                    turn(act_to_float<BF16>(low(p[w])), act_to_float<BF16>(low(q[w])), 8 * x.chunk + 2 * w, &f0, &s0);
                    turn(act_to_float<BF16>(high(p[w])), act_to_float<BF16>(high(q[w])), 8 * x.chunk + 2 * w + 1, &f1, &s1);
                    p[w] = f0 | (static_cast<uint32_t>(f1) << 16);
                    q[w] = s0 | (static_cast<uint32_t>(s1) << 16);
                }
                if (to) *reinterpret_cast<u32x4_t*>(to + 8 * x.chunk + half) = q;
            }
        } else if (PAIRS == 1) {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int pair = 4 * x.chunk + w;
                if (pair < half) {
                    uint16_t f, s;
                    turn(act_to_float<BF16>(low(p[w])), act_to_float<BF16>(high(p[w])), pair, &f, &s);
                    p[w] = f | (static_cast<uint32_t>(s) << 16);
                }
            }
        } else {
            // The partners lie anywhere in the head; q may be turned in place: the lanes of a head are in one wave (8 or 16 of them), whose
            // loads all come before its stores (the barrier keeps the compiler to it).
            uint16_t own[8], other[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int col = 8 * x.chunk + e;
                own[e] = e & 1 ? high(p[e >> 1]) : low(p[e >> 1]);
                other[e] = col < r ? x.src[col < half ? col + half : col - half] : 0;
            }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int col = 8 * x.chunk + e;
                if (col >= r) continue;
                uint16_t f, s;
                if (col < half) { turn(act_to_float<BF16>(own[e]), act_to_float<BF16>(other[e]), col, &f, &s); own[e] = f; }
                else { turn(act_to_float<BF16>(other[e]), act_to_float<BF16>(own[e]), col - half, &f, &s); own[e] = s; }
            }
#pragma unroll
            for (int w = 0; w < 4; ++w) p[w] = own[2 * w] | (static_cast<uint32_t>(own[2 * w + 1]) << 16);
        }
        if (to) *reinterpret_cast<u32x4_t*>(to + 8 * x.chunk) = p;
    };
#pragma unroll
    for (int k = 0; k < KEEP; ++k)
        if (u0 + k * step < units) finish(find(u0 + k * step), lo[k], PAIRS == 0 ? hi[k] : lo[k]);
    for (int u = u0 + KEEP * step; u < units; u += step) {
        const Unit x = find(u);
        const u32x4_t p = *reinterpret_cast<const u32x4_t*>(x.src + 8 * x.chunk);
        finish(x, p, PAIRS == 0 ? *reinterpret_cast<const u32x4_t*>(x.src + 8 * x.chunk + (!x.value && x.chunk < turned ? half : 0)) : p);
    }
}

template <bool BF16, bool COPIES>
static void launch_rope_form(const PagedRopeArgs& a, dim3 grid, hipStream_t stream) {
    if (a.layout == 1) hipLaunchKernelGGL((paged_rope_kernel<BF16, 1, COPIES>), grid, dim3(256), 0, stream, a);
    else if (a.rotary_dim % 16 == 0) hipLaunchKernelGGL((paged_rope_kernel<BF16, 0, COPIES>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((paged_rope_kernel<BF16, 2, COPIES>), grid, dim3(256), 0, stream, a);
}

hipError_t launch_paged_rope(const PagedRopeArgs& a, hipStream_t stream) {
    if (a.T == 0) return hipSuccess;
    // few tokens: a row's units go to several workgroups, about one unit per thread
    const int chunks = (a.nh + 2 * a.kv.nkv) * (a.kv.d >> 3);
    const int parts = a.T >= 512 ? 1 : std::min((chunks + 511) / 512, 16);
    const dim3 grid(a.T + (a.copies.n ? std::min(a.B * a.kv.nkv, 256) : 0), parts);
    if (a.copies.n) launch_rope_form<false, true>(a, grid, stream);   // (inside the layers, whose cache is fp16)
    else if (a.kv.bf16) launch_rope_form<true, false>(a, grid, stream);
    else launch_rope_form<false, false>(a, grid, stream);
    return hipGetLastError();
}

}  // namespace qtale
