// Attention over pages in 4 bits where few queries meet many keys: the form of paged_decode.hip (a workgroup of four waves per (sequence, kv head, 16
// (query, head) pairs), or per span of keys; a wave's step is 32 keys; the pairs are the 16 columns of both products), with codes as operands.
//
// A nibble at bits 0 - 3 of a 16-bit word is, read as fp16, the subnormal number c 2^-24, and at bits 4 - 7 it is 16 c 2^-24: the matrix cores take
// both as they are, exactly.  So a 32-bit word of eight codes becomes an operand with one shift and four ANDs.  The 16 goes into the queries'
// elements (powers of two), for values into the result.  Scales stay outside the products, in 32 bits, where they are exact too:
//   score = s_j (q . c_j - z_j sum(q)),   out = sum_j (p_j t_j) (c'_j - z'_j) / sum_j p_j,
// the sum with z' as one more fragment of the second product whose operand rows are all z', so that both parts see the same rounded p t.
// Queries are fp16 relative to their row's power of two (exact, but for elements 2^-34 of the largest), whatever the cache's type, and p t is fp16
// relative to a running power of two of the t that the row has seen, which it follows upwards: it is off by 2^-11 of itself, as the output's own rounding is, or by
// 2^-35 of the largest p times the largest t.  (fp16 caches hardly reach that; a bf16 row that sees values 2^24 above those that it weighs loses bits.)  All codes are finite, so that a row reaches a NaN (scale) only through a key that it sees.
//
// A wave's step of 32 keys takes sixteen words of codes per lane apart (five instructions each) for 18 or 9 MFMAs.  What bounds it: HBM where all CUs are
// filled, 64 x 4000 keys, 32 heads of 128, 171 us, 6.5 TB/s; else the time that a CU's own loads take: 33 x 3000 keys, 8 heads, 28 us and 5 for the
// pieces, 3.4 TB/s (spans for three workgroups per CU; compiled for four, with 7 registers of 128 spilled); 48 x 4 tokens under a window of 1024, heads of 64, 17 us.  (The 16-bit cache takes 69 us for 33 x 3000, four times the bytes.)
#include <algorithm>

#include "paged4.h"
#include "paged_attn.h"

namespace qtale {

constexpr int kStepKeys = 32;                    // per wave
constexpr int kUnitSteps = 4;                    // spans are cut at multiples of this: a step per wave
constexpr float kLift4 = 0x1p12f;                // the largest probability goes in as 2^12 when the reference point moves (kDecodeLift)

// Units of a sequence in a call with spans; 0: not this kernel's.  A sequence without keys has one, in which its zeros are written.
__device__ __forceinline__ int seq_units4(const PagedAttnDev& p, int b) {
    const SeqView s(p, b);
    if (s.n == 0 || (p.take != 0 && s.n * p.rep > kDecodeCols)) return 0;
    return max((KeySteps<kStepKeys>(s.first, s.first + s.n - 1, s.len, p.window, p.sinks).steps + kUnitSteps - 1) / kUnitSteps, 1);
}

// A word's eight codes as the operand of a k-step: elements 2 i, 2 i + 1 are its codes at bits 4 i and 16 + 4 i, those of odd i times 16.
__device__ __forceinline__ u32x4_t codes4(uint32_t w) {
    const uint32_t y = w >> 8;
    return u32x4_t{w & 0x000f000fu, w & 0x00f000f0u, y & 0x000f000fu, y & 0x00f000f0u};
}

template <int D, bool BF16, bool SPANS>
__global__ void __launch_bounds__(256, 4)
paged4_decode_kernel(PagedAttnDev p) {
    constexpr int S = D / 32;                    // k-steps of the scores, and words of codes per lane and 16 keys
    constexpr int F = D / 16;                    // output fragments, and columns of V per lane
    typedef uint32_t Words __attribute__((ext_vector_type(S)));
    const int hk = blockIdx.x;                   // kv heads fastest
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4;
    __shared__ float sm[4][kDecodeCols][D + 2];
    __shared__ int ends[SPANS ? kSpanSeqs : 1];                  // units up to and with sequence b

    int b = blockIdx.z, cur = 0, end = 0, total = 0, spans = 1;
    uint32_t span = 0;
    if (SPANS) {
        for (int b0 = 0; b0 < p.B; b0 += 64) {
            int sum = b0 + lane < p.B ? seq_units4(p, b0 + lane) : 0;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int y = __shfl_up(sum, o, 64);
                if (lane >= o) sum += y;
            }
            if (wave == 0) ends[b0 + lane] = total + sum;
            total += __shfl(sum, 63, 64);
        }
        total = __builtin_amdgcn_readfirstlane(total);
        spans = min(p.spans, total);
        span = blockIdx.y;
        if (static_cast<int>(span) >= spans) return;
        cur = static_cast<int>(static_cast<uint64_t>(span) * total / static_cast<uint32_t>(spans));
        end = static_cast<int>(static_cast<uint64_t>(span + 1) * total / static_cast<uint32_t>(spans));
        __syncthreads();
        b = 0;
        for (int b0 = 0; b0 < p.B; b0 += 64) b += __popcll(__ballot(b0 + lane < p.B && ends[min(b0 + lane, p.B - 1)] <= cur));
    }
    const int begin = cur;
again:                                                           // the pieces of a span
    b = __builtin_amdgcn_readfirstlane(b);
    SeqView s(p, b);
    s.uniform();
    // this workgroup's columns c0 .. c0 + cols - 1 of the sequence's, of queries q_lo .. q_hi (with spans there are no more than sixteen)
    const int c0 = SPANS ? 0 : static_cast<int>(blockIdx.y) * kDecodeCols, all_cols = s.n * p.rep;
    if (!SPANS && (all_cols <= c0 || (p.take != 0 && all_cols > kDecodeCols))) return;
    const int cols = min(all_cols - c0, kDecodeCols);
    const int q_lo = SPANS ? 0 : __builtin_amdgcn_readfirstlane(c0 / p.rep), q_hi = SPANS ? s.n - 1 : __builtin_amdgcn_readfirstlane((c0 + cols - 1) / p.rep);
    const KeySteps<kStepKeys> walk(s.first + q_lo, s.first + q_hi, s.len, p.window, p.sinks);
    int first_step = 0, last_step = walk.steps;
    bool whole = true;
    int seq_begin = 0, seq_end = 0;
    if (SPANS) {
        seq_begin = b > 0 ? __builtin_amdgcn_readfirstlane(ends[b - 1]) : 0;
        seq_end = __builtin_amdgcn_readfirstlane(ends[b]);
        first_step = (cur - seq_begin) * kUnitSteps;
        if (end < seq_end) last_step = min(last_step, (end - seq_begin) * kUnitSteps);
        whole = cur == seq_begin && end >= seq_end;
    }
    const int col = c0 + min(c, cols - 1);                       // this lane's column: query col / rep, head col % rep
    const int qi = col / p.rep, head = hk * p.rep + col - qi * p.rep;
    const int place = s.first + qi;                              // the query's place in its slot
    const int reach = p.window > 0 ? place - p.window : INT32_MIN;   // keys after it are in its window

    const int s0 = first_step + wave, s1 = last_step;            // this wave's steps: s0, s0 + 4, ...
    const PageRow pages(p, s.slot);
    const int hi = walk.hi, lo = walk.lo, n_minus = q_hi - q_lo;
    const uint32_t params_at = static_cast<uint32_t>(D / 2) << p.shift, block = params_at + (4u << p.shift);

    // page ids of the two fragments of a step: read one step before the loads that use them
    struct Ids { int a, b; };
    auto ids_of = [&](int st) {
        const int kb = walk.key(min(st, walk.steps - 1));
        return Ids{pages.at(kb), pages.at(kb + 16)};
    };
    Words kn[2], vn[2];
    u32x4_t kp[2], vp[2];                                        // words s | z << 16 of keys 4 g .. 4 g + 3 of each fragment
    const uint32_t k_off = c * (D / 2) + (D / 8) * g, v_off = g * (2 * D) + (D / 8) * c;
    auto load = [](__amdgpu_buffer_rsrc_t buf, uint32_t off, uint32_t base) {
        if constexpr (S == 4) return __builtin_amdgcn_raw_buffer_load_b128(buf, off, base, 2);   // read once: non-temporal
        else return __builtin_amdgcn_raw_buffer_load_b64(buf, off, base, 2);
    };
    auto fetch = [&](const uint16_t* pool, int kb, Ids id, uint32_t off, Words* to, u32x4_t* params) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int page = u ? id.b : id.a;                    // (of a page that is gone: an empty buffer, zeros)
            const auto buf = buffer_of(reinterpret_cast<const char*>(pool) + (static_cast<size_t>(max(page, 0)) * p.nkv + hk) * block, page < 0 ? 0 : block);
            const uint32_t t = (kb + 16 * u) & ((1 << p.shift) - 1);
            to[u] = load(buf, off, t * (D / 2));
            params[u] = __builtin_amdgcn_raw_buffer_load_b128(buf, 16 * g, params_at + 4 * t, 2);
        }
    };

    // queries: k-step k of lane g has columns (D / 4) g + 8 k .., as fp16 with the row's largest at 2^13; unq: what a unit of the products stands
    // for, with the scale and log2(e)
    u32x4_t q[S];
    float q_sum = 0.0f, unq;
    {
        const uint16_t* qrow = p.q + (s.row0 + qi) * p.q_stride + head * D + (D / 4) * g;
        u32x4_t raw[S];
        float big = 0.0f;
#pragma unroll
        for (int k = 0; k < S; ++k) {
            raw[k] = *reinterpret_cast<const u32x4_t*>(qrow + 8 * k);
#pragma unroll
            for (int w = 0; w < 4; ++w) big = fmaxf(big, fmaxf(fabsf(Act16<BF16>::low(raw[k][w])), fabsf(Act16<BF16>::high(raw[k][w]))));
        }
        big = fmaxf(big, __shfl_xor(big, 16, 64));
        big = fmaxf(big, __shfl_xor(big, 32, 64));
        const int e = min(max(static_cast<int>(__float_as_uint(big) >> 23) - 127, -100), 127);
        const float f = ldexpf(1.0f, 13 - e);
#pragma unroll
        for (int k = 0; k < S; ++k)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const uint32_t h = Act16<false>::pack(Act16<BF16>::low(raw[k][w]) * f, Act16<BF16>::high(raw[k][w]) * f);
                q_sum += Act16<false>::low(h) + Act16<false>::high(h);
                q[k][w] = w & 1 ? Act16<false>::pack(Act16<false>::low(h) * 0.0625f, Act16<false>::high(h) * 0.0625f) : h;
            }
        q_sum += __shfl_xor(q_sum, 16, 64);
        q_sum += __shfl_xor(q_sum, 32, 64);
        unq = ldexpf(p.scale_log2, e + 24 - 13);
    }

    // probabilities are 2^(score - m_run), m_run a score itself (less a lift it would be rounded, and from 2^27 on by more than fp16 has room for); the lift goes
    // in with the values' scales, which are relative to t_ref
    float m_run = kPagedNone, l_run = 0.0f, t_ref = 0x1p-100f, t_inv = kLift4 * 0x1p100f;
    float4_t o[F + 1];                                           // (the last: zero points)
#pragma unroll
    for (int f = 0; f <= F; ++f) o[f] = float4_t{0.f, 0.f, 0.f, 0.f};
    auto step = [&](int kb, Ids id, auto next) {
        float sc[8], t[8];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            float4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < S; ++k) sum = Act16<false>::mfma16(codes4(kn[u][k]), q[k], sum);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float z = half_bits_to_float(static_cast<uint16_t>(kp[u][r] >> 16));   // z 2^-24, as the codes
                sc[4 * u + r] = fmaf(-z, q_sum, sum[r]) * (act_to_float<BF16>(static_cast<uint16_t>(kp[u][r] & 0xffffu)) * unq);
            }
        }
        next(0);
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = act_to_float<BF16>(static_cast<uint16_t>(vp[e >> 2][e & 3] & 0xffffu));
        // every key of the step is seen by every query, unless the step lies at an end of the keys or a page is gone
        if (!(kb + kStepKeys <= min(s.first + q_lo + 1, hi) && (kb >= lo + n_minus || kb + kStepKeys <= p.sinks) && (id.a | id.b) >= 0)) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int key = kb + 16 * (e >> 2) + 4 * g + (e & 3);
                const bool seen = (key <= place) & (key < hi) & ((e >> 2 ? id.b : id.a) >= 0) & ((key > reach) | (key < p.sinks));
                sc[e] = seen ? sc[e] : -INFINITY;
                t[e] = seen ? t[e] : 0.0f;                       // (what lies in unused places may be anything)
            }
        }
        float mx = sc[0], tx = t[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) { mx = fmaxf(mx, sc[e]); tx = fmaxf(tx, t[e]); }
        if (__any((mx - m_run > kDecodeHead) | (tx > t_ref))) {
            mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));              // the column's largest: all its lanes move together
            tx = fmaxf(tx, __shfl_xor(tx, 16, 64));
            tx = fmaxf(tx, __shfl_xor(tx, 32, 64));
            const float m_new = mx - m_run > kDecodeHead ? mx : m_run;
            const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
            // the next power of two but one
            const float t_new = tx > t_ref ? fminf(ldexpf(1.0f, static_cast<int>(__float_as_uint(tx) >> 23) - 127 + 2), 0x1p126f) : t_ref;
            const float beta = alpha * (t_ref * (1.0f / t_new));
            l_run *= alpha;
#pragma unroll
            for (int f = 0; f <= F; ++f)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[f][r] *= beta;
            m_run = m_new;
            t_ref = t_new;
            t_inv = kLift4 / t_new;
        }
        u32x4_t ph, zv;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const float p0 = __builtin_amdgcn_exp2f(sc[e] - m_run), p1 = __builtin_amdgcn_exp2f(sc[e + 1] - m_run);
            l_run += p0 + p1;
            ph[e >> 1] = Act16<false>::pack(p0 * (t[e] * t_inv), p1 * (t[e + 1] * t_inv));
            zv[e >> 1] = __builtin_amdgcn_perm(vp[e >> 2][(e & 3) + 1], vp[e >> 2][e & 3], 0x07060302u) & 0x000f000fu;   // (in unused places it may be anything)
        }
        o[F] = Act16<false>::mfma16(zv, ph, o[F]);
        // words 2 h, 2 h + 1 of a lane: columns F c + 4 h .. + 3 of its keys 4 g + {0, 1} and {2, 3}
#pragma unroll
        for (int h = 0; h < S / 2; ++h) {
            const u32x4_t w0 = codes4(vn[0][2 * h]), w1 = codes4(vn[0][2 * h + 1]), w2 = codes4(vn[1][2 * h]), w3 = codes4(vn[1][2 * h + 1]);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[4 * h + i] = Act16<false>::mfma16(u32x4_t{w0[i], w1[i], w2[i], w3[i]}, ph, o[4 * h + i]);
        }
        next(1);
    };
    if (s0 < s1) {
        Ids id = ids_of(s0), id_next = ids_of(s0 + 4);
        int kb = walk.key(s0);
        fetch(p.k, kb, id, k_off, kn, kp);
        fetch(p.v, kb, id, v_off, vn, vp);
        for (int st = s0; st < s1; st += 4) {
            const bool more = st + 4 < s1;
            const int kb_next = walk.key(st + 4);
            const Ids id_after = ids_of(st + 8);
            // (past the last step the buffers are empty: such loads touch nothing)
            if (!more) id_next = Ids{-1, -1};
            step(kb, id, [&](int what) {
                if (what == 0) {
                    fetch(p.k, kb_next, id_next, k_off, kn, kp);
                    __builtin_amdgcn_sched_barrier(0);
                } else {
                    __builtin_amdgcn_sched_barrier(0);
                    fetch(p.v, kb_next, id_next, v_off, vn, vp);
                }
            });
            kb = kb_next;
            id = id_next;
            id_next = id_after;
        }
    }

    // the four waves meet in LDS
    l_run += __shfl_xor(l_run, 16, 64);
    l_run += __shfl_xor(l_run, 32, 64);
    if (c < cols) {
        constexpr float UNIT = 0x1p24f / kLift4;                 // (apart from t_ref, which may be 2^126)
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int r = 0; r < 4; ++r) sm[wave][c][F * (4 * g + r) + f] = ((f & 1 ? o[f][r] * 0.0625f : o[f][r]) - o[F][r]) * UNIT * t_ref;
        if (g == 0) { sm[wave][c][D] = m_run; sm[wave][c][D + 1] = l_run; }
    }
    __syncthreads();
    // the launch that adds the chunk kernel's key ranges finds none in these rows
    if (p.take != 0 && p.ranges > 1 && (!SPANS || cur == seq_begin) && tid < cols) {
        const int i = (c0 + tid) / p.rep;
        p.part[((static_cast<size_t>(s.row0 + i) * p.nh + hk * p.rep + c0 + tid - i * p.rep) * p.ranges) * part_stride(D) + D + 2] = 0.0f;
    }
    // a piece that begins its span goes to the span's first place, another one (it reaches the span's end) to the second
    float* piece = SPANS ? p.span_part + ((static_cast<size_t>(hk) * p.spans + span) * 2 + (cur == begin ? 0 : 1)) * (kDecodeCols * part_stride(D)) : nullptr;
    if (SPANS && hk == 0 && tid == 0 && cur == seq_begin) {
        // the span of unit x is the last one that begins at or before it
        const int last = whole ? static_cast<int>(span) : static_cast<int>((static_cast<uint64_t>(seq_end) * static_cast<uint32_t>(spans) - 1) / static_cast<uint32_t>(total));
        p.pieces[b] = int4{static_cast<int>(span), last - static_cast<int>(span) + 1, cur == begin ? 0 : 1, 0};
    }
    for (int x = tid; x < cols * (D / 2); x += 256) {
        const int r = x / (D / 2), e = 2 * (x % (D / 2));
        float mn = kPagedNone;
#pragma unroll
        for (int w = 0; w < 4; ++w) mn = fmaxf(mn, sm[w][r][D]);
        float n0 = 0.0f, n1 = 0.0f, den = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = __builtin_amdgcn_exp2f(sm[w][r][D] - mn);
            n0 += sm[w][r][e] * f;
            n1 += sm[w][r][e + 1] * f;
            den += sm[w][r][D + 1] * f;
        }
        if (!whole) {
            float* dst = piece + r * part_stride(D);
            *reinterpret_cast<float2_t*>(dst + e) = float2_t{n0, n1};
            if (e == 0) *reinterpret_cast<float2_t*>(dst + D) = float2_t{mn, den};
        } else {
            const int i = (c0 + r) / p.rep, h = hk * p.rep + c0 + r - i * p.rep;
            const float inv = den != 0.0f ? 1.0f / den : 0.0f;   // a row that sees no key is zero
            *reinterpret_cast<uint32_t*>(p.out + (s.row0 + i) * p.out_stride + h * D + e) = Act16<BF16>::pack(n0 * inv, n1 * inv);
        }
    }
    if (SPANS && end > seq_end) {
        cur = seq_end;
        while (ends[++b] == cur) {}                              // (a later sequence holds unit `cur`)
        __syncthreads();                                         // the sums have been read
        goto again;
    }
}

template <int D, bool BF16>
static hipError_t decode4_form(const PagedAttnDev& a, hipStream_t stream) {
    if (a.spans > 0) {
        hipLaunchKernelGGL((paged4_decode_kernel<D, BF16, true>), dim3(a.nkv, a.spans), dim3(256), 0, stream, a);
        PagedAttnDev sums = a;
        sums.scale_log2 = 1.0f;                                  // (reference points of this kernel are scaled scores)
        return launch_paged_pieces(sums, D, BF16, stream);
    }
    // a sequence's columns next to each other: the workgroups that share its keys run together
    const dim3 grid(a.nkv, (a.cols + kDecodeCols - 1) / kDecodeCols, a.B);
    hipLaunchKernelGGL((paged4_decode_kernel<D, BF16, false>), grid, dim3(256), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_paged4_decode(const PagedAttnDev& a, int d, hipStream_t stream) {
    if (d == 128) return a.bf16 ? decode4_form<128, true>(a, stream) : decode4_form<128, false>(a, stream);
    return a.bf16 ? decode4_form<64, true>(a, stream) : decode4_form<64, false>(a, stream);
}

}  // namespace qtale
