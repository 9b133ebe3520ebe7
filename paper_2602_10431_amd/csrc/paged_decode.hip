// Attention over pages where few queries meet many keys: (query, head) pairs of a key/value head by sixteen, so a single token of up to 16 heads per
// kv head, or a few tokens.
//
// One workgroup of four waves per (sequence, kv head, 16 pairs), or per span of keys; the pairs are the 16 columns of both products.  A wave's step is 32 keys:
//   S = K Q^T: two fragments of 16 keys; lane (c, g) = (lane % 16, lane / 16) holds 16 bytes of key c per instruction, an operand as loaded;
//   O^T += V^T P^T: the scores of keys 4 g + r of both fragments are in lane (c, g), which is operand order if product index 8 g + e is key
//   4 g + e (e < 4) or 16 + 4 g + e - 4.  Lane (c, g) loads columns F c .. F c + F - 1 of those eight keys; byte permutes make fragments.
// 16 consecutive keys lie in one page whatever its size, so a fragment has one base address, kept in scalar registers as a buffer whose length
// ends at the last key: loads past it, and of pages that are gone, return zeros (a zero probability times what lies in unused memory, NaN
// maybe, would be NaN).  Probabilities are 32-bit sums; as operands they go in as two 16-bit terms, p = hi + lo, through two products into one
// accumulator, which leaves 2^-16 (bf16) or 2^-22 of them (fp16; or 2^-37 of the largest, kDecodeLift): the matrix cores have time (about a tenth of
// the stream's), and a bf16 probability alone would add as much error as the output's own rounding.
// Calls of more than 16 pairs per sequence come here while their workgroups fit the chip about once: each reads the sequence's keys, from L2 but for
// the first, and the longest is done sooner than a workgroup of the chunk kernel, whose waves take a tile after the other (plan_paged_attention).
// What bounds it is the stream of keys and values, and a CU takes in no more than about 50 GB/s (1 x 3000 keys, 32 workgroups: 33 us, whatever
// the waves per workgroup).  So with few (sequence, kv head) pairs the keys of the call, laid end to end over its sequences, are cut into equally
// long spans, one per workgroup that fits the chip; a span may end one sequence and begin the next, and a second launch adds the pieces.
// Measured: 64 sequences of 2048 keys, 32 kv heads 312 us, 6.9 TB/s; 33 of 3000 (500 to 4500), 8 kv heads of 4 query heads 69 us, 5.9 TB/s, 4.6 us of it
// the second launch; 1 of 700, 32 kv heads 10.8 us, where a launch alone takes 4 and the rest is the 350 KB per workgroup at a CU's rate.
#include <algorithm>

#include "paged_attn.h"

namespace qtale {

constexpr int kStepKeys = 32;                    // per wave
constexpr int kUnitSteps = 4;                    // spans are cut at multiples of this: a step per wave

// Units of a sequence in a call with spans; 0: not this kernel's.  A sequence without keys has one, in which its zeros are written.
__device__ __forceinline__ int seq_units(const PagedAttnDev& p, int b) {
    const SeqView s(p, b);
    if (s.n == 0 || (p.take != 0 && s.n * p.rep > kDecodeCols)) return 0;
    return max((KeySteps<kStepKeys>(s.first, s.first + s.n - 1, s.len, p.window, p.sinks).steps + kUnitSteps - 1) / kUnitSteps, 1);
}

// STREAM: keys as non-temporal loads too, not only values.  Where the workgroups fill the chip evenly (spans, or many of them) the stream gains, us
// without / with: 33 x 3000 keys of 8 kv heads 74 / 69, 20 x 6000 85 / 80, heads of 64 49 / 47; 64 x 2048 of 32 kv heads 324 / 313, 128 x 1000 of 8
// 81.7 / 79.3; where some CUs are left with one workgroup more than others those have less of it each: 48 x 1028 37.6 / 40.8, 100 x 2000 139 / 142.
// Heads of 64 gain it with spans only, however many workgroups: 128 x 1000 keys of 8 kv heads 43.0 / 42.6, 128 x 2000 81.1 / 81.7, 150 x 1500 73.2 / 74.7,
// 256 x 1000 81.9 / 82.7, 200 x 2000 of 1000 to 3000 137 / 143.
template <int D, bool BF16, bool SPANS, bool STREAM>
__global__ void __launch_bounds__(256, D == 64 ? 4 : 3)
paged_decode_kernel(PagedAttnDev p) {
    using A = Act16<BF16>;
    constexpr int S = D / 32;                    // k-steps of the scores
    constexpr int F = D / 16;                    // output fragments, and columns of V per lane
    typedef uint32_t VWords __attribute__((ext_vector_type(F / 2)));
    const int hk = blockIdx.x;                   // kv heads fastest
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4;
    __shared__ float sm[4][kDecodeCols][D + 2];
    __shared__ uint32_t s_redo;                                  // columns whose sum is not finite
    __shared__ int ends[SPANS ? kSpanSeqs : 1];                  // units up to and with sequence b

    int b = blockIdx.z, cur = 0, end = 0, total = 0, spans = 1;
    uint32_t span = 0;
    if (SPANS) {
        for (int b0 = 0; b0 < p.B; b0 += 64) {
            int sum = b0 + lane < p.B ? seq_units(p, b0 + lane) : 0;
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
    u32x4_t q[S];
    const uint16_t* qrow = p.q + (s.row0 + qi) * p.q_stride + head * D + 8 * g;
#pragma unroll
    for (int k = 0; k < S; ++k) q[k] = *reinterpret_cast<const u32x4_t*>(qrow + 32 * k);

    const int s0 = first_step + wave, s1 = last_step;            // this wave's steps: s0, s0 + 4, ...
    const PageRow pages(p, s.slot);
    const int hi = walk.hi, lo = walk.lo, n_minus = q_hi - q_lo;
    const size_t head_elems = static_cast<size_t>(D) << p.shift;

    // page ids of the two fragments of a step: read one step before the loads that use them
    struct Ids { int a, b; };
    auto ids_of = [&](int st) {
        const int kb = walk.key(min(st, walk.steps - 1));
        return Ids{pages.at(kb), pages.at(kb + 16)};
    };
    auto buffer = [&](const uint16_t* pool, int page, int key) {
        const int rows = page < 0 ? 0 : min(max(hi - key, 0), 16);
        const size_t at = (static_cast<size_t>(max(page, 0)) * p.nkv + hk) * head_elems + static_cast<size_t>(key & ((1 << p.shift) - 1)) * D;
        return buffer_of(pool + at, rows * (2 * D));
    };
    u32x4_t kn[2][S];
    VWords vn[8];
    const uint32_t k_off = c * (2 * D) + 16 * g, v_off = 4 * g * (2 * D) + 2 * F * c;
    auto fetch_k = [&](int kb, Ids id) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const auto buf = buffer(p.k, u ? id.b : id.a, kb + 16 * u);
#pragma unroll
            for (int k = 0; k < S; ++k) kn[u][k] = __builtin_amdgcn_raw_buffer_load_b128(buf, k_off + 64 * k, 0, STREAM ? 2 : 0);
        }
    };
    auto fetch_v = [&](int kb, Ids id) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const auto buf = buffer(p.v, u ? id.b : id.a, kb + 16 * u);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (D == 128) vn[4 * u + e] = __builtin_amdgcn_raw_buffer_load_b128(buf, v_off + 2 * D * e, 0, 2);   // read once: non-temporal
                else vn[4 * u + e] = __builtin_amdgcn_raw_buffer_load_b64(buf, v_off + 2 * D * e, 0, 2);
            }
        }
    };
    auto scores = [&](const u32x4_t* k) {
        float4_t sum[S / 2];
#pragma unroll
        for (int i = 0; i < S; i += 2) {
            sum[i / 2] = A::mfma16(k[i], q[i], float4_t{0.f, 0.f, 0.f, 0.f});
            sum[i / 2] = A::mfma16(k[i + 1], q[i + 1], sum[i / 2]);
        }
        return S == 2 ? sum[0] : sum[0] + sum[S / 2 - 1];
    };
    const float sc = p.scale_log2;               // probabilities are 2^((score - m_run) sc + lift)
    constexpr float LIFT = kDecodeLift<BF16>;
    float m_run = kPagedNone, l_run = 0.0f;
    float4_t o[F];
#pragma unroll
    for (int f = 0; f < F; ++f) o[f] = float4_t{0.f, 0.f, 0.f, 0.f};
    auto absorb = [&](const float4_t& st0, const float4_t& st1) {   // 32 keys; masked scores are -inf
        float mx = fmaxf(fmaxf(fmaxf(st0[0], st0[1]), fmaxf(st0[2], st0[3])), fmaxf(fmaxf(st1[0], st1[1]), fmaxf(st1[2], st1[3])));
        if (__any((mx - m_run) * sc > kDecodeHead)) {
            mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));              // the column's largest score: all its lanes move together
            const float m_new = (mx - m_run) * sc > kDecodeHead ? mx : m_run;
            const float alpha = __builtin_amdgcn_exp2f((m_run - m_new) * sc);
            l_run *= alpha;
#pragma unroll
            for (int f = 0; f < F; ++f)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[f][r] *= alpha;
            m_run = m_new;
        }
        u32x4_t ph, pl;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const float p0 = __builtin_amdgcn_exp2f(fmaf((e < 4 ? st0[e & 3] : st1[e & 3]) - m_run, sc, LIFT));
            const float p1 = __builtin_amdgcn_exp2f(fmaf((e < 4 ? st0[(e & 3) + 1] : st1[(e & 3) + 1]) - m_run, sc, LIFT));
            l_run += p0 + p1;
            const uint32_t h = A::pack(p0, p1);
            ph[e >> 1] = h;
            pl[e >> 1] = A::pack(p0 - A::low(h), p1 - A::high(h));
        }
#pragma unroll
        for (int f = 0; f < F; ++f) {
            u32x4_t va;
#pragma unroll
            for (int e = 0; e < 8; e += 2) va[e >> 1] = __builtin_amdgcn_perm(vn[e + 1][f >> 1], vn[e][f >> 1], f & 1 ? 0x07060302u : 0x05040100u);
            o[f] = A::mfma16(va, ph, o[f]);
            o[f] = A::mfma16(va, pl, o[f]);
        }
    };
    auto step = [&](int kb, Ids id, auto next) {
        float4_t st[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) st[u] = scores(kn[u]);
        next(0);
        // every key of the step is seen by every query, unless the step lies at an end of the keys or a page is gone
        if (!(kb + kStepKeys <= min(s.first + q_lo + 1, hi) && (kb >= lo + n_minus || kb + kStepKeys <= p.sinks) && (id.a | id.b) >= 0)) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int key = kb + 16 * u + 4 * g + r;
                    const bool seen = (key <= place) & (key < hi) & ((u ? id.b : id.a) >= 0) & ((key > reach) | (key < p.sinks));
                    st[u][r] = seen ? st[u][r] : -INFINITY;
                    const bool out = (key < lo) & (key >= p.sinks);   // before every query's window: whatever is there stays out of the products
#pragma unroll
                    for (int w = 0; w < F / 2; ++w) vn[4 * u + r][w] = out ? 0u : vn[4 * u + r][w];
                }
        }
        absorb(st[0], st[1]);
        next(1);
    };
    if (s0 < s1) {
        Ids id = ids_of(s0), id_next = ids_of(s0 + 4);
        int kb = walk.key(s0);
        fetch_k(kb, id);
        fetch_v(kb, id);
        for (int st = s0; st < s1; st += 4) {
            const bool more = st + 4 < s1;
            const int kb_next = walk.key(st + 4);
            const Ids id_after = ids_of(st + 8);
            // (past the last step the buffers are empty: such loads touch nothing)
            if (!more) id_next = Ids{-1, -1};
            step(kb, id, [&](int what) {
                if (what == 0) {
                    fetch_k(kb_next, id_next);
                    __builtin_amdgcn_sched_barrier(0);
                } else {
                    __builtin_amdgcn_sched_barrier(0);
                    fetch_v(kb_next, id_next);
                }
            });
            kb = kb_next;
            id = id_next;
            id_next = id_after;
        }
    }

    // the four waves meet in LDS
    if (tid == 0) s_redo = 0;
    l_run += __shfl_xor(l_run, 16, 64);
    l_run += __shfl_xor(l_run, 32, 64);
    if (c < cols) {
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int r = 0; r < 4; ++r) sm[wave][c][F * (4 * g + r) + f] = o[f][r];
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
    for (int t = tid; t < cols * (D / 2); t += 256) {
        const int r = t / (D / 2), e = 2 * (t % (D / 2));
        float mn = kPagedNone;
#pragma unroll
        for (int w = 0; w < 4; ++w) mn = fmaxf(mn, sm[w][r][D]);
        float n0 = 0.0f, n1 = 0.0f, den = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = __builtin_amdgcn_exp2f((sm[w][r][D] - mn) * sc);
            n0 += sm[w][r][e] * f;
            n1 += sm[w][r][e + 1] * f;
            den += sm[w][r][D + 1] * f;
        }
        if (n_minus > 0 && fmaf(n0, 0.0f, fmaf(n1, 0.0f, den * 0.0f)) != 0.0f) atomicOr(&s_redo, 1u << r);
        if (!whole) {
            float* dst = piece + r * part_stride(D);
            *reinterpret_cast<float2_t*>(dst + e) = float2_t{n0, n1};
            if (e == 0) *reinterpret_cast<float2_t*>(dst + D) = float2_t{mn, den};
        } else {
            const int i = (c0 + r) / p.rep, h = hk * p.rep + c0 + r - i * p.rep;
            const float inv = den != 0.0f ? 1.0f / den : 0.0f;   // a row that sees no key is zero
            *reinterpret_cast<uint32_t*>(p.out + (s.row0 + i) * p.out_stride + h * D + e) = A::pack(n0 * inv, n1 * inv);
        }
    }
    // Several queries: a value that is not finite, seen by the later ones, has met the earlier ones' zeros (redo_column).  A single query meets
    // no key that it does not see.
    if (n_minus > 0) {
        __syncthreads();
        uint32_t redo = s_redo;
#pragma unroll 1
        for (int j = 0; redo != 0; ++j, redo &= redo - 1) {
            if ((j & 3) != wave) continue;
            const int r = __ffs(static_cast<int>(redo)) - 1, i = (c0 + r) / p.rep, h = hk * p.rep + c0 + r - i * p.rep;
            float num[D / 64], m, l;
            redo_column<D, BF16>(p, walk, s.slot, hk, p.q + (s.row0 + i) * p.q_stride + h * D, s.first + i, first_step, last_step, LIFT, num, &m, &l);
            put_column<D, BF16>(num, m, l, whole ? nullptr : piece + r * part_stride(D), p.out + (s.row0 + i) * p.out_stride + h * D);
        }
    }
    if (SPANS && end > seq_end) {
        cur = seq_end;
        while (ends[++b] == cur) {}                              // (a later sequence holds unit `cur`)
        __syncthreads();                                         // the sums have been read
        goto again;
    }
}

// Adds the pieces of a (sequence, kv head, column): 1024 / D groups of D / 4 lanes take every so manieth piece and meet in LDS.
template <int D, bool BF16>
__global__ void __launch_bounds__(256)
paged_pieces_kernel(PagedAttnDev p) {
    constexpr int W = part_stride(D), LANES = D / 4, GROUPS = 256 / LANES;
    __shared__ float4_t nums[GROUPS][LANES];
    __shared__ float2_t stats[GROUPS];
    const int hk = blockIdx.x, b = blockIdx.y, r = blockIdx.z, lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
    const int4 at = p.pieces[b];                                 // (of a sequence that is not the decode kernel's: not written, not used)
    const int row0 = p.offs[b], n = p.offs[b + 1] - row0, cols = n * p.rep;
    if (n <= 0 || cols > kDecodeCols || r >= cols || at.y <= 1) return;
    const float* span0 = p.span_part + (static_cast<size_t>(hk) * p.spans + at.x) * (2 * kDecodeCols * W);
    RangeSum sum{p.scale_log2};
    sum.add_all<D>(group, GROUPS, at.y, lane, [&](int z) { return span0 + (static_cast<size_t>(2 * z + (z == 0 ? at.z : 0)) * kDecodeCols + r) * W; });
    nums[group][lane] = sum.num;
    if (lane == 0) stats[group] = float2_t{sum.m, sum.den};
    __syncthreads();
    if (group != 0) return;
    float4_t x[GROUPS - 1];
    float2_t s[GROUPS - 1];
    bool on[GROUPS - 1];
#pragma unroll
    for (int k = 0; k < GROUPS - 1; ++k) { x[k] = nums[k + 1][lane]; s[k] = stats[k + 1]; on[k] = k + 1 < at.y; }
    sum.add<GROUPS - 1>(x, s, on);
    const int i = r / p.rep, h = hk * p.rep + r - i * p.rep;
    sum.put<BF16>(p.out + (row0 + i) * p.out_stride + h * D, lane);
}

// (a.cols <= 16)
hipError_t launch_paged_pieces(const PagedAttnDev& a, int d, int bf16, hipStream_t stream) {
    const dim3 grid(a.nkv, a.B, a.cols), block(256);
    if (d == 128) {
        if (bf16) hipLaunchKernelGGL((paged_pieces_kernel<128, true>), grid, block, 0, stream, a);
        else hipLaunchKernelGGL((paged_pieces_kernel<128, false>), grid, block, 0, stream, a);
    } else {
        if (bf16) hipLaunchKernelGGL((paged_pieces_kernel<64, true>), grid, block, 0, stream, a);
        else hipLaunchKernelGGL((paged_pieces_kernel<64, false>), grid, block, 0, stream, a);
    }
    return hipGetLastError();
}

template <int D, bool BF16>
static hipError_t decode_form(const PagedAttnDev& a, hipStream_t stream) {
    // a sequence's columns next to each other: the workgroups that share its keys run together
    const dim3 grid(a.nkv, (a.cols + kDecodeCols - 1) / kDecodeCols, a.B);
    if (a.spans > 0) {
        hipLaunchKernelGGL((paged_decode_kernel<D, BF16, true, true>), dim3(a.nkv, a.spans), dim3(256), 0, stream, a);
        return launch_paged_pieces(a, D, BF16, stream);
    } else if (D == 128 && a.stream_keys) {
        hipLaunchKernelGGL((paged_decode_kernel<D, BF16, false, D == 128>), grid, dim3(256), 0, stream, a);
    } else {
        hipLaunchKernelGGL((paged_decode_kernel<D, BF16, false, false>), grid, dim3(256), 0, stream, a);
    }
    return hipGetLastError();
}

hipError_t launch_paged_decode(const PagedAttnDev& a, int d, int bf16, hipStream_t stream) {
    if (d == 128) return bf16 ? decode_form<128, true>(a, stream) : decode_form<128, false>(a, stream);
    return bf16 ? decode_form<64, true>(a, stream) : decode_form<64, false>(a, stream);
}

}  // namespace qtale
