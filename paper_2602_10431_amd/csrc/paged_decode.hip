// Attention over pages where few queries meet many keys: at most 16 (query, head) pairs per key/value head, so a single token of up to 16
// heads per kv head, or a few tokens.
//
// One workgroup of four waves per (sequence, kv head[, key range]); the pairs are the 16 columns of both products.  A wave's step is 32 keys:
//   S = K Q^T: two fragments of 16 keys; lane (c, g) = (lane % 16, lane / 16) holds 16 bytes of key c per instruction, an operand as loaded;
//   O^T += V^T P^T: the scores of keys 4 g + r of both fragments are in lane (c, g), which is operand order if product index 8 g + e is key
//   4 g + e (e < 4) or 16 + 4 g + e - 4.  Lane (c, g) loads columns F c .. F c + F - 1 of those eight keys; byte permutes make fragments.
// 16 consecutive keys lie in one page whatever its size, so a fragment has one base address, kept in scalar registers as a buffer whose length
// ends at the last key: loads past it, and of pages that are gone, return zeros (a zero probability times what lies in unused memory, NaN
// maybe, would be NaN).  Probabilities are 32-bit sums; as operands they go in as two 16-bit terms, p = hi + lo, through two products into one
// accumulator, which leaves 2^-16 (bf16) or 2^-22 of them: the matrix cores have time (about a tenth of the stream's), and a bf16 probability
// alone would add as much error as the output's own rounding.
// What bounds it is the stream of keys and values.  Few (sequence, kv head) pairs: the keys of the call are cut into ranges of equal length so
// that `target` workgroups run, and a second launch adds the ranges' sums.
#include <algorithm>

#include "paged_attn.h"

namespace qtale {

constexpr int kStepKeys = 32;                    // per wave
constexpr int kRangeSteps = kDecodeRangeKeys / kStepKeys;   // two per wave

// Steps of a sequence's call, and how a call with key ranges is cut: ranges of `per` steps, numbered through the sequences in order.
__device__ __forceinline__ int seq_steps(const PagedAttnDev& p, int b, bool* mine) {
    const SeqView s(p, b);
    *mine = s.n > 0 && (p.take == 0 || s.n * p.rep <= kDecodeCols);
    return *mine ? KeySteps<kStepKeys>(s.first, s.first + s.n - 1, s.len, p.window, p.sinks).steps : 0;
}

__device__ __forceinline__ int wave_total(int v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

template <int D, bool BF16, bool SPLIT>
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

    int b = blockIdx.y, z = 0, ranges = 1, per = 0;
    if (SPLIT) {
        int total = 0;
        for (int b0 = 0; b0 < p.B; b0 += 64) {
            bool mine = false;
            total += wave_total(b0 + lane < p.B ? seq_steps(p, b0 + lane, &mine) : 0);
        }
        const int wanted = max(p.target / p.nkv, 1);             // ranges of the call, per kv head
        per = ((total + wanted - 1) / wanted + kRangeSteps - 1) / kRangeSteps * kRangeSteps;
        per = max(per, kRangeSteps);
        int item = blockIdx.y, found = -1;
        for (int b0 = 0; b0 < p.B && found < 0; b0 += 64) {
            bool mine = false;
            const int steps = b0 + lane < p.B ? seq_steps(p, b0 + lane, &mine) : 0;
            const int n = mine ? min(max((steps + per - 1) / per, 1), p.ranges) : 0;
            int before = n;                                      // inclusive prefix sum over the lanes
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int y = __shfl_up(before, o, 64);
                if (lane >= o) before += y;
            }
            const uint64_t past = __ballot(before > item);
            if (past) {
                const int at = __ffsll(static_cast<long long>(past)) - 1;
                found = b0 + at;
                ranges = __shfl(n, at, 64);
                z = item - (__shfl(before, at, 64) - ranges);
            } else {
                item -= __shfl(before, 63, 64);
            }
        }
        if (found < 0) return;
        b = __builtin_amdgcn_readfirstlane(found);
        z = __builtin_amdgcn_readfirstlane(z);
        ranges = __builtin_amdgcn_readfirstlane(ranges);
    }
    SeqView s(p, b);
    s.uniform();
    const int cols = s.n * p.rep;
    if (s.n == 0 || (p.take != 0 && cols > kDecodeCols)) return;
    const int col = min(c, cols - 1);                            // this lane's column: query col / rep, head col % rep
    const int qi = col / p.rep, head = hk * p.rep + col - qi * p.rep;
    const int place = s.first + qi;                              // the query's place in its slot
    const int reach = p.window > 0 ? place - p.window : INT32_MIN;   // keys after it are in its window
    u32x4_t q[S];
    const uint16_t* qrow = p.q + (s.row0 + qi) * p.q_stride + head * D + 8 * g;
#pragma unroll
    for (int k = 0; k < S; ++k) q[k] = *reinterpret_cast<const u32x4_t*>(qrow + 32 * k);

    const KeySteps<kStepKeys> walk(s.first, s.first + s.n - 1, s.len, p.window, p.sinks);
    int s0 = wave, s1 = walk.steps;                              // this wave's steps: s0, s0 + 4, ...
    if (SPLIT) {
        s0 += z * per;
        if (z < ranges - 1) s1 = min(s1, (z + 1) * per);         // (the last range takes what is left)
    }
    const PageRow pages(p, s.slot);
    const int first = s.first, hi = walk.hi, lo = walk.lo, n_minus = s.n - 1;
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
            for (int k = 0; k < S; ++k) kn[u][k] = __builtin_amdgcn_raw_buffer_load_b128(buf, k_off + 64 * k, 0, 0);
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
    constexpr float kTop = 4.0f;                 // probabilities are 2^(score - m_run), at most 2^kTop
    const float sc = p.scale_log2;
    float m_run = kPagedNone, l_run = 0.0f;
    float4_t o[F];
#pragma unroll
    for (int f = 0; f < F; ++f) o[f] = float4_t{0.f, 0.f, 0.f, 0.f};
    auto absorb = [&](const float4_t& st0, const float4_t& st1) {   // 32 keys; masked scores are -inf
        float mx = fmaxf(fmaxf(fmaxf(st0[0], st0[1]), fmaxf(st0[2], st0[3])), fmaxf(fmaxf(st1[0], st1[1]), fmaxf(st1[2], st1[3]))) * sc;
        if (__any(mx > m_run + kTop)) {
            mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));              // the column's largest score: all its lanes move together
            const float m_new = mx > m_run + kTop ? mx : m_run;
            const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
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
            const float p0 = __builtin_amdgcn_exp2f(fmaf(e < 4 ? st0[e & 3] : st1[e & 3], sc, -m_run));
            const float p1 = __builtin_amdgcn_exp2f(fmaf(e < 4 ? st0[(e & 3) + 1] : st1[(e & 3) + 1], sc, -m_run));
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
        if (!(kb + kStepKeys <= min(first + 1, hi) && (kb >= lo + n_minus || kb + kStepKeys <= p.sinks) && (id.a | id.b) >= 0)) {
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
    __shared__ float sm[4][kDecodeCols][D + 2];
    __shared__ uint32_t s_redo;                                  // columns whose sum is not finite
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
    for (int t = tid; t < min(cols, kDecodeCols) * (D / 2); t += 256) {
        const int r = t / (D / 2), e = 2 * (t % (D / 2));
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
        const int i = r / p.rep, h = hk * p.rep + r - i * p.rep;
        if (n_minus > 0 && fmaf(n0, 0.0f, fmaf(n1, 0.0f, den * 0.0f)) != 0.0f) atomicOr(&s_redo, 1u << r);
        if (SPLIT && ranges > 1) {
            float* dst = p.part + (static_cast<size_t>(s.row0 + i) * p.nh + h) * p.n_split * part_stride(D) + static_cast<size_t>(z) * part_stride(D);
            *reinterpret_cast<float2_t*>(dst + e) = float2_t{n0, n1};
            if (e == 0) *reinterpret_cast<float4_t*>(dst + D) = float4_t{mn, den, static_cast<float>(ranges), 0.0f};
        } else {
            const float inv = den != 0.0f ? 1.0f / den : 0.0f;   // a row that sees no key is zero
            *reinterpret_cast<uint32_t*>(p.out + (s.row0 + i) * p.out_stride + h * D + e) = A::pack(n0 * inv, n1 * inv);
            if (SPLIT && e == 0) p.part[(static_cast<size_t>(s.row0 + i) * p.nh + h) * p.n_split * part_stride(D) + D + 2] = 1.0f;
        }
    }
    // Several queries: a value that is not finite, seen by the later ones, has met the earlier ones' zeros (redo_column).  A single query meets
    // no key that it does not see.
    if (n_minus == 0) return;
    __syncthreads();
    uint32_t redo = s_redo;
    const int begin = SPLIT ? z * per : 0, end = SPLIT && z < ranges - 1 ? min((z + 1) * per, walk.steps) : walk.steps;
#pragma unroll 1
    for (int j = 0; redo != 0; ++j, redo &= redo - 1) {
        if ((j & 3) != wave) continue;
        const int r = __ffs(static_cast<int>(redo)) - 1, i = r / p.rep, h = hk * p.rep + r - i * p.rep;
        float num[D / 64], m, l;
        redo_column<D, BF16>(p, walk, s.slot, hk, p.q + (s.row0 + i) * p.q_stride + h * D, s.first + i, begin, end, num, &m, &l);
        put_column<D, BF16>(p, s.row0 + i, h, z, ranges, num, m, l);
    }
}

// Adds the key ranges of a (row, head): one wave each.  The reference point of a range without keys lets it drop out.
template <int D, bool BF16>
__global__ void __launch_bounds__(256)
paged_combine_kernel(PagedAttnDev p, int T) {
    const int pair = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (pair >= T * p.nh || pair / p.nh >= p.offs[p.B]) return;
    constexpr int E = D / 64, W = part_stride(D);
    const float* src = p.part + static_cast<size_t>(pair) * p.n_split * W;
    const int ranges = min(static_cast<int>(src[D + 2]), p.n_split);
    if (ranges <= 1) return;
    float m = kPagedNone;
    for (int r = lane; r < ranges; r += 64) m = fmaxf(m, src[static_cast<size_t>(r) * W + D]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    float num[E], den = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) num[e] = 0.0f;
#pragma unroll 4
    for (int r = 0; r < ranges; ++r) {
        const float* row = src + static_cast<size_t>(r) * W;
        const float f = __builtin_amdgcn_exp2f(row[D] - m);
#pragma unroll
        for (int e = 0; e < E; ++e) num[e] += row[E * lane + e] * f;
        den += row[D + 1] * f;
    }
    const float inv = den != 0.0f ? 1.0f / den : 0.0f;
    uint16_t* out = p.out + (pair / p.nh) * p.out_stride + (pair % p.nh) * D;
    if constexpr (E == 2) *reinterpret_cast<uint32_t*>(out + 2 * lane) = Act16<BF16>::pack(num[0] * inv, num[1] * inv);
    else out[lane] = static_cast<uint16_t>(Act16<BF16>::pack(num[0] * inv, 0.0f) & 0xffffu);
}

template <int D, bool BF16>
static hipError_t decode_form(const PagedAttnDev& a, hipStream_t stream) {
    const bool split = a.n_split > 1;
    // every sequence has a range, and the target is passed by less than one per sequence
    const dim3 grid(a.nkv, split ? a.B + std::max(a.target / a.nkv, 1) : a.B), block(256);
    if (split) hipLaunchKernelGGL((paged_decode_kernel<D, BF16, true>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((paged_decode_kernel<D, BF16, false>), grid, block, 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_paged_decode(const PagedAttnDev& a, int d, int bf16, hipStream_t stream) {
    if (d == 128) return bf16 ? decode_form<128, true>(a, stream) : decode_form<128, false>(a, stream);
    return bf16 ? decode_form<64, true>(a, stream) : decode_form<64, false>(a, stream);
}

hipError_t launch_paged_combine(const PagedAttnDev& a, int d, int bf16, int T, hipStream_t stream) {
    const dim3 grid((static_cast<int64_t>(T) * a.nh + 3) / 4), block(256);
    if (d == 128) {
        if (bf16) hipLaunchKernelGGL((paged_combine_kernel<128, true>), grid, block, 0, stream, a, T);
        else hipLaunchKernelGGL((paged_combine_kernel<128, false>), grid, block, 0, stream, a, T);
    } else {
        if (bf16) hipLaunchKernelGGL((paged_combine_kernel<64, true>), grid, block, 0, stream, a, T);
        else hipLaunchKernelGGL((paged_combine_kernel<64, false>), grid, block, 0, stream, a, T);
    }
    return hipGetLastError();
}

}  // namespace qtale
