// Attention over pages in 4 bits, one wave per (row, head): a lane scores a key at a time and owns d / 64 columns of the result.
#include "paged4.h"
#include "paged_attn.h"

namespace qtale {

template <int D, bool BF16>
__global__ void __launch_bounds__(64)
paged4_simple_kernel(PagedAttnDev p, int T) {
    constexpr int E = D / 64;
    const int row = blockIdx.x, head = blockIdx.y, lane = threadIdx.x;
    if (row >= p.offs[p.B]) return;
    int b = 0;
    for (int b0 = 0; b0 < p.B; b0 += 64) b += __popcll(__ballot(b0 + lane < p.B && p.offs[min(b0 + lane, p.B - 1) + 1] <= row));
    if (b >= p.B) return;
    const SeqView s(p, b);
    const int place = s.first + row - s.row0, hk = head / p.rep;
    const KeySteps<64> walk(place, place, s.len, p.window, p.sinks);
    const Block4 block{D, p.shift};
    __shared__ float q[D];
    float qsum = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        q[lane + 64 * e] = act_to_float<BF16>(p.q[row * p.q_stride + head * D + lane + 64 * e]);
        qsum += q[lane + 64 * e];
    }
    qsum = wave_sum(qsum);
    __syncthreads();
    float m = kPagedNone, l = 0.0f, num[E] = {};
    for (int st = 0; st < walk.steps; ++st) {
        const int key = walk.key(st) + lane;
        int page = -1;
        if (key <= place && key < walk.hi && (p.window == 0 || key > place - p.window || key < p.sinks))
            page = p.table[static_cast<size_t>(s.slot) * p.max_pages + min(key >> p.shift, p.max_pages - 1)];
        const bool seen = static_cast<uint32_t>(page) < static_cast<uint32_t>(p.n_pages);
        uint64_t who = __ballot(seen);
        if (who == 0) continue;
        const int t = key & ((1 << p.shift) - 1);
        float score = -INFINITY, vs = 0.0f, vz = 0.0f;
        size_t base = 0;
        if (seen) {
            base = (static_cast<size_t>(page) * p.nkv + hk) * block.bytes();
            const char* k = reinterpret_cast<const char*>(p.k) + base;
            float sum = 0.0f;
            for (int w = 0; w < D / 8; ++w) {
                const uint32_t x = *reinterpret_cast<const uint32_t*>(k + block.key(t) + 4 * w);
                for (int e = 0; e < 8; ++e) sum = fmaf(static_cast<float>(x >> (4 * (e >> 1) + 16 * (e & 1)) & 15u), q[8 * w + e], sum);
            }
            const uint32_t kp = *reinterpret_cast<const uint32_t*>(k + block.param(t));
            const uint32_t vp = *reinterpret_cast<const uint32_t*>(reinterpret_cast<const char*>(p.v) + base + block.param(t));
            score = (sum - static_cast<float>(kp >> 16) * qsum) * scale4(kp, BF16);
            vs = scale4(vp, BF16);
            vz = static_cast<float>(vp >> 16);
        }
        const float m_new = fmaxf(m, wave_max(score)), alpha = __builtin_amdgcn_exp2f((m - m_new) * p.scale_log2);
        const float w = seen ? __builtin_amdgcn_exp2f((score - m_new) * p.scale_log2) : 0.0f;
        m = m_new;
        l = l * alpha + wave_sum(w);
        for (int e = 0; e < E; ++e) num[e] *= alpha;
        for (; who != 0; who &= who - 1) {
            const int j = __ffsll(static_cast<long long>(who)) - 1;
            const float wj = __shfl(w, j, 64) * __shfl(vs, j, 64), zj = __shfl(vz, j, 64);
            const size_t at = __shfl(base, j, 64);
            const int tj = __shfl(t, j, 64), col = E * lane;
            const uint32_t x = *reinterpret_cast<const uint16_t*>(reinterpret_cast<const char*>(p.v) + at + block.value(tj, col & ~3)) >> (4 * (col & 3));
            for (int e = 0; e < E; ++e) num[e] = fmaf(wj, static_cast<float>(x >> (4 * e) & 15u) - zj, num[e]);
        }
    }
    put_column<D, BF16>(num, m, l, nullptr, p.out + row * p.out_stride + head * D);
}

hipError_t launch_paged4_simple(const PagedAttnDev& a, int d, int T, hipStream_t stream) {
    const dim3 grid(T, a.nh), block(64);
    if (d == 128) {
        if (a.bf16) hipLaunchKernelGGL((paged4_simple_kernel<128, true>), grid, block, 0, stream, a, T);
        else hipLaunchKernelGGL((paged4_simple_kernel<128, false>), grid, block, 0, stream, a, T);
    } else {
        if (a.bf16) hipLaunchKernelGGL((paged4_simple_kernel<64, true>), grid, block, 0, stream, a, T);
        else hipLaunchKernelGGL((paged4_simple_kernel<64, false>), grid, block, 0, stream, a, T);
    }
    return hipGetLastError();
}

}  // namespace qtale
