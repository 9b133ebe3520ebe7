// Low-rank adapters of many requests beside a shared projection: y_i += scale[a] up_a (down_a A_i), a the adapter of row i.
//
// Both products run on the matrix cores in tiles of 16 rows (or 64) that know nothing of the rows' order: a tile walks the adapters that occur in it, and a
// row takes the result of its own and leaves the others'.  A decode step's tile of 16 requests reads each of its adapters once, which has to be; a
// prompt's tile meets one.  Operands of rows that the result leaves out cannot reach it, whatever they hold (a select, not a product with zero).
//   inner  D[r][row] = down_a A^T, K cut over the waves of a workgroup and over workgroups, so that a few requests fill the chip;
//          a part's sums are written, and added by the second kernel: no atomics, the same bits every time
//   outer  D[n][row] = up_a inner^T: inner values go in as fp16 relative to their row's power of two, off by 2^-11 of each (or 2^-36 of the
//          row's largest), as the rows that they come from are; the sum with the shared product, which stays in 32 bits until then, is rounded once
#include <algorithm>

#include "lora.h"
#include "qtale_dev.h"

namespace qtale {

__device__ __forceinline__ float4_t mfma(const half8_t& a, const half8_t& b, const float4_t& c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// Number that row i (the lane's) chooses its adapters by: -1 for none.
__device__ __forceinline__ int choice_of(const LoraRows& rows, int i, int M) {
    if (i >= M) return -1;
    int seq = i;
    if (rows.row_seq) {
        seq = rows.row_seq[i];
        if (static_cast<uint32_t>(seq) >= static_cast<uint32_t>(rows.n_seq)) return -1;
    }
    return max(rows.adapter[seq], -1);
}
// ... which a linear may have an adapter for or not
__device__ __forceinline__ int adapter_of(const LoraDev& l, int choice) { return static_cast<uint32_t>(choice) < static_cast<uint32_t>(l.n) ? choice : -1; }
__device__ __forceinline__ int rank_of(const LoraDev& l, int a) { return l.rank ? min(max(l.rank[a], 0), l.R) : l.R; }

// As the shared product's results: saturating; a NaN stays one.
__device__ __forceinline__ uint16_t to_half(float f) { return f == f ? float_to_half_bits(f) : 0x7e00u; }

struct LoraInner {
    LoraDev l[kLoraMost];
    float* inner[kLoraMost];
    LoraRows rows;
    const uint16_t* A;
    int parts;
};

// One workgroup of NW waves per (16 RT rows, part of K[, adapter of the tile]); NR tiles of 16 inner values.  ALONE: each adapter of the tile has its own
// workgroup.
template <int RT, int NR, int NW, bool ALONE>
__global__ void __launch_bounds__(64 * NW)
lora_inner_kernel(LoraInner p) {
    const LoraDev& l = p.l[blockIdx.z];
    const int M = p.rows.count ? min(*p.rows.count, p.rows.M) : p.rows.M;
    const int row0 = blockIdx.x * (16 * RT), part = ALONE ? blockIdx.y >> 4 : blockIdx.y;
    if (row0 >= M) return;
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    __shared__ float4_t sums[NW - 1][RT * NR][64];
    const int mine = adapter_of(l, choice_of(p.rows, row0 + lane, lane < 16 * RT ? M : 0));   // lane x: row x of the tile
    int own[RT];                                                 // this lane's columns: rows c, 16 + c, ...
#pragma unroll
    for (int t = 0; t < RT; ++t) own[t] = __shfl(mine, 16 * t + c, 64);
    uint64_t left = __ballot(mine >= 0);
    int skip = ALONE ? blockIdx.y & 15 : 0;
    const int units = (l.K + 127) / 128, step = NW * p.parts;    // units of 128 columns of K: this wave's are part * NW + wave, + step, ...
    const size_t stride = static_cast<size_t>(p.rows.M) * l.R;
    const uint16_t* rows_at[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) rows_at[t] = p.A + static_cast<size_t>(min(row0 + 16 * t + c, M - 1)) * l.K;
    while (left != 0) {
        const int a = __builtin_amdgcn_readlane(mine, __builtin_amdgcn_readfirstlane(__ffsll(static_cast<long long>(left)) - 1));
        left &= ~__ballot(mine == a);
        if (ALONE && skip-- > 0) continue;
        const int rank = rank_of(l, a);
        const uint16_t* down = l.down + static_cast<size_t>(a) * l.R * l.K;
        float4_t acc[RT][NR];
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int r = 0; r < NR; ++r) acc[t][r] = float4_t{0.f, 0.f, 0.f, 0.f};
        for (int u = part * NW + wave; u < units; u += step) {
            half8_t x[4][RT], w[4][NR];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = u * 128 + 32 * j + 8 * g;
                const bool in = k < l.K;                         // (K is a multiple of 8)
#pragma unroll
                for (int t = 0; t < RT; ++t) x[j][t] = *reinterpret_cast<const half8_t*>(rows_at[t] + (in ? k : 0));
#pragma unroll
                for (int r = 0; r < NR; ++r) w[j][r] = *reinterpret_cast<const half8_t*>(down + static_cast<size_t>(min(16 * r + c, l.R - 1)) * l.K + (in ? k : 0));
                if (!in) {
#pragma unroll
                    for (int t = 0; t < RT; ++t) x[j][t] = half8_t{};
#pragma unroll
                    for (int r = 0; r < NR; ++r) w[j][r] = half8_t{};
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int t = 0; t < RT; ++t)
#pragma unroll
                    for (int r = 0; r < NR; ++r) acc[t][r] = mfma(w[j][r], x[j][t], acc[t][r]);
        }
        // the waves meet in LDS; the first writes
        if (wave > 0) {
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int r = 0; r < NR; ++r) sums[wave - 1][t * NR + r][lane] = acc[t][r];
        }
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int r = 0; r < NR; ++r) {
                    float4_t y = acc[t][r];
#pragma unroll
                    for (int w = 0; w < NW - 1; ++w) y += sums[w][t * NR + r][lane];
                    // lane (c, g): row c, inner values 16 r + 4 g .. + 3 (R is a multiple of 8)
                    if (own[t] == a && 16 * r + 4 * g < rank)
                        *reinterpret_cast<float4_t*>(p.inner[blockIdx.z] + part * stride + static_cast<size_t>(row0 + 16 * t + c) * l.R + 16 * r + 4 * g) = y;
                }
        }
        if (ALONE) return;
        __syncthreads();
    }
}

// Inner values of this lane's row (one that there is) as operands, zeros from `rank` on: k-step s has values 32 s + 8 g ..; returns the power of two that a
// unit of the products stands for.  All loads go out together and without a branch: what is not wanted is loaded from a place that is there.
template <int NS>
__device__ __forceinline__ float inner_operand(const LoraDev& l, int rank, const float* inner, int parts, size_t stride, int row, int g, half8_t* x) {
    constexpr int AT_ONCE = NS == 1 ? 4 : 2;
    float v[NS][8], big = 0.0f;
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[s][e] = 0.0f;
    const float* at = inner + static_cast<size_t>(row) * l.R;
    for (int z0 = 0; z0 < parts; z0 += AT_ONCE) {
        float4_t y[AT_ONCE][NS][2];
#pragma unroll
        for (int z = 0; z < AT_ONCE; ++z)
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                const float* from = at + min(z0 + z, parts - 1) * stride + min(32 * s + 8 * g, l.R - 8);
                y[z][s][0] = *reinterpret_cast<const float4_t*>(from);
                y[z][s][1] = *reinterpret_cast<const float4_t*>(from + 4);
            }
#pragma unroll
        for (int z = 0; z < AT_ONCE; ++z)
#pragma unroll
            for (int s = 0; s < NS; ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[s][e] += z0 + z < parts ? y[z][s][e >> 2][e & 3] : 0.0f;
    }
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[s][e] = 32 * s + 8 * g + e < rank ? v[s][e] : 0.0f;
            big = fmaxf(big, fabsf(v[s][e]));
        }
    big = fmaxf(big, __shfl_xor(big, 16, 64));
    big = fmaxf(big, __shfl_xor(big, 32, 64));
    const int e = min(max(static_cast<int>(__float_as_uint(big) >> 23) - 127, -100), 127);
    const float f = ldexpf(1.0f, 12 - e);
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[s][i] = static_cast<half_t>(v[s][i] * f);
    return ldexpf(1.0f, e - 12);
}
__device__ __forceinline__ float scale_of(const LoraDev& l, int a) { return l.scale ? l.scale[a] : 1.0f; }

// Many rows: the parts' sums as operands, once: [M][32 NS] fp16 relative to the row's power of two, zeros from its adapter's rank on, then [M] of what a
// unit of the products stands for (0 for a row without an adapter).
struct LoraPack {
    LoraDev l[kLoraMost];
    float* inner[kLoraMost];
    uint16_t* out[kLoraMost];
    LoraRows rows;
    int parts;
};
__host__ __device__ inline int operand_width(int R) { return R <= 32 ? 32 : R <= 64 ? 64 : 128; }
__device__ __forceinline__ const float* operand_units(const uint16_t* operands, int R, int M) { return reinterpret_cast<const float*>(operands + static_cast<size_t>(M) * operand_width(R)); }

__global__ void __launch_bounds__(256)
lora_pack_kernel(LoraPack p) {
    const LoraDev& l = p.l[blockIdx.y];
    const int M = p.rows.count ? min(*p.rows.count, p.rows.M) : p.rows.M;
    if (static_cast<int>(blockIdx.x) * 16 >= M) return;          // (M on the device may be 0: there is no row then to load in the others' place)
    const int row = blockIdx.x * 16 + (threadIdx.x >> 4), r0 = 8 * (threadIdx.x & 15), at_row = min(row, M - 1);
    const size_t stride = static_cast<size_t>(p.rows.M) * l.R;
    const float* from = p.inner[blockIdx.y] + static_cast<size_t>(at_row) * l.R + min(r0, l.R - 8);
    float4_t y[8][2];
#pragma unroll
    for (int z = 0; z < 8; ++z) {
        y[z][0] = *reinterpret_cast<const float4_t*>(from + min(z, p.parts - 1) * stride);
        y[z][1] = *reinterpret_cast<const float4_t*>(from + min(z, p.parts - 1) * stride + 4);
    }
    const int a = adapter_of(l, choice_of(p.rows, at_row, M));
    const int rank = a >= 0 ? rank_of(l, a) : 0;
    float v[8], big = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        v[e] = 0.0f;
#pragma unroll
        for (int z = 0; z < 8; ++z) v[e] += z < p.parts ? y[z][e >> 2][e & 3] : 0.0f;
        v[e] = r0 + e < rank ? v[e] : 0.0f;
        big = fmaxf(big, fabsf(v[e]));
    }
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) big = fmaxf(big, __shfl_xor(big, o, 64));
    if (row >= M) return;
    const int e = min(max(static_cast<int>(__float_as_uint(big) >> 23) - 127, -100), 127), width = operand_width(l.R);
    const float f = ldexpf(1.0f, 12 - e);
    half8_t x;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = static_cast<half_t>(v[i] * f);
    uint16_t* out = p.out[blockIdx.y];
    if (r0 < width) *reinterpret_cast<half8_t*>(out + static_cast<size_t>(row) * width + r0) = x;
    if (r0 == 0) const_cast<float*>(operand_units(out, l.R, p.rows.M))[row] = a >= 0 ? ldexpf(scale_of(l, a), e - 12) : 0.0f;
}

struct LoraOuter {
    LoraDev l[2];
    const float* inner[2];
    int parts[2];
    LoraRows rows;
    const float* base;           // (what is added to, elsewhere) [M][ldb], ldb at least 2 N for swiglu
    int ldb;
    void* out;
    int ldo;
};
enum { LORA_ROUND, LORA_ADD_F32, LORA_SWIGLU };

// A wave's products of 16 NT columns from n0 on: product j has columns n0 + 4 NT (i / 4) + 4 j + i % 4, i < 16, so that lane (c, g), which gets i = 4 g .. 4 g + 3
// of each, has 4 NT columns in a row of the matrix that it reads and writes.
// up_a of product j's columns (lane c: i = c), k-step s: inner values 32 s + 8 g ..
template <int NS, int NT>
__device__ __forceinline__ void up_operand(const LoraDev& l, int a, int n0, int j, u32x4_t* w) {
    const int c = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
    const uint16_t* at = l.up + (static_cast<size_t>(a) * l.N + min(n0 + 4 * NT * (c >> 2) + 4 * j + (c & 3), l.N - 1)) * l.R;
#pragma unroll
    for (int s = 0; s < NS; ++s) w[s] = *reinterpret_cast<const u32x4_t*>(at + min(32 * s + 8 * g, l.R - 8));
}
// What lies past the rank may be anything: bits of this lane's operands that stay.
template <int NS>
__device__ __forceinline__ void rank_mask(int rank, u32x4_t* mask) {
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e) mask[s][e] = (32 * s + 8 * g + 2 * e < rank ? 0xffffu : 0u) | (32 * s + 8 * g + 2 * e + 1 < rank ? 0xffff0000u : 0u);
}
template <int NS>
__device__ __forceinline__ float4_t outer_product(const u32x4_t* w, const u32x4_t* mask, const half8_t* x) {
    float4_t y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < NS; ++s) y = mfma(__builtin_bit_cast(half8_t, w[s] & mask[s]), x[s], y);
    return y;
}

// Eight values of a row: what is there and what is added (two products' four).
template <int FORM> struct OuterRow;
template <> struct OuterRow<LORA_ADD_F32> {
    float4_t old[2];
    __device__ __forceinline__ void read(const LoraOuter& p, size_t row, int n, int) {
        const float4_t* from = reinterpret_cast<const float4_t*>(static_cast<const float*>(p.out) + row * p.ldo + n);
        old[0] = from[0];
        old[1] = from[1];
    }
    __device__ __forceinline__ void write(const LoraOuter& p, size_t row, int n, const float4_t* y, const float4_t*) const {
        float4_t* to = reinterpret_cast<float4_t*>(static_cast<float*>(p.out) + row * p.ldo + n);
        to[0] = old[0] + y[0];
        to[1] = old[1] + y[1];
    }
};
__device__ __forceinline__ u32x4_t halves(const float* y) {
    u32x4_t w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = to_half(y[2 * e]) | static_cast<uint32_t>(to_half(y[2 * e + 1])) << 16;
    return w;
}
template <> struct OuterRow<LORA_ROUND> {
    float4_t old[2];
    __device__ __forceinline__ void read(const LoraOuter& p, size_t row, int n, int) {
        const float4_t* from = reinterpret_cast<const float4_t*>(p.base + row * p.ldb + n);
        old[0] = from[0];
        old[1] = from[1];
    }
    __device__ __forceinline__ void write(const LoraOuter& p, size_t row, int n, const float4_t* y, const float4_t*) const {
        float sum[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = old[e >> 2][e & 3] + y[e >> 2][e & 3];
        *reinterpret_cast<u32x4_t*>(static_cast<uint16_t*>(p.out) + row * p.ldo + n) = halves(sum);
    }
};
template <> struct OuterRow<LORA_SWIGLU> {
    float4_t gate[2], up[2];
    __device__ __forceinline__ void read(const LoraOuter& p, size_t row, int n, int N) {
        const float* from = p.base + row * p.ldb + n;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            gate[h] = reinterpret_cast<const float4_t*>(from)[h];
            up[h] = reinterpret_cast<const float4_t*>(from + N)[h];
        }
    }
    __device__ __forceinline__ void write(const LoraOuter& p, size_t row, int n, const float4_t* yg, const float4_t* yu) const {
        float out[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = gate[e >> 2][e & 3] + yg[e >> 2][e & 3];
            out[e] = x * __builtin_amdgcn_rcpf(1.0f + __expf(-x)) * (up[e >> 2][e & 3] + yu[e >> 2][e & 3]);   // (off by 2^-22 or so)
        }
        *reinterpret_cast<u32x4_t*>(static_cast<uint16_t*>(p.out) + row * p.ldo + n) = halves(out);
    }
};

// Few rows, which mostly choose differently: a workgroup per (16 rows, 256 NT columns, number that some of the rows choose by), which writes those rows.
// The rows' operands are made once, by a wave per linear, in LDS; a wave's first columns are on their way meanwhile.
template <int NS, int FORM, int NT>
__global__ void __launch_bounds__(256)
lora_few_kernel(LoraOuter p, int steps) {
    constexpr int NL = FORM == LORA_SWIGLU ? 2 : 1;
    const int M = p.rows.count ? min(*p.rows.count, p.rows.M) : p.rows.M;
    const int row0 = blockIdx.x * 16, lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int N = FORM == LORA_SWIGLU ? p.ldo : p.l[0].N;
    if (row0 >= M) return;
    __shared__ half8_t operands[NL][NS][64];
    __shared__ float units[NL][16];
    const int mine = choice_of(p.rows, row0 + lane, lane < 16 ? M : 0);   // lane x: row x of the tile
    // rows that there are (and have something to add, where nothing else is done), then those of the blockIdx.z-th choice
    uint64_t rows = __ballot(lane < 16 && row0 + lane < M && (FORM != LORA_ADD_F32 || adapter_of(p.l[0], mine) >= 0));
    int choice = -1;
    for (int skip = blockIdx.z; rows != 0; --skip) {
        choice = __builtin_amdgcn_readlane(mine, __builtin_amdgcn_readfirstlane(__ffsll(static_cast<long long>(rows)) - 1));
        const uint64_t same = __ballot(mine == choice) & rows;
        if (skip == 0) { rows = same; break; }
        rows &= ~same;
    }
    if (rows == 0) return;                                       // (the same in all waves)
    const bool own = (rows >> c & 1) != 0;
    const size_t row = row0 + c;
    int a[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) a[i] = adapter_of(p.l[i], choice);
    u32x4_t w[NL][NT][NS];
    OuterRow<FORM> there[NT / 2];
    auto fetch = [&](int n0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            if (a[i] < 0) continue;                              // (the same in all lanes)
#pragma unroll
            for (int j = 0; j < NT; ++j) up_operand<NS, NT>(p.l[i], a[i], n0, j, w[i][j]);
        }
        if (own) {                                               // (N is a multiple of 8)
#pragma unroll
            for (int h = 0; h < NT / 2; ++h) there[h].read(p, row, min(n0 + 4 * NT * g + 8 * h, N - 8), N);
        }
    };
    int n0 = (blockIdx.y * steps * 4 + wave) * (16 * NT);
    fetch(n0);
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        if (wave != i || a[i] < 0) continue;
        half8_t x[NS];
        const float unit = inner_operand<NS>(p.l[i], rank_of(p.l[i], a[i]), p.inner[i], p.parts[i], static_cast<size_t>(p.rows.M) * p.l[i].R, min(row0 + c, M - 1), g, x);
#pragma unroll
        for (int s = 0; s < NS; ++s) operands[i][s][lane] = x[s];
        if (g == 0) units[i][c] = unit * scale_of(p.l[i], a[i]);
    }
    u32x4_t mask[NL][NS];
#pragma unroll
    for (int i = 0; i < NL; ++i) rank_mask<NS>(a[i] >= 0 ? rank_of(p.l[i], a[i]) : 0, mask[i]);
    __syncthreads();
    half8_t x[NL][NS];
    float unit[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) {
#pragma unroll
        for (int s = 0; s < NS; ++s) x[i][s] = operands[i][s][lane];
        unit[i] = units[i][c];
    }
#pragma unroll 1
    for (int step = 0; step < steps && n0 < N; ++step, n0 += 64 * NT) {
        float4_t y[NL][NT];
#pragma unroll
        for (int i = 0; i < NL; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                y[i][j] = float4_t{0.f, 0.f, 0.f, 0.f};
                if (a[i] >= 0) y[i][j] = outer_product<NS>(w[i][j], mask[i], x[i]) * unit[i];
            }
#pragma unroll
        for (int h = 0; h < NT / 2; ++h)
            if (own && n0 + 4 * NT * g + 8 * h < N) there[h].write(p, row, n0 + 4 * NT * g + 8 * h, &y[0][2 * h], &y[NL - 1][2 * h]);
        if (step + 1 < steps) fetch(n0 + 64 * NT);
    }
}

constexpr int many_tiles(int ns, int form) { return ns * (form == LORA_SWIGLU ? 2 : 1) >= 4 ? 2 : 4; }   // (registers)

// Many rows, operands made (lora_pack_kernel): a wave per 64 rows and 16 NT columns, 16 rows at a time, the next ones on their way.  It walks the adapters
// that the rows have, mostly one, and keeps its part of up until another comes.
template <int NS, int FORM>
__global__ void __launch_bounds__(256)
lora_many_kernel(LoraOuter p) {
    constexpr int NT = many_tiles(NS, FORM), NL = FORM == LORA_SWIGLU ? 2 : 1;
    const int M = p.rows.count ? min(*p.rows.count, p.rows.M) : p.rows.M;
    // Workgroups go round-robin to the 8 XCDs: each has its own blocks of columns, whose part of up its L2 holds for all rows.
    const int chunks = (p.rows.M + 63) / 64, local = blockIdx.x >> 3, block = local / chunks * 8 + (blockIdx.x & 7);
    const int row0 = (local % chunks) * 64, lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int N = FORM == LORA_SWIGLU ? p.ldo : p.l[0].N, n0 = (block * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * (16 * NT);
    if (row0 >= M || n0 >= N) return;
    struct Rows {                                                // what the wave reads of 16 rows
        half8_t x[NL][NS];
        float unit[NL];
        OuterRow<FORM> there[NT / 2];
    };
    auto read = [&](int t, Rows& to) __attribute__((always_inline)) {
        const size_t row = min(row0 + 16 * t + c, M - 1);
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            if (p.l[i].n == 0) continue;
            const uint16_t* operands = reinterpret_cast<const uint16_t*>(p.inner[i]);
            const int width = operand_width(p.l[i].R);
#pragma unroll
            for (int s = 0; s < NS; ++s) to.x[i][s] = *reinterpret_cast<const half8_t*>(operands + row * width + min(32 * s + 8 * g, width - 8));
            to.unit[i] = operand_units(operands, p.l[i].R, p.rows.M)[row];
        }
#pragma unroll
        for (int h = 0; h < NT / 2; ++h) to.there[h].read(p, row, min(n0 + 4 * NT * g + 8 * h, N - 8), N);   // (N is a multiple of 8)
    };
    Rows now, next;
    read(0, now);
    const int mine = choice_of(p.rows, row0 + lane, M);          // lane x: row x of the 64
    const uint64_t rows = __ballot(row0 + lane < M && (FORM != LORA_ADD_F32 || adapter_of(p.l[0], mine) >= 0));
    u32x4_t w[NL][NT][NS], mask[NL][NS];
    int held[NL];                                                // the adapter whose part of up is there
#pragma unroll
    for (int i = 0; i < NL; ++i) held[i] = -1;
#pragma unroll 1
    for (int t = 0; t < 4 && row0 + 16 * t < M; ++t) {
        if (t < 3) read(t + 1, next);
        const uint32_t own = static_cast<uint32_t>(rows >> (16 * t)) & 0xffffu;
        const int choice = __shfl(mine, 16 * t + c, 64);         // of this lane's row
        float4_t y[NL][NT];
#pragma unroll
        for (int i = 0; i < NL; ++i) {
#pragma unroll
            for (int j = 0; j < NT; ++j) y[i][j] = float4_t{0.f, 0.f, 0.f, 0.f};
            uint32_t left = own & static_cast<uint32_t>(__ballot(adapter_of(p.l[i], mine) >= 0) >> (16 * t));
            while (left != 0) {
                const int a = __builtin_amdgcn_readlane(mine, __builtin_amdgcn_readfirstlane(16 * t + __ffs(static_cast<int>(left)) - 1));
                left &= ~static_cast<uint32_t>(__ballot(mine == a) >> (16 * t));
                if (a != held[i]) {
                    held[i] = a;
#pragma unroll
                    for (int j = 0; j < NT; ++j) up_operand<NS, NT>(p.l[i], a, n0, j, w[i][j]);
                    rank_mask<NS>(rank_of(p.l[i], a), mask[i]);
                }
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const float4_t d = outer_product<NS>(w[i][j], mask[i], now.x[i]);
#pragma unroll
                    for (int r = 0; r < 4; ++r) y[i][j][r] = choice == a ? d[r] * now.unit[i] : y[i][j][r];
                }
            }
        }
        if ((own >> c & 1) != 0) {
#pragma unroll
            for (int h = 0; h < NT / 2; ++h)
                if (n0 + 4 * NT * g + 8 * h < N) now.there[h].write(p, row0 + 16 * t + c, n0 + 4 * NT * g + 8 * h, &y[0][2 * h], &y[NL - 1][2 * h]);
        }
        now = next;
    }
}

// Rows up to which they are taken to choose differently: a workgroup per choice of a tile's rows, instead of one that walks them.  us, the whole linear, with /
// without, 4096 -> 4096: 200 rows with 60 adapters 42.5 / 88, in requests of 40 rows 40 / 42; 500 rows with 60 adapters 68 / 94, in requests of 100
// rows 45.7 / 43.5; 900 rows 99 / 116, in requests of 90 74 / 69.  (So many rows are mostly prompts.)
constexpr int kLoraAlone = 256;

// Parts of K: workgroups that fill the chip, each wave with a unit of 128 columns at least.
constexpr int kManyFill = 512;
// Rows of a tile: more read less of down, if few adapters meet in one.  Tiles of 16 / 64, us, the whole linear, 14336 -> 4096 with rank 32 in requests of 100: 512 rows
// 112 / 121, 1024 160 / 166, 1536 241 / 238, 2048 302 / 281, 3000 445 / 436, 4000 549 / 518; of 500: 1024 158 / 166, 2048 282 / 278, 4000 522 / 506; of 25: 2048 306 / 314,
// 4000 553 / 565.  4096 -> 4096 with rank 16 in requests of 100: 1024 62.5 / 64.7, 2048 103 / 100, 4000 178 / 174.  Rows that all choose for themselves lose by 64 at
// every size (4096 -> 4096: 1024 121 / 212, 4000 332 / 423): so many rows are prompts.
static int inner_tile(int M) { return M <= 2048 ? 16 : 64; }
static int inner_parts(int M, int K, int n) {
    const int units = (K + 127) / 128;
    if (M <= kLoraAlone) return std::min(std::max(units / 8, 1), 4);
    const int wgs = (M + inner_tile(M) - 1) / inner_tile(M) * n;
    return std::min(std::min((kManyFill + wgs - 1) / wgs, 8), std::max(units / 4, 1));
}
size_t lora_inner_bytes(int R, int M) {
    // enough for any number of rows up to M: parts * M <= 8 M, and <= 64 kManyFill + M
    const size_t rows = std::min<size_t>(static_cast<size_t>(8) * M, static_cast<size_t>(kManyFill) * 64 + M);
    return (rows * R * 4 + 255) / 256 * 256 + (static_cast<size_t>(M) * (2 * operand_width(R) + 4) + 255) / 256 * 256;
}

template <int RT, int NR, int NW, bool ALONE>
static void inner_launch(const LoraInner& p, int tiles, int n, hipStream_t stream) {
    hipLaunchKernelGGL((lora_inner_kernel<RT, NR, NW, ALONE>), dim3(tiles, (ALONE ? 16 : 1) * p.parts, n), dim3(64 * NW), 0, stream, p);
}

hipError_t launch_lora_inner(const LoraDev* l, int n, const LoraRows& rows, const void* A, float* const* inner, const float** operands, int* parts,
                             hipStream_t stream) {
    LoraInner p{};
    int R = 0;
    for (int i = 0; i < n; ++i) {
        p.l[i] = l[i];
        p.inner[i] = inner[i];
        R = std::max(R, l[i].R);
    }
    p.rows = rows; p.A = static_cast<const uint16_t*>(A);
    p.parts = inner_parts(rows.M, l[0].K, n);
    for (int i = 0; i < n; ++i) parts[i] = p.parts;
    // Few rows, whose adapters mostly differ: a workgroup per adapter of the tile.  Many: a tile's adapters one after the
    // other, mostly one.
    const int tile = inner_tile(rows.M), tiles = (rows.M + tile - 1) / tile;
    if (rows.M <= kLoraAlone) {
        if (R <= 16) inner_launch<1, 1, 8, true>(p, tiles, n, stream);
        else if (R <= 32) inner_launch<1, 2, 8, true>(p, tiles, n, stream);
        else if (R <= 64) inner_launch<1, 4, 8, true>(p, tiles, n, stream);
        else inner_launch<1, 8, 8, true>(p, tiles, n, stream);
    } else if (tile == 16) {
        if (R <= 16) inner_launch<1, 1, 4, false>(p, tiles, n, stream);
        else if (R <= 32) inner_launch<1, 2, 4, false>(p, tiles, n, stream);
        else if (R <= 64) inner_launch<1, 4, 4, false>(p, tiles, n, stream);
        else inner_launch<1, 8, 4, false>(p, tiles, n, stream);
    } else {
        if (R <= 16) inner_launch<4, 1, 4, false>(p, tiles, n, stream);
        else if (R <= 32) inner_launch<4, 2, 4, false>(p, tiles, n, stream);
        else if (R <= 64) inner_launch<4, 4, 4, false>(p, tiles, n, stream);
        else inner_launch<4, 8, 4, false>(p, tiles, n, stream);
    }
    if (rows.M > kLoraAlone) {                                   // the sums become operands, behind the parts
        LoraPack k{};
        for (int i = 0; i < n; ++i) {
            k.l[i] = l[i];
            k.inner[i] = inner[i];
            k.out[i] = reinterpret_cast<uint16_t*>(inner[i] + (static_cast<size_t>(p.parts) * rows.M * l[i].R + 63) / 64 * 64);
        }
        k.rows = rows; k.parts = p.parts;
        hipLaunchKernelGGL(lora_pack_kernel, dim3((rows.M + 15) / 16, n), dim3(256), 0, stream, k);
        for (int i = 0; i < n; ++i) operands[i] = reinterpret_cast<const float*>(k.out[i]);
    } else {
        for (int i = 0; i < n; ++i) operands[i] = inner[i];
    }
    return hipGetLastError();
}

template <int NS, int FORM>
static void outer_rank(const LoraOuter& p, int N, hipStream_t stream) {
    constexpr int NT = 2, WIDE = 64 * many_tiles(NS, FORM);
    // Few rows: about four workgroups per CU if they all choose differently.  (64 rows of 40 adapters, gate/up of 11008, us: one step of 256 columns 29.5, of
    // 512 23, of 1024 18; four steps of 128 15.5.)
    const int blocks = (N + 64 * NT - 1) / (64 * NT), steps = std::min(std::max(static_cast<int>(static_cast<int64_t>(p.rows.M) * blocks / 1024), 1), 8);
    // (neighbours share a part of up)
    if (p.rows.M <= kLoraAlone)
        hipLaunchKernelGGL((lora_few_kernel<NS, FORM, NT>), dim3((p.rows.M + 15) / 16, (blocks + steps - 1) / steps, 16), dim3(256), 0, stream, p, steps);
    else
        hipLaunchKernelGGL((lora_many_kernel<NS, FORM>), dim3((p.rows.M + 63) / 64 * (((N + WIDE - 1) / WIDE + 7) / 8 * 8)), dim3(256), 0, stream, p);
}
template <int FORM>
static hipError_t outer_form(const LoraOuter& p, int R, int N, hipStream_t stream) {
    if (p.rows.M <= 0) return hipSuccess;
    if (R <= 32) outer_rank<1, FORM>(p, N, stream);
    else if (R <= 64) outer_rank<2, FORM>(p, N, stream);
    else outer_rank<4, FORM>(p, N, stream);
    return hipGetLastError();
}

hipError_t launch_lora_add(const LoraDev& l, const LoraRows& rows, const float* inner, int parts, float* out, int ldo, hipStream_t stream) {
    LoraOuter p{};
    p.l[0] = l; p.inner[0] = inner; p.parts[0] = parts; p.rows = rows; p.out = out; p.ldo = ldo;
    return outer_form<LORA_ADD_F32>(p, l.R, l.N, stream);
}
hipError_t launch_lora_round(const LoraDev& l, const LoraRows& rows, const float* inner, int parts, const float* base, int ldb, void* out, int ldo,
                             hipStream_t stream) {
    LoraOuter p{};
    p.l[0] = l; p.inner[0] = inner; p.parts[0] = parts; p.rows = rows; p.base = base; p.ldb = ldb; p.out = out; p.ldo = ldo;
    return outer_form<LORA_ROUND>(p, l.R, l.N, stream);
}

hipError_t launch_lora_swiglu(const LoraDev& lg, const LoraDev& lu, const LoraRows& rows, const float* inner_g, const float* inner_u, int parts_g, int parts_u,
                              const float* base, void* out, int N, hipStream_t stream) {
    LoraOuter p{};
    p.l[0] = lg; p.l[1] = lu; p.inner[0] = inner_g; p.inner[1] = inner_u; p.parts[0] = parts_g; p.parts[1] = parts_u;
    p.rows = rows; p.base = base; p.ldb = 2 * N; p.out = out; p.ldo = N;
    return outer_form<LORA_SWIGLU>(p, std::max(lg.R, lu.R), N, stream);
}

}  // namespace qtale
