// Low-rank adapters of many requests beside a shared projection: y_i += scale[a] up_a (down_a A_i), a the adapter of row i.
//
// Both products run on the matrix cores in tiles of 16 rows (or 64) that know nothing of the rows' order: a tile walks the adapters that occur in it, and a
// row takes the result of its own and leaves the others'.  A decode step's tile of 16 requests reads each of its adapters once, which has to be; a
// prompt's tile meets one.  Operands of rows that the result leaves out cannot reach it, whatever they hold (a select, not a product with zero).
//   inner  D[r][row] = down_a A^T, K cut over the waves of a workgroup and over workgroups (lora_splits), so that a few requests fill the chip;
//          a part's sums are written, and added by the second kernel: no atomics, the same bits every time
//   outer  D[n][row] = up_a inner^T: inner values go in as fp16 relative to their row's power of two, off by 2^-12 of each (or 2^-36 of the
//          row's largest): less than the rounding of the result they are added to
#include <algorithm>

#include "lora.h"
#include "qtale_dev.h"

namespace qtale {

__device__ __forceinline__ float4_t mfma(const half8_t& a, const half8_t& b, const float4_t& c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// Adapter of row i (the lane's): -1 for none.
__device__ __forceinline__ int adapter_of(const LoraDev& l, const LoraRows& rows, int i, int M) {
    if (i >= M) return -1;
    int seq = i;
    if (rows.row_seq) {
        seq = rows.row_seq[i];
        if (static_cast<uint32_t>(seq) >= static_cast<uint32_t>(rows.n_seq)) return -1;
    }
    const int a = rows.adapter[seq];
    return static_cast<uint32_t>(a) < static_cast<uint32_t>(l.n) ? a : -1;
}
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

// One workgroup per (16 RT rows, part of K[, adapter of the tile]); NR tiles of 16 inner values.  ALONE: each adapter of the tile has its own workgroup.
template <int RT, int NR, bool ALONE>
__global__ void __launch_bounds__(256)
lora_inner_kernel(LoraInner p) {
    const LoraDev& l = p.l[blockIdx.z];
    const int M = p.rows.count ? min(*p.rows.count, p.rows.M) : p.rows.M;
    const int row0 = blockIdx.x * (16 * RT), part = ALONE ? blockIdx.y >> 4 : blockIdx.y;
    if (row0 >= M) return;
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    __shared__ float4_t sums[3][RT * NR][64];
    const int mine = adapter_of(l, p.rows, row0 + lane, lane < 16 * RT ? M : 0);   // lane x: row x of the tile
    int own[RT];                                                 // this lane's columns: rows c, 16 + c, ...
#pragma unroll
    for (int t = 0; t < RT; ++t) own[t] = __shfl(mine, 16 * t + c, 64);
    uint64_t left = __ballot(mine >= 0);
    int skip = ALONE ? blockIdx.y & 15 : 0;
    const int units = (l.K + 127) / 128, step = 4 * p.parts;     // units of 128 columns of K: this wave's are part * 4 + wave, + step, ...
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
        for (int u = part * 4 + wave; u < units; u += step) {
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
        // the four waves meet in LDS; the first writes
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
                    const float4_t y = (acc[t][r] + sums[0][t * NR + r][lane]) + (sums[1][t * NR + r][lane] + sums[2][t * NR + r][lane]);
                    // lane (c, g): row c, inner values 16 r + 4 g .. + 3 (R is a multiple of 8)
                    if (own[t] == a && 16 * r + 4 * g < rank)
                        *reinterpret_cast<float4_t*>(p.inner[blockIdx.z] + part * stride + static_cast<size_t>(row0 + 16 * t + c) * l.R + 16 * r + 4 * g) = y;
                }
        }
        if (ALONE) return;
        __syncthreads();
    }
}

// Inner values of this lane's row as operands: k-step s has values 32 s + 8 g ..; *unit: what a unit of the products stands for.
template <int NS>
__device__ __forceinline__ void inner_operand(const LoraDev& l, int a, const float* inner, int parts, size_t stride, int row, int g, half8_t* x, float* unit) {
    float v[NS][8], big = 0.0f;
    const int rank = a >= 0 ? rank_of(l, a) : 0;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        const int r0 = 32 * s + 8 * g;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[s][e] = 0.0f;
        if (r0 < rank) {
            const float* at = inner + static_cast<size_t>(row) * l.R + r0;
            for (int z = 0; z < parts; ++z) {
                const float4_t y0 = *reinterpret_cast<const float4_t*>(at + z * stride), y1 = *reinterpret_cast<const float4_t*>(at + z * stride + 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) { v[s][e] += y0[e]; v[s][4 + e] += y1[e]; }
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[s][e] = r0 + e < rank ? v[s][e] : 0.0f;
            big = fmaxf(big, fabsf(v[s][e]));
        }
    }
    big = fmaxf(big, __shfl_xor(big, 16, 64));
    big = fmaxf(big, __shfl_xor(big, 32, 64));
    const int e = min(max(static_cast<int>(__float_as_uint(big) >> 23) - 127, -100), 127);
    const float f = ldexpf(1.0f, 12 - e);
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[s][i] = static_cast<half_t>(v[s][i] * f);
    *unit = a >= 0 ? ldexpf(l.scale ? l.scale[a] : 1.0f, e - 12) : 0.0f;
}

// y[j] = up_a inner of columns n0 + 16 j + 4 g .. + 3 and the lane's row, for the rows' own adapters (0 for those without); left: rows that have one.
template <int NS, int NT>
__device__ __forceinline__ void outer_product(const LoraDev& l, uint64_t left, int mine, int own, const half8_t* x, int n0, float4_t* y) {
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
#pragma unroll
    for (int j = 0; j < NT; ++j) y[j] = float4_t{0.f, 0.f, 0.f, 0.f};
    while (left != 0) {
        const int a = __builtin_amdgcn_readlane(mine, __builtin_amdgcn_readfirstlane(__ffsll(static_cast<long long>(left)) - 1));
        left &= ~__ballot(mine == a);
        const int rank = rank_of(l, a);
        half8_t w[NT][NS];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const uint16_t* at = l.up + (static_cast<size_t>(a) * l.N + min(n0 + 16 * j + c, l.N - 1)) * l.R;
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                const int r0 = 32 * s + 8 * g;
                w[j][s] = half8_t{};
                if (r0 < rank) w[j][s] = *reinterpret_cast<const half8_t*>(at + r0);
                if (r0 + 8 > rank && r0 < rank) {                // what lies past the rank may be anything
#pragma unroll
                    for (int e = 0; e < 8; ++e) w[j][s][e] = r0 + e < rank ? w[j][s][e] : static_cast<half_t>(0.0f);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            float4_t d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < NS; ++s) d = mfma(w[j][s], x[s], d);
#pragma unroll
            for (int r = 0; r < 4; ++r) y[j][r] = own == a ? d[r] : y[j][r];
        }
    }
}

struct LoraOuter {
    LoraDev l[2];
    const float* inner[2];
    int parts[2];
    LoraRows rows;
    const uint16_t* base;        // swiglu: [M][2 N]
    void* out;
    int ldo;
};
enum { LORA_ADD_F16, LORA_ADD_F32, LORA_SWIGLU };
constexpr int kOuterTiles = 4;   // of 16 columns per wave

// One wave per 16 rows x 64 columns.
template <int NS, int FORM>
__global__ void __launch_bounds__(256)
lora_outer_kernel(LoraOuter p) {
    constexpr int NT = kOuterTiles, NL = FORM == LORA_SWIGLU ? 2 : 1;
    const int M = p.rows.count ? min(*p.rows.count, p.rows.M) : p.rows.M;
    const int row0 = blockIdx.x * 16, lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int N = FORM == LORA_SWIGLU ? p.ldo : p.l[0].N, n0 = (blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * (16 * NT);
    if (row0 >= M || n0 >= N) return;
    const int row = row0 + c;
    float4_t y[NL][NT];
    bool has = FORM == LORA_SWIGLU;                              // whether the lane's row is written
#pragma unroll
    for (int i = 0; i < NL; ++i) {
#pragma unroll
        for (int j = 0; j < NT; ++j) y[i][j] = float4_t{0.f, 0.f, 0.f, 0.f};
        const LoraDev& l = p.l[i];
        if (l.n == 0) continue;
        const int mine = adapter_of(l, p.rows, row0 + lane, lane < 16 ? M : 0), own = __shfl(mine, c, 64);
        const uint64_t left = __ballot(mine >= 0);
        if (left == 0) continue;
        has |= own >= 0;
        half8_t x[NS];
        float unit;
        inner_operand<NS>(l, own, p.inner[i], p.parts[i], static_cast<size_t>(p.rows.M) * l.R, row, g, x, &unit);
        outer_product<NS, NT>(l, left, mine, own, x, n0, y[i]);
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) y[i][j][r] = own >= 0 ? y[i][j][r] * unit : 0.0f;
    }
    if (row >= M || !has) return;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int n = n0 + 16 * j + 4 * g;
        if (n >= N) continue;                                    // (N is a multiple of 8)
        const size_t at = static_cast<size_t>(row) * p.ldo + n;
        if (FORM == LORA_ADD_F32) {
            float4_t* to = reinterpret_cast<float4_t*>(static_cast<float*>(p.out) + at);
            *to = *to + y[0][j];
        } else if (FORM == LORA_ADD_F16) {
            U2* to = reinterpret_cast<U2*>(static_cast<uint16_t*>(p.out) + at);
            const U2 b = *to;
            const uint32_t w[2] = {b.x, b.y};
            uint16_t h[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) h[r] = to_half(half_bits_to_float(static_cast<uint16_t>(w[r >> 1] >> (16 * (r & 1)) & 0xffffu)) + y[0][j][r]);
            *to = U2{h[0] | static_cast<uint32_t>(h[1]) << 16, h[2] | static_cast<uint32_t>(h[3]) << 16};
        } else {
            const uint16_t* from = p.base + static_cast<size_t>(row) * 2 * N + n;
            const U2 bg = *reinterpret_cast<const U2*>(from), bu = *reinterpret_cast<const U2*>(from + N);
            const uint32_t wg[2] = {bg.x, bg.y}, wu[2] = {bu.x, bu.y};
            uint16_t h[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float gate = half_bits_to_float(static_cast<uint16_t>(wg[r >> 1] >> (16 * (r & 1)) & 0xffffu)) + y[0][j][r];
                const float up = half_bits_to_float(static_cast<uint16_t>(wu[r >> 1] >> (16 * (r & 1)) & 0xffffu)) + y[NL - 1][j][r];
                h[r] = to_half(gate / (1.0f + __expf(-gate)) * up);
            }
            *reinterpret_cast<U2*>(static_cast<uint16_t*>(p.out) + at) = U2{h[0] | static_cast<uint32_t>(h[1]) << 16, h[2] | static_cast<uint32_t>(h[3]) << 16};
        }
    }
}

// Parts of K that fill the chip: tiles of 64 rows, three workgroups per CU.
constexpr int kInnerFill = 768;
int lora_splits(int M) { return std::min(std::max((kInnerFill * 64 + M - 1) / std::max(M, 1), 1), 8); }
size_t lora_inner_bytes(int R, int M) {
    // enough for any number of rows up to M: parts * M <= 8 M, and <= 64 * kInnerFill + M
    const size_t rows = std::min<size_t>(static_cast<size_t>(8) * M, static_cast<size_t>(kInnerFill) * 64 + M);
    return (rows * R * 4 + 255) / 256 * 256;
}

template <int RT, bool ALONE>
static void inner_form(const LoraInner& p, int R, dim3 grid, hipStream_t stream) {
    if (R <= 16) hipLaunchKernelGGL((lora_inner_kernel<RT, 1, ALONE>), grid, dim3(256), 0, stream, p);
    else if (R <= 32) hipLaunchKernelGGL((lora_inner_kernel<RT, 2, ALONE>), grid, dim3(256), 0, stream, p);
    else if (R <= 64) hipLaunchKernelGGL((lora_inner_kernel<RT, 4, ALONE>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((lora_inner_kernel<RT, 8, ALONE>), grid, dim3(256), 0, stream, p);
}

hipError_t launch_lora_inner(const LoraDev* l, int n, const LoraRows& rows, const void* A, float* const* inner, int* parts, hipStream_t stream) {
    if (rows.M <= 0 || n <= 0) return hipSuccess;
    LoraInner p{};
    int R = 0;
    for (int i = 0; i < n; ++i) {
        p.l[i] = l[i];
        p.inner[i] = inner[i];
        R = std::max(R, l[i].R);
    }
    p.rows = rows; p.A = static_cast<const uint16_t*>(A);
    p.parts = std::max(1, std::min(lora_splits(rows.M), (l[0].K + 511) / 512));
    for (int i = 0; i < n; ++i) parts[i] = p.parts;
    // Few rows, whose adapters mostly differ: a workgroup per adapter of the tile.  Many: a tile's adapters one after the other, mostly one.
    if (rows.M <= 256) inner_form<1, true>(p, R, dim3((rows.M + 15) / 16, 16 * p.parts, n), stream);
    else inner_form<4, false>(p, R, dim3((rows.M + 63) / 64, p.parts, n), stream);
    return hipGetLastError();
}

template <int FORM>
static hipError_t outer_form(const LoraOuter& p, int R, int N, hipStream_t stream) {
    if (p.rows.M <= 0) return hipSuccess;
    const dim3 grid((p.rows.M + 15) / 16, (N + 64 * kOuterTiles - 1) / (64 * kOuterTiles));   // (neighbours share a part of up)
    if (R <= 32) hipLaunchKernelGGL((lora_outer_kernel<1, FORM>), grid, dim3(256), 0, stream, p);
    else if (R <= 64) hipLaunchKernelGGL((lora_outer_kernel<2, FORM>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((lora_outer_kernel<4, FORM>), grid, dim3(256), 0, stream, p);
    return hipGetLastError();
}

hipError_t launch_lora_add(const LoraDev& l, const LoraRows& rows, const float* inner, int parts, void* out, int ldo, int f32, hipStream_t stream) {
    LoraOuter p{};
    p.l[0] = l; p.inner[0] = inner; p.parts[0] = parts; p.rows = rows; p.out = out; p.ldo = ldo;
    return f32 ? outer_form<LORA_ADD_F32>(p, l.R, l.N, stream) : outer_form<LORA_ADD_F16>(p, l.R, l.N, stream);
}

hipError_t launch_lora_swiglu(const LoraDev& lg, const LoraDev& lu, const LoraRows& rows, const float* inner_g, const float* inner_u, int parts_g, int parts_u,
                              const void* base, void* out, int N, hipStream_t stream) {
    LoraOuter p{};
    p.l[0] = lg; p.l[1] = lu; p.inner[0] = inner_g; p.inner[1] = inner_u; p.parts[0] = parts_g; p.parts[1] = parts_u;
    p.rows = rows; p.base = static_cast<const uint16_t*>(base); p.out = out; p.ldo = N;
    return outer_form<LORA_SWIGLU>(p, std::max(lg.R, lu.R), N, stream);
}

}  // namespace qtale
