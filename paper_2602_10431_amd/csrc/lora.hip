// Low-rank adapters: a row's inner values, one wave each, and their product with its adapter's second matrix, one thread per value.
#include "lora.h"

#include "qtale_dev.h"

namespace qtale {

__device__ __forceinline__ int adapter_of(const LoraDev& l, const LoraRows& rows, int i) {
    const int seq = rows.row_seq ? rows.row_seq[i] : i;
    if (rows.row_seq && static_cast<uint32_t>(seq) >= static_cast<uint32_t>(rows.n_seq)) return -1;
    const int a = rows.adapter[seq];
    return static_cast<uint32_t>(a) < static_cast<uint32_t>(l.n) ? a : -1;
}
__device__ __forceinline__ int rank_of(const LoraDev& l, int a) { return a < 0 ? 0 : l.rank ? min(max(l.rank[a], 0), l.R) : l.R; }

__global__ void __launch_bounds__(256)
lora_inner_kernel(LoraDev l, LoraRows rows, const uint16_t* A, float* inner) {
    const int i = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (rows.count && i >= *rows.count) return;
    const int a = adapter_of(l, rows, i), rank = rank_of(l, a);
    for (int r = wave; r < l.R; r += 4) {
        float sum = 0.0f;
        if (r < rank) {
            const uint16_t* w = l.down + (static_cast<size_t>(a) * l.R + r) * l.K;
            const uint16_t* x = A + static_cast<size_t>(i) * l.K;
            for (int k = lane; k < l.K; k += 64) sum = fmaf(half_bits_to_float(x[k]), half_bits_to_float(w[k]), sum);
            sum = wave_sum(sum);
        }
        if (lane == 0) inner[static_cast<size_t>(i) * l.R + r] = sum;
    }
}

__device__ __forceinline__ float lora_value(const LoraDev& l, int a, const float* inner, int n) {
    const int rank = rank_of(l, a);
    if (rank == 0) return 0.0f;
    const uint16_t* w = l.up + (static_cast<size_t>(a) * l.N + n) * l.R;
    float sum = 0.0f;
    for (int r = 0; r < rank; ++r) sum = fmaf(half_bits_to_float(w[r]), inner[r], sum);
    return l.scale ? sum * l.scale[a] : sum;
}

// As the shared product's results: saturating; a NaN stays one.
__device__ __forceinline__ uint16_t to_half(float f) { return f == f ? float_to_half_bits(f) : 0x7e00u; }

template <bool F32>
__global__ void __launch_bounds__(256)
lora_add_kernel(LoraDev l, LoraRows rows, const float* inner, void* out, int ldo) {
    const int i = blockIdx.y, n = blockIdx.x * 256 + threadIdx.x;
    if (n >= l.N || (rows.count && i >= *rows.count)) return;
    const int a = adapter_of(l, rows, i);
    if (a < 0) return;
    const float add = lora_value(l, a, inner + static_cast<size_t>(i) * l.R, n);
    const size_t at = static_cast<size_t>(i) * ldo + n;
    if (F32) static_cast<float*>(out)[at] += add;
    else static_cast<uint16_t*>(out)[at] = to_half(half_bits_to_float(static_cast<uint16_t*>(out)[at]) + add);
}

__global__ void __launch_bounds__(256)
lora_swiglu_kernel(LoraDev lg, LoraDev lu, LoraRows rows, const float* inner_g, const float* inner_u, const uint16_t* gate, const uint16_t* up,
                   uint16_t* out, int N) {
    const int i = blockIdx.y, n = blockIdx.x * 256 + threadIdx.x;
    if (n >= N || (rows.count && i >= *rows.count)) return;
    const size_t at = static_cast<size_t>(i) * N + n;
    float g = half_bits_to_float(gate[at]), u = half_bits_to_float(up[at]);
    if (lg.n > 0) g += lora_value(lg, adapter_of(lg, rows, i), inner_g + static_cast<size_t>(i) * lg.R, n);
    if (lu.n > 0) u += lora_value(lu, adapter_of(lu, rows, i), inner_u + static_cast<size_t>(i) * lu.R, n);
    out[at] = to_half(g / (1.0f + expf(-g)) * u);
}

size_t lora_inner_bytes(int R, int M) { return (static_cast<size_t>(M) * R * 4 + 255) / 256 * 256; }

hipError_t launch_lora_inner(const LoraDev& l, const LoraRows& rows, const void* A, float* inner, hipStream_t stream) {
    hipLaunchKernelGGL(lora_inner_kernel, dim3(rows.M), dim3(256), 0, stream, l, rows, static_cast<const uint16_t*>(A), inner);
    return hipGetLastError();
}
hipError_t launch_lora_add(const LoraDev& l, const LoraRows& rows, const float* inner, void* out, int ldo, int f32, hipStream_t stream) {
    const dim3 grid((l.N + 255) / 256, rows.M);
    if (f32) hipLaunchKernelGGL(lora_add_kernel<true>, grid, dim3(256), 0, stream, l, rows, inner, out, ldo);
    else hipLaunchKernelGGL(lora_add_kernel<false>, grid, dim3(256), 0, stream, l, rows, inner, out, ldo);
    return hipGetLastError();
}
hipError_t launch_lora_swiglu(const LoraDev& lg, const LoraDev& lu, const LoraRows& rows, const float* inner_g, const float* inner_u,
                              const void* gate, const void* up, void* out, int N, hipStream_t stream) {
    hipLaunchKernelGGL(lora_swiglu_kernel, dim3((N + 255) / 256, rows.M), dim3(256), 0, stream, lg, lu, rows, inner_g, inner_u,
                       static_cast<const uint16_t*>(gate), static_cast<const uint16_t*>(up), static_cast<uint16_t*>(out), N);
    return hipGetLastError();
}

}  // namespace qtale
