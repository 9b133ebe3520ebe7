// Low-rank adapters of many requests beside a shared projection: what the kernels take, and their launchers.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace qtale {

struct LoraDev {
    const uint16_t *down, *up;   // fp16 [n][R][K], [n][N][R]
    const int32_t* rank;         // nullable: R
    const float* scale;          // nullable: 1
    int n, R, N, K;              // n == 0: no adapters
};
// Which adapter a row has: adapter[row_seq ? row_seq[i] : i]
struct LoraRows {
    const int32_t* adapter;
    const int32_t* row_seq;      // nullable
    const int32_t* count;        // nullable: rows on the device (M is its bound)
    int M;
    int n_seq;                   // with row_seq: entries of adapter
};
size_t lora_inner_bytes(int R, int M);           // of one linear's inner values

// inner = down_a A_i of every row, [M][R] fp32
hipError_t launch_lora_inner(const LoraDev& l, const LoraRows& rows, const void* A, float* inner, hipStream_t stream);
// out (fp16, or fp32 if f32; ldo elements between rows) += scale up_a inner_i
hipError_t launch_lora_add(const LoraDev& l, const LoraRows& rows, const float* inner, void* out, int ldo, int f32, hipStream_t stream);
// out [M][N] = silu(gate + ...) * (up + ...), gate and up fp16 [M][N]
hipError_t launch_lora_swiglu(const LoraDev& lg, const LoraDev& lu, const LoraRows& rows, const float* inner_g, const float* inner_u,
                              const void* gate, const void* up, void* out, int N, hipStream_t stream);

}  // namespace qtale
