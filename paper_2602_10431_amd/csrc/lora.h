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
constexpr int kLoraMost = 3;     // linears with the same input that one launch takes

size_t lora_inner_bytes(int R, int M);           // of one linear's inner values, for up to M rows

// inner = down_a A_i of every row, for `n` linears of one input [M][K]: in parts over K for the calls below, or, of many rows, their sums as the second
// product's operands.  What belongs to no adapter, or lies past a rank, is not written.  *operands, *parts (host out): of each linear, for the calls below
hipError_t launch_lora_inner(const LoraDev* l, int n, const LoraRows& rows, const void* A, float* const* inner, const float** operands, int* parts,
                             hipStream_t stream);
// out (ldo elements between rows) += scale up_a inner_i
hipError_t launch_lora_add(const LoraDev& l, const LoraRows& rows, const float* operands, int parts, float* out, int ldo, hipStream_t stream);
// out (fp16, ldo elements between rows) = base (ldb) + scale up_a inner_i, rounded once; rows without an adapter (of l without any: all) are base, rounded
hipError_t launch_lora_round(const LoraDev& l, const LoraRows& rows, const float* operands, int parts, const float* base, int ldb, void* out, int ldo,
                             hipStream_t stream);
// out [M][N] = silu(gate + ...) * (up + ...); base [M][2 N]: gate's columns, then up's
hipError_t launch_lora_swiglu(const LoraDev& lg, const LoraDev& lu, const LoraRows& rows, const float* operands_g, const float* operands_u, int parts_g,
                              int parts_u, const float* base, void* out, int N, hipStream_t stream);

}  // namespace qtale
