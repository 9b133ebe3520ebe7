// Host side of the adapters' C ABI (include/qtale.h): argument validation before any HIP call, then the launches.
#include <algorithm>

#include "lora_check.h"
#include "qtale_kernels.h"

using namespace qtale;

namespace {

#define HIP_TRY(expr)                                   \
    do {                                                \
        hipError_t e__ = (expr);                        \
        if (e__ != hipSuccess) return QTALE_ERR_HIP;    \
    } while (0)

int check_base(const qtale_qlinear* w, int bits, int group) {
    if (!w || w->N <= 0 || w->K <= 0) return QTALE_ERR_INVALID_ARG;
    if (bits != 4 && bits != 3 && bits != 2) return QTALE_ERR_UNSUPPORTED;
    if (group != 32 && group != 64 && group != 128) return QTALE_ERR_UNSUPPORTED;
    return w->K % 8 != 0 || w->N % 8 != 0 ? QTALE_ERR_SHAPE : QTALE_OK;
}

int check_lora_call(const int32_t* adapter, const void* A, const void* out, const void* ws, size_t have, size_t need) {
    if (!adapter || !A || !out || !ws || reinterpret_cast<uintptr_t>(ws) % 256 != 0) return QTALE_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(A) | reinterpret_cast<uintptr_t>(out)) % 16 != 0) return QTALE_ERR_INVALID_ARG;
    return have < need ? QTALE_ERR_WORKSPACE_TOO_SMALL : QTALE_OK;
}

// The shared product alone in fp32 (it is rounded with what the adapters add), of one linear or of two side by side ([M][2 N]).
hipError_t base_linear(const qtale_qlinear* w, const qtale_qlinear* w2, int bits, int group, const void* A, int M, float* out, hipStream_t stream) {
    GemmArgs g{};
    g.A = A; g.M_max = M; g.rows_exact = 1; g.K = w->K; g.group = group; g.bits = bits; g.n_w = w2 ? 2 : 1;
    g.w[0] = {w->prepacked, w->N, w->K};
    if (w2) g.w[1] = {w2->prepacked, w2->N, w2->K};
    g.epilogue = EPI_STORE_F16; g.out_f32 = 1; g.out = out; g.ldo = w->N * g.n_w;
    return launch_gemm_w4a16(g, stream);
}

// Rows that are done at a time, which bounds the scratch.  (Each product fills the chip many times over.)
constexpr int kRowsAtOnce = 8192;
size_t rows_bytes(int M, int N) { return (static_cast<size_t>(M) * N * 4 + 255) / 256 * 256; }
size_t inner_bytes(const qtale_lora* l, int M) { return l ? lora_inner_bytes(l->max_rank, M) : 0; }

}  // namespace

extern "C" {

size_t qtale_lora_workspace_bytes(const qtale_lora* a, const qtale_lora* b, int M) {
    if (!a || check_lora(a, a->N, a->K, false) || (b && check_lora(b, a->N, a->K, false)) || M < 0 || a->N <= 0 || a->K <= 0) return 0;
    M = std::min(M, kRowsAtOnce);
    return 256 + inner_bytes(a, M) + inner_bytes(b, M) + (b ? 2 : 1) * rows_bytes(M, a->N);
}

int qtale_linear_lora_w4a16(const qtale_qlinear* w, int bits, int group, const qtale_lora* lora, const int32_t* adapter, const void* A, int M,
                            void* out, void* workspace, size_t workspace_bytes, void* stream) {
    int e = check_base(w, bits, group);
    if (e || (e = check_lora(lora, w->N, w->K, M > 0))) return e;
    if (M < 0) return QTALE_ERR_INVALID_ARG;
    if (M == 0) return QTALE_OK;
    if (!w->prepacked) return QTALE_ERR_INVALID_ARG;
    if ((e = check_lora_call(adapter, A, out, workspace, workspace_bytes, qtale_lora_workspace_bytes(lora, nullptr, M)))) return e;
    const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const LoraDev l = lora_device(lora);
    float* inner = static_cast<float*>(workspace);
    float* base = reinterpret_cast<float*>(static_cast<char*>(workspace) + inner_bytes(lora, std::min(M, kRowsAtOnce)));
    for (int m = 0; m < M; m += kRowsAtOnce) {
        const int n = std::min(M - m, kRowsAtOnce);
        const LoraRows rows{adapter + m, nullptr, nullptr, n, 0};
        const uint16_t* x = static_cast<const uint16_t*>(A) + static_cast<size_t>(m) * w->K;
        const float* operands = nullptr;
        int parts = 0;
        HIP_TRY(launch_lora_inner(&l, 1, rows, x, &inner, &operands, &parts, s));
        HIP_TRY(base_linear(w, nullptr, bits, group, x, n, base, s));
        HIP_TRY(launch_lora_round(l, rows, operands, parts, base, w->N, static_cast<uint16_t*>(out) + static_cast<size_t>(m) * w->N, w->N, s));
    }
    return QTALE_OK;
}

int qtale_swiglu_lora_w4a16(const qtale_qlinear* gate, const qtale_qlinear* up, int bits, int group, const qtale_lora* lora_gate,
                            const qtale_lora* lora_up, const int32_t* adapter, const void* A, int M, void* out, void* workspace,
                            size_t workspace_bytes, void* stream) {
    int e = check_base(gate, bits, group);
    if (e || (e = check_base(up, bits, group))) return e;
    if (gate->N != up->N || gate->K != up->K) return QTALE_ERR_SHAPE;
    if (!lora_gate && !lora_up) return QTALE_ERR_INVALID_ARG;
    if (lora_gate && (e = check_lora(lora_gate, gate->N, gate->K, M > 0))) return e;
    if (lora_up && (e = check_lora(lora_up, up->N, up->K, M > 0))) return e;
    if (M < 0) return QTALE_ERR_INVALID_ARG;
    if (M == 0) return QTALE_OK;
    if (!gate->prepacked || !up->prepacked) return QTALE_ERR_INVALID_ARG;
    // (a size for one of them counts the rows' buffers too: the pair's size with the larger rank twice is enough for either)
    const int most = std::min(M, kRowsAtOnce);
    const size_t need = 256 + inner_bytes(lora_gate, most) + inner_bytes(lora_up, most) + 2 * rows_bytes(most, gate->N);
    if ((e = check_lora_call(adapter, A, out, workspace, workspace_bytes, need))) return e;
    const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const LoraDev lg = lora_device(lora_gate), lu = lora_device(lora_up);
    char* at = static_cast<char*>(workspace);
    float* inner_g = reinterpret_cast<float*>(at);
    float* inner_u = reinterpret_cast<float*>(at += inner_bytes(lora_gate, most));
    float* base = reinterpret_cast<float*>(at += inner_bytes(lora_up, most));
    for (int m = 0; m < M; m += kRowsAtOnce) {
        const int rows_here = std::min(M - m, kRowsAtOnce);
        const LoraRows rows{adapter + m, nullptr, nullptr, rows_here, 0};
        const uint16_t* x = static_cast<const uint16_t*>(A) + static_cast<size_t>(m) * gate->K;
        LoraDev l[2];
        float* inner[2];
        const float* operands[2] = {nullptr, nullptr};
        int parts[2] = {0, 0}, n = 0;
        if (lg.n) { l[n] = lg; inner[n++] = inner_g; }
        if (lu.n) { l[n] = lu; inner[n++] = inner_u; }
        HIP_TRY(launch_lora_inner(l, n, rows, x, inner, operands, parts, s));
        HIP_TRY(base_linear(gate, up, bits, group, x, rows_here, base, s));
        HIP_TRY(launch_lora_swiglu(lg, lu, rows, operands[0], operands[n - 1], parts[0], parts[n - 1], base,
                                   static_cast<uint16_t*>(out) + static_cast<size_t>(m) * gate->N, gate->N, s));
    }
    return QTALE_OK;
}

}  // extern "C"
