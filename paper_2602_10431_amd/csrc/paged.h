// The paged K/V cache inside the library: its device view, how queries meet pages, and the launchers of its kernels.
//
// A slot is the cache of one sequence at one layer: table[slot][j] is the page of its tokens j * P .. j * P + P - 1 (-1: none, its tokens are
// not seen), kv_len[slot] its tokens, kv_cap[slot] the tokens its pages have room for.  A page is [n_kv_heads][P][d], so the keys of a head in
// a page are contiguous; pages of all layers come from one pool.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace qtale {

struct PagedDev {
    uint16_t *k, *v;             // [n_pages][nkv][P][d] fp16 or bf16
    int32_t* refs;               // [n_pages]
    uint32_t* bits;              // [ceil(n_pages / 32)]
    int32_t* table;              // [n_layers][n_slots][max_pages]
    int32_t *len, *cap;          // [n_layers][n_slots]
    int n_pages, shift, nkv, d, n_layers, n_slots, max_pages, bf16;   // P = 1 << shift
};

// ---- pages (pages.hip) ----------------------------------------------------------------------------
constexpr int kReserveItems = 2048;              // (layer, sequence) pairs that a reserving workgroup holds at once; bound on B
size_t pages_workspace_bytes(const PagedDev& p, int B);
hipError_t launch_pages_init(const PagedDev& p, hipStream_t stream);
hipError_t launch_pages_fork(const PagedDev& p, const int32_t* src, const int32_t* dst, int n, hipStream_t stream);
hipError_t launch_pages_drop(const PagedDev& p, const int32_t* slots, int n, bool release, int window, int sinks, hipStream_t stream);
// layer < 0: every layer.  first/missing nullable; first [layers of the call][B]: the lengths before; then kv_len advances.
// split: also the launch that copies shared pages; without it the next launch on the list has to.
hipError_t launch_pages_reserve(const PagedDev& p, int layer, const int32_t* seq_offsets, const int32_t* slots, int B, int32_t* first,
                                int32_t* missing, bool split, void* workspace, hipStream_t stream);
hipError_t launch_pages_compact(const PagedDev& p, int32_t* n_live, void* workspace, hipStream_t stream);
hipError_t launch_pages_copy(const PagedDev& from, const PagedDev& to, const int32_t* src, const int32_t* dst, int n, hipStream_t stream);

// ---- rotary embedding + append (paged_rope.hip) ---------------------------------------------------
struct SplitList {               // pages to copy (pages_reserve_kernel's list)
    const int32_t* n;
    const int4* entries;         // from, to, tokens, -
};
SplitList pages_split_list(void* workspace);

struct PagedRopeArgs {
    PagedDev kv;                 // table and len of the layer
    int layout, rotary_dim;      // 0 half, 1 interleaved
    const double* freqs;         // device [rotary_dim / 2]
    float magnitude;
    const uint16_t *q, *k, *v;
    uint16_t* q_out;
    int64_t q_stride, k_stride, v_stride, q_out_stride;              // elements between tokens
    int nh, T, B;
    const int32_t* seq_offsets;
    const int32_t* slots;        // nullable
    const int32_t* first;        // nullable: kv_len - new tokens
    const int32_t* positions;
    const int32_t* rows;         // nullable: token of row i is rows[i]
    const int32_t* count;        // nullable: rows on the device (T is its bound)
    SplitList copies;            // nullable: pages that the workgroups past the T rows copy
};
hipError_t launch_paged_rope(const PagedRopeArgs& a, hipStream_t stream);

// ---- attention (paged_decode.hip, paged_prefill.hip) ----------------------------------------------
struct PagedAttnDev {
    const uint16_t* q;
    uint16_t* out;
    int64_t q_stride, out_stride;
    const uint16_t *k, *v;
    const int32_t *table, *len;  // of the layer
    const int32_t *offs, *slots, *first;
    int B, nh, nkv, rep, shift, max_pages, n_slots, n_pages;
    int window, sinks, max_len;
    float scale_log2;
    int take;                    // 0: every sequence; 1: only those of this kernel (the other one is launched too)
    // chunk kernel: column tiles (bound), key ranges that one may be cut into (1: none), workgroups that the call's ranges are to be, and the
    // ranges' sums [T * nh][ranges][part_stride(d)]
    int items, ranges, target;
    float* part;
    // decode kernel: spans per kv head that the call's keys are cut into (0: a workgroup per sequence), the sums of a span's first and last
    // piece [nkv][spans][2][kDecodeCols][part_stride(d)], and where a sequence's pieces are: [B] (first span, pieces, place of the first, -)
    int spans, cols;             // cols: bound on the columns of a sequence of this kernel
    int stream_keys;             // without spans: non-temporal keys
    float* span_part;
    int4* pieces;
};
struct PagedAttnPlan {
    bool decode, chunk;          // which kernels run
    int cols, spans, stream_keys;    // decode; cols: bound on those of a sequence of its
    int ranges, target, groups, items;   // chunk; groups of waves per workgroup that share its keys, 0: the wide form
    bool too_large;              // more workgroups than a grid has
    size_t decode_bytes, bytes;  // of workspace: the decode kernel's, all
};
constexpr int kDecodeCols = 16;                  // (query, head) pairs per kv head that a workgroup of the decode kernel holds
constexpr int kChunkCols = 128;                  // ... and a workgroup of the chunk kernel
constexpr int kWideCols = 256;                   // ... of its form with two halves that take turns
constexpr int kChunkTileKeys = 64;
constexpr int kSpanSeqs = 1024;                  // bound on the sequences of a call that is cut into spans
constexpr int part_stride(int d) { return d + 4; }   // floats of a column's sums: numerators, reference point, denominator, (chunk) ranges, unused
PagedAttnPlan plan_paged_attention(int nh, int nkv, int d, int T, int B, int max_new, int max_len, int window, int sinks);
size_t paged_attention_bytes(int nh, int nkv, int d, int T, int B);   // of workspace, for any call of at most T tokens and B sequences
// All launches of a call; a: everything but `take` and what follows it, which the plan says.
hipError_t launch_paged_attention(PagedAttnDev a, const PagedAttnPlan& plan, int d, int bf16, int T, float* workspace, hipStream_t stream);
hipError_t launch_paged_decode(const PagedAttnDev& a, int d, int bf16, hipStream_t stream);
hipError_t launch_paged_chunk(const PagedAttnDev& a, int groups, int d, int bf16, hipStream_t stream);
hipError_t launch_chunk_combine(const PagedAttnDev& a, int d, int bf16, int T, hipStream_t stream);

#ifdef __HIP_DEVICE_COMPILE__
#define QT_CONST_AS __attribute__((address_space(4)))
#else
#define QT_CONST_AS
#endif

// The keys that queries p0 .. p1 of a slot with `len` tokens may see, as steps of G keys: those of the first tokens that stay, then those of
// the window.  Steps next to each other in memory are walked as one run.
template <int G>
struct KeySteps {
    int lo, hi, first_steps, base, steps;        // window [lo, hi); steps [0, first_steps) start at key 0, the others at `base`
    __device__ __forceinline__ KeySteps(int p0, int p1, int len, int window, int sinks) {
        hi = max(min(p1 + 1, len), 0);
        lo = window > 0 ? max(p0 + 1 - window, 0) : 0;
        const int stay = min(min(sinks, lo), hi);
        first_steps = (stay + G - 1) / G;
        base = lo & ~(G - 1);
        if (first_steps * G >= base) { first_steps = 0; if (stay > 0) base = 0; }
        steps = first_steps + (hi > base ? (hi - base + G - 1) / G : 0);
    }
    __device__ __forceinline__ int key(int s) const { return s < first_steps ? s * G : base + (s - first_steps) * G; }
};

}  // namespace qtale
