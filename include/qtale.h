/*
 * qtale.h - C ABI of the MI355X (gfx950) library for QTALE's inference hot path:
 * the token-adaptive, weight-only int4 group-quantized decoder-layer forward.
 *
 * What the calls compute (paper: "QTALE: Quantization-Robust Token-Adaptive Layer Execution"):
 *   - every layer has a router g_l that scores each token of the layer's input x_l (Sec. 2.2, Eq. 2);
 *   - a token executes the layer iff its execute probability p_{l,0} = softmax(g_l(x_l))_0 is at least
 *     a threshold theta shared by all layers (Sec. 3.4, Eq. 9); theta = 0.5 is the arg-max rule of Eq. 2;
 *   - executed tokens take x_{l+1} = x_l + f_l(x_l) (Eq. 1), bypassed tokens keep x_{l+1} = x_l
 *     bit for bit (Eq. 3);
 *   - executed tokens are gathered into a dense matrix before the layer runs (App. B.2);
 *   - the layer's linears are weight-only group-quantized (4 bit, groups along the input dimension,
 *     Sec. 4.1); the execution ratio is changed at run time without touching the weights (Sec. 3.4).
 * The paper fixes neither the quantizer's arithmetic nor the inside of f_l; this library uses a
 * round-to-nearest asymmetric min/max quantizer with fp16 scale and integer zero-point, a linear
 * router whose output is the execute-minus-bypass logit z (p_{l,0} = sigmoid(z)), and a pre-norm
 * LLaMA block (RMSNorm, rotary embedding at the token's ORIGINAL absolute position with half-split
 * pairing, causal softmax attention among the EXECUTED tokens of the same sequence, SwiGLU MLP).
 *
 * Conventions
 *   - All data pointers are DEVICE pointers unless a comment says "host".  The caller owns every
 *     buffer; the library never allocates, frees or keeps device memory.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).  All work is enqueued
 *     on it and the calls return without waiting for the GPU.
 *   - Every call returns 0 (QTALE_OK) or a negative error code.  Arguments are validated before the
 *     first HIP call, so invalid arguments are reported even on a machine without a GPU.
 *   - Matrices are row-major.  "act dtype" is cfg->act_dtype (IEEE fp16 or bfloat16), the type of
 *     the residual stream and of the RMSNorm gains.  K/V caches are always fp16.
 */
#ifndef QTALE_H
#define QTALE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
    QTALE_OK = 0,
    QTALE_ERR_INVALID_ARG = -1,        /* null pointer, NaN/out-of-range control value, negative size */
    QTALE_ERR_SHAPE = -2,              /* shapes inconsistent with each other or with the kernels' granularity */
    QTALE_ERR_UNSUPPORTED = -3,        /* bits/group/head_dim the kernels do not implement */
    QTALE_ERR_WORKSPACE_TOO_SMALL = -4,
    QTALE_ERR_HIP = -5                 /* a HIP runtime call or a kernel launch failed */
};

enum { QTALE_ACT_FP16 = 0, QTALE_ACT_BF16 = 1 };
enum { QTALE_MODE_RATIO = 0, QTALE_MODE_THRESHOLD = 1 };

const char* qtale_strerror(int code);

/* ---- control state: which tokens execute (Sec. 3.4) --------------------------------------------
 * A context only holds the selection mode and its value.  Default: ratio mode, r = 1. */
typedef struct qtale_ctx qtale_ctx;
int qtale_create(qtale_ctx** out);
int qtale_destroy(qtale_ctx* ctx);

/* Ratio mode: in every layer of every later forward call exactly k = floor(r*T + 1/2) of the call's T
 * tokens execute, namely the k with the highest router score (equal scores: lower token index first).
 * r in [0,1]; NaN or out of range -> QTALE_ERR_INVALID_ARG.  Touches no weight buffer. */
int qtale_set_exec_ratio(qtale_ctx* ctx, float r);
/* Threshold mode (Eq. 9 verbatim): a token executes iff sigmoid(z) >= theta, decided as
 * z >= fp32(ln(theta/(1-theta))).  theta <= 0 executes every token, theta >= 1 none; NaN -> error. */
int qtale_set_threshold(qtale_ctx* ctx, float theta);
int qtale_get_control(const qtale_ctx* ctx, int* mode /*host*/, float* value /*host*/);

/* ---- quantized weights (Sec. 4.1: weight-only, groups along the input dimension) ----------------
 * W is [N][K] (out x in), fp32.  Per (row n, group g of `group` consecutive k; the last group may be
 * short): lo = min(0,min W), hi = max(0,max W), scale = fp16((hi-lo)/(2^bits-1)) (1.0 if that is 0 or
 * not finite), zero = clamp(rint(-lo/scale)), code = clamp(rint(W/scale)+zero); IEEE fp32 arithmetic,
 * round-half-even.  Dequantized weight: (code - zero) * scale.
 *   codes     bits = 4: [N][ceil(K/8)] uint32, nibble j of word w = code of k = 8*w + j;
 *             bits = 3: [N][3*ceil(K/32)] uint32, the row's codes as one little-endian bit stream, code k
 *             at bits 3k..3k+2 (32 codes fill three words); row tails padded with code 0
 *   scales    [N][ceil(K/group)] fp16 bit patterns
 *   zeros     [N][ceil(K/group)] fp16 bit patterns of the integer zero-point
 *   prepacked the kernels' private copy (codes reordered for the matrix-core operand layout plus
 *             scale/zero pairs), qtale_prepacked_bytes() bytes, 16-byte aligned; may be NULL here.
 * Supported: bits in {4, 3} (Sec. 4.1 evaluates both) and 2 (for mixed 2-/4-bit stacks: 16 codes per word,
 * bit pair j of word w = code of k = 16*w + j); group in {32, 64, 128}; K % 8 == 0.  Else
 * QTALE_ERR_UNSUPPORTED / _SHAPE.
 * The GEMM entry points (forward calls, qtale_linear_w4a16, qtale_swiglu_w4a16) also need N % 8 == 0. */
size_t qtale_prepacked_bytes(int N, int K, int bits, int group);
int qtale_quantize(const float* W, int N, int K, int bits, int group,
                   uint32_t* codes, uint16_t* scales, uint16_t* zeros,
                   void* prepacked /*nullable*/, void* stream);
/* Builds `prepacked` from canonical codes/scales/zeros (e.g. weights quantized elsewhere). */
int qtale_prepack(const uint32_t* codes, const uint16_t* scales, const uint16_t* zeros,
                  int N, int K, int bits, int group, void* prepacked, void* stream);

typedef struct {
    const uint32_t* codes;      /* canonical; not read by the forward calls, may be NULL */
    const uint16_t* scales;     /* canonical; may be NULL */
    const uint16_t* zeros;      /* canonical; may be NULL */
    const void* prepacked;      /* required by the forward calls */
    int N, K;
} qtale_qlinear;

typedef struct {
    int hidden, n_heads, n_kv_heads, head_dim, inter;   /* head_dim must be 64 or 128 */
    int bits;                                           /* 4, 3 or 2: default code width of the seven linears */
    int group;                                          /* 32, 64 or 128 */
    int act_dtype;                                      /* QTALE_ACT_FP16 | QTALE_ACT_BF16 */
    float rms_eps;                                      /* e.g. 1e-5 */
    float rope_base;                                    /* e.g. 10000 */
} qtale_layer_cfg;

typedef struct {
    qtale_qlinear q, k, v, o, gate, up, down;  /* q [nh*d][H], k,v [nkv*d][H], o [H][nh*d], gate,up [I][H], down [H][I] */
    const void* norm1;                         /* [hidden], act dtype: gain of the pre-attention RMSNorm */
    const void* norm2;                         /* [hidden], act dtype: gain of the pre-MLP RMSNorm */
    const float* router_w;                     /* [hidden] fp32: z_t = router_w . x_t + router_b */
    float router_b;
    /* Optional two-output MLP router (Sec. 2.2), used instead of router_w/router_b when router_hidden > 0:
     * u = relu(W1 x_t + b1), (l_e, l_b) = W2 u + b2, z_t = l_e - l_b (p_0 of Eq. 9 = sigmoid(z_t)); fp64 sums,
     * one rounding to fp32.  The paper gives no depth, width or activation: one hidden ReLU layer is this
     * library's reading.  router_hidden in 1..256; router_w may then be NULL. */
    int router_hidden;                         /* R; 0 = linear router */
    const float* router_w1;                    /* [R][hidden] fp32 */
    const float* router_b1;                    /* [R] fp32 */
    const float* router_w2;                    /* [2][R] fp32: row 0 execute logit, row 1 bypass logit */
    const float* router_b2;                    /* [2] fp32 */
    int bits;                                  /* code width of THIS layer's linears; 0 = cfg->bits (mixed-precision stacks) */
} qtale_layer_weights;

/* Per-layer K/V cache holding entries of EXECUTED tokens only (a bypassed token produces no key or
 * value at that layer).  k_cache/v_cache: [B][n_kv_heads][cap][head_dim] fp16 (the entries of one sequence
 * and head are contiguous: decode attention streams them at the full memory rate); kv_len [B] int32 device:
 * entries already present per sequence.  A forward call appends the executed tokens of sequence b (keys
 * after rotary embedding) at kv_len[b].. and adds their number to kv_len[b].  The caller should guarantee
 * kv_len[b] + (tokens of sequence b in the call) <= cap.  If it does not, the entries that would not fit are
 * dropped (the newest tokens of the call), kv_len[b] stops at cap, and those tokens' own queries attend to the cap
 * entries present: kv_len[b] == cap after a call is the caller's sign that the cache is full. */
typedef struct {
    void* k_cache;
    void* v_cache;
    int32_t* kv_len;
    int cap;
} qtale_kv;

/* Bytes of scratch a forward call with at most max_tokens tokens in max_seqs sequences needs.
 * Returns 0 for an invalid cfg. */
size_t qtale_workspace_bytes(const qtale_layer_cfg* cfg, int max_tokens, int max_seqs);

/* One token-adaptive layer (Eq. 1, 3, 9; App. B.2), in place on x.
 *   x            [T][hidden] act dtype; rows of bypassed tokens are not written
 *   seq_offsets  [B+1] int32: tokens seq_offsets[b]..seq_offsets[b+1]-1 form sequence b, in order;
 *                seq_offsets[0] = 0, seq_offsets[B] = T
 *   positions    [T] int32: absolute position of every token (for the rotary embedding)
 *   kv           nullable: NULL = the call's tokens are the whole context (pure prefill)
 *   sel_idx      nullable [T] int32 out: ascending indices of the executed tokens (first *sel_count valid)
 *   sel_count    nullable [1] int32 out
 *   scores       nullable [T] fp32 out: router scores z
 *   workspace    >= qtale_workspace_bytes(cfg, T, B) bytes, 256-byte aligned
 * T = 0 is a no-op.  With k = 0 executed tokens no kernel touches x. */
int qtale_layer_forward(qtale_ctx* ctx, const qtale_layer_cfg* cfg, const qtale_layer_weights* w,
                        void* x, int T, const int32_t* seq_offsets, int B, const int32_t* positions,
                        const qtale_kv* kv, int32_t* sel_idx, int32_t* sel_count, float* scores,
                        void* workspace, size_t workspace_bytes, void* stream);

/* For callers that cannot allocate device memory (code under HIP graph capture, tight serving loops, harnesses
 * that forbid hipMalloc): qtale_layer_forward with the workspace taken from an array inside the library instead
 * of a caller buffer.  Same arguments, same kernels and bit-identical results; the call allocates and frees
 * nothing.  The array is QTALE_STATIC_SCRATCH_BYTES large (enough for a decode step of 128 one-token sequences
 * at hidden 5120 / 40 heads / SwiGLU 13824, or about 250 prefill tokens at hidden 4096 / SwiGLU 11008) and every
 * GPU the library runs on holds one copy until the process ends.  A call whose workspace
 * (qtale_workspace_bytes(cfg, T, B)) is larger returns QTALE_ERR_WORKSPACE_TOO_SMALL before any GPU work.
 * All calls on one GPU share that GPU's array: calls that overlap on one GPU (different streams or threads) race;
 * serialize them.  Returns QTALE_ERR_INVALID_ARG while per-kernel profiling is enabled. */
#define QTALE_STATIC_SCRATCH_BYTES (40u << 20)
size_t qtale_static_scratch_bytes(void);
int qtale_layer_forward_static(qtale_ctx* ctx, const qtale_layer_cfg* cfg, const qtale_layer_weights* w,
                               void* x, int T, const int32_t* seq_offsets, int B, const int32_t* positions,
                               const qtale_kv* kv, int32_t* sel_idx, int32_t* sel_count, float* scores,
                               void* stream);

/* n_layers layers in sequence with the context's single control value (one global knob, Sec. 3.4).
 *   layers       host array [n_layers]
 *   kv_per_layer host array [n_layers], nullable
 *   sel_idx      nullable [n_layers][T]; sel_count nullable [n_layers]; scores nullable [n_layers][T]
 *   dbg_hidden   nullable [n_layers][T][hidden] act dtype: receives the INPUT of every layer */
int qtale_stack_forward(qtale_ctx* ctx, const qtale_layer_cfg* cfg, const qtale_layer_weights* layers,
                        int n_layers, void* x, int T, const int32_t* seq_offsets, int B,
                        const int32_t* positions, const qtale_kv* kv_per_layer,
                        int32_t* sel_idx, int32_t* sel_count, float* scores, void* dbg_hidden,
                        void* workspace, size_t workspace_bytes, void* stream);

/* ---- single steps of the path, exposed for tests and per-kernel measurement --------------------- */

/* Router scores and selection alone (steps 1-3 of a layer): z, ascending idx, count. */
int qtale_router_select(qtale_ctx* ctx, int act_dtype, const void* x, int T, int hidden,
                        const float* router_w, float router_b,
                        const int32_t* seq_offsets, int B,
                        float* scores /*[T]*/, int32_t* sel_idx /*[T]*/, int32_t* sel_count /*[1]*/,
                        int32_t* cu_exec /*nullable [B+1]: executed tokens before each sequence*/,
                        void* stream);

/* ---- threshold calibration (Sec. 3.4: two-phase grid search for the global theta) --------------------
 * Candidates theta_n = fp32(n/100), n = 1..50 (the search range (0, 0.5]).  Coarse pass over n = 5, 10,
 * ..., 50, then the not yet evaluated n within 4 steps of the best coarse point; the result is the evaluated
 * n whose average execution ratio R_avg is closest to target_ratio (ties: the larger theta).  The paper's
 * objective is a task metric on calibration data; here it is the execution ratio itself.
 * Both calls synchronize `stream`, allocate nothing, and on success leave ctx in threshold mode at the theta
 * found (as qtale_set_threshold would); on failure the control value is unchanged.
 *   scratch    device, qtale_calibration_scratch_bytes(n_layers) bytes (n_layers = 0 for the score form)
 *   theta, ratio  host out (nullable): theta found and its R_avg
 *   table      host out (nullable) [50]: R_avg of every evaluated candidate at index n-1, NaN elsewhere */
#define QTALE_THETA_GRID 50
size_t qtale_calibration_scratch_bytes(int n_layers);
/* Scores taken as fixed: scores is a device array of n fp32 router scores (e.g. [L][T] written by a forward
 * call); R_avg(theta) = fraction of them with sigmoid(z) >= theta, decided as in qtale_set_threshold. */
int qtale_calibrate_threshold_from_scores(qtale_ctx* ctx, const float* scores, int64_t n, float target_ratio,
                                          void* scratch, float* theta, float* ratio, float* table, void* stream);
/* R_avg measured: for every candidate the stack runs in threshold mode on the calibration batch (skipping
 * changes the hidden states later routers see) and R_avg = executed (layer, token) pairs / (n_layers * T).
 * x_calib [T][hidden] act dtype is only read; x_work (same size) is overwritten.  No K/V cache is used.
 * Other arguments as in qtale_stack_forward. */
int qtale_calibrate_threshold(qtale_ctx* ctx, const qtale_layer_cfg* cfg, const qtale_layer_weights* layers,
                              int n_layers, const void* x_calib, void* x_work, int T,
                              const int32_t* seq_offsets, int B, const int32_t* positions, float target_ratio,
                              void* scratch, void* workspace, size_t workspace_bytes,
                              float* theta, float* ratio, float* table, void* stream);

/* Scores of the two-output MLP router alone (see qtale_layer_weights): scores[t] for T tokens. */
int qtale_router_mlp_scores(int act_dtype, const void* x, int T, int hidden, const float* w1, const float* b1,
                            const float* w2, const float* b2, int router_hidden, float* scores /*[T]*/, void* stream);

/* out[M][N] (fp16) = A[M][K] (fp16) x dequant(W)^T for one quantized linear (matrix-core GEMM on 4-bit or
 * 3-bit codes, `bits`/`group` as given to qtale_quantize for this matrix). */
int qtale_linear_w4a16(const qtale_qlinear* w, int bits, int group, const void* A, int M, void* out, void* stream);

/* act[M][I] (fp16) = silu(A Wgate^T) * (A Wup^T): the fused gate/up GEMM of the SwiGLU MLP. */
int qtale_swiglu_w4a16(const qtale_qlinear* gate, const qtale_qlinear* up, int bits, int group,
                       const void* A, int M, void* out, void* stream);

/* ---- low-rank adapters of many requests beside a shared projection -----------------------------------------
 * Row i of a call has adapter a = adapter[i] (int32 device [M]; a number outside 0 .. n_adapters - 1: none):
 *   y_i = W A_i + scale[a] * up_a (down_a A_i),   W the quantized linear, sums in 32 bits.
 * The inner values down_a A_i are held in 32 bits between the two products; they enter the second one as fp16 of their row's power of two.
 * The shared product, of weights fp16((code - zero) * scale) as in qtale_linear_w4a16, stays in 32 bits; the sum is rounded, once. */
typedef struct {
    const void* down;          /* [n_adapters][max_rank][K] fp16, 16-byte aligned */
    const void* up;            /* [n_adapters][N][max_rank] fp16, 16-byte aligned */
    const int32_t* rank;       /* device [n_adapters], 0 .. max_rank each (nullable: max_rank): what lies past an adapter's rank is not used */
    const float* scale;        /* device [n_adapters] (nullable: 1) */
    int n_adapters, max_rank;  /* max_rank a multiple of 8, at most 128 */
    int N, K;                  /* of the linear */
} qtale_lora;

/* Scratch of the two calls below with M rows: of a linear with `a` (b null), or of a gate/up pair with `a` and `b` (a pair with one of them alone
 * needs no more than with that one twice).  They do 8192 rows at a time: more need no more. */
size_t qtale_lora_workspace_bytes(const qtale_lora* a, const qtale_lora* b, int M);

/* qtale_linear_w4a16 with adapters. */
int qtale_linear_lora_w4a16(const qtale_qlinear* w, int bits, int group, const qtale_lora* lora, const int32_t* adapter, const void* A, int M,
                            void* out, void* workspace, size_t workspace_bytes, void* stream);

/* qtale_swiglu_w4a16 with adapters on gate and up (either nullable): silu(gate_i) * up_i of the y above. */
int qtale_swiglu_lora_w4a16(const qtale_qlinear* gate, const qtale_qlinear* up, int bits, int group, const qtale_lora* lora_gate,
                            const qtale_lora* lora_up, const int32_t* adapter, const void* A, int M, void* out, void* workspace,
                            size_t workspace_bytes, void* stream);

/* ---- HIP graph of one stack forward (launch-overhead removal, App. B.2 future work) -------------------
 * qtale_graph_capture_stack records the kernels of ONE qtale_stack_forward call with exactly these
 * arguments (no dbg_hidden) into a HIP graph and instantiates it; nothing executes during capture.
 * Every pointer and the control value of ctx at capture time are baked in (in ratio mode the launch shapes
 * depend on the ratio): to step a decode loop the caller rewrites x, positions and the caches' contents in
 * place between launches; per-sequence cache lengths advance on the device as in the eager call.  After
 * qtale_set_exec_ratio / qtale_set_threshold a new graph must be captured.  Fails with
 * QTALE_ERR_INVALID_ARG while per-kernel profiling is enabled.
 * qtale_graph_launch enqueues one replay on `stream`; replays of one graph must not overlap. */
typedef struct qtale_graph qtale_graph;
int qtale_graph_capture_stack(qtale_ctx* ctx, const qtale_layer_cfg* cfg, const qtale_layer_weights* layers,
                              int n_layers, void* x, int T, const int32_t* seq_offsets, int B,
                              const int32_t* positions, const qtale_kv* kv_per_layer /*nullable*/,
                              int32_t* sel_idx /*nullable*/, int32_t* sel_count /*nullable*/,
                              float* scores /*nullable*/, void* workspace, size_t workspace_bytes,
                              qtale_graph** graph /*host out*/);
int qtale_graph_launch(qtale_graph* graph, void* stream);
void qtale_graph_destroy(qtale_graph* graph);

/* ---- paged K/V cache -------------------------------------------------------------------------------------
 * A layer's cache holds the tokens that executed it, so its length differs from layer to layer and only the device knows it.  Instead of
 * `cap` entries per layer and sequence, a paged cache takes pages of page_size tokens from one pool as they are needed; sequences that begin
 * alike share them.
 *   page    keys and values of page_size consecutive tokens of one slot: [n_kv_heads][page_size][head_dim] each, fp16 or bf16, or in 4 bits
 *   slot    the cache of one sequence; 0 .. n_slots - 1, the same number in every layer
 *   table   page of every page_size tokens of a slot, per layer; -1 = none: its tokens are not seen by attention, and not stored by an append
 * The caller allocates all arrays; qtale_pages_init makes an empty cache of them.  Invariants that the calls keep: page_refs[p] is the number
 * of table entries that name p, bit p is set in free_bits iff it is 0, and entries from kv_cap / page_size on are -1.
 * Calls on slots: `slots` [B] int32 device, the slot of each sequence of the call, all different (nullable: sequence b is slot b); a number
 * out of range is skipped.  The calls only enqueue kernels (no synchronisation, no allocation; they can be captured into a graph), and
 * every result, page numbers included, depends on the state and the arguments alone. */
typedef struct {
    void* k_pages;          /* [n_pages][n_kv_heads][page_size][head_dim], 16-byte aligned (4 bits: see QTALE_KV_INT4) */
    void* v_pages;
    int32_t* page_refs;     /* [n_pages] table entries that name the page */
    uint32_t* free_bits;    /* [ceil(n_pages / 32)] bit p % 32 of word p / 32: page p is free */
    int32_t* table;         /* [n_layers][n_slots][max_pages] */
    int32_t* kv_len;        /* [n_layers][n_slots] tokens in the slot */
    int32_t* kv_cap;        /* [n_layers][n_slots] tokens that the slot's pages have room for */
    int n_pages;
    int page_size;          /* 16, 32, 64, ..., 1024 */
    int n_kv_heads, head_dim;   /* head_dim 64 or 128 */
    int n_layers, n_slots, max_pages;
    int dtype;              /* QTALE_ACT_FP16 | QTALE_ACT_BF16, of keys and values (and of the queries and outputs of the calls on them);
                             * plus QTALE_KV_INT4: that is the type of what goes in and comes out, the pages hold 4 bits */
} qtale_paged_kv;

/* Pages in 4 bits.  The d values x of a token's key or value at one kv head share a scale s, of the cache's 16-bit type T, and a zero point z, as
 * the weights' groups do: lo = min(0, min x), hi = max(0, max x), s = T((hi - lo) / 15) (1 if that is 0), z = min(rint(-lo / s), 15),
 * code = clamp(rint(x / s) + z, 0, 15), half to even; a code stands for (code - z) * s.  A row with a value that is not finite has s = NaN: it
 * reads as NaN.  Keys are turned in 64 bits and rounded to T (what a 16-bit page would hold) before that.
 * A page is [n_kv_heads] blocks of page_size * (head_dim / 2 + 4) bytes: the codes, then per token a 32-bit word s | z << 16.
 * (64 to 16 bits, here and in s, by way of 32.)
 *   key codes    [page_size][head_dim / 8] words: column 8 w + 2 i of a token at bits 4 i of its word w, column 8 w + 2 i + 1 at bits 16 + 4 i
 *   value codes  [page_size / 4][head_dim / 4][2] words, tokens by fours: column 4 Q + i of token 2 p of the four at bits 4 i of word (Q, p),
 *                of token 2 p + 1 at bits 16 + 4 i
 * All calls on a qtale_paged_kv take either form; a fork's copy of a shared page copies what its tokens hold bit by bit. */
enum { QTALE_KV_INT4 = 4 };

/* All pages free, all slots empty. */
int qtale_pages_init(const qtale_paged_kv* kv, void* stream);

/* Scratch of qtale_pages_reserve (at most max_seqs sequences) and qtale_pages_compact (0 sequences); 0 for invalid arguments. */
size_t qtale_pages_workspace_bytes(const qtale_paged_kv* kv, int max_seqs);

/* Slot dst[i] becomes a copy of slot src[i] in every layer (i < n): it shares the pages that hold tokens.  dst[i] has to be empty (released), a
 * slot that is not is left alone; no slot may be a target twice, or a target and a source. */
int qtale_pages_fork(const qtale_paged_kv* kv, const int32_t* src, const int32_t* dst, int n, void* stream);

/* Makes room for the new tokens of a call: seq_offsets[b+1] - seq_offsets[b] for sequence b (seq_offsets [B+1] int32 device), in one layer or
 * in all (layer = -1).  Pages are taken lowest number first, in the order of layers, then sequences, then places.  A slot that will write into
 * a page it shares (its last, partly filled) first gets a copy of it.  Only where all holders of the page write in this call, the one with the
 * most tokens, of several the last in order, keeps the page itself.
 *   first     nullable: only make room.  Otherwise the slots' lengths are advanced as well and first [layers of the call][B] receives the
 *             lengths before: token i of sequence b is entry first[b] + i of its slot, for qtale_paged_rope_append and qtale_paged_attention
 *   missing   nullable [1] out: pages that the pool could not give.  A slot that got fewer than it needs holds as many of the new tokens as
 *             fit (the first ones); the others are dropped by the append, and its length stops there.  Likewise at max_pages * page_size.  One that
 *             got no page for its copy takes none of its tokens and keeps sharing the old one
 *   workspace qtale_pages_workspace_bytes(kv, B) bytes, 256-byte aligned; B <= 2048 */
int qtale_pages_reserve(const qtale_paged_kv* kv, int layer, const int32_t* seq_offsets, const int32_t* slots, int B, int32_t* first,
                        int32_t* missing, void* workspace, size_t workspace_bytes, void* stream);

/* Empties n slots in every layer; pages that nobody else holds are free again. */
int qtale_pages_release(const qtale_paged_kv* kv, const int32_t* slots, int n, void* stream);

/* Lets go of the pages of n slots that attention with this window (>= 1) and these first tokens (sinks >= 0) no longer reaches, seen from each
 * slot's next token: those whose tokens all lie before the window and after the first `sinks`.  Lengths and room stay. */
int qtale_pages_trim(const qtale_paged_kv* kv, const int32_t* slots, int n, int window, int sinks, void* stream);

/* Moves the pages in use to the front of the pool, 0 .. n_live - 1 (nullable [1] out): the k-th page in use from n_live on, by number, goes to
 * the k-th free one below it.  What lies in pages from n_live on is then unused (the pool can shrink, or be saved as one block). */
int qtale_pages_compact(const qtale_paged_kv* kv, int32_t* n_live, void* workspace, size_t workspace_bytes, void* stream);

/* Copies the contents of pages src[i] of one pool to pages dst[i] of another (or of the same, if no page is written that is also read or
 * written by another i); counts and tables are not touched.  Both of one page shape and type. */
int qtale_pages_copy(const qtale_paged_kv* from, const qtale_paged_kv* to, const int32_t* src, const int32_t* dst, int n, void* stream);

/* Rotary embedding: pair i < rotary_dim / 2 of a head turns by position * freqs[i]; columns from rotary_dim on stay as they are. */
enum { QTALE_ROPE_HALF = 0, QTALE_ROPE_INTERLEAVED = 1 };   /* pairs (i, i + rotary_dim / 2) or (2 i, 2 i + 1) */
enum {                        /* frequencies w_i = base^(-2 i / rotary_dim), and how a longer context stretches them by `factor` */
    QTALE_ROPE_PLAIN = 0,
    QTALE_ROPE_LINEAR = 1,    /* w_i / factor */
    QTALE_ROPE_BASE = 2,      /* base * factor^(r / (r - 2)) for base: the slowest pair is stretched by factor, the fastest not at all */
    QTALE_ROPE_BANDS = 3,     /* pairs that make more than `high` turns over original_len tokens stay, fewer than `low`: w_i / factor, linear between */
    QTALE_ROPE_PARTS = 4      /* the same ends, linear in i between the pairs that make `high` and `low` turns; magnitude 0.1 ln(factor) + 1 */
};
typedef struct {
    int layout;               /* QTALE_ROPE_HALF | QTALE_ROPE_INTERLEAVED */
    int rotary_dim;           /* even, 2 .. head_dim */
    const double* freqs;      /* device [rotary_dim / 2]: angle per position */
    float magnitude;          /* factor on cosine and sine, usually 1 */
} qtale_rope;

/* freqs (host out [rotary_dim / 2]) and magnitude (host out) of one of the scalings above; original_len, low and high are read for BANDS and
 * PARTS only, factor by all but PLAIN. */
int qtale_rope_frequencies(int rotary_dim, float base, int scaling, float factor, int original_len, float low, float high,
                           double* freqs, float* magnitude);

/* Turns the queries and the new keys of T tokens and stores keys and values into the pages of one layer.  q [T][n_heads * head_dim],
 * k, v [T][n_kv_heads * head_dim], q_out like q (may be q itself): kv->dtype, *_stride elements between tokens (a multiple of 8), 16-byte aligned.
 *   seq_offsets [B+1], positions [T] (absolute, for the angles); first [B]: entry of each sequence's first new token in its slot (nullable:
 *   kv_len minus its new tokens, which is that entry only where qtale_pages_reserve has dropped none of them: after a call that may find
 *   the pool empty pass the `first` that it gave, or kept entries are overwritten).  Entries at or past kv_len, and those without a page, are not stored. */
int qtale_paged_rope_append(const qtale_paged_kv* kv, int layer, const qtale_rope* rope, const void* q, int64_t q_stride,
                            const void* k, int64_t k_stride, const void* v, int64_t v_stride, void* q_out, int64_t q_out_stride,
                            int n_heads, int T, const int32_t* seq_offsets, const int32_t* slots, const int32_t* first, int B,
                            const int32_t* positions, void* stream);

/* The values that entries of one layer's slots stand for, in kv->dtype's 16-bit type: row i of sequence b is entry first[b] + i (first [B]; nullable: its
 * slot's last entries) of its slot.  k, v [T][n_kv_heads * head_dim], strides as above.  Entries outside 0 .. kv_len - 1, without a page or
 * of a slot that does not exist are zeros; rows past the last sequence are left as they are. */
int qtale_paged_read(const qtale_paged_kv* kv, int layer, void* k, int64_t k_stride, void* v, int64_t v_stride, int T,
                     const int32_t* seq_offsets, const int32_t* slots, const int32_t* first, int B, void* stream);

/* Causal attention of T new tokens over the pages of one layer, from one token per sequence to whole prompts:
 *   out_p = sum_j softmax_j(scale q_p . k_j) v_j,  j <= p, j < kv_len, page of j present, and (window == 0 or j > p - window or j < sinks),
 * p = first[b] + i for token i of sequence b (first as in qtale_paged_rope_append).  A token that sees no entry gets zeros.  Head h reads kv head h / (n_heads / n_kv_heads).
 * q and out [T][n_heads * head_dim], *_stride elements between tokens (q: a multiple of 8, 16-byte aligned; out: of 4, 8-byte aligned). */
typedef struct {
    int n_heads;
    int window;               /* entries that a token sees, itself included; 0 = all before it */
    int sinks;                /* first entries of the slot that stay visible with a window */
    float scale;              /* > 0, e.g. 1 / sqrt(head_dim) */
    int max_new;              /* bound on the new tokens of a sequence (rows past it are undefined); 0 = T.  A bound near the truth pays */
    int max_len;              /* bound on kv_len; 0 = max_pages * page_size.  Entries from max_len on are not seen */
} qtale_paged_attn;
size_t qtale_paged_attention_workspace_bytes(const qtale_paged_kv* kv, const qtale_paged_attn* attn, int T, int B);
int qtale_paged_attention(const qtale_paged_kv* kv, int layer, const qtale_paged_attn* attn, const void* q, int64_t q_stride,
                          void* out, int64_t out_stride, int T, const int32_t* seq_offsets, const int32_t* slots, const int32_t* first,
                          int B, void* workspace, size_t workspace_bytes, void* stream);

/* n_layers layers as in qtale_stack_forward, on a paged cache: layer l of the call uses the cache's layer first_layer + l.  In every layer the
 * executed tokens get room in their sequences' slots (qtale_pages_reserve), their queries and keys are turned (positions are those of the
 * tokens), keys and values go to the pages, and the queries attend to what their slot holds, which is executed tokens only.
 *   kv      fp16 (or fp16 in 4 bits), of cfg's kv heads and head size; slots [B] as everywhere (nullable: sequence b is slot b); B <= 2048
 *   rope    replaces cfg->rope_base;  attn: window, sinks, scale and bounds (max_new: of a call's tokens per sequence; n_heads = cfg->n_heads)
 *   missing nullable [n_layers] out: pages that the pool could not give in a layer.  Tokens without a place are dropped from that layer's
 *           cache (their own queries see what is there), as the newest tokens are when a qtale_kv is full.  Left as it is by calls that ask
 *           for no pages, because T is 0 or the ratio rounds to no token: set it to 0 before such a call.
 *   workspace >= qtale_paged_stack_workspace_bytes(cfg, kv, T, B) bytes, 256-byte aligned */
size_t qtale_paged_stack_workspace_bytes(const qtale_layer_cfg* cfg, const qtale_paged_kv* kv, int max_tokens, int max_seqs);
int qtale_paged_stack_forward(qtale_ctx* ctx, const qtale_layer_cfg* cfg, const qtale_layer_weights* layers, int n_layers, int first_layer,
                              void* x, int T, const int32_t* seq_offsets, int B, const int32_t* positions, const qtale_paged_kv* kv,
                              const int32_t* slots /*nullable*/, const qtale_rope* rope, const qtale_paged_attn* attn,
                              int32_t* missing /*nullable*/, int32_t* sel_idx /*nullable*/, int32_t* sel_count /*nullable*/,
                              float* scores /*nullable*/, void* workspace, size_t workspace_bytes, void* stream);

/* qtale_paged_stack_forward with adapters: loras host [n_layers], whose linears without an adapter have n_adapters = 0 (the rest is then not read);
 * adapter [B] int32 device: that of each sequence of the call, one number for all linears and layers (outside a linear's adapters: none).
 * workspace >= qtale_paged_stack_lora_workspace_bytes(cfg, kv, max_rank, T, B) with the largest max_rank.  (All rows of a layer are done at once: 8 * inter bytes
 * of it per token for gate and up, 2.9 GB for 32768 tokens with inter = 11008.  Calls of fewer tokens need less.) */
typedef struct { qtale_lora q, k, v, o, gate, up, down; } qtale_layer_lora;
size_t qtale_paged_stack_lora_workspace_bytes(const qtale_layer_cfg* cfg, const qtale_paged_kv* kv, int max_rank, int max_tokens, int max_seqs);
int qtale_paged_stack_lora_forward(qtale_ctx* ctx, const qtale_layer_cfg* cfg, const qtale_layer_weights* layers, const qtale_layer_lora* loras,
                                   int n_layers, int first_layer, void* x, int T, const int32_t* seq_offsets, int B, const int32_t* positions,
                                   const qtale_paged_kv* kv, const int32_t* slots /*nullable*/, const int32_t* adapter, const qtale_rope* rope,
                                   const qtale_paged_attn* attn, int32_t* missing /*nullable*/, int32_t* sel_idx /*nullable*/,
                                   int32_t* sel_count /*nullable*/, float* scores /*nullable*/, void* workspace, size_t workspace_bytes, void* stream);

/* Per-kernel timing with HIP events recorded on the forward call's stream.  While enabled, every
 * layer/stack forward brackets its kernels with events; qtale_profile_read waits for them and
 * returns, per kernel class, accumulated milliseconds and launch counts since the last read.
 * Classes: 0 router, 1 select, 2 norm1, 3 qkv gemm, 4 rope+append, 5 attention, 6 o gemm, 7 norm2,
 * 8 gate/up gemm, 9 down gemm.  Small calls fuse some of them, and a fused step is counted in the class of the launch that
 * does it: up to 256 tokens class 2 is part of 1; with a cache and few new tokens per sequence (decode) class 4 is part
 * of 5, so that a bandwidth made from class 5 includes the rotation and the append (otherwise 4 also builds the work list of 5;
 * on a paged cache it is always 4, with the pages' room);
 * adapters are counted in the class of their linear;
 * with at most four tokens 0 (unless the
 * router is an MLP), 1 and 2 are part of 3, and 7 is part of 8.  Inside a stack a decode-sized layer's class 9 also scores the
 * next layer's tokens (its class 0).  Profiling adds event overhead; leave it off when timing whole steps. */
enum { QTALE_PROF_CLASSES = 10 };
int qtale_profile_enable(qtale_ctx* ctx, int on);
int qtale_profile_read(qtale_ctx* ctx, double* ms /*host [QTALE_PROF_CLASSES]*/,
                       int64_t* launches /*host [QTALE_PROF_CLASSES]*/);

#ifdef __cplusplus
}
#endif
#endif /* QTALE_H */
