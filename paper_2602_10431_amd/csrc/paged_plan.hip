// Which launches a call of attention over pages makes, from what the host knows of it.
#include <algorithm>

#include "paged.h"

namespace qtale {

// CUs of the current device (queried once per device).
static int device_cus() {
    static int cus[64] = {0};
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
    if (cus[dev] == 0) {
        int n = 0;
        if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) n = 256;
        cus[dev] = n;
    }
    return cus[dev];
}

// Spans per kv head that fill the chip once with the decode kernel's workgroups.
static int decode_spans(int nkv, int d) { return std::max((d == 64 ? 4 : 3) * device_cus() / nkv, 1); }
static size_t decode_bytes(int nkv, int d, int B) {
    const size_t pieces = (static_cast<size_t>(std::min(B, kSpanSeqs)) * sizeof(int4) + 255) / 256 * 256;
    return pieces + static_cast<size_t>(decode_spans(nkv, d)) * nkv * 2 * kDecodeCols * part_stride(d) * 4;
}
// Pages in 4 bits: whether sixteen columns at a time, which unpack in registers, take less time than tiles of 128 columns, which unpack once for all
// of them but pass LDS and barriers.  Estimates in us, from runs of either alone.  A workgroup of the decode kernel walks a key in 6.2 ns (heads of 64: 5.6)
// until a CU's others hold it up, 4.0 (3.1) ns for each of those.  A workgroup of the chunk kernel takes 8 us and 2.2 us per tile of 64 keys, two on a CU 2.9
// per tile; ranges cost 14 us and 0.5 ns per row of sums.  us, decode / chunk kernel, heads of 128, 4 per kv head (8): 1 x 32 tokens on 1500 keys 15 /
// 56, on 4000 30 / 31; 1 x 64 on 24000 138 / 64; 64 x 8 on 2000 46 / 98; 64 x 32 on 1000 96 / 64; 4 x 1000 on 0 113 / 76, 2 x 2000 162 / 119; 8 x 128 on
// 2000 74 / 81; one per kv head (32) 4 x 1000 111 / 75; heads of 64 48 x 6 on 3000 34 / 101, 64 x 16 on 3000 82 / 108.
static bool decode4_pays(int nh, int nkv, int d, int T, int B, int64_t max_new, int64_t seen, bool window) {
    const int rep = nh / nkv, cus = device_cus();
    const int64_t cols = max_new * rep, sixteens = (cols + kDecodeCols - 1) / kDecodeCols, live = std::min(B, T);
    if (sixteens > 65535) return false;                          // (a grid's second extent)
    auto workgroups = [&](int64_t per) {                         // per CU
        return static_cast<double>(std::min((T * static_cast<int64_t>(rep) + (per - 1) * live) / per, live * ((cols + per - 1) / per)) * nkv) / cus;
    };
    const double longest = static_cast<double>(seen), mean = window ? longest : std::max(longest - 0.5 * static_cast<double>(max_new), 0.0);
    const double by = workgroups(kDecodeCols), decode = 5.0 + 1.2 * by + 0.001 * mean * (d == 64 ? std::max(5.6, 3.1 * by) : std::max(6.2, 4.0 * by));
    const double r = std::max(workgroups(kChunkCols), 1e-3), most = longest / kChunkTileKeys, some = mean / kChunkTileKeys;
    const double whole = 8.0 * std::max(0.5 * r, 1.0) + std::max(2.2 * most, 1.45 * r * some + (r > 2.0 ? 2.2 * (most - some) : 0.0));
    const double ranges = std::max(std::min({2.0 / r, most / 8, 32.0}), 1.0);
    const double cut = 22.0 + std::max(2.2 * most / ranges, 1.45 * r * some) + 0.0005 * T * nh * ranges;
    return decode < std::min(whole, cut);
}
PagedAttnPlan plan_paged_attention(int q4, int nh, int nkv, int d, int T, int B, int max_new, int max_len, int window, int sinks) {
    PagedAttnPlan l{};
    const int rep = nh / nkv, cus = device_cus();
    const int64_t seen = window > 0 ? std::min<int64_t>(max_len, static_cast<int64_t>(window) + sinks + max_new) : max_len;   // keys of a sequence
    const int64_t cols = static_cast<int64_t>(max_new) * rep, sixteens = (cols + kDecodeCols - 1) / kDecodeCols, scaled = seen * d / 128;
    int64_t items = (static_cast<int64_t>(T) * rep + static_cast<int64_t>(kChunkCols - 1) * std::min(B, T)) / kChunkCols;
    // chunk kernel: workgroups, tiles of a sequence's keys, and whether those are cut into ranges (few column tiles, where that saves more than
    // adding the ranges costs, about 24 tiles of time)
    const int64_t wgs = std::max<int64_t>(items * nkv, 1), tiles = (seen + kChunkTileKeys - 1) / kChunkTileKeys, two = 2 * cus;
    const bool cut = tiles * (two - wgs) > 24 * two;
    // (Figures of chunks in fp16, here and below, are from before kChunkLift, which adds 1 to 2 % to every form.)
    // The decode kernel takes sequences of up to sixteen columns, for which a chunk's workgroup would run mostly empty, and larger ones while its
    // workgroups, each walking all keys, fill the chip about once.  us, it / chunk kernel, heads of 128, 4 per kv head (8): 1 x 32 tokens on 700
    // keys 12 / 19, on 1500 18 / 28, on 4000 (cut) 40 / 24; 4 x 64 on 300 13 / 17, on 700 20 / 22, on 1500 35 / 31; 16 x 8 on 1500 23 / 32, on 4000
    // 51 / 64 (cut); 16 x 24 on 100 11 / 12, on 300 22 / 16; 32 x 8 on 1500 40 / 45, 24 x 8 on 6000 143 / 135; one per kv head (32) 4 x 32 on 700
    // 14 / 21, 4 x 64 on 700 21 / 22; heads of 64 8 x 48 on 100 8 / 11.6.
    const int64_t by_sixteen = sixteens * B * nkv;
    const bool fits = by_sixteen <= cus ? !cut || 2 * wgs >= cus : by_sixteen <= 2 * cus ? scaled <= (sixteens == 2 ? 4000 : 900) : by_sixteen <= 3 * cus && scaled <= 160;
    l.chunk = cols > kDecodeCols && !(q4 ? decode4_pays(nh, nkv, d, T, B, max_new, seen, window > 0) : fits);
    // Both run where the call seems to hold sequences of either kind: the mean is far below the longest.
    l.decode = !l.chunk || (4 * static_cast<int64_t>(T) < static_cast<int64_t>(B) * max_new && rep <= kDecodeCols);
    l.cols = static_cast<int>(l.chunk ? std::min<int64_t>(kDecodeCols, cols) : cols);
    // Spans cost about 5 us (finding the piece, a second launch) and save what a workgroup per (sequence, kv head) leaves idle: the fuller those fill
    // the CUs, the longer the keys have to be.  us without / with spans, 8 kv heads of 128, sequences of 0.5 to 1.5 times the mean: 4 x 400 keys
    // 9.1 / 10.8, 4 x 1500 27 / 13.6, 16 x 700 16.1 / 16.4, 16 x 2200 39 / 31, 24 x 2200 44.7 / 45.6, 32 x 3000 71 / 72, 32 x 12000 269 / 246,
    // 40 x 700 27.0 / 27.6, 40 x 2200 81 / 69, 60 x 2200 94.6 / 96.6, 60 x 12000 495 / 448; heads of 64 8 x 1500 13.2 / 13.6.
    const int64_t pairs = static_cast<int64_t>(B) * nkv, filled = (pairs + cus - 1) / cus * cus;
    if (l.decode && l.cols <= kDecodeCols && B <= kSpanSeqs && pairs < 2 * cus && scaled * (10 * filled - 9 * pairs) > 8000 * filled) l.spans = decode_spans(nkv, d);
    l.stream_keys = pairs >= 4 * cus;
    l.ranges = l.groups = 1;
    if (l.chunk && q4) {
        // Ranges for two workgroups per CU.  us, with / without: heads of 128, 4 per kv head, 64 rows on 24000 keys 68 / 961, 500 295 / 985, 1000 on 6000 173 / 295;
        // one per kv head 700 on 4000 113 / 206 (unpacking before the scores' products, as the forms then were).
        if (cut) {
            l.target = static_cast<int>(two);
            l.ranges = static_cast<int>(std::max<int64_t>(std::min<int64_t>({2 * ((two + wgs - 1) / wgs), tiles / 8, 32}), 1));
        }
    } else if (l.chunk) {
        // Ranges for two workgroups per CU; else, where the tiles fill less than 7/8 of the CUs' places, two groups of waves per workgroup, which share a
        // tile's keys.  us, ranges / groups / neither: heads of 128, 4 per kv head, 500 rows on 24000 keys 218 / 393 / -, 2 x 300 on 2000
        // 59 / 61 / -, 1500 on 0 50 / 35 / 44, 1000 on 0 - / 23.6 / 27.3; heads of 64 2 x 700 on 1400 52 / 45 / 58, 1500 on 0 30 / 24 / 34; one
        // head per kv head, 200 on 3000 33 / 57 / -, 40 heads 2 x 700 on 1000 - / 68 / 58; 4 x 4096 - / 704 / 603.
        // Many and long: the wide form, if its workgroups, one per CU at a time, end together.  us, it / chunk kernel: heads of 128, 4 per kv
        // head, 4 x 4096 574 / 603, 1 x 4096 133 / 144, 2 x 2048 88 / 92, 3 x 750 to 2250 104 / 97, 8 x 512 52 / 48; one per kv head
        // 4 x 1000 75 / 67; under a window of 1000 99 / 81; heads of 64 4 x 4096 411 / 326.
        const int64_t wide = (static_cast<int64_t>(T) * rep + static_cast<int64_t>(kWideCols - 1) * std::min(B, T)) / kWideCols;
        const int64_t rounds = (wide * nkv + cus - 1) / cus;
        if (cut) {
            l.target = static_cast<int>(two);
            l.ranges = static_cast<int>(std::max<int64_t>(std::min<int64_t>({2 * ((two + wgs - 1) / wgs), tiles / 8, 32}), 1));
        } else if (8 * wgs < (d == 64 ? 28 : 14) * cus && tiles >= 8) {
            l.groups = 2;
        } else if (d == 128 && tiles >= 32 && rounds >= 2 && (rounds >= 6 || 8 * wide * nkv >= 7 * cus * rounds)) {
            l.groups = 0;
            items = wide;
        }
    }
    l.items = static_cast<int>(std::min<int64_t>(items, INT32_MAX));
    l.too_large = items * nkv * l.ranges > INT32_MAX || static_cast<int64_t>(T) * nh > INT32_MAX;
    if (l.spans) l.decode_bytes = decode_bytes(nkv, d, B);
    l.bytes = 256 + l.decode_bytes + (l.ranges > 1 ? static_cast<size_t>(T) * nh * l.ranges * part_stride(d) * 4 : 0);
    return l;
}

size_t paged_attention_bytes(int nh, int nkv, int d, int T, int B) {
    // ranges exist below two workgroups per CU, of 128 columns each: that bounds T * nh, and 2 (2 CUs / workgroups + 1) ranges the product
    const size_t columns = static_cast<size_t>(2 * device_cus()) * kChunkCols, sums = std::min<size_t>(static_cast<size_t>(T) * nh * 32, 4 * columns);
    return (256 + decode_bytes(nkv, d, B) + sums * part_stride(d) * 4 + 255) / 256 * 256;
}

hipError_t launch_paged_attention(PagedAttnDev a, const PagedAttnPlan& plan, int d, int T, float* workspace, hipStream_t stream) {
    const int bf16 = a.bf16;
    a.take = plan.decode && plan.chunk;
    a.items = plan.items; a.ranges = plan.ranges; a.target = plan.target;
    a.spans = plan.spans; a.stream_keys = plan.stream_keys; a.cols = plan.cols;
    char* at = reinterpret_cast<char*>(workspace);
    a.pieces = reinterpret_cast<int4*>(at);
    a.span_part = reinterpret_cast<float*>(at + (static_cast<size_t>(std::min(a.B, kSpanSeqs)) * sizeof(int4) + 255) / 256 * 256);
    a.part = reinterpret_cast<float*>(at + plan.decode_bytes);
    hipError_t e = hipSuccess;
    if (a.q4) {
        if (plan.decode && (e = launch_paged4_decode(a, d, stream)) != hipSuccess) return e;
        if (plan.chunk && (e = launch_paged4_chunk(a, d, stream)) != hipSuccess) return e;
        a.scale_log2 = 1.0f;                                     // (reference points of these kernels are scaled scores)
        return plan.ranges > 1 ? launch_chunk_combine(a, d, bf16, T, stream) : e;
    }
    if (plan.decode && (e = launch_paged_decode(a, d, bf16, stream)) != hipSuccess) return e;
    if (plan.chunk && (e = launch_paged_chunk(a, plan.groups, d, bf16, stream)) != hipSuccess) return e;
    return plan.ranges > 1 ? launch_chunk_combine(a, d, bf16, T, stream) : e;
}

}  // namespace qtale
