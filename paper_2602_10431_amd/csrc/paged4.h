// Pages in 4 bits: where a token's codes, scale and zero point lie in its head's block, and what they stand for.
//   keys    [P][d / 8] words, column 8 w + 2 i at bits 4 i of word w, 8 w + 2 i + 1 at bits 16 + 4 i: `word >> 4 i & 0x000f000f` is two columns that
//           follow each other, in the order of a matrix operand
//   values  [P / 4][d / 4][2] words, column 4 Q + i of tokens 2 p and 2 p + 1 of the four at bits 4 i and 16 + 4 i of word (Q, p): the same shifts give
//           one column of two tokens that follow each other, which is how the second product takes them, without a permutation
//   then P words s | z << 16: scale in the cache's 16-bit type, zero point as a whole number
#pragma once
#include "paged.h"
#include "qtale_dev.h"

namespace qtale {

struct Block4 {                                  // offsets in a head's block, in bytes
    int d, shift;
    __device__ __forceinline__ uint32_t key(int t) const { return static_cast<uint32_t>(t) * (d >> 1); }
    __device__ __forceinline__ uint32_t value(int t, int col) const {     // the 16-bit piece of columns col .. col + 3
        return static_cast<uint32_t>(t >> 2) * (2 * d) + 2 * col + 2 * (t & 3);
    }
    __device__ __forceinline__ uint32_t param(int t) const { return (static_cast<uint32_t>(d >> 1) << shift) + 4 * t; }
    __device__ __forceinline__ size_t bytes() const { return static_cast<size_t>((d >> 1) + 4) << shift; }
};

__device__ __forceinline__ float scale4(uint32_t param, int bf16) { return act_to_float(static_cast<uint16_t>(param & 0xffffu), bf16); }

// Entry of a slot that row i of a call is: its page and place (page < 0: there is none).  by: rows of its sequence and before
struct RowEntry { int page, place; };
template <class Offsets>
__device__ __forceinline__ RowEntry entry_of_row(const PagedDev& kv, const Offsets* seq_offsets, const int32_t* slots, const int32_t* first, int B, int i) {
    const int lane = threadIdx.x & 63;
    int b = 0;                                   // the number of sequences that end at or before the row
    for (int b0 = 0; b0 < B; b0 += 64) b += __popcll(__ballot(b0 + lane < B && seq_offsets[min(b0 + lane, B - 1) + 1] <= i));
    RowEntry r{-1, 0};
    if (b >= B) return r;
    const int slot = slots ? slots[b] : b;
    if (static_cast<uint32_t>(slot) >= static_cast<uint32_t>(kv.n_slots)) return r;
    const int begin = seq_offsets[b], len = kv.len[slot];
    const int at = (first ? first[b] : len - (seq_offsets[b + 1] - begin)) + (i - begin);
    if (at < 0 || at >= len || (at >> kv.shift) >= kv.max_pages) return r;
    const int page = kv.table[static_cast<size_t>(slot) * kv.max_pages + (at >> kv.shift)];
    if (static_cast<uint32_t>(page) < static_cast<uint32_t>(kv.n_pages)) r = RowEntry{page, at & ((1 << kv.shift) - 1)};
    return r;
}

}  // namespace qtale
