// What the two paged attention kernels share: 16-bit types on the matrix cores, page loads that return zeros outside the keys, partial sums.
#pragma once
#include "paged.h"
#include "qtale_dev.h"

namespace qtale {

constexpr float kPagedNone = -1.0e30f;           // reference point of a row that has seen no key

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

// Operands travel as 16-byte words whatever their type.
template <bool BF16>
struct Act16 {
    static __device__ __forceinline__ float16_t mfma32(const u32x4_t& a, const u32x4_t& b, const float16_t& c) {
        if constexpr (BF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
        else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ float4_t mfma16(const u32x4_t& a, const u32x4_t& b, const float4_t& c) {
        if constexpr (BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
        else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float x, float y) {      // nearest even, one instruction
        const float2_t v = {x, y};
        if constexpr (BF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
        else return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, half2_t));
    }
    static __device__ __forceinline__ float low(uint32_t w) { return act_to_float<BF16>(static_cast<uint16_t>(w & 0xffffu)); }
    static __device__ __forceinline__ float high(uint32_t w) {
        if constexpr (BF16) return __uint_as_float(w & 0xffff0000u);
        else return act_to_float<false>(static_cast<uint16_t>(w >> 16));
    }
};

// A buffer of `bytes` bytes from `base` on, both the same in every lane: loads past them return zeros and touch no memory.  (Named lane by
// lane, because what the compiler cannot see to be uniform it would load in a loop over the lanes' descriptors.)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void* base, int bytes) {
    const uint64_t a = reinterpret_cast<uint64_t>(base);
    const uint64_t lo = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(a))), hi = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(a >> 32)));
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(lo | hi << 32), 0, __builtin_amdgcn_readfirstlane(bytes), 0x00027000);
}

// Table row of a slot, read through the scalar cache (no kernel that reads it writes it).
struct PageRow {
    const QT_CONST_AS int32_t* row;
    int shift, last, n_pages;
    __device__ __forceinline__ PageRow(const PagedAttnDev& p, int slot)
        : row((const QT_CONST_AS int32_t*)(p.table + static_cast<size_t>(slot) * p.max_pages)), shift(p.shift), last(p.max_pages - 1), n_pages(p.n_pages) {}
    // page of a key (the same in every lane), -1 if there is none
    __device__ __forceinline__ int at(int key) const {
        const int page = row[__builtin_amdgcn_readfirstlane(min(key >> shift, last))];
        return page < n_pages ? page : -1;
    }
};

// What a launch has to know of a sequence: its rows, its slot's tokens, the place of its first row in the slot.
struct SeqView {
    int row0, n, slot, len, first;
    __device__ __forceinline__ SeqView(const PagedAttnDev& p, int b) {
        row0 = p.offs[b];
        n = max(p.offs[b + 1] - row0, 0);
        slot = p.slots ? p.slots[b] : b;
        const bool ok = static_cast<uint32_t>(slot) < static_cast<uint32_t>(p.n_slots);
        if (!ok) slot = 0;
        len = ok ? min(p.len[slot], p.max_len) : 0;
        first = p.first ? p.first[b] : (ok ? p.len[slot] : 0) - n;
    }
    // for a sequence that the whole wave works on: into scalar registers
    __device__ __forceinline__ void uniform() {
        row0 = __builtin_amdgcn_readfirstlane(row0);
        n = __builtin_amdgcn_readfirstlane(n);
        slot = __builtin_amdgcn_readfirstlane(slot);
        len = __builtin_amdgcn_readfirstlane(len);
        first = __builtin_amdgcn_readfirstlane(first);
    }
};

}  // namespace qtale
