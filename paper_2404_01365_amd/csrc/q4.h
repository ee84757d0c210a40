// The cache in 4 bits as kernels see it: where a page keeps what, and what its codes stand for.
#pragma once

#include "layer.h"

namespace griffin {

typedef __attribute__((ext_vector_type(2))) _Float16 q4_pair;

// Sizes of one kv head's part of a page: page_size rows of codes, then page_size rows of (scale, middle) words
struct Q4Shape {
    uint32_t row_bytes, groups, group_shift, pairs_at, head_bytes;
    int32_t page_shift, last_page, kv_heads;
};

inline Q4Shape q4_shape(const griffin_kv_cache_q4 &C)
{
    Q4Shape s;
    s.row_bytes = (uint32_t)(C.dim + 31) / 32 * 16;
    s.groups = (uint32_t)(C.dim + C.group - 1) / C.group;
    s.group_shift = __builtin_ctz(C.group);
    s.pairs_at = s.row_bytes * C.page_size;
    s.head_bytes = s.pairs_at + s.groups * 4 * C.page_size;
    s.page_shift = __builtin_ctz(C.page_size);
    s.last_page = (int32_t)(C.n_pages - 1);
    s.kv_heads = C.kv_heads;
    return s;
}

// Codes of features f .. f + 7 are one word.  With a code's four bits as the last of an fp16's whose unit is one, 1024 + (c + 8), taking away 1032 leaves c
// exactly, two codes an instruction.  Features (0, 4), (1, 5), (2, 6), (3, 7) come out as pairs: those are four bits apart in both halves of the word.
// One instruction takes both constants only if one of them is in a vector register, where the compiler would not put it by itself.
__device__ __forceinline__ q4_pair q4_code_pair(uint32_t bits)       // codes in bits 0 .. 3 and 16 .. 19; others are cut away
{
    uint32_t mask = 0x000F000Fu;
    asm("" : "+v"(mask));
    return __builtin_bit_cast(q4_pair, (bits & mask) | 0x64006400u) - q4_pair{(_Float16)1032, (_Float16)1032};
}

// middle + scale c, rounded once
__device__ __forceinline__ q4_pair q4_value_pair(uint32_t bits, q4_pair scale, q4_pair middle)
{
    return __builtin_elementwise_fma(q4_code_pair(bits), scale, middle);
}

// the two of a (scale, middle) word, twice each
__device__ __forceinline__ q4_pair q4_scales(uint32_t pair) { return __builtin_bit_cast(q4_pair, __builtin_amdgcn_perm(pair, pair, 0x01000100)); }
__device__ __forceinline__ q4_pair q4_middles(uint32_t pair) { return __builtin_bit_cast(q4_pair, __builtin_amdgcn_perm(pair, pair, 0x03020302)); }

}  // namespace griffin
