// Internal helpers that lynx_kvcache.hip and lynx_attention.hip share (not part of the C ABI).
#pragma once

#include "../../include/lynx/attention.h"
#include "lynx_common.h"

namespace lynx {

constexpr int kMaxHeads = 1024;
constexpr int kMaxGroup = 256;
constexpr int kMaxContext = 1 << 29;        // most tokens that a row of the block table can hold

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

int check_cache(const char *who, const void *k_cache, const void *v_cache, int cache_format, float k_scale, float v_scale,
                int num_pages, int page_size, int QH, int KVH, int D);
int check_rows(const char *who, const char *what, const void *ptr, int64_t stride, int heads, int D);

// Two floats as bf16 (to nearest, ties to even), the first in the low half: one instruction.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const f32x2 v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

}  // namespace lynx
