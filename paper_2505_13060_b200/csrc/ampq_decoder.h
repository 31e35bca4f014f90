// What the operators around a decoder's linear layers share (ampq_heads.cu,
// ampq_embed.cu, ampq_distill.cu).
#pragma once
#include "ampq_ckpt.h"

namespace ampq {

inline bool known_index(int type) { return type == AMPQ_I32 || type == AMPQ_I64; }
inline size_t index_bytes(int type) { return type == AMPQ_I64 ? 8 : 4; }

__device__ __forceinline__ long long load_index(const void* p, long long i, bool wide) {
    return wide ? __ldg(static_cast<const long long*>(p) + i) : (long long)__ldg(static_cast<const int*>(p) + i);
}

__device__ __forceinline__ float load_param(const void* p, long long i, bool bf16) {
    return bf16 ? load_elem(static_cast<const __nv_bfloat16*>(p) + i) : load_elem(static_cast<const float*>(p) + i);
}

// 2^x to two units in the last place; 0 below the normal numbers.
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

}  // namespace ampq
