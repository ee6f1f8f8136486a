// What the units of the paged KV cache share: element types, checks of their arguments.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/rtn.h"
#include "rtn_device.h"

namespace rtn {

typedef __bf16 bf16_t;
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef _Float16 half4_t __attribute__((ext_vector_type(4)));
typedef short short4_t __attribute__((ext_vector_type(4)));
typedef float float16_t __attribute__((ext_vector_type(16)));

// An element type: vectors of it and the matrix instructions on them (fp32 sums).
template <int TYPE> struct Elem;
template <> struct Elem<RTN_TYPE_F16> {
    typedef half_t one;
    typedef half8_t x8;
    typedef half4_t x4;
    static __device__ __forceinline__ float4_t mfma16(x8 a, x8 b, float4_t c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ float16_t mfma32(x8 a, x8 b, float16_t c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
template <> struct Elem<RTN_TYPE_BF16> {
    typedef bf16_t one;
    typedef bf16x8_t x8;
    typedef bf16x4_t x4;
    static __device__ __forceinline__ float4_t mfma16(x8 a, x8 b, float4_t c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ float16_t mfma32(x8 a, x8 b, float16_t c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};

// Sums over the lanes before and including this one: four shifts within rows of 16, then the rows' last sums to the rows behind.  (Six vector
// instructions; by way of LDS, as shuffles go, a scan takes half a microsecond of a call of a few.)
template <int CTRL, int ROWS, typename T>
__device__ __forceinline__ T from_lane(T x) {                // zero where there is no such lane
    return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, ROWS, 0xF, false));
}

template <typename T>
__device__ __forceinline__ T wave_scan(T x) {
    x += from_lane<0x111, 0xF>(x);                           // row_shr:1, 2, 4, 8
    x += from_lane<0x112, 0xF>(x);
    x += from_lane<0x114, 0xF>(x);
    x += from_lane<0x118, 0xF>(x);
    x += from_lane<0x142, 0xA>(x);                           // row_bcast:15 into rows 1 and 3, row_bcast:31 into 2 and 3
    x += from_lane<0x143, 0xC>(x);
    return x;
}

// The largest of the lanes up to this one, of values that are not negative.
__device__ __forceinline__ int wave_max(int x) {
    x = max(x, from_lane<0x111, 0xF>(x));
    x = max(x, from_lane<0x112, 0xF>(x));
    x = max(x, from_lane<0x114, 0xF>(x));
    x = max(x, from_lane<0x118, 0xF>(x));
    x = max(x, from_lane<0x142, 0xA>(x));
    x = max(x, from_lane<0x143, 0xC>(x));
    return x;
}

// Host-side checks.
inline bool aligned_to(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

inline bool page_size_valid(int ps) { return ps >= 16 && ps <= 256 && (ps & (ps - 1)) == 0; }

// A launch's threads are counted in 32 bits.
inline bool launchable(int64_t workgroups, int threads) { return workgroups <= (int64_t)UINT32_MAX / threads; }

inline int log2_of(int pow2) { return 31 - __builtin_clz((unsigned)pow2); }

// Strides of whole 16-byte pieces; a page's heads and tokens are addressed with 32 bits from its start.
inline rtn_status check_cache(const rtn_kv_cache* c) {
    if (!c || !c->dev_k || !c->dev_v) return RTN_ERR_NULL;
    if (c->dtype != RTN_TYPE_F16 && c->dtype != RTN_TYPE_BF16) return RTN_ERR_CONFIG;
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return RTN_ERR_SHAPE;
    if (!page_size_valid(c->page_size) || c->kv_heads < 1 || c->kv_heads > 1024 || c->pages < 1 || c->pages > INT32_MAX / c->page_size) return RTN_ERR_SHAPE;
    if (c->page_stride < 0 || c->head_stride < 0 || c->token_stride < c->head_dim) return RTN_ERR_SHAPE;
    if (c->page_stride % 8 || c->head_stride % 8 || c->token_stride % 8) return RTN_ERR_ALIGN;
    // (offsets in bytes stay within 63 bits)
    if ((double)c->page_stride * (double)c->pages + (double)c->head_stride * (double)c->kv_heads > 0x1p48) return RTN_ERR_SHAPE;
    if (c->token_stride > ((int64_t)1 << 30) / c->page_size) return RTN_ERR_SHAPE;
    if (!aligned_to(c->dev_k, 16) || !aligned_to(c->dev_v, 16)) return RTN_ERR_ALIGN;
    return RTN_OK;
}

}  // namespace rtn
