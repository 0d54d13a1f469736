// Device-side pieces that the kernels of the paged key-value cache share: element types, rows of 16 bytes, pages.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <stdint.h>

#include "fcsim_kv.h"

namespace fcsim_kv_dev {

// The cache as a kernel sees it.  Offsets are 64-bit: a pool passes 2^31 elements long before it fills the memory.
struct Pool {
    char *k, *v;
    float* weight;
    const float *k_scale, *v_scale;
    int64_t stride_page, stride_slot, stride_head;  // elements
    int n_pages, page_size, n_kv, head_dim;
    uint64_t page_magic;  // ceil(2^63 / page_size)
};

// t / page_size by a multiplication, exact for t < 2^31.
__device__ __forceinline__ int page_of(const Pool& pool, int t) {
    const uint32_t x = (uint32_t)t << 1;
    const uint64_t low = (uint64_t)x * (uint32_t)pool.page_magic;
    return (int)(((uint64_t)x * (uint32_t)(pool.page_magic >> 32) + (low >> 32)) >> 32);
}

// Sets a bit of the caller's status word (if there is one).
__device__ __forceinline__ void flag(int32_t* status, int bit) {
    if (status) atomicOr(status, bit);
}

struct F16 {
    static constexpr int bytes = 2;
    static __device__ __forceinline__ float2 unpack(uint32_t w) {
        return __half22float2(*reinterpret_cast<const __half2*>(&w));
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<uint32_t*>(&h);
    }
};
struct BF16 {
    static constexpr int bytes = 2;
    static __device__ __forceinline__ float2 unpack(uint32_t w) {
        return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<uint32_t*>(&h);
    }
};
struct E4M3 {
    static constexpr int bytes = 1;
    // two stored bytes (the low half of w) as two halves, exactly
    static __device__ __forceinline__ uint32_t halves(uint32_t w) {
        uint32_t h;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)w));
        return h;
    }
    // round to nearest even; beyond +-448 the largest value
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    }
};

}  // namespace fcsim_kv_dev
