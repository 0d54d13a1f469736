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
};

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

// 8 elements of a row, at a multiple of 8 elements.
template <class T>
__device__ __forceinline__ void load8(const char* p, float (&x)[8]) {
    if constexpr (T::bytes == 2) {
        uint4 w = *reinterpret_cast<const uint4*>(p);
        float2 a = T::unpack(w.x), b = T::unpack(w.y), c = T::unpack(w.z), d = T::unpack(w.w);
        x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y, x[4] = c.x, x[5] = c.y, x[6] = d.x, x[7] = d.y;
    } else {
        uint2 w = *reinterpret_cast<const uint2*>(p);
        float2 a = F16::unpack(E4M3::halves(w.x & 0xffff)), b = F16::unpack(E4M3::halves(w.x >> 16));
        float2 c = F16::unpack(E4M3::halves(w.y & 0xffff)), d = F16::unpack(E4M3::halves(w.y >> 16));
        x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y, x[4] = c.x, x[5] = c.y, x[6] = d.x, x[7] = d.y;
    }
}
template <class T>
__device__ __forceinline__ void store8(char* p, const float (&x)[8]) {
    if constexpr (T::bytes == 2) {
        *reinterpret_cast<uint4*>(p) =
            make_uint4(T::pack(x[0], x[1]), T::pack(x[2], x[3]), T::pack(x[4], x[5]), T::pack(x[6], x[7]));
    } else {
        *reinterpret_cast<uint2*>(p) = make_uint2(T::pack(x[0], x[1]) | (T::pack(x[2], x[3]) << 16),
                                                  T::pack(x[4], x[5]) | (T::pack(x[6], x[7]) << 16));
    }
}

}  // namespace fcsim_kv_dev
