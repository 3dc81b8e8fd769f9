// Helpers of the kernels that work on rows of logits [R, A] (action sampling, policy loss): rows may
// start at any element, so a row is walked as a ragged head, 16-byte vectors and a ragged tail.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace rlcs_rows {

struct bf16 { uint16_t bits; };

template <typename T> struct Vec;                       // one 16-byte access

__device__ __forceinline__ float max_nan(float a, float b) {      // NaN if either is
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

__device__ __forceinline__ uint32_t max_nan_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

template <> struct Vec<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void unpack(const uint4& v, float* f) {
        f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ uint4 pack(const float* f) {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
    static __device__ __forceinline__ float load(const float* p) { return *p; }
    static constexpr uint32_t kNothing = 0xff800000u;           // -inf throughout
    static __device__ __forceinline__ uint32_t most(uint32_t a, uint32_t b) {
        return __float_as_uint(max_nan(__uint_as_float(a), __uint_as_float(b)));
    }
    static __device__ __forceinline__ float most_of(uint32_t a) { return __uint_as_float(a); }
    static __device__ __forceinline__ uint32_t most_number(uint32_t a, uint32_t b) {      // NaN aside
        return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
    }
    static __device__ __forceinline__ float most_number_of(uint32_t a) { return fmaxf(__uint_as_float(a), -INFINITY); }
    static constexpr uint32_t kFloor = 0xf149f2cau;             // -1e30
    static __device__ __forceinline__ uint4 floored(const uint4& v) {      // nothing below about -1e30
        return make_uint4(most(v.x, kFloor), most(v.y, kFloor), most(v.z, kFloor), most(v.w, kFloor));
    }
    static __device__ __forceinline__ void store(float* p, float v) { *p = v; }
};

template <> struct Vec<bf16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void two(uint32_t w, float* f) {
        f[0] = __uint_as_float(w << 16);
        f[1] = __uint_as_float(w & 0xffff0000u);
    }
    static __device__ __forceinline__ void unpack(const uint4& v, float* f) {
        two(v.x, f); two(v.y, f + 2); two(v.z, f + 4); two(v.w, f + 6);
    }
    static __device__ __forceinline__ uint32_t pair(float lo, float hi) {
        uint32_t r;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
    static __device__ __forceinline__ uint4 pack(const float* f) {
        return make_uint4(pair(f[0], f[1]), pair(f[2], f[3]), pair(f[4], f[5]), pair(f[6], f[7]));
    }
    static constexpr uint32_t kNothing = 0xff80ff80u;
    static __device__ __forceinline__ uint32_t most(uint32_t a, uint32_t b) { return max_nan_bf16x2(a, b); }
    static __device__ __forceinline__ float most_of(uint32_t a) {
        return max_nan(__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u));
    }
    static __device__ __forceinline__ uint32_t most_number(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ float most_number_of(uint32_t a) {
        return fmaxf(fmaxf(__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u)), -INFINITY);
    }
    static constexpr uint32_t kFloor = 0xf149f149u;
    static __device__ __forceinline__ uint4 floored(const uint4& v) {      // nothing below about -1e30
        return make_uint4(most(v.x, kFloor), most(v.y, kFloor), most(v.z, kFloor), most(v.w, kFloor));
    }
    static __device__ __forceinline__ float load(const bf16* p) { return __uint_as_float((uint32_t)p->bits << 16); }
    static __device__ __forceinline__ void store(bf16* p, float v) { p->bits = (uint16_t)(pair(v, 0.f) & 0xffffu); }
};

// Where the 16-byte vectors of a row lie: elements [0, head) one by one, `vecs` vectors from `head`, the rest one by one.
struct Span {
    int head, vecs;
};

template <typename T> __host__ __device__ __forceinline__ Span span_of(const T* row, int n) {
    const int off = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    int head = off ? Vec<T>::N - off : 0;
    if (head > n) head = n;
    return Span{head, (n - head) / Vec<T>::N};
}

template <typename T> __device__ __forceinline__ T warp_max(T v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) { const T u = __shfl_xor_sync(~0u, v, o); v = u > v ? u : v; }
    return v;
}

template <typename T> __device__ __forceinline__ T warp_sum(T v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}

}  // namespace rlcs_rows
