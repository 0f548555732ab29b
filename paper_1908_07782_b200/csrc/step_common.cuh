// Device helpers shared by the kernels of the local step (clipping, group norm, grouped products).
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace combo_step {

// Programmatic dependent launch: wait for the preceding kernel of the stream / let the next one become resident.
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

__device__ __forceinline__ float widen_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float widen_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);   // round to nearest even, once
    return *reinterpret_cast<uint32_t*>(&v);
}

// Two binary32 values in one 64-bit register, the operand form of the f32x2 instructions: one instruction, two
// IEEE operations, each rounded as the scalar one.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair(float lo, float hi) {
    return ((f32x2)__float_as_uint(hi) << 32) | (f32x2)__float_as_uint(lo);
}
__device__ __forceinline__ float lo_of(f32x2 v) { return __uint_as_float((uint32_t)v); }
__device__ __forceinline__ float hi_of(f32x2 v) { return __uint_as_float((uint32_t)(v >> 32)); }
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
    f32x2 d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ f32x2 neg2(f32x2 a) { return a ^ 0x8000000080000000ull; }

// One element / one 16-byte vector of a type as binary32, and back (rounded to nearest even).
template <int EB> struct Elem;
template <> struct Elem<4> {
    static constexpr int V = 4;
    typedef float type;
    __device__ static __forceinline__ float get(const void* p) { return *static_cast<const float*>(p); }
    __device__ static __forceinline__ void put(void* p, float v) { *static_cast<float*>(p) = v; }
    __device__ static __forceinline__ void unpack(const uint4& v, float (&x)[4]) {
        x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
    }
    __device__ static __forceinline__ uint4 pack(const float (&x)[4]) {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
};
template <> struct Elem<2> {
    static constexpr int V = 8;
    typedef __nv_bfloat16 type;
    __device__ static __forceinline__ float get(const void* p) {
        return __uint_as_float((uint32_t)*static_cast<const unsigned short*>(p) << 16);
    }
    __device__ static __forceinline__ void put(void* p, float v) { *static_cast<__nv_bfloat16*>(p) = __float2bfloat16_rn(v); }
    __device__ static __forceinline__ void unpack(const uint4& v, float (&x)[8]) {
        x[0] = widen_lo(v.x); x[1] = widen_hi(v.x); x[2] = widen_lo(v.y); x[3] = widen_hi(v.y);
        x[4] = widen_lo(v.z); x[5] = widen_hi(v.z); x[6] = widen_lo(v.w); x[7] = widen_hi(v.w);
    }
    __device__ static __forceinline__ uint4 pack(const float (&x)[8]) {
        return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
    }
};

template <typename T> __device__ __forceinline__ T warp_sum(T v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

}  // namespace combo_step
