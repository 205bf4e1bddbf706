// aspis_elements.h -- what the streaming kernels share: element types with
// their 16-byte vectors, and sums over lanes and workgroups in a fixed order.
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

#include "../../include/aspis.h"

namespace aspis {

namespace {

// Sixteen bytes of a tensor.  The address is aligned to the element only;
// gfx950 takes such vector accesses.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef u32x4 u32x4_at4 __attribute__((aligned(4)));
typedef u32x4 u32x4_at2 __attribute__((aligned(2)));
typedef u32x2 u32x2_at2 __attribute__((aligned(2)));
#define GLOBAL __attribute__((address_space(1)))

// ---------------------------------------------------------------------------
// element types: V elements per 16 bytes, to and from f32

struct F32 {
    typedef float T;
    typedef u32x4_at4 Vec;
    static constexpr int V = 4;
    static constexpr uint32_t kLowest = 0xFF800000u;   // -inf, in every element of a word
    __device__ static float get(T x) { return x; }
    __device__ static T put(float x) { return x; }
    __device__ static void unpack(u32x4 w, float (&x)[V]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = __uint_as_float(w[j]);
    }
    __device__ static u32x4 pack(const float (&x)[V]) {
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = __float_as_uint(x[j]);
        return w;
    }
};

struct BF16 {
    typedef __bf16 T;
    typedef u32x4_at2 Vec;
    static constexpr int V = 8;
    static constexpr uint32_t kLowest = 0xFF80FF80u;
    __device__ static float get(T x) { return (float)x; }
    __device__ static T put(float x) { return (__bf16)x; }
    __device__ static void unpack(u32x4 w, float (&x)[V]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[2 * j] = __uint_as_float(w[j] << 16);
            x[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
        }
    }
    __device__ static u32x4 pack(const float (&x)[V]) {
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            w[j] = __builtin_bit_cast(
                uint32_t, __builtin_convertvector((f32x2){x[2 * j], x[2 * j + 1]}, b2));
        return w;
    }
};

struct F16 {
    typedef _Float16 T;
    typedef u32x4_at2 Vec;
    static constexpr int V = 8;
    static constexpr uint32_t kLowest = 0xFC00FC00u;
    __device__ static float get(T x) { return (float)x; }
    __device__ static T put(float x) { return (_Float16)x; }
    __device__ static void unpack(u32x4 w, float (&x)[V]) {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t word = w[j];   // (a bit cast of w[j] itself reads w[0])
            const h2 h = __builtin_bit_cast(h2, word);
            x[2 * j] = (float)h[0];
            x[2 * j + 1] = (float)h[1];
        }
    }
    __device__ static u32x4 pack(const float (&x)[V]) {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            w[j] = __builtin_bit_cast(
                uint32_t, __builtin_convertvector((f32x2){x[2 * j], x[2 * j + 1]}, h2));
        return w;
    }
};

template <typename E>
using Ptr = const typename E::T GLOBAL *;
template <typename E>
using MutPtr = typename E::T GLOBAL *;

// A product rounded to E.  To f16 the compiler would make one instruction of
// both where a single element is stored, which adds +0 and so makes +0 of -0,
// unlike those of pack: the same element would have other bits by where it
// stands.  It is not to see that x is a product.
template <typename E>
__device__ __forceinline__ typename E::T put_product(float x) {
    if constexpr (E::V == 8) asm("" : "+v"(x));
    return E::put(x);
}

// Once: the data is not needed again soon (non-temporal).
enum class Use { Again, Once };

template <typename E, Use USE = Use::Again>
__device__ __forceinline__ u32x4 load_vec(Ptr<E> p) {
    const typename E::Vec GLOBAL *q = (const typename E::Vec GLOBAL *)p;
    if constexpr (USE == Use::Once) return __builtin_nontemporal_load(q);
    return *q;
}
template <typename E, Use USE = Use::Again>
__device__ __forceinline__ void store_vec(MutPtr<E> p, u32x4 v) {
    typename E::Vec GLOBAL *q = (typename E::Vec GLOBAL *)p;
    if constexpr (USE == Use::Once) __builtin_nontemporal_store((typename E::Vec)v, q);
    else *q = v;
}

// Calls f with the element type of a dtype code (uniform over the workgroup).
template <typename F>
__device__ __forceinline__ void with_type(int dtype, F &&f) {
    if (dtype == ASPIS_F32) f(F32());
    else if (dtype == ASPIS_BF16) f(BF16());
    else f(F16());
}

// ---------------------------------------------------------------------------
// sums

// v of the lane that the DPP control names.
template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
    const uint64_t w = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)w, CTRL, 0xF, 0xF, true);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(w >> 32), CTRL, 0xF, 0xF, true);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// Over groups of L consecutive lanes (a power of two <= 64), to every lane.
// Both partners of a step add the same two values, so all lanes agree.  Up
// to 16 lanes by DPP: within quads, then the mirrors pair the quads.
template <int L>
__device__ __forceinline__ double lanes_sum(double v) {
    if constexpr (L >= 2) v += dpp<0xB1>(v);    // quad_perm 1,0,3,2
    if constexpr (L >= 4) v += dpp<0x4E>(v);    // quad_perm 2,3,0,1
    if constexpr (L >= 8) v += dpp<0x141>(v);   // row_half_mirror
    if constexpr (L >= 16) v += dpp<0x140>(v);  // row_mirror
    if constexpr (L >= 32) v += __shfl_xor(v, 16, 64);
    if constexpr (L >= 64) v += __shfl_xor(v, 32, 64);
    return v;
}

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v),
                                                                 CTRL, 0xF, 0xF, true));
}
struct Sum {
    __device__ float operator()(float a, float b) const { return a + b; }
};
struct Max {   // of two numbers, or the one that is not NaN
    __device__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
// The same of floats, by an operation that does not mind the order of its two
// operands.
template <int L, typename Op>
__device__ __forceinline__ float lanes_join(float v, Op op) {
    if constexpr (L >= 2) v = op(v, dpp<0xB1>(v));
    if constexpr (L >= 4) v = op(v, dpp<0x4E>(v));
    if constexpr (L >= 8) v = op(v, dpp<0x141>(v));
    if constexpr (L >= 16) v = op(v, dpp<0x140>(v));
    if constexpr (L >= 32) v = op(v, __shfl_xor(v, 16, 64));
    if constexpr (L >= 64) v = op(v, __shfl_xor(v, 32, 64));
    return v;
}

// Over the workgroup of B threads, to every thread.  Two barriers: the
// second lets the caller use it again at once.
template <int B>
__device__ __forceinline__ double block_sum(double v) {
    v = lanes_sum<64>(v);
    if constexpr (B == 64) return v;
    __shared__ double part[B / 64];
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = v;
    __syncthreads();
    double s = part[0];
#pragma unroll
    for (int w = 1; w < B / 64; ++w) s += part[w];
    __syncthreads();
    return s;
}

}  // namespace

}  // namespace aspis
