// Items of 4 and 2 bytes as the agent's update reads and writes them: 16 bytes at a time where a row is aligned.
#pragma once
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cham {

typedef float float2v __attribute__((ext_vector_type(2)));

struct F32 {
    using item = float;
    typedef unsigned words __attribute__((ext_vector_type(4), aligned(4)));         // 16 bytes that begin at any item
    static constexpr int kVec = 4;              // items in 16 bytes
    static constexpr uint32_t kMasked = 0xff800000u;         // -inf
    static __device__ __forceinline__ float get(item x) { return x; }
    static __device__ __forceinline__ item put(float x) { return x; }
    static __device__ __forceinline__ void unpack(const uint4 &v, float (&x)[4])
    {
        x[0] = __uint_as_float(v.x);
        x[1] = __uint_as_float(v.y);
        x[2] = __uint_as_float(v.z);
        x[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&x)[4])
    {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
};

struct BF16 {
    using item = __bf16;
    typedef unsigned words __attribute__((ext_vector_type(4), aligned(2)));
    static constexpr int kVec = 8;
    static constexpr uint32_t kMasked = 0xff80u;
    static __device__ __forceinline__ float get(item x) { return (float)x; }
    static __device__ __forceinline__ item put(float x) { return (item)x; }        // to the nearest, ties to even
    static __device__ __forceinline__ void unpack(const uint4 &v, float (&x)[8])
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ uint4 pack(const float (&x)[8])
    {
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2v p = {x[2 * i], x[2 * i + 1]};                            // both in one instruction
            w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, b2));
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

struct F16 {
    using item = _Float16;
    typedef unsigned words __attribute__((ext_vector_type(4), aligned(2)));
    static constexpr int kVec = 8;
    static constexpr uint32_t kMasked = 0xfc00u;
    // x as fp32: the compiler folds a product and its rounding to f16 into one operation where it can, which depends on the
    // code around it, and a result would depend on the alignment of its row
    static __device__ __forceinline__ float held(float x)
    {
        asm volatile("" : "+v"(x));
        return x;
    }
    static __device__ __forceinline__ float get(item x) { return (float)x; }
    static __device__ __forceinline__ item put(float x) { return (item)held(x); }
    static __device__ __forceinline__ void unpack(const uint4 &v, float (&x)[8])
    {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const h2 p = __builtin_bit_cast(h2, w[i]);
            x[2 * i] = (float)p.x;
            x[2 * i + 1] = (float)p.y;
        }
    }
    static __device__ __forceinline__ uint4 pack(const float (&x)[8])
    {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2v p = {held(x[2 * i]), held(x[2 * i + 1])};
            w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, h2));
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

inline int type_bytes(int type) { return type == 0 ? 4 : 2; }     // CHAM_TYPE_F32, _BF16, _F16

// Items in front of the first 16-byte boundary at or behind p, at most n.
template <typename T>
__device__ __forceinline__ int64_t items_to_boundary(const typename T::item *p, int64_t n)
{
    const int64_t h = (int64_t)((16u - ((unsigned)reinterpret_cast<uintptr_t>(p) & 15u)) & 15u) / (int64_t)sizeof(*p);
    return h < n ? h : n;
}

}  // namespace cham
