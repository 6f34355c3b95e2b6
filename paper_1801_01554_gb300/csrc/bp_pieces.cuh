// Rows in 16-byte pieces: what the kernels of bp_blocks.h load and store.
#pragma once

#include "bp_experts_device.cuh"

namespace bp {
namespace {

// V values of a row, 16 bytes of it (or one float32 where rows are not whole 16-byte pieces).
template <class T, int V>
struct Piece {
    uint4 u;
    __device__ __forceinline__ void load(const T* p) {   // (volatile: a batch of loads stays a batch)
        if constexpr (V == 1) asm volatile("ld.global.nc.u32 %0, [%1];" : "=r"(u.x) : "l"(p));
        else asm volatile("ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p));
    }
    // Where the buffer may also be written by this launch (in place).
    __device__ __forceinline__ void load_rw(const T* p) {
        if constexpr (V == 1) asm volatile("ld.global.u32 %0, [%1];" : "=r"(u.x) : "l"(p) : "memory");
        else asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p) : "memory");
    }
    __device__ __forceinline__ void values(float (&v)[V]) const {
        const unsigned w[4] = {u.x, u.y, u.z, u.w};
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = __uint_as_float(w[i]);
        }
    }
    // The values rounded to T.
    __device__ __forceinline__ void set(const float (&v)[V]) {
        if constexpr (sizeof(T) == 2) {
            unsigned w[4];
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                w[i] = *reinterpret_cast<const unsigned*>(&h);
            }
            u = make_uint4(w[0], w[1], w[2], w[3]);
        } else if constexpr (V == 1) {
            u.x = __float_as_uint(v[0]);
        } else {
            u = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        }
    }
    __device__ __forceinline__ void store(T* p) const {
        if constexpr (V == 1) *reinterpret_cast<unsigned*>(p) = u.x;
        else *reinterpret_cast<uint4*>(p) = u;
    }
};
// float32 values, in 16-byte pieces where V > 1.
template <int V>
__device__ __forceinline__ void store_floats(float* p, const float (&v)[V]) {
    if constexpr (V == 1) {
        *p = v[0];
    } else {
#pragma unroll
        for (int i = 0; i < V; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    }
}

// As another SM has just written them (from L2).
template <int V>
__device__ __forceinline__ void load_floats_l2(const float* p, float (&v)[V]) {
    if constexpr (V == 1) {
        v[0] = __ldcg(p);
    } else {
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const float4 x = __ldcg(reinterpret_cast<const float4*>(p + i));
            v[i] = x.x, v[i + 1] = x.y, v[i + 2] = x.z, v[i + 3] = x.w;
        }
    }
}

}  // namespace
}  // namespace bp
