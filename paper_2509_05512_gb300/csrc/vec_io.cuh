// vec_io.cuh -- loads and stores of VEC consecutive elements (8, 4 or 1) of a bf16 or fp32
// tensor as fp32 values, in the widest accesses (8 and 4 elements: VEC x the element's size up
// to 16 bytes, which the address must be aligned to).
#pragma once
#include <cuda_bf16.h>

#include <cstdint>

namespace quan {

__device__ __forceinline__ void bf16x2_to_f32(uint32_t v, float& lo, float& hi) {
    lo = __uint_as_float(v << 16);
    hi = __uint_as_float(v & 0xFFFF0000u);
}

__device__ __forceinline__ uint32_t f32_to_bf16x2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// The words of VEC elements as they are in memory, so that a load can be issued long before
// its values are needed and takes no more registers than its bytes.
template <typename T, int VEC>
struct Raw {
    static constexpr int WORDS = VEC * static_cast<int>(sizeof(T)) / 4 > 0
                                     ? VEC * static_cast<int>(sizeof(T)) / 4
                                     : 1;
    uint32_t w[WORDS];

    __device__ __forceinline__ void load(const T* p) {
        if constexpr (VEC == 1 && sizeof(T) == 2) {
            w[0] = *reinterpret_cast<const unsigned short*>(p);
        } else if constexpr (WORDS == 1) {
            w[0] = *reinterpret_cast<const uint32_t*>(p);
        } else if constexpr (WORDS == 2) {
            const uint2 v = *reinterpret_cast<const uint2*>(p);
            w[0] = v.x, w[1] = v.y;
        } else {
#pragma unroll
            for (int i = 0; i < WORDS; i += 4) {
                const uint4 v = *reinterpret_cast<const uint4*>(
                    reinterpret_cast<const uint32_t*>(p) + i);
                w[i] = v.x, w[i + 1] = v.y, w[i + 2] = v.z, w[i + 3] = v.w;
            }
        }
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[i] = 0u;
    }
    __device__ __forceinline__ void values(float (&v)[VEC]) const {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = __uint_as_float(w[i]);
        } else if constexpr (VEC == 1) {
            v[0] = __uint_as_float(w[0] << 16);
        } else {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) bf16x2_to_f32(w[i], v[2 * i], v[2 * i + 1]);
        }
    }
    __device__ __forceinline__ void set(const float (&v)[VEC]) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) w[i] = __float_as_uint(v[i]);
        } else if constexpr (VEC == 1) {
            w[0] = f32_to_bf16x2(v[0], 0.0f);
        } else {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) w[i] = f32_to_bf16x2(v[2 * i], v[2 * i + 1]);
        }
    }
    __device__ __forceinline__ void store(T* p) const {
        if constexpr (VEC == 1 && sizeof(T) == 2) {
            *reinterpret_cast<unsigned short*>(p) = static_cast<unsigned short>(w[0]);
        } else if constexpr (WORDS == 1) {
            *reinterpret_cast<uint32_t*>(p) = w[0];
        } else if constexpr (WORDS == 2) {
            *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        } else {
#pragma unroll
            for (int i = 0; i < WORDS; i += 4)
                *reinterpret_cast<uint4*>(reinterpret_cast<uint32_t*>(p) + i) =
                    make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
        }
    }
};

// Bytes the accesses of Raw<T, VEC> need their address aligned to.
template <typename T, int VEC>
constexpr int raw_align() {
    return VEC * static_cast<int>(sizeof(T)) > 16 ? 16 : VEC * static_cast<int>(sizeof(T));
}

}  // namespace quan
