// philox.cuh -- the counter-based generator of the dropout masks: Philox4x32-10 (Salmon,
// Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011).  A block of
// 128 random bits is a function of a 64-bit counter and a 64-bit key alone, so a mask is
// computed again wherever it is needed and never stored.
//
// A block serves eight elements with 16 bits each: element i of a tensor takes bits
// 16 (i mod 8) and up of block offset + i / 8.  Sixteen bits give every probability in steps of
// 2^-16, and halve the integer work, which at 32 bits an element would bound the kernel:
// a block is 20 wide multiplications and 20 three-input xors, about 60 issue slots, 7.5 an
// element, where streaming bf16 at 6.7 TB/s leaves about 22 an element.
#pragma once
#include <cstdint>

#include "internal.h"

namespace quan {

__device__ __forceinline__ uint4 philox4x32_10(unsigned long long block, uint32_t key0,
                                               uint32_t key1) {
    uint32_t c0 = static_cast<uint32_t>(block), c1 = static_cast<uint32_t>(block >> 32);
    uint32_t c2 = 0, c3 = 0;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const unsigned long long a = static_cast<unsigned long long>(c0) * 0xD2511F53u;
        const unsigned long long b = static_cast<unsigned long long>(c2) * 0xCD9E8D57u;
        c0 = static_cast<uint32_t>(b >> 32) ^ c1 ^ key0;
        c1 = static_cast<uint32_t>(b);
        c2 = static_cast<uint32_t>(a >> 32) ^ c3 ^ key1;
        c3 = static_cast<uint32_t>(a);
        key0 += 0x9E3779B9u;
        key1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}

// The draws of a block's eight elements: element j is kept when keep(j).  A draw is compared in
// the upper half of a word, so the odd ones need no shift.
struct Dropout8 {
    uint32_t w[4];
    __device__ __forceinline__ void none() { w[0] = w[1] = w[2] = w[3] = 0u; }
    __device__ __forceinline__ void draw(const DropoutArgs& d, unsigned long long block) {
        const uint4 r = philox4x32_10(block, d.key0, d.key1);
        w[0] = r.x, w[1] = r.y, w[2] = r.z, w[3] = r.w;
    }
    __device__ __forceinline__ bool keep(const DropoutArgs& d, int j) const {
        return (j & 1 ? w[j >> 1] : w[j >> 1] << 16) >= d.bound;
    }
    // The eight elements from element s of this block on, `next` holding the block after it.
    __device__ __forceinline__ void shift(const Dropout8& next, int s) {
        const int n = s >> 1;
        uint32_t a[8] = {w[0], w[1], w[2], w[3], next.w[0], next.w[1], next.w[2], next.w[3]};
#pragma unroll
        for (int k = 0; k < 6; ++k) a[k] = n & 2 ? a[k + 2] : a[k];
#pragma unroll
        for (int k = 0; k < 5; ++k) a[k] = n & 1 ? a[k + 1] : a[k];
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = s & 1 ? (a[k] >> 16) | (a[k + 1] << 16) : a[k];
    }
};

// The counter base of a call: the offset, and the device word when there is one.
__device__ __forceinline__ unsigned long long dropout_base(const DropoutArgs& d) {
    return d.offset + (d.counter ? *d.counter : 0ull);
}

}  // namespace quan
