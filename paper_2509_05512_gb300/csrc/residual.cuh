// residual.cuh -- what the kernels of the residual join share: a thread's channels, its place in a row,
// sums over the threads of a statistic, and the random numbers of a dropout.
#pragma once
#include <cuda_bf16.h>

#include "internal.h"
#include "philox.cuh"
#include "ptx.cuh"
#include "vec_io.cuh"

namespace quan {

struct JoinParams {
    const void *x, *h, *y, *dy, *dn;  // forward: x, h; backward: h, y, dy, dn
    const float *post, *gate, *pre;
    void *out_y, *out_n;               // forward: y, n; backward: dx, dh
    float *part_gate;                  // backward: sums of dgate, a row a unit
    float *part_post, *part_pre;       // and of dpost and dpre, a row a block
    long long rows, rows_per_image;
    int C, S, groups, tps, slots;
    long long units, chunk_rows;       // backward: units of chunk_rows rows within an image
    int chunks;                        // units of an image
    long long part_stride;             // between the rows of two blocks
    float alpha, eps, inv_s;
    DropoutArgs drop;
    // the norm in 8 bits as well: its values, scales and the lanes that a statistic takes (below)
    uint8_t* q8;
    float* s8;
    long long s8_pitch;
    int q8_pitch, kblk, red;
};

// The join with 8-bit rows (join_f8.cu) of rows that it takes, `whole`: one statistic a row.
bool join_f8_aligned(const JoinArgs& a);
cudaError_t launch_join_f8(const JoinParams& p, bool f32, bool whole, int num_sms,
                           cudaStream_t stream);

namespace {

// Eight consecutive channels of a thread, loaded LV at a time; `left` of them exist.
template <typename T, int LV>
struct Chunk {
    Raw<T, LV> r[8 / LV];
    __device__ __forceinline__ void load(const T* p, int left) {
#pragma unroll
        for (int i = 0; i < 8 / LV; ++i) {
            if (i * LV < left)
                r[i].load(p + i * LV);
            else
                r[i].zero();
        }
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < 8 / LV; ++i) r[i].zero();
    }
    __device__ __forceinline__ void values(float (&v)[8]) const {
#pragma unroll
        for (int i = 0; i < 8 / LV; ++i) {
            float w[LV];
            r[i].values(w);
#pragma unroll
            for (int j = 0; j < LV; ++j) v[i * LV + j] = w[j];
        }
    }
    __device__ __forceinline__ void set_store(const float (&v)[8], T* p, int left) {
#pragma unroll
        for (int i = 0; i < 8 / LV; ++i) {
            if (i * LV < left) {
                float w[LV];
#pragma unroll
                for (int j = 0; j < LV; ++j) w[j] = v[i * LV + j];
                r[i].set(w);
                r[i].store(p + i * LV);
            }
        }
    }
};

// Where a thread stands: its slot (row of the block's rows), group and chunks.
struct Place {
    int slot, seg, ts;
};
__device__ __forceinline__ Place place_of(const JoinParams& p) {
    const int tpr = p.groups * p.tps;
    Place q;
    q.slot = threadIdx.x / tpr;
    const int t = threadIdx.x - q.slot * tpr;
    q.seg = t / p.tps;
    q.ts = t - q.seg * p.tps;
    return q;
}

// Sum of v over the tps threads of a group.  Every thread of the block calls it together.
// CROSS (tps > 32): through shared memory, one word a warp, two buffers in turn: who writes a
// buffer has passed the other one's barrier, which every reader of this one reached after it.
template <bool CROSS, int N>
__device__ __forceinline__ void group_sum(float (&v)[N], int tps, float (&both)[2][96],
                                          int& turn) {
    if constexpr (!CROSS) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            if (o >= tps) continue;
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
        }
    } else {
        float* sm = both[turn];
        turn ^= 1;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
        }
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        const int wps = tps >> 5, first = warp & ~(wps - 1);
        if (lane == 0) {
#pragma unroll
            for (int k = 0; k < N; ++k) sm[32 * k + warp] = v[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            v[k] = lane < wps ? sm[32 * k + first + lane] : 0.0f;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
        }
    }
}

// A thread's share of a per-channel vector (1 without one).  A plain load: the grid before this
// one may be its writer, and the read-only path is for what nothing writes while the kernel runs.
// (32 x 56 x 56 x 256 bf16: 38.9 and 64.7 us; 39.3 and 65.3 where the compiler places the loads.)
template <int NC>
__device__ __forceinline__ void load_columns(const float* v, const JoinParams& p, const Place& q,
                                             float scale, float (&out)[NC][8]) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int col = (q.ts + c * p.tps) * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            out[c][j] = (v && col + j < p.S) ? scale * ld_global_f32(v + q.seg * p.S + col + j)
                                             : scale;
    }
}

// The draws of the eight elements from linear index i on.
template <bool ALIGNED>
__device__ __forceinline__ void draw_from(Dropout8& m, const DropoutArgs& d,
                                          unsigned long long base, long long i) {
    const unsigned long long block = base + (static_cast<unsigned long long>(i) >> 3);
    m.draw(d, block);
    if constexpr (!ALIGNED) {
        const int s = static_cast<int>(i & 7);
        if (s != 0) {
            Dropout8 next;
            next.draw(d, block + 1);
            m.shift(next, s);
        }
    }
}

}  // namespace
}  // namespace quan
