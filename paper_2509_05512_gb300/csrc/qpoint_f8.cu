// qpoint_f8.cu -- the pointwise (1x1) quaternion convolution in 8-bit floating point: x is
// quantised in the call, the letters once (f8.cuh), both with a scale for each block of 128:
//   activations  128 channels of one component of one row;
//   letters      128 output x 128 input channels of one letter.
// With q the 8-bit values, s the scales, L = co xor ci and sgn Eq. 6's signs,
//   y[m][co][n] = sum over ci, blocks b of  sgn(co, ci) s_x[ci][b][m] s_w[L][n / 128][b]
//                 sum over k in b of  q_x[m][ci][k] q_w[L][n][k].
// The input gradient is the same product with dy in place of x and the letters transposed, whose
// signs are those of conj(W): letters i, j and k negated.
//
// Layouts: q_x [row][4][Kp] and q_w [4][Nq][Kp] with Kp = Kq rounded up to 16, zeros in the
// padding; s_x [4][blocks][rows rounded up to 128], s_w [4][ceil(Nq / 128)][blocks].
//
// Inputs are read with plain loads only: these grids start while the one before them may still
// write what they read, and the read-only path may be used only for what nothing writes while
// the kernel runs.
#include <cuda_bf16.h>

#include <atomic>
#include <cstdio>

#include "f8.cuh"
#include "internal.h"
#include "ptx.cuh"
#include "tc_common.cuh"
#include "vec_io.cuh"

namespace quan {
namespace {

// Eight consecutive bf16 channels from k on (the row has Kq of them), 0 past the end.
template <bool VEC>
__device__ __forceinline__ void load_x8(const __nv_bfloat16* p, int k, int Kq, float (&v)[8]) {
    if (VEC) {  // Kq is a multiple of 8
        Raw<__nv_bfloat16, 8> r;
        if (k < Kq)
            r.load(p + k);
        else
            r.zero();
        r.values(v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = k + j < Kq ? __bfloat162float(p[k + j]) : 0.0f;
    }
}

// Scale of the 128 channels that a half-warp holds, eight a lane.
__device__ __forceinline__ float half_warp_scale(const float (&v)[8], float& inv) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, abs_bits(v[j]));
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    return f8_scale(__uint_as_float(m), inv);
}

// Eight consecutive bf16 channels as words, LV channels a load (their address aligned to that);
// `left` of them exist, a multiple of LV where LV > 1, the others are 0.
template <int LV>
__device__ __forceinline__ void load_words8(const __nv_bfloat16* p, int left, uint32_t (&w)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = 0u;
    if constexpr (LV == 8) {
        if (left > 0) {
            const uint4 v = *reinterpret_cast<const uint4*>(p);
            w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
        }
    } else if constexpr (LV == 2) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (2 * j < left) w[j] = reinterpret_cast<const uint32_t*>(p)[j];
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < left)
                w[j / 2] |=
                    static_cast<uint32_t>(reinterpret_cast<const unsigned short*>(p)[j])
                    << (16 * (j & 1));
    }
}

// Channels a load may take of rows of n channels, all tensors or'ed into `address`.
int load_channels(int n, uintptr_t address) {
    return n % 8 == 0 && address % 16 == 0 ? 8 : (n % 2 == 0 && address % 4 == 0 ? 2 : 1);
}

// ------------------------------------------------------------------ letters

struct F8Letters {
    const __nv_bfloat16* w[4];  // [rows][cols]
    int rows, cols;             // Qout, Qin
    uint8_t* q;                 // [4][N][Kp]: N = rows, K = cols, or the other way round
    float* scale;               // [4][N blocks][K blocks]
    int Kp, nblk, kblk;
};

// One 128 x 128 block of one letter: its scale, then its 8-bit values, which the transposed form
// turns in shared memory so that it too is written along its rows.  A thread has eight channels of
// eight rows, all loaded before the first is looked at: a block is one trip to memory (LV channels
// a load).  The letters of 512 -> 1024: 1.9 us (transposed 2.8), of 4096 -> 4096 4.5 us, 2.8 TB/s
// (transposed 6.3).
template <bool TRANSPOSE, int LV>
__global__ void __launch_bounds__(256) f8_letters_kernel(const F8Letters p) {
    __shared__ uint8_t tile[128 * 129];  // 129: neither direction meets a bank twice
    __shared__ uint32_t top[8];
    griddep_launch_dependents();
    griddep_wait();
    const int letter = blockIdx.z, r0 = blockIdx.y * 128, c0 = blockIdx.x * 128;
    const int tr = threadIdx.x >> 4, tc = (threadIdx.x & 15) * 8;  // rows tr + 16 i
    const __nv_bfloat16* w = p.w[letter] + c0 + tc;
    uint32_t v[8][4], m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = r0 + tr + 16 * i;
        load_words8<LV>(w + static_cast<long long>(r) * p.cols, r < p.rows ? p.cols - c0 - tc : 0,
                        v[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) m = __vmaxu2(m, v[i][j] & 0x7FFF7FFFu);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, o));
    if ((threadIdx.x & 31) == 0) top[threadIdx.x >> 5] = m;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 8; ++k) m = __vmaxu2(m, top[k]);
    float inv;
    const float s = f8_scale(__uint_as_float(max(m << 16, m & 0xFFFF0000u)), inv);
    const int nb = TRANSPOSE ? blockIdx.x : blockIdx.y, kb = TRANSPOSE ? blockIdx.y : blockIdx.x;
    if (threadIdx.x == 0)
        p.scale[(static_cast<long long>(letter) * p.nblk + nb) * p.kblk + kb] = s;
    const int N = TRANSPOSE ? p.cols : p.rows;
    uint8_t* q = p.q + static_cast<long long>(letter) * N * p.Kp + kb * 128;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        uint32_t h[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float lo, hi;
            bf16x2_to_f32(v[i][j], lo, hi);
            h[j] = f8x2_from_f32(lo * inv, hi * inv);
        }
        const int r = tr + 16 * i;
        if constexpr (TRANSPOSE) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                tile[r * 129 + tc + j] = static_cast<uint8_t>(h[j >> 1] >> (8 * (j & 1)));
        } else if (r0 + r < N && kb * 128 + tc < p.Kp) {
            *reinterpret_cast<uint2*>(q + static_cast<long long>(r0 + r) * p.Kp + tc) =
                make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
        }
    }
    if constexpr (TRANSPOSE) {
        __syncthreads();
        for (int i = threadIdx.x; i < 128 * 32; i += 256) {
            const int n = i >> 5, k = (i & 31) * 4;
            if (c0 + n >= N || kb * 128 + k >= p.Kp) continue;
            uint32_t h = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                h |= static_cast<uint32_t>(tile[(k + j) * 129 + n]) << (8 * j);
            *reinterpret_cast<uint32_t*>(q + static_cast<long long>(c0 + n) * p.Kp + k) = h;
        }
    }
}

// ------------------------------------------------------------------ the product

struct F8Params {
    const __nv_bfloat16* x;  // [rows][4 Kq], or null:
    const uint8_t* xq;       // [rows][4][Kp]
    const float* xs;         // [4][kblk][pitch]
    long long pitch;
    const uint8_t* wq;       // [4][Nq][Kp]
    const float* ws;         // [4][nblk][kblk]
    EpilogueArgs ep;
    __nv_bfloat16* out;      // [rows][4 Nq]
    long long rows;
    int Kq, Nq, Kp, kblk, nblk;
    int conj;  // letters i, j and k enter negated
    int act;
};

__device__ __forceinline__ void f8_store(const F8Params& p, long long row, int co, int n,
                                         float acc) {
    const int c = co * p.Nq + n;
    if (p.ep.bias) acc += p.ep.bias[c];
    if (p.ep.scale) acc = fmaf(p.ep.scale[c], acc, p.ep.shift[c]);
    p.out[row * (4LL * p.Nq) + c] = __float2bfloat16_rn(f8_act(acc, p.act));
}

// A warp per quaternion output channel, RT rows a block: the block quantises its rows' channels
// 512 at a time into shared memory (as the values they stand for), each lane multiplies four
// channels of a block of 128, and the warp adds its lanes at the end.  Every product is exact in
// fp32.  Q8: the rows come in 8 bits and are only read back.
constexpr int ROWS_K = 512;
template <int RT, bool VEC, bool Q8>
__global__ void __launch_bounds__(256) qpoint_rows_kernel(const F8Params p) {
    __shared__ float xs[RT][4][ROWS_K];
    griddep_launch_dependents();
    griddep_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int half = threadIdx.x >> 4, hl = threadIdx.x & 15;
    const int n = blockIdx.y * 8 + warp;
    const long long row0 = static_cast<long long>(blockIdx.x) * RT;
    float acc[RT][4] = {};
    for (int k0 = 0; k0 < p.Kq; k0 += ROWS_K) {
        __syncthreads();
        for (int u = half; u < RT * 16; u += 16) {
            const int r = u >> 4, ci = (u >> 2) & 3, b = u & 3;
            const int k = k0 + b * F8_BLOCK + hl * 8;
            if constexpr (Q8) {
                const int kb = k0 / F8_BLOCK + b;
                uint2 w = make_uint2(0u, 0u);
                float s = 0.0f;
                if (row0 + r < p.rows && k < p.Kp) {
                    w = *reinterpret_cast<const uint2*>(p.xq + ((row0 + r) * 4 + ci) * p.Kp + k);
                    s = p.xs[(static_cast<long long>(ci) * p.kblk + kb) * p.pitch + row0 + r];
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float d[4];
                    f8x4_to_f32(j ? w.y : w.x, d);
                    *reinterpret_cast<float4*>(&xs[r][ci][b * F8_BLOCK + hl * 8 + 4 * j]) =
                        make_float4(d[0] * s, d[1] * s, d[2] * s, d[3] * s);
                }
                continue;
            }
            float v[8], inv;
            if (row0 + r < p.rows) {
                load_x8<VEC>(p.x + (row0 + r) * (4LL * p.Kq) + ci * p.Kq, k, p.Kq, v);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = 0.0f;
            }
            const float s = half_warp_scale(v, inv);
#pragma unroll
            for (int j = 0; j < 8; j += 4) {
                float d[4];
                f8x4_to_f32(f8x4_from_f32(v[j] * inv, v[j + 1] * inv, v[j + 2] * inv,
                                          v[j + 3] * inv), d);
                *reinterpret_cast<float4*>(&xs[r][ci][b * F8_BLOCK + hl * 8 + j]) =
                    make_float4(d[0] * s, d[1] * s, d[2] * s, d[3] * s);
            }
        }
        __syncthreads();
        if (n >= p.Nq) continue;
        // the four blocks' letters and scales first, then the products
        uint32_t q[ROWS_K / F8_BLOCK][4];
        float sw[ROWS_K / F8_BLOCK][4];
#pragma unroll
        for (int b = 0; b < ROWS_K / F8_BLOCK; ++b) {
            const int kb = k0 / F8_BLOCK + b, k = kb * F8_BLOCK + lane * 4;
#pragma unroll
            for (int L = 0; L < 4; ++L) {
                q[b][L] = k < p.Kp ? *reinterpret_cast<const uint32_t*>(
                                         p.wq + (static_cast<long long>(L) * p.Nq + n) * p.Kp + k)
                                   : 0u;
                sw[b][L] = kb < p.kblk
                               ? p.ws[(static_cast<long long>(L) * p.nblk + n / F8_BLOCK) *
                                          p.kblk + kb]
                               : 0.0f;
            }
        }
#pragma unroll
        for (int b = 0; b < ROWS_K / F8_BLOCK; ++b) {
            if (k0 + b * F8_BLOCK >= p.Kq) break;
            float w[4][4];
#pragma unroll
            for (int L = 0; L < 4; ++L) {
                const float s = p.conj && L > 0 ? -sw[b][L] : sw[b][L];
                f8x4_to_f32(q[b][L], w[L]);
#pragma unroll
                for (int j = 0; j < 4; ++j) w[L][j] *= s;
            }
#pragma unroll
            for (int r = 0; r < RT; ++r) {
#pragma unroll
                for (int ci = 0; ci < 4; ++ci) {
                    const float4 x4 =
                        *reinterpret_cast<const float4*>(&xs[r][ci][b * F8_BLOCK + lane * 4]);
                    const float xv[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
                    for (int co = 0; co < 4; ++co)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            acc[r][co] = fmaf(
                                (tc::NEG_MASK >> (4 * co + ci)) & 1u ? -w[co ^ ci][j]
                                                                     : w[co ^ ci][j],
                                xv[j], acc[r][co]);
                }
            }
        }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int co = 0; co < 4; ++co) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1)
                acc[r][co] += __shfl_xor_sync(0xffffffffu, acc[r][co], o);
        }
    if (n < p.Nq && lane < 4) {
#pragma unroll
        for (int r = 0; r < RT; ++r)
            if (row0 + r < p.rows) {
                const float v = lane == 0 ? acc[r][0]
                                          : (lane == 1 ? acc[r][1]
                                                       : (lane == 2 ? acc[r][2] : acc[r][3]));
                f8_store(p, row0 + r, lane, n, v);
            }
    }
}

template <int RT>
cudaError_t launch_rows(const F8Params& p, bool vec, cudaStream_t stream) {
    const dim3 g(static_cast<unsigned>((p.rows + RT - 1) / RT),
                 static_cast<unsigned>((p.Nq + 7) / 8));
    if (p.xq) return launch_pdl(qpoint_rows_kernel<RT, true, true>, g, dim3(256), 0, stream, p);
    return vec ? launch_pdl(qpoint_rows_kernel<RT, true, false>, g, dim3(256), 0, stream, p)
               : launch_pdl(qpoint_rows_kernel<RT, false, false>, g, dim3(256), 0, stream, p);
}

// ------------------------------------------------------------------ rows in 8 bits

// GL lanes a block of 128 channels, eight channels a lane: the block's scale, then its 8-bit
// values.  GL = 16, or 8 or 4 where a component has no more than 64 or 32 channels.  Bound by HBM:
// 2 bytes read, 1 written a channel.
struct F8Rows {
    const __nv_bfloat16* x;  // [rows][4 Kq]
    uint8_t* q;              // [rows][4][Kp]
    float* scale;            // [4][kblk][pitch]
    long long rows, pitch;
    int Kq, Kp, kblk;
    int group;  // rows side by side in a block of threads
};

// A block of threads takes 256 / GL of a row's blocks side by side (grid.y counts these), or as
// many whole rows as fit, and F8_ROWS_UNROLL such row groups, whose loads all go out first; so a
// thread's component and block, the results of two divisions, hold for all of them.  102,400 x 512
// channels: 28 us, 5.6 TB/s (a division a block: 36).
constexpr int F8_ROWS_UNROLL = 4;

template <int GL, int LV>
__global__ void __launch_bounds__(256) f8_rows_kernel(const F8Rows p) {
    griddep_launch_dependents();
    griddep_wait();
    const int hl = threadIdx.x & (GL - 1);
    const unsigned per_row = 4u * p.kblk, unit = blockIdx.y * (256u / GL) + threadIdx.x / GL;
    const unsigned r0 = unit / per_row, rest = unit - r0 * per_row;
    const unsigned ci = rest / p.kblk, b = rest - ci * p.kblk;
    const int k = static_cast<int>(b) * F8_BLOCK + hl * 8;
    // units past the row groups' whole rows have nothing to do
    const bool mine = r0 < static_cast<unsigned>(p.group);
    const long long row0 = static_cast<long long>(blockIdx.x) * (p.group * F8_ROWS_UNROLL) + r0;
    const __nv_bfloat16* x = p.x + row0 * (4LL * p.Kq) + static_cast<int>(ci) * p.Kq + k;
    uint32_t w[F8_ROWS_UNROLL][4];  // eight bf16 channels
#pragma unroll
    for (int i = 0; i < F8_ROWS_UNROLL; ++i)
        load_words8<LV>(x + static_cast<long long>(i * p.group) * (4LL * p.Kq),
                        mine && row0 + i * p.group < p.rows ? p.Kq - k : 0, w[i]);
#pragma unroll
    for (int i = 0; i < F8_ROWS_UNROLL; ++i) {
        // largest magnitude: the bits without the sign order as the numbers do, NaN above all
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) m = __vmaxu2(m, w[i][j] & 0x7FFF7FFFu);
#pragma unroll
        for (int o = GL / 2; o > 0; o >>= 1) m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, o));
        m = max(m << 16, m & 0xFFFF0000u);
        const long long row = row0 + i * p.group;
        if (!mine || row >= p.rows) continue;
        float inv;
        const float s = f8_scale(__uint_as_float(m), inv);
        if (hl == 0) p.scale[(static_cast<long long>(ci) * p.kblk + b) * p.pitch + row] = s;
        uint32_t q[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float lo, hi;
            bf16x2_to_f32(w[i][j], lo, hi);
            q[j] = f8x2_from_f32(lo * inv, hi * inv);
        }
        if (k < p.Kp)
            *reinterpret_cast<uint2*>(p.q + (row * 4 + static_cast<int>(ci)) * p.Kp + k) =
                make_uint2(q[0] | (q[1] << 16), q[2] | (q[3] << 16));
    }
}

template <int GL>
cudaError_t launch_f8_rows(F8Rows r, cudaStream_t stream) {
    const int per_row = 4 * r.kblk, units = 256 / GL;
    r.group = per_row < units ? units / per_row : 1;
    const dim3 g(static_cast<unsigned>((r.rows + r.group * F8_ROWS_UNROLL - 1) /
                                       (r.group * F8_ROWS_UNROLL)),
                 static_cast<unsigned>((per_row + units - 1) / units));
    switch (load_channels(r.Kq, reinterpret_cast<uintptr_t>(r.x))) {
        case 8: return launch_pdl(f8_rows_kernel<GL, 8>, g, dim3(256), 0, stream, r);
        case 2: return launch_pdl(f8_rows_kernel<GL, 2>, g, dim3(256), 0, stream, r);
        default: return launch_pdl(f8_rows_kernel<GL, 1>, g, dim3(256), 0, stream, r);
    }
}

// Rows read back: a thread takes eight channels of a component of F8_DEQUANT_UNROLL rows, as above, all
// loads first.  The last rows go first: their writer has just left them in L2.  Bound by HBM: 1 byte
// read, 2 written a channel.  25,600 rows of 4096: 48 us, 6.5 TB/s (60 with 16 channels a thread, from
// the first rows on); 100,352 of 256: 14 us, 5.5 TB/s.
struct F8Dequant {
    const uint8_t* q;    // [rows][4][Kp]
    const float* scale;  // [4][kblk][pitch]
    __nv_bfloat16* out;  // [rows][4 Kq]
    long long rows, pitch;
    int Kq, Kp, kblk;
    int group;  // rows side by side in a block of threads
};

constexpr int F8_DEQUANT_UNROLL = 8;

__global__ void __launch_bounds__(256) f8_dequant_kernel(const F8Dequant p) {
    griddep_launch_dependents();
    griddep_wait();
    const unsigned units = p.Kq / 8, per_row = 4u * units;
    const unsigned unit = blockIdx.y * 256u + threadIdx.x;
    const unsigned r0 = unit / per_row, rest = unit - r0 * per_row;
    const unsigned ci = rest / units, k = (rest - ci * units) * 8;
    if (r0 >= static_cast<unsigned>(p.group)) return;
    const long long row0 = static_cast<long long>(gridDim.x - 1 - blockIdx.x) *
                               (p.group * F8_DEQUANT_UNROLL) + r0;
    const uint8_t* q = p.q + (row0 * 4 + ci) * p.Kp + k;
    const float* scale =
        p.scale + (static_cast<long long>(ci) * p.kblk + k / F8_BLOCK) * p.pitch + row0;
    __nv_bfloat16* out = p.out + row0 * (4LL * p.Kq) + static_cast<long long>(ci) * p.Kq + k;
    const int left = p.rows - row0 < p.group * F8_DEQUANT_UNROLL
                         ? static_cast<int>(p.rows - row0)
                         : p.group * F8_DEQUANT_UNROLL;
    uint2 w[F8_DEQUANT_UNROLL];
    float s[F8_DEQUANT_UNROLL];
#pragma unroll
    for (int i = 0; i < F8_DEQUANT_UNROLL; ++i)
        if (i * p.group < left) {
            w[i] = *reinterpret_cast<const uint2*>(q + static_cast<long long>(i * p.group) *
                                                           (4LL * p.Kp));
            s[i] = scale[i * p.group];
        }
#pragma unroll
    for (int i = 0; i < F8_DEQUANT_UNROLL; ++i)
        if (i * p.group < left) {
            float v[8], d[4];
            f8x4_to_f32(w[i].x, d);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = d[j] * s[i];
            f8x4_to_f32(w[i].y, d);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[4 + j] = d[j] * s[i];
            Raw<__nv_bfloat16, 8> o;
            o.set(v);
            o.store(out + static_cast<long long>(i * p.group) * (4LL * p.Kq));
        }
}

// The same of components that are not whole chunks of eight: eight elements of the output a thread,
// wherever rows and components begin, `group` rows (a multiple of eight) a column of blocks.  PAIR,
// components of eight channels or more: a thread's elements are a run of one component and perhaps the
// start of the next, which follows it in memory whatever row it is of, so that two loads of eight bytes
// hold the run and a third the start, shifted together; at most three scales.  Bound by its instructions (80%
// of the issue slots).  100,352 rows of 244:
// 22.5 us (39.7 by single bytes, eight rows a block); 4805 of 340: 3.0 (4.9); 401,408 of 20: 13.2 (51.9
// with blocks of eight rows, 20 threads of 256).
template <bool PAIR>
__global__ void __launch_bounds__(256) f8_dequant_any_kernel(const F8Dequant p) {
    griddep_launch_dependents();
    griddep_wait();
    const long long row0 = static_cast<long long>(gridDim.x - 1 - blockIdx.x) * p.group;
    const int rows = p.rows - row0 < p.group ? static_cast<int>(p.rows - row0) : p.group;
    const unsigned C = 4u * p.Kq, n = rows * C;
    __nv_bfloat16* out = p.out + row0 * C;
    const bool aligned = (reinterpret_cast<uintptr_t>(out) & 15u) == 0;
    for (unsigned f = 8u * (blockIdx.y * 256u + threadIdx.x); f < n; f += 8u * 256u * gridDim.y) {
        unsigned r = f / C, k = f - r * C, ci = k / p.Kq;
        k -= ci * p.Kq;
        const uint8_t* q = p.q + ((row0 + r) * 4 + ci) * p.Kp;
        float v[8];
        if constexpr (PAIR) {
            const float* scale = p.scale + row0 + r;
            const int run = p.Kq - k < 8u ? static_cast<int>(p.Kq - k) : 8;  // of this component
            const int block = F8_BLOCK - static_cast<int>(k % F8_BLOCK);     // of this scale
            const unsigned from = k & ~7u, bits = 8u * (k & 7u);
            using Eight = unsigned long long;
            Eight w = *reinterpret_cast<const Eight*>(q + from);
            Eight after = 0;
            if (bits && from + 8u < static_cast<unsigned>(p.Kp))
                after = *reinterpret_cast<const Eight*>(q + from + 8);
            const long long at = (static_cast<long long>(ci) * p.kblk + k / F8_BLOCK) * p.pitch;
            const float s0 = scale[at];
            float s1 = 0.0f, s2 = 0.0f;
            if (block < run) s1 = scale[at + p.pitch];
            Eight next = 0;
            if (f + run < n && run < 8) {
                next = *reinterpret_cast<const Eight*>(q + p.Kp);
                s2 = ci == 3 ? scale[1] : scale[static_cast<long long>(ci + 1) * p.kblk * p.pitch];
            }
            if (bits) w = (w >> bits) | (after << (64u - bits));
            if (run < 8) w = (w & ((1ull << (8 * run)) - 1)) | (next << (8 * run));
            float d[4];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                f8x4_to_f32(static_cast<uint32_t>(w >> (32 * i)), d);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    v[4 * i + j] = d[j] * (4 * i + j >= run ? s2 : 4 * i + j >= block ? s1 : s0);
            }
        } else {
            float s = 0.0f;
            bool fresh = true;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = 0.0f;
                if (f + j >= n) continue;
                if (fresh) s = p.scale[static_cast<long long>(ci) * p.pitch + row0 + r];
                v[j] = f8_to_f32(q[k]) * s;
                fresh = ++k == static_cast<unsigned>(p.Kq);
                if (fresh) {
                    k = 0;
                    q += p.Kp;
                    if (++ci == 4) ci = 0, ++r;
                }
            }
        }
        if (aligned && f + 8 <= n) {
            Raw<__nv_bfloat16, 8> o;
            o.set(v);
            o.store(out + f);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (f + j < n) out[f + j] = __float2bfloat16_rn(v[j]);
        }
    }
}

#include "qpoint_f8_tc.cuh"

int blocks_of(int q) { return (q + F8_BLOCK - 1) / F8_BLOCK; }

}  // namespace

int f8_pitch(int Kq) { return (Kq + 15) / 16 * 16; }

// Whole tiles of rows, so that a tile's scales are read without a bound (what stands past the rows is
// never used).
long long f8_scale_pitch(long long rows) { return (rows + F8_BM - 1) / F8_BM * F8_BM; }

cudaError_t launch_f8_dequant(const void* q, const float* scale, long long rows, int Kq, void* out,
                              cudaStream_t stream) {
    F8Dequant p = {static_cast<const uint8_t*>(q), scale, static_cast<__nv_bfloat16*>(out), rows,
                   f8_scale_pitch(rows), Kq, f8_pitch(Kq), blocks_of(Kq), 0};
    if (Kq % 8 != 0 || reinterpret_cast<uintptr_t>(out) % 16 != 0) {
        // 4096 elements or eight rows a column, 4096 elements a block
        p.group = Kq < 128 ? 8 * (128 / Kq) : 8;
        const dim3 g(static_cast<unsigned>((rows + p.group - 1) / p.group),
                     static_cast<unsigned>((static_cast<long long>(p.group) * 4 * Kq + 4095) / 4096));
        return Kq < 8 ? launch_pdl(f8_dequant_any_kernel<false>, g, dim3(256), 0, stream, p)
                      : launch_pdl(f8_dequant_any_kernel<true>, g, dim3(256), 0, stream, p);
    }
    const int per_row = Kq / 2;
    p.group = per_row < 256 ? 256 / per_row : 1;
    return launch_pdl(f8_dequant_kernel,
                      dim3(static_cast<unsigned>((rows + p.group * F8_DEQUANT_UNROLL - 1) /
                                                 (p.group * F8_DEQUANT_UNROLL)),
                           static_cast<unsigned>((per_row + 255) / 256)),
                      dim3(256), 0, stream, p);
}

cudaError_t launch_f8_letters(const void* const w[4], int Qout, int Qin, bool transpose, void* q,
                              float* scale, cudaStream_t stream) {
    F8Letters p;
    for (int L = 0; L < 4; ++L) p.w[L] = static_cast<const __nv_bfloat16*>(w[L]);
    p.rows = Qout;
    p.cols = Qin;
    p.q = static_cast<uint8_t*>(q);
    p.scale = scale;
    p.Kp = f8_pitch(transpose ? Qout : Qin);
    p.nblk = blocks_of(transpose ? Qin : Qout);
    p.kblk = blocks_of(transpose ? Qout : Qin);
    const dim3 g(static_cast<unsigned>(blocks_of(Qin)), static_cast<unsigned>(blocks_of(Qout)),
                 4);
    uintptr_t at = 0;
    for (int L = 0; L < 4; ++L) at |= reinterpret_cast<uintptr_t>(w[L]);
#define QUAN_LETTERS(LV)                                                                   \
    (transpose ? launch_pdl(f8_letters_kernel<true, LV>, g, dim3(256), 0, stream, p)       \
               : launch_pdl(f8_letters_kernel<false, LV>, g, dim3(256), 0, stream, p))
    switch (load_channels(Qin, at)) {
        case 8: return QUAN_LETTERS(8);
        case 2: return QUAN_LETTERS(2);
        default: return QUAN_LETTERS(1);
    }
#undef QUAN_LETTERS
}

namespace {

// The CUDA-core kernel: one row always, a few rows while their products are few.  Measured (us,
// CUDA cores and tensor cores with their quantisation): 1 row 512 -> 1024 2.1 and 5.2, 1 row
// 4096 -> 4096 5.6 and 17; 4 rows 4096 -> 4096 14.4 and 16.5, 8 rows 18.2 and 16.9; 8 rows
// 2048 -> 2048 8.3 and 10.4, 16 rows 11.0 and 10.3; 16 rows 512 -> 1024 5.5 and 5.7.
bool f8_few_rows(long long rows, int Kq, int Nq) {
    return rows == 1 || (rows <= 16 && rows * Kq * Nq <= (1 << 22));
}

size_t quantised_bytes(long long rows, int Kq) {
    return (static_cast<size_t>(rows) * 4 * f8_pitch(Kq) + 255) / 256 * 256;
}

// Quaternion output channels of a tile, by the estimated time of the waves of tiles (1280 rows
// 4096 -> 1024: 23.4, 18.8 and 25.3 us with 64, 32 and 16; 128 rows: 20.4, 15.9, 13.5; 20,000 rows
// 2048 -> 512: 54.3, 58.1, 70.7).
int f8_tile_width(long long rows, int Kq, int Nq, int num_sms) {
    // measured ns of a partial, and of a tile's beginning and end
    const int widths[3] = {64, 32, 16}, partial[3] = {456, 341, 272}, rest[3] = {2300, 1800, 950};
    int best = 64;
    double least = 0.0;
    // (below 32 rows the many CTAs of the narrowest tiles wait for the same few lines of x:
    // 24 rows 4096 -> 4096 26 us, 16.5 with 32 channels a tile)
    for (int i = 0; i < (rows < 32 ? 2 : 3); ++i) {
        const long long tiles = (rows + F8_BM - 1) / F8_BM * ((Nq + widths[i] - 1) / widths[i]);
        const long long waves = (tiles + num_sms - 1) / num_sms;
        const double t = static_cast<double>(waves) *
                         (4.0 * blocks_of(Kq) * partial[i] + rest[i]);
        if (i == 0 || t < least) best = widths[i], least = t;
    }
    return best;
}

template <int BNQ, bool SILU, bool AFFINE>
cudaError_t launch_f8_form(const CUtensorMap& mx, const CUtensorMap& mw, const F8TcParams& p,
                         int num_sms, cudaStream_t stream) {
    using C = F8Cfg<BNQ>;
    auto* kern = qpoint_f8_kernel<BNQ, SILU, AFFINE>;
    // once a device: the shared memory, and a look at the registers that the exchange counts on
    static std::atomic<unsigned long long> ready{0};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !((ready.load(std::memory_order_acquire) >> dev) & 1ull)) {
        cudaFuncAttributes a;
        if ((e = cudaFuncGetAttributes(&a, kern)) != cudaSuccess) return e;
        if (a.numRegs < F8_REGS) return cudaErrorInvalidKernelImage;
        e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 C::SMEM_BYTES);
        if (e != cudaSuccess) return e;
        if (dev < 64) ready.fetch_or(1ull << dev, std::memory_order_release);
    }
    const int grid = p.num_tiles < num_sms ? p.num_tiles : num_sms;
    return launch_pdl(kern, dim3(static_cast<unsigned>(grid)), dim3(F8_THREADS),
                      C::SMEM_BYTES, stream, mx, mw, p);
}

template <int BNQ>
cudaError_t launch_f8_tc(const CUtensorMap& mx, const CUtensorMap& mw, const F8TcParams& p,
                         int num_sms, cudaStream_t stream) {
    if (p.act == 2) return launch_f8_form<BNQ, true, true>(mx, mw, p, num_sms, stream);
    return p.ep.bias || p.ep.scale ? launch_f8_form<BNQ, false, true>(mx, mw, p, num_sms, stream)
                                   : launch_f8_form<BNQ, false, false>(mx, mw, p, num_sms, stream);
}

}  // namespace

size_t qpoint_f8_workspace_bytes(long long rows, int Kq, int Nq) {
    if (f8_few_rows(rows, Kq, Nq)) return 0;
    return quantised_bytes(rows, Kq) + static_cast<size_t>(f8_scale_pitch(rows)) * 4 * blocks_of(Kq) * 4;
}

cudaError_t launch_qpoint_f8(const void* x, const float* xscale, const void* wq, const float* ws,
                             const EpilogueArgs& ep, long long rows, int Kq, int Nq, bool conj,
                             int act, void* workspace, void* out, int num_sms,
                             unsigned long long wait_limit_ns, int inject_stall,
                             cudaStream_t stream, char* err, size_t errlen) {
    const int Kp = f8_pitch(Kq), kblk = blocks_of(Kq), nblk = blocks_of(Nq);
    const bool vec = Kq % 8 == 0 && reinterpret_cast<uintptr_t>(x) % 16 == 0;
    auto* xb = static_cast<const __nv_bfloat16*>(x);
    auto* ob = static_cast<__nv_bfloat16*>(out);
    const long long pitch = f8_scale_pitch(rows);
    if (f8_few_rows(rows, Kq, Nq)) {
        const F8Params p = {xscale ? nullptr : xb,
                            xscale ? static_cast<const uint8_t*>(x) : nullptr,
                            xscale, pitch, static_cast<const uint8_t*>(wq), ws, ep, ob, rows, Kq,
                            Nq, Kp, kblk, nblk, conj ? 1 : 0, act};
        return rows == 1 ? launch_rows<1>(p, vec, stream) : launch_rows<4>(p, vec, stream);
    }
    const void* xq = x;
    const float* xs = xscale;
    if (!xscale) {
        auto* q = static_cast<uint8_t*>(workspace);
        auto* s = reinterpret_cast<float*>(q + quantised_bytes(rows, Kq));
        const F8Rows r = {xb, q, s, rows, pitch, Kq, Kp, kblk, 0};
        const cudaError_t e = Kq <= 32   ? launch_f8_rows<4>(r, stream)
                              : Kq <= 64 ? launch_f8_rows<8>(r, stream)
                                         : launch_f8_rows<16>(r, stream);
        if (e != cudaSuccess) return e;
        xq = q;
        xs = s;
    }

    const int bnq = f8_tile_width(rows, Kq, Nq, num_sms);
    CUtensorMap mx, mw;
    const unsigned long long dx[3] = {static_cast<unsigned long long>(Kq), 4,
                                      static_cast<unsigned long long>(rows)};
    const unsigned long long sx[2] = {static_cast<unsigned long long>(Kp), 4ull * Kp};
    const unsigned bx[3] = {F8_BLOCK, 1, F8_BM};
    const unsigned long long dw[3] = {static_cast<unsigned long long>(Kq),
                                      static_cast<unsigned long long>(Nq), 4};
    const unsigned long long sw[2] = {static_cast<unsigned long long>(Kp),
                                      static_cast<unsigned long long>(Nq) * Kp};
    const unsigned bw[3] = {F8_BLOCK, static_cast<unsigned>(bnq), 4};
    if (!encode_bytes_3d(&mx, xq, dx, sx, bx) || !encode_bytes_3d(&mw, wq, dw, sw, bw)) {
        snprintf(err, errlen, "cuTensorMapEncodeTiled failed for the 8-bit tensors");
        return cudaErrorInvalidValue;
    }
    F8TcParams p = {};
    p.xs = xs;
    p.ws = ws;
    p.ep = ep;
    p.out = ob;
    p.rows = rows;
    p.pitch = pitch;
    p.Kq = Kq;
    p.Nq = Nq;
    p.kblk = kblk;
    p.nblk = nblk;
    p.conj = conj ? 1 : 0;
    p.act = act;
    p.ntiles = (Nq + bnq - 1) / bnq;
    p.num_tiles = static_cast<int>((rows + F8_BM - 1) / F8_BM * p.ntiles);
    const uintptr_t a = reinterpret_cast<uintptr_t>(out);
    p.store = Nq % 16 == 0 && a % 32 == 0  ? F8_STORE_SECTOR
              : Nq % 8 == 0 && a % 16 == 0 ? F8_STORE_16
              : Nq % 2 == 0 && a % 4 == 0  ? F8_STORE_4
                                           : F8_STORE_2;
    p.wait_limit_ns = wait_limit_ns;
    p.inject_stall = inject_stall;
    switch (bnq) {
        case 64: return launch_f8_tc<64>(mx, mw, p, num_sms, stream);
        case 32: return launch_f8_tc<32>(mx, mw, p, num_sms, stream);
        default: return launch_f8_tc<16>(mx, mw, p, num_sms, stream);
    }
}

cudaError_t read_and_clear_status_f8(unsigned* status, cudaStream_t stream) {
    cudaError_t e = cudaMemcpyFromSymbolAsync(status, g_status, sizeof(unsigned), 0,
                                              cudaMemcpyDeviceToHost, stream);
    if (e != cudaSuccess) return e;
    e = cudaStreamSynchronize(stream);
    if (e != cudaSuccess) return e;
    const unsigned zero = 0;
    e = cudaMemcpyToSymbolAsync(g_status, &zero, sizeof(unsigned), 0, cudaMemcpyHostToDevice,
                                stream);
    if (e != cudaSuccess) return e;
    return cudaStreamSynchronize(stream);
}

}  // namespace quan
