// qpoint_w4.cu -- the pointwise (1x1) quaternion convolution of a few pixels with letters in 4 bits.
//
// A group is `group` (32, 64 or 128) input channels of one output channel of one letter: its scale s is
// max |v| / 7 rounded to bf16 (1 where that is 0; NaN where the group holds an infinity or a NaN, so
// that everything computed from it is NaN), its values q = v / s rounded to a whole number in -7 .. 7.
// With L = co xor ci and sgn Eq. 6's signs,
//   out[m][co][n] = sum over ci, groups b of  sgn(co, ci) s[L][n][b] sum over k in b of q[L][n][k] x[m][ci][k].
// bf16 holds q and x exactly and the tensor cores add their products in fp32; a group's sum is
// multiplied by its scale in fp32, so nothing is rounded to fewer bits but the output.
//
// Bound by the letters' bytes (half a byte for the four products that a letter's element has a row), and
// with one pixel by the trip to memory.  A warp-level MMA (m16n8k16) takes 16 output channels of one
// letter as its rows; its 8 columns are the four output components of two pixels, column (m, co)
// holding component co xor L of pixel m with Eq. 6's sign.  So an element of a letter is read and
// widened once for all four components, and the quaternion product needs no other arithmetic.
//
// Device time: one pixel 512 -> 1024 1.7 us; 8192 -> 8192 8.3 us with the letters in memory (8.9 MB with
// their scales: 1.3 us at HBM's rate), 7.1 with them in L2; 49 pixels 2048 -> 2048 8.1 us (8.5 with SiLU and
// vectors), 13 pixels 1172 -> 2804 6.3 us.  At 8192 -> 8192 clusters of four blocks share a tile's inputs:
// 512 blocks with 98 registers a thread, 304 at once, so that a second wave's letters wait for the
// first's joins.  Other clusters there, from memory and L2: one block 9.5 and 8.2, two 6.7 and 5.5, eight
// 13.2 and 11.4.
//
// Layout of the letters: [L][16 output channels][64 input channels] blocks of 512 bytes, a lane's 16
// bytes side by side: word s of lane 4 g + t has q + 8 of channels g and g + 8, inputs
// k = 32 (s / 2) + 8 t + 4 (s mod 2) + 0 .. 3, so that a lane's inputs of a block are two runs of eight.
// Nibble i, i < 4, is (g + 8 (i mod 2), k + 2 (i / 2)), nibble i + 4 its neighbour in k: one mask gives
// a register of the MMA.  Scales: bf16 [L][16 output channels][group][g][g or g + 8].
//
// Inputs are read with plain loads only, behind the wait for the grid before this one.
#include <cuda_bf16.h>

#include <atomic>

#include "f8.cuh"
#include "internal.h"
#include "ptx.cuh"
#include "tc_common.cuh"
#include "vec_io.cuh"

namespace quan {
namespace {

constexpr int W4_TILE_N = 16, W4_TILE_K = 64, W4_BLOCK_BYTES = 512;

// Channels a load may take of rows of n channels at `address`.
int load_channels(int n, uintptr_t address) {
    return n % 8 == 0 && address % 16 == 0 ? 8 : (n % 2 == 0 && address % 4 == 0 ? 2 : 1);
}

// Eight consecutive bf16 channels as words, LV channels a load; `left` of them exist, a multiple of LV
// where LV > 1, the others are 0.
template <int LV>
__device__ __forceinline__ void load_words8(const __nv_bfloat16* p, int left, uint32_t* w) {
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
                w[j / 2] |= static_cast<uint32_t>(reinterpret_cast<const unsigned short*>(p)[j])
                            << (16 * (j & 1));
    }
}

// ------------------------------------------------------------------ letters

struct W4Letters {
    const __nv_bfloat16* w[4];  // [Qo][Qi]
    int Qo, Qi, group, groups;  // groups: of a row
    uint32_t* q;
    __nv_bfloat16* scale;
    int ntiles, ktiles;
};

// 16 output x 128 input channels of one letter a block: a thread has eight inputs of one output, 4, 8
// or 16 threads a group; the values meet in shared memory and leave as the product reads them.
template <int LV>
__global__ void __launch_bounds__(256) w4_letters_kernel(const W4Letters p) {
    __shared__ uint8_t tile[16][128];
    griddep_launch_dependents();
    griddep_wait();
    const int letter = blockIdx.z, nt = blockIdx.y, k0 = blockIdx.x * 128;
    const int r = threadIdx.x >> 4, k = k0 + (threadIdx.x & 15) * 8, n = nt * 16 + r;
    uint32_t w[4], m = 0;
    load_words8<LV>(p.w[letter] + static_cast<long long>(n) * p.Qi + k,
                    n < p.Qo ? p.Qi - k : 0, w);
#pragma unroll
    for (int j = 0; j < 4; ++j) m = __vmaxu2(m, w[j] & 0x7FFF7FFFu);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1)
        if (8 * o < p.group) m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, o));
    m = max(m << 16, m & 0xFFFF0000u);
    float s = __bfloat162float(__float2bfloat16_rn(__uint_as_float(m) / 7.0f));
    if (s == 0.0f) s = 1.0f;
    const bool bad = m >= 0x7F800000u;
    if (bad) s = __uint_as_float(0x7FC00000u);
    if (k % p.group == 0 && k / p.group < p.groups)
        p.scale[((static_cast<long long>(letter) * p.ntiles + nt) * p.groups + k / p.group) * 16 +
                2 * (r & 7) + (r >> 3)] = __float2bfloat16_rn(s);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float v[2];
        bf16x2_to_f32(w[j], v[0], v[1]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float q = fminf(fmaxf(rintf(v[i] / s), -7.0f), 7.0f);
            tile[r][(threadIdx.x & 15) * 8 + 2 * j + i] =
                static_cast<uint8_t>(bad ? 8 : static_cast<int>(q) + 8);
        }
    }
    __syncthreads();
    {
        const int kt = threadIdx.x >> 7, lane = (threadIdx.x >> 2) & 31, step = threadIdx.x & 3;
        const int g = lane >> 2, t = lane & 3, ktile = blockIdx.x * 2 + kt;
        const int at = kt * 64 + 32 * (step >> 1) + 8 * t + 4 * (step & 1);
        uint32_t word = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            word |= static_cast<uint32_t>(tile[g + 8 * (i & 1)][at + 2 * ((i & 3) >> 1) + (i >> 2)])
                    << (4 * i);
        if (ktile < p.ktiles)
            p.q[(((static_cast<long long>(letter) * p.ntiles + nt) * p.ktiles + ktile) * 32 + lane) *
                    4 + step] = word;
    }
}

// ------------------------------------------------------------------ the product

struct W4Params {
    const __nv_bfloat16* x;  // [rows][4 Qi]
    const uint4* q;
    const uint32_t* scale;  // pairs of bf16
    EpilogueArgs ep;
    __nv_bfloat16* out;  // [rows][4 Qo]
    long long rows;
    int Qi, Qo, ntiles, ktiles, groups, act;
    int wide;   // 1 for groups of 128
    int split;  // blocks of a cluster that share a tile's inputs
};

__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0,
                                         uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, "
        "{%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Eight 4-bit values as the registers of an MMA: 128 + (q + 8) by its bits, less 136 (exact).
__device__ __forceinline__ void widen(uint32_t w, uint32_t (&a)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t u = ((w >> (4 * i)) & 0x000F000Fu) | 0x43004300u;
        asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(a[i]) : "r"(u), "r"(0x43084308u));
    }
}

constexpr int W4_WARPS = 8;

// The warps' sums, and the cluster's, in a fixed order, and the output.  `part`: a row of NT x 128 values
// a warp, element e of a tile's 16 x 8 being channel e mod 16 of column e / 16.
template <int NT>
__device__ __forceinline__ void w4_finish(const W4Params& p, float (&acc)[NT][4],
                                          float (*part)[NT * 128], int rank, int nt,
                                          long long row0) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            part[warp][j * 128 + (2 * t + (e & 1)) * 16 + g + 8 * (e >> 1)] = acc[j][e];
    __syncthreads();
    constexpr int MINE = (NT * 128 + 32 * W4_WARPS - 1) / (32 * W4_WARPS);
    float sum[MINE];
#pragma unroll
    for (int e = 0; e < MINE; ++e) {
        const int at = threadIdx.x + e * 32 * W4_WARPS;
        sum[e] = 0.0f;
        if (at < NT * 128) {
#pragma unroll
            for (int w = 0; w < W4_WARPS; ++w) sum[e] += part[w][at];
        }
    }
    if (p.split > 1) {
        cluster_sync_all();  // the first block has read what the others write over
        if (rank > 0) {
#pragma unroll
            for (int e = 0; e < MINE; ++e) {
                const int at = threadIdx.x + e * 32 * W4_WARPS;
                if (at < NT * 128)
                    st_shared_cluster(mapa_shared(smem_u32(&part[rank][at]), 0),
                                      __float_as_uint(sum[e]));
            }
        }
        cluster_sync_all();
        if (rank > 0) return;
#pragma unroll
        for (int e = 0; e < MINE; ++e) {
            const int at = threadIdx.x + e * 32 * W4_WARPS;
            if (at < NT * 128)
                for (int r = 1; r < p.split; ++r) sum[e] += part[r][at];
        }
    }
#pragma unroll
    for (int e = 0; e < MINE; ++e) {
        const int at = threadIdx.x + e * 32 * W4_WARPS;
        const int n = nt * 16 + (at & 15), column = at >> 4;
        const long long row = row0 + (column >> 2);
        if (at >= NT * 128 || n >= p.Qo || row >= p.rows) continue;
        const int c = (column & 3) * p.Qo + n;
        float v = sum[e];
        if (p.ep.bias) v += p.ep.bias[c];
        if (p.ep.scale) v = fmaf(p.ep.scale[c], v, p.ep.shift[c]);
        p.out[row * (4LL * p.Qo) + c] = __float2bfloat16_rn(f8_act(v, p.act));
    }
}

// 16 output channels and 2 NT pixels a block, or a cluster that splits the inputs.  A warp takes a
// letter's block of 64 inputs at a time.
template <int NT, bool G32>
__global__ void __launch_bounds__(32 * W4_WARPS) qpoint_w4_kernel(const W4Params p) {
    __shared__ float part[W4_WARPS][NT * 128];
    griddep_launch_dependents();
    griddep_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const unsigned tile = blockIdx.x / static_cast<unsigned>(p.split);
    const int rank = static_cast<int>(blockIdx.x - tile * p.split), nt = blockIdx.y;
    const long long row0 = static_cast<long long>(tile) * (2 * NT);
    // this lane's column of an MMA: pixel and output component
    const int co = g & 3;
    float acc[NT][4] = {};
    const int items = 4 * p.ktiles, per = (items + p.split - 1) / p.split;
    const int end = (rank + 1) * per < items ? (rank + 1) * per : items;
    constexpr int U = NT == 1 ? 4 : 2;  // blocks whose loads go out together
    for (int i0 = rank * per + warp; i0 < end; i0 += U * W4_WARPS) {
        uint4 q[U];
        uint32_t s[U][2], x[U][NT][8];
        auto load_x = [&](int i, int j, uint32_t (&w)[8]) {
            const int L = i & 3, k = (i >> 2) * W4_TILE_K + 8 * t, ci = co ^ L;
            const long long row = row0 + 2 * j + (g >> 2);
            const uint32_t neg = (tc::NEG_MASK >> (4 * co + ci)) & 1u ? 0x80008000u : 0u;
            const __nv_bfloat16* src =
                p.x + row * (4LL * p.Qi) + static_cast<long long>(ci) * p.Qi + k;
            const int left = row < p.rows ? p.Qi - k : 0;
            load_words8<8>(src, left, w);
            load_words8<8>(src + 32, left - 32, w + 4);
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] ^= neg;
        };
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * W4_WARPS;
            if (i >= end) break;
            const int L = i & 3, kt = i >> 2;
            const long long block = (static_cast<long long>(L) * p.ntiles + nt) * p.ktiles + kt;
            q[u] = p.q[block * 32 + lane];
            const uint32_t* sc = p.scale + (static_cast<long long>(L) * p.ntiles + nt) * p.groups * 8;
            // (64 inputs are two groups of 32, one of 64 or half of one of 128)
            if constexpr (G32) {
                s[u][0] = sc[2 * kt * 8 + g];
                s[u][1] = 2 * kt + 1 < p.groups ? sc[(2 * kt + 1) * 8 + g] : 0u;
            } else {
                s[u][0] = sc[(kt >> p.wide) * 8 + g];
            }
#pragma unroll
            for (int j = 0; j < NT; ++j) load_x(i, j, x[u][j]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * W4_WARPS;
            if (i >= end) break;
            uint32_t a[4][4];
            widen(q[u].x, a[0]);
            widen(q[u].y, a[1]);
            widen(q[u].z, a[2]);
            widen(q[u].w, a[3]);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const uint32_t(&b)[8] = x[u][j];
#pragma unroll
                for (int h = 0; h < (G32 ? 2 : 1); ++h) {
                    float c[4] = {};
#pragma unroll
                    for (int e = 0; e < (G32 ? 2 : 4); ++e)
                        mma_bf16(c, a[2 * h + e], b[4 * h + 2 * e], b[4 * h + 2 * e + 1]);
                    float lo, hi;
                    bf16x2_to_f32(s[u][h], lo, hi);
                    acc[j][0] = fmaf(lo, c[0], acc[j][0]);
                    acc[j][1] = fmaf(lo, c[1], acc[j][1]);
                    acc[j][2] = fmaf(hi, c[2], acc[j][2]);
                    acc[j][3] = fmaf(hi, c[3], acc[j][3]);
                }
            }
        }
    }
    w4_finish<NT>(p, acc, part, rank, nt, row0);
}

// The same with the pixels' channels staged in shared memory, KT blocks of 64 inputs at a time: for
// more pixels than fit a lane's registers, and where their channels cannot be loaded eight at a time.
// Components of pixels stand 64 bytes past a multiple of 128 apart, so that the two that a quarter of a
// warp reads lie in different banks.  49 rows 2048 -> 2048: 12.4 us with loads of their own for every
// MMA, whose trips to L2 added up.
template <int NT>
struct W4Stage {
    static constexpr int KT = NT >= 8 ? 8 : NT == 4 ? 16 : 32;
    static constexpr int PITCH = KT * W4_TILE_K * 2 + 64;  // bytes of a component
    static constexpr int BYTES = 2 * NT * 4 * PITCH;
};

template <int NT, int LV, bool G32>
__global__ void __launch_bounds__(32 * W4_WARPS) qpoint_w4_staged_kernel(const W4Params p) {
    using S = W4Stage<NT>;
    static_assert(S::BYTES >= W4_WARPS * NT * 128 * 4, "the warps' sums take the stage's place");
    extern __shared__ int4 stage[];
    griddep_launch_dependents();
    griddep_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const unsigned tile = blockIdx.x / static_cast<unsigned>(p.split);
    const int rank = static_cast<int>(blockIdx.x - tile * p.split), nt = blockIdx.y;
    const long long row0 = static_cast<long long>(tile) * (2 * NT);
    const int co = g & 3, per = (p.ktiles + p.split - 1) / p.split;
    const int last = (rank + 1) * per < p.ktiles ? (rank + 1) * per : p.ktiles;
    char* xs = reinterpret_cast<char*>(stage);
    float acc[NT][4] = {};
    constexpr int U = 4;  // blocks of letters whose loads go out together
    for (int k0 = rank * per; k0 < last; k0 += S::KT) {
        const int kts = last - k0 < S::KT ? last - k0 : S::KT, items = 4 * kts;
        uint4 q[U];
        uint32_t s[U][2];
        auto letters = [&](int first) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = first + u * W4_WARPS;
                if (i >= items) break;
                const int L = i & 3, kt = k0 + (i >> 2);
                const long long block = (static_cast<long long>(L) * p.ntiles + nt) * p.ktiles + kt;
                q[u] = p.q[block * 32 + lane];
                const uint32_t* sc =
                    p.scale + (static_cast<long long>(L) * p.ntiles + nt) * p.groups * 8;
                if constexpr (G32) {
                    s[u][0] = sc[2 * kt * 8 + g];
                    s[u][1] = 2 * kt + 1 < p.groups ? sc[(2 * kt + 1) * 8 + g] : 0u;
                } else {
                    s[u][0] = sc[(kt >> p.wide) * 8 + g];
                }
            }
        };
        letters(warp);
        // the pixels' channels of these blocks, eight a thread, 0 past the last
        for (int i = threadIdx.x; i < 2 * NT * 4 * 8 * kts; i += 32 * W4_WARPS) {
            const int c = i / (8 * kts), k = (i - c * 8 * kts) * 8;  // component of a pixel
            const long long row = row0 + (c >> 2);
            const int at = k0 * W4_TILE_K + k, left = row < p.rows ? p.Qi - at : 0;
            const __nv_bfloat16* src =
                p.x + row * (4LL * p.Qi) + static_cast<long long>(c & 3) * p.Qi + at;
            uint32_t w[4];
            load_words8<LV>(src, left, w);
            *reinterpret_cast<uint4*>(xs + c * S::PITCH + k * 2) =
                make_uint4(w[0], w[1], w[2], w[3]);
        }
        __syncthreads();
        for (int i0 = warp; i0 < items; i0 += U * W4_WARPS) {
            if (i0 != warp) letters(i0);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * W4_WARPS;
                if (i >= items) break;
                const int L = i & 3, ci = co ^ L;
                const uint32_t neg = (tc::NEG_MASK >> (4 * co + ci)) & 1u ? 0x80008000u : 0u;
                const char* at = xs + ((g >> 2) * 4 + ci) * S::PITCH + (i >> 2) * 128 + 16 * t;
                uint32_t a[4][4];
                widen(q[u].x, a[0]);
                widen(q[u].y, a[1]);
                widen(q[u].z, a[2]);
                widen(q[u].w, a[3]);
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const uint4 b0 = *reinterpret_cast<const uint4*>(at + j * 8 * S::PITCH);
                    const uint4 b1 = *reinterpret_cast<const uint4*>(at + j * 8 * S::PITCH + 64);
                    const uint32_t b[8] = {b0.x ^ neg, b0.y ^ neg, b0.z ^ neg, b0.w ^ neg,
                                           b1.x ^ neg, b1.y ^ neg, b1.z ^ neg, b1.w ^ neg};
#pragma unroll
                    for (int h = 0; h < (G32 ? 2 : 1); ++h) {
                        float c[4] = {};
#pragma unroll
                        for (int e = 0; e < (G32 ? 2 : 4); ++e)
                            mma_bf16(c, a[2 * h + e], b[4 * h + 2 * e], b[4 * h + 2 * e + 1]);
                        float lo, hi;
                        bf16x2_to_f32(s[u][h], lo, hi);
                        acc[j][0] = fmaf(lo, c[0], acc[j][0]);
                        acc[j][1] = fmaf(lo, c[1], acc[j][1]);
                        acc[j][2] = fmaf(hi, c[2], acc[j][2]);
                        acc[j][3] = fmaf(hi, c[3], acc[j][3]);
                    }
                }
            }
        }
        __syncthreads();  // before the stage is filled again
    }
    w4_finish<NT>(p, acc, reinterpret_cast<float(*)[NT * 128]>(stage), rank, nt, row0);
}

template <int NT, int LV, bool G32>
cudaError_t launch_w4_form(W4Params p, int num_sms, cudaStream_t stream) {
    // staged for more than four pixels, or channels that are not loaded eight at a time
    constexpr bool STAGED = NT > 2 || LV != 8;
    const long long tiles = (p.rows + 2 * NT - 1) / (2 * NT);
    // the inputs are split in two, and again, while the blocks are fewer than the SMs (without a stage,
    // than two an SM) and a warp keeps two blocks of letters
    p.split = 1;
    while (p.split < 8 && tiles * p.ntiles * p.split < (STAGED ? 1 : 2) * num_sms &&
           4 * p.ktiles >= 4 * W4_WARPS * p.split)
        p.split *= 2;
    const dim3 g(static_cast<unsigned>(tiles * p.split), static_cast<unsigned>(p.ntiles));
    const unsigned cluster = static_cast<unsigned>(p.split);
    if constexpr (STAGED) {
        constexpr int BYTES = W4Stage<NT>::BYTES;
        auto* kern = qpoint_w4_staged_kernel<NT, LV, G32>;
        static std::atomic<unsigned long long> ready{0};  // once a device: the shared memory
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        if (dev >= 64 || !((ready.load(std::memory_order_acquire) >> dev) & 1ull)) {
            e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, BYTES);
            if (e != cudaSuccess) return e;
            if (dev < 64) ready.fetch_or(1ull << dev, std::memory_order_release);
        }
        return launch_pdl_cluster(kern, g, dim3(32 * W4_WARPS), cluster, BYTES, stream, p);
    } else {
        return launch_pdl_cluster(qpoint_w4_kernel<NT, G32>, g, dim3(32 * W4_WARPS), cluster, 0,
                                  stream, p);
    }
}

template <int NT>
cudaError_t launch_w4_nt(const W4Params& p, bool g32, int num_sms, cudaStream_t stream) {
    switch (load_channels(p.Qi, reinterpret_cast<uintptr_t>(p.x))) {
        case 8: return g32 ? launch_w4_form<NT, 8, true>(p, num_sms, stream)
                           : launch_w4_form<NT, 8, false>(p, num_sms, stream);
        case 2: return g32 ? launch_w4_form<NT, 2, true>(p, num_sms, stream)
                           : launch_w4_form<NT, 2, false>(p, num_sms, stream);
        default: return g32 ? launch_w4_form<NT, 1, true>(p, num_sms, stream)
                            : launch_w4_form<NT, 1, false>(p, num_sms, stream);
    }
}

int tiles_of(int n, int tile) { return (n + tile - 1) / tile; }

}  // namespace

size_t w4_bytes(int Qi, int Qo) {
    return size_t(4) * tiles_of(Qo, W4_TILE_N) * tiles_of(Qi, W4_TILE_K) * W4_BLOCK_BYTES;
}

size_t w4_scales(int Qi, int Qo, int group) {
    return size_t(4) * tiles_of(Qo, W4_TILE_N) * tiles_of(Qi, group) * 16;
}

cudaError_t launch_w4_letters(const void* const w[4], int Qo, int Qi, int group, void* q,
                              void* scale, cudaStream_t stream) {
    W4Letters p;
    uintptr_t at = 0;
    for (int L = 0; L < 4; ++L) {
        p.w[L] = static_cast<const __nv_bfloat16*>(w[L]);
        at |= reinterpret_cast<uintptr_t>(w[L]);
    }
    p.Qo = Qo;
    p.Qi = Qi;
    p.group = group;
    p.groups = tiles_of(Qi, group);
    p.q = static_cast<uint32_t*>(q);
    p.scale = static_cast<__nv_bfloat16*>(scale);
    p.ntiles = tiles_of(Qo, W4_TILE_N);
    p.ktiles = tiles_of(Qi, W4_TILE_K);
    const dim3 g(static_cast<unsigned>(tiles_of(Qi, 128)), static_cast<unsigned>(p.ntiles), 4);
    switch (load_channels(Qi, at)) {
        case 8: return launch_pdl(w4_letters_kernel<8>, g, dim3(256), 0, stream, p);
        case 2: return launch_pdl(w4_letters_kernel<2>, g, dim3(256), 0, stream, p);
        default: return launch_pdl(w4_letters_kernel<1>, g, dim3(256), 0, stream, p);
    }
}

cudaError_t launch_qpoint_w4(const void* x, const void* q, const void* scale,
                             const EpilogueArgs& ep, long long rows, int Qi, int Qo, int group,
                             int act, void* out, int num_sms, cudaStream_t stream) {
    const W4Params p = {static_cast<const __nv_bfloat16*>(x), static_cast<const uint4*>(q),
                        static_cast<const uint32_t*>(scale), ep, static_cast<__nv_bfloat16*>(out),
                        rows, Qi, Qo, tiles_of(Qo, W4_TILE_N), tiles_of(Qi, W4_TILE_K),
                        tiles_of(Qi, group), act, group == 128 ? 1 : 0, 1};
    const bool g32 = group == 32;
    return rows <= 2   ? launch_w4_nt<1>(p, g32, num_sms, stream)
           : rows <= 4 ? launch_w4_nt<2>(p, g32, num_sms, stream)
           : rows <= 8 ? launch_w4_nt<4>(p, g32, num_sms, stream)
                       : launch_w4_nt<8>(p, g32, num_sms, stream);
}

}  // namespace quan
