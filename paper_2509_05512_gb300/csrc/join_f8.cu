// join_f8.cu -- the residual join whose norm comes out in 8 bits (residual.cu has the formulas and the
// form for any rows), for rows whose components are whole chunks of eight channels, 16-byte aligned.
//
// A row's components lie on TPS lanes each whatever its statistics are, so a block of 128 is a run of
// neighbouring lanes.  With a statistic for each component a lane has eight channels, and sums are
// taken in residual_join's order: the same bits.  With one for the row (WHOLE) it has 16, which halves
// the exchange between lanes.  R rows a thread are under way together, the next R loaded ahead.
// Everything elementwise goes by twos (f32x2), rounded as one by one.
//
// Bound by HBM beside the instructions of reductions and conversions.  32 x 56 x 56 x 256 bf16, a
// statistic a component: 33 us, 5.4 TB/s (39 by residual.cu's form).  The norm of 25,600 rows of 4096,
// a statistic a row: 58 us, 5.4 TB/s (138; 103 with eight channels a lane and 64-bit indexes).
#include <cuda_bf16.h>

#include <atomic>

#include "f8.cuh"
#include "internal.h"
#include "pairs.cuh"
#include "residual.cuh"

namespace quan {
namespace {

// The join's form for a component of up to 8 CPT TPS channels.
template <int TPS, bool WHOLE>
struct JoinF8Cfg {
    static constexpr int CPT = WHOLE ? 2 : 1;  // chunks a lane
    static constexpr int LANES = 4 * TPS;      // of a row
    static constexpr int RED = WHOLE ? LANES : TPS;
    static constexpr int THREADS = LANES > 256 ? LANES : 256;
    static constexpr int SLOTS = THREADS / LANES;
};

// Sums over the RED lanes of a statistic, as group_sum orders them.
template <int TPS, bool WHOLE, int R>
__device__ __forceinline__ void statistic(float (&v)[R], float (*both)[R][32], int& turn) {
    using C = JoinF8Cfg<TPS, WHOLE>;
    constexpr int LOW = C::RED < 32 ? C::RED : 32;
#pragma unroll
    for (int o = LOW / 2; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < R; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    if constexpr (C::RED > 32) {
        constexpr int WPS = C::RED / 32;  // warps of a statistic
        float(*sm)[32] = both[turn];
        turn ^= 1;
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        if (lane == 0) {
#pragma unroll
            for (int i = 0; i < R; ++i) sm[i][warp] = v[i];
        }
        __syncthreads();
        const int at = (warp & ~(WPS - 1)) + (lane & (WPS - 1));
#pragma unroll
        for (int i = 0; i < R; ++i) v[i] = sm[i][at];
#pragma unroll
        for (int o = WPS / 2; o > 0; o >>= 1)
#pragma unroll
            for (int i = 0; i < R; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    }
}

template <typename T, int TPS, bool WHOLE, bool BRANCH, int R>
__global__ void __launch_bounds__(JoinF8Cfg<TPS, WHOLE>::THREADS)
    join_f8_kernel(const JoinParams p) {
    using C = JoinF8Cfg<TPS, WHOLE>;
    constexpr int CPT = C::CPT, V = 8 * CPT;                       // channels a lane
    constexpr int GL = TPS * CPT < 16 ? TPS : 16 / CPT;            // lanes of a block of 128
    __shared__ float sm[2][R][32];
    int turn = 0;
    griddep_launch_dependents();
    griddep_wait();
    const int slot = threadIdx.x / C::LANES, seg = threadIdx.x / TPS % 4, ts = threadIdx.x % TPS;
    const int col = ts * V, rows = static_cast<int>(p.rows);
    float pg[V], pre[V];
    // a lane's share of a per-channel vector
    auto columns = [&](const float* v, float scale, float (&out)[V]) {
#pragma unroll
        for (int j = 0; j < V; ++j)
            out[j] = (v && col + j < p.S) ? scale * ld_global_f32(v + seg * p.S + col + j) : scale;
    };
    auto load_gate = [&](int image) {
        float post[V];
        columns(p.post, p.alpha * p.drop.factor, post);
        columns(p.gate ? p.gate + static_cast<long long>(image) * p.C : nullptr, 1.0f, pg);
#pragma unroll
        for (int j = 0; j < V; ++j) pg[j] *= post[j];
    };
    if (BRANCH) load_gate(0);
    columns(p.pre, 1.0f, pre);
    const unsigned long long base = BRANCH && p.drop.draws ? dropout_base(p.drop) : 0ull;
    const T *x = static_cast<const T*>(p.x), *h = static_cast<const T*>(p.h);
    T* y = static_cast<T*>(p.out_y);
    __nv_bfloat16* n = static_cast<__nv_bfloat16*>(p.out_n);
    float* scale = p.s8 + (static_cast<long long>(seg) * p.kblk + col / F8_BLOCK) * p.s8_pitch;
    // a lane's first chunk of eight of a row, counted over the tensor, and of its 8-bit row
    const unsigned row_chunks = p.C / 8, row_q = 4 * p.q8_pitch / 8;
    const unsigned mine = (seg * p.S + col) / 8, mine_q = (seg * p.q8_pitch + col) / 8;
    const int step = gridDim.x * (C::SLOTS * R);
    Raw<T, 8> nx[R][CPT], nh[R][CPT];
    auto fetch = [&](int r0) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int row = r0 + i * C::SLOTS;
            const unsigned at = row * row_chunks + mine;
#pragma unroll
            for (int c = 0; c < CPT; ++c) {
                if (row < rows && col + 8 * c < p.S) {
                    nx[i][c].load(x + 8ull * (at + c));
                    if (BRANCH) nh[i][c].load(h + 8ull * (at + c));
                } else {
                    nx[i][c].zero();
                    if (BRANCH) nh[i][c].zero();
                }
            }
        }
    };
    auto values = [](const Raw<T, 8>(&r)[CPT], float (&v)[V]) {
#pragma unroll
        for (int c = 0; c < CPT; ++c) {
            float w[8];
            r[c].values(w);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[8 * c + j] = w[j];
        }
    };
    // v *= f w
    auto scaled = [](float (&v)[V], float f, const float (&w)[V]) {
        const float2 ff = make_float2(f, f);
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            const float2 r = mul2(make_float2(v[j], v[j + 1]),
                                  mul2(ff, make_float2(w[j], w[j + 1])));
            v[j] = r.x, v[j + 1] = r.y;
        }
    };
    const int rows_per_image = static_cast<int>(p.rows_per_image);
    int row0 = blockIdx.x * (C::SLOTS * R) + slot;
    int image_end = BRANCH && p.gate ? rows_per_image : rows;
    fetch(row0);
    // (rows < 2^31 - step, so that no index passes an int)
    for (; row0 - slot < rows; row0 += step) {
        float v[R][V], u[R][V];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            values(nx[i], v[i]);
            if (BRANCH) values(nh[i], u[i]);
        }
        fetch(row0 + step);
        if constexpr (BRANCH) {
            float r1[R];
#pragma unroll
            for (int i = 0; i < R; ++i) r1[i] = 0.0f;
            if (p.post) {
#pragma unroll
                for (int i = 0; i < R; ++i)
#pragma unroll
                    for (int j = 0; j < V; ++j) r1[i] = fmaf(u[i][j], u[i][j], r1[i]);
                statistic<TPS, WHOLE, R>(r1, sm, turn);
            }
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const int row = row0 + i * C::SLOTS;
                r1[i] = p.post ? rsqrtf(fmaf(r1[i], p.inv_s, p.eps)) : 1.0f;
                if (row >= image_end && row < rows) {
                    const int image = row / rows_per_image;
                    image_end = (image + 1) * rows_per_image;
                    load_gate(image);
                }
                const unsigned at = row * row_chunks + mine;
                scaled(u[i], r1[i], pg);
                if (p.drop.draws) {
#pragma unroll
                    for (int c = 0; c < CPT; ++c) {
                        Dropout8 m;
                        m.draw(p.drop, base + at + c);
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            u[i][8 * c + j] = m.keep(p.drop, j) ? u[i][8 * c + j] : 0.0f;
                    }
                } else if (p.drop.bound != 0) {  // nothing is kept
#pragma unroll
                    for (int j = 0; j < V; ++j) u[i][j] = 0.0f;
                }
#pragma unroll
                for (int j = 0; j < V; j += 2) {
                    const float2 r = add2(make_float2(v[i][j], v[i][j + 1]),
                                          make_float2(u[i][j], u[i][j + 1]));
                    v[i][j] = r.x, v[i][j + 1] = r.y;
                }
#pragma unroll
                for (int c = 0; c < CPT; ++c)
                    if (row < rows && col + 8 * c < p.S) {
                        float w[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) w[j] = v[i][8 * c + j];
                        Raw<T, 8> o;
                        o.set(w);
                        o.store(y + 8ull * (at + c));
                    }
            }
        }
        float r2[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            r2[i] = 0.0f;
#pragma unroll
            for (int j = 0; j < V; ++j) r2[i] = fmaf(v[i][j], v[i][j], r2[i]);
        }
        statistic<TPS, WHOLE, R>(r2, sm, turn);
        // (bf16 first: the values that quantising the bf16 norm gives)
        uint32_t w[R][V / 2], m[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            scaled(v[i], rsqrtf(fmaf(r2[i], p.inv_s, p.eps)), pre);
            m[i] = 0u;
#pragma unroll
            for (int j = 0; j < V / 2; ++j) {
                w[i][j] = col + 8 * (j / 4) < p.S ? f32_to_bf16x2(v[i][2 * j], v[i][2 * j + 1]) : 0u;
                m[i] = __vmaxu2(m[i], w[i][j] & 0x7FFF7FFFu);
            }
        }
#pragma unroll
        for (int o = GL / 2; o > 0; o >>= 1)
#pragma unroll
            for (int i = 0; i < R; ++i)
                m[i] = __vmaxu2(m[i], __shfl_xor_sync(0xffffffffu, m[i], o));
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int row = row0 + i * C::SLOTS;
            float inv;
            const float s = f8_scale(__uint_as_float(max(m[i] << 16, m[i] & 0xFFFF0000u)), inv);
            const float2 ii = make_float2(inv, inv);
            if (row >= rows) continue;
            if (ts % GL == 0 && col < p.S) scale[row] = s;
            const unsigned at = row * row_chunks + mine, at_q = row * row_q + mine_q;
#pragma unroll
            for (int c = 0; c < CPT; ++c) {
                uint32_t b[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float2 e;
                    bf16x2_to_f32(w[i][4 * c + j], e.x, e.y);
                    e = mul2(e, ii);
                    b[j] = f8x2_from_f32(e.x, e.y);
                }
                if (col + 8 * c < p.q8_pitch)
                    *reinterpret_cast<uint2*>(p.q8 + 8ull * (at_q + c)) =
                        make_uint2(b[0] | (b[1] << 16), b[2] | (b[3] << 16));
                if (n && col + 8 * c < p.S)
                    *reinterpret_cast<uint4*>(n + 8ull * (at + c)) = make_uint4(
                        w[i][4 * c], w[i][4 * c + 1], w[i][4 * c + 2], w[i][4 * c + 3]);
            }
        }
    }
}

template <typename T, int TPS, bool WHOLE, bool BRANCH>
cudaError_t launch_form(const JoinParams& p, int num_sms, cudaStream_t stream) {
    using C = JoinF8Cfg<TPS, WHOLE>;
    // two rows of two tensors in bf16, or of one: what leaves two or three blocks an SM
    constexpr int R = C::CPT * static_cast<int>(sizeof(T)) * (BRANCH ? 2 : 1) <= 4 ? 2 : 1;
    auto* kern = join_f8_kernel<T, TPS, WHOLE, BRANCH, R>;
    static std::atomic<int> at_once{0};  // blocks an SM: a block takes rows until none is left
    int per_sm = at_once.load(std::memory_order_relaxed);
    if (per_sm == 0) {
        const cudaError_t e =
            cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kern, C::THREADS, 0);
        if (e != cudaSuccess) return e;
        if (per_sm < 1) per_sm = 1;
        at_once.store(per_sm, std::memory_order_relaxed);
    }
    const long long blocks = (p.rows + C::SLOTS * R - 1) / (C::SLOTS * R);
    const long long cap = static_cast<long long>(num_sms) * per_sm;
    return launch_pdl(kern, dim3(static_cast<unsigned>(blocks < cap ? blocks : cap)),
                      dim3(C::THREADS), 0, stream, p);
}

template <typename T, bool WHOLE, bool BRANCH>
cudaError_t launch_tps(const JoinParams& p, int num_sms, cudaStream_t stream) {
    int tps = 2;
    while (tps * (WHOLE ? 16 : 8) < p.S) tps *= 2;
    switch (tps) {
        case 2: return launch_form<T, 2, WHOLE, BRANCH>(p, num_sms, stream);
        case 4: return launch_form<T, 4, WHOLE, BRANCH>(p, num_sms, stream);
        case 8: return launch_form<T, 8, WHOLE, BRANCH>(p, num_sms, stream);
        case 16: return launch_form<T, 16, WHOLE, BRANCH>(p, num_sms, stream);
        case 32: return launch_form<T, 32, WHOLE, BRANCH>(p, num_sms, stream);
        case 64: return launch_form<T, 64, WHOLE, BRANCH>(p, num_sms, stream);
        default:
            if constexpr (!WHOLE) return launch_form<T, 128, WHOLE, BRANCH>(p, num_sms, stream);
            return cudaErrorInvalidValue;
    }
}

template <typename T>
cudaError_t launch_type(const JoinParams& p, bool whole, int num_sms, cudaStream_t stream) {
    if (whole)
        return p.h ? launch_tps<T, true, true>(p, num_sms, stream)
                   : launch_tps<T, true, false>(p, num_sms, stream);
    return p.h ? launch_tps<T, false, true>(p, num_sms, stream)
               : launch_tps<T, false, false>(p, num_sms, stream);
}

}  // namespace

bool join_f8_aligned(const JoinArgs& a) {
    const void* t[] = {a.x, a.h, a.out_y, a.out_n};
    uintptr_t at = 0;
    for (const void* v : t) at |= reinterpret_cast<uintptr_t>(v);
    // (chunks of eight, and rows with a grid's step, are counted in 32 bits)
    return a.C % 32 == 0 && a.C <= 4096 && at % 16 == 0 && a.rows < (1LL << 30) &&
           a.rows * ((a.C + 63) / 64 * 64 / 8) < (1LL << 32);
}

cudaError_t launch_join_f8(const JoinParams& p, bool f32, bool whole, int num_sms,
                           cudaStream_t stream) {
    return f32 ? launch_type<float>(p, whole, num_sms, stream)
               : launch_type<__nv_bfloat16>(p, whole, num_sms, stream);
}

}  // namespace quan
