// residual.cu -- the join of a residual block's branch with its stream, its gradients, and
// dropout.  Rows are pixels, C channels each; the norms are root-mean-square norms over the
// whole row (groups = 1) or over each quaternion component by itself (groups = 4), S = C / groups
// channels wide:
//   u = h / rms(h) * post            (post-norm of the branch; u = h without one)
//   d = dropout(u),  y = x + alpha * gate * d
//   n = y / rms(y) * pre             (the next branch's pre-norm), rms(v)^2 = mean(v^2) + eps
// and, from dy = dL/dy (the stream's) and dn = dL/dn, with r1 = 1 / rms(h), r2 = 1 / rms(y),
// t = dn * pre:
//   dx = dy + r2 (t - y r2^2 mean(t y)),     dpre  = sum of dn y r2
//   s = alpha dropout'(dx), v = s gate,      dgate = sum of s u,  dpost = sum of v h r1
//   w = v post,  dh = r1 (w - h r1^2 mean(w h))
// (dropout' = the same mask and factor).  All arithmetic and every sum is fp32; a tensor element
// is rounded once, on its way out, and n is taken of y before that rounding.  The gradients need
// no statistics kept from the forward call: they read h and y whole anyway.
//
// Both directions are one pass, each tensor read or written once.  A row stays in registers
// between its two reductions: tps threads (a power of two) hold a group, eight consecutive channels
// a thread (at most two such chunks), so that narrow rows share a warp and reduce with shuffles,
// wide ones a block of up to 512 threads (8192 channels at most).  Column sums stay in each thread's
// registers for all of its block's rows; blocks leave one row of partial sums each, added in a fixed
// order by a second launch, so that repeated calls give the same bits.
//
// Measured on 32 x 56 x 56 x 256 bf16 with dropout: forward 38.2 us, 5.4 TB/s, bound by HBM with the
// generator's integer work beside it (two rows under way a thread: 55 without the row ahead);
// gradients 64 us, 4.8 TB/s, at no single limit: about 470 instructions for eight elements of four
// tensors take two thirds of the issue slots, HBM is at half, and 16 warps an SM leave fixed
// latencies uncovered (the row ahead: 85 without; three blocks an SM spill: 89).
#include <cuda_bf16.h>

#include <atomic>

#include "internal.h"
#include "philox.cuh"
#include "ptx.cuh"
#include "vec_io.cuh"

namespace quan {
namespace {

// ------------------------------------------------------------------ dropout

// UNROLL blocks of eight elements a thread, their loads first.  32 x 112 x 112 x 64 bf16: 17.6 us,
// 5.8 TB/s, HBM beside the generator's integer issue (22 us with one block a thread).
template <typename T, bool VEC, int UNROLL>
__global__ void __launch_bounds__(256) dropout_kernel(const T* x, long long n, DropoutArgs d,
                                                      T* out) {
    griddep_launch_dependents();
    griddep_wait();
    const unsigned long long base = dropout_base(d);
    const long long g0 = static_cast<long long>(blockIdx.x) * (256 * UNROLL) + threadIdx.x;
    Raw<T, 8> r[UNROLL];
    if (VEC) {
#pragma unroll
        for (int i = 0; i < UNROLL; ++i)
            if (8 * (g0 + 256 * i) + 8 <= n) r[i].load(x + 8 * (g0 + 256 * i));
    }
#pragma unroll
    for (int i = 0; i < UNROLL; ++i) {
        const long long g = g0 + 256 * i;
        if (8 * g >= n) break;
        Dropout8 m;
        m.none();
        if (d.draws) m.draw(d, base + g);
        if (VEC && 8 * g + 8 <= n) {
            float v[8];
            r[i].values(v);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = m.keep(d, j) ? v[j] * d.factor : 0.0f;
            r[i].set(v);
            r[i].store(out + 8 * g);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (8 * g + j >= n) break;
                Raw<T, 1> e;
                float w[1];
                e.load(x + 8 * g + j);
                e.values(w);
                w[0] = m.keep(d, j) ? w[0] * d.factor : 0.0f;
                e.set(w);
                e.store(out + 8 * g + j);
            }
        }
    }
}

// ------------------------------------------------------------------ the join

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

template <typename T, int LV, int NC, bool CROSS>
__global__ void __launch_bounds__(CROSS ? 512 : 256) join_fwd_kernel(const JoinParams p) {
    __shared__ float sm[2][96];
    int turn = 0;
    griddep_launch_dependents();
    griddep_wait();
    const Place q = place_of(p);
    // pg = alpha gate post / (1 - p): what a kept element of h / rms(h) is multiplied by
    float pg[NC][8], pre[NC][8];
    auto load_gate = [&](long long image) {
        float post[NC][8];
        load_columns<NC>(p.post, p, q, p.alpha * p.drop.factor, post);
        load_columns<NC>(p.gate ? p.gate + image * p.C : nullptr, p, q, 1.0f, pg);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) pg[c][j] *= post[c][j];
    };
    load_gate(0);
    load_columns<NC>(p.pre, p, q, 1.0f, pre);
    const unsigned long long base = p.drop.draws ? dropout_base(p.drop) : 0ull;
    const T *x = static_cast<const T*>(p.x), *h = static_cast<const T*>(p.h);
    T *y = static_cast<T*>(p.out_y), *n = static_cast<T*>(p.out_n);
    const long long step = static_cast<long long>(gridDim.x) * p.slots;
    // a row's tensors are loaded one row ahead
    Chunk<T, LV> nx[NC], nh[NC];
    auto fetch = [&](long long row) {
        const long long at = row * p.C + q.seg * p.S;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = (q.ts + c * p.tps) * 8;
            const int left = row < p.rows && q.slot < p.slots ? p.S - col : 0;
            nx[c].load(x + at + col, left);
            if (h) nh[c].load(h + at + col, left);
        }
    };
    long long row = static_cast<long long>(blockIdx.x) * p.slots + q.slot;
    long long image = 0, image_end = p.rows_per_image;
    fetch(row);
    for (long long r0 = static_cast<long long>(blockIdx.x) * p.slots; r0 < p.rows;
         r0 += step, row += step) {
        const bool active = row < p.rows && q.slot < p.slots;
        const long long at = row * p.C + q.seg * p.S;
        float v[NC][8], u[NC][8];
        int left[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            left[c] = active ? p.S - (q.ts + c * p.tps) * 8 : 0;
            nx[c].values(v[c]);
            if (h) nh[c].values(u[c]);
        }
        fetch(row + step);
        Chunk<T, LV> o;
        if (h) {
            if (p.gate && active && row >= image_end) {
                image = row / p.rows_per_image;
                image_end = (image + 1) * p.rows_per_image;
                load_gate(image);
            }
            float r1 = 1.0f;
            if (p.post) {
                float ss[1] = {0.0f};
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) ss[0] = fmaf(u[c][j], u[c][j], ss[0]);
                group_sum<CROSS, 1>(ss, p.tps, sm, turn);
                r1 = rsqrtf(fmaf(ss[0], p.inv_s, p.eps));
            }
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int col = (q.ts + c * p.tps) * 8;
                // (the product is selected, not a factor: an infinity that is dropped is 0)
                Dropout8 m;
                m.none();
                if (p.drop.draws) draw_from<LV == 8>(m, p.drop, base, at + col);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float d = u[c][j] * (r1 * pg[c][j]);
                    v[c][j] += m.keep(p.drop, j) ? d : 0.0f;
                }
                o.set_store(v[c], y + at + col, left[c]);
            }
        }
        if (n) {
            float ss[1] = {0.0f};
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) ss[0] = fmaf(v[c][j], v[c][j], ss[0]);
            group_sum<CROSS, 1>(ss, p.tps, sm, turn);
            const float r2 = rsqrtf(fmaf(ss[0], p.inv_s, p.eps));
#pragma unroll
            for (int c = 0; c < NC; ++c) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[c][j] *= r2 * pre[c][j];
                o.set_store(v[c], n + at + (q.ts + c * p.tps) * 8, left[c]);
            }
        }
    }
}

// Adds a column sum over the block's slots and stores it to dst[C].  `sm` holds slots x C words
// (not used by a block of one slot).
template <int NC>
__device__ __forceinline__ void flush_columns(const JoinParams& p, const Place& q,
                                              float (&acc)[NC][8], float* sm, float* dst) {
    if (p.slots > 1) __syncthreads();
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int col = (q.ts + c * p.tps) * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (col + j < p.S && q.slot < p.slots) {
                const int at = q.seg * p.S + col + j;
                if (p.slots > 1)
                    sm[q.slot * p.C + at] = acc[c][j];
                else
                    dst[at] = acc[c][j];
            }
            acc[c][j] = 0.0f;
        }
    }
    if (p.slots > 1) {
        __syncthreads();
        for (int c = threadIdx.x; c < p.C; c += blockDim.x) {
            float s = 0.0f;
            for (int k = 0; k < p.slots; ++k) s += sm[k * p.C + c];
            dst[c] = s;
        }
    }
}

template <typename T, int LV, int NC, bool CROSS>
__global__ void __launch_bounds__(CROSS ? 512 : 256, CROSS ? 1 : 2) join_bwd_kernel(const JoinParams p) {
    __shared__ float sm[2][96];
    int turn = 0;
    extern __shared__ float cols[];
    griddep_launch_dependents();
    griddep_wait();
    const Place q = place_of(p);
    // With c = alpha / (1 - p), k the mask and e = sum over an image's rows of k dx h r1:
    // dgate = c post e and dpost = sum over images of c gate e, so one sum serves both;
    // w = k dx pg with pg = c gate post.
    float pg[NC][8], pre[NC][8];
    float e[NC][8] = {}, a_pre[NC][8] = {}, a_post[NC][8] = {};
    const float factor = p.alpha * p.drop.factor;  // (0 when nothing is kept)
    load_columns<NC>(p.pre, p, q, 1.0f, pre);
    const unsigned long long base = p.drop.draws ? dropout_base(p.drop) : 0ull;
    const T *h = static_cast<const T*>(p.h), *y = static_cast<const T*>(p.y);
    const T *dy = static_cast<const T*>(p.dy), *dn = static_cast<const T*>(p.dn);
    T *dx = static_cast<T*>(p.out_y), *dh = static_cast<T*>(p.out_n);
    for (long long u = blockIdx.x; u < p.units; u += gridDim.x) {
        const long long image = u / p.chunks, k = u - image * p.chunks;
        const long long first = image * p.rows_per_image + k * p.chunk_rows;
        long long last = first + p.chunk_rows;
        if (last > (image + 1) * p.rows_per_image) last = (image + 1) * p.rows_per_image;
        const float* gate = p.gate ? p.gate + image * p.C : nullptr;
        {
            float post[NC][8];
            load_columns<NC>(p.post, p, q, 1.0f, post);
            load_columns<NC>(gate, p, q, factor, pg);
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) pg[c][j] *= post[c][j];
        }
        // a row's tensors are loaded one row ahead, where the registers allow it (16 words of
        // bf16; fp32 rows have twice the bytes under way as it is)
        constexpr bool AHEAD = sizeof(T) == 2 && NC == 1;
        Chunk<T, LV> cdy[NC], cdn[NC], cy[NC], ch[NC];
        auto fetch = [&](long long row, long long at) {
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int col = (q.ts + c * p.tps) * 8;
                const int left = row < last && q.slot < p.slots ? p.S - col : 0;
                if (dy)
                    cdy[c].load(dy + at + col, left);
                else
                    cdy[c].zero();
                if (dn) {
                    cdn[c].load(dn + at + col, left);
                    cy[c].load(y + at + col, left);
                }
                if (h) ch[c].load(h + at + col, left);
            }
        };
        const long long at_step = static_cast<long long>(p.slots) * p.C;
        long long row = first + q.slot, at = row * p.C + q.seg * p.S;
        if (AHEAD) fetch(row, at);
        for (long long r0 = first; r0 < last; r0 += p.slots, row += p.slots) {
            if constexpr (!AHEAD) {  // (one register pair less across the row)
                at = row * p.C + q.seg * p.S;
                fetch(row, at);
            }
            const bool active = row < last && q.slot < p.slots;
            float g[NC][8], yv[NC][8], nv[NC][8], hv[NC][8];
            int left[NC];
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                left[c] = active ? p.S - (q.ts + c * p.tps) * 8 : 0;
                cdy[c].values(g[c]);
                if (dn) {
                    cy[c].values(yv[c]);
                    cdn[c].values(nv[c]);
                }
                if (h) ch[c].values(hv[c]);
            }
            const long long here = at;
            if constexpr (AHEAD) {
                at += at_step;
                fetch(row + p.slots, at);
            }
            float s3[3] = {0.0f, 0.0f, 0.0f};  // sums of h^2, y^2 and t y
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                if (dn) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        s3[1] = fmaf(yv[c][j], yv[c][j], s3[1]);
                        s3[2] = fmaf(nv[c][j] * pre[c][j], yv[c][j], s3[2]);
                    }
                }
                if (h) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) s3[0] = fmaf(hv[c][j], hv[c][j], s3[0]);
                }
            }
            group_sum<CROSS, 3>(s3, p.tps, sm, turn);
            const float r1 = p.post ? rsqrtf(fmaf(s3[0], p.inv_s, p.eps)) : 1.0f;
            Chunk<T, LV> o;
            if (dn) {
                const float r2 = rsqrtf(fmaf(s3[1], p.inv_s, p.eps));
                const float m = -s3[2] * p.inv_s * r2 * r2 * r2;
#pragma unroll
                for (int c = 0; c < NC; ++c) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float rn = r2 * nv[c][j];
                        g[c][j] = fmaf(rn, pre[c][j], fmaf(m, yv[c][j], g[c][j]));
                        a_pre[c][j] = fmaf(rn, yv[c][j], a_pre[c][j]);
                    }
                    o.set_store(g[c], dx + here + (q.ts + c * p.tps) * 8, left[c]);
                }
            } else if (dx) {
#pragma unroll
                for (int c = 0; c < NC; ++c)
                    o.set_store(g[c], dx + here + (q.ts + c * p.tps) * 8, left[c]);
            }
            if (h) {
                float w1[1] = {0.0f};
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    Dropout8 m;
                    m.none();
                    if (p.drop.draws)
                        draw_from<LV == 8>(m, p.drop, base, here + (q.ts + c * p.tps) * 8);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        // (both factors are selected: what is dropped has no part, be it infinite)
                        const bool keep = m.keep(p.drop, j);
                        const float gk = keep ? g[c][j] : 0.0f, hk = keep ? hv[c][j] : 0.0f;
                        e[c][j] = fmaf(gk * r1, hk, e[c][j]);
                        g[c][j] = gk * pg[c][j];  // w
                        w1[0] = fmaf(g[c][j], hk, w1[0]);
                    }
                }
                if (p.post) {
                    group_sum<CROSS, 1>(w1, p.tps, sm, turn);
                    const float m = -w1[0] * p.inv_s * r1 * r1 * r1;
#pragma unroll
                    for (int c = 0; c < NC; ++c)
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            g[c][j] = fmaf(m, hv[c][j], r1 * g[c][j]);
                }
#pragma unroll
                for (int c = 0; c < NC; ++c)
                    o.set_store(g[c], dh + here + (q.ts + c * p.tps) * 8, left[c]);
            }
        }
        if (p.part_post || p.part_gate) {
            float v[NC][8];
            load_columns<NC>(gate, p, q, factor, v);
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) a_post[c][j] = fmaf(v[c][j], e[c][j], a_post[c][j]);
            load_columns<NC>(p.post, p, q, factor, v);
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    v[c][j] *= e[c][j];
                    e[c][j] = 0.0f;
                }
            if (p.part_gate) flush_columns<NC>(p, q, v, cols, p.part_gate + u * p.C);
        }
    }
    const long long b = blockIdx.x * p.part_stride;
    if (p.part_post) flush_columns<NC>(p, q, a_post, cols, p.part_post + b);
    if (p.part_pre) flush_columns<NC>(p, q, a_pre, cols, p.part_pre + b);
}

// out[v][c] = sum over k < count of part[v stride_v + k stride_k + c], for the vectors v of
// blockIdx.y; 32 channels a block, 32 threads a channel, joined in a fixed order.
struct ColumnSum {
    const float* part;
    float* out;
    long long stride_v, stride_k;
    int count;
};
__global__ void __launch_bounds__(1024)
    join_columns_kernel(ColumnSum a, ColumnSum b, ColumnSum c, int C) {
    __shared__ float sm[32][33];
    griddep_launch_dependents();
    griddep_wait();
    const long long v = blockIdx.y;
    const ColumnSum& s = v == 0 ? a : (v == 1 ? b : c);
    if (!s.out) return;
    const long long w = v < 2 ? 0 : v - 2;
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
    const int col = blockIdx.x * 32 + lane;
    float acc = 0.0f;
    if (col < C) {
        const float* src = s.part + w * s.stride_v + col;
#pragma unroll 8
        for (int k = part; k < s.count; k += 32) acc += src[k * s.stride_k];
    }
    sm[part][lane] = acc;
    __syncthreads();
    // warp `part` adds the 32 parts of channel `part` of the block
    float t = sm[lane][part];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    const int mine = blockIdx.x * 32 + part;
    if (lane == 0 && mine < C) s.out[w * C + mine] = t;
}

constexpr int JOIN_MAX_THREADS = 512;

// Threads of a group, chunks a thread, threads of a block and rows side by side in it.
struct JoinPlan {
    int tps, nc, threads, slots;
    long long chunk_rows, units;  // backward
    int chunks, grid;
};

bool join_plan(int C, int groups, JoinPlan* pl) {
    const int S = C / groups;
    for (pl->nc = 1; pl->nc <= 2; ++pl->nc) {
        pl->tps = 1;
        while (pl->tps * 8 * pl->nc < S) pl->tps *= 2;
        if (pl->tps * groups <= JOIN_MAX_THREADS) break;
    }
    if (pl->nc > 2) return false;
    const int tpr = pl->tps * groups;
    pl->threads = tpr > 256 ? tpr : 256;
    pl->slots = pl->threads / tpr;
    return true;
}

// Backward: rows are cut into units within an image, so many that the SMs have a few blocks
// each; a block takes units until none is left.
void join_units(JoinPlan* pl, long long rows, long long images, int num_sms) {
    const long long per_image = rows / images;
    const long long target = static_cast<long long>(num_sms) * (pl->threads > 256 ? 1 : 2);
    long long chunks = (target + images - 1) / images;
    const long long most = (per_image + pl->slots - 1) / pl->slots;
    if (chunks > most) chunks = most;
    long long r = (per_image + chunks - 1) / chunks;
    r = (r + pl->slots - 1) / pl->slots * pl->slots;
    pl->chunk_rows = r;
    pl->chunks = static_cast<int>((per_image + r - 1) / r);
    pl->units = images * pl->chunks;
    pl->grid = static_cast<int>(pl->units < target ? pl->units : target);
}

template <typename T>
int load_width(int S, int C, const void* const* t, int n) {
    uintptr_t a = 0;
    for (int i = 0; i < n; ++i) a |= reinterpret_cast<uintptr_t>(t[i]);
    const int row = C * static_cast<int>(sizeof(T));
    if (S % 8 == 0 && row % 16 == 0 && a % raw_align<T, 8>() == 0) return 8;
    if (S % 4 == 0 && a % raw_align<T, 4>() == 0) return 4;
    return 1;
}

// A thread's one or two chunks; two only where a row takes more than the block's threads, so
// where its sums cross warps.  Forward, a block takes rows until none is left, and there are as many
// blocks as run at once (`blocks` at most): with twice as many the last ones run by themselves
// (32 x 56 x 56 x 256: 40 us, 38 with one wave).
template <typename T, int LV, int NC, bool CROSS>
cudaError_t launch_join_nc(const JoinParams& p, const JoinPlan& pl, bool backward,
                           long long blocks, int num_sms, cudaStream_t stream) {
    const dim3 b(static_cast<unsigned>(pl.threads));
    if (backward) {
        const size_t smem = pl.slots > 1 ? static_cast<size_t>(pl.slots) * p.C * 4 : 0;
        return launch_pdl(join_bwd_kernel<T, LV, NC, CROSS>,
                          dim3(static_cast<unsigned>(blocks)), b, smem, stream, p);
    }
    static std::atomic<int> at_once[2];  // blocks an SM, of 256 and of 512 threads
    std::atomic<int>& known = at_once[pl.threads > 256];
    int per_sm = known.load(std::memory_order_relaxed);
    if (per_sm == 0) {
        const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(
            &per_sm, join_fwd_kernel<T, LV, NC, CROSS>, pl.threads, 0);
        if (e != cudaSuccess) return e;
        if (per_sm < 1) per_sm = 1;
        known.store(per_sm, std::memory_order_relaxed);
    }
    const long long cap = static_cast<long long>(num_sms) * per_sm;
    return launch_pdl(join_fwd_kernel<T, LV, NC, CROSS>,
                      dim3(static_cast<unsigned>(blocks < cap ? blocks : cap)), b, 0, stream, p);
}

template <typename T, int LV>
cudaError_t launch_join_lv(const JoinParams& p, const JoinPlan& pl, bool backward,
                           long long blocks, int num_sms, cudaStream_t stream) {
    if (pl.nc == 2)
        return launch_join_nc<T, LV, 2, true>(p, pl, backward, blocks, num_sms, stream);
    return pl.tps > 32
               ? launch_join_nc<T, LV, 1, true>(p, pl, backward, blocks, num_sms, stream)
               : launch_join_nc<T, LV, 1, false>(p, pl, backward, blocks, num_sms, stream);
}

template <typename T>
cudaError_t launch_join_t(const JoinParams& p, const JoinPlan& pl, int lv, bool backward,
                          long long blocks, int num_sms, cudaStream_t stream) {
    return lv == 8   ? launch_join_lv<T, 8>(p, pl, backward, blocks, num_sms, stream)
           : lv == 4 ? launch_join_lv<T, 4>(p, pl, backward, blocks, num_sms, stream)
                     : launch_join_lv<T, 1>(p, pl, backward, blocks, num_sms, stream);
}

void fill(JoinParams* p, const JoinArgs& a, const JoinPlan& pl) {
    p->x = a.x;
    p->h = a.h;
    p->y = a.y;
    p->dy = a.dy;
    p->dn = a.dn;
    p->post = a.post;
    p->gate = a.gate;
    p->pre = a.pre;
    p->out_y = a.out_y;
    p->out_n = a.out_n;
    p->rows = a.rows;
    p->rows_per_image = a.rows / a.images;
    p->C = a.C;
    p->S = a.C / a.groups;
    p->groups = a.groups;
    p->tps = pl.tps;
    p->slots = pl.slots;
    p->alpha = a.alpha;
    p->eps = a.eps;
    p->inv_s = 1.0f / static_cast<float>(p->S);
    p->drop = a.drop;
}

int join_load_width(const JoinArgs& a) {
    const void* t[] = {a.x, a.h, a.y, a.dy, a.dn, a.out_y, a.out_n};
    return a.f32 ? load_width<float>(a.C / a.groups, a.C, t, 7)
                 : load_width<__nv_bfloat16>(a.C / a.groups, a.C, t, 7);
}

}  // namespace

DropoutArgs dropout_args(float p, unsigned long long seed, unsigned long long offset,
                         const unsigned long long* counter) {
    DropoutArgs d;
    const uint32_t t = static_cast<uint32_t>(p * 65536.0 + 0.5);
    d.draws = t > 0 && t < 65536u;
    d.bound = t < 65536u ? t << 16 : 1u << 16;
    d.factor = t < 65536u ? static_cast<float>(65536.0 / (65536.0 - static_cast<double>(t))) : 0.0f;
    d.key0 = static_cast<uint32_t>(seed);
    d.key1 = static_cast<uint32_t>(seed >> 32);
    d.offset = offset;
    d.counter = counter;
    return d;
}

cudaError_t launch_dropout(const void* x, long long n, bool f32, const DropoutArgs& d, void* out,
                           int num_sms, cudaStream_t stream) {
    if (n == 0) return cudaSuccess;
    const bool vec = (reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(out)) % 16 == 0;
    const long long groups = (n + 7) / 8;
    // four blocks of eight a thread once that still fills the SMs twice
    const bool many = groups >= 4LL * 256 * 2 * 8 * num_sms;
    const long long per = 256 * (many ? 4 : 1);
    const dim3 g(static_cast<unsigned>((groups + per - 1) / per)), b(256);
#define QUAN_DROPOUT(T, VEC, U)                                                          \
    launch_pdl(dropout_kernel<T, VEC, U>, g, b, 0, stream, static_cast<const T*>(x), n, d, \
               static_cast<T*>(out))
    if (f32)
        return vec ? (many ? QUAN_DROPOUT(float, true, 4) : QUAN_DROPOUT(float, true, 1))
                   : (many ? QUAN_DROPOUT(float, false, 4) : QUAN_DROPOUT(float, false, 1));
    return vec ? (many ? QUAN_DROPOUT(__nv_bfloat16, true, 4) : QUAN_DROPOUT(__nv_bfloat16, true, 1))
               : (many ? QUAN_DROPOUT(__nv_bfloat16, false, 4)
                       : QUAN_DROPOUT(__nv_bfloat16, false, 1));
#undef QUAN_DROPOUT
}

bool join_supported(int C, int groups) {
    JoinPlan pl;
    return join_plan(C, groups, &pl);
}

cudaError_t launch_join_fwd(const JoinArgs& a, int num_sms, cudaStream_t stream) {
    if (a.rows == 0) return cudaSuccess;
    JoinPlan pl;
    join_plan(a.C, a.groups, &pl);
    JoinParams p = {};
    fill(&p, a, pl);
    const long long blocks = (a.rows + pl.slots - 1) / pl.slots;
    const int lv = join_load_width(a);
    return a.f32 ? launch_join_t<float>(p, pl, lv, false, blocks, num_sms, stream)
                 : launch_join_t<__nv_bfloat16>(p, pl, lv, false, blocks, num_sms, stream);
}

// Partial sums: one row of dpost and dpre a block, and one row of dgate a unit, unless there is
// just one (it then is the result).
size_t join_bwd_workspace_bytes(long long rows, int C, int groups, long long images,
                                int num_sms) {
    JoinPlan pl;
    if (rows == 0 || !join_plan(C, groups, &pl)) return 0;
    join_units(&pl, rows, images, num_sms);
    const size_t w = pl.grid > 1 ? 2u * static_cast<size_t>(pl.grid) : 0;
    const size_t g = pl.chunks > 1 ? static_cast<size_t>(pl.units) : 0;
    return (w + g) * C * sizeof(float);
}

cudaError_t launch_join_bwd(const JoinArgs& a, float* workspace, float* dpost, float* dgate,
                            float* dpre, int num_sms, cudaStream_t stream) {
    if (a.rows == 0) {
        float* out[] = {dpost, dgate, dpre};
        for (int k = 0; k < 3; ++k) {
            if (!out[k]) continue;
            const size_t n = static_cast<size_t>(a.C) * (k == 1 ? a.images : 1);
            const cudaError_t e = cudaMemsetAsync(out[k], 0, n * sizeof(float), stream);
            if (e != cudaSuccess) return e;
        }
        return cudaSuccess;
    }
    JoinPlan pl;
    join_plan(a.C, a.groups, &pl);
    join_units(&pl, a.rows, a.images, num_sms);
    JoinParams p = {};
    fill(&p, a, pl);
    p.units = pl.units;
    p.chunk_rows = pl.chunk_rows;
    p.chunks = pl.chunks;
    const long long C = a.C;
    float* gate_part = workspace + (pl.grid > 1 ? 2LL * pl.grid * C : 0);
    p.part_gate = a.gate ? (pl.chunks > 1 ? gate_part : dgate) : nullptr;
    // (one block: its sums are the results)
    const bool many = pl.grid > 1;
    p.part_post = dpost ? (many ? workspace : dpost) : nullptr;
    p.part_pre = dpre ? (many ? workspace + C : dpre) : nullptr;
    p.part_stride = 2 * C;
    const int lv = join_load_width(a);
    cudaError_t e =
        a.f32 ? launch_join_t<float>(p, pl, lv, true, pl.grid, num_sms, stream)
              : launch_join_t<__nv_bfloat16>(p, pl, lv, true, pl.grid, num_sms, stream);
    if (e != cudaSuccess) return e;
    const bool sum_g = a.gate && pl.chunks > 1;
    if (!(many && (dpost || dpre)) && !sum_g) return cudaSuccess;
    const ColumnSum post = {p.part_post, many ? dpost : nullptr, 0, 2 * C, pl.grid};
    const ColumnSum pre = {p.part_pre, many ? dpre : nullptr, 0, 2 * C, pl.grid};
    const ColumnSum gate = {gate_part, dgate, pl.chunks * C, C, pl.chunks};
    const dim3 g(static_cast<unsigned>((a.C + 31) / 32),
                 static_cast<unsigned>(2 + (sum_g ? a.images : 0)));
    return launch_pdl(join_columns_kernel, g, dim3(1024), 0, stream, post, pre, gate, a.C);
}

}  // namespace quan
