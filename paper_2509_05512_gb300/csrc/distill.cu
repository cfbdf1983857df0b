// distill.cu -- the loss that trains classes from a teacher's top logits, and its gradient.
//
// A row (pixel) has V logits z and `top` slots, each a class i_k and the teacher's logit t_k of it.  A
// slot whose class is outside [0, V) or whose t_k is -inf is empty.  With p = softmax(t / T) over the
// other slots and q = softmax(z / T) over the classes,
//   loss = T^2 sum over k of p_k (ln p_k - ln q_(i_k)),
//   dz_v = g T (q_v - sum over the k with i_k = v of p_k),      g = dL/dloss,
// both 0 for a row of empty slots.  (T^2 keeps the gradient's size as T grows: q - p falls as 1 / T.)
// With m = max z, S = sum of 2^((z - m) c), c = log2(e) / T:  lse = m / T + ln S is all that the gradient
// needs of the forward pass, q_v = e^(z_v / T - lse).
//
// Everything is fp32; a gradient is rounded once.  A slot's class may come twice: the first of its slots
// adds the others' p in their order, so that no sum depends on which thread comes first.
#include <cuda_bf16.h>

#include "internal.h"
#include "ptx.cuh"
#include "vec_io.cuh"

namespace quan {
namespace {

constexpr float LOG2E = 1.44269504f;
constexpr int LOSS = 1, GRAD = 2;  // what a launch computes: one of them, or both

struct DistillParams {
    const void *z, *index, *teacher;
    const float *lse_in, *dloss;  // GRAD: the forward pass's (without LOSS), and g (null: 1)
    float *loss, *lse;
    void* dz;
    long long rows, pitch;
    int classes, top;
    int index64, teacher_f32;
    float inv_t, c, t2, scale;  // 1 / T, log2(e) / T, T^2, what g is multiplied by (with T)
};

// The elements of a row, 16 bytes a chunk at addresses that are multiples of 16: the row's first and
// last chunk may hold elements of its neighbours, which are not used.
template <typename T>
struct RowView {
    static constexpr int E = 16 / static_cast<int>(sizeof(T));
    const T* base;   // the first chunk
    int head, n;     // the row is elements head .. head + n - 1 from there
    const T *first, *last;  // the tensor
    __device__ __forceinline__ RowView(const T* tensor, long long elements, long long at, int len) {
        first = tensor;
        last = tensor + elements;
        const T* row = tensor + at;
        head = static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T));
        base = row - head;
        n = len;
    }
    __device__ __forceinline__ int chunks() const { return (head + n + E - 1) / E; }
    // A chunk as it is in memory.  Only one that reaches past the tensor's ends goes element by
    // element.
    __device__ __forceinline__ void load(int chunk, Raw<T, E>& r) const {
        const T* p = base + chunk * E;
        if (p >= first && p + E <= last) {
            r.load(p);
        } else {
            float v[E];
#pragma unroll
            for (int j = 0; j < E; ++j) {
                Raw<T, 1> e;
                float w[1] = {0.0f};
                if (p + j >= first && p + j < last) {
                    e.load(p + j);
                    e.values(w);
                }
                v[j] = w[0];
            }
            r.set(v);
        }
    }
    // A chunk's values, -inf outside the row's first `len` elements.
    __device__ __forceinline__ void values(int chunk, const Raw<T, E>& r, int len,
                                           float (&v)[E]) const {
        r.values(v);
        const int lo = head - chunk * E, hi = head + len - chunk * E;
        if (lo > 0 || hi < E) {
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (j < lo || j >= hi) v[j] = -INFINITY;
        }
    }
    // Writes a chunk's values to the row's place in `out`, a tensor laid out as this one.
    __device__ __forceinline__ void store(int chunk, const float (&v)[E], T* out_row) const {
        T* p = out_row - head + chunk * E;
        const int lo = head - chunk * E, hi = head + n - chunk * E;
        if (lo <= 0 && hi >= E && (reinterpret_cast<uintptr_t>(p) & 15u) == 0) {
            Raw<T, E> r;
            r.set(v);
            r.store(p);
        } else {
#pragma unroll
            for (int j = 0; j < E; ++j) {
                if (j < lo || j >= hi) continue;
                Raw<T, 1> e;
                const float w[1] = {v[j]};
                e.set(w);
                e.store(p + j);
            }
        }
    }
};

template <typename T>
__device__ __forceinline__ float element(const T* p) {
    Raw<T, 1> e;
    float v[1];
    e.load(p);
    e.values(v);
    return v[0];
}

template <typename T>
__device__ __forceinline__ void put(T* p, float x) {
    Raw<T, 1> e;
    const float v[1] = {x};
    e.set(v);
    e.store(p);
}

// Slot k of a row: its class (-1 when empty) and the teacher's logit.
__device__ __forceinline__ int slot(const DistillParams& p, long long row, int k, float& t) {
    const long long at = row * p.top + k;
    const long long id = p.index64 ? static_cast<const long long*>(p.index)[at]
                                   : static_cast<const int*>(p.index)[at];
    t = p.teacher_f32 ? element(static_cast<const float*>(p.teacher) + at)
                      : element(static_cast<const __nv_bfloat16*>(p.teacher) + at);
    return id >= 0 && id < p.classes && t != -INFINITY ? static_cast<int>(id) : -1;
}

// A sum of 2^((z - m) c) for another maximum.  (Without a number so far, m = -inf, it is 0, or NaN
// from a NaN.)
__device__ __forceinline__ float shifted(float s, float m, float top, float c) {
    return m == -INFINITY ? s : s * ex2_approx_ftz((m - top) * c);
}

constexpr int DISTILL_THREADS = 256;
constexpr int DISTILL_WARPS = DISTILL_THREADS / 32;

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Max and sum over the block; `sm` holds a word a warp.
template <bool MAX>
__device__ __forceinline__ float block_reduce(float v, float* sm) {
    v = MAX ? warp_max(v) : warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = v;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    v = lane < DISTILL_WARPS ? sm[lane] : (MAX ? -INFINITY : 0.0f);
    return MAX ? warp_max(v) : warp_sum(v);
}

// A block a row; the logits are read once for the sums and once for the gradient.  Loss and gradient
// of 4096 x 32768 bf16: 149 us (the second reading mostly from L2); of 100,352 x 100: 403 us, where a
// block has 13 chunks to read and a dozen barriers.
template <typename T, int MODE>
__global__ void __launch_bounds__(DISTILL_THREADS) distill_kernel(const DistillParams p) {
    constexpr int E = RowView<T>::E;
    extern __shared__ float slots[];  // p_k, the row's logit at class k, class k
    float *sp = slots, *sz = slots + p.top;
    int* si = reinterpret_cast<int*>(slots + 2 * p.top);
    __shared__ float sm[DISTILL_WARPS];
    griddep_launch_dependents();
    griddep_wait();
    const long long row = blockIdx.x;
    const T* z = static_cast<const T*>(p.z);
    const RowView<T> view(z, p.rows * p.pitch, row * p.pitch,
                          MODE & GRAD ? static_cast<int>(p.pitch) : p.classes);
    const T* zrow = z + row * p.pitch;
    // the teacher's side
    float tm = -INFINITY, some = 0.0f;
    for (int k = threadIdx.x; k < p.top; k += DISTILL_THREADS) {
        float t;
        const int id = slot(p, row, k, t);
        si[k] = id;
        sp[k] = t;
        if (id >= 0) {
            sz[k] = element(zrow + id);
            tm = fmaxf(tm, t);
            some = 1.0f;
        }
    }
    tm = block_reduce<true>(tm, sm);
    some = block_reduce<true>(some, sm);
    float ts = 0.0f;
    for (int k = threadIdx.x; k < p.top; k += DISTILL_THREADS)
        if (si[k] >= 0) ts += expf((sp[k] - tm) * p.inv_t);
    ts = block_reduce<false>(ts, sm);
    const float ln_ts = logf(ts);
    // the student's
    float m = 0.0f, ln_s = 0.0f, inv_s = 1.0f, lse = 0.0f;
    const int chunks = view.chunks();
    if (MODE & LOSS) {
        m = -INFINITY;
        float s = 0.0f;
        for (int i = threadIdx.x; i < chunks; i += DISTILL_THREADS) {
            Raw<T, E> r;
            float v[E], top = m;
            view.load(i, r);
            view.values(i, r, p.classes, v);
#pragma unroll
            for (int j = 0; j < E; ++j) top = fmaxf(top, v[j]);
            const float at = top == -INFINITY ? 0.0f : top;
            s = shifted(s, m, at, p.c);
#pragma unroll
            for (int j = 0; j < E; ++j) s += ex2_approx_ftz((v[j] - at) * p.c);
            m = top;
        }
        const float top = block_reduce<true>(m, sm);
        s = block_reduce<false>(shifted(s, m, top, p.c), sm);
        m = top;
        inv_s = 1.0f / s;
        ln_s = logf(s);
        lse = fmaf(m, p.inv_t, ln_s);
        float loss = 0.0f;
        for (int k = threadIdx.x; k < p.top; k += DISTILL_THREADS) {
            if (si[k] < 0) continue;
            const float lnp = (sp[k] - tm) * p.inv_t - ln_ts, pk = expf(lnp);
            // (a slot whose share has vanished has no part, be its class impossible)
            if (!(pk == 0.0f)) loss = fmaf(pk, lnp - ((sz[k] - m) * p.inv_t - ln_s), loss);
        }
        loss = block_reduce<false>(loss, sm);
        if (threadIdx.x == 0) {
            p.loss[row] = some > 0.0f ? p.t2 * loss : 0.0f;
            if (p.lse) p.lse[row] = lse;
        }
    } else {
        lse = p.lse_in[row];
    }
    if (MODE & GRAD) {
        T* out = static_cast<T*>(p.dz) + row * p.pitch;
        const float g = some > 0.0f ? (p.dloss ? p.dloss[row] : 1.0f) * p.scale : 0.0f;
        auto q_of = [&](float v) {
            return MODE & LOSS ? ex2_approx_ftz((v - m) * p.c) * inv_s
                               : ex2_approx_ftz(fmaf(v, p.inv_t, -lse) * LOG2E);
        };
        // the slots' elements, before any of the row is written (dz may be z)
        __syncthreads();
        for (int k = threadIdx.x; k < p.top; k += DISTILL_THREADS)
            if (si[k] >= 0) sp[k] = expf((sp[k] - tm) * p.inv_t - ln_ts);
        for (int i = threadIdx.x; i < chunks; i += DISTILL_THREADS) {
            Raw<T, E> r;
            float v[E];
            view.load(i, r);
            view.values(i, r, p.classes, v);
            const int behind = view.head + p.classes - i * E;  // from here on: padding
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const float d = g * q_of(v[j]);
                v[j] = g == 0.0f || j >= behind ? 0.0f : d;
            }
            view.store(i, v, out);
        }
        __syncthreads();
        if (g != 0.0f) {
            for (int k = threadIdx.x; k < p.top; k += DISTILL_THREADS) {
                const int id = si[k];
                if (id < 0) continue;
                float share = 0.0f;
                bool mine = true;
                for (int j = 0; j < p.top; ++j) {
                    if (si[j] != id) continue;
                    if (j < k) mine = false;
                    share += sp[j];
                }
                if (mine) put(out + id, g * (q_of(sz[k]) - share));
            }
        }
    }
}

template <typename T>
cudaError_t launch_distill_t(const DistillParams& p, cudaStream_t stream) {
    const dim3 g(static_cast<unsigned>(p.rows)), b(DISTILL_THREADS);
    const size_t smem = static_cast<size_t>(p.top) * 12;
    if (!p.dz) return launch_pdl(distill_kernel<T, LOSS>, g, b, smem, stream, p);
    return p.loss ? launch_pdl(distill_kernel<T, LOSS | GRAD>, g, b, smem, stream, p)
                  : launch_pdl(distill_kernel<T, GRAD>, g, b, smem, stream, p);
}

}  // namespace

cudaError_t launch_distill(const DistillArgs& a, int num_sms, cudaStream_t stream) {
    if (a.rows == 0) return cudaSuccess;
    DistillParams p = {};
    p.z = a.z;
    p.index = a.index;
    p.teacher = a.teacher;
    p.lse_in = a.lse_in;
    p.dloss = a.dloss;
    p.loss = a.loss;
    p.lse = a.lse;
    p.dz = a.dz;
    p.rows = a.rows;
    p.pitch = a.pitch;
    p.classes = a.classes;
    p.top = a.top;
    p.index64 = a.index64;
    p.teacher_f32 = a.teacher_f32;
    p.inv_t = 1.0f / a.temperature;
    p.c = static_cast<float>(1.4426950408889634 / static_cast<double>(a.temperature));
    p.t2 = a.temperature * a.temperature;
    p.scale = a.scale * a.temperature;
    return a.f32 ? launch_distill_t<float>(p, stream) : launch_distill_t<__nv_bfloat16>(p, stream);
}

}  // namespace quan
