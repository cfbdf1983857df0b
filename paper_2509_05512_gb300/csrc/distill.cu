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
//
// A row is read once and its gradient written once, with what a row needs in between on the chip: rows
// of up to 4 KB as tiles of many rows (distill_tile_kernel), longer ones whole in a ring of shared
// memory (distill_ring_kernel), single ones, those of more than 64 KB and the gradient alone of rows below
// 48 KB or of few by blocks that keep their part in registers (distill_row_kernel).  Bound: HBM for long rows; for short ones the
// instructions of their slots and reductions.  Loss and gradient, device time: 4096 x 32768 bf16 90 us,
// 6.0 TB/s (149 by a block a row that reads it twice); 100,352 x 100 bf16, ten slots, 17.6 us, 2.9 TB/s
// (403); gradient of 333 x 10007 fp32 6.5 us; loss of one row of 65,536 fp32 4.1 us.
#include <cuda_bf16.h>

#include <atomic>

#include "internal.h"
#include "pairs.cuh"
#include "ptx.cuh"
#include "vec_io.cuh"

namespace quan {
namespace {

constexpr float LOG2E = 1.44269504f;
constexpr int DISTILL_TOP = 256;    // slots a row at most
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
    const T* base;           // the first chunk
    int head, n;             // the row is elements head .. head + n - 1 from there
    const T *first, *last;   // the tensor
    __device__ __forceinline__ RowView(const T* tensor, long long elements, long long at, int len) {
        first = tensor;
        last = tensor + elements;
        const T* row = tensor + at;
        head = static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T));
        base = row - head;
        n = len;
    }
    __device__ __forceinline__ int chunks() const { return (head + n + E - 1) / E; }
    // All of a chunk is in the row's first `len` elements.
    __device__ __forceinline__ bool whole(int chunk, int len) const {
        return chunk * E >= head && (chunk + 1) * E <= head + len;
    }
    // Some of it is past the tensor's ends.
    __device__ __forceinline__ bool outside(int chunk) const {
        const T* p = base + chunk * E;
        return p < first || p + E > last;
    }
    // A chunk of which not all is in the row's first `len` elements, the others -inf.
    __device__ __forceinline__ void load_masked(int chunk, int len, Raw<T, E>& r) const {
        const T* p = base + chunk * E;
        const int lo = head - chunk * E, hi = lo + len;
        float v[E];
#pragma unroll
        for (int j = 0; j < E; ++j) {
            Raw<T, 1> e;
            float w[1] = {-INFINITY};
            if (j >= lo && j < hi) {
                e.load(p + j);
                e.values(w);
            }
            v[j] = w[0];
        }
        r.set(v);
    }
    // Writes what the row has of a chunk to its place in `out`, element by element: 0 past the
    // first `len`.
    __device__ __forceinline__ void store_part(int chunk, const Raw<T, E>& r, int len,
                                               T* out_row) const {
        T* p = out_row - head + chunk * E;
        const int lo = head - chunk * E;
        float v[E];
        r.values(v);
#pragma unroll
        for (int j = 0; j < E; ++j) {
            if (j < lo || j >= lo + n) continue;
            Raw<T, 1> e;
            const float w[1] = {j < lo + len ? v[j] : 0.0f};
            e.set(w);
            e.store(p + j);
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

// Slot k of a row: its class (-1 when empty) and the teacher's logit; `at`: row top + k.
__device__ __forceinline__ long long slot_class(const DistillParams& p, long long at) {
    return p.index64 ? static_cast<const long long*>(p.index)[at]
                     : static_cast<const int*>(p.index)[at];
}
__device__ __forceinline__ float slot_logit(const DistillParams& p, long long at) {
    return p.teacher_f32 ? element(static_cast<const float*>(p.teacher) + at)
                         : element(static_cast<const __nv_bfloat16*>(p.teacher) + at);
}
__device__ __forceinline__ int slot_id(const DistillParams& p, long long id, float t) {
    return id >= 0 && id < p.classes && t != -INFINITY ? static_cast<int>(id) : -1;
}
__device__ __forceinline__ int slot(const DistillParams& p, long long row, int k, float& t) {
    t = slot_logit(p, row * p.top + k);
    return slot_id(p, slot_class(p, row * p.top + k), t);
}

// A sum of 2^((z - m) c) for another maximum.  (Without a number so far, m = -inf, it is 0, or NaN
// from a NaN.)
__device__ __forceinline__ float shifted(float s, float m, float top, float c) {
    return m == -INFINITY ? s : s * ex2_approx_ftz((m - top) * c);
}

// Max and sum over the lanes of a group of `lanes` (a power of two) of a warp.
__device__ __forceinline__ float lanes_max(float v, int lanes) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        if (o < lanes) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ float lanes_sum(float v, int lanes) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        if (o < lanes) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// A row's slots, `top4` (top rounded up to 4) each: the class or -1, the teacher's logit and then p,
// ln p, the student's logit of the class, and what all slots of the class put on it, -1 but in the
// first of them.
constexpr int SLOT_BYTES = 20;
struct Slots {
    int* id;
    float *p, *lnp, *z, *share;
    int top, top4;
    __device__ __forceinline__ Slots(void* at, int slots) {
        top = slots;
        top4 = (slots + 3) & ~3;
        id = static_cast<int*>(at);
        p = reinterpret_cast<float*>(id + top4);
        lnp = p + top4;
        z = lnp + top4;
        share = z + top4;
    }
};

// The teacher's side of a row by a warp: p and ln p of each slot; whether there is one.
__device__ __forceinline__ bool teacher_side(const Slots& s, const DistillParams& p, int lane) {
    float m = -INFINITY, sum = 0.0f;
    bool any = false;
    for (int k = lane; k < s.top; k += 32)
        if (s.id[k] >= 0) {
            m = fmaxf(m, s.p[k]);
            any = true;
        }
    m = lanes_max(m, 32);
    for (int k = lane; k < s.top; k += 32)
        if (s.id[k] >= 0) sum += ex2_approx_ftz((s.p[k] - m) * p.c);
    sum = lanes_sum(sum, 32);
    const float ln_sum = logf(sum), inv = 1.0f / sum;
    for (int k = lane; k < s.top; k += 32)
        if (s.id[k] >= 0) {
            const float x = s.p[k] - m;
            s.p[k] = ex2_approx_ftz(x * p.c) * inv;
            s.lnp[k] = fmaf(x, p.inv_t, -ln_sum);
        }
    return __any_sync(0xffffffffu, any);
}

// A row's loss over T^2 by a warp: slot by slot, so that a student near its teacher loses nothing to
// sums that cancel.  (A slot whose share has vanished has no part, be its class impossible.)
__device__ __forceinline__ float slots_loss(const Slots& s, const DistillParams& p, int lane, float m,
                                            float ln_s) {
    float loss = 0.0f;
    for (int k = lane; k < s.top; k += 32)
        if (s.id[k] >= 0 && !(s.p[k] == 0.0f))
            loss = fmaf(s.p[k], s.lnp[k] - ((s.z[k] - m) * p.inv_t - ln_s), loss);
    return lanes_sum(loss, 32);
}

// What all slots of slot k's class put on it, or -1 where an earlier slot has that class.
__device__ __forceinline__ float class_share(const Slots& s, int k) {
    const int id = s.id[k];
    int same = 0;
    for (int j = 0; j < s.top4; j += 4) {
        const int4 o = *reinterpret_cast<const int4*>(s.id + j);
        same += (o.x == id) + (o.y == id) + (o.z == id) + (o.w == id);
    }
    if (same == 1) return s.p[k];
    float share = 0.0f;
#pragma unroll 1
    for (int j = 0; j < s.top; ++j)
        if (s.id[j] == id) {
            if (j < k) return -1.0f;
            share += s.p[j];
        }
    return share;
}

// 16 bytes to shared memory, asynchronously; a thread waits for its own copies with copies_wait.
__device__ __forceinline__ void copy_async(void* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src)
                 : "memory");
}
__device__ __forceinline__ void copies_commit() {
    asm volatile("cp.async.commit_group;" ::: "memory");
}
template <int N>
__device__ __forceinline__ void copies_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// v becomes 2^((v - at) c); `sum` takes its elements by twos.
template <int N>
__device__ __forceinline__ void powers(float (&v)[N], float at, float c, float2& sum) {
    const float2 a = make_float2(-at, -at), cc = make_float2(c, c);
#pragma unroll
    for (int j = 0; j + 1 < N; j += 2) {
        const float2 x = mul2(add2(make_float2(v[j], v[j + 1]), a), cc);
        v[j] = ex2_approx_ftz(x.x);
        v[j + 1] = ex2_approx_ftz(x.y);
        sum = add2(sum, make_float2(v[j], v[j + 1]));
    }
    if constexpr (N % 2 == 1) {
        v[N - 1] = ex2_approx_ftz((v[N - 1] - at) * c);
        sum.x += v[N - 1];
    }
}
template <int N>
__device__ __forceinline__ void times(float (&v)[N], float f) {
    const float2 ff = make_float2(f, f);
#pragma unroll
    for (int j = 0; j + 1 < N; j += 2) {
        const float2 x = mul2(make_float2(v[j], v[j + 1]), ff);
        v[j] = x.x;
        v[j + 1] = x.y;
    }
    if constexpr (N % 2 == 1) v[N - 1] *= f;
}

// Largest of the elements seen so far; bf16 by twos.
template <typename T, int N>
struct Largest;
template <int N>
struct Largest<float, N> {
    float m = -INFINITY;
    __device__ __forceinline__ void add(const Raw<float, N>& r) {
#pragma unroll
        for (int j = 0; j < N; ++j) m = fmaxf(m, __uint_as_float(r.w[j]));
    }
    __device__ __forceinline__ float get() const { return m; }
};
template <int N>
struct Largest<__nv_bfloat16, N> {
    uint32_t m = 0xFF80FF80u;  // -inf
    __device__ __forceinline__ void add(const Raw<__nv_bfloat16, N>& r) {
#pragma unroll
        for (int j = 0; j < N / 2; ++j)
            asm("max.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(r.w[j]));
    }
    __device__ __forceinline__ float get() const {
        float lo, hi;
        bf16x2_to_f32(m, lo, hi);
        return fmaxf(lo, hi);
    }
};

// ------------------------------------------------------------------ long rows

constexpr int ROW_THREADS = 512, ROW_WARPS = ROW_THREADS / 32, ROW_CLUSTER = 8;

// A row by `parts` blocks of a cluster, NCH chunks of it a thread, which stay in registers between the
// sums and the gradient (what a row has beyond that is read twice, or for the loss alone once, NCH chunks
// on their way together).  The first warp does the teacher's
// side while the row's loads are under way; maximum and sum are joined over warps and, pushed into the
// other blocks' shared memory, over the cluster.
template <typename T, int MODE, int NCH>
__global__ void __launch_bounds__(ROW_THREADS, 2) distill_row_kernel(const DistillParams p,
                                                                     int parts) {
    constexpr int E = RowView<T>::E;
    extern __shared__ int4 dynamic[];
    __shared__ float warp_m[ROW_WARPS], warp_s[ROW_WARPS], part_m[ROW_CLUSTER], part_s[ROW_CLUSTER];
    __shared__ int counts;
    const Slots s(dynamic, p.top);
    griddep_launch_dependents();
    griddep_wait();
    const long long row = blockIdx.x / static_cast<unsigned>(parts);
    const int part = static_cast<int>(blockIdx.x - row * parts);
    const int tid = threadIdx.x, lane = tid & 31, warps = blockDim.x >> 5;
    const T* z = static_cast<const T*>(p.z);
    const RowView<T> view(z, p.rows * p.pitch, row * p.pitch,
                          MODE & GRAD ? static_cast<int>(p.pitch) : p.classes);
    const int chunks = view.chunks(), per = (chunks + parts - 1) / parts;
    const int first = part * per, end = first + per < chunks ? first + per : chunks;
    auto fetch = [&](int i, Raw<T, E>& q) {
        if (view.whole(i, p.classes))
            q.load(view.base + i * E);
        else
            view.load_masked(i, p.classes, q);
    };
    Raw<T, E> r[NCH];
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
        const int i = first + tid + k * static_cast<int>(blockDim.x);
        if (i < end) fetch(i, r[k]);
    }
    const int rest = first + tid + NCH * static_cast<int>(blockDim.x);
    const float g_row = MODE & GRAD && p.dloss ? p.dloss[row] : 1.0f;
    if ((MODE & LOSS) && parts > 1)  // (every block runs: it may be written to)
        asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    // this block's part of the row, for slots: chunk of a class
    auto here = [&](int id) {
        const int chunk = (view.head + id) / E;
        return chunk >= first && chunk < end;
    };
    if (tid < 32) {
        const T* zrow = z + row * p.pitch;
        for (int k = lane; k < s.top4; k += 32) {
            float t = 0.0f;
            const int id = k < s.top ? slot(p, row, k, t) : -1;
            s.id[k] = id;
            s.p[k] = t;
            if (id >= 0 && (((MODE & LOSS) && part == 0) || here(id))) s.z[k] = element(zrow + id);
        }
        __syncwarp();
        const bool some = teacher_side(s, p, lane);
        if (lane == 0) counts = some;
    }
    float m = -INFINITY, sum = 0.0f;
    if (MODE & LOSS) {
        Largest<T, E> largest;
#pragma unroll
        for (int k = 0; k < NCH; ++k)
            if (first + tid + k * static_cast<int>(blockDim.x) < end) largest.add(r[k]);
        m = largest.get();
        const float at = m == -INFINITY ? 0.0f : m;
        float2 sums = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < NCH; ++k) {
            if (first + tid + k * static_cast<int>(blockDim.x) >= end) continue;
            float v[E];
            r[k].values(v);
            powers(v, at, p.c, sums);
        }
        sum = sums.x + sums.y;
        constexpr int U = MODE & GRAD ? 1 : NCH;  // (the gradient's chunks take the registers)
#pragma unroll 1
        for (int i0 = rest; i0 < end; i0 += U * static_cast<int>(blockDim.x)) {
            Raw<T, E> q[U];
            Largest<T, E> other;
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int i = i0 + k * static_cast<int>(blockDim.x);
                if (i < end) fetch(i, q[k]);
            }
#pragma unroll
            for (int k = 0; k < U; ++k)
                if (i0 + k * static_cast<int>(blockDim.x) < end) other.add(q[k]);
            const float top = fmaxf(m, other.get()), now = top == -INFINITY ? 0.0f : top;
            sums = make_float2(shifted(sum, m, now, p.c), 0.0f);
#pragma unroll
            for (int k = 0; k < U; ++k) {
                if (i0 + k * static_cast<int>(blockDim.x) >= end) continue;
                float v[E];
                q[k].values(v);
                powers(v, now, p.c, sums);
            }
            sum = sums.x + sums.y;
            m = top;
        }
        const float top = lanes_max(m, 32);
        sum = lanes_sum(shifted(sum, m, top, p.c), 32);
        if (lane == 0) {
            warp_m[tid >> 5] = top;
            warp_s[tid >> 5] = sum;
        }
    }
    __syncthreads();
    const bool some = counts != 0;
    if (MODE & GRAD)
        for (int k = tid; k < s.top; k += blockDim.x)
            s.share[k] = s.id[k] >= 0 ? class_share(s, k) : -1.0f;
    float inv_s = 1.0f, lse = 0.0f;
    if (MODE & LOSS) {
        const float wm = lane < warps ? warp_m[lane] : -INFINITY;
        m = lanes_max(wm, 32);
        sum = lanes_sum(lane < warps ? shifted(warp_s[lane], wm, m, p.c) : 0.0f, 32);
        if (parts > 1) {
            asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
            if (tid < parts) {
                st_shared_cluster(mapa_shared(smem_u32(part_m + part), tid), __float_as_uint(m));
                st_shared_cluster(mapa_shared(smem_u32(part_s + part), tid), __float_as_uint(sum));
            }
            cluster_sync_all();
            const float pm = lane < parts ? part_m[lane] : -INFINITY;
            m = lanes_max(pm, 32);
            sum = lanes_sum(lane < parts ? shifted(part_s[lane], pm, m, p.c) : 0.0f, 32);
        }
        inv_s = 1.0f / sum;
        const float ln_s = logf(sum);
        lse = fmaf(m, p.inv_t, ln_s);
        if (part == 0 && tid < 32) {
            const float loss = slots_loss(s, p, lane, m, ln_s);
            if (lane == 0) {
                p.loss[row] = some ? p.t2 * loss : 0.0f;
                if (p.lse) p.lse[row] = lse;
            }
        }
    } else {
        lse = p.lse_in[row];
    }
    if (MODE & GRAD) {
        T* out = static_cast<T*>(p.dz) + row * p.pitch;
        const float g = some ? g_row * p.scale : 0.0f;
        auto q_of = [&](float v) {
            return MODE & LOSS ? ex2_approx_ftz((v - m) * p.c) * inv_s
                               : ex2_approx_ftz(fmaf(v, p.inv_t, -lse) * LOG2E);
        };
        const bool aligned = (reinterpret_cast<uintptr_t>(out - view.head) & 15u) == 0;
        auto write = [&](int i, const Raw<T, E>& q) {
            float v[E];
            q.values(v);
            if constexpr (MODE & LOSS) {
                float2 sums = make_float2(0.0f, 0.0f);
                powers(v, m, p.c, sums);
                times(v, g * inv_s);
            } else {
#pragma unroll
                for (int j = 0; j < E; ++j) v[j] = g * q_of(v[j]);
            }
            if (g == 0.0f) {
#pragma unroll
                for (int j = 0; j < E; ++j) v[j] = 0.0f;
            }
            Raw<T, E> o;
            o.set(v);
            if (aligned && view.whole(i, p.classes))
                o.store(out - view.head + i * E);
            else
                view.store_part(i, o, p.classes, out);
        };
#pragma unroll
        for (int k = 0; k < NCH; ++k) {
            const int i = first + tid + k * static_cast<int>(blockDim.x);
            if (i < end) write(i, r[k]);
        }
#pragma unroll 1
        for (int i = rest; i < end; i += blockDim.x) {
            Raw<T, E> q;
            fetch(i, q);
            write(i, q);
        }
        __syncthreads();  // the slots' classes, over what was just written
        for (int k = tid; k < s.top && g != 0.0f; k += blockDim.x) {
            const int id = s.id[k];
            if (id >= 0 && s.share[k] != -1.0f && here(id))
                put(out + id, g * (q_of(s.z[k]) - s.share[k]));
        }
    }
}

// ------------------------------------------------------------------ many long rows

__device__ __forceinline__ void named_bar_arrive(int id, int count) {
    asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(count) : "memory");
}

// Whole rows, one after the other, by CT threads with NCH chunks each at most and H warps beside
// them for the slots.  Two rows are on their way into shared memory while one is worked on: a thread
// copies, and later reads, its own chunks, so no barrier stands between.  It takes its powers against
// its own maximum and keeps them: one power an element, and a factor a thread,
// 2^((own max - max) c) g / S, once the row's maximum and sum are known.  Helper warp h joins the
// warps' sums of every H-th row, while they take the next row's maximum, and does its slots ahead of
// time, its loss, and its classes' elements behind the others.  (The gradient alone has its lse, and
// nothing to join.)
//
// 4096 x 32768 bf16, loss and gradient: 89.7 us, 89% of the bytes' floor (101 where the threads wait
// for the joined sums with nothing else to do, 156 with two powers an element and bounds at every
// chunk).  Rows that fill fewer threads take blocks of 256 or 128, two to four an SM; of those one
// helper a block was the slower side (20,000 x 3000, loss: 90 us; 45 with two, in bf16 as in fp32).
//
// A helper's time grows with the slots, and past its rows' share of the threads' it bounds the row: loss
// of 20,000 x 3000 bf16 47 us with 16 slots, 61 with 64, 87 with 128, 112 with 192; loss and gradient of
// 4096 x 16,000 bf16 47, 60, 86 and 119, where each slot is compared with every other.  Past about 200
// slots the loss of rows that fill 128 threads has blocks of too much shared memory for four an SM, which
// its grid counts on: the fourth quarter runs as a second wave (267 us with 256).
template <typename T, int MODE, int CT_>
struct RingCfg {
    // Helper warps: fp32 keeps half the powers, which leaves four room beside fewer threads too
    // (8000 x 4000, loss and gradient: 45 us, 57 with two; in bf16 they spill: 101 and 68 for
    // 10,000 x 5001).
    static constexpr bool GRADIENT = (MODE & GRAD) != 0;
    static constexpr int CT = CT_, NCH = 8, H = CT == 512 || (GRADIENT && sizeof(T) == 4) ? 4 : 2;
    static constexpr int THREADS = CT + 32 * H;
    static constexpr int STAGES = 3;
    static constexpr int STAGE_CHUNKS = NCH * CT;
    // Blocks an SM: with powers kept, three of 128 threads, which have 113 or 85 registers.
    static constexpr int BLOCKS = GRADIENT && CT == 128 ? 3 : 512 / CT;
    static size_t smem(int top) {
        return size_t(16) * STAGES * STAGE_CHUNKS + size_t(SLOT_BYTES) * H * ((top + 3) & ~3);
    }
};

// `most`: chunks of any row at most.
template <typename T, int MODE, int CT>
__global__ void __launch_bounds__(RingCfg<T, MODE, CT>::THREADS, RingCfg<T, MODE, CT>::BLOCKS)
    distill_ring_kernel(const DistillParams p, int most) {
    using C = RingCfg<T, MODE, CT>;
    constexpr int E = RowView<T>::E, H = C::H, NCH = C::NCH, WARPS = CT / 32;
    extern __shared__ int4 dynamic[];
    // the warps' maxima and sums of two rows in turn, and what a helper makes of them
    __shared__ float sum_m[2][WARPS], sum_s[2][WARPS], row_m[H], row_f[H];
    griddep_launch_dependents();
    griddep_wait();
    const int tid = threadIdx.x, lane = tid & 31;
    const T* z = static_cast<const T*>(p.z);
    const long long step = gridDim.x;
    const int len = MODE & GRAD ? static_cast<int>(p.pitch) : p.classes;
    if (tid < CT) {
        int4* ring = dynamic + tid;
        auto view_of = [&](long long row) {  // (its loads stay in the row: no look at the tensor's ends)
            return RowView<T>(z, 0, row * p.pitch, len);
        };
        // Of a thread's chunks, the first `wholes` are all classes (but for chunk 0 of a row that does
        // not begin on a chunk).
        auto wholes = [&](const RowView<T>& view) {
            const int n = (view.head + p.classes) / E - tid + CT - 1;
            return n < CT ? 0 : n / CT;
        };
        auto fetch = [&](long long row, int stage) {
            if (row < p.rows) {
                const RowView<T> view = view_of(row);
                const int n = wholes(view);
                const bool part0 = tid == 0 && view.head != 0;
                int4* dst = ring + stage * C::STAGE_CHUNKS;
                const T* src = view.base + tid * E;
#pragma unroll
                for (int k = 0; k < NCH; ++k)
                    if (k < n && !(k == 0 && part0)) copy_async(dst + k * CT, src + k * CT * E);
                // its other chunks, up to what any row has: -inf where there is no class
                if (part0) {
                    Raw<T, E> r;
                    view.load_masked(0, p.classes, r);
                    r.store(reinterpret_cast<T*>(dst));
                }
#pragma unroll 1
                for (int i = tid + (n == 0 && part0 ? 1 : n) * CT; i < most; i += CT) {
                    Raw<T, E> r;
                    view.load_masked(i, p.classes, r);
                    r.store(reinterpret_cast<T*>(dst + (i - tid)));
                }
            }
            copies_commit();
        };
        // chunks that no row has
        for (int i = tid + (most - tid + CT - 1) / CT * CT; i < C::STAGES * C::STAGE_CHUNKS; i += CT)
            if (i % C::STAGE_CHUNKS >= most) {
                Raw<T, E> r;
#pragma unroll
                for (int j = 0; j < 4; ++j) r.w[j] = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;
                r.store(reinterpret_cast<T*>(dynamic + i));
            }
        long long row = blockIdx.x;
        fetch(row, 0);
        fetch(row + step, 1);
        int stage = 0, h = 0, buf = 0;
        // largest of this thread's elements of the row in a stage
        auto largest_of = [&](int st) {
            const T* from = reinterpret_cast<const T*>(ring + st * C::STAGE_CHUNKS);
            Largest<T, E> largest;
#pragma unroll
            for (int k = 0; k < NCH; ++k)
                if ((k & ~1) * CT < most) {
                    Raw<T, E> r;
                    r.load(from + k * CT * E);
                    largest.add(r);
                }
            return largest.get();
        };
        copies_wait<1>();
        float m = MODE & LOSS ? largest_of(0) : 0.0f;
        for (; row < p.rows; row += step) {
            // (the stage that this overwrites was read a row ago, by this thread)
            fetch(row + 2 * step, stage == 0 ? 2 : stage - 1);
            T* mine = reinterpret_cast<T*>(ring + stage * C::STAGE_CHUNKS);
            float e[NCH][E];
            const float at = m == -INFINITY ? 0.0f : m;
            float2 sums = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int k = 0; k < NCH; ++k)
                if ((k & ~1) * CT < most) {
                    Raw<T, E> r;
                    r.load(mine + k * CT * E);
                    r.values(e[k]);
                    if (MODE & LOSS) powers(e[k], at, p.c, sums);
                }
            stage = stage == 2 ? 0 : stage + 1;
            if (MODE & LOSS) {
                const float top = lanes_max(m, 32);
                const float sum = lanes_sum(shifted(sums.x + sums.y, m, top, p.c), 32);
                if (lane == 0) {
                    sum_m[buf][tid >> 5] = top;
                    sum_s[buf][tid >> 5] = sum;
                }
                named_bar_arrive(1 + h, CT + 32);
            }
            copies_wait<1>();  // (past the last row: nothing is under way, and what is read not used)
            if (MODE & LOSS) m = largest_of(stage);
            named_bar_sync(1 + H + h, CT + 32);
            if (MODE & GRAD) {
                const float g = row_f[h], of_row = row_m[h];
                // (a thread with no finite logit has at = 0, which may be far above the row's maximum)
                const float f =
                    MODE & LOSS ? ex2_approx_ftz(fminf((at - of_row) * p.c, 0.0f)) * g : g;
                if (!(MODE & LOSS)) {
#pragma unroll
                    for (int k = 0; k < NCH; ++k)
                        if ((k & ~1) * CT < most) {
#pragma unroll
                            for (int j = 0; j < E; ++j)
                                e[k][j] = ex2_approx_ftz(fmaf(e[k][j], p.inv_t, -of_row) * LOG2E);
                        }
                }
                const RowView<T> view = view_of(row);
                T* out = static_cast<T*>(p.dz) + row * p.pitch;
                T* place = out - view.head + tid * E;
                const bool part0 = tid == 0 && view.head != 0;
                const int n = (reinterpret_cast<uintptr_t>(place) & 15u) == 0 ? wholes(view) : 0;
                const uint32_t keep = g == 0.0f ? 0u : ~0u;  // (0 whatever the logits are)
                const int chunks = view.chunks();
                // chunks that are not all classes, or not on 16 bytes: back to their place in the
                // ring until the next row is fetched there, and from there element by element
                // (what no row has keeps its -inf)
                const bool parts = part0 || tid + n * CT < chunks;
#pragma unroll
                for (int k = 0; k < NCH; ++k)
                    if ((k & ~1) * CT < most) {
                        Raw<T, E> o;
                        times(e[k], f);
                        o.set(e[k]);
#pragma unroll
                        for (int j = 0; j < 4; ++j) o.w[j] &= keep;
                        if (k < n && (k > 0 || !part0)) o.store(place + k * CT * E);
                    }
                if (parts) {
#pragma unroll
                    for (int k = 0; k < NCH; ++k)
                        if (((k == 0 && part0) || k >= n) && tid + k * CT < chunks) {
                            Raw<T, E> o;
                            o.set(e[k]);
#pragma unroll
                            for (int j = 0; j < 4; ++j) o.w[j] &= keep;
                            o.store(mine + k * CT * E);
                        }
                    auto part = [&](int i) {
                        Raw<T, E> o;
                        o.load(mine + (i - tid) * E);
                        view.store_part(i, o, p.classes, out);
                    };
                    if (part0 && n > 0) part(0);
#pragma unroll 1
                    for (int i = tid + n * CT; i < chunks; i += CT) part(i);
                }
                named_bar_arrive(1 + 2 * H + h, CT + 32);
            }
            h = h == H - 1 ? 0 : h + 1;
            buf ^= 1;
        }
        return;
    }
    const int h = (tid - CT) >> 5;
    const Slots s(reinterpret_cast<char*>(dynamic + C::STAGES * C::STAGE_CHUNKS) +
                      h * ((p.top + 3) & ~3) * SLOT_BYTES, p.top);
    const int buf = h & 1;
    // A lane's first slot and the row's weight are loaded a turn ahead, the student's logit behind
    // the loss (a row's logits are overwritten only after its helper has come to its sums).
    long long row = blockIdx.x + h * step, raw = -1;
    float t0 = 0.0f, z0 = 0.0f, weight = 1.0f, lse0 = 0.0f;
    auto ahead = [&](long long r) {
        raw = -1;
        if (r >= p.rows) return;
        if (MODE & GRAD && p.dloss) weight = p.dloss[r];
        if (MODE == GRAD) lse0 = p.lse_in[r];
        if (lane < s.top) {
            raw = slot_class(p, r * p.top + lane);
            t0 = slot_logit(p, r * p.top + lane);
        }
    };
    auto gather = [&](long long r) {
        const int id = slot_id(p, raw, t0);
        if (id >= 0) z0 = element(z + r * p.pitch + id);
    };
    ahead(row);
    gather(row);
    for (; row < p.rows; row += H * step) {
        const T* zrow = z + row * p.pitch;
        const float g_row = weight, lse = lse0;
        if (lane < s.top4) {
            s.id[lane] = slot_id(p, raw, t0);
            s.p[lane] = t0;
            s.z[lane] = z0;
        }
        ahead(row + H * step);
        for (int k = lane + 32; k < s.top4; k += 32) {
            float t = 0.0f;
            const int id = k < s.top ? slot(p, row, k, t) : -1;
            s.id[k] = id;
            s.p[k] = t;
            if (id >= 0) s.z[k] = element(zrow + id);
        }
        __syncwarp();
        const bool some = teacher_side(s, p, lane);
        if (MODE & GRAD) {
            __syncwarp();
            for (int k = lane; k < s.top; k += 32)
                s.share[k] = s.id[k] >= 0 ? class_share(s, k) : -1.0f;
        }
        const float g = some ? g_row * p.scale : 0.0f;
        float m = lse, inv_s = 1.0f;
        if (MODE & LOSS) {
            named_bar_sync(1 + h, CT + 32);
            const float wm = lane < WARPS ? sum_m[buf][lane] : -INFINITY;
            m = lanes_max(wm, 32);
            const float sum =
                lanes_sum(lane < WARPS ? shifted(sum_s[buf][lane], wm, m, p.c) : 0.0f, 32);
            inv_s = 1.0f / sum;
            if (lane == 0) {
                row_m[h] = m;
                row_f[h] = g == 0.0f ? 0.0f : g * inv_s;
            }
            __syncwarp();
            named_bar_arrive(1 + H + h, CT + 32);
            const float ln_s = logf(sum), loss = slots_loss(s, p, lane, m, ln_s);
            if (lane == 0) {
                p.loss[row] = some ? p.t2 * loss : 0.0f;
                if (p.lse) p.lse[row] = fmaf(m, p.inv_t, ln_s);
            }
        } else {
            if (lane == 0) {
                row_m[h] = lse;
                row_f[h] = g;
            }
            __syncwarp();
            named_bar_arrive(1 + H + h, CT + 32);
        }
        gather(row + H * step);
        if (MODE & GRAD) {
            named_bar_sync(1 + 2 * H + h, CT + 32);
            T* out = static_cast<T*>(p.dz) + row * p.pitch;
            for (int k = lane; k < s.top && g != 0.0f; k += 32)
                if (s.id[k] >= 0 && s.share[k] != -1.0f)
                    put(out + s.id[k],
                        g * ((MODE & LOSS ? ex2_approx_ftz((s.z[k] - m) * p.c) * inv_s
                                          : ex2_approx_ftz(fmaf(s.z[k], p.inv_t, -m) * LOG2E)) -
                             s.share[k]));
        }
        __syncwarp();
        static_assert(H % 2 == 0, "a helper's rows have one buffer of sums");
    }
}

// Chunks of a row at most: one more than its bytes where rows do not begin on a chunk.
int row_chunks(const DistillParams& p, int size) {
    const long long bytes = p.pitch * size;
    const bool whole = (static_cast<uintptr_t>(bytes) | reinterpret_cast<uintptr_t>(p.z)) % 16 == 0;
    return static_cast<int>((bytes + 15) / 16) + (whole ? 0 : 1);
}

template <typename T, int MODE, int CT>
cudaError_t launch_distill_ring(const DistillParams& p, int num_sms, cudaStream_t stream) {
    using C = RingCfg<T, MODE, CT>;
    auto* kern = distill_ring_kernel<T, MODE, CT>;
    static std::atomic<unsigned long long> ready{0};  // once a device: the shared memory
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !((ready.load(std::memory_order_acquire) >> dev) & 1ull)) {
        e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 static_cast<int>(C::smem(DISTILL_TOP)));
        if (e != cudaSuccess) return e;
        if (dev < 64) ready.fetch_or(1ull << dev, std::memory_order_release);
    }
    const long long most = static_cast<long long>(num_sms) * C::BLOCKS;
    const dim3 g(static_cast<unsigned>(p.rows < most ? p.rows : most));
    return launch_pdl(kern, g, dim3(C::THREADS), C::smem(p.top), stream, p,
                      row_chunks(p, sizeof(T)));
}

// ------------------------------------------------------------------ short rows

constexpr int TILE_THREADS = 256;

// Blocks an SM that the compiler is asked for: loss and gradient in bf16 keep two powers a word, and
// gain from a block more than they would get (60,000 rows of 1000: 80 us without, 74 with four); for
// the others it is left to choose (0).
constexpr int tile_blocks(int size, int mode, int words) {
    return size == 2 && mode == (LOSS | GRAD) && words <= 16 ? (words <= 8 ? 5 : 4) : 0;
}

// A tile of 256 / LANES rows a block.  The rows lie one after the other, so the tile is read and
// written in whole chunks wherever its rows begin; in shared memory a row is LANES lanes of a warp, at
// most W of its 4-byte words and K of its slots each, whose powers stay in registers, and the gradient
// takes the logits' place: 100,352 x 100 bf16 with ten slots 17.6 us, bound by its instructions (31 with
// the slots in shared memory and each compared with every other).  A class that several slots have shows by a byte a class: each slot writes
// its number there and looks whether it still stands.
template <typename T, int MODE, int LANES, int W, int K>
__global__ void __launch_bounds__(TILE_THREADS, tile_blocks(sizeof(T), MODE, W))
    distill_tile_kernel(const DistillParams p) {
    constexpr int E = RowView<T>::E, N = 4 / static_cast<int>(sizeof(T));
    constexpr int ROWS = TILE_THREADS / LANES;
    extern __shared__ int4 dynamic[];
    griddep_launch_dependents();
    griddep_wait();
    const int tid = threadIdx.x, tr = tid / LANES, lane = tid % LANES;
    const long long row0 = static_cast<long long>(blockIdx.x) * ROWS, row = row0 + tr;
    const int rows = p.rows - row0 < ROWS ? static_cast<int>(p.rows - row0) : ROWS;
    const int pitch = static_cast<int>(p.pitch);
    const RowView<T> view(static_cast<const T*>(p.z), p.rows * p.pitch, row0 * p.pitch,
                          rows * pitch);
    const int chunks = view.chunks();
    int4* tile = dynamic;
    uint8_t* owner =
        reinterpret_cast<uint8_t*>(tile + (ROWS * pitch + E - 1) / E + 1) + tr * pitch;
    for (int i = tid; i < chunks; i += TILE_THREADS) {
        if (!view.outside(i)) {
            copy_async(tile + i, view.base + i * E);
        } else {
            Raw<T, E> r;
            view.load_masked(i, view.n, r);
            r.store(reinterpret_cast<T*>(tile + i));
        }
    }
    copies_commit();
    // the teacher's side: p, and the sum of p ln p
    const bool active = tr < rows;
    long long raw[K];
    float t[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const long long at = row * p.top + lane + k * LANES;
        raw[k] = -1;
        t[k] = 0.0f;
        if (active && lane + k * LANES < p.top) {
            raw[k] = slot_class(p, at);
            t[k] = slot_logit(p, at);
        }
    }
    float g = MODE & GRAD && p.dloss && active ? p.dloss[row] : 1.0f;
    float lse = MODE == GRAD && active ? p.lse_in[row] : 0.0f;
    int id[K];
    float tm = -INFINITY;
    bool any = false;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        id[k] = slot_id(p, raw[k], t[k]);
        if (id[k] >= 0) {
            tm = fmaxf(tm, t[k]);
            any = true;
        }
    }
    tm = lanes_max(tm, LANES);
    const unsigned votes = __ballot_sync(0xffffffffu, any);
    const unsigned of_row = (0xffffffffu >> (32 - LANES)) << ((tid & 31) - lane);
    const bool some = (votes & of_row) != 0;
    float ts = 0.0f, lnp[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        lnp[k] = t[k] - tm;
        t[k] = id[k] >= 0 ? ex2_approx_ftz(lnp[k] * p.c) : 0.0f;
        ts += t[k];
    }
    ts = lanes_sum(ts, LANES);
    const float inv_ts = 1.0f / ts, ln_ts = logf(ts);
    // the share of each class, in the first of its slots
    bool lost = false;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        lnp[k] = fmaf(lnp[k], p.inv_t, -ln_ts);
        t[k] *= inv_ts;
        if (id[k] >= 0) owner[id[k]] = static_cast<uint8_t>(lane + k * LANES);
    }
    __syncwarp();
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (id[k] >= 0) lost = lost || owner[id[k]] != lane + k * LANES;
    if (__any_sync(0xffffffffu, lost)) {
        // (the first slot stands for all of its class, their p ln p included)
        float share[K], sum[K];
        bool first[K];
#pragma unroll
        for (int k = 0; k < K; ++k) share[k] = sum[k] = 0.0f, first[k] = true;
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll 1
            for (int l = 0; l < LANES; ++l) {
                const int from = (tid & 31) - lane + l;
                const int other = __shfl_sync(0xffffffffu, id[j], from);
                const float part = __shfl_sync(0xffffffffu, t[j], from);
                const float ln = __shfl_sync(0xffffffffu, lnp[j], from);
#pragma unroll
                for (int k = 0; k < K; ++k)
                    if (other == id[k] && other >= 0) {
                        share[k] += part;
                        if (!(part == 0.0f)) sum[k] = fmaf(part, ln, sum[k]);
                        if (l + j * LANES < lane + k * LANES) first[k] = false;
                    }
            }
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (id[k] >= 0) {
                if (share[k] != t[k]) lnp[k] = sum[k] / share[k];
                t[k] = share[k];
                if (!first[k]) id[k] = -1;
            }
    }
    copies_wait<0>();
    __syncthreads();
    // the row's words: `odd` elements of the row before it stand in the first one
    T* mine = reinterpret_cast<T*>(tile) + view.head + tr * pitch;
    const int odd = N == 2 ? (view.head + tr * pitch) & 1 : 0;
    T* words = mine - odd;
    const int classes = active ? p.classes : 0;
    float v[W][N];
    Largest<T, N> largest;
#pragma unroll
    for (int j = 0; j < W; ++j) {
        const int e0 = N * (lane + j * LANES) - odd;  // element of the word's first
        Raw<T, N> r;
        r.w[0] = N == 2 ? 0xFF80FF80u : 0xFF800000u;  // -inf
        if (e0 < classes) r.load(words + N * (lane + j * LANES));
        if (N == 2 && j == 0 && e0 < 0) r.w[0] = (r.w[0] & 0xFFFF0000u) | 0xFF80u;
        if (N == 2 && e0 + 1 >= classes) r.w[0] = (r.w[0] & 0xFFFFu) | 0xFF800000u;
        if (MODE & LOSS) largest.add(r);
        r.values(v[j]);
    }
    float m = 0.0f, ln_s = 0.0f, inv_s = 1.0f;
    if (MODE & LOSS) {
        m = lanes_max(largest.get(), LANES);
        const float at = m == -INFINITY ? 0.0f : m;
        float2 sums = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int j = 0; j < W; ++j) {
                powers(v[j], at, p.c, sums);
        }
        const float sum = lanes_sum(sums.x + sums.y, LANES);
        inv_s = 1.0f / sum;
        ln_s = logf(sum);
        lse = fmaf(m, p.inv_t, ln_s);
    }
    g = some ? g * p.scale : 0.0f;
    auto q_of = [&](float x) {
        return MODE & LOSS ? ex2_approx_ftz((x - m) * p.c) * inv_s
                           : ex2_approx_ftz(fmaf(x, p.inv_t, -lse) * LOG2E);
    };
    float loss = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (id[k] < 0) continue;
        const float z = element(mine + id[k]);
        if (MODE & LOSS)  // (slot by slot, as slots_loss)
            if (!(t[k] == 0.0f)) loss = fmaf(t[k], lnp[k] - ((z - m) * p.inv_t - ln_s), loss);
        if (MODE & GRAD) t[k] = g * (q_of(z) - t[k]);  // the gradient there
    }
    if (MODE & LOSS) {
        loss = lanes_sum(loss, LANES);
        if (active && lane == 0) {
            p.loss[row] = some ? p.t2 * loss : 0.0f;
            if (p.lse) p.lse[row] = lse;
        }
    }
    if (MODE & GRAD) {
        __syncwarp();  // every slot's logit is read
        const float gs = g * inv_s;
        const uint32_t keep = g == 0.0f ? 0u : ~0u;  // (0 whatever the logits are)
        const int end = active ? pitch : -1;
#pragma unroll
        for (int j = 0; j < W; ++j) {
                const int e0 = N * (lane + j * LANES) - odd;
            if (!(MODE & LOSS)) {
#pragma unroll
                for (int i = 0; i < N; ++i) v[j][i] = q_of(v[j][i]);
            }
            times(v[j], gs);
            Raw<T, N> r;
            r.set(v[j]);
            r.w[0] &= keep;
            if (e0 + N > p.classes) r.w[0] &= e0 + 1 == p.classes ? 0xFFFFu : 0u;  // padding
            T* at = words + N * (lane + j * LANES);
            if (N == 1 ? e0 < end : (j > 0 || e0 >= 0) && e0 + 1 < end) {
                r.store(at);
            } else if (N == 2 && e0 < end) {  // a word that two rows share
                const bool high = j == 0 && e0 < 0;
                *reinterpret_cast<unsigned short*>(high ? at + 1 : at) =
                    static_cast<unsigned short>(high ? r.w[0] >> 16 : r.w[0]);
            }
        }
        __syncwarp();
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (id[k] >= 0 && g != 0.0f) put(mine + id[k], t[k]);
        __syncthreads();
        T* out = static_cast<T*>(p.dz) + row0 * p.pitch;
        const bool aligned = (reinterpret_cast<uintptr_t>(out - view.head) & 15u) == 0;
        for (int i = tid; i < chunks; i += TILE_THREADS) {
            Raw<T, E> r;
            r.load(reinterpret_cast<const T*>(tile + i));
            if (aligned && view.whole(i, view.n))
                r.store(out - view.head + i * E);
            else
                view.store_part(i, r, view.n, out);
        }
    }
}

size_t tile_bytes(const DistillParams& p, int size, int lanes) {
    const size_t rows = TILE_THREADS / lanes;
    return ((rows * p.pitch * size + 15) / 16 + 1) * 16 + rows * p.pitch;
}

template <typename T, int MODE, int LANES, int W, int K>
cudaError_t launch_distill_tile(const DistillParams& p, cudaStream_t stream) {
    constexpr int ROWS = TILE_THREADS / LANES;
    return launch_pdl(distill_tile_kernel<T, MODE, LANES, W, K>,
                      dim3(static_cast<unsigned>((p.rows + ROWS - 1) / ROWS)), dim3(TILE_THREADS),
                      tile_bytes(p, sizeof(T), LANES), stream, p);
}

// The least multiple of four words a lane that holds a row (100,000 rows of 300 bf16 with 32 slots, ten
// words of 16: 69 us with 16, 55 with 12).
template <typename T, int MODE, int LANES>
cudaError_t launch_distill_lanes(const DistillParams& p, int words, cudaStream_t stream) {
    return words <= 8    ? launch_distill_tile<T, MODE, LANES, 8, 4>(p, stream)
           : words <= 12 ? launch_distill_tile<T, MODE, LANES, 12, 4>(p, stream)
                         : launch_distill_tile<T, MODE, LANES, 16, 4>(p, stream);
}

template <typename T, int MODE>
cudaError_t launch_distill_mode(const DistillParams& p, int num_sms, cudaStream_t stream) {
    constexpr int size = static_cast<int>(sizeof(T));
    constexpr size_t SMEM = 48 << 10;
    // a row's words, with one that it may share: up to 16 and four slots a lane, up to 32 and eight
    // of a whole warp
    const bool even = (static_cast<uintptr_t>(p.pitch * size) | reinterpret_cast<uintptr_t>(p.z)) % 4 == 0;
    const long long words = p.pitch * size / 4 + (even ? 0 : 1);
    if (words <= 32 * 32) {
        int lanes = 4;
        while (lanes < 32 && (16 * lanes < words || 4 * lanes < p.top ||
                              tile_bytes(p, size, lanes) > SMEM))
            lanes *= 2;
        if (tile_bytes(p, size, lanes) <= SMEM) {
            const int each = static_cast<int>((words + lanes - 1) / lanes);  // words a lane
            if (p.top > 4 * lanes) return launch_distill_tile<T, MODE, 32, 32, 8>(p, stream);
            if (each > 16) return launch_distill_tile<T, MODE, 32, 32, 4>(p, stream);
            switch (lanes) {
                case 4: return launch_distill_lanes<T, MODE, 4>(p, each, stream);
                case 8: return launch_distill_lanes<T, MODE, 8>(p, each, stream);
                case 16: return launch_distill_lanes<T, MODE, 16>(p, each, stream);
                default: return launch_distill_lanes<T, MODE, 32>(p, each, stream);
            }
        }
    }
    // blocks of a row: as many as its chunks need to stay in registers, more while there are
    // fewer blocks than SMs and a block keeps 256 chunks; the loss of longer rows keeps nothing, and
    // takes two blocks an SM (1000 x 100,000 fp32: 80 us, 185 with eight blocks a row)
    const int n = row_chunks(p, size);
    int parts = 1;
    const bool keeps = (MODE & GRAD) != 0 || n <= ROW_THREADS * 8;
    while (parts < ROW_CLUSTER &&
           (keeps ? n > parts * ROW_THREADS * 8 || (2 * parts * p.rows <= num_sms && n >= 512 * parts)
                  : parts * p.rows < 2 * num_sms))
        parts *= 2;
    const int per = (n + parts - 1) / parts;
    if (parts == 1 && n <= ROW_THREADS * 8) {
        // the gradient alone: rows that keep most of a ring's chunks busy, four a block or more
        // (4096 x 32768 bf16 84 us, 120 by a block a row; 1300 x 10007 fp32 26 and 21)
        if constexpr (MODE == GRAD) {
            if (n > ROW_THREADS * 6 && p.rows >= 4LL * num_sms)
                return launch_distill_ring<T, MODE, 512>(p, num_sms, stream);
        } else {
            if (n <= 1024) return launch_distill_ring<T, MODE, 128>(p, num_sms, stream);
            if (n <= 2048) return launch_distill_ring<T, MODE, 256>(p, num_sms, stream);
            return launch_distill_ring<T, MODE, 512>(p, num_sms, stream);
        }
    }
    const bool wide = per > 4 * ROW_THREADS;
    int threads = (per + (wide ? 8 : 4) - 1) / (wide ? 8 : 4);
    threads = threads < 128 ? 128 : threads > ROW_THREADS ? ROW_THREADS : (threads + 31) & ~31;
    const size_t smem = static_cast<size_t>((p.top + 3) & ~3) * SLOT_BYTES;
    const dim3 g(static_cast<unsigned>(p.rows * parts)), b(static_cast<unsigned>(threads));
    const unsigned cluster = MODE & LOSS ? static_cast<unsigned>(parts) : 1u;
    return wide ? launch_pdl_cluster(distill_row_kernel<T, MODE, 8>, g, b, cluster, smem, stream, p,
                                     parts)
                : launch_pdl_cluster(distill_row_kernel<T, MODE, 4>, g, b, cluster, smem, stream, p,
                                     parts);
}

template <typename T>
cudaError_t launch_distill_t(const DistillParams& p, int num_sms, cudaStream_t stream) {
    if (!p.dz) return launch_distill_mode<T, LOSS>(p, num_sms, stream);
    return p.loss ? launch_distill_mode<T, LOSS | GRAD>(p, num_sms, stream)
                  : launch_distill_mode<T, GRAD>(p, num_sms, stream);
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
    return a.f32 ? launch_distill_t<float>(p, num_sms, stream)
                 : launch_distill_t<__nv_bfloat16>(p, num_sms, stream);
}

}  // namespace quan
