// qpoint_f8_tc.cuh -- the 8-bit pointwise product on the tensor cores.  Included by qpoint_f8.cu
// inside its anonymous namespace.
//
// A tile is 128 rows x BNQ quaternion output channels, all four output components.  For one
// K block b (128 channels) and one input component ci a single MMA chain multiplies the rows'
// component ci by the four letters stacked, N = 4 BNQ columns in the order r, i, j, k:
//   P[m][L BNQ + n] = sum over k in b of q_x[m][ci][k] q_w[L][n][k]        (M 128, K 128)
// and column group L of it belongs to output component co = L xor ci.  So the Hamilton product's
// signs and its exchange of components cost nothing: the operands stay as they are in memory,
// the letters of a K block serve all four input components (32 KB beside 4 x 16 KB of rows for
// 4 x 512 clocks of MMAs, half of what a plain 128 x 256 tile of the real block matrix copies),
// and the epilogue threads of component co read column group co xor ci and add it times
//   sgn(co, ci) s_x[ci][b][m] s_w[L][b]
// to their fp32 accumulators.  The scales change every 128 channels, so no sum runs in the tensor
// core for longer than that.  Bound: the MMAs (8192 products a clock and SM) as long as a
// partial's 128 x 256 values are taken out of TMEM, one fused multiply-add each (256 clocks of
// the SM's FMA lanes), in the 512 clocks that the next partial's MMAs take: hence two TMEM
// buffers, and eight epilogue warps that load a chunk of columns while they add the one before.
// A thread keeps 2 x BNQ accumulators, so the epilogue's two warpgroups take registers that the
// other warps hand back.  The factors are multiplied by a warp of their own, a K block ahead, into
// shared memory: loaded by the epilogue's threads they put a load's latency, 500 clocks, into
// every block (495 against 452 us for 25,600 rows 4096 -> 4096).
//
// What bounds it now: a buffer's round trip.  A partial's MMAs take 514 clocks, and 390 more pass
// from their issue to their arrival at the epilogue; taking the partial out takes the slowest of
// eight warps about 700, the way back to the issuer 200; two buffers make that about 1000 clocks a
// partial: 25,600 rows 4096 -> 4096 365 us, 2.35 PFLOP/s.  Buffers of 128 columns, twice as many,
// hide the trip, but an MMA of 128 columns takes 94 clocks, not 64 (the rows' operand is read
// again): as two halves of a tile 511 us for the call that takes 420; as tiles of 32 channels on two
// CTAs an SM 437, bound by the copies from L2, 39 bytes a clock and SM.
//
// BNQ = 64, 32 or 16: with few row tiles the narrower ones spread the letters over more SMs (see
// f8_tile_width).
//
// Roles (12 warps, one CTA per SM, persistent over tiles, channel tiles first):
//   warp 0      TMA producer: per K block the letters' box, then the rows' box of each component;
//   warps 1, 2  MMA issuers, one a TMEM buffer, taking partials in turn: the waits and commits of
//               the one pass while the other's MMAs run, 5% over one issuer (warp 1 owns TMEM);
//   warp 3      the factors of a K block: sgn(co, ci) s_x s_w for the tile's rows;
//   warps 4..11 epilogue: components 2 g and 2 g + 1 of warpgroup g = 0 or 1 (warps 4..7, 8..11),
//               TMEM lane quadrant warp mod 4.
// Waits are bounded like every kernel here (tc_common.cuh).

constexpr int F8_THREADS = 12 * 32;
constexpr int F8_EPI_WARP0 = 4;
constexpr int F8_EPI_WARPS = 8;
constexpr int F8_BM = 128;
// Registers a thread: at launch, and after the warpgroups' exchange.  An increase waits until
// the block's own registers cover it, so the shares must not pass the launch's total.
constexpr int F8_REGS = 168, F8_REGS_ISSUE = 56, F8_REGS_EPI = 224;
static_assert(128 * F8_REGS_ISSUE + 256 * F8_REGS_EPI <= F8_THREADS * F8_REGS, "register shares");

struct F8TcParams {
    const float* xs;  // [4][kblk][pitch]
    const float* ws;  // [4][nblk][kblk]
    EpilogueArgs ep;
    __nv_bfloat16* out;  // [rows][4 Nq]
    long long rows;
    long long pitch;  // rows rounded up to whole tiles
    int Kq, Nq, kblk, nblk;
    int conj, act;
    int ntiles, num_tiles;
    int store;  // how the output leaves (f8_store_tile), by Nq and its alignment
    unsigned long long wait_limit_ns;
    int inject_stall;
};

template <int BNQ>
struct F8Cfg {
    static constexpr int A_STAGE = F8_BM * F8_BLOCK;    // one component of 128 rows: 16 KB
    static constexpr int B_STAGE = 4 * BNQ * F8_BLOCK;  // four letters
    static constexpr int A_STAGES = 4, B_STAGES = 2;  // a K block of rows, two of letters
    static constexpr int RING = A_STAGES * A_STAGE + B_STAGES * B_STAGE;
    static constexpr int VEC = F8_EPI_WARPS * 2 * 2 * BNQ * 4;  // each epilogue warp's vectors
    static constexpr int OUT_PITCH = 2 * BNQ + 16;  // staged output row: no bank twice in a quarter
    static constexpr int OUT = F8_EPI_WARPS * 32 * OUT_PITCH;
    static constexpr int S_STAGES = 2, S_STAGE = 4 * 4 * F8_BM * 4;  // factors of a K block: 8 KB
    static constexpr int SCALES = S_STAGES * S_STAGE;
    // full and done (A), full and empty (B, factors), acce (2 buffers), drain (2 issuers)
    static constexpr int NUM_BARS = 2 * (A_STAGES + B_STAGES + S_STAGES) + 2 + 2;
    static constexpr int SMEM_BYTES = 1024 + RING + SCALES + OUT + VEC + NUM_BARS * 8 + 32;
    static constexpr uint32_t DESC_HI = tc::desc_hi(8 * 128, tc::desc_layout(128));
    static constexpr uint32_t TMEM_COLS = 2 * 4 * BNQ;  // 512, 256 or 128
    // kind::f8f6f4: e4m3 A and B (format 0), fp32 D, both K-major
    static constexpr uint32_t IDESC = (1u << 4) | (static_cast<uint32_t>(4 * BNQ / 8) << 17) |
                                      (static_cast<uint32_t>(F8_BM / 16) << 24);
    static_assert(SMEM_BYTES <= 227 * 1024, "8-bit ring");
};

// D[tmem] (+)= A[smem] * B[smem]^T, kind::f8f6f4, K = 32.
__device__ __forceinline__ void umma_f8(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t hi,
                                        uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 ad, bd;\n\t"
        "mov.b64 ad, {%1, %3};\n\t"
        "mov.b64 bd, {%2, %3};\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], ad, bd, %4, p;\n\t}" ::"r"(d_tmem),
        "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate)
        : "memory");
}

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const void* map, uint32_t bar, int c0,
                                            int c1, int c2, uint64_t policy) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        ".L2::cache_hint [%0], [%1, {%2, %3, %4}], [%5], %6;" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(bar), "l"(policy)
        : "memory");
}

__device__ __forceinline__ float lds_f1(uint32_t addr) {
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
// v with its sign flipped.
__device__ __forceinline__ float negate_if(float v, uint32_t flip) {
    return __uint_as_float(__float_as_uint(v) ^ (flip << 31));
}

template <int N>
__device__ __forceinline__ void f8_load(uint32_t taddr, uint32_t (&v)[N]) {
#pragma unroll
    for (int k = 0; k < N; k += 16)
        tmem_ld_32x32b_x16(taddr + k, *reinterpret_cast<uint32_t(*)[16]>(&v[k]));
}
template <int N>
__device__ __forceinline__ void f8_add(const uint32_t (&v)[N], float f, float* acc) {
#pragma unroll
    for (int j = 0; j < N; ++j) acc[j] = fmaf(f, __uint_as_float(v[j]), acc[j]);
}

// 32 bytes of one row in one store: a whole sector.
__device__ __forceinline__ void st_global_na_32(void* p, const uint32_t (&v)[8]) {
    asm volatile("st.global.L1::no_allocate.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(
                     p),
                 "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]),
                 "r"(v[7])
                 : "memory");
}

// How a tile's output leaves, in order of preference:
enum : int {
    F8_STORE_SECTOR = 0,  // Nq a multiple of 16, 32-byte aligned: each thread its row's sectors
    F8_STORE_16 = 1,      // Nq a multiple of 8, 16-byte aligned: staged, 16 bytes along the rows
    F8_STORE_4 = 2,       // Nq even, 4-byte aligned: staged, 4 bytes along the rows
    F8_STORE_2 = 3        // else: staged, 2 bytes
};

// Staged rows along the rows, U channels a store; T has U channels.
template <int BNQ, typename T, int U>
__device__ __forceinline__ void f8_copy_rows(uint32_t stage, __nv_bfloat16* o, int Nq, int rows,
                                             int left) {
    constexpr int PER_ROW = BNQ / U;
    const int lane = threadIdx.x & 31;
#pragma unroll 4
    for (int i = lane; i < 32 * PER_ROW; i += 32) {
        const int r = i / PER_ROW, n = U * (i % PER_ROW);
        if (r < rows && n < left) {
            T h;
            if constexpr (sizeof(T) == 2)
                asm volatile("ld.shared.u16 %0, [%1];"
                             : "=h"(h)
                             : "r"(stage + r * F8Cfg<BNQ>::OUT_PITCH + 2 * n)
                             : "memory");
            else
                asm volatile("ld.shared.u32 %0, [%1];"
                             : "=r"(h)
                             : "r"(stage + r * F8Cfg<BNQ>::OUT_PITCH + 2 * n)
                             : "memory");
            *reinterpret_cast<T*>(o + r * (4LL * Nq) + n) = h;
        }
    }
}

// A warp's 32 rows of a tile, components co0 and co0 + 1 of BNQ channels, out of its threads'
// accumulators (a row a thread): affine, activation, one rounding, and out.  Whole sectors are
// stored by the thread that has them (102,400 rows 512 -> 1024: 113 us; 118 staged in shared
// memory, 117 staged and copied by TMA); rows that do not start at one are staged and stored along
// the rows (7473 rows 520 -> 328: 49 us when each thread stores its own row, staged 17).
template <int BNQ, bool SILU, bool AFFINE, bool SECTOR>
__device__ __forceinline__ void f8_store_tile(const float (&acc)[2][BNQ], const float* scale,
                                              const float* shift, uint32_t stage,
                                              const F8TcParams& p, long long row0, int co0,
                                              int n0) {
    using C = F8Cfg<BNQ>;
    const int lane = threadIdx.x & 31;
    const int rows =
        row0 < p.rows ? static_cast<int>(p.rows - row0 < 32 ? p.rows - row0 : 32) : 0;
    const int left = p.Nq - n0;
    const float least = p.act == 1 ? 0.0f : __uint_as_float(0xFF800000u);  // ReLU; NaN stays
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        __nv_bfloat16* o = p.out + row0 * (4LL * p.Nq) + (co0 + c) * p.Nq + n0;
        if constexpr (!SECTOR) __syncwarp();  // the other component's reads
#pragma unroll
        for (int g = 0; g < BNQ; g += 16) {
            uint32_t v[8];
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                float z[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) z[k] = acc[c][g + j + k];
                if constexpr (AFFINE) {
                    const float4 sc = *reinterpret_cast<const float4*>(scale + c * BNQ + g + j);
                    const float4 sh = *reinterpret_cast<const float4*>(shift + c * BNQ + g + j);
                    z[0] = fmaf(sc.x, z[0], sh.x);
                    z[1] = fmaf(sc.y, z[1], sh.y);
                    z[2] = fmaf(sc.z, z[2], sh.z);
                    z[3] = fmaf(sc.w, z[3], sh.w);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    z[k] = SILU ? f8_silu(z[k]) : (z[k] < least ? least : z[k]);
                v[j / 2] = tc::pack_bf16x2(z[0], z[1]);
                v[j / 2 + 1] = tc::pack_bf16x2(z[2], z[3]);
            }
            if constexpr (SECTOR) {
                if (lane < rows && g < left) st_global_na_32(o + lane * (4LL * p.Nq) + g, v);
            } else {
                const uint32_t at = stage + lane * C::OUT_PITCH + 2 * g;
                sts_u4(at, make_uint4(v[0], v[1], v[2], v[3]));
                sts_u4(at + 16, make_uint4(v[4], v[5], v[6], v[7]));
            }
        }
        if constexpr (SECTOR) continue;
        __syncwarp();
        if (p.store == F8_STORE_16) {
            constexpr int PER_ROW = BNQ / 8;  // 16-byte units
#pragma unroll
            for (int i = 0; i < PER_ROW; ++i) {
                const int r = i * (32 / PER_ROW) + lane / PER_ROW, u = lane % PER_ROW;
                if (r < rows && 8 * u < left)
                    st_global_na(o + r * (4LL * p.Nq) + 8 * u,
                                 lds_u4(stage + r * C::OUT_PITCH + 16 * u));
            }
        } else if (p.store == F8_STORE_4) {
            f8_copy_rows<BNQ, uint32_t, 2>(stage, o, p.Nq, rows, left);
        } else if (p.store == F8_STORE_2) {
            f8_copy_rows<BNQ, uint16_t, 1>(stage, o, p.Nq, rows, left);
        }
    }
}

// SILU or not (ReLU or none then), and whether the epilogue has per-channel vectors: forms of their
// own, for the epilogue's code is as long as the rest.  One form with every branch took 157 us
// for 102,400 rows 512 -> 1024 with SiLU where these took 144 (139 by now).
template <int BNQ, bool SILU, bool AFFINE>
__global__ void __launch_bounds__(F8_THREADS, 1)
    qpoint_f8_kernel(const __grid_constant__ CUtensorMap tmap_x,
                     const __grid_constant__ CUtensorMap tmap_w, const F8TcParams p) {
    using C = F8Cfg<BNQ>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const uint32_t ring_a = smem_u32(smem), ring_b = ring_a + C::A_STAGES * C::A_STAGE;
    float* vectors = reinterpret_cast<float*>(smem + C::RING + C::SCALES + C::OUT);
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::RING + C::SCALES + C::VEC + C::OUT);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + C::NUM_BARS);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    // what an abort has to wait for, written by the roles as they end: the stages of rows that were
    // filled and the parities of their last fills, the same of letters; whether MMAs were issued
    volatile uint32_t* left = tmem_slot + 2;  // [4], [2]
    const uint32_t bar0 = smem_u32(bars);
    const uint32_t full_a = bar0, done_a = full_a + 8u * C::A_STAGES;
    const uint32_t full_b = done_a + 8u * C::A_STAGES, empty_b = full_b + 8u * C::B_STAGES;
    const uint32_t full_s = empty_b + 8u * C::B_STAGES, empty_s = full_s + 8u * C::S_STAGES;
    const uint32_t acce = empty_s + 8u * C::S_STAGES, drain_bar = acce + 16u;
    const uint32_t factors = ring_a + C::RING;  // [stage][ci][co][row]
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint64_t limit = p.wait_limit_ns;
    auto wait = [&](uint32_t bar, uint32_t parity, unsigned code) {
        return tc::wait_or_abort(bar, parity, limit, abort_flag, code);
    };

    griddep_launch_dependents();
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::A_STAGES; ++i) {
            mbar_init(full_a + 8u * i, 1);
            mbar_init(done_a + 8u * i, 1);
        }
        for (int i = 0; i < C::B_STAGES; ++i) {
            mbar_init(full_b + 8u * i, 1);
            mbar_init(empty_b + 8u * i, 2);
        }
        for (int i = 0; i < C::S_STAGES; ++i) {
            mbar_init(full_s + 8u * i, 32);
            mbar_init(empty_s + 8u * i, F8_EPI_WARPS);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(acce + 8u * b, F8_EPI_WARPS);
            mbar_init(drain_bar + 8u * b, 1);
        }
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 0 && lane == 0) {
        tma_prefetch_desc(&tmap_x);
        tma_prefetch_desc(&tmap_w);
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(tmem_slot), C::TMEM_COLS);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;

    if (warp < F8_EPI_WARP0)
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(F8_REGS_ISSUE));
    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer
        if (lane == 0) {
            griddep_wait();  // the quantised rows are complete
            const uint64_t pol_x = l2_policy_evict_normal(), pol_w = l2_policy_evict_last();
            uint32_t filled_a = 0, parity_a = 0, filled_b = 0, parity_b = 0;
            uint32_t phase_a = 0, phase_b = 0;
            int sa = 0, sb = 0;
            bool ok = true;
            for (int t = blockIdx.x; ok && t < p.num_tiles; t += gridDim.x) {
                const int mt = t / p.ntiles, nt = t - mt * p.ntiles;
                for (int kb = 0; ok && kb < p.kblk; ++kb) {
                    if (!wait(empty_b + 8u * sb, phase_b ^ 1u, STATUS_TIMEOUT_PRODUCER)) {
                        ok = false;
                        break;
                    }
                    mbar_arrive_expect_tx(full_b + 8u * sb, C::B_STAGE);
                    filled_b |= 1u << sb;
                    parity_b = (parity_b & ~(1u << sb)) | (phase_b << sb);
                    tma_load_3d(ring_b + sb * C::B_STAGE, &tmap_w, full_b + 8u * sb,
                                kb * F8_BLOCK, nt * BNQ, 0, pol_w);
                    if (++sb == C::B_STAGES) sb = 0, phase_b ^= 1u;
                    for (int ci = 0; ci < 4; ++ci) {
                        if (!wait(done_a + 8u * sa, phase_a ^ 1u, STATUS_TIMEOUT_PRODUCER)) {
                            ok = false;
                            break;
                        }
                        mbar_arrive_expect_tx(full_a + 8u * sa, C::A_STAGE);
                        filled_a |= 1u << sa;
                        parity_a = (parity_a & ~(1u << sa)) | (phase_a << sa);
                        tma_load_3d(ring_a + sa * C::A_STAGE, &tmap_x, full_a + 8u * sa,
                                    kb * F8_BLOCK, ci, mt * F8_BM, pol_x);
                        if (++sa == C::A_STAGES) sa = 0, phase_a ^= 1u;
                    }
                }
            }
            left[0] = filled_a, left[1] = parity_a, left[2] = filled_b, left[3] = parity_b;
        }
    } else if (warp <= 2) {
        // ------------------------------------------------------------ MMA issuers
        if (lane == 0) {
            const int buf = warp - 1;  // this issuer's TMEM buffer, and its partials' parity
            bool ok = true, issued = false;
            if (p.inject_stall) {
                // Failure injection: wait on a barrier nothing arrives on.
                wait(drain_bar, 0, STATUS_TIMEOUT_MMA);
                ok = false;
            }
            const uint32_t d = tmem_base + static_cast<uint32_t>(buf * 4 * BNQ);
            int sa = buf, sb = 0;
            uint32_t phase_a = 0, phase_b = 0, use = 0;
            for (int t = blockIdx.x; ok && t < p.num_tiles; t += gridDim.x) {
                for (int kb = 0; ok && kb < p.kblk; ++kb) {
                    const int left = p.Kq - kb * F8_BLOCK;  // channels of this block
                    const int steps = left >= F8_BLOCK ? 4 : (left + 31) / 32;
                    if (!wait(full_b + 8u * sb, phase_b, STATUS_TIMEOUT_MMA)) {
                        ok = false;
                        break;
                    }
                    const uint32_t b_lo = tc::desc_lo(ring_b + sb * C::B_STAGE);
                    for (int half = 0; half < 2; ++half) {  // components buf and buf + 2
                        if (!wait(acce + 8u * buf, use ^ 1u, STATUS_TIMEOUT_MMA) ||
                            !wait(full_a + 8u * sa, phase_a, STATUS_TIMEOUT_MMA)) {
                            ok = false;
                            break;
                        }
                        use ^= 1u;
                        tc_fence_after();
                        const uint32_t a_lo = tc::desc_lo(ring_a + sa * C::A_STAGE);
                        for (int kk = 0; kk < steps; ++kk)  // 32 channels: 32 bytes into a row
                            umma_f8(d, a_lo + 2 * kk, b_lo + 2 * kk, C::DESC_HI, C::IDESC,
                                    kk != 0 ? 1u : 0u);
                        issued = true;
                        umma_commit(done_a + 8u * sa);
                        if (half == 1) umma_commit(empty_b + 8u * sb);
                        if ((sa += 2) >= C::A_STAGES) sa = buf, phase_a ^= 1u;
                    }
                    if (++sb == C::B_STAGES) sb = 0, phase_b ^= 1u;
                }
            }
            left[4 + buf] = issued;
        }
    } else if (warp == 3) {
        // ------------------------------------------------------------ factors
        // sgn(co, ci) s_x[ci][kb][row] s_w[co xor ci][kb], four rows a lane
        griddep_wait();
        bool ok = true;
        uint32_t ss = 0, phase = 0;
        for (int t = blockIdx.x; ok && t < p.num_tiles; t += gridDim.x) {
            const int mt = t / p.ntiles, nt = t - mt * p.ntiles;
            const float* xs = p.xs + static_cast<long long>(mt) * F8_BM + 4 * lane;
            const float* ws = p.ws + static_cast<long long>(nt * BNQ / F8_BLOCK) * p.kblk;
            for (int kb = 0; kb < p.kblk; ++kb, xs += p.pitch, ++ws) {
                float4 x[4];
                float w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    x[k] = *reinterpret_cast<const float4*>(xs + k * p.kblk * p.pitch);
                    w[k] = ws[static_cast<long long>(k) * p.nblk * p.kblk];
                }
                ok = __all_sync(0xffffffffu,
                                wait(empty_s + 8u * ss, phase ^ 1u, STATUS_TIMEOUT_PRODUCER));
                if (!ok) break;
                const uint32_t dst = factors + ss * C::S_STAGE + 16u * lane;
#pragma unroll
                for (int ci = 0; ci < 4; ++ci)
#pragma unroll
                    for (int co = 0; co < 4; ++co) {
                        const uint32_t flip = ((tc::NEG_MASK >> (4 * co + ci)) & 1u) ^
                                              (co != ci ? static_cast<uint32_t>(p.conj) : 0u);
                        const float f = negate_if(w[co ^ ci], flip);
                        const float4 v = make_float4(f * x[ci].x, f * x[ci].y, f * x[ci].z,
                                                     f * x[ci].w);
                        sts_u4(dst + (4 * ci + co) * (F8_BM * 4),
                               *reinterpret_cast<const uint4*>(&v));
                    }
                mbar_arrive(full_s + 8u * ss);
                if (++ss == C::S_STAGES) ss = 0, phase ^= 1u;
            }
        }
    } else if (warp >= F8_EPI_WARP0) {
        // ---------------------------------------------------------------- epilogue
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(F8_REGS_EPI));
        griddep_wait();  // the rows' scales; the output no longer read by an earlier kernel
        constexpr int CH = BNQ == 16 ? 16 : 32;  // columns of a load
        constexpr int PER = BNQ / CH;            // loads of a component
        const int co0 = 2 * ((warp - F8_EPI_WARP0) / 4), qd = warp & 3;
        float* scale = vectors + (warp - F8_EPI_WARP0) * 4 * BNQ;  // [2][BNQ]
        float* shift = scale + 2 * BNQ;
        const uint32_t stage = smem_u32(smem + C::RING + C::SCALES) +
                               (warp - F8_EPI_WARP0) * 32 * C::OUT_PITCH;
        // factors of this lane's row for component co0; co0 + 1 is 512 bytes on, ci 2 KB a step
        const uint32_t mine = factors + co0 * (F8_BM * 4) + 4u * (qd * 32 + lane);
        uint32_t ss = 0, phase_s = 0;
        int it = 0;
        bool ok = true;
        for (int t = blockIdx.x; ok && t < p.num_tiles; t += gridDim.x) {
            const int mt = t / p.ntiles, nt = t - mt * p.ntiles;
            const int n0 = nt * BNQ;
            if constexpr (AFFINE) {
                __syncwarp();  // the previous tile's reads
                // (every load before the first store, which the compiler has to take for one to
                // these vectors)
                float sc[2 * BNQ / 32], b[2 * BNQ / 32], sh[2 * BNQ / 32];
#pragma unroll
                for (int k = 0; k < 2 * BNQ / 32; ++k) {
                    const int j = lane + 32 * k, n = n0 + (j & (BNQ - 1));
                    const int c = (co0 + j / BNQ) * p.Nq + n;
                    const bool col = n < p.Nq;
                    sc[k] = p.ep.scale && col ? p.ep.scale[c] : 1.0f;
                    sh[k] = p.ep.scale && col ? p.ep.shift[c] : 0.0f;
                    b[k] = p.ep.bias && col ? p.ep.bias[c] : 0.0f;
                }
#pragma unroll
                for (int k = 0; k < 2 * BNQ / 32; ++k) {
                    scale[lane + 32 * k] = sc[k];
                    shift[lane + 32 * k] = fmaf(sc[k], b[k], sh[k]);
                }
                __syncwarp();
            }
            float acc[2][BNQ];
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int j = 0; j < BNQ; ++j) acc[c][j] = 0.0f;
            const int partials = 4 * p.kblk;
#pragma unroll 1
            for (int i = 0; i < partials; ++i, ++it) {
                const int ci = i & 3, buf = it & 1;
                bool got = true;
                if (ci == 0) got = wait(full_s + 8u * ss, phase_s, STATUS_TIMEOUT_EPILOGUE);
                got = got && wait(done_a + 8u * (it & (C::A_STAGES - 1)),
                                  (it / C::A_STAGES) & 1, STATUS_TIMEOUT_EPILOGUE);
                ok = __all_sync(0xffffffffu, got);
                if (!ok) break;
                const uint32_t fa = mine + ss * C::S_STAGE + ci * (4 * F8_BM * 4);
                const float f[2] = {lds_f1(fa), lds_f1(fa + F8_BM * 4)};
                if (ci == 3) {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(empty_s + 8u * ss);
                    if (++ss == C::S_STAGES) ss = 0, phase_s ^= 1u;
                }
                tc_fence_after();
                const uint32_t taddr = tmem_base + (static_cast<uint32_t>(qd * 32) << 16) +
                                       static_cast<uint32_t>(buf * 4 * BNQ);
                const uint32_t t0 = taddr + (co0 ^ ci) * BNQ, t1 = taddr + (co0 ^ 1 ^ ci) * BNQ;
                // chunk k: columns CH (k mod PER) and up of component co0 + k / PER
                uint32_t v[2][CH];
                f8_load<CH>(t0, v[0]);
#pragma unroll
                for (int k = 0; k < 2 * PER; ++k) {
                    tmem_ld_wait();
                    if (k + 1 < 2 * PER) {
                        f8_load<CH>((k + 1 < PER ? t0 : t1) + CH * ((k + 1) % PER),
                                    v[(k + 1) & 1]);
                    } else {
                        // the partial is in registers: hand the buffer back to the issuer
                        tc_fence_before();
                        if (lane == 0) mbar_arrive_relaxed(acce + 8u * buf);
                    }
                    f8_add<CH>(v[k & 1], f[k / PER], &acc[k / PER][CH * (k % PER)]);
                }
            }
            if (!ok) break;
            const long long row0 = static_cast<long long>(mt) * F8_BM + qd * 32;
            if (p.store == F8_STORE_SECTOR)
                f8_store_tile<BNQ, SILU, AFFINE, true>(acc, scale, shift, stage, p, row0, co0, n0);
            else
                f8_store_tile<BNQ, SILU, AFFINE, false>(acc, scale, shift, stage, p, row0, co0,
                                                        n0);
        }
    }

    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {
        // Behind the barrier, for a role may end before another gives up: no copy may land in
        // shared memory that is another CTA's by then, and no MMA write TMEM that was released.
        if (threadIdx.x == 0) {
            tc::drain_fills(full_a, C::A_STAGES, left[0], left[1], limit);
            tc::drain_fills(full_b, C::B_STAGES, left[2], left[3], limit);
        }
        if ((warp == 1 || warp == 2) && lane == 0 && left[3 + warp]) {
            const uint32_t bar = drain_bar + 8u * (warp - 1);
            umma_commit(bar);
            tc::drain_fills(bar, 1, 1u, 0u, limit);
        }
        __syncthreads();
    }
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc(tmem_base, C::TMEM_COLS);
    }
}
