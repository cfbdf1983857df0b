// internal.h -- launch interfaces shared by the C-ABI front end (quan_api.cu) and the
// kernels.  Not part of the public header.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <cstdint>

namespace quan {

// Geometry and epilogue of one quaternion convolution call.  Channels are real
// channels; Q = C / 4 quaternion channels per component block.
struct ConvShape {
    int N, H, W, Cin, Cout, kh, kw, stride, pad, act;
    int Ho, Wo, Qin, Qout;
    long long M;  // N * Ho * Wo output pixels
    int sep;      // 1: the separable form of Eq. 7 (per-component convolutions, sign mix);
                  // 2 (tensor-core path only): its transpose, the input gradient's
                  // convolution (block (q, p) = sign(p, q) W_q)
};

struct EpilogueArgs {
    const float* bias;   // [Cout] or null
    const float* scale;  // [Cout] or null (IQBN scale, with shift)
    const float* shift;  // [Cout] or null
    const void* residual;  // [M][Cout] (same dtype as out) or null
};

// Device status word bits (set by kernels whose bounded waits ran out).
enum : unsigned {
    STATUS_TIMEOUT_PRODUCER = 1u,
    STATUS_TIMEOUT_MMA = 2u,
    STATUS_TIMEOUT_EPILOGUE = 4u,
    STATUS_TIMEOUT_DRAIN = 8u,
};

struct TcOptions {
    int kappa;                    // quaternion input channels per K block (16, 32 or 64); 0 = auto
    int bnq;                      // quaternion output channels per tile (16, 32 or 64); 0 = auto
    int max_ctas;                 // persistent grid cap; 0 = number of SMs
    int mode;                     // 0 auto, 1 one MMA per (q, p), 2 paired output components,
                                  // 3 weight-stationary
    int ws_halo;                  // weight-stationary: stage row blocks with halos (1) when
                                  // the shape allows it, else one im2col box per tap (0)
    int ws_issuers;               // weight-stationary MMA issuers: 0 auto, 2 or 3
    int vs_rows;                  // vertical-tap kernel: output rows per band, 0 auto, 1..4
    void* sk_ws;                  // caller workspace for K ranges split over the CTAs (the
    size_t sk_ws_bytes;           // quad/pair kernel's partial tiles and flags), or null
    unsigned long long wait_limit_ns;
    int inject_stall;             // failure-injection: the MMA role never consumes
};

// Tensor-core path (tcgen05 + TMA), bf16 in/out, fp32 accumulation.
bool tc_supported(const ConvShape& s, const void* x, const void* const w[4], const void* out,
                  const EpilogueArgs& ep);
cudaError_t launch_qconv_tc(const ConvShape& s, const void* x, const void* const w[4],
                            const EpilogueArgs& ep, void* out, const TcOptions& opt,
                            int num_sms, cudaStream_t stream, char* err, size_t errlen);
// Input gradient of a stride-2 forward convolution f by the parity classes of its pixels
// (f.sep: 0 or 2), letters in bwd_transform's layout.
bool tc_parity_supported(const ConvShape& f);
cudaError_t launch_qconv_tc_parity(const ConvShape& f, const void* dy, const void* const w[4],
                                   void* dx, const TcOptions& opt, int num_sms,
                                   cudaStream_t stream, char* err, size_t errlen);
cudaError_t read_and_clear_status(unsigned* status, cudaStream_t stream);
// Workspace bytes that let a quad/pair-kernel launch on a device of num_sms SMs split its
// K ranges evenly over its CTAs (one fp32 partial tile and one flag per CTA).
size_t tc_split_workspace_bytes(int num_sms);
// The convolution s and a 1x1 shortcut (Qout_sc quaternion output channels, no padding, the
// same stride) on the same input x in one tensor-core launch; its own letters, epilogue
// vectors (no residual), activation and output.
bool tc_shortcut_supported(const ConvShape& s, const void* x, const void* const w[4],
                           const void* out, const EpilogueArgs& ep, const void* const wsc[4],
                           int qout_sc, const EpilogueArgs& ep_sc, const void* out_sc,
                           const TcOptions& opt);
cudaError_t launch_qconv_tc_shortcut(const ConvShape& s, const void* x, const void* const w[4],
                                     const EpilogueArgs& ep, void* out,
                                     const void* const wsc[4], int qout_sc, int act_sc,
                                     const EpilogueArgs& ep_sc, void* out_sc,
                                     const TcOptions& opt, int num_sms, cudaStream_t stream,
                                     char* err, size_t errlen);
// Name of the tensor-core kernel the calling thread's last launch_qconv_tc used.
const char* last_tc_kernel();

// Which form the calling thread's last launch of a kernel with several behind one name took
// (for the tests, through quan_last_variant): "direct", "mma" or "tiles" for the kernels without
// tcgen05, "single" or "pairs" for the pointwise kernel.
extern thread_local const char* last_variant;

// Without tcgen05, any shape: a thread per output (qconv_direct.cuh), warp-level MMAs (bf16) or
// tiled CUDA-core products, whichever takes least; T = __nv_bfloat16 or float.
cudaError_t launch_qconv_simt_bf16(const ConvShape& s, const void* x, const void* const w[4],
                                   const EpilogueArgs& ep, void* out, int num_sms,
                                   cudaStream_t stream);
cudaError_t launch_qconv_simt_f32(const ConvShape& s, const void* x, const void* const w[4],
                                  const EpilogueArgs& ep, void* out, int num_sms,
                                  cudaStream_t stream);

// Warp-level tensor-core kernels (mma.sync) for bf16 layers off the tcgen05 kernels' channel
// grid: the convolution, its input gradient and its weight gradient (zeroes dW_L, then adds).
bool mma_fwd_supported(const ConvShape& s, const void* x, const void* out, const void* residual);
cudaError_t launch_mma_fwd(const ConvShape& s, const void* x, const void* const w[4],
                           const EpilogueArgs& ep, void* out, int num_sms, cudaStream_t stream);
// Estimated time (us) of the first two.
double mma_fwd_time(const ConvShape& s, int num_sms);
double mma_bwd_data_time(const ConvShape& s, int num_sms);
bool mma_bwd_data_supported(const ConvShape& s, const void* dy, const void* dx);
cudaError_t launch_mma_bwd_data(const ConvShape& s, const void* dy, const void* const w[4],
                                void* dx, int num_sms, cudaStream_t stream);
bool mma_bwd_weight_supported(const ConvShape& s, const void* x, const void* dy);
cudaError_t launch_mma_bwd_weight(const ConvShape& s, const void* x, const void* dy,
                                  float* const dw[4], int num_sms, cudaStream_t stream);

// Launch with programmatic stream serialization: the kernel may start while the previous
// kernel in the stream is finishing (once all of that grid's CTAs have signalled), runs its
// prologue (barriers, TMEM, descriptor prefetch) and waits with griddepcontrol.wait before
// its first global access.  Every kernel of this library follows that rule.
// launch_pdl_cluster: the same in clusters of `cluster` blocks along x.
template <typename... KArgs, typename... Args>
cudaError_t launch_pdl_cluster(void (*kern)(KArgs...), dim3 grid, dim3 block, unsigned cluster,
                               size_t smem, cudaStream_t stream, Args&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, static_cast<KArgs>(args)...);
}

template <typename... KArgs, typename... Args>
cudaError_t launch_pdl(void (*kern)(KArgs...), dim3 grid, dim3 block, size_t smem,
                       cudaStream_t stream, Args&&... args) {
    return launch_pdl_cluster(kern, grid, block, 1u, smem, stream, static_cast<Args&&>(args)...);
}

// Poincare RGB -> quaternion mapping (Eq. 4): fp32 [npix][3] -> bf16 [npix][4].
cudaError_t launch_poincare(const float* rgb, long long npix, void* out, int num_sms,
                            cudaStream_t stream);

// Backward of the pre-epilogue convolution (s.sep selects the separable form, Eq. 8-10).
// Bytes of the transformed letters bwd_transform writes: 4 x [Qin][kh][kw][Qout] bf16.
size_t bwd_data_workspace_bytes(int Cin, int Cout, int kh, int kw);
// out_L[ci][kh-1-dh][kw-1-dw][co] = s_L * w_L[co][dh][dw][ci], the four letters one after
// the other: the forward weights of the stride-1 input gradient; s = (+1, -1, -1, -1)
// (the conjugate, full form) when conj, else +1 (the separable form's signs are applied
// by the MMA table).
cudaError_t launch_bwd_transform(int Cin, int Cout, int kh, int kw, const void* const w[4],
                                 bool conj, void* out, int num_sms, cudaStream_t stream);
// dy [N][Ho][Wo][C] with s - 1 zeros inserted between pixels, [N][Hu][Wu][C] (C % 8 == 0,
// 16-byte aligned): the input of a strided forward's input-gradient convolution.
cudaError_t launch_bwd_upsample(const void* dy, int N, int Ho, int Wo, int C, int s, int Hu,
                                int Wu, void* u, int num_sms, cudaStream_t stream);
// dx [N][H][W][Cin] from dy [N][Ho][Wo][Cout] without tcgen05, any stride.
cudaError_t launch_bwd_data_simt(const ConvShape& s, const void* dy, const void* const w[4],
                                 void* dx, int num_sms, cudaStream_t stream);
// Library-owned device scratch of quan_qconv2d_bwd_data_static (one per device, in the
// module's static device memory): its size, and its address on the current device.
constexpr size_t BWD_STATIC_SCRATCH_BYTES = size_t(2) << 20;
cudaError_t bwd_static_scratch_address(void** ptr);
// Tensor-core weight gradient, both forms (s.sep) (stride 1 or 2, Cin and Cout multiples of 64,
// Cout <= 256 or a multiple of 256, 16-byte aligned x and dy).  Zeroes dW_L, then adds.
bool bwd_weight_tc_supported(const ConvShape& s, const void* x, const void* dy);
cudaError_t launch_bwd_weight_tc(const ConvShape& s, const void* x, const void* dy,
                                 float* const dw[4], int num_sms,
                                 unsigned long long wait_limit_ns, cudaStream_t stream,
                                 char* err, size_t errlen);
// Four fp32 arrays of n elements set to zero in one launch.
cudaError_t launch_zero4(float* const t[4], long long n, int num_sms, cudaStream_t stream);
// dW_L fp32 [Qout][kh][kw][Qin] (zeroed, then accumulated) without tcgen05.
cudaError_t launch_bwd_weight_simt(const ConvShape& s, const void* x, const void* dy,
                                   float* const dw[4], int num_sms, cudaStream_t stream);

// Training-mode IQBN (Eq. 11-12) over bf16 [npix][C].  The 16-byte vector path needs C a
// multiple of 8 (at most 2048) and 16-byte aligned tensors; otherwise C <= 256.
bool iqbn_vec_ok(int C, const void* a, const void* b);
bool iqbn_supported(int C, const void* a, const void* b);
// Partial sums of at most IQBN_MAX_PARTIALS blocks: workspace fp32 [blocks][2][C].
constexpr int IQBN_MAX_PARTIALS = 1024;
size_t iqbn_stats_workspace_bytes(int C);
cudaError_t launch_iqbn_stats(const void* x, long long npix, int C, void* workspace,
                              float* mean, float* var, int num_sms, cudaStream_t stream);
cudaError_t launch_iqbn_apply(const void* x, long long npix, int C, const float* mean,
                              const float* var, const float* gamma, const float* beta, float eps,
                              int act, void* out, int num_sms, cudaStream_t stream);

// The 4-channel stem convolution and its 3x3/2, padding-1 max pooling in one kernel:
// out [N][(Ho - 1) / 2 + 1][(Wo - 1) / 2 + 1][64] bf16 (Cin = 4, Cout = 64, stride 2, even W,
// Wo <= 128).
bool tc_stem_pool_supported(const ConvShape& s, const void* x, const void* const w[4],
                            const void* out, const EpilogueArgs& ep);
cudaError_t launch_qconv_stem_pool(const ConvShape& s, const void* x, const void* const w[4],
                                   const EpilogueArgs& ep, void* out, const TcOptions& opt,
                                   int num_sms, cudaStream_t stream, char* err, size_t errlen);

// The same from fp32 RGB pixels [N][H][W][3] (W a multiple of 32), the Poincare mapping of
// Eq. 4 done in the kernel's loader; s is the convolution's shape (Cin = 4).
bool tc_stem_pool_rgb_supported(const ConvShape& s, const float* rgb, const void* const w[4],
                                const void* out, const EpilogueArgs& ep);
cudaError_t launch_qconv_stem_pool_rgb(const ConvShape& s, const float* rgb,
                                       const void* const w[4], const EpilogueArgs& ep, void* out,
                                       const TcOptions& opt, int num_sms, cudaStream_t stream,
                                       char* err, size_t errlen);

// Dropout (philox.cuh): the mask of one call.
struct DropoutArgs {
    uint32_t bound;  // an element is kept when its 16 bits, as the upper half of a word, are >= it
    int draws;       // 0: no bits are drawn, every element has zeros (all are kept with bound 0,
                     // none with bound 2^16)
    float factor;    // 1 / (1 - p); 0 for p = 1
    uint32_t key0, key1;
    unsigned long long offset;
    const unsigned long long* counter;  // device word added to offset, or null
};
// p in [0, 1] rounded to a step of 2^-16.
DropoutArgs dropout_args(float p, unsigned long long seed, unsigned long long offset,
                         const unsigned long long* counter);
cudaError_t launch_dropout(const void* x, long long n, bool f32, const DropoutArgs& d, void* out,
                           int num_sms, cudaStream_t stream);

// The residual join and its gradients (residual.cu).  Forward: x, h, out_y (y), out_n (n);
// backward: h, y, dy, dn, out_y (dx), out_n (dh).  Absent tensors and vectors are null.
struct JoinArgs {
    const void *x, *h, *y, *dy, *dn;
    const float *post, *gate, *pre;  // [C], [images][C], [C]
    void *out_y, *out_n;
    long long rows, images;
    int C, groups;
    bool f32;
    float alpha, eps;
    DropoutArgs drop;
    // forward: n in 8 bits, laid out as the 8-bit product's rows, and out_n, if given, in bf16
    void* q8;
    float* s8;
};
bool join_supported(int C, int groups);
cudaError_t launch_join_fwd(const JoinArgs& a, int num_sms, cudaStream_t stream);
size_t join_bwd_workspace_bytes(long long rows, int C, int groups, long long images, int num_sms);
cudaError_t launch_join_bwd(const JoinArgs& a, float* workspace, float* dpost, float* dgate,
                            float* dpre, int num_sms, cudaStream_t stream);

// Distillation from a teacher's top logits (distill.cu): the loss (dz null), its gradient (loss null,
// lse_in given) or both.
struct DistillArgs {
    const void *z, *index, *teacher;
    const float *lse_in, *dloss;
    float *loss, *lse;
    void* dz;
    long long rows, pitch;
    int classes, top;
    bool f32, teacher_f32, index64;
    float temperature, scale;
};
cudaError_t launch_distill(const DistillArgs& a, int num_sms, cudaStream_t stream);

// The pointwise product in 8-bit floating point (qpoint_f8.cu) of Kq input and Nq output
// quaternion channels.  f8_pitch: bytes of a row of 8-bit channels of one component.
int f8_pitch(int Kq);
cudaError_t launch_f8_letters(const void* const w[4], int Qout, int Qin, bool transpose, void* q,
                              float* scale, cudaStream_t stream);
// Status word of its kernels, as read_and_clear_status.
cudaError_t read_and_clear_status_f8(unsigned* status, cudaStream_t stream);
// Tiled map of a byte tensor of three dimensions, innermost first (strides: of the outer two, in
// bytes), boxes with the 128-byte swizzle, 0 past the ends (qconv_tc.cu).
bool encode_bytes_3d(CUtensorMap* map, const void* base, const unsigned long long dims[3],
                     const unsigned long long strides[2], const unsigned box[3]);
size_t qpoint_f8_workspace_bytes(long long rows, int Kq, int Nq);
// Rows in 8 bits: words between the scales of two blocks, and the rows read back to bf16.
long long f8_scale_pitch(long long rows);
cudaError_t launch_f8_dequant(const void* q, const float* scale, long long rows, int Kq, void* out,
                              cudaStream_t stream);
// xscale: x is rows in 8 bits already, and these are their scales; no workspace then.
cudaError_t launch_qpoint_f8(const void* x, const float* xscale, const void* wq, const float* ws,
                             const EpilogueArgs& ep, long long rows, int Kq, int Nq, bool conj,
                             int act, void* workspace, void* out, int num_sms,
                             unsigned long long wait_limit_ns, int inject_stall,
                             cudaStream_t stream, char* err, size_t errlen);

// The pointwise product with 4-bit letters (qpoint_w4.cu): bytes of the letters, number of scales.
size_t w4_bytes(int Qi, int Qo);
size_t w4_scales(int Qi, int Qo, int group);
cudaError_t launch_w4_letters(const void* const w[4], int Qo, int Qi, int group, void* q,
                              void* scale, cudaStream_t stream);
cudaError_t launch_qpoint_w4(const void* x, const void* q, const void* scale,
                             const EpilogueArgs& ep, long long rows, int Qi, int Qo, int group,
                             int act, void* out, int num_sms, cudaStream_t stream);

// Per-real-channel max pooling, bf16 NHWC.
cudaError_t launch_maxpool_bf16(const void* x, int N, int H, int W, int C, int k, int stride,
                                int pad, void* out, int num_sms, cudaStream_t stream);

}  // namespace quan
