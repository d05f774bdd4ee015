// C-ABI entry points of libhinm: host-side argument validation and kernel dispatch.
// Every check here runs before anything is launched, so the error paths need no GPU.
#include "hinm_internal.h"

#include "linear_tile.h"
#include "mx4_form.h"
#include "prepared_layout.h"
#include "hinm_calib.h"


namespace {

using namespace hinm;

hinm_status check_shape(const hinm_shape* s) {
  if (!s) return HINM_ERR_NULL;
  if (s->dtype != HINM_F16 && s->dtype != HINM_BF16) return HINM_ERR_DTYPE;
  if (s->M <= 0 || s->K <= 0 || s->V <= 0 || s->Kv <= 0) return HINM_ERR_SHAPE;
  if (s->M % s->V != 0) return HINM_ERR_SHAPE;
  if (s->Kv > s->K || s->Kv % 8 != 0) return HINM_ERR_SHAPE;
  return HINM_OK;
}

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

hinm_status check_spmm(const hinm_shape* s, int32_t N, const void* vals, const uint8_t* nm_idx,
                       const int32_t* vec_idx, const void* X, int64_t ldx, const void* Y, int64_t ldy,
                       uint32_t flags) {
  hinm_status st = check_shape(s);
  if (st != HINM_OK) return st;
  if (!vals || !nm_idx || !vec_idx || !X || !Y) return HINM_ERR_NULL;
  if (N <= 0 || ldx < N || ldy < N) return HINM_ERR_SHAPE;
  if (N > 1 && (ldx % 8 != 0 || ldy % 8 != 0)) return HINM_ERR_SHAPE;
  if (!aligned(vals, 16) || !aligned(X, 16) || !aligned(Y, 16)) return HINM_ERR_SHAPE;
  const uint32_t known = HINM_EPI_RELU | HINM_OUT_F32 | HINM_KERNEL_REFERENCE | HINM_KERNEL_SMFMAC | HINM_KERNEL_GEMV;
  if (flags & ~known) return HINM_ERR_UNSUPPORTED;
  const uint32_t forced = flags & (HINM_KERNEL_REFERENCE | HINM_KERNEL_SMFMAC | HINM_KERNEL_GEMV);
  if (forced & (forced - 1)) return HINM_ERR_UNSUPPORTED;  // at most one kernel may be forced
  return HINM_OK;
}

hinm_status run_spmm(const SpmmArgs& a, uint32_t flags, hipStream_t stream) {
  hipError_t e;
  if (flags & HINM_KERNEL_REFERENCE) {
    e = launch_spmm_reference(a, stream);
  } else if (flags & HINM_KERNEL_SMFMAC) {
    if (spmm_tile_supported(a)) e = launch_spmm_tile(a, stream);
    else if (spmm_skinny_supported(a)) e = launch_spmm_skinny(a, stream);
    else return HINM_ERR_UNSUPPORTED;
  } else if (flags & HINM_KERNEL_GEMV) {
    if (a.N > 16 || !spmm_skinny_supported(a)) return HINM_ERR_UNSUPPORTED;
    e = launch_spmm_skinny(a, stream);
  } else {
    // by shape: a moderate number of columns -> wave-private kernel; one column, or up to sixteen where one round of its
    // workgroups does -> k-split skinny kernel (bandwidth-bound on the packed weights); otherwise the tile kernel; shapes
    // none covers fall back to the plain kernel.
    if (spmm_mid_canonical_preferred(a)) e = launch_spmm_mid_canonical(a, stream);
    else if (a.N <= 16 && spmm_skinny_supported(a)) e = launch_spmm_skinny(a, stream);
    else if (spmm_tile_supported(a)) e = launch_spmm_tile(a, stream);
    else if (spmm_skinny_supported(a)) e = launch_spmm_skinny(a, stream);
    else e = launch_spmm_reference(a, stream);
  }
  return e == hipSuccess ? HINM_OK : HINM_ERR_DEVICE;
}

size_t elem_bytes_out(uint32_t flags) { return (flags & HINM_OUT_F32) ? 4 : 2; }

// ---- 4-bit form and norms around a block ---------------------------------------------------------------
bool known_dtype(int32_t d) { return d == HINM_F16 || d == HINM_BF16; }
hinm_status launched(hipError_t e) { return e == hipSuccess ? HINM_OK : HINM_ERR_DEVICE; }

// What sizes may be (index arithmetic in 32 bits beside it), and the workgroups of a launch (of up to 512 threads).
constexpr int32_t kMostSize = 1 << 30;
constexpr int64_t kMostGroups = 1 << 22;

// rows of `length` values in 4-bit form
hinm_status check_form(const uint8_t* codes, const uint8_t* scales) {
  if (!codes || !scales) return HINM_ERR_NULL;
  return aligned(codes, 16) && aligned(scales, 16) ? HINM_OK : HINM_ERR_SHAPE;
}

// workgroups that quantise a matrix: 32 x 256 values along the rows, 128 x 64 down the columns
bool too_many_to_quantize(int32_t rows, int32_t cols, bool columns) {
  const int64_t pieces = columns ? (int64_t)((cols + 63) / 64) * 2 * mx4_lines(rows) : (int64_t)mx4_row_blocks(rows) * mx4_lines(cols);
  return pieces >= 2 * kMostGroups;
}

hinm_status check_product(int32_t M, int32_t N, int32_t K, int32_t dtype, const void* Y, int64_t ldy, uint32_t flags) {
  if (!known_dtype(dtype)) return HINM_ERR_DTYPE;
  if (M <= 0 || N <= 0 || K <= 0) return HINM_ERR_SHAPE;
  if (!Y) return HINM_ERR_NULL;
  if (ldy < N || !aligned(Y, (flags & HINM_OUT_F32) ? 4 : 2)) return HINM_ERR_SHAPE;
  if (flags & ~(uint32_t)(HINM_EPI_RELU | HINM_OUT_F32)) return HINM_ERR_UNSUPPORTED;
  // workgroups of one launch: 32 rows for one column, otherwise at most 128 x 128 outputs
  if (M > kMostSize || N > kMostSize || K > kMostSize) return HINM_ERR_UNSUPPORTED;
  if (N == 1 ? M / 32 >= kMostGroups : (int64_t)((M + 127) / 128) * ((N + 127) / 128) >= kMostGroups) return HINM_ERR_UNSUPPORTED;
  return HINM_OK;
}

struct LinearPlan {
  size_t codes, scales;  // bytes of the activations' 4-bit form, each rounded to 256
};
LinearPlan linear_plan(int32_t K, int32_t N) {
  const size_t c = (size_t)mx4_code_bytes(N, K), s = (size_t)mx4_scale_bytes(N, K);
  return {(c + 255) & ~size_t{255}, (s + 255) & ~size_t{255}};
}

// a workgroup has 64 tokens, and some 64 of them the chunks of such a strip
constexpr int32_t kMostTokens = 1 << 22;

hinm_status check_norm(int32_t K, int32_t N, int32_t dtype) {
  if (!known_dtype(dtype)) return HINM_ERR_DTYPE;
  if (K <= 0 || N <= 0) return HINM_ERR_SHAPE;
  return N > kMostTokens || K > kMostSize ? HINM_ERR_UNSUPPORTED : HINM_OK;
}

// Channels' gradients of several strips of tokens are added by workgroups of 1024 threads, 32 channels each; a launch has less than
// 2^32 threads.
bool too_many_to_add(int32_t K, int32_t N) { return K > 32 * (kMostGroups - 1) && N > 64; }

// ---- dense layers --------------------------------------------------------------------------------------
// M x N results of sums over K: what a launch has workgroups for, 64 x 64 results each at the least
hinm_status check_dense(int32_t M, int32_t K, int32_t N) {
  if (M <= 0 || K <= 0 || N <= 0) return HINM_ERR_SHAPE;
  if (M > kMostSize || K > kMostSize || N > kMostSize) return HINM_ERR_UNSUPPORTED;
  return (int64_t)((M + 63) / 64) * ((N + 63) / 64) >= kMostGroups ? HINM_ERR_UNSUPPORTED : HINM_OK;
}
// ... of a layer forward, whose few tokens have workgroups of 16 rows and up to 1024 threads; a launch has less than 2^32 threads
hinm_status check_layer(int32_t M, int32_t K, int32_t N) {
  return N <= kFewTokens && M / 16 >= kMostGroups - 8 ? HINM_ERR_UNSUPPORTED : check_dense(M, K, N);
}
// ... of a layer's gradients
hinm_status check_dense_grad(int32_t M, int32_t K, int32_t N) {
  const hinm_status st = check_dense(K, M, N);
  return st != HINM_OK ? st : check_dense(M, N, K);
}
// The gradients' products take whole pieces of rows: dZ has them, and dY where it takes dZ's place, or it is written there as it is; X
// of few tokens is copied, but not of so few that dW has a kernel which takes rows of any kind.
constexpr int32_t kMostCopiedTokens = 64;
struct LinearGradPlan {
  int64_t ldz;              // of dZ and of X's copy
  size_t dz, x, product;  // bytes of dZ and of X's copy, rounded to 256, and of the products' partial sums
};
LinearGradPlan linear_grad_plan(int32_t M, int32_t K, int32_t N) {
  LinearGradPlan p;
  p.ldz = ((int64_t)N + 7) / 8 * 8;
  p.dz = ((size_t)M * p.ldz * 2 + 255) & ~size_t{255};
  p.x = N > kOuterTokens && N <= kMostCopiedTokens ? ((size_t)K * p.ldz * 2 + 255) & ~size_t{255} : 0;
  const size_t x = dense_product_workspace_bytes(K, N, M, kAcross, kAcross), w = dense_product_workspace_bytes(M, K, N, kAlong, kAlong);
  p.product = x > w ? x : w;
  return p;
}
// ... from dZ (dY where that takes its place) on, which lies in whole pieces.
struct LinearGradProducts {
  DenseProduct of_x, of_w;
  bool wants_x, wants_w, copied, pair;  // X to whole pieces first; both products in one launch
  const void* X;                        // as the call has it
  int64_t ldx;
  void* x_copy;
};
LinearGradProducts linear_grad_products(const LinearGradPlan& p, int32_t M, int32_t K, int32_t N, int32_t dtype, const void* W, int64_t ldw,
                                        const void* X, int64_t ldx, const void* dz, int64_t ldz, void* dX, void* dW, bool out_f32,
                                        void* workspace, LaunchPlan* record) {
  uint8_t* const x_copy = static_cast<uint8_t*>(workspace) + p.dz;
  void* const partials = x_copy + p.x;
  const bool copied = dW && p.x && pieces_of_rows(X, ldx, N) != kAligned;
  LinearGradProducts g{{K, N, M, dtype, kAcross, kAcross, W, ldw, dz, ldz,
                        {K, N, nullptr, nullptr, 0, kAligned, nullptr, dX, ldx, kActNone, false}, partials, record},
                       {M, K, N, dtype, kAlong, kAlong, dz, ldz, copied ? x_copy : X, copied ? p.ldz : ldx,
                        {M, K, nullptr, nullptr, 0, kAligned, nullptr, dW, ldw, kActNone, out_f32}, partials, record},
                       dX != nullptr, dW != nullptr, copied, false, X, ldx, x_copy};
  g.pair = dX && dW && dense_pair_serves(g.of_w, g.of_x);
  return g;
}
// ... with the sums of dZ's rows to `sums`, unless it is NULL, where both products are one launch
hipError_t launch_grad_products(const LinearGradProducts& g, float* sums, hipStream_t stream) {
  LaunchPlan* const record = g.of_w.plan;
  hipError_t e = hipSuccess;
  if (g.copied && record) plan_record(record, "linear_copy_kernel block=256");
  else if (g.copied) e = launch_row_copy(g.X, g.ldx, g.x_copy, g.of_w.ldb, g.of_w.N, g.of_w.K, stream);
  if (e != hipSuccess) return e;
  if (g.pair) return launch_dense_pair(g.of_w, g.of_x, sums, stream);
  if (g.wants_x) e = launch_dense_product(g.of_x, stream);
  return e == hipSuccess && g.wants_w ? launch_dense_product(g.of_w, stream) : e;
}

// ---- hinm_pack_static: the score workspace of the pack kernels in a file-scope device array -------------
// One binary64 score per tile and column, at most kStaticScoreCount of them (4 MiB).  Every GPU the library runs
// on holds its own copy of the array at its own address until the process ends.
constexpr size_t kStaticScoreCount = (size_t)HINM_PACK_STATIC_MAX_SCORES;
static __device__ __align__(256) double scratch[kStaticScoreCount];

// In host code `scratch` is only a stand-in for the symbol: the device address comes from
// hipGetSymbolAddress, once per device with that device current, and is kept per device.
constexpr int kStaticMaxDevices = 64;
hipError_t static_scores(double** out) {
  static std::atomic<double*> per_device[kStaticMaxDevices];
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= kStaticMaxDevices) return hipErrorInvalidDevice;
  double* p = per_device[dev].load(std::memory_order_acquire);
  if (!p) {
    void* addr = nullptr;
    e = hipGetSymbolAddress(&addr, HIP_SYMBOL(scratch));
    if (e != hipSuccess) return e;
    if (!addr) return hipErrorInvalidSymbol;
    p = static_cast<double*>(addr);
    per_device[dev].store(p, std::memory_order_release);  // two first calls racing store the same address
  }
  *out = p;
  return hipSuccess;
}

}  // namespace

extern "C" {

hinm_status hinm_pack_sizes(const hinm_shape* shape, size_t* vals_bytes, size_t* nm_bytes, size_t* vec_bytes,
                            size_t* workspace_bytes) {
  hinm_status st = check_shape(shape);
  if (st != HINM_OK) return st;
  const size_t M = shape->M, K = shape->K, Kv = shape->Kv, T = shape->M / shape->V;
  if (vals_bytes) *vals_bytes = M * (Kv / 2) * 2;
  if (nm_bytes) *nm_bytes = M * (Kv / 8);
  if (vec_bytes) *vec_bytes = T * Kv * sizeof(int32_t);
  if (workspace_bytes) *workspace_bytes = T * K * sizeof(double);
  return HINM_OK;
}

static hinm_status run_pack(const hinm_shape* shape, const void* W, const float* rho, bool with_rho,
                            const int32_t* tile_order, void* vals, uint8_t* nm_idx, bool with_nm, int32_t* vec_idx,
                            void* workspace, size_t workspace_bytes, void* stream) {
  hinm_status st = check_shape(shape);
  if (st != HINM_OK) return st;
  if (!W || !vals || !vec_idx || (with_nm && !nm_idx) || (with_rho && !rho)) return HINM_ERR_NULL;
  size_t need = 0;
  hinm_pack_sizes(shape, nullptr, nullptr, nullptr, &need);
  if (!workspace || workspace_bytes < need || !aligned(workspace, 8)) return HINM_ERR_WORKSPACE;
  if (!aligned(vals, with_nm ? 8 : 16) || !aligned(vec_idx, 4) || !aligned(W, 2)) return HINM_ERR_SHAPE;
  if (with_rho && !aligned(rho, 4)) return HINM_ERR_SHAPE;
  if (tile_order && (!aligned(tile_order, 4) || shape->K > kPackOrderMaxK)) return HINM_ERR_UNSUPPORTED;
  const PackArgs a{*shape, W, rho, tile_order, vals, with_nm ? nm_idx : nullptr, vec_idx,
                   static_cast<double*>(workspace)};
  hipError_t e = launch_pack(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? HINM_OK : HINM_ERR_DEVICE;
}

hinm_status hinm_pack(const hinm_shape* shape, const void* W, void* vals, uint8_t* nm_idx, int32_t* vec_idx,
                      void* workspace, size_t workspace_bytes, void* stream) {
  return run_pack(shape, W, nullptr, false, nullptr, vals, nm_idx, true, vec_idx, workspace, workspace_bytes, stream);
}

hinm_status hinm_pack_static(const hinm_shape* shape, const void* W, void* vals, uint8_t* nm_idx, int32_t* vec_idx,
                             void* stream) {
  hinm_status st = check_shape(shape);
  if (st != HINM_OK) return st;
  if (!W || !vals || !nm_idx || !vec_idx) return HINM_ERR_NULL;
  // the size limit comes before anything touches the device
  if ((size_t)(shape->M / shape->V) * (size_t)shape->K > kStaticScoreCount) return HINM_ERR_WORKSPACE;
  if (!aligned(vals, 8) || !aligned(vec_idx, 4) || !aligned(W, 2)) return HINM_ERR_SHAPE;
  double* scores = nullptr;
  if (static_scores(&scores) != hipSuccess) return HINM_ERR_DEVICE;
  // every score the select step reads is written by the score step of the same call: nothing to clear
  const PackArgs a{*shape, W, nullptr, nullptr, vals, nm_idx, vec_idx, scores};
  hipError_t e = launch_pack(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? HINM_OK : HINM_ERR_DEVICE;
}

hinm_status hinm_pack_ordered(const hinm_shape* shape, const void* W, const int32_t* tile_order, void* vals,
                              uint8_t* nm_idx, int32_t* vec_idx, void* workspace, size_t workspace_bytes,
                              void* stream) {
  return run_pack(shape, W, nullptr, false, tile_order, vals, nm_idx, true, vec_idx, workspace, workspace_bytes,
                  stream);
}

hinm_status hinm_pack_scored(const hinm_shape* shape, const void* W, const float* rho, const int32_t* tile_order,
                             void* vals, uint8_t* nm_idx, int32_t* vec_idx, void* workspace, size_t workspace_bytes,
                             void* stream) {
  return run_pack(shape, W, rho, true, tile_order, vals, nm_idx, true, vec_idx, workspace, workspace_bytes, stream);
}

hinm_status hinm_pack_vectors(const hinm_shape* shape, const void* W, const float* rho, const int32_t* tile_order,
                              void* vals_v, int32_t* vec_idx, void* workspace, size_t workspace_bytes, void* stream) {
  return run_pack(shape, W, rho, rho != nullptr, tile_order, vals_v, nullptr, false, vec_idx, workspace,
                  workspace_bytes, stream);
}

hinm_status hinm_apply_row_order(const void* src, void* dst, const int32_t* row_order, int32_t rows, size_t row_bytes,
                                 void* stream) {
  if (!src || !dst || !row_order) return HINM_ERR_NULL;
  if (rows <= 0 || row_bytes == 0 || row_bytes % 4 != 0 || !aligned(src, 4) || !aligned(dst, 4) || !aligned(row_order, 4) ||
      src == dst)
    return HINM_ERR_SHAPE;
  return launch_gather_rows(src, dst, row_order, rows, row_bytes, static_cast<hipStream_t>(stream)) == hipSuccess
             ? HINM_OK
             : HINM_ERR_DEVICE;
}

hinm_status hinm_tile_order(const hinm_shape* shape, const int32_t* vec_idx, int32_t* tile_order, void* stream) {
  hinm_status st = check_shape(shape);
  if (st != HINM_OK) return st;
  if (!vec_idx || !tile_order) return HINM_ERR_NULL;
  if (!aligned(vec_idx, 4) || !aligned(tile_order, 4)) return HINM_ERR_SHAPE;
  if (shape->K > kPackOrderMaxK) return HINM_ERR_UNSUPPORTED;
  return launch_tile_order(*shape, vec_idx, tile_order, static_cast<hipStream_t>(stream)) == hipSuccess ? HINM_OK
                                                                                                          : HINM_ERR_DEVICE;
}

static hinm_status check_icp_shape(const hinm_shape* shape) {
  hinm_status st = check_shape(shape);
  if (st != HINM_OK) return st;
  if (shape->Kv / 4 > kIcpMaxPartitions || shape->M / shape->V > 65535 || shape->V > 65535) return HINM_ERR_UNSUPPORTED;
  return HINM_OK;
}

hinm_status hinm_icp_sizes(const hinm_shape* shape, size_t* workspace_bytes) {
  hinm_status st = check_icp_shape(shape);
  if (st != HINM_OK) return st;
  if (!workspace_bytes) return HINM_ERR_NULL;
  *workspace_bytes = icp_workspace_layout(*shape).total_bytes;
  return HINM_OK;
}

hinm_status hinm_icp_search(const hinm_shape* shape, const void* W, const float* rho, int32_t* vec_idx,
                            const uint8_t* samples, int32_t iters, double* objective, void* workspace,
                            size_t workspace_bytes, void* stream) {
  hinm_status st = check_icp_shape(shape);
  if (st != HINM_OK) return st;
  if ((!W && !rho) || !vec_idx || (iters > 0 && !samples)) return HINM_ERR_NULL;
  if (iters < 0) return HINM_ERR_SHAPE;
  if (!aligned(vec_idx, 4) || (rho && !aligned(rho, 4)) || (!rho && !aligned(W, 2)) ||
      (objective && !aligned(objective, 8)))
    return HINM_ERR_SHAPE;
  const size_t need = icp_workspace_layout(*shape).total_bytes;
  if (!workspace || workspace_bytes < need || !aligned(workspace, 256)) return HINM_ERR_WORKSPACE;
  if (iters == 0) return HINM_OK;
  const IcpArgs a{*shape, W, rho, vec_idx, samples, iters, objective, workspace};
  hipError_t e = launch_icp_search(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? HINM_OK : HINM_ERR_DEVICE;
}

static hinm_status check_ocp_shape(const hinm_shape* shape, int32_t n_samples) {
  hinm_status st = check_shape(shape);
  if (st != HINM_OK) return st;
  if (n_samples < 1 || n_samples > shape->V) return HINM_ERR_SHAPE;
  if (shape->M / shape->V > kIcpMaxPartitions || shape->K > kOcpMaxK || shape->V > kOcpMaxV) return HINM_ERR_UNSUPPORTED;
  return HINM_OK;
}

hinm_status hinm_ocp_sizes(const hinm_shape* shape, int32_t n_samples, size_t* workspace_bytes) {
  hinm_status st = check_ocp_shape(shape, n_samples);
  if (st != HINM_OK) return st;
  if (!workspace_bytes) return HINM_ERR_NULL;
  *workspace_bytes = ocp_workspace_layout(*shape, n_samples).total_bytes;
  return HINM_OK;
}

hinm_status hinm_ocp_search(const hinm_shape* shape, const void* W, const float* rho, int32_t* row_order,
                            const int32_t* samples, const int32_t* clusters, int32_t n_samples, int32_t iters,
                            double* objective, void* workspace, size_t workspace_bytes, void* stream) {
  hinm_status st = check_ocp_shape(shape, n_samples);
  if (st != HINM_OK) return st;
  if ((!W && !rho) || !row_order || (iters > 0 && !samples)) return HINM_ERR_NULL;
  if (iters < 0) return HINM_ERR_SHAPE;
  if (!aligned(row_order, 4) || !aligned(samples, 4) || !aligned(clusters, 4) || (rho && !aligned(rho, 4)) ||
      (!rho && !aligned(W, 2)) || (objective && !aligned(objective, 8)))
    return HINM_ERR_SHAPE;
  const size_t need = ocp_workspace_layout(*shape, n_samples).total_bytes;
  if (!workspace || workspace_bytes < need || !aligned(workspace, 256)) return HINM_ERR_WORKSPACE;
  if (iters == 0) return HINM_OK;
  const OcpArgs a{*shape, W, rho, row_order, samples, clusters, n_samples, iters, objective, workspace};
  hipError_t e = launch_ocp_search(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? HINM_OK : HINM_ERR_DEVICE;
}

static hinm_status check_cluster_shape(const hinm_shape* shape, int32_t n_samples) {
  hinm_status st = check_ocp_shape(shape, n_samples);
  if (st != HINM_OK) return st;
  if ((int64_t)(shape->M / shape->V) * n_samples > kIcpMaxPartitions) return HINM_ERR_UNSUPPORTED;
  return HINM_OK;
}

hinm_status hinm_ocp_cluster_sizes(const hinm_shape* shape, int32_t n_samples, size_t* workspace_bytes) {
  hinm_status st = check_cluster_shape(shape, n_samples);
  if (st != HINM_OK) return st;
  if (!workspace_bytes) return HINM_ERR_NULL;
  *workspace_bytes = kmeans_workspace_layout(*shape, n_samples).total_bytes;
  return HINM_OK;
}

hinm_status hinm_ocp_cluster(const hinm_shape* shape, const void* W, const float* rho, const int32_t* row_order,
                             const int32_t* samples, int32_t n_samples, int32_t rounds, double* centroids,
                             int32_t init_centroids, int32_t* clusters, double* objective, void* workspace,
                             size_t workspace_bytes, void* stream) {
  hinm_status st = check_cluster_shape(shape, n_samples);
  if (st != HINM_OK) return st;
  if ((!W && !rho) || !row_order || !samples || !centroids || !clusters) return HINM_ERR_NULL;
  if (rounds < 1) return HINM_ERR_SHAPE;
  if (!aligned(row_order, 4) || !aligned(samples, 4) || !aligned(clusters, 4) || !aligned(centroids, 8) ||
      (rho && !aligned(rho, 4)) || (!rho && !aligned(W, 2)) || (objective && !aligned(objective, 8)))
    return HINM_ERR_SHAPE;
  const size_t need = kmeans_workspace_layout(*shape, n_samples).total_bytes;
  if (!workspace || workspace_bytes < need || !aligned(workspace, 256)) return HINM_ERR_WORKSPACE;
  const KmeansArgs a{*shape, W, rho, row_order, samples, n_samples, rounds, centroids, init_centroids != 0,
                     clusters, objective, workspace};
  hipError_t e = launch_ocp_cluster(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? HINM_OK : HINM_ERR_DEVICE;
}

hinm_status hinm_unpack(const hinm_shape* shape, const void* vals, const uint8_t* nm_idx, const int32_t* vec_idx,
                        void* W_out, void* stream) {
  hinm_status st = check_shape(shape);
  if (st != HINM_OK) return st;
  if (!vals || !nm_idx || !vec_idx || !W_out) return HINM_ERR_NULL;
  hipError_t e = launch_unpack(*shape, vals, nm_idx, vec_idx, W_out, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? HINM_OK : HINM_ERR_DEVICE;
}

hinm_status hinm_spmm(const hinm_shape* shape, int32_t N, const void* vals, const uint8_t* nm_idx,
                      const int32_t* vec_idx, const int32_t* pi_in, const int32_t* pi_out, const void* X, int64_t ldx,
                      void* Y, int64_t ldy, uint32_t flags, void* workspace, size_t workspace_bytes, void* stream) {
  (void)workspace;
  (void)workspace_bytes;
  hinm_status st = check_spmm(shape, N, vals, nm_idx, vec_idx, X, ldx, Y, ldy, flags);
  if (st != HINM_OK) return st;
  SpmmArgs a{*shape, N, vals, nm_idx, vec_idx, pi_in, pi_out, X, ldx, Y, ldy,
             (flags & HINM_EPI_RELU) != 0, (flags & HINM_OUT_F32) != 0};
  return run_spmm(a, flags, static_cast<hipStream_t>(stream));
}

hinm_status hinm_spmm_vectors(const hinm_shape* shape, int32_t N, const void* vals_v, const int32_t* vec_idx,
                              const int32_t* pi_in, const int32_t* pi_out, const void* X, int64_t ldx, void* Y,
                              int64_t ldy, uint32_t flags, void* stream) {
  hinm_status st = check_shape(shape);
  if (st != HINM_OK) return st;
  if (!vals_v || !vec_idx || !X || !Y) return HINM_ERR_NULL;
  if (N <= 0 || ldx < N || ldy < N) return HINM_ERR_SHAPE;
  if (N > 1 && (ldx % 8 != 0 || ldy % 8 != 0)) return HINM_ERR_SHAPE;
  if (!aligned(vals_v, 16) || !aligned(X, 16) || !aligned(Y, 16)) return HINM_ERR_SHAPE;
  if (flags & ~(uint32_t)(HINM_EPI_RELU | HINM_OUT_F32 | HINM_KERNEL_REFERENCE | HINM_VARIANT_MASK))
    return HINM_ERR_UNSUPPORTED;
  const int variant = (int)((flags & HINM_VARIANT_MASK) >> HINM_VARIANT_SHIFT);
  if (variant && (flags & HINM_KERNEL_REFERENCE)) return HINM_ERR_UNSUPPORTED;
  const VectorsArgs a{*shape, N, vals_v, vec_idx, pi_in, pi_out, X, ldx, Y, ldy,
                      (flags & HINM_EPI_RELU) != 0, (flags & HINM_OUT_F32) != 0, variant};
  hipError_t e;
  const bool rings = variant >= kRingFirstVariant && variant <= kRingLastVariant;
  // a pinned kernel must fit the shape
  if (variant && !(rings ? spmm_ring_vectors_supported(a) : spmm_vectors_mfma_supported(a))) return HINM_ERR_UNSUPPORTED;
  if (!(flags & HINM_KERNEL_REFERENCE) && !variant && N == 1)
    e = launch_spmm_vectors_gemv(a, static_cast<hipStream_t>(stream));
  else if (rings || (!(flags & HINM_KERNEL_REFERENCE) && !variant && spmm_ring_vectors_preferred(a)))
    e = launch_spmm_ring_vectors(a, static_cast<hipStream_t>(stream));
  else if (!(flags & HINM_KERNEL_REFERENCE) && !variant && spmm_mid_vectors_preferred(a))
    e = launch_spmm_mid_vectors(a, static_cast<hipStream_t>(stream));
  else if (!(flags & HINM_KERNEL_REFERENCE) && spmm_vectors_mfma_supported(a))
    e = launch_spmm_vectors_mfma(a, static_cast<hipStream_t>(stream));
  else
    e = launch_spmm_vectors_plain(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? HINM_OK : HINM_ERR_DEVICE;
}

// Which kernel family a prepared call runs on; everything that can make the call fail is decided here, on the
// host, before anything is launched (hinm_chain validates every layer with it before its first launch).
enum class PreparedRoute { Mid, MidRing, Rows16, Skinny, Panel, Tile, TileRing };

static hinm_status check_prepared_call(const hinm_shape* shape, int32_t N, const void* prepared, const void* X,
                                       int64_t ldx, const void* Y, int64_t ldy, uint32_t flags, void* workspace,
                                       size_t workspace_bytes, PreparedRoute* route);
static hinm_status run_prepared(const hinm_shape* shape, int32_t N, const void* prepared, const void* X, int64_t ldx,
                                void* Y, int64_t ldy, uint32_t flags, void* workspace, size_t workspace_bytes,
                                PreparedRoute route, hipStream_t stream, LaunchPlan* plan);

static hinm_status check_chain(int32_t L, const hinm_layer* layers, int32_t N, size_t* bytes_per_buffer) {
  if (!layers) return HINM_ERR_NULL;
  if (L <= 0 || N <= 0) return HINM_ERR_SHAPE;
  size_t widest = 0;
  for (int l = 0; l < L; ++l) {
    hinm_status st = check_shape(&layers[l].shape);
    if (st != HINM_OK) return st;
    if (!layers[l].prepared && (!layers[l].vals || !layers[l].nm_idx || !layers[l].vec_idx)) return HINM_ERR_NULL;
    if (layers[l].shape.dtype != layers[0].shape.dtype) return HINM_ERR_DTYPE;
    if (l > 0 && layers[l].shape.K != layers[l - 1].shape.M) return HINM_ERR_SHAPE;
    if (l + 1 < L && (layers[l].flags & HINM_OUT_F32)) return HINM_ERR_UNSUPPORTED;
    if (l + 1 < L) {
      const size_t b = (size_t)layers[l].shape.M * (size_t)((N + 7) / 8 * 8) * 2;
      widest = b > widest ? b : widest;
    }
  }
  *bytes_per_buffer = (widest + 255) / 256 * 256;
  return HINM_OK;
}

hinm_status hinm_chain_sizes(int32_t L, const hinm_layer* layers, int32_t N, size_t* scratch_bytes) {
  if (!scratch_bytes) return HINM_ERR_NULL;
  size_t per = 0;
  hinm_status st = check_chain(L, layers, N, &per);
  if (st != HINM_OK) return st;
  *scratch_bytes = (L <= 1) ? 0 : (L == 2 ? per : 2 * per);
  return HINM_OK;
}

hinm_status hinm_chain(int32_t L, const hinm_layer* layers, int32_t N, const void* X, int64_t ldx, void* Y,
                       int64_t ldy, void* scratch, size_t scratch_bytes, void* stream) {
  size_t per = 0;
  hinm_status st = check_chain(L, layers, N, &per);
  if (st != HINM_OK) return st;
  if (!X || !Y) return HINM_ERR_NULL;
  const size_t need = (L <= 1) ? 0 : (L == 2 ? per : 2 * per);
  if (need > 0 && (!scratch || scratch_bytes < need || !aligned(scratch, 256))) return HINM_ERR_WORKSPACE;
  // one column is packed: 4096 x 11008 at 50 % gathers its input from 22 KB then, not from 176 KB, and stages it in LDS
  // (13.6 -> 8.9 us behind an 11008 x 4096 layer)
  const int64_t ldh = N == 1 ? 1 : (N + 7) / 8 * 8;
  // validate every layer's call before launching the first one
  constexpr int kKeptRoutes = 8;
  PreparedRoute routes[kKeptRoutes], route;  // of the first layers; the others' are worked out again
  for (int l = 0; l < L; ++l) {
    const void* in = (l == 0) ? X : scratch;
    void* out = (l == L - 1) ? Y : scratch;
    if (layers[l].prepared)
      st = check_prepared_call(&layers[l].shape, N, layers[l].prepared, in, l == 0 ? ldx : ldh, out,
                               l == L - 1 ? ldy : ldh, layers[l].flags, nullptr, 0, &(l < kKeptRoutes ? routes[l] : route));
    else
      st = check_spmm(&layers[l].shape, N, layers[l].vals, layers[l].nm_idx, layers[l].vec_idx, in,
                      l == 0 ? ldx : ldh, out, l == L - 1 ? ldy : ldh, layers[l].flags);
    if (st != HINM_OK) return st;
  }
  char* buf[2] = {static_cast<char*>(scratch), static_cast<char*>(scratch) + per};
  const void* in = X;
  int64_t ld_in = ldx;
  for (int l = 0; l < L; ++l) {
    const bool last = (l == L - 1);
    void* out = last ? Y : static_cast<void*>(buf[l & 1]);
    const int64_t ld_out = last ? ldy : ldh;
    const hinm_layer& ly = layers[l];
    if (ly.prepared) {
      if (l < kKeptRoutes) route = routes[l];
      else check_prepared_call(&ly.shape, N, ly.prepared, in, ld_in, out, ld_out, ly.flags, nullptr, 0, &route);
      st = run_prepared(&ly.shape, N, ly.prepared, in, ld_in, out, ld_out, ly.flags, nullptr, 0, route,
                        static_cast<hipStream_t>(stream), nullptr);
    } else {
      SpmmArgs a{ly.shape, N, ly.vals, ly.nm_idx, ly.vec_idx, ly.pi_in, ly.pi_out, in, ld_in, out, ld_out,
                 (ly.flags & HINM_EPI_RELU) != 0, (ly.flags & HINM_OUT_F32) != 0};
      st = run_spmm(a, ly.flags, static_cast<hipStream_t>(stream));
    }
    if (st != HINM_OK) return st;
    in = out;
    ld_in = ld_out;
  }
  return HINM_OK;
}


hinm_status hinm_prepare_sizes(const hinm_shape* shape, size_t* prepared_bytes) {
  hinm_status st = check_shape(shape);
  if (st != HINM_OK) return st;
  if (!prepared_bytes) return HINM_ERR_NULL;
  if (shape->V % 32 != 0 || shape->V > 128) return HINM_ERR_UNSUPPORTED;
  *prepared_bytes = prepared_layout(*shape).total_bytes;
  return HINM_OK;
}

hinm_status hinm_prepare(const hinm_shape* shape, const void* vals, const uint8_t* nm_idx, const int32_t* vec_idx,
                         const int32_t* pi_in, const int32_t* pi_out, void* prepared, size_t prepared_bytes,
                         void* stream) {
  size_t need = 0;
  hinm_status st = hinm_prepare_sizes(shape, &need);
  if (st != HINM_OK) return st;
  if (!vals || !nm_idx || !vec_idx || !prepared) return HINM_ERR_NULL;
  if (prepared_bytes < need || !aligned(prepared, 256)) return HINM_ERR_WORKSPACE;
  hipError_t e = launch_prepare(*shape, vals, nm_idx, vec_idx, pi_in, pi_out, prepared,
                                static_cast<hipStream_t>(stream));
  return e == hipSuccess ? HINM_OK : HINM_ERR_DEVICE;
}

hinm_status hinm_spmm_prepared_workspace(const hinm_shape* shape, int32_t N, size_t* workspace_bytes) {
  size_t need = 0;
  hinm_status st = hinm_prepare_sizes(shape, &need);
  if (st != HINM_OK) return st;
  if (!workspace_bytes) return HINM_ERR_NULL;
  if (N <= 0) return HINM_ERR_SHAPE;
  *workspace_bytes = (N <= 32) ? skinny_prepared_workspace_bytes(*shape, N) : 0;
  return HINM_OK;
}

static PreparedArgs prepared_args(const hinm_shape* shape, int32_t N, const void* prepared, const void* X, int64_t ldx,
                                  void* Y, int64_t ldy, uint32_t flags, void* workspace, size_t workspace_bytes) {
  return PreparedArgs{*shape, N, prepared, X, ldx, Y, ldy, (flags & HINM_EPI_RELU) != 0, (flags & HINM_OUT_F32) != 0,
                      (int)((flags & HINM_VARIANT_MASK) >> HINM_VARIANT_SHIFT), workspace, workspace_bytes};
}

// with_mid = false: as if there were no kernel for a moderate number of columns (what the measurement launches of the
// tile kernel go by, which serve shapes that now run on that kernel too).
static hinm_status route_prepared(const PreparedArgs& a, PreparedRoute* route, bool with_mid = true) {
  const hinm_shape* shape = &a.s;
  const int32_t N = a.N;
  if (a.tile_variant >= kRingFirstVariant && a.tile_variant <= kRingLastVariant) {
    if (!spmm_ring_prepared_supported(a)) return HINM_ERR_UNSUPPORTED;
    *route = PreparedRoute::TileRing;
    return HINM_OK;
  }
  // From 65 columns on: the kernel with private rings wherever it can run, unless one of the kernels for fewer columns is
  // estimated to take less (with a margin, spmm_rings.hip).  Up to five steps it and the one for a moderate number of columns
  // are within a tenth of each other (3008 x 560, Kv = 280, N = 273 5.4 us there and 5.9; 1312 x 1048, V = 32, Kv = 264, N = 681
  // 5.4 and 5.3).
  const bool ring = with_mid && a.tile_variant == 0 && N > 64 && spmm_ring_prepared_supported(a);
  if (with_mid && a.tile_variant == 0 && spmm_mid_prepared_preferred(a)) {
    *route = ring && shape->Kv > 5 * 64 && spmm_ring_prepared_us(a, true) < spmm_mid_prepared_us(a) ? PreparedRoute::MidRing : PreparedRoute::Mid;
    return HINM_OK;
  }
  // What the kernel for a moderate number of columns leaves: one column, up to 64 columns (128 on the smallest layers) where it
  // is behind, V % 64 != 0 beyond 768 of its blocks, and many columns.  Up to 64 columns that is the 16-row kernel (16x16x64
  // form, faster than the 32-row one on every decode shape tried, by 8-10 % with 344 row blocks of 32 and by 15-37 % with
  // 128); variant 11 pins it for any N, 19 its form with the input rows resident in LDS (16 columns only).
  if (a.tile_variant == 19 && !spmm_rows16_resident_supported(a)) return HINM_ERR_UNSUPPORTED;
  // Beyond, up to 2048 columns, it is the 16-row kernel while its cost, which grows with M * Kv * ceil(N / 16), stays under
  // the tile kernels' floor of one serial pass over the kept columns (about 15 us per 1024 of them, a little more per column
  // on short passes): V = 32 and 96 with long passes among products, and every shape for hinm_calib_tile_part, which goes by
  // the choice between these two alone.  The constants are fitted to timings of 42 (layer, N) pairs between 512 x 4608
  // and 8192 x 8192 and checked on some 250 more at other N.
  bool few_columns = N <= 64;
  if (!few_columns && N <= 2048) {
    const double units = (double)shape->M * ((N + 15) / 16);
    // the tile kernels' pass: 15 us per 1024 kept columns (12 with tiles of up to 64 rows: smaller stages,
    // 128-column stages where the step count is even), and on short passes 2 us more, 4 with 128-row tiles
    const double tile_floor_us =
        shape->V >= 96 ? 1.0 + 15.0 * shape->Kv / 1024.0 + (shape->Kv <= 1024 ? (shape->V >= 128 ? 4.0 : 2.0) : 0.0)
                       : 2.0 + 12.0 * shape->Kv / 1024.0 + (shape->Kv <= 1024 ? 2.0 : 0.0);
    // with two column blocks per workgroup the 16-row kernel measured 19-34 % faster, with four as much again
    const int blocks_per_wg = spmm_rows16_prepared_blocks_per_wg(a);
    const double pair_factor = blocks_per_wg == 4 ? 0.58 : blocks_per_wg == 2 ? 0.78 : 1.0;
    // beyond 512 columns X (K x N) often outgrows one L2 and the gathers slow down, those that use a quarter
    // or half of each cache line first (measured on small layers up to N = 4096: the kernel still wins to
    // 1024..2048 columns on layers of a few hundred rows)
    const bool x_beyond_l2 = (double)shape->K * N * 2 > 3.5e6;
    const double l2_factor = !x_beyond_l2 ? 1.0 : N > 1024 ? 2.0 : (N > 512 && blocks_per_wg < 4) ? 1.5 : 1.0;
    // on tall layers of 32-row tiles that cost is 1.6 times the estimate (median of 430 drawn ones; 13664 x 3936, Kv = 496,
    // N = 84 11.1 us, rings 8.7; 12640 x 13784, Kv = 1720, N = 96 31.5 and 17.0): said to the rings alone, whose estimate is
    // of such layers
    const double cost = units * (0.14 * shape->Kv + 40.0) * 1e-6 * l2_factor * pair_factor;
    few_columns = 2.5 + cost < tile_floor_us &&
                  !(ring && spmm_ring_prepared_us(a, false) <= 2.5 + cost * (shape->V == 32 ? 1.6 : 1.0));
  }
  if (a.tile_variant == 11 || a.tile_variant == 19 || (a.tile_variant == 0 && few_columns)) {
    if ((N + 15) / 16 > 65535) return HINM_ERR_UNSUPPORTED;
    *route = PreparedRoute::Rows16;
  } else if (N <= 32 && (a.tile_variant == 0 || a.tile_variant == 12)) {  // variant 12 pins the 32-row skinny kernel
    const size_t need = skinny_prepared_workspace_bytes(*shape, N);
    if (need > 0 && (!a.workspace || a.workspace_bytes < need || !aligned(a.workspace, 256)))
      return HINM_ERR_WORKSPACE;
    *route = PreparedRoute::Skinny;
  } else {
    if (N == 1 || a.ldx % 8 != 0 || a.ldy % 8 != 0 || a.tile_variant == 12) return HINM_ERR_UNSUPPORTED;
    // 128-row tiles leave the panel kernel's waves two tiles' registers and no depth: rings are ahead on all of 50 drawn layers
    // (1.24 times; 2304 x 856, Kv = 432, N = 3153 20.5 against 11.4 us); up to 96 rows the two are level or the panel is ahead
    // (64 rows: 0.99, 13440 x 704, Kv = 176, N = 7601 58 against 82 us).
    const bool panel = (a.tile_variant == 15) ||
                       (a.tile_variant == 0 && !(ring && shape->V == 128) && spmm_panel_prepared_preferred(a));
    if (panel && !spmm_panel_prepared_supported(a)) return HINM_ERR_UNSUPPORTED;
    *route = panel ? PreparedRoute::Panel : ring ? PreparedRoute::TileRing : PreparedRoute::Tile;
  }
  return HINM_OK;
}

static hinm_status check_prepared_call(const hinm_shape* shape, int32_t N, const void* prepared, const void* X,
                                       int64_t ldx, const void* Y, int64_t ldy, uint32_t flags, void* workspace,
                                       size_t workspace_bytes, PreparedRoute* route) {
  size_t need = 0;
  hinm_status st = hinm_prepare_sizes(shape, &need);
  if (st != HINM_OK) return st;
  if (!prepared || !X || !Y) return HINM_ERR_NULL;
  if (N <= 0 || ldx < N || ldy < N) return HINM_ERR_SHAPE;
  if (N > 1 && (ldx % 8 != 0 || ldy % 8 != 0)) return HINM_ERR_SHAPE;
  if (!aligned(prepared, 256) || !aligned(X, 16) || !aligned(Y, 16)) return HINM_ERR_SHAPE;
  if (flags & ~(uint32_t)(HINM_EPI_RELU | HINM_OUT_F32 | HINM_VARIANT_MASK)) return HINM_ERR_UNSUPPORTED;
  return route_prepared(prepared_args(shape, N, prepared, X, ldx, const_cast<void*>(Y), ldy, flags, workspace,
                                      workspace_bytes), route);
}

// The call has passed check_prepared_call, which found its route (once a call: with up to three estimates it costs 0.1 us).
static hinm_status run_prepared(const hinm_shape* shape, int32_t N, const void* prepared, const void* X, int64_t ldx,
                                void* Y, int64_t ldy, uint32_t flags, void* workspace, size_t workspace_bytes,
                                PreparedRoute route, hipStream_t stream, LaunchPlan* plan) {
  PreparedArgs a = prepared_args(shape, N, prepared, X, ldx, Y, ldy, flags, workspace, workspace_bytes);
  a.plan = plan;
  hipError_t e = hipSuccess;
  switch (route) {
    case PreparedRoute::Mid: e = launch_spmm_mid_prepared(a, stream); break;
    case PreparedRoute::Rows16: e = launch_spmm_rows16_prepared(a, stream); break;
    case PreparedRoute::Skinny: e = launch_spmm_skinny_prepared(a, stream); break;
    case PreparedRoute::Panel: e = launch_spmm_panel_prepared(a, stream); break;
    case PreparedRoute::Tile: e = launch_spmm_tile_prepared(a, stream); break;
    case PreparedRoute::MidRing:
    case PreparedRoute::TileRing: e = launch_spmm_ring_prepared(a, route == PreparedRoute::MidRing, stream); break;
  }
  return e == hipSuccess ? HINM_OK : HINM_ERR_DEVICE;
}

hinm_status hinm_spmm_prepared(const hinm_shape* shape, int32_t N, const void* prepared, const void* X, int64_t ldx,
                               void* Y, int64_t ldy, uint32_t flags, void* workspace, size_t workspace_bytes,
                               void* stream) {
  PreparedRoute route;
  hinm_status st = check_prepared_call(shape, N, prepared, X, ldx, Y, ldy, flags, workspace, workspace_bytes, &route);
  if (st != HINM_OK) return st;
  return run_prepared(shape, N, prepared, X, ldx, Y, ldy, flags, workspace, workspace_bytes, route,
                      static_cast<hipStream_t>(stream), nullptr);
}

hinm_status hinm_spmm_prepared_plan(const hinm_shape* shape, int32_t N, int64_t ldx, int64_t ldy, uint32_t flags,
                                    char* text, size_t text_bytes, int32_t* launches) {
  if (!text || text_bytes == 0) return HINM_ERR_NULL;
  text[0] = 0;
  // stand-ins with the alignment of real buffers: a dry run dereferences nothing
  void* const fake = reinterpret_cast<void*>(uintptr_t{1} << 20);
  PreparedRoute route;
  hinm_status st = check_prepared_call(shape, N, fake, fake, ldx, fake, ldy, flags, fake, ~size_t{0}, &route);
  if (st != HINM_OK) return st;
  LaunchPlan plan{text, text_bytes};
  st = run_prepared(shape, N, fake, fake, ldx, fake, ldy, flags, fake, ~size_t{0}, route, nullptr, &plan);
  if (launches) *launches = plan.launches;
  return st;
}

hinm_status hinm_calib_tile_part(const hinm_shape* shape, int32_t N, const void* prepared, const void* X, int64_t ldx,
                                 int32_t part, void* stream) {
  // Y is never written: any aligned non-NULL stand-in passes the checks
  void* const no_y = reinterpret_cast<void*>(uintptr_t{1} << 20);
  PreparedRoute route;
  hinm_status st = check_prepared_call(shape, N, prepared, X, ldx, no_y, (N + 7) / 8 * 8, 0, nullptr, 0, &route);
  if (st != HINM_OK) return st;
  if (part != 1 && part != 2) return HINM_ERR_UNSUPPORTED;
  PreparedArgs a = prepared_args(shape, N, prepared, X, ldx, no_y, (N + 7) / 8 * 8, 0, nullptr, 0);
  st = route_prepared(a, &route, false);
  if (st != HINM_OK) return st;
  if (route != PreparedRoute::Tile) return HINM_ERR_UNSUPPORTED;
  hipError_t e = launch_spmm_tile_prepared_part(a, part, static_cast<hipStream_t>(stream));
  if (e == hipErrorNotSupported) return HINM_ERR_UNSUPPORTED;
  return e == hipSuccess ? HINM_OK : HINM_ERR_DEVICE;
}

hinm_status hinm_calib_mid_plan(const hinm_shape* shape, int32_t N, int32_t form, char* text, size_t text_bytes) {
  hinm_status st = check_shape(shape);
  if (st != HINM_OK) return st;
  if (!text || text_bytes == 0) return HINM_ERR_NULL;
  if (N <= 0 || form < 0 || form > 1) return HINM_ERR_SHAPE;
  text[0] = 0;
  const int64_t ld = N == 1 ? 1 : ((int64_t)N + 7) / 8 * 8;
  LaunchPlan plan{text, text_bytes};
  hipError_t e = hipSuccess;
  if (form == 0) {
    SpmmArgs a{*shape, N, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, ld, nullptr, ld, false, false, &plan};
    if (spmm_mid_canonical_preferred(a)) e = launch_spmm_mid_canonical(a, nullptr);
  } else {
    VectorsArgs a{*shape, N, nullptr, nullptr, nullptr, nullptr, nullptr, ld, nullptr, ld, false, false, 0, &plan};
    if (spmm_mid_vectors_preferred(a) && !spmm_ring_vectors_preferred(a)) e = launch_spmm_mid_vectors(a, nullptr);
  }
  return e == hipSuccess ? HINM_OK : HINM_ERR_DEVICE;
}

hinm_status hinm_mx4_sizes(int32_t rows, int32_t length, size_t* code_bytes, size_t* scale_bytes) {
  if (rows <= 0 || length <= 0) return HINM_ERR_SHAPE;
  if (rows > kMostSize || length > kMostSize) return HINM_ERR_UNSUPPORTED;
  if (code_bytes) *code_bytes = (size_t)mx4_code_bytes(rows, length);
  if (scale_bytes) *scale_bytes = (size_t)mx4_scale_bytes(rows, length);
  return HINM_OK;
}

hinm_status hinm_mx4_quantize(int32_t rows, int32_t cols, int32_t dtype, const void* src, int64_t ld, int32_t along,
                              uint8_t* codes, uint8_t* scales, void* stream) {
  if (!known_dtype(dtype)) return HINM_ERR_DTYPE;
  if (rows <= 0 || cols <= 0) return HINM_ERR_SHAPE;
  if (!src) return HINM_ERR_NULL;
  const hinm_status st = check_form(codes, scales);
  if (st != HINM_OK) return st;
  if (ld < cols || !aligned(src, 2)) return HINM_ERR_SHAPE;
  if (along != HINM_MX4_ROWS && along != HINM_MX4_COLUMNS) return HINM_ERR_UNSUPPORTED;
  if (rows > kMostSize || cols > kMostSize || too_many_to_quantize(rows, cols, along == HINM_MX4_COLUMNS)) return HINM_ERR_UNSUPPORTED;
  return launched(launch_mx4_quantize(rows, cols, dtype, src, ld, along == HINM_MX4_COLUMNS, codes, scales,
                                      static_cast<hipStream_t>(stream)));
}

hinm_status hinm_mx4_unpack(int32_t rows, int32_t length, int32_t dtype, const uint8_t* codes, const uint8_t* scales, void* dst,
                            int64_t ld, void* stream) {
  if (!known_dtype(dtype)) return HINM_ERR_DTYPE;
  if (rows <= 0 || length <= 0) return HINM_ERR_SHAPE;
  if (!dst) return HINM_ERR_NULL;
  const hinm_status st = check_form(codes, scales);
  if (st != HINM_OK) return st;
  if (ld < length || !aligned(dst, 2)) return HINM_ERR_SHAPE;
  if (rows > kMostSize || length > kMostSize || (int64_t)mx4_row_blocks(rows) * mx4_groups(length) >= 2 * kMostGroups)
    return HINM_ERR_UNSUPPORTED;
  return launched(launch_mx4_unpack(rows, length, dtype, codes, scales, dst, ld, static_cast<hipStream_t>(stream)));
}

hinm_status hinm_mx4_product(int32_t M, int32_t N, int32_t K, int32_t dtype, const uint8_t* a_codes, const uint8_t* a_scales,
                             const uint8_t* b_codes, const uint8_t* b_scales, void* Y, int64_t ldy, uint32_t flags,
                             void* stream) {
  hinm_status st = check_product(M, N, K, dtype, Y, ldy, flags);
  if (st != HINM_OK) return st;
  if ((st = check_form(a_codes, a_scales)) != HINM_OK || (st = check_form(b_codes, b_scales)) != HINM_OK) return st;
  const Mx4ProductArgs a{M, N, K, dtype, a_codes, a_scales, b_codes, b_scales, Y, ldy, (flags & HINM_EPI_RELU) != 0,
                         (flags & HINM_OUT_F32) != 0};
  return launched(launch_mx4_product(a, static_cast<hipStream_t>(stream)));
}

hinm_status hinm_mx4_linear_workspace(int32_t M, int32_t K, int32_t N, size_t* workspace_bytes) {
  if (!workspace_bytes) return HINM_ERR_NULL;
  if (M <= 0 || K <= 0 || N <= 0) return HINM_ERR_SHAPE;
  if (M > kMostSize || K > kMostSize || N > kMostSize) return HINM_ERR_UNSUPPORTED;
  const LinearPlan p = linear_plan(K, N);
  *workspace_bytes = p.codes + p.scales;
  return HINM_OK;
}

hinm_status hinm_mx4_linear(int32_t M, int32_t K, int32_t N, int32_t dtype, const uint8_t* codes, const uint8_t* scales,
                            const void* X, int64_t ldx, void* Y, int64_t ldy, uint32_t flags, void* workspace,
                            size_t workspace_bytes, void* stream) {
  hinm_status st = check_product(M, N, K, dtype, Y, ldy, flags);
  if (st != HINM_OK) return st;
  if (!X) return HINM_ERR_NULL;
  if ((st = check_form(codes, scales)) != HINM_OK) return st;
  if (ldx < N || !aligned(X, 2)) return HINM_ERR_SHAPE;
  const LinearPlan p = linear_plan(K, N);
  if (!workspace || workspace_bytes < p.codes + p.scales || !aligned(workspace, 256)) return HINM_ERR_WORKSPACE;
  uint8_t* x_codes = static_cast<uint8_t*>(workspace);
  uint8_t* x_scales = x_codes + p.codes;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const Mx4ProductArgs a{M, N, K, dtype, codes, scales, x_codes, x_scales, Y, ldy, (flags & HINM_EPI_RELU) != 0,
                         (flags & HINM_OUT_F32) != 0};
  if (mx4_quantises_on_the_way(a)) return launched(launch_mx4_on_the_way(a, X, ldx, s));
  if (too_many_to_quantize(K, N, true)) return HINM_ERR_UNSUPPORTED;
  const hipError_t e = launch_mx4_quantize(K, N, dtype, X, ldx, true, x_codes, x_scales, s);
  return launched(e == hipSuccess ? launch_mx4_product(a, s) : e);
}

hinm_status hinm_calib_mx4_plan(int32_t M, int32_t N, int32_t K, int32_t dtype, uint32_t flags, int32_t quantize, char* text,
                                size_t text_bytes) {
  if (!text || text_bytes == 0) return HINM_ERR_NULL;
  text[0] = 0;
  void* const fake = reinterpret_cast<void*>(uintptr_t{1} << 20);  // never dereferenced
  const hinm_status st = check_product(M, N, K, dtype, fake, N, flags);
  if (st != HINM_OK) return st;
  LaunchPlan plan{text, text_bytes};
  const Mx4ProductArgs a{M, N, K, dtype, nullptr, nullptr, nullptr, nullptr, fake, N, (flags & HINM_EPI_RELU) != 0,
                         (flags & HINM_OUT_F32) != 0, &plan};
  if (quantize && mx4_quantises_on_the_way(a)) return launched(launch_mx4_on_the_way(a, fake, N, nullptr));
  if (quantize && too_many_to_quantize(K, N, true)) return HINM_ERR_UNSUPPORTED;
  if (quantize) plan_record(&plan, "mx4_columns_kernel<DT=%d>", dtype);
  return launched(launch_mx4_product(a, nullptr));
}

hinm_status hinm_block_norm_workspace(int32_t K, int32_t N, size_t* workspace_bytes) {
  if (!workspace_bytes) return HINM_ERR_NULL;
  const hinm_status st = check_norm(K, N, HINM_F16);
  if (st != HINM_OK) return st;
  *workspace_bytes = block_norm_workspace_bytes(K, N);
  return HINM_OK;
}

hinm_status hinm_block_norm(int32_t K, int32_t N, int32_t dtype, float residual_scale, float eps, const void* x, const void* y,
                            const float* w_post, const float* gate, const float* token_gate, const float* w_pre, void* h,
                            int64_t ld_stream, void* u, int64_t ld_block, float* rstd_y, float* rstd_h, void* workspace,
                            size_t workspace_bytes, void* stream) {
  const hinm_status st = check_norm(K, N, dtype);
  if (st != HINM_OK) return st;
  if (!x || (w_pre && !u) || (!w_pre && !h)) return HINM_ERR_NULL;
  if (!y && (w_post || gate || token_gate)) return HINM_ERR_NULL;
  if (ld_stream < N || ((y || w_pre) && ld_block < N)) return HINM_ERR_SHAPE;
  if (!aligned(x, 2) || !aligned(y, 2) || !aligned(h, 2) || !aligned(u, 2)) return HINM_ERR_SHAPE;
  for (const float* p : {w_post, gate, token_gate, w_pre, const_cast<const float*>(rstd_y), const_cast<const float*>(rstd_h)})
    if (!aligned(p, 4)) return HINM_ERR_SHAPE;
  const size_t need = block_norm_workspace_bytes(K, N);
  if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 256))) return HINM_ERR_WORKSPACE;
  const BlockNormArgs a{K, N, dtype, residual_scale, eps, x, y, w_post, gate, token_gate, w_pre, h, ld_stream,
                        w_pre ? u : nullptr, ld_block, w_post ? rstd_y : nullptr, w_pre ? rstd_h : nullptr,
                        static_cast<float*>(workspace)};
  return launched(launch_block_norm(a, static_cast<hipStream_t>(stream)));
}

hinm_status hinm_block_norm_grad_workspace(int32_t K, int32_t N, size_t* workspace_bytes) {
  if (!workspace_bytes) return HINM_ERR_NULL;
  const hinm_status st = check_norm(K, N, HINM_F16);
  if (st != HINM_OK) return st;
  *workspace_bytes = block_norm_grad_workspace_bytes(K, N);
  return HINM_OK;
}

hinm_status hinm_block_norm_grad(int32_t K, int32_t N, int32_t dtype, float residual_scale, const void* h, const void* y,
                                 const float* w_post, const float* gate, const float* token_gate, const float* w_pre,
                                 const float* rstd_y, const float* rstd_h, const void* dh, const void* du, void* dx,
                                 int64_t ld_stream, void* dy, int64_t ld_block, float* dw_post, float* dgate,
                                 float* dtoken_gate, float* dw_pre, void* workspace, size_t workspace_bytes, void* stream) {
  const hinm_status st = check_norm(K, N, dtype);
  if (st != HINM_OK) return st;
  if (w_pre ? (!h || !du || !rstd_h) : (du || !dh)) return HINM_ERR_NULL;
  if ((w_post && !rstd_y) || (!y && (w_post || gate || token_gate || dy))) return HINM_ERR_NULL;
  if ((dw_post && !w_post) || (dgate && !gate) || (dtoken_gate && !token_gate) || (dw_pre && !w_pre)) return HINM_ERR_NULL;
  if (((h && w_pre) || dh || dx) && ld_stream < N) return HINM_ERR_SHAPE;
  if ((y || du || dy) && ld_block < N) return HINM_ERR_SHAPE;
  for (const void* p : {h, y, dh, du, const_cast<const void*>(dx), const_cast<const void*>(dy)})
    if (!aligned(p, 2)) return HINM_ERR_SHAPE;
  for (const float* p : {w_post, gate, token_gate, w_pre, rstd_y, rstd_h, const_cast<const float*>(dw_post),
                         const_cast<const float*>(dgate), const_cast<const float*>(dtoken_gate), const_cast<const float*>(dw_pre)})
    if (!aligned(p, 4)) return HINM_ERR_SHAPE;
  if (too_many_to_add(K, N) && (dw_post || dgate || dw_pre)) return HINM_ERR_UNSUPPORTED;
  const size_t need = block_norm_grad_workspace_bytes(K, N);
  if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 256))) return HINM_ERR_WORKSPACE;
  const BlockNormGradArgs a{K, N, dtype, residual_scale, h, y, w_post, gate, token_gate, w_pre, rstd_y, rstd_h, dh, du, dx,
                            ld_stream, dy, ld_block, dw_post, dgate, dtoken_gate, dw_pre, static_cast<float*>(workspace)};
  return launched(launch_block_norm_grad(a, static_cast<hipStream_t>(stream)));
}

hinm_status hinm_linear_workspace(int32_t M, int32_t K, int32_t N, size_t* workspace_bytes) {
  if (!workspace_bytes) return HINM_ERR_NULL;
  const hinm_status st = check_layer(M, K, N);
  if (st != HINM_OK) return st;
  *workspace_bytes = dense_product_workspace_bytes(M, N, K, kAlong, kAcross);
  return HINM_OK;
}

hinm_status hinm_linear(int32_t M, int32_t K, int32_t N, int32_t dtype, const void* W, int64_t ldw, const void* X, int64_t ldx,
                        const float* bias, const void* residual, int64_t ldr, void* Z, void* Y, int64_t ldy, uint32_t flags,
                        void* workspace, size_t workspace_bytes, void* stream) {
  if (!known_dtype(dtype)) return HINM_ERR_DTYPE;
  const hinm_status st = check_layer(M, K, N);
  if (st != HINM_OK) return st;
  if (!W || !X || !Y) return HINM_ERR_NULL;
  const bool out_f32 = (flags & HINM_OUT_F32) != 0;
  if (ldw < K || ldx < N || ldy < N || (residual && ldr < N)) return HINM_ERR_SHAPE;
  if (!aligned(W, 2) || !aligned(X, 2) || !aligned(residual, 2) || !aligned(Z, 2) || !aligned(Y, out_f32 ? 4 : 2) || !aligned(bias, 4))
    return HINM_ERR_SHAPE;
  const int act = activation_of(flags);
  if (act < 0 || (flags & ~(kActFlags | HINM_OUT_F32))) return HINM_ERR_UNSUPPORTED;
  const size_t need = dense_product_workspace_bytes(M, N, K, kAlong, kAcross);
  if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 256))) return HINM_ERR_WORKSPACE;
  const LinearEpilogue to{M, N, bias, static_cast<const uint16_t*>(residual), ldr, pieces_of_rows(residual, ldr, N),
                          static_cast<uint16_t*>(Z), Y, ldy, act, out_f32};
  return launched(launch_dense_product({M, N, K, dtype, kAlong, kAcross, W, ldw, X, ldx, to, workspace}, static_cast<hipStream_t>(stream)));
}

hinm_status hinm_linear_grad_workspace(int32_t M, int32_t K, int32_t N, size_t* workspace_bytes) {
  if (!workspace_bytes) return HINM_ERR_NULL;
  const hinm_status st = check_dense_grad(M, K, N);
  if (st != HINM_OK) return st;
  const LinearGradPlan p = linear_grad_plan(M, K, N);
  *workspace_bytes = p.dz + p.x + p.product;
  return HINM_OK;
}

hinm_status hinm_linear_grad(int32_t M, int32_t K, int32_t N, int32_t dtype, const void* W, int64_t ldw, const void* X, int64_t ldx,
                             const void* Z, const void* dY, int64_t ldy, void* dX, void* dW, float* dbias, uint32_t flags,
                             void* workspace, size_t workspace_bytes, void* stream) {
  if (!known_dtype(dtype)) return HINM_ERR_DTYPE;
  hinm_status st = check_dense_grad(M, K, N);
  if (st != HINM_OK) return st;
  const int act = activation_of(flags);
  if (!dY || (!dX && !dW && !dbias) || (dX && !W) || (dW && !X) || (act > kActNone && !Z)) return HINM_ERR_NULL;
  const bool out_f32 = (flags & HINM_OUT_F32) != 0;
  if (ldy < N || (dX && (ldw < K || ldx < N)) || (dW && (ldw < K || ldx < N))) return HINM_ERR_SHAPE;
  if (!aligned(W, 2) || !aligned(X, 2) || !aligned(Z, 2) || !aligned(dY, 2) || !aligned(dX, 2) || !aligned(dW, out_f32 ? 4 : 2) ||
      !aligned(dbias, 4))
    return HINM_ERR_SHAPE;
  if (act < 0 || (flags & ~(kActFlags | HINM_OUT_F32))) return HINM_ERR_UNSUPPORTED;
  const LinearGradPlan p = linear_grad_plan(M, K, N);
  if (!workspace || workspace_bytes < p.dz + p.x + p.product || !aligned(workspace, 256)) return HINM_ERR_WORKSPACE;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const bool as_it_is = act == kActNone && pieces_of_rows(dY, ldy, N) == kAligned;
  uint16_t* const dz = as_it_is || (!dX && !dW) ? nullptr : static_cast<uint16_t*>(workspace);
  const LinearGradProducts g = linear_grad_products(p, M, K, N, dtype, W, ldw, X, ldx, dz ? dz : dY, dz ? p.ldz : ldy, dX, dW, out_f32,
                                                    workspace, nullptr);
  const bool sums_in_pair = g.pair && dbias && !dz && M <= kMostGroups;
  hipError_t e = hipSuccess;
  if (dz || (dbias && !sums_in_pair)) {
    const void* z = act == kActNone ? nullptr : Z;
    e = launch_linear_slope({M, N, static_cast<const uint16_t*>(z), static_cast<const uint16_t*>(dY), ldy,
                             lesser(pieces_of_rows(z, ldy, N), pieces_of_rows(dY, ldy, N)), act, dz, p.ldz, dbias}, dtype, s);
  }
  return launched(e == hipSuccess ? launch_grad_products(g, sums_in_pair ? dbias : nullptr, s) : e);
}

hinm_status hinm_calib_linear_plan(int32_t M, int32_t K, int32_t N, int32_t dtype, int32_t which, int32_t is_aligned, char* text,
                                   size_t text_bytes) {
  if (!text || text_bytes == 0) return HINM_ERR_NULL;
  text[0] = 0;
  if (!known_dtype(dtype)) return HINM_ERR_DTYPE;
  const hinm_status st = which == 0 ? check_layer(M, K, N) : check_dense_grad(M, K, N);
  if (st != HINM_OK) return st;
  if (which < 0 || which > 3) return HINM_ERR_UNSUPPORTED;
  LaunchPlan plan{text, text_bytes};
  const void* const aligned_at = reinterpret_cast<const void*>(uintptr_t{1} << 20);  // never dereferenced
  const void* const at = reinterpret_cast<const void*>((uintptr_t{1} << 20) + (is_aligned ? 0 : 2));
  auto pitch = [](int32_t n) { return ((int64_t)n + 7) / 8 * 8; };
  void* const written = const_cast<void*>(aligned_at);
  if (which == 0) {
    const LinearEpilogue to{M, N, nullptr, nullptr, 0, kAligned, nullptr, nullptr, pitch(N), kActNone, false};
    return launched(launch_dense_product({M, N, K, dtype, kAlong, kAcross, at, pitch(K), aligned_at, pitch(N), to, written, &plan}, nullptr));
  }
  return launched(launch_grad_products(linear_grad_products(linear_grad_plan(M, K, N), M, K, N, dtype, which == 2 ? aligned_at : at, pitch(K),
                                                            which == 2 ? at : aligned_at, pitch(N), aligned_at, pitch(N),
                                                            which == 2 ? nullptr : written, which == 1 ? nullptr : written, false, written,
                                                            &plan), nullptr, nullptr));
}

hinm_status hinm_layer_norm_workspace(int32_t K, int32_t N, size_t* workspace_bytes) {
  if (!workspace_bytes) return HINM_ERR_NULL;
  const hinm_status st = check_norm(K, N, HINM_F16);
  if (st != HINM_OK) return st;
  *workspace_bytes = layer_norm_workspace_bytes(K, N);
  return HINM_OK;
}

hinm_status hinm_layer_norm(int32_t K, int32_t N, int32_t dtype, float eps, const void* x, int64_t ldx, const float* w, const float* b,
                            void* u, int64_t ldu, float* mean, float* rstd, void* workspace, size_t workspace_bytes, void* stream) {
  const hinm_status st = check_norm(K, N, dtype);
  if (st != HINM_OK) return st;
  if (!x || !u) return HINM_ERR_NULL;
  if (ldx < N || ldu < N || !aligned(x, 2) || !aligned(u, 2)) return HINM_ERR_SHAPE;
  if (!aligned(w, 4) || !aligned(b, 4) || !aligned(mean, 4) || !aligned(rstd, 4)) return HINM_ERR_SHAPE;
  const size_t need = layer_norm_workspace_bytes(K, N);
  if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 256))) return HINM_ERR_WORKSPACE;
  return launched(launch_layer_norm({K, N, dtype, eps, x, ldx, w, b, u, ldu, mean, rstd, static_cast<float*>(workspace)},
                                    static_cast<hipStream_t>(stream)));
}

hinm_status hinm_layer_norm_grad_workspace(int32_t K, int32_t N, size_t* workspace_bytes) {
  if (!workspace_bytes) return HINM_ERR_NULL;
  const hinm_status st = check_norm(K, N, HINM_F16);
  if (st != HINM_OK) return st;
  *workspace_bytes = layer_norm_grad_workspace_bytes(K, N);
  return HINM_OK;
}

hinm_status hinm_layer_norm_grad(int32_t K, int32_t N, int32_t dtype, const void* x, int64_t ldx, const float* w, const float* mean,
                                 const float* rstd, const void* du, int64_t ldu, const void* dh, void* dx, float* dw, float* db,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  const hinm_status st = check_norm(K, N, dtype);
  if (st != HINM_OK) return st;
  if (!x || !mean || !rstd || !du || (!dx && !dw && !db)) return HINM_ERR_NULL;
  if (ldx < N || ldu < N) return HINM_ERR_SHAPE;
  for (const void* p : {x, du, dh, const_cast<const void*>(dx)})
    if (!aligned(p, 2)) return HINM_ERR_SHAPE;
  for (const float* p : {w, mean, rstd, const_cast<const float*>(dw), const_cast<const float*>(db)})
    if (!aligned(p, 4)) return HINM_ERR_SHAPE;
  if (too_many_to_add(K, N) && (dw || db)) return HINM_ERR_UNSUPPORTED;
  const size_t need = layer_norm_grad_workspace_bytes(K, N);
  if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 256))) return HINM_ERR_WORKSPACE;
  return launched(launch_layer_norm_grad({K, N, dtype, x, ldx, w, mean, rstd, du, ldu, dh, dx, dw, db, static_cast<float*>(workspace)},
                                         static_cast<hipStream_t>(stream)));
}

const char* hinm_status_str(hinm_status s) {
  switch (s) {
    case HINM_OK: return "ok";
    case HINM_ERR_NULL: return "null pointer argument";
    case HINM_ERR_SHAPE: return "invalid shape, leading dimension or alignment";
    case HINM_ERR_DTYPE: return "unsupported dtype";
    case HINM_ERR_WORKSPACE: return "workspace missing, misaligned or too small";
    case HINM_ERR_UNSUPPORTED: return "request not supported by this build";
    case HINM_ERR_DEVICE: return "HIP launch failed";
  }
  return "unknown status";
}

int32_t hinm_version(void) { return 1000 * 0 + 1; }

}  // extern "C"
