// The C ABI of libqlin (declared in include/qlin.h): argument validation on
// the host, then launches on the caller's stream.  No call allocates memory.
#include <atomic>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <mutex>
#include <utility>

#include "qlin_attention.h"
#include "qlin_internal.h"
#include "qlin_tiles.h"

namespace qlin {
namespace {

// Device status word: kernels record device-side failures here.
__device__ unsigned g_status_word;

std::mutex g_dev_mutex;
unsigned* g_status_ptr[kMaxDevices] = {};
int g_num_sms[kMaxDevices] = {};
std::atomic<uint64_t> g_timeout_ns{2000000000ull};
thread_local char g_last_error[256] = "";

qlin_status cuda_fail(cudaError_t e) {
  std::snprintf(g_last_error, sizeof g_last_error, "%s: %s", cudaGetErrorName(e),
                cudaGetErrorString(e));
  return QLIN_ERR_CUDA;
}

// Per-device state, set up on the first call made on that device: the
// address of the status word and the SM count.
qlin_status device_state(unsigned** status, Device* out) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_fail(e);
  if (dev < 0 || dev >= kMaxDevices) return QLIN_ERR_UNSUPPORTED;
  std::lock_guard<std::mutex> lock(g_dev_mutex);
  if (g_status_ptr[dev] == nullptr) {
    int major = 0, minor = 0, sms = 0;
    if ((e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev)) != cudaSuccess ||
        (e = cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev)) != cudaSuccess ||
        (e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess)
      return cuda_fail(e);
    if (major != 10 || minor != 3) {
      std::snprintf(g_last_error, sizeof g_last_error,
                    "libqlin is built for sm_103a; device %d is sm_%d%d", dev, major, minor);
      return QLIN_ERR_UNSUPPORTED;
    }
    void* p = nullptr;
    if ((e = cudaGetSymbolAddress(&p, g_status_word)) != cudaSuccess) return cuda_fail(e);
    g_status_ptr[dev] = static_cast<unsigned*>(p);
    g_num_sms[dev] = sms;
  }
  *status = g_status_ptr[dev];
  *out = {dev, g_num_sms[dev]};
  return QLIN_OK;
}

// Scratch of qlin_quantize_act_nvfp4_noalloc: a static device array, so the
// entry point needs no allocation.  Host code may only use its device address
// (looked up once per device), never the symbol itself.
static __device__ __align__(256) unsigned char g_noalloc_scratch[QLIN_NOALLOC_SCRATCH_BYTES];
unsigned char* g_noalloc_ptr[kMaxDevices] = {};

qlin_status noalloc_scratch(unsigned char** out) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_fail(e);
  if (dev < 0 || dev >= kMaxDevices) return QLIN_ERR_UNSUPPORTED;
  std::lock_guard<std::mutex> lock(g_dev_mutex);
  if (g_noalloc_ptr[dev] == nullptr) {
    void* p = nullptr;
    if ((e = cudaGetSymbolAddress(&p, g_noalloc_scratch)) != cudaSuccess) return cuda_fail(e);
    g_noalloc_ptr[dev] = static_cast<unsigned char*>(p);
  }
  *out = g_noalloc_ptr[dev];
  return QLIN_OK;
}

uint64_t timeout() { return g_timeout_ns.load(std::memory_order_relaxed); }

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

bool shape_ok(int64_t rows, int64_t K) { return rows >= 1 && K >= 64 && K % 64 == 0; }

qlin_status check_nvfp4(const qlin_nvfp4_t* t, int64_t rows, int64_t K) {
  if (t == nullptr || t->codes == nullptr || t->scales == nullptr || t->tensor_scale == nullptr)
    return QLIN_ERR_INVALID_ARG;
  if (t->rows != rows || t->K != K || !shape_ok(rows, K)) return QLIN_ERR_INVALID_ARG;
  if (!aligned(t->codes, 16) || !aligned(t->scales, 16) || !aligned(t->tensor_scale, 4))
    return QLIN_ERR_MISALIGNED;
  return QLIN_OK;
}

qlin_status check_fp8(const qlin_fp8_t* t, int64_t rows, int64_t K) {
  if (t == nullptr || t->codes == nullptr || t->scale == nullptr) return QLIN_ERR_INVALID_ARG;
  if (t->rows != rows || t->K != K || !shape_ok(rows, K)) return QLIN_ERR_INVALID_ARG;
  if (!aligned(t->codes, 16) || !aligned(t->scale, 4)) return QLIN_ERR_MISALIGNED;
  return QLIN_OK;
}

qlin_status check_workspace(void* ws, size_t ws_bytes) {
  if (ws == nullptr || ws_bytes < qlin_workspace_size(0, 0)) return QLIN_ERR_WORKSPACE;
  // 8-byte aligned: the one-read quantizer reads its amax and arrival words
  // as one 64-bit load
  if (!aligned(ws, 8)) return QLIN_ERR_MISALIGNED;
  return QLIN_OK;
}

#define QLIN_TRY(expr)                 \
  do {                                 \
    qlin_status st__ = (expr);         \
    if (st__ != QLIN_OK) return st__;  \
  } while (0)

#define QLIN_CUDA(expr)                          \
  do {                                           \
    cudaError_t e__ = (expr);                    \
    if (e__ != cudaSuccess) return cuda_fail(e__); \
  } while (0)

}  // namespace
// Workspace words: the dynamic quantizers' amax and counts (kGridSyncWords from
// word 0; zero between calls), and qlin_linear_dynamic's max |y| from the GEMM
// epilogue and the epilogue's departure count (words 5 and 6; zero between
// calls).
constexpr int kWsQuant = 0;
constexpr int kWsChainAmax = 5;
static_assert(kWsQuant + kGridSyncWords <= kWsChainAmax, "separate words");

}  // namespace qlin

using namespace qlin;

extern "C" {

size_t qlin_nvfp4_scale_bytes(int64_t rows, int64_t K) {
  if (!shape_ok(rows, K)) return 0;
  return (size_t)(((rows + 127) / 128) * (K / 64) * 512);
}

size_t qlin_workspace_size(int64_t M, int64_t K) {
  (void)M;
  (void)K;
  return 256;
}

qlin_status qlin_quantize_act_nvfp4(const void* x_bf16, int64_t M, int64_t K,
                                    const float* static_scale, qlin_nvfp4_t* out,
                                    void* workspace, size_t ws_bytes, void* stream) {
  if (x_bf16 == nullptr || !shape_ok(M, K)) return QLIN_ERR_INVALID_ARG;
  QLIN_TRY(check_nvfp4(out, M, K));
  if (!aligned(x_bf16, 16)) return QLIN_ERR_MISALIGNED;
  if (static_scale != nullptr && !aligned(static_scale, 4)) return QLIN_ERR_MISALIGNED;
  if (static_scale == nullptr) QLIN_TRY(check_workspace(workspace, ws_bytes));
  unsigned* status;
  Device dev;
  QLIN_TRY(device_state(&status, &dev));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (static_scale == nullptr) {
    QLIN_CUDA(launch_quant_nvfp4_dynamic(x_bf16, M, K, *out,
                                         static_cast<unsigned*>(workspace) + kWsQuant, false, s,
                                         dev, grid_wait(timeout())));
  } else {
    QLIN_CUDA(launch_quant_nvfp4(x_bf16, M, K, static_scale, *out, s, dev));
  }
  return QLIN_OK;
}

qlin_status qlin_quantize_act_nvfp4_noalloc(const void* x_bf16, int64_t M, int64_t K,
                                            qlin_nvfp4_t* out, void* stream) {
  if (x_bf16 == nullptr || !shape_ok(M, K)) return QLIN_ERR_INVALID_ARG;
  QLIN_TRY(check_nvfp4(out, M, K));
  if (!aligned(x_bf16, 16)) return QLIN_ERR_MISALIGNED;
  if (qlin_workspace_size(M, K) > QLIN_NOALLOC_SCRATCH_BYTES) {
    std::snprintf(g_last_error, sizeof g_last_error,
                  "shape [%lld, %lld] needs more than %d bytes of static scratch",
                  (long long)M, (long long)K, QLIN_NOALLOC_SCRATCH_BYTES);
    return QLIN_ERR_WORKSPACE;
  }
  unsigned* status;
  Device dev;
  QLIN_TRY(device_state(&status, &dev));
  unsigned char* scratch = nullptr;
  QLIN_TRY(noalloc_scratch(&scratch));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  // the scratch words are cleared by the launch that uses them
  QLIN_CUDA(launch_quant_nvfp4_dynamic(x_bf16, M, K, *out,
                                       reinterpret_cast<unsigned*>(scratch) + kWsQuant, true, s,
                                       dev, grid_wait(timeout())));
  return QLIN_OK;
}

qlin_status qlin_quantize_act_fp8(const void* x_bf16, int64_t M, int64_t K,
                                  const float* static_scale, qlin_fp8_t* out, void* workspace,
                                  size_t ws_bytes, void* stream) {
  if (x_bf16 == nullptr || !shape_ok(M, K)) return QLIN_ERR_INVALID_ARG;
  QLIN_TRY(check_fp8(out, M, K));
  if (out->per_channel) return QLIN_ERR_INVALID_ARG;
  if (!aligned(x_bf16, 16)) return QLIN_ERR_MISALIGNED;
  if (static_scale != nullptr && !aligned(static_scale, 4)) return QLIN_ERR_MISALIGNED;
  if (static_scale == nullptr) QLIN_TRY(check_workspace(workspace, ws_bytes));
  unsigned* status;
  Device dev;
  QLIN_TRY(device_state(&status, &dev));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (static_scale == nullptr) {
    QLIN_CUDA(launch_quant_fp8_dynamic(x_bf16, M, K, *out,
                                       static_cast<unsigned*>(workspace) + kWsQuant, false, s, dev,
                                       grid_wait(timeout())));
  } else {
    QLIN_CUDA(launch_quant_fp8(x_bf16, M, K, static_scale, *out, s, dev, status, timeout()));
  }
  return QLIN_OK;
}

qlin_status qlin_quantize_weight(const void* w_bf16, int64_t N, int64_t K, qlin_format fmt,
                                 void* out_desc, void* workspace, size_t ws_bytes, void* stream) {
  if (w_bf16 == nullptr || out_desc == nullptr || !shape_ok(N, K)) return QLIN_ERR_INVALID_ARG;
  if (!aligned(w_bf16, 16)) return QLIN_ERR_MISALIGNED;
  if (fmt == QLIN_FMT_NVFP4) {
    return qlin_quantize_act_nvfp4(w_bf16, N, K, nullptr, static_cast<qlin_nvfp4_t*>(out_desc),
                                   workspace, ws_bytes, stream);
  }
  if (fmt != QLIN_FMT_FP8) return QLIN_ERR_UNSUPPORTED;
  qlin_fp8_t* out = static_cast<qlin_fp8_t*>(out_desc);
  QLIN_TRY(check_fp8(out, N, K));
  if (!out->per_channel) return QLIN_ERR_INVALID_ARG;
  unsigned* status;
  Device dev;
  QLIN_TRY(device_state(&status, &dev));
  QLIN_CUDA(launch_quant_fp8_rows(w_bf16, N, K, *out, static_cast<cudaStream_t>(stream), dev));
  return QLIN_OK;
}

static qlin_status check_fp8_block(const qlin_fp8_block_t* t, int32_t block_rows) {
  if (t == nullptr || t->codes == nullptr || t->scales == nullptr || !shape_ok(t->rows, t->K) ||
      t->block_rows != block_rows)
    return QLIN_ERR_INVALID_ARG;
  if (!aligned(t->codes, 16) || !aligned(t->scales, 4)) return QLIN_ERR_MISALIGNED;
  return QLIN_OK;
}

// Bias, activation and residual of a linear into its GEMM's arguments (M, N set).
static qlin_status set_epilogue(GemmArgs& a, const qlin_epilogue_t* ep) {
  if (ep == nullptr) return QLIN_OK;
  if (ep->act < QLIN_ACT_NONE || ep->act > QLIN_ACT_GELU) return QLIN_ERR_INVALID_ARG;
  if (ep->residual != nullptr && ep->residual_stride < a.N) return QLIN_ERR_INVALID_ARG;
  if (!aligned(ep->bias, 16) || !aligned(ep->residual, 16) ||
      (ep->residual != nullptr && ep->residual_stride % 8 != 0))
    return QLIN_ERR_MISALIGNED;
  // (in place: a thread reads what it writes, at the same address)
  if (ep->residual != nullptr && ep->residual == a.y && ep->residual_stride != a.N && a.M > 1)
    return QLIN_ERR_INVALID_ARG;
  a.bias = ep->bias;
  a.residual = ep->residual;
  a.residual_stride = ep->residual_stride;
  a.act = ep->act;
  a.epilogue = a.epilogue || a.bias != nullptr || a.residual != nullptr || a.act != QLIN_ACT_NONE;
  return QLIN_OK;
}

// The plain GEMMs always take whole tensor-core tiles, so that their sums keep their
// order; the linears take the few-token kernel or tiles with a split K where those apply.
static cudaError_t launch_linear(GemmArgs& a, cudaStream_t s, Device dev, unsigned* status) {
  const GemmKind kind = a.fp4 ? GemmKind::kNvfp4 : a.bf16 ? GemmKind::k16 : GemmKind::kFp8;
  // (the few-token kernel counts a row's bytes in 32 bits)
  if (a.few_ok && a.K <= (int64_t)1 << 28 &&
      few_tokens(a.bf16, a.M, a.N, k_row_bytes(kind, a.K), dev.num_sms) &&
      !split_over_few(kind, a.M, a.N, a.K, dev.num_sms))
    return launch_few(a, s, dev);
  a.split = a.few_ok ? choose_split_k(kind, a.M, a.N, a.K, dev.num_sms) : 1;
  return launch_gemm(a, s, dev, status, timeout());
}

static qlin_status gemm_common(bool fp4, const void* Aany, const void* Wany, void* y,
                               const float* next_scale, qlin_nvfp4_t* y_q, int64_t rq_col0,
                               void* stream, unsigned* y_amax = nullptr,
                               qlin_fp8_t* y_q8 = nullptr, float* y_sdec = nullptr,
                               const qlin_epilogue_t* ep = nullptr, bool linear = false) {
  GemmArgs a{};
  a.y_amax = y_amax;
  a.y_departures = y_amax != nullptr ? y_amax + 1 : nullptr;
  a.y_sdec = y_sdec;
  a.fp4 = fp4;
  if (fp4) {
    const qlin_nvfp4_t* A = static_cast<const qlin_nvfp4_t*>(Aany);
    const qlin_nvfp4_t* W = static_cast<const qlin_nvfp4_t*>(Wany);
    if (A == nullptr || W == nullptr) return QLIN_ERR_INVALID_ARG;
    QLIN_TRY(check_nvfp4(A, A->rows, A->K));
    QLIN_TRY(check_nvfp4(W, W->rows, A->K));
    a.a_codes = A->codes;
    a.w_codes = W->codes;
    a.sfa = A->scales;
    a.sfb = W->scales;
    a.sdec_a = A->tensor_scale;
    a.sdec_w = W->tensor_scale;
    a.M = A->rows;
    a.N = W->rows;
    a.K = A->K;
  } else {
    const qlin_fp8_t* A = static_cast<const qlin_fp8_t*>(Aany);
    const qlin_fp8_t* W = static_cast<const qlin_fp8_t*>(Wany);
    if (A == nullptr || W == nullptr) return QLIN_ERR_INVALID_ARG;
    QLIN_TRY(check_fp8(A, A->rows, A->K));
    QLIN_TRY(check_fp8(W, W->rows, A->K));
    if (A->per_channel && !linear) return QLIN_ERR_INVALID_ARG;
    a.a_per_row = A->per_channel != 0;
    // (the plain epilogue reads W's row scales 16 bytes at a time)
    a.epilogue = a.a_per_row || (W->per_channel && !aligned(W->scale, 16));
    a.a_codes = A->codes;
    a.w_codes = W->codes;
    a.sdec_a = A->scale;
    a.sdec_w = W->scale;
    a.w_per_channel = W->per_channel ? 1 : 0;
    a.M = A->rows;
    a.N = W->rows;
    a.K = A->K;
  }
  if (a.N % 64 != 0) return QLIN_ERR_INVALID_ARG;
  if (a.M > (int64_t)1 << 31 || a.N > (int64_t)1 << 31) return QLIN_ERR_UNSUPPORTED;
  if (y != nullptr && !aligned(y, 16)) return QLIN_ERR_MISALIGNED;
  a.y = y;
  QLIN_TRY(set_epilogue(a, ep));
  a.few_ok = linear;
  if (next_scale != nullptr) {
    // the re-quantized operand: NVFP4 after an NVFP4 GEMM, FP8 after an FP8 one
    const int64_t rq_cols = fp4 ? (y_q ? y_q->K : 0) : (y_q8 ? y_q8->K : 0);
    if ((fp4 ? y_q == nullptr : y_q8 == nullptr) || !aligned(next_scale, 4))
      return QLIN_ERR_INVALID_ARG;
    if (rq_cols < 64 || rq_cols % 64 != 0 || rq_col0 < 0 || rq_col0 % 64 != 0 ||
        rq_col0 + rq_cols > a.N)
      return QLIN_ERR_INVALID_ARG;
    if (fp4) {
      QLIN_TRY(check_nvfp4(y_q, a.M, y_q->K));
      a.rq_codes = y_q->codes;
      a.rq_scales = y_q->scales;
      a.rq_tensor_scale = y_q->tensor_scale;
    } else {
      QLIN_TRY(check_fp8(y_q8, a.M, y_q8->K));
      if (y_q8->per_channel) return QLIN_ERR_INVALID_ARG;
      a.rq_codes = y_q8->codes;
      a.rq_tensor_scale = y_q8->scale;
    }
    a.next_scale = next_scale;
    a.rq_col0 = rq_col0;
    a.rq_cols = rq_cols;
  } else if (y == nullptr) {
    return QLIN_ERR_INVALID_ARG;  // nothing to write
  }
  unsigned* status;
  Device dev;
  QLIN_TRY(device_state(&status, &dev));
  cudaError_t e = launch_linear(a, static_cast<cudaStream_t>(stream), dev, status);
  if (e != cudaSuccess) return cuda_fail(e);
  return QLIN_OK;
}

qlin_status qlin_gemm_nvfp4(const qlin_nvfp4_t* A, const qlin_nvfp4_t* W, void* y_bf16,
                            void* stream) {
  if (y_bf16 == nullptr) return QLIN_ERR_INVALID_ARG;
  return gemm_common(true, A, W, y_bf16, nullptr, nullptr, 0, stream);
}

qlin_status qlin_gemm_fp8(const qlin_fp8_t* A, const qlin_fp8_t* W, void* y_bf16, void* stream) {
  if (y_bf16 == nullptr) return QLIN_ERR_INVALID_ARG;
  return gemm_common(false, A, W, y_bf16, nullptr, nullptr, 0, stream);
}

qlin_status qlin_linear_fused(const qlin_nvfp4_t* A, const qlin_nvfp4_t* W, void* y_bf16,
                              const float* next_scale, qlin_nvfp4_t* y_q, int64_t rq_col0,
                              void* stream) {
  return gemm_common(true, A, W, y_bf16, next_scale, y_q, rq_col0, stream);
}

// The unquantized 16-bit linear (bf16 or fp16 operands and output).
static qlin_status gemm16(const void* a16, int64_t lda, const void* w16, int64_t M, int64_t N,
                          int64_t K, void* y16, void* stream, bool fp16,
                          const qlin_epilogue_t* ep = nullptr, bool linear = false) {
  if (a16 == nullptr || w16 == nullptr || y16 == nullptr) return QLIN_ERR_INVALID_ARG;
  if (M < 1 || K < 64 || K % 64 != 0 || N < 64 || N % 64 != 0 || lda < K)
    return QLIN_ERR_INVALID_ARG;
  if (M > (int64_t)1 << 31 || N > (int64_t)1 << 31) return QLIN_ERR_UNSUPPORTED;
  if (!aligned(a16, 16) || !aligned(w16, 16) || !aligned(y16, 16) || (lda * 2) % 16 != 0)
    return QLIN_ERR_MISALIGNED;
  GemmArgs a{};
  a.bf16 = true;
  a.fp16 = fp16;
  a.a_codes = a16;
  a.a_row_bytes = lda * 2;
  a.w_codes = w16;
  a.y = y16;
  a.M = M;
  a.N = N;
  a.K = K;
  QLIN_TRY(set_epilogue(a, ep));
  a.few_ok = linear;
  unsigned* status;
  Device dev;
  QLIN_TRY(device_state(&status, &dev));
  cudaError_t e = launch_linear(a, static_cast<cudaStream_t>(stream), dev, status);
  if (e != cudaSuccess) return cuda_fail(e);
  return QLIN_OK;
}

qlin_status qlin_gemm_bf16(const void* a_bf16, int64_t lda, const void* w_bf16, int64_t M,
                           int64_t N, int64_t K, void* y_bf16, void* stream) {
  return gemm16(a_bf16, lda, w_bf16, M, N, K, y_bf16, stream, false);
}

qlin_status qlin_gemm_fp16(const void* a_fp16, int64_t lda, const void* w_fp16, int64_t M,
                           int64_t N, int64_t K, void* y_fp16, void* stream) {
  return gemm16(a_fp16, lda, w_fp16, M, N, K, y_fp16, stream, true);
}

qlin_status qlin_linear_dynamic(const qlin_nvfp4_t* A, const qlin_nvfp4_t* W, void* y_bf16,
                                qlin_nvfp4_t* y_q, void* workspace, size_t ws_bytes,
                                void* stream) {
  if (A == nullptr || W == nullptr || y_bf16 == nullptr || y_q == nullptr)
    return QLIN_ERR_INVALID_ARG;
  QLIN_TRY(check_nvfp4(y_q, A->rows, W->rows));
  QLIN_TRY(check_workspace(workspace, ws_bytes));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  unsigned* amax = static_cast<unsigned*>(workspace) + kWsChainAmax;
  // y and its tensor scale in one GEMM (its last CTA writes S_dec into y_q's
  // tensor scale and resets the scratch words), then the quantizer of y with
  // that scale
  QLIN_TRY(gemm_common(true, A, W, y_bf16, nullptr, nullptr, 0, stream, amax, nullptr,
                       y_q->tensor_scale));
  unsigned* status;
  Device dev;
  QLIN_TRY(device_state(&status, &dev));
  QLIN_CUDA(launch_quant_nvfp4_after(y_bf16, A->rows, W->rows, y_q->tensor_scale, *y_q, s, dev,
                                     status, timeout()));
  return QLIN_OK;
}

qlin_status qlin_linear_fused_fp8(const qlin_fp8_t* A, const qlin_fp8_t* W, void* y_bf16,
                                  const float* next_scale, qlin_fp8_t* y_q, int64_t rq_col0,
                                  void* stream) {
  if (next_scale == nullptr) return QLIN_ERR_INVALID_ARG;
  return gemm_common(false, A, W, y_bf16, next_scale, nullptr, rq_col0, stream, nullptr, y_q);
}

qlin_status qlin_linear_nvfp4(const qlin_nvfp4_t* A, const qlin_nvfp4_t* W,
                              const qlin_epilogue_t* epilogue, void* y_bf16,
                              const float* next_scale, qlin_nvfp4_t* y_q, int64_t rq_col0,
                              void* stream) {
  return gemm_common(true, A, W, y_bf16, next_scale, y_q, rq_col0, stream, nullptr, nullptr,
                     nullptr, epilogue, true);
}

qlin_status qlin_linear_fp8(const qlin_fp8_t* A, const qlin_fp8_t* W,
                            const qlin_epilogue_t* epilogue, void* y_bf16,
                            const float* next_scale, qlin_fp8_t* y_q, int64_t rq_col0,
                            void* stream) {
  return gemm_common(false, A, W, y_bf16, next_scale, nullptr, rq_col0, stream, nullptr, y_q,
                     nullptr, epilogue, true);
}

qlin_status qlin_linear_fp8_block(const qlin_fp8_block_t* A, const qlin_fp8_block_t* W,
                                  const qlin_epilogue_t* epilogue, void* y_bf16, void* stream) {
  QLIN_TRY(check_fp8_block(A, 1));
  QLIN_TRY(check_fp8_block(W, 128));
  if (y_bf16 == nullptr || A->K != W->K || W->rows % 64 != 0) return QLIN_ERR_INVALID_ARG;
  if (A->rows > (int64_t)1 << 31 || W->rows > (int64_t)1 << 31 || A->K > INT32_MAX) return QLIN_ERR_UNSUPPORTED;
  if (!aligned(y_bf16, 16)) return QLIN_ERR_MISALIGNED;
  GemmArgs a{};
  a.blocks = true;
  a.a_codes = A->codes;
  a.w_codes = W->codes;
  a.sdec_a = A->scales;
  a.sdec_w = W->scales;
  a.M = A->rows;
  a.N = W->rows;
  a.K = A->K;
  a.y = y_bf16;
  QLIN_TRY(set_epilogue(a, epilogue));
  unsigned* status;
  Device dev;
  QLIN_TRY(device_state(&status, &dev));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (a.K <= (int64_t)1 << 28 && few_block_tokens(a.M, a.N, a.K, dev.num_sms))
    QLIN_CUDA(launch_few(a, s, dev));
  else
    QLIN_CUDA(launch_gemm_block(a, s, dev, status, timeout()));
  return QLIN_OK;
}

qlin_status qlin_linear_bf16(const void* a_bf16, int64_t lda, const void* w_bf16, int64_t M,
                             int64_t N, int64_t K, const qlin_epilogue_t* epilogue,
                             void* y_bf16, void* stream) {
  return gemm16(a_bf16, lda, w_bf16, M, N, K, y_bf16, stream, false, epilogue, true);
}

qlin_status qlin_linear_fp16(const void* a_fp16, int64_t lda, const void* w_fp16, int64_t M,
                             int64_t N, int64_t K, const qlin_epilogue_t* epilogue,
                             void* y_fp16, void* stream) {
  return gemm16(a_fp16, lda, w_fp16, M, N, K, y_fp16, stream, true, epilogue, true);
}

static qlin_status check_rmsnorm(const qlin_rmsnorm_t* a) {
  if (a == nullptr || a->x == nullptr || !shape_ok(a->M, a->K)) return QLIN_ERR_INVALID_ARG;
  if (a->dtype != QLIN_BF16 && a->dtype != QLIN_FP16) return QLIN_ERR_INVALID_ARG;
  if (!(a->eps > 0.0f) || !std::isfinite(a->eps)) return QLIN_ERR_INVALID_ARG;
  if (a->sum != nullptr && a->residual == nullptr) return QLIN_ERR_INVALID_ARG;
  if (a->x_stride < a->K || (a->residual != nullptr && a->residual_stride < a->K) ||
      (a->sum != nullptr && a->sum_stride < a->K))
    return QLIN_ERR_INVALID_ARG;
  if (a->M > INT32_MAX || a->K > INT32_MAX) return QLIN_ERR_UNSUPPORTED;
  if (!aligned(a->x, 16) || !aligned(a->residual, 16) || !aligned(a->sum, 16) ||
      !aligned(a->weight, 16) || a->x_stride % 8 != 0 ||
      (a->residual != nullptr && a->residual_stride % 8 != 0) ||
      (a->sum != nullptr && a->sum_stride % 8 != 0))
    return QLIN_ERR_MISALIGNED;
  // in place only with equal strides
  if (a->sum != nullptr && a->M > 1 &&
      ((a->sum == a->x && a->sum_stride != a->x_stride) ||
       (a->sum == a->residual && a->sum_stride != a->residual_stride)))
    return QLIN_ERR_INVALID_ARG;
  return QLIN_OK;
}

static qlin_status rmsnorm(const qlin_rmsnorm_t* args, void* y16, const float* static_scale,
                           const qlin_fp8_t* fp8, const qlin_nvfp4_t* nvfp4, void* stream) {
  unsigned* status;
  Device dev;
  QLIN_TRY(device_state(&status, &dev));
  QLIN_CUDA(launch_rmsnorm(*args, y16, static_scale, fp8, nvfp4, static_cast<cudaStream_t>(stream), dev));
  return QLIN_OK;
}

qlin_status qlin_rmsnorm(const qlin_rmsnorm_t* args, void* y, void* stream) {
  QLIN_TRY(check_rmsnorm(args));
  if (y == nullptr) return QLIN_ERR_INVALID_ARG;
  if (!aligned(y, 16)) return QLIN_ERR_MISALIGNED;
  if (y == args->sum || (args->M > 1 && ((y == args->x && args->x_stride != args->K) ||
                                         (y == args->residual && args->residual_stride != args->K))))
    return QLIN_ERR_INVALID_ARG;
  return rmsnorm(args, y, nullptr, nullptr, nullptr, stream);
}

qlin_status qlin_rmsnorm_fp8(const qlin_rmsnorm_t* args, const float* static_scale,
                             qlin_fp8_t* out, void* stream) {
  QLIN_TRY(check_rmsnorm(args));
  QLIN_TRY(check_fp8(out, args->M, args->K));
  if ((static_scale == nullptr) != (out->per_channel != 0)) return QLIN_ERR_INVALID_ARG;
  if (!aligned(static_scale, 4)) return QLIN_ERR_MISALIGNED;
  return rmsnorm(args, nullptr, static_scale, out, nullptr, stream);
}

qlin_status qlin_rmsnorm_nvfp4(const qlin_rmsnorm_t* args, const float* static_scale,
                               qlin_nvfp4_t* out, void* stream) {
  QLIN_TRY(check_rmsnorm(args));
  QLIN_TRY(check_nvfp4(out, args->M, args->K));
  if (static_scale == nullptr) return QLIN_ERR_INVALID_ARG;
  if (!aligned(static_scale, 4)) return QLIN_ERR_MISALIGNED;
  return rmsnorm(args, nullptr, static_scale, nullptr, out, stream);
}

qlin_status qlin_rope(const qlin_rope_t* a, void* stream) {
  if (a == nullptr || a->x == nullptr || a->y == nullptr || a->positions == nullptr ||
      a->turns == nullptr)
    return QLIN_ERR_INVALID_ARG;
  if (a->tokens < 1 || a->heads < 1 || a->rot_dim < 2 || a->rot_dim % 2 != 0 ||
      a->rot_dim > a->head_dim || a->axes < 1 || a->axes > 4)
    return QLIN_ERR_INVALID_ARG;
  if ((a->position_bits != 32 && a->position_bits != 64) ||
      (a->layout != QLIN_ROPE_INTERLEAVED && a->layout != QLIN_ROPE_HALF) ||
      (a->dtype != QLIN_BF16 && a->dtype != QLIN_FP16))
    return QLIN_ERR_INVALID_ARG;
  int64_t pairs = 0;
  for (int i = 0; i < a->axes; ++i) {
    if (a->axis_pairs[i] < 0) return QLIN_ERR_INVALID_ARG;
    pairs += a->axis_pairs[i];
  }
  if (pairs != a->rot_dim / 2) return QLIN_ERR_INVALID_ARG;
  if (a->x == a->y &&
      (a->x_token_stride != a->y_token_stride || a->x_head_stride != a->y_head_stride))
    return QLIN_ERR_INVALID_ARG;
  // heads * head_dim is indexed in 32 bits
  if (a->head_dim > 1024 || a->tokens > INT32_MAX || a->heads > INT32_MAX / 1024)
    return QLIN_ERR_UNSUPPORTED;
  if (!aligned(a->x, 2) || !aligned(a->y, 2) || !aligned(a->turns, 8) ||
      !aligned(a->positions, a->position_bits / 8))
    return QLIN_ERR_MISALIGNED;
  // heads of y that lie over one another (an expanded tensor, say)
  auto apart = [&](int64_t n, int64_t stride) {
    return n == 1 || stride >= a->head_dim || stride <= -(int64_t)a->head_dim;
  };
  if (!apart(a->tokens, a->y_token_stride) || !apart(a->heads, a->y_head_stride)) return QLIN_ERR_INVALID_ARG;
  unsigned* status;
  Device dev;
  QLIN_TRY(device_state(&status, &dev));
  QLIN_CUDA(launch_rope(*a, dev.num_sms, static_cast<cudaStream_t>(stream)));
  return QLIN_OK;
}

size_t qlin_fp8_block_scales(int64_t rows, int64_t K, int32_t block_rows) {
  if (!shape_ok(rows, K) || (block_rows != 1 && block_rows != 128)) return 0;
  return (size_t)((K + 127) / 128) * (size_t)((rows + block_rows - 1) / block_rows);
}

qlin_status qlin_quantize_fp8_block(const void* x, int32_t dtype, int64_t x_stride,
                                    const qlin_fp8_block_t* out, void* stream) {
  if (x == nullptr || out == nullptr || (dtype != QLIN_BF16 && dtype != QLIN_FP16)) return QLIN_ERR_INVALID_ARG;
  if (out->block_rows != 1 && out->block_rows != 128) return QLIN_ERR_INVALID_ARG;
  QLIN_TRY(check_fp8_block(out, out->block_rows));
  if (x_stride < out->K) return QLIN_ERR_INVALID_ARG;
  if (!aligned(x, 16) || x_stride % 8 != 0) return QLIN_ERR_MISALIGNED;
  // (CTAs are counted in 31 bits: at least 2^36 elements)
  if (out->rows > INT32_MAX || out->K > INT32_MAX || qlin_fp8_block_scales(out->rows, out->K, out->block_rows) > INT32_MAX)
    return QLIN_ERR_UNSUPPORTED;
  unsigned* status;
  Device dev;
  QLIN_TRY(device_state(&status, &dev));
  QLIN_CUDA(launch_quant_fp8_block(x, x_stride, dtype == QLIN_FP16, *out, static_cast<cudaStream_t>(stream)));
  return QLIN_OK;
}

// Whether n0 x n1 rows of `width` elements, s0 and s1 elements apart, lie beside one another.
static bool rows_beside(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t width) {
  using Wide = __int128;   // (strides are any 64-bit numbers)
  Wide outer = s0 < 0 ? -(Wide)s0 : s0, inner = s1 < 0 ? -(Wide)s1 : s1;
  if (n0 == 1) outer = (Wide)1 << 100;
  if (n1 == 1) inner = (Wide)1 << 100;
  if (outer < inner) {
    std::swap(outer, inner);
    std::swap(n0, n1);
  }
  if (inner < width) return false;
  if (n0 == 1 || outer >= (n1 - 1) * inner + width) return true;
  // rows that interleave: the inner one nearest to each outer step (steps past the inner rows' extent meet none)
  for (Wide i = 1; i < n0 && i * outer < (n1 - 1) * inner + width; ++i) {
    const Wide j = i * outer / inner;
    for (Wide k = j; k <= j + 1 && k < n1; ++k) {
      const Wide d = i * outer - k * inner;
      if (d < width && d > -(Wide)width) return false;
    }
  }
  return true;
}

static qlin_status check_cache(const qlin_cache_t* c) {
  if (c == nullptr || c->k == nullptr || c->v == nullptr || c->page_table == nullptr || c->cached == nullptr ||
      c->q_start == nullptr)
    return QLIN_ERR_INVALID_ARG;
  if (c->sequences < 1 || c->pages < 1 || c->page_size < 1 || c->table_width < 1 || c->heads < 1 ||
      c->head_dim < 1 || c->format < QLIN_CACHE_BF16 || c->format > QLIN_CACHE_E4M3)
    return QLIN_ERR_INVALID_ARG;
  if (c->format == QLIN_CACHE_E4M3 && (c->k_scale == nullptr || c->v_scale == nullptr)) return QLIN_ERR_INVALID_ARG;
  if (c->k_page_stride < 0 || c->k_slot_stride < 0 || c->k_head_stride < 0 || c->v_page_stride < 0 ||
      c->v_slot_stride < 0 || c->v_head_stride < 0 || (c->sequences > 1 && c->table_stride < c->table_width))
    return QLIN_ERR_INVALID_ARG;
  if (c->head_dim > 256 || c->heads > 65536 || c->sequences > 1 << 24) return QLIN_ERR_UNSUPPORTED;
  if (!aligned(c->page_table, 4) || !aligned(c->cached, 4) || !aligned(c->q_start, 4) || !aligned(c->k_scale, 4) ||
      !aligned(c->v_scale, 4))
    return QLIN_ERR_MISALIGNED;
  return QLIN_OK;
}

qlin_status qlin_cache_append(const qlin_cache_t* c, const qlin_cache_append_t* a, void* stream) {
  QLIN_TRY(check_cache(c));
  if (a == nullptr || a->k == nullptr || a->v == nullptr || a->tokens < 1 ||
      (a->dtype != QLIN_BF16 && a->dtype != QLIN_FP16))
    return QLIN_ERR_INVALID_ARG;
  if (a->q != nullptr && (a->q_out == nullptr || a->q_heads < 1)) return QLIN_ERR_INVALID_ARG;
  // cache rows of new tokens must not lie over one another
  auto rows_apart = [&](int64_t page, int64_t slot, int64_t head) {
    return (c->pages == 1 || page >= c->head_dim) && (c->page_size == 1 || slot >= c->head_dim) &&
           (c->heads == 1 || head >= c->head_dim);
  };
  if (!rows_apart(c->k_page_stride, c->k_slot_stride, c->k_head_stride) ||
      !rows_apart(c->v_page_stride, c->v_slot_stride, c->v_head_stride))
    return QLIN_ERR_INVALID_ARG;
  if (c->format != QLIN_CACHE_E4M3 && c->format != a->dtype) return QLIN_ERR_UNSUPPORTED;
  if (a->turns != nullptr) {
    if (a->rot_dim < 2 || a->rot_dim % 2 != 0 || a->rot_dim > c->head_dim || a->axes < 1 || a->axes > 4 ||
        (a->layout != QLIN_ROPE_INTERLEAVED && a->layout != QLIN_ROPE_HALF) ||
        (a->positions != nullptr && a->position_bits != 32 && a->position_bits != 64) ||
        (a->positions == nullptr && a->axes != 1))
      return QLIN_ERR_INVALID_ARG;
    int64_t pairs = 0;
    for (int i = 0; i < a->axes; ++i) {
      if (a->axis_pairs[i] < 0) return QLIN_ERR_INVALID_ARG;
      pairs += a->axis_pairs[i];
    }
    if (pairs != a->rot_dim / 2) return QLIN_ERR_INVALID_ARG;
    if (!aligned(a->turns, 8) || (a->positions != nullptr && !aligned(a->positions, a->position_bits / 8)))
      return QLIN_ERR_MISALIGNED;
  }
  if (a->q != nullptr) {
    if (a->q == a->q_out &&
        (a->q_token_stride != a->q_out_token_stride || a->q_head_stride != a->q_out_head_stride))
      return QLIN_ERR_INVALID_ARG;
    if (a->tokens > 1 << 28 || a->q_heads > 65536) return QLIN_ERR_UNSUPPORTED;
    if (!rows_beside(a->tokens, a->q_out_token_stride, a->q_heads, a->q_out_head_stride, c->head_dim))
      return QLIN_ERR_INVALID_ARG;
    if (!aligned(a->q, 2) || !aligned(a->q_out, 2)) return QLIN_ERR_MISALIGNED;
  }
  if (a->tokens > 1 << 28) return QLIN_ERR_UNSUPPORTED;
  if (!aligned(a->k, 2) || !aligned(a->v, 2) ||
      (c->format != QLIN_CACHE_E4M3 && (!aligned(c->k, 2) || !aligned(c->v, 2))))
    return QLIN_ERR_MISALIGNED;
  unsigned* status;
  Device dev;
  QLIN_TRY(device_state(&status, &dev));
  QLIN_CUDA(launch_cache_append(*c, *a, static_cast<cudaStream_t>(stream), dev, status));
  return QLIN_OK;
}

size_t qlin_cache_attention_workspace_size(void) { return (size_t)kWorkspaceBytes; }

qlin_status qlin_cache_attention(const qlin_cache_t* c, const qlin_cache_attention_t* a, void* workspace,
                                 size_t ws_bytes, void* stream) {
  QLIN_TRY(check_cache(c));
  if (a == nullptr || a->q == nullptr || a->out == nullptr || a->tokens < 1 || a->q_heads < 1 ||
      (a->dtype != QLIN_BF16 && a->dtype != QLIN_FP16) || a->q_heads % c->heads != 0)
    return QLIN_ERR_INVALID_ARG;
  // (below 2^127: times log2(e) it is finite)
  if (!std::isnormal(a->scale) || !(a->scale > 0.0f) || a->scale >= 0x1p127f) return QLIN_ERR_INVALID_ARG;
  if (a->mask != nullptr && (a->mask_words < 1 || (a->tokens > 1 && a->mask_stride < 0))) return QLIN_ERR_INVALID_ARG;
  if (a->q == a->out &&
      (a->q_token_stride != a->out_token_stride || a->q_head_stride != a->out_head_stride))
    return QLIN_ERR_INVALID_ARG;
  if (c->head_dim % 16 != 0 || (c->format != QLIN_CACHE_E4M3 && c->format != a->dtype)) return QLIN_ERR_UNSUPPORTED;
  // (rows, and the tiles of a call, are counted in 31 and 43 bits)
  if (a->tokens > 1 << 24 || a->q_heads > 65536 || a->tokens * (a->q_heads / c->heads) > (int64_t)1 << 30)
    return QLIN_ERR_UNSUPPORTED;
  const int64_t per16 = c->format == QLIN_CACHE_E4M3 ? 16 : 8;
  const int64_t strides = c->k_page_stride | c->k_slot_stride | c->k_head_stride | c->v_page_stride |
                          c->v_slot_stride | c->v_head_stride;
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || strides % per16 != 0 || !aligned(a->q, 16) ||
      !aligned(a->out, 16) ||
      ((a->q_token_stride | a->q_head_stride | a->out_token_stride | a->out_head_stride) & 7) != 0 ||
      !aligned(a->lse, 4) || !aligned(a->mask, 8))
    return QLIN_ERR_MISALIGNED;
  if (!rows_beside(a->tokens, a->out_token_stride, a->q_heads, a->out_head_stride, c->head_dim))
    return QLIN_ERR_INVALID_ARG;
  if (workspace == nullptr || ws_bytes < qlin_cache_attention_workspace_size()) return QLIN_ERR_WORKSPACE;
  if (!aligned(workspace, 16)) return QLIN_ERR_MISALIGNED;
  unsigned* status;
  Device dev;
  QLIN_TRY(device_state(&status, &dev));
  QLIN_CUDA(launch_cache_attention(*c, *a, workspace, static_cast<cudaStream_t>(stream), dev, status, timeout()));
  return QLIN_OK;
}

qlin_status qlin_rope_turns(int32_t rot_dim, double base, int32_t scaling, double factor,
                            double trained_length, double beta_fast, double beta_slow,
                            uint64_t* turns, float* magnitude) {
  if (turns == nullptr || magnitude == nullptr || rot_dim < 2 || rot_dim % 2 != 0)
    return QLIN_ERR_INVALID_ARG;
  if (!std::isfinite(base) || !(base > 1.0) || scaling < QLIN_ROPE_NONE || scaling > QLIN_ROPE_YARN)
    return QLIN_ERR_INVALID_ARG;
  if (scaling == QLIN_ROPE_NONE) factor = 1.0;
  if (!std::isfinite(factor) || !(factor >= 1.0)) return QLIN_ERR_INVALID_ARG;
  const double kTwoPi = 6.283185307179586476925;
  const double R = rot_dim;
  double low = 0.0, high = 0.0;   // YARN: the ramp's first and last pair
  if (scaling == QLIN_ROPE_YARN) {
    if (!std::isfinite(trained_length) || !(trained_length > 0.0) || !(beta_slow > 0.0) ||
        !std::isfinite(beta_fast) || !(beta_fast > beta_slow))
      return QLIN_ERR_INVALID_ARG;
    // the pair that turns `beta` times over the trained length
    auto pair_of = [&](double beta) {
      return R * std::log(trained_length / (beta * kTwoPi)) / (2.0 * std::log(base));
    };
    low = std::max(std::floor(pair_of(beta_fast)), 0.0);
    high = std::min(std::ceil(pair_of(beta_slow)), R - 1.0);
  }
  double b = base;
  if (scaling == QLIN_ROPE_NTK && rot_dim > 2) {
    b = base * std::pow(factor, R / (R - 2.0));
    if (!std::isfinite(b)) return QLIN_ERR_INVALID_ARG;
  }
  for (int i = 0; i < rot_dim / 2; ++i) {
    double f = std::pow(b, -2.0 * i / R);
    if (scaling == QLIN_ROPE_LINEAR || (scaling == QLIN_ROPE_NTK && rot_dim == 2)) f /= factor;
    if (scaling == QLIN_ROPE_YARN) {
      const double ramp = std::min(std::max((i - low) / std::max(high - low, 1e-3), 0.0), 1.0);
      f = f * (1.0 - ramp) + f / factor * ramp;
    }
    turns[i] = (uint64_t)std::nearbyint(std::ldexp(f / kTwoPi, 64));   // f <= 1: below 2^62
  }
  *magnitude = scaling == QLIN_ROPE_YARN ? (float)(0.1 * std::log(factor) + 1.0) : 1.0f;
  return QLIN_OK;
}

qlin_status qlin_sync_status(void* stream) {
  unsigned* status;
  Device dev;
  QLIN_TRY(device_state(&status, &dev));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  QLIN_CUDA(cudaStreamSynchronize(s));
  unsigned word = 0;
  QLIN_CUDA(cudaMemcpy(&word, status, sizeof word, cudaMemcpyDeviceToHost));
  if (word != 0) {
    const unsigned zero = 0;
    QLIN_CUDA(cudaMemcpy(status, &zero, sizeof zero, cudaMemcpyHostToDevice));
    return word == kErrTimeout ? QLIN_ERR_TIMEOUT : word == kErrInvalid ? QLIN_ERR_INVALID_ARG : QLIN_ERR_CUDA;
  }
  return QLIN_OK;
}

qlin_status qlin_selftest_bounded_wait(uint64_t timeout_ns, void* stream) {
  unsigned* status;
  Device dev;
  QLIN_TRY(device_state(&status, &dev));
  timeout_ns = std::min<uint64_t>(std::max<uint64_t>(timeout_ns, 1000ull), 2000000000ull);
  QLIN_CUDA(launch_wait_selftest(timeout_ns, static_cast<cudaStream_t>(stream), status));
  return QLIN_OK;
}

void qlin_set_wait_timeout_ns(uint64_t ns) {
  g_timeout_ns.store(std::max<uint64_t>(ns, 1000ull), std::memory_order_relaxed);
}

const char* qlin_status_str(qlin_status s) {
  switch (s) {
    case QLIN_OK: return "ok";
    case QLIN_ERR_INVALID_ARG: return "invalid argument";
    case QLIN_ERR_UNSUPPORTED: return "unsupported";
    case QLIN_ERR_MISALIGNED: return "misaligned pointer";
    case QLIN_ERR_CUDA: return "CUDA error";
    case QLIN_ERR_TIMEOUT: return "device wait timed out";
    case QLIN_ERR_WORKSPACE: return "workspace missing or too small";
  }
  return "unknown status";
}

const char* qlin_last_error(void) { return g_last_error; }

}  // extern "C"
