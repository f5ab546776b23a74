// Host side of rotary positions, 4-bit products and drawing tokens: implements the C
// ABI of ravel_decode.h.  (ravel_cache_append_rotary sits with the cache, cache_host.cpp.)
#include <cuda_runtime.h>

#include <atomic>
#include <cfloat>
#include <cmath>
#include <cstdio>
#include <new>

#include "../../include/ravel_decode.h"
#include "decode.h"
#include "rotary_host.h"

using namespace ravel;

struct ravel_w4_ctx {
  W4Matrix m{};
  int device = 0, num_sms = 0;
  ErrorWord* err = nullptr;
  int* err_host = nullptr;   // pinned, mapped: the error word's mirror
};

namespace {

thread_local char t_error[192] = "";

ravel_status fail(ravel_status s, const char* msg) {
  snprintf(t_error, sizeof t_error, "%s", msg);
  return s;
}

ravel_status cuda_fail(cudaError_t e, const char* what) {
  cudaGetLastError();   // (reported here: the step's launches ask for the last error)
  snprintf(t_error, sizeof t_error, "%s: %s", what, cudaGetErrorString(e));
  return e == cudaErrorMemoryAllocation ? RAVEL_ENOMEM : RAVEL_ECUDA;
}

// Calls on a handle run on its device, whatever the current one is.
struct OnDevice {
  int was = -1;
  cudaError_t e;
  explicit OnDevice(int device) {
    e = cudaGetDevice(&was);
    if (e == cudaSuccess && was != device) e = cudaSetDevice(device);
    else was = -1;
  }
  ~OnDevice() {
    if (was >= 0) cudaSetDevice(was);
  }
};

bool known(int dtype) { return dtype == RAVEL_FP32 || dtype == RAVEL_BF16; }
Dtype type_of(int dtype) { return dtype == RAVEL_BF16 ? DT_BF16 : DT_F32; }
int size_of(int dtype) { return dtype == RAVEL_BF16 ? 2 : 4; }

// The current device's SMs; once per device before anything is launched on it.
cudaError_t sm_count(int* out) {
  static std::atomic<int> counts[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const bool kept = dev >= 0 && dev < 64;
  *out = kept ? counts[dev].load(std::memory_order_relaxed) : 0;
  if (*out) return cudaSuccess;
  e = cudaDeviceGetAttribute(out, cudaDevAttrMultiProcessorCount, dev);
  if (e == cudaSuccess) e = init_draw_kernels();
  if (e == cudaSuccess && kept) counts[dev].store(*out, std::memory_order_relaxed);
  return e;
}

void free_matrix(ravel_w4_t* w) {
  if (w->m.codes) cudaFree(w->m.codes);
  if (w->m.sz) cudaFree(w->m.sz);
  if (w->err) cudaFree(w->err);
  if (w->err_host) cudaFreeHost(w->err_host);
  delete w;
}

const double kTwoPi = 6.283185307179586476925;

// f_i
double rotary_frequency(const ravel_rotary_config& c, int i) {
  if (c.frequencies) return c.frequencies[i];
  const double f = std::pow(c.base, -2.0 * i / c.dims);
  double g = 0.0;
  if (c.original_length > 0) {
    g = (c.original_length * f / kTwoPi - c.low) / (c.high - c.low);
    g = g < 0.0 ? 0.0 : g > 1.0 ? 1.0 : g;
  }
  return g >= 1.0 ? f : f * (g + (1.0 - g) / c.factor);
}

const char* rotary_fault(const ravel_rotary_config& c) {
  if (c.dims < 2 || c.dims % 2 || c.dims > 256) return "dims must be even, 2 to 256";
  if (c.interleaved != 0 && c.interleaved != 1) return "interleaved must be 0 or 1";
  if (!(std::fabs(c.amplitude) <= FLT_MAX)) return "amplitude must be finite in fp32";
  if (!c.frequencies) {
    if (!(c.base > 0) || !std::isfinite(c.base)) return "base must be positive";
    if (!(c.factor > 0) || !std::isfinite(c.factor)) return "factor must be positive";
    if (!(c.original_length >= 0) || !std::isfinite(c.original_length)) return "original_length must not be negative";
    if (c.original_length > 0 && !(c.low >= 0 && c.low < c.high && std::isfinite(c.high))) return "0 <= low < high is wanted";
  }
  for (int i = 0; i < c.dims / 2; ++i)   // (a small base or factor makes large ones)
    if (!std::isfinite(rotary_frequency(c, i))) return "frequencies must be finite";
  return nullptr;
}

}  // namespace

namespace ravel {

unsigned long long rotary_turns(const ravel_rotary_config& c, int i) {
  // turns per position modulo 1: whole turns do nothing at whole positions
  double turns = rotary_frequency(c, i) / kTwoPi;
  turns -= std::floor(turns);
  // (two halves: 2^64 itself is no uint64)
  const double high = std::floor(turns * 4294967296.0);
  const double low = std::floor((turns * 4294967296.0 - high) * 4294967296.0 + 0.5);
  return ((unsigned long long)high << 32) + (unsigned long long)low;
}

}  // namespace ravel

extern "C" {

const char* ravel_decode_last_error(void) { return t_error; }

ravel_status ravel_rotary_create(const ravel_rotary_config* cfg, int device, ravel_rotary_t** out) {
  if (!cfg || !out) return fail(RAVEL_EINVAL, "rotary_create: null argument");
  *out = nullptr;
  if (const char* why = rotary_fault(*cfg)) return fail(RAVEL_EINVAL, why);
  unsigned long long table[128] = {};
  for (int i = 0; i < cfg->dims / 2; ++i) table[i] = rotary_turns(*cfg, i);
  ravel_rotary_t* r = new (std::nothrow) ravel_rotary_t();
  if (!r) return fail(RAVEL_ENOMEM, "rotary_create: no memory");
  r->device = device;
  r->table.dims = cfg->dims;
  r->table.interleaved = cfg->interleaved;
  r->table.amplitude = (float)cfg->amplitude;
  OnDevice on(device);
  cudaError_t e = on.e;
  unsigned long long* f = nullptr;
  if (e == cudaSuccess) e = sm_count(&r->num_sms);
  if (e == cudaSuccess) e = cudaMalloc((void**)&f, sizeof table);
  if (e == cudaSuccess) e = cudaMemcpy(f, table, sizeof table, cudaMemcpyHostToDevice);
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  r->table.f = f;
  if (e != cudaSuccess) {
    const ravel_status s = cuda_fail(e, "rotary_create");
    if (f) cudaFree(f);
    delete r;
    return s;
  }
  *out = r;
  return RAVEL_OK;
}

void ravel_rotary_destroy(ravel_rotary_t* r) {
  if (!r) return;
  OnDevice on(r->device);
  if (on.e == cudaSuccess) {
    cudaDeviceSynchronize();
    cudaFree((void*)r->table.f);
  }
  delete r;
}

ravel_status ravel_rotary_apply(ravel_rotary_t* r, int batch, int n, int heads, int hd, int dtype, const void* x,
                                long long x_robot_stride, long long x_token_stride, void* out, long long out_robot_stride,
                                long long out_token_stride, const int* starts, const int* positions, const int* counts,
                                void* stream) {
  if (!r) return fail(RAVEL_EINVAL, "rotary_apply: null argument");
  if (!known(dtype)) return fail(RAVEL_EINVAL, "rotary_apply: unknown dtype");
  if (x_robot_stride < 0 || x_token_stride < 0 || out_robot_stride < 0 || out_token_stride < 0)
    return fail(RAVEL_EINVAL, "rotary_apply: negative stride");
  if (x == out && (x_robot_stride != out_robot_stride || x_token_stride != out_token_stride))
    return fail(RAVEL_EINVAL, "rotary_apply: in place, x and out need the same strides");
  if (batch < 0 || batch > 65535 || n < 0 || n > (1 << 30) || heads < 0 || heads > 65535)
    return fail(RAVEL_ESHAPE, "rotary_apply: up to 65535 robots and heads, 2^30 tokens");
  if (hd < r->table.dims || hd > 256) return fail(RAVEL_ESHAPE, "rotary_apply: hd outside [dims, 256]");
  if (batch == 0 || n == 0 || heads == 0) return RAVEL_OK;
  if (!x || !out) return fail(RAVEL_EINVAL, "rotary_apply: null argument");
  if (((uintptr_t)x | (uintptr_t)out) % size_of(dtype)) return fail(RAVEL_EINVAL, "rotary_apply: unaligned x or out");
  if (rows_overlap(batch, n, (long long)heads * hd, out_robot_stride, out_token_stride))
    return fail(RAVEL_EINVAL, "rotary_apply: rows of out overlap");
  RotaryArgs a{r->table, x,     out, x_robot_stride, x_token_stride, out_robot_stride, out_token_stride, batch, n, heads, hd,
               starts,   positions, counts, 16, r->num_sms, 0};
  const long long es = size_of(dtype);
  const uintptr_t all = (uintptr_t)x | (uintptr_t)out | (uintptr_t)(x_robot_stride * es) | (uintptr_t)(x_token_stride * es) |
                        (uintptr_t)(out_robot_stride * es) | (uintptr_t)(out_token_stride * es);
  while (all % a.align) a.align /= 2;
  OnDevice on(r->device);
  cudaError_t e = on.e;
  if (e == cudaSuccess) e = launch_rotary(a, type_of(dtype), (cudaStream_t)stream);
  return e == cudaSuccess ? RAVEL_OK : cuda_fail(e, "rotary_apply");
}

ravel_status ravel_w4_create(int N, int K, int group, int device, ravel_w4_t** out) {
  if (!out) return fail(RAVEL_EINVAL, "w4_create: null argument");
  *out = nullptr;
  if (group != 32 && group != 64 && group != 128) return fail(RAVEL_EINVAL, "w4_create: group must be 32, 64 or 128");
  if (N < 1 || K < 1 || N > (1 << 24) || K > (1 << 24)) return fail(RAVEL_ESHAPE, "w4_create: N and K must be 1 to 2^24");
  ravel_w4_t* w = new (std::nothrow) ravel_w4_t();
  if (!w) return fail(RAVEL_ENOMEM, "w4_create: no memory");
  W4Matrix& m = w->m = W4Matrix(N, K, group);
  w->device = device;
  const size_t codes = (size_t)m.tiles * m.kblocks * 512, sz = ((size_t)m.tiles * m.groups + kPadGroups) * 64;
  OnDevice on(device);
  cudaError_t e = on.e;
  if (e == cudaSuccess) e = sm_count(&w->num_sms);
  if (e == cudaSuccess) e = init_w4_kernels();
  if (e == cudaSuccess) e = cudaMalloc((void**)&m.codes, codes);
  if (e == cudaSuccess) e = cudaMalloc((void**)&m.sz, sz);
  if (e == cudaSuccess) e = cudaMemset(m.codes, 0, codes);
  if (e == cudaSuccess) e = cudaMemset(m.sz, 0, sz);
  ErrorWord word{0, nullptr};
  if (e == cudaSuccess) e = cudaMalloc((void**)&w->err, sizeof word);
  if (e == cudaSuccess) e = cudaHostAlloc((void**)&w->err_host, sizeof(int), cudaHostAllocMapped);
  if (e == cudaSuccess) *w->err_host = 0;
  if (e == cudaSuccess) e = cudaHostGetDevicePointer((void**)&word.mirror, w->err_host, 0);
  if (e == cudaSuccess) e = cudaMemcpy(w->err, &word, sizeof word, cudaMemcpyHostToDevice);
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (e != cudaSuccess) {
    const ravel_status s = cuda_fail(e, "w4_create");
    free_matrix(w);
    cudaGetLastError();
    return s;
  }
  *out = w;
  return RAVEL_OK;
}

void ravel_w4_destroy(ravel_w4_t* w) {
  if (!w) return;
  OnDevice on(w->device);
  if (on.e == cudaSuccess) cudaDeviceSynchronize();
  free_matrix(w);
}

ravel_status ravel_w4_reset(ravel_w4_t* w) {
  if (!w) return fail(RAVEL_EINVAL, "w4_reset: null argument");
  OnDevice on(w->device);
  cudaError_t e = on.e;
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemset(w->err, 0, sizeof(int));
  if (e != cudaSuccess) return cuda_fail(e, "w4_reset");
  *w->err_host = 0;
  return RAVEL_OK;
}

ravel_status ravel_w4_load(ravel_w4_t* w, const void* codes, const void* scales, const void* zeros, void* stream) {
  if (!w || !codes || !scales || !zeros) return fail(RAVEL_EINVAL, "w4_load: null argument");
  if ((uintptr_t)scales % 2) return fail(RAVEL_EINVAL, "w4_load: scales must be aligned");
  OnDevice on(w->device);
  cudaError_t e = on.e;
  cudaStreamCaptureStatus cs = cudaStreamCaptureStatusNone;
  if (e == cudaSuccess) e = cudaStreamIsCapturing((cudaStream_t)stream, &cs);
  if (e == cudaSuccess && cs != cudaStreamCaptureStatusNone)
    return fail(RAVEL_EINVAL, "w4_load: not on a stream that is being captured");
  if (e == cudaSuccess)
    e = launch_w4_load(w->m, (const uint8_t*)codes, (const uint16_t*)scales, (const uint8_t*)zeros, (cudaStream_t)stream);
  if (e == cudaSuccess) e = cudaStreamSynchronize((cudaStream_t)stream);
  return e == cudaSuccess ? RAVEL_OK : cuda_fail(e, "w4_load");
}

ravel_status ravel_w4_quantize(const void* W, int N, int K, int ldw, int dtype, int group, void* codes, void* scales,
                               void* zeros, void* stream) {
  if (!W || !codes || !scales || !zeros) return fail(RAVEL_EINVAL, "w4_quantize: null argument");
  if (!known(dtype)) return fail(RAVEL_EINVAL, "w4_quantize: unknown dtype");
  if (group != 32 && group != 64 && group != 128) return fail(RAVEL_EINVAL, "w4_quantize: group must be 32, 64 or 128");
  if ((uintptr_t)W % size_of(dtype) || (uintptr_t)scales % 2) return fail(RAVEL_EINVAL, "w4_quantize: unaligned W or scales");
  if (N < 1 || K < 1 || ldw < K || N > (1 << 24) || K > (1 << 24)) return fail(RAVEL_ESHAPE, "w4_quantize: N, K or ldw");
  if ((long long)N * ((K + group - 1) / group) > (1ll << 31))
    return fail(RAVEL_ESHAPE, "w4_quantize: at most 2^31 groups");
  const cudaError_t e = launch_w4_quantize(W, N, K, ldw, type_of(dtype), group, (uint8_t*)codes, (uint16_t*)scales,
                                           (uint8_t*)zeros, (cudaStream_t)stream);
  return e == cudaSuccess ? RAVEL_OK : cuda_fail(e, "w4_quantize");
}

ravel_status ravel_w4_read(ravel_w4_t* w, void* out, int ldo, int dtype, void* stream) {
  if (!w || !out) return fail(RAVEL_EINVAL, "w4_read: null argument");
  if (!known(dtype)) return fail(RAVEL_EINVAL, "w4_read: unknown dtype");
  if (ldo < w->m.K) return fail(RAVEL_ESHAPE, "w4_read: ldo below K");
  if ((uintptr_t)out % size_of(dtype)) return fail(RAVEL_EINVAL, "w4_read: unaligned out");
  OnDevice on(w->device);
  cudaError_t e = on.e;
  if (e == cudaSuccess) e = launch_w4_read(w->m, out, ldo, type_of(dtype), (cudaStream_t)stream);
  return e == cudaSuccess ? RAVEL_OK : cuda_fail(e, "w4_read");
}

ravel_status ravel_w4_gemm(const ravel_w4_t* w, const void* X, int M, int lda, int epi, void* out, int ldo, int out_dtype,
                           const float* bias, void* stream) {
  if (!w) return fail(RAVEL_EINVAL, "w4_gemm: null argument");
  if (epi < 0 || epi > 3 || !known(out_dtype)) return fail(RAVEL_EINVAL, "w4_gemm: unknown epilogue or dtype");
  if (epi == EPI_ADD_F32 && out_dtype != RAVEL_FP32) return fail(RAVEL_EINVAL, "w4_gemm: epilogue 2 adds to float32");
  if (epi == EPI_GEGLU && (w->m.N % 128 || out_dtype != RAVEL_BF16))
    return fail(RAVEL_EINVAL, "w4_gemm: epilogue 3 takes N % 128 == 0 and a bf16 out");
  if (M < 0 || M > (1 << 19) || lda < w->m.K || ldo < (epi == EPI_GEGLU ? w->m.N / 2 : w->m.N))
    return fail(RAVEL_ESHAPE, "w4_gemm: M outside [0, 2^19], lda below K or ldo below the outputs");
  if ((uintptr_t)X % 2 || (uintptr_t)out % size_of(out_dtype)) return fail(RAVEL_EINVAL, "w4_gemm: unaligned X or out");
  if (M == 0) return RAVEL_OK;
  if (!X || !out) return fail(RAVEL_EINVAL, "w4_gemm: null argument");
  const int bits = *(volatile int*)w->err_host;
  if (bits) {
    snprintf(t_error, sizeof t_error, "device error word 0x%x", bits);
    return bits & ERR_TIMEOUT ? RAVEL_ETIMEOUT : RAVEL_EDEVICE;
  }
  W4Args a{w->m, X, out, bias, M, lda, ldo, epi, out_dtype == RAVEL_BF16, 0, w->num_sms, &w->err->bits};
  a.vec = (uintptr_t)X % 16 == 0 && lda % 8 == 0;
  OnDevice on(w->device);
  cudaError_t e = on.e;
  if (e == cudaSuccess) e = launch_w4_gemm(a, (cudaStream_t)stream);
  return e == cudaSuccess ? RAVEL_OK : cuda_fail(e, "w4_gemm");
}

ravel_status ravel_draw_tokens(const void* logits, int batch, int vocab, long long row_stride, int dtype, const float* u,
                               const float* temperature, const int* top_k, const float* top_p, const float* min_p,
                               int* tokens, float* log_probs, void* stream) {
  if (!known(dtype)) return fail(RAVEL_EINVAL, "draw_tokens: unknown dtype");
  if (batch < 0 || batch > 65535 || vocab < 1 || vocab > (1 << 20))
    return fail(RAVEL_ESHAPE, "draw_tokens: up to 65535 rows of 1 to 2^20 tokens");
  if (batch > 1 && row_stride < vocab) return fail(RAVEL_ESHAPE, "draw_tokens: rows overlap");
  if (batch == 0) return RAVEL_OK;
  if (!logits || !u || !tokens) return fail(RAVEL_EINVAL, "draw_tokens: null argument");
  if ((uintptr_t)logits % size_of(dtype)) return fail(RAVEL_EINVAL, "draw_tokens: unaligned logits");
  DrawArgs a{logits, batch, vocab, row_stride, u, temperature, top_p, min_p, top_k, tokens, log_probs, 0};
  cudaError_t e = sm_count(&a.num_sms);
  if (e == cudaSuccess) e = launch_draw(a, type_of(dtype), (cudaStream_t)stream);
  return e == cudaSuccess ? RAVEL_OK : cuda_fail(e, "draw_tokens");
}

}  // extern "C"
