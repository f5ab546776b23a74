// Host side of the 8-bit context cache: owns its storage and workspace and
// implements the C ABI of ravel_cache.h.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <new>
#include <string>
#include <vector>

#include "../../include/ravel_cache.h"
#include "cache.h"
#include "rotary_host.h"

using namespace ravel;

struct ravel_cache_ctx {
  ravel_cache_config cfg{};
  Dtype dt = DT_F32;
  size_t esize = 4;
  int device = 0, num_sms = 0, clusters[9] = {};
  int hdp = 0, T = 0;            // held row bytes; capacity rounded up
  size_t rows = 0, blocks = 0;   // per layer: bytes of K (or V), exponents
  uint8_t *k = nullptr, *v = nullptr;
  int8_t *ke = nullptr, *ve = nullptr;
  float* part = nullptr;
  float2 *part_ml = nullptr, *row_ml = nullptr;
  unsigned* arrived = nullptr;
  uint8_t* q_ws = nullptr;
  float* mass_ws = nullptr;
  size_t mass_ws_bytes = 0;
  ErrorWord* err = nullptr;
  int* err_host = nullptr;       // pinned, mapped: the error word's mirror
  std::vector<void*> allocs;
  std::vector<CacheMaps> maps;   // by layer
  std::string last_error;

  CacheLayer layer(int l) const {
    return CacheLayer{k + rows * l, v + rows * l, ke + blocks * l, ve + blocks * l, cfg.n_kv_heads, cfg.head_dim, hdp, T};
  }
};

namespace {

ravel_status fail(ravel_cache_t* c, ravel_status s, const char* msg) {
  try {
    if (c) c->last_error = msg;
  } catch (...) {   // no memory for the text: the status stands
  }
  return s;
}

ravel_status cuda_fail(ravel_cache_t* c, cudaError_t e, const char* what) {
  char buf[160];
  cudaGetLastError();   // (reported here: the step's launches ask for the last error)
  snprintf(buf, sizeof buf, "%s: %s", what, cudaGetErrorString(e));
  return fail(c, e == cudaErrorMemoryAllocation ? RAVEL_ENOMEM : RAVEL_ECUDA, buf);
}

// What every call checks: the layer, the batch and an error that earlier work raised.
ravel_status check_call(ravel_cache_t* c, int layer, int batch, const char* what) {
  char buf[96];
  if (layer < 0 || layer >= c->cfg.layers || batch < 1 || batch > c->cfg.max_batch) {
    snprintf(buf, sizeof buf, "%s: layer or batch outside the configuration", what);
    return fail(c, RAVEL_ESHAPE, buf);
  }
  const int bits = *(volatile int*)c->err_host;
  if (bits) {
    snprintf(buf, sizeof buf, "device error word 0x%x", bits);
    return fail(c, (bits & ERR_TIMEOUT) ? RAVEL_ETIMEOUT : RAVEL_EDEVICE, buf);
  }
  const cudaError_t e = cudaSetDevice(c->device);
  return e == cudaSuccess ? RAVEL_OK : cuda_fail(c, e, "cudaSetDevice");
}

bool aligned16(const void* p, long long s0, long long s1, size_t es) {
  return ((uintptr_t)p | (uintptr_t)(s0 * (long long)es) | (uintptr_t)(s1 * (long long)es)) % 16 == 0;
}

const char* config_fault(const ravel_cache_config& c) {
  if (c.layers < 1 || c.n_q_heads < 1 || c.n_kv_heads < 1 || c.max_tokens < 1 || c.max_batch < 1 || c.max_queries < 1)
    return "every size must be at least 1";
  if (c.n_q_heads % c.n_kv_heads) return "n_q_heads must be a multiple of n_kv_heads";
  if (c.head_dim < 8 || c.head_dim % 8 || c.head_dim > 256) return "head_dim must be a multiple of 8, at most 256";
  if (c.dtype != RAVEL_FP32 && c.dtype != RAVEL_BF16) return "unknown dtype";
  if (c.n_kv_heads > 65535 || c.max_batch > 65535) return "at most 65535 KV heads and robots";
  // (rows of a layer are counted in 32 bits, and what a CTA steps past the last one as well; the
  // product of three 32-bit sizes could pass 64)
  if ((double)c.max_batch * c.n_kv_heads * ((double)c.max_tokens + kCacheRound) > 2147483648.0 - 65536.0)
    return "max_batch * n_kv_heads * max_tokens must be below 2^31 - 2^16";
  if ((long long)c.max_queries * c.n_q_heads > (1 << 30)) return "max_queries * n_q_heads must be at most 2^30";
  return nullptr;
}

}  // namespace

extern "C" {

const char* ravel_cache_last_error(const ravel_cache_t* c) { return c ? c->last_error.c_str() : ""; }

ravel_status ravel_cache_create(const ravel_cache_config* cfg, int device, ravel_cache_t** out) {
  if (!cfg || !out) return RAVEL_EINVAL;
  *out = nullptr;
  if (const char* why = config_fault(*cfg)) {
    fprintf(stderr, "ravel_cache_create: %s\n", why);
    return RAVEL_ESHAPE;
  }
  ravel_cache_t* c = new (std::nothrow) ravel_cache_t();
  if (!c) return RAVEL_ENOMEM;
  c->cfg = *cfg;
  c->dt = cfg->dtype == RAVEL_BF16 ? DT_BF16 : DT_F32;
  c->esize = cfg->dtype == RAVEL_BF16 ? 2 : 4;
  c->device = device;
  c->hdp = (cfg->head_dim + 63) / 64 * 64;
  c->T = (cfg->max_tokens + kCacheRound - 1) / kCacheRound * kCacheRound;
  const size_t heads = (size_t)cfg->max_batch * cfg->n_kv_heads;
  c->rows = heads * c->T * c->hdp;
  c->blocks = heads * (c->T / kCacheBlock);
  cudaError_t e = cudaSetDevice(device);
  const char* what = "cudaSetDevice";
  auto get = [&](auto** p, size_t bytes) {
    if (e != cudaSuccess) return;
    what = "allocation";
    e = cudaMalloc((void**)p, bytes);
    if (e != cudaSuccess) return;
    c->allocs.push_back(*p);   // (reserved below: does not throw)
    what = "clear";
    e = cudaMemset(*p, 0, bytes);   // codes and exponents that nobody wrote are finite
  };
  try {
    c->allocs.reserve(16);
    c->maps.resize(cfg->layers);
  } catch (...) {
    delete c;
    return RAVEL_ENOMEM;
  }
  get(&c->k, c->rows * cfg->layers);
  get(&c->v, c->rows * cfg->layers);
  get(&c->ke, c->blocks * cfg->layers);
  get(&c->ve, c->blocks * cfg->layers);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&c->num_sms, cudaDevAttrMultiProcessorCount, device);
  const size_t part_rows = std::max((size_t)kCacheSplitCtas * 16, (size_t)c->num_sms * kCacheTcRows);
  get(&c->part, sizeof(float) * part_rows * c->hdp);
  get(&c->part_ml, sizeof(float2) * part_rows);
  get(&c->arrived, sizeof(unsigned) * kCacheSplitCtas);
  get(&c->row_ml, sizeof(float2) * cfg->max_batch * (size_t)cfg->n_q_heads * cfg->max_queries);
  const int G = cfg->n_q_heads / cfg->n_kv_heads;
  c->mass_ws_bytes = cache_mass_ws_bytes((int)heads, cfg->n_kv_heads, G, cfg->dtype == RAVEL_FP32 ? (long long)cfg->max_queries * G : 16,
                                         c->T, c->num_sms);
  get(&c->mass_ws, c->mass_ws_bytes);
  get(&c->q_ws, (size_t)c->num_sms * kCacheTcRows * c->hdp * 2);
  get(&c->err, sizeof(ErrorWord));
  if (e == cudaSuccess) {
    what = "set-up";
    ErrorWord w{0, nullptr};
    e = cudaHostAlloc((void**)&c->err_host, sizeof(int), cudaHostAllocMapped);
    if (e == cudaSuccess) *c->err_host = 0;
    if (e == cudaSuccess) e = cudaHostGetDevicePointer((void**)&w.mirror, c->err_host, 0);
    if (e == cudaSuccess) e = cudaMemcpy(c->err, &w, sizeof w, cudaMemcpyHostToDevice);
    for (int l = 0; l < cfg->layers && e == cudaSuccess; ++l) e = encode_layer(&c->maps[l], c->layer(l), cfg->max_batch);
    if (e == cudaSuccess) e = init_cache_kernels();
    if (e == cudaSuccess) e = init_cache_tc_kernels(c->hdp, c->clusters);
    if (e == cudaSuccess) e = init_cache_mass_tc_kernels();
    if (e == cudaSuccess) e = cudaDeviceSynchronize();
  }
  if (e != cudaSuccess) {
    fprintf(stderr, "ravel_cache_create: %s: %s\n", what, cudaGetErrorString(e));
    ravel_cache_destroy(c);
    cudaGetLastError();   // (as in cuda_fail)
    return e == cudaErrorMemoryAllocation ? RAVEL_ENOMEM : RAVEL_ECUDA;
  }
  *out = c;
  return RAVEL_OK;
}

void ravel_cache_destroy(ravel_cache_t* c) {
  if (!c) return;
  cudaSetDevice(c->device);
  cudaDeviceSynchronize();
  for (void* p : c->allocs) cudaFree(p);
  if (c->err_host) cudaFreeHost(c->err_host);
  delete c;
}

ravel_status ravel_cache_reset(ravel_cache_t* c) {
  if (!c) return RAVEL_EINVAL;
  cudaError_t e = cudaSetDevice(c->device);
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemset(c->err, 0, sizeof(int));
  if (e != cudaSuccess) return cuda_fail(c, e, "reset");
  *c->err_host = 0;
  return RAVEL_OK;
}

ravel_status ravel_cache_append(ravel_cache_t* c, int layer, int batch, int n, const void* k, const void* v,
                                long long robot_stride, long long token_stride, const int* starts, const int* counts,
                                void* stream) {
  if (!c || !k || !v) return fail(c, RAVEL_EINVAL, "append: null argument");
  if (robot_stride < 0 || token_stride < 0) return fail(c, RAVEL_EINVAL, "append: negative stride");
  ravel_status s = check_call(c, layer, batch, "append");
  if (s != RAVEL_OK) return s;
  if (n < 1 || n > c->cfg.max_tokens) return fail(c, RAVEL_ESHAPE, "append: n outside [1, max_tokens]");
  AppendArgs a{c->layer(layer), k, v, robot_stride, token_stride, batch, n, c->cfg.max_tokens, starts, counts, 0,
               &c->err->bits};
  a.vec = aligned16(k, robot_stride, token_stride, c->esize) && aligned16(v, 0, 0, 1);
  const cudaError_t e = launch_cache_append(a, c->dt, (cudaStream_t)stream);
  return e == cudaSuccess ? RAVEL_OK : cuda_fail(c, e, "append");
}

ravel_status ravel_cache_append_rotary(ravel_cache_t* c, int layer, const ravel_rotary_t* r, int batch, int n, const void* q,
                                       long long q_robot_stride, long long q_token_stride, void* q_out,
                                       long long q_out_robot_stride, long long q_out_token_stride, const void* k,
                                       long long k_robot_stride, long long k_token_stride, const void* v,
                                       long long v_robot_stride, long long v_token_stride, const int* starts,
                                       const int* positions, const int* counts, void* stream) {
  if (!c || !r || !k || !v) return fail(c, RAVEL_EINVAL, "append_rotary: null argument");
  if (!q != !q_out) return fail(c, RAVEL_EINVAL, "append_rotary: q and q_out go together");
  if (q_robot_stride < 0 || q_token_stride < 0 || q_out_robot_stride < 0 || q_out_token_stride < 0 || k_robot_stride < 0 ||
      k_token_stride < 0 || v_robot_stride < 0 || v_token_stride < 0)
    return fail(c, RAVEL_EINVAL, "append_rotary: negative stride");
  if (q && q == q_out && (q_robot_stride != q_out_robot_stride || q_token_stride != q_out_token_stride))
    return fail(c, RAVEL_EINVAL, "append_rotary: in place, q and q_out need the same strides");
  ravel_status s = check_call(c, layer, batch, "append_rotary");
  if (s != RAVEL_OK) return s;
  if (n < 1 || n > c->cfg.max_tokens) return fail(c, RAVEL_ESHAPE, "append_rotary: n outside [1, max_tokens]");
  if (((uintptr_t)q | (uintptr_t)q_out | (uintptr_t)k | (uintptr_t)v) % c->esize)
    return fail(c, RAVEL_EINVAL, "append_rotary: unaligned q, q_out, k or v");
  if (q && (long long)c->cfg.n_q_heads * c->hdp > (1 << 30))   // (places in a token's queries are counted in 32 bits)
    return fail(c, RAVEL_ESHAPE, "append_rotary: more than 2^30 values in the query heads of a token");
  if (q && rows_overlap(batch, n, (long long)c->cfg.n_q_heads * c->cfg.head_dim, q_out_robot_stride, q_out_token_stride))
    return fail(c, RAVEL_EINVAL, "append_rotary: rows of q_out overlap");
  if (r->table.dims > c->cfg.head_dim) return fail(c, RAVEL_ESHAPE, "append_rotary: the table has more dims than a head");
  if (r->device != c->device) return fail(c, RAVEL_EINVAL, "append_rotary: the table is on another device");
  AppendRotaryArgs a{c->layer(layer), r->table, q, k, v, q_out, q_robot_stride, q_token_stride, q_out_robot_stride,
                     q_out_token_stride, k_robot_stride, k_token_stride, v_robot_stride, v_token_stride, batch, n,
                     c->cfg.n_q_heads / c->cfg.n_kv_heads, c->cfg.max_tokens, starts, positions, counts, 0, 0, 16, c->num_sms, &c->err->bits};
  a.kv_vec = aligned16(k, k_robot_stride, k_token_stride, c->esize) && aligned16(v, v_robot_stride, v_token_stride, c->esize);
  a.q_vec = aligned16(q, q_robot_stride, q_token_stride, c->esize) &&
            aligned16(q_out, q_out_robot_stride, q_out_token_stride, c->esize);
  const long long es = (long long)c->esize;
  const uintptr_t all = (uintptr_t)q | (uintptr_t)q_out | (uintptr_t)(q_robot_stride * es) | (uintptr_t)(q_token_stride * es) |
                        (uintptr_t)(q_out_robot_stride * es) | (uintptr_t)(q_out_token_stride * es);
  while (all % a.q_align) a.q_align /= 2;
  const cudaError_t e = launch_cache_append_rotary(a, c->dt, (cudaStream_t)stream);
  return e == cudaSuccess ? RAVEL_OK : cuda_fail(c, e, "append_rotary");
}

ravel_status ravel_cache_attend(ravel_cache_t* c, int layer, int batch, int n, const void* q, long long q_robot_stride,
                                long long q_token_stride, void* out, long long out_robot_stride,
                                long long out_token_stride, const int* lengths, const int* counts, int max_length,
                                int causal, int window, int sinks, float scale, float* mass, long long mass_stride,
                                int mass_add, void* stream) {
  if (!c || !q || !out || !lengths) return fail(c, RAVEL_EINVAL, "attend: null argument");
  if (q_robot_stride < 0 || q_token_stride < 0 || out_robot_stride < 0 || out_token_stride < 0)
    return fail(c, RAVEL_EINVAL, "attend: negative stride");
  if ((causal != 0 && causal != 1) || (mass_add != 0 && mass_add != 1) || window < 0 || sinks < 0 ||
      (window > 0 && !causal) || (sinks > 0 && window == 0))
    return fail(c, RAVEL_EINVAL, "attend: a window needs causal = 1, sinks need a window, none is negative");
  if (!(scale >= 0.f) || std::isinf(scale)) return fail(c, RAVEL_EINVAL, "attend: scale must be finite and not negative");
  ravel_status s = check_call(c, layer, batch, "attend");
  if (s != RAVEL_OK) return s;
  if (n < 1 || n > c->cfg.max_queries) return fail(c, RAVEL_ESHAPE, "attend: n outside [1, max_queries]");
  if (max_length < 0 || max_length > c->cfg.max_tokens)
    return fail(c, RAVEL_ESHAPE, "attend: max_length outside [0, max_tokens]");
  if (mass && mass_stride < max_length) return fail(c, RAVEL_ESHAPE, "attend: mass_stride below max_length");
  CacheAttnArgs a{};
  a.c = c->layer(layer);
  a.maps = &c->maps[layer];
  a.q = q;
  a.out = out;
  a.q_robot = q_robot_stride;
  a.q_token = q_token_stride;
  a.out_robot = out_robot_stride;
  a.out_token = out_token_stride;
  a.lengths = lengths;
  a.counts = counts;
  a.batch = batch;
  a.n = n;
  a.G = c->cfg.n_q_heads / c->cfg.n_kv_heads;
  a.by_G = LaunchDiv(a.G);
  a.by_heads = LaunchDiv(c->cfg.n_kv_heads);
  a.max_length = max_length;
  a.causal = causal;
  // (a window or sinks of the whole length hide nothing; bounded, positions stay in 32 bits)
  a.window = window > max_length ? 0 : window;
  a.sinks = a.window ? (sinks > max_length ? max_length : sinks) : 0;
  const float sc = scale > 0.f ? scale : 1.f / std::sqrt((float)c->cfg.head_dim);
  a.scale_log2 = sc * 1.4426950408889634f;
  a.mass = mass;
  a.mass_stride = mass_stride;
  a.mass_add = mass_add;
  a.vec = aligned16(q, q_robot_stride, q_token_stride, c->esize);
  a.num_sms = c->num_sms;
  a.clusters = c->clusters;
  a.part = c->part;
  a.part_ml = c->part_ml;
  a.arrived = c->arrived;
  a.row_ml = c->row_ml;
  a.q_ws = c->q_ws;
  a.mass_ws = c->mass_ws;
  a.mass_ws_bytes = c->mass_ws_bytes;
  a.err = &c->err->bits;
  const cudaError_t e = launch_cache_attend(a, c->dt, (cudaStream_t)stream);
  return e == cudaSuccess ? RAVEL_OK : cuda_fail(c, e, "attend");
}

ravel_status ravel_cache_evict(ravel_cache_t* c, int layer, ravel_cache_t* to, int to_layer, int batch,
                               const int* lengths, const float* mass, long long mass_stride, int keep, int sinks,
                               int recent, int* new_lengths, int* index, float* new_mass, void* stream) {
  if (!c || !to || !lengths || !mass || !new_lengths || !index) return fail(c, RAVEL_EINVAL, "evict: null argument");
  if (c == to && layer == to_layer) return fail(c, RAVEL_EINVAL, "evict: a layer cannot be evicted into itself");
  if (sinks < 0 || recent < 0 || mass_stride < 0) return fail(c, RAVEL_EINVAL, "evict: negative argument");
  ravel_status s = check_call(c, layer, batch, "evict");
  if (s != RAVEL_OK) return s;
  if (to_layer < 0 || to_layer >= to->cfg.layers || batch > to->cfg.max_batch ||
      to->cfg.n_kv_heads != c->cfg.n_kv_heads || to->cfg.head_dim != c->cfg.head_dim || to->device != c->device)
    return fail(c, RAVEL_ESHAPE, "evict: the other cache does not fit");
  if (keep < 1 || keep > to->cfg.max_tokens || (long long)sinks + recent > keep)
    return fail(c, RAVEL_ESHAPE, "evict: keep outside [max(1, sinks + recent), max_tokens]");
  EvictArgs a{c->layer(layer), to->layer(to_layer), batch, keep, sinks, recent, c->cfg.max_tokens, lengths, mass,
              mass_stride, new_lengths, index, new_mass, &c->err->bits};
  const cudaError_t e = launch_cache_evict(a, (cudaStream_t)stream);
  return e == cudaSuccess ? RAVEL_OK : cuda_fail(c, e, "evict");
}

ravel_status ravel_cache_read(ravel_cache_t* c, int layer, int batch, int n, const int* firsts, const int* lengths,
                              void* k, void* v, void* stream) {
  if (!c || !k || !v) return fail(c, RAVEL_EINVAL, "read: null argument");
  ravel_status s = check_call(c, layer, batch, "read");
  if (s != RAVEL_OK) return s;
  if (n < 1 || n > c->T) return fail(c, RAVEL_ESHAPE, "read: n outside [1, max_tokens rounded up to 128]");
  ReadArgs a{c->layer(layer), batch, n, c->cfg.max_tokens, firsts, lengths, k, v, 0, &c->err->bits};
  a.vec = aligned16(k, 0, 0, 1) && aligned16(v, 0, 0, 1);
  const cudaError_t e = launch_cache_read(a, c->dt, (cudaStream_t)stream);
  return e == cudaSuccess ? RAVEL_OK : cuda_fail(c, e, "read");
}

}  // extern "C"
