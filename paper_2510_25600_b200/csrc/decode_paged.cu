// purekv_decode_paged: attention of one new token per request over the pages of a cache.
#include <cmath>

#include <cuda_fp8.h>

#include "common.cuh"
#include "paged.cuh"
#include "paged_args.cuh"

namespace purekv {

struct DecodePagedArgs {
  const uint8_t* q;  // strides in bytes
  int64_t q_tok, q_head;
  const uint8_t *k_pool, *v_pool;
  const float *k_scale, *v_scale;
  PagedView view;
  int32_t n_req, n_q_heads, n_kv_heads, group;
  float scale_log2;
  void* o;
  float* lse;
  int32_t* status;
};

template <typename C>
__device__ __forceinline__ float held(const C* p) { return (float)*p; }

// One CTA per (head, request): four warps take the keys in turn, a lane D / 32 of the row's elements.
template <typename T, typename C, int D>
__global__ void __launch_bounds__(128) decode_paged_simple_kernel(const DecodePagedArgs a) {
  constexpr int E = D / 32;
  __shared__ float s_o[4][D], s_m[4], s_l[4];
  const int32_t h = blockIdx.x, r = blockIdx.y, g = h / a.group, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int32_t len = a.view.seq_lens[r], n = min(max(len, 0), a.view.capacity());
  if (len > n && threadIdx.x == 0) atomicExch(a.status, (int32_t)PUREKV_ERR_BAD_PAGE);
  const int32_t* list = a.view.table + r * a.view.table_stride;
  const float ks = a.k_scale ? a.k_scale[g] : 1.f, vs = a.v_scale ? a.v_scale[g] : 1.f;
  float q[E], acc[E], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    q[e] = (float)reinterpret_cast<const T*>(a.q + r * a.q_tok + h * a.q_head)[lane * E + e] * a.scale_log2 * ks;
    acc[e] = 0.f;
  }
  for (int32_t j = warp; j < n; j += 4) {
    const int64_t at = a.view.row_offset(list, j);
    if (at < 0) {
      if (lane == 0) atomicExch(a.status, (int32_t)PUREKV_ERR_BAD_PAGE);
      continue;
    }
    const C* k = reinterpret_cast<const C*>(a.k_pool + at + g * a.view.head_stride) + lane * E;
    const C* v = reinterpret_cast<const C*>(a.v_pool + at + g * a.view.head_stride) + lane * E;
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) s = fmaf(q[e], held(k + e), s);
#pragma unroll
    for (int mask = 16; mask >= 1; mask >>= 1) s += __shfl_xor_sync(0xffffffffu, s, mask);
    const float top = fmaxf(m, s), ref = top == -INFINITY ? 0.f : top;
    const float alpha = exp2f(m - ref), p = exp2f(s - ref);
    l = l * alpha + p;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = acc[e] * alpha + p * held(v + e);
    m = top;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) s_o[warp][lane * E + e] = acc[e];
  if (lane == 0) {
    s_m[warp] = m;
    s_l[warp] = l;
  }
  __syncthreads();
  const float top = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3])), ref = top == -INFINITY ? 0.f : top;
  float w[4], sum = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    w[i] = exp2f(s_m[i] - ref);
    sum += w[i] * s_l[i];
  }
  const int64_t out = (int64_t)r * a.n_q_heads + h;
  for (int32_t c = threadIdx.x; c < D; c += 128) {
    const float x = w[0] * s_o[0][c] + w[1] * s_o[1][c] + w[2] * s_o[2][c] + w[3] * s_o[3][c];
    reinterpret_cast<T*>(a.o)[out * D + c] = (T)(n > 0 ? x / sum * vs : 0.f);
  }
  if (a.lse && threadIdx.x == 0) a.lse[out] = n > 0 ? (ref + log2f(sum)) * 0.6931471805599453f : -INFINITY;
}

template <typename T, typename C>
static purekv_status launch_simple(const DecodePagedArgs& a, int32_t head_dim, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)a.n_q_heads, (unsigned)a.n_req);
  cfg.blockDim = dim3(128);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (head_dim == 64)
    PK_CUDA(cudaLaunchKernelEx(&cfg, decode_paged_simple_kernel<T, C, 64>, a));
  else
    PK_CUDA(cudaLaunchKernelEx(&cfg, decode_paged_simple_kernel<T, C, 128>, a));
  return PUREKV_OK;
}

}  // namespace purekv

using namespace purekv;

extern "C" {

size_t purekv_decode_paged_ws_bytes(int32_t n_req, int32_t max_len, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                    purekv_dtype dtype) {
  (void)n_req; (void)max_len; (void)n_q_heads; (void)n_kv_heads; (void)head_dim; (void)dtype;
  return 0;
}

purekv_status purekv_decode_paged(const void* q, int64_t q_token_stride, int64_t q_head_stride, void* o, float* lse,
                                  const purekv_pages* pages, int32_t max_len, int32_t n_q_heads, purekv_dtype dtype,
                                  float softmax_scale, void* ws, size_t ws_bytes, int32_t* status, void* stream) {
  static const char* const kName = "purekv_decode_paged";
  PK_REQUIRE(dtype == PUREKV_BF16 || dtype == PUREKV_FP32, PUREKV_ERR_INVALID_ARG, "%s: q is bf16 or fp32", kName);
  PK_REQUIRE(pages, PUREKV_ERR_INVALID_ARG, "%s: no pages", kName);
  const purekv_status st = check_pages(pages, dtype, kName);
  if (st != PUREKV_OK) return st;
  PK_REQUIRE(n_q_heads > 0 && n_q_heads % pages->n_kv_heads == 0, PUREKV_ERR_INVALID_ARG,
             "%s: n_q_heads must be a positive multiple of n_kv_heads", kName);
  PK_REQUIRE(pages->head_dim == 64 || pages->head_dim == 128, PUREKV_ERR_UNSUPPORTED, "%s: head_dim must be 64 or 128", kName);
  PK_REQUIRE(max_len >= 0, PUREKV_ERR_INVALID_ARG, "%s: max_len is negative", kName);
  PK_REQUIRE(n_q_heads <= 65535 && pages->n_req <= 65535, PUREKV_ERR_UNSUPPORTED, "%s: too many heads or requests", kName);
  if (pages->n_req == 0) return PUREKV_OK;
  PK_REQUIRE(q && o, PUREKV_ERR_INVALID_ARG, "%s: null pointer", kName);
  const int64_t esz = dtype == PUREKV_BF16 ? 2 : 4;
  PK_REQUIRE(((uintptr_t)q | (uintptr_t)o) % 16 == 0 &&
                 (pages->n_req == 1 || (q_token_stride >= 0 && q_token_stride * esz % 16 == 0)) &&
                 (n_q_heads == 1 || (q_head_stride >= 0 && q_head_stride * esz % 16 == 0)),
             PUREKV_ERR_INVALID_ARG, "%s: pointers and strides must be multiples of 16 bytes", kName);
  DecodePagedArgs a = {};
  a.q = (const uint8_t*)q;
  a.q_tok = q_token_stride * esz;
  a.q_head = q_head_stride * esz;
  a.k_pool = (const uint8_t*)pages->k;
  a.v_pool = (const uint8_t*)pages->v;
  a.k_scale = pages->k_scale;
  a.v_scale = pages->v_scale;
  a.view = view_of(pages);
  a.n_req = pages->n_req;
  a.n_q_heads = n_q_heads;
  a.n_kv_heads = pages->n_kv_heads;
  a.group = n_q_heads / pages->n_kv_heads;
  a.scale_log2 = (softmax_scale > 0.f ? softmax_scale : 1.f / sqrtf((float)pages->head_dim)) * 1.4426950408889634f;
  a.o = o;
  a.lse = lse;
  a.status = status;
  if (!status) {
    const purekv_status s2 = default_status_word(&a.status);
    if (s2 != PUREKV_OK) return s2;
  }
  (void)ws; (void)ws_bytes;
  cudaStream_t sm = (cudaStream_t)stream;
  if (dtype == PUREKV_FP32) return launch_simple<float, float>(a, pages->head_dim, sm);
  return pages->dtype == PUREKV_E4M3 ? launch_simple<__nv_bfloat16, __nv_fp8_e4m3>(a, pages->head_dim, sm)
                                     : launch_simple<__nv_bfloat16, __nv_bfloat16>(a, pages->head_dim, sm);
}

}  // extern "C"
