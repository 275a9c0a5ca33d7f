// purekv_append_paged and purekv_compact_paged: rows of K and V into the pages of a cache.
//
// Append.  A token's heads turn by the same angles: a block takes a few tokens, forms their angles once (64-bit product of position
// and frequency, reduced to a fraction of a turn, fp32 sine and cosine) in shared memory, and its threads go over the tokens' head
// rows, 2 x 16 bytes at a time: the two chunks whose elements rotate into one another.  The K rows go to k_out and to their slot in the
// pages, q to q_out.  Bound by HBM for prompts, by the chain of position, page and row loads for single tokens.
//
// Compact.  A warp takes 16 kept rows: each lane looks one row's source and slot up, and the warp then copies row by row.
#include <algorithm>

#include <cuda_fp8.h>

#include "common.cuh"
#include "paged.cuh"
#include "paged_args.cuh"

namespace purekv {

constexpr int kAppendThreads = 256;
constexpr int kMaxAxes = 4;

struct AppendArgs {
  const uint8_t *q, *k, *v;  // strides in bytes
  int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head;
  uint8_t *q_out, *k_out;
  uint8_t *k_pool, *v_pool;
  bool store;  // into the pools; false: a rotation alone
  const float *k_scale, *v_scale;
  PagedView view;
  const int32_t* positions;  // null: no rotation
  int64_t axis_stride;
  const double* inv_freq;
  int32_t half;               // pairs that turn
  int32_t axis_end[kMaxAxes];  // pairs of the axes up to and including this one
  int32_t interleaved;
  const int32_t* cu_new;
  int32_t n_req, n_tokens, n_q_heads, n_kv_heads, head_dim;
  int32_t rows_per_token;  // q's, k's and v's head rows
  FastDiv row_lanes;       // threads of a head row: one for each two chunks
  FastDiv rows_div;
  int32_t* status;
};

// 16 bytes of the input as fp32, and back
template <typename T>
struct Chunk;
template <>
struct Chunk<__nv_bfloat16> {
  static constexpr int E = 8;
  static __device__ __forceinline__ void get(uint4 u, float (&f)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 put(const float (&f)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(f[2 * i + 1]), "f"(f[2 * i]));
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <>
struct Chunk<float> {
  static constexpr int E = 4;
  static __device__ __forceinline__ void get(uint4 u, float (&f)[4]) {
    f[0] = __uint_as_float(u.x); f[1] = __uint_as_float(u.y); f[2] = __uint_as_float(u.z); f[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ uint4 put(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
};

// Eight values as e4m3, nearest, ties to even, saturating; NaN stays NaN.  The quotient is the correctly rounded one: a product with
// the reciprocal would fall on the other side of a rounding boundary now and then.
__device__ __forceinline__ uint2 to_e4m3(const float (&f)[8], float scale) {
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(__fdiv_rn(f[4 * i + 1], scale)), "f"(__fdiv_rn(f[4 * i], scale)));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(__fdiv_rn(f[4 * i + 3], scale)), "f"(__fdiv_rn(f[4 * i + 2], scale)));
    w[i] = (uint32_t)lo | ((uint32_t)hi << 16);
  }
  return make_uint2(w[0], w[1]);
}

// T: the tokens' type; E8: the pools hold e4m3; TOK: tokens of a block.  Dynamic shared memory: TOK x half (cos, sin).
template <typename T, bool E8, int TOK>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(const AppendArgs a) {
  constexpr int E = Chunk<T>::E;
  extern __shared__ float2 s_turn[];
  __shared__ int64_t s_dst[TOK];
  const int32_t tid = threadIdx.x, t0 = blockIdx.x * TOK, n_tok = min(TOK, a.n_tokens - t0);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");

  if (a.positions)
    for (int32_t i = tid; i < n_tok * a.half; i += kAppendThreads) {
      const int32_t tok = i / a.half, pair = i - tok * a.half;
      int32_t axis = 0;
      while (axis < kMaxAxes - 1 && pair >= a.axis_end[axis]) ++axis;
      const double turns = (double)a.positions[axis * a.axis_stride + t0 + tok] * a.inv_freq[pair] * 0.15915494309189533577;  // 1 / 2 pi
      float sn, cs;
      sincospif(2.f * (float)(turns - rint(turns)), &sn, &cs);
      s_turn[i] = make_float2(cs, sn);
    }
  if (a.store && tid >= kAppendThreads - TOK) {
    const int32_t tok = tid - (kAppendThreads - TOK), t = t0 + tok;
    int64_t dst = -1;
    if (tok < n_tok) {
      int32_t r = t, row = -1, len = 0;
      if (a.cu_new) {
        r = request_of(a.cu_new, a.n_req, t);
        const int32_t end = a.cu_new[r + 1];
        if (a.cu_new[r] <= t && t < end) {
          len = a.view.seq_lens[r];
          row = len - (end - t);
        }
      } else {
        len = a.view.seq_lens[r];
        row = len - 1;
      }
      if (len > 0) {
        dst = a.view.row_offset(a.view.table + r * a.view.table_stride, row);
        if (dst < 0) atomicExch(a.status, (int32_t)PUREKV_ERR_BAD_PAGE);
      }
    }
    s_dst[tok] = dst;
  }
  __syncthreads();

  const int32_t lanes = (int32_t)a.row_lanes.d, n_items = n_tok * a.rows_per_token * lanes;
  const int32_t rc = a.half / E;  // chunks of the first halves (half-split pairs)
  for (int32_t item = tid; item < n_items; item += kAppendThreads) {
    const int32_t row = (int32_t)a.row_lanes.quotient((uint32_t)item), j = item - row * lanes;
    const int32_t tok = (int32_t)a.rows_div.quotient((uint32_t)row);
    int32_t h = row - tok * a.rows_per_token;
    const int64_t t = t0 + tok;
    const int32_t nq = a.q ? a.n_q_heads : 0, nk = a.k ? a.n_kv_heads : 0;
    const bool is_q = h < nq, is_v = h >= nq + nk;
    const uint8_t* src;
    if (is_q) {
      src = a.q + t * a.q_tok + h * a.q_head;
    } else if (!is_v) {
      h -= nq;
      src = a.k + t * a.k_tok + h * a.k_head;
    } else {
      h -= nq + nk;
      src = a.v + t * a.v_tok + h * a.v_head;
    }
    const bool split = !a.interleaved && !is_v && a.positions && j < rc;
    const int32_t ca = split ? j : 2 * j, cb = split ? j + rc : 2 * j + 1;  // (2 rc + 2 (j - rc) = 2 j past the halves)
    float x[E], y[E];
    Chunk<T>::get(reinterpret_cast<const uint4*>(src)[ca], x);
    Chunk<T>::get(reinterpret_cast<const uint4*>(src)[cb], y);
    if (split) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float2 w = s_turn[tok * a.half + ca * E + e];
        const float xe = x[e], ye = y[e];
        x[e] = xe * w.x - ye * w.y;
        y[e] = ye * w.x + xe * w.y;
      }
    } else if (a.interleaved && !is_v && a.positions) {
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        auto turn = [&](float (&z)[E], int32_t c) {
          const int32_t pair = (c * E + e) / 2;
          if (pair >= a.half) return;
          const float2 w = s_turn[tok * a.half + pair];
          const float ze = z[e], zo = z[e + 1];
          z[e] = ze * w.x - zo * w.y;
          z[e + 1] = zo * w.x + ze * w.y;
        };
        turn(x, ca);
        turn(y, cb);
      }
    }
    if (!is_v) {
      uint8_t* out = is_q ? a.q_out : a.k_out;
      if (out) {
        uint4* o4 = reinterpret_cast<uint4*>(out + (t * (is_q ? a.n_q_heads : a.n_kv_heads) + h) * a.head_dim * (int64_t)sizeof(T));
        o4[ca] = Chunk<T>::put(x);
        o4[cb] = Chunk<T>::put(y);
      }
    }
    if (!is_q && a.store && s_dst[tok] >= 0) {
      uint8_t* dst = (is_v ? a.v_pool : a.k_pool) + s_dst[tok] + h * a.view.head_stride;
      if constexpr (E8) {
        const float* sc = is_v ? a.v_scale : a.k_scale;
        const float scale = sc ? sc[h] : 1.f;
        reinterpret_cast<uint2*>(dst)[ca] = to_e4m3(x, scale);
        reinterpret_cast<uint2*>(dst)[cb] = to_e4m3(y, scale);
      } else {
        reinterpret_cast<uint4*>(dst)[ca] = Chunk<T>::put(x);
        reinterpret_cast<uint4*>(dst)[cb] = Chunk<T>::put(y);
      }
    }
  }
}

constexpr int kCompactRows = 16;  // rows of a warp

struct CompactArgs {
  const uint8_t *k, *v;
  int64_t layer_bytes;  // between layers of k and v
  uint8_t *k_pool, *v_pool;
  int64_t pool_layer_bytes;
  const float *k_scale, *v_scale;
  PagedView view;
  const int32_t *idx, *cu_seqlens, *cu_kept;
  int64_t total_tokens, n_rows;  // rows of all layers and heads
  int32_t n_req, k_tot, n_kv_heads, chunks;  // 16-byte chunks of a source row
  int32_t* status;
};

template <typename T, bool E8>
__global__ void __launch_bounds__(256) compact_paged_kernel(const CompactArgs a) {
  const int32_t lane = threadIdx.x & 31;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int64_t warp = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5, n_warps = ((int64_t)gridDim.x * blockDim.x) >> 5;
  const int64_t per_layer = (int64_t)a.k_tot * a.n_kv_heads;
  for (int64_t first = warp * kCompactRows; first < a.n_rows; first += n_warps * kCompactRows) {
    int64_t src = -1, dst = -1;
    int32_t scale_at = 0;
    if (lane < kCompactRows && first + lane < a.n_rows) {
      const int64_t x = first + lane;
      const int32_t layer = (int32_t)(x / per_layer), in_layer = (int32_t)(x - layer * per_layer);
      const int32_t t = in_layer / a.n_kv_heads, g = in_layer - t * a.n_kv_heads;
      const int32_t r = request_of(a.cu_kept, a.n_req, t);
      const int32_t end = a.cu_kept[r + 1], at = a.cu_seqlens[r], len = a.cu_seqlens[r + 1] - at;
      const int32_t i = a.idx[((int64_t)layer * a.n_kv_heads + g) * a.k_tot + t], rows = a.view.seq_lens[r];
      if (a.cu_kept[r] <= t && t < end && rows > 0) {
        dst = a.view.row_offset(a.view.table + r * a.view.table_stride, rows - (end - t));
        const int64_t token = (int64_t)at + i;
        if (dst < 0 || i < 0 || i >= len || at < 0 || token >= a.total_tokens) {
          dst = -1;
          atomicExch(a.status, (int32_t)PUREKV_ERR_BAD_PAGE);
        } else {
          src = layer * a.layer_bytes + (token * a.n_kv_heads + g) * (int64_t)a.chunks * 16;
          dst += layer * a.pool_layer_bytes + g * a.view.head_stride;
          scale_at = layer * a.n_kv_heads + g;
        }
      }
    }
    for (int32_t c = lane; c < kCompactRows * a.chunks; c += 32) {
      const int32_t row = c / a.chunks, chunk = c - row * a.chunks;
      const int64_t s = __shfl_sync(0xffffffffu, src, row), d = __shfl_sync(0xffffffffu, dst, row);
      const int32_t sc = __shfl_sync(0xffffffffu, scale_at, row);
      if (d < 0) continue;
      const uint4 ku = reinterpret_cast<const uint4*>(a.k + s)[chunk], vu = reinterpret_cast<const uint4*>(a.v + s)[chunk];
      if constexpr (E8) {
        float f[8];
        Chunk<T>::get(ku, f);
        reinterpret_cast<uint2*>(a.k_pool + d)[chunk] = to_e4m3(f, a.k_scale ? a.k_scale[sc] : 1.f);
        Chunk<T>::get(vu, f);
        reinterpret_cast<uint2*>(a.v_pool + d)[chunk] = to_e4m3(f, a.v_scale ? a.v_scale[sc] : 1.f);
      } else {
        reinterpret_cast<uint4*>(a.k_pool + d)[chunk] = ku;
        reinterpret_cast<uint4*>(a.v_pool + d)[chunk] = vu;
      }
    }
  }
}

template <typename Kernel, typename Args>
static purekv_status launch_pdl(Kernel kernel, unsigned blocks, unsigned threads, size_t smem, cudaStream_t stream, const Args& a) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // see griddepcontrol in the kernels
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  PK_CUDA(cudaLaunchKernelEx(&cfg, kernel, a));
  return PUREKV_OK;
}

template <typename T, bool E8>
static purekv_status launch_append(const AppendArgs& a, cudaStream_t stream) {
  const size_t turn = (size_t)a.half * sizeof(float2);
  if (a.n_tokens <= 148 * 8) return launch_pdl(append_kernel<T, E8, 1>, (unsigned)a.n_tokens, kAppendThreads, turn, stream, a);
  return launch_pdl(append_kernel<T, E8, 4>, (unsigned)((a.n_tokens + 3) / 4), kAppendThreads, 4 * turn, stream, a);
}

}  // namespace purekv

using namespace purekv;

extern "C" {

purekv_status purekv_append_paged(const void* q, int64_t q_token_stride, int64_t q_head_stride, const void* k, int64_t k_token_stride,
                                  int64_t k_head_stride, const void* v, int64_t v_token_stride, int64_t v_head_stride, void* q_out,
                                  void* k_out, const purekv_pages* pages, const purekv_rope* rope, const int32_t* cu_new,
                                  int32_t n_tokens, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, purekv_dtype dtype,
                                  int32_t* status, void* stream) {
  static const char* const kName = "purekv_append_paged";
  PK_REQUIRE(dtype == PUREKV_BF16 || dtype == PUREKV_FP32, PUREKV_ERR_INVALID_ARG, "%s: q, k and v are bf16 or fp32", kName);
  PK_REQUIRE(n_tokens >= 0 && n_q_heads >= 0 && n_kv_heads >= 0 && head_dim > 0, PUREKV_ERR_INVALID_ARG, "%s: bad sizes", kName);
  PK_REQUIRE(head_dim % 16 == 0 && head_dim <= 512 && n_q_heads <= 65536 && n_kv_heads <= 65536, PUREKV_ERR_UNSUPPORTED,
             "%s: head_dim must be a multiple of 16, at most 512, and heads at most 65536", kName);
  AppendArgs a = {};
  const int64_t esz = dtype == PUREKV_BF16 ? 2 : 4;
  if (pages) {
    const purekv_status st = check_pages(pages, dtype, kName);
    if (st != PUREKV_OK) return st;
    PK_REQUIRE(pages->n_kv_heads == n_kv_heads && pages->head_dim == head_dim, PUREKV_ERR_INVALID_ARG,
               "%s: the pages have other heads than k and v", kName);
    PK_REQUIRE(cu_new || pages->n_req == n_tokens, PUREKV_ERR_INVALID_ARG, "%s: without cu_new there is one token per request", kName);
  }
  if (n_tokens == 0) return PUREKV_OK;
  PK_REQUIRE((q != nullptr) == (q_out != nullptr), PUREKV_ERR_INVALID_ARG, "%s: q and q_out come together", kName);
  PK_REQUIRE((k != nullptr) == (pages != nullptr || k_out != nullptr) && (v != nullptr) == (pages != nullptr), PUREKV_ERR_INVALID_ARG,
             "%s: k comes with pages or k_out, v with pages", kName);
  PK_REQUIRE((!q || n_q_heads > 0) && (!k || n_kv_heads > 0), PUREKV_ERR_INVALID_ARG, "%s: no heads", kName);
  auto rows = [&](const void* p, int64_t tok, int64_t head, int32_t heads) {
    return !p || ((uintptr_t)p % 16 == 0 && (n_tokens == 1 || (tok >= 0 && tok * esz % 16 == 0)) && (heads == 1 || (head >= 0 && head * esz % 16 == 0)));
  };
  PK_REQUIRE(rows(q, q_token_stride, q_head_stride, n_q_heads) && rows(k, k_token_stride, k_head_stride, n_kv_heads) &&
                 rows(v, v_token_stride, v_head_stride, n_kv_heads) && ((uintptr_t)q_out | (uintptr_t)k_out) % 16 == 0,
             PUREKV_ERR_INVALID_ARG, "%s: pointers and strides must be multiples of 16 bytes", kName);
  if (rope) {
    PK_REQUIRE(rope->positions && rope->inv_freq && (uintptr_t)rope->inv_freq % 8 == 0, PUREKV_ERR_INVALID_ARG, "%s: null positions or frequencies", kName);
    PK_REQUIRE(rope->rotary_dim > 0 && rope->rotary_dim <= head_dim && rope->rotary_dim % 16 == 0, PUREKV_ERR_UNSUPPORTED,
               "%s: rotary_dim must be a multiple of 16, at most head_dim", kName);
    PK_REQUIRE(rope->n_axes >= 1 && rope->n_axes <= kMaxAxes, PUREKV_ERR_INVALID_ARG, "%s: 1 to %d axes", kName, kMaxAxes);
    int64_t sum = 0;
    for (int32_t i = 0; i < rope->n_axes; ++i) {
      PK_REQUIRE(rope->sections[i] >= 0, PUREKV_ERR_INVALID_ARG, "%s: a negative section", kName);
      sum += rope->sections[i];
      a.axis_end[i] = (int32_t)std::min<int64_t>(sum, 1 << 20);
    }
    PK_REQUIRE(sum == rope->rotary_dim / 2, PUREKV_ERR_INVALID_ARG, "%s: the sections must sum to rotary_dim / 2", kName);
    for (int32_t i = rope->n_axes; i < kMaxAxes; ++i) a.axis_end[i] = 1 << 20;
    PK_REQUIRE(rope->n_axes == 1 || rope->axis_stride >= n_tokens, PUREKV_ERR_INVALID_ARG, "%s: the axes' positions overlap", kName);
    a.positions = rope->positions;
    a.axis_stride = rope->axis_stride;
    a.inv_freq = rope->inv_freq;
    a.half = rope->rotary_dim / 2;
    a.interleaved = rope->interleaved != 0;
  }
  if (!q && !k) return PUREKV_OK;
  if (pages) {
    a.k_pool = (uint8_t*)pages->k;
    a.v_pool = (uint8_t*)pages->v;
    a.k_scale = pages->k_scale;
    a.v_scale = pages->v_scale;
    a.view = view_of(pages);
    a.n_req = pages->n_req;
    a.store = pages->n_req > 0;
    a.status = status;
    if (!status) {
      const purekv_status st = default_status_word(&a.status);
      if (st != PUREKV_OK) return st;
    }
  }
  a.q = (const uint8_t*)q;
  a.k = (const uint8_t*)k;
  a.v = (const uint8_t*)v;
  a.q_tok = q_token_stride * esz; a.q_head = q_head_stride * esz;
  a.k_tok = k_token_stride * esz; a.k_head = k_head_stride * esz;
  a.v_tok = v_token_stride * esz; a.v_head = v_head_stride * esz;
  a.q_out = (uint8_t*)q_out;
  a.k_out = (uint8_t*)k_out;
  a.cu_new = cu_new;
  a.n_tokens = n_tokens;
  a.n_q_heads = n_q_heads;
  a.n_kv_heads = n_kv_heads;
  a.head_dim = head_dim;
  a.rows_per_token = (q ? n_q_heads : 0) + (k ? n_kv_heads : 0) + (v ? n_kv_heads : 0);
  a.row_lanes = FastDiv::of((int32_t)(head_dim * esz / 32));
  a.rows_div = FastDiv::of(a.rows_per_token);
  cudaStream_t sm = (cudaStream_t)stream;
  if (dtype == PUREKV_FP32) return launch_append<float, false>(a, sm);
  return pages && pages->dtype == PUREKV_E4M3 ? launch_append<__nv_bfloat16, true>(a, sm) : launch_append<__nv_bfloat16, false>(a, sm);
}

purekv_status purekv_compact_paged(const void* k, const void* v, int64_t layer_stride, int32_t n_layers, const int32_t* idx,
                                   const int32_t* cu_seqlens, int64_t total_tokens, const int32_t* cu_kept, int32_t k_tot,
                                   purekv_dtype dtype, const purekv_pages* pages, int32_t* status, void* stream) {
  static const char* const kName = "purekv_compact_paged";
  PK_REQUIRE(dtype == PUREKV_BF16 || dtype == PUREKV_FP32, PUREKV_ERR_INVALID_ARG, "%s: k and v are bf16 or fp32", kName);
  PK_REQUIRE(pages, PUREKV_ERR_INVALID_ARG, "%s: no pages", kName);
  const purekv_status st = check_pages(pages, dtype, kName);
  if (st != PUREKV_OK) return st;
  PK_REQUIRE(n_layers >= 0 && k_tot >= 0 && total_tokens >= 0 && total_tokens <= INT32_MAX, PUREKV_ERR_INVALID_ARG, "%s: bad sizes", kName);
  if (n_layers == 0 || k_tot == 0 || pages->n_req == 0) return PUREKV_OK;
  PK_REQUIRE(k && v && idx && cu_seqlens && cu_kept, PUREKV_ERR_INVALID_ARG, "%s: null pointer", kName);
  PK_REQUIRE((int64_t)k_tot * pages->n_kv_heads <= INT32_MAX, PUREKV_ERR_UNSUPPORTED, "%s: too many rows in a layer", kName);
  PK_REQUIRE(pages->head_dim % 16 == 0 && pages->head_dim <= 512, PUREKV_ERR_UNSUPPORTED,
             "%s: head_dim must be a multiple of 16, at most 512", kName);
  const int64_t esz = dtype == PUREKV_BF16 ? 2 : 4, out_esz = bytes_of(pages->dtype);
  PK_REQUIRE(((uintptr_t)k | (uintptr_t)v) % 16 == 0 && (n_layers == 1 || layer_stride * esz % 16 == 0), PUREKV_ERR_INVALID_ARG,
             "%s: pointers and strides must be multiples of 16 bytes", kName);
  PK_REQUIRE(n_layers == 1 || layer_stride >= total_tokens * pages->n_kv_heads * pages->head_dim, PUREKV_ERR_INVALID_ARG,
             "%s: layer_stride smaller than one layer", kName);
  PK_REQUIRE(n_layers == 1 || (pages->layer_stride > 0 && pages->layer_stride * out_esz % 16 == 0), PUREKV_ERR_INVALID_ARG,
             "%s: the pools' layer_stride must be positive and a multiple of 16 bytes", kName);
  CompactArgs a = {};
  a.k = (const uint8_t*)k;
  a.v = (const uint8_t*)v;
  a.layer_bytes = layer_stride * esz;
  a.k_pool = (uint8_t*)pages->k;
  a.v_pool = (uint8_t*)pages->v;
  a.pool_layer_bytes = pages->layer_stride * out_esz;
  a.k_scale = pages->k_scale;
  a.v_scale = pages->v_scale;
  a.view = view_of(pages);
  a.idx = idx;
  a.cu_seqlens = cu_seqlens;
  a.cu_kept = cu_kept;
  a.total_tokens = total_tokens;
  a.n_rows = (int64_t)k_tot * pages->n_kv_heads * n_layers;
  a.n_req = pages->n_req;
  a.k_tot = k_tot;
  a.n_kv_heads = pages->n_kv_heads;
  a.chunks = (int32_t)(pages->head_dim * esz / 16);
  a.status = status;
  if (!status) {
    const purekv_status s2 = default_status_word(&a.status);
    if (s2 != PUREKV_OK) return s2;
  }
  const int64_t blocks = (a.n_rows + 8 * kCompactRows - 1) / (8 * kCompactRows);
  const unsigned grid = (unsigned)std::min<int64_t>(blocks, 148 * 8);
  cudaStream_t sm = (cudaStream_t)stream;
  if (dtype == PUREKV_FP32) return launch_pdl(compact_paged_kernel<float, false>, grid, 256, 0, sm, a);
  return pages->dtype == PUREKV_E4M3 ? launch_pdl(compact_paged_kernel<__nv_bfloat16, true>, grid, 256, 0, sm, a)
                                     : launch_pdl(compact_paged_kernel<__nv_bfloat16, false>, grid, 256, 0, sm, a);
}

}  // extern "C"
