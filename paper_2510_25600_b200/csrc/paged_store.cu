// purekv_append_paged and purekv_compact_paged: rows of K and V into the pages of a cache.
//
// Append.  A token's heads turn by the same angles.  A thread stands for two 16-byte chunks of one head row, those whose elements
// rotate into one another, and takes them of all the block's tokens: it asks for all of them, the block then forms the tokens' angles
// (64-bit product of position and frequency, reduced to a fraction of a turn, fp32 sine and cosine) in shared memory and looks their
// slots in the pages up, and the thread rotates and stores: q to q_out, k to k_out and its slot, v to its slot.  Bound by HBM for
// prompts (74 000 tokens of 28 / 4 heads, k kept beside: 228 us = 6.35 TB/s), by the chain of position, page and row loads for single tokens.
//
// Compact.  A warp takes a batch of kept rows at a time, whose sources and slots its lanes look up, a row each.  A batch is four stages of a
// ring in shared memory (cp.async; a thread stores what it has loaded, so no thread waits for another): as a stage has been stored, the same
// stage of the next batch is asked for, so that three to four are always on their way -- the rows lie 256 bytes here and there, and it
// takes about 130 KB per SM on their way to keep HBM busy (registers hold half of that: 191 us for 1.3 million rows, now 164 = 5.8 TB/s).
#include <algorithm>

#include <cuda_fp8.h>

#include "common.cuh"
#include "paged.cuh"
#include "paged_args.cuh"

namespace purekv {

constexpr int kAppendThreads = 512;  // at most
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

// Eight values times `inverse`, the reciprocal of their scale, as e4m3: nearest, ties to even, saturating; NaN stays NaN.  (A correction
// of the product to the correctly rounded quotient: 1.3 million rows 171 us with it and 164 without, 128 tokens 3.3 and 3.0.)
__device__ __forceinline__ uint2 to_e4m3(const float (&f)[8], float inverse) {
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float2 a = __fmul2_rn(make_float2(f[4 * i], f[4 * i + 1]), make_float2(inverse, inverse));
    const float2 b = __fmul2_rn(make_float2(f[4 * i + 2], f[4 * i + 3]), make_float2(inverse, inverse));
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(a.y), "f"(a.x));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(b.y), "f"(b.x));
    w[i] = (uint32_t)lo | ((uint32_t)hi << 16);
  }
  return make_uint2(w[0], w[1]);
}

// T: the tokens' type; E8: the pools hold e4m3; TOK: tokens of a block.  grid (tokens / TOK, parts of a token's chunk pairs).  Dynamic
// shared memory: TOK x half (cos, sin).
template <typename T, bool E8, int TOK>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(const __grid_constant__ AppendArgs a) {
  constexpr int E = Chunk<T>::E;
  extern __shared__ float2 s_turn[];
  __shared__ int64_t s_dst[TOK];
  const int32_t tid = threadIdx.x, t0 = blockIdx.x * TOK, n_tok = min(TOK, a.n_tokens - t0);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");

  // this thread's head row, and its two chunks
  const int32_t item = blockIdx.y * blockDim.x + tid, lanes = (int32_t)a.row_lanes.d;
  const int32_t row = (int32_t)a.row_lanes.quotient((uint32_t)item), j = item - row * lanes;
  const bool there = row < a.rows_per_token;
  const int32_t nq = a.q ? a.n_q_heads : 0, nk = a.k ? a.n_kv_heads : 0;
  const bool is_q = row < nq, is_v = row >= nq + nk, turns = a.positions && !is_v;
  const int32_t h = is_q ? row : is_v ? row - nq - nk : row - nq;
  const int64_t tok_stride = is_q ? a.q_tok : is_v ? a.v_tok : a.k_tok;
  const uint8_t* src = (is_q ? a.q + h * a.q_head : is_v ? a.v + h * a.v_head : a.k + h * a.k_head) + t0 * tok_stride;
  const int32_t rc = a.half / E;  // chunks of the first halves (half-split pairs)
  const bool rotates = turns && j < rc;  // (of the row's chunks 2 rc hold what turns; interleaved, its chunks 2 j and 2 j + 1 hold whole pairs)
  const bool split = rotates && !a.interleaved;
  const int32_t ca = split ? j : 2 * j, cb = split ? j + rc : 2 * j + 1;  // (2 rc + 2 (j - rc) = 2 j past the halves)
  uint4 ux[TOK], uy[TOK];
#pragma unroll
  for (int u = 0; u < TOK; ++u)
    if (there && u < n_tok) {
      ux[u] = reinterpret_cast<const uint4*>(src + u * tok_stride)[ca];
      uy[u] = reinterpret_cast<const uint4*>(src + u * tok_stride)[cb];
    }

  if (a.positions)
    for (int32_t i = tid; i < n_tok * a.half; i += blockDim.x) {
      const int32_t tok = i / a.half, pair = i - tok * a.half;
      const int32_t axis = (pair >= a.axis_end[0]) + (pair >= a.axis_end[1]) + (pair >= a.axis_end[2]);
      const double full = (double)a.positions[axis * a.axis_stride + t0 + tok] * a.inv_freq[pair] * 0.15915494309189533577;  // 1 / 2 pi
      // The fraction of a turn as a 32-bit number and what is left of it, which moves sine and cosine by its product with the other: without
      // that, rounding the fraction would move them by up to 1.6 times 2^-24, more than all that follows.
      const double fraction = full - rint(full);
      const float held = (float)fraction, left = (float)(fraction - held) * 6.283185307f;
      float sn, cs;
      sincospif(2.f * held, &sn, &cs);
      s_turn[i] = make_float2(fmaf(-left, sn, cs), fmaf(left, cs, sn));
    }
  if (a.store && tid >= (int32_t)blockDim.x - TOK) {
    const int32_t tok = tid - ((int32_t)blockDim.x - TOK), t = t0 + tok;
    int64_t dst = -1;
    if (tok < n_tok) {
      int32_t r = t, at = -1, len = 0;
      if (a.cu_new) {
        r = request_of(a.cu_new, a.n_req, t);
        const int32_t end = a.cu_new[r + 1];
        if (a.cu_new[r] <= t && t < end) {
          len = a.view.seq_lens[r];
          at = len - (end - t);
        }
      } else {
        len = a.view.seq_lens[r];
        at = len - 1;
      }
      if (len > 0) {
        dst = a.view.row_offset(a.view.table + r * a.view.table_stride, at);
        if (dst < 0) atomicExch(a.status, (int32_t)PUREKV_ERR_BAD_PAGE);
      }
    }
    s_dst[tok] = dst;
  }
  __syncthreads();
  if (!there) return;

  uint8_t* const out = is_q ? a.q_out : is_v ? nullptr : a.k_out;
  const int64_t out_row = (int64_t)a.head_dim * sizeof(T), out_tok = (is_q ? a.n_q_heads : a.n_kv_heads) * out_row;
  uint8_t* const pool = (is_v ? a.v_pool : a.k_pool) + h * a.view.head_stride;
  const bool store = a.store && !is_q;
  const float* const scales = is_v ? a.v_scale : a.k_scale;
  const float inverse = E8 && store && scales ? 1.f / scales[h] : 1.f;
#pragma unroll
  for (int u = 0; u < TOK; ++u) {
    if (u >= n_tok) break;
    float x[E], y[E];
    Chunk<T>::get(ux[u], x);
    Chunk<T>::get(uy[u], y);
    const float2* turn = s_turn + u * a.half;
    if (split) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float2 w = turn[ca * E + e];
        const float xe = x[e], ye = y[e];
        x[e] = xe * w.x - ye * w.y;
        y[e] = ye * w.x + xe * w.y;
      }
      ux[u] = Chunk<T>::put(x);  // (what does not turn stays as it is, a NaN's bits too)
      uy[u] = Chunk<T>::put(y);
    } else if (rotates) {
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        auto rotate = [&](float (&z)[E], int32_t c) {
          const float2 w = turn[(c * E + e) / 2];
          const float ze = z[e], zo = z[e + 1];
          z[e] = ze * w.x - zo * w.y;
          z[e + 1] = zo * w.x + ze * w.y;
        };
        rotate(x, ca);
        rotate(y, cb);
      }
      ux[u] = Chunk<T>::put(x);
      uy[u] = Chunk<T>::put(y);
    }
    if (out) {
      uint4* o4 = reinterpret_cast<uint4*>(out + (t0 + u) * out_tok + h * out_row);
      o4[ca] = ux[u];
      o4[cb] = uy[u];
    }
    if (store && s_dst[u] >= 0) {
      uint8_t* dst = pool + s_dst[u];
      if constexpr (E8) {
        reinterpret_cast<uint2*>(dst)[ca] = to_e4m3(x, inverse);
        reinterpret_cast<uint2*>(dst)[cb] = to_e4m3(y, inverse);
      } else {
        reinterpret_cast<uint4*>(dst)[ca] = ux[u];
        reinterpret_cast<uint4*>(dst)[cb] = uy[u];
      }
    }
  }
}

constexpr int kCompactBlocks = 3;      // of 256 threads per SM
constexpr int kCompactStages = 4;
constexpr int kCompactRequests = 256;  // whose offsets a block keeps in shared memory

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

// CH: 16-byte chunks of a source row, 8, 16 or 32: a stage is 64 / CH rows of K and of V.  0: a.chunks of them, a batch of 16 rows
// without a ring (other head dimensions).
template <int CH>
__host__ __device__ constexpr int compact_rows() { return CH ? 64 / CH * kCompactStages : 16; }
template <typename T, bool E8, int CH>
__global__ void __launch_bounds__(256, kCompactBlocks) compact_paged_kernel(const __grid_constant__ CompactArgs a) {
  constexpr int kRows = compact_rows<CH>(), kPerStage = CH ? 64 / CH : 8;
  extern __shared__ __align__(16) uint8_t s_ring[];  // [warp][stage][2][K, V][lane] of 16 bytes
  __shared__ int32_t s_kept[kCompactRequests + 1], s_first[kCompactRequests + 1], s_lens[kCompactRequests];
  const int32_t lane = threadIdx.x & 31, chunks = CH ? CH : a.chunks;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int32_t *cu_kept = a.cu_kept, *cu_seqlens = a.cu_seqlens, *seq_lens = a.view.seq_lens;
  if (a.n_req <= kCompactRequests) {
    for (int32_t r = threadIdx.x; r <= a.n_req; r += blockDim.x) {
      s_kept[r] = cu_kept[r];
      s_first[r] = cu_seqlens[r];
      if (r < a.n_req) s_lens[r] = seq_lens[r];
    }
    __syncthreads();
    cu_kept = s_kept;
    cu_seqlens = s_first;
    seq_lens = s_lens;
  }
  const int64_t warp = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5, step = (((int64_t)gridDim.x * blockDim.x) >> 5) * kRows;
  const int32_t per_layer = a.k_tot * a.n_kv_heads;
  struct Row {  // dst < 0: nothing to copy
    int64_t src, dst;
    float ks, vs;  // reciprocals of the scales
  };
  // lane's row of the rows from `first` on, which lie in layer `layer` from row `at` on
  auto look = [&](int64_t first, int32_t layer, int32_t at) {
    Row w = {-1, -1, 1.f, 1.f};
    if (lane >= kRows || first + lane >= a.n_rows) return w;
    at += lane;
    while (at >= per_layer) {
      at -= per_layer;
      ++layer;
    }
    const int32_t t = at / a.n_kv_heads, g = at - t * a.n_kv_heads;
    const int32_t i = a.idx[((int64_t)layer * a.n_kv_heads + g) * a.k_tot + t];
    const int32_t r = request_of(cu_kept, a.n_req, t);
    const int32_t begin = cu_kept[r], end = cu_kept[r + 1], from = cu_seqlens[r], len = cu_seqlens[r + 1] - from, rows = seq_lens[r];
    if (t < begin || t >= end || rows <= 0) return w;
    const int64_t dst = a.view.row_offset(a.view.table + r * a.view.table_stride, rows - (end - t)), token = (int64_t)from + i;
    if (dst < 0 || i < 0 || i >= len || from < 0 || token >= a.total_tokens) {
      atomicExch(a.status, (int32_t)PUREKV_ERR_BAD_PAGE);
      return w;
    }
    w.src = layer * a.layer_bytes + (token * a.n_kv_heads + g) * (int64_t)chunks * 16;
    w.dst = dst + layer * a.pool_layer_bytes + g * a.view.head_stride;
    if constexpr (E8) {
      if (a.k_scale) w.ks = 1.f / a.k_scale[layer * a.n_kv_heads + g];
      if (a.v_scale) w.vs = 1.f / a.v_scale[layer * a.n_kv_heads + g];
    }
    return w;
  };
  auto store = [&](uint8_t* k_dst, uint8_t* v_dst, int32_t chunk, uint4 ku, uint4 vu, float ks, float vs) {
    if constexpr (E8) {
      float f[8];
      Chunk<T>::get(ku, f);
      reinterpret_cast<uint2*>(k_dst)[chunk] = to_e4m3(f, ks);
      Chunk<T>::get(vu, f);
      reinterpret_cast<uint2*>(v_dst)[chunk] = to_e4m3(f, vs);
    } else {
      reinterpret_cast<uint4*>(k_dst)[chunk] = ku;
      reinterpret_cast<uint4*>(v_dst)[chunk] = vu;
    }
  };
  // where the warp is: the first of its batch's rows, its layer and its row there; moved on without a division
  int64_t first = warp * kRows;
  int32_t layer = (int32_t)(first / per_layer), at = (int32_t)(first - (int64_t)layer * per_layer);
  const int32_t step_layers = (int32_t)(step / per_layer), step_rows = (int32_t)(step - (int64_t)step_layers * per_layer);
  auto look_on = [&]() {
    layer += step_layers;
    at += step_rows;
    if (at >= per_layer) {
      at -= per_layer;
      ++layer;
    }
    return look(first + step, layer, at);
  };
  Row w = look(first, layer, at);
  if constexpr (CH > 0) {
    uint8_t* const mine = s_ring + (threadIdx.x >> 5) * (kCompactStages * 2048) + lane * 16;
    auto ask = [&](const Row& x, int stage) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int32_t c = lane + 32 * u, row = stage * kPerStage + c / chunks;
        const int64_t from = __shfl_sync(0xffffffffu, x.src, row) + (c % chunks) * 16;
        const uint32_t to = (uint32_t)__cvta_generic_to_shared(mine + stage * 2048 + u * 1024);
        if (__shfl_sync(0xffffffffu, x.dst, row) >= 0) {
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(a.k + from) : "memory");
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + 512), "l"(a.v + from) : "memory");
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int stage = 0; stage < kCompactStages; ++stage) ask(w, stage);
    while (first < a.n_rows) {
      const Row next = look_on();
      __syncwarp();
#pragma unroll
      for (int stage = 0; stage < kCompactStages; ++stage) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kCompactStages - 1) : "memory");
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int32_t c = lane + 32 * u, row = stage * kPerStage + c / chunks;
          const int64_t to = __shfl_sync(0xffffffffu, w.dst, row);
          const float ks = E8 ? __shfl_sync(0xffffffffu, w.ks, row) : 1.f, vs = E8 ? __shfl_sync(0xffffffffu, w.vs, row) : 1.f;
          if (to >= 0) {
            const uint4* held = reinterpret_cast<const uint4*>(mine + stage * 2048 + u * 1024);
            store(a.k_pool + to, a.v_pool + to, c % chunks, held[0], held[32], ks, vs);
          }
        }
        ask(next, stage);
      }
      first += step;
      w = next;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
  } else {
    while (first < a.n_rows) {
      for (int32_t c = lane; c < kRows * chunks; c += 32) {  // (the same trips for every lane: 16 rows of an even number of chunks)
        const int32_t row = c / chunks, chunk = c - row * chunks;
        const int64_t from = __shfl_sync(0xffffffffu, w.src, row) + chunk * 16, to = __shfl_sync(0xffffffffu, w.dst, row);
        const float ks = E8 ? __shfl_sync(0xffffffffu, w.ks, row) : 1.f, vs = E8 ? __shfl_sync(0xffffffffu, w.vs, row) : 1.f;
        if (to >= 0)
          store(a.k_pool + to, a.v_pool + to, chunk, *reinterpret_cast<const uint4*>(a.k + from), *reinterpret_cast<const uint4*>(a.v + from), ks, vs);
      }
      w = look_on();
      first += step;
    }
  }
}

template <typename Kernel, typename Args>
static purekv_status launch_pdl(Kernel kernel, dim3 blocks, unsigned threads, size_t smem, cudaStream_t stream, const Args& a) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = blocks;
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
  const int32_t pairs = a.rows_per_token * (int32_t)a.row_lanes.d, parts = (pairs + kAppendThreads - 1) / kAppendThreads;
  const unsigned threads = (unsigned)(((pairs + parts - 1) / parts + 31) / 32 * 32);
  const size_t turn = (size_t)a.half * sizeof(float2);
  // a token per block while that is not more than the SMs take at once
  if (a.n_tokens <= 148 * 4) return launch_pdl(append_kernel<T, E8, 1>, dim3((unsigned)a.n_tokens, (unsigned)parts), threads, turn, stream, a);
  return launch_pdl(append_kernel<T, E8, 4>, dim3((unsigned)((a.n_tokens + 3) / 4), (unsigned)parts), threads, 4 * turn, stream, a);
}

template <typename T, bool E8, int CH>
static purekv_status launch_compact_as(const CompactArgs& a, cudaStream_t stream) {
  constexpr int64_t kRows = 8 * compact_rows<CH>();  // of a block's warps, a batch each
  auto kernel = compact_paged_kernel<T, E8, CH>;
  static std::atomic<uint64_t> smem_allowed{0};
  const purekv_status st = allow_max_dynamic_smem(kernel, smem_allowed);
  if (st != PUREKV_OK) return st;
  // as many blocks as the SMs hold at once
  return launch_pdl(kernel, dim3((unsigned)std::min<int64_t>((a.n_rows + kRows - 1) / kRows, 148 * kCompactBlocks)), 256,
                    CH ? 8 * kCompactStages * 2048 : 0, stream, a);
}
template <typename T, bool E8>
static purekv_status launch_compact_paged(const CompactArgs& a, cudaStream_t stream) {
  switch (a.chunks) {
    case 8: return launch_compact_as<T, E8, 8>(a, stream);
    case 16: return launch_compact_as<T, E8, 16>(a, stream);
    case 32: return launch_compact_as<T, E8, 32>(a, stream);
    default: return launch_compact_as<T, E8, 0>(a, stream);
  }
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
      const purekv_status st = default_status_word(kWordPaged, &a.status);
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
  PK_REQUIRE((int64_t)k_tot * pages->n_kv_heads <= 1 << 30, PUREKV_ERR_UNSUPPORTED, "%s: too many rows in a layer", kName);
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
    const purekv_status s2 = default_status_word(kWordPaged, &a.status);
    if (s2 != PUREKV_OK) return s2;
  }
  cudaStream_t sm = (cudaStream_t)stream;
  if (dtype == PUREKV_FP32) return launch_compact_paged<float, false>(a, sm);
  return pages->dtype == PUREKV_E4M3 ? launch_compact_paged<__nv_bfloat16, true>(a, sm)
                                     : launch_compact_paged<__nv_bfloat16, false>(a, sm);
}

}  // extern "C"
