// purekv_decode_paged: attention of one new token per request over the pages of a cache.
//
// What it computes, per request r and KV head g with its G query heads: one read of the request's K and V rows serves the whole group.
// Bound by HBM for much work (2 G operations per byte at most), by a chain of latencies for little: lengths, pages, rows, products,
// the join.
//
// Two kernels share everything but the way work reaches a CTA:
//  * even (CLUSTER): grid (C, heads, requests); a cluster of C CTAs owns one (request, KV head) and its parts meet in distributed
//    shared memory.  One launch, no workspace.
//  * balanced: one wave of persistent CTAs; the (KV head, request, tile of keys) triples in that order are cut into equal runs, whatever
//    the lengths are -- they are read on the device -- and a run goes on loading across the ends of requests.  (Head by head, so that
//    CTAs at work on the heads of a request are at the same rows at the same time: those lie side by side in memory.)  A request that a cut
//    goes through leaves partial results in the workspace, which a second, small kernel joins.
//
// Inside a CTA every warp takes TK keys of a tile at a time through a ring of its own in shared memory (cp.async, ST stages), looks the
// pages of its next keys up one step ahead, and keeps (reference maximum, sum, unnormalised output) in registers; the warps' results are
// joined at the end of a request.  Rows that do not exist are not read and weigh nothing.
#include <algorithm>
#include <cmath>

#include <cuda_fp16.h>

#include "cluster.cuh"
#include "common.cuh"
#include "decode.cuh"
#include "paged.cuh"
#include "paged_args.cuh"

namespace purekv {

struct DecodePagedArgs {
  const uint8_t* q;  // strides in bytes
  int64_t q_tok, q_head;
  const uint8_t *k_pool, *v_pool;
  const float *k_scale, *v_scale;
  PagedView view;
  int32_t n_req, n_q_heads, group;
  int32_t blocks;    // of query heads per KV head: 1, or more where a group has more heads than a tile has rows
  int32_t v_heads;   // KV heads x blocks
  float scale_log2;
  void* o;
  float* lse;
  int32_t* status;
  int32_t* chains;   // balanced form: per CTA what it leaves to be joined (ChainRecord)
  float* part;       //   and two slots of partial results per CTA
};

constexpr int kDpClusterMax = 16;

// ---- the three ways of multiplying --------------------------------------------------------------------------------------
// Each has: TK keys per trip, KS and VS bytes between rows of K and V in shared memory, R query heads per tile, `Shared` for what
// the CTA shares; and the state of one warp.  load() starts the loads of a group's queries, ready() puts them to use behind a barrier,
// trip() takes TK keys, finish() leaves the warp's output rows in shared memory and returns (reference, sum) per row.

// On tensor cores a group's heads are the N = 8 columns of m16n8k16 tiles and 16 keys, or 16 of V's columns, their rows: S^T = K Q^T
// and O^T += V^T P^T, so that up to eight heads waste no row of a tile (half the instructions and the accumulators of tiles with heads as
// rows).  mma.sync, not tcgen05: a step is bound by HBM, and a warp that goes from S to P to O in registers needs no other's help.
// A lane holds, for two heads, the logits of two keys; the maxima over the keys are taken across lanes, P is turned into the B operand by
// a transposition of 8 x 8 blocks, and O's rescaling needs no exchange, since its columns are S's.
__device__ __forceinline__ uint32_t dp_transpose(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// NT column tiles (of eight heads) and MT row tiles (of 16 keys): references, sums and weights.  sc[..][0, 1]: key g8, heads 2t and 2t + 1
// of the lane's g8 = lane / 4, t = lane % 4; [2, 3]: key g8 + 8.  Before: logits in log2 units, -inf for keys that are not there; after:
// the weights.  Returns whether O has to be multiplied by alpha.
template <int MT, int NT>
__device__ __forceinline__ bool dp_softmax(float (&sc)[MT][NT][4], float (&m)[NT][2], float (&l)[NT][2], float (&alpha)[NT][2]) {
  bool grew = false;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      float mx = fmaxf(sc[0][nt][x], sc[0][nt][2 + x]);
#pragma unroll
      for (int mt = 1; mt < MT; ++mt) mx = fmaxf(mx, fmaxf(sc[mt][nt][x], sc[mt][nt][2 + x]));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
      const bool up = mx > m[nt][x];
      alpha[nt][x] = up ? dec_ex2(m[nt][x] - mx) : 1.f;
      m[nt][x] = up ? mx : m[nt][x];
      grew |= up;
    }
  grew = __any_sync(0xffffffffu, grew);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const float ref = m[nt][x] == -INFINITY ? 0.f : m[nt][x];
      float sum = 0.f;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        sc[mt][nt][x] = dec_ex2(sc[mt][nt][x] - ref);
        sc[mt][nt][2 + x] = dec_ex2(sc[mt][nt][2 + x] - ref);
        sum += sc[mt][nt][x] + sc[mt][nt][2 + x];
      }
      l[nt][x] = fmaf(l[nt][x], alpha[nt][x], sum);
    }
  return grew;
}
template <int N, int NT>
__device__ __forceinline__ void dp_rescale(float (&o)[N][NT][4], const float (&alpha)[NT][2]) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int x = 0; x < 4; ++x) o[i][nt][x] *= alpha[nt][x & 1];
}
// Sums over the lanes that share heads, and (reference, sum) of each head.
template <int NT>
__device__ __forceinline__ void dp_finish_sums(const float (&m)[NT][2], float (&l)[NT][2], float (*ml)[2]) {
  const int lane = threadIdx.x & 31, g8 = lane >> 2, t = lane & 3;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      l[nt][x] += __shfl_xor_sync(0xffffffffu, l[nt][x], 4);
      l[nt][x] += __shfl_xor_sync(0xffffffffu, l[nt][x], 8);
      l[nt][x] += __shfl_xor_sync(0xffffffffu, l[nt][x], 16);
      if (g8 == 0) {
        ml[8 * nt + 2 * t + x][0] = m[nt][x];
        ml[8 * nt + 2 * t + x][1] = l[nt][x];
      }
    }
}

// bf16 pools.  Rows padded by 16 bytes, so that ldmatrix reads eight of them without bank conflicts.
template <int D_, int NT>
struct Bf16Rows {
  static constexpr int D = D_, TK = 16, RowBytes = D * 2, KS = RowBytes + 16, VS = RowBytes + 16, R = 8 * NT;
  using Out = __nv_bfloat16;
  struct Shared {};
  uint32_t qb[D / 16][NT][2];
  float o[D / 16][NT][4], m[NT][2], l[NT][2], unit;

  __device__ __forceinline__ void load(const DecodePagedArgs& a, Shared&, int32_t r, int32_t g, int32_t h0, int32_t nh) {
    const int lane = threadIdx.x & 31, g8 = lane >> 2, t = lane & 3;
    unit = a.scale_log2;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int32_t h = g8 + 8 * nt;
      const uint32_t* p = reinterpret_cast<const uint32_t*>(a.q + r * a.q_tok + (h0 + (h < nh ? h : 0)) * a.q_head) + t;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        qb[ks][nt][0] = h < nh ? p[ks * 8] : 0u;
        qb[ks][nt][1] = h < nh ? p[ks * 8 + 4] : 0u;
      }
      m[nt][0] = m[nt][1] = -INFINITY;
      l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
      for (int n = 0; n < D / 16; ++n)
#pragma unroll
        for (int x = 0; x < 4; ++x) o[n][nt][x] = 0.f;
    }
  }
  __device__ __forceinline__ void ready(Shared&) {}

  __device__ __forceinline__ void trip(uint32_t st, uint32_t mask, Shared&, int) {
    const int lane = threadIdx.x & 31, g8 = lane >> 2;
    const uint32_t k_at = st + ((lane & 7) + 8 * ((lane >> 3) & 1)) * KS + (lane >> 4) * 16;
    float sc[1][NT][4] = {}, odd[NT][4] = {};  // two chains of products
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      uint32_t k[4];
      dec_ldsm(k_at + ks * 32, k);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) dec_mma(ks & 1 ? odd[nt] : sc[0][nt], k, qb[ks][nt][0], qb[ks][nt][1]);
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int x = 0; x < 4; ++x) sc[0][nt][x] = mask >> (g8 + 8 * (x >> 1)) & 1 ? (sc[0][nt][x] + odd[nt][x]) * unit : -INFINITY;
    float alpha[NT][2];
    if (dp_softmax<1, NT>(sc, m, l, alpha)) dp_rescale(o, alpha);
    uint32_t p[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      p[nt][0] = dp_transpose(dec_pack_bf16(sc[0][nt][0], sc[0][nt][1]));
      p[nt][1] = dp_transpose(dec_pack_bf16(sc[0][nt][2], sc[0][nt][3]));
    }
    const uint32_t v_at = st + TK * KS + ((lane & 7) + 8 * (lane >> 4)) * VS + ((lane >> 3) & 1) * 16;
#pragma unroll
    for (int n = 0; n < D / 16; ++n) {
      uint32_t v[4];
      dec_ldsm_t(v_at + n * 32, v);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) dec_mma(o[n][nt], v, p[nt][0], p[nt][1]);
    }
  }

  __device__ __forceinline__ void finish(float* rows, int ld, float (*ml)[2]) {
    const int lane = threadIdx.x & 31, g8 = lane >> 2, t = lane & 3;
    dp_finish_sums<NT>(m, l, ml);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int n = 0; n < D / 16; ++n)
#pragma unroll
        for (int x = 0; x < 4; ++x) rows[(8 * nt + 2 * t + (x & 1)) * ld + 16 * n + g8 + 8 * (x >> 1)] = o[n][nt][x];
  }
};

// e4m3 pools: every e4m3 number is an fp16 number, so the tiles are fp16 with exact keys and values; the queries' rows are brought into
// fp16's range by a power of two each, and the weights, at most 1, lose less in fp16 than in bf16.  The scale of the keys goes into the
// logits' factor, that of the values into the output.  A lane reads 16 bytes of a key at once: the order in which a dot product takes its
// terms is free, so the queries' fragments are laid out to match.  Of the values, ldmatrix transposes pairs of bytes: a register
// holds two columns of two keys, which go to two tiles, of the even columns and of the odd ones.
template <int D_, int NT>
struct E4m3Rows {
  // Row strides without bank conflicts: for keys eight lanes read 16 bytes of two rows, for values of eight rows.
  static constexpr int D = D_, TK = 32, RowBytes = D, KS = D == 128 ? 144 : 64, VS = D + 16, R = 8 * NT, CL = D / 64;
  using Out = __nv_bfloat16;
  struct Shared {};
  uint32_t qb[D / 16][NT][2];
  float o[D / 16][NT][4], m[NT][2], l[NT][2], unit[NT][2];

  static __device__ __forceinline__ uint32_t half2_of(uint16_t pair) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(pair));
    return r;
  }
  static __device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  }
  static __device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
  }

  __device__ __forceinline__ void load(const DecodePagedArgs& a, Shared&, int32_t r, int32_t g, int32_t h0, int32_t nh) {
    const int lane = threadIdx.x & 31, g8 = lane >> 2, t = lane & 3;
    const float per_key = a.scale_log2 * (a.k_scale ? a.k_scale[g] : 1.f);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int32_t h = g8 + 8 * nt;
      uint32_t w[8 * CL];  // q[16 CL t .. + 16 CL) of head h
      if (h < nh) {
        const uint4* p = reinterpret_cast<const uint4*>(a.q + r * a.q_tok + (h0 + h) * a.q_head) + 2 * CL * t;
#pragma unroll
        for (int i = 0; i < 2 * CL; ++i) {
          const uint4 u = p[i];
          w[4 * i] = u.x; w[4 * i + 1] = u.y; w[4 * i + 2] = u.z; w[4 * i + 3] = u.w;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8 * CL; ++i) w[i] = 0u;
      }
      uint32_t top = 0u;  // the largest exponent of the head's elements
#pragma unroll
      for (int i = 0; i < 8 * CL; ++i) top = max(top, max(w[i] >> 7 & 0xffu, w[i] >> 23 & 0xffu));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      // elements below 2^15, exact down to 2^-28 of the largest; a head below 2^-112 has logits of nothing and stays as it is
      const bool as_is = top < 15u;
      const float down = as_is ? 1.f : __uint_as_float((268u - top) << 23);
      const float up = per_key * (as_is ? 1.f : __uint_as_float((top - 14u) << 23));
      unit[nt][0] = __shfl_sync(0xffffffffu, up, 8 * t);  // of the heads whose logits the lane holds
      unit[nt][1] = __shfl_sync(0xffffffffu, up, 8 * t + 4);
#pragma unroll
      for (int i = 0; i < 8 * CL; ++i)  // word i: elements 2i, 2i + 1 = k slots of step i / 2, the lower or the upper pair
        qb[i / 2][nt][i & 1] = pack_half(__uint_as_float(w[i] << 16) * down, __uint_as_float(w[i] & 0xffff0000u) * down);
      m[nt][0] = m[nt][1] = -INFINITY;
      l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
      for (int n = 0; n < D / 16; ++n)
#pragma unroll
        for (int x = 0; x < 4; ++x) o[n][nt][x] = 0.f;
    }
  }
  __device__ __forceinline__ void ready(Shared&) {}

  __device__ __forceinline__ void trip(uint32_t st, uint32_t mask, Shared&, int) {
    const int lane = threadIdx.x & 31, g8 = lane >> 2, t = lane & 3;
    float sc[2][NT][4] = {};
#pragma unroll
    for (int j = 0; j < CL; ++j)
#pragma unroll
      for (int mt = 0; mt < 2; ++mt) {
        uint32_t w[2][4];  // keys g8 and g8 + 8
#pragma unroll
        for (int x = 0; x < 2; ++x)
          asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                       : "=r"(w[x][0]), "=r"(w[x][1]), "=r"(w[x][2]), "=r"(w[x][3])
                       : "r"(st + (16 * mt + 8 * x + g8) * KS + (CL * t + j) * 16) : "memory");
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const uint32_t a0 = half2_of((uint16_t)w[0][s]), a2 = half2_of((uint16_t)(w[0][s] >> 16));
          const uint32_t a1 = half2_of((uint16_t)w[1][s]), a3 = half2_of((uint16_t)(w[1][s] >> 16));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) mma(sc[mt][nt], a0, a1, a2, a3, qb[4 * j + s][nt][0], qb[4 * j + s][nt][1]);
        }
      }
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int x = 0; x < 4; ++x) sc[mt][nt][x] = mask >> (16 * mt + g8 + 8 * (x >> 1)) & 1 ? sc[mt][nt][x] * unit[nt][x & 1] : -INFINITY;
    float alpha[NT][2];
    if (dp_softmax<2, NT>(sc, m, l, alpha)) dp_rescale(o, alpha);
    const uint32_t v_at = st + TK * KS + ((lane & 7) + 8 * ((lane >> 3) & 1)) * VS + (lane >> 4) * 16;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      uint32_t p[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        p[nt][0] = dp_transpose(pack_half(sc[mt][nt][0], sc[mt][nt][1]));
        p[nt][1] = dp_transpose(pack_half(sc[mt][nt][2], sc[mt][nt][3]));
      }
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {  // 32 columns: b[0] and b[1] keys 2t, 2t + 1 and 2t + 8, 2t + 9 of the first 16, b[2] and b[3] of the others
        uint32_t b[4], lo[4], hi[4];
        dec_ldsm_t(v_at + mt * 16 * VS + c * 32, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          lo[i] = half2_of((uint16_t)b[i]);
          hi[i] = half2_of((uint16_t)(b[i] >> 16));
        }
        uint32_t even[4], odd[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          even[i] = __byte_perm(lo[i], hi[i], 0x5410);
          odd[i] = __byte_perm(lo[i], hi[i], 0x7632);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          mma(o[2 * c][nt], even[0], even[2], even[1], even[3], p[nt][0], p[nt][1]);
          mma(o[2 * c + 1][nt], odd[0], odd[2], odd[1], odd[3], p[nt][0], p[nt][1]);
        }
      }
    }
  }

  __device__ __forceinline__ void finish(float* rows, int ld, float (*ml)[2]) {
    const int lane = threadIdx.x & 31, g8 = lane >> 2, t = lane & 3;
    dp_finish_sums<NT>(m, l, ml);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          *reinterpret_cast<float2*>(rows + (8 * nt + 2 * t + (x & 1)) * ld + 32 * c + 16 * (x >> 1) + 2 * g8) = make_float2(o[2 * c][nt][x], o[2 * c + 1][nt][x]);
  }
};

// fp32 pools: CUDA cores (tf32 would not keep fp32's accuracy).  For the logits a lane takes 32 elements of one key and all heads; for
// the output D / 32 columns of every key.
template <int D_, int GP>
struct Fp32Rows {
  static constexpr int D = D_, TK = D == 64 ? 16 : 8, RowBytes = D * 4, KS = RowBytes + 16, VS = RowBytes + 16, R = GP, E = D / 32;
  using Out = float;
  struct Shared {
    float q[GP][D];
    float p[8][TK][GP];  // per warp
  };
  static constexpr int kQPerThread = (GP * D + 127) / 128;  // at least 128 threads
  float staged[kQPerThread];
  float o[GP][E], m[GP], l[GP];

  __device__ __forceinline__ void load(const DecodePagedArgs& a, Shared&, int32_t r, int32_t g, int32_t h0, int32_t nh) {
#pragma unroll
    for (int i = 0; i < kQPerThread; ++i) {
      const int32_t x = threadIdx.x + i * (int32_t)blockDim.x, h = x / D;
      staged[i] = h < nh && x < GP * D ? reinterpret_cast<const float*>(a.q + r * a.q_tok + (h0 + h) * a.q_head)[x % D] * a.scale_log2 : 0.f;
    }
#pragma unroll
    for (int h = 0; h < GP; ++h) {
#pragma unroll
      for (int e = 0; e < E; ++e) o[h][e] = 0.f;
      m[h] = -INFINITY;
      l[h] = 0.f;
    }
  }
  __device__ __forceinline__ void ready(Shared& s) {
#pragma unroll
    for (int i = 0; i < kQPerThread; ++i) {
      const int32_t x = threadIdx.x + i * (int32_t)blockDim.x;
      if (x < GP * D) (&s.q[0][0])[x] = staged[i];
    }
  }

  __device__ __forceinline__ void trip(uint32_t st, uint32_t mask, Shared& s, int warp) {
    const int lane = threadIdx.x & 31, key = lane % TK, part = lane / TK;
    float dot[GP];
#pragma unroll
    for (int h = 0; h < GP; ++h) dot[h] = 0.f;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      float4 k;
      asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                   : "=f"(k.x), "=f"(k.y), "=f"(k.z), "=f"(k.w) : "r"(st + key * KS + part * 128 + c * 16) : "memory");
#pragma unroll
      for (int h = 0; h < GP; ++h) {
        const float4 q = *reinterpret_cast<const float4*>(&s.q[h][part * 32 + c * 4]);
        dot[h] = fmaf(q.x, k.x, dot[h]); dot[h] = fmaf(q.y, k.y, dot[h]);
        dot[h] = fmaf(q.z, k.z, dot[h]); dot[h] = fmaf(q.w, k.w, dot[h]);
      }
    }
#pragma unroll
    for (int h = 0; h < GP; ++h) {
#pragma unroll
      for (int x = TK; x < 32; x *= 2) dot[h] += __shfl_xor_sync(0xffffffffu, dot[h], x);
      const float z = mask >> key & 1 ? dot[h] : -INFINITY;
      float mx = z;
#pragma unroll
      for (int x = 1; x < TK; x *= 2) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, x));
      if (mx > m[h]) {  // the same for the warp
        const float alpha = dec_ex2(m[h] - mx);
        l[h] *= alpha;
#pragma unroll
        for (int e = 0; e < E; ++e) o[h][e] *= alpha;
        m[h] = mx;
      }
      const float p = dec_ex2(z - (m[h] == -INFINITY ? 0.f : m[h]));
      if (part == 0) {
        l[h] += p;
        s.p[warp][key][h] = p;
      }
    }
    __syncwarp();
    const uint32_t v_at = st + TK * KS + lane * (4 * E);
#pragma unroll
    for (int j = 0; j < TK; ++j) {
      float v[E];
      if constexpr (E == 2)
        asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v[0]), "=f"(v[1]) : "r"(v_at + j * VS) : "memory");
      else
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(v_at + j * VS) : "memory");
#pragma unroll
      for (int h = 0; h < GP; ++h) {
        const float p = s.p[warp][j][h];
#pragma unroll
        for (int e = 0; e < E; ++e) o[h][e] = fmaf(p, v[e], o[h][e]);
      }
    }
  }

  __device__ __forceinline__ void finish(float* rows, int ld, float (*ml)[2]) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int h = 0; h < GP; ++h) {
#pragma unroll
      for (int x = 16; x >= 1; x /= 2) l[h] += __shfl_xor_sync(0xffffffffu, l[h], x);
      if (lane == 0) {
        ml[h][0] = m[h];
        ml[h][1] = l[h];
      }
#pragma unroll
      for (int e = 0; e < E; ++e) rows[h * ld + lane * E + e] = o[h][e];
    }
  }
};

// ---- the kernel ---------------------------------------------------------------------------------------------------------
template <class E>
__host__ __device__ constexpr int dp_stage_bytes() { return E::TK * (E::KS + E::VS); }
// A warp's output rows start eight banks apart; they are laid over the stage that the warp used last.
template <class E>
__host__ __device__ constexpr int dp_ld() { return E::D + 8; }
template <class E, int ST>
__host__ __device__ constexpr int dp_warp_bytes() {
  static_assert(ST == 1 || E::R * dp_ld<E>() * 4 <= dp_stage_bytes<E>(), "a warp's rows fit a stage");
  return ST * dp_stage_bytes<E>() > E::R * dp_ld<E>() * 4 ? ST * dp_stage_bytes<E>() : E::R * dp_ld<E>() * 4;
}
// Partial results of one slot: [R][D] unnormalised outputs, [R] references, [R] sums
template <class E>
__host__ __device__ constexpr int64_t dp_part_floats() { return (int64_t)E::R * (E::D + 2); }

// What a CTA of the balanced form leaves: the request and virtual head whose first part it is (in its second slot), and how many
// parts there are (the others in the first slots of the CTAs that follow); 0: nothing.
struct ChainRecord {
  int32_t r, vh, parts, pad;
};

// Row of a request: weight of a warp's, a CTA's or a part's result.  Nothing summed (sum 0) weighs nothing; a NaN sum stays NaN.
__device__ __forceinline__ float dp_weight(float m, float l, float ref) { return l == 0.f ? 0.f : dec_ex2(m - ref); }
__device__ __forceinline__ float dp_seen(float m, float l) { return l == 0.f ? -INFINITY : m; }
__device__ __forceinline__ float dp_finite(float m) { return m == -INFINITY ? 0.f : m; }

template <typename T>
__device__ __forceinline__ void dp_store4(T* dst, float4 v);
template <>
__device__ __forceinline__ void dp_store4(__nv_bfloat16* dst, float4 v) {
  *reinterpret_cast<uint2*>(dst) = make_uint2(dec_pack_bf16(v.x, v.y), dec_pack_bf16(v.z, v.w));
}
template <>
__device__ __forceinline__ void dp_store4(float* dst, float4 v) { *reinterpret_cast<float4*>(dst) = v; }

template <class E, int W, int ST, bool CLUSTER, bool WHOLE, int OCC>
__global__ void __launch_bounds__(W * 32, OCC) decode_paged_kernel(const __grid_constant__ DecodePagedArgs a) {
  constexpr int D = E::D, R = E::R, TK = E::TK, TILE = W * TK, kThreads = W * 32, kStage = dp_stage_bytes<E>(), LD = dp_ld<E>();
  constexpr int kWarpBytes = dp_warp_bytes<E, ST>();
  using Out = typename E::Out;
  extern __shared__ __align__(16) uint8_t dp_smem[];
  __shared__ float s_ml[W][R][2];
  __shared__ uint32_t s_mask[W][ST];
  __shared__ __align__(16) typename E::Shared s_e;
  __shared__ __align__(16) float s_part[CLUSTER ? R * D : 1];          // what the cluster's CTAs send this one: [source][head][its columns]
  __shared__ __align__(8) float s_pml[CLUSTER ? kDpClusterMax : 1][R][2];  // every CTA's (reference, sum) per head
  __shared__ int64_t s_scan[W + 1];
  __shared__ int32_t s_req, s_tile;

  const int32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int32_t C = CLUSTER ? (int32_t)gridDim.x : 1, rank = CLUSTER ? (int32_t)blockIdx.x : 0;
  const int32_t capacity = min(a.view.capacity(), INT32_MAX - 65536);  // (row numbers past the last tile stay in 32 bits)
  // The next kernel of the stream may be placed meanwhile; what the previous one wrote is complete and visible behind the wait.
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (CLUSTER && C > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");  // "started": awaited before the sends
  asm volatile("griddepcontrol.wait;" ::: "memory");

  auto rows_of = [&](int32_t r) {
    const int32_t len = a.view.seq_lens[r];
    return min(max(len, 0), capacity);
  };
  // the next request that has rows, or the next head's first one (there is one, or the lengths have changed under the kernel: then
  // whatever request comes last)
  auto next_request = [&](int32_t& i, int32_t& v, int32_t& rows) {
    do {
      if (i + 1 == a.n_req) {
        if (v + 1 == a.v_heads) break;
        i = -1;
        ++v;
      }
      rows = rows_of(++i);
    } while (rows == 0);
  };
  auto tiles_of = [&](int32_t n) { return (n + TILE - 1) / TILE; };

  // This CTA's tiles: `total` of them, from tile `tile` of (request r, virtual head vh) on.
  int32_t r, vh, tile, n;
  int64_t total, all = 0, runs = 0, first = 0;
  if constexpr (CLUSTER) {
    r = blockIdx.z;
    vh = blockIdx.y;
    n = rows_of(r);
    if (a.view.seq_lens[r] > capacity && tid == 0) atomicExch(a.status, (int32_t)PUREKV_ERR_BAD_PAGE);
    const int32_t share = (tiles_of(n) + C - 1) / C;
    tile = min(rank * share, tiles_of(n));
    total = min(share, tiles_of(n) - tile);
  } else {
    const int32_t ctas = gridDim.x, c = blockIdx.x;
    // all tiles, and requests without rows: their outputs are zero
    int64_t sum = 0;
    for (int32_t i = tid; i < a.n_req; i += kThreads) sum += tiles_of(rows_of(i));
#pragma unroll
    for (int x = 16; x >= 1; x /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, x);
    if (lane == 0) s_scan[warp] = sum;
    __syncthreads();
    int64_t per_head = 0;
    for (int w = 0; w < W; ++w) per_head += s_scan[w];
    all = per_head * a.v_heads;
    runs = min((int64_t)ctas, all);  // (each of a tile or more)
    first = c < runs ? all * c / runs : all;
    total = c < runs ? all * (c + 1) / runs - first : 0;
    vh = total > 0 ? (int32_t)(first / per_head) : 0;
    const int64_t of_head = first - vh * per_head;
    // the request in which tile `of_head` lies: running sums over the requests, kThreads at a time
    int64_t before = 0;
    for (int32_t i0 = 0; i0 < a.n_req && total > 0; i0 += kThreads) {
      const int32_t i = i0 + tid;
      const int64_t mine = i < a.n_req ? (int64_t)tiles_of(rows_of(i)) : 0;
      int64_t upto = mine;
#pragma unroll
      for (int x = 1; x < 32; x *= 2) {
        const int64_t y = __shfl_up_sync(0xffffffffu, upto, x);
        if (lane >= x) upto += y;
      }
      __syncthreads();
      if (lane == 31) s_scan[warp] = upto;
      __syncthreads();
      int64_t chunk = 0;
      for (int w = 0; w < W; ++w) {
        if (w < warp) upto += s_scan[w];
        chunk += s_scan[w];
      }
      upto += before;
      if (upto - mine <= of_head && of_head < upto) {
        s_req = i;
        s_tile = (int32_t)(of_head - (upto - mine));
      }
      before += chunk;
      if (before > of_head) break;
    }
    __syncthreads();
    r = total > 0 ? s_req : 0;
    n = total > 0 ? rows_of(r) : 0;
    tile = total > 0 ? s_tile : 0;
    for (int32_t i = c; i < a.n_req; i += ctas) {
      const int32_t len = a.view.seq_lens[i];
      if (len > capacity && tid == 0) atomicExch(a.status, (int32_t)PUREKV_ERR_BAD_PAGE);
      if (rows_of(i) > 0) continue;
      for (int32_t x = tid; x < a.n_q_heads * (D / 4); x += kThreads)
        dp_store4(reinterpret_cast<Out*>(a.o) + (int64_t)i * a.n_q_heads * D + 4 * x, make_float4(0.f, 0.f, 0.f, 0.f));
      if (a.lse)
        for (int32_t x = tid; x < a.n_q_heads; x += kThreads) a.lse[(int64_t)i * a.n_q_heads + x] = -INFINITY;
    }
    if (tid == 0) reinterpret_cast<ChainRecord*>(a.chains)[c].parts = 0;
  }

  // ---- loads.  The cursor (fr, fvh, ftile, fn) runs ahead of the products, over the ends of requests.
  int32_t fr = r, fvh = vh, ftile = tile, fn = n;
  int64_t f_left = total;
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(dp_smem) + (uint32_t)warp * kWarpBytes;
  // The page of a row, its slot there and its KV head.  WHOLE (a page holds whole trips): of the trip's first row, `there` of whose
  // rows are wanted; otherwise of row `lane` of the trip, `there` 1 if it is wanted.
  struct Look {
    int32_t page, slot, g, there;
  };
  auto look = [&]() {
    Look k = {-1, 0, 0, 0};
    if (f_left > 0) {
      const int32_t row = ftile * TILE + warp * TK + (WHOLE ? 0 : lane);
      k.there = WHOLE ? min(max(fn - row, 0), TK) : lane < TK && row < fn;
      if (k.there > 0) {
        const uint32_t p = a.view.page_size.quotient((uint32_t)row);
        k.slot = row - (int32_t)(p * a.view.page_size.d);
        k.page = a.view.table[(int64_t)fr * a.view.table_stride + p];
      }
      k.g = a.blocks == 1 ? fvh : fvh / a.blocks;
      --f_left;
      if (++ftile == tiles_of(fn)) {
        ftile = 0;
        if (!CLUSTER && f_left > 0) next_request(fr, fvh, fn);
      }
    }
    return k;
  };
  constexpr int CPR = E::RowBytes / 16, RPI = 32 / CPR;  // 16-byte chunks of a row, rows of a warp's request
  auto copy = [](uint32_t dst, const uint8_t* src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); };
  auto copy_or_zero = [](uint32_t dst, const uint8_t* src, bool there) {  // zeros for rows that do not exist: nothing is read
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16u : 0u) : "memory");
  };
  auto fetch = [&](int32_t stage, const Look& k) {
    const uint32_t dst = ring + (uint32_t)stage * kStage + (lane / CPR) * E::KS + (lane % CPR) * 16;
    const uint32_t dst_v = ring + (uint32_t)stage * kStage + TK * E::KS + (lane / CPR) * E::VS + (lane % CPR) * 16;
    const int64_t off = k.there > 0 ? a.view.offset(k.page, (uint32_t)k.slot) : -1;
    uint32_t mask;
    if constexpr (WHOLE) {
      mask = off < 0 ? 0u : k.there == 32 ? 0xffffffffu : (1u << k.there) - 1u;
      if (k.there > 0 && off < 0 && lane == 0) atomicExch(a.status, (int32_t)PUREKV_ERR_BAD_PAGE);
      if (mask) {
        const int64_t from = off + (int64_t)k.g * a.view.head_stride + (lane / CPR) * a.view.token_stride + (lane % CPR) * 16;
        const uint8_t *kp = a.k_pool + from, *vp = a.v_pool + from;
        const int64_t step = RPI * a.view.token_stride;
        if (k.there == TK) {
#pragma unroll
          for (int i = 0; i < TK / RPI; ++i, kp += step, vp += step) {
            copy(dst + i * RPI * E::KS, kp);
            copy(dst_v + i * RPI * E::VS, vp);
          }
        } else {
#pragma unroll
          for (int i = 0; i < TK / RPI; ++i, kp += step, vp += step) {
            const bool there = i * RPI + lane / CPR < k.there;
            copy_or_zero(dst + i * RPI * E::KS, there ? kp : a.k_pool, there);
            copy_or_zero(dst_v + i * RPI * E::VS, there ? vp : a.v_pool, there);
          }
        }
      }
    } else {
      mask = __ballot_sync(0xffffffffu, off >= 0);
      if (__ballot_sync(0xffffffffu, k.there > 0) != mask && lane == 0) atomicExch(a.status, (int32_t)PUREKV_ERR_BAD_PAGE);
      if (mask) {
        const int64_t mine = off + (int64_t)k.g * a.view.head_stride;
#pragma unroll
        for (int i = 0; i < TK / RPI; ++i) {
          const int row = i * RPI + lane / CPR;
          const int64_t from = __shfl_sync(0xffffffffu, mine, row) + (lane % CPR) * 16;
          const bool there = mask >> row & 1;
          copy_or_zero(dst + i * RPI * E::KS, a.k_pool + (there ? from : 0), there);
          copy_or_zero(dst_v + i * RPI * E::VS, a.v_pool + (there ? from : 0), there);
        }
      }
    }
    if (lane == 0) s_mask[warp][stage] = mask;
    asm volatile("cp.async.commit_group;" ::: "memory");  // (empty past the end: the group count stays in step)
  };
  Look next;
  {
    Look ahead[ST > 1 ? ST - 1 : 1];
#pragma unroll
    for (int s = 0; s < (ST > 1 ? ST - 1 : 1); ++s) ahead[s] = look();
#pragma unroll
    for (int s = 0; s < (ST > 1 ? ST - 1 : 1); ++s) fetch(s, ahead[s]);
    next = look();
  }

  E e;
  auto heads_at = [&](int32_t v, int32_t& g, int32_t& h0, int32_t& nh) {
    g = a.blocks == 1 ? v : v / a.blocks;
    const int32_t b = v - g * a.blocks;
    h0 = g * a.group + b * R;
    nh = min(R, a.group - b * R);
  };
  int32_t g, h0, nh;
  heads_at(vh, g, h0, nh);
  e.load(a, s_e, r, g, h0, nh);
  e.ready(s_e);
  __syncthreads();

  int32_t stage = 0;
  bool from_start = tile == 0;  // whether this CTA has the request's first tile
  for (int64_t i = 0;; ++i) {
    bool end_of_request = true, end_of_run = true;
    if (i < total) {
      if constexpr (ST > 1) {
        fetch(stage == 0 ? ST - 1 : stage - 1, next);
        next = look();
      }
      asm volatile("cp.async.wait_group %0;" ::"n"(ST - 1) : "memory");
      __syncwarp();
      const uint32_t mask = s_mask[warp][stage];
      if (mask) e.trip(ring + (uint32_t)stage * kStage, mask, s_e, warp);
      __syncwarp();  // every lane has read the stage before the next fetch overwrites it
      end_of_request = ++tile == tiles_of(n);
      end_of_run = i + 1 == total;
      if constexpr (ST == 1) {
        if (!end_of_run && !end_of_request) {
          fetch(0, next);
          next = look();
        }
      }
      if (!end_of_request && !end_of_run) {
        stage = stage + 1 == ST ? 0 : stage + 1;
        continue;
      }
    } else if (!CLUSTER) {
      break;  // a run without tiles
    }

    // ---- the warps' results side by side, each over the stage that its warp has just used up
    e.finish(reinterpret_cast<float*>(dp_smem + warp * kWarpBytes + stage * kStage), LD, s_ml[warp]);
    const int32_t r_done = r, h0_done = h0, nh_done = nh, g_done = g, vh_done = vh, n_done = n;
    if (!CLUSTER && !end_of_run) {  // the next request's queries, while this one's results are joined
      next_request(r, vh, n);
      tile = 0;
      heads_at(vh, g, h0, nh);
      e.load(a, s_e, r, g, h0, nh);
    }
    __syncthreads();
    if constexpr (CLUSTER) {
      if (C > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    }
    const float vs = a.v_scale ? a.v_scale[g_done] : 1.f;
    const bool whole = CLUSTER ? C == 1 : from_start && end_of_request;
    const int32_t cols = D / C;  // columns of every head that each CTA of the cluster finishes
    float* slot = nullptr;
    if constexpr (!CLUSTER) slot = a.part + (2 * (int64_t)blockIdx.x + (from_start ? 1 : 0)) * dp_part_floats<E>();
    for (int32_t x = tid; x < nh_done * (D / 4); x += kThreads) {  // one thread per four columns of a head
      const int32_t h = x / (D / 4), col = 4 * (x % (D / 4));
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < W; ++w) top = fmaxf(top, dp_seen(s_ml[w][h][0], s_ml[w][h][1]));
      const float ref = dp_finite(top);
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
      float l = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float wgt = dp_weight(s_ml[w][h][0], s_ml[w][h][1], ref);
        const float4 v4 = *reinterpret_cast<const float4*>(dp_smem + w * kWarpBytes + stage * kStage + (h * LD + col) * 4);
        acc.x = fmaf(wgt, v4.x, acc.x); acc.y = fmaf(wgt, v4.y, acc.y); acc.z = fmaf(wgt, v4.z, acc.z); acc.w = fmaf(wgt, v4.w, acc.w);
        l = fmaf(wgt, s_ml[w][h][1], l);
      }
      if (whole) {
        const int64_t hq = (int64_t)r_done * a.n_q_heads + h0_done + h;
        const float inv = n_done > 0 ? vs / l : 0.f;
        dp_store4(reinterpret_cast<Out*>(a.o) + hq * D + col, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
        if (col == 0 && a.lse) a.lse[hq] = n_done > 0 ? (ref + log2f(l)) * 0.6931471805599453f : -INFINITY;
      } else if constexpr (CLUSTER) {
        const uint32_t to = (uint32_t)(col / cols);
        asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(dec_mapa(s_part + (rank * nh_done + h) * cols + col % cols, to)),
                     "f"(acc.x), "f"(acc.y), "f"(acc.z), "f"(acc.w) : "memory");
        if (col % cols == 0)
          asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(dec_mapa(s_pml[rank][h], to)), "f"(ref), "f"(l) : "memory");
      } else {
        *reinterpret_cast<float4*>(slot + h * D + col) = acc;
        if (col == 0) {
          slot[R * D + h] = ref;
          slot[R * D + R + h] = l;
        }
      }
    }
    if constexpr (CLUSTER) {
      break;
    } else {
      if (from_start && !end_of_request && tid == 0) {  // the first of several parts: the one that holds the request's last tile is
        const int64_t last = first + i + (tiles_of(n_done) - tile);  // tile `last` of all, in run (last + 1) runs - 1 over all
        const int32_t until = (int32_t)(((last + 1) * runs - 1) / all);
        reinterpret_cast<ChainRecord*>(a.chains)[blockIdx.x] = {r_done, vh_done, until - (int32_t)blockIdx.x + 1, 0};
      }
      if (end_of_run) break;
      e.ready(s_e);
      __syncthreads();
      from_start = true;
      stage = stage + 1 == ST ? 0 : stage + 1;
    }
  }

  if constexpr (CLUSTER) {
    if (C == 1) return;
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    // four threads per output value, each over every fourth CTA's share (nh * cols * 4 is a multiple of 16: whole quarters)
    const int32_t cols = D / C, part = tid & 3;
    const float vs = a.v_scale ? a.v_scale[g] : 1.f;
    for (int32_t x0 = 0; x0 < nh * cols * 4; x0 += kThreads) {
      const int32_t x = x0 + tid, y = min(x, nh * cols * 4 - 1), h = (y >> 2) / cols, c = (y >> 2) % cols;
      float top = -INFINITY;
#pragma unroll
      for (int k = 0; k < kDpClusterMax / 4; ++k) {
        const int32_t j = part + 4 * k;
        if (j < C) top = fmaxf(top, dp_seen(s_pml[j][h][0], s_pml[j][h][1]));
      }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const float ref = dp_finite(top);
      float acc = 0.f, l = 0.f;
#pragma unroll
      for (int k = 0; k < kDpClusterMax / 4; ++k) {
        const int32_t j = part + 4 * k;
        if (j < C) {
          const float wgt = dp_weight(s_pml[j][h][0], s_pml[j][h][1], ref);
          acc = fmaf(wgt, s_part[(j * nh + h) * cols + c], acc);
          l = fmaf(wgt, s_pml[j][h][1], l);
        }
      }
      acc += __shfl_xor_sync(0xffffffffu, acc, 1);
      l += __shfl_xor_sync(0xffffffffu, l, 1);
      acc += __shfl_xor_sync(0xffffffffu, acc, 2);
      l += __shfl_xor_sync(0xffffffffu, l, 2);
      if (part == 0 && x < nh * cols * 4) {
        const int64_t hq = (int64_t)r * a.n_q_heads + h0 + h;
        reinterpret_cast<Out*>(a.o)[hq * D + rank * cols + c] = (Out)(n > 0 ? acc * (vs / l) : 0.f);
        if (rank == 0 && c == 0 && a.lse) a.lse[hq] = n > 0 ? (ref + log2f(l)) * 0.6931471805599453f : -INFINITY;
      }
    }
  }
}

// Joins the parts of the requests that cuts went through: grid (half of the balanced form's CTAs, heads of a tile), a block looks
// after two CTAs' chains.  Each D / 4 threads take eight parts at a time, all loads of which are asked for before the first is used, and
// run a softmax of their own over them; the groups meet in shared memory.
template <class E>
__global__ void __launch_bounds__(256) decode_paged_join_kernel(const __grid_constant__ DecodePagedArgs a) {
  constexpr int D = E::D, R = E::R, kGroup = D / 4, kGroups = 256 / kGroup, kAtOnce = 8;
  __shared__ float s_ml[kGroups][2];
  __shared__ __align__(16) float4 s_acc[kGroups][kGroup];
  const int32_t h = blockIdx.y, grp = threadIdx.x / kGroup, c = threadIdx.x % kGroup;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const ChainRecord both[2] = {reinterpret_cast<const ChainRecord*>(a.chains)[2 * blockIdx.x], reinterpret_cast<const ChainRecord*>(a.chains)[2 * blockIdx.x + 1]};
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const ChainRecord chain = both[which];
    const int32_t g = a.blocks == 1 ? chain.vh : chain.vh / a.blocks, b = chain.vh - g * a.blocks;
    if (chain.parts == 0 || h >= min(R, a.group - b * R)) continue;  // the same for the block
    const int64_t cta = 2 * blockIdx.x + which;
    float ref = -INFINITY, l = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int32_t i0 = grp; i0 < chain.parts; i0 += kAtOnce * kGroups) {
      float mi[kAtOnce], li[kAtOnce];
      float4 v[kAtOnce];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const int32_t i = i0 + k * kGroups;
        mi[k] = -INFINITY;
        li[k] = 0.f;
        v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i < chain.parts) {
          const float* slot = a.part + (2 * (cta + i) + (i == 0 ? 1 : 0)) * dp_part_floats<E>();
          mi[k] = slot[R * D + h];
          li[k] = slot[R * D + R + h];
          v[k] = *reinterpret_cast<const float4*>(slot + h * D + 4 * c);
        }
      }
      float top = ref;
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) top = fmaxf(top, dp_seen(mi[k], li[k]));
      const float alpha = dp_weight(ref, l, dp_finite(top));
      ref = top;
      l *= alpha;
      acc.x *= alpha; acc.y *= alpha; acc.z *= alpha; acc.w *= alpha;
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const float w = dp_weight(mi[k], li[k], dp_finite(ref));
        l = fmaf(w, li[k], l);
        acc.x = fmaf(w, v[k].x, acc.x); acc.y = fmaf(w, v[k].y, acc.y); acc.z = fmaf(w, v[k].z, acc.z); acc.w = fmaf(w, v[k].w, acc.w);
      }
    }
    if (c == 0) {
      s_ml[grp][0] = ref;
      s_ml[grp][1] = l;
    }
    s_acc[grp][c] = acc;
    __syncthreads();
    if (grp == 0) {
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < kGroups; ++i) top = fmaxf(top, dp_seen(s_ml[i][0], s_ml[i][1]));
      const float to = dp_finite(top);
      acc = make_float4(0.f, 0.f, 0.f, 0.f);
      l = 0.f;
#pragma unroll
      for (int i = 0; i < kGroups; ++i) {
        const float w = dp_weight(s_ml[i][0], s_ml[i][1], to);
        const float4 v = s_acc[i][c];
        l = fmaf(w, s_ml[i][1], l);
        acc.x = fmaf(w, v.x, acc.x); acc.y = fmaf(w, v.y, acc.y); acc.z = fmaf(w, v.z, acc.z); acc.w = fmaf(w, v.w, acc.w);
      }
      const int64_t hq = (int64_t)chain.r * a.n_q_heads + g * a.group + b * R + h;
      const float inv = (a.v_scale ? a.v_scale[g] : 1.f) / l;
      dp_store4(reinterpret_cast<typename E::Out*>(a.o) + hq * D + 4 * c, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
      if (c == 0 && a.lse) a.lse[hq] = (to + log2f(l)) * 0.6931471805599453f;
    }
    __syncthreads();
  }
}

// ---- launching ----------------------------------------------------------------------------------------------------------
struct DpLaunch {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  DpLaunch(dim3 grid, int threads, size_t smem, cudaStream_t stream) {
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // see griddepcontrol in the kernels
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
  }
};

template <class E, int W, int ST, bool WHOLE, int OCC>
static purekv_status launch_even(const DecodePagedArgs& a, int32_t cl, cudaStream_t stream) {
  auto kernel = decode_paged_kernel<E, W, ST, true, WHOLE, OCC>;
  static std::atomic<uint64_t> smem_allowed{0}, wide_allowed{0};
  const purekv_status st = allow_max_dynamic_smem(kernel, smem_allowed);
  if (st != PUREKV_OK) return st;
  if (cl > 8) {  // clusters of more than eight CTAs are opt-in, once per device
    int dev = -1;
    PK_CUDA(cudaGetDevice(&dev));
    if (!(wide_allowed.load(std::memory_order_acquire) & (1ull << dev))) {
      PK_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
      wide_allowed.fetch_or(1ull << dev, std::memory_order_release);
    }
  }
  DpLaunch l(dim3(1), W * 32, (size_t)W * dp_warp_bytes<E, ST>(), stream);
  l.cfg.numAttrs = 2;
  auto set_size = [&](int32_t c) {
    l.cfg.gridDim = dim3((unsigned)c, (unsigned)a.v_heads, (unsigned)a.n_req);
    l.attr[1].val.clusterDim.x = (unsigned)c;
  };
  set_size(cluster_that_fits(cl, [&](int32_t c) {
    set_size(c);
    return clusters_at_once(kernel, l.cfg);
  }));
  PK_CUDA(cudaLaunchKernelEx(&l.cfg, kernel, a));
  return PUREKV_OK;
}

template <class E, int W, int ST, bool WHOLE, int OCC>
static purekv_status launch_balanced(const DecodePagedArgs& a, int32_t ctas, cudaStream_t stream) {
  auto kernel = decode_paged_kernel<E, W, ST, false, WHOLE, OCC>;
  static std::atomic<uint64_t> smem_allowed{0};
  const purekv_status st = allow_max_dynamic_smem(kernel, smem_allowed);
  if (st != PUREKV_OK) return st;
  DpLaunch l(dim3((unsigned)ctas), W * 32, (size_t)W * dp_warp_bytes<E, ST>(), stream);
  PK_CUDA(cudaLaunchKernelEx(&l.cfg, kernel, a));
  DpLaunch j(dim3((unsigned)(ctas / 2), (unsigned)std::min(E::R, a.group)), 256, 0, stream);
  PK_CUDA(cudaLaunchKernelEx(&j.cfg, decode_paged_join_kernel<E>, a));
  return PUREKV_OK;
}

constexpr int32_t kDpCtas = 296;  // CTAs of the balanced form: two per SM

// How a call is launched: C CTAs per (request, head) in a cluster, or 0 for the balanced form.
struct DpForm {
  int32_t cluster;
};
static DpForm dp_form(int64_t base, int64_t bound) {
  int32_t c = 1;
  while (c < kDpClusterMax && bound > 128 * c && base * 2 * c <= (c < 4 ? 128 : 64)) c *= 2;
  return {bound <= 128 * (int64_t)c * 2 ? c : 0};
}

template <class E, int ST8, bool WHOLE>
static purekv_status launch_form(const DecodePagedArgs& a, const DpForm& f, cudaStream_t stream) {
  if (f.cluster) return launch_even<E, 8, ST8, WHOLE, 1>(a, f.cluster, stream);
  return launch_balanced<E, 4, ST8, WHOLE, 2>(a, kDpCtas, stream);
}
template <class E, int ST8>
static purekv_status launch_rows(const DecodePagedArgs& a, const DpForm& f, cudaStream_t stream) {
  return a.view.page_size.d % E::TK == 0 ? launch_form<E, ST8, true>(a, f, stream) : launch_form<E, ST8, false>(a, f, stream);
}

static int32_t dp_rows(int32_t group, purekv_dtype dtype) { return dtype == PUREKV_FP32 ? (group <= 2 ? 2 : 8) : group <= 8 ? 8 : 16; }

static int64_t dp_ws(const DpForm& f, int32_t group, int32_t head_dim, purekv_dtype dtype) {
  if (f.cluster) return 0;
  return 256 + kDpCtas * (int64_t)sizeof(ChainRecord) + 2 * kDpCtas * (int64_t)dp_rows(group, dtype) * (head_dim + 2) * 4;
}

}  // namespace purekv

using namespace purekv;

extern "C" {

size_t purekv_decode_paged_ws_bytes(int32_t n_req, int32_t max_len, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                    purekv_dtype dtype) {
  if (n_req <= 0 || n_q_heads <= 0 || n_kv_heads <= 0 || n_q_heads % n_kv_heads || head_dim <= 0) return 0;
  const int32_t group = n_q_heads / n_kv_heads, rows = dp_rows(group, dtype), blocks = (group + rows - 1) / rows;
  return (size_t)dp_ws(dp_form((int64_t)n_req * n_kv_heads * blocks, max_len > 0 ? max_len : INT32_MAX), group, head_dim, dtype);
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
  a.group = n_q_heads / pages->n_kv_heads;
  const int32_t rows = dp_rows(a.group, dtype);
  a.blocks = (a.group + rows - 1) / rows;
  a.v_heads = pages->n_kv_heads * a.blocks;
  a.scale_log2 = (softmax_scale > 0.f ? softmax_scale : 1.f / sqrtf((float)pages->head_dim)) * 1.4426950408889634f;
  a.o = o;
  a.lse = lse;
  a.status = status;
  const DpForm form = dp_form((int64_t)a.n_req * a.v_heads, max_len > 0 ? max_len : INT32_MAX);
  if (!form.cluster) {
    PK_REQUIRE(ws && ws_bytes >= (size_t)dp_ws(form, a.group, pages->head_dim, dtype), PUREKV_ERR_WORKSPACE,
               "%s: workspace of %zu bytes is too small", kName, ws_bytes);
    a.chains = (int32_t*)(((uintptr_t)ws + 255) & ~(uintptr_t)255);
    a.part = (float*)(a.chains + kDpCtas * (sizeof(ChainRecord) / 4));
  }
  if (!status) {
    const purekv_status s2 = default_status_word(&a.status);
    if (s2 != PUREKV_OK) return s2;
  }
  cudaStream_t sm = (cudaStream_t)stream;
  const bool wide = pages->head_dim == 128;
  if (dtype == PUREKV_FP32) {
    if (rows == 2) return wide ? launch_rows<Fp32Rows<128, 2>, 3>(a, form, sm) : launch_rows<Fp32Rows<64, 2>, 3>(a, form, sm);
    return wide ? launch_rows<Fp32Rows<128, 8>, 3>(a, form, sm) : launch_rows<Fp32Rows<64, 8>, 3>(a, form, sm);
  }
  if (pages->dtype == PUREKV_E4M3) {
    if (rows == 8) return wide ? launch_rows<E4m3Rows<128, 1>, 3>(a, form, sm) : launch_rows<E4m3Rows<64, 1>, 5>(a, form, sm);
    return wide ? launch_rows<E4m3Rows<128, 2>, 2>(a, form, sm) : launch_rows<E4m3Rows<64, 2>, 5>(a, form, sm);
  }
  if (rows == 8) return wide ? launch_rows<Bf16Rows<128, 1>, 3>(a, form, sm) : launch_rows<Bf16Rows<64, 1>, 5>(a, form, sm);
  return wide ? launch_rows<Bf16Rows<128, 2>, 3>(a, form, sm) : launch_rows<Bf16Rows<64, 2>, 5>(a, form, sm);
}

}  // extern "C"
