// purekv_decode_paged: attention of one new token per request over the pages of a cache.
//
// What it computes, per request r and KV head g with its G query heads: one read of the request's K and V rows serves the whole group.
// Bound by HBM for much work (2 G operations per byte at most), by a chain of latencies for little: lengths, pages, rows, products,
// the join.
//
// Two kernels share everything but the way work reaches a CTA:
//  * even (CLUSTER): grid (C, heads, requests); a cluster of C CTAs owns one (request, KV head) and its parts meet in distributed
//    shared memory.  One launch, no workspace.
//  * balanced: one wave of persistent CTAs; the (request, KV head, tile of keys) triples in that order are cut into equal runs, whatever
//    the lengths are -- they are read on the device -- and a run goes on loading across the ends of requests.  A request that a cut
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

// bf16 pools: mma.sync, the group's heads are the rows of m16n8k16 tiles.  (M = 16 is far below a tcgen05 tile's 128 rows, and the
// step is bound by HBM.)  Rows padded by 16 bytes, so that ldmatrix reads eight of them without bank conflicts.
template <int D_, int RW>
struct Bf16Rows {
  static constexpr int D = D_, TK = 16, RowBytes = D * 2, KS = RowBytes + 16, VS = RowBytes + 16, R = 8 * RW;
  using Out = __nv_bfloat16;
  struct Shared {};
  uint32_t qa[D / 16][4];
  float o[D / 8][4], m[2], l[2], unit;

  __device__ __forceinline__ void load(const DecodePagedArgs& a, Shared&, int32_t r, int32_t g, int32_t h0, int32_t nh, int32_t) {
    const int lane = threadIdx.x & 31, g8 = lane >> 2, t = lane & 3;
    unit = a.scale_log2;
#pragma unroll
    for (int rw = 0; rw < RW; ++rw) {
      const int32_t h = g8 + 8 * rw;
      const uint32_t* p = reinterpret_cast<const uint32_t*>(a.q + r * a.q_tok + (h0 + (h < nh ? h : 0)) * a.q_head) + t;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        qa[ks][rw] = h < nh ? p[ks * 8] : 0u;
        qa[ks][2 + rw] = h < nh ? p[ks * 8 + 4] : 0u;
      }
    }
    if constexpr (RW == 1)
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) qa[ks][1] = qa[ks][3] = 0u;
#pragma unroll
    for (int n = 0; n < D / 8; ++n)
#pragma unroll
      for (int x = 0; x < 4; ++x) o[n][x] = 0.f;
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.f;
  }
  __device__ __forceinline__ void ready(Shared&) {}

  __device__ __forceinline__ void trip(uint32_t st, uint32_t mask, Shared&, int) {
    const int lane = threadIdx.x & 31, t = lane & 3;
    const uint32_t k_at = st + ((lane & 7) + 8 * (lane >> 4)) * KS + ((lane >> 3) & 1) * 16;
    float sc[2][4] = {};
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      uint32_t b[4];
      dec_ldsm(k_at + ks * 32, b);
      dec_mma(sc[0], qa[ks], b[0], b[1]);
      dec_mma(sc[1], qa[ks], b[2], b[3]);
    }
#pragma unroll
    for (int tl = 0; tl < 2; ++tl)
#pragma unroll
      for (int x = 0; x < 4; ++x) sc[tl][x] = mask >> (8 * tl + 2 * t + (x & 1)) & 1 ? sc[tl][x] * unit : -INFINITY;
    uint32_t pa[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int rw = 0; rw < RW; ++rw) {
      float mx = fmaxf(fmaxf(sc[0][2 * rw], sc[0][2 * rw + 1]), fmaxf(sc[1][2 * rw], sc[1][2 * rw + 1]));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
      if (mx > m[rw]) {  // the same for the four threads of the row
        const float alpha = dec_ex2(m[rw] - mx);
        l[rw] *= alpha;
#pragma unroll
        for (int n = 0; n < D / 8; ++n) {
          o[n][2 * rw] *= alpha;
          o[n][2 * rw + 1] *= alpha;
        }
        m[rw] = mx;
      }
      const float ref = m[rw] == -INFINITY ? 0.f : m[rw];
      const float p00 = dec_ex2(sc[0][2 * rw] - ref), p01 = dec_ex2(sc[0][2 * rw + 1] - ref);
      const float p10 = dec_ex2(sc[1][2 * rw] - ref), p11 = dec_ex2(sc[1][2 * rw + 1] - ref);
      l[rw] += (p00 + p01) + (p10 + p11);
      pa[rw] = dec_pack_bf16(p00, p01);  // the accumulators of S are the A operand of P V
      pa[2 + rw] = dec_pack_bf16(p10, p11);
    }
    const uint32_t v_at = st + TK * KS + ((lane & 7) + 8 * ((lane >> 3) & 1)) * VS + (lane >> 4) * 16;
#pragma unroll
    for (int n = 0; n < D / 8; n += 2) {
      uint32_t b[4];
      dec_ldsm_t(v_at + n * 16, b);
      dec_mma(o[n], pa, b[0], b[1]);
      dec_mma(o[n + 1], pa, b[2], b[3]);
    }
  }

  __device__ __forceinline__ void finish(float* rows, int ld, float (*ml)[2]) {
    const int lane = threadIdx.x & 31, g8 = lane >> 2, t = lane & 3;
#pragma unroll
    for (int rw = 0; rw < RW; ++rw) {
      l[rw] += __shfl_xor_sync(0xffffffffu, l[rw], 1);
      l[rw] += __shfl_xor_sync(0xffffffffu, l[rw], 2);
      if (t == 0) {
        ml[g8 + 8 * rw][0] = m[rw];
        ml[g8 + 8 * rw][1] = l[rw];
      }
#pragma unroll
      for (int n = 0; n < D / 8; ++n)
        *reinterpret_cast<float2*>(rows + (g8 + 8 * rw) * ld + n * 8 + 2 * t) = make_float2(o[n][2 * rw], o[n][2 * rw + 1]);
    }
  }
};

// e4m3 pools: every e4m3 number is an fp16 number, so the tiles are fp16 with exact keys and values; the queries' rows are brought into
// fp16's range by a power of two each, and the weights, at most 1, lose less in fp16 than in bf16.  The scale of the keys goes into the
// logits' factor, that of the values into the output.  A lane reads 16 bytes of a key at once: the order in which a dot product takes its
// terms is free, so the queries' fragments are laid out to match.  Of the values, ldmatrix transposes pairs of bytes: a register
// holds two columns of two keys, which go to two tiles, of the even columns and of the odd ones.
template <int D_, int RW>
struct E4m3Rows {
  // Row strides without bank conflicts: for keys eight lanes read 16 bytes of two rows, for values of eight rows.
  static constexpr int D = D_, TK = 32, RowBytes = D, KS = D == 128 ? 144 : 64, VS = D + 16, R = 8 * RW, CL = D / 64;
  using Out = __nv_bfloat16;
  struct Shared {};
  uint32_t qa[D / 16][4];
  float o[D / 8][4], m[2], l[2], unit[2];

  static __device__ __forceinline__ uint32_t half2_of(uint16_t pair) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(pair));
    return r;
  }
  static __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
  static __device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
  }

  __device__ __forceinline__ void load(const DecodePagedArgs& a, Shared&, int32_t r, int32_t g, int32_t h0, int32_t nh, int32_t) {
    const int lane = threadIdx.x & 31, g8 = lane >> 2, t = lane & 3;
    const float per_key = a.scale_log2 * (a.k_scale ? a.k_scale[g] : 1.f);
#pragma unroll
    for (int rw = 0; rw < 2; ++rw) {
      const int32_t h = g8 + 8 * rw;
      uint32_t w[8 * CL];  // q[16 CL t .. + 16 CL) of head h
      if (rw < RW && h < nh) {
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
      const float down = as_is ? 1.f : __uint_as_float((268u - top) << 23), up = as_is ? 1.f : __uint_as_float((top - 14u) << 23);
      unit[rw] = per_key * up;
#pragma unroll
      for (int i = 0; i < 8 * CL; ++i) {  // word i: elements 2i, 2i + 1 = k slots of step i / 2, the lower or the upper pair
        const uint32_t x = pack_half(__uint_as_float(w[i] << 16) * down, __uint_as_float(w[i] & 0xffff0000u) * down);
        qa[i / 2][(i & 1) * 2 + rw] = x;
      }
    }
#pragma unroll
    for (int n = 0; n < D / 8; ++n)
#pragma unroll
      for (int x = 0; x < 4; ++x) o[n][x] = 0.f;
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.f;
  }
  __device__ __forceinline__ void ready(Shared&) {}

  __device__ __forceinline__ void trip(uint32_t st, uint32_t mask, Shared&, int) {
    const int lane = threadIdx.x & 31, g8 = lane >> 2, t = lane & 3;
    float sc[4][4] = {};
#pragma unroll
    for (int tl = 0; tl < 4; ++tl)
#pragma unroll
      for (int j = 0; j < CL; ++j) {
        uint32_t w[4];
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(st + (8 * tl + g8) * KS + (CL * t + j) * 16) : "memory");
#pragma unroll
        for (int s = 0; s < 4; ++s) mma(sc[tl], qa[4 * j + s], half2_of((uint16_t)w[s]), half2_of((uint16_t)(w[s] >> 16)));
      }
#pragma unroll
    for (int tl = 0; tl < 4; ++tl)
#pragma unroll
      for (int x = 0; x < 4; ++x) sc[tl][x] = mask >> (8 * tl + 2 * t + (x & 1)) & 1 ? sc[tl][x] * unit[x >> 1] : -INFINITY;
    uint32_t pa[2][4] = {};
#pragma unroll
    for (int rw = 0; rw < RW; ++rw) {
      float mx = fmaxf(sc[0][2 * rw], sc[0][2 * rw + 1]);
#pragma unroll
      for (int tl = 1; tl < 4; ++tl) mx = fmaxf(mx, fmaxf(sc[tl][2 * rw], sc[tl][2 * rw + 1]));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
      if (mx > m[rw]) {
        const float alpha = dec_ex2(m[rw] - mx);
        l[rw] *= alpha;
#pragma unroll
        for (int n = 0; n < D / 8; ++n) {
          o[n][2 * rw] *= alpha;
          o[n][2 * rw + 1] *= alpha;
        }
        m[rw] = mx;
      }
      const float ref = m[rw] == -INFINITY ? 0.f : m[rw];
#pragma unroll
      for (int tl = 0; tl < 4; ++tl) {
        const float p0 = dec_ex2(sc[tl][2 * rw] - ref), p1 = dec_ex2(sc[tl][2 * rw + 1] - ref);
        l[rw] += p0 + p1;
        pa[tl >> 1][(tl & 1) * 2 + rw] = pack_half(p0, p1);
      }
    }
    const uint32_t v_at = st + TK * KS + ((lane & 7) + 8 * ((lane >> 3) & 1)) * VS + (lane >> 4) * 16;
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {  // 32 columns
        uint32_t b[4];
        dec_ldsm_t(v_at + half * 16 * VS + c * 32, b);
#pragma unroll
        for (int i = 0; i < 2; ++i) {  // 16 columns: b[2i] of keys 2t, 2t + 1 and b[2i + 1] of keys 2t + 8, 2t + 9
          const uint32_t a0 = half2_of((uint16_t)b[2 * i]), a1 = half2_of((uint16_t)(b[2 * i] >> 16));
          const uint32_t c0 = half2_of((uint16_t)b[2 * i + 1]), c1 = half2_of((uint16_t)(b[2 * i + 1] >> 16));
          mma(o[4 * c + 2 * i], pa[half], __byte_perm(a0, a1, 0x5410), __byte_perm(c0, c1, 0x5410));
          mma(o[4 * c + 2 * i + 1], pa[half], __byte_perm(a0, a1, 0x7632), __byte_perm(c0, c1, 0x7632));
        }
      }
  }

  __device__ __forceinline__ void finish(float* rows, int ld, float (*ml)[2]) {
    const int lane = threadIdx.x & 31, g8 = lane >> 2, t = lane & 3;
#pragma unroll
    for (int rw = 0; rw < RW; ++rw) {
      l[rw] += __shfl_xor_sync(0xffffffffu, l[rw], 1);
      l[rw] += __shfl_xor_sync(0xffffffffu, l[rw], 2);
      if (t == 0) {
        ml[g8 + 8 * rw][0] = m[rw];
        ml[g8 + 8 * rw][1] = l[rw];
      }
#pragma unroll
      for (int c = 0; c < D / 16; ++c)
        *reinterpret_cast<float4*>(rows + (g8 + 8 * rw) * ld + 16 * c + 4 * t) =
            make_float4(o[2 * c][2 * rw], o[2 * c + 1][2 * rw], o[2 * c][2 * rw + 1], o[2 * c + 1][2 * rw + 1]);
    }
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

  __device__ __forceinline__ void load(const DecodePagedArgs& a, Shared&, int32_t r, int32_t g, int32_t h0, int32_t nh, int32_t) {
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

template <class E, int W, int ST, bool CLUSTER, int OCC>
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
  __shared__ int64_t s_at;
  __shared__ int32_t s_req;

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
  // the next request that has rows (there is one, or the lengths have changed under the kernel: then the last request, as it is)
  auto next_request = [&](int32_t& i, int32_t& rows) {
    rows = 0;
    while (rows == 0 && i + 1 < a.n_req) rows = rows_of(++i);
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
    for (int w = 0; w < W; ++w) all += s_scan[w];
    all *= a.v_heads;
    runs = min((int64_t)ctas, all);  // (each of a tile or more)
    first = c < runs ? all * c / runs : all;
    total = c < runs ? all * (c + 1) / runs - first : 0;
    // the request in which tile `first` lies: running sums over the requests, kThreads at a time
    int64_t before = 0;
    for (int32_t i0 = 0; i0 < a.n_req && total > 0; i0 += kThreads) {
      const int32_t i = i0 + tid;
      const int64_t mine = i < a.n_req ? (int64_t)tiles_of(rows_of(i)) * a.v_heads : 0;
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
      if (upto - mine <= first && first < upto) {
        s_req = i;
        s_at = first - (upto - mine);
      }
      before += chunk;
      if (before > first) break;
    }
    __syncthreads();
    r = total > 0 ? s_req : 0;
    n = total > 0 ? rows_of(r) : 0;
    const int64_t at = total > 0 ? s_at : 0;
    vh = n ? (int32_t)(at / tiles_of(n)) : 0;
    tile = n ? (int32_t)(at - (int64_t)vh * tiles_of(n)) : 0;
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
  struct Look {  // the page of lane's row (there < 0: no such row is wanted), its slot and its KV head
    int32_t page, slot, g;
  };
  auto look = [&]() {
    Look k = {-1, -1, 0};
    if (f_left > 0) {
      const int32_t row = ftile * TILE + warp * TK + lane;
      if (lane < TK && row < fn) {
        const uint32_t p = a.view.page_size.quotient((uint32_t)row);
        k.slot = row - (int32_t)(p * a.view.page_size.d);
        k.page = a.view.table[(int64_t)fr * a.view.table_stride + p];
      }
      k.g = a.blocks == 1 ? fvh : fvh / a.blocks;
      --f_left;
      if (++ftile == tiles_of(fn)) {
        ftile = 0;
        if (++fvh == a.v_heads && !CLUSTER) {
          fvh = 0;
          if (f_left > 0) next_request(fr, fn);
        }
      }
    }
    return k;
  };
  constexpr int CPR = E::RowBytes / 16, RPI = 32 / CPR;  // 16-byte chunks of a row, rows of a warp's request
  auto fetch = [&](int32_t stage, const Look& k) {
    int64_t off = k.slot >= 0 ? a.view.offset(k.page, (uint32_t)k.slot) : -1;
    const uint32_t mask = __ballot_sync(0xffffffffu, off >= 0);
    if (__ballot_sync(0xffffffffu, k.slot >= 0) != mask && lane == 0) atomicExch(a.status, (int32_t)PUREKV_ERR_BAD_PAGE);
    if (lane == 0) s_mask[warp][stage] = mask;
    if (mask) {
      off += (int64_t)k.g * a.view.head_stride;
      const uint32_t dst = ring + (uint32_t)stage * kStage + (lane / CPR) * E::KS + (lane % CPR) * 16;
      const uint32_t dst_v = ring + (uint32_t)stage * kStage + TK * E::KS + (lane / CPR) * E::VS + (lane % CPR) * 16;
#pragma unroll
      for (int i = 0; i < TK / RPI; ++i) {
        const int row = i * RPI + lane / CPR;
        const int64_t src = __shfl_sync(0xffffffffu, off, row) + (lane % CPR) * 16;
        const uint32_t bytes = mask >> row & 1 ? 16u : 0u;  // zeros for rows that do not exist
        const int64_t from = bytes ? src : 0;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + i * RPI * E::KS), "l"(a.k_pool + from), "r"(bytes) : "memory");
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst_v + i * RPI * E::VS), "l"(a.v_pool + from), "r"(bytes) : "memory");
      }
    }
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
  e.load(a, s_e, r, g, h0, nh, warp);
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
      if (++vh == a.v_heads) {
        vh = 0;
        next_request(r, n);
      }
      tile = 0;
      heads_at(vh, g, h0, nh);
      e.load(a, s_e, r, g, h0, nh, warp);
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

// Joins the parts of the requests that cuts went through: grid (CTAs of the balanced form, heads of a tile), a thread per column.
template <class E>
__global__ void __launch_bounds__(E::D) decode_paged_join_kernel(const __grid_constant__ DecodePagedArgs a) {
  constexpr int D = E::D, R = E::R;
  __shared__ float s_w[D], s_red[D / 32];
  const int32_t c = threadIdx.x, h = blockIdx.y, lane = c & 31, warp = c >> 5;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const ChainRecord chain = reinterpret_cast<const ChainRecord*>(a.chains)[blockIdx.x];
  if (chain.parts == 0) return;
  const int32_t g = chain.vh / a.blocks, b = chain.vh - g * a.blocks;
  if (h >= min(R, a.group - b * R)) return;
  auto slot = [&](int32_t i) { return a.part + (i == 0 ? 2 * (int64_t)blockIdx.x + 1 : 2 * ((int64_t)blockIdx.x + i)) * dp_part_floats<E>(); };
  float top = -INFINITY;
  for (int32_t i = c; i < chain.parts; i += D) top = fmaxf(top, dp_seen(slot(i)[R * D + h], slot(i)[R * D + R + h]));
#pragma unroll
  for (int x = 16; x >= 1; x /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
  if (lane == 0) s_red[warp] = top;
  __syncthreads();
  top = s_red[0];
#pragma unroll
  for (int w = 1; w < D / 32; ++w) top = fmaxf(top, s_red[w]);
  const float ref = dp_finite(top);
  float acc = 0.f, l = 0.f;
  for (int32_t i0 = 0; i0 < chain.parts; i0 += D) {
    const int32_t np = min(D, chain.parts - i0);
    __syncthreads();
    if (c < np) {
      const float li = slot(i0 + c)[R * D + R + h];
      s_w[c] = dp_weight(slot(i0 + c)[R * D + h], li, ref);
      l = fmaf(s_w[c], li, l);
    }
    __syncthreads();
#pragma unroll 4
    for (int32_t i = 0; i < np; ++i) acc = fmaf(s_w[i], slot(i0 + i)[h * D + c], acc);
  }
#pragma unroll
  for (int x = 16; x >= 1; x /= 2) l += __shfl_xor_sync(0xffffffffu, l, x);
  __syncthreads();
  if (lane == 0) s_red[warp] = l;
  __syncthreads();
  l = 0.f;
#pragma unroll
  for (int w = 0; w < D / 32; ++w) l += s_red[w];
  const int64_t hq = (int64_t)chain.r * a.n_q_heads + g * a.group + b * R + h;
  reinterpret_cast<typename E::Out*>(a.o)[hq * D + c] = (typename E::Out)(acc * ((a.v_scale ? a.v_scale[g] : 1.f) / l));
  if (c == 0 && a.lse) a.lse[hq] = (ref + log2f(l)) * 0.6931471805599453f;
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

template <class E, int W, int ST, int OCC>
static purekv_status launch_even(const DecodePagedArgs& a, int32_t cl, cudaStream_t stream) {
  auto kernel = decode_paged_kernel<E, W, ST, true, OCC>;
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

template <class E, int W, int ST, int OCC>
static purekv_status launch_balanced(const DecodePagedArgs& a, int32_t ctas, cudaStream_t stream) {
  auto kernel = decode_paged_kernel<E, W, ST, false, OCC>;
  static std::atomic<uint64_t> smem_allowed{0};
  const purekv_status st = allow_max_dynamic_smem(kernel, smem_allowed);
  if (st != PUREKV_OK) return st;
  DpLaunch l(dim3((unsigned)ctas), W * 32, (size_t)W * dp_warp_bytes<E, ST>(), stream);
  PK_CUDA(cudaLaunchKernelEx(&l.cfg, kernel, a));
  DpLaunch j(dim3((unsigned)ctas, (unsigned)std::min(E::R, a.group)), E::D, 0, stream);
  PK_CUDA(cudaLaunchKernelEx(&j.cfg, decode_paged_join_kernel<E>, a));
  return PUREKV_OK;
}

constexpr int32_t kDpCtas = 148;  // CTAs of the balanced form: one per SM

// How a call is launched: C CTAs per (request, head) in a cluster, or 0 for the balanced form.
struct DpForm {
  int32_t cluster;
};
static DpForm dp_form(int64_t base, int64_t bound) {
  int32_t c = 1;
  while (c < kDpClusterMax && bound > 128 * c && base * 2 * c <= (c < 4 ? 128 : 64)) c *= 2;
  return {bound <= 128 * (int64_t)c * 2 ? c : 0};
}

template <class E, int ST8>
static purekv_status launch_form(const DecodePagedArgs& a, const DpForm& f, cudaStream_t stream) {
  if (f.cluster) return launch_even<E, 8, ST8, 1>(a, f.cluster, stream);
  return launch_balanced<E, 8, ST8, 1>(a, kDpCtas, stream);
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
    if (rows == 2) return wide ? launch_form<Fp32Rows<128, 2>, 3>(a, form, sm) : launch_form<Fp32Rows<64, 2>, 3>(a, form, sm);
    return wide ? launch_form<Fp32Rows<128, 8>, 3>(a, form, sm) : launch_form<Fp32Rows<64, 8>, 3>(a, form, sm);
  }
  if (pages->dtype == PUREKV_E4M3) {
    if (rows == 8) return wide ? launch_form<E4m3Rows<128, 1>, 3>(a, form, sm) : launch_form<E4m3Rows<64, 1>, 5>(a, form, sm);
    return wide ? launch_form<E4m3Rows<128, 2>, 2>(a, form, sm) : launch_form<E4m3Rows<64, 2>, 5>(a, form, sm);
  }
  if (rows == 8) return wide ? launch_form<Bf16Rows<128, 1>, 3>(a, form, sm) : launch_form<Bf16Rows<64, 1>, 5>(a, form, sm);
  return wide ? launch_form<Bf16Rows<128, 2>, 3>(a, form, sm) : launch_form<Bf16Rows<64, 2>, 5>(a, form, sm);
}

}  // extern "C"
