// purekv_decode_paged: attention of one new token per request over the pages of a cache.
//
// What it computes, per request r and KV head g with its G query heads: one read of the request's K and V rows serves the whole group.
// Bound by HBM for much work (2 G operations per byte at most), by a chain of latencies for little: lengths, pages, rows, products,
// the join.
//
// Two kernels share everything but the way work reaches a CTA:
//  * even (CLUSTER): grid (C, heads, requests); a cluster of C CTAs owns one (request, KV head) and its parts meet in distributed
//    shared memory.  One launch, no workspace.
//  * balanced: the (KV head, request, tile of keys) triples in that order are cut into runs, whatever the lengths are -- they are read on
//    the device -- and a block is launched for each: first the long runs, as many as CTAs are at work at once, then the short ones
//    (paged_runs.cuh).  A CTA that comes to the end of its run takes over a block that has not started (cluster launch control), since
//    SMs do not stream equally fast, and goes on loading across the ends of requests and runs.  In which order blocks start and are handed
//    out does not matter.  (Head by head, so that CTAs at work on the heads of a request are at the same rows at the same time: those lie
//    side by side in memory.)  A request that a cut goes through leaves partial results in the workspace, which a second, small kernel joins.
//
// Inside a CTA every warp takes TK keys of a tile at a time through a ring of its own in shared memory (ST stages), filled by the copy
// engine (balanced form, pages that hold whole trips or of which a trip holds several) or by cp.async, looks the pages of its next keys up
// one step ahead, and keeps (reference maximum, sum, unnormalised output) in registers; the warps' results are joined at the end of a
// request.  Rows that do not exist are not read and weigh nothing.
//
// Waits on copies and answers are bounded.  A lane whose wait runs out goes on to the end of the tile, with whatever lies there; there its
// warp agrees to stop, and at the barrier at the request's end the CTA does: no vote or matrix product is reached by some lanes only.
// The CTA leaves once what is under way into its shared memory has landed.
#include <algorithm>
#include <cmath>

#include <cuda_fp16.h>

#include "cluster.cuh"
#include "common.cuh"
#include "decode.cuh"
#include "paged.cuh"
#include "paged_args.cuh"
#include "paged_runs.cuh"
#include "tc_util.cuh"

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
  // balanced form: per run what it leaves to be joined (ChainRecord) and two slots of partial results; CTAs at work at once; long and
  // short runs of a head; the limit of waits
  int32_t* chains;
  float* part;
  int32_t at_once, n_long, n_short;
  uint64_t wait_ns;
};

constexpr int kDpClusterMax = 16;
constexpr int kDpGroups = 128;   // of requests: their running sums of tiles lie in shared memory
constexpr int kDpSteals = 8;     // answers to requests for runs that a CTA keeps: more than runs its loads can be ahead of its products
constexpr int kDpShorts = 3;     // short runs for every CTA at work
constexpr uint64_t kDpNoWaitNs = 1000;           // limits below are no time at all: what is not there when it is asked about is late
constexpr uint64_t kDpSettleNs = 1000000000ull;  // of the wait for what is in flight, before a CTA that gave up leaves

// Tiles of one head: `left` of them, from tile `tile` of request r (n rows) on, tile `at` of the head's.
struct DpRun {
  int32_t id, vh, r, tile, n;
  int64_t at, left;
};

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
// the weights.  Returns whether O has to be multiplied by alpha.  The reference lies UP below the largest logit, so that weights go up to
// 2^UP (references and sums go together, so nobody else has to know).
template <int UP, int MT, int NT>
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
      if constexpr (UP > 0) mx -= (float)UP;
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

// How rows lie in a stage.  Copied by threads (SW false): one after the other, each padded so that no two of the rows that an
// instruction reads share banks.  Copied by the copy engine (SW true): in parts of 128 bytes, a part's rows one after the other, the
// 16-byte chunks of a row swizzled (by 128 bytes; 64-byte rows by 64).  In both, `at` is the address of chunk c of row `row`, given
// that the rows of one instruction agree in row - row % 8.
template <int TK, int RowBytes, int Stride, bool SW>
struct RowsAt {
  static __device__ __forceinline__ uint32_t at(uint32_t base, int row, int c) {
    if constexpr (!SW) return base + row * Stride + c * 16;
    else if constexpr (RowBytes == 64) return base + row * 64 + ((c ^ (row >> 1 & 3)) * 16);
    else return base + (c >> 3) * (TK * 128) + row * 128 + (((c & 7) ^ (row & 7)) * 16);
  }
};

// The rows of a trip that exist, a bit each.
template <int TK>
struct MaskOf { using type = uint32_t; };
template <>
struct MaskOf<64> { using type = uint64_t; };

// bf16 pools.  Padding of 16 bytes, so that ldmatrix reads eight rows without bank conflicts.  The weights are rounded to bf16 for the
// product with the values, as tiles have one type, and their sum is not: 2^-8 of each at most, independent of one another, 0.8e-3 of the
// result's norm beside the 1.7e-3 of its own rounding (1.9e-3 together).  What rounding leaves of the weights, as a second product, would
// remove that for twice the products with the values.
template <int D_, int NT, int MT, bool SW_>
struct Bf16Rows {
  static constexpr bool SW = SW_;
  static constexpr int D = D_, TK = 16 * MT, RowBytes = D * 2, KS = RowBytes + (SW ? 0 : 16), VS = KS, R = 8 * NT;
  using At = RowsAt<TK, RowBytes, KS, SW>;
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

  using Mask = typename MaskOf<TK>::type;
  __device__ __forceinline__ void trip(uint32_t st, Mask mask, Shared&, int) {
    const int lane = threadIdx.x & 31, g8 = lane >> 2;
    float sc[MT][NT][4] = {}, odd[MT][NT][4] = {};  // two chains of products
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        uint32_t k[4];
        dec_ldsm(At::at(st, 16 * mt + (lane & 7) + 8 * ((lane >> 3) & 1), 2 * ks + (lane >> 4)), k);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) dec_mma(ks & 1 ? odd[mt][nt] : sc[mt][nt], k, qb[ks][nt][0], qb[ks][nt][1]);
      }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          sc[mt][nt][x] = mask >> (16 * mt + g8 + 8 * (x >> 1)) & 1 ? (sc[mt][nt][x] + odd[mt][nt][x]) * unit : -INFINITY;
    float alpha[NT][2];
    if (dp_softmax<0, MT, NT>(sc, m, l, alpha)) dp_rescale(o, alpha);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      uint32_t p[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        p[nt][0] = dp_transpose(dec_pack_bf16(sc[mt][nt][0], sc[mt][nt][1]));
        p[nt][1] = dp_transpose(dec_pack_bf16(sc[mt][nt][2], sc[mt][nt][3]));
      }
#pragma unroll
      for (int n = 0; n < D / 16; ++n) {
        uint32_t v[4];
        dec_ldsm_t(At::at(st + TK * KS, 16 * mt + (lane & 7) + 8 * (lane >> 4), 2 * n + ((lane >> 3) & 1)), v);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) dec_mma(o[n][nt], v, p[nt][0], p[nt][1]);
      }
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
// fp16's range by a power of two each.  The weights go up to 2^15 (fp16 ends at 65504): they keep 11 bits down to 2^-29 of the largest
// and are off by 2^-40 of it at most below, so that not even a million keys of 2^-26 are lost, as they would be with weights up to 1.  The
// scale of the keys goes into the logits' factor, that of the values into the output.  A lane reads 16 bytes of a key at once:
// the order in which a dot product takes its terms is free, so the queries' fragments are laid out to match.  Of the values,
// ldmatrix transposes 16 x 16 bytes: a register holds a column of four keys, whose halves are two registers of a tile of V^T once they
// are fp16; the keys' rows in the tiles of logits are in the order that this gives.  (Transposed in pairs of bytes, and the columns sorted
// out after the conversion, it is a quarter more instructions, which set the pace under the power cap: 128 requests of 2900-5100 rows, 8 KV
// heads, call after call at 1640 MHz, 181 us against 174.)
template <int D_, int NT, int MT, bool SW_>
struct E4m3Rows {
  static constexpr bool SW = SW_;
  // Row strides without bank conflicts: for keys eight lanes read 16 bytes of two rows, for values of eight rows.
  static constexpr int D = D_, TK = 16 * MT, RowBytes = D, KS = SW ? D : D == 128 ? 144 : 64, VS = SW ? D : D + 16, R = 8 * NT, CL = D / 64;
  using KAt = RowsAt<TK, RowBytes, KS, SW>;
  using VAt = RowsAt<TK, RowBytes, VS, SW>;
  using Out = __nv_bfloat16;
  struct Shared {};
  static constexpr int kUp = 15;
  uint32_t qb[D / 16][NT][2];
  float o[D / 16][NT][4], m[NT][2], l[NT][2], unit[NT][2];

  // The key of 16 in row g8 (x 0) or g8 + 8 (x 1) of a tile of logits.
  static __device__ __forceinline__ int key(int g8, int x) { return 4 * (g8 >> 1) + (g8 & 1) + 2 * x; }
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

  using Mask = typename MaskOf<TK>::type;
  __device__ __forceinline__ void trip(uint32_t st, Mask mask, Shared&, int) {
    const int lane = threadIdx.x & 31, g8 = lane >> 2, t = lane & 3;
    float sc[MT][NT][4] = {};
#pragma unroll
    for (int j = 0; j < CL; ++j)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        uint32_t w[2][4];  // the keys of rows g8 and g8 + 8 of the tile
#pragma unroll
        for (int x = 0; x < 2; ++x)
          asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                       : "=r"(w[x][0]), "=r"(w[x][1]), "=r"(w[x][2]), "=r"(w[x][3])
                       : "r"(KAt::at(st, 16 * mt + key(g8, x), CL * t + j)) : "memory");
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const uint32_t a0 = half2_of((uint16_t)w[0][s]), a2 = half2_of((uint16_t)(w[0][s] >> 16));
          const uint32_t a1 = half2_of((uint16_t)w[1][s]), a3 = half2_of((uint16_t)(w[1][s] >> 16));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) mma(sc[mt][nt], a0, a1, a2, a3, qb[4 * j + s][nt][0], qb[4 * j + s][nt][1]);
        }
      }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int x = 0; x < 4; ++x) sc[mt][nt][x] = mask >> (16 * mt + key(g8, x >> 1)) & 1 ? sc[mt][nt][x] * unit[nt][x & 1] : -INFINITY;
    float alpha[NT][2];
    if (dp_softmax<kUp, MT, NT>(sc, m, l, alpha)) dp_rescale(o, alpha);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      uint32_t p[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        p[nt][0] = dp_transpose(pack_half(sc[mt][nt][0], sc[mt][nt][1]));
        p[nt][1] = dp_transpose(pack_half(sc[mt][nt][2], sc[mt][nt][3]));
      }
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {  // 32 columns: r[0], r[1] columns g8 and g8 + 8 of keys 4t .. 4t + 3, r[2], r[3] the same of the other 16
        uint32_t r[4];
        asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0, %1, %2, %3}, [%4];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                     : "r"(VAt::at(st + TK * KS, 16 * mt + (lane & 15), 2 * c + (lane >> 4))) : "memory");
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const uint32_t a0 = half2_of((uint16_t)r[2 * y]), a2 = half2_of((uint16_t)(r[2 * y] >> 16));
          const uint32_t a1 = half2_of((uint16_t)r[2 * y + 1]), a3 = half2_of((uint16_t)(r[2 * y + 1] >> 16));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) mma(o[2 * c + y][nt], a0, a1, a2, a3, p[nt][0], p[nt][1]);
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
      for (int n = 0; n < D / 16; ++n)
#pragma unroll
        for (int x = 0; x < 4; ++x) rows[(8 * nt + 2 * t + (x & 1)) * ld + 16 * n + g8 + 8 * (x >> 1)] = o[n][nt][x];
  }
};

// fp32 pools: CUDA cores (tf32 would not keep fp32's accuracy).  For the logits a lane takes 32 elements of one key and all heads; for
// the output D / 32 columns of every key.
template <int D_, int GP, bool SW_>
struct Fp32Rows {
  static constexpr bool SW = SW_;
  static constexpr int D = D_, TK = D == 64 ? 16 : 8, RowBytes = D * 4, KS = RowBytes + (SW ? 0 : 16), VS = KS, R = GP, E = D / 32;
  using At = RowsAt<TK, RowBytes, KS, SW>;
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

  using Mask = uint32_t;
  __device__ __forceinline__ void trip(uint32_t st, Mask mask, Shared& s, int warp) {
    const int lane = threadIdx.x & 31, key = lane % TK, part = lane / TK;
    float dot[GP];
#pragma unroll
    for (int h = 0; h < GP; ++h) dot[h] = 0.f;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      float4 k;
      asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                   : "=f"(k.x), "=f"(k.y), "=f"(k.z), "=f"(k.w) : "r"(At::at(st, key, part * 8 + c)) : "memory");
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
#pragma unroll
    for (int j = 0; j < TK; ++j) {
      float v[E];
      if constexpr (E == 2)
        asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v[0]), "=f"(v[1]) : "r"(At::at(st + TK * KS, j, lane >> 1) + (lane & 1) * 8) : "memory");
      else
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(At::at(st + TK * KS, j, lane)) : "memory");
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
// A warp's output rows start eight banks apart where there is room; they are laid over the stage that the warp used last.
template <class E>
__host__ __device__ constexpr int dp_ld() { return E::R * (E::D + 8) * 4 <= dp_stage_bytes<E>() ? E::D + 8 : E::D; }
template <class E, int ST>
__host__ __device__ constexpr int dp_warp_bytes() {
  static_assert(ST == 1 || E::R * dp_ld<E>() * 4 <= dp_stage_bytes<E>(), "a warp's rows fit a stage");
  return ST * dp_stage_bytes<E>() > E::R * dp_ld<E>() * 4 ? ST * dp_stage_bytes<E>() : E::R * dp_ld<E>() * 4;
}
// Partial results of one slot: [R][D] unnormalised outputs, [R] references, [R] sums
__host__ __device__ constexpr int64_t dp_part_floats(int rows, int d) { return (int64_t)rows * (d + 2); }

// What a run of the balanced form leaves: the request and virtual head whose first part it is (in its second slot), and how many
// parts there are (the others in the first slots of the head's runs that follow); 0: nothing.
struct ChainRecord {
  int32_t r, vh, parts, pad;
};

// Row of a request: weight of a warp's, a CTA's or a part's result.  Nothing summed (sum 0) weighs nothing; a NaN sum stays NaN.
__device__ __forceinline__ float dp_weight(float m, float l, float ref) { return l == 0.f ? 0.f : dec_ex2(m - ref); }
__device__ __forceinline__ float dp_seen(float m, float l) { return l == 0.f ? -INFINITY : m; }
__device__ __forceinline__ float dp_finite(float m) { return m == -INFINITY ? 0.f : m; }
// What a request's sums are multiplied by, and its log-sum-exp: 0 and -inf where no key weighs anything (no rows, or none that is there).
__device__ __forceinline__ float dp_over(float scale, float l) { return l == 0.f ? 0.f : scale / l; }
__device__ __forceinline__ float dp_lse(float ref, float l) { return (ref + log2f(l)) * 0.6931471805599453f; }

template <typename T>
__device__ __forceinline__ void dp_store4(T* dst, float4 v);
template <>
__device__ __forceinline__ void dp_store4(__nv_bfloat16* dst, float4 v) {
  *reinterpret_cast<uint2*>(dst) = make_uint2(dec_pack_bf16(v.x, v.y), dec_pack_bf16(v.z, v.w));
}
template <>
__device__ __forceinline__ void dp_store4(float* dst, float4 v) { *reinterpret_cast<float4*>(dst) = v; }

// How rows come into shared memory: each by its own page (cp.async); a trip's rows from one page (cp.async), where a page holds whole
// trips; the same by the copy engine.
enum DpLoad { kDpRows, kDpWhole, kDpEngine };
// The pools as the copy engine sees them, in bytes: (128 of a row, slot of a page, part of a row, head, page).  A trip's rows are `boxes`
// boxes: one of all parts where a page holds whole trips, otherwise one for each part and page.
struct DpMaps {
  CUtensorMap k, v;
  int32_t boxes;
};

template <class E, int W, int ST, bool CLUSTER, DpLoad LOAD, int OCC>
__global__ void __launch_bounds__(W * 32, OCC) decode_paged_kernel(const __grid_constant__ DecodePagedArgs a, const __grid_constant__ DpMaps maps) {
  constexpr bool WHOLE = LOAD != kDpRows;
  static_assert(E::SW == (LOAD == kDpEngine), "the copy engine swizzles");
  constexpr int D = E::D, R = E::R, TK = E::TK, TILE = W * TK, kThreads = W * 32, kStage = dp_stage_bytes<E>(), LD = dp_ld<E>();
  constexpr int kWarpBytes = dp_warp_bytes<E, ST>();
  using Out = typename E::Out;
  extern __shared__ __align__(16) uint8_t dp_smem_raw[];
  // (the swizzle counts from multiples of 1024 bytes)
  uint8_t* const dp_smem = LOAD == kDpEngine ? dp_smem_raw + (-(int32_t)__cvta_generic_to_shared(dp_smem_raw) & 1023) : dp_smem_raw;
  __shared__ float s_ml[W][R][2];
  using Mask = typename E::Mask;
  __shared__ Mask s_mask[W][ST];
  __shared__ __align__(8) uint64_t s_full[LOAD == kDpEngine ? W : 1][ST];  // a stage's copies have arrived
  __shared__ int s_late;
  __shared__ __align__(16) typename E::Shared s_e;
  __shared__ __align__(16) float s_part[CLUSTER ? R * D : 1];          // what the cluster's CTAs send this one: [source][head][its columns]
  __shared__ __align__(8) float s_pml[CLUSTER ? kDpClusterMax : 1][R][2];  // every CTA's (reference, sum) per head
  __shared__ int64_t s_sum[W];
  __shared__ int64_t s_tiles[CLUSTER ? 1 : kDpGroups];                // running sums of the requests' tiles, by groups of requests
  __shared__ int32_t s_rows[CLUSTER ? 1 : kDpGroups];                 // rows of the last request of each group
  __shared__ __align__(16) ulonglong2 s_stolen[CLUSTER ? 1 : kDpSteals];  // answers to this CTA's requests for runs
  __shared__ __align__(8) uint64_t s_answered[CLUSTER ? 1 : kDpSteals];
  __shared__ DpRun s_run[CLUSTER ? 1 : W][kDpSteals];                 // per warp: the runs that its loads have entered
  __shared__ int32_t s_found[2];                                      // a run that one thread has found, and the answers it has read

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
  // the next request that has rows (there is one, or the lengths have changed under the kernel: then the last request)
  auto next_request = [&](int32_t& i, int32_t& rows) {
    while (i + 1 < a.n_req && (rows = rows_of(++i)) == 0) {}
  };
  auto tiles_of = [&](int32_t n) { return (n + TILE - 1) / TILE; };

  // The work at hand: `left` tiles from tile `tile` of (request r with n rows, virtual head vh) on.
  DpRun run = {};
  int32_t f_answers = 0;  // read so far
  bool late = false;      // a wait of this warp's ran out: it asks for, loads and multiplies nothing any more
  // Whether a barrier's phase has come, for the calling thread; false if the limit passes, or has passed for another thread of the CTA.
  auto arrives = [&](uint32_t bar, uint32_t phase) {
    if (tc::mbar_test(bar, phase)) return true;
    if (a.wait_ns >= kDpNoWaitNs) return tc::mbar_wait(bar, phase, &s_late, a.wait_ns);
    *(volatile int*)&s_late = 1;
    return false;
  };
  RunCuts cuts = {};
  auto take = [&](int32_t b) {
    const int32_t j = cuts.piece_of(b);
    DpRun x = {b, b - j * a.v_heads, 0, 0, 0, cuts.starts_at(j), cuts.tiles(b)};
    if (x.left > 0) {
      // the group of requests in which tile x.at lies, then the request
      uint32_t hit = __ballot_sync(0xffffffffu, s_tiles[lane * (kDpGroups / 32) + kDpGroups / 32 - 1] > x.at);
      const int32_t first = (__ffs(hit) - 1) * (kDpGroups / 32);
      hit = __ballot_sync(0xffffffffu, lane < kDpGroups / 32 && s_tiles[first + lane % (kDpGroups / 32)] > x.at);
      const int32_t group = first + __ffs(hit) - 1, per_group = (a.n_req + kDpGroups - 1) / kDpGroups;
      int64_t before = group > 0 ? s_tiles[group - 1] : 0;
      if (per_group == 1) {
        x.r = group;
        x.n = s_rows[group];
        x.tile = (int32_t)(x.at - before);
        return x;
      }
      for (int32_t i0 = group * per_group; i0 < a.n_req; i0 += 32) {
        const int32_t rows = i0 + lane < a.n_req ? rows_of(i0 + lane) : 0;
        int64_t upto = tiles_of(rows);
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
          const int64_t y = __shfl_up_sync(0xffffffffu, upto, d);
          if (lane >= d) upto += y;
        }
        hit = __ballot_sync(0xffffffffu, before + upto > x.at);
        if (hit) {
          const int32_t l0 = __ffs(hit) - 1;
          x.r = i0 + l0;
          x.n = __shfl_sync(0xffffffffu, rows, l0);
          x.tile = (int32_t)(x.at - (before + __shfl_sync(0xffffffffu, upto, l0) - tiles_of(x.n)));
          break;
        }
        before += __shfl_sync(0xffffffffu, upto, 31);
      }
    }
    return x;
  };
  // Thread 0 asks for a run that no CTA has started; the answer comes to its slot and barrier.
  auto ask = [&](int32_t k) {
    const uint32_t slot = (uint32_t)__cvta_generic_to_shared(&s_stolen[k % kDpSteals]), bar = (uint32_t)__cvta_generic_to_shared(&s_answered[k % kDpSteals]);
    tc::mbar_expect_tx(bar, 16);
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(slot), "r"(bar) : "memory");
  };
  // The run of answer k, -1 if there is none, -2 if the answer is late.
  auto answer = [&](int32_t k) {
    if (!arrives((uint32_t)__cvta_generic_to_shared(&s_answered[k % kDpSteals]), (uint32_t)(k / kDpSteals) & 1u)) return -2;
    const volatile ulonglong2& h = s_stolen[k % kDpSteals];
    const uint64_t lo = h.x, hi = h.y;
    uint32_t yes, b;
    asm volatile(
        "{\n .reg .b128 h;\n .reg .pred p;\n mov.b128 h, {%2, %3};\n clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, h;\n"
        " selp.u32 %0, 1, 0, p;\n mov.u32 %1, 0;\n @p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, h;\n}\n"
        : "=r"(yes), "=r"(b) : "l"(lo), "l"(hi));
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // read before a later answer overwrites it
    return yes ? (int32_t)b : -1;
  };
  ChainRecord* const chains = reinterpret_cast<ChainRecord*>(a.chains);
  // Answer k has come into shared memory, which the CTA must not leave before.
  auto settle_answer = [&](int32_t k) {
    volatile int again = 0;
    tc::mbar_wait((uint32_t)__cvta_generic_to_shared(&s_answered[k % kDpSteals]), (uint32_t)(k / kDpSteals) & 1u, &again, kDpSettleNs);
  };
  // The next run with tiles among those that no CTA has started, `k` answers having been read; without tiles if there are none.  One
  // thread asks for the block: the answers' slots are its own as long as no warp waits for one.
  auto find = [&](int32_t& k) {
    if constexpr (LOAD == kDpEngine) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the rows laid over the stages, before they are copied into again
    if (tid == 0) {
      auto next = [&] {
        const int32_t b = answer(k);
        if (b == -2) {
          atomicExch(a.status, (int32_t)PUREKV_ERR_TIMEOUT);
          settle_answer(k);
        }
        ++k;
        return b;
      };
      s_found[0] = next_run(cuts, [&] { ask(k); }, next, [&](int32_t b) { chains[b].parts = 0; });
      s_found[1] = k;
    }
    __syncthreads();
    k = s_found[1];
    const int32_t b = s_found[0];
    return b < 0 ? DpRun{} : take(b);
  };
  if constexpr (CLUSTER) {
    run = {0, (int32_t)blockIdx.y, (int32_t)blockIdx.z, 0, rows_of(blockIdx.z), 0, 0};
    if (a.view.seq_lens[run.r] > capacity && tid == 0) atomicExch(a.status, (int32_t)PUREKV_ERR_BAD_PAGE);
    const int32_t tiles = tiles_of(run.n), share = (tiles + C - 1) / C;
    run.tile = min(rank * share, tiles);
    run.left = min(share, tiles - run.tile);
  } else {
    if (tid < kDpSteals) tc::mbar_init((uint32_t)__cvta_generic_to_shared(&s_answered[tid]), 1);
    if (LOAD == kDpEngine && lane < ST) tc::mbar_init((uint32_t)__cvta_generic_to_shared(&s_full[warp][lane]), 1);
    if (tid == 0) s_late = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    constexpr int kPer = kDpGroups / kThreads;  // groups of a thread
    const int32_t per_group = (a.n_req + kDpGroups - 1) / kDpGroups;
    int64_t mine[kPer], sum = 0;
#pragma unroll
    for (int x = 0; x < kPer; ++x) {
      const int32_t i0 = (tid * kPer + x) * per_group;
      for (int32_t i = i0; i < min(i0 + per_group, a.n_req); ++i) {
        const int32_t rows = rows_of(i);
        s_rows[tid * kPer + x] = rows;
        sum += tiles_of(rows);
      }
      mine[x] = sum;
    }
    int64_t upto = sum, all = 0;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int64_t y = __shfl_up_sync(0xffffffffu, upto, d);
      if (lane >= d) upto += y;
    }
    if (lane == 31) s_sum[warp] = upto;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) {
      if (w < warp) upto += s_sum[w];
      all += s_sum[w];
    }
#pragma unroll
    for (int x = 0; x < kPer; ++x) s_tiles[tid * kPer + x] = upto - sum + mine[x];
    __syncthreads();
    cuts = RunCuts::of(all, a.v_heads, a.at_once, a.n_long, a.n_short);
    if (tid == 0) chains[blockIdx.x].parts = 0;
    run = take(blockIdx.x);
    if (run.left <= 0) {
      run = find(f_answers);
      if (run.left <= 0) return;
    }
    if (tid == 0) ask(f_answers);
  }

  // Whether this warp's copies into `stage` have arrived (phase: of the stage's barrier), for the calling lane.
  auto arrived = [&](int32_t stage, uint32_t phase) {
    if constexpr (LOAD == kDpEngine) {
      return arrives((uint32_t)__cvta_generic_to_shared(&s_full[warp][stage]), phase);
    } else {
      asm volatile("cp.async.wait_group %0;" ::"n"(ST - 1) : "memory");
      return true;
    }
  };

  const int32_t box_rows = LOAD == kDpEngine ? TK / maps.boxes : TK;

  // ---- loads.  The cursor runs ahead of the products, over the ends of requests and of runs.
  DpRun f = run;
  int32_t f_runs = 1;  // entered
  bool f_more = !CLUSTER, f_empty = false;  // a further run is asked for; the last one asked for had no tiles
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(dp_smem) + (uint32_t)warp * kWarpBytes;
  // The page of a row, its slot there and its KV head.  WHOLE: of the trip's first row, `there` of whose rows are wanted (copy engine:
  // of the first row of box `lane`, if there are several, and of that box); otherwise of row `lane` of the trip, `there` 1 if it is
  // wanted.
  struct Look {
    int32_t page, slot, g, there;
  };
  auto look = [&]() {
    Look k = {-1, 0, 0, 0};
    if constexpr (!CLUSTER) {
      if (f.left == 0 && f_more && !late) {
        const int32_t b = answer(f_answers);
        late = __any_sync(0xffffffffu, b == -2);  // (for one lane, so for all: what follows is the warp's together)
        if (!late) {
          ++f_answers;
          f_more = false;
        }
        if (!late && b >= 0) {
          if (tid == 0) chains[b].parts = 0;
          const DpRun x = take(b);
          if (x.left > 0) {
            f = x;
            f_more = true;
            if (tid == 0) ask(f_answers);
            if (lane == 0) s_run[warp][f_runs % kDpSteals] = x;
            ++f_runs;
          } else {
            f_empty = true;
          }
        }
      }
    }
    if (f.left > 0) {
      int32_t row = f.tile * TILE + warp * TK + (WHOLE ? 0 : lane);
      if constexpr (LOAD == kDpEngine) {
        if (maps.boxes > 1) row += lane * box_rows;
        k.there = maps.boxes == 1 || lane < maps.boxes ? min(max(f.n - row, 0), box_rows) : 0;
      } else {
        k.there = WHOLE ? min(max(f.n - row, 0), TK) : lane < TK && row < f.n;
      }
      if (k.there > 0) {
        const uint32_t p = a.view.page_size.quotient((uint32_t)row);
        k.slot = row - (int32_t)(p * a.view.page_size.d);
        k.page = a.view.table[(int64_t)f.r * a.view.table_stride + p];
      }
      k.g = a.blocks == 1 ? f.vh : f.vh / a.blocks;
      --f.left;
      if (++f.tile == tiles_of(f.n)) {
        f.tile = 0;
        if (!CLUSTER && f.left > 0) next_request(f.r, f.n);
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
    Mask mask;
    if constexpr (LOAD == kDpEngine) {
      mask = off < 0 ? (Mask)0 : (Mask)(~(Mask)0 >> (8 * sizeof(Mask) - k.there));
      uint32_t rows = off >= 0 ? (uint32_t)box_rows : 0u;  // copied: whole boxes; what lies behind the request's last row is masked (keys) or overwritten (values) later
      bool missing = k.there > 0 && off < 0;
      if (maps.boxes > 1) {
        mask = off < 0 ? (Mask)0 : mask << (lane * box_rows);
        uint32_t lo = __reduce_or_sync(0xffffffffu, (uint32_t)mask);
        if constexpr (sizeof(Mask) == 8) mask = lo | (Mask)__reduce_or_sync(0xffffffffu, (uint32_t)(mask >> 32)) << 32;
        else mask = lo;
        rows = __popc(__ballot_sync(0xffffffffu, off >= 0)) * box_rows;
        missing = __any_sync(0xffffffffu, missing);
      }
      const uint32_t bar = (uint32_t)__cvta_generic_to_shared(&s_full[warp][stage]), to = ring + (uint32_t)stage * kStage;
      auto load = [&](uint32_t dst, const CUtensorMap* map, int32_t part, int32_t slot, int32_t page) {
        asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
                     ::"r"(dst), "l"(map), "r"(bar), "r"(0), "r"(slot), "r"(part), "r"(k.g), "r"(page) : "memory");
      };
      if (lane == 0) {
        if (missing) atomicExch(a.status, (int32_t)PUREKV_ERR_BAD_PAGE);
        if (rows) tc::mbar_expect_tx(bar, rows * 2 * E::RowBytes);
        else tc::mbar_arrive(bar);  // (the barrier's phases stay in step with the stages)
      }
      if (maps.boxes == 1) {
        if (lane == 0 && rows) {
          load(to, &maps.k, 0, k.slot, k.page);
          load(to + TK * E::KS, &maps.v, 0, k.slot, k.page);
        }
      } else {
        constexpr int kParts = E::RowBytes < 128 ? 1 : E::RowBytes / 128, kInner = E::RowBytes / kParts;
        __syncwarp();  // (the barrier expects the bytes before they come)
        const int32_t box = lane % maps.boxes, part = lane / maps.boxes;
        const int32_t page = __shfl_sync(0xffffffffu, off >= 0 ? k.page : -1, box);
        if (page >= 0 && part < kParts) {
          const uint32_t dst = to + part * (TK * kInner) + box * box_rows * kInner;
          load(dst, &maps.k, part, 0, page);
          load(dst + TK * E::KS, &maps.v, part, 0, page);
        }
      }
    } else if constexpr (WHOLE) {
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
    if constexpr (LOAD != kDpEngine) asm volatile("cp.async.commit_group;" ::: "memory");  // (empty past the end: the group count stays in step)
  };
  // A wait ran out: all of the CTA's threads leave, once what is under way into shared memory has landed, copies into any stage (into the
  // one just used up, `stage`, they have unless they are the late ones) and an answer.
  auto leave = [&](int32_t stage, uint32_t phase) {
    if (late && lane == 0) atomicExch(a.status, (int32_t)PUREKV_ERR_TIMEOUT);
    if constexpr (LOAD == kDpEngine) {
      volatile int again = 0;
      for (int32_t i = 0; i < ST; ++i, stage = stage + 1 == ST ? 0 : stage + 1, phase ^= stage == 0)
        tc::mbar_wait((uint32_t)__cvta_generic_to_shared(&s_full[warp][stage]), phase, &again, kDpSettleNs);
    } else {
      asm volatile("cp.async.wait_all;" ::: "memory");
    }
    if (tid == 0 && f_more) settle_answer(f_answers);
  };

  E e;
  auto heads_at = [&](int32_t v, int32_t& g, int32_t& h0, int32_t& nh) {
    g = a.blocks == 1 ? v : v / a.blocks;
    const int32_t b = v - g * a.blocks;
    h0 = g * a.group + b * R;
    nh = min(R, a.group - b * R);
  };
  int32_t g, h0, nh;
  int32_t stage = 0, c_runs = 1;  // c_runs: runs entered by the products
  uint32_t phase = 0;
  bool from_start;  // whether this run has the request's first tile
[[maybe_unused]] begin:
  Look next;
  {
    Look ahead[ST > 1 ? ST - 1 : 1];
#pragma unroll
    for (int s = 0; s < (ST > 1 ? ST - 1 : 1); ++s) ahead[s] = look();
#pragma unroll
    for (int s = 0; s < (ST > 1 ? ST - 1 : 1); ++s) fetch(stage + s < ST ? stage + s : stage + s - ST, ahead[s]);
    next = look();
  }
  heads_at(run.vh, g, h0, nh);
  e.load(a, s_e, run.r, g, h0, nh);
  e.ready(s_e);
  __syncthreads();
  from_start = run.tile == 0;
  while (true) {
    bool end_of_request = true;
    if (run.left > 0) {
      if constexpr (ST > 1) {
        fetch(stage == 0 ? ST - 1 : stage - 1, next);
        next = look();
      }
      late = late || !arrived(stage, phase);  // (if so the tile is whatever lies there, and the warp's last one)
      __syncwarp();
      const Mask mask = s_mask[warp][stage];
      if constexpr (LOAD == kDpEngine) {
        constexpr Mask kAll = (Mask)(~(Mask)0 >> (8 * sizeof(Mask) - TK));
        if (mask != 0 && mask != kAll) {  // zeros for the values that are not the request's: whatever lies there has weight 0, but may be NaN
          constexpr int kChunks = E::RowBytes / 16, kPart = kChunks < 8 ? kChunks : 8;  // of a row, of a part of a row
          for (int32_t x = lane; x < TK * kChunks; x += 32) {
            const int32_t row = x / kChunks, c = x % kChunks;
            if (mask >> row & 1) continue;
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(ring + (uint32_t)stage * kStage + TK * E::KS + (c / kPart) * (TK * 128) + row * (kPart * 16) + (c % kPart) * 16), "r"(0) : "memory");
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // before the copy engine writes there again
          __syncwarp();
        }
      }
      if (mask) e.trip(ring + (uint32_t)stage * kStage, mask, s_e, warp);
      __syncwarp();  // every lane has read the stage before the next fetch overwrites it
      if constexpr (!CLUSTER) late = __any_sync(0xffffffffu, late);
      --run.left;
      ++run.at;
      end_of_request = ++run.tile == tiles_of(run.n);
      if constexpr (ST == 1) {
        static_assert(CLUSTER, "one stage: nothing is loaded across the ends of requests");
        if (run.left > 0) {
          fetch(0, next);
          next = look();
        }
      }
      if (!end_of_request && run.left > 0 && !late) {
        stage = stage + 1 == ST ? 0 : stage + 1;
        phase ^= stage == 0;
        continue;
      }
    }

    // ---- the warps' results side by side, each over the stage that its warp has just used up
    e.finish(reinterpret_cast<float*>(dp_smem + warp * kWarpBytes + stage * kStage), LD, s_ml[warp]);
    const DpRun done = run;
    const int32_t h0_done = h0, nh_done = nh, g_done = g;
    bool more = false;
    if constexpr (!CLUSTER) {  // the next request's queries, while this one's results are joined
      if (run.left > 0) {
        next_request(run.r, run.n);
        run.tile = 0;
        more = true;
      } else if (c_runs < f_runs) {
        __syncwarp();
        run = s_run[warp][c_runs++ % kDpSteals];
        more = true;
      }
      if (more) {
        heads_at(run.vh, g, h0, nh);
        e.load(a, s_e, run.r, g, h0, nh);
      }
    }
    __syncthreads();
    const bool quit = !CLUSTER && *(volatile int*)&s_late;  // a warp's wait ran out: the results are nobody's (no warp waits again before the next barrier)
    if constexpr (CLUSTER) {
      if (C > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    }
    const float vs = a.v_scale ? a.v_scale[g_done] : 1.f;
    const bool whole = CLUSTER ? C == 1 : from_start && end_of_request;
    const int32_t cols = D / C;  // columns of every head that each CTA of the cluster finishes
    float* slot = nullptr;
    if constexpr (!CLUSTER) slot = a.part + (2 * (int64_t)done.id + (from_start ? 1 : 0)) * dp_part_floats(R, D);
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
        const int64_t hq = (int64_t)done.r * a.n_q_heads + h0_done + h;
        const float inv = dp_over(vs, l);
        dp_store4(reinterpret_cast<Out*>(a.o) + hq * D + col, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
        if (col == 0 && a.lse) a.lse[hq] = dp_lse(ref, l);
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
      if (from_start && !end_of_request && tid == 0) {  // the first of several parts; the last is the run with the request's last tile
        const int64_t last = done.at - 1 + (tiles_of(done.n) - done.tile);
        chains[done.id] = {done.r, done.vh, cuts.piece_with(last) - cuts.piece_of(done.id) + 1, 0};
      }
      if (quit) return leave(stage, phase);
      if (!more) break;
      e.ready(s_e);
      if constexpr (LOAD == kDpEngine) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the rows laid over the stages, before they are copied into again
      __syncthreads();
      from_start = run.tile == 0;
      stage = stage + 1 == ST ? 0 : stage + 1;
      phase ^= stage == 0;
    }
  }
  if constexpr (!CLUSTER) {
    // Runs without tiles are the last ones, but nothing says that CTAs start in that order: others may be left behind one.  They are
    // begun as the first one was; the ring goes on where it is, a round later (its other stages were asked for nothing).
    if (f_empty) {
      run = find(f_answers);
      if (run.left > 0) {
        if (tid == 0) ask(f_answers);
        f = run;
        f_more = true;
        f_empty = false;
        phase ^= 1u;
        goto begin;
      }
    }
  }

  if constexpr (CLUSTER) {
    if (C == 1) return;
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    // four threads per four output values, each over every fourth CTA's share
    const int32_t quads = D / C / 4, part = tid & 3, items = nh * quads * 4;
    const float vs = a.v_scale ? a.v_scale[g] : 1.f;
    for (int32_t x0 = 0; x0 < items; x0 += kThreads) {
      const int32_t x = x0 + tid, y = min(x, items - 1), h = (y >> 2) / quads, c = (y >> 2) % quads;
      float mi[kDpClusterMax / 4], li[kDpClusterMax / 4], top = -INFINITY;
#pragma unroll
      for (int k = 0; k < kDpClusterMax / 4; ++k) {
        const int32_t j = part + 4 * k;
        const float2 ml = j < C ? *reinterpret_cast<const float2*>(s_pml[j][h]) : make_float2(0.f, 0.f);
        mi[k] = ml.x;
        li[k] = ml.y;
        top = fmaxf(top, dp_seen(ml.x, ml.y));
      }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const float ref = dp_finite(top);
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
      float l = 0.f;
#pragma unroll
      for (int k = 0; k < kDpClusterMax / 4; ++k) {
        const int32_t j = part + 4 * k;
        if (j < C) {
          const float wgt = dp_weight(mi[k], li[k], ref);
          const float4 v = *reinterpret_cast<const float4*>(s_part + ((j * nh + h) * quads + c) * 4);
          acc.x = fmaf(wgt, v.x, acc.x); acc.y = fmaf(wgt, v.y, acc.y); acc.z = fmaf(wgt, v.z, acc.z); acc.w = fmaf(wgt, v.w, acc.w);
          l = fmaf(wgt, li[k], l);
        }
      }
#pragma unroll
      for (int d = 1; d <= 2; d *= 2) {
        acc.x += __shfl_xor_sync(0xffffffffu, acc.x, d);
        acc.y += __shfl_xor_sync(0xffffffffu, acc.y, d);
        acc.z += __shfl_xor_sync(0xffffffffu, acc.z, d);
        acc.w += __shfl_xor_sync(0xffffffffu, acc.w, d);
        l += __shfl_xor_sync(0xffffffffu, l, d);
      }
      if (part == 0 && x < items) {
        const int64_t hq = (int64_t)run.r * a.n_q_heads + h0 + h;
        const float inv = dp_over(vs, l);
        dp_store4(reinterpret_cast<Out*>(a.o) + hq * D + (rank * quads + c) * 4, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
        if (rank == 0 && c == 0 && a.lse) a.lse[hq] = dp_lse(ref, l);
      }
    }
  }
}

// Joins the parts of the requests that cuts went through: grid (runs / J, heads of a tile / HPB).  A block looks after J runs' chains, one
// after the other, and HPB heads of each: D / 4 threads per head, and as many groups of those as 256 threads hold.  A group takes AO parts
// at a time, all loads of which are asked for before the first is used, and runs a softmax of its own over them; the groups meet in
// shared memory.  OCC blocks per SM.  Requests without rows get their zeros here.
template <typename Out, int D, int R, int HPB, int J, int AO, int OCC>
__global__ void __launch_bounds__(256, OCC) decode_paged_join_kernel(const __grid_constant__ DecodePagedArgs a) {
  constexpr int kHead = D / 4, kGroup = HPB * kHead, kGroups = 256 / kGroup, kAtOnce = AO;
  static_assert(kGroups >= 1, "a head's columns fit a block");
  __shared__ float s_ml[kGroups][HPB][2];
  __shared__ __align__(16) float4 s_acc[kGroups][kGroup];
  const int32_t grp = threadIdx.x / kGroup, in_grp = threadIdx.x % kGroup, hb = in_grp / kHead, c = in_grp % kHead, h = blockIdx.y * HPB + hb;
  const int32_t runs = a.v_heads * (a.n_long + a.n_short);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  ChainRecord chains[J];
#pragma unroll
  for (int k = 0; k < J; ++k) {
    const int32_t b = blockIdx.x + k * gridDim.x;  // (neighbours begin the same request for different heads)
    chains[k] = b < runs ? reinterpret_cast<const ChainRecord*>(a.chains)[b] : ChainRecord{};
  }
  for (int32_t r = blockIdx.x; r < a.n_req; r += gridDim.x) {
    const int32_t len = a.view.seq_lens[r];
    if (len > a.view.capacity() && blockIdx.y == 0 && threadIdx.x == 0) atomicExch(a.status, (int32_t)PUREKV_ERR_BAD_PAGE);
    if (min(len, a.view.capacity()) > 0) continue;
    for (int32_t hq = h; hq < a.n_q_heads; hq += gridDim.y * HPB)
      if (grp == 0) {
        dp_store4(reinterpret_cast<Out*>(a.o) + ((int64_t)r * a.n_q_heads + hq) * D + 4 * c, make_float4(0.f, 0.f, 0.f, 0.f));
        if (c == 0 && a.lse) a.lse[(int64_t)r * a.n_q_heads + hq] = -INFINITY;
      }
  }
#pragma unroll
  for (int which = 0; which < J; ++which) {
    const ChainRecord chain = chains[which];
    const int64_t first = blockIdx.x + (int64_t)which * gridDim.x;
    // the same for the block.  (A record is always whole, unless a wait ran out or the lengths changed under the kernels: then it may be
    // anything, and nothing follows it anywhere.)
    if (chain.parts <= 0 || chain.r < 0 || chain.r >= a.n_req || chain.vh < 0 || chain.vh >= a.v_heads || first + (int64_t)(chain.parts - 1) * a.v_heads >= runs)
      continue;
    const int32_t g = a.blocks == 1 ? chain.vh : chain.vh / a.blocks, b = chain.vh - g * a.blocks, nh = min(R, a.group - b * R);
    float ref = -INFINITY, l = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int32_t i0 = grp; i0 < chain.parts && h < nh; i0 += kAtOnce * kGroups) {
      float mi[kAtOnce], li[kAtOnce];
      float4 v[kAtOnce];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const int32_t i = i0 + k * kGroups;
        mi[k] = -INFINITY;
        li[k] = 0.f;
        v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i < chain.parts) {
          const float* slot = a.part + (2 * (first + (int64_t)i * a.v_heads) + (i == 0 ? 1 : 0)) * dp_part_floats(R, D);
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
    if constexpr (kGroups > 1) {
      if (c == 0) {
        s_ml[grp][hb][0] = ref;
        s_ml[grp][hb][1] = l;
      }
      s_acc[grp][in_grp] = acc;
      __syncthreads();
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < kGroups; ++i) top = fmaxf(top, dp_seen(s_ml[i][hb][0], s_ml[i][hb][1]));
      ref = dp_finite(top);
      acc = make_float4(0.f, 0.f, 0.f, 0.f);
      l = 0.f;
#pragma unroll
      for (int i = 0; i < kGroups; ++i) {
        const float w = dp_weight(s_ml[i][hb][0], s_ml[i][hb][1], ref);
        const float4 v = s_acc[i][in_grp];
        l = fmaf(w, s_ml[i][hb][1], l);
        acc.x = fmaf(w, v.x, acc.x); acc.y = fmaf(w, v.y, acc.y); acc.z = fmaf(w, v.z, acc.z); acc.w = fmaf(w, v.w, acc.w);
      }
      __syncthreads();
    }
    if (grp == 0 && h < nh) {
      const int64_t hq = (int64_t)chain.r * a.n_q_heads + g * a.group + b * R + h;
      const float inv = dp_over(a.v_scale ? a.v_scale[g] : 1.f, l);
      dp_store4(reinterpret_cast<Out*>(a.o) + hq * D + 4 * c, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
      if (c == 0 && a.lse) a.lse[hq] = dp_lse(dp_finite(ref), l);
    }
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

template <class E, int W, int ST, DpLoad LOAD, int OCC>
static purekv_status launch_even(const DecodePagedArgs& a, int32_t cl, cudaStream_t stream) {
  auto kernel = decode_paged_kernel<E, W, ST, true, LOAD, OCC>;
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
  PK_CUDA(cudaLaunchKernelEx(&l.cfg, kernel, a, DpMaps{}));
  return PUREKV_OK;
}

template <class E, int W, int ST, DpLoad LOAD, int OCC>
static purekv_status launch_balanced(const DecodePagedArgs& a, const DpMaps& maps, cudaStream_t stream) {
  auto kernel = decode_paged_kernel<E, W, ST, false, LOAD, OCC>;
  static std::atomic<uint64_t> smem_allowed{0};
  const purekv_status st = allow_max_dynamic_smem(kernel, smem_allowed);
  if (st != PUREKV_OK) return st;
  const int32_t runs = a.v_heads * (a.n_long + a.n_short);
  DpLaunch l(dim3((unsigned)runs), W * 32, (size_t)W * dp_warp_bytes<E, ST>() + (LOAD == kDpEngine ? 1024 : 0), stream);
  PK_CUDA(cudaLaunchKernelEx(&l.cfg, kernel, a, maps));
  // What cuts can go through are segments, a request's tiles of one head.  Short chains, of up to five parts on average: a block
  // each, all heads, few registers.  Longer ones: two heads and four chains a block.  Few, of very many parts: a head each.  Decode of 128
  // requests of 2900-5100 rows, us, by these three: 164, 169, 182 (e4m3 168, 171, 184); one of 60 000 rows among 63 of 100-2000: 61, 58, 65; 128 of
  // 2900-5100 with 4 heads in e4m3: 98, 103; two of 150-250 thousand: 250, 236, 235.
  const int64_t segments = (int64_t)a.n_req * a.v_heads;
  const int32_t heads = std::min(E::R, a.group);
  auto join = [&](auto kernel, int32_t chains, int32_t heads_each) -> purekv_status {
    DpLaunch j(dim3((unsigned)((runs + chains - 1) / chains), (unsigned)((heads + heads_each - 1) / heads_each)), 256, 0, stream);
    PK_CUDA(cudaLaunchKernelEx(&j.cfg, kernel, a));
    return PUREKV_OK;
  };
  using Out = typename E::Out;
  constexpr int kWide = E::R < 8 ? E::R : 8;
  if (segments * 4 >= runs) return join(decode_paged_join_kernel<Out, E::D, E::R, kWide, 1, 4, 4>, 1, kWide);
  if (segments * 16 >= runs) return join(decode_paged_join_kernel<Out, E::D, E::R, 2, 4, 4, 4>, 4, 2);
  return join(decode_paged_join_kernel<Out, E::D, E::R, 1, 8, 8, 1>, 8, 1);
}

// How a call is launched: C CTAs per (request, head) in a cluster, or, with 0, the balanced form with so many long and short runs of a
// head.
struct DpForm {
  int32_t cluster, at_once, n_long, n_short;
  int32_t per_sm = 1;  // even form, CTAs of a head: 1 alone on its SM; 2 of four warps, two or three per SM; with rings of one stage 3 of four, 4 of eight
};
// Measured over 1-128 requests of 16-64 000 rows, 4 and 2 KV heads, all three types (us).  A CTA alone on its SM streams 75 GB/s, all
// together 6.3 TB/s; the even form costs 4 us besides, the balanced one 14.  Clusters: as many CTAs as find an SM each (128, or 64 for
// clusters of eight and more: 8 requests of 1200 bf16 rows 7.7 with 4 CTAs each, 16 with 8), but not for less than 130 KB of
// a head's rows (200 bf16 rows: 4.7 with one CTA, 5.0 with 4; 500: 7.3 and 5.1), and no pairs for less than 200 KB (64 heads of 300
// rows: 6.2 alone, 6.9 in pairs; of 500 7.8 and 6.9).  Balanced from 380 MB on, which is 60 us: the even form may still be level there if all
// requests are as long as the longest, but nothing says so (128 of 2900-5100 rows: 167 against 173; one of 60 000 among 63 of 100-2000: 57
// against 450), and where the even form's longest share takes longer (one request of 64 000 rows, 4 heads: 39 against 36, in e4m3 26 and 25).  Lengths are
// unknown here but for the longest: a batch with one long request among short ones is taken for as much work as if all were as long (63 of 200
// rows and one of 6000, one head: 28, 17 in the balanced form, which a hint of 0 gives).
static DpForm dp_form(int64_t n_req, int64_t v_heads, int64_t longest, int32_t head_dim, purekv_dtype held, int32_t at_once) {
  const int64_t row_bytes = 2 * head_dim * bytes_of(held);
  const int64_t base = n_req * v_heads, bytes = longest * row_bytes;  // of one head's rows
  int32_t c = 1;
  if (bytes > 130000) {
    while (c < kDpClusterMax && longest > 64 * c && base * 2 * c <= (c < 4 ? 128 : 64)) c *= 2;
    if (c == 2 && bytes <= 200000) c = 1;
  }
  const double all = (double)base * bytes / 6.3e6, share = (double)((base * c + 147) / 148) * bytes / c / 75e3;
  if (all < 60. && std::max(all, share) + 4. < all + 14.) {
    // more heads than SMs: several CTAs on each, so that one streams while another starts or ends.  Requests of one trip of four warps,
    // or of eight, take rings of one stage (4, e4m3 8 KV heads, us, against eight warps with a ring of three: 128 requests of 100-200 rows 18
    // and 28); others two or three CTAs of four warps (128 requests of 300-500 bf16 rows 25 and 30, e4m3 18 and 25).
    const int32_t one_trip = held == PUREKV_E4M3 ? 256 : 128;
    const int32_t per_sm = base <= 148 ? 1 : longest <= 64 ? 3 : longest <= one_trip && held != PUREKV_FP32 ? 4 : longest > 2048 ? 1 : 2;
    return {c, 0, 0, 0, per_sm};
  }
  // (no short runs, but one to be at hand, where the longest requests to be expected would not make any)
  const int64_t shorts = longest < INT32_MAX && n_req * ((longest + 63) / 64) * v_heads <= RunCuts::kFew * at_once ? v_heads : kDpShorts * at_once;
  return {0, at_once, (int32_t)std::max<int64_t>(1, at_once / v_heads), (int32_t)((shorts + v_heads - 1) / v_heads)};
}

// The pools for the copy engine; false where it cannot take them.
template <class E>
static bool dp_maps(const DecodePagedArgs& a, int32_t n_kv_heads, DpMaps* maps) {
  const tc::EncodeTiledFn encode = tc::encode_fn();
  if (!encode || a.view.n_pages == 0) return false;
  constexpr cuuint32_t kInner = E::RowBytes < 128 ? E::RowBytes : 128, kParts = E::RowBytes / kInner;
  auto stride = [](int64_t s) { return (cuuint64_t)(s > 0 ? s : E::RowBytes); };  // (0: a dimension of size 1)
  const cuuint64_t dims[5] = {kInner, (cuuint64_t)a.view.page_size.d, kParts, (cuuint64_t)n_kv_heads, (cuuint64_t)a.view.n_pages};
  const cuuint64_t strides[4] = {stride(a.view.token_stride), 128, stride(a.view.head_stride), stride(a.view.page_stride)};
  const bool whole = a.view.page_size.d % E::TK == 0;
  if (!whole && (E::TK % a.view.page_size.d || a.view.page_size.d < 8)) return false;  // (the swizzle repeats every eight rows)
  maps->boxes = whole ? 1 : E::TK / (int32_t)a.view.page_size.d;
  const cuuint32_t box[5] = {kInner, (cuuint32_t)(E::TK / maps->boxes), whole ? kParts : 1, 1, 1}, each[5] = {1, 1, 1, 1, 1};
  const uint8_t* pools[2] = {a.k_pool, a.v_pool};
  CUtensorMap* out[2] = {&maps->k, &maps->v};
  for (int i = 0; i < 2; ++i)
    if (encode(out[i], CU_TENSOR_MAP_DATA_TYPE_UINT8, 5, const_cast<uint8_t*>(pools[i]), dims, strides, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE,
               kInner == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
               kParts > 1 ? CU_TENSOR_MAP_L2_PROMOTION_L2_256B : kInner == 128 ? CU_TENSOR_MAP_L2_PROMOTION_L2_128B : CU_TENSOR_MAP_L2_PROMOTION_L2_64B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return false;
  return true;
}

// E: the engine for rows copied by threads; X: the same for rows that the copy engine brings.  ST8 and ST4: stages of each warp with
// eight warps in a CTA and with two CTAs of four.
template <class E, class X, int ST8, int ST4, int OCC4>
static purekv_status launch_rows(const DecodePagedArgs& a, int32_t n_kv_heads, const DpForm& f, cudaStream_t stream) {
  const bool whole = a.view.page_size.d % E::TK == 0;
  if (f.cluster && f.per_sm == 3) return launch_even<E, 4, 1, kDpRows, (E::R > 8 ? 2 : 3)>(a, f.cluster, stream);
  if constexpr (E::RowBytes < 4 * E::D) {  // (dp_form has no such CTAs for fp32)
    if (f.cluster && f.per_sm == 4) return launch_even<E, 8, 1, kDpRows, (E::R > 8 ? 1 : 2)>(a, f.cluster, stream);
  }
  if (f.cluster && f.per_sm == 2) return launch_even<E, 4, (OCC4 == 3 ? 2 : 3), kDpRows, OCC4>(a, f.cluster, stream);
  if (f.cluster) return whole ? launch_even<E, 8, ST8, kDpWhole, 1>(a, f.cluster, stream) : launch_even<E, 8, ST8, kDpRows, 1>(a, f.cluster, stream);
  DpMaps maps = {};
  if (dp_maps<X>(a, n_kv_heads, &maps)) return launch_balanced<X, 4, ST4, kDpEngine, OCC4>(a, maps, stream);
  return launch_balanced<E, 4, OCC4 == 3 ? 2 : ST8, kDpRows, OCC4>(a, maps, stream);
}


static int32_t dp_rows(int32_t group, purekv_dtype dtype) { return dtype == PUREKV_FP32 ? (group <= 2 ? 2 : 8) : group <= 8 ? 8 : 16; }

// CTAs of the balanced form at work: two per SM, or three where the products and not the loads take the time: of e4m3, which has to
// become fp16, with up to eight heads (128 requests of 2900-5100 rows, 8 KV heads, call after call under the power cap, us: pages of 16 rows 197 with two, 178 with three; of 64 rows 183 and 173).
constexpr int dp_ctas(bool e4m3, int rows) { return e4m3 && rows == 8 ? 3 : 2; }
static int32_t dp_at_once(int32_t rows, purekv_dtype held) { return 148 * dp_ctas(held == PUREKV_E4M3, rows); }

static int64_t dp_ws(const DpForm& f, int64_t v_heads, int32_t group, int32_t head_dim, purekv_dtype dtype) {
  if (f.cluster) return 0;
  const int64_t runs = v_heads * (f.n_long + f.n_short);
  return 256 + runs * (int64_t)sizeof(ChainRecord) + 2 * runs * dp_rows(group, dtype) * (head_dim + 2) * 4;
}

}  // namespace purekv

using namespace purekv;

extern "C" {

size_t purekv_decode_paged_ws_bytes(int32_t n_req, int32_t max_len, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                    purekv_dtype dtype) {
  if (n_req <= 0 || n_q_heads <= 0 || n_kv_heads <= 0 || n_q_heads % n_kv_heads || head_dim <= 0) return 0;
  const int32_t group = n_q_heads / n_kv_heads, rows = dp_rows(group, dtype), blocks = (group + rows - 1) / rows;
  const int64_t v_heads = (int64_t)n_kv_heads * blocks;
  // (of the pools' types that go with dtype, e4m3 has the shorter rows: either may need the larger workspace)
  const int64_t longest = max_len > 0 ? max_len : INT32_MAX;
  auto need = [&](purekv_dtype held) {
    const DpForm f = dp_form(n_req, v_heads, longest, head_dim, held, dp_at_once(rows, held));
    return dp_ws(f, v_heads, group, head_dim, dtype);
  };
  return (size_t)std::max(need(dtype), dtype == PUREKV_FP32 ? 0 : need(PUREKV_E4M3));
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
  const DpForm form = dp_form(a.n_req, a.v_heads, max_len > 0 ? max_len : INT32_MAX, pages->head_dim, pages->dtype,
                              dp_at_once(rows, pages->dtype));
  if (!form.cluster) {
    PK_REQUIRE(ws && ws_bytes >= (size_t)dp_ws(form, a.v_heads, a.group, pages->head_dim, dtype), PUREKV_ERR_WORKSPACE,
               "%s: workspace of %zu bytes is too small", kName, ws_bytes);
    a.chains = (int32_t*)(((uintptr_t)ws + 255) & ~(uintptr_t)255);
    a.at_once = form.at_once;
    a.n_long = form.n_long;
    a.n_short = form.n_short;
    a.wait_ns = wait_limit_ns();
    a.part = (float*)(a.chains + (int64_t)a.v_heads * (a.n_long + a.n_short) * (sizeof(ChainRecord) / 4));
  }
  if (!status) {
    const purekv_status s2 = default_status_word(kWordPaged, &a.status);
    if (s2 != PUREKV_OK) return s2;
  }
  cudaStream_t sm = (cudaStream_t)stream;
  const bool wide = pages->head_dim == 128;
  // rows of a trip: 8 KB of K and V, or 4 where threads look a row up each
#define PK_FP32(D, N) launch_rows<Fp32Rows<D, N, false>, Fp32Rows<D, N, true>, 3, 3, 2>(a, pages->n_kv_heads, form, sm)
#define PK_ROWS(ENGINE, D, N, MT, MT4, ST8, ST4, OCC4) launch_rows<ENGINE<D, N, MT, false>, ENGINE<D, N, MT4, true>, ST8, ST4, OCC4>(a, pages->n_kv_heads, form, sm)
  if (dtype == PUREKV_FP32) {
    if (rows == 2) return wide ? PK_FP32(128, 2) : PK_FP32(64, 2);
    return wide ? PK_FP32(128, 8) : PK_FP32(64, 8);
  }
  if (pages->dtype == PUREKV_E4M3) {
    if (rows == 8) return wide ? PK_ROWS(E4m3Rows, 128, 1, 2, 2, 3, 2, 3) : PK_ROWS(E4m3Rows, 64, 1, 2, 4, 5, 2, 3);
    return wide ? PK_ROWS(E4m3Rows, 128, 2, 2, 2, 2, 3, 2) : PK_ROWS(E4m3Rows, 64, 2, 2, 4, 5, 3, 2);
  }
  if (rows == 8) return wide ? PK_ROWS(Bf16Rows, 128, 1, 1, 1, 3, 3, 2) : PK_ROWS(Bf16Rows, 64, 1, 1, 2, 5, 3, 2);
  return wide ? PK_ROWS(Bf16Rows, 128, 2, 1, 1, 3, 3, 2) : PK_ROWS(Bf16Rows, 64, 2, 1, 2, 5, 3, 2);
#undef PK_FP32
#undef PK_ROWS
}

}  // extern "C"
