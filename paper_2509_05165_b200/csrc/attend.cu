// Attention of a few query rows over an 8-bit cache (kvc_attend).
//
// HBM is the bound: 2 d bytes of codes per token and KV head, against 4 d products per query row.  Two kernels, three with weights:
//
// attend_split_kernel   one CTA per SM.  The tokens of all heads, in granules of kGranule (and kSetup granules more per head,
//   for what starting one costs), are laid end to end and cut into equal shares, one per CTA, whatever the lengths.  A CTA
//   whose share lies within one head spreads it over its warps, 32 tokens each in turn, and joins their results; one that
//   holds several heads cuts its share once more, one piece per warp, and each warp works for itself.  A lane copies the very
//   16-byte pieces it will use (cp.async into its own places in shared memory, kStages deep, no barrier), turns the codes into
//   fp16 and feeds mma.m16n8k16: S^T = K Q^T with the tokens as rows, then O^T = V^T P^T, eight query rows to a column tile
//   (kTiles of them share the converted codes).  Operand layouts: the order of the summed index is free as long as both
//   operands agree, so lane (g, t) takes token g's entries 16 t .. 16 t + 15 of each 64 as its k slots, and entries (d / 8) g ..
//   of its tokens of V as its rows; a transpose of P's 8 x 8 tiles (movmatrix) is the only exchange between lanes.  Legacy
//   mma on purpose: while HBM brings a token's codes, the scheduler that will work on it has 44 clocks, and eight query rows take
//   8 of them in mma (8.0 per m16n8k16, measured).  Through tcgen05 the converted codes have to go back to shared memory first and
//   change hands between roles, 1.4 us per 128 tokens of waits alone: 109 us for the four rows over 128K tokens below, 41 for 32K
//   tokens, in the form that was tried.
// attend_join_kernel    joins the parts of a row (log-sum-exp).
// attend_weight_kernel  adds the rows' weights from the logits, which the first kernel leaves in the workspace (they stay in L2; the
//   softmax's denominator is known only after the last token).
//
// Numbers: codes are exact in fp16.  A query row is scaled by a power of two to below 2 and rounded to fp16, which is exact
// for bf16 but for entries 2^17 times smaller than the row's largest (fp16's smallest step is 2^-24, a bf16 has 8 bits); fp32
// rows go as two fp16 (within 2^-23 of the row's largest entry), and so does P in front of V then (22 bits).  For bf16 outputs P is
// one fp16: 11 bits, off by at most 2^-11 of sum p |v| where the output's own rounding is 2^-8 of its value, for half the
// products with V.  Products, softmax and sums are fp32; log-sum-exps and weights take P before it is rounded.  V's exponents differ from block
// to block: P goes in relative to 2^M, M a running maximum of logit + exponent, which keeps the largest terms of a row at
// full precision whatever block they are in, and 2^5 times larger, so that 2^17 weights of 2^-26 are not lost beside one of
// 1/2, as they are in an fp16 of at most 1.  References only move when they are exceeded by 2^10 (2^60 for the sums): until
// then no lane needs another's maximum (with a maximum per step, four rows over 128K tokens took 79 us instead of 68).
//
// B200: 8 sequences of 32768 tokens, 8 heads of 128, one row of 32 query heads 89 us (537 MB of codes, 6.0 TB/s); one such
// sequence with weights 22.6 us, of which about 7 are the launches' own; four rows of 28 query heads over 131072 tokens of 4 heads
// 55 us (2.4 TB/s): latency.  The accumulators fill the registers, and the two warps per scheduler that this leaves issue in a third
// of the cycles (mma pipe 31 %, DRAM 31 %): a step's products with K, its softmax and its products with V follow one another.
#include <math.h>

#include "cache8.cuh"

namespace kvc {
namespace {

constexpr int kGranule = 64;              // tokens: unit of the split
constexpr int kSetup = 2;                 // granules that a head's start counts as
constexpr int kAttWarps = 8;              // (12 with fewer registers each: 32 ragged sequences 51 -> 53 us, four rows over 128K tokens in two
                                          // tiles of 16 64 -> 77)
constexpr int kMaxCtas = 256;             // bounds the workspace, whatever the device
constexpr int kMaxRows = 64;              // query rows of a KV head that one launch takes (bounds the logits kept)
constexpr float kSlackSum = 60.f;         // logits may exceed the reference of the sums by this much (see Form for V's)
constexpr float kNone = -3e38f;           // "no logit yet": finite, so that differences are numbers
constexpr int kJoinThreads = 256;
constexpr int kJoinWarps = kJoinThreads / 32;
constexpr int kJoinEach = 4;              // tokens of a thread
constexpr int kJoinTokens = kJoinThreads * kJoinEach;

struct AttendParams {
  Cache c;
  int Hq, G, rows, causal;
  float scale;
  long long qs[3], os[3];
  // of this launch: query rows row0 .. row0 + live - 1 of the G * rows of a KV head, in row_tiles tiles of 8 * kTiles
  int row0, live, row_tiles, tile_rows, ctas, warps, logit_rows, device;
  float* part_o;                          // [slot][tile_rows][d]
  float2* part_ml;                        // [slot][tile_rows]: largest logit (in powers of two), sum of 2^(logit - it)
  float* logits;                          // [unit][row tile][token][logit_rows]
  float* lse2;                            // [unit][live]
  int* before;                            // [units + 1]: granules (with kSetup) in front of a head, per row tile; all of them last
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void mma16816(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// Four codes as two pairs of fp16.
template <int kFormat>
__device__ __forceinline__ void to_half2(uint32_t w, uint32_t* lo, uint32_t* hi) {
  if (kFormat == KVC_E4M3) {
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(*lo) : "h"((uint16_t)w));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(*hi) : "h"((uint16_t)(w >> 16)));
  } else {
    // 0x6400 + u is 1024 + u in fp16; u = code + 128
    const uint32_t u = w ^ 0x80808080u;
    const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
    const __half2 off = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));
    const __half2 x = __hsub2(*reinterpret_cast<const __half2*>(&a), off), y = __hsub2(*reinterpret_cast<const __half2*>(&b), off);
    *lo = *reinterpret_cast<const uint32_t*>(&x);
    *hi = *reinterpret_cast<const uint32_t*>(&y);
  }
}

// (through L1: K's copies touch half a line each, the other half by the next copy; past L1 a cache larger than L2 came in at 4.6
// TB/s instead of 6.0)
template <int kBytes>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, bool live) {
  if (kBytes == 16)
    asm volatile("cp.async.ca.shared.global.L2::256B [%0], [%1], 16, %2;" :: "r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
  else
    asm volatile("cp.async.ca.shared.global.L2::128B [%0], [%1], 8, %2;" :: "r"(dst), "l"(src), "r"(live ? 8 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int n>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(n) : "memory"); }

__device__ __forceinline__ int row_count(const AttendParams& P, const int32_t* row_counts, int b) {
  const int n = row_counts == nullptr ? P.rows : row_counts[b];
  return n < 0 ? 0 : (n > P.rows ? P.rows : n);
}
// Tokens that row rr (of the G * rows of a KV head) sees; -1: there is no such row.
__device__ __forceinline__ long long tokens_seen(const AttendParams& P, int rr, int last, int rows, long long len) {
  const int m = rr % P.rows;
  if (rr >= last || m >= rows) return -1;
  const long long n = P.causal ? len - (rows - 1 - m) : len;
  return n < 0 ? 0 : n;
}
// Granules of a head's row tile, what starting it costs included.
__device__ __forceinline__ int granules(long long len) { return len == 0 ? 0 : (int)((len + kGranule - 1) / kGranule) + kSetup; }

// `total` granules (of all heads and row tiles: under 2^31, see resolve_attend) cut into `parts` shares, as many of them as there are
// granules at most: share i, and the share of a place.  The first `more` shares hold one granule more than the others.
struct Shares {
  uint32_t each, more;
  int parts;
  __device__ __forceinline__ Shares(int total, int parts_) : parts(min(total, parts_)) {
    each = (uint32_t)total / (uint32_t)parts;
    more = (uint32_t)total - each * parts;
  }
  __device__ __forceinline__ int begin(int i) const { return (int)(each * i + min((uint32_t)i, more)); }
  __device__ __forceinline__ int of(int place) const {
    const uint32_t larger = more * (each + 1);
    return (uint32_t)place < larger ? (uint32_t)place / (each + 1) : more + ((uint32_t)place - larger) / each;
  }
};

// Warps, stages and shared memory of a form of attend_split_kernel.
template <typename T, int kD, int kTiles>
struct Form {
  static constexpr bool kTwo = sizeof(T) == 4;         // fp32: Q and P as two fp16 each
  // P goes into V as 2^kLift p, relative to a reference that it may exceed by 2^kSlack: 2^15 fits fp16, and its smallest steps are
  // 2^-29 of the row's largest weight (fp32: 2^-36, at the price of references that move more often)
  static constexpr float kLift = kTwo ? 12.f : 5.f, kSlack = kTwo ? 3.f : 10.f;
  static constexpr bool kQShared = kTiles == 4;        // Q's operands in shared memory (else in registers)
  static constexpr int kWarps = kAttWarps;
  static constexpr int kHalves = kTiles == 4 ? 1 : 2;  // a step's 32 tokens at once, or 16 by 16 (four tiles: the registers)
  static constexpr int kThreads = kWarps * 32;
  static constexpr int kSteps = kD / 16;               // k steps of Q K^T, and row tiles of V^T
  static constexpr int kKPieces = kD / 64;             // 16-byte pieces of a token's K per lane
  static constexpr int kVBytes = kD / 8;               // a lane's bytes of a token's V
  static constexpr int kStages = kD == 128 ? 2 : 3;
  static constexpr int kStageBytes = 32 * 2 * kD;      // per warp: 32 tokens of K and V
  static constexpr int kVBase = 32 * kD;
  static constexpr int kRows = 8 * kTiles;
  static constexpr int kPitch = kD + 4;
  static constexpr int kQBytes = kQShared ? kTiles * kSteps * 32 * 8 : 0;      // per warp
  static constexpr int kWarpBytes = kStages * kStageBytes + kQBytes;
  static constexpr int kJoinBytes = kWarps * kRows * kPitch * 4;
  static constexpr int kSmem = kWarps * kWarpBytes > kJoinBytes ? kWarps * kWarpBytes : kJoinBytes;
};

template <typename T, int kFormat, int kD, int kTiles, bool kWeight>
__global__ void __launch_bounds__(Form<T, kD, kTiles>::kThreads, 1)
attend_split_kernel(const __grid_constant__ AttendParams P, const T* __restrict__ q, const int32_t* __restrict__ row_counts) {
  using F = Form<T, kD, kTiles>;
  constexpr bool kTwo = F::kTwo;
  constexpr int kWarps = F::kWarps, kThreads = F::kThreads, kSteps = F::kSteps, kStages = F::kStages, kRows = F::kRows, kPitch = F::kPitch, kH = F::kHalves;
  extern __shared__ __align__(128) char smem[];
  __shared__ int s_sum[kWarps];
  __shared__ int s_unit[kWarps + 1], s_before[kWarps + 1];      // the head that each warp's piece starts in; last: the whole share's
  __shared__ float s_stat[kWarps][kRows][2];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  grid_dependency_wait();
  const Cache& c = P.c;
  const int units = c.units();

  // ---- this CTA's share, and the heads that it and its warps' pieces start in
  const int per = (units + kThreads - 1) / kThreads;
  const int u0 = tid * per, u1 = min(u0 + per, units);
  int mine = 0;
  for (int u = u0; u < u1; ++u) mine += granules(c.length(u));
  int incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += y;
  }
  if (lane == 31) s_sum[warp] = incl;
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const int y = s_sum[w];
    if (w < warp) incl += y;
    total += y;
  }
  if (blockIdx.x == 0) {                               // for attend_join_kernel
    int b = incl - mine;
    for (int u = u0; u < u1; ++u) {
      P.before[u] = b;
      b += granules(c.length(u));
    }
    if (tid == 0) P.before[units] = total;
  }
  total *= P.row_tiles;
  if (total == 0) return;
  const Shares ctas(total, P.ctas);
  if ((int)blockIdx.x >= ctas.parts) return;
  const int share0 = ctas.begin(blockIdx.x), share1 = ctas.begin(blockIdx.x + 1);
  // the head that holds place p: found by the thread that has it
  auto find = [&](int p, int which) {
    int v = (incl - mine) * P.row_tiles;
    if (v > p || p >= incl * P.row_tiles) return;
    for (int u = u0;; ++u) {
      const int n = granules(c.length(u)) * P.row_tiles;
      if (p < v + n) {
        s_unit[which] = u;
        s_before[which] = v;
        return;
      }
      v += n;
    }
  };
  find(share0, kWarps);
  __syncthreads();
  int at = share0, end = share1;                       // the place, and its end
  int unit = s_unit[kWarps], before = s_before[kWarps];        // .. and where the row tile begins that it lies in
  int len = (int)c.length(unit), n_gran = granules(len);
  int rt = P.row_tiles > 1 ? (at - before) / n_gran : 0;
  before += rt * n_gran;
  // within one row tile of one head: all warps work on it together; else each on a piece of its own
  const bool together = share1 <= before + n_gran;
  if (!together) {
    const Shares pieces(share1 - share0, kWarps);
    for (int w = 0; w < pieces.parts; ++w) find(share0 + pieces.begin(w), w);
    __syncthreads();
    if (warp >= pieces.parts) return;                  // (no barrier follows for a CTA of several heads)
    at = share0 + pieces.begin(warp);
    end = share0 + pieces.begin(warp + 1);
    unit = s_unit[warp];
    before = s_before[warp];
    len = (int)c.length(unit);
    n_gran = granules(len);
    rt = P.row_tiles > 1 ? (at - before) / n_gran : 0;
    before += rt * n_gran;
  }
  const int warp_in = together ? warp : 0, warps_in = together ? kWarps : 1;
  const int st = (int)c.st[2];                         // (a row's stride; 31 bits, checked by the host)

  char* my_smem = smem + warp * F::kWarpBytes;
  const uint32_t my_smem_addr = (uint32_t)__cvta_generic_to_shared(my_smem);

  while (true) {
    // ---- a part of one row tile of one head: tokens [lo, hi)
    const int b = unit / c.Hkv, h = unit - b * c.Hkv;
    const int upto = min(end, before + n_gran);
    const int lo = max(at - before - kSetup, 0) * kGranule;
    const int hi = (int)min((long long)max(upto - before - kSetup, 0) * kGranule, (long long)len);
    const int rows = row_count(P, row_counts, b);
    const int first_row = P.row0 + rt * kRows, last_row = min(P.row0 + P.live, first_row + kRows);
    const int live_rows = last_row - first_row;

    if (hi > lo) {
    const int8_t *ke = c.k_exp + (long long)unit * c.blocks, *ve = c.v_exp + (long long)unit * c.blocks;
    const int stride = 32 * warps_in;                  // tokens from one step of a warp to its next
    const int first = lo + 32 * warp_in;
    const int iters = hi > first ? (hi - first + stride - 1) / stride : 0;
    // the lane's places in the next 32 tokens to copy
    const uint8_t* kp = c.k + c.base(unit) + (long long)(first + g) * st + 16 * t;
    const uint8_t* vp = c.v + c.base(unit) + (long long)(first + 2 * t) * st + F::kVBytes * g;
    const long long advance = (long long)stride * st;

    // K, and V, of step `it` into stage it % kStages, each a group of copies.  Rows behind the end are filled with zeros.
    auto fetch_k = [&](int it) {
      if (it < iters) {
        const uint32_t dst = my_smem_addr + (it % kStages) * F::kStageBytes;
        const int left = hi - first - it * stride;     // tokens from this step on
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool live = left >= 32 || 8 * i + g < left;
          const uint8_t* src = live ? kp + (long long)(8 * i) * st : c.k;
#pragma unroll
          for (int p = 0; p < F::kKPieces; ++p) copy_async<16>(dst + ((i * F::kKPieces + p) * 32 + lane) * 16, src + (live ? 64 * p : 0), live);
        }
        kp += advance;
      }
      copy_commit();
    };
    auto fetch_v = [&](int it) {
      if (it < iters) {
        const uint32_t dst = my_smem_addr + (it % kStages) * F::kStageBytes + F::kVBase;
        const int left = hi - first - it * stride;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int tok = 16 * (i >> 2) + 8 * ((i >> 1) & 1) + (i & 1);
          const bool live = left >= 32 || tok + 2 * t < left;
          copy_async<F::kVBytes>(dst + (i * 32 + lane) * F::kVBytes, live ? vp + (long long)tok * st : c.v, live);
        }
        vp += advance;
      }
      copy_commit();
    };
#pragma unroll
    for (int s = 0; s < kStages; ++s) {
      fetch_k(s);
      fetch_v(s);
    }

    // exponents of the two halves of 32 tokens, K's and V's: a lane reads those of one step in 32, four bytes in one register
    uint32_t exps = 0;
    auto fetch_exps = [&](int it) {
      const int tok = first + (it + lane) * stride;
      if (it + lane < iters) {
        const int at0 = tok >> c.block_shift, at1 = min(tok + 16, hi - 1) >> c.block_shift;
        exps = (uint32_t)(uint8_t)__ldg(ke + at0) | (uint32_t)(uint8_t)__ldg(ke + at1) << 8 | (uint32_t)(uint8_t)__ldg(ve + at0) << 16 |
               (uint32_t)(uint8_t)__ldg(ve + at1) << 24;
      }
    };
    fetch_exps(0);

    // ---- Q: row 8 n + g of the tile, its entries in the lane's k slots, scaled by a power of two to below 2
    uint32_t qh[F::kQShared ? 1 : kTiles][kSteps][2], ql[kTwo ? kTiles : 1][kTwo ? kSteps : 1][2];
    uint2* sq = reinterpret_cast<uint2*>(my_smem + kStages * F::kStageBytes) + lane;      // [tile][step][lane]
    float factor[kTiles][2];                           // of the columns 2 t, 2 t + 1: logit = accumulator * factor * 2^ke
    int seen[kTiles][2], seen_least = 0x7fffffff;      // (lengths fit 31 bits)
#pragma unroll
    for (int n = 0; n < kTiles; ++n) {
      const int rr = first_row + 8 * n + g;
      float x[kD / 4];
      float top = 0.f;
      const bool there = tokens_seen(P, rr, last_row, rows, len) >= 0;
      const T* src = q + b * P.qs[0] + (there ? h * P.G + rr / P.rows : 0) * P.qs[1] + (there ? rr % P.rows : 0) * P.qs[2] + 16 * t;
#pragma unroll
      for (int p = 0; p < kD / 64; ++p)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float* y = x + 16 * p + 8 * i;
          if (there) load8<T>(src + 64 * p + 8 * i, y);
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            if (!there) y[u] = 0.f;
            top = fmaxf(top, fabsf(y[u]));
          }
        }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const int e = min(max((int)(__float_as_uint(top) >> 23) - 127, -120), 126);
      // (an infinity makes the whole row NaN, as one does by itself; fmaxf passes NaN over)
      const float down = __float_as_uint(top) < 0x7f800000u ? pow2(-e) : __int_as_float(0x7fffffff), up = pow2(e) * P.scale * 1.44269504088896341f;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        uint32_t w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float a = x[4 * s + 2 * i] * down, z = x[4 * s + 2 * i + 1] * down;
          w[i] = pack_half2(a, z);
          if (kTwo) {
            const __half2 hh = *reinterpret_cast<const __half2*>(&w[i]);
            ql[n][s][i] = pack_half2(a - __low2float(hh), z - __high2float(hh));
          }
        }
        if (F::kQShared) {
          sq[(n * kSteps + s) * 32] = make_uint2(w[0], w[1]);      // (its own lane reads it back)
        } else {
          qh[n][s][0] = w[0];
          qh[n][s][1] = w[1];
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        factor[n][i] = __shfl_sync(0xffffffffu, up, (2 * t + i) * 4);
        seen[n][i] = (int)tokens_seen(P, first_row + 8 * n + 2 * t + i, last_row, rows, len);
        if (seen[n][i] >= 0) seen_least = min(seen_least, seen[n][i]);
      }
    }
    seen_least = __reduce_min_sync(0xffffffffu, seen_least);

    float o[kTiles][kSteps][4], top_s[kTiles][2], top_v[kTiles][2], sum[kTiles][2];
#pragma unroll
    for (int n = 0; n < kTiles; ++n) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[n][s][i] = 0.f;
#pragma unroll
      for (int i = 0; i < 2; ++i) { top_s[n][i] = kNone; top_v[n][i] = kNone; sum[n][i] = 0.f; }
    }
    float* logit_row = nullptr;
    if (kWeight) logit_row = P.logits + ((long long)unit * P.row_tiles + rt) * c.cap * P.logit_rows + 2 * t;

    for (int it = 0; it < iters; ++it) {
      if (it > 0 && (it & 31) == 0) fetch_exps(it);
      const uint32_t four = __shfl_sync(0xffffffffu, exps, it & 31);
      copy_wait<2 * kStages - 1>();                    // K of this step is there; behind it, V and kStages - 1 steps more
      const char* stage = my_smem + (it % kStages) * F::kStageBytes;
#pragma unroll 1
      for (int half = 0; half < 2; half += kH) {       // kH times 16 tokens at once
      const uint32_t mine = half == 0 ? four : four >> 8;
      const int ek[2] = {(int8_t)mine, (int8_t)(mine >> 8)}, ev[2] = {(int8_t)(mine >> 16), (int8_t)(mine >> 24)};
      const int tok0 = first + it * stride + 16 * half;

      // ---- logits, in powers of two: lane holds tokens g and g + 8 (of each 16), columns 2 t and 2 t + 1
      float sc[kH][kTiles][4];
#pragma unroll
      for (int f = 0; f < kH; ++f)
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) sc[f][n][i] = 0.f;
#pragma unroll
      for (int p = 0; p < F::kKPieces; ++p) {
        uint32_t x[2 * kH][4];
#pragma unroll
        for (int i = 0; i < 2 * kH; ++i) {
          const uint4 w = *reinterpret_cast<const uint4*>(stage + (((2 * half + i) * F::kKPieces + p) * 32 + lane) * 16);
          x[i][0] = w.x; x[i][1] = w.y; x[i][2] = w.z; x[i][3] = w.w;
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          uint32_t a[kH][4];
#pragma unroll
          for (int f = 0; f < kH; ++f) {
            to_half2<kFormat>(x[2 * f][s], &a[f][0], &a[f][2]);
            to_half2<kFormat>(x[2 * f + 1][s], &a[f][1], &a[f][3]);
          }
#pragma unroll
          for (int n = 0; n < kTiles; ++n) {
            uint32_t b0, b1;
            if (F::kQShared) {
              const uint2 w = sq[(n * kSteps + 4 * p + s) * 32];
              b0 = w.x; b1 = w.y;
            } else {
              b0 = qh[n][4 * p + s][0]; b1 = qh[n][4 * p + s][1];
            }
#pragma unroll
            for (int f = 0; f < kH; ++f) {
              mma16816(sc[f][n], a[f], b0, b1);
              if (kTwo) mma16816(sc[f][n], a[f], ql[n][4 * p + s][0], ql[n][4 * p + s][1]);
            }
          }
        }
      }
      if (half + kH == 2) fetch_k(it + kStages);       // (into the place just read)
#pragma unroll
      for (int f = 0; f < kH; ++f) {
        const float kf = pow2_clamped(ek[f]);
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) sc[f][n][i] *= factor[n][i & 1] * kf;
      }
      if (tok0 + 16 * kH > seen_least) {
#pragma unroll
        for (int f = 0; f < kH; ++f)
#pragma unroll
          for (int n = 0; n < kTiles; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (tok0 + 16 * f + 8 * (i >> 1) + g >= seen[n][i & 1]) sc[f][n][i] = -INFINITY;
      }
      if (kWeight) {
#pragma unroll
        for (int f = 0; f < kH; ++f)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int tok = tok0 + 16 * f + 8 * i + g;
            if (tok < hi) {
#pragma unroll
              for (int n = 0; n < kTiles; ++n)
                if (8 * n + 2 * t < P.logit_rows)
                  *reinterpret_cast<float2*>(logit_row + (long long)tok * P.logit_rows + 8 * n) = make_float2(sc[f][n][2 * i], sc[f][n][2 * i + 1]);
            }
          }
      }

      // ---- references of the logits and of logit + V's exponent.  They move when a lane finds one exceeded by more than the slack:
      // then to the maxima of these tokens over all lanes, and sums and outputs follow.
      const float evf[2] = {(float)ev[0], (float)ev[1]};
      auto tops = [&](int n, int i, float* ms, float* mv) {      // of the lane's tokens
        *ms = fmaxf(sc[0][n][i], sc[0][n][2 + i]);
        *mv = *ms + evf[0];
        if (kH == 2) {
          const float m1 = fmaxf(sc[kH - 1][n][i], sc[kH - 1][n][2 + i]);
          *ms = fmaxf(*ms, m1);
          *mv = fmaxf(*mv, m1 + evf[1]);
        }
      };
      float over = -INFINITY;
#pragma unroll
      for (int n = 0; n < kTiles; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float ms, mv;
          tops(n, i, &ms, &mv);
          over = fmaxf(over, mv - top_v[n][i] - F::kSlack);
          over = fmaxf(over, ms - top_s[n][i] - kSlackSum);
        }
      if (__any_sync(0xffffffffu, over > 0.f)) {
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float ms, mv;
            tops(n, i, &ms, &mv);
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) {
              ms = fmaxf(ms, __shfl_xor_sync(0xffffffffu, ms, x));
              mv = fmaxf(mv, __shfl_xor_sync(0xffffffffu, mv, x));
            }
            ms = fmaxf(ms, top_s[n][i]);
            mv = fmaxf(mv, top_v[n][i]);
            sum[n][i] *= ex2(top_s[n][i] - ms);
            const float r = ex2(top_v[n][i] - mv);
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
              o[n][s][i] *= r;
              o[n][s][2 + i] *= r;
            }
            top_s[n][i] = ms;
            top_v[n][i] = mv;
          }
      }

      // ---- P, and its share of the outputs
      if (half == 0) copy_wait<2 * kStages - (kH == 2 ? 1 : 2)>();      // V of this step is there (K of a step more has been asked for or not)
#pragma unroll
      for (int f = 0; f < kH; ++f) {
        uint32_t ph[kTiles][2], pl[kTwo ? kTiles : 1][2];
#pragma unroll
        for (int n = 0; n < kTiles; ++n) {
          float up[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) up[i] = top_s[n][i] + evf[f] - top_v[n][i] + F::kLift;
          const bool far = fmaxf(up[0], up[1]) > 100.f;         // (V's exponents so far apart that p may be no fp32 where its product is)
          up[0] = ex2(up[0]);
          up[1] = ex2(up[1]);
          float p[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            p[i] = ex2(sc[f][n][i] - top_s[n][i & 1]);
            sum[n][i & 1] += p[i];
            p[i] *= up[i & 1];
          }
          if (far) {
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = ex2(sc[f][n][i] + (evf[f] - top_v[n][i & 1] + F::kLift));
          }
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t w = pack_half2(p[2 * i], p[2 * i + 1]);
            ph[n][i] = transpose8x8(w);
            if (kTwo) {
              const __half2 hh = *reinterpret_cast<const __half2*>(&w);
              pl[n][i] = transpose8x8(pack_half2(p[2 * i] - __low2float(hh), p[2 * i + 1] - __high2float(hh)));
            }
          }
        }
        const char* sv = stage + F::kVBase + (4 * (half + f) * 32 + lane) * F::kVBytes;
        uint32_t v[4][F::kVBytes / 4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (kD == 128) {
            const uint4 w = *reinterpret_cast<const uint4*>(sv + i * 32 * F::kVBytes);
            v[i][0] = w.x; v[i][1] = w.y; v[i][F::kVBytes / 4 - 2] = w.z; v[i][F::kVBytes / 4 - 1] = w.w;
          } else {
            const uint2 w = *reinterpret_cast<const uint2*>(sv + i * 32 * F::kVBytes);
            v[i][0] = w.x; v[i][1] = w.y;
          }
        }
#pragma unroll
        for (int w = 0; w < F::kVBytes / 4; ++w) {
          // bytes of two tokens side by side: entry 4 w + 2 x (+ 1) of tokens 2 t, 2 t + 1 and of the two 8 further on
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            uint32_t a[4];
            to_half2<kFormat>(__byte_perm(v[0][w], v[1][w], x == 0 ? 0x5140 : 0x7362), &a[0], &a[1]);
            to_half2<kFormat>(__byte_perm(v[2][w], v[3][w], x == 0 ? 0x5140 : 0x7362), &a[2], &a[3]);
#pragma unroll
            for (int n = 0; n < kTiles; ++n) {
              mma16816(o[n][2 * w + x], a, ph[n][0], ph[n][1]);
              if (kTwo) mma16816(o[n][2 * w + x], a, pl[n][0], pl[n][1]);
            }
          }
        }
      }
      }
      fetch_v(it + kStages);
    }
    copy_wait<0>();
#pragma unroll
    for (int n = 0; n < kTiles; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) sum[n][i] += __shfl_xor_sync(0xffffffffu, sum[n][i], x);
    const long long slot = (long long)blockIdx.x * kWarps + (together ? 0 : warp) + (long long)unit * P.row_tiles + rt;

    if (!together) {
      // ---- this warp's part as it is.  Four entries of the lane's kD / 8 at a time: place 8 k + g of a row holds entries
      // (kD / 8) g + 4 k ..
#pragma unroll
      for (int n = 0; n < kTiles; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int row = 8 * n + 2 * t + i;
          if (row < live_rows) {
            const float r = ex2(top_v[n][i] - F::kLift - top_s[n][i]);
            float* dst = P.part_o + (slot * kRows + row) * kD + 4 * g;
#pragma unroll
            for (int k = 0; k < kSteps / 2; ++k)
              *reinterpret_cast<float4*>(dst + 32 * k) =
                  make_float4(o[n][2 * k][i] * r, o[n][2 * k][2 + i] * r, o[n][2 * k + 1][i] * r, o[n][2 * k + 1][2 + i] * r);
            if (g == 0) P.part_ml[slot * kRows + row] = make_float2(top_s[n][i], sum[n][i]);
          }
        }
    } else {
      // ---- the warps' parts joined: relative to the CTA's largest logit of each row
      if (g == 0) {
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            s_stat[warp][8 * n + 2 * t + i][0] = top_s[n][i];
            s_stat[warp][8 * n + 2 * t + i][1] = sum[n][i];
          }
      }
      __syncthreads();                                 // (also: nobody reads the stages any more)
      float* so = reinterpret_cast<float*>(smem);      // [warp][row][kPitch]
#pragma unroll
      for (int n = 0; n < kTiles; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int row = 8 * n + 2 * t + i;
          float m = s_stat[0][row][0];
#pragma unroll
          for (int w = 1; w < kWarps; ++w) m = fmaxf(m, s_stat[w][row][0]);
          const float r = ex2(top_v[n][i] - F::kLift - m);
          float* dst = so + (warp * kRows + row) * kPitch + 4 * g;
#pragma unroll
          for (int k = 0; k < kSteps / 2; ++k)
            *reinterpret_cast<float4*>(dst + 32 * k) =
                make_float4(o[n][2 * k][i] * r, o[n][2 * k][2 + i] * r, o[n][2 * k + 1][i] * r, o[n][2 * k + 1][2 + i] * r);
        }
      __syncthreads();
      for (int i = tid; i < live_rows * (kD / 4); i += kThreads) {
        const int row = i / (kD / 4), x = i - row * (kD / 4);
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float4 y = *reinterpret_cast<const float4*>(so + (w * kRows + row) * kPitch + 4 * x);
          a.x += y.x; a.y += y.y; a.z += y.z; a.w += y.w;
        }
        *reinterpret_cast<float4*>(P.part_o + (slot * kRows + row) * kD + 4 * x) = a;
      }
      if (tid < live_rows) {
        float m = s_stat[0][tid][0], l = 0.f;
        for (int w = 1; w < kWarps; ++w) m = fmaxf(m, s_stat[w][tid][0]);
        for (int w = 0; w < kWarps; ++w) l += s_stat[w][tid][1] * ex2(s_stat[w][tid][0] - m);
        P.part_ml[slot * kRows + tid] = make_float2(m, l);
      }
    }
    }                                                  // (hi > lo)

    if (together) return;
    at = upto;
    if (at >= end) return;
    // the next row tile, or the next head that holds tokens
    before += n_gran;
    if (++rt == P.row_tiles) {
      rt = 0;
      do len = (int)c.length(++unit); while (len == 0);     // (one is left: at < end <= total)
      n_gran = granules(len);
    }
  }
}

// The parts of a row tile: up to three runs of slots, of the warps of its first CTA, of whole CTAs, of the warps of its last.
struct Parts {
  int slot[3], n[3], step1;                            // the middle run's slots lie step1 apart
  __device__ __forceinline__ int count() const { return n[0] + n[1] + n[2]; }
  __device__ __forceinline__ long long operator[](int i) const {
    return i < n[0] ? slot[0] + i : i < n[0] + n[1] ? slot[1] + (i - n[0]) * step1 : slot[2] + (i - n[0] - n[1]);
  }
};

__device__ __forceinline__ Parts parts_of(const AttendParams& P, int unit, int rt) {
  Parts r{};
  r.step1 = P.warps;
  const int b = P.before[unit], n = P.before[unit + 1] - b, total = P.before[P.c.units()];
  if (n == 0) return r;
  const Shares ctas(total * P.row_tiles, P.ctas);
  const int u = unit * P.row_tiles + rt, v0 = b * P.row_tiles + rt * n, v1 = v0 + n;
  const int c0 = ctas.of(v0 + kSetup), c1 = ctas.of(v1 - 1);
  int mid0 = c0, mid1 = c1;                            // CTAs that lie wholly inside
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    const int cta = side == 0 ? c0 : c1;
    const int s0 = ctas.begin(cta), s1 = ctas.begin(cta + 1);
    if ((side == 1 && c1 == c0) || (v0 <= s0 && s1 <= v1)) continue;
    const Shares pieces(s1 - s0, P.warps);
    const int w0 = pieces.of(max(v0 + kSetup, s0) - s0), w1 = pieces.of(min(v1, s1) - s0 - 1);
    r.slot[2 * side] = cta * P.warps + w0 + u;
    r.n[2 * side] = w1 - w0 + 1;
    if (side == 0) mid0 = c0 + 1; else mid1 = c1 - 1;
  }
  r.slot[1] = mid0 * P.warps + u;
  r.n[1] = max(mid1 - mid0 + 1, 0);
  return r;
}

// A CTA writes 2^row_shift query rows' outputs of a head, and their log-sum-exps in powers of two for attend_weight_kernel.  The
// warps share the rows out; a warp takes every so many-th part of its row (of 64 entries: two parts at a time), statistics and
// output in one go, against a running maximum, and the warps meet once.
template <typename T, int kD>
__global__ void __launch_bounds__(kJoinThreads)
attend_join_kernel(const __grid_constant__ AttendParams P, const int32_t* __restrict__ row_counts, T* __restrict__ out,
                   float* __restrict__ lse, int row_shift) {
  constexpr int kLanes = kD / 4;                       // lanes of a part's row, 16 bytes each
  constexpr int kPer = 32 / kLanes;                    // parts a warp reads side by side
  constexpr int kGroups = kJoinWarps * kPer;
  __shared__ float2 s_ml[kGroups];
  __shared__ float4 s_o[kGroups][kLanes];
  grid_dependency_wait();
  const Cache& c = P.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, units = c.units();
  const int per_unit = (P.live + (1 << row_shift) - 1) >> row_shift, unit = blockIdx.x / per_unit;
  const int r0 = (blockIdx.x - unit * per_unit) << row_shift;
  const int x = lane % kLanes, group = warp * kPer + lane / kLanes, groups = kGroups >> row_shift;      // of a row
  const int r = r0 + group / groups, rt = min(r, P.live - 1) / P.tile_rows, row = min(r, P.live - 1) - rt * P.tile_rows;
  const Parts parts = parts_of(P, unit, rt);
  const int n = parts.count();
  float m = kNone, l = 0.f;
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i0 = group % groups; i0 < n; i0 += 4 * groups) {      // four parts in flight
    float2 ml[4];
    float4 y[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = i0 + k * groups;
      ml[k] = make_float2(kNone, 0.f);
      y[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (i < n) {
        const long long at = parts[i] * P.tile_rows + row;
        ml[k] = P.part_ml[at];
        y[k] = *reinterpret_cast<const float4*>(P.part_o + at * kD + 4 * x);
      }
    }
    const float top = fmaxf(m, fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x)));
    const float down = ex2(m - top);
    l *= down; a.x *= down; a.y *= down; a.z *= down; a.w *= down;
    m = top;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float f = ex2(ml[k].x - top);
      l += ml[k].y * f;
      a.x += y[k].x * f; a.y += y[k].y * f; a.z += y[k].z * f; a.w += y[k].w * f;
    }
  }
  s_o[group][x] = a;
  if (x == 0) s_ml[group] = make_float2(m, l);
  __syncthreads();
  // thread: an output's 16 bytes
  const int out_row = tid / kLanes, at = tid - out_row * kLanes, r1 = r0 + out_row;
  const int b = unit / c.Hkv, h = unit - b * c.Hkv;
  const int rr = P.row0 + r1, j = h * P.G + rr / P.rows, mm = rr % P.rows;
  if (out_row >= 1 << row_shift || r1 >= P.live || mm >= row_count(P, row_counts, b)) return;      // (rows that the sequence has not got stay as they are)
  float top = kNone;
  for (int k = out_row * groups; k < (out_row + 1) * groups; ++k) top = fmaxf(top, s_ml[k].x);
  l = 0.f;
  a = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k = out_row * groups; k < (out_row + 1) * groups; ++k) {
    const float2 ml = s_ml[k];
    const float4 y = s_o[k][at];
    const float f = ex2(ml.x - top);
    l += ml.y * f;
    a.x += y.x * f; a.y += y.y * f; a.z += y.z * f; a.w += y.w * f;
  }
  const bool none = l == 0.f;                          // (the row sees no token; a sum of NaN stays one)
  const float inv = none ? 0.f : 1.f / l;
  // place 8 k + g holds entries (kD / 8) g + 4 k ..
  T* dst = out + b * P.os[0] + j * P.os[1] + mm * P.os[2] + (kD / 8) * (at & 7) + 4 * (at >> 3);
  a.x *= inv; a.y *= inv; a.z *= inv; a.w *= inv;
  if (sizeof(T) == 2) {
    const __nv_bfloat162 lo = __floats2bfloat162_rn(a.x, a.y), hi = __floats2bfloat162_rn(a.z, a.w);
    *reinterpret_cast<uint2*>(dst) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
  } else {
    *reinterpret_cast<float4*>(dst) = a;
  }
  if (at == 0) P.lse2[(long long)unit * P.live + r1] = none ? INFINITY : top + log2f(l);
  if (at == 0 && lse != nullptr)
    lse[((long long)b * P.Hq + j) * P.rows + mm] = none ? -INFINITY : (top + log2f(l)) * 0.693147180559945309f;
}

// weight_out = weight_in + the sum of 2^(logit - log-sum-exp) over the rows: four tokens of a head per thread.
__global__ void __launch_bounds__(kJoinThreads)
attend_weight_kernel(const __grid_constant__ AttendParams P, const int32_t* __restrict__ row_counts, const float* weight_in, float* weight_out) {
  __shared__ float s_lse[kMaxRows];
  grid_dependency_wait();
  const Cache& c = P.c;
  const int tid = threadIdx.x, unit = blockIdx.y;
  const long long len = c.length(unit), tok0 = (long long)blockIdx.x * kJoinTokens + tid;
  if (tok0 - tid >= len) return;
  const int rows = row_count(P, row_counts, unit / c.Hkv);
  const float* logits = P.logits + ((long long)unit * P.row_tiles * c.cap + tok0) * P.logit_rows;
  float2 x0[kJoinEach][2];                             // the first rows' logits
  float w[kJoinEach];
#pragma unroll
  for (int k = 0; k < kJoinEach; ++k) {
    const long long tok = tok0 + k * kJoinThreads;
    w[k] = 0.f;
    x0[k][0] = x0[k][1] = make_float2(0.f, 0.f);
    if (tok < len) {
      if (weight_in != nullptr) w[k] = weight_in[(long long)unit * c.cap + tok];
      const float* y = logits + (long long)k * kJoinThreads * P.logit_rows;
      x0[k][0] = *reinterpret_cast<const float2*>(y);
      if (P.logit_rows > 2) x0[k][1] = *reinterpret_cast<const float2*>(y + 2);
    }
  }
  // (infinity weighs nothing: rows that are not there, or see no token)
  if (tid < kMaxRows) s_lse[tid] = tid < P.live && (P.row0 + tid) % P.rows < rows ? P.lse2[(long long)unit * P.live + tid] : INFINITY;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kJoinEach; ++k) {
    const long long tok = tok0 + k * kJoinThreads;
    if (tok >= len) continue;
    float sum = ex2(x0[k][0].x - s_lse[0]) + ex2(x0[k][0].y - s_lse[1]);
    if (P.logit_rows > 2) sum += ex2(x0[k][1].x - s_lse[2]) + ex2(x0[k][1].y - s_lse[3]);
    for (int rt = 0; rt < P.row_tiles; ++rt) {
      const float* y = logits + ((long long)rt * c.cap + (long long)k * kJoinThreads) * P.logit_rows;
      const int n = min(P.live - rt * P.tile_rows, P.tile_rows);
      for (int i = rt == 0 ? 4 : 0; i < n; i += 2) {
        const float2 v = *reinterpret_cast<const float2*>(y + i);
        sum += ex2(v.x - s_lse[rt * P.tile_rows + i]);
        if (i + 1 < n) sum += ex2(v.y - s_lse[rt * P.tile_rows + i + 1]);
      }
    }
    weight_out[(long long)unit * c.cap + tok] = w[k] + sum;
  }
}

kvc_status resolve_attend(const kvc_cache* cache, const kvc_attend_desc* d, AttendParams* P) {
  kvc_status s = resolve_cache(cache, "cache", &P->c);
  if (s != KVC_OK) return s;
  KVC_REQUIRE8(d != nullptr, KVC_ERR_INVALID_ARG, "desc is NULL");
  KVC_REQUIRE8(d->n_q_heads >= 1 && d->n_q_heads % P->c.Hkv == 0, KVC_ERR_INVALID_ARG, "n_q_heads must be a multiple of the cache's n_kv_heads");
  KVC_REQUIRE8(d->n_q_heads <= kMaxQHeads, KVC_ERR_UNSUPPORTED, "more than %d query heads", kMaxQHeads);
  KVC_REQUIRE8(d->rows >= 1, KVC_ERR_INVALID_ARG, "rows must be >= 1");
  KVC_REQUIRE8(d->rows <= 65536, KVC_ERR_UNSUPPORTED, "rows > 65536");
  if ((s = check_dtype(d->dtype)) != KVC_OK) return s;
  KVC_REQUIRE8(d->causal == 0 || d->causal == 1, KVC_ERR_INVALID_ARG, "causal must be 0 or 1");
  KVC_REQUIRE8(d->reserved_ == 0, KVC_ERR_INVALID_ARG, "reserved_ must be 0");
  KVC_REQUIRE8(isfinite(d->scale), KVC_ERR_INVALID_ARG, "scale is not finite");
  KVC_REQUIRE8(P->c.st[2] < (1LL << 31), KVC_ERR_UNSUPPORTED, "tokens of the cache lie 2^31 bytes or more apart");
  // (places in the granules of all heads and row tiles are 32-bit numbers)
  KVC_REQUIRE8((long long)P->c.units() * (P->c.cap / kGranule + 1 + kSetup) * (kMaxRows / 8) < (1LL << 31), KVC_ERR_UNSUPPORTED,
               "batch * n_kv_heads * capacity must be below 2^34");
  P->Hq = d->n_q_heads; P->G = d->n_q_heads / P->c.Hkv; P->rows = d->rows; P->causal = d->causal;
  P->scale = d->scale > 0.f ? d->scale : 1.0f / sqrtf((float)P->c.d);
  const int eb = d->dtype == KVC_F32 ? 4 : 2;
  if ((s = resolve_strides(d->q_stride, P->c.Bt, P->Hq, P->rows, P->c.d, eb, false, "q_stride", P->qs)) != KVC_OK) return s;
  return resolve_strides(d->out_stride, P->c.Bt, P->Hq, P->rows, P->c.d, eb, true, "out_stride", P->os);
}

// Query rows that share the codes' conversion: 8, 16 or, in bf16, 32 (fp32 keeps twice the operands).
int tile_rows_of(int live, int dtype) { return live <= 8 ? 8 : live <= 16 || dtype == KVC_F32 ? 16 : 32; }

struct AttendLayout {
  int live, tile_rows, row_tiles, logit_rows;
  size_t o, ml, before, lse2, logits, total;
};

AttendLayout attend_layout(const AttendParams& P, int dtype, bool with_weight) {
  AttendLayout y;
  const long long all = (long long)P.G * P.rows;
  y.live = (int)(all < kMaxRows ? all : kMaxRows);
  y.tile_rows = tile_rows_of(y.live, dtype);
  y.row_tiles = (y.live + y.tile_rows - 1) / y.tile_rows;
  y.logit_rows = 2;
  while (y.logit_rows < y.live && y.logit_rows < y.tile_rows) y.logit_rows *= 2;
  const size_t slots = (size_t)kMaxCtas * kAttWarps + (size_t)P.c.units() * y.row_tiles;
  y.o = 0;
  y.ml = align_up(slots * y.tile_rows * P.c.d * sizeof(float));
  y.before = y.ml + align_up(slots * y.tile_rows * sizeof(float2));
  y.lse2 = y.before + align_up(((size_t)P.c.units() + 1) * sizeof(int));
  y.logits = y.lse2 + align_up((size_t)P.c.units() * kMaxRows * sizeof(float));
  y.total = y.logits + (with_weight ? align_up((size_t)P.c.units() * y.row_tiles * P.c.cap * y.logit_rows * sizeof(float)) : 0);
  return y;
}

template <typename T, int kFormat, int kD, int kTiles, bool kWeight>
kvc_status launch_split(AttendParams& P, const T* q, const int32_t* row_counts, cudaStream_t st) {
  using F = Form<T, kD, kTiles>;
  static_assert(F::kSmem <= 220 * 1024, "shared memory and slots");
  auto kernel = attend_split_kernel<T, kFormat, kD, kTiles, kWeight>;
  P.warps = F::kWarps;
  static std::atomic<uint64_t> done{0};
  KVC_CUDA(allow_smem(kernel, F::kSmem, done, P.device));
  KVC_CUDA(launch_dependent(kernel, dim3(P.ctas), dim3(F::kThreads), F::kSmem, st, P, q, row_counts));
  KVC_LAUNCH_CHECK("attend_split_kernel");
  return KVC_OK;
}

template <typename T, int kFormat, int kD>
kvc_status launch_split_form(AttendParams& P, bool weight, const T* q, const int32_t* row_counts, cudaStream_t st) {
  if (P.tile_rows == 8)
    return weight ? launch_split<T, kFormat, kD, 1, true>(P, q, row_counts, st) : launch_split<T, kFormat, kD, 1, false>(P, q, row_counts, st);
  if (P.tile_rows == 16)
    return weight ? launch_split<T, kFormat, kD, 2, true>(P, q, row_counts, st) : launch_split<T, kFormat, kD, 2, false>(P, q, row_counts, st);
  if constexpr (sizeof(T) == 2)
    return weight ? launch_split<T, kFormat, kD, 4, true>(P, q, row_counts, st) : launch_split<T, kFormat, kD, 4, false>(P, q, row_counts, st);
  set_error("no form of attend_split_kernel for tiles of %d rows", P.tile_rows);
  return KVC_ERR_UNSUPPORTED;
}

template <typename T>
kvc_status run_attend(AttendParams& P, const AttendLayout& y, const T* q, const int32_t* row_counts, T* out, float* lse,
                      const float* weight_in, float* weight_out, cudaStream_t st) {
  const bool weight = weight_out != nullptr, e4m3 = P.c.format == KVC_E4M3;
  const long long all = (long long)P.G * P.rows;
  for (long long row0 = 0; row0 < all; row0 += y.live) {
    P.row0 = (int)row0;
    P.live = (int)(all - row0 < y.live ? all - row0 : y.live);
    P.row_tiles = (P.live + y.tile_rows - 1) / y.tile_rows;
    kvc_status s;
    if (P.c.d == 128)
      s = e4m3 ? launch_split_form<T, KVC_E4M3, 128>(P, weight, q, row_counts, st) : launch_split_form<T, KVC_INT8, 128>(P, weight, q, row_counts, st);
    else
      s = e4m3 ? launch_split_form<T, KVC_E4M3, 64>(P, weight, q, row_counts, st) : launch_split_form<T, KVC_INT8, 64>(P, weight, q, row_counts, st);
    if (s != KVC_OK) return s;
    // a CTA per row while that keeps the GPU busy; many heads, whose parts are few: several rows in a CTA
    int shift = 0;
    while (shift < 3 && (P.live >> shift) > 1 && (long long)P.c.units() * ((P.live + (1 << shift) - 1) >> shift) > 2LL * P.ctas) ++shift;
    KVC_CUDA(launch_dependent(P.c.d == 128 ? attend_join_kernel<T, 128> : attend_join_kernel<T, 64>,
                              dim3((unsigned)P.c.units() * ((P.live + (1 << shift) - 1) >> shift)), dim3(kJoinThreads), 0, st, P, row_counts,
                              out, lse, shift));
    KVC_LAUNCH_CHECK("attend_join_kernel");
    if (!weight) continue;
    KVC_CUDA(launch_dependent(attend_weight_kernel, dim3((unsigned)((P.c.cap + kJoinTokens - 1) / kJoinTokens), P.c.units()), dim3(kJoinThreads),
                              0, st, P, row_counts, weight_in, weight_out));
    KVC_LAUNCH_CHECK("attend_weight_kernel");
    weight_in = weight_out;                          // (later rows add to what the first ones gave)
  }
  return KVC_OK;
}

}  // namespace
}  // namespace kvc

using namespace kvc;

extern "C" {

kvc_status kvc_attend_workspace_size(const kvc_cache* cache, const kvc_attend_desc* desc, int32_t with_weight, size_t* bytes) {
  AttendParams P;
  const kvc_status s = resolve_attend(cache, desc, &P);
  if (s != KVC_OK) return s;
  KVC_REQUIRE8(bytes != nullptr, KVC_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = attend_layout(P, desc->dtype, with_weight != 0).total;
  return KVC_OK;
}

kvc_status kvc_attend(const kvc_cache* cache, const kvc_attend_desc* desc, const void* q, const int32_t* row_counts, void* out, float* lse,
                      const float* weight_in, float* weight_out, void* workspace, size_t workspace_bytes, void* stream) {
  AttendParams P;
  kvc_status s = resolve_attend(cache, desc, &P);
  if (s != KVC_OK) return s;
  KVC_REQUIRE8(q && out && aligned16(q) && aligned16(out), KVC_ERR_INVALID_ARG, "q or out is NULL or not 16-byte aligned");
  KVC_REQUIRE8(weight_in == nullptr || weight_out != nullptr, KVC_ERR_INVALID_ARG, "weight_in without weight_out");
  const AttendLayout y = attend_layout(P, desc->dtype, weight_out != nullptr);
  KVC_REQUIRE8(workspace != nullptr, KVC_ERR_WORKSPACE, "workspace is NULL (%zu bytes needed)", y.total);
  KVC_REQUIRE8((reinterpret_cast<uintptr_t>(workspace) & 255u) == 0, KVC_ERR_WORKSPACE, "workspace is not 256-byte aligned");
  KVC_REQUIRE8(workspace_bytes >= y.total, KVC_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, y.total);
  if ((s = require_device()) != KVC_OK) return s;
  int dev = 0, sms = 0;
  KVC_CUDA(cudaGetDevice(&dev));
  KVC_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  P.ctas = sms < kMaxCtas ? sms : kMaxCtas;
  P.device = dev;
  P.tile_rows = y.tile_rows; P.logit_rows = y.logit_rows;
  P.part_o = (float*)((char*)workspace + y.o);
  P.part_ml = (float2*)((char*)workspace + y.ml);
  P.before = (int*)((char*)workspace + y.before);
  P.lse2 = (float*)((char*)workspace + y.lse2);
  P.logits = (float*)((char*)workspace + y.logits);
  return desc->dtype == KVC_F32 ? run_attend<float>(P, y, (const float*)q, row_counts, (float*)out, lse, weight_in, weight_out, (cudaStream_t)stream)
                                : run_attend<__nv_bfloat16>(P, y, (const __nv_bfloat16*)q, row_counts, (__nv_bfloat16*)out, lse, weight_in,
                                                            weight_out, (cudaStream_t)stream);
}

}  // extern "C"
