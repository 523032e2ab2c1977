// Attention of a few query rows over an 8-bit cache (kvc_attend).
//
// HBM is the bound: 2 d bytes of codes per token and KV head, against 4 d products per query row.  Two kernels:
//
// attend_split_kernel   one CTA per SM.  The tokens of all heads, in granules of kGranule, are laid end to end and cut into
//   equal shares, one per CTA, whatever the lengths: a CTA may hold a part of one long head or many short ones.  Its warps
//   take 32 tokens in turn, each for itself: a lane copies the very 16-byte pieces it will use (cp.async into its own
//   places in shared memory, kStages deep, no barrier), turns the codes into fp16 and feeds mma.m16n8k16: S^T = K Q^T with the
//   tokens as rows, then O^T = V^T P^T, eight query rows to a column tile (kTiles of them share the converted codes).
//   Operand layouts: the order of the summed index is free as long as both operands agree, so lane (g, t) takes token
//   g's entries 16 t .. 16 t + 15 of each 64 as its k slots, and entries (d / 8) g .. of its tokens of V as its rows; a
//   transpose of P's 8 x 8 tiles (movmatrix) is the only exchange between lanes.  Legacy mma on purpose: the tensor pipe needs
//   a quarter of the time the codes take to arrive, and codes go from registers into it; through tcgen05 they would have to
//   be written back to shared memory as fp16 first.
// attend_join_kernel    joins the parts of a row (log-sum-exp), and adds the row's weights from the logits, which the first
//   kernel leaves in the workspace (they stay in L2; the softmax's denominator is known only after the last token).
//
// Numbers: codes are exact in fp16.  A query row is scaled by a power of two to below 2 and rounded to fp16, which is exact
// for bf16 but for entries 2^14 times smaller than the row's largest; fp32 rows go as two fp16 (22 bits), and so does P in
// front of V then (one fp16, 11 bits, for bf16 outputs).  Products, softmax and sums are fp32.  V's exponents differ from block
// to block: P goes in relative to 2^M, M the running maximum of logit + exponent, which keeps the largest terms of a row at
// full precision whatever block they are in, and 2^15 times larger, so that 2^17 weights of 2^-26 are not lost beside one
// of 1/2, as they are in an fp16 of at most 1.
#include <math.h>

#include "cache8.cuh"

namespace kvc {
namespace {

constexpr int kWarps = 12;                // (8: xx, 16 do not fit the registers)
constexpr int kAttThreads = kWarps * 32;
constexpr int kGranule = 64;              // tokens: unit of the split
constexpr int kMaxCtas = 256;             // bounds the workspace, whatever the device
constexpr int kMaxRows = 64;              // query rows of a KV head that one launch takes (bounds the logits kept)
constexpr float kLift = 15.f;             // P goes into V as 2^15 p: fp16 then tells weights apart down to 2^-40 of the largest
constexpr float kNone = -3e38f;           // "no logit yet": finite, so that differences are numbers
constexpr int kJoinThreads = 128;
constexpr int kJoinTokens = 512;

struct AttendParams {
  Cache c;
  int Hq, G, rows, causal;
  float scale;
  long long qs[3], os[3];
  // of this launch: query rows row0 .. row0 + live - 1 of the G * rows of a KV head, in row_tiles tiles of 8 * kTiles
  int row0, live, row_tiles, tile_rows, ctas, logit_rows;
  float* part_o;                          // [slot][tile_rows][d]
  float2* part_ml;                        // [slot][tile_rows]: largest logit (in powers of two), sum of 2^(logit - it)
  float* logits;                          // [unit][row tile][token][logit_rows]
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void mma16816(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
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

template <int kBytes>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, bool live) {
  if (kBytes == 16)
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" :: "r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
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
// CTAs that get a share of `total` granules: each at least one, so that the parts of a head lie in consecutive CTAs.
__device__ __forceinline__ int sharers(const AttendParams& P, long long total) { return total < P.ctas ? max((int)total, 1) : P.ctas; }
__device__ __forceinline__ int granules(const AttendParams& P, int unit) { return (int)((P.c.length(unit) + kGranule - 1) / kGranule); }

template <int kFormat, int kD, int kTiles, bool kSplitF32, bool kWeight>
struct Warp {
  static constexpr int kSteps = kD / 16;               // k steps of Q K^T, and row tiles of V^T
  static constexpr int kKPieces = kD / 64;             // 16-byte pieces of a token's K per lane
  static constexpr int kVBytes = kD / 8;               // a lane's bytes of a token's V
  static constexpr int kStages = kD == 128 ? 2 : 3;
  static constexpr int kStageBytes = 32 * 2 * kD;      // per warp: 32 tokens of K and V
  static constexpr int kVBase = 32 * kD;
};

template <typename T, int kFormat, int kD, int kTiles, bool kWeight>
__global__ void __launch_bounds__(kAttThreads, 1)
attend_split_kernel(const __grid_constant__ AttendParams P, const T* __restrict__ q, const int32_t* __restrict__ row_counts) {
  constexpr bool kTwo = sizeof(T) == 4;                // fp32: Q and P as two fp16 each
  using W = Warp<kFormat, kD, kTiles, kTwo, kWeight>;
  constexpr int kSteps = W::kSteps, kStages = W::kStages, kRowsTile = 8 * kTiles, kPitch = kD + 4;
  extern __shared__ __align__(128) char smem[];
  __shared__ long long s_sum[kWarps];
  __shared__ int s_unit;
  __shared__ long long s_before, s_total;
  __shared__ float s_stat[kWarps][kRowsTile][2];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  grid_dependency_wait();
  const Cache& c = P.c;
  const int units = c.units();

  // ---- this CTA's share: granules [at, end) of all of them, and the unit that `at` lies in
  {
    const int per = (units + kAttThreads - 1) / kAttThreads;
    const int u0 = tid * per, u1 = min(u0 + per, units);
    long long mine = 0;
    for (int u = u0; u < u1; ++u) mine += granules(P, u);
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    if (lane == 31) s_sum[warp] = incl;
    __syncthreads();
    long long total = 0;
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) incl += s_sum[w];
      total += s_sum[w];
    }
    total *= P.row_tiles;
    const long long at = total * blockIdx.x / sharers(P, total);
    long long before = (incl - mine) * P.row_tiles;
    if (tid == 0) s_total = total;
    if (total > 0 && before <= at && at < incl * P.row_tiles) {
      int u = u0;
      for (;; ++u) {
        const long long n = (long long)granules(P, u) * P.row_tiles;
        if (at < before + n) break;
        before += n;
      }
      s_unit = u;
      s_before = before;
    }
    __syncthreads();
  }
  const long long total = s_total;
  const int ctas = sharers(P, total);
  if (total == 0 || (int)blockIdx.x >= ctas) return;
  long long at = total * blockIdx.x / ctas;
  const long long end = total * (blockIdx.x + 1) / ctas;
  int unit = s_unit;
  long long before = s_before;

  char* my_smem = smem + warp * (kStages * W::kStageBytes);
  const uint32_t my_smem_addr = (uint32_t)__cvta_generic_to_shared(my_smem);
  int rt = (int)((at - before) / granules(P, unit));
  before += (long long)rt * granules(P, unit);

  while (true) {
    // ---- a part of one row tile of one head: tokens [lo, hi)
    const int b = unit / c.Hkv, h = unit - b * c.Hkv;
    const long long len = c.length(unit);
    const int n_gran = granules(P, unit);
    const long long lo = (at - before) * kGranule;
    const long long upto = min(end - before, (long long)n_gran);
    const long long hi = min(upto * kGranule, len);
    const int rows = row_count(P, row_counts, b);
    const int first_row = P.row0 + rt * kRowsTile, last_row = min(P.row0 + P.live, first_row + kRowsTile);

    const uint8_t *kc = c.k + c.base(unit), *vc = c.v + c.base(unit);
    const int8_t *ke = c.k_exp + (long long)unit * c.blocks, *ve = c.v_exp + (long long)unit * c.blocks;
    const int iters = (int)((hi - lo + 32 * kWarps - 1 - 32 * warp) / (32 * kWarps));      // 0 for warps behind the end

    auto fetch = [&](int it) {                       // 32 tokens of K and V into stage it % kStages
      if (it < iters) {
        const uint32_t dst = my_smem_addr + (it % kStages) * W::kStageBytes;
        const long long tok0 = lo + (long long)(it * kWarps + warp) * 32;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const long long tok = tok0 + 8 * i + g;
          const bool live = tok < hi;
          const uint8_t* src = kc + (live ? tok : 0) * c.st[2] + 16 * t;
#pragma unroll
          for (int p = 0; p < W::kKPieces; ++p) copy_async<16>(dst + ((i * W::kKPieces + p) * 32 + lane) * 16, src + 64 * p, live);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const long long tok = tok0 + 16 * (i >> 2) + 8 * ((i >> 1) & 1) + 2 * t + (i & 1);
          const bool live = tok < hi;
          copy_async<W::kVBytes>(dst + W::kVBase + (i * 32 + lane) * W::kVBytes, vc + (live ? tok : 0) * c.st[2] + W::kVBytes * g, live);
        }
      }
      copy_commit();
    };
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) fetch(s);

    // ---- Q: row 8 n + g of the tile, its entries in the lane's k slots, scaled by a power of two to below 2
    uint32_t qh[kTiles][kSteps][2], ql[kTwo ? kTiles : 1][kTwo ? kSteps : 1][2];
    float factor[kTiles][2];                         // of the columns 2 t, 2 t + 1: logit = accumulator * factor * 2^ke
    int seen[kTiles][2], seen_least = 0x7fffffff;    // (lengths fit 31 bits)
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
      const float down = pow2(-e), up = pow2(e) * P.scale * 1.44269504088896341f;
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float a = x[4 * s + 2 * i] * down, z = x[4 * s + 2 * i + 1] * down;
          qh[n][s][i] = pack_half2(a, z);
          if (kTwo) {
            const __half2 hh = *reinterpret_cast<const __half2*>(&qh[n][s][i]);
            ql[n][s][i] = pack_half2(a - __low2float(hh), z - __high2float(hh));
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

    // exponents of the two halves of 32 tokens, read one step ahead
    int ek[2], ev[2], ek_next[2] = {0, 0}, ev_next[2] = {0, 0};
    auto fetch_exps = [&](int it) {
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const long long tok = lo + (long long)(it * kWarps + warp) * 32 + 16 * f;
        if (it < iters && tok < hi) {
          ek_next[f] = __ldg(ke + (tok >> c.block_shift));
          ev_next[f] = __ldg(ve + (tok >> c.block_shift));
        }
      }
    };
    fetch_exps(0);

    for (int it = 0; it < iters; ++it) {
      ek[0] = ek_next[0]; ek[1] = ek_next[1]; ev[0] = ev_next[0]; ev[1] = ev_next[1];
      fetch_exps(it + 1);
      fetch(it + kStages - 1);
      copy_wait<kStages - 1>();
      const char* st = my_smem + (it % kStages) * W::kStageBytes;
      const long long tok0 = lo + (long long)(it * kWarps + warp) * 32;

      // ---- logits, in powers of two: lane holds tokens g and g + 8 (of each 16), columns 2 t and 2 t + 1
      float sc[2][kTiles][4];
#pragma unroll
      for (int f = 0; f < 2; ++f) {
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) sc[f][n][i] = 0.f;
#pragma unroll
        for (int p = 0; p < W::kKPieces; ++p) {
          const uint4 w0 = *reinterpret_cast<const uint4*>(st + (((2 * f) * W::kKPieces + p) * 32 + lane) * 16);
          const uint4 w1 = *reinterpret_cast<const uint4*>(st + (((2 * f + 1) * W::kKPieces + p) * 32 + lane) * 16);
          const uint32_t x0[4] = {w0.x, w0.y, w0.z, w0.w}, x1[4] = {w1.x, w1.y, w1.z, w1.w};
#pragma unroll
          for (int s = 0; s < 4; ++s) {
            uint32_t a[4];
            to_half2<kFormat>(x0[s], &a[0], &a[2]);
            to_half2<kFormat>(x1[s], &a[1], &a[3]);
#pragma unroll
            for (int n = 0; n < kTiles; ++n) {
              mma16816(sc[f][n], a, qh[n][4 * p + s][0], qh[n][4 * p + s][1]);
              if (kTwo) mma16816(sc[f][n], a, ql[n][4 * p + s][0], ql[n][4 * p + s][1]);
            }
          }
        }
        const float kf = pow2_clamped(ek[f]);
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) sc[f][n][i] *= factor[n][i & 1] * kf;
      }
      if (tok0 + 32 > seen_least) {
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
          for (int n = 0; n < kTiles; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (tok0 + 16 * f + 8 * (i >> 1) + g >= seen[n][i & 1]) sc[f][n][i] = -INFINITY;
      }
      if (kWeight) {
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const long long tok = tok0 + 16 * f + 8 * i + g;
            if (tok < hi) {
#pragma unroll
              for (int n = 0; n < kTiles; ++n)
                if (8 * n + 2 * t < P.logit_rows)
                  *reinterpret_cast<float2*>(logit_row + tok * P.logit_rows + 8 * n) = make_float2(sc[f][n][2 * i], sc[f][n][2 * i + 1]);
            }
          }
      }

      // ---- running maxima of the logits and of logit + V's exponent; sums and outputs follow them
      const bool same = ev[0] == ev[1];
#pragma unroll
      for (int n = 0; n < kTiles; ++n) {
        float ms[2], mv[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float m0 = fmaxf(sc[0][n][i], sc[0][n][2 + i]), m1 = fmaxf(sc[1][n][i], sc[1][n][2 + i]);
          if (same) {
            m0 = fmaxf(m0, m1);
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) m0 = fmaxf(m0, __shfl_xor_sync(0xffffffffu, m0, x));
            m1 = m0;
          } else {
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) {
              m0 = fmaxf(m0, __shfl_xor_sync(0xffffffffu, m0, x));
              m1 = fmaxf(m1, __shfl_xor_sync(0xffffffffu, m1, x));
            }
          }
          ms[i] = fmaxf(top_s[n][i], fmaxf(m0, m1));
          mv[i] = fmaxf(top_v[n][i], fmaxf(m0 + ev[0], m1 + ev[1]));
        }
        const bool grew = ms[0] > top_s[n][0] || ms[1] > top_s[n][1] || mv[0] > top_v[n][0] || mv[1] > top_v[n][1];
        if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            sum[n][i] *= ex2(top_s[n][i] - ms[i]);
            const float r = ex2(top_v[n][i] - mv[i]);
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
              o[n][s][i] *= r;
              o[n][s][2 + i] *= r;
            }
            top_s[n][i] = ms[i];
            top_v[n][i] = mv[i];
          }
        }
      }

      // ---- P, and its share of the outputs
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        uint32_t ph[kTiles][2], pl[kTwo ? kTiles : 1][2];
#pragma unroll
        for (int n = 0; n < kTiles; ++n) {
          float up[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) up[i] = top_s[n][i] + ev[f] - top_v[n][i] + kLift;
          const bool far = fmaxf(up[0], up[1]) > 126.f;         // (V's exponents more than 2^111 apart: the factor is no fp32)
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
            for (int i = 0; i < 4; ++i) p[i] = ex2(sc[f][n][i] + (ev[f] - top_v[n][i & 1] + kLift));
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
        const char* sv = st + W::kVBase + (4 * f * 32 + lane) * W::kVBytes;
        uint32_t v[4][W::kVBytes / 4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (kD == 128) {
            const uint4 w = *reinterpret_cast<const uint4*>(sv + i * 32 * W::kVBytes);
            v[i][0] = w.x; v[i][1] = w.y; v[i][W::kVBytes / 4 - 2] = w.z; v[i][W::kVBytes / 4 - 1] = w.w;
          } else {
            const uint2 w = *reinterpret_cast<const uint2*>(sv + i * 32 * W::kVBytes);
            v[i][0] = w.x; v[i][1] = w.y;
          }
        }
#pragma unroll
        for (int w = 0; w < W::kVBytes / 4; ++w) {
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
    copy_wait<0>();

    // ---- the warps' parts joined: relative to the CTA's largest logit of each row
#pragma unroll
    for (int n = 0; n < kTiles; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) sum[n][i] += __shfl_xor_sync(0xffffffffu, sum[n][i], x);
        if (g == 0) {
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
        const float r = ex2(top_v[n][i] - kLift - m);
        float* dst = so + (warp * kRowsTile + row) * kPitch + 4 * g;
        // four entries of the lane's kD / 8 at a time: place 8 k + g of the row holds entries (kD / 8) g + 4 k ..
#pragma unroll
        for (int k = 0; k < kSteps / 2; ++k)
          *reinterpret_cast<float4*>(dst + 32 * k) =
              make_float4(o[n][2 * k][i] * r, o[n][2 * k][2 + i] * r, o[n][2 * k + 1][i] * r, o[n][2 * k + 1][2 + i] * r);
      }
    __syncthreads();
    const long long slot = (long long)blockIdx.x + (long long)unit * P.row_tiles + rt;
    for (int i = tid; i < kRowsTile * (kD / 4); i += kAttThreads) {
      const int row = i / (kD / 4), x = i - row * (kD / 4);
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float4 y = *reinterpret_cast<const float4*>(so + (w * kRowsTile + row) * kPitch + 4 * x);
        a.x += y.x; a.y += y.y; a.z += y.z; a.w += y.w;
      }
      *reinterpret_cast<float4*>(P.part_o + (slot * kRowsTile + row) * kD + 4 * x) = a;
    }
    if (tid < kRowsTile) {
      float m = s_stat[0][tid][0], l = 0.f;
      for (int w = 1; w < kWarps; ++w) m = fmaxf(m, s_stat[w][tid][0]);
      for (int w = 0; w < kWarps; ++w) l += s_stat[w][tid][1] * ex2(s_stat[w][tid][0] - m);
      P.part_ml[slot * kRowsTile + tid] = make_float2(m, l);
    }

    at = before + upto;
    if (at >= end) break;
    // the next row tile, or the next head that holds tokens
    before += n_gran;
    if (++rt == P.row_tiles) {
      rt = 0;
      do ++unit; while (granules(P, unit) == 0);     // (one is left: at < end <= total)
    }
    __syncthreads();                                 // the shared memory is free again
  }
}

// Parts of row tile (unit, rt): slots first .. last, or none (last < first).
struct Parts {
  long long first, last;
};

__device__ __forceinline__ Parts parts_of(const AttendParams& P, int unit, int rt, long long before, long long total) {
  const long long n = granules(P, unit);
  Parts r{0, -1};
  if (n == 0) return r;
  const int ctas = sharers(P, total);
  const long long u = (long long)unit * P.row_tiles + rt, t0 = before * P.row_tiles + rt * n;
  r.first = ((t0 + 1) * ctas - 1) / total + u;
  r.last = ((t0 + n) * ctas - 1) / total + u;
  return r;
}

// One warp: the largest logit of a row over its parts, and the sum of 2^(logit - it).
__device__ __forceinline__ float2 join_stats(const AttendParams& P, const Parts& r, int row) {
  const int lane = threadIdx.x & 31;
  float m = kNone, l = 0.f;
  for (long long s = r.first + lane; s <= r.last; s += 32) m = fmaxf(m, P.part_ml[s * P.tile_rows + row].x);
#pragma unroll
  for (int x = 1; x < 32; x <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
  for (long long s = r.first + lane; s <= r.last; s += 32) {
    const float2 a = P.part_ml[s * P.tile_rows + row];
    l += a.y * ex2(a.x - m);
  }
#pragma unroll
  for (int x = 1; x < 32; x <<= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
  return make_float2(m, l);
}

// The first units * live CTAs write a query row's output each; the others add the weights of kJoinTokens tokens of a head.
template <typename T, int kD>
__global__ void __launch_bounds__(kJoinThreads)
attend_join_kernel(const __grid_constant__ AttendParams P, const int32_t* __restrict__ row_counts, T* __restrict__ out,
                   float* __restrict__ lse, const float* weight_in, float* weight_out, int chunks) {
  __shared__ long long s_sum[2][kJoinThreads / 32];
  __shared__ float s_lse[kMaxRows];
  __shared__ float4 s_o[kJoinThreads / 32][32];
  grid_dependency_wait();
  const Cache& c = P.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, units = c.units();
  const bool is_row = blockIdx.x < (unsigned)(units * P.live);
  const int job = is_row ? blockIdx.x : blockIdx.x - units * P.live;
  const int unit = is_row ? job / P.live : job / chunks;
  const long long len = c.length(unit);
  const long long tok0 = is_row ? 0 : (long long)(job - unit * chunks) * kJoinTokens;
  if (!is_row && tok0 >= len) return;
  // granules before this unit, and all of them
  long long before = 0, total = 0;
  for (int u = tid; u < units; u += kJoinThreads) {
    const int n = granules(P, u);
    total += n;
    if (u < unit) before += n;
  }
#pragma unroll
  for (int x = 1; x < 32; x <<= 1) {
    before += __shfl_xor_sync(0xffffffffu, before, x);
    total += __shfl_xor_sync(0xffffffffu, total, x);
  }
  if (lane == 0) { s_sum[0][warp] = before; s_sum[1][warp] = total; }
  __syncthreads();
  before = 0; total = 0;
  for (int w = 0; w < kJoinThreads / 32; ++w) { before += s_sum[0][w]; total += s_sum[1][w]; }
  total *= P.row_tiles;
  const int b = unit / c.Hkv, h = unit - b * c.Hkv;
  const int rows = row_count(P, row_counts, b);

  if (is_row) {
    const int r = job - unit * P.live, rr = P.row0 + r, rt = r / P.tile_rows, row = r - rt * P.tile_rows;
    const int m = rr % P.rows, j = h * P.G + rr / P.rows;
    if (m >= rows) return;                           // a row that the sequence has not got
    const Parts parts = parts_of(P, unit, rt, before, total);
    const float2 ml = join_stats(P, parts, row);     // (every warp for itself)
    constexpr int kLanes = kD / 4;                   // lanes of a part's row, 16 bytes each
    constexpr int kPer = 32 / kLanes;                // parts a warp reads side by side
    const int x = lane % kLanes;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (long long s = parts.first + warp * kPer + lane / kLanes; s <= parts.last; s += kPer * (kJoinThreads / 32)) {
      const float4 y = *reinterpret_cast<const float4*>(P.part_o + (s * P.tile_rows + row) * kD + 4 * x);
      const float f = ex2(P.part_ml[s * P.tile_rows + row].x - ml.x);
      a.x += y.x * f; a.y += y.y * f; a.z += y.z * f; a.w += y.w * f;
    }
    s_o[warp][lane] = a;
    __syncthreads();
    if (tid < kLanes) {
      for (int w = 0; w < kJoinThreads / 32; ++w)
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
          if (w + k == 0) continue;
          const float4 y = s_o[w][tid + k * kLanes];
          a.x += y.x; a.y += y.y; a.z += y.z; a.w += y.w;
        }
      const float inv = ml.y > 0.f ? 1.f / ml.y : 0.f;
      // place 8 k + g holds entries (kD / 8) g + 4 k ..
      T* dst = out + b * P.os[0] + j * P.os[1] + m * P.os[2] + (kD / 8) * (tid & 7) + 4 * (tid >> 3);
      a.x *= inv; a.y *= inv; a.z *= inv; a.w *= inv;
      if (sizeof(T) == 2) {
        const __nv_bfloat162 lo = __floats2bfloat162_rn(a.x, a.y), hi = __floats2bfloat162_rn(a.z, a.w);
        *reinterpret_cast<uint2*>(dst) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
      } else {
        *reinterpret_cast<float4*>(dst) = a;
      }
      if (tid == 0 && lse != nullptr)
        lse[((long long)b * P.Hq + j) * P.rows + m] = ml.y > 0.f ? (ml.x + log2f(ml.y)) * 0.693147180559945309f : -INFINITY;
    }
    return;
  }

  // ---- weights: the logits' log-sum-exps, then the tokens
  for (int r = warp; r < P.live; r += kJoinThreads / 32) {
    const int rt = r / P.tile_rows;
    const float2 ml = join_stats(P, parts_of(P, unit, rt, before, total), r - rt * P.tile_rows);
    if (lane == 0) s_lse[r] = ml.y > 0.f && (P.row0 + r) % P.rows < rows ? ml.x + log2f(ml.y) : INFINITY;     // (infinity: weighs nothing)
  }
  __syncthreads();
  for (long long tok = tok0 + tid; tok < min(tok0 + kJoinTokens, len); tok += kJoinThreads) {
    float w = 0.f;
    for (int rt = 0; rt < P.row_tiles; ++rt) {
      const float* s = P.logits + (((long long)unit * P.row_tiles + rt) * c.cap + tok) * P.logit_rows;
      const int n = min(P.live - rt * P.tile_rows, P.tile_rows);
      for (int i = 0; i < n; i += 2) {
        const float2 x = *reinterpret_cast<const float2*>(s + i);
        w += ex2(x.x - s_lse[rt * P.tile_rows + i]);
        if (i + 1 < n) w += ex2(x.y - s_lse[rt * P.tile_rows + i + 1]);
      }
    }
    const long long i = (long long)unit * c.cap + tok;
    weight_out[i] = (weight_in == nullptr ? 0.f : weight_in[i]) + w;
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
  P->Hq = d->n_q_heads; P->G = d->n_q_heads / P->c.Hkv; P->rows = d->rows; P->causal = d->causal;
  P->scale = d->scale > 0.f ? d->scale : 1.0f / sqrtf((float)P->c.d);
  const int eb = d->dtype == KVC_F32 ? 4 : 2;
  if ((s = resolve_strides(d->q_stride, P->c.Bt, P->Hq, P->rows, P->c.d, eb, false, "q_stride", P->qs)) != KVC_OK) return s;
  return resolve_strides(d->out_stride, P->c.Bt, P->Hq, P->rows, P->c.d, eb, true, "out_stride", P->os);
}

// Query rows of a KV head in one launch: tiles of 8, or of 16 where there are more (the codes' conversion is shared).
int tile_rows_of(int live) { return live <= 8 ? 8 : 16; }

struct AttendLayout {
  int live, tile_rows, row_tiles, logit_rows;
  size_t o, ml, logits, total;
};

AttendLayout attend_layout(const AttendParams& P, bool with_weight) {
  AttendLayout y;
  const long long all = (long long)P.G * P.rows;
  y.live = (int)(all < kMaxRows ? all : kMaxRows);
  y.tile_rows = tile_rows_of(y.live);
  y.row_tiles = (y.live + y.tile_rows - 1) / y.tile_rows;
  y.logit_rows = 2;
  while (y.logit_rows < y.live && y.logit_rows < y.tile_rows) y.logit_rows *= 2;
  const size_t slots = (size_t)kMaxCtas + (size_t)P.c.units() * y.row_tiles;
  y.o = 0;
  y.ml = align_up(slots * y.tile_rows * P.c.d * sizeof(float));
  y.logits = y.ml + align_up(slots * y.tile_rows * sizeof(float2));
  y.total = y.logits + (with_weight ? align_up((size_t)P.c.units() * y.row_tiles * P.c.cap * y.logit_rows * sizeof(float)) : 0);
  return y;
}

template <typename T, int kFormat, int kD, int kTiles, bool kWeight>
kvc_status launch_split(const AttendParams& P, const T* q, const int32_t* row_counts, cudaStream_t st) {
  using W = Warp<kFormat, kD, kTiles, sizeof(T) == 4, kWeight>;
  auto kernel = attend_split_kernel<T, kFormat, kD, kTiles, kWeight>;
  constexpr int stages = kWarps * W::kStages * W::kStageBytes, join = kWarps * 8 * kTiles * (kD + 4) * (int)sizeof(float);
  constexpr int smem = stages > join ? stages : join;
  KVC_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  KVC_CUDA(launch_dependent(kernel, dim3(P.ctas), dim3(kAttThreads), smem, st, P, q, row_counts));
  KVC_LAUNCH_CHECK("attend_split_kernel");
  return KVC_OK;
}

template <typename T, int kFormat, int kD>
kvc_status launch_split_form(const AttendParams& P, bool weight, const T* q, const int32_t* row_counts, cudaStream_t st) {
  if (P.tile_rows == 8)
    return weight ? launch_split<T, kFormat, kD, 1, true>(P, q, row_counts, st) : launch_split<T, kFormat, kD, 1, false>(P, q, row_counts, st);
  return weight ? launch_split<T, kFormat, kD, 2, true>(P, q, row_counts, st) : launch_split<T, kFormat, kD, 2, false>(P, q, row_counts, st);
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
    const long long chunks = weight ? (P.c.cap + kJoinTokens - 1) / kJoinTokens : 0;
    const long long ctas = P.c.units() * (P.live + chunks);
    KVC_REQUIRE8(ctas < (1LL << 31), KVC_ERR_UNSUPPORTED, "batch * n_kv_heads * capacity is too large");
    KVC_CUDA(launch_dependent(P.c.d == 128 ? attend_join_kernel<T, 128> : attend_join_kernel<T, 64>, dim3((unsigned)ctas), dim3(kJoinThreads),
                              0, st, P, row_counts, out, lse, weight_in, weight_out, (int)chunks));
    KVC_LAUNCH_CHECK("attend_join_kernel");
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
  *bytes = attend_layout(P, with_weight != 0).total;
  return KVC_OK;
}

kvc_status kvc_attend(const kvc_cache* cache, const kvc_attend_desc* desc, const void* q, const int32_t* row_counts, void* out, float* lse,
                      const float* weight_in, float* weight_out, void* workspace, size_t workspace_bytes, void* stream) {
  AttendParams P;
  kvc_status s = resolve_attend(cache, desc, &P);
  if (s != KVC_OK) return s;
  KVC_REQUIRE8(q && out && aligned16(q) && aligned16(out), KVC_ERR_INVALID_ARG, "q or out is NULL or not 16-byte aligned");
  KVC_REQUIRE8(weight_in == nullptr || weight_out != nullptr, KVC_ERR_INVALID_ARG, "weight_in without weight_out");
  const AttendLayout y = attend_layout(P, weight_out != nullptr);
  KVC_REQUIRE8(workspace != nullptr, KVC_ERR_WORKSPACE, "workspace is NULL (%zu bytes needed)", y.total);
  KVC_REQUIRE8((reinterpret_cast<uintptr_t>(workspace) & 255u) == 0, KVC_ERR_WORKSPACE, "workspace is not 256-byte aligned");
  KVC_REQUIRE8(workspace_bytes >= y.total, KVC_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, y.total);
  if ((s = require_device()) != KVC_OK) return s;
  int dev = 0, sms = 0;
  KVC_CUDA(cudaGetDevice(&dev));
  KVC_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  P.ctas = sms < kMaxCtas ? sms : kMaxCtas;
  P.tile_rows = y.tile_rows; P.logit_rows = y.logit_rows;
  P.part_o = (float*)((char*)workspace + y.o);
  P.part_ml = (float2*)((char*)workspace + y.ml);
  P.logits = (float*)((char*)workspace + y.logits);
  return desc->dtype == KVC_F32 ? run_attend<float>(P, y, (const float*)q, row_counts, (float*)out, lse, weight_in, weight_out, (cudaStream_t)stream)
                                : run_attend<__nv_bfloat16>(P, y, (const __nv_bfloat16*)q, row_counts, (__nv_bfloat16*)out, lse, weight_in,
                                                            weight_out, (cudaStream_t)stream);
}

}  // extern "C"
