// Rotary positions (kvc_rotary): pair i of a row at position p is turned by the angle p f_i.
//
// Every value is read once and written once; the bound is HBM.  The angles of a row are the same in all of its heads, so a CTA
// takes a tile of rows of one sequence with all heads (or, for few rows, a share of the heads), forms the tile's cosines and
// sines in shared memory once, and each thread keeps its eight pairs of them in registers while it goes from head to head,
// kRotUnroll heads' loads (32 bytes of a row each, 64 in fp32) in flight.
// Angles: p f_i / 2pi in 64 bits, the whole turns taken off there (fp32 loses 0.008 rad at p = 131072, more than half a
// step of bf16), the rest of a turn in fp32 through sincospif.
// B200: 16001 tokens of 32 + 8 heads of 128 in bf16 58.5 us, 5.6 TB/s of reads and writes (a copy: 6.5); one token of 32
// sequences 2.3 us, a launch.
#include <math.h>

#include "cache8.cuh"

namespace kvc {
namespace {

constexpr int kRotThreads = 256;
constexpr int kRotRows = 8;                  // rows of a tile (16 with four heads in flight: 65 us instead of 62 for the prompt below)
constexpr int kRotUnroll = 2;                // heads in flight

struct RotaryParams {
  int Hq, Hkv, d, rows, rot, tile_shift, heads_per_cta;      // tiles of 2^tile_shift rows
  long long qs[3], ks[3], qo[3], ko[3];
  long long pos_stride;
  float mscale;
  double turn[64];                           // f_i / 2pi, negated for the inverse
};

template <typename T>
__device__ __forceinline__ void store8(T* p, const float* x) {
  if (sizeof(T) == 2) {
    uint4 w;
    uint32_t* u = &w.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      u[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    __stcs(reinterpret_cast<uint4*>(p), w);              // (written once, not read here: 62 -> 58.5 us for the prompt above; a decoded
                                                         // token's rows, a few KB that the next kernel reads, are found in L2 all the same)
  } else {
    __stcs(reinterpret_cast<float4*>(p), make_float4(x[0], x[1], x[2], x[3]));
    __stcs(reinterpret_cast<float4*>(p + 4), make_float4(x[4], x[5], x[6], x[7]));
  }
}

// A step of a thread: 16 values of a row, eight pairs or, behind rot_dim, a copy.
template <typename T, bool kInterleaved>
__global__ void __launch_bounds__(kRotThreads)
rotary_kernel(const __grid_constant__ RotaryParams P, const T* q, const T* k, const int64_t* __restrict__ positions, T* q_out,
              T* k_out) {
  __shared__ float2 cs[kRotRows * 64];
  grid_dependency_wait();
  const int row0 = blockIdx.x << P.tile_shift, b = blockIdx.y;
  const int n = min(1 << P.tile_shift, P.rows - row0), half = P.rot >> 1;
  for (int i = threadIdx.x; i < n * half; i += kRotThreads) {
    const int r = i / half, j = i - r * half;
    const double t = (double)positions[b * P.pos_stride + row0 + r] * P.turn[j];
    float s, c;
    sincospif(2.f * (float)(t - rint(t)), &s, &c);
    cs[i] = make_float2(c * P.mscale, s * P.mscale);
  }
  __syncthreads();

  // thread: a step c of a row r, of every `side`-th head
  const int steps_shift = P.d == 128 ? 3 : 2, shift = steps_shift + P.tile_shift, side = kRotThreads >> shift;
  const int c = threadIdx.x & ((1 << steps_shift) - 1), r = (threadIdx.x & ((1 << shift) - 1)) >> steps_shift;
  if (r >= n) return;
  const bool copy = 16 * c >= P.rot;
  const int first = copy || kInterleaved ? 16 * c : 8 * c, second = copy || kInterleaved ? 16 * c + 8 : half + 8 * c;
  float2 a[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) a[j] = copy ? make_float2(1.f, 0.f) : cs[r * half + 8 * c + j];
  const long long row = row0 + r;
  const T *qi = q + b * P.qs[0] + row * P.qs[2], *ki = k + b * P.ks[0] + row * P.ks[2];
  T *qo = q_out + b * P.qo[0] + row * P.qo[2], *ko = k_out + b * P.ko[0] + row * P.ko[2];
  const int head1 = min((int)(blockIdx.z + 1) * P.heads_per_cta, P.Hq + P.Hkv);
  for (int h0 = blockIdx.z * P.heads_per_cta + (threadIdx.x >> shift); h0 < head1; h0 += side * kRotUnroll) {
    Raw8<T> w[kRotUnroll][2];
#pragma unroll
    for (int u = 0; u < kRotUnroll; ++u) {
      const int h = h0 + u * side;
      if (h >= head1) break;
      const T* in = h < P.Hq ? qi + h * P.qs[1] : ki + (h - P.Hq) * P.ks[1];
      w[u][0].load_coherent(in + first);      // (an output may be its input)
      w[u][1].load_coherent(in + second);
    }
#pragma unroll
    for (int u = 0; u < kRotUnroll; ++u) {
      const int h = h0 + u * side;
      if (h >= head1) break;
      T* out = h < P.Hq ? qo + h * P.qo[1] : ko + (h - P.Hq) * P.ko[1];
      if (copy) {
        w[u][0].store(out + first);
        w[u][1].store(out + second);
        continue;
      }
      float x[16], y[16];
      w[u][0].values(x);
      w[u][1].values(x + 8);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int i0 = kInterleaved ? 2 * j : j, i1 = kInterleaved ? 2 * j + 1 : 8 + j;
        y[i0] = x[i0] * a[j].x - x[i1] * a[j].y;
        y[i1] = x[i1] * a[j].x + x[i0] * a[j].y;
      }
      store8(out + first, y);
      store8(out + second, y + 8);
    }
  }
}

template <typename T>
kvc_status launch_rotary(bool interleaved, const RotaryParams& P, dim3 grid, const void* q, const void* k,
                         const int64_t* positions, void* q_out, void* k_out, cudaStream_t st) {
  auto kernel = interleaved ? rotary_kernel<T, true> : rotary_kernel<T, false>;
  KVC_CUDA(launch_dependent(kernel, grid, dim3(kRotThreads), 0, st, P, (const T*)q, (const T*)k, positions, (T*)q_out, (T*)k_out));
  KVC_LAUNCH_CHECK("rotary_kernel");
  return KVC_OK;
}

}  // namespace
}  // namespace kvc

using namespace kvc;

extern "C" {

kvc_status kvc_rope_init(kvc_rope* R, int32_t rot_dim, int32_t interleaved, double theta, int32_t scaling, double factor,
                         double turns_low, double turns_high, double original_ctx, double mscale) {
  KVC_REQUIRE8(R != nullptr, KVC_ERR_INVALID_ARG, "rope is NULL");
  KVC_REQUIRE8(rot_dim >= 16 && rot_dim <= 128 && rot_dim % 16 == 0, KVC_ERR_UNSUPPORTED, "rot_dim must be a multiple of 16 within [16, 128]");
  KVC_REQUIRE8(interleaved == 0 || interleaved == 1, KVC_ERR_INVALID_ARG, "interleaved must be 0 or 1");
  KVC_REQUIRE8(isfinite(theta) && theta > 1.0, KVC_ERR_INVALID_ARG, "theta must be finite and > 1");
  KVC_REQUIRE8(scaling >= KVC_ROPE_NONE && scaling <= KVC_ROPE_YARN, KVC_ERR_INVALID_ARG, "unknown scaling");
  KVC_REQUIRE8(scaling == KVC_ROPE_NONE || (isfinite(factor) && factor >= 1.0), KVC_ERR_INVALID_ARG, "factor must be finite and >= 1");
  if (scaling == KVC_ROPE_BANDED || scaling == KVC_ROPE_YARN) {
    KVC_REQUIRE8(isfinite(turns_high) && turns_low > 0 && turns_high > turns_low, KVC_ERR_INVALID_ARG, "0 < turns_low < turns_high is needed");
    KVC_REQUIRE8(isfinite(original_ctx) && original_ctx > 0, KVC_ERR_INVALID_ARG, "original_ctx must be positive");
  }
  KVC_REQUIRE8(isfinite(mscale) && mscale >= 0, KVC_ERR_INVALID_ARG, "mscale must be finite and >= 0");
  const double two_pi = 6.283185307179586476925286766559;
  const double lt = log(theta);
  double first = 0, last = 0;
  if (scaling == KVC_ROPE_YARN) {
    first = floor(rot_dim * log(original_ctx / (turns_high * two_pi)) / (2.0 * lt));
    last = ceil(rot_dim * log(original_ctx / (turns_low * two_pi)) / (2.0 * lt));
    if (first < 0) first = 0;
    if (last > rot_dim - 1) last = rot_dim - 1;
  }
  for (int i = 0; i < 64; ++i) {
    double f = i < rot_dim / 2 ? pow(theta, -2.0 * i / rot_dim) : 0.0;
    if (scaling == KVC_ROPE_LINEAR) {
      f /= factor;
    } else if (scaling == KVC_ROPE_BANDED) {
      double keep = (original_ctx * f / two_pi - turns_low) / (turns_high - turns_low);
      keep = keep < 0 ? 0 : (keep > 1 ? 1 : keep);
      f = keep * f + (1.0 - keep) * f / factor;
    } else if (scaling == KVC_ROPE_YARN) {
      const double width = last - first > 0.001 ? last - first : 0.001;
      double ramp = (i - first) / width;
      ramp = ramp < 0 ? 0 : (ramp > 1 ? 1 : ramp);
      f = (1.0 - ramp) * f + ramp * f / factor;
    }
    R->turn[i] = f / two_pi;
  }
  R->rot_dim = rot_dim;
  R->interleaved = interleaved;
  R->mscale = mscale > 0 ? mscale : scaling == KVC_ROPE_YARN ? 0.1 * log(factor) + 1.0 : 1.0;
  return KVC_OK;
}

kvc_status kvc_rotary(const kvc_rope* R, const kvc_rope_desc* D, const void* q, const void* k, const int64_t* positions, int64_t pos_stride,
                      void* q_out, void* k_out, void* stream) {
  KVC_REQUIRE8(R != nullptr && D != nullptr, KVC_ERR_INVALID_ARG, "rope or desc is NULL");
  KVC_REQUIRE8(D->batch >= 1 && D->rows >= 1, KVC_ERR_INVALID_ARG, "batch and rows must be >= 1");
  KVC_REQUIRE8(D->batch <= 65535, KVC_ERR_UNSUPPORTED, "batch > 65535");
  KVC_REQUIRE8(D->rows <= (1 << 30), KVC_ERR_UNSUPPORTED, "rows > 2^30");
  KVC_REQUIRE8(D->head_dim == 64 || D->head_dim == 128, KVC_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
  KVC_REQUIRE8(R->rot_dim >= 16 && R->rot_dim <= D->head_dim && R->rot_dim % 16 == 0, KVC_ERR_UNSUPPORTED,
               "rot_dim must be a multiple of 16 within [16, head_dim]");
  kvc_status s = check_dtype(D->dtype);
  if (s != KVC_OK) return s;
  KVC_REQUIRE8(D->inverse == 0 || D->inverse == 1, KVC_ERR_INVALID_ARG, "inverse must be 0 or 1");
  KVC_REQUIRE8(D->reserved_ == 0, KVC_ERR_INVALID_ARG, "reserved_ must be 0");
  KVC_REQUIRE8(q != nullptr || k != nullptr, KVC_ERR_INVALID_ARG, "q and k are both NULL");
  KVC_REQUIRE8((q == nullptr) == (q_out == nullptr) && (k == nullptr) == (k_out == nullptr), KVC_ERR_INVALID_ARG,
               "q and q_out, k and k_out go together");
  KVC_REQUIRE8(positions != nullptr && pos_stride >= 0, KVC_ERR_INVALID_ARG, "positions is NULL or pos_stride negative");
  const void* ptrs[4] = {q, k, q_out, k_out};
  for (const void* p : ptrs) KVC_REQUIRE8(aligned16(p), KVC_ERR_INVALID_ARG, "q, k and the outputs must be 16-byte aligned");
  RotaryParams P;
  P.Hq = q ? D->n_q_heads : 0;
  P.Hkv = k ? D->n_kv_heads : 0;
  KVC_REQUIRE8((!q || D->n_q_heads >= 1) && (!k || D->n_kv_heads >= 1), KVC_ERR_INVALID_ARG, "head counts must be >= 1");
  KVC_REQUIRE8(P.Hq <= kMaxQHeads && P.Hkv <= kMaxQHeads, KVC_ERR_UNSUPPORTED, "more than %d heads", kMaxQHeads);
  P.d = D->head_dim; P.rows = D->rows; P.rot = R->rot_dim; P.pos_stride = pos_stride;
  const int eb = D->dtype == KVC_F32 ? 4 : 2;
  if (q && (s = resolve_strides(D->q_stride, D->batch, P.Hq, P.rows, P.d, eb, false, "q_stride", P.qs)) != KVC_OK) return s;
  if (q && (s = resolve_strides(D->q_out_stride, D->batch, P.Hq, P.rows, P.d, eb, true, "q_out_stride", P.qo)) != KVC_OK) return s;
  if (k && (s = resolve_strides(D->k_stride, D->batch, P.Hkv, P.rows, P.d, eb, false, "k_stride", P.ks)) != KVC_OK) return s;
  if (!q) P.qs[0] = P.qs[1] = P.qs[2] = P.qo[0] = P.qo[1] = P.qo[2] = 0;
  if (!k) P.ks[0] = P.ks[1] = P.ks[2] = P.ko[0] = P.ko[1] = P.ko[2] = 0;
  if (k && (s = resolve_strides(D->k_out_stride, D->batch, P.Hkv, P.rows, P.d, eb, true, "k_out_stride", P.ko)) != KVC_OK) return s;
  P.mscale = (float)R->mscale;
  if ((s = require_device()) != KVC_OK) return s;
  for (int i = 0; i < 64; ++i) P.turn[i] = D->inverse ? -R->turn[i] : R->turn[i];

  P.tile_shift = 0;
  while ((1 << P.tile_shift) < kRotRows && (1 << P.tile_shift) < P.rows) ++P.tile_shift;
  const long long tiles = ((long long)P.rows + (1 << P.tile_shift) - 1) >> P.tile_shift;
  const int heads = P.Hq + P.Hkv;
  // few rows: a CTA takes only as many heads as give each of its threads a step
  P.heads_per_cta = heads;
  if (tiles * D->batch < 296) {
    const int steps = (P.d / 16) << P.tile_shift;
    P.heads_per_cta = kRotThreads / steps < heads ? kRotThreads / steps : heads;
  }
  const dim3 grid((unsigned)tiles, D->batch, (heads + P.heads_per_cta - 1) / P.heads_per_cta);
  const bool il = R->interleaved != 0;
  return D->dtype == KVC_F32 ? launch_rotary<float>(il, P, grid, q, k, positions, q_out, k_out, (cudaStream_t)stream)
                             : launch_rotary<__nv_bfloat16>(il, P, grid, q, k, positions, q_out, k_out, (cudaStream_t)stream);
}

}  // extern "C"
