// Rotary positions (kvc_rotary): pair i of a row at position p is turned by the angle p f_i.
//
// Every value is read once and written once; the bound is HBM.  The angles of a row are the same in all of its heads, so
// a CTA takes a tile of rows of one sequence with all heads (or, for few rows, a share of the heads), forms the tile's
// cosines and sines in shared memory once, and streams the heads past them, 32 bytes of a row per thread and step.
// Angles: p f_i / 2pi in 64 bits, the whole turns taken off there (fp32 loses 0.008 rad at p = 131072, more than half a
// step of bf16), the rest of a turn in fp32 through sincospif.
#include <math.h>

#include "cache8.cuh"

namespace kvc {
namespace {

constexpr int kRotThreads = 256;
constexpr int kRotRows = 16;                 // rows of a tile

struct RotaryParams {
  int Hq, Hkv, d, rows, rot, tile_rows, heads_per_cta;
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
    *reinterpret_cast<uint4*>(p) = w;
  } else {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
  }
}

template <typename T>
__device__ __forceinline__ void load8_any(const T* p, float* x) {   // (through the coherent path: an output may be its input)
  if (sizeof(T) == 2) {
    const uint4 w = ld16(p);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(u[i] << 16);
      x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  } else {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
}

// A step of a thread: 16 values of a row, eight pairs or, behind rot_dim, a copy.
template <typename T, bool kInterleaved>
__global__ void __launch_bounds__(kRotThreads)
rotary_kernel(const __grid_constant__ RotaryParams P, const T* q, const T* k, const int64_t* __restrict__ positions, T* q_out,
              T* k_out) {
  __shared__ float2 cs[kRotRows * 64];
  grid_dependency_wait();
  const int row0 = blockIdx.x * P.tile_rows, b = blockIdx.y;
  const int n = min(P.tile_rows, P.rows - row0), half = P.rot >> 1;
  for (int i = threadIdx.x; i < n * half; i += kRotThreads) {
    const int r = i / half, j = i - r * half;
    const double t = (double)positions[b * P.pos_stride + row0 + r] * P.turn[j];
    float s, c;
    sincospif(2.f * (float)(t - rint(t)), &s, &c);
    cs[i] = make_float2(c * P.mscale, s * P.mscale);
  }
  __syncthreads();

  const int steps_shift = P.d == 128 ? 3 : 2;               // log2 of steps per row
  const int per_head = n << steps_shift;
  const int head0 = blockIdx.z * P.heads_per_cta;
  const int heads = min(P.heads_per_cta, P.Hq + P.Hkv - head0);
  for (int i = threadIdx.x; i < per_head * heads; i += kRotThreads) {
    const int hh = i / per_head, rest = i - hh * per_head;
    const int r = rest >> steps_shift, c = rest & ((1 << steps_shift) - 1);
    int h = head0 + hh;
    const T* in;
    T* out;
    if (h < P.Hq) {
      in = q + b * P.qs[0] + h * P.qs[1] + (row0 + r) * P.qs[2];
      out = q_out + b * P.qo[0] + h * P.qo[1] + (row0 + r) * P.qo[2];
    } else {
      h -= P.Hq;
      in = k + b * P.ks[0] + h * P.ks[1] + (row0 + r) * P.ks[2];
      out = k_out + b * P.ko[0] + h * P.ko[1] + (row0 + r) * P.ko[2];
    }
    float x[16], y[16];
    if (16 * c >= P.rot) {
      load8_any(in + 16 * c, x);
      load8_any(in + 16 * c + 8, x + 8);
      store8(out + 16 * c, x);
      store8(out + 16 * c + 8, x + 8);
      continue;
    }
    const int first = kInterleaved ? 16 * c : 8 * c, second = kInterleaved ? 16 * c + 8 : half + 8 * c;
    load8_any(in + first, x);
    load8_any(in + second, x + 8);
    const float2* a = cs + r * half + 8 * c;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int u = kInterleaved ? 2 * j : j, v = kInterleaved ? 2 * j + 1 : 8 + j;
      y[u] = x[u] * a[j].x - x[v] * a[j].y;
      y[v] = x[v] * a[j].x + x[u] * a[j].y;
    }
    store8(out + first, y);
    store8(out + second, y + 8);
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
  if (k && (s = resolve_strides(D->k_out_stride, D->batch, P.Hkv, P.rows, P.d, eb, true, "k_out_stride", P.ko)) != KVC_OK) return s;
  P.mscale = (float)R->mscale;
  if ((s = require_device()) != KVC_OK) return s;
  for (int i = 0; i < 64; ++i) P.turn[i] = D->inverse ? -R->turn[i] : R->turn[i];

  P.tile_rows = P.rows < kRotRows ? P.rows : kRotRows;
  const long long tiles = (P.rows + P.tile_rows - 1) / P.tile_rows;
  const int heads = P.Hq + P.Hkv;
  // few rows: a CTA takes only as many heads as give each of its threads a step
  P.heads_per_cta = heads;
  if (tiles * D->batch < 296) {
    const int steps = P.tile_rows * P.d / 16;
    P.heads_per_cta = (kRotThreads + steps - 1) / steps;
    if (P.heads_per_cta > heads) P.heads_per_cta = heads;
  }
  const dim3 grid((unsigned)tiles, D->batch, (heads + P.heads_per_cta - 1) / P.heads_per_cta);
  const bool il = R->interleaved != 0;
  return D->dtype == KVC_F32 ? launch_rotary<float>(il, P, grid, q, k, positions, q_out, k_out, (cudaStream_t)stream)
                             : launch_rotary<__nv_bfloat16>(il, P, grid, q, k, positions, q_out, k_out, (cudaStream_t)stream);
}

}  // extern "C"
