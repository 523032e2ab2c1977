// Attention of a few query rows over an 8-bit cache (kvc_attend), first form: one CTA per KV head walks its tokens for
// one query row after another, fp32 throughout.
#include "cache8.cuh"

namespace kvc {
namespace {

constexpr int kAttThreads = 256;

struct AttendParams {
  Cache c;
  int Hq, G, rows, causal;
  float scale;
  long long qs[3], os[3];
};

__device__ __forceinline__ float block_reduce(float x, bool is_max, float* scratch) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float y = __shfl_xor_sync(0xffffffffu, x, o);
    x = is_max ? fmaxf(x, y) : x + y;
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = x;
  __syncthreads();
  x = scratch[0];
  for (int i = 1; i < kAttThreads / 32; ++i) x = is_max ? fmaxf(x, scratch[i]) : x + scratch[i];
  return x;
}

template <typename T, int kFormat>
__global__ void __launch_bounds__(kAttThreads)
attend_kernel(const __grid_constant__ AttendParams P, const T* __restrict__ q, const int32_t* __restrict__ row_counts,
              T* __restrict__ out, float* __restrict__ lse, const float* weight_in, float* weight_out, float* __restrict__ logits) {
  __shared__ float sq[128], scratch[8], so[kAttThreads];
  grid_dependency_wait();
  const Cache& c = P.c;
  const int unit = blockIdx.x, b = unit / c.Hkv, h = unit - b * c.Hkv, tid = threadIdx.x;
  const long long len = c.length(unit);
  int rows = row_counts == nullptr ? P.rows : row_counts[b];
  rows = rows < 0 ? 0 : (rows > P.rows ? P.rows : rows);
  const uint8_t *kc = c.k + c.base(unit), *vc = c.v + c.base(unit);
  const int8_t *ke = c.k_exp + (long long)unit * c.blocks, *ve = c.v_exp + (long long)unit * c.blocks;
  float* s = logits + unit * c.cap;
  if (weight_out != nullptr)
    for (long long i = tid; i < len; i += kAttThreads) weight_out[unit * c.cap + i] = weight_in == nullptr ? 0.f : weight_in[unit * c.cap + i];
  for (int gr = 0; gr < P.G * rows; ++gr) {
    const int j = h * P.G + gr / rows, m = gr % rows;
    long long seen = P.causal ? len - (rows - 1 - m) : len;
    if (seen < 0) seen = 0;
    __syncthreads();
    if (tid < c.d) sq[tid] = (float)q[b * P.qs[0] + j * P.qs[1] + m * P.qs[2] + tid] * P.scale;
    __syncthreads();
    float top = -INFINITY;
    for (long long i = tid; i < seen; i += kAttThreads) {
      const uint8_t* row = kc + i * c.st[2];
      float dot = 0.f;
      for (int x = 0; x < c.d; x += 4) {
        float y[4];
        decode4<kFormat>(*reinterpret_cast<const uint32_t*>(row + x), y);
        for (int u = 0; u < 4; ++u) dot += sq[x + u] * y[u];
      }
      dot *= pow2_clamped(ke[i >> c.block_shift]);
      s[i] = dot;
      top = fmaxf(top, dot);
    }
    top = block_reduce(top, true, scratch);
    float sum = 0.f;
    for (long long i = tid; i < seen; i += kAttThreads) {
      s[i] = expf(s[i] - top);
      sum += s[i];
    }
    sum = block_reduce(sum, false, scratch);        // (its barriers also make the logits visible to the CTA)
    const float inv = seen > 0 ? 1.f / sum : 0.f;
    if (weight_out != nullptr)
      for (long long i = tid; i < seen; i += kAttThreads) weight_out[unit * c.cap + i] += s[i] * inv;
    const int x = tid % c.d, part = tid / c.d, parts = kAttThreads / c.d;
    float acc = 0.f;
    for (long long i = part; i < seen; i += parts) {
      float y[4];
      decode4<kFormat>(vc[i * c.st[2] + x], y);
      acc += s[i] * (y[0] * pow2_clamped(ve[i >> c.block_shift]));
    }
    so[tid] = acc;
    __syncthreads();
    if (part == 0) {
      for (int u = 1; u < parts; ++u) acc += so[u * c.d + x];
      out[b * P.os[0] + j * P.os[1] + m * P.os[2] + x] = (T)(acc * inv);
    }
    if (tid == 0 && lse != nullptr) lse[((long long)b * P.Hq + j) * P.rows + m] = seen > 0 ? top + logf(sum) : -INFINITY;
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

size_t attend_workspace_bytes(const AttendParams& P, bool with_weight) { return align_up((size_t)P.c.units() * P.c.cap * sizeof(float)); }

}  // namespace
}  // namespace kvc

using namespace kvc;

extern "C" {

kvc_status kvc_attend_workspace_size(const kvc_cache* cache, const kvc_attend_desc* desc, int32_t with_weight, size_t* bytes) {
  AttendParams P;
  const kvc_status s = resolve_attend(cache, desc, &P);
  if (s != KVC_OK) return s;
  KVC_REQUIRE8(bytes != nullptr, KVC_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = attend_workspace_bytes(P, with_weight != 0);
  return KVC_OK;
}

kvc_status kvc_attend(const kvc_cache* cache, const kvc_attend_desc* desc, const void* q, const int32_t* row_counts, void* out, float* lse,
                      const float* weight_in, float* weight_out, void* workspace, size_t workspace_bytes, void* stream) {
  AttendParams P;
  kvc_status s = resolve_attend(cache, desc, &P);
  if (s != KVC_OK) return s;
  KVC_REQUIRE8(q && out && aligned16(q) && aligned16(out), KVC_ERR_INVALID_ARG, "q or out is NULL or not 16-byte aligned");
  KVC_REQUIRE8(weight_in == nullptr || weight_out != nullptr, KVC_ERR_INVALID_ARG, "weight_in without weight_out");
  const size_t need = attend_workspace_bytes(P, weight_out != nullptr);
  KVC_REQUIRE8(workspace != nullptr, KVC_ERR_WORKSPACE, "workspace is NULL (%zu bytes needed)", need);
  KVC_REQUIRE8((reinterpret_cast<uintptr_t>(workspace) & 255u) == 0, KVC_ERR_WORKSPACE, "workspace is not 256-byte aligned");
  KVC_REQUIRE8(workspace_bytes >= need, KVC_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, need);
  if ((s = require_device()) != KVC_OK) return s;
  const bool e4m3 = P.c.format == KVC_E4M3;
  const dim3 grid(P.c.units());
  cudaStream_t st = (cudaStream_t)stream;
  if (desc->dtype == KVC_F32)
    KVC_CUDA(launch_dependent(e4m3 ? attend_kernel<float, KVC_E4M3> : attend_kernel<float, KVC_INT8>, grid, dim3(kAttThreads), 0, st, P,
                              (const float*)q, row_counts, (float*)out, lse, weight_in, weight_out, (float*)workspace));
  else
    KVC_CUDA(launch_dependent(e4m3 ? attend_kernel<__nv_bfloat16, KVC_E4M3> : attend_kernel<__nv_bfloat16, KVC_INT8>, grid,
                              dim3(kAttThreads), 0, st, P, (const __nv_bfloat16*)q, row_counts, (__nv_bfloat16*)out, lse, weight_in,
                              weight_out, (float*)workspace));
  KVC_LAUNCH_CHECK("attend_kernel");
  return KVC_OK;
}

}  // extern "C"
