// Eviction from an 8-bit cache by accumulated attention weight (kvc_evict).
//
// Two kernels.  evict_select_kernel, one CTA per head: the k-th largest of the weights before the protected rows is found
// digit by digit (11, 11 and 10 bits of an order-preserving key, a histogram in shared memory each), then the kept
// positions are written in order by counting along the row.  evict_move_kernel, a job per block of the new cache (see
// cache8.cuh): kept rows are read once, take the exponent of their new block and are written once.
#include "cache8.cuh"

namespace kvc {
namespace {

constexpr int kSelThreads = 1024;
constexpr int kBins = 2048;

struct EvictParams {
  Cache src, dst;
  long long budget, recent;
};

// Exclusive prefix sum over the CTA of a 0/1 flag, and the total; two barriers.
__device__ __forceinline__ int flag_scan(bool flag, int* warp_sums, int* total) {
  const uint32_t m = __ballot_sync(0xffffffffu, flag);
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  if (lane == 0) warp_sums[w] = __popc(m);
  __syncthreads();
  const int mine = lane < kSelThreads / 32 ? warp_sums[lane] : 0;
  const int before = __reduce_add_sync(0xffffffffu, lane < w ? mine : 0);
  *total = __reduce_add_sync(0xffffffffu, mine);
  __syncthreads();
  return before + __popc(m & ((1u << lane) - 1u));
}

__global__ void __launch_bounds__(kSelThreads)
evict_select_kernel(const __grid_constant__ EvictParams P, const float* __restrict__ weight, int32_t* __restrict__ idx_out,
                    float* __restrict__ weight_out) {
  __shared__ int hist[kBins];
  __shared__ int warp_sums[kSelThreads / 32];
  __shared__ int s_bin, s_before;
  grid_dependency_wait();
  const int unit = blockIdx.x, tid = threadIdx.x;
  const long long n = P.src.length(unit);
  const float* w = weight + unit * P.src.cap;
  int32_t* idx = idx_out + unit * P.budget;
  float* wo = weight_out == nullptr ? nullptr : weight_out + unit * P.dst.cap;
  const long long kept = n < P.budget ? n : P.budget;
  if (tid == 0) P.dst.lengths[unit] = (int32_t)kept;
  for (long long i = kept + tid; i < P.budget; i += kSelThreads) idx[i] = -1;
  if (n <= P.budget) {
    for (long long i = tid; i < n; i += kSelThreads) {
      idx[i] = (int32_t)i;
      if (wo != nullptr) wo[i] = w[i];
    }
    return;
  }
  // the heaviest `want` of the first `m` rows (keys ascend as weights descend)
  const long long m = n - P.recent;
  int want = (int)(P.budget - P.recent);
  uint32_t prefix = 0;                  // the digits found so far
  int ties = 0;                         // of the rows with exactly the threshold's key, the first `ties` are kept
  if (want > 0) {
    int shift = 32;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      const int bits = pass == 2 ? 10 : 11;
      for (int i = tid; i < kBins; i += kSelThreads) hist[i] = 0;
      __syncthreads();
      const int up = shift;             // bits from `up` on are fixed
      shift -= bits;
      for (long long i = tid; i < m; i += kSelThreads) {
        const uint32_t key = score_to_key(w[i]);
        if (pass == 0 || (key >> up) == (prefix >> up)) atomicAdd(&hist[(key >> shift) & ((1 << bits) - 1)], 1);
      }
      __syncthreads();
      // the bin that the want-th row falls into: two bins per thread, scanned over the CTA
      const int a = hist[2 * tid], b = hist[2 * tid + 1];
      int x = a + b;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if ((tid & 31) >= o) x += y;
      }
      if ((tid & 31) == 31) warp_sums[tid >> 5] = x;
      __syncthreads();
      const int other = warp_sums[tid & 31];
      const int before = __reduce_add_sync(0xffffffffu, (tid & 31) < (tid >> 5) ? other : 0) + x - a - b;
      if (before < want && want <= before + a + b) {
        const int first = want <= before + a;
        s_bin = first ? 2 * tid : 2 * tid + 1;
        s_before = first ? before : before + a;
      }
      __syncthreads();
      prefix |= (uint32_t)s_bin << shift;
      want -= s_before;
      __syncthreads();
    }
    ties = want;
  }
  // positions in order
  long long done = 0;
  int ties_done = 0;
  for (long long i0 = 0; i0 < m; i0 += kSelThreads) {
    const long long i = i0 + tid;
    const float x = i < m ? w[i] : 0.f;
    const uint32_t key = score_to_key(x);
    const bool equal = i < m && ties > 0 && key == prefix;
    int total;
    const int rank = flag_scan(equal, warp_sums, &total) + ties_done;
    const bool keep = i < m && ties > 0 && (key < prefix || (equal && rank < ties));
    ties_done += total;
    const int at = flag_scan(keep, warp_sums, &total);
    if (keep) {
      idx[done + at] = (int32_t)i;
      if (wo != nullptr) wo[done + at] = x;
    }
    done += total;
  }
  for (long long i = tid; i < P.recent; i += kSelThreads) {
    idx[P.budget - P.recent + i] = (int32_t)(m + i);
    if (wo != nullptr) wo[P.budget - P.recent + i] = w[m + i];
  }
}

template <int kFormat>
__global__ void __launch_bounds__(512)
evict_move_kernel(const __grid_constant__ EvictParams P, const int32_t* __restrict__ idx_out) {
  __shared__ float2 scratch[16];
  grid_dependency_wait();
  const int unit = blockIdx.y;
  const int n = (int)P.dst.length(unit);
  const JobLane<16> j(P.dst.block_shift, P.dst.d);
  const int slots = blockDim.x / j.threads;
  if (((long long)blockIdx.x * slots << P.dst.block_shift) >= n) return;
  const int blk = blockIdx.x * slots + j.slot;
  const long long row0 = (long long)blk << P.dst.block_shift;
  const int32_t* idx = idx_out + unit * P.budget;
  const uint8_t *ks = P.src.k + P.src.base(unit), *vs = P.src.v + P.src.base(unit);
  const long long eb = (long long)unit * P.src.blocks;
  int at[2];
#pragma unroll
  for (int g = 0; g < 2; ++g) at[g] = row0 + j.row(g) < n ? idx[row0 + j.row(g)] : -1;
  uint4 kx[2], vx[2];
  int ks_e[2], vs_e[2];
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    kx[g] = vx[g] = make_uint4(0, 0, 0, 0);
    ks_e[g] = vs_e[g] = kExpMin;
    if (at[g] >= 0) {
      const long long o = at[g] * P.src.st[2] + j.col(g);
      kx[g] = ld16_stream(ks + o);
      vx[g] = ld16_stream(vs + o);
      ks_e[g] = P.src.k_exp[eb + (at[g] >> P.src.block_shift)];
      vs_e[g] = P.src.v_exp[eb + (at[g] >> P.src.block_shift)];
    }
  }
  float2 top = make_float2(0.f, 0.f);
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const uint32_t km = max_codes<kFormat>(max_codes<kFormat>(max_codes<kFormat>(max_codes<kFormat>(0, kx[g].x), kx[g].y), kx[g].z), kx[g].w);
    const uint32_t vm = max_codes<kFormat>(max_codes<kFormat>(max_codes<kFormat>(max_codes<kFormat>(0, vx[g].x), vx[g].y), vx[g].z), vx[g].w);
    top.x = fmaxf(top.x, max_value<kFormat>(km) * pow2_clamped(ks_e[g]));
    top.y = fmaxf(top.y, max_value<kFormat>(vm) * pow2_clamped(vs_e[g]));
  }
  top = job_max(top, j, scratch);
  if (row0 >= n) return;
  const int ke = exponent_of<kFormat>(top.x), ve = exponent_of<kFormat>(top.y);
  uint8_t *ko = P.dst.k + P.dst.base(unit), *vo = P.dst.v + P.dst.base(unit);
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    if (at[g] < 0) continue;
    const long long o = (row0 + j.row(g)) * P.dst.st[2] + j.col(g);
    *reinterpret_cast<uint4*>(ko + o) = ks_e[g] == ke ? kx[g] : recode<kFormat>(kx[g], pow2_clamped(ks_e[g] - ke));
    *reinterpret_cast<uint4*>(vo + o) = vs_e[g] == ve ? vx[g] : recode<kFormat>(vx[g], pow2_clamped(vs_e[g] - ve));
  }
  if (j.t == 0) {
    P.dst.k_exp[(long long)unit * P.dst.blocks + blk] = (int8_t)ke;
    P.dst.v_exp[(long long)unit * P.dst.blocks + blk] = (int8_t)ve;
  }
}

bool overlap(const void* a, long long na, const void* b, long long nb) {
  const char *x = (const char*)a, *y = (const char*)b;
  return x < y + nb && y < x + na;
}

long long span(const Cache& c) { return (c.Bt - 1) * c.st[0] + (c.Hkv - 1) * c.st[1] + (c.cap - 1) * c.st[2] + c.d; }

}  // namespace
}  // namespace kvc

using namespace kvc;

extern "C" kvc_status kvc_evict(const kvc_cache* src, const kvc_cache* dst, const float* weight, int64_t budget, int64_t recent,
                                int32_t* idx_out, float* weight_out, void* stream) {
  EvictParams P;
  kvc_status s;
  if ((s = resolve_cache(src, "src", &P.src)) != KVC_OK) return s;
  if ((s = resolve_cache(dst, "dst", &P.dst)) != KVC_OK) return s;
  const Cache &a = P.src, &b = P.dst;
  KVC_REQUIRE8(a.Bt == b.Bt && a.Hkv == b.Hkv && a.d == b.d && a.format == b.format, KVC_ERR_INVALID_ARG,
               "src and dst differ in batch, head count, head_dim or format");
  KVC_REQUIRE8(budget >= 1 && budget <= b.cap, KVC_ERR_INVALID_ARG, "budget must lie in [1, dst->capacity]");
  KVC_REQUIRE8(recent >= 0 && recent <= budget, KVC_ERR_INVALID_ARG, "recent must lie in [0, budget]");
  KVC_REQUIRE8(weight != nullptr && idx_out != nullptr, KVC_ERR_INVALID_ARG, "weight or idx_out is NULL");
  const long long sa = span(a), sb = span(b), U = a.units();
  KVC_REQUIRE8(!overlap(a.k, sa, b.k, sb) && !overlap(a.k, sa, b.v, sb) && !overlap(a.v, sa, b.k, sb) && !overlap(a.v, sa, b.v, sb) &&
                   !overlap(a.k_exp, U * a.blocks, b.k_exp, U * b.blocks) && !overlap(a.v_exp, U * a.blocks, b.v_exp, U * b.blocks) &&
                   !overlap(a.lengths, 4 * U, b.lengths, 4 * U),
               KVC_ERR_INVALID_ARG, "src and dst share memory");
  KVC_REQUIRE8(weight_out == nullptr || !overlap(weight, 4 * U * a.cap, weight_out, 4 * U * b.cap), KVC_ERR_INVALID_ARG,
               "weight and weight_out share memory");
  if ((s = require_device()) != KVC_OK) return s;
  P.budget = budget; P.recent = recent;
  cudaStream_t st = (cudaStream_t)stream;
  KVC_CUDA(launch_dependent(evict_select_kernel, dim3((unsigned)U), dim3(kSelThreads), 0, st, P, weight, idx_out, weight_out));
  KVC_LAUNCH_CHECK("evict_select_kernel");
  const int threads = job_cta_threads(b);
  const long long per_cta = (long long)(threads / (b.block * b.d / 32)) * b.block;
  KVC_CUDA(launch_dependent(b.format == KVC_E4M3 ? evict_move_kernel<KVC_E4M3> : evict_move_kernel<KVC_INT8>,
                            dim3((unsigned)((budget + per_cta - 1) / per_cta), (unsigned)U), dim3(threads), 0, st, P, idx_out));
  KVC_LAUNCH_CHECK("evict_move_kernel");
  return KVC_OK;
}
