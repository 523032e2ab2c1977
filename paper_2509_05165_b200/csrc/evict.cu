// Eviction from an 8-bit cache by accumulated attention weight (kvc_evict).
//
// Two kernels.  evict_select_kernel, a cluster of up to eight CTAs per head: the weights before the protected rows are read
// once into shared memory, as order-preserving keys, a share per CTA; the key of the last one to keep is found by counting how
// many lie below seven places of the range that it is in (eleven steps at most; a histogram of digits takes three, but its
// atomics crowd into a few bins: 34 us for 64 heads of 32768 rows; it is taken for short ones); the kept positions are written in
// order.  evict_move_kernel, a job per block of the new cache (see cache8.cuh): kept rows are
// read once, take the exponent of their new block and are written once.
// B200: 256 heads from 2112 rows to 2048 selection 12 us, moving 48 us (268 MB, 5.6 TB/s); 64 heads of up to 32768 rows to 8192
// selection 25 us, moving 18 us.
#include "cache8.cuh"

namespace kvc {
namespace {

constexpr int kSelThreads = 256;        // (1024: a step's barriers wait for 32 warps; 256 heads of 2112 rows 20 -> 53 us with one pivot)
constexpr int kSelWarps = kSelThreads / 32;
constexpr int kPivots = 7;
constexpr int kBins = 8 * kSelThreads;
constexpr int kSelHistogram = 8192;     // rows of one CTA up to which a histogram of digits is taken (256 heads of 2112 rows 20 -> 12 us)
constexpr int kSelKeep = 40960;         // keys that a CTA keeps in shared memory (160 KB); what is behind them is read again
constexpr int kSelCluster = 8;

struct EvictParams {
  Cache src, dst;
  long long budget, recent;
};

// What the CTAs of a cluster tell one another, by turns in two places.
struct Exchange {
  uint32_t warp[2][kSelWarps][8];
  uint32_t cta[2][kSelCluster][8];
};

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}

// Sums of each of v's kN numbers over the CTA, left in x.cta[turn][rank] of every CTA of the cluster.
template <int kN>
__device__ __forceinline__ void tell(Exchange& x, int turn, uint32_t rank, int ctas, const uint32_t (&v)[kN]) {
  const int tid = threadIdx.x;
#pragma unroll
  for (int j = 0; j < kN; ++j) {
    const uint32_t sum = __reduce_add_sync(0xffffffffu, v[j]);
    if ((tid & 31) == j) x.warp[turn][tid >> 5][j] = sum;
  }
  __syncthreads();
  if (tid < 8 * ctas && (tid & 7) < kN) {
    const int j = tid & 7;
    uint32_t sum = 0;
#pragma unroll
    for (int w = 0; w < kSelWarps; ++w) sum += x.warp[turn][w][j];
    const uint32_t mine = (uint32_t)__cvta_generic_to_shared(&x.cta[turn][rank][j]);
    uint32_t theirs;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(theirs) : "r"(mine), "r"(tid >> 3));
    asm volatile("st.shared::cluster.u32 [%0], %1;" :: "r"(theirs), "r"(sum) : "memory");
  }
  if (ctas == 1) {
    __syncthreads();
  } else {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
}

__global__ void __launch_bounds__(kSelThreads)
evict_select_kernel(const __grid_constant__ EvictParams P, int ctas, const float* __restrict__ weight, int32_t* __restrict__ idx_out,
                    float* __restrict__ weight_out) {
  extern __shared__ __align__(16) uint32_t s_key[];
  __shared__ Exchange x;
  __shared__ __align__(16) uint32_t hist[kBins];
  __shared__ int s_bin, s_before;
  grid_dependency_wait();
  const uint32_t rank = ctas == 1 ? 0 : cluster_rank();
  const int unit = blockIdx.x / ctas, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int n = (int)P.src.length(unit), budget = (int)P.budget, recent = (int)P.recent;
  const float* w = weight + unit * P.src.cap;
  int32_t* idx = idx_out + unit * P.budget;
  float* wo = weight_out == nullptr ? nullptr : weight_out + unit * P.dst.cap;
  const int kept = min(n, budget), first = rank * kSelThreads + tid, step = ctas * kSelThreads;
  if (first == 0) P.dst.lengths[unit] = kept;
  for (long long i = kept + first; i < budget; i += step) idx[i] = -1;
  if (n <= budget) {
    for (long long i = first; i < n; i += step) {
      idx[i] = (int32_t)i;
      if (wo != nullptr) wo[i] = w[i];
    }
    return;
  }
  // behind the others: the protected rows
  const int m = n - recent, want = budget - recent;
  for (long long i = first; i < recent; i += step) {
    idx[want + i] = (int32_t)(m + i);
    if (wo != nullptr) wo[want + i] = w[m + i];
  }
  if (want == 0) return;

  // this CTA's rows, in fours: row0 .. row0 + mine - 1, as keys that ascend as weights descend; padded with the largest key
  const int each = (int)(((long long)m + 4 * ctas - 1) / (4 * ctas)) * 4;
  const long long row0 = (long long)rank * each;
  const int mine = (int)max(min((long long)each, m - row0), 0LL), held = min(mine, kSelKeep), fours = (held + 3) / 4;
  w += row0;
  for (int i0 = tid; i0 < 4 * fours; i0 += 8 * kSelThreads) {
    float y[8];                                      // (eight loads in flight)
#pragma unroll
    for (int u = 0; u < 8; ++u) y[u] = i0 + u * kSelThreads < held ? __ldg(w + i0 + u * kSelThreads) : 0.f;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int i = i0 + u * kSelThreads;
      if (i < 4 * fours) s_key[i] = i < held ? score_to_key(y[u]) : 0xffffffffu;
    }
  }
  __syncthreads();

  // The smallest key that at least `want` rows do not exceed lies in [low, hi].
  const uint4* fours_of = reinterpret_cast<const uint4*>(s_key);
  uint32_t low = 0, hi = 0xffffffffu;
  int low_count = 0, ties = -1, turn = 0;            // rows below `low`; of the rows with the last key, the first `ties` are kept
  if (ctas > 1)                                      // (a CTA's shared memory is written to by the others once all of them run)
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (ctas == 1 && mine <= kSelHistogram) {
    // digit by digit (11, 11 and 10 bits): the digit that the want-th row has, among the rows with the digits found so far
    int want_left = want, shift = 32;
    hi = 0;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int bits = pass == 2 ? 10 : 11;
      const uint32_t fixed = pass == 0 ? 0u : ~0u << shift;
      shift -= bits;
      for (int i = tid; i < kBins / 4; i += kSelThreads) reinterpret_cast<uint4*>(hist)[i] = make_uint4(0, 0, 0, 0);
      __syncthreads();
      for (int i = tid; i < mine; i += kSelThreads) {
        const uint32_t key = s_key[i];
        if (((key ^ hi) & fixed) == 0) atomicAdd(&hist[(key >> shift) & ((1u << bits) - 1)], 1u);
      }
      __syncthreads();
      const uint4 a = reinterpret_cast<const uint4*>(hist)[2 * tid], b = reinterpret_cast<const uint4*>(hist)[2 * tid + 1];
      const uint32_t bin[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
      uint32_t sum = 0;
#pragma unroll
      for (int u = 0; u < 8; ++u) sum += bin[u];
      uint32_t incl = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
      }
      if (lane == 31) x.warp[0][warp][0] = incl;
      __syncthreads();
      uint32_t before = incl - sum;
      for (int w = 0; w < warp; ++w) before += x.warp[0][w][0];
      if ((int)before < want_left && want_left <= (int)(before + sum)) {
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          if ((int)before < want_left && want_left <= (int)(before + bin[u])) {
            s_bin = 8 * tid + u;
            s_before = before;
          }
          before += bin[u];
        }
      }
      __syncthreads();
      hi |= (uint32_t)s_bin << shift;
      want_left -= s_before;                         // (both written again behind the next barriers)
    }
    low = hi;
    ties = want_left;
  }
  while (low < hi) {
    const uint32_t range = hi - low, stride = (range >> 3) + 1;
    uint32_t pivot[kPivots], count[kPivots];         // places in (low, hi], keys below them
#pragma unroll
    for (int j = 0; j < kPivots; ++j) {
      pivot[j] = low + min(stride * (j + 1), range);
      count[j] = 0;
    }
    for (int i = tid; i < fours; i += kSelThreads) {
      const uint4 k = fours_of[i];
#pragma unroll
      for (int j = 0; j < kPivots; ++j) count[j] += (k.x < pivot[j]) + (k.y < pivot[j]) + (k.z < pivot[j]) + (k.w < pivot[j]);
    }
    for (long long i = held + tid; i < mine; i += kSelThreads) {
      const uint32_t key = score_to_key(w[i]);
#pragma unroll
      for (int j = 0; j < kPivots; ++j) count[j] += key < pivot[j];
    }
    tell(x, turn, rank, ctas, count);
    uint32_t total = 0;                              // lane j: of pivot j
    if (lane < kPivots)
      for (int c = 0; c < ctas; ++c) total += x.cta[turn][c][lane];
    turn ^= 1;
    const uint32_t exact = __ballot_sync(0xffffffffu, lane < kPivots && (int)total == want);
    const int below = __popc(__ballot_sync(0xffffffffu, lane < kPivots && (int)total < want));      // (counts do not fall with the pivots)
    const uint32_t from = low;
    if (exact != 0) {                                // all keys below that pivot are kept
      hi = from + min(stride * __ffs(exact), range) - 1;
      ties = 0x7fffffff;
      break;
    }
    if (below < kPivots) hi = from + min(stride * (below + 1), range) - 1;
    if (below > 0) {
      low = from + min(stride * below, range);
      low_count = (int)__shfl_sync(0xffffffffu, total, below - 1);
    }
  }
  if (ties < 0) ties = want - low_count;

  // Positions in order.  A row in front of which lie l rows with smaller keys and q with the last key goes to place
  // l + min(q, ties).
  uint32_t both[2] = {0, 0};
  for (int i = tid; i < fours; i += kSelThreads) {
    const uint4 k = fours_of[i];
    both[0] += (k.x < hi) + (k.y < hi) + (k.z < hi) + (k.w < hi);
    const int at = 4 * i;
    both[1] += (k.x == hi && at < held) + (k.y == hi && at + 1 < held) + (k.z == hi && at + 2 < held) + (k.w == hi && at + 3 < held);
  }
  for (long long i = held + tid; i < mine; i += kSelThreads) {
    const uint32_t key = score_to_key(w[i]);
    both[0] += key < hi;
    both[1] += key == hi;
  }
  tell(x, turn, rank, ctas, both);
  int less = 0, equal = 0;
  for (uint32_t c = 0; c < rank; ++c) {
    less += x.cta[turn][c][0];
    equal += x.cta[turn][c][1];
  }
  for (long long i0 = 0; i0 < mine; i0 += 4 * kSelThreads) {     // four rows in a row per thread
    const long long at = i0 + 4 * tid;
    uint32_t key[4];
    int flags = 0;                                   // smaller keys; equal ones, 2^16 times
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      key[u] = 0xffffffffu;
      if (at + u >= mine) continue;
      key[u] = at + u < held ? s_key[at + u] : score_to_key(w[at + u]);
      flags += (key[u] < hi ? 1 : 0) + (key[u] == hi ? 1 << 16 : 0);
    }
    int incl = flags;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    turn ^= 1;                                       // (one barrier per step: the sums of the step before are in the other place)
    if (lane == 31) x.warp[turn][warp][0] = incl;
    __syncthreads();
    const int other = lane < kSelWarps ? x.warp[turn][lane][0] : 0;
    const int before = __reduce_add_sync(0xffffffffu, lane < warp ? other : 0) + incl - flags;
    const int all = __reduce_add_sync(0xffffffffu, other);
    int l = less + (before & 0xffff), q = equal + (before >> 16);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (at + u >= mine) continue;
      if (key[u] < hi || (key[u] == hi && q < ties)) {
        const int place = l + min(q, ties);
        idx[place] = (int32_t)(row0 + at + u);
        if (wo != nullptr) wo[place] = w[at + u];
      }
      l += key[u] < hi;
      q += key[u] == hi;
    }
    less += all & 0xffff;
    equal += all >> 16;
  }
}

// CTAs per head: as many as keep the keys in shared memory, and as fit the GPU at once (four per SM) if they have 4096 keys each.
int select_ctas(long long cap, long long units, int sms) {
  int c = 1;
  while (c < kSelCluster && (cap > (long long)c * kSelKeep || (units * c * 2 <= 4 * sms && cap > (long long)c * 4096))) c *= 2;
  return c;
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
      const long long o = at[g] * P.src.st[2] + j.col;
      kx[g] = ld16_stream(ks + o);
      vx[g] = ld16_stream(vs + o);
      ks_e[g] = P.src.k_exp[eb + (at[g] >> P.src.block_shift)];
      vs_e[g] = P.src.v_exp[eb + (at[g] >> P.src.block_shift)];
    }
  }
  constexpr int kDown = 8;                             // (448 * 2^121 and 2^-9 * 2^-100, both 2^-8 times, are normal fp32 numbers)
  float2 top = make_float2(0.f, 0.f);
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const uint32_t km = max_codes<kFormat>(max_codes<kFormat>(max_codes<kFormat>(max_codes<kFormat>(0, kx[g].x), kx[g].y), kx[g].z), kx[g].w);
    const uint32_t vm = max_codes<kFormat>(max_codes<kFormat>(max_codes<kFormat>(max_codes<kFormat>(0, vx[g].x), vx[g].y), vx[g].z), vx[g].w);
    top.x = fmaxf(top.x, max_value<kFormat>(km) * pow2_clamped(ks_e[g] - kDown));
    top.y = fmaxf(top.y, max_value<kFormat>(vm) * pow2_clamped(vs_e[g] - kDown));
  }
  top = job_max(top, j, scratch);
  if (row0 >= n) return;
  const int ke = exponent_of<kFormat>(top.x, kDown), ve = exponent_of<kFormat>(top.y, kDown);
  uint8_t *ko = P.dst.k + P.dst.base(unit), *vo = P.dst.v + P.dst.base(unit);
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    if (at[g] < 0) continue;
    const long long o = (row0 + j.row(g)) * P.dst.st[2] + j.col;
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
                   !overlap(a.k_exp, U * a.blocks, b.v_exp, U * b.blocks) && !overlap(a.v_exp, U * a.blocks, b.k_exp, U * b.blocks) &&
                   !overlap(a.lengths, 4 * U, b.lengths, 4 * U),
               KVC_ERR_INVALID_ARG, "src and dst share memory");
  KVC_REQUIRE8(weight_out == nullptr || !overlap(weight, 4 * U * a.cap, weight_out, 4 * U * b.cap), KVC_ERR_INVALID_ARG,
               "weight and weight_out share memory");
  if ((s = require_device()) != KVC_OK) return s;
  P.budget = budget; P.recent = recent;
  cudaStream_t st = (cudaStream_t)stream;
  int dev = 0, sms = 0;
  KVC_CUDA(cudaGetDevice(&dev));
  KVC_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  const int ctas = select_ctas(a.cap, U, sms);
  const long long each = ((a.cap + 4 * ctas - 1) / (4 * ctas)) * 4;
  static std::atomic<uint64_t> done{0};
  KVC_CUDA(allow_smem(evict_select_kernel, kSelKeep * 4, done, dev));
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ctas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(U * ctas));
  cfg.blockDim = dim3(kSelThreads);
  cfg.dynamicSmemBytes = (size_t)(each < kSelKeep ? each : kSelKeep) * 4;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  KVC_CUDA(cudaLaunchKernelEx(&cfg, evict_select_kernel, P, ctas, weight, idx_out, weight_out));
  KVC_LAUNCH_CHECK("evict_select_kernel");
  const int threads = job_cta_threads(b);
  const long long per_cta = (long long)(threads / (b.block * b.d / 32)) * b.block;
  KVC_CUDA(launch_dependent(b.format == KVC_E4M3 ? evict_move_kernel<KVC_E4M3> : evict_move_kernel<KVC_INT8>,
                            dim3((unsigned)((budget + per_cta - 1) / per_cta), (unsigned)U), dim3(threads), 0, st, P, idx_out));
  KVC_LAUNCH_CHECK("evict_move_kernel");
  return KVC_OK;
}
