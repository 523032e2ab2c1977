// The 8-bit cache (kvc.h): taking kept rows in (kvc_cache_gather), new tokens (kvc_cache_append), values back
// (kvc_cache_read).
//
// The unit of work is a block of tokens of one head, K or V: its exponent needs the largest of its block * d values before
// the first code can be rounded, so a job of block * d / 32 threads holds a block of K and the one of V beside it in registers,
// 32 values of each per thread (as loaded: maxima are taken over the bits), reduces both maxima at once and writes codes.
// Every source row is read once and every code written once; HBM is the bound.
// B200: gathering 32 layers of 8 heads, about 1024 of 8192 rows of 128 each, into e4m3 39 us (202 MB, 5.2 TB/s; warps
// issue in 56 % of the cycles); reading 2048 places of them back as bf16 52 us (336 MB, 6.4 TB/s).
#include "cache8.cuh"

namespace kvc {
namespace {

// ---- kept rows of a prefilled cache -----------------------------------------------------------------------------------

struct GatherLayer {
  const void *k, *v;
  uint8_t *ko, *vo;
  int8_t *ke, *ve;
  int32_t* lengths;
  long long cap, blocks, st[3];
};

struct CacheGatherParams {
  int L, Bt, Hkv, d, block_shift, per_head;
  long long N, kvs[3];
  GatherLayer layer[KVC_MAX_LAYERS];
};

template <typename T, int kFormat>
__global__ void __launch_bounds__(512)
cache_gather_kernel(const __grid_constant__ CacheGatherParams P, const int32_t* __restrict__ idx,
                    const int32_t* __restrict__ n_keep, int32_t* device_status) {
  __shared__ float2 scratch[16];
  grid_dependency_wait();
  const int l = blockIdx.z, unit = blockIdx.y, b = unit / P.Hkv, h = unit - b * P.Hkv;
  const GatherLayer& y = P.layer[l];
  long long kept = P.N;
  if (n_keep != nullptr) {
    kept = P.per_head ? n_keep[((long long)b * P.L + l) * P.Hkv + h] : n_keep[(long long)b * P.L + l];
    kept = kept < 0 ? 0 : (kept > P.N ? P.N : kept);
  }
  const int n = (int)min(kept, y.cap);                 // (capacities are below 2^31 - 1024)
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    y.lengths[unit] = n;
    if (kept > n && device_status != nullptr) atomicExch(device_status, KVC_ERR_CAPACITY);
  }

  const JobLane<8> j(P.block_shift, P.d);
  const int slots = blockDim.x / j.threads;
  if (((long long)blockIdx.x * slots << P.block_shift) >= n) return;    // (the whole CTA)
  const int blk = blockIdx.x * slots + j.slot, row0 = blk << P.block_shift;
  const int left = n - row0 - j.row0;                  // of the thread's rows, those with g * row_step < left are there
  const long long from = b * P.kvs[0] + h * P.kvs[1] + j.col;
  const T *ks = reinterpret_cast<const T*>(y.k) + from, *vs = reinterpret_cast<const T*>(y.v) + from;
  const int32_t* map = idx == nullptr ? nullptr : idx + (((long long)l * P.Bt + b) * P.Hkv + h) * P.N + row0 + j.row0;
  int at[4];
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    at[g] = -1;
    if (g * j.row_step < left) {
      at[g] = map == nullptr ? row0 + j.row(g) : map[g * j.row_step];
      if (at[g] >= P.N) at[g] = -1;
    }
  }
  Raw8<T> kx[4], vx[4];
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    if (at[g] >= 0) {
      const long long o = at[g] * P.kvs[2];
      kx[g].load(ks + o);
      vx[g].load(vs + o);
    } else {
      kx[g].zero();
      vx[g].zero();
    }
  }
  uint32_t km = 0, vm = 0;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    km = kx[g].max_bits(km);
    vm = vx[g].max_bits(vm);
  }
  float2 top = job_max(make_float2(Raw8<T>::top(km), Raw8<T>::top(vm)), j, scratch);
  if (row0 >= n) return;
  // the thread's row g: its token's place among the values (as above), -1 if there is none
  const auto row = [&](int g) -> long long {
    if (g * j.row_step >= left) return -1;
    const int t = map == nullptr ? row0 + j.row(g) : map[g * j.row_step];
    return t < 0 || t >= P.N ? -1 : t * P.kvs[2];
  };
  const bool finite = all_finite(top);
  if (!finite) top = finite_max(ks, vs, row, j, scratch, device_status);
  const int ke = exponent_of<kFormat>(top.x), ve = exponent_of<kFormat>(top.y);
  const float kf = pow2(-ke), vf = pow2(-ve);
  long long to = b * y.st[0] + h * y.st[1] + (row0 + j.row0) * y.st[2] + j.col;
  const long long step = j.row_step * y.st[2];
  if (finite) {
#pragma unroll
    for (int g = 0; g < 4; ++g, to += step) {
      if (g * j.row_step < left) {
        *reinterpret_cast<uint2*>(y.ko + to) = kx[g].template encode<kFormat>(kf);
        *reinterpret_cast<uint2*>(y.vo + to) = vx[g].template encode<kFormat>(vf);
      }
    }
  } else {
#pragma unroll 1
    for (int g = 0; g * j.row_step < left && g < 4; ++g, to += step) {
      const long long o = row(g);
      *reinterpret_cast<uint2*>(y.ko + to) = o < 0 ? make_uint2(0, 0) : encode_any<kFormat>(ks + o, kf);
      *reinterpret_cast<uint2*>(y.vo + to) = o < 0 ? make_uint2(0, 0) : encode_any<kFormat>(vs + o, vf);
    }
  }
  if (j.t == 0) {
    y.ke[(long long)unit * y.blocks + blk] = (int8_t)ke;
    y.ve[(long long)unit * y.blocks + blk] = (int8_t)ve;
  }
}

// ---- new tokens -------------------------------------------------------------------------------------------------------

struct AppendParams {
  Cache c;
  int rows, jobs_per_cta;                // jobs_per_cta: blocks (of K and V) that a CTA takes
  long long ns[3];
  bool write_lengths;                    // the lengths are written here (else by append_lengths_kernel)
};

__device__ __forceinline__ int rows_of(const AppendParams& P, const int32_t* n_new, int b) {
  const int n = n_new == nullptr ? P.rows : n_new[b];
  return n < 0 ? 0 : (n > P.rows ? P.rows : n);
}

// Eight codes in place, rounded again for an exponent larger by -down.
template <int kFormat>
__device__ __forceinline__ void regrow(uint8_t* p, int down) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  const float f = pow2_clamped(down);
  float y[8];
  decode4<kFormat>(w.x, y);
  decode4<kFormat>(w.y, y + 4);
  *reinterpret_cast<uint2*>(p) = make_uint2(encode4<kFormat>(y[0], y[1], y[2], y[3], f), encode4<kFormat>(y[4], y[5], y[6], y[7], f));
}

// A CTA takes blocks blockIdx.x * jobs_per_cta .. of the ones that a head's new rows touch, counted from its open block.
template <typename T, int kFormat>
__global__ void __launch_bounds__(512)
cache_append_kernel(const __grid_constant__ AppendParams P, const T* __restrict__ k_new, const T* __restrict__ v_new,
                    const int32_t* __restrict__ n_new, int32_t* lengths_out, float* __restrict__ weight, int32_t* device_status) {
  __shared__ float2 scratch[16];
  grid_dependency_wait();
  const Cache& c = P.c;
  const int unit = blockIdx.y, b = unit / c.Hkv, h = unit - b * c.Hkv;
  const int len = (int)c.length(unit);
  const int want = rows_of(P, n_new, b);
  const int n = (int)min((long long)want, c.cap - len);
  __syncthreads();                       // every thread has the length before it may change
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    if (P.write_lengths) lengths_out[unit] = len + n;
    if (n < want && device_status != nullptr) atomicExch(device_status, KVC_ERR_CAPACITY);
  }
  if (n == 0) return;
  const JobLane<8> j(c.block_shift, c.d);
  const int slots = blockDim.x / j.threads;
  const int blk0 = len >> c.block_shift, touched = ((len + n - 1) >> c.block_shift) - blk0 + 1;
  const int last = min((int)(blockIdx.x + 1) * P.jobs_per_cta, touched);
  const long long from = b * P.ns[0] + h * P.ns[1];
  for (int jb = blockIdx.x * P.jobs_per_cta; jb < last; jb += slots) {
    const bool live = jb + j.slot < last;
    const int blk = blk0 + jb + j.slot, row0 = blk << c.block_shift;
    Raw8<T> kx[4], vx[4];
    uint32_t km = 0, vm = 0;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int r = row0 + j.row(g) - len;                // the row's number among the new ones
      if (live && r >= 0 && r < n) {
        const long long at = from + r * P.ns[2] + j.col;
        kx[g].load(k_new + at);
        vx[g].load(v_new + at);
        if (weight != nullptr && j.col == 0) weight[unit * c.cap + len + r] = 0.f;
      } else {
        kx[g].zero();
        vx[g].zero();
      }
    }
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      km = kx[g].max_bits(km);
      vm = vx[g].max_bits(vm);
    }
    float2 top = job_max(make_float2(Raw8<T>::top(km), Raw8<T>::top(vm)), j, scratch);
    if (!live) continue;
    const bool finite = all_finite(top);
    if (!finite) {
      const auto row = [&](int g) -> long long {
        const int r = row0 + j.row(g) - len;
        return r >= 0 && r < n ? from + r * P.ns[2] + j.col : -1;
      };
      top = finite_max(k_new, v_new, row, j, scratch, device_status);
    }
    const long long eat = (long long)unit * c.blocks + blk;
    int ke = exponent_of<kFormat>(top.x), ve = exponent_of<kFormat>(top.y);
    const bool open = row0 < len;                         // the block has rows already
    int kwas = kExpMin, vwas = kExpMin;
    if (open) {
      kwas = c.k_exp[eat];
      vwas = c.v_exp[eat];
      ke = max(ke, kwas);
      ve = max(ve, vwas);
    }
    const long long to = c.base(unit);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int r = row0 + j.row(g);
      const long long o = to + r * c.st[2] + j.col;
      if (r >= len && r < len + n) {
        if (!finite) {                                      // (some of the job's values: read again)
          const long long at = from + (r - len) * P.ns[2] + j.col;
          *reinterpret_cast<uint2*>(c.k + o) = encode_any<kFormat>(k_new + at, pow2(-ke));
          *reinterpret_cast<uint2*>(c.v + o) = encode_any<kFormat>(v_new + at, pow2(-ve));
          continue;
        }
        *reinterpret_cast<uint2*>(c.k + o) = kx[g].template encode<kFormat>(pow2(-ke));
        *reinterpret_cast<uint2*>(c.v + o) = vx[g].template encode<kFormat>(pow2(-ve));
      } else if (open && r < len && (ke > kwas || ve > vwas)) {      // a code under a larger exponent: rounded again
        if (ke > kwas) regrow<kFormat>(c.k + o, kwas - ke);
        if (ve > vwas) regrow<kFormat>(c.v + o, vwas - ve);
      }
    }
    // every thread of the job has read the old exponents before they change
    job_barrier(j);
    if (j.t == 0) {
      c.k_exp[eat] = (int8_t)ke;
      c.v_exp[eat] = (int8_t)ve;
    }
  }
}

__global__ void append_lengths_kernel(const __grid_constant__ AppendParams P, const int32_t* __restrict__ n_new, int32_t* lengths_out) {
  grid_dependency_wait();
  const int unit = blockIdx.x * blockDim.x + threadIdx.x;
  if (unit >= P.c.units()) return;
  const long long len = P.c.length(unit), want = rows_of(P, n_new, unit / P.c.Hkv);
  lengths_out[unit] = (int32_t)(len + (want < P.c.cap - len ? want : P.c.cap - len));
}

// ---- values back ------------------------------------------------------------------------------------------------------

// 32 bytes, a whole sector, at once (its address is a multiple of 16 at least).
__device__ __forceinline__ void st32(void* p, const uint32_t* u) {
  if ((reinterpret_cast<uintptr_t>(p) & 31u) == 0) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 :: "l"(p), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]) : "memory");
  } else {
    reinterpret_cast<uint4*>(p)[0] = make_uint4(u[0], u[1], u[2], u[3]);
    reinterpret_cast<uint4*>(p)[1] = make_uint4(u[4], u[5], u[6], u[7]);
  }
}

struct ReadParams {
  Cache c;
  long long rows;
};

constexpr int kReadEach = 4;             // pieces of 16 codes per thread, asked for together

template <typename T, int kFormat>
__global__ void __launch_bounds__(256)
cache_read_kernel(const __grid_constant__ ReadParams P, const int32_t* __restrict__ first, T* __restrict__ k_out, T* __restrict__ v_out) {
  grid_dependency_wait();
  const Cache& c = P.c;
  const int unit = blockIdx.y;
  const bool is_v = k_out == nullptr || blockIdx.z == 1;
  const int shift = c.d == 128 ? 3 : 2;                   // log2(d / 16)
  const long long len = c.length(unit), row_first = first == nullptr ? 0 : first[unit];
  const uint8_t* codes = (is_v ? c.v : c.k) + c.base(unit);
  const int8_t* exps = (is_v ? c.v_exp : c.k_exp) + (long long)unit * c.blocks;
  T* out = (is_v ? v_out : k_out) + unit * P.rows * c.d;
  const long long total = P.rows << shift;
  for (long long i0 = (long long)blockIdx.x * (256 * kReadEach) + threadIdx.x; i0 < total; i0 += (long long)gridDim.x * (256 * kReadEach)) {
    uint4 w[kReadEach];
    float f[kReadEach];
#pragma unroll
    for (int u = 0; u < kReadEach; ++u) {
      const long long i = i0 + 256 * u, r = row_first + (i >> shift);
      w[u] = make_uint4(0, 0, 0, 0);
      f[u] = 0.f;
      if (i < total && r >= 0 && r < len) {
        w[u] = ld16_stream(codes + r * c.st[2] + (int)(i & ((1 << shift) - 1)) * 16);
        f[u] = pow2_clamped(exps[r >> c.block_shift]);
      }
    }
#pragma unroll
    for (int u = 0; u < kReadEach; ++u) {
      const long long i = i0 + 256 * u;
      if (i >= total) break;
      T* o = out + (i << 4);
      const uint32_t v[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
#pragma unroll
      for (int h = 0; h < (int)sizeof(T) / 2; ++h) {        // 32 bytes of output at a time
        constexpr int kWords = 8 / (int)sizeof(T);          // of codes
        uint32_t y[8];
#pragma unroll
        for (int q = 0; q < kWords; ++q) {
          float x[4];
          decode4<kFormat>(v[kWords * h + q], x);
          if (sizeof(T) == 2) {
            const __nv_bfloat162 s = __floats2bfloat162_rn(x[0] * f[u], x[1] * f[u]), t = __floats2bfloat162_rn(x[2] * f[u], x[3] * f[u]);
            y[2 * q] = *reinterpret_cast<const uint32_t*>(&s);
            y[2 * q + 1] = *reinterpret_cast<const uint32_t*>(&t);
          } else {
#pragma unroll
            for (int z = 0; z < 4; ++z) y[(4 * q + z) & 7] = __float_as_uint(x[z] * f[u]);
          }
        }
        st32(reinterpret_cast<char*>(o) + 32 * h, y);
      }
    }
  }
}

template <typename T>
kvc_status run_gather(const CacheGatherParams& P, int format, int block, long long most_cap, const int32_t* idx, const int32_t* n_keep,
                      int32_t* status, cudaStream_t st) {
  const int job = block * P.d / 32, threads = job > 256 ? job : 256;
  const long long rows = most_cap < P.N ? most_cap : P.N, per_cta = (long long)(threads / job) * block;
  const dim3 grid((unsigned)((rows + per_cta - 1) / per_cta), P.Bt * P.Hkv, P.L);
  auto kernel = format == KVC_E4M3 ? cache_gather_kernel<T, KVC_E4M3> : cache_gather_kernel<T, KVC_INT8>;
  KVC_CUDA(launch_dependent(kernel, grid, dim3(threads), 0, st, P, idx, n_keep, status));
  KVC_LAUNCH_CHECK("cache_gather_kernel");
  return KVC_OK;
}

}  // namespace

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

kvc_status check_dtype(int32_t dtype) {
  KVC_REQUIRE8(dtype == KVC_F32 || dtype == KVC_BF16, KVC_ERR_INVALID_ARG, "unknown dtype");
  return KVC_OK;
}

kvc_status resolve_strides(const int64_t* given, int batch, int heads, long long rows, int d, int elem_bytes, bool written,
                           const char* name, long long* out) {
  if (given == nullptr || given[0] == 0) {
    out[2] = d; out[1] = rows * d; out[0] = out[1] * heads;
    return KVC_OK;
  }
  for (int i = 0; i < 3; ++i) {
    KVC_REQUIRE8(given[i] >= (i == 2 ? d : 0) && given[i] % (16 / elem_bytes) == 0, KVC_ERR_INVALID_ARG,
                 "%s[%d] must be a non-negative multiple of 16 bytes (rows >= head_dim apart)", name, i);
    out[i] = given[i];
  }
  if (!written) return KVC_OK;
  // dimensions from the narrowest on: each must step over all that the narrower ones span
  const long long size[3] = {batch, heads, rows};
  int order[3] = {0, 1, 2};
  for (int i = 0; i < 2; ++i)
    for (int k = i + 1; k < 3; ++k)
      if (out[order[k]] < out[order[i]]) { const int t = order[i]; order[i] = order[k]; order[k] = t; }
  long long extent = d;
  for (int i : order) {
    if (size[i] <= 1) continue;
    KVC_REQUIRE8(out[i] >= extent, KVC_ERR_INVALID_ARG, "%s: rows of an array that is written to overlap", name);
    extent += out[i] * (size[i] - 1);
  }
  return KVC_OK;
}

kvc_status resolve_cache(const kvc_cache* c, const char* name, Cache* out) {
  KVC_REQUIRE8(c != nullptr, KVC_ERR_INVALID_ARG, "%s is NULL", name);
  KVC_REQUIRE8(c->batch >= 1 && c->n_kv_heads >= 1, KVC_ERR_INVALID_ARG, "%s: batch and n_kv_heads must be >= 1", name);
  KVC_REQUIRE8((long long)c->batch * c->n_kv_heads <= 65535, KVC_ERR_UNSUPPORTED, "%s: batch * n_kv_heads > 65535", name);
  KVC_REQUIRE8(c->head_dim == 64 || c->head_dim == 128, KVC_ERR_UNSUPPORTED, "%s: head_dim must be 64 or 128", name);
  KVC_REQUIRE8(c->block == 16 || c->block == 32 || c->block == 64 || c->block == 128, KVC_ERR_UNSUPPORTED,
               "%s: block must be 16, 32, 64 or 128", name);
  KVC_REQUIRE8(c->format == KVC_INT8 || c->format == KVC_E4M3, KVC_ERR_INVALID_ARG, "%s: unknown format", name);
  KVC_REQUIRE8(c->reserved_ == 0, KVC_ERR_INVALID_ARG, "%s: reserved_ must be 0", name);
  KVC_REQUIRE8(c->capacity >= 1, KVC_ERR_INVALID_ARG, "%s: capacity must be >= 1", name);
  KVC_REQUIRE8(c->capacity < (1LL << 31) - 1024, KVC_ERR_UNSUPPORTED, "%s: capacity must be < 2^31 - 1024", name);
  KVC_REQUIRE8(c->k && c->v && c->k_exp && c->v_exp && c->lengths, KVC_ERR_INVALID_ARG, "%s: k, v, k_exp, v_exp or lengths is NULL", name);
  KVC_REQUIRE8(aligned16(c->k) && aligned16(c->v), KVC_ERR_INVALID_ARG, "%s: k or v is not 16-byte aligned", name);
  KVC_REQUIRE8((reinterpret_cast<uintptr_t>(c->lengths) & 3u) == 0, KVC_ERR_INVALID_ARG, "%s: lengths is not 4-byte aligned", name);
  out->Bt = c->batch; out->Hkv = c->n_kv_heads; out->d = c->head_dim; out->block = c->block; out->format = c->format;
  out->block_shift = c->block == 16 ? 4 : c->block == 32 ? 5 : c->block == 64 ? 6 : 7;
  out->cap = c->capacity;
  out->blocks = (c->capacity + c->block - 1) / c->block;
  out->k = (uint8_t*)c->k; out->v = (uint8_t*)c->v; out->k_exp = c->k_exp; out->v_exp = c->v_exp; out->lengths = c->lengths;
  return resolve_strides(c->stride, c->batch, c->n_kv_heads, c->capacity, c->head_dim, 1, true, name, out->st);
}

}  // namespace kvc

using namespace kvc;

extern "C" {

kvc_status kvc_cache_gather(const kvc_desc* d, const void* const* k, const void* const* v, const int32_t* idx, const int32_t* n_keep,
                            int32_t per_head, const kvc_cache* caches, int32_t* device_status, void* stream) {
  Problem P;
  kvc_status s = resolve_desc(d, &P);
  if (s != KVC_OK) return s;
  KVC_REQUIRE8(k != nullptr && v != nullptr, KVC_ERR_INVALID_ARG, "k or v pointer array is NULL");
  KVC_REQUIRE8(caches != nullptr, KVC_ERR_INVALID_ARG, "caches is NULL");
  KVC_REQUIRE8(per_head == 0 || per_head == 1, KVC_ERR_INVALID_ARG, "per_head must be 0 or 1");
  KVC_REQUIRE8((long long)P.Bt * P.Hkv <= 65535, KVC_ERR_UNSUPPORTED, "batch * n_kv_heads > 65535");
  CacheGatherParams gp;
  gp.L = P.L; gp.Bt = P.Bt; gp.Hkv = P.Hkv; gp.d = P.d; gp.per_head = per_head; gp.N = P.N;
  for (int i = 0; i < 3; ++i) gp.kvs[i] = P.kvs[i];
  long long most = 0;
  for (int l = 0; l < P.L; ++l) {
    Cache c;
    if ((s = resolve_cache(caches + l, "caches", &c)) != KVC_OK) return s;
    KVC_REQUIRE8(c.Bt == P.Bt && c.Hkv == P.Hkv && c.d == P.d, KVC_ERR_INVALID_ARG, "caches[%d] has another batch, head count or head_dim than desc", l);
    KVC_REQUIRE8(c.block == caches[0].block && c.format == caches[0].format, KVC_ERR_INVALID_ARG,
                 "caches[%d] has another block or format than caches[0]", l);
    KVC_REQUIRE8(k[l] && v[l] && aligned16(k[l]) && aligned16(v[l]), KVC_ERR_INVALID_ARG, "k[%d] or v[%d] is NULL or not 16-byte aligned", l, l);
    gp.block_shift = c.block_shift;
    gp.layer[l] = GatherLayer{k[l], v[l], c.k, c.v, c.k_exp, c.v_exp, c.lengths, c.cap, c.blocks, {c.st[0], c.st[1], c.st[2]}};
    if (c.cap > most) most = c.cap;
  }
  if ((s = require_device()) != KVC_OK) return s;
  return P.dtype == KVC_F32
             ? run_gather<float>(gp, caches[0].format, caches[0].block, most, idx, n_keep, device_status, (cudaStream_t)stream)
             : run_gather<__nv_bfloat16>(gp, caches[0].format, caches[0].block, most, idx, n_keep, device_status, (cudaStream_t)stream);
}

kvc_status kvc_cache_append(const kvc_cache* cache, const void* k_new, const void* v_new, int32_t dtype, int32_t rows,
                            const int64_t* stride, const int32_t* n_new, int32_t* lengths_out, float* weight,
                            int32_t* device_status, void* stream) {
  AppendParams P;
  kvc_status s = resolve_cache(cache, "cache", &P.c);
  if (s != KVC_OK) return s;
  if ((s = check_dtype(dtype)) != KVC_OK) return s;
  KVC_REQUIRE8(k_new && v_new && aligned16(k_new) && aligned16(v_new), KVC_ERR_INVALID_ARG, "k_new or v_new is NULL or not 16-byte aligned");
  KVC_REQUIRE8(rows >= 1, KVC_ERR_INVALID_ARG, "rows must be >= 1");
  KVC_REQUIRE8(rows <= (1 << 30), KVC_ERR_UNSUPPORTED, "rows > 2^30");
  if ((s = resolve_strides(stride, P.c.Bt, P.c.Hkv, rows, P.c.d, dtype == KVC_F32 ? 4 : 2, false, "stride", P.ns)) != KVC_OK) return s;
  if ((s = require_device()) != KVC_OK) return s;
  P.rows = rows;
  if (lengths_out == nullptr) lengths_out = P.c.lengths;
  // (a head's new rows touch at most this many blocks, wherever its open block ends)
  const long long touched = ((long long)rows + P.c.block - 2) / P.c.block + 1;
  // up to four blocks: one CTA per head, which can then write the length itself; more: as many blocks as a CTA has jobs
  P.jobs_per_cta = touched <= 4 ? (int)touched : job_cta_threads(P.c) / (P.c.block * P.c.d / 32);
  const long long steps = (touched + P.jobs_per_cta - 1) / P.jobs_per_cta;
  P.write_lengths = steps == 1 || lengths_out != P.c.lengths;
  const dim3 grid((unsigned)steps, P.c.units()), threads(job_cta_threads(P.c));
  const bool e4m3 = P.c.format == KVC_E4M3;
  cudaStream_t st = (cudaStream_t)stream;
  if (dtype == KVC_F32)
    KVC_CUDA(launch_dependent(e4m3 ? cache_append_kernel<float, KVC_E4M3> : cache_append_kernel<float, KVC_INT8>, grid, threads, 0, st, P,
                              (const float*)k_new, (const float*)v_new, n_new, lengths_out, weight, device_status));
  else
    KVC_CUDA(launch_dependent(e4m3 ? cache_append_kernel<__nv_bfloat16, KVC_E4M3> : cache_append_kernel<__nv_bfloat16, KVC_INT8>, grid,
                              threads, 0, st, P, (const __nv_bfloat16*)k_new, (const __nv_bfloat16*)v_new, n_new, lengths_out, weight,
                              device_status));
  KVC_LAUNCH_CHECK("cache_append_kernel");
  if (!P.write_lengths) {
    KVC_CUDA(launch_dependent(append_lengths_kernel, dim3((P.c.units() + 127) / 128), dim3(128), 0, st, P, n_new, lengths_out));
    KVC_LAUNCH_CHECK("append_lengths_kernel");
  }
  return KVC_OK;
}

kvc_status kvc_cache_read(const kvc_cache* cache, const int32_t* first, int64_t rows, int32_t dtype, void* k_out, void* v_out, void* stream) {
  ReadParams P;
  kvc_status s = resolve_cache(cache, "cache", &P.c);
  if (s != KVC_OK) return s;
  if ((s = check_dtype(dtype)) != KVC_OK) return s;
  KVC_REQUIRE8(k_out != nullptr || v_out != nullptr, KVC_ERR_INVALID_ARG, "k_out and v_out are both NULL");
  KVC_REQUIRE8(aligned16(k_out) && aligned16(v_out), KVC_ERR_INVALID_ARG, "k_out or v_out is not 16-byte aligned");
  KVC_REQUIRE8(rows >= 1, KVC_ERR_INVALID_ARG, "rows must be >= 1");
  KVC_REQUIRE8(rows < (1LL << 31), KVC_ERR_UNSUPPORTED, "rows must be < 2^31");
  if ((s = require_device()) != KVC_OK) return s;
  P.rows = rows;
  const long long items = rows * P.c.d / 16;
  long long ctas = (items + 256 * kReadEach - 1) / (256 * kReadEach);
  if (ctas > 65536) ctas = 65536;
  const dim3 grid((unsigned)ctas, P.c.units(), k_out != nullptr && v_out != nullptr ? 2 : 1);
  const bool e4m3 = P.c.format == KVC_E4M3;
  cudaStream_t st = (cudaStream_t)stream;
  if (dtype == KVC_F32)
    KVC_CUDA(launch_dependent(e4m3 ? cache_read_kernel<float, KVC_E4M3> : cache_read_kernel<float, KVC_INT8>, grid, dim3(256), 0, st, P,
                              first, (float*)k_out, (float*)v_out));
  else
    KVC_CUDA(launch_dependent(e4m3 ? cache_read_kernel<__nv_bfloat16, KVC_E4M3> : cache_read_kernel<__nv_bfloat16, KVC_INT8>, grid,
                              dim3(256), 0, st, P, first, (__nv_bfloat16*)k_out, (__nv_bfloat16*)v_out));
  KVC_LAUNCH_CHECK("cache_read_kernel");
  return KVC_OK;
}

}  // extern "C"
