// The 8-bit cache of kvc.h: resolved descriptor, exponents and codes.  Shared by cache8.cu, evict.cu and attend.cu.
#pragma once

#include <cuda_fp8.h>

#include <atomic>

#include "kvc_internal.cuh"

namespace kvc {

constexpr int kExpMin = -100, kExpMax = 121;   // 2^e and 2^-e are normal fp32 numbers with room for the codes

// A kvc_cache with its strides filled in.
struct Cache {
  int Bt, Hkv, d, block, block_shift, format;
  long long cap, blocks;                  // blocks: exponents per head
  long long st[3];                        // in codes (bytes)
  uint8_t *k, *v;
  int8_t *k_exp, *v_exp;
  int32_t* lengths;
  __host__ __device__ int units() const { return Bt * Hkv; }
  __device__ __forceinline__ long long base(int unit) const { return (unit / Hkv) * st[0] + (unit % Hkv) * st[1]; }
  // rows in use, whatever the caller's array holds
  __device__ __forceinline__ long long length(int unit) const {
    const long long n = lengths[unit];
    return n < 0 ? 0 : (n > cap ? cap : n);
  }
};

kvc_status resolve_cache(const kvc_cache* c, const char* name, Cache* out);
// Element strides (batch, head, row) of a [batch, heads, rows, d] array: checked, or dense.  An array that is written to
// must not overlap itself.
kvc_status resolve_strides(const int64_t* given, int batch, int heads, long long rows, int d, int elem_bytes, bool written,
                           const char* name, long long* out);
// kvc_dtype of an argument that is not part of a kvc_desc.
kvc_status check_dtype(int32_t dtype);
bool aligned16(const void* p);

#define KVC_REQUIRE8(cond, code, ...)     \
  do {                                    \
    if (!(cond)) {                        \
      ::kvc::set_error(__VA_ARGS__);      \
      return code;                        \
    }                                     \
  } while (0)

#ifdef __CUDACC__

// 2^e for e in [-126, 127]
__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }
__device__ __forceinline__ float pow2_clamped(int e) { return pow2(min(max(e, -126), 127)); }

// The smallest e with amax <= qmax 2^e: with amax = m 2^E, m in [1, 2), that is E minus the exponent of qmax, and one
// more where m exceeds qmax's own significand (448 = 1.75 * 2^8, 127 = 1.984375 * 2^6).  Zero and subnormal amax end at
// the lower bound.  `up`: amax (finite) stands for amax * 2^up; codes can stand for more than fp32 holds.
template <int kFormat>
__device__ __forceinline__ int exponent_of(float amax, int up = 0) {
  const uint32_t b = __float_as_uint(amax);
  const int E = (int)(b >> 23) - 127 + up;
  const uint32_t m = b & 0x7fffffu;
  const int e = kFormat == KVC_E4M3 ? E - 8 + (m > 0x600000u) : E - 6 + (m > 0x7e0000u);
  return min(max(e, kExpMin), kExpMax);
}

// Codes of four values x * f (f a power of two, so the product is exact but for what rounds to zero): rounded to
// nearest, ties to even, held at the largest code.
template <int kFormat>
__device__ __forceinline__ uint32_t encode4(float x0, float x1, float x2, float x3, float f) {
  if (kFormat == KVC_E4M3) {
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(x1 * f), "f"(x0 * f));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(x3 * f), "f"(x2 * f));
    return (uint32_t)lo | ((uint32_t)hi << 16);
  }
  const int a = min(max(__float2int_rn(x0 * f), -127), 127), b = min(max(__float2int_rn(x1 * f), -127), 127);
  const int c = min(max(__float2int_rn(x2 * f), -127), 127), d = min(max(__float2int_rn(x3 * f), -127), 127);
  return (a & 255) | ((b & 255) << 8) | ((c & 255) << 16) | ((uint32_t)d << 24);
}

// The values of four codes, without the exponent.
template <int kFormat>
__device__ __forceinline__ void decode4(uint32_t w, float* x) {
  if (kFormat == KVC_E4M3) {
    uint32_t a, b;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(a) : "h"((uint16_t)w));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(b) : "h"((uint16_t)(w >> 16)));
    const float2 fa = __half22float2(*reinterpret_cast<__half2*>(&a)), fb = __half22float2(*reinterpret_cast<__half2*>(&b));
    x[0] = fa.x; x[1] = fa.y; x[2] = fb.x; x[3] = fb.y;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(w >> (8 * i));
  }
}

__device__ __forceinline__ uint4 ld16(const void* p) { return *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ uint4 ld16_stream(const void* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

// The largest magnitude among 8-bit codes, as fp32.  pairs: two 16-bit maxima, of e4m3 magnitudes (as codes, whose order is
// that of the values) or of int8 magnitudes.
template <int kFormat>
__device__ __forceinline__ uint32_t max_codes(uint32_t pairs, uint32_t w) {
  if (kFormat == KVC_E4M3) return __vmaxu2(__vmaxu2(pairs, w & 0x007f007fu), (w >> 8) & 0x007f007fu);
  uint32_t a, b;                          // sign-extended (a selector's fourth bit copies the byte's sign)
  asm("prmt.b32 %0, %1, 0, 0x9180;" : "=r"(a) : "r"(w));
  asm("prmt.b32 %0, %1, 0, 0xb3a2;" : "=r"(b) : "r"(w));
  return __vmaxu2(__vmaxu2(pairs, __vabs2(a)), __vabs2(b));
}
template <int kFormat>
__device__ __forceinline__ float max_value(uint32_t pairs) {
  const uint32_t m = max(pairs & 0xffffu, pairs >> 16);
  // (e4m3: the bits moved to fp32's place, whose exponents are biased by 120 more)
  return kFormat == KVC_E4M3 ? __uint_as_float(m << 20) * pow2(120) : (float)m;
}

// A block's tokens as one job of block * d / 32 threads with 32 values of K and of V each, in groups of kGroup values of a row.
// The jobs of a CTA lie side by side; a job is one warp or whole warps.
// A job's threads are a multiple of a row's groups, so a thread has the same place in each of its rows.
template <int kGroup>
struct JobLane {
  static constexpr int kGroups = 32 / kGroup;
  int threads, slot, t, row0, row_step, col;           // rows row0, row0 + row_step, ..; entries from col on
  __device__ __forceinline__ JobLane(int block_shift, int d) {
    const int per_row_shift = (d == 128 ? 7 : 6) - (kGroup == 8 ? 3 : 4);      // log2(d / kGroup)
    const int shift = block_shift + (d == 128 ? 2 : 1);
    threads = 1 << shift;
    slot = threadIdx.x >> shift;
    t = threadIdx.x & (threads - 1);
    row0 = t >> per_row_shift;
    row_step = threads >> per_row_shift;
    col = (t & ((1 << per_row_shift) - 1)) * kGroup;
  }
  __device__ __forceinline__ int row(int g) const { return row0 + g * row_step; }
};

// A job's threads meet (a warp, or whole warps: barrier 1 + slot).
template <typename Job>
__device__ __forceinline__ void job_barrier(const Job& j) {
  if (j.threads == 32) __syncwarp();
  else asm volatile("bar.sync %0, %1;" :: "r"(1 + j.slot), "r"(j.threads) : "memory");
}

// The largest of a job's threads' values, of K and of V: non-negative, and compared by their bits, in which NaN is above infinity.
// kTogether: every thread of the CTA calls it; else whole jobs do.  scratch: one per warp.
template <bool kTogether = true, typename Job>
__device__ __forceinline__ float2 job_max(float2 x, const Job& j, float2* scratch) {
  uint32_t k = __reduce_max_sync(0xffffffffu, __float_as_uint(x.x)), v = __reduce_max_sync(0xffffffffu, __float_as_uint(x.y));
  if (j.threads > 32) {
    const auto meet = [&] { if (kTogether) __syncthreads(); else job_barrier(j); };
    meet();                               // (the scratch of the call before has been read)
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = make_float2(__uint_as_float(k), __uint_as_float(v));
    meet();
    const int w0 = j.slot * (j.threads >> 5);
    for (int i = 0; i < (j.threads >> 5); ++i) {
      k = max(k, __float_as_uint(scratch[w0 + i].x));
      v = max(v, __float_as_uint(scratch[w0 + i].y));
    }
  }
  return make_float2(__uint_as_float(k), __uint_as_float(v));
}

__device__ __forceinline__ bool all_finite(float2 top) { return max(__float_as_uint(top.x), __float_as_uint(top.y)) < 0x7f800000u; }

// Eight values as they lie in memory.
template <typename T>
struct Raw8 {
  uint4 w[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {          // (read once: past L1)
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = ld16_stream(reinterpret_cast<const char*>(p) + 16 * i);
  }
  __device__ __forceinline__ void load_coherent(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = ld16(reinterpret_cast<const char*>(p) + 16 * i);
  }
  __device__ __forceinline__ void store(T* p) const {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) *reinterpret_cast<uint4*>(reinterpret_cast<char*>(p) + 16 * i) = w[i];
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = make_uint4(0, 0, 0, 0);
  }
  __device__ __forceinline__ void values(float* x) const {
    const uint32_t* u = &w[0].x;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) * 2; ++i) {
      if (sizeof(T) == 2) {
        x[2 * i] = __uint_as_float(u[i] << 16);
        x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
      } else {
        x[i] = __uint_as_float(u[i]);
      }
    }
  }
  // The magnitudes' bits, whose order is the values'; of bf16 two maxima side by side (see top()).
  __device__ __forceinline__ uint32_t max_bits(uint32_t m) const {
    const uint32_t* u = &w[0].x;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) * 2; ++i) m = sizeof(T) == 2 ? __vmaxu2(m, u[i] & 0x7fff7fffu) : max(m, u[i] & 0x7fffffffu);
    return m;
  }
  // max_bits of the finite values; NaN become zero.
  __device__ __forceinline__ uint32_t max_finite_bits(uint32_t m) {
    uint32_t* u = &w[0].x;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) * 2; ++i) {
      if (sizeof(T) == 2) {
        const uint32_t lo = u[i] & 0x7fffu, hi = (u[i] >> 16) & 0x7fffu;
        if (lo > 0x7f80u) u[i] &= 0xffff0000u;
        if (hi > 0x7f80u) u[i] &= 0x0000ffffu;
        m = __vmaxu2(m, (lo < 0x7f80u ? lo : 0u) | (hi < 0x7f80u ? hi << 16 : 0u));
      } else {
        const uint32_t mag = u[i] & 0x7fffffffu;
        if (mag > 0x7f800000u) u[i] = 0;
        if (mag < 0x7f800000u) m = max(m, mag);
      }
    }
    return m;
  }
  static __device__ __forceinline__ float top(uint32_t m) {
    return __uint_as_float(sizeof(T) == 2 ? max(m << 16, m & 0xffff0000u) : m);
  }
  template <int kFormat>
  __device__ __forceinline__ uint2 encode(float f) const {
    float x[8];
    values(x);
    return make_uint2(encode4<kFormat>(x[0], x[1], x[2], x[3], f), encode4<kFormat>(x[4], x[5], x[6], x[7], f));
  }
};

// A job's largest values where some are not finite: of the finite ones.  The rows are read again, one at a time, so that the
// way without such rows keeps its registers (64; with the rows kept for both, 97).  row(g): where row g of the thread lies, -1 if
// there is none.  The status word, if it holds no error yet, says so.  Whole jobs call it.
template <typename T, typename Job, typename Row>
__device__ __forceinline__ float2 finite_max(const T* k, const T* v, const Row& row, const Job& j, float2* scratch, int32_t* device_status) {
  if (j.t == 0 && device_status != nullptr) atomicCAS(device_status, KVC_OK, KVC_ERR_NOT_FINITE);
  uint32_t km = 0, vm = 0;
#pragma unroll 1
  for (int g = 0; g < 4; ++g) {
    const long long at = row(g);
    if (at < 0) continue;
    Raw8<T> x;
    x.load(k + at);
    km = x.max_finite_bits(km);
    x.load(v + at);
    vm = x.max_finite_bits(vm);
  }
  return job_max<false>(make_float2(Raw8<T>::top(km), Raw8<T>::top(vm)), j, scratch);
}
// Codes of eight such values: a NaN is taken as zero, an infinity is held at the largest code.
template <int kFormat, typename T>
__device__ __forceinline__ uint2 encode_any(const T* p, float f) {
  Raw8<T> x;
  x.load(p);
  x.max_finite_bits(0);
  return x.template encode<kFormat>(f);
}

// Sixteen codes rounded again after a change of exponent.
template <int kFormat>
__device__ __forceinline__ uint4 recode(uint4 w, float f) {
  uint32_t* u = &w.x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float x[4];
    decode4<kFormat>(u[i], x);
    u[i] = encode4<kFormat>(x[0], x[1], x[2], x[3], f);
  }
  return w;
}

template <typename T>
__device__ __forceinline__ void load8(const T* p, float* x) {
  Raw8<T> r;
  r.load(p);
  r.values(x);
}

// cudaFuncSetAttribute's opt-in to more shared memory, once per kernel and device (`done`: a word of the call site's own).
template <typename Kernel>
inline cudaError_t allow_smem(Kernel kernel, int bytes, std::atomic<uint64_t>& done, int dev) {
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if ((done.load(std::memory_order_relaxed) & bit) != 0) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

// Threads of a CTA that works on blocks: at least 256, and whole jobs.
inline int job_cta_threads(const Cache& c) {
  const int t = c.block * c.d / 32;
  return t > 256 ? t : 256;
}

#endif  // __CUDACC__

}  // namespace kvc
