// Root-mean-square norm with the residual's addition and 8-bit codes, one scale per row (q4_rmsnorm_quantize).
//
// With h the row (after the addition, rounded to its type) and v_i = h_i g_i:
//   scale = max |v| / sqrt(mean h^2 + eps) / 127,  code_i = rne(127 v_i / max |v|).
// Codes need the row's maximum, the scale its sum of squares as well; both come from one reduction.
//
// Codes are those of exact arithmetic.  In fp32 t = v (127 / max |v|) is off by at most three roundings, 127 * 3 * 2^-24 < 2.3e-5; an
// element whose t lies further than that from a half is decided by it (t is not rounded itself: a fused operation adds the number
// that leaves its nearest integer, another takes the distance).  The others are decided in double, where v is exact and a half is
// decided by exact products (exact_code); the maximum is then taken from the exact products too.
#include <cuda_bf16.h>

#include "q4_internal.h"

namespace q4 {

namespace {

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32(float v) { return v; }
template <> __device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32(float v) { return __float2bfloat16_rn(v); }

// 16 bytes of a row
template <typename T>
union Vec {
  static constexpr int N = 16 / (int)sizeof(T);
  uint4 v16;
  uint2 v8[2];
  uint32_t v4[4];
  T e[N];
  __device__ Vec() {}
};
// Rows that are not 16-byte aligned.  The 16 bytes of a vector lie across two aligned granules, `shift` bytes into the first (the
// same for all vectors of a row): both are read and put together.  A granule is read as a whole only where it lies inside
// [lo, hi), the tensor's first and last byte; else the vector's elements are read one by one.  Elements from n on become 0.
__device__ __forceinline__ uint4 across(const uint4& a, const uint4& b, int shift) {   // bytes [shift, shift + 16) of (a, b)
  const int bits = (shift & 3) * 8;
  switch (shift >> 2) {
    case 0:
      return make_uint4(__funnelshift_r(a.x, a.y, bits), __funnelshift_r(a.y, a.z, bits), __funnelshift_r(a.z, a.w, bits), __funnelshift_r(a.w, b.x, bits));
    case 1:
      return make_uint4(__funnelshift_r(a.y, a.z, bits), __funnelshift_r(a.z, a.w, bits), __funnelshift_r(a.w, b.x, bits), __funnelshift_r(b.x, b.y, bits));
    case 2:
      return make_uint4(__funnelshift_r(a.z, a.w, bits), __funnelshift_r(a.w, b.x, bits), __funnelshift_r(b.x, b.y, bits), __funnelshift_r(b.y, b.z, bits));
    default:
      return make_uint4(__funnelshift_r(a.w, b.x, bits), __funnelshift_r(b.x, b.y, bits), __funnelshift_r(b.y, b.z, bits), __funnelshift_r(b.z, b.w, bits));
  }
}
template <typename T>
__device__ __forceinline__ void load_across(Vec<T>& v, const T* p, int n, uintptr_t lo, uintptr_t hi) {
  constexpr int N = Vec<T>::N;
  const uintptr_t at = reinterpret_cast<uintptr_t>(p), granule = at & ~(uintptr_t)15;
  v.v16 = make_uint4(0, 0, 0, 0);
  if (n <= 0) return;
  if (granule >= lo && granule + 32 <= hi) {
    const uint4* g = reinterpret_cast<const uint4*>(granule);
    v.v16 = across(g[0], g[1], (int)(at & 15));
    if (n < N) {
#pragma unroll
      for (int i = 1; i < N; ++i)
        if (i >= n) v.e[i] = T(0.0f);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n) v.e[i] = p[i];
  }
}
// By whole warps, lane l holding the l-th of neighbouring vectors: a lane stores the granule that its vector and its neighbour's lie
// in; the ends of what the warp holds are stored element by element.
template <typename T>
__device__ __forceinline__ void store_across(const Vec<T>& v, T* p, int n) {
  constexpr int N = Vec<T>::N;
  const int lane = threadIdx.x & 31, shift = (int)(reinterpret_cast<uintptr_t>(p) & 15);
  const bool full = n >= N;
  if (shift == 0) {                                            // the same for the whole warp
    if (full) {
      *reinterpret_cast<uint4*>(p) = v.v16;
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (i < n) p[i] = v.e[i];
    }
    return;
  }
  uint4 before;
  before.x = __shfl_up_sync(0xffffffffu, v.v16.x, 1);
  before.y = __shfl_up_sync(0xffffffffu, v.v16.y, 1);
  before.z = __shfl_up_sync(0xffffffffu, v.v16.z, 1);
  before.w = __shfl_up_sync(0xffffffffu, v.v16.w, 1);
  const bool next_full = __shfl_down_sync(0xffffffffu, full, 1) && lane < 31;
  const int in_front = (16 - shift) / (int)sizeof(T);          // elements of the vector in its first granule
  if (full && lane > 0) *reinterpret_cast<uint4*>(reinterpret_cast<uint8_t*>(p) - shift) = across(before, v.v16, 16 - shift);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const bool alone = full ? (i < in_front ? lane == 0 : !next_full) : i < n;
    if (alone) p[i] = v.e[i];
  }
}
// gains of elements [at, at + N) (at a multiple of N, gain 16-byte aligned); 0 behind the last
template <int N>
__device__ __forceinline__ void load_gain(float (&g)[N], const float* gain, int at, int k) {
  if (at + N <= k) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const float4 f = __ldg(reinterpret_cast<const float4*>(gain + at + i));
      g[i] = f.x;
      g[i + 1] = f.y;
      g[i + 2] = f.z;
      g[i + 3] = f.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) g[i] = at + i < k ? __ldg(gain + at + i) : 0.0f;
  }
}
// N codes given as integers in fp32, one byte each
template <int N>
__device__ __forceinline__ void store_codes(int8_t* q, const int (&c)[N]) {
  uint32_t w[N / 4];
#pragma unroll
  for (int i = 0; i < N / 4; ++i)
    w[i] = __byte_perm(__byte_perm(c[4 * i], c[4 * i + 1], 0x0040), __byte_perm(c[4 * i + 2], c[4 * i + 3], 0x0040), 0x5410);
  if (N == 8)
    *reinterpret_cast<uint2*>(q) = make_uint2(w[0], w[N / 4 - 1]);
  else
    *reinterpret_cast<uint32_t*>(q) = w[0];
}

__device__ __forceinline__ float larger(float a, float b) {   // a NaN stays
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
__device__ __forceinline__ double larger(double a, double b) { return fmax(a, b); }

// Sum and maximum over the THREADS threads of a row, the same in all of them.
template <int THREADS, typename F>
__device__ __forceinline__ void row_reduce(F& sum, F& top, F (*s)[2]) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    sum += __shfl_xor_sync(0xffffffffu, sum, o);
    top = larger(top, __shfl_xor_sync(0xffffffffu, top, o));
  }
  if (THREADS > 32) {
    if ((threadIdx.x & 31) == 0) {
      s[threadIdx.x >> 5][0] = sum;
      s[threadIdx.x >> 5][1] = top;
    }
    __syncthreads();
    sum = top = F(0);
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
      sum += s[w][0];
      top = larger(top, s[w][1]);
    }
    __syncthreads();
  }
}
template <int THREADS>
__device__ __forceinline__ bool row_any(bool v) {
  return THREADS > 32 ? __syncthreads_or(v) != 0 : __any_sync(0xffffffffu, v) != 0;
}

// 127 v / top rounded to the nearest integer, halves to even; v and top are products of two fp32 values, of 48 bits at most.  Of the
// quotient only its last bits are uncertain (by 127 * 3 * 2^-53), so that it decides unless it lies within 10^-9 of some n + 1/2, where the
// sign of 254 |v| - (2 n + 1) top does.  Those products take up to
// 56 bits: each is a rounded one and what fused operations find it to lack.  The rounded ones lie within 2 % of each other, so that their
// difference is exact, and so is that of the lacks, a few of their last places; one rounding of the sum keeps the sign.
__device__ __forceinline__ int exact_code(double v, double top) {
  constexpr double MAGIC64 = 6755399441055744.0;   // 1.5 * 2^52: adding it leaves the nearest integer in the low bits
  const double q = 127.0 * v / top, m = __dadd_rn(q, MAGIC64);
  if (fabs(q - (m - MAGIC64)) < 0.5 - 1e-9) return __double2loint(m);
  const double size = fabs(v);
  const int n = (int)fabs(q);
  const double odd = 2 * n + 1, a = __dmul_rn(254.0, size), b = __dmul_rn(odd, top);   // (rounded: not fused with what follows)
  const double over = (a - b) + (fma(254.0, size, -a) - fma(odd, top, -b));
  const int code = n + (over > 0.0 || (over == 0.0 && (n & 1)));
  return v < 0.0 ? -code : code;
}

// A row in double, from memory: for rows that hold no more than zeros, a NaN or infinity, or values whose squares or products leave
// the range of fp32, and for rows too long for registers.  Elements vec, vec + THREADS, ... of N are thread `t`'s, as everywhere; they are
// counted without a sign, as the step behind the last one of a row of nearly 2^31 passes that.
template <typename T, int THREADS>
__device__ __noinline__ void norm_row(const NormArgs& a, long long row, int t, double (*s)[2]) {
  constexpr int N = Vec<T>::N;
  const T* h = a.sum ? static_cast<const T*>(a.sum) + row * a.s_ld : static_cast<const T*>(a.x) + row * a.x_ld;
  int8_t* q = a.q + row * a.k_pad;
  __syncwarp();   // (a neighbour may have stored part of a vector of the sum; wider groups have met at a barrier since)
  double sum = 0.0, top = 0.0;
  bool bad = false;
  const uint32_t k = a.k, k_pad = a.k_pad;
  for (uint32_t v = t; v * N < k; v += THREADS)
    for (uint32_t i = v * N; i < min(v * N + N, k); ++i) {
      const double f = to_f32<T>(h[i]), p = fabs(f * (double)a.gain[i]);
      sum += f * f;
      top = fmax(top, p);
      bad = bad || !(fabs(f) <= 3.5e38) || !(p <= 1e300);
    }
  bad = row_any<THREADS>(bad);
  row_reduce<THREADS>(sum, top, s);
  for (uint32_t v = t; v * N < k_pad; v += THREADS) {
    int c[N];
    for (int i = 0; i < N; ++i) {
      const uint32_t at = v * N + i;
      c[i] = at < k && !bad && top > 0.0 ? exact_code((double)to_f32<T>(h[at]) * (double)a.gain[at], top) : 0;
    }
    store_codes<N>(q + v * N, c);
  }
  if (t == 0) a.scale[row] = bad ? __int_as_float(0x7fffffff) : (float)((top > 0.0 ? top / sqrt(sum / a.k + (double)a.eps) : 1.0) / 127.0);
}

constexpr float MAGIC = 12582912.0f;   // 1.5 * 2^23: adding it leaves the nearest integer in the low bits
constexpr float SETTLED = 0.5f - 3.2e-5f;

__device__ __forceinline__ float max_abs3(float a, float b, float c) {   // of the magnitudes, a NaN stays
  float d;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

__device__ __forceinline__ uint4 load_once(const void* p) {   // past the L1, which keeps the gains
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
template <typename T>
__device__ __forceinline__ void unpack(const Vec<T>& v, float (&f)[Vec<T>::N]) {
#pragma unroll
  for (int i = 0; i < Vec<T>::N; ++i) f[i] = to_f32<T>(v.e[i]);
}
template <>
__device__ __forceinline__ void unpack<__nv_bfloat16>(const Vec<__nv_bfloat16>& v, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(v.v4[i] << 16);
    f[2 * i + 1] = __uint_as_float(v.v4[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void pack(Vec<float>& v, const float (&f)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v.e[i] = f[i];
}
__device__ __forceinline__ void pack(Vec<__half>& v, const float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2 p = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
    v.v4[i] = *reinterpret_cast<const uint32_t*>(&p);
  }
}
__device__ __forceinline__ void pack(Vec<__nv_bfloat16>& v, const float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
    v.v4[i] = *reinterpret_cast<const uint32_t*>(&p);
  }
}

// A row per group of THREADS threads; everything is read and written once, the products v lie in registers, NV vectors of 16 bytes of
// the row a thread.  WHOLE: rows are 16-byte aligned and a multiple of that long.
// Long rows are bound by memory (4096 x 4096 with a residual: fp32 36.9 us, 5.9 TB/s; bf16 24.5 us, 4.8 TB/s), short ones of 16 bits
// by their instructions, about 14 for each element, and waits that few warps cover (16000 x 1280 fp16 alone: 17.7 us, 3.5 TB/s; with a
// sixth vector that holds nothing 20.6; with the next row copied ahead to shared memory 22).  One warp a row needs no barrier;
// wider groups take rows that a warp's registers do not hold, and few rows, where a row's latency is the call's (16 x 1024: 2.2 us).
// Forming the products again for the codes, for registers of half as many bits, took 10 % more.  Rows that are not 16-byte
// aligned (4096 x 4001 bf16) take 49 us; element by element they took 75.
// Threads of a block: four rows of one warp, or one row.  Blocks of an SM: 64 registers a thread for up to 16 elements, 80 for up to
// 40, 96 and 128 for up to 48 and 64.
__host__ __device__ constexpr int norm_threads(int threads) { return threads > 32 ? threads : 128; }
__host__ __device__ constexpr int norm_blocks(int threads, int elements) {
  return 128 * (elements <= 16 ? 8 : elements <= 40 ? 6 : elements <= 48 ? 5 : 4) / norm_threads(threads);
}
template <typename T, int THREADS, int NV, bool WHOLE>
__global__ void __launch_bounds__(norm_threads(THREADS), norm_blocks(THREADS, NV * (16 / (int)sizeof(T)))) k_rmsnorm_quantize(const __grid_constant__ NormArgs a) {
  constexpr int N = Vec<T>::N, ROWS = norm_threads(THREADS) / THREADS;
  __shared__ float s_part[THREADS / 32][2];
  __shared__ double s_part64[THREADS / 32][2];
  const int t = threadIdx.x % THREADS;
  const uintptr_t lo_x = reinterpret_cast<uintptr_t>(a.x), hi_x = lo_x + ((a.rows - 1) * a.x_ld + a.k) * sizeof(T);
  const uintptr_t lo_r = reinterpret_cast<uintptr_t>(a.residual), hi_r = lo_r + ((a.rows - 1) * a.r_ld + a.k) * sizeof(T);
  pdl_wait();
  pdl_trigger();
  for (long long row = (long long)blockIdx.x * ROWS + threadIdx.x / THREADS; row < a.rows; row += (long long)gridDim.x * ROWS) {
    const T* x = static_cast<const T*>(a.x) + row * a.x_ld;
    const T* h = x;
    int8_t* q = a.q + row * a.k_pad;
    auto load = [&](Vec<T>& v, const T* p, int at, uintptr_t lo, uintptr_t hi) {
      if (!WHOLE)
        load_across<T>(v, p + at, a.k - at, lo, hi);
      else
        v.v16 = at < a.k ? load_once(p + at) : make_uint4(0, 0, 0, 0);
    };
    Vec<T> raw[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) load(raw[j], x, (t + j * THREADS) * N, lo_x, hi_x);
    if (a.residual) {
      const T* r = static_cast<const T*>(a.residual) + row * a.r_ld;
      T* out = static_cast<T*>(a.sum) + row * a.s_ld;
      Vec<T> add[NV];
#pragma unroll
      for (int j = 0; j < NV; ++j) load(add[j], r, (t + j * THREADS) * N, lo_r, hi_r);
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int at = (t + j * THREADS) * N;
        float f[N], g[N];
        unpack<T>(raw[j], f);
        unpack<T>(add[j], g);
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = __fadd_rn(f[i], g[i]);
        pack(raw[j], f);
        if (!WHOLE)
          store_across<T>(raw[j], out + at, a.k - at);
        else if (at < a.k)
          *reinterpret_cast<uint4*>(out + at) = raw[j].v16;
      }
      h = out;
    }
    float v[NV][N], sum = 0.0f, top = 0.0f;
    {
      uint64_t squares = pk2(0.0f, 0.0f);
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float g[N], f[N];
        load_gain<N>(g, a.gain, (t + j * THREADS) * N, a.k);
        unpack<T>(raw[j], f);
#pragma unroll
        for (int i = 0; i < N; i += 2) {
          const uint64_t f2 = pk2(f[i], f[i + 1]);
          squares = fma2(f2, f2, squares);
          upk2(mul2(f2, pk2(g[i], g[i + 1])), v[j][i], v[j][i + 1]);
          top = max_abs3(top, v[j][i], v[j][i + 1]);
        }
      }
      float odd;
      upk2(squares, sum, odd);
      sum += odd;
    }
    row_reduce<THREADS>(sum, top, s_part);
    // (a NaN or infinity of the row is in the sum, one of the gain, or of both, in the maximum)
    if (!(top > 1e-30f && top < 1e37f && sum > 1e-30f && sum < 1e38f)) {
      norm_row<T, THREADS>(a, row, t, s_part64);
      continue;
    }
    if (t == 0) a.scale[row] = __fdiv_rn(__fdiv_rn(top, __fsqrt_rn(__fadd_rn(__fdiv_rn(sum, (float)a.k), a.eps))), 127.0f);
    const float inv = __fdiv_rn(127.0f, top);
    const uint64_t inv2 = pk2(inv, inv), magic2 = pk2(MAGIC, MAGIC);
    uint32_t unsettled = 0;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int at = (t + j * THREADS) * N;
      int c[N];
      float off = 0.0f;
#pragma unroll
      for (int i = 0; i < N; i += 2) {   // m = the nearest integer plus MAGIC, off: distance from it
        const uint64_t v2 = pk2(v[j][i], v[j][i + 1]), m = fma2(v2, inv2, magic2);
        float m0, m1, d0, d1;
        upk2(m, m0, m1);
        upk2(fma2(v2, inv2, sub2(magic2, m)), d0, d1);
        off = max_abs3(off, d0, d1);
        c[i] = __float_as_int(m0);
        c[i + 1] = __float_as_int(m1);
      }
      if (at < a.k_pad) store_codes<N>(q + at, c);
      if (off > SETTLED) unsettled |= 1u << j;
    }
    if (!row_any<THREADS>(unsettled != 0)) continue;
    __syncwarp();   // as in norm_row: elements of the sum are read again
    double exact = 0.0, unused = 0.0;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (fabsf(v[j][i]) == top) {
          const int at = (t + j * THREADS) * N + i;
          exact = fmax(exact, fabs((double)to_f32<T>(h[at]) * (double)a.gain[at]));
        }
    row_reduce<THREADS>(unused, exact, s_part64);
#pragma unroll 1
    for (int j = 0; j < NV; ++j) {
      if (!(unsettled >> j & 1)) continue;
      for (int i = 0; i < N; ++i) {
        const int at = (t + j * THREADS) * N + i;
        if (at >= a.k) break;
        const float f = to_f32<T>(h[at]), g = a.gain[at], p = __fmul_rn(f, g), m = __fmaf_rn(p, inv, MAGIC);
        if (fabsf(__fmaf_rn(p, inv, __fsub_rn(MAGIC, m))) > SETTLED) q[at] = (int8_t)exact_code((double)f * (double)g, exact);
      }
    }
  }
}

// Rows of any length, from memory in double.
template <typename T>
__global__ void __launch_bounds__(512) k_rmsnorm_quantize_long(const __grid_constant__ NormArgs a) {
  __shared__ double s_part64[16][2];
  pdl_wait();
  pdl_trigger();
  for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
    if (a.residual) {
      constexpr int N = Vec<T>::N;
      const T *x = static_cast<const T*>(a.x) + row * a.x_ld, *r = static_cast<const T*>(a.residual) + row * a.r_ld;
      T* out = static_cast<T*>(a.sum) + row * a.s_ld;
      const uint32_t k = a.k;
      for (uint32_t v = threadIdx.x; v * N < k; v += 512)
        for (uint32_t i = v * N; i < min(v * N + N, k); ++i) out[i] = from_f32<T>(__fadd_rn(to_f32<T>(x[i]), to_f32<T>(r[i])));
    }
    norm_row<T, 512>(a, row, threadIdx.x, s_part64);
  }
}

template <typename T, int THREADS, int NV, bool WHOLE>
cudaError_t launch_rows(const NormArgs& a, cudaStream_t s) {
  constexpr int ROWS = norm_threads(THREADS) / THREADS;
  const long long blocks = (a.rows + ROWS - 1) / ROWS;
  return launch_ex(k_rmsnorm_quantize<T, THREADS, NV, WHOLE>, dim3((unsigned)(blocks < (1 << 20) ? blocks : 1 << 20)),
                   dim3(norm_threads(THREADS)), 0, s, true, 1, a);
}
// Vectors of a thread at most: 48 elements of 16 bits, 32 of 32; in the widest group 64 of 16 bits.
template <typename T> constexpr int MOST = sizeof(T) == 4 ? 8 : 6;
template <typename T, int THREADS>
cudaError_t launch_group(const NormArgs& a, int nv, bool whole, cudaStream_t s) {
  constexpr int ALL = THREADS == 512 ? 8 : MOST<T>;
  if (whole) switch (nv) {
    case 1: case 2: return launch_rows<T, THREADS, 2, true>(a, s);
    case 3: return launch_rows<T, THREADS, 3, true>(a, s);
    case 4: return launch_rows<T, THREADS, 4, true>(a, s);
    case 5: return launch_rows<T, THREADS, 5, true>(a, s);
    case 6: return launch_rows<T, THREADS, 6, true>(a, s);
    default: return launch_rows<T, THREADS, ALL, true>(a, s);
  }
  return nv <= 2   ? launch_rows<T, THREADS, 2, false>(a, s)
         : nv <= 4 ? launch_rows<T, THREADS, 4, false>(a, s)
         : nv <= 6 ? launch_rows<T, THREADS, 6, false>(a, s)
                   : launch_rows<T, THREADS, ALL, false>(a, s);
}
template <typename T>
cudaError_t launch_norm(const NormArgs& a, cudaStream_t s) {
  // rows of x, residual and sum that are multiples of 16 bytes long and apart
  uintptr_t low = reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.residual) | reinterpret_cast<uintptr_t>(a.sum) | a.k * sizeof(T);
  if (a.rows > 1) low |= (uintptr_t)(a.x_ld | a.r_ld | a.s_ld) * sizeof(T);
  const bool whole = low % 16 == 0;
  const int vectors = a.k_pad / Vec<T>::N;
  // The narrowest group that holds a row, then wider ones while the rows' threads would not fill the SMs (768 threads are what one holds
  // of most of these kernels; for narrow groups and 16 bits twice as many).  bf16, us: rows of 4096 with 128 threads of 4 vectors and with 256
  // of 2, 300 rows 5.2 and 4.9, 1200 rows 7.7 and 8.2, 16000 rows 55 and 71; rows of 1024 with 32 of 4 and 64 of 2, 2048 rows 5.9 and
  // 4.8, 16000 rows 15.6 and 19.3.
  const long long fill = 768LL * sm_count();
  int threads = 32;
  while (threads < 512 && vectors > threads * MOST<T>) threads *= 2;
  while (threads < 128 && vectors > threads * 2 && a.rows * threads < fill * (4 / (int)sizeof(T))) threads *= 2;
  while (threads >= 128 && threads < 512 && vectors > threads * 3 && a.rows * threads < fill) threads *= 2;
  const int nv = (vectors + threads - 1) / threads;
  if (threads == 32) return launch_group<T, 32>(a, nv, whole, s);
  if (threads == 64) return launch_group<T, 64>(a, nv, whole, s);
  if (threads == 128) return launch_group<T, 128>(a, nv, whole, s);
  if (threads == 256) return launch_group<T, 256>(a, nv, whole, s);
  if (nv <= 8) return launch_group<T, 512>(a, nv, whole, s);
  return launch_ex(k_rmsnorm_quantize_long<T>, dim3((unsigned)(a.rows < (1 << 20) ? a.rows : 1 << 20)), dim3(512), 0, s, true, 1, a);
}

}  // namespace

cudaError_t launch_rmsnorm_quantize(const NormArgs& a, int dtype, cudaStream_t s) {
  timing_begin(s);
  const cudaError_t e = dtype == Q4_F32 ? launch_norm<float>(a, s) : dtype == Q4_F16 ? launch_norm<__half>(a, s) : launch_norm<__nv_bfloat16>(a, s);
  timing_end(s);
  ++g_launches;
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace q4
