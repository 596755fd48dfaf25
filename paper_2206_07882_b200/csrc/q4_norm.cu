// Root-mean-square norm with the residual's addition and 8-bit codes, one scale per row (q4_rmsnorm_quantize).
//
// With h the row (after the addition, rounded to its type) and v_i = h_i g_i:
//   scale = max |v| / sqrt(mean h^2 + eps) / 127,  code_i = rne(127 v_i / max |v|).
// Codes need the row's maximum, the scale its sum of squares as well; both come from one reduction.
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

// One block per row, all in double: v = h g has at most 48 bits, so products are exact.
template <typename T>
__global__ void __launch_bounds__(256) k_rmsnorm_quantize(const NormArgs a) {
  __shared__ double s_sum[8], s_max[8];
  const T* gain_row = nullptr;
  (void)gain_row;
  for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row * a.x_ld;
    const T* r = a.residual ? static_cast<const T*>(a.residual) + row * a.r_ld : nullptr;
    T* h = a.sum ? static_cast<T*>(a.sum) + row * a.s_ld : nullptr;
    auto value = [&](int i) {   // h_i; the thread that stores element i is the one that reads it again
      return to_f32<T>(r ? h[i] : x[i]);
    };
    if (r)
      for (int i = threadIdx.x; i < a.k; i += 256) h[i] = from_f32<T>(__fadd_rn(to_f32<T>(x[i]), to_f32<T>(r[i])));
    double sum = 0.0, top = 0.0;
    bool bad = false;
    for (int i = threadIdx.x; i < a.k; i += 256) {
      const float f = value(i);
      const double v = fabs((double)f * (double)a.gain[i]);
      sum += (double)f * (double)f;
      bad = bad || !(v <= 1.7e308) || !(fabsf(f) <= 3.4028235e38f);
      top = fmax(top, v);
    }
    for (int o = 16; o > 0; o >>= 1) {
      sum += __shfl_xor_sync(0xffffffffu, sum, o);
      top = fmax(top, __shfl_xor_sync(0xffffffffu, top, o));
    }
    if ((threadIdx.x & 31) == 0) {
      s_sum[threadIdx.x >> 5] = sum;
      s_max[threadIdx.x >> 5] = top;
    }
    bad = __syncthreads_or(bad) != 0;
    sum = top = 0.0;
    for (int w = 0; w < 8; ++w) {
      sum += s_sum[w];
      top = fmax(top, s_max[w]);
    }
    int8_t* q = a.q + row * a.k_pad;
    for (int i = threadIdx.x; i < a.k_pad; i += 256)
      q[i] = i < a.k && !bad && top > 0.0 ? (int8_t)__double2int_rn(127.0 * ((double)value(i) * (double)a.gain[i]) / top) : (int8_t)0;
    if (threadIdx.x == 0)
      a.scale[row] = bad ? __int_as_float(0x7fffffff) : (float)((top > 0.0 ? top / sqrt(sum / a.k + (double)a.eps) : 1.0) / 127.0);
    __syncthreads();
  }
}

}  // namespace

cudaError_t launch_rmsnorm_quantize(const NormArgs& a, int dtype, cudaStream_t s) {
  const unsigned blocks = (unsigned)(a.rows < (1 << 20) ? a.rows : (1 << 20));
  timing_begin(s);
  const cudaError_t e = dtype == Q4_F32   ? launch_ex(k_rmsnorm_quantize<float>, dim3(blocks), dim3(256), 0, s, false, 1, a)
                        : dtype == Q4_F16 ? launch_ex(k_rmsnorm_quantize<__half>, dim3(blocks), dim3(256), 0, s, false, 1, a)
                                          : launch_ex(k_rmsnorm_quantize<__nv_bfloat16>, dim3(blocks), dim3(256), 0, s, false, 1, a);
  timing_end(s);
  ++g_launches;
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace q4
