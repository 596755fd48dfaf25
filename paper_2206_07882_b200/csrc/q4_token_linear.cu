// Linear layer on 8-bit codes with a scale for every token and every output channel (q4_linear_token_scales).
//
// out[m, n] = (sum_k x[m, k] w[n, k]) (sx[m] sw[n]) + b[n], the sum in int32.
#include <cuda_bf16.h>
#include <string.h>

#include "q4_internal.h"
#include "q4_mma.cuh"

namespace q4 {

namespace {

constexpr int BK = 128;        // codes per row of an operand tile
constexpr int CH = 128;        // output channels of a tile: the lanes of the accumulator
constexpr uint32_t WAIT_LIMIT = 1u << 22;

template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32(float v) { return __float2bfloat16_rn(v); }

__host__ __device__ constexpr int stages(int tok) { return tok <= 32 ? 8 : tok <= 64 ? 6 : tok <= 128 ? 6 : 4; }
__host__ __device__ constexpr size_t smem_bytes(int tok) { return (size_t)stages(tok) * (CH + tok) * BK + 1024; }

// Channels are the rows (lanes) of the accumulator and tokens its columns: a warp's 32 lanes store 32 neighbouring channels
// of one token.
template <int TOK, typename T>
__global__ void __launch_bounds__(192, 1)
k_token_linear(const __grid_constant__ CUtensorMap tma_w, const __grid_constant__ CUtensorMap tma_x, const TokenLinearArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  constexpr int NS = stages(TOK), W_BYTES = CH * BK, STAGE = W_BYTES + TOK * BK;
  constexpr uint32_t TCOLS = TOK < 32 ? 32 : TOK;
  __shared__ uint64_t full[NS], empty[NS], acc_full;
  __shared__ uint32_t tmem_base_s, failed;
  __shared__ float s_x[TOK];
  const int tid = threadIdx.x, warp = uniform_warp(), lane = tid & 31;
  const int n0 = blockIdx.x * CH, m0 = blockIdx.y * TOK, nk = (a.K + BK - 1) / BK;
  if (tid == 0) {
    for (int s = 0; s < NS; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    mbar_init(&acc_full, 1);
    failed = 0;
    fence_barrier_init();
    fence_proxy_async();
  }
  if (warp == 5) tmem_alloc(&tmem_base_s, TCOLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base_s;
  pdl_wait();
  if (warp == 4) {
    const uint32_t on = elect_one();
    bool ok = true;
    for (int i = 0; i < nk && ok; ++i) {
      const int s = i % NS;
      ok = i < NS || mbar_wait_warp(&empty[s], (uint32_t)(i / NS - 1) & 1u, WAIT_LIMIT);
      if (!ok) {
        failed = 1;
        ring_landed(full, NS, i);
        break;
      }
      mbar_expect_tx(on, &full[s], STAGE);
      tma_load_2d(on, smem + s * STAGE, &tma_w, i * BK, n0, &full[s]);
      tma_load_2d(on, smem + s * STAGE + W_BYTES, &tma_x, i * BK, m0, &full[s]);
    }
  } else if (warp == 5) {
    const uint32_t idesc = umma_idesc_i8(CH, TOK), on = elect_one();
    bool ok = true;
    for (int i = 0; i < nk && ok; ++i) {
      const int s = i % NS;
      ok = mbar_wait_warp(&full[s], (uint32_t)(i / NS) & 1u, WAIT_LIMIT);
      if (!ok) {
        failed = 1;
        ring_landed(full, NS, nk);
        break;
      }
      tc_fence_after();
      const uint64_t dw = umma_desc_sw128(smem_u32(smem + s * STAGE)), dx = umma_desc_sw128(smem_u32(smem + s * STAGE + W_BYTES));
#pragma unroll
      for (int kk = 0; kk < BK / 32; ++kk) umma_i8(on, tmem, dw + 2 * kk, dx + 2 * kk, idesc, (i | kk) != 0);
      umma_commit(on, &empty[s]);
    }
    umma_commit(on, &acc_full);
  } else {
    for (int c = tid; c < TOK; c += 128) s_x[c] = m0 + c < a.M ? a.x_scale[m0 + c] : 0.0f;
    asm volatile("bar.sync 1, 128;" ::: "memory");
    const int n = n0 + warp * 32 + lane;
    const float sw = n < a.N ? a.w_scale[n] : 0.0f, b = a.bias && n < a.N ? a.bias[n] : 0.0f;
    const bool ok = mbar_wait(&acc_full, 0, WAIT_LIMIT) && *reinterpret_cast<volatile uint32_t*>(&failed) == 0;
    tc_fence_after();
    if (!ok && a.status && lane == 0) atomicExch(a.status, Q4_ERR_TIMEOUT);
    T* out = static_cast<T*>(a.out) + n;
    for (int c0 = 0; c0 < TOK; c0 += 16) {
      int r[16];
      tmem_ld16(tmem + ((uint32_t)(warp * 32) << 16) + c0, r);
      tmem_ld_wait();
      if (!ok || n >= a.N) continue;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int m = m0 + c0 + i;
        if (m < a.M) out[(long long)m * a.ldo] = from_f32<T>(__fmaf_rn((float)r[i], __fmul_rn(s_x[c0 + i], sw), b));
      }
    }
  }
  pdl_trigger();
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 5) tmem_dealloc(tmem, TCOLS);
}

template <int TOK, typename T>
cudaError_t launch_tile(const TokenLinearArgs& a, cudaStream_t s) {
  static bool configured_on[MAX_DEVICES];
  bool& configured = configured_on[device_slot()];
  if (!configured) {
    const cudaError_t e = cudaFuncSetAttribute(k_token_linear<TOK, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes(TOK));
    if (e != cudaSuccess) return e;
    configured = true;
  }
  CUtensorMap tw, tx;
  if (!make_tmap_i8(&tw, a.wq, a.K, a.N, a.K, CH) || !make_tmap_i8(&tx, a.xq, a.K, a.M, a.K, TOK)) return cudaErrorInvalidValue;
  return launch_ex(k_token_linear<TOK, T>, dim3((a.N + CH - 1) / CH, (a.M + TOK - 1) / TOK), dim3(192), smem_bytes(TOK), s, true, 1,
                   tw, tx, a);
}
template <typename T>
cudaError_t launch_typed(const TokenLinearArgs& a, cudaStream_t s) {
  return a.M <= 16   ? launch_tile<16, T>(a, s)
         : a.M <= 64 ? launch_tile<64, T>(a, s)
                     : launch_tile<256, T>(a, s);
}

}  // namespace

cudaError_t launch_token_linear(const TokenLinearArgs& a, int dtype, cudaStream_t s) {
  timing_begin(s);
  const cudaError_t e = dtype == Q4_F32   ? launch_typed<float>(a, s)
                        : dtype == Q4_F16 ? launch_typed<__half>(a, s)
                                          : launch_typed<__nv_bfloat16>(a, s);
  timing_end(s);
  ++g_launches;
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace q4
