// Linear layer on 8-bit codes with a scale for every token and every output channel (q4_linear_token_scales).
//
// out[m, n] = (sum_k x[m, k] w[n, k]) (sx[m] sw[n]) + b[n], the sum in int32.
//
// Channels are the rows (lanes) of the accumulator in tensor memory and tokens its columns, whatever their numbers: a warp's 32
// lanes store 32 neighbouring channels of one token, a channel's scale and bias stay in a register, and few tokens make a narrow
// tile.  Codes are the tensor cores' operands as they are stored.
#include <cuda_bf16.h>
#include <math.h>
#include <string.h>

#include "q4_internal.h"
#include "q4_mma.cuh"

namespace q4 {

namespace {

constexpr int BK = 128;        // codes per row of an operand tile
constexpr int CH = 128;        // output channels of a CTA's tile, of most

template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ void record_timeout(int32_t* status) {
  if (status) atomicExch(status, Q4_ERR_TIMEOUT);
}

// COLS accumulator columns of a warp's 32 lanes, from `taddr` on, to tokens 0 .. min(COLS, tokens) - 1 at `out` (this lane's channel).
// Two sets of registers: the next columns are on their way out of tensor memory while these are stored; `drained` is called once
// all have been read.
template <typename T, int COLS, typename F>
__device__ __forceinline__ void store_columns(uint32_t taddr, T* out, long long ldo, const float* scale, float sw, float b, int tokens, F drained) {
  constexpr int STEP = COLS < 32 ? COLS : 32;
  int r[2][STEP];
  tmem_ld(taddr, r[0]);
#pragma unroll
  for (int c0 = 0; c0 < COLS; c0 += STEP) {
    const int set = c0 / STEP & 1;
    tmem_ld_wait();
    if (c0 + STEP < COLS)
      tmem_ld(taddr + c0 + STEP, r[set ^ 1]);
    else
      drained();
    if (c0 + STEP <= tokens) {
      float4 sc[STEP / 4];
#pragma unroll
      for (int i = 0; i < STEP / 4; ++i) sc[i] = *reinterpret_cast<const float4*>(scale + c0 + 4 * i);
      auto store = [&](int v, float s) {
        *out = from_f32<T>(__fmaf_rn((float)v, __fmul_rn(s, sw), b));
        out += ldo;
      };
#pragma unroll
      for (int i = 0; i < STEP / 4; ++i) {
        store(r[set][4 * i], sc[i].x);
        store(r[set][4 * i + 1], sc[i].y);
        store(r[set][4 * i + 2], sc[i].z);
        store(r[set][4 * i + 3], sc[i].w);
      }
    } else if (c0 < tokens) {
#pragma unroll
      for (int i = 0; i < STEP; ++i) {
        if (c0 + i < tokens) *out = from_f32<T>(__fmaf_rn((float)r[set][i], __fmul_rn(scale[c0 + i], sw), b));
        out += ldo;
      }
    }
  }
}

// ---- one CTA a tile; up to 8 CTAs of a cluster share a tile's K
// Tiles of 64 channels are for SMs that tiles of 128 would leave idle (32 x 4096 x 4096 7.1 -> 6.2 us, 16 x 5120 x 4096 7.5 -> 6.9).
// What few tokens need is operand bytes in flight, as their weights come from memory once: up to 216 KB in the CTAs of an SM.
// The CTAs of a split exchange their int32 sums through distributed shared memory (in place of the rings, once all of them are
// through), each finishing a part of the tokens, so a split changes no result.
constexpr int MAX_STAGES = 21;
constexpr size_t RING_SM = 216 * 1024;   // bytes of rings on an SM
__host__ __device__ constexpr int stage_bytes(int tok, int chn) { return (chn + tok) * BK; }
__host__ __device__ constexpr int blocks_per_sm(int tok) { return tok <= 16 ? 3 : 2; }
template <int TOK, int CHN, typename T>
__global__ void __launch_bounds__(192, blocks_per_sm(TOK))
k_token_linear(const __grid_constant__ CUtensorMap tma_w, const __grid_constant__ CUtensorMap tma_x, const TokenLinearArgs a, const int tiles_n,
               const int split, const int NS) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  int32_t* part = reinterpret_cast<int32_t*>(smem);   // [split][TOK / split / 4][CHN][4] (or 2 for 4), the sums of all CTAs of a split
  constexpr int W_BYTES = CHN * BK, STAGE = W_BYTES + TOK * BK;
  constexpr uint32_t TCOLS = TOK < 32 ? 32 : TOK;
  __shared__ uint64_t full[MAX_STAGES], empty[MAX_STAGES], acc_full;
  __shared__ uint32_t tmem_base_s, failed;
  __shared__ __align__(16) float s_x[TOK];
  const int tid = threadIdx.x, warp = uniform_warp(), lane = tid & 31;
  const int rank = blockIdx.x % split, tile = blockIdx.x / split;
  const int n0 = tile % tiles_n * CHN, m0 = tile / tiles_n * TOK, all = (a.K + BK - 1) / BK;
  const int k0 = all * rank / split, nk = all * (rank + 1) / split - k0;   // (at least one chunk each)
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
  if (warp == 4 && lane == 0) {
    prefetch_tmap(&tma_w);
    prefetch_tmap(&tma_x);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base_s;
  pdl_wait();
  bool ok = true;
  if (warp == 4) {
    const uint32_t on = elect_one();
    int s = 0;
    uint32_t ph = 1;
    for (int i = 0; i < nk && !a.skip_producer; ++i) {
      ok = i < NS || mbar_wait_warp(&empty[s], ph, a.wait_limit);
      if (!ok) {
        ring_landed(full, NS, i);
        break;
      }
      mbar_expect_tx(on, &full[s], STAGE);
      tma_load_2d(on, smem + s * STAGE, &tma_w, (k0 + i) * BK, n0, &full[s]);
      tma_load_2d(on, smem + s * STAGE + W_BYTES, &tma_x, (k0 + i) * BK, m0, &full[s]);
      if (++s == NS) {
        s = 0;
        ph ^= 1;
      }
    }
  } else if (warp == 5) {
    const uint32_t idesc = umma_idesc_i8(CHN, TOK), on = elect_one();
    bool ready = mbar_test(&full[0], 0);
    int s = 0;
    uint32_t ph = 0;
    for (int i = 0; i < nk; ++i) {
      ok = mbar_wait_warp_tested(ready, &full[s], ph, a.wait_limit);
      if (!ok) {
        if (!a.skip_producer) ring_landed(full, NS, nk);
        break;
      }
      tc_fence_after();
      const int st = s;
      if (++s == NS) {
        s = 0;
        ph ^= 1;
      }
      ready = mbar_test(&full[s], ph);
      const uint64_t dw = umma_desc_sw128(smem_u32(smem + st * STAGE)), dx = umma_desc_sw128(smem_u32(smem + st * STAGE + W_BYTES));
#pragma unroll
      for (int kk = 0; kk < BK / 32; ++kk) umma_i8(on, tmem, dw + 2 * kk, dx + 2 * kk, idesc, (i | kk) != 0);
      umma_commit(on, &empty[st]);
    }
    if (!ok) {   // recorded before the epilogue is released, so that it stores nothing
      failed = 1;
      __threadfence_block();
      __syncwarp();
    }
    umma_commit(on, &acc_full);
  } else {
    for (int c = tid; c < TOK; c += 128) s_x[c] = m0 + c < a.M ? __ldg(a.x_scale + m0 + c) : 0.0f;
    asm volatile("bar.sync 1, 128;" ::: "memory");
    ok = mbar_wait(&acc_full, 0, a.wait_limit);
    ok = ok && *reinterpret_cast<volatile uint32_t*>(&failed) == 0;
    tc_fence_after();
  }
  pdl_trigger();
  if (!ok && lane == 0) {
    record_timeout(a.status);
    failed = 1;
  }
  // 64 rows of an accumulator lie in the first 16 lanes of each warp's 32
  const int ch = warp * (CHN / 4) + lane % (CHN / 4), n = n0 + ch;
  const bool mine = (CHN == CH || lane < CHN / 4) && n < a.N;
  __syncwarp();
  if (split > 1) {
    const int log_each = 31 - __clz(TOK / split);
    cluster_arrive();
    cluster_wait();                  // every CTA's products are done (or given up, with its copies landed): its ring may be written to
    const int each = TOK / split;    // tokens that a CTA finishes
    const uint32_t to = smem_u32(part) + (uint32_t)(rank * each * CHN) * 4;
    if (warp < 4) {
#pragma unroll
      for (int c0 = 0; c0 < TOK; c0 += 16) {
        int r[16];
        tmem_ld(tmem + ((uint32_t)(warp * 32) << 16) + c0, r);
        tmem_ld_wait();
        if (!mine) continue;
        if (each >= 4) {
#pragma unroll
          for (int i = 0; i < 16; i += 4)
            st_cluster(cluster_addr_of(to + (uint32_t)(((c0 + i) & (each - 1)) * CHN + 4 * ch) * 4, (c0 + i) >> log_each), r[i], r[i + 1], r[i + 2], r[i + 3]);
        } else {                     // each is 2
#pragma unroll
          for (int i = 0; i < 16; i += 2) st_cluster(cluster_addr_of(to + (uint32_t)(2 * ch) * 4, (c0 + i) >> 1), r[i], r[i + 1]);
        }
      }
      if (!ok)                       // nobody stores anything of this tile
        for (int p = 0; p < split; ++p) st_cluster(cluster_addr(&failed, p), 1);
    }
    __syncwarp();
    cluster_arrive();
    cluster_wait();
    if (warp < 4 && mine && *reinterpret_cast<volatile uint32_t*>(&failed) == 0) {
      const int first = rank * each;
      const float sw = __ldg(a.w_scale + n), b = a.bias ? __ldg(a.bias + n) : 0.0f;
      T* out = static_cast<T*>(a.out) + (long long)(m0 + first) * a.ldo + n;
      auto finish = [&](int c, int sum, float sx) {
        if (m0 + first + c < a.M) out[(long long)c * a.ldo] = from_f32<T>(__fmaf_rn((float)sum, __fmul_rn(sx, sw), b));
      };
      if (each >= 4) {
#pragma unroll 2
        for (int c = 0; c < each; c += 4) {
          int4 sum = make_int4(0, 0, 0, 0);
#pragma unroll 4
          for (int p = 0; p < split; ++p) {
            const int4 v = *reinterpret_cast<const int4*>(part + (p * each + c) * CHN + 4 * ch);
            sum.x += v.x;
            sum.y += v.y;
            sum.z += v.z;
            sum.w += v.w;
          }
          const float4 sx = *reinterpret_cast<const float4*>(s_x + first + c);
          finish(c, sum.x, sx.x);
          finish(c + 1, sum.y, sx.y);
          finish(c + 2, sum.z, sx.z);
          finish(c + 3, sum.w, sx.w);
        }
      } else {
        int2 sum = make_int2(0, 0);
#pragma unroll 8
        for (int p = 0; p < split; ++p) {
          const int2 v = *reinterpret_cast<const int2*>(part + p * 2 * CHN + 2 * ch);
          sum.x += v.x;
          sum.y += v.y;
        }
        finish(0, sum.x, s_x[first]);
        finish(1, sum.y, s_x[first + 1]);
      }
    }
  } else if (warp < 4) {
    const float sw = mine ? __ldg(a.w_scale + n) : 0.0f, b = a.bias && mine ? __ldg(a.bias + n) : 0.0f;
    store_columns<T, TOK>(tmem + ((uint32_t)(warp * 32) << 16), static_cast<T*>(a.out) + (long long)m0 * a.ldo + n, a.ldo, s_x, sw, b,
                          ok && mine ? a.M - m0 : 0, [] {});
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 5) tmem_dealloc(tmem, TCOLS);
}

// ---- two CTAs a tile of 256 channels x 256 or 128 tokens, persistent
// A stage is 128 channels and 128 tokens of 128 codes in each CTA, 32 KB for 2 x 128 x 256 x 128 products: half of what a CTA
// alone would fetch for its 128 x 256 tile, whose operands come out of the L2 slower than the tensor cores take them.
// Tensor memory holds two accumulators of 256 columns: the epilogue stores one while the next tile is summed up.
// Tiles of 128 tokens fetch half as much again for a product, but leave fewer pairs idle
// (300 x 11000 x 8192 29 us, with 256 tokens 43; 512 x 32000 x 14000 220 and 175).
constexpr int PAIR_GROUP = 8;
__host__ __device__ constexpr int pair_stage(int pt) { return (CH + pt / 2) * BK; }
__host__ __device__ constexpr int pair_stages(int pt) { return pt == 256 ? 6 : 8; }
template <int PT, typename T>
__global__ void __launch_bounds__(320, 1)
k_token_linear_pair(const __grid_constant__ CUtensorMap tma_w, const __grid_constant__ CUtensorMap tma_x, const TokenLinearArgs a,
                    const int tiles_n, const int tiles_m) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  constexpr int NS = pair_stages(PT), STAGE = pair_stage(PT);
  __shared__ uint64_t full[NS], empty[NS], acc_full[2], acc_empty[2];   // full and acc_empty: those of rank 0 count
  __shared__ uint32_t tmem_base_s;
  __shared__ __align__(16) float s_x[2][PT];
  const int tid = threadIdx.x, warp = uniform_warp(), lane = tid & 31;
  const uint32_t rank = pair_rank();
  const int pairs = gridDim.x / 2, n_tiles = tiles_n * tiles_m, nk = (a.K + BK - 1) / BK;
  if (tid == 0) {
    for (int s = 0; s < NS; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&acc_full[b], 1);
      mbar_init(&acc_empty[b], 16);   // the epilogue warps of both CTAs
    }
    fence_barrier_init();
    fence_proxy_async();
  }
  if (warp == 9) tmem_alloc_pair(&tmem_base_s, 2 * PT);
  if (warp == 8 && lane == 0) {
    prefetch_tmap(&tma_w);
    prefetch_tmap(&tma_x);
  }
  tc_fence_before();
  __syncthreads();
  cluster_arrive();
  cluster_wait();                    // barriers and tensor memory of both CTAs are there
  tc_fence_after();
  const uint32_t tmem = tmem_base_s;
  pdl_wait();
  // Tiles in columns of 8 channel tiles, so that the pairs at work at one time share their operands' rows in the L2
  auto place = [&](int t, int& n0, int& m0) {
    const int group = t / (PAIR_GROUP * tiles_m), first = group * PAIR_GROUP, wide = min(PAIR_GROUP, tiles_n - first);
    const int at = t - group * PAIR_GROUP * tiles_m;
    n0 = (first + at % wide) * 2 * CH + (int)rank * CH;
    m0 = at / wide * PT;
  };
  bool ok = true;
  if (warp == 8) {
    const uint32_t on = elect_one();
    int s = 0, filled = 0;
    uint32_t ph = 1;
    for (int t = blockIdx.x / 2; t < n_tiles && ok && !a.skip_producer; t += pairs) {
      int n0, m0;
      place(t, n0, m0);
      for (int i = 0; i < nk; ++i) {
        ok = filled < NS || mbar_wait_warp(&empty[s], ph, a.wait_limit);
        if (!ok) break;
        ++filled;
        const uint32_t bar = cluster_addr(&full[s], 0);
        if (rank == 0) mbar_expect_tx(on, &full[s], 2 * STAGE);
        tma_load_2d_pair(on, smem + s * STAGE, &tma_w, i * BK, n0, bar);
        tma_load_2d_pair(on, smem + s * STAGE + CH * BK, &tma_x, i * BK, m0 + (int)rank * (PT / 2), bar);
        if (++s == NS) {
          s = 0;
          ph ^= 1;
        }
      }
    }
    if (ok) {   // the last MMAs' arrivals on this CTA's barriers are in before it can leave
      for (int j = 0; j < min(filled, NS); ++j)
        ok = mbar_wait_warp(&empty[j], (uint32_t)((filled - j + NS - 1) / NS - 1) & 1u, a.wait_limit) && ok;
    } else if (rank == 0) {
      ring_landed(full, NS, filled);
    }
  } else if (warp == 9) {
    if (rank == 0) {
      const uint32_t idesc = umma_idesc_i8(2 * CH, PT), on = elect_one();
      bool ready = mbar_test(&full[0], 0);
      int s = 0, it = 0, used = 0;
      uint32_t ph = 0;
      for (int t = blockIdx.x / 2; t < n_tiles && ok; t += pairs, ++it) {
        const int buf = it & 1, use = it >> 1;
        if (use >= 1) ok = __all_sync(0xffffffffu, mbar_wait_cluster(&acc_empty[buf], (use - 1) & 1, a.wait_limit)) != 0;
        if (!ok) break;
        tc_fence_after();
        const uint32_t d = tmem + (uint32_t)(buf * PT);
        for (int i = 0; i < nk; ++i) {
          ok = mbar_wait_warp_tested(ready, &full[s], ph, a.wait_limit);
          if (!ok) break;
          ++used;
          tc_fence_after();
          const int st = s;
          if (++s == NS) {
            s = 0;
            ph ^= 1;
          }
          ready = mbar_test(&full[s], ph);
          const uint64_t dw = umma_desc_sw128(smem_u32(smem + st * STAGE)), dx = umma_desc_sw128(smem_u32(smem + st * STAGE + CH * BK));
#pragma unroll
          for (int kk = 0; kk < BK / 32; ++kk) umma_i8_pair(on, d, dw + 2 * kk, dx + 2 * kk, idesc, (i | kk) != 0);
          umma_commit_pair(on, &empty[st]);
        }
        if (ok) umma_commit_pair(on, &acc_full[buf]);
      }
      if (!ok && !a.skip_producer) ring_landed(full, NS, used + NS);   // what the producers may have issued
    }
  } else {
    int it = 0;
    for (int t = blockIdx.x / 2; t < n_tiles; t += pairs, ++it) {
      const int buf = it & 1, use = it >> 1;
      int n0, m0;
      place(t, n0, m0);
      const int n = n0 + warp % 4 * 32 + lane, first = warp / 4 * (PT / 2);   // four warps for each half of the tokens
      for (int c = tid; c < PT; c += 256) s_x[buf][c] = m0 + c < a.M ? __ldg(a.x_scale + m0 + c) : 0.0f;
      const float sw = n < a.N ? __ldg(a.w_scale + n) : 0.0f, b = a.bias && n < a.N ? __ldg(a.bias + n) : 0.0f;
      asm volatile("bar.sync 1, 256;" ::: "memory");   // (nobody is still at the tile before the last, which used this buffer)
      ok = ok && __all_sync(0xffffffffu, mbar_wait_cluster(&acc_full[buf], use & 1, a.wait_limit)) != 0;
      if (!ok) continue;                               // stores nothing any more, but meets the others at the barrier
      tc_fence_after();
      const uint32_t taddr = tmem + (uint32_t)(buf * PT + first) + ((uint32_t)(warp % 4 * 32) << 16);
      store_columns<T, PT / 2>(taddr, static_cast<T*>(a.out) + n + (long long)(m0 + first) * a.ldo, a.ldo, s_x[buf] + first, sw, b,
                               n < a.N ? a.M - m0 - first : 0, [&] {   // hand the accumulator back before the last stores
                                 tc_fence_before();
                                 __syncwarp();
                                 if (lane == 0) mbar_arrive_cluster(cluster_addr(&acc_empty[buf], 0));
                               });
    }
  }
  pdl_trigger();
  if (!ok && lane == 0) record_timeout(a.status);
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  cluster_arrive();
  cluster_wait();                    // no CTA leaves, or frees its tensor memory, while the other may still use it
  if (warp == 9) tmem_dealloc_pair(tmem, 2 * PT);
}

template <typename K>
cudaError_t allow_smem(K kernel, size_t bytes, bool* configured_on) {
  bool& configured = configured_on[device_slot()];
  if (configured) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  configured = e == cudaSuccess;
  return e;
}

// Clusters of `size` CTAs with an SM each that run at once: fewer than SMs / size, as a cluster lies inside one group of SMs (here
// 33 of 4 and 15 of 8).  More share SMs, or wait for another to end: 64 x 1024 x 8192, 16 clusters of 8, took 9.7 us
// with whole SMs for rings and 6.4 with halves.
int clusters_at_once(int size) {
  static int known_on[MAX_DEVICES][2];
  int& known = known_on[device_slot()][size == 8];
  if (known == 0) {
    static bool configured_on[MAX_DEVICES];
    cudaLaunchConfig_t c = {};
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = size;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    c.gridDim = dim3(size * sm_count());
    c.blockDim = dim3(192);
    c.dynamicSmemBytes = RING_SM + 1024;
    c.attrs = &at;
    c.numAttrs = 1;
    int n = 0;
    if (allow_smem(k_token_linear<32, CH, float>, RING_SM + 1024, configured_on) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, k_token_linear<32, CH, float>, &c) != cudaSuccess || n <= 0) {
      (void)cudaGetLastError();      // (a guess does as well)
      return sm_count() * 3 / 4 / size;
    }
    known = n;
  }
  return known;
}

// CTAs of an SM: clusters of a split in turn on the SMs that hold one at a time
int ctas_of_sm(long long tiles, int split) {
  const long long at_once = split > 1 ? clusters_at_once(split) : sm_count();
  return (int)((tiles + at_once - 1) / at_once);
}

template <int TOK, int CHN, typename T>
cudaError_t launch_tile(const TokenLinearArgs& a, int split, cudaStream_t s) {
  static bool configured_on[MAX_DEVICES];
  cudaError_t e = allow_smem(k_token_linear<TOK, CHN, T>, RING_SM + 1024, configured_on);
  if (e != cudaSuccess) return e;
  CUtensorMap tw, tx;
  if (!make_tmap_i8(&tw, a.wq, a.K, a.N, a.K, CHN) || !make_tmap_i8(&tx, a.xq, a.K, a.M, a.K, TOK)) return cudaErrorInvalidValue;
  const int tiles_n = (a.N + CHN - 1) / CHN, tiles_m = (a.M + TOK - 1) / TOK;
  // the CTAs of an SM share the room for rings; a ring needs no more stages than its part of K has chunks, but holds the sums of a split
  const long long ctas = (long long)tiles_n * tiles_m * split;
  const int each = ctas_of_sm((long long)tiles_n * tiles_m, split);
  const int on_sm = each < blocks_per_sm(TOK) ? each : blocks_per_sm(TOK), chunks = ((a.K + BK - 1) / BK + split - 1) / split;
  int ns = (int)((RING_SM - 1024 * on_sm) / on_sm / stage_bytes(TOK, CHN));
  ns = ns < chunks ? ns : chunks;
  ns = ns < 4 ? 4 : ns > MAX_STAGES ? MAX_STAGES : ns;
  const size_t bytes = (size_t)ns * stage_bytes(TOK, CHN) + 1024;
  return launch_ex(k_token_linear<TOK, CHN, T>, dim3((unsigned)ctas), dim3(192), bytes, s, true, (unsigned)split, tw, tx, a, tiles_n, split, ns);
}
template <int PT, typename T>
cudaError_t launch_pair(const TokenLinearArgs& a, cudaStream_t s) {
  static bool configured_on[MAX_DEVICES];
  const size_t bytes = (size_t)pair_stages(PT) * pair_stage(PT) + 1024;
  cudaError_t e = allow_smem(k_token_linear_pair<PT, T>, bytes, configured_on);
  if (e != cudaSuccess) return e;
  CUtensorMap tw, tx;
  if (!make_tmap_i8(&tw, a.wq, a.K, a.N, a.K, CH) || !make_tmap_i8(&tx, a.xq, a.K, a.M, a.K, PT / 2)) return cudaErrorInvalidValue;
  const int tiles_n = (a.N + 2 * CH - 1) / (2 * CH), tiles_m = (a.M + PT - 1) / PT;
  const long long tiles = (long long)tiles_n * tiles_m;
  if (tiles > INT32_MAX / 2) return cudaErrorInvalidValue;
  const int pairs = tiles < sm_count() / 2 ? (int)tiles : sm_count() / 2;
  return launch_ex(k_token_linear_pair<PT, T>, dim3((unsigned)(2 * pairs)), dim3(320), bytes, s, true, 2, tw, tx, a, tiles_n, tiles_m);
}

// Time of a launch in us, fitted to all kernels' times at some 600 shapes (1 to 8192 tokens, 512 to 50257 channels, 640 to 14000
// codes); the kernel with the least is taken, of equal ones that with more tokens a tile, which reads weights less often.  At those
// shapes the choice takes 0.4 % longer than the fastest on average.  (Fitted by hand on one B200; another chip wants its own.)
// Examples, us for 32 / 64 tokens a tile / pairs of 128 / of 256:
// 64 x 4096 x 4096 7.8 / 8.3 / - / -, 300 x 5120 x 4096 19 / 13.1 / 10.9 / 15.5, 512 x 11000 x 8192 107 / 71 / 40 / 44.
// A CTA alone: a tile's chunk of 128 codes takes as long as its operands need from the L2 (18 to 24 KB), the CTAs of an SM one after
// the other, their epilogues behind the first, and all bytes at least their time in memory.  A split exchanges sums, 1 to 2.2 us
// for 16 to 64 tokens (16 bytes a store; single words took 1.2 to 3.4), and pays where few tiles have a long K (16 x 1024 x 4096:
// 5.6 -> 3.6, 256 x 1024 x 14000: 18 -> 10.9).
double memory_time(const TokenLinearArgs& a, int bytes) { return ((double)a.N * a.K + (double)a.M * a.K + (double)a.M * a.N * bytes) / 6.2e6; }
double single_cost(const TokenLinearArgs& a, int tok, int chn, int split, int bytes) {
  const double chunk = chn == 128 ? (tok == 16 ? 0.125 : tok == 32 ? 0.13 : 0.183) : (tok == 16 ? 0.11 : tok == 32 ? 0.116 : 0.155);
  const double joined = split == 1 ? 0.0 : tok == 16 ? 1.0 : tok == 32 ? 1.5 : 2.2;
  const int chunks = ((a.K + BK - 1) / BK + split - 1) / split;
  const double each = ctas_of_sm((long long)((a.N + chn - 1) / chn) * ((a.M + tok - 1) / tok), split);
  const double memory = memory_time(a, bytes), sums = each * chunks * chunk + (each - 1.0) * 0.024 * tok;
  return (chn == 128 ? 2.1 : 2.05) + joined + (memory > sums ? memory : sums);
}
// A pair: a chunk for both its CTAs' 256 x 256 or 256 x 128; rounds of tiles behind the first at least their epilogue.
double pair_cost(const TokenLinearArgs& a, int tok, int bytes) {
  const long long tiles = (long long)((a.N + 2 * CH - 1) / (2 * CH)) * ((a.M + tok - 1) / tok), pairs = sm_count() / 2;
  const double chunks = (tok == 256 ? 0.35 : 0.215) * ((a.K + BK - 1) / BK), memory = memory_time(a, bytes), epilogue = 2.1;
  const double sums = chunks + (double)((tiles + pairs - 1) / pairs - 1) * (chunks > epilogue ? chunks : epilogue);
  return (tok == 256 ? 4.8 : 4.55) + (memory > sums ? memory : sums);
}

template <int CHN, typename T>
cudaError_t launch_single(const TokenLinearArgs& a, int tok, int split, cudaStream_t s) {
  return tok == 16   ? launch_tile<16, CHN, T>(a, split, s)
         : tok == 32 ? launch_tile<32, CHN, T>(a, split, s)
                     : launch_tile<64, CHN, T>(a, split, s);
}
template <typename T>
cudaError_t launch_typed(const TokenLinearArgs& a, cudaStream_t s) {
  const int chunks = (a.K + BK - 1) / BK;
  double least = 1e300;
  int tok = 0, chn = CH, split = 1;
  for (int t = 16; t <= 64; t *= 2) {
    if (t == 16 ? a.M > 16 : t / 2 >= a.M) continue;                  // (more tiles of 16 tokens never paid)
    for (int n = 64; n <= CH; n *= 2) {
      const long long tiles = (long long)((a.N + n - 1) / n) * ((a.M + t - 1) / t);
      if (tiles > (n == CH ? INT32_MAX / 2 : sm_count())) continue;   // (tiles of 64 channels: for SMs that would be idle)
      for (int p = 1; p <= 8; p *= p == 1 ? 4 : 2) {                  // two chunks at least for each part
        if (p > 1 && (chunks < 2 * p || ctas_of_sm(tiles, p) > blocks_per_sm(t))) break;
        const double c = single_cost(a, t, n, p, sizeof(T));
        if (c < least || (c == least && t >= tok)) {
          least = c;
          tok = t;
          chn = n;
          split = p;
        }
      }
    }
  }
  for (int t = 128; t <= 256 && a.M > 64; t *= 2) {
    const double c = pair_cost(a, t, sizeof(T));
    if (c <= least) {
      least = c;
      tok = t;
    }
  }
  return tok > 64 || tok == 0 ? (tok == 128 ? launch_pair<128, T>(a, s) : launch_pair<256, T>(a, s))
         : chn == CH          ? launch_single<CH, T>(a, tok, split, s)
                              : launch_single<64, T>(a, tok, split, s);
}

}  // namespace

cudaError_t launch_token_linear(TokenLinearArgs a, int dtype, cudaStream_t s) {
  test_gemm_waits(&a.skip_producer, &a.wait_limit);
  timing_begin(s);
  const cudaError_t e = dtype == Q4_F32   ? launch_typed<float>(a, s)
                        : dtype == Q4_F16 ? launch_typed<__half>(a, s)
                                          : launch_typed<__nv_bfloat16>(a, s);
  timing_end(s);
  ++g_launches;
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace q4
