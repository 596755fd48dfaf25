// Label-synchronous beam search over whole vocabularies: selection of the best W of W x V proposals (q4_lm_beam_select) and
// the move of the beams' states that follows it (q4_beam_reorder).
#include <cuda_bf16.h>
#include <math.h>
#include <string.h>

#include "q4_internal.h"

namespace q4 {

namespace {

constexpr int MAX_BEAMS = 32;

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32(float v) { return v; }
template <> __device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }

// What a row leaves for the merge: its log-sum-exp (NaN: the row proposes nothing) and its W best logits, best first, equal
// ones by label; label -1 behind the last.
struct RowBest {
  double lse;
  float value[MAX_BEAMS];
  int32_t label[MAX_BEAMS];
};

// (value, label) a before b
__device__ __forceinline__ bool before(float va, int la, float vb, int lb) { return va > vb || (va == vb && la < lb); }

template <typename T>
__global__ void __launch_bounds__(256) k_lm_rows(const LmSelectArgs a, RowBest* best) {
  __shared__ double s_sum[8];
  __shared__ float s_val[8];
  __shared__ int s_lab[8];
  const long long row = blockIdx.x;
  const int tid = threadIdx.x;
  const T* z = static_cast<const T*>(a.logits) + row * a.ld;
  RowBest& out = best[row];
  if (!isfinite(a.score[row]) || (a.done && a.done[row])) return;   // the merge does not look at the row
  float top = -INFINITY;
  bool bad = false;
  for (int k = tid; k < a.V; k += 256) {
    const float v = to_f32<T>(z[k]);
    bad = bad || !(v < INFINITY);
    top = fmaxf(top, v);
  }
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if ((tid & 31) == 0) s_val[tid >> 5] = top;
  bad = __syncthreads_or(bad) != 0;
  for (int w = 0; w < 8; ++w) top = fmaxf(top, s_val[w]);
  if (bad || top == -INFINITY) {
    if (tid == 0) out.lse = NAN;
    return;
  }
  double sum = 0.0;
  for (int k = tid; k < a.V; k += 256) sum += exp((double)to_f32<T>(z[k]) - (double)top);
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if ((tid & 31) == 0) s_sum[tid >> 5] = sum;
  __syncthreads();
  if (tid == 0) {
    sum = 0.0;
    for (int w = 0; w < 8; ++w) sum += s_sum[w];
    out.lse = (double)top + log(sum);
  }
  float last_v = INFINITY;
  int last_k = -1;
  for (int i = 0; i < a.W; ++i) {
    float v = -INFINITY;
    int lab = INT32_MAX;
    for (int k = tid; k < a.V; k += 256) {
      const float f = to_f32<T>(z[k]);
      if (f > -INFINITY && before(last_v, last_k, f, k) && before(f, k, v, lab)) {
        v = f;
        lab = k;
      }
    }
    for (int o = 16; o > 0; o >>= 1) {
      const float ov = __shfl_xor_sync(0xffffffffu, v, o);
      const int ol = __shfl_xor_sync(0xffffffffu, lab, o);
      if (before(ov, ol, v, lab)) {
        v = ov;
        lab = ol;
      }
    }
    __syncthreads();
    if ((tid & 31) == 0) {
      s_val[tid >> 5] = v;
      s_lab[tid >> 5] = lab;
    }
    __syncthreads();
    for (int w = 0; w < 8; ++w)
      if (before(s_val[w], s_lab[w], v, lab)) {
        v = s_val[w];
        lab = s_lab[w];
      }
    if (tid == 0) {
      out.value[i] = v;
      out.label[i] = lab == INT32_MAX ? -1 : lab;
    }
    if (lab == INT32_MAX) {
      for (int j = i + 1 + tid; j < a.W; j += 256) out.label[j] = -1;
      break;
    }
    last_v = v;
    last_k = lab;
  }
}

// One warp per utterance: lane w walks down the list of beam w.
__global__ void __launch_bounds__(32) k_lm_merge(const LmSelectArgs a, const RowBest* best) {
  const int b = blockIdx.x, w = threadIdx.x;
  const long long row = (long long)b * a.W + w;
  const bool mine = w < a.W && isfinite(a.score[row]), ended = mine && a.done && a.done[row];
  const RowBest* list = best + row;
  const double score = mine ? (double)a.score[row] : 0.0;
  const bool rows = mine && !ended && !isnan(list->lse);
  int at = 0;
  for (int i = 0; i < a.W; ++i) {
    double c = -INFINITY;
    int lab = -1;
    if (ended && at == 0) {
      c = score;
      lab = a.eos;
    } else if (rows && at < a.W && list->label[at] >= 0) {
      c = score + (((double)list->value[at] - list->lse) + (double)a.rho);
      lab = list->label[at];
      if (!isfinite((float)c)) c = -INFINITY;
    }
    double m = c;
    for (int o = 16; o > 0; o >>= 1) m = fmax(m, __shfl_xor_sync(0xffffffffu, m, o));
    const bool none = m == -INFINITY;
    const int win = __ffs(__ballot_sync(0xffffffffu, c == m)) - 1;
    if (w == win) {
      const long long o = (long long)b * a.W + i;
      a.parent[o] = none ? -1 : w;
      a.token[o] = none ? -1 : lab;
      a.score_out[o] = none ? -INFINITY : (float)c;
      if (a.done_out) a.done_out[o] = !none && lab == a.eos;
      ++at;
    }
  }
}

// Moves of up to Q4_REORDER_MAX tensors, cut into vectors of `width` bytes.
struct MoveItem {
  const uint8_t* src;
  uint8_t* dst;
  long long src_row, dst_row, src_step[2], dst_step[2];
  long long n0, n1, per_row;   // vectors of a row
  int32_t width;
  uint32_t first_block;
};
struct Moves {
  MoveItem item[Q4_REORDER_MAX];
  int32_t n_items, B, W;
  const int32_t* parent;
};
constexpr int MOVE_VECTORS = 1024;   // of a block

template <typename V>
__device__ __forceinline__ void move_vectors(const MoveItem& t, const Moves& a, long long base) {
  const long long total = t.n0 * t.n1 * a.B * a.W * t.per_row;
  for (int i = threadIdx.x; i < MOVE_VECTORS; i += blockDim.x) {
    const long long v = base + i;
    if (v >= total) return;
    const long long r = v / t.per_row, col = v % t.per_row;
    const long long i1 = r % t.n1, bw = (r / t.n1) % ((long long)a.B * a.W), i0 = r / t.n1 / ((long long)a.B * a.W);
    const int p = a.parent[bw];
    if (p < 0 || p >= a.W) continue;
    const long long from = bw / a.W * a.W + p;
    reinterpret_cast<V*>(t.dst + i0 * t.dst_step[0] + i1 * t.dst_step[1] + bw * t.dst_row)[col] =
        reinterpret_cast<const V*>(t.src + i0 * t.src_step[0] + i1 * t.src_step[1] + from * t.src_row)[col];
  }
}

__global__ void __launch_bounds__(256) k_beam_reorder(const __grid_constant__ Moves a) {
  int it = 0;
  while (it + 1 < a.n_items && blockIdx.x >= a.item[it + 1].first_block) ++it;
  const MoveItem& t = a.item[it];
  const long long base = (long long)(blockIdx.x - t.first_block) * MOVE_VECTORS;
  switch (t.width) {
    case 16: move_vectors<uint4>(t, a, base); break;
    case 8: move_vectors<uint2>(t, a, base); break;
    case 4: move_vectors<uint32_t>(t, a, base); break;
    case 2: move_vectors<uint16_t>(t, a, base); break;
    default: move_vectors<uint8_t>(t, a, base);
  }
}

}  // namespace

size_t lm_select_workspace(int B, int W, int V) {
  (void)V;
  return align_up((size_t)B * W * sizeof(RowBest));
}

cudaError_t launch_lm_select(const LmSelectArgs& a, int dtype, cudaStream_t s) {
  RowBest* best = reinterpret_cast<RowBest*>(a.workspace);
  const dim3 rows((unsigned)(a.B * a.W));
  timing_begin(s);
  cudaError_t e = dtype == Q4_F32   ? launch_ex(k_lm_rows<float>, rows, dim3(256), 0, s, false, 1, a, best)
                  : dtype == Q4_F16 ? launch_ex(k_lm_rows<__half>, rows, dim3(256), 0, s, false, 1, a, best)
                                    : launch_ex(k_lm_rows<__nv_bfloat16>, rows, dim3(256), 0, s, false, 1, a, best);
  timing_end(s);
  if (e != cudaSuccess) return e;
  timing_begin(s);
  e = launch_ex(k_lm_merge, dim3((unsigned)a.B), dim3(32), 0, s, false, 1, a, static_cast<const RowBest*>(best));
  timing_end(s);
  g_launches += 2;
  return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t launch_beam_reorder(const q4_reorder* items, int n_items, const int32_t* parent, int B, int W, cudaStream_t s) {
  Moves m;
  memset(&m, 0, sizeof(m));
  m.B = B;
  m.W = W;
  m.parent = parent;
  unsigned long long blocks = 0;
  for (int i = 0; i < n_items; ++i) {
    const q4_reorder& q = items[i];
    if (q.row_bytes == 0 || q.n[0] == 0 || q.n[1] == 0) continue;
    MoveItem& t = m.item[m.n_items++];
    t.src = static_cast<const uint8_t*>(q.src);
    t.dst = static_cast<uint8_t*>(q.dst);
    t.src_row = q.src_row_step;
    t.dst_row = q.dst_row_step;
    t.n0 = q.n[0];
    t.n1 = q.n[1];
    unsigned long long low = reinterpret_cast<uintptr_t>(q.src) | reinterpret_cast<uintptr_t>(q.dst) | (unsigned long long)q.row_bytes;
    if ((long long)B * W > 1) low |= (unsigned long long)(q.src_row_step | q.dst_row_step);
    for (int d = 0; d < 2; ++d) {
      t.src_step[d] = q.src_step[d];
      t.dst_step[d] = q.dst_step[d];
      if (q.n[d] > 1) low |= (unsigned long long)(q.src_step[d] | q.dst_step[d]);
    }
    t.width = low % 16 == 0 ? 16 : low % 8 == 0 ? 8 : low % 4 == 0 ? 4 : low % 2 == 0 ? 2 : 1;
    t.per_row = q.row_bytes / t.width;
    t.first_block = (unsigned)blocks;
    blocks += (unsigned long long)((t.n0 * t.n1 * B * W * t.per_row + MOVE_VECTORS - 1) / MOVE_VECTORS);
    if (blocks > 0x7fffffffull) return cudaErrorInvalidValue;
  }
  if (blocks == 0) return cudaSuccess;
  timing_begin(s);
  const cudaError_t e = launch_ex(k_beam_reorder, dim3((unsigned)blocks), dim3(256), 0, s, false, 1, m);
  timing_end(s);
  ++g_launches;
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace q4
