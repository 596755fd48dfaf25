// Label-synchronous beam search over whole vocabularies: selection of the best W of W x V proposals (q4_lm_beam_select) and
// the move of the beams' states that follows it (q4_beam_reorder).
#include <cuda_bf16.h>
#include <math.h>
#include <string.h>

#include "q4_internal.h"

namespace q4 {

namespace {

constexpr int MAX_BEAMS = 32;

// 2^x on the base-2 unit (ex2.approx: relative error 2^-22), results below 2^-126 are 0: terms of a sum that has a term of 1
__device__ __forceinline__ float exp2_unit(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32(float v) { return v; }
template <> __device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }

constexpr float LOG2E = 1.4426950408889634f;

// A row of logits is cut into `parts` segments.  What a segment leaves for the merge: its maximum and its sum of exponentials
// relative to it (NaN: the row holds a NaN or +inf), and its W best logits above -inf, best first, equal ones by label; label -1
// behind the last.
struct PartSum {
  float top;
  float pad;
  double sum;
};
struct Best {
  float value;
  int32_t label;
};
struct RowParts {
  PartSum* sums;            // [B W, parts]
  Best* best;               // [B W, parts, W]
  int32_t parts;
  int32_t vectors;          // 16-byte vectors of a segment
};

// (value, label) a before b
__device__ __forceinline__ bool before(float va, int la, float vb, int lb) { return va > vb || (va == vb && la < lb); }

template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int N = 4;
  __device__ static __forceinline__ void get(const uint4& r, float (&v)[4]) {
    v[0] = __uint_as_float(r.x);
    v[1] = __uint_as_float(r.y);
    v[2] = __uint_as_float(r.z);
    v[3] = __uint_as_float(r.w);
  }
};
template <> struct Vec<__half> {
  static constexpr int N = 8;
  __device__ static __forceinline__ void get(const uint4& r, float (&v)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      v[2 * i] = f.x;
      v[2 * i + 1] = f.y;
    }
  }
};
template <> struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  __device__ static __forceinline__ void get(const uint4& r, float (&v)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
};
template <typename T> __device__ __forceinline__ uint4 lowest_vector();
template <> __device__ __forceinline__ uint4 lowest_vector<float>() { return make_uint4(0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u); }
template <> __device__ __forceinline__ uint4 lowest_vector<__half>() { return make_uint4(0xFC00FC00u, 0xFC00FC00u, 0xFC00FC00u, 0xFC00FC00u); }
template <> __device__ __forceinline__ uint4 lowest_vector<__nv_bfloat16>() { return make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u); }

constexpr int ROW_NT = 256, ROW_VECTORS = 4, ROW_GROUPS = ROW_NT / 4, ROW_LIST = 512, ROW_STAGES = 3;
constexpr int ROW_TURN = ROW_NT * ROW_VECTORS;                    // 16-byte vectors that a block reads in one turn
constexpr int ROW_RING = ROW_STAGES * ROW_TURN * 16;              // bytes

__device__ __forceinline__ void copy_async16(uint4* dst, const uint4* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void copy_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// One pass over a segment: running maximum and sum of every thread, and the candidates for the segment's W best.
// A bound on those comes from the first turn: the W-th best of the maxima of 64 groups of four threads.  W of its elements are
// no smaller, so of the elements behind it only larger ones count (equal ones come later in the order).  About 20 (W = 16) to
// 45 (W = 32) elements of a turn pass a bound like that; they are ranked at the end.  A list that overflows (equal or rising
// logits) is given up for W passes over the segment.
// Every thread copies the vectors it will read itself into shared memory, two turns ahead: no barrier in the loop, no registers
// for what is on its way, and four blocks of an SM keep 128 KB in flight.
template <typename T>
__global__ void __launch_bounds__(ROW_NT, 4) k_lm_rows(const LmSelectArgs a, const RowParts p) {
  constexpr int N = Vec<T>::N;
  extern __shared__ uint4 s_ring[];
  __shared__ __align__(16) Best s_list[ROW_LIST];
  __shared__ __align__(16) float s_group[ROW_GROUPS];
  __shared__ float s_top[ROW_NT / 32];
  __shared__ double s_sum[ROW_NT / 32];
  __shared__ float s_bound;
  __shared__ int s_n;
  const long long row = blockIdx.x / p.parts;
  const int part = blockIdx.x % p.parts, tid = threadIdx.x, W = a.W;
  pdl_wait();
  pdl_trigger();   // the merge waits for this grid's end before it reads anything
  if (!isfinite(a.score[row]) || (a.done && a.done[row])) return;   // the merge does not look at the row
  const T* z = static_cast<const T*>(a.logits) + row * a.ld;
  // elements in front of the first 16-byte boundary, vectors, and elements behind the last whole vector
  const int head = min((int)(((16 - (reinterpret_cast<uintptr_t>(z) & 15)) & 15) / sizeof(T)), a.V);
  const int n_vec = (a.V - head) / N;
  const uint4* body = reinterpret_cast<const uint4*>(z + head);
  const int v0 = min(part * p.vectors, n_vec), v1 = part + 1 == p.parts ? n_vec : min(v0 + p.vectors, n_vec);
  const int turns = max((v1 - v0 + ROW_TURN - 1) / ROW_TURN, 1);
  auto fetch = [&](int t) {
    if (t < turns) {
      uint4* slot = s_ring + (t % ROW_STAGES) * ROW_TURN + tid;
#pragma unroll
      for (int j = 0; j < ROW_VECTORS; ++j) {
        const int v = v0 + t * ROW_TURN + j * ROW_NT + tid;
        if (v < v1) copy_async16(slot + j * ROW_NT, body + v);
      }
    }
    copy_async_commit();
  };
#pragma unroll
  for (int t = 0; t < ROW_STAGES - 1; ++t) fetch(t);
  const int tail = head + n_vec * N;
  int extra_at = -1;
  if (part == 0 && tid < head) extra_at = tid;
  if (part + 1 == p.parts && tid >= 32 && tid < 32 + a.V - tail) extra_at = tail + tid - 32;
  const float extra = extra_at >= 0 ? to_f32<T>(z[extra_at]) : -INFINITY;
  if (tid == 0) s_n = 0;

  float m = extra != extra ? -INFINITY : extra, bound = 0.0f;
  float sum = extra == -INFINITY ? 0.0f : extra < INFINITY ? 1.0f : NAN;   // a NaN or +inf makes the row's sum NaN
  for (int t = 0; t < turns; ++t) {
    copy_async_wait<ROW_STAGES - 2>();
    const uint4* slot = s_ring + (t % ROW_STAGES) * ROW_TURN + tid;
    const int left = v1 - (v0 + t * ROW_TURN + tid);              // vectors from this thread's first one to the end
    auto vector = [&](int j, float (&x)[N]) { Vec<T>::get(j * ROW_NT < left ? slot[j * ROW_NT] : lowest_vector<T>(), x); };
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < ROW_VECTORS; ++j) {
      float x[N];
      vector(j, x);
#pragma unroll
      for (int i = 0; i < N; ++i) top = fmaxf(top, x[i]);
    }
    fetch(t + ROW_STAGES - 1);
    if (t == 0) {
      float g = fmaxf(top, m);
      g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, 1));
      g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, 2));
      if ((tid & 3) == 0) s_group[tid >> 2] = g;
      __syncthreads();
      if (tid < ROW_GROUPS) {
        const float mine = s_group[tid];
        int rank = 0;
#pragma unroll
        for (int i = 0; i < ROW_GROUPS; i += 4) {
          const float4 o = *reinterpret_cast<const float4*>(s_group + i);
          rank += (o.x > mine || (o.x == mine && i < tid)) + (o.y > mine || (o.y == mine && i + 1 < tid)) +
                  (o.z > mine || (o.z == mine && i + 2 < tid)) + (o.w > mine || (o.w == mine && i + 3 < tid));
        }
        if (rank == W - 1) s_bound = mine;
      }
      __syncthreads();
      bound = s_bound;
      if (extra > -INFINITY && extra >= bound) {
        const int at = atomicAdd(&s_n, 1);
        if (at < ROW_LIST) s_list[at] = Best{extra, extra_at};
      }
    }
    // (elements of the first turn count from the bound on, later ones above it only)
    if (t == 0 ? top >= bound && top > -INFINITY : top > bound) {
#pragma unroll
      for (int j = 0; j < ROW_VECTORS; ++j) {
        float x[N];
        vector(j, x);
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (t == 0 ? x[i] >= bound && x[i] > -INFINITY : x[i] > bound) {
            const int at = atomicAdd(&s_n, 1);
            if (at < ROW_LIST) s_list[at] = Best{x[i], head + (v0 + t * ROW_TURN + j * ROW_NT + tid) * N + i};
          }
      }
    }
    const float next_m = fmaxf(m, top), base = next_m > -INFINITY ? next_m : 0.0f;
    float part_sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < ROW_VECTORS; ++j) {
      float x[N];
      vector(j, x);
#pragma unroll
      for (int i = 0; i < N; ++i) part_sum[i & 1] += exp2_unit((x[i] - base) * LOG2E);
    }
    sum = sum * exp2_unit((m - base) * LOG2E) + (part_sum[0] + part_sum[1]);
    m = next_m;
  }

  float top = m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if ((tid & 31) == 0) s_top[tid >> 5] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < ROW_NT / 32; ++w) top = fmaxf(top, s_top[w]);
  double total = (double)(sum * exp2_unit((m - (top > -INFINITY ? top : 0.0f)) * LOG2E));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  if ((tid & 31) == 0) s_sum[tid >> 5] = total;
  __syncthreads();
  const long long out = row * p.parts + part;
  if (tid == 0) {
    total = 0.0;
#pragma unroll
    for (int w = 0; w < ROW_NT / 32; ++w) total += s_sum[w];
    p.sums[out] = PartSum{top, 0.0f, total};
  }
  Best* best = p.best + out * W;
  const int n = s_n;
  if (n <= ROW_LIST) {
    constexpr int UNROLL = 8;
    const int n_pad = (n + UNROLL - 1) / UNROLL * UNROLL;   // (ROW_LIST is a multiple)
    if (n + tid < n_pad) s_list[n + tid] = Best{-INFINITY, INT32_MAX};
    __syncthreads();
    for (int i = tid; i < max(n, W); i += ROW_NT) {
      if (i >= n) {
        best[i] = Best{-INFINITY, -1};
        continue;
      }
      const Best mine = s_list[i];
      int rank = 0;
      for (int j = 0; j < n_pad; j += UNROLL)
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) rank += before(s_list[j + u].value, s_list[j + u].label, mine.value, mine.label);
      if (rank < W) best[rank] = mine;
    }
    return;
  }
  const int from = part == 0 ? 0 : head + v0 * N, to = part + 1 == p.parts ? a.V : head + v1 * N;
  Best last{INFINITY, -1};
  for (int i = 0; i < W; ++i) {
    Best b{-INFINITY, INT32_MAX};
    for (int k = from + tid; k < to; k += ROW_NT) {
      const float f = to_f32<T>(z[k]);
      if (f > -INFINITY && before(last.value, last.label, f, k) && before(f, k, b.value, b.label)) b = Best{f, k};
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const Best c{__shfl_xor_sync(0xffffffffu, b.value, o), __shfl_xor_sync(0xffffffffu, b.label, o)};
      if (before(c.value, c.label, b.value, b.label)) b = c;
    }
    __syncthreads();
    if ((tid & 31) == 0) s_list[tid >> 5] = b;
    __syncthreads();
    for (int w = 0; w < ROW_NT / 32; ++w)
      if (before(s_list[w].value, s_list[w].label, b.value, b.label)) b = s_list[w];
    if (tid == 0) best[i] = b.label == INT32_MAX ? Best{-INFINITY, -1} : b;   // (overflowed: there are more than W)
    last = b;
  }
}

// One block per utterance.  A proposal's score is score[w] + (z - lse + rho) in double; lse from the segments' sums.
// As in k_lm_rows the W-th best of the maxima of 128 groups (rounded down to fp32, so it errs on the safe side) bounds the W best
// from below, and the proposals that reach it are ranked.  Every entry of the lists has a thread of its own where there are enough: a
// walk down the lists took 20 us in dependent loads.
struct Proposal {
  double c;
  float z;
  int32_t label, beam;
};
__device__ __forceinline__ bool before(const Proposal& a, const Proposal& b) {
  return a.c > b.c || (a.c == b.c && (a.beam < b.beam || (a.beam == b.beam && before(a.z, a.label, b.z, b.label))));
}
constexpr int MERGE_NT = 512, MERGE_GROUPS = 128, MERGE_LIST = 512;

__global__ void __launch_bounds__(MERGE_NT) k_lm_merge(const LmSelectArgs a, const RowParts p) {
  __shared__ double s_score[MAX_BEAMS], s_lse[MAX_BEAMS];   // lse NaN: the beam proposes nothing
  __shared__ int s_ended[MAX_BEAMS];
  __shared__ __align__(16) float s_group[MERGE_GROUPS];
  __shared__ Proposal s_list[MERGE_LIST];
  __shared__ float s_bound;
  __shared__ int s_n;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, W = a.W;
  const long long row0 = (long long)blockIdx.x * W;
  if (tid == 0) s_n = 0;
  pdl_wait();
  // entries of all lists of the utterance, entry ((w parts + i) W + j): place j of segment i of beam w
  const int per_beam = p.parts * W, entries = W * per_beam;
  const Best* all = p.best + row0 * per_beam;
  const Best first = tid < entries ? all[tid] : Best{};     // on its way while the sums are put together
  for (int w = warp; w < W; w += MERGE_NT / 32) {
    const float score = a.score[row0 + w];
    const bool ended = isfinite(score) && a.done && a.done[row0 + w];
    double lse = NAN;
    if (isfinite(score) && !ended) {
      const PartSum* ps = p.sums + (row0 + w) * p.parts;
      PartSum mine = lane < p.parts ? ps[lane] : PartSum{-INFINITY, 0.0f, 0.0};
      float top = mine.top;
      for (int i = lane + 32; i < p.parts; i += 32) top = fmaxf(top, ps[i].top);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      if (top > -INFINITY && top < INFINITY) {
        double sum = mine.sum * (double)exp2_unit((mine.top - top) * LOG2E);
        for (int i = lane + 32; i < p.parts; i += 32) sum += ps[i].sum * (double)exp2_unit((ps[i].top - top) * LOG2E);
        for (int o = 16; o > 0; o >>= 1)
          if (o < p.parts) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        lse = (double)top + log(sum);
      }
    }
    if (lane == 0) {
      s_score[w] = score;
      s_lse[w] = lse;
      s_ended[w] = ended;
    }
  }
  __syncthreads();
  auto proposal = [&](int e, const Best& b) {
    const int w = e / per_beam;
    Proposal q{-INFINITY, -INFINITY, -1, w};
    if (s_ended[w]) {
      if (e == w * per_beam) q.c = s_score[w], q.z = 0.0f, q.label = a.eos;
    } else if (!isnan(s_lse[w]) && b.label >= 0) {
      q.c = s_score[w] + (((double)b.value - s_lse[w]) + (double)a.rho);
      q.z = b.value;
      q.label = b.label;
      if (!isfinite((float)q.c)) q.c = -INFINITY;
    }
    return q;
  };
  Proposal mine{-INFINITY, -INFINITY, -1, 0};
  if (tid < entries) mine = proposal(tid, first);
  float head = __double2float_rd(mine.c);
  for (int e = tid + MERGE_NT; e < entries; e += MERGE_NT) head = fmaxf(head, __double2float_rd(proposal(e, all[e]).c));
#pragma unroll
  for (int o = 1; o < MERGE_NT / MERGE_GROUPS; o <<= 1) head = fmaxf(head, __shfl_xor_sync(0xffffffffu, head, o));
  if (tid % (MERGE_NT / MERGE_GROUPS) == 0) s_group[tid / (MERGE_NT / MERGE_GROUPS)] = head;
  __syncthreads();
  if (tid < MERGE_GROUPS) {
    const float g = s_group[tid];
    int rank = 0;
#pragma unroll
    for (int i = 0; i < MERGE_GROUPS; i += 4) {
      const float4 o = *reinterpret_cast<const float4*>(s_group + i);
      rank += (o.x > g || (o.x == g && i < tid)) + (o.y > g || (o.y == g && i + 1 < tid)) + (o.z > g || (o.z == g && i + 2 < tid)) +
              (o.w > g || (o.w == g && i + 3 < tid));
    }
    if (rank == W - 1) s_bound = g;
  }
  __syncthreads();
  const double bound = s_bound;
  auto offer = [&](const Proposal& q) {
    if (q.c > -INFINITY && q.c >= bound) {
      const int at = atomicAdd(&s_n, 1);
      if (at < MERGE_LIST) s_list[at] = q;
    }
  };
  offer(mine);
  for (int e = tid + MERGE_NT; e < entries; e += MERGE_NT) offer(proposal(e, all[e]));
  __syncthreads();
  const int n = s_n;
  auto store = [&](int i, const Proposal& q, bool some) {
    const long long o = row0 + i;
    a.parent[o] = some ? q.beam : -1;
    a.token[o] = some ? q.label : -1;
    a.score_out[o] = some ? (float)q.c : -INFINITY;
    if (a.done_out) a.done_out[o] = some && q.label == a.eos;
  };
  if (n <= MERGE_LIST) {
    for (int i = tid; i < max(n, W); i += MERGE_NT) {
      if (i >= n) {
        store(i, Proposal{}, false);
        continue;
      }
      const Proposal q = s_list[i];
      int rank = 0;
#pragma unroll 4
      for (int j = 0; j < n; ++j) rank += before(s_list[j], q);
      if (rank < W) store(rank, q, true);
    }
    return;
  }
  // more proposals at the bound than the list holds (equal beams of equal logits): one after the other
  Proposal last{INFINITY, INFINITY, -1, -1};
  for (int i = 0; i < W; ++i) {
    Proposal b{-INFINITY, -INFINITY, INT32_MAX, INT32_MAX};
    for (int e = tid; e < entries; e += MERGE_NT) {
      const Proposal q = proposal(e, all[e]);
      if (q.c > -INFINITY && before(last, q) && before(q, b)) b = q;
    }
    __syncthreads();
    s_list[tid] = b;
    __syncthreads();
    for (int j = 0; j < MERGE_NT; ++j)
      if (before(s_list[j], b)) b = s_list[j];
    if (tid == 0) store(i, b, true);                        // (overflowed: there are more than W)
    last = b;
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

// Segments of a row: at least as many as keep their lists short (8 bounds of 4096 elements, see k_lm_rows), and more while there
// are fewer than 4 blocks per SM and segments of more than one such bound; they are as long as one another.
static RowParts row_parts(int B, int W, int V, int bytes, uint8_t* workspace) {
  const long long rows = (long long)B * W;
  const int per_block = ROW_TURN * (16 / bytes);                  // elements of one turn of a block
  const long long fill = (4LL * sm_count() + rows - 1) / rows;
  long long parts = ((long long)V + per_block - 1) / per_block;
  const long long least = (parts + 7) / 8;
  parts = parts < fill ? parts : fill;
  parts = parts > least ? parts : least;
  RowParts p;
  p.parts = (int)parts;
  const long long vectors = (V * (long long)bytes + 15) / 16;
  p.vectors = (int)((vectors + parts - 1) / parts);
  p.sums = reinterpret_cast<PartSum*>(workspace);
  p.best = reinterpret_cast<Best*>(workspace + align_up((size_t)rows * parts * sizeof(PartSum)));
  return p;
}

size_t lm_select_workspace(int B, int W, int V) {
  size_t n = 0;
  for (int bytes = 2; bytes <= 4; bytes += 2) {
    const size_t parts = (size_t)row_parts(B > 0 ? B : 1, W, V, bytes, nullptr).parts, rows = (size_t)B * W;
    const size_t need = align_up(rows * parts * sizeof(PartSum)) + align_up(rows * parts * W * sizeof(Best));
    n = need > n ? need : n;
  }
  return n;
}

template <typename T>
static cudaError_t launch_rows(const LmSelectArgs& a, const RowParts& p, cudaStream_t s) {
  static bool configured_on[MAX_DEVICES];
  bool& configured = configured_on[device_slot()];
  if (!configured) {
    const cudaError_t e = cudaFuncSetAttribute(k_lm_rows<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, ROW_RING);
    if (e != cudaSuccess) return e;
    configured = true;
  }
  return launch_ex(k_lm_rows<T>, dim3((unsigned)((long long)a.B * a.W * p.parts)), dim3(ROW_NT), ROW_RING, s, true, 1, a, p);
}
cudaError_t launch_lm_select(const LmSelectArgs& a, int dtype, cudaStream_t s) {
  const RowParts p = row_parts(a.B, a.W, a.V, dtype == Q4_F32 ? 4 : 2, a.workspace);
  if ((long long)a.B * a.W * p.parts > 0x7fffffffLL) return cudaErrorInvalidValue;
  timing_begin(s);
  cudaError_t e = dtype == Q4_F32 ? launch_rows<float>(a, p, s) : dtype == Q4_F16 ? launch_rows<__half>(a, p, s) : launch_rows<__nv_bfloat16>(a, p, s);
  timing_end(s);
  if (e != cudaSuccess) return e;
  timing_begin(s);
  e = launch_ex(k_lm_merge, dim3((unsigned)a.B), dim3(MERGE_NT), 0, s, true, 1, a, p);
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
