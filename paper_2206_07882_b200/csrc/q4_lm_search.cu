// Label-synchronous beam search over whole vocabularies: selection of the best W of W x V proposals (q4_lm_beam_select) and
// the move of the beams' states that follows it (q4_beam_reorder).
#include <cuda_bf16.h>
#include <math.h>
#include <string.h>

#include "q4_internal.h"

namespace q4 {

namespace {

constexpr int MAX_BEAMS = 32;

// (a NaN loses against a number)
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
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
constexpr double LOG2E_EXCESS = (double)LOG2E * 0.693147180559945309417232 - 1.0;   // of the rounded constant

// A row of logits is cut into `parts` segments.  What a segment leaves for the merge: its log-sum-exp (-inf: nothing but -inf;
// NaN: a NaN or +inf), and its W best logits above -inf, best first, equal ones by label; label -1 behind the last.
struct Best {
  float value;
  int32_t label;
};
struct RowParts {
  double* lse;              // [B W, parts]
  Best* best;               // [B W, parts, W]
  int32_t parts;
  int32_t vectors;          // 16-byte vectors of a segment
  uint32_t inv_width, inv_parts;   // 2^32 / W rounded up and 2^32 / parts rounded down: entries of a row to segments, segments to places
};

// (value, label) a before b
__device__ __forceinline__ bool before(float va, int la, float vb, int lb) { return va > vb || (va == vb && la < lb); }

__device__ __forceinline__ uint4 load_once(const uint4* p) {   // past the L1: 4 % of a call
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int N = 4;
  __device__ static __forceinline__ void get(const uint4& r, float (&v)[4]) {
    v[0] = __uint_as_float(r.x);
    v[1] = __uint_as_float(r.y);
    v[2] = __uint_as_float(r.z);
    v[3] = __uint_as_float(r.w);
  }
  __device__ static __forceinline__ float top(const uint4& r) {
    return fmaxf(max3(__uint_as_float(r.x), __uint_as_float(r.y), __uint_as_float(r.z)), __uint_as_float(r.w));
  }
};
template <typename T2> __device__ __forceinline__ T2 max_of_pairs(const uint4& r) {   // (a NaN loses here too)
  const T2* p = reinterpret_cast<const T2*>(&r);
  return __hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3]));
}
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
  __device__ static __forceinline__ float top(const uint4& r) {
    const float2 f = __half22float2(max_of_pairs<__half2>(r));
    return fmaxf(f.x, f.y);
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
  __device__ static __forceinline__ float top(const uint4& r) {
    const float2 f = __bfloat1622float2(max_of_pairs<__nv_bfloat162>(r));
    return fmaxf(f.x, f.y);
  }
};
template <typename T> __device__ __forceinline__ uint4 lowest_vector();
template <> __device__ __forceinline__ uint4 lowest_vector<float>() { return make_uint4(0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u); }
template <> __device__ __forceinline__ uint4 lowest_vector<__half>() { return make_uint4(0xFC00FC00u, 0xFC00FC00u, 0xFC00FC00u, 0xFC00FC00u); }
template <> __device__ __forceinline__ uint4 lowest_vector<__nv_bfloat16>() { return make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u); }

constexpr int ROW_NT = 128, ROW_BLOCKS = 7;       // threads of a block, blocks of an SM
constexpr int ROW_VECTORS = 4, ROW_TURNS = 16, ROW_GROUPS = 64;
constexpr int ROW_TURN = ROW_NT * ROW_VECTORS;    // 16-byte vectors that a block reads in one turn
constexpr int ROW_NOTED = 512, ROW_LIST = 1024, MERGE_LIST = MAX_BEAMS * MAX_BEAMS;

// Sums of exponentials are kept as s 2^n, n an integer: a term is 2^(x log2 e - n), one fused multiply-add and the base-2 unit,
// and a change of n is exact.  The rounded constant raises e to 1 + LOG2E_EXCESS, which is taken out again at the maximum.
// n stays within 2^21: logits below that are nothing beside any above, and a segment whose maximum lies outside of +-10^6 is
// summed in another way (`far`).
__device__ __forceinline__ float sum_scale(float m) { return fminf(fmaxf(rintf(m * LOG2E), -2097152.0f), 2097152.0f); }
__device__ __forceinline__ float pow2_down(float d) {   // 2^d, d <= 0 an integer; 0 below 2^-126
  return __int_as_float((int)(fmaxf(d, -127.0f) + 127.0f) << 23);
}

// A proposal's score in double as an integer of the same order (comparisons of doubles take several times as long), and what
// decides between equal ones.
struct Proposal {
  long long key;
  float z;
  int32_t label, beam;
};
constexpr long long NO_PROPOSAL = (long long)0x800fffffffffffffULL;   // the key of -inf
__device__ __forceinline__ long long order_key(double c) {
  const long long b = __double_as_longlong(c + 0.0);       // (-0 becomes 0)
  return b >= 0 ? b : b ^ 0x7fffffffffffffffLL;
}
// the keys of -+(2 - 2^-24) 2^127: scores between them are finite in fp32
constexpr long long LOWEST_SCORE = (long long)0xB81000000FFFFFFFULL, HIGHEST_SCORE = 0x47EFFFFFF0000000LL;
__device__ __forceinline__ double key_score(long long k) { return __longlong_as_double(k >= 0 ? k : k ^ 0x7fffffffffffffffLL); }
__device__ __forceinline__ bool before(const Proposal& a, const Proposal& b) {
  return a.key > b.key || (a.key == b.key && (a.beam < b.beam || (a.beam == b.beam && before(a.z, a.label, b.z, b.label))));
}

struct RowShared {            // of a segment
  uint4 vector[ROW_NOTED];    // noted vectors of logits, and their numbers
  int32_t number[ROW_NOTED];
  float value[ROW_LIST];      // candidates
  int32_t label[ROW_LIST];
};
struct MergeShared {
  double base[MAX_BEAMS], lse[MAX_BEAMS];   // score + rho and log-sum-exp of a beam's row; an ended beam's score
  int32_t kind[MAX_BEAMS];                  // 0: the beam proposes nothing, 1: labels, 2: it has ended
  uint32_t like[MAX_BEAMS], any_like;       // earlier beams whose rows may be equal; beams that have any
  long long key[MERGE_LIST];
  float z[MERGE_LIST];
  int32_t label[MERGE_LIST], beam[MERGE_LIST], pick[MERGE_LIST];
};
struct SelectShared {
  union {
    RowShared row;
    MergeShared merge;
  };
  Best best[ROW_NT / 32];
  double sum[ROW_NT / 32];
  float group[ROW_GROUPS], top[ROW_NT / 32], scale[ROW_NT / 32], bound[2];
  int32_t noted, n, picked, last;
};
static_assert(sizeof(SelectShared) * ROW_BLOCKS <= 200 * 1024, "shared memory of an SM");

// The W-th largest of the block's ROW_GROUPS group maxima, at least (W of the elements are no smaller): every thread of the first
// two warps counts what is larger than its own, and the smallest of those with fewer than W larger ones is taken.
__device__ __forceinline__ float group_bound(SelectShared& sh, float mine, int W) {
  constexpr int EACH = ROW_NT / ROW_GROUPS;
  static_assert(ROW_GROUPS == 64 && EACH >= 1 && EACH <= 32, "two warps count, groups lie within a warp");
#pragma unroll
  for (int o = 1; o < EACH; o <<= 1) mine = fmaxf(mine, __shfl_xor_sync(0xffffffffu, mine, o));
  const int tid = threadIdx.x;
  if (tid % EACH == 0) sh.group[tid / EACH] = mine;
  __syncthreads();
  if (tid < ROW_GROUPS) {
    mine = sh.group[tid];
    int larger = 0;
#pragma unroll
    for (int i = 0; i < ROW_GROUPS; i += 4) {
      const float4 o = *reinterpret_cast<const float4*>(sh.group + i);
      larger += (o.x > mine) + (o.y > mine) + (o.z > mine) + (o.w > mine);
    }
    float low = larger < W ? mine : INFINITY;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) low = fminf(low, __shfl_xor_sync(0xffffffffu, low, o));
    if ((tid & 31) == 0) sh.bound[tid >> 5] = low;
  }
  __syncthreads();
  return fminf(sh.bound[0], sh.bound[1]);
}

// The candidates of sh.row that reach `bound`, all of them offered before, as the list `best` of the W best; false if there are more
// than the list holds.
__device__ __forceinline__ void offer_candidate(SelectShared& sh, float bound, float v, int label) {
  if (v >= bound && v > -INFINITY) {
    const int at = atomicAdd(&sh.n, 1);
    if (at < ROW_LIST) {
      sh.row.value[at] = v;
      sh.row.label[at] = label;
    }
  }
}
__device__ __forceinline__ bool rank_candidates(const SelectShared& sh, int n, int W, Best* best) {
  if (n > ROW_LIST) return false;
  for (int i = threadIdx.x; i < max(n, W); i += ROW_NT) {
    if (i >= n) {
      best[i] = Best{-INFINITY, -1};
      continue;
    }
    const float mine = sh.row.value[i];
    const int label = sh.row.label[i];
    int rank = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) rank += before(sh.row.value[j], sh.row.label[j], mine, label);
    if (rank < W) best[rank] = Best{mine, label};
  }
  return true;
}
// The same by W passes over get(from) .. get(to - 1) (counted without a sign: the step behind the last of nearly 2^31 passes that)
template <typename F>
__device__ __forceinline__ void best_by_passes(SelectShared& sh, F get, uint32_t from, uint32_t to, int W, Best* best) {
  const int tid = threadIdx.x;
  Best last{INFINITY, -1};
  for (int i = 0; i < W; ++i) {
    Best b{-INFINITY, INT32_MAX};
    for (uint32_t k = from + tid; k < to; k += ROW_NT) {
      const Best c = get(k);
      if (c.value > -INFINITY && before(last.value, last.label, c.value, c.label) && before(c.value, c.label, b.value, b.label)) b = c;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const Best c{__shfl_xor_sync(0xffffffffu, b.value, o), __shfl_xor_sync(0xffffffffu, b.label, o)};
      if (before(c.value, c.label, b.value, b.label)) b = c;
    }
    __syncthreads();
    if ((tid & 31) == 0) sh.best[tid >> 5] = b;
    __syncthreads();
    for (int w = 0; w < ROW_NT / 32; ++w)
      if (before(sh.best[w].value, sh.best[w].label, b.value, b.label)) b = sh.best[w];
    if (tid == 0) best[i] = b.label == INT32_MAX ? Best{-INFINITY, -1} : b;
    last = b;
  }
}

// One pass over a segment of at most 16 turns: running maximum and sum of every thread, and the segment's candidates.
// The W-th best of the running maxima of 64 groups of threads (group_bound), taken in turns 1, 2, 4, 8 and 16, bounds the
// segment's W best from below.  Vectors with an element above it are noted: of the turn that it was taken in also those that
// reach it, W of which are no smaller; behind that turn only larger ones, as equal ones come later in the order.  About 18 (W = 16) to
// 45 (W = 32) elements pass between two bounds.  The noted vectors' elements that reach the last bound are ranked.  More than the
// lists take (equal or rising logits) are given up for W passes over the segment.
// The next turn's vectors are on their way into registers while a turn is worked on: 56 KB in the seven blocks of an SM.
// Bound by memory: 64 x 16 rows of 32000 fp32 logits, 131 MB, take 28 us with a fifth of the beams ended; a kernel that only
// reads 134 MB in blocks like these takes 25 us, in the best of blocks 23.  Tried at 64 x 16 x 32768: candidates read again once the last
// bound was known 14 us more, one bound of the first turn 9 us more, two turns ahead by asynchronous copies to shared memory no
// gain, five blocks with twice the vectors 6 us more (two waves of blocks).
template <typename T>
__device__ __forceinline__ void best_of_segment(const LmSelectArgs& a, const RowParts& p, long long row, int part, SelectShared& sh) {
  constexpr int N = Vec<T>::N;
  RowShared& list = sh.row;
  const int tid = threadIdx.x, W = a.W;
  const T* z = static_cast<const T*>(a.logits) + row * a.ld;
  // elements in front of the first 16-byte boundary, vectors, and elements behind the last whole vector
  const int head = min((int)(((16 - (reinterpret_cast<uintptr_t>(z) & 15)) & 15) / sizeof(T)), a.V);
  const int n_vec = (a.V - head) / N;
  const int v0 = min(part * p.vectors, n_vec), v1 = part + 1 == p.parts ? n_vec : min(v0 + p.vectors, n_vec);
  const int turns = (v1 - v0 + ROW_TURN - 1) / ROW_TURN;
  const uint4* src = reinterpret_cast<const uint4*>(z + head) + v0 + tid;
  int left = v1 - v0 - tid;                        // vectors from src on
  auto fetch = [&](uint4 (&raw)[ROW_VECTORS]) {
    if (left > (ROW_VECTORS - 1) * ROW_NT) {
#pragma unroll
      for (int j = 0; j < ROW_VECTORS; ++j) raw[j] = load_once(src + j * ROW_NT);
    } else {
#pragma unroll
      for (int j = 0; j < ROW_VECTORS; ++j) raw[j] = j * ROW_NT < left ? load_once(src + j * ROW_NT) : lowest_vector<T>();
    }
    src += ROW_TURN;
    left -= ROW_TURN;
  };
  uint4 raw_a[ROW_VECTORS], raw_b[ROW_VECTORS];
  fetch(raw_a);
  const int tail = head + n_vec * N;
  const float first = part == 0 && tid < head ? to_f32<T>(z[tid]) : -INFINITY;
  const float last = part + 1 == p.parts && tid < a.V - tail ? to_f32<T>(z[tail + tid]) : -INFINITY;
  if (tid == 0) sh.n = sh.noted = 0;

  float m = first != first ? -INFINITY : first, scale = sum_scale(m), bound = -INFINITY, limit = -INFINITY;
  // A turn's 16 or 32 terms are added in fp32, four chains of them, turns in double: 10 roundings of 2^-24 at most, where fp32 alone
  // would add one a turn.  (A NaN makes the sum NaN.)
  double sum = exp2_unit(__fmaf_rn(first, LOG2E, -scale));
  auto turn = [&](const uint4 (&raw)[ROW_VECTORS], int t) {
    float vector_top[ROW_VECTORS], top = -INFINITY;
#pragma unroll
    for (int j = 0; j < ROW_VECTORS; ++j) vector_top[j] = Vec<T>::top(raw[j]);
#pragma unroll
    for (int j = 0; j < ROW_VECTORS; j += 2) top = max3(top, vector_top[j], vector_top[j + 1]);
    m = fmaxf(m, top);
    if ((t & (t + 1)) == 0) {
      bound = group_bound(sh, m, W);
      limit = nextafterf(bound, -INFINITY);
    }
    if (top > limit) {
#pragma unroll
      for (int j = 0; j < ROW_VECTORS; ++j)
        if (vector_top[j] > limit) {
          const int at = atomicAdd(&sh.noted, 1);
          if (at < ROW_NOTED) {
            list.vector[at] = raw[j];
            list.number[at] = v0 + t * ROW_TURN + j * ROW_NT + tid;
          }
        }
    }
    limit = bound;
    const float now = sum_scale(m);
    const uint64_t mul = pk2(LOG2E, LOG2E), sub = pk2(-now, -now);
    uint64_t part_sum[2] = {pk2(0.0f, 0.0f), pk2(0.0f, 0.0f)};
#pragma unroll
    for (int j = 0; j < ROW_VECTORS; ++j) {
      float x[N];
      Vec<T>::get(raw[j], x);
#pragma unroll
      for (int i = 0; i < N; i += 2) {
        float e0, e1;
        upk2(fma2(pk2(x[i], x[i + 1]), mul, sub), e0, e1);
        part_sum[(i >> 1) & 1] = add2(part_sum[(i >> 1) & 1], pk2(exp2_unit(e0), exp2_unit(e1)));
      }
    }
    float even, odd;
    upk2(add2(part_sum[0], part_sum[1]), even, odd);
    sum = fma(sum, (double)pow2_down(scale - now), (double)(even + odd));
    scale = now;
  };
  for (int t = 0; t < turns; t += 2) {   // two sets of registers: one on its way, one worked on
    fetch(raw_b);
    turn(raw_a, t);
    if (t + 1 == turns) break;
    fetch(raw_a);
    turn(raw_b, t + 1);
  }
  m = fmaxf(m, last);
  const float now = sum_scale(m);
  sum = fma(sum, (double)pow2_down(scale - now), (double)exp2_unit(__fmaf_rn(last, LOG2E, -now)));
  scale = now;

  // candidates: elements that reach the last bound (without turns there is none)
  __syncthreads();
  const int noted = sh.noted;
  offer_candidate(sh, bound, first, tid);
  offer_candidate(sh, bound, last, tail + tid);
  for (int i = tid; i < min(noted, ROW_NOTED); i += ROW_NT) {
    float x[N];
    Vec<T>::get(list.vector[i], x);
    const int label = head + list.number[i] * N;
#pragma unroll
    for (int j = 0; j < N; ++j) offer_candidate(sh, bound, x[j], label + j);
  }
  // the segment's log-sum-exp
  float top = m, most = scale;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
  }
  if ((tid & 31) == 0) {
    sh.top[tid >> 5] = top;
    sh.scale[tid >> 5] = most;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < ROW_NT / 32; ++w) {
    top = fmaxf(top, sh.top[w]);
    most = fmaxf(most, sh.scale[w]);
  }
  const bool far = top > -INFINITY && fabsf(top) > 1e6f;
  double total = sum * (double)pow2_down(scale - most);
  const uint32_t from = part == 0 ? 0 : head + v0 * N, to = part + 1 == p.parts ? a.V : head + v1 * N;
  if (far) {   // differences from the maximum, which are exact where they count
    total = 0.0;
    for (uint32_t k = from + tid; k < to; k += ROW_NT) total += (double)exp2_unit((to_f32<T>(z[k]) - top) * LOG2E);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  if ((tid & 31) == 0) sh.sum[tid >> 5] = total;
  const int n = sh.n;
  __syncthreads();
  const long long out = row * p.parts + part;
  if (tid == ROW_NT - 1) {   // (a warp that has nothing to rank, mostly)
    total = 0.0;
#pragma unroll
    for (int w = 0; w < ROW_NT / 32; ++w) total += sh.sum[w];
    const double excess = far ? 0.0 : LOG2E_EXCESS * (double)top, base = far ? (double)top : (double)most * 0.693147180559945309417232;
    p.lse[out] = top == -INFINITY ? (total == 0.0 ? -INFINITY : NAN) : base + log(total) - excess;
  }
  Best* best = p.best + out * W;
  if (noted > ROW_NOTED || !rank_candidates(sh, n, W, best))
    best_by_passes(sh, [&](uint32_t k) { return Best{to_f32<T>(z[k]), (int32_t)k}; }, from, to, W, best);
}

// A row's segments put together in the place of the first one: the sum of their shares of the log-sum-exp, and the W best of their
// lists, by a bound from group maxima as in a segment.  What other blocks wrote is read past the L1.
__device__ __forceinline__ Best load_best(const Best* p) {
  const int2 v = __ldcg(reinterpret_cast<const int2*>(p));
  return Best{__int_as_float(v.x), v.y};
}
__device__ __forceinline__ void merge_row(const RowParts& p, long long row, int W, SelectShared& sh) {
  const int tid = threadIdx.x, entries = p.parts * W;
  Best* best = p.best + row * entries;
  double* parts = p.lse + row * p.parts;
  // Lists begin with their best: each is read from another place on, so that the threads of a group meet early and late ones.  (Read
  // all from their first ones, the low places' groups give a bound below most entries: 32 x 128256 fp32 37 us, so 21.)
  auto entry = [&](int e) {
    const int list = W > 1 ? (int)__umulhi(e, p.inv_width) : e, at = e - list * W + (int)__umulhi(list * W, p.inv_parts);
    return load_best(best + list * W + (at < W ? at : at - W));
  };
  constexpr int EACH = 4;
  Best mine[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) mine[i] = tid + i * ROW_NT < entries ? entry(tid + i * ROW_NT) : Best{-INFINITY, -1};
  if (tid == 0) sh.n = 0;
  float head = -INFINITY;
#pragma unroll
  for (int i = 0; i < EACH; ++i) head = fmaxf(head, mine[i].value);
#pragma unroll 4
  for (int e = tid + EACH * ROW_NT; e < entries; e += ROW_NT) head = fmaxf(head, entry(e).value);
  const float bound = group_bound(sh, head, W);
#pragma unroll
  for (int i = 0; i < EACH; ++i) offer_candidate(sh, bound, mine[i].value, mine[i].label);
#pragma unroll 4
  for (int e = tid + EACH * ROW_NT; e < entries; e += ROW_NT) {
    const Best b = entry(e);
    offer_candidate(sh, bound, b.value, b.label);
  }
  if (tid < 32) {
    double top = -INFINITY, sum = 0.0;
    bool bad = false;
    for (int j = tid; j < p.parts; j += 32) {
      const double v = __ldcg(parts + j);
      top = fmax(top, v);
      bad = bad || isnan(v);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmax(top, __shfl_xor_sync(0xffffffffu, top, o));
    for (int j = tid; j < p.parts; j += 32) sum += (double)exp2_unit((float)(__ldcg(parts + j) - top) * LOG2E);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    bad = __any_sync(0xffffffffu, bad);
    if (tid == 0) parts[0] = bad ? NAN : top + log(sum);
  }
  __syncthreads();                             // (all entries have been read, but for the passes below)
  if (!rank_candidates(sh, sh.n, W, best)) {
    // many equal ones: best of passes into shared memory first, as it takes the place of what the passes read
    __syncthreads();
    Best* found = reinterpret_cast<Best*>(sh.row.value);
    best_by_passes(sh, [&](uint32_t k) { return load_best(best + k); }, 0, entries, W, found);
    __syncthreads();
    if (tid < W) best[tid] = found[tid];
  }
}

// How far sums of equal rows may lie apart: each is off by less than 5e-6 (terms by 2^-22 and by what rounds their arguments, 10
// roundings of 2^-24, the same again where segments are joined)
constexpr double SAME_SUM = 1e-5;

// Whether two rows hold the same values, by the whole block.  Only beams that are all but certainly alike come here: 15 us for 50257 labels
// (1 x 32 x 50257 fp32 with all beams alike 400 us, with none 22).  More loads under way at a time cost registers that every row would miss.
template <typename T>
__device__ __forceinline__ bool same_rows(const T* x, const T* y, int V) {
  constexpr int EACH = 8;
  bool same = true;
  for (int left = V - (int)threadIdx.x; left > 0 && same; left -= left > ROW_NT * EACH ? ROW_NT * EACH : left) {
    const T *xs = x + (V - left), *ys = y + (V - left);
    T u[EACH], v[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      u[i] = i * ROW_NT < left ? xs[i * ROW_NT] : T(0.0f);
      v[i] = i * ROW_NT < left ? ys[i * ROW_NT] : T(0.0f);
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) same = to_f32<T>(u[i]) == to_f32<T>(v[i]) && same;
  }
  return __syncthreads_and(same) != 0;
}

// The W best proposals of an utterance from its rows' lists.  A proposal's score is score[w] + rho + (z - lse) in double (the logits may
// be far larger than their differences).  As for a segment a bound from group maxima (rounded down to fp32, so it errs on
// the safe side) leaves few proposals to rank; where the best are in few groups (beams far apart, or many beams alike) it leaves
// hundreds, and a second bound is taken among those.
// Double precision is slow to wait for: two additions and two conversions an entry, everything else is done on the keys.
template <typename T>
__device__ __forceinline__ void merge_rows(const LmSelectArgs& a, const RowParts& p, int utterance, SelectShared& sh) {
  MergeShared& mg = sh.merge;
  const int tid = threadIdx.x, W = a.W, entries = W * W;   // entry w W + j: place j of beam w
  const long long row0 = (long long)utterance * W;
  const int over = 65536 / W + 1;                          // e / W = e over >> 16 for e < 1024
  constexpr int EACH = MERGE_LIST / ROW_NT;
  Best mine[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int e = tid + i * ROW_NT, w = e * over >> 16;
    mine[i] = e < entries ? load_best(p.best + (row0 + w) * p.parts * W + (e - w * W)) : Best{-INFINITY, -1};
  }
  if (tid < 32) {
    const float score = tid < W ? a.score[row0 + tid] : -INFINITY;
    const bool ended = tid < W && a.done && a.done[row0 + tid] && isfinite(score);
    const double lse = tid < W ? __ldcg(p.lse + (row0 + tid) * p.parts) : NAN;   // (a beam that is empty or ended left none: not used)
    const bool rows = isfinite(score) && !ended && isfinite(lse);           // (not finite: nothing but -inf, a NaN or +inf)
    // Beams of equal scores and equal rows have equal proposals, but rows that begin at different places of 16 bytes are summed in
    // another order.  Such a beam takes the sum of the first one like it.  Asked for here: same score, another place of 16 bytes, and a
    // sum that differs, by no more than that makes it; the rows themselves are compared below.
    uint32_t alike = __match_any_sync(0xffffffffu, rows ? __float_as_uint(score + 0.0f) : 0x7fc00000u | tid) & ((1u << tid) - 1), like = 0;
    const uint32_t place = (uint32_t)(((row0 + tid) * a.ld * (long long)sizeof(T)) & 15);
    while (__any_sync(0xffffffffu, alike != 0)) {
      const int w = alike ? __ffs(alike) - 1 : tid;
      const double other = __shfl_sync(0xffffffffu, lse, w);
      const uint32_t other_place = __shfl_sync(0xffffffffu, place, w);
      if (alike == 0) continue;
      alike &= alike - 1;
      if (place != other_place && lse != other && fabs(lse - other) <= SAME_SUM) like |= 1u << w;
    }
    if (tid < W) {
      mg.base[tid] = ended ? (double)score : (double)score + (double)a.rho;
      mg.lse[tid] = lse;
      mg.kind[tid] = ended ? 2 : rows ? 1 : 0;
      mg.like[tid] = like;
    }
    like = __ballot_sync(0xffffffffu, like != 0);
    if (tid == 0) mg.any_like = like;
  }
  if (tid == 0) sh.n = sh.picked = 0;
  __syncthreads();
  for (uint32_t left = mg.any_like; left; left &= left - 1) {   // seldom any
    const int w = __ffs(left) - 1;
    const T* z = static_cast<const T*>(a.logits) + row0 * a.ld;
    for (uint32_t like = mg.like[w]; like; like &= like - 1) {
      const int v = __ffs(like) - 1;
      if (!same_rows(z + w * a.ld, z + v * a.ld, a.V)) continue;
      if (tid == 0) mg.lse[w] = mg.lse[v];
      break;
    }
    __syncthreads();
  }
  long long key[EACH], head = NO_PROPOSAL;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int e = tid + i * ROW_NT, w = e * over >> 16;
    key[i] = NO_PROPOSAL;
    if (e >= entries) continue;
    const int kind = mg.kind[w];
    if (kind == 1 && mine[i].label >= 0) {
      const long long k = order_key(mg.base[w] + ((double)mine[i].value - mg.lse[w]));
      if (k > LOWEST_SCORE && k < HIGHEST_SCORE) key[i] = k;
    } else if (kind == 2 && e == w * W) {
      key[i] = order_key(mg.base[w]);
      mine[i] = Best{0.0f, a.eos};
    }
    head = max(head, key[i]);
  }
  long long bound = order_key((double)group_bound(sh, __double2float_rd(key_score(head)), W));
#pragma unroll
  for (int i = 0; i < EACH; ++i)
    if (key[i] > NO_PROPOSAL && key[i] >= bound) {
      const int at = atomicAdd(&sh.n, 1);
      mg.key[at] = key[i];
      mg.z[at] = mine[i].value;
      mg.label[at] = mine[i].label;
      mg.beam[at] = (tid + i * ROW_NT) * over >> 16;
    }
  __syncthreads();
  int n = sh.n;
  const bool many = n > ROW_NT;
  if (many) {
    head = NO_PROPOSAL;
    for (int i = tid; i < n; i += ROW_NT) head = max(head, mg.key[i]);
    bound = order_key((double)group_bound(sh, __double2float_rd(key_score(head)), W));
    for (int i = tid; i < n; i += ROW_NT)
      if (mg.key[i] >= bound) mg.pick[atomicAdd(&sh.picked, 1)] = i;
    __syncthreads();
    n = sh.picked;
  }
  auto store = [&](int i, const Proposal& q, bool some) {
    const long long o = row0 + i;
    a.parent[o] = some ? q.beam : -1;
    a.token[o] = some ? q.label : -1;
    a.score_out[o] = some ? (float)key_score(q.key) : -INFINITY;
    if (a.done_out) a.done_out[o] = some && q.label == a.eos;
  };
  auto place = [&](int i) { return many ? mg.pick[i] : i; };
  auto listed = [&](int i) { return Proposal{mg.key[i], mg.z[i], mg.label[i], mg.beam[i]}; };
  for (int i = tid; i < max(n, W); i += ROW_NT) {
    if (i >= n) {
      store(i, Proposal{}, false);
      continue;
    }
    const Proposal q = listed(place(i));
    int rank = 0, equal = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) {
      const long long k = mg.key[place(j)];
      rank += k > q.key;
      equal += k == q.key;
    }
    if (rank < W && equal > 1)
      for (int j = 0; j < n; ++j) rank += mg.key[place(j)] == q.key && before(listed(place(j)), q);
    if (rank < W) store(rank, q, true);
  }
}

// One block per segment; the last of a row's blocks to be through merges the row, the last of an utterance's rows the utterance.
// A block that arrives publishes what its threads wrote (a barrier, then a releasing count), the last one reads the others' after
// the count, which acquires, past the L1.  The counts wrap to 0 for the next call.
__device__ __forceinline__ bool last_to_arrive(uint32_t* count, uint32_t of, SelectShared& sh) {
  __syncthreads();
  if (threadIdx.x == 0) {
    uint32_t before;
    asm volatile("atom.acq_rel.gpu.global.inc.u32 %0, [%1], %2;" : "=r"(before) : "l"(count), "r"(of - 1) : "memory");
    sh.last = before == of - 1;
  }
  __syncthreads();
  return sh.last != 0;
}
template <typename T>
__global__ void __launch_bounds__(ROW_NT, ROW_BLOCKS) k_lm_select(const LmSelectArgs a, const RowParts p) {
  __shared__ __align__(16) SelectShared sh;
  const long long row = blockIdx.x / p.parts;
  const int part = blockIdx.x % p.parts, utterance = (int)(row / a.W);
  pdl_wait();
  pdl_trigger();   // (nothing of a later kernel starts to read or write before this grid has ended)
  const bool live = isfinite(a.score[row]) && !(a.done && a.done[row]);
  if (live) best_of_segment<T>(a, p, row, part, sh);
  if (p.parts > 1) {
    if (!last_to_arrive(a.arrived + a.B + row, p.parts, sh)) return;
    if (live) merge_row(p, row, a.W, sh);
  }
  if (last_to_arrive(a.arrived + utterance, a.W, sh)) merge_rows<T>(a, p, utterance, sh);
}

// Moves of up to Q4_REORDER_MAX tensors, rows cut into vectors of `width` bytes.  A block takes a piece of one long row or some
// short rows; where its rows lie is worked out once a row and kept in shared memory, so that a vector costs one 32-bit multiplication
// beside its load and store.
struct MoveItem {
  const uint8_t* src;
  uint8_t* dst;
  long long src_row, dst_row, src_step[2], dst_step[2];
  long long rows, n1, per_row;    // rows of all steps; vectors of a row
  long long piece;                // vectors of a row that a block takes
  int32_t width;
  int32_t block_rows;             // rows of a block; more than one: whole rows
  uint32_t pieces;                // blocks of a row
  uint32_t over;                  // 2^32 / per_row, rounded up, for blocks of several rows
  uint32_t first_block;
};
struct Moves {
  MoveItem item[Q4_REORDER_MAX];
  int32_t n_items, B, W;
  const int32_t* parent;
};
constexpr int MOVE_NT = 256, MOVE_EACH = 8, MOVE_ROWS = 256;   // vectors of a thread, most rows of a block
constexpr int MOVE_VECTORS = MOVE_NT * MOVE_EACH;

template <typename V>
__device__ __forceinline__ void move_vectors(const MoveItem& t, const uint8_t* const* from, uint8_t* const* to, long long first, int n) {
#pragma unroll 1
  for (int i0 = threadIdx.x; i0 < n; i0 += MOVE_NT * 4) {
    V v[4];
    V* at[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {   // loads of four vectors, then their stores
      const int i = i0 + j * MOVE_NT;
      at[j] = nullptr;
      if (i >= n) continue;
      const int r = t.block_rows == 1 ? 0 : t.per_row == 1 ? i : (int)__umulhi((uint32_t)i, t.over);
      const long long col = t.block_rows > 1 ? i - r * (int)t.per_row : first + i;
      if (to[r] == nullptr) continue;
      v[j] = __ldg(reinterpret_cast<const V*>(from[r]) + col);
      at[j] = reinterpret_cast<V*>(to[r]) + col;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (at[j]) *at[j] = v[j];
  }
}

__global__ void __launch_bounds__(MOVE_NT) k_beam_reorder(const __grid_constant__ Moves a) {
  __shared__ const uint8_t* s_from[MOVE_ROWS];
  __shared__ uint8_t* s_to[MOVE_ROWS];     // null: left as it is
  int it = 0;
  while (it + 1 < a.n_items && blockIdx.x >= a.item[it + 1].first_block) ++it;
  const MoveItem& t = a.item[it];
  const uint32_t block = blockIdx.x - t.first_block;
  const long long row0 = t.block_rows > 1 ? (long long)block * t.block_rows : block / t.pieces;
  const long long first = t.block_rows > 1 ? 0 : block % t.pieces * t.piece;   // vector of the row that the block starts at
  const int rows = (int)(t.rows - row0 < t.block_rows ? t.rows - row0 : t.block_rows);
  pdl_wait();
  pdl_trigger();
  if ((int)threadIdx.x < rows) {
    const long long r = row0 + threadIdx.x, beams = (long long)a.B * a.W;
    const long long i1 = r % t.n1, bw = r / t.n1 % beams, i0 = r / t.n1 / beams;
    const int p = a.parent[bw];
    s_from[threadIdx.x] = t.src + i0 * t.src_step[0] + i1 * t.src_step[1] + (bw / a.W * a.W + p) * t.src_row;
    s_to[threadIdx.x] = p >= 0 && p < a.W ? t.dst + i0 * t.dst_step[0] + i1 * t.dst_step[1] + bw * t.dst_row : nullptr;
  }
  __syncthreads();
  const int n = t.block_rows > 1 ? rows * (int)t.per_row : (int)(t.per_row - first < t.piece ? t.per_row - first : t.piece);
  switch (t.width) {
    case 16: move_vectors<uint4>(t, s_from, s_to, first, n); break;
    case 8: move_vectors<uint2>(t, s_from, s_to, first, n); break;
    case 4: move_vectors<uint32_t>(t, s_from, s_to, first, n); break;
    case 2: move_vectors<uint16_t>(t, s_from, s_to, first, n); break;
    default: move_vectors<uint8_t>(t, s_from, s_to, first, n);
  }
}

}  // namespace

// Segments of a row: as many as fill the block slots of the device once, at most one a turn, at least so many that none has more than
// 16 turns.  (Two or four times as many, us: 64 x 16 x 32000 31 -> 39 / 50, 100 x 16 x 8000 31 -> 45 / 56.)
static RowParts row_parts(int B, int W, int V, int bytes, uint8_t* workspace) {
  const long long rows = (long long)B * W, slots = (long long)ROW_BLOCKS * sm_count();
  const long long turns = ((long long)V + ROW_TURN * (16 / bytes) - 1) / (ROW_TURN * (16 / bytes)), least = (turns + ROW_TURNS - 1) / ROW_TURNS;
  long long parts = slots / rows;
  if (parts > turns) parts = turns;
  if (parts < least) parts = least;
  RowParts p;
  p.parts = (int)parts;
  p.inv_width = 0xffffffffu / W + 1;   // (entries of a row are fewer than 2^32 / W)
  p.inv_parts = 0xffffffffu / p.parts;
  const long long vectors = (V * (long long)bytes + 15) / 16;
  p.vectors = (int)((vectors + parts - 1) / parts);
  p.lse = reinterpret_cast<double*>(workspace);
  p.best = reinterpret_cast<Best*>(workspace + align_up((size_t)rows * parts * sizeof(double)));
  return p;
}

size_t lm_select_workspace(int B, int W, int V) {
  size_t n = 0;
  for (int bytes = 2; bytes <= 4; bytes += 2) {
    const size_t parts = (size_t)row_parts(B > 0 ? B : 1, W, V, bytes, nullptr).parts, rows = (size_t)B * W;
    const size_t need = align_up(rows * parts * sizeof(double)) + align_up(rows * parts * W * sizeof(Best));
    n = need > n ? need : n;
  }
  return n;
}

template <typename T>
static cudaError_t launch_select(const LmSelectArgs& a, const RowParts& p, cudaStream_t s) {
  return launch_ex(k_lm_select<T>, dim3((unsigned)((long long)a.B * a.W * p.parts)), dim3(ROW_NT), 0, s, true, 1, a, p);
}
cudaError_t launch_lm_select(const LmSelectArgs& a, int dtype, cudaStream_t s) {
  const RowParts p = row_parts(a.B, a.W, a.V, dtype == Q4_F32 ? 4 : 2, a.workspace);
  if ((long long)a.B * a.W * p.parts > 0x7fffffffLL) return cudaErrorInvalidValue;
  timing_begin(s);
  const cudaError_t e = dtype == Q4_F32   ? launch_select<float>(a, p, s)
                        : dtype == Q4_F16 ? launch_select<__half>(a, p, s)
                                          : launch_select<__nv_bfloat16>(a, p, s);
  timing_end(s);
  ++g_launches;
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
    t.rows = q.n[0] * q.n[1] * B * W;
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
    const long long pieces = (t.per_row + MOVE_VECTORS - 1) / MOVE_VECTORS;
    t.block_rows = (int)(MOVE_VECTORS / t.per_row < MOVE_ROWS ? MOVE_VECTORS / t.per_row : MOVE_ROWS);
    if (t.block_rows < 1) t.block_rows = 1;
    if (t.block_rows > 1) t.over = (uint32_t)((0x100000000LL + t.per_row - 1) / t.per_row);   // (not used for rows of one vector)
    t.pieces = (unsigned)pieces;
    t.piece = (t.per_row + pieces - 1) / pieces;
    t.first_block = (unsigned)blocks;
    const long long need = t.block_rows > 1 ? (t.rows + t.block_rows - 1) / t.block_rows : t.rows * pieces;
    if (pieces > 0x7fffffff || need > 0x7fffffff || (blocks += (unsigned long long)need) > 0x7fffffffull) return cudaErrorInvalidValue;
  }
  if (blocks == 0) return cudaSuccess;
  timing_begin(s);
  const cudaError_t e = launch_ex(k_beam_reorder, dim3((unsigned)blocks), dim3(MOVE_NT), 0, s, true, 1, m);
  timing_end(s);
  ++g_launches;
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace q4
