// Token log probabilities (gfx950): log probability of a given id, entropy and
// the most likely ids of each row of logits, and the gradient.
#include <float.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "sara_internal.h"

namespace sara {

// With z = x / T, m the row's largest logit, c = log2(e) / T and u = (x - m) c:
//   s = sum 2^u,  t = sum 2^u u
//   logp(id) = (x_id - m) / T - log s,   H = log s - log(2) t / s
// one pass over the row with a running (m, s, t).  Logits enter as x - m, never as x c:
// the type's lowest value (a mask) would overflow there, and a row of nothing else is uniform.  t sums u, not
// x - m: |2^u u| is at most 0.54, where 2^u (x - m) overflows for logits as large as an accepted temperature allows.
// Running sums start at m = -FLT_MAX, so that x - m is -inf (weight 0), not NaN, for masked ids.
struct RowSum { float m, s, t; };
constexpr RowSum kEmptySum = {-FLT_MAX, 0.f, 0.f};

// (m, s, t) under the larger maximum `m`.  The old maximum may be a mask's, so that u is huge
// and r is 0: r u is formed first, and u is held above -inf.
__device__ __forceinline__ void rescale(RowSum& a, float m, float c) {
  const float u = (a.m - m) * c, r = __builtin_amdgcn_exp2f(u);
  a.t = fmaf(r * fmaxf(u, -FLT_MAX), a.s, r * a.t);
  a.s *= r;
  a.m = m;
}
__device__ __forceinline__ void merge(RowSum& a, RowSum b, float c) {
  const float m = fmaxf(a.m, b.m);
  rescale(a, m, c);
  rescale(b, m, c);
  a.s += b.s;
  a.t += b.t;
}
// weight 0 of a masked id times its -inf must count as 0; a NaN stays in s
__device__ __forceinline__ void add_logit(RowSum& a, float x, float c) {
  const float u = (x - a.m) * c, e = __builtin_amdgcn_exp2f(u);
  a.s += e;
  a.t = fmaf(e, fmaxf(u, -FLT_MAX), a.t);
}

// Reductions over a wave along its rows of 16 lanes and then across them; the result of lane 63 is everyone's.
template <int CTRL> __device__ __forceinline__ float from_lane(float v, float none) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(__float_as_uint(none), __float_as_uint(v), CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ float lane_value(float v, int lane) {
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane));
}
__device__ __forceinline__ float wave_max(float v) {
  v = fmaxf(v, from_lane<0x111>(v, -INFINITY));      // row_shr 1, 2, 4, 8
  v = fmaxf(v, from_lane<0x112>(v, -INFINITY));
  v = fmaxf(v, from_lane<0x114>(v, -INFINITY));
  v = fmaxf(v, from_lane<0x118>(v, -INFINITY));
  v = fmaxf(v, from_lane<0x142>(v, -INFINITY));      // row_bcast 15, 31
  v = fmaxf(v, from_lane<0x143>(v, -INFINITY));
  return lane_value(v, 63);
}
__device__ __forceinline__ float wave_sum(float v) {
  v += from_lane<0x111>(v, 0.f);
  v += from_lane<0x112>(v, 0.f);
  v += from_lane<0x114>(v, 0.f);
  v += from_lane<0x118>(v, 0.f);
  // the broadcasts reach rows that already hold complete sums: rows 1 and 3 take row 0's and 2's, rows 2 and 3 row 1's
  v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x142, 0xA, 0xF, false));
  v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x143, 0xC, 0xF, false));
  return lane_value(v, 63);
}
__device__ __forceinline__ RowSum wave_merge(RowSum a, float c) {
  rescale(a, wave_max(a.m), c);
  return RowSum{a.m, wave_sum(a.s), wave_sum(a.t)};
}

// The k (<= 32) best (logit, id) of what a wave has seen, rank i in lane i: larger logits first, the lower id among
// equals.  Empty ranks hold (-inf, -1), which no -inf logit and no NaN beats.  The floor is a
// value that k of the logits are known to reach: below it nothing is let in.
struct TopList {
  float v;
  int id;
  float last_v;    // what a newcomer has to beat: rank k - 1 or, while that is empty, the floor
  int last_id;
  float floor_v;
  int floor_id;
};
constexpr TopList kEmptyTop = {-INFINITY, -1, -INFINITY, -1, -INFINITY, -1};
__device__ __forceinline__ bool beats(float v, int id, float lv, int lid) { return v > lv || (v == lv && id < lid); }
// the k-th largest of the lanes' values: the smallest of those that fewer than k are above, counted in 64 steps of three
// instructions (taking the largest k times took 0.3 us a time)
__device__ __forceinline__ float kth_largest(int k, float v) {
  if (k == 1) return wave_max(v);
  int above = 0;
#pragma unroll 16
  for (int j = 0; j < 64; ++j) above += lane_value(v, j) > v;
  return -wave_max(above < k ? -v : -INFINITY);
}
__device__ __forceinline__ void set_floor(TopList& l, float f) {
  if (f > -INFINITY) {
    l.last_v = l.floor_v = f;
    l.last_id = l.floor_id = 0x7FFFFFFF;
  }
}
// lane i gets lane i - 1's value, lane 0 its own
__device__ __forceinline__ int lane_below(int v) { return __builtin_amdgcn_update_dpp(v, v, 0x138, 0xF, 0xF, false); }
__device__ __forceinline__ void top_insert(TopList& l, int k, float v, int id) {
  const int lane = threadIdx.x & 63;
  const bool after = beats(v, id, l.v, l.id);        // the list is sorted: a run of lanes from the new entry's rank on
  const float pv = __uint_as_float(lane_below(__float_as_uint(l.v)));
  const int pid = lane_below(l.id);
  const bool here = after && (lane == 0 || !beats(v, id, pv, pid));
  if (lane < k) {
    l.v = here ? v : after ? pv : l.v;
    l.id = here ? id : after ? pid : l.id;
  }
  l.last_v = lane_value(l.v, k - 1);
  l.last_id = __builtin_amdgcn_readlane(l.id, k - 1);
  if (l.last_id < 0) { l.last_v = l.floor_v; l.last_id = l.floor_id; }
}
// each lane offers one (v, id)
__device__ __forceinline__ void top_offer(TopList& l, int k, float v, int id) {
  unsigned long long who = __ballot(beats(v, id, l.last_v, l.last_id));
  while (who) {
    const int src = __ffsll(who) - 1;
    top_insert(l, k, lane_value(v, src), __builtin_amdgcn_readlane(id, src));
    who = __ballot(beats(v, id, l.last_v, l.last_id)) & (who & (who - 1));
  }
}

// Candidates of a block's (or wave's) k best, gathered in any order and then ranked all at once.  More than 64 can reach
// a floor where logits are equal; then n exceeds 64 and the list has to be built by offers.
struct Pool { int n; float v[64]; int id[64]; };
__device__ __forceinline__ void pool_add(Pool& p, bool keep, float v, int id) {
  const unsigned long long who = __ballot(keep);
  if (!who) return;
  const int lane = threadIdx.x & 63;
  int at = 0;
  if (lane == 0) at = atomicAdd(&p.n, __popcll(who));
  at = __builtin_amdgcn_readfirstlane(at) + __popcll(who & ((1ull << lane) - 1));
  if (keep && at < 64) { p.v[at] = v; p.id[at] = id; }
}
// the k best of a pool of n <= 64, rank i in lane i: by a wave
__device__ __forceinline__ TopList pool_best(const Pool& p, int n, int k) {
  const int lane = threadIdx.x & 63;
  TopList l = kEmptyTop;
  const float v = lane < n ? p.v[lane] : -INFINITY;
  const int id = lane < n ? p.id[lane] : -1;
  int rank = lane < n ? 0 : lane;
#pragma unroll 4
  for (int j = 0; j < n; ++j) rank += lane < n && beats(lane_value(v, j), __builtin_amdgcn_readlane(id, j), v, id);
  const float rv = __uint_as_float(__builtin_amdgcn_ds_permute(4 * rank, __float_as_uint(v)));
  const int ri = __builtin_amdgcn_ds_permute(4 * rank, id);
  if (lane < min(n, k)) { l.v = rv; l.id = ri; }
  return l;
}

// The largest of three, NaN if any is.  fmaxf would pass over a NaN, but it makes every operand quiet that may be
// signalling, an instruction each, and the bare maximum loses its other operands to a signalling one.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float m;
  asm("v_maximum3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(a), "v"(b), "v"(c));
  return m;
}

template <typename T> struct Vec16 {
  static constexpr int N = 16 / sizeof(T);
  __device__ static void unpack(u32x4 w, float* x);
};
template <> __device__ __forceinline__ void Vec16<float>::unpack(u32x4 w, float* x) {
#pragma unroll
  for (int q = 0; q < 4; ++q) x[q] = __uint_as_float(w[q]);
}
template <> __device__ __forceinline__ void Vec16<uint16_t>::unpack(u32x4 w, float* x) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    x[2 * q] = __uint_as_float(w[q] << 16);
    x[2 * q + 1] = __uint_as_float(w[q] & 0xFFFF0000u);
  }
}

struct ScoreOut {
  float *logp, *entropy, *stats;
  int32_t* top_id;
  float* top_logp;
};

// (x - m) / T - log s.  Of two finite logits x - m may be -inf, which T above 5e35 would bring back: then each is divided.
__device__ __forceinline__ float log_prob(float x, float m, float inv_t, float logs) {
  const float d = x - m;
  return d < -FLT_MAX ? fmaf(x, inv_t, -m * inv_t) - logs : fmaf(d, inv_t, -logs);
}

// a row's outputs from its sums and its sorted list
__device__ __forceinline__ void write_row(const ScoreOut& out, int r, RowSum a, bool has_tok, float x_tok,
                                          const TopList& l, int k, float inv_t) {
  const int lane = threadIdx.x & 63;
  const bool none = a.s == 0.f;                     // no id above -inf
  const float logs = logf(a.s);
  if (lane == 0) {
    if (out.logp) out.logp[r] = !has_tok ? 0.f : none ? -INFINITY : log_prob(x_tok, a.m, inv_t, logs);
    if (out.entropy) out.entropy[r] = none ? 0.f : fmaf(-0.69314718f, a.t / a.s, logs);
    if (out.stats) *(float2*)(out.stats + 2 * (size_t)r) = make_float2(none ? -INFINITY : a.m, a.s);
  }
  if (lane < k) {
    out.top_id[(size_t)r * k + lane] = l.id;
    out.top_logp[(size_t)r * k + lane] = l.id < 0 ? -INFINITY : log_prob(l.v, a.m, inv_t, logs);
  }
}

// Block (split, row).  The row's 16-byte aligned vectors are shared out over the splits, the few logits before the
// first and after the last go to split 0.  A lane sums U vectors (a group) under one look at its maximum.
// Top ids: while they stream by, a lane keeps only its largest logit and that one's group, and the largest of its other
// groups.  Over the waves lane i keeps the largest of their lanes i; the k-th largest of these 64 is a floor that k logits
// reach, so only the lanes whose maximum reaches it, little more than k, hold any of the k best: their group is read
// again (all their groups if a second one reaches the floor), what reaches the floor is gathered in LDS and ranked at
// once.  Logits equal to the floor can be too many for that; then waves offer theirs one by one to sorted lists.
// Offering logits as they come took 30-60 us more for 2,048 bf16 rows x 151,936 ids (k = 8-20), which sum in 105.
// STREAM: non-temporal loads (see launch_score).
// Bound by memory from some 100 rows on: 2,048 bf16 rows x 151,936 ids 98 us (6.3 TB/s), 512 fp32 rows with 8 top ids 61
// (5.1); one row with 5 top ids is two launches of 6.4 and 4.5 us.
template <typename T, int W, bool TOP, bool STREAM>
__global__ __launch_bounds__(64 * W) void k_token_logprobs(const T* __restrict__ logits, int64_t row_stride, int V,
    const int32_t* __restrict__ tok, float c, float inv_t, int n_top, int splits, float* __restrict__ part, ScoreOut out) {
  const int k = TOP ? n_top : 0;
  constexpr int N = Vec16<T>::N, U = 4;
  __shared__ RowSum sum_w[W];
  __shared__ float max_w[TOP ? W : 1][64];
  __shared__ Pool pool;
  __shared__ float lv_w[W][32];
  __shared__ int li_w[W][32];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int r = blockIdx.y, sp = blockIdx.x;
  const T* x = logits + (size_t)r * row_stride;
  const int head = min(V, (int)((16 - ((uintptr_t)x & 15)) & 15) / (int)sizeof(T));
  const int nv = (V - head) / N, tail = V - head - nv * N;
  const u32x4* xv = (const u32x4*)(x + head);
  const int v0 = (int)((int64_t)nv * sp / splits), v1 = (int)((int64_t)nv * (sp + 1) / splits);
  const int tk = tok[r];
  const bool has_tok = tk >= 0 && tk < V;
  const float x_tok = has_tok && wave == 0 ? ld_f32<T>(x, tk) : 0.f;
  RowSum a = kEmptySum;
  float m1 = -INFINITY, m2 = -INFINITY;                // the lane's largest logit, and outside of its group
  int g1 = 0, groups = 0;
  auto note = [&](float mx, int g) {
    m2 = fmaxf(m2, fminf(m1, mx));
    g1 = mx > m1 ? g : g1;
    m1 = fmaxf(m1, mx);
  };
  auto take = [&](const u32x4* w, int n, bool valid) {
    float f[U][N], all = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u >= n) break;
      Vec16<T>::unpack(w[u], f[u]);
      if (!valid)
#pragma unroll
        for (int q = 0; q < N; ++q) f[u][q] = -INFINITY;
#pragma unroll
      for (int q = 0; q < N; q += 2) all = max3(all, f[u][q], f[u][q + 1]);
    }
    if (all != all) {                                  // the largest of the numbers
      all = -INFINITY;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (u >= n) break;
#pragma unroll
        for (int q = 0; q < N; ++q) all = f[u][q] > all ? f[u][q] : all;
      }
    }
    if (all > a.m) rescale(a, all, c);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u >= n) break;
#pragma unroll
      for (int q = 0; q < N; ++q) add_logit(a, f[u][q], c);
    }
    if (TOP) note(all, groups);
    ++groups;
  };
  constexpr int step = U * W * 64;
  const int b0 = v0 + wave * 64;                       // lane 0's first vector
  const int whole = b0 + (U - 1) * W * 64 + 64 > v1 ? 0 : (v1 - 64 - (U - 1) * W * 64 - b0) / step + 1;   // full groups
  {
    // one group in flight while another is summed
    u32x4 w0[U], w1[U];
    auto load = [&](u32x4* w, int g) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const u32x4* p = xv + (b0 + lane + g * step + u * W * 64);
        w[u] = STREAM ? __builtin_nontemporal_load(p) : *p;
      }
    };
    if (whole > 0) load(w0, 0);
    for (int g = 0; g < whole; g += 2) {
      if (g + 1 < whole) load(w1, g + 1);
      take(w0, U, true);
      if (g + 1 < whole) {
        if (g + 2 < whole) load(w0, g + 2);
        take(w1, U, true);
      }
    }
  }
  for (int b = b0 + whole * step; b < v1; b += W * 64) {   // groups of one vector, the last one ragged
    const u32x4 w = xv[min(b + lane, v1 - 1)];
    take(&w, 1, b + lane < v1);
  }
  const bool ends = sp == 0 && wave == 0;              // one more group: head + tail < 2 N <= 16 logits, one a lane
  auto end_id = [&](int i) { return i < head ? i : V - tail + (i - head); };
  if (ends) {
    const float f = lane < head + tail ? ld_f32<T>(x, end_id(lane)) : -INFINITY;
    if (f > a.m) rescale(a, f, c);
    add_logit(a, f, c);
    if (TOP) note(f == f ? f : -INFINITY, groups);
  }
  TopList l = kEmptyTop;
  if (TOP) {
    max_w[wave][lane] = m1;
    if (threadIdx.x == 0) pool.n = 0;
    __syncthreads();
    float most = max_w[0][lane];
#pragma unroll
    for (int w = 1; w < W; ++w) most = fmaxf(most, max_w[w][lane]);
    const float floor_v = kth_largest(k, most);
    // element i of group g of lane `src`: its id, or -1
    auto element = [&](int src, int g, int i) {
      if (g >= groups) return i == 0 && src < head + tail ? end_id(src) : -1;
      const int first = b0 + src + min(g, whole) * step + max(g - whole, 0) * W * 64;
      const int vec = first + i / N * W * 64;
      return i < (g < whole ? U * N : N) && vec < v1 ? head + vec * N + i % N : -1;
    };
    auto each_candidate = [&](auto offer) {
      auto offer_id = [&](int id) { offer(id >= 0 ? ld_f32<T>(x, id) : -INFINITY, id); };
      unsigned long long few = __ballot(m1 > -INFINITY && m1 >= floor_v);
      unsigned long long more = __ballot(m2 > -INFINITY && m2 >= floor_v) & few;
      few &= ~more;
      constexpr int PER = U * N, AT_ONCE = 64 / PER;   // lanes whose groups are read together
      while (few) {
        int id = -1;
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
          if (!few) break;
          const int src = __ffsll(few) - 1, g = __builtin_amdgcn_readlane(g1, src);
          few &= few - 1;
          if (lane / PER == i) id = element(src, g, lane % PER);
        }
        offer_id(id);
      }
      while (more) {
        const int src = __ffsll(more) - 1;
        more &= more - 1;
        const int n = (groups + (ends ? 1 : 0)) * PER;
        for (int e = lane; e - lane < n; e += 64) offer_id(e < n ? element(src, e / PER, e % PER) : -1);
      }
    };
    each_candidate([&](float v, int id) { pool_add(pool, v > -INFINITY && v >= floor_v, v, id); });
    __syncthreads();
    if (pool.n > 64) {
      set_floor(l, floor_v);
      each_candidate([&](float v, int id) { top_offer(l, k, v, id); });
    }
  }
  a = wave_merge(a, c);
  if (lane == 0) sum_w[wave] = a;
  if (lane < k) { lv_w[wave][lane] = l.v; li_w[wave][lane] = l.id; }
  __syncthreads();
  if (wave) return;
  for (int w = 1; w < W; ++w) merge(a, sum_w[w], c);
  if (TOP) {
    if (pool.n <= 64) l = pool_best(pool, pool.n, k);
    else
      for (int w = 1; w < W; ++w) top_offer(l, k, lane < k ? lv_w[w][lane] : -INFINITY, lane < k ? li_w[w][lane] : -1);
  }
  if (splits == 1) {
    write_row(out, r, a, has_tok, x_tok, l, k, inv_t);
    return;
  }
  float* p = part + ((size_t)r * splits + sp) * (4 + 2 * k);
  if (lane == 0) { p[0] = a.m; p[1] = a.s; p[2] = a.t; }
  if (lane < k) { p[4 + lane] = l.v; p[4 + k + lane] = __int_as_float(l.id); }
}

// A wave per row joins its splits (at most 64): sums by lane, top ids as above from the splits' sorted lists.  38 splits
// with 5 top ids: 4.5 us; 64 rows of 16 with 20: 7.2.
template <typename T>
__global__ __launch_bounds__(64) void k_token_logprobs_join(const T* __restrict__ logits, int64_t row_stride, int V,
    const int32_t* __restrict__ tok, float c, float inv_t, int k, int splits, const float* __restrict__ part,
    ScoreOut out) {
  const int lane = threadIdx.x, r = blockIdx.x;
  const int tk = tok[r];
  const bool has_tok = tk >= 0 && tk < V;
  const float x_tok = has_tok ? ld_f32<T>(logits + (size_t)r * row_stride, tk) : 0.f;
  const float* p = part + (size_t)r * splits * (4 + 2 * k);
  RowSum a = kEmptySum;
  if (lane < splits) { const float* q = p + (size_t)lane * (4 + 2 * k); a = RowSum{q[0], q[1], q[2]}; }
  a = wave_merge(a, c);
  TopList l = kEmptyTop;
  if (k > 0) {
    // floor: the k-th largest of 64 entries, as many from the front of each split's list
    __shared__ Pool pool;
    if (lane == 0) pool.n = 0;
    auto value = [&](int split, int rank) { return p[(size_t)split * (4 + 2 * k) + 4 + rank]; };
    const float floor_v = kth_largest(k, lane / splits < k ? value(lane % splits, lane / splits) : -INFINITY);
    auto each_entry = [&](auto offer) {
#pragma unroll 4
      for (int e0 = 0; e0 < splits * k; e0 += 64) {
        const int e = min(e0 + lane, splits * k - 1);
        const float* q = p + (size_t)(e / k) * (4 + 2 * k) + 4 + e % k;
        const bool in = e0 + lane < splits * k;
        offer(in ? q[0] : -INFINITY, in ? __float_as_int(q[k]) : -1);
      }
    };
    each_entry([&](float v, int id) { pool_add(pool, v > -INFINITY && v >= floor_v, v, id); });
    const int n = __builtin_amdgcn_readfirstlane(pool.n);
    if (n <= 64) {
      l = pool_best(pool, n, k);
    } else {
      set_floor(l, floor_v);
      each_entry([&](float v, int id) { top_offer(l, k, v, id); });
    }
  }
  write_row(out, r, a, has_tok, x_tok, l, k, inv_t);
}

// dx_j = (1/T) [ g ([j = tok] - p_j) - h p_j (log p_j + H) ],  p_j = 2^((x_j - m) c) / s.
// With u = (x_j - m) c:  dx_j = (2^u (A + B u) + [j = tok] g) / T,
//   A = -(g + h (H - log s)) / s,  B = -h log(2) / s.
// No power of T enters A or B and u is held above -150, where 2^u is 0 already: at every accepted temperature a masked
// id gets 0, and 1 / T overflows only where the gradient does.
// The rounded d and d c alone would cost the p of an id far below the largest |d c| 2^-23 of itself: nothing
// beside the rounding of a bf16 gradient, but an fp32 one adds what the difference and the product lost (c in
// two parts), which its twice as many bytes hide.
// Bound by memory: 2,048 bf16 rows x 151,936 ids 197 us (6.3 TB/s), read and written past the caches.
// VEC: logits and gradient rows lie alike modulo 16 bytes.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void k_token_logprobs_grad(const T* logits, int64_t row_stride, int V,
    const int32_t* __restrict__ tok, const float* __restrict__ stats, const float* __restrict__ entropy,
    const float* __restrict__ g_logp, const float* __restrict__ g_ent, float c, float c_lo, float inv_t, T* grad,
    int64_t grad_stride) {
  constexpr int N = Vec16<T>::N;
  const int r = blockIdx.y;
  const T* x = logits + (size_t)r * row_stride;
  T* y = grad + (size_t)r * grad_stride;
  const int tk = tok[r];
  const float m = stats[2 * (size_t)r], s = stats[2 * (size_t)r + 1];
  const float g = tk >= 0 && tk < V && g_logp ? g_logp[r] : 0.f, h = g_ent ? g_ent[r] : 0.f;
  const bool none = s == 0.f || (g == 0.f && h == 0.f);   // nothing left of the row, or nothing asked of it
  const float A = -(g + (h == 0.f ? 0.f : h * (entropy[r] - logf(s)))) / s, B = -0.69314718f * h / s;
  // T times the gradient of a logit, but for the token's own g
  auto one = [&](float f) {
    const float d = f - m, a = d * c;
    float e = __builtin_amdgcn_exp2f(a);
    if (sizeof(T) == 4) {
      const float x1 = d + m, dl = (f - x1) + ((x1 - d) - m);
      const float lost = fmaf(dl, c, fmaf(d, c_lo, fmaf(d, c, -a)));   // not a number where d c overflows, and e is 0
      e = a > -150.f ? fmaf(e, lost * 0.69314718f, e) : e;
    }
    return e * fmaf(B, fmaxf(a, -150.f), A);             // a NaN is in e
  };
  const int stride = gridDim.x * 256, t0 = blockIdx.x * 256 + threadIdx.x;
  if (!VEC) {
    for (int j = t0; j < V; j += stride) st_f32<T>(y, j, none ? 0.f : (one(ld_f32<T>(x, j)) + (j == tk ? g : 0.f)) * inv_t);
    return;
  }
  const int head = min(V, (int)((16 - ((uintptr_t)x & 15)) & 15) / (int)sizeof(T));
  const int nv = (V - head) / N, tail = V - head - nv * N;
  for (int b = t0; b < nv; b += stride) {
    u32x4 w = {0, 0, 0, 0};
    if (!none) {
      float f[N];
      Vec16<T>::unpack(__builtin_nontemporal_load((const u32x4*)(x + head) + b), f);
#pragma unroll
      for (int q = 0; q < N; ++q) f[q] = one(f[q]);
      const int at = tk - (head + b * N);
      if (at >= 0 && at < N)
#pragma unroll
        for (int q = 0; q < N; ++q) f[q] += q == at ? g : 0.f;
#pragma unroll
      for (int q = 0; q < N; ++q) f[q] *= inv_t;
#pragma unroll
      for (int q = 0; q < 4; ++q) w[q] = sizeof(T) == 2 ? pack_bf16(f[2 * q], f[2 * q + 1]) : __float_as_uint(f[q]);
    }
    __builtin_nontemporal_store(w, (u32x4*)(y + head) + b);
  }
  if (t0 < head + tail) {
    const int j = t0 < head ? t0 : V - tail + (t0 - head);
    st_f32<T>(y, j, none ? 0.f : (one(ld_f32<T>(x, j)) + (j == tk ? g : 0.f)) * inv_t);
  }
}

// Waves of a block and splits of a row.  From 512 rows on a block has a row to itself, of 8 waves where rows are long (600
// bf16 rows x 151,936 ids with 20 top ids: 50 us, against 54 with 4 waves; 512 fp32 rows with 8: 61 either way, 66 as two
// splits of 4 waves and a join), of 4 where they are not (700 bf16 rows x 32,016 ids: 17 us, against 20; x 100,000: 34
// either way).  Fewer rows are split until 1,024 blocks share them, but not below 4,096 ids, about what a block's start
// and the join cost.
static int score_waves(int n_rows, int V) { return n_rows >= 512 && V >= 98304 ? 8 : 4; }
static int score_splits(int n_rows, int V) {
  if (n_rows >= 512) return 1;
  const int by_rows = (1024 + n_rows - 1) / n_rows, by_size = (V + 4095) / 4096;
  return std::max(1, std::min(std::min(by_rows, by_size), 64));
}

int64_t score_workspace(int n_rows, int V, int k) {
  const int sp = score_splits(n_rows, V);
  return sp == 1 ? 0 : (int64_t)sizeof(float) * n_rows * sp * (4 + 2 * k);
}

template <typename T>
static void launch_score(const T* logits, int64_t row_stride, int n_rows, int V, const int32_t* tok, float temp, int k,
                         const ScoreOut& out, float* ws, hipStream_t st) {
  const float inv_t = 1.f / temp, c = (float)(1.4426950408889634 / (double)temp);
  const int sp = score_splits(n_rows, V);
  // Logits that a gradient may soon read again are left in the last-level cache (256 MB) where much of them fits: 155 MB
  // of bf16, forward and gradient 81 us against 86 with non-temporal loads.  Past twice its size nothing would be left:
  // 622 MB, forward alone 102 us non-temporal against 114.
  const bool stream = (double)n_rows * V * sizeof(T) > 512.0e6;
  // a grid's y extent is 16 bits
  for (int r0 = 0; r0 < n_rows; r0 += 65535) {
    const int n = std::min(65535, n_rows - r0);
    ScoreOut o = out;
    if (o.logp) o.logp += r0;
    if (o.entropy) o.entropy += r0;
    if (o.stats) o.stats += 2 * (size_t)r0;
    if (k) { o.top_id += (size_t)r0 * k; o.top_logp += (size_t)r0 * k; }
    const T* x = logits + (size_t)r0 * row_stride;
    auto go = [&](auto kernel, int waves) {
      hipLaunchKernelGGL(kernel, dim3(sp, n), dim3(64 * waves), 0, st, x, row_stride, V, tok + r0, c, inv_t, k, sp, ws, o);
    };
    auto by_loads = [&](auto w, auto top) {
      if (stream) go(k_token_logprobs<T, w.value, top.value, true>, w.value);
      else go(k_token_logprobs<T, w.value, top.value, false>, w.value);
    };
    auto by_top = [&](auto w) { k ? by_loads(w, std::true_type{}) : by_loads(w, std::false_type{}); };
    if (score_waves(n_rows, V) == 8) by_top(std::integral_constant<int, 8>{});
    else by_top(std::integral_constant<int, 4>{});
    if (sp > 1)
      hipLaunchKernelGGL(k_token_logprobs_join<T>, dim3(n), dim3(64), 0, st, x, row_stride, V, tok + r0, c, inv_t, k, sp,
                         ws, o);
  }
}

int launch_token_logprobs(const void* logits, int dtype, int64_t row_stride, int n_rows, int V, const int32_t* tok,
                          float temp, int k, float* logp, float* entropy, float* stats, int32_t* top_id, float* top_logp,
                          void* ws, hipStream_t st) {
  const ScoreOut out = {logp, entropy, stats, top_id, top_logp};
  if (dtype == SARA_BF16)
    launch_score((const uint16_t*)logits, row_stride, n_rows, V, tok, temp, k, out, (float*)ws, st);
  else
    launch_score((const float*)logits, row_stride, n_rows, V, tok, temp, k, out, (float*)ws, st);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SARA_OK : hip_fail(e, "token log probabilities launch");
}

template <typename T>
static void launch_score_grad(const T* x, int64_t xs, int n_rows, int V, const int32_t* tok, const float* stats,
                              const float* entropy, const float* g_logp, const float* g_ent, float temp, T* y, int64_t ys,
                              hipStream_t st) {
  const double cd = 1.4426950408889634 / (double)temp;
  const float inv_t = 1.f / temp, c = (float)cd, c_lo = (float)(cd - (double)c);
  const bool vec = ((uintptr_t)x - (uintptr_t)y) % 16 == 0 && (n_rows == 1 || ((xs - ys) * (int64_t)sizeof(T)) % 16 == 0);
  const int per = 256 * Vec16<T>::N * 4;
  for (int r0 = 0; r0 < n_rows; r0 += 65535) {
    const int n = std::min(65535, n_rows - r0);
    auto go = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3((V + per - 1) / per, n), dim3(256), 0, st, x + (size_t)r0 * xs, xs, V, tok + r0,
                         stats + 2 * (size_t)r0, entropy ? entropy + r0 : nullptr, g_logp ? g_logp + r0 : nullptr,
                         g_ent ? g_ent + r0 : nullptr, c, c_lo, inv_t, y + (size_t)r0 * ys, ys);
    };
    if (vec) go(k_token_logprobs_grad<T, true>);
    else go(k_token_logprobs_grad<T, false>);
  }
}

int launch_token_logprobs_grad(const void* logits, int dtype, int64_t row_stride, int n_rows, int V, const int32_t* tok,
                               const float* stats, const float* entropy, const float* g_logp, const float* g_ent,
                               float temp, void* grad, int64_t grad_stride, hipStream_t st) {
  if (dtype == SARA_BF16)
    launch_score_grad((const uint16_t*)logits, row_stride, n_rows, V, tok, stats, entropy, g_logp, g_ent, temp,
                      (uint16_t*)grad, grad_stride, st);
  else
    launch_score_grad((const float*)logits, row_stride, n_rows, V, tok, stats, entropy, g_logp, g_ent, temp, (float*)grad,
                      grad_stride, st);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SARA_OK : hip_fail(e, "token log probabilities gradient launch");
}

}  // namespace sara
