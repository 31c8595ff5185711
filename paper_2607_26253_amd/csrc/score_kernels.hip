// Token log probabilities (gfx950): log probability of a given id, entropy and
// the most likely ids of each row of logits, and the gradient.
#include <float.h>
#include <math.h>

#include <algorithm>

#include "sara_internal.h"

namespace sara {

// With z = x / T, m the row's largest logit and c = log2(e) / T:
//   s = sum 2^((x - m) c),  t = sum 2^((x - m) c) (x - m)
//   logp(id) = (x_id - m) / T - log s,   H = log s - t / (T s)
// one pass over the row with a running (m, s, t).  Logits enter as x - m, never as x c:
// the type's lowest value (a mask) would overflow there, and a row of nothing else is uniform.
// Running sums start at m = -FLT_MAX, so that x - m is -inf (weight 0), not NaN, for masked ids.
struct RowSum { float m, s, t; };
constexpr RowSum kEmptySum = {-FLT_MAX, 0.f, 0.f};

// (m, s, t) under the larger maximum `m`.  The old maximum may be a mask's, so that d is huge
// and r is 0: r d is formed first, and d is held above -inf.
__device__ __forceinline__ void rescale(RowSum& a, float m, float c) {
  const float d = a.m - m, r = __builtin_amdgcn_exp2f(d * c);
  a.t = fmaf(r * fmaxf(d, -FLT_MAX), a.s, r * a.t);
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
  const float d = x - a.m, e = __builtin_amdgcn_exp2f(d * c);
  a.s += e;
  a.t = fmaf(e, fmaxf(d, -FLT_MAX), a.t);
}

// The k (<= 32) best (logit, id) of what a wave has seen, rank i in lane i: larger logits
// first, the lower id among equals.  Empty ranks hold (-inf, -1), which no -inf logit and no NaN beats.
struct TopList {
  float v;
  int id;
  float last_v;   // rank k - 1, in all lanes
  int last_id;
};
__device__ __forceinline__ bool beats(float v, int id, float lv, int lid) { return v > lv || (v == lv && id < lid); }
__device__ __forceinline__ void top_insert(TopList& l, int k, float v, int id) {
  const int lane = threadIdx.x & 63;
  const int at = __ffsll((unsigned long long)__ballot(beats(v, id, l.v, l.id))) - 1;
  const float pv = __shfl_up(l.v, 1, 64);
  const int pid = __shfl_up(l.id, 1, 64);
  l.v = lane < at ? l.v : lane == at ? v : pv;
  l.id = lane < at ? l.id : lane == at ? id : pid;
  if (lane >= k) { l.v = -INFINITY; l.id = -1; }
  l.last_v = __shfl(l.v, k - 1, 64);
  l.last_id = __shfl(l.id, k - 1, 64);
}
// each lane offers one (v, id)
__device__ __forceinline__ void top_offer(TopList& l, int k, float v, int id) {
  unsigned long long who = __ballot(beats(v, id, l.last_v, l.last_id));
  while (who) {
    const int src = __ffsll(who) - 1;
    top_insert(l, k, __shfl(v, src, 64), __shfl(id, src, 64));
    who &= who - 1;
    who &= __ballot(beats(v, id, l.last_v, l.last_id));
  }
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

// a row's outputs from its sums and its sorted list
__device__ __forceinline__ void write_row(const ScoreOut& out, int r, RowSum a, bool has_tok, float x_tok,
                                          const TopList& l, int k, float inv_t) {
  const int lane = threadIdx.x & 63;
  const bool none = a.s == 0.f;                     // no id above -inf
  const float logs = logf(a.s);
  if (lane == 0) {
    if (out.logp) out.logp[r] = !has_tok ? 0.f : none ? -INFINITY : fmaf(x_tok - a.m, inv_t, -logs);
    if (out.entropy) out.entropy[r] = none ? 0.f : fmaf(-inv_t, a.t / a.s, logs);
    if (out.stats) *(float2*)(out.stats + 2 * (size_t)r) = make_float2(none ? -INFINITY : a.m, a.s);
  }
  if (lane < k) {
    out.top_id[(size_t)r * k + lane] = l.id;
    out.top_logp[(size_t)r * k + lane] = l.id < 0 ? -INFINITY : fmaf(l.v - a.m, inv_t, -logs);
  }
}

__device__ __forceinline__ RowSum wave_merge(RowSum a, float c) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    RowSum b = {__shfl_xor(a.m, o, 64), __shfl_xor(a.s, o, 64), __shfl_xor(a.t, o, 64)};
    merge(a, b, c);
  }
  return a;
}

// Block (split, row).  The row's 16-byte aligned vectors are shared out over the splits, the
// few logits before the first and after the last go to split 0.
template <typename T, int W>
__global__ __launch_bounds__(64 * W) void k_token_logprobs(const T* __restrict__ logits, int64_t row_stride, int V,
    const int32_t* __restrict__ tok, float c, float inv_t, int k, int splits, float* __restrict__ part, ScoreOut out) {
  constexpr int N = Vec16<T>::N, U = 4;
  __shared__ RowSum sum_w[W];
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
  TopList l = {-INFINITY, -1, -INFINITY, -1};
  auto take = [&](u32x4 w, int vec, bool valid) {
    float f[N];
    Vec16<T>::unpack(w, f);
    if (!valid)
#pragma unroll
      for (int q = 0; q < N; ++q) f[q] = -INFINITY;
    float mx = f[0];
#pragma unroll
    for (int q = 1; q < N; ++q) mx = fmaxf(mx, f[q]);
    if (mx > a.m) rescale(a, mx, c);
#pragma unroll
    for (int q = 0; q < N; ++q) add_logit(a, f[q], c);
    if (k > 0 && __ballot(mx >= l.last_v)) {
#pragma unroll
      for (int q = 0; q < N; ++q) top_offer(l, k, f[q], head + vec * N + q);
    }
  };
  for (int b = v0 + wave * 64; b < v1; b += W * 64 * U) {
    u32x4 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = xv[min(b + u * W * 64 + lane, v1 - 1)];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = b + u * W * 64;
      if (at < v1) take(w[u], at + lane, at + lane < v1);
    }
  }
  if (sp == 0 && wave == 0) {                        // head + tail < 2 N <= 16 logits
    const int id = lane < head ? lane : V - tail + (lane - head);
    const float f = lane < head + tail ? ld_f32<T>(x, id) : -INFINITY;
    if (f > a.m) rescale(a, f, c);
    add_logit(a, f, c);
    if (k > 0) top_offer(l, k, f, id);
  }
  a = wave_merge(a, c);
  if (lane == 0) sum_w[wave] = a;
  if (lane < k) { lv_w[wave][lane] = l.v; li_w[wave][lane] = l.id; }
  __syncthreads();
  if (wave) return;
  for (int w = 1; w < W; ++w) {
    merge(a, sum_w[w], c);
    if (k > 0) top_offer(l, k, lane < k ? lv_w[w][lane] : -INFINITY, lane < k ? li_w[w][lane] : -1);
  }
  if (splits == 1) {
    write_row(out, r, a, has_tok, x_tok, l, k, inv_t);
    return;
  }
  float* p = part + ((size_t)r * splits + sp) * (4 + 2 * k);
  if (lane == 0) { p[0] = a.m; p[1] = a.s; p[2] = a.t; }
  if (lane < k) { p[4 + lane] = l.v; p[4 + k + lane] = __int_as_float(l.id); }
}

// a wave per row joins its splits (at most 64)
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
  TopList l = {-INFINITY, -1, -INFINITY, -1};
  for (int e0 = 0; e0 < splits * k; e0 += 64) {
    const int e = e0 + lane;
    const float* q = p + (size_t)(e / k) * (4 + 2 * k) + 4 + e % k;
    const bool in = e < splits * k;
    top_offer(l, k, in ? q[0] : -INFINITY, in ? __float_as_int(q[k]) : -1);
  }
  write_row(out, r, a, has_tok, x_tok, l, k, inv_t);
}

// dx_j = (1/T) [ g ([j = tok] - p_j) - h p_j (log p_j + H) ],  p_j = 2^((x_j - m) c) / s.
// With d = x_j - m:  dx_j = 2^(d c) (A + B d) + [j = tok] g / T,
//   A = -(g + h (H - log s)) / (T s),  B = -h / (T^2 s).
// The rounded d and d c alone would cost the p of an id far below the largest |d c| 2^-23 of itself: nothing
// beside the rounding of a bf16 gradient, but an fp32 one adds what the difference and the product lost (c in
// two parts), which its twice as many bytes hide.
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
  const float A = -(g + (h == 0.f ? 0.f : h * (entropy[r] - logf(s)))) * inv_t / s, B = -h * inv_t * inv_t / s;
  const float at_tok = g * inv_t;
  auto one = [&](float f, int j) {
    const float d = f - m, a = d * c;
    float e = __builtin_amdgcn_exp2f(a);
    if (sizeof(T) == 4) {
      const float x1 = d + m, dl = (f - x1) + ((x1 - d) - m);
      const float lost = fmaf(dl, c, fmaf(d, c_lo, fmaf(d, c, -a)));   // not a number where d c overflows, and e is 0
      e = a > -150.f ? fmaf(e, lost * 0.69314718f, e) : e;
    }
    // where d matters (d c > -150) it is far above this bound, which keeps B d finite for masked ids
    const float v = e * fmaf(B, fmaxf(d, -1e20f), A);
    return (d != d ? d : v) + (j == tk ? at_tok : 0.f);
  };
  const int stride = gridDim.x * 256, t0 = blockIdx.x * 256 + threadIdx.x;
  if (!VEC) {
    for (int j = t0; j < V; j += stride) st_f32<T>(y, j, none ? 0.f : one(ld_f32<T>(x, j), j));
    return;
  }
  const int head = min(V, (int)((16 - ((uintptr_t)x & 15)) & 15) / (int)sizeof(T));
  const int nv = (V - head) / N, tail = V - head - nv * N;
  for (int b = t0; b < nv; b += stride) {
    u32x4 w = {0, 0, 0, 0};
    if (!none) {
      float f[N];
      Vec16<T>::unpack(((const u32x4*)(x + head))[b], f);
#pragma unroll
      for (int q = 0; q < N; ++q) f[q] = one(f[q], head + b * N + q);
#pragma unroll
      for (int q = 0; q < 4; ++q) w[q] = sizeof(T) == 2 ? pack_bf16(f[2 * q], f[2 * q + 1]) : __float_as_uint(f[q]);
    }
    ((u32x4*)(y + head))[b] = w;
  }
  if (t0 < head + tail) {
    const int j = t0 < head ? t0 : V - tail + (t0 - head);
    st_f32<T>(y, j, none ? 0.f : one(ld_f32<T>(x, j), j));
  }
}

int score_splits(int n_rows, int V) {
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
  // a grid's y extent is 16 bits
  for (int r0 = 0; r0 < n_rows; r0 += 65535) {
    const int n = std::min(65535, n_rows - r0);
    ScoreOut o = out;
    if (o.logp) o.logp += r0;
    if (o.entropy) o.entropy += r0;
    if (o.stats) o.stats += 2 * (size_t)r0;
    if (k) { o.top_id += (size_t)r0 * k; o.top_logp += (size_t)r0 * k; }
    const T* x = logits + (size_t)r0 * row_stride;
    hipLaunchKernelGGL((k_token_logprobs<T, 4>), dim3(sp, n), dim3(256), 0, st, x, row_stride, V, tok + r0, c, inv_t, k,
                       sp, ws, o);
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
