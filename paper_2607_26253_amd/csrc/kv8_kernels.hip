// KV cache in 8 bits (gfx950): quantising writes, reads, and attention over its pages.
//
// A page holds 16 tokens of one sequence: codes k, v [page][KV head][16][HD], one byte each (int8, or
// fp8 e4m3), and for each page and KV head two exponent bytes: value = code 2^(b - 127), b = 255 is NaN.
// A power of two as scale makes x / scale exact, so a code is the one rounding between a value and its
// cached form, a value is exact in bf16 (but for e4m3 at b = 1 or 2, below bf16's 2^-133), and a page whose scale grows (a token larger than its others
// is appended) re-rounds its codes by a shift: it ends as if written at once, but for codes that the
// shift leaves halfway.  Against amax / 127 it costs int8 up to one bit and e4m3 nothing.
#include <math.h>

#include <algorithm>

#include "sara_internal.h"

namespace sara {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------------------
// codes
// ---------------------------------------------------------------------------
// 127 = 1.984375 2^6 and 448 = 1.75 2^8: amax rounds up to the next power of two above those mantissas
template <int FMT> __device__ __forceinline__ int exponent_of(uint32_t amax_bits) {
  if (amax_bits >= 0x7F800000u) return 255;
  return FMT == SARA_KV8_INT8 ? max(1, (int)((amax_bits + 0x1FFFFu) >> 23) - 6)
                              : max(1, (int)((amax_bits + 0x1FFFFFu) >> 23) - 8);
}
__device__ __forceinline__ float exponent_scale(int b) {
  return b == 255 ? __uint_as_float(0x7FC00000u) : ldexpf(1.f, b - 127);
}
// four codes from values already divided by their scale (|y| <= 127 or 448)
template <int FMT> __device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  if (FMT == SARA_KV8_INT8) {
    const uint32_t x = __float2int_rn(a), y = __float2int_rn(b), z = __float2int_rn(c), w = __float2int_rn(d);
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(w, z, 0x0C0C0400u), __builtin_amdgcn_perm(y, x, 0x0C0C0400u),
                                 0x05040100u);
  }
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}
// byte B of a word, signed, as a float: one instruction (left to itself the compiler shifts first)
template <int B> __device__ __forceinline__ float byte_f32(uint32_t w) {
  float f;
  if (B == 0) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=v"(f) : "v"(w));
  if (B == 1) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(f) : "v"(w));
  if (B == 2) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(f) : "v"(w));
  if (B == 3) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(f) : "v"(w));
  return f;
}
template <int FMT> __device__ __forceinline__ void decode4(uint32_t w, float* f) {
  if (FMT == SARA_KV8_INT8) {
    f[0] = byte_f32<0>(w); f[1] = byte_f32<1>(w); f[2] = byte_f32<2>(w); f[3] = byte_f32<3>(w);
  } else {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    f[0] = lo[0]; f[1] = lo[1]; f[2] = hi[0]; f[3] = hi[1];
  }
}
// four codes as bf16, exactly
template <int FMT> __device__ __forceinline__ u32x2 codes_bf16(uint32_t w) {
  if (FMT == SARA_KV8_E4M3)
    return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true))};
  float f[4];
  decode4<FMT>(w, f);
  return u32x2{__builtin_amdgcn_perm(__float_as_uint(f[1]), __float_as_uint(f[0]), 0x07060302u),
               __builtin_amdgcn_perm(__float_as_uint(f[3]), __float_as_uint(f[2]), 0x07060302u)};
}

// four codes times a power of two as bf16, exactly but for what bf16 does not hold (values below 2^-133, inf)
template <int FMT> __device__ __forceinline__ u32x2 values_bf16(uint32_t w, float scale) {
  if (FMT == SARA_KV8_INT8) {
    float f[4];
    decode4<FMT>(w, f);
    return u32x2{__builtin_amdgcn_perm(__float_as_uint(f[1] * scale), __float_as_uint(f[0] * scale), 0x07060302u),
                 __builtin_amdgcn_perm(__float_as_uint(f[3] * scale), __float_as_uint(f[2] * scale), 0x07060302u)};
  }
  return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true))};
}

// The first exponent byte whose scale takes some code past the largest finite number, and four codes under such a byte
// held at the largest multiple of the scale that is finite (b = 255, a page of NaN, leaves none).
template <int FMT> constexpr int kFirstInf = FMT == SARA_KV8_INT8 ? 249 : 247;
template <int FMT> __device__ __forceinline__ uint32_t finite_codes(uint32_t w, int b) {
  const int top = FMT == SARA_KV8_INT8 ? (1 << (255 - b)) - 1 : 8 * (262 - b) - 1;   // below 2^(255 - b), as a code
  uint32_t r = 0;
#pragma unroll
  for (int i = 0; i < 32; i += 8) {
    const int c = (int)(w << (24 - i)) >> 24;
    r |= (uint32_t)((FMT == SARA_KV8_INT8 ? min(max(c, -top), top) : (c & 0x80) | min(c & 0x7F, top)) & 255) << i;
  }
  return r;
}

// ---------------------------------------------------------------------------
// ragged work
// ---------------------------------------------------------------------------
// Sequences own rows [off[i], off[i + 1]).  A launch numbers its items without a pass over the sequences:
// sequence i's begin at off[i] mul / DIV + add i, which leaves room for floor(rows mul / DIV) + add of them.
// The sequence of item b (-1: none), by a wave that cuts the range 64-fold a step.
// What the caller needs of the sequence next comes with the last step: its rows and its entry of `per_seq`.
struct SeqRows { int seq, first, r0, r1, value; };
template <int DIV>
__device__ __forceinline__ SeqRows find_seq(const int32_t* off, const int32_t* per_seq, int n_seqs, int n_rows, int b, int mul,
                                            int add) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = n_seqs;
  while (true) {
    const int step = (hi - lo + 63) >> 6;
    const int i = lo + lane * step;
    int at = 0x7FFFFFFF, o0 = 0, o1 = 0, value = 0;
    if (i < hi) {
      o0 = off[i];
      if (step <= 1) { o1 = off[i + 1]; value = per_seq[i]; }
      at = (int)((int64_t)o0 * mul / DIV) + add * i;
    }
    const int n = __popcll(__ballot(at <= b));
    if (n == 0) return SeqRows{-1, 0, 0, 0, 0};
    lo += (n - 1) * step;
    hi = min(hi, lo + step);
    if (step > 1) continue;
    SeqRows s = {__builtin_amdgcn_readfirstlane(lo), __builtin_amdgcn_readlane(at, n - 1), __builtin_amdgcn_readlane(o0, n - 1),
                 __builtin_amdgcn_readlane(o1, n - 1), __builtin_amdgcn_readlane(value, n - 1)};
    s.r0 = min(max(s.r0, 0), n_rows);
    s.r1 = min(max(s.r1, s.r0), n_rows);
    return s;
  }
}

// rows of sequence i: [r0, r1), held inside the caller's tensor
__device__ __forceinline__ void seq_rows(const int32_t* off, int i, int n_rows, int& r0, int& r1) {
  r0 = off ? min(max(off[i], 0), n_rows) : i;
  r1 = off ? min(max(off[i + 1], r0), n_rows) : i + 1;
}

// ---------------------------------------------------------------------------
// write and read
// ---------------------------------------------------------------------------
struct KvRows {   // rows of K and V in the caller's tensors, strides in elements
  void *k, *v;
  int64_t k_row, k_head, v_row, v_head;
};

// A wave per (page, KV head, K or V): which page, or false where there is none.  A start below 0 begins at a page below 0.
struct PageUnit {
  int seq, page, head, r0, len, start;   // page: its index in the sequence; rows r0 + t <-> positions start + t
  bool is_v;
};
__device__ __forceinline__ bool page_unit(int unit, int hkv, const int32_t* start, const int32_t* off, int n_seqs,
                                          int n_rows, PageUnit& u) {
  u.is_v = unit & 1;
  const int rest = unit >> 1, item = rest / hkv;
  u.head = rest - item * hkv;
  SeqRows s = {item, item, item, item + 1, 0};
  if (off) s = find_seq<16>(off, start, n_seqs, n_rows, item, 1, 2);
  else if (item < n_seqs) s.value = start[item];
  if (s.seq < 0 || s.seq >= n_seqs || item < s.first) return false;
  u.seq = s.seq;
  u.r0 = s.r0;
  u.len = s.r1 - s.r0;
  u.start = s.value;
  if (u.len <= 0) return false;
  u.page = (u.start >> 4) + (item - s.first);
  return u.page <= (int)(((int64_t)u.start + u.len - 1) >> 4);
}

// Lane: 8 consecutive dims of 128 / HD token rows of every 8 (HD 64) or 4 (HD 128) of the page.
template <int HD> struct PageLanes {
  static constexpr int TPR = HD / 8;          // lanes a token row
  static constexpr int RPI = 64 / TPR;        // token rows an instruction
  static constexpr int NI = kBlockTok / RPI;  // instructions a page
};

// 8 elements as they lie in memory
template <typename T> struct Raw8 { u32x4 w[sizeof(T) / 2]; };
template <typename T> __device__ __forceinline__ Raw8<T> load_raw8(const T* p) {
  Raw8<T> r;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.w[i] = ((const u32x4*)p)[i];
  return r;
}
__device__ __forceinline__ void unpack8(const Raw8<uint16_t>& r, float* f) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    f[2 * q] = __uint_as_float(r.w[0][q] << 16);
    f[2 * q + 1] = __uint_as_float(r.w[0][q] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void unpack8(const Raw8<float>& r, float* f) {
#pragma unroll
  for (int q = 0; q < 8; ++q) f[q] = __uint_as_float(r.w[q >> 2][q & 3]);
}
template <typename T> __device__ __forceinline__ void load8(const T* p, float* f) { unpack8(load_raw8<T>(p), f); }

// The larger of `most` and the magnitudes of 8 elements, as bits (NaN above inf above all); bf16 as two halves a word.
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t magnitude(uint32_t most, const Raw8<uint16_t>& r) {
  u16x2 m = __builtin_bit_cast(u16x2, most);
#pragma unroll
  for (int q = 0; q < 4; ++q) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, r.w[0][q] & 0x7FFF7FFFu));
  return __builtin_bit_cast(uint32_t, m);
}
__device__ __forceinline__ uint32_t magnitude(uint32_t most, const Raw8<float>& r) {
#pragma unroll
  for (int q = 0; q < 8; ++q) most = max(most, r.w[q >> 2][q & 3] & 0x7FFFFFFFu);
  return most;
}
template <typename T> __device__ __forceinline__ uint32_t magnitude_bits(uint32_t most) {
  return sizeof(T) == 4 ? most : max(most << 16, most & 0xFFFF0000u);
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  auto with = [&](auto ctrl) { v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl.value, 0xF, 0xF, false)); };
  with(std::integral_constant<int, 0x111>{});        // row_shr 1, 2, 4, 8
  with(std::integral_constant<int, 0x112>{});
  with(std::integral_constant<int, 0x114>{});
  with(std::integral_constant<int, 0x118>{});
  with(std::integral_constant<int, 0x142>{});        // row_bcast 15, 31
  with(std::integral_constant<int, 0x143>{});
  return __builtin_amdgcn_readlane(v, 63);
}

// Codes of 8 elements at a page's exponent b < 255.  int8: the fma rounds x / scale to an integer in the low bits of
// 1.5 2^23, ties to even.
template <int FMT, typename T> __device__ __forceinline__ u32x2 quantise8(const Raw8<T>& r, int b) {
  if constexpr (FMT == SARA_KV8_INT8) {
    const float inv = ldexpf(1.f, 127 - b), magic = 12582912.f;
    float f[8];
    uint32_t c[8];
    unpack8(r, f);
#pragma unroll
    for (int q = 0; q < 8; ++q) c[q] = __float_as_uint(fmaf(f[q], inv, magic));
    u32x2 w;
#pragma unroll
    for (int q = 0; q < 2; ++q)
      w[q] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(c[4 * q + 3], c[4 * q + 2], 0x0C0C0400u),
                                   __builtin_amdgcn_perm(c[4 * q + 1], c[4 * q], 0x0C0C0400u), 0x05040100u);
    return w;
  } else {
    const float inv = ldexpf(1.f, 127 - b);
    float f[8];
    unpack8(r, f);
#pragma unroll
    for (int q = 0; q < 8; ++q) f[q] *= inv;
    return u32x2{encode4<FMT>(f[0], f[1], f[2], f[3]), encode4<FMT>(f[4], f[5], f[6], f[7])};
  }
}

template <typename T> __device__ __forceinline__ void store8(T* p, const float* f);
template <> __device__ __forceinline__ void store8<uint16_t>(uint16_t* p, const float* f) {
  *(u32x4*)p = u32x4{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])};
}
template <> __device__ __forceinline__ void store8<float>(float* p, const float* f) {
  *(f32x4*)p = f32x4{f[0], f[1], f[2], f[3]};
  *(f32x4*)(p + 4) = f32x4{f[4], f[5], f[6], f[7]};
}

// A wave has a page's 16 rows of one head in registers: their largest magnitude gives the scale, the codes follow with no
// second read, and a page that keeps earlier tokens is re-rounded by the same wave.  Bound by memory on a pool (256
// prompts of 128-512 tokens, 21 us; with the read back 50 us, 4.98 TB/s) and by its load chain on a token (2.2 us).
template <int HD, int FMT, typename T>
__global__ __launch_bounds__(256) void k_kv8_write(sara_kv8_cache c, KvRows src, const int32_t* __restrict__ pages,
    int max_pages, const int32_t* __restrict__ start, const int32_t* __restrict__ off, int n_seqs, int n_rows) {
  typedef PageLanes<HD> PL;
  PageUnit u;
  if (!page_unit(blockIdx.x * 4 + (threadIdx.x >> 6), c.n_kv_heads, start, off, n_seqs, n_rows, u)) return;
  if (u.start < 0 || u.page >= max_pages) return;
  const int id = pages[(size_t)u.seq * max_pages + u.page];
  if (id < 0 || id >= c.n_pages) return;
  const int lane = threadIdx.x & 63, d0 = 8 * (lane % PL::TPR), row = lane / PL::TPR;
  const T* x = (const T*)(u.is_v ? src.v : src.k) + (u.is_v ? src.v_head : src.k_head) * u.head + d0;
  const int64_t stride = u.is_v ? src.v_row : src.k_row;
  const int t0 = 16 * u.page - u.start;                 // row of the page's slot 0, below 0 where it keeps tokens
  const size_t block = (size_t)id * c.n_kv_heads + u.head;
  uint8_t* codes = (uint8_t*)(u.is_v ? c.v : c.k) + (block * kBlockTok + row) * HD + d0;
  uint8_t* exp = (u.is_v ? c.v_exp : c.k_exp) + block;
  Raw8<T> r[PL::NI];
  uint32_t most = 0;
#pragma unroll
  for (int j = 0; j < PL::NI; ++j) {
    const int t = t0 + j * PL::RPI + row;
    r[j] = load_raw8<T>(x + (size_t)(u.r0 + min(max(t, 0), u.len - 1)) * stride);   // rows outside repeat one of the page's
  }
#pragma unroll
  for (int j = 0; j < PL::NI; ++j) most = magnitude(most, r[j]);
  int b = exponent_of<FMT>(wave_max(magnitude_bits<T>(most)));
  if (t0 < 0) {
    const int old = *exp;
    b = max(b, old);
    if (b > old && b < 255) {
#pragma unroll
      for (int j = 0; j < PL::NI; ++j)
        if (t0 + j * PL::RPI + row < 0) {
          u32x2* p = (u32x2*)(codes + (size_t)j * PL::RPI * HD);
          const u32x2 w = *p;
          float g[8];
          decode4<FMT>(w.x, g);
          decode4<FMT>(w.y, g + 4);
#pragma unroll
          for (int q = 0; q < 8; ++q) g[q] = ldexpf(g[q], old - b);
          *p = u32x2{encode4<FMT>(g[0], g[1], g[2], g[3]), encode4<FMT>(g[4], g[5], g[6], g[7])};
        }
    }
  }
#pragma unroll
  for (int j = 0; j < PL::NI; ++j) {
    const int t = t0 + j * PL::RPI + row;
    if (t >= 0 && t < u.len) *(u32x2*)(codes + (size_t)j * PL::RPI * HD) = b == 255 ? u32x2{0u, 0u} : quantise8<FMT, T>(r[j], b);
  }
  if (lane == 0) *exp = (uint8_t)b;
}

// The same units as the write.  Rows of positions without a page are 0.  The pool above: 21 us.
template <int HD, int FMT, typename T>
__global__ __launch_bounds__(256) void k_kv8_read(sara_kv8_cache c, KvRows dst, const int32_t* __restrict__ pages,
    int max_pages, const int32_t* __restrict__ start, const int32_t* __restrict__ off, int n_seqs, int n_rows) {
  typedef PageLanes<HD> PL;
  PageUnit u;
  if (!page_unit(blockIdx.x * 4 + (threadIdx.x >> 6), c.n_kv_heads, start, off, n_seqs, n_rows, u)) return;
  const int id = u.page >= 0 && u.page < max_pages ? pages[(size_t)u.seq * max_pages + u.page] : -1;
  const bool have = id >= 0 && id < c.n_pages;
  const int lane = threadIdx.x & 63, d0 = 8 * (lane % PL::TPR), row = lane / PL::TPR;
  const size_t block = (size_t)(have ? id : 0) * c.n_kv_heads + u.head;
  const uint8_t* codes = (const uint8_t*)(u.is_v ? c.v : c.k) + (block * kBlockTok + row) * HD + d0;
  const int b = (u.is_v ? c.v_exp : c.k_exp)[block];
  const float scale = exponent_scale(b);
  T* y = (T*)(u.is_v ? dst.v : dst.k) + (u.is_v ? dst.v_head : dst.k_head) * u.head + d0;
  const int64_t stride = u.is_v ? dst.v_row : dst.k_row;
  const int t0 = 16 * u.page - u.start;
#pragma unroll
  for (int j = 0; j < PL::NI; ++j) {
    const int t = t0 + j * PL::RPI + row;
    if (t < 0 || t >= u.len) continue;
    float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (have) {
      const u32x2 w = *(const u32x2*)(codes + (size_t)j * PL::RPI * HD);
      decode4<FMT>(w.x, f);
      decode4<FMT>(w.y, f + 4);
#pragma unroll
      for (int q = 0; q < 8; ++q) f[q] *= scale;
    }
    store8<T>(y + (size_t)(u.r0 + t) * stride, f);
  }
}

// ---------------------------------------------------------------------------
// attention
// ---------------------------------------------------------------------------
struct AttnArgs {
  const void* q;
  void* out;
  int64_t q_row, q_head, o_row, o_head;   // strides in elements
  const int32_t *pages, *ctx, *off;
  int max_pages, max_ctx, n_seqs, n_rows, hq;
  int splits, pps, splits_tile, pps_tile; // most splits of a row and pages a split, in the two kernels below
  float scale_log2;
  // partial results (HD numerators, maximum, sum): k_kv8_attn's [sequence][KV head][column][split], k_kv8_attn_tile's
  // [row][head][split]
  float *part, *part_tile;
};

// fp32 as a sum of P bf16 numbers: 8 bits (bf16 inputs are one exactly), 16, or 24
template <int P> __device__ __forceinline__ void split_bf16(float a, float b, uint32_t* w) {
#pragma unroll
  for (int i = 0; i < P; ++i) {
    w[i] = pack_bf16(a, b);
    if (i + 1 == P) break;
    asm("" : "+v"(w[i]));                                  // else the compiler rounds `a` a second time for its part
    a -= __uint_as_float(w[i] << 16);
    b -= __uint_as_float(w[i] & 0xFFFF0000u);
  }
}

// byte i of four words to word i
__device__ __forceinline__ void transpose4(uint32_t* r) {
  const uint32_t a = __builtin_amdgcn_perm(r[1], r[0], 0x05010400u), b = __builtin_amdgcn_perm(r[1], r[0], 0x07030602u);
  const uint32_t c = __builtin_amdgcn_perm(r[3], r[2], 0x05010400u), d = __builtin_amdgcn_perm(r[3], r[2], 0x07030602u);
  r[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
  r[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
  r[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
  r[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

// Sequences with more columns (query tokens x heads of a KV head) than this go through k_kv8_attn_tile.
constexpr int kFewColumns = 32;
constexpr int kTileWaves = 4;          // one for each page of a key block

// The value m subtracted from a column's scores follows them only once they pass it, and is then set this much above them
// (base 2): weights stay at or below 1, and most key blocks leave the sums where they are (16 sequences of 256 queries
// over 4,000 tokens: 226 us, against 229 with the maximum itself).
constexpr float kSlack = 8.f;

template <int HD> struct FewLds {
  float m_w[4][16], l_w[4][16], o_w[4][16][HD + 4];
};

// Block (16 columns of one sequence and KV head, split): column = query token x head of the group.  The 4
// waves take the split's pages in pairs, wave w pairs w, w + 4, ...; the next pair's K codes are loaded once
// the scores are there, its V codes at the end.  Per pair:
//   S^T = K q^T   codes as bf16 (exact), the page's scale on the fp32 scores
//   online softmax per column in base 2 over the 4 lanes that hold it; m, l: the value that was subtracted
//                 and the sum
//   O^T += V^T P^T   the score registers are the B operand (4 tokens of each page a lane); V's bytes
//                 are transposed in registers; P, times the page's V scale, enters as PP bf16 parts
//                 (2: 2^-17 of a weight; 3 for fp32 queries), so the product adds no rounding of its own
// Queries of fp32 enter as 3 bf16 parts.  A column without a visible key gives 0.
// What bounds it is the pages' memory traffic from some 100 rows on (512 rows at 256-1,700 tokens: 51 us, 5.1 TB/s; 32
// rows at 3,000-4,600 in splits: 15.7 us, 4.0 TB/s), below that its load round trips (one row at 333: 7.1 us).  Blocks of
// 8 waves take 6.7 us there, but 22 for the 32 rows' 18.2 with the join.
// A weight times its page's scale is held to bf16's range: below 2^-126 it may count as 0, which matters where all of V is
// below about 1e-30 (at 1e-24 fp32 queries lose nothing).
template <int HD, int FMT, typename T>
__device__ __forceinline__ void attn_few(const sara_kv8_cache& c, const AttnArgs& a, FewLds<HD>& lds, int bx, int split) {
  constexpr int NK = HD / 64, NT = HD / 16, DV = HD / 16;   // 16-byte K loads, dim tiles, V dims a lane
  constexpr int QP = sizeof(T) == 2 ? 1 : 3, PP = sizeof(T) == 2 ? 2 : 3;
  auto &m_w = lds.m_w, &l_w = lds.l_w;
  auto& o_w = lds.o_w;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int col = lane & 15, grp = lane >> 4;
  const int hkv = c.n_kv_heads, G = a.hq / hkv;
  const int item = bx / hkv, g = bx - item * hkv;
  const int tiles = a.off ? kFewColumns / 16 : (G + 15) / 16;
  const int seq = item / tiles, c0 = 16 * (item - seq * tiles);
  int r0, r1;
  seq_rows(a.off, seq, a.n_rows, r0, r1);
  const int n_cols = (r1 - r0) * G;
  if (c0 >= n_cols || (a.off && n_cols > kFewColumns)) return;
  const int p0 = split * a.pps;
  // ids of 32 of the wave's page pairs, one a lane; the first are loaded beside the context's length
  const int32_t* table = a.pages + (size_t)seq * a.max_pages;
  auto load_ids = [&](int it) { return table[min(p0 + 2 * wave + 8 * (it + (lane >> 1)) + (lane & 1), a.max_pages - 1)]; };
  int ids = load_ids(0);
  const int ctx = max(a.ctx[seq], 0);
  const bool too_long = ctx > a.max_ctx;                 // more than the launch was sized for: the rows are NaN
  const int np = too_long ? 0 : (ctx + 15) >> 4;
  const int p1 = min(np, p0 + a.pps);
  if (p0 >= p1 && split > 0) return;
  // this lane's column: query row and head, and how many keys it sees
  const int cc = min(c0 + col, n_cols - 1), qt = cc / G, head = g * G + cc - qt * G;
  const int before = ctx - (r1 - r0);                    // keys before the first query (below 0: its row sees none)
  const int seen = before + qt + 1;
  const int seen_all = before + c0 / G + 1;              // keys that every column sees
  u32x4 qf[QP][2 * NK];
  {
    const T* q = (const T*)a.q + (size_t)(r0 + qt) * a.q_row + (size_t)head * a.q_head;
#pragma unroll
    for (int i = 0; i < 2 * NK; ++i) {
      const T* qp = q + 64 * (i >> 1) + 16 * grp + 8 * (i & 1);
      if constexpr (QP == 1) {
        qf[0][i] = *(const u32x4*)qp;
      } else {
        float f[8];
        load8<T>(qp, f);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t w[QP];
          split_bf16<QP>(f[2 * j], f[2 * j + 1], w);
#pragma unroll
          for (int p = 0; p < QP; ++p) qf[p][i][j] = w[p];
        }
      }
    }
  }
  const int n_it = p1 <= p0 + 2 * wave ? 0 : (p1 - p0 - 2 * wave + 7) / 8;
  u32x4 kr[2][NK];
  uint32_t vr[2][4][DV / 4];
  int ke[2], ve[2];
  size_t v_block[2];
  bool have[2], v_have[2];
  // K codes and the exponents of pair `it`; its V codes follow by load_v, once V's registers are free
  auto load_k = [&](int it) {
    if (it > 0 && (it & 31) == 0) ids = load_ids(it);
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int id = __builtin_amdgcn_readlane(ids, 2 * (it & 31) + p);
      have[p] = p0 + 2 * wave + 8 * it + p < p1 && id >= 0 && id < c.n_pages;
      v_block[p] = (size_t)(have[p] ? id : 0) * hkv + g;
      const uint8_t* kp = (const uint8_t*)c.k + (v_block[p] * kBlockTok + col) * HD + 16 * grp;
#pragma unroll
      for (int i = 0; i < NK; ++i) kr[p][i] = *(const u32x4*)(kp + 64 * i);
      ke[p] = c.k_exp[v_block[p]];
      ve[p] = c.v_exp[v_block[p]];
    }
  };
  auto load_v = [&]() {
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      v_have[p] = have[p];
      const uint8_t* vp = (const uint8_t*)c.v + (v_block[p] * kBlockTok + 4 * grp) * HD + DV * col;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int w = 0; w < DV / 4; ++w) vr[p][j][w] = *(const uint32_t*)(vp + j * HD + 4 * w);
    }
  };
  float m = -INFINITY, l = 0.f;
  f32x4 o[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (n_it > 0) {
    load_k(0);
    __builtin_amdgcn_sched_barrier(0);                     // K first: a wait for it must not be one for V (9% at 512 rows)
    load_v();
  }
  for (int it = 0; it < n_it; ++it) {
    f32x4 s[2];
    float vs[2];
    float mx = m;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      s[p] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 2 * NK; ++i) {
        const u32x2 x = codes_bf16<FMT>(kr[p][i >> 1][2 * (i & 1)]), y = codes_bf16<FMT>(kr[p][i >> 1][2 * (i & 1) + 1]);
        const bf16x8 kf = __builtin_bit_cast(bf16x8, u32x4{x.x, x.y, y.x, y.y});
#pragma unroll
        for (int qp = QP - 1; qp >= 0; --qp)
          s[p] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, __builtin_bit_cast(bf16x8, qf[qp][i]), s[p], 0, 0, 0);
      }
      // a page of NaN scale in K or V makes the scores of its keys NaN, so it reaches only the columns that
      // see them; its V then counts as 0
      const bool bad = ke[p] == 255 || ve[p] == 255;
      const float ks = bad ? __uint_as_float(0x7FC00000u) : ldexpf(a.scale_log2, ke[p] - 127);
      vs[p] = bad ? 0.f : ldexpf(1.f, ve[p] - 127);
      s[p] *= ks;
    }
    if (it + 1 < n_it) load_k(it + 1);
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int k0 = 16 * (p0 + 2 * wave + 8 * it + p);
      if (!v_have[p] || k0 + 16 > seen_all) {
        const int left = v_have[p] ? seen - k0 - 4 * grp : 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) s[p][q] = q < left ? s[p][q] : -INFINITY;
        // codes past the sequence's last token may be anything
        const int live = v_have[p] ? ctx - k0 - 4 * grp : 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int w = 0; w < DV / 4; ++w) vr[p][j][w] = j < live ? vr[p][j][w] : 0u;
      }
      mx = fmaxf(mx, fmaxf(fmaxf(s[p][0], s[p][1]), fmaxf(s[p][2], s[p][3])));
    }
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    if (__any(mx > m)) {
      const float to = mx > m ? mx + kSlack : m;
      const float al = __builtin_amdgcn_exp2f(m - (to == -INFINITY ? 0.f : to));
      l *= al;
#pragma unroll
      for (int i = 0; i < NT; ++i) o[i] *= al;
      m = to;
    }
    const float sub = m == -INFINITY ? 0.f : m;           // nothing seen yet: every weight is 0
    u32x4 pf[PP];
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int q = 0; q < 4; q += 2) {
        const float e0 = __builtin_amdgcn_exp2f(s[p][q] - sub), e1 = __builtin_amdgcn_exp2f(s[p][q + 1] - sub);
        l += e0 + e1;
        uint32_t w[PP];
        split_bf16<PP>(e0 * vs[p], e1 * vs[p], w);
#pragma unroll
        for (int i = 0; i < PP; ++i) pf[i][2 * p + (q >> 1)] = w[i];
      }
#pragma unroll
    for (int w = 0; w < DV / 4; ++w) {
      uint32_t x[4] = {vr[0][0][w], vr[0][1][w], vr[0][2][w], vr[0][3][w]};
      uint32_t y[4] = {vr[1][0][w], vr[1][1][w], vr[1][2][w], vr[1][3][w]};
      transpose4(x);
      transpose4(y);
#pragma unroll
      for (int i = 0; i < 4; ++i) {                       // dim DV col + 4 w + i of tile 4 w + i
        const u32x2 u = codes_bf16<FMT>(x[i]), v = codes_bf16<FMT>(y[i]);
        const bf16x8 vf = __builtin_bit_cast(bf16x8, u32x4{u.x, u.y, v.x, v.y});
#pragma unroll
        for (int p = PP - 1; p >= 0; --p)
          o[4 * w + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, __builtin_bit_cast(bf16x8, pf[p]), o[4 * w + i], 0, 0, 0);
      }
    }
    if (it + 1 < n_it) load_v();
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  // join the waves: lane (col, grp) holds dims DV (4 grp + q) + t of its column
  if (grp == 0) { m_w[wave][col] = m; l_w[wave][col] = l; }
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int t = 0; t < NT; t += 4)
      *(f32x4*)&o_w[wave][col][DV * (4 * grp + q) + t] = f32x4{o[t][q], o[t + 1][q], o[t + 2][q], o[t + 3][q]};
  __syncthreads();
  constexpr int TPC = HD / 4, CPP = 256 / TPC;
  const int cols = min(16, n_cols - c0);
  for (int x = (int)threadIdx.x / TPC; x < cols; x += CPP) {
    const int d4 = 4 * ((int)threadIdx.x % TPC);
    const float mx = fmaxf(fmaxf(m_w[0][x], m_w[1][x]), fmaxf(m_w[2][x], m_w[3][x]));
    const float sub = mx == -INFINITY ? 0.f : mx;
    f32x4 num = {0.f, 0.f, 0.f, 0.f};
    float den = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float wt = __builtin_amdgcn_exp2f(m_w[w][x] - sub);
      num += wt * *(const f32x4*)&o_w[w][x][d4];
      den += wt * l_w[w][x];
    }
    const int t = (c0 + x) / G, h = g * G + (c0 + x) - t * G;
    if (np <= a.pps) {
      T* dst = (T*)a.out + (size_t)(r0 + t) * a.o_row + (size_t)h * a.o_head + d4;
      float f[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) f[q] = too_long ? __uint_as_float(0x7FC00000u) : den == 0.f ? 0.f : num[q] / den;
      if constexpr (sizeof(T) == 2) *(uint2*)dst = make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]));
      else *(f32x4*)dst = f32x4{f[0], f[1], f[2], f[3]};
    } else {
      const int slots = a.off ? kFewColumns : G;
      float* dst = a.part + ((((size_t)seq * hkv + g) * slots + c0 + x) * a.splits + split) * (HD + 2);
      *(f32x2*)(dst + d4) = f32x2{num[0], num[1]};
      *(f32x2*)(dst + d4 + 2) = f32x2{num[2], num[3]};
      if (d4 == 0) *(f32x2*)(dst + HD) = f32x2{mx, den};
    }
  }
}

template <int HD> struct TileLds {
  u32x4 kf[2][2 * (HD / 16) * 64], vf[2][4 * (HD / 32) * 64];
};

// The same attention for sequences of many columns: a block owns 128 of them, a wave 32, and all its waves
// read the same 64-key blocks of K and V from LDS, as bf16 values (code times scale, exact), converted once a block.
// Per key block and wave:
//   S^T = K q^T    v_mfma_f32_32x32x16_bf16: lane (col l % 32, h = l / 32) gets keys 8 (i / 4) + 4 h + i % 4, i < 16
//   online softmax in base 2, a column in two lanes; O is rescaled only when some column's maximum moved
//   O^T += V^T P^T    scores 0..7 and 8..15 of a lane are the B operands of two 16-key steps (keys 4 h + 0..3 and
//                  8 + 4 h + 0..3 of a page), P in PP bf16 parts as above
// LDS holds the operands in fragment order.  K: 16 dims of a key are one 16-byte load and the 16 bytes of two lanes;
// slots are xor-ed with the dim step so that the 8 threads of a token row write to different banks.  V: 4 dims of 8
// tokens are transposed in registers; row r of a 32-dim tile is dim 4 (r % 8) + r / 8, which spreads the writes and
// leaves a lane 16 consecutive dims of the output.
// What bounds it is VALU issue: a wave and key block has 473 vector instructions (e4m3: 349), 32 exponentials among them,
// which take 60% of the kernel's cycles (51%), beside 48 MFMAs of 32 cycles in 40% (44%).  So both run side by side: the codes of block kb + 1 wait in registers and become bf16 in LDS between the score
// MFMAs of block kb, their successors load behind them, and the weights of 16 keys are made between the MFMAs of the
// 16 before.  16 sequences of 256 queries, the last of 4,000 tokens, 16 heads: 215 us (605 TFLOP/s; e4m3 197); one prompt
// of 4,590: 166 (520), against 182 with conversion, softmax and MFMAs one after the other.  Blocks of 8 waves over 256
// columns convert half as much each; they are level on other sizes and lose there (360 us, against 233 of blocks of 4 in
// that version of the loop).
// Queries of fp32 have 96 MFMAs (three parts of q, three of a weight) beside 718 vector instructions, and 256 registers: one
// block a CU, whose one wave a SIMD overlaps little: vector issue 43%, MFMAs 40%.  Three prompts of 1,100-4,590: 408 us,
// against 218 in bf16.
template <int HD, int FMT, typename T>
__device__ __forceinline__ void attn_tile(const sara_kv8_cache& c, const AttnArgs& a, TileLds<HD>& lds, int bx, int n_bx, int split) {
  constexpr int NW = kTileWaves, NKS = HD / 16, NDT = HD / 32;
  constexpr int QP = sizeof(T) == 2 ? 1 : 3, PP = sizeof(T) == 2 ? 2 : 3;
  constexpr int KU = NKS / NW, KR = 64 / NKS;                        // staging: K units a thread, token rows a unit of a wave
  typedef float f32x16 __attribute__((ext_vector_type(16)));
  auto &kf = lds.kf;
  auto &vf = lds.vf;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 31, h = lane >> 5;
  const int hkv = c.n_kv_heads, G = a.hq / hkv;
  const int item = n_bx / hkv - 1 - bx / hkv, g = bx % hkv;          // long tiles first
  const SeqRows sr = find_seq<32 * NW>(a.off, a.ctx, a.n_seqs, a.n_rows, item, G, 1);
  const int seq = sr.seq, r0 = sr.r0, r1 = sr.r1;
  if (seq < 0 || item < sr.first) return;
  const int n_cols = (r1 - r0) * G, c0 = 32 * NW * (item - sr.first);
  if (c0 >= n_cols || n_cols <= kFewColumns) return;
  const int ctx = max(sr.value, 0);
  const bool too_long = ctx > a.max_ctx;
  const int np = too_long ? 0 : (ctx + 15) >> 4;
  const int p0 = split * a.pps_tile;
  if (p0 >= np && split > 0) return;
  const int before = ctx - (r1 - r0);
  const int c_last = min(c0 + 32 * NW, n_cols) - 1;
  const int keys = min(max(before + c_last / G + 1, 0), ctx);       // keys that some column of the block sees
  const int p1 = min(min(np, p0 + a.pps_tile), (keys + 15) >> 4);
  const int nkb = p1 > p0 ? (p1 - p0 + 3) >> 2 : 0;
  const int wc0 = c0 + 32 * wave;
  const bool live = wc0 < n_cols;
  const int cc = min(wc0 + col, n_cols - 1), qt = cc / G, head = g * G + cc - qt * G;
  const int seen = live ? before + qt + 1 : 0;                      // keys this lane's column sees
  const int w_seen = live ? before + min(wc0 + 31, n_cols - 1) / G + 1 : 0;   // that some column of the wave sees
  const int w_all = before + wc0 / G + 1;                           // that every column of the wave sees
  // a negative scale becomes the sign of q; the floor keeps a masked -inf from meeting a scale of 0
  const float sl2 = fmaxf(fabsf(a.scale_log2), 1e-37f);
  u32x4 qf[QP][NKS];
  {
    const uint32_t flip = a.scale_log2 < 0.f ? 0x80008000u : 0u;
    const T* q = (const T*)a.q + (size_t)(r0 + qt) * a.q_row + (size_t)head * a.q_head + 8 * h;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) {
      if constexpr (QP == 1) {
        qf[0][ks] = *(const u32x4*)(q + 16 * ks) ^ flip;
      } else {
        float f[8];
        load8<T>(q + 16 * ks, f);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t w[QP];
          split_bf16<QP>(f[2 * j], f[2 * j + 1], w);
#pragma unroll
          for (int p = 0; p < QP; ++p) qf[p][ks][j] = w[p] ^ flip;
        }
      }
    }
  }
  const int32_t* table = a.pages + (size_t)seq * a.max_pages;
  // lane i: page i of a stretch of 64 (16 key blocks), its exponent bytes (0x10000: no page, 0x20000: NaN, 0x40000: values may be inf)
  int ids = 0, meta = 0;
  // A wave stages KR token rows of K at a time, all of one page, and the V of one page: pages, exponents and addresses
  // are scalars.  K: lane (token row lane / NKS, 16 dims).  V: lane (8 tokens v_half, 4 dims 4 v_dim).
  const int k_row = lane / NKS, k_step = lane % NKS, v_dim = lane % (HD / 4), v_half = lane / (HD / 4) & 1;
  u32x4 kr[KU];
  uint32_t vr[8];
  int km[KU], vm;
  auto first_row = [&](int x) { return (wave + NW * x) * KR; };      // of the wave's unit x
  auto load = [&](int kb) {
    if ((kb & 15) == 0) {
      const int pg = p0 + 4 * kb + lane;
      const int id = pg < p1 ? table[pg] : -1;
      const bool have = id >= 0 && id < c.n_pages;
      ids = have ? id : 0;
      const size_t block = (size_t)ids * hkv + g;
      const int ke = c.k_exp[block], ve = c.v_exp[block];
      meta = ke | ve << 8 | (have ? 0 : 0x10000) | (ke == 255 || ve == 255 ? 0x20000 : 0) |
             (max(ke, ve) >= kFirstInf<FMT> ? 0x40000 : 0);
    }
    const int at = 4 * (kb & 15);
    auto page = [&](const void* codes, int pg, int& info) {
      info = __builtin_amdgcn_readlane(meta, at + pg);
      return (const uint8_t*)codes + ((size_t)__builtin_amdgcn_readlane(ids, at + pg) * hkv + g) * (kBlockTok * HD);
    };
#pragma unroll
    for (int x = 0; x < KU; ++x) {
      const uint8_t* kp = page(c.k, first_row(x) >> 4, km[x]) + (first_row(x) & 15) * HD;
      kr[x] = *(const u32x4*)(kp + (k_row * HD + 16 * k_step));
    }
    const uint8_t* vp = page(c.v, wave, vm);
#pragma unroll
    for (int j = 0; j < 8; ++j) vr[j] = *(const uint32_t*)(vp + ((j + 4 * (j >> 2) + 4 * v_half) * HD + 4 * v_dim));
  };
  // The loaded codes go to LDS in PIECES pieces of about ten instructions, after `settle`.  A value that rounded past the
  // largest finite number must not enter LDS as inf: a weight of 0, or a q of 0, would make it NaN for columns that do not
  // see its key or its dim.
  constexpr int PIECES = 4 * KU + 8;
  float k_scale[KU], v_scale;
  u32x4 w_k, w_v;
  auto settle = [&](int kb) {
    int large = vm & 0x40000;
#pragma unroll
    for (int x = 0; x < KU; ++x) large |= km[x] & 0x40000;
    const int tokens = (vm & 0x30000) ? 0 : min(ctx - 16 * (p0 + 4 * kb + wave), 16);
    if ((large ? 0 : tokens) < 16) {                       // one branch for all that is rare (two cost 1.5% of a prompt)
      if (large) {
#pragma unroll
        for (int x = 0; x < KU; ++x)
          if ((km[x] & 255) >= kFirstInf<FMT>)
#pragma unroll
            for (int q = 0; q < 4; ++q) kr[x][q] = finite_codes<FMT>(kr[x][q], km[x] & 255);
        if ((vm >> 8 & 255) >= kFirstInf<FMT>)
#pragma unroll
          for (int j = 0; j < 8; ++j) vr[j] = finite_codes<FMT>(vr[j], vm >> 8 & 255);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) vr[j] = j + 4 * (j >> 2) + 4 * v_half < tokens ? vr[j] : 0u;
    }
#pragma unroll
    for (int x = 0; x < KU; ++x) {
      // a NaN page (its K or its V) is seen through its keys' scores: a NaN scale, or the code of NaN
      const bool bad = km[x] & 0x20000;
      if (FMT == SARA_KV8_E4M3 && bad) kr[x] = u32x4{0x7F7F7F7Fu, 0x7F7F7F7Fu, 0x7F7F7F7Fu, 0x7F7F7F7Fu};
      k_scale[x] = bad ? (FMT == SARA_KV8_E4M3 ? 1.f : __uint_as_float(0x7FC00000u)) : ldexpf(1.f, (km[x] & 255) - 127);
    }
    v_scale = (vm & 0x20000) ? 0.f : ldexpf(1.f, (vm >> 8 & 255) - 127);
  };
  auto store = [&](int i, int buf) {
    if (i < 4 * KU) {
      const int x = i >> 2, q = i & 3, r = first_row(x) + k_row;
      const u32x2 y = values_bf16<FMT>(kr[x][q], k_scale[x]);
      w_k[2 * (q & 1)] = y.x;
      w_k[2 * (q & 1) + 1] = y.y;
      if (q & 1) kf[buf][((r >> 5) * NKS + k_step) * 64 + 32 * (q >> 1) + ((r & 31) ^ (k_step & 7))] = w_k;
      return;
    }
    const int j = (i - 4 * KU) >> 1, half = i & 1;         // 4 KU is even
    if (i == 4 * KU) {
      transpose4(vr);
      transpose4(vr + 4);
    }
    const u32x2 y = values_bf16<FMT>(vr[4 * half + j], v_scale);
    w_v[2 * half] = y.x;
    w_v[2 * half + 1] = y.y;
    if (half && (HD == 128 || lane < HD / 2)) vf[buf][(wave * NDT + (v_dim >> 3)) * 64 + 32 * v_half + 8 * j + (v_dim & 7)] = w_v;
  };
  float m = -INFINITY, l = 0.f;
  f32x16 o[NDT];
#pragma unroll
  for (int t = 0; t < NDT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
  auto v_frag = [&](int buf, int st, int t) { return vf[buf][(st * NDT + t) * 64 + lane]; };
  // Scores of a key block, each MFMA beside a piece of the next block's way to LDS.  LDS reads run half of the MFMAs ahead.
  f32x16 s[2];
  u32x4 vv[2][NDT];
  auto scores = [&](int buf) {
    auto k_frag = [&](int b, int ks) { return kf[buf][(b * NKS + ks) * 64 + 32 * h + (col ^ (ks & 7))]; };
    u32x4 kk[2][NKS];
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) kk[0][ks] = k_frag(0, ks);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[b][i] = 0.f;
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) {
        const int n = b * NKS + ks;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int p = QP - 1; p >= 0; --p)
          s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kk[b][ks]), __builtin_bit_cast(bf16x8, qf[p][ks]),
                                                         s[b], 0, 0, 0);
        if (b == 0) kk[1][ks] = k_frag(1, ks);
        else if (ks < NDT) vv[0][ks] = v_frag(buf, 0, ks);
#pragma unroll
        for (int i = PIECES * n / (2 * NKS); i < PIECES * (n + 1) / (2 * NKS); ++i) store(i, buf ^ 1);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto compute = [&](int kb, int buf, int absent) {
    const int k0 = 16 * (p0 + 4 * kb);
    if (k0 + 64 > w_all || absent) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const bool in = k0 + 32 * b + 8 * (i >> 2) + 4 * h + (i & 3) < seen && !(absent >> (2 * b + (i >> 3)) & 1);
          s[b][i] = in ? s[b][i] : -INFINITY;
        }
    }
    float mx = s[0][0];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[b][i]);
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    mx = fmaxf(m, mx * sl2);
    if (__any(mx > m)) {
      const float to = mx > m ? mx + kSlack : m;
      const float al = __builtin_amdgcn_exp2f(m - (to == -INFINITY ? 0.f : to));
      l *= al;
#pragma unroll
      for (int t = 0; t < NDT; ++t) o[t] *= al;
      m = to;
    }
    const float sub = m == -INFINITY ? 0.f : m;
    // weights of keys pair j of step st, in PP bf16 parts
    u32x4 pf[2][PP];
    auto weights = [&](int st, int j) {
      const int i = 8 * (st & 1) + 2 * j;
      const float e0 = __builtin_amdgcn_exp2f(fmaf(s[st >> 1][i], sl2, -sub));
      const float e1 = __builtin_amdgcn_exp2f(fmaf(s[st >> 1][i + 1], sl2, -sub));
      l += e0 + e1;
      uint32_t w[PP];
      split_bf16<PP>(e0, e1, w);
#pragma unroll
      for (int p = 0; p < PP; ++p) pf[st & 1][p][j] = w[p];
    };
#pragma unroll
    for (int j = 0; j < 4; ++j) weights(0, j);
    // a step's MFMAs in four groups, each with a quarter of the next step's weights
    constexpr int M = NDT * PP;
#pragma unroll
    for (int st = 0; st < 4; ++st) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        __builtin_amdgcn_sched_barrier(0);
        if (st < 3 && j < NDT) vv[(st + 1) & 1][j] = v_frag(buf, st + 1, j);
#pragma unroll
        for (int n = M * j / 4; n < M * (j + 1) / 4; ++n) {
          const int t = n % NDT, p = PP - 1 - n / NDT;
          o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vv[st & 1][t]),
                                                         __builtin_bit_cast(bf16x8, pf[st & 1][p]), o[t], 0, 0, 0);
        }
        if (st < 3) weights(st + 1, j);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // bit i: page i of the key block has no page id
  auto absent_pages = [&](int kb) { return (int)(__ballot(meta & 0x10000) >> (4 * (kb & 15)) & 15); };
  // Key block kb is in LDS, kb + 1 in registers; kb + 2 is loaded once those are free.
  int absent = 0, next_absent = 0;
  if (nkb > 0) {
    load(0);
    absent = absent_pages(0);
    settle(0);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) store(i, 0);
    if (nkb > 1) {
      load(1);
      next_absent = absent_pages(1);
    }
  }
  __syncthreads();
  for (int kb = 0; kb < nkb; ++kb) {
    const int buf = kb & 1;
    const bool mine = 16 * (p0 + 4 * kb) < w_seen;         // else no column of the wave sees the block
    settle(kb + 1);                                        // past the last block: stale codes, to a buffer that is not read
    if (mine) {
      scores(buf);
    } else {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) store(i, buf ^ 1);
    }
    const int now_absent = absent;
    absent = next_absent;
    if (kb + 2 < nkb) {
      load(kb + 2);
      next_absent = absent_pages(kb + 2);
    }
    if (mine) compute(kb, buf, now_absent);
    __syncthreads();
  }
  l += __shfl_xor(l, 32, 64);
  if (!live || wc0 + col >= n_cols) return;
  const float inv = too_long ? __uint_as_float(0x7FC00000u) : l == 0.f ? 0.f : 1.f / l;
  const bool whole = np <= a.pps_tile;
  T* out = (T*)a.out + (size_t)(r0 + qt) * a.o_row + (size_t)head * a.o_head + 16 * h;
  float* part = a.part_tile + (((size_t)(r0 + qt) * a.hq + head) * a.splits_tile + split) * (HD + 2);
#pragma unroll
  for (int t = 0; t < NDT; ++t) {
    float f[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) f[e] = o[t][4 * (e & 3) + (e >> 2)];
    if (whole) {
#pragma unroll
      for (int e = 0; e < 16; ++e) f[e] *= inv;
      store8<T>(out + 32 * t, f);
      store8<T>(out + 32 * t + 8, f + 8);
    } else {
#pragma unroll
      for (int e = 0; e < 16; e += 2) *(f32x2*)(part + 32 * t + 16 * h + e) = f32x2{f[e], f[e + 1]};
    }
  }
  if (!whole && h == 0) *(f32x2*)(part + HD) = f32x2{m, l};
}

template <int HD, int FMT, typename T>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 3 : 2) void k_kv8_attn(sara_kv8_cache c, AttnArgs a) {
  __shared__ __attribute__((aligned(16))) FewLds<HD> lds;
  attn_few<HD, FMT, T>(c, a, lds, blockIdx.x, blockIdx.y);
}
template <int HD, int FMT, typename T>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void k_kv8_attn_tile(sara_kv8_cache c, AttnArgs a) {
  __shared__ __attribute__((aligned(16))) TileLds<HD> lds;
  attn_tile<HD, FMT, T>(c, a, lds, blockIdx.x, gridDim.x, blockIdx.y);
}
// Both in one launch (see launch_kv8_attention): n_tile x splits_tile blocks of tiles, then n_few x splits of few columns.
template <int HD, int FMT, typename T>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void k_kv8_attn_both(sara_kv8_cache c, AttnArgs a, int n_tile, int n_few) {
  __shared__ __attribute__((aligned(16))) union { FewLds<HD> few; TileLds<HD> tile; } lds;
  const int b = blockIdx.x, few = b - n_tile * a.splits_tile;
  if (few < 0) attn_tile<HD, FMT, T>(c, a, lds.tile, b % n_tile, n_tile, b / n_tile);
  else attn_few<HD, FMT, T>(c, a, lds.few, few % n_few, few / n_few);
}

// A block per (row, head) joins the splits of rows that have more than one: its 4 waves take every fourth split,
// kJoin of them in flight, and meet in LDS.  TILE: the rows of k_kv8_attn_tile, found by their number; else those of
// k_kv8_attn, `cols` columns for each sequence and KV head.
constexpr int kJoin = 4;
template <int HD, typename T, bool TILE>
__global__ __launch_bounds__(256) void k_kv8_attn_join(AttnArgs a, int hkv, int cols) {
  constexpr int DL = HD / 64;                            // dims a lane
  __shared__ float m_w[4], l_w[4], o_w[4][HD];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, G = a.hq / hkv;
  int seq, row, h, r0, r1, ctx;
  if (TILE) {
    row = blockIdx.x / a.hq;
    h = blockIdx.x - row * a.hq;
    const SeqRows sr = find_seq<1>(a.off, a.ctx, a.n_seqs, a.n_rows, row, 1, 0);
    ctx = sr.value;
    if (sr.seq < 0 || row < sr.r0 || row >= sr.r1 || (sr.r1 - sr.r0) * G <= kFewColumns) return;
  } else {
    const int gc = blockIdx.x / cols, x = blockIdx.x - gc * cols;
    seq = gc / hkv;
    ctx = a.ctx[seq];
    seq_rows(a.off, seq, a.n_rows, r0, r1);
    const int n_cols = (r1 - r0) * G;
    if (x >= n_cols || (a.off && n_cols > kFewColumns)) return;
    row = r0 + x / G;
    h = (gc - seq * hkv) * G + x % G;
  }
  const int pps = TILE ? a.pps_tile : a.pps;
  const int ns = (((ctx + 15) >> 4) + pps - 1) / pps;
  if (ctx > a.max_ctx || ns <= 1) return;
  const float* p = TILE ? a.part_tile + ((size_t)row * a.hq + h) * a.splits_tile * (HD + 2)
                        : a.part + (size_t)blockIdx.x * a.splits * (HD + 2);
  float m = -INFINITY, l = 0.f, o[DL] = {};
  for (int s0 = wave; s0 < ns; s0 += 4 * kJoin) {
    float pm[kJoin], pl[kJoin], po[kJoin][DL];
#pragma unroll
    for (int i = 0; i < kJoin; ++i) {
      const float* q = p + (size_t)min(s0 + 4 * i, ns - 1) * (HD + 2);
      const f32x2 ml = *(const f32x2*)(q + HD);
      pm[i] = s0 + 4 * i < ns ? ml[0] : -INFINITY;
      pl[i] = ml[1];
      if (DL == 2) {
        const f32x2 v = *(const f32x2*)(q + 2 * lane);
        po[i][0] = v[0];
        po[i][DL - 1] = v[1];
      } else {
        po[i][0] = q[lane];
      }
    }
    float mx = m;
#pragma unroll
    for (int i = 0; i < kJoin; ++i) mx = fmaxf(mx, pm[i]);
    const float sub = mx == -INFINITY ? 0.f : mx;
    const float al = __builtin_amdgcn_exp2f(m - sub);
    l *= al;
#pragma unroll
    for (int d = 0; d < DL; ++d) o[d] *= al;
#pragma unroll
    for (int i = 0; i < kJoin; ++i) {
      const float w = __builtin_amdgcn_exp2f(pm[i] - sub);
      l = fmaf(w, pl[i], l);
#pragma unroll
      for (int d = 0; d < DL; ++d) o[d] = fmaf(w, po[i][d], o[d]);
    }
    m = mx;
  }
  if (lane == 0) { m_w[wave] = m; l_w[wave] = l; }
#pragma unroll
  for (int d = 0; d < DL; ++d) o_w[wave][DL * lane + d] = o[d];
  __syncthreads();
  if (threadIdx.x >= HD) return;
  const float mx = fmaxf(fmaxf(m_w[0], m_w[1]), fmaxf(m_w[2], m_w[3]));
  const float sub = mx == -INFINITY ? 0.f : mx;
  float num = 0.f, den = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float wt = __builtin_amdgcn_exp2f(m_w[w] - sub);
    num = fmaf(wt, o_w[w][threadIdx.x], num);
    den = fmaf(wt, l_w[w], den);
  }
  st_f32<T>((T*)a.out + (size_t)row * a.o_row + (size_t)h * a.o_head, threadIdx.x, den == 0.f ? 0.f : num / den);
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------
template <typename F> static int kv8_dispatch(const sara_kv8_cache& c, int dtype, F&& go) {
  auto by_type = [&](auto hd, auto fmt) {
    if (dtype == SARA_BF16) go(hd, fmt, uint16_t{});
    else go(hd, fmt, float{});
  };
  auto by_fmt = [&](auto hd) {
    if (c.format == SARA_KV8_INT8) by_type(hd, std::integral_constant<int, SARA_KV8_INT8>{});
    else by_type(hd, std::integral_constant<int, SARA_KV8_E4M3>{});
  };
  if (c.head_dim == 64) by_fmt(std::integral_constant<int, 64>{});
  else by_fmt(std::integral_constant<int, 128>{});
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SARA_OK : hip_fail(e, "8-bit KV cache launch");
}

// blocks of a write or read: four units of (page, KV head, K or V)
int64_t kv8_rows_blocks(int n_seqs, int n_rows, bool ragged, int hkv) {
  const int64_t items = ragged ? (int64_t)n_rows / 16 + 2 * (int64_t)n_seqs : n_seqs;
  return (items * hkv * 2 + 3) / 4;
}

int launch_kv8_rows(bool write, const sara_kv8_cache& c, void* k, void* v, int dtype, int64_t k_row, int64_t k_head,
                    int64_t v_row, int64_t v_head, int n_rows, const int32_t* pages, int max_pages, const int32_t* start,
                    const int32_t* off, int n_seqs, hipStream_t st) {
  const KvRows rows = {k, v, k_row, k_head, v_row, v_head};
  const dim3 grid((uint32_t)kv8_rows_blocks(n_seqs, n_rows, off != nullptr, c.n_kv_heads));
  return kv8_dispatch(c, dtype, [&](auto hd, auto fmt, auto t) {
    if (write)
      hipLaunchKernelGGL((k_kv8_write<hd.value, fmt.value, decltype(t)>), grid, dim3(256), 0, st, c, rows, pages,
                         max_pages, start, off, n_seqs, n_rows);
    else
      hipLaunchKernelGGL((k_kv8_read<hd.value, fmt.value, decltype(t)>), grid, dim3(256), 0, st, c, rows, pages, max_pages,
                         start, off, n_seqs, n_rows);
  });
}

Kv8Split kv8_split(int n_rows, int hq, int hkv, int hd, int n_seqs, int max_ctx, bool ragged) {
  const int G = hq / hkv, np = std::max(1, (max_ctx + 15) / 16);
  // Pages a split so that about `blocks` blocks share the work, at least `least`, in steps of `step`, and at most
  // 128 splits a row.  A split costs its block about 4 us before the first pages are there and the join launch 4 us
  // more: one row at context 333 takes 7.2 us in one split, 8.6 in three.  With the join, by pages a split: 32 rows at
  // 3,000-4,600 take 19.7 us (16), 18.7 (24, this rule's), 20.0 (32), 18.2 (40); one at 65,537 17.7 (24), 15.9 (32), 16.1
  // (40, this rule's), 18.6 (64); one at 40,000 13.6 (24, this rule's), 14.1 (32).  Where the rule's 24 pages make more
  // blocks than fit at once, coarser splits would gain: 4 rows at 40,000 24.5 (24), 20.7 (40); 8 at 16,000 18.6 (24), 16.7 (32).
  auto share = [&](int64_t items, int64_t blocks, int least, int step) {
    const int64_t want = std::min<int64_t>(128, std::max<int64_t>(1, blocks / std::max<int64_t>(1, items * hkv)));
    return (int)std::max<int64_t>(least, ((np + want - 1) / want + step - 1) / step * step);
  };
  Kv8Split s = {};
  s.items = (int64_t)n_seqs * (ragged ? kFewColumns / 16 : (G + 15) / 16);
  s.tile_items = ragged && (int64_t)n_rows * G > kFewColumns ? (int64_t)n_rows * G / (32 * kTileWaves) + n_seqs : 0;
  s.pps = share(ragged ? n_seqs : s.items, 1024, 24, 8);
  // tiles of 128 columns: two blocks a CU are resident.  16 sequences of 64 queries over 4,000 tokens: 115 us, against 130
  // in steps of 64 pages; 256 queries over 16,000: 86, against 105, and 93 with 1,024 blocks
  s.pps_tile = s.tile_items ? share(s.tile_items, 512, 32, 16) : s.pps;
  s.splits = (np + s.pps - 1) / s.pps;
  s.splits_tile = s.tile_items ? (np + s.pps_tile - 1) / s.pps_tile : 0;
  const int64_t one = (int64_t)sizeof(float) * (hd + 2);
  if (s.splits > 1) s.part_bytes = (one * n_seqs * hkv * (ragged ? kFewColumns : G) * s.splits + 15) / 16 * 16;
  if (s.splits_tile > 1) s.part_tile_bytes = one * n_rows * hq * s.splits_tile;
  return s;
}

int launch_kv8_attention(const sara_kv8_cache& c, const void* q, int dtype, int64_t q_row, int64_t q_head, int n_rows,
                         int hq, const int32_t* pages, int max_pages, const int32_t* ctx, const int32_t* off, int n_seqs,
                         int max_ctx, float scale, void* out, int64_t o_row, int64_t o_head, void* ws, hipStream_t st) {
  const Kv8Split s = kv8_split(n_rows, hq, c.n_kv_heads, c.head_dim, n_seqs, max_ctx, off != nullptr);
  const AttnArgs a = {q, out, q_row, q_head, o_row, o_head, pages, ctx, off, max_pages, max_ctx, n_seqs, n_rows, hq,
                      s.splits, s.pps, s.splits_tile, s.pps_tile, scale * 1.4426950408889634f, (float*)ws,
                      (float*)((char*)ws + s.part_bytes)};
  return kv8_dispatch(c, dtype, [&](auto hd, auto fmt, auto t) {
    const int n_few = (int)(s.items * c.n_kv_heads), n_tile = (int)(s.tile_items * c.n_kv_heads);
    // One launch for both where the blocks of few columns fit beside each other at the tiles' two a CU: 64 sequences of
    // 1-33 fp32 queries over up to 63 tokens 12.4 -> 8.0 us, of 1-33 bf16 ones over up to 500 31.2 -> 22.9.  More of them
    // lose the third wave a SIMD that streaming pages wants: 512 sequences of 1-2 queries over 1,000 tokens 70 -> 80.
    if (s.tile_items && (int64_t)n_few * s.splits <= 512) {
      hipLaunchKernelGGL((k_kv8_attn_both<hd.value, fmt.value, decltype(t)>), dim3(n_tile * s.splits_tile + n_few * s.splits), dim3(256),
                         0, st, c, a, n_tile, n_few);
    } else {
      hipLaunchKernelGGL((k_kv8_attn<hd.value, fmt.value, decltype(t)>), dim3(n_few, s.splits), dim3(256), 0, st, c, a);
      if (s.tile_items)
        hipLaunchKernelGGL((k_kv8_attn_tile<hd.value, fmt.value, decltype(t)>), dim3(n_tile, s.splits_tile), dim3(256), 0, st, c, a);
    }
    if (s.splits > 1) {
      const int cols = off ? kFewColumns : hq / c.n_kv_heads;
      hipLaunchKernelGGL((k_kv8_attn_join<hd.value, decltype(t), false>), dim3((uint32_t)((int64_t)n_seqs * c.n_kv_heads * cols)),
                         dim3(256), 0, st, a, c.n_kv_heads, cols);
    }
    if (s.splits_tile > 1)
      hipLaunchKernelGGL((k_kv8_attn_join<hd.value, decltype(t), true>), dim3((uint32_t)((int64_t)n_rows * hq)), dim3(256), 0,
                         st, a, c.n_kv_heads, 0);
  });
}

}  // namespace sara
