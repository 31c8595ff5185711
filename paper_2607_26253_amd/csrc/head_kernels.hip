// Token log probabilities from hidden states and the LM head (gfx950), without logits in memory, and both gradients.
//
// x_nv = h_n . W_v is formed tile by tile in fp32 and used where it is:
//   forward    with z = x / T: per row the running maximum m, s = sum 2^u and t = sum 2^u u, u = (x - m) log2(e) / T;
//              logp = (x_tok - m) / T - log s, H = log s - log(2) t / s
//   gradient   D_nv = g ([v = tok] - p) - h p (log p + H) by pieces of the vocabulary, from x formed again;
//              dH = D W / T and dW = D^T H / T, half of the power of two in 1 / T with D and half with the results: an
//              accepted temperature takes neither out of the range of fp32
// 8 N d V operations a training step where 6 would do with the logits kept: 2 against [rows][vocab] written and read.
#include <float.h>
#include <limits.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "sara_internal.h"

namespace sara {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------------------
// products of 256 x 256 tiles
// ---------------------------------------------------------------------------
// An operand of a product over k, in parts (fp32 numbers enter as sums of bf16 parts):
//   kPacked   [32 elements of k][16 rows] blocks of 1 KiB in fragment order: lane (row, grp) of the MFMA holds k 8 grp ..+7
//   kPackedT  the same blocks, of the transpose: k runs over their rows
//   kCols     element (k, m) at p[k stride + m]
//   kRowPairs element (m, k) at p[m stride + k]; loaded 64 elements of k at a time, whole lines of memory
enum { kPacked, kPackedT, kCols, kRowPairs };
struct Mat {
  const uint16_t* p;
  int64_t stride, part;     // of kPacked and kPackedT: the 16-row tiles of a k block
};

// What a row needs for its D: 2^u (A + B u) + [v = tok] g; logits above `large` make elements
// that are taken more exactly.  on: 0 where nothing is asked of the row, 2 where elements may pass bf16's range, else 1.
struct HeadRow { float m, A, B, g, large; int32_t tok, on; };

// The first of a number's bf16 parts is bf16's largest finite number where rounding would pass it: the parts that follow
// hold what is left, as ever.  An infinity stays one.
constexpr float kBf16Max = 0x1.FEp127f;
__device__ __forceinline__ float first_part(float f) {
  return fabsf(f) < INFINITY ? __builtin_amdgcn_fmed3f(f, -kBf16Max, kBf16Max) : f;
}

struct HeadTile {
  Mat a, b;                 // M side and N side of C[m][n] = sum_k a(m, k) b(n, k)
  int M, N, K;
  int n_pairs;              // the part pairs whose products are summed, 4 bits each (part of a, part of b << 2), smallest first
  uint32_t pairs;
  int steps;                // 32-wide k steps of a split
  int row0, m_parts;        // stats: row of the call's first, rows of a slice of `parts`
  int v0;                   // first vocabulary id of the N side
  float c, inv_t;
  const int32_t* tok;
  float* x_tok;
  float4* parts;            // [tile column][m_parts]: (m, s, t)
  const HeadRow* rows;
  uint16_t* d;              // D, packed: [part][32 ids][16 rows]
  int64_t d_part;
  int d_tiles;              // 16-row tiles
  // D's last part is kept where it counts.  Bytes: does a 256-row tile need it in a 32-id step (of dH), a 256-id tile in a
  // 32-row step (of dW)?  Written by the tiles of D; read in the products, where `sparse` is that part of a (0: none).
  uint8_t *id_flags, *row_flags;
  const uint8_t* flags;
  int id_flags_stride, row_flags_stride, flags_stride, sparse;
  float* slab;              // [split][M][N]
  void* out;                // weight gradient
  int64_t out_stride;
  int out_f32, add;         // add: to what is there
};

__device__ __attribute__((aligned(16))) const uint32_t kZeroUnit[4] = {0, 0, 0, 0};

enum { kStats, kSlab, kWeight, kGradRows };   // kGradRows + p: p parts of every element of D

constexpr int kTileLds = 163840;       // all of a compute unit's
constexpr int kTileThreads = 256;
struct TileEpilogue {                  // in the ring's place once the products are done
  float red[3][2][256];
  HeadRow rows[256];
  uint32_t bits[4];
};

// One wave's quarter of a tile: acc[n][m] of lane (row, grp) is row 16 m + row, columns 16 n + 4 grp ..+3.  The 256
// accumulators of a lane live in accumulation registers throughout; they are only touched by these.
typedef f32x4 TileAcc[8][8];
__device__ __forceinline__ void acc_zero(f32x4& a) {
  asm volatile("v_accvgpr_write_b32 %0, 0\n\tv_accvgpr_write_b32 %1, 0\n\tv_accvgpr_write_b32 %2, 0\n\tv_accvgpr_write_b32 %3, 0"
               : "=a"(a[0]), "=a"(a[1]), "=a"(a[2]), "=a"(a[3]));
}
__device__ __forceinline__ float acc_read(float a) {
  float x;
  asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(a));   // volatile: a value read twice is not kept in between
  return x;
}
__device__ __forceinline__ f32x4 acc_read4(const f32x4& a) {
  return f32x4{acc_read(a[0]), acc_read(a[1]), acc_read(a[2]), acc_read(a[3])};
}
__device__ __forceinline__ void acc_mfma(f32x4& c, bf16x8 x, bf16x8 y) {
  asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(x), "v"(y));
}

// The softmax statistics of a block's tile: per row over its columns below N.
__device__ __forceinline__ void tile_stats(TileAcc& acc, const HeadTile& a, TileEpilogue& lds, int tm0, int tn0, int bn) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, row = lane & 15, grp = lane >> 4;
  const int wm = wave >> 1, wn = wave & 1;
  const int left = a.N - (tn0 + 128 * wn) - 4 * grp;        // columns of this lane's first tile and on
  const bool full = a.N - (tn0 + 128 * wn) >= 128;
#pragma unroll
  for (int m = 0; m < 8; ++m) {
    const int r = 128 * wm + 16 * m + row;
    f32x4 z[8];
#pragma unroll
    for (int n = 0; n < 8; ++n) z[n] = acc_read4(acc[n][m]);
    const int at = lds.rows[r].tok - tn0 - 128 * wn;        // the row's id, if it is here
    if (at >= 0 && at < 128 && (at >> 2 & 3) == grp && tm0 + r < a.M) {
      float x = 0.f;
#pragma unroll
      for (int n = 0; n < 8; ++n)
#pragma unroll
        for (int q = 0; q < 4; ++q) x = at >> 4 == n && (at & 3) == q ? z[n][q] : x;
      a.x_tok[a.row0 + tm0 + r] = x;
    }
    float mx = -FLT_MAX, mn = FLT_MAX;
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float x = z[n][q];
        if (!full) x = 16 * n + q < left ? x : NAN;        // neither largest nor smallest
        mx = fmaxf(mx, x);
        mn = fminf(mn, x);
      }
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    float s = mn == -INFINITY ? NAN : 0.f, t = 0.f;        // a logit that is not finite makes the row NaN
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float u = (z[n][q] - mx) * a.c;
        if (!full) u = 16 * n + q < left ? u : -INFINITY;
        const float e = __builtin_amdgcn_exp2f(u);
        s += e;
        t = fmaf(e, fmaxf(u, -FLT_MAX), t);
      }
    s += __shfl_xor(s, 16, 64);
    t += __shfl_xor(t, 16, 64);
    s += __shfl_xor(s, 32, 64);
    t += __shfl_xor(t, 32, 64);
    if (grp == 0) { lds.red[0][wn][r] = mx; lds.red[1][wn][r] = s; lds.red[2][wn][r] = t; }
  }
  __syncthreads();
  const int r = threadIdx.x;
  if (tm0 + r >= a.M) return;
  const float m = fmaxf(lds.red[0][0][r], lds.red[0][1][r]);
  float s = 0.f, t = 0.f;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const float u = (lds.red[0][w][r] - m) * a.c, e = __builtin_amdgcn_exp2f(u);
    s = fmaf(e, lds.red[1][w][r], s);
    t += fmaf(e * fmaxf(u, -FLT_MAX), lds.red[1][w][r], e * lds.red[2][w][r]);
  }
  a.parts[(size_t)bn * a.m_parts + tm0 + r] = make_float4(m, s, t, 0.f);
}

// 32 ids of D lie in fragments in the order that leaves a lane's eight values together: place 8 g + 4 b + q holds id
// 16 b + 4 g + q.  Products over ids take the other operand in that order, D^T gives its rows back.
__device__ __forceinline__ int id_of_place(int p) { return 16 * (p >> 2 & 1) + 4 * (p >> 3) + (p & 3); }

// PARTS of every element of D, and the last part of the steps of 32 ids or rows that have a large one (a.id_flags).
template <int PARTS>
__device__ __forceinline__ void tile_grad(TileAcc& acc, const HeadTile& a, TileEpilogue& lds, int tm0, int tn0) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, row = lane & 15, grp = lane >> 4;
  const int wm = wave >> 1, wn = wave & 1;
  const int col = tn0 + 128 * wn + 4 * grp;
  const bool full = tn0 + 256 <= a.N;
  uint32_t my_ids = 0, my_rows = 0;                          // steps of this wave's that want the last part
  if (a.id_flags) {
    uint32_t bits = 0;                                       // of the wave: ids in bits 0..3, rows in bits 4..7
#pragma unroll
    for (int m = 0; m < 8; ++m) {
      const HeadRow& hr = lds.rows[128 * wm + 16 * m + row];
      const float large = hr.large;
      const int at = hr.tok - a.v0 - col;                    // the row's id itself is taken for large
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x4 x = acc_read4(acc[2 * j][m]), y = acc_read4(acc[2 * j + 1][m]);
        const float mx = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])));
        if (__any(mx > large || (unsigned)(at + 4 * grp - 32 * j) < 32u)) bits |= 1u << j | 16u << (m >> 1);
      }
    }
    if (lane == 0) lds.bits[wave] = bits;
    __syncthreads();
    my_ids = __builtin_amdgcn_readfirstlane((lds.bits[wn] | lds.bits[2 + wn]) & 15);
    my_rows = __builtin_amdgcn_readfirstlane((lds.bits[2 * wm] | lds.bits[2 * wm + 1]) >> 4);
    if (threadIdx.x < 16) {
      const int i = threadIdx.x & 3, half = threadIdx.x >> 2 & 1;
      if (threadIdx.x < 8)
        a.id_flags[(int64_t)(tm0 >> 8) * a.id_flags_stride + (tn0 >> 5) + threadIdx.x] = (lds.bits[half] | lds.bits[2 + half]) >> i & 1;
      else
        a.row_flags[(int64_t)(tn0 >> 8) * a.row_flags_stride + (tm0 >> 5) + threadIdx.x - 8] =
            (lds.bits[2 * half] | lds.bits[2 * half + 1]) >> (4 + i) & 1;
    }
  }
#pragma unroll
  for (int m = 0; m < 8; ++m) {
    __builtin_amdgcn_sched_barrier(0);                       // else the rows' values gather in front
    const HeadRow hr = lds.rows[128 * wm + 16 * m + row];
    const int at = hr.tok - a.v0 - col;                      // 32 j + 16 b + q where it is this lane's
    const bool huge = __any(hr.on == 2);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      // A row that is off has A = B = 0 and no id here; one that met a NaN has it in A
      float f[8];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const f32x4 z = acc_read4(acc[2 * j + b][m]);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          // x formed again may lie above the forward's maximum by its rounding, which a low temperature would blow up
          const float u = __builtin_amdgcn_fmed3f((z[q] - hr.m) * a.c, -150.f, 0.f);
          f[4 * b + q] = __builtin_amdgcn_exp2f(u) * fmaf(hr.B, u, hr.A);
        }
      }
      if (__any((unsigned)(at - 32 * j) < 32u && (at & 12) == 0))
#pragma unroll
        for (int n = 0; n < 8; ++n) f[n] += at == 32 * j + 16 * (n >> 2) + (n & 3) ? hr.g : 0.f;
      if (!full)
#pragma unroll
        for (int n = 0; n < 8; ++n) f[n] = col + 32 * j + 16 * (n >> 2) + (n & 3) < a.N ? f[n] : 0.f;
      u32x4* y = (u32x4*)(a.d + ((int64_t)((tn0 >> 5) + 4 * wn + j) * a.d_tiles + ((tm0 + 128 * wm + 16 * m) >> 4)) * 512);   // scalar
      auto store = [&](int p, auto may_pass) {               // rounded; f keeps the rest
        u32x4 w;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint32_t x = may_pass.value ? pack_bf16(first_part(f[2 * q]), first_part(f[2 * q + 1])) : pack_bf16(f[2 * q], f[2 * q + 1]);
          asm("" : "+v"(x));                                 // what was rounded is what is subtracted
          f[2 * q] -= __uint_as_float(x << 16);
          f[2 * q + 1] -= __uint_as_float(x & 0xFFFF0000u);
          w[q] = x;
        }
        (y + p * (a.d_part / 8))[lane] = w;
      };
      if (huge) store(0, std::true_type{});
      else store(0, std::false_type{});
#pragma unroll
      for (int p = 1; p < PARTS; ++p) store(p, std::false_type{});
      if ((my_ids >> j | my_rows >> (m >> 1)) & 1) store(PARTS, std::false_type{});
    }
  }
}

// C[m][n] = sum over part pairs and k of a(m, k) b(n, k), 256 x 256 a block of 4 waves (v_mfma_f32_16x16x32_bf16, 128 x 128 a
// wave).  Operands go straight to LDS, 16 bytes a lane, in 32-wide k stages: a ring of five for both, or (PAIRS: kRowPairs) of
// four for a and of three 64-wide ones for b.  What limits the loads is how many lines they touch: 32-wide pieces of rows of
// a row-major matrix took 0.67 us a stage and compute unit, whole lines 0.44, blocks 0.40 (the MFMAs of a stage: 0.43 at
// 2.4 GHz).  In LDS the 16-byte units of a row (32-byte units of kCols) are exchanged so that the 16 lanes which a read
// serves at a time meet different banks; fragments of operands that lie across k are read transposed
// (ds_read_b64_tr_b16), k in the order of id_of_place.  Rows past the end repeat the last one and are dropped; k past the
// end is zero on both sides.
//
// In step s the fragments of stage s are in registers; between its 64 MFMAs a wave reads those of stage s + 1 and sends for
// later stages, into slots whose reads are over.  One barrier a step: before it a wave waits for its own loads of stage
// s + 1, so all have landed behind it.  The loads are written in assembly: the compiler would wait for all of them
// before each LDS read.
//
// 4,093 rows of width 1,536 over 151,936 ids run at 1.17 PFLOP/s in all (a library's product of 16,384 cubed: 1.38): 44 us a
// round of tiles, of which some 9 go to the statistics and 4 to the first loads, with nothing of the next tile under way.  2,048
// rows over 57,344 ids: D 346 us, dH 285, dW 337 (1.04, 1.27 and 1.07 PFLOP/s).
template <int AK, int BK, int EPI>
__global__ __launch_bounds__(kTileThreads, 1) void k_head_tile(HeadTile a) {
  constexpr bool PAIRS = BK == kRowPairs;
  constexpr int RA = PAIRS ? 4 : 5, A_SLOT = PAIRS ? 16384 : 32768;      // slots of a, their pitch
  constexpr int RB = PAIRS ? 3 : 5, B_SLOT = 32768, B_AT = PAIRS ? 65536 : 16384;
  constexpr int AHEAD = PAIRS ? 4 : 5;                                   // stages that a's loads run ahead
  __shared__ __attribute__((aligned(1024))) char ring[kTileLds];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int row = lane & 15, grp = lane >> 4;
  const int wm = wave >> 1, wn = wave & 1;
  // Each XCD takes a contiguous stretch of an order that walks 4 row tiles by every column tile, one split after the other
  int bn, bm, split;
  {
    const int nb = (a.N + 255) >> 8, mb = (a.M + 255) >> 8, tiles = nb * mb, total = gridDim.x;
    const int x = blockIdx.x & 7, per = total >> 3, rem = total & 7;
    const int all = x * per + min(x, rem) + (blockIdx.x >> 3);
    split = all / tiles;
    const int lin = all - split * tiles;
    const int gs = 4 * nb, g = lin / gs, gm = min(4, mb - 4 * g), r = lin - g * gs;
    bm = 4 * g + r % gm;
    bn = r / gm;
  }
  const int tm0 = 256 * bm, tn0 = 256 * bn;
  const int k_steps = (a.K + 31) >> 5, s0 = split * a.steps, ns = min(a.steps, k_steps - s0), dense = ns * a.n_pairs;
  // Steps that want D's last part, 64 a lane; they come first.  left: how many are still to be sent.
  constexpr bool SPARSE = EPI == kSlab || EPI == kWeight;
  uint64_t wanted = 0, sp_bits = 0;
  int sp_lane = -1, sp_at = 0, sp_left = 0;
  auto sp_next = [&]() {
    sp_bits &= sp_bits - 1;
    if (sp_bits == 0) {
      const uint64_t who = __ballot(wanted != 0) & (sp_lane < 0 ? ~0ull : ~((2ull << sp_lane) - 1));
      sp_lane = __ffsll((unsigned long long)who) - 1;
      sp_bits = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(wanted >> 32), sp_lane) << 32 |
                (uint32_t)__builtin_amdgcn_readlane((int)wanted, sp_lane);
    }
    sp_at = 64 * sp_lane + __ffsll((unsigned long long)sp_bits) - 1;
  };
  if (SPARSE && a.sparse) {
    const uint8_t* f = a.flags + (int64_t)bm * a.flags_stride + s0 + 64 * lane;
    int n = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (64 * lane + 16 * i < ns) {
        const u32x4 w = *(const u32x4*)(f + 16 * i);
#pragma unroll
        for (int q = 0; q < 16; ++q)
          if (64 * lane + 16 * i + q < ns) wanted |= (uint64_t)(w[q >> 2] >> (8 * (q & 3)) & 1) << (16 * i + q);
      }
    n = __popcll(wanted);
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) n += __shfl_xor(n, x, 64);
    sp_left = __builtin_amdgcn_readfirstlane(n);
    if (sp_left > 0) sp_next();
  }
  const int total = dense + sp_left;
  // A wave loads 4 KiB of either operand in a step: where a lane's 16 bytes come from at k = 0, and the k they hold
  auto unit = [&](auto kind, const Mat& mat, int t0, int n, int f, int& k_of) {
    k_of = 0;
    if constexpr (kind.value == kPacked) return mat.p + ((t0 >> 4) + f) * 512 + lane * 8;
    if constexpr (kind.value == kPackedT)
      return mat.p + ((int64_t)min((t0 >> 5) + (f >> 1), ((n + 31) >> 5) - 1) * mat.stride + (f & 1)) * 512 + lane * 8;
    if constexpr (kind.value == kCols) {
      const int kr = 2 * f + (lane >> 5), u = lane & 31;
      k_of = kr;
      return mat.p + kr * mat.stride + min(t0 + 16 * ((u >> 1) ^ (kr & 15)) + 8 * (u & 1), n - 8);
    }
    const int r = 8 * f + (lane >> 3), u = (lane & 7) ^ (r >> 1 & 7);
    k_of = 8 * u;
    return mat.p + (int64_t)min(t0 + r, n - 1) * mat.stride + 8 * u;
  };
  constexpr std::integral_constant<int, AK> ak{};
  constexpr std::integral_constant<int, BK> bk{};
  const int64_t a_step = AK == kPacked ? a.a.stride * 512 : 1024;
  const int64_t b_step = BK == kPacked ? a.b.stride * 512 : BK == kPackedT ? 1024 : BK == kCols ? 32 * a.b.stride : 64;
  constexpr int BF = PAIRS ? 8 : 4;                        // loads of b that a wave keeps addresses of
  const uint16_t *fa[4], *fb[BF];
  int unused;
#pragma unroll
  for (int j = 0; j < 4; ++j) fa[j] = unit(ak, a.a, tm0, a.M, 4 * wave + j, unused);
#pragma unroll
  for (int j = 0; j < BF; ++j) fb[j] = unit(bk, a.b, tn0, a.N, BF * wave + j, unused);
  const uint32_t ring_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)ring;
  auto load = [&](const char* p, uint32_t at) {
    // m0, where in LDS the load goes, is read as the load is issued; as an output the compiler knows that it is overwritten
    uint32_t m0;
    asm volatile("s_mov_b32 %0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off" : "={m0}"(m0) : "s"(ring_at + at), "v"(p));
  };
  // The next stage to load.  For `run` stages the addresses only grow; then comes k that ends inside a stage or the next pair
  // of parts.  Past the last stage it is loaded again, to slots that nobody reads, so that the count of loads in flight
  // stays exact.
  int i_pair = 0, i_step = 0, i_seen = 0, run = 0;
  bool tail = false;
  int64_t a_at = 0, b_at = 0, a_grow = 2 * a_step, b_grow = 2 * b_step;   // added to the addresses, in bytes
  uint32_t a_slot = 0, b_slot = 0;
  auto place = [&]() {
    const bool sp = SPARSE && sp_left > 0;
    const int pair = sp ? a.sparse : a.pairs >> (4 * i_pair) & 15, ks = s0 + (sp ? sp_at : i_step);
    const int kb = PAIRS ? i_seen >> 1 : ks;
    a_at = 2 * ((pair & 3) * a.a.part + ks * a_step);
    b_at = 2 * ((pair >> 2) * a.b.part + kb * b_step);
    run = sp ? 0 : ns - 1 - i_step;
    if constexpr (BK == kCols || BK == kRowPairs) {        // not padded with zeros
      constexpr int W = PAIRS ? 64 : 32;
      const bool ends = W * (kb + 1) > a.K;
      if (ends || tail) {
#pragma unroll
        for (int j = 0; j < BF; ++j) {
          int k;
          const uint16_t* p = unit(bk, a.b, tn0, a.N, BF * wave + j, k);
          fb[j] = W * kb + k < a.K ? p : (const uint16_t*)((const char*)kZeroUnit - b_at);
        }
      }
      tail = ends;
      const int full = a.K / W;                            // stages (or pairs) before the one that ends inside
      if (!ends && !sp) run = min(run, (PAIRS ? 2 * full - i_seen : full - ks) - 1);
    }
  };
  auto grow = [&](int odd) {                               // odd: of the stage just sent
    a_slot = a_slot == (RA - 1) * A_SLOT ? 0 : a_slot + A_SLOT;
    if (!PAIRS || odd) b_slot = b_slot == (RB - 1) * B_SLOT ? 0 : b_slot + B_SLOT;
    a_at += a_grow;
    if (!PAIRS || odd) b_at += b_grow;
  };
  auto plain = [&](int n) { run -= n; i_step += n; i_seen += n; };   // n stages were sent so
  auto next = [&](int odd) {
    grow(odd);
    if (run > 0) { plain(1); return; }
    ++i_seen;
    if (SPARSE && sp_left > 0) {
      if (--sp_left > 0) sp_next();
      place();
    } else if (i_pair * ns + i_step + 1 < dense) {
      if (++i_step == ns) { i_step = 0; ++i_pair; }
      place();
    } else if (a_grow != 0) {                              // that was the last
      a_at -= a_grow;
      if (!PAIRS || odd) b_at -= b_grow;
      a_grow = b_grow = 0;
      run = INT_MAX;
    }
  };
  // With pairs, the b of stages s + 4 and s + 5 goes with steps s and s + 1 (s even): half of its rows each
  auto send_b = [&](int j, int half) { load((const char*)fb[4 * half + j] + b_at, B_AT + b_slot + (BF * wave + 4 * half + j) * 1024); };
  auto send_a = [&](int j) { load((const char*)fa[j] + a_at, a_slot + (4 * wave + j) * 1024); };
  typedef __attribute__((address_space(3))) s16x4* Lds8;
  // byte address of fragment i of this wave's half of an operand; of those read transposed, the part with k below 16.  The
  // 16 columns of a transposed b's fragments 2 j and 2 j + 1 are fours of 32 in turn, so that a lane's results are eight in a row.
  auto address = [&](auto kind, bool b, int i) {
    const int t = 8 * (b ? wn : wm) + i;
    if constexpr (kind.value == kPacked) return t * 1024 + (row + 16 * grp) * 16;
    const int c = b ? (row & 3) * 16 + (t & 1) * 8 : (row & 3) * 8 + (t & 1) * 32;   // byte of 32 columns
    if constexpr (kind.value == kPackedT) return (t >> 1) * 2048 + (c >> 4) * 256 + (4 * grp + (row >> 2)) * 16 + (c & 15);
    const int k = 4 * grp + (row >> 2);
    if constexpr (kind.value == kCols) return k * 512 + ((((t & ~1) + (c >> 5)) ^ k) * 32) + (c & 31);
    return (16 * t + row) * 128;
  };
  s16x4 lo;
  auto read = [&](auto kind, bool b, uint32_t slot, int i, int part, int half, bf16x8& f) {
    const char* p = ring + slot + address(kind, b, i);
    if constexpr (kind.value == kPacked) {
      if (part == 0) f = __builtin_bit_cast(bf16x8, *(const u32x4*)p);
    } else if constexpr (kind.value == kRowPairs) {
      if (part == 0) f = __builtin_bit_cast(bf16x8, *(const u32x4*)(p + (((4 * half + grp) ^ (row >> 1)) * 16)));
    } else if (part == 0) {
      lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds8)(const s16x4*)p);
    } else {
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds8)(const s16x4*)(p + (kind.value == kPackedT ? 1024 : 8192)));
      f = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  };
  auto barrier = [&]() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  TileAcc acc;
#pragma unroll
  for (int n = 0; n < 8; ++n)
#pragma unroll
    for (int m = 0; m < 8; ++m) acc_zero(acc[n][m]);
  bf16x8 wf[2][8], xf[2][8];
  place();
#pragma unroll
  for (int s = 0; s < AHEAD; ++s) {
#pragma unroll
    for (int j = 0; j < 4; ++j) send_b(j, PAIRS ? s & 1 : 0);
#pragma unroll
    for (int j = 0; j < 4; ++j) send_a(j);
    next(s & 1);
  }
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(PAIRS ? 20 : 32) : "memory");   // stage 0 has landed
  barrier();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    read(bk, true, B_AT, i, 0, 0, wf[0][i]);
    read(bk, true, B_AT, i, 1, 0, wf[0][i]);
    read(ak, false, 0, i, 0, 0, xf[0][i]);
    read(ak, false, 0, i, 1, 0, xf[0][i]);
  }
  uint32_t a_read = A_SLOT, b_read = PAIRS ? 0 : B_SLOT;   // the slots of stage s + 1
  auto step = [&](auto par, auto is_plain) {
    constexpr int P = par.value;                           // s & 1
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(PAIRS ? (P ? 9 : 16) : 24) : "memory");
    barrier();
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int n = 0; n < 8; ++n) {
        acc_mfma(acc[n][i], wf[P][n], xf[P][i]);
        __builtin_amdgcn_sched_barrier(0);
        if (n < 2) read(bk, true, B_AT + b_read, i, n, P ^ 1, wf[P ^ 1][i]);
        else if (n < 4) read(ak, false, a_read, i, n - 2, 0, xf[P ^ 1][i]);
        else if (i < 4 && n == 5) send_b(i, PAIRS ? P : 0);
        else if (i < 4 && n == 7) send_a(i);
        else if (is_plain.value && i == 5 && n == 5) grow(P);   // scalar work in the MFMAs' shade
        __builtin_amdgcn_sched_barrier(0);
      }
    a_read = a_read == (RA - 1) * A_SLOT ? 0 : a_read + A_SLOT;
    if (!PAIRS || P == 0) b_read = b_read == (RB - 1) * B_SLOT ? 0 : b_read + B_SLOT;
    if (!is_plain.value) next(P);
  };
  constexpr std::integral_constant<int, 0> even{};
  constexpr std::integral_constant<int, 1> odd{};
  for (int s = 0; s < total;) {
    const int n = min(run, total - s) & ~1;
    for (int i = 0; i < n; i += 2) {
      step(even, std::true_type{});
      step(odd, std::true_type{});
    }
    plain(n);
    s += n;
    if (s < total) { step(even, std::false_type{}); ++s; }
    if (s < total) { step(odd, std::false_type{}); ++s; }
  }
  // the repeated loads, and the results on their way to the accumulators
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_nop 15\n\ts_nop 15" ::: "memory");
  barrier();
  TileEpilogue& lds = *(TileEpilogue*)ring;
  if constexpr (EPI == kStats) {
    const int tok = tm0 + (int)threadIdx.x < a.M ? a.tok[a.row0 + tm0 + threadIdx.x] : -1;
    lds.rows[threadIdx.x].tok = tok >= a.v0 && tok < a.v0 + a.N ? tok - a.v0 : -1;
    __syncthreads();
    tile_stats(acc, a, lds, tm0, tn0, bn + (a.v0 >> 8));
  } else if constexpr (EPI > kGradRows) {
    lds.rows[threadIdx.x] = a.rows[tm0 + threadIdx.x];
    __syncthreads();
    tile_grad<EPI - kGradRows>(acc, a, lds, tm0, tn0);
  } else {
    const int c0 = tn0 + 128 * wn + 8 * grp;
#pragma unroll
    for (int m = 0; m < 8; ++m) {
      const int p = 16 * (m & 1) + row;
      const int r = tm0 + 128 * wm + (EPI == kWeight ? 32 * (m >> 1) + id_of_place(p) : 16 * m + row);
      if (r >= a.M) continue;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int col = c0 + 32 * j;
        if (col >= a.N) continue;                          // N is a multiple of 4
        f32x4 v[2] = {acc_read4(acc[2 * j][m]), acc_read4(acc[2 * j + 1][m])};
        if (EPI == kWeight) { v[0] *= a.inv_t; v[1] *= a.inv_t; }
        if (EPI == kSlab || a.out_f32) {
          f32x4* y = (f32x4*)(EPI == kSlab ? a.slab + ((int64_t)split * a.M + r) * a.N + col : (float*)a.out + r * a.out_stride + col);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (col + 4 * h >= a.N) continue;
            if (a.add) v[h] += y[h];
            y[h] = v[h];
          }
        } else {
          u32x4* y = (u32x4*)((uint16_t*)a.out + r * a.out_stride + col);   // bf16: N is a multiple of 8
          if (a.add) {
            const u32x4 w = *y;
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q >> 2][q & 3] += __uint_as_float(q & 1 ? w[q >> 1] & 0xFFFF0000u : w[q >> 1] << 16);
          }
          *y = u32x4{pack_bf16(v[0][0], v[0][1]), pack_bf16(v[0][2], v[0][3]), pack_bf16(v[1][0], v[1][1]), pack_bf16(v[1][2], v[1][3])};
        }
      }
    }
  }
}

// ---------------------------------------------------------------------------
// few rows
// ---------------------------------------------------------------------------
struct HeadSum { float m, s, t; };
__device__ __forceinline__ void head_merge(HeadSum& a, HeadSum b, float c) {
  const float m = fmaxf(a.m, b.m);
  const float ua = (a.m - m) * c, ub = (b.m - m) * c;
  const float ea = __builtin_amdgcn_exp2f(ua), eb = __builtin_amdgcn_exp2f(ub);
  a.t = fmaf(ea * fmaxf(ua, -FLT_MAX), a.s, ea * a.t) + fmaf(eb * fmaxf(ub, -FLT_MAX), b.s, eb * b.t);
  a.s = fmaf(ea, a.s, eb * b.s);
  a.m = m;
}

// Up to 16 NT rows: W streams past them.  A block of 8 waves takes 128 ids at a time, a wave 16 of them, in 128-byte blocks of
// k: a lane loads 32 consecutive bytes of an id's row, the hidden states lie in LDS (`chunk` blocks of k at a time).
// fp32 runs on v_mfma_f32_16x16x4_f32.  Bound by W's way from memory: 151,936 ids of width 1,536 in bf16, 467 MB, take 100 us for
// one row (4.7 TB/s), 105 for 17 to 32 and 116 for 35 to 64, whose hidden states pass LDS in two and three chunks; in fp32, 933 MB, 198, 215
// and 300, of which the matrix instructions of 64 rows are some 190.  Eight blocks of k in flight leave 17 to 32 rows no
// registers for their sums: the call took 136 us in bf16 and 264 in fp32, for 110 and 217.
struct HeadFew {
  const char *h, *w;
  int64_t h_stride, w_stride;   // bytes
  int n_rows, units, V;         // units: 16-byte units of a row
  const int32_t* tok;
  float c;
  float* x_tok;
  float4* parts;                // [block][16 NT]
};
constexpr int kFewLds = 65536;
template <typename T, int NT>
__global__ __launch_bounds__(512, 4) void k_head_few(HeadFew a) {
  constexpr int CB = kFewLds / (16 * NT * 128);            // 128-byte blocks of k of a chunk
  constexpr int DEPTH = NT == 1 ? 8 : 4;                   // blocks of k in flight; CB is a multiple
  __shared__ u32x4 hs[kFewLds / 16];
  __shared__ HeadSum red[8][16 * NT];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, row = lane & 15, grp = lane >> 4;
  const int blocks = (a.units + 7) >> 3, chunks = (blocks + CB - 1) / CB;
  int tok[NT];
  HeadSum sum[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    tok[t] = 16 * t + row < a.n_rows ? a.tok[16 * t + row] : -1;
    sum[t] = HeadSum{-FLT_MAX, 0.f, 0.f};
  }
  auto stage = [&](int chunk) {
    const int nb = min(CB, (blocks - chunk * CB + DEPTH - 1) / DEPTH * DEPTH);   // blocks past the end are zeros on both sides
    for (int i = threadIdx.x; i < nb * 16 * NT * 8; i += 512) {
      const int u = i & 7, r = (i >> 3) % (16 * NT), b = i / (128 * NT);
      const int unit = 8 * (chunk * CB + b) + u;
      u32x4 v = {0, 0, 0, 0};
      if (r < a.n_rows && unit < a.units) v = *(const u32x4*)(a.h + r * a.h_stride + 16 * (int64_t)unit);
      hs[(b * 16 * NT + r) * 8 + (u ^ (r & 7))] = v;
    }
  };
  if (chunks == 1) {
    stage(0);
    __syncthreads();
  }
  for (int64_t v0 = 128 * (int64_t)blockIdx.x; v0 < a.V; v0 += 128 * (int64_t)gridDim.x) {
    const int id = (int)v0 + 16 * wave;
    const char* w = a.w + min((int64_t)id + row, (int64_t)a.V - 1) * a.w_stride + 32 * grp;
    // Several sums of a logit, of smaller numbers and fewer roundings in a row: with one the largest logit of a row was
    // off by some 2e-6, and so was the sum of exponentials
    constexpr int SUMS = NT == 4 ? 2 : 4;
    f32x4 part[NT][SUMS], acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < SUMS; ++i) part[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    u32x4 r[DEPTH][2];
    auto load = [&](int b, int slot) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const bool in = 8 * b + 2 * grp + s < a.units;
        const char* p = in ? w + 128 * (int64_t)b + 16 * s : (const char*)kZeroUnit;
        r[slot][s] = __builtin_nontemporal_load((const __attribute__((address_space(1))) u32x4*)p);
      }
    };
#pragma unroll
    for (int i = 0; i < DEPTH; ++i) load(i, i);            // blocks past the end are zeros
    for (int chunk = 0; chunk < chunks; ++chunk) {
      if (chunks > 1) {
        __syncthreads();
        stage(chunk);
        __syncthreads();
      }
      const int b0 = chunk * CB, nb = min(CB, blocks - b0);
      for (int b = 0; b < nb; b += DEPTH) {
#pragma unroll
        for (int i = 0; i < DEPTH; ++i) {
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              const u32x4 h = hs[((b + i) * 16 * NT + 16 * t + row) * 8 + ((2 * grp + s) ^ (row & 7))];
              f32x4& z = part[t][(2 * i + s) % SUMS];
              if constexpr (sizeof(T) == 2) {
                z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, r[i][s]), __builtin_bit_cast(bf16x8, h),
                                                            z, 0, 0, 0);
              } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  z = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(r[i][s][e]), __uint_as_float(h[e]), z, 0, 0, 0);
              }
            }
          __builtin_amdgcn_sched_barrier(0);               // else the loads gather behind the products
          load(b0 + b + i + DEPTH, i);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    // lane (row, grp): ids id + 4 grp ..+3 of rows 16 t + row
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int n = SUMS / 2; n > 0; n /= 2)
#pragma unroll
        for (int i = 0; i < n; ++i) part[t][i] += part[t][i + n];
      acc[t] = part[t][0];
      const int at = tok[t] - id - 4 * grp, left = a.V - id - 4 * grp;
      if (at >= 0 && at < 4 && left > at) {
        float x = acc[t][0];
#pragma unroll
        for (int q = 1; q < 4; ++q) x = at == q ? acc[t][q] : x;
        a.x_tok[16 * t + row] = x;
      }
      HeadSum one = {-FLT_MAX, 0.f, 0.f};                  // a logit that is not finite makes the row NaN
#pragma unroll
      for (int q = 0; q < 4; ++q) one.m = fmaxf(one.m, q < left ? acc[t][q] : NAN);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float x = acc[t][q], u = q < left ? (x - one.m) * a.c : -INFINITY;
        const float e = q < left && x == -INFINITY ? NAN : __builtin_amdgcn_exp2f(u);
        one.s += e;
        one.t = fmaf(e, fmaxf(u, -FLT_MAX), one.t);
      }
      head_merge(sum[t], one, a.c);
    }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
#pragma unroll
    for (int x = 16; x < 64; x <<= 1)
      head_merge(sum[t], HeadSum{__shfl_xor(sum[t].m, x, 64), __shfl_xor(sum[t].s, x, 64), __shfl_xor(sum[t].t, x, 64)}, a.c);
    if (grp == 0) red[wave][16 * t + row] = sum[t];
  }
  __syncthreads();
  if (threadIdx.x < 16 * NT) {
    HeadSum all = red[0][threadIdx.x];
    for (int w = 1; w < 8; ++w) head_merge(all, red[w][threadIdx.x], a.c);
    a.parts[(size_t)blockIdx.x * 16 * NT + threadIdx.x] = make_float4(all.m, all.s, all.t, 0.f);
  }
}

// A block joins the slices of RB rows: 256 / RB threads a row.  594 slices of 2,048 rows: 10 us (19 with 16 rows a block).
template <int RB>
__global__ __launch_bounds__(256) void k_head_join(const float4* __restrict__ parts, int slices, int m_parts, int row0, int n_rows,
    int V, const int32_t* __restrict__ tok, const float* __restrict__ x_tok, float c, float inv_t, float* logp, float* entropy,
    float* stats) {
  constexpr int TR = 256 / RB;
  __shared__ HeadSum red[TR][RB];
  const int ri = threadIdx.x % RB, sl = threadIdx.x / RB, r = blockIdx.x * RB + ri;
  HeadSum sum = {-FLT_MAX, 0.f, 0.f};
  if (r < n_rows)
    for (int i = sl; i < slices; i += TR) {
      const float4 p = parts[(size_t)i * m_parts + r];
      head_merge(sum, HeadSum{p.x, p.y, p.z}, c);
    }
  red[sl][ri] = sum;
  for (int half = TR / 2; half > 0; half >>= 1) {
    __syncthreads();
    if (sl < half) {
      HeadSum x = red[sl][ri];
      head_merge(x, red[sl + half][ri], c);
      red[sl][ri] = x;
    }
  }
  if (sl != 0 || r >= n_rows) return;
  const HeadSum x = red[0][ri];
  const int tk = tok[row0 + r];
  const float ls = logf(x.s);
  if (logp) logp[row0 + r] = tk >= 0 && tk < V ? (x_tok[row0 + r] - x.m) * inv_t - ls : 0.f;
  if (entropy) entropy[row0 + r] = ls - 0.69314718f * (x.t / x.s);
  if (stats) *(float2*)(stats + 2 * (size_t)(row0 + r)) = make_float2(x.s == x.s ? x.m : NAN, x.s);
}

// ---------------------------------------------------------------------------
// operands
// ---------------------------------------------------------------------------
// Rows of a matrix packed, as P bf16 parts: rows past the end, those of `rows` that are off and elements past d are 0.  A block
// takes 16 rows, a wave 32 elements of k at a time.
template <typename T, int P>
__global__ __launch_bounds__(256) void k_head_pack(const T* __restrict__ x, int64_t stride, int n_rows, int d,
    const HeadRow* __restrict__ rows, uint16_t* __restrict__ y, int tiles, int k_blocks) {
  const int lane = threadIdx.x & 63, r = blockIdx.x * 16 + (lane & 15);
  const bool have = r < n_rows && (!rows || rows[r].on);
  for (int kb = blockIdx.y * 4 + (threadIdx.x >> 6); kb < k_blocks; kb += 4 * gridDim.y) {
    const int k = 32 * kb + 8 * (lane >> 4);
    float f[8] = {};
    if (have) {
      if constexpr (sizeof(T) == 2) {
        if (k < d) {
          const u32x4 w = *(const u32x4*)(x + r * stride + k);
          if (P == 1) {
            *(u32x4*)(y + ((int64_t)kb * tiles + blockIdx.x) * 512 + lane * 8) = w;
            continue;
          }
        }
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (k + 4 * h < d) {                             // d is a multiple of 4
            const f32x4 w = *(const f32x4*)(x + r * stride + k + 4 * h);
#pragma unroll
            for (int q = 0; q < 4; ++q) f[4 * h + q] = w[q];
          }
      }
    }
#pragma unroll
    for (int p = 0; p < P; ++p) {
      u32x4 w;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t v = p == 0 ? pack_bf16(first_part(f[2 * q]), first_part(f[2 * q + 1])) : pack_bf16(f[2 * q], f[2 * q + 1]);
        asm("" : "+v"(v));
        f[2 * q] -= __uint_as_float(v << 16);
        f[2 * q + 1] -= __uint_as_float(v & 0xFFFF0000u);
        w[q] = v;
      }
      *(u32x4*)(y + (((int64_t)p * k_blocks + kb) * tiles + blockIdx.x) * 512 + lane * 8) = w;
    }
  }
}

// A bf16 number is off by up to 2^-8 of itself; a gradient row is made of few large elements of D and many small ones, whose
// errors are independent.  Elements above kBig of a row's scale get one part more (32 x 256 of their neighbours with
// them), which leaves some 2^-9 sqrt(kBig) of the row.
constexpr float kBig = 1.f / 16;

struct HeadGrads {
  int n_rows, V;
  const int32_t* tok;
  const float *stats, *entropy, *g_logp, *g_ent;
  float scale, inv_c;
};
__device__ __forceinline__ HeadRow head_row(const HeadGrads& a, int r) {
  HeadRow o = {0.f, 0.f, 0.f, 0.f, 0.f, -1, 0};
  if (r >= a.n_rows) return o;
  const int tk = a.tok[r];
  const bool has = tk >= 0 && tk < a.V;
  const float m = a.stats[2 * (size_t)r], s = a.stats[2 * (size_t)r + 1];
  const float g = has && a.g_logp ? a.g_logp[r] : 0.f, h = a.g_ent ? a.g_ent[r] : 0.f;
  if (g == 0.f && h == 0.f) return o;
  // 1 / s is the largest p: |g| (1 - 1 / s) is at most |D| at the row's id, the other term |D| at its likeliest.  Where
  // 2^u |A| and 2^u |B u| <= 1.07 2^(u / 2) |B| are below half of kBig of that, D is below kBig of it.
  const float hl = h == 0.f ? 0.f : h * (a.entropy[r] - logf(s)), A = -(g + hl) / s, B = -0.69314718f * h / s;
  const float half = 0.5f * kBig * (fabsf(g) * (1.f - 1.f / s) + fabsf(hl) / s);
  const float u = B == 0.f ? log2f(2.f * half / fabsf(A)) : fminf(log2f(half / fabsf(A)), 2.f * log2f(half / (1.07f * fabsf(B))));
  const float most = a.scale * (fabsf(A) + 0.54f * fabsf(B) + fabsf(g));   // 2^u |u| <= 0.531
  return HeadRow{m, a.scale * A, a.scale * B, a.scale * g, m + fminf(u, 0.f) * a.inv_c, has ? tk : -1, most > 0.5f * kBf16Max ? 2 : 1};
}

__global__ __launch_bounds__(256) void k_head_rows(HeadGrads a, int rows_out, HeadRow* __restrict__ out) {
  const int r = blockIdx.x * 256 + threadIdx.x;
  if (r < rows_out) out[r] = head_row(a, r);
}

// ---------------------------------------------------------------------------
// small problems
// ---------------------------------------------------------------------------
// Tiles of 32 x 32 on v_mfma_f32_16x16x4_f32, whose products of bf16 or fp32 numbers are exact before their sum in fp32: no
// operand is packed or taken in parts, and D stays in fp32.  The four waves of a block take every fourth 16 elements of k,
// straight from memory to registers four steps ahead, and join their sums in LDS.  509 fp32 rows of width 256 over 512 ids:
// statistics 7 us, D 8, both gradients 9, most of that a launch and its load round trips.  With many tiles a compute unit takes
// 2.4 us for a tile and 256 of k, twice its matrix instructions' time: loads in pieces of 64 bytes.
struct Rows { const void* p; int64_t stride; };

struct HeadSmall {
  HeadGrads g;              // of the forward: n_rows, V and tok
  Rows h, w;
  int d, m_parts;
  float c, inv_t;
  float* x_tok;
  float4* parts;            // [32 ids][m_parts]
  float* D;                 // [rows, a multiple of 32][ld], zero past the last row and id
  int ld, h_blocks;         // blocks of dH, those of dW follow
  int h_tiles, h_steps;     // of a split of dH's contraction; with several their sums go to slab [split][rows][d]
  float* slab;
  HeadRow* rows;
  void *gh, *gw;
  int64_t gh_stride, gw_stride;
  int gw_f32, add;
};

// 16 columns (or rows) of an operand by 16 of k: element (m, k) at p[m stride + k], or ACROSS at p[k stride + m].  Lane
// (m, grp) takes k = 16 step + 4 grp ..+3; those at K and past it are 0, as are (ON) rows k that are off.
template <typename T, bool ACROSS, bool ON>
struct SmallOperand {
  static constexpr int W = sizeof(T) == 2 && !ACROSS ? 2 : 4;
  struct Raw { uint32_t w[W]; int on[ON ? 4 : 1]; };
  const T* p;
  const HeadRow* rows;
  int64_t stride;
  int K, k0;
  __device__ SmallOperand(Rows m, const HeadRow* r, int t0, int n, int K_) : rows(r), stride(m.stride), K(K_) {
    const int lane = threadIdx.x & 63, at = min(t0 + (lane & 15), n - 1);
    k0 = 4 * (lane >> 4);
    p = (const T*)m.p + (ACROSS ? at : at * m.stride);
  }
  __device__ __forceinline__ void load(Raw& x, int step) const {
    const int k = k0 + 16 * step;
    if constexpr (ACROSS) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int kk = min(k + j, K - 1);
        if constexpr (sizeof(T) == 2) x.w[j] = p[kk * stride];
        else x.w[j] = __float_as_uint(p[kk * stride]);
        if (ON) x.on[j] = rows[kk].on;
      }
    } else {                                               // K is a multiple of 4
      const T* q = p + min(k, K - 4);
      if constexpr (sizeof(T) == 2) { const u32x2 v = *(const u32x2*)q; x.w[0] = v[0]; x.w[1] = v[1]; }
      else { const u32x4 v = *(const u32x4*)q; x.w[0] = v[0]; x.w[1] = v[1]; x.w[2] = v[2]; x.w[3] = v[3]; }
    }
  }
  __device__ __forceinline__ f32x4 value(const Raw& x, int step) const {
    const int k = k0 + 16 * step;
    f32x4 f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (W == 2) f[j] = __uint_as_float(j & 1 ? x.w[j >> 1] & 0xFFFF0000u : x.w[j >> 1] << 16);
      else f[j] = __uint_as_float(sizeof(T) == 2 ? x.w[j] << 16 : x.w[j]);
      f[j] = k + j < K && (!ON || x.on[ON ? j : 0]) ? f[j] : 0.f;
    }
    return f;
  }
};

struct SmallLds {
  float part[4][32][36];
  HeadRow rows[32];
};

// Of the tile's sum over the 16-wide steps [first, steps) of k: columns 4 (t % 8) ..+3 of row t / 8 for thread t
template <typename A, typename B>
__device__ __forceinline__ f32x4 small_tile(const A& a0, const A& a1, const B& b0, const B& b1, int first, int steps, SmallLds& lds) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, row = lane & 15, grp = lane >> 4;
  constexpr int DEPTH = 4;
  struct { typename A::Raw a[2]; typename B::Raw b[2]; } at[DEPTH];
  auto load = [&](int s, int u) {
    const int st = min(s, steps - 1);
    a0.load(at[u].a[0], st);
    a1.load(at[u].a[1], st);
    b0.load(at[u].b[0], st);
    b1.load(at[u].b[1], st);
  };
  f32x4 acc[2][2] = {};
#pragma unroll
  for (int u = 0; u < DEPTH; ++u) load(first + wave + 4 * u, u);
  for (int s = first + wave; s < steps; s += 4 * DEPTH) {
#pragma unroll
    for (int u = 0; u < DEPTH; ++u) {
      const int st = s + 4 * u;
      if (st < steps) {
        const f32x4 x[2] = {a0.value(at[u].a[0], st), a1.value(at[u].a[1], st)};
        const f32x4 y[2] = {b0.value(at[u].b[0], st), b1.value(at[u].b[1], st)};
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int n = 0; n < 2; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[m][j], y[n][j], acc[m][n], 0, 0, 0);
      }
      load(st + 4 * DEPTH, u);
    }
  }
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int q = 0; q < 4; ++q) lds.part[wave][16 * m + 4 * grp + q][16 * n + row] = acc[m][n][q];
  __syncthreads();
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < 4; ++w) v += *(const f32x4*)&lds.part[w][threadIdx.x >> 3][4 * (threadIdx.x & 7)];
  return v;
}

// The statistics of a tile of logits, or its D
template <typename T, bool GRAD>
__global__ __launch_bounds__(256, 2) void k_head_small(HeadSmall a) {
  __shared__ __attribute__((aligned(16))) SmallLds lds;
  const int M = a.g.n_rows, V = a.g.V, mb = (M + 31) >> 5, bn = blockIdx.x / mb, m0 = 32 * (blockIdx.x - bn * mb), n0 = 32 * bn;
  if (GRAD && threadIdx.x < 32) {
    const HeadRow r = head_row(a.g, m0 + threadIdx.x);
    lds.rows[threadIdx.x] = r;
    if (bn == 0) a.rows[m0 + threadIdx.x] = r;
  }
  typedef SmallOperand<T, false, false> Op;
  const f32x4 z = small_tile(Op(a.h, nullptr, m0, M, a.d), Op(a.h, nullptr, m0 + 16, M, a.d), Op(a.w, nullptr, n0, V, a.d),
                             Op(a.w, nullptr, n0 + 16, V, a.d), 0, (a.d + 15) >> 4, lds);
  const int ri = threadIdx.x >> 3, r = m0 + ri, id = n0 + 4 * (threadIdx.x & 7), left = V - id;
  if constexpr (GRAD) {
    const HeadRow hr = lds.rows[ri];
    f32x4 y;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      // x formed again may lie above the forward's maximum by its rounding, which a low temperature would blow up
      const float u = __builtin_amdgcn_fmed3f((z[q] - hr.m) * a.c, -150.f, 0.f);
      y[q] = __builtin_amdgcn_exp2f(u) * fmaf(hr.B, u, hr.A) + (id + q == hr.tok ? hr.g : 0.f);
      if (!hr.on || q >= left) y[q] = 0.f;
    }
    *(f32x4*)(a.D + (int64_t)r * a.ld + id) = y;
  } else {
    const int tok = r < M ? a.g.tok[r] - id : -1;
    HeadSum sum = {-FLT_MAX, 0.f, 0.f};                    // a logit that is not finite makes the row NaN
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      sum.m = fmaxf(sum.m, q < left ? z[q] : NAN);
      if (q == tok && q < left) a.x_tok[r] = z[q];
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float u = q < left ? (z[q] - sum.m) * a.c : -INFINITY;
      const float e = q < left && z[q] == -INFINITY ? NAN : __builtin_amdgcn_exp2f(u);
      sum.s += e;
      sum.t = fmaf(e, fmaxf(u, -FLT_MAX), sum.t);
    }
#pragma unroll
    for (int x = 1; x < 8; x <<= 1)
      head_merge(sum, HeadSum{__shfl_xor(sum.m, x, 64), __shfl_xor(sum.s, x, 64), __shfl_xor(sum.t, x, 64)}, a.c);
    if ((threadIdx.x & 7) == 0 && r < M) a.parts[(size_t)bn * a.m_parts + r] = make_float4(sum.m, sum.s, sum.t, 0.f);
  }
}

// dH = D W and dW = D^T H
template <typename T>
__global__ __launch_bounds__(256, 2) void k_head_small_grads(HeadSmall a) {
  __shared__ __attribute__((aligned(16))) SmallLds lds;
  const int R = a.g.n_rows, V = a.g.V, nb = (a.d + 31) >> 5;
  const bool of_h = (int)blockIdx.x < a.h_blocks;
  const int split = of_h ? blockIdx.x / a.h_tiles : 0;
  const int b = of_h ? blockIdx.x - split * a.h_tiles : blockIdx.x - a.h_blocks, bm = b / nb, m0 = 32 * bm, n0 = 32 * (b - bm * nb);
  const int ri = m0 + (threadIdx.x >> 3), col = n0 + 4 * (threadIdx.x & 7);
  const Rows D = {a.D, a.ld};
  f32x4 v;
  if (of_h) {
    typedef SmallOperand<float, false, false> A;
    typedef SmallOperand<T, true, false> B;
    v = small_tile(A(D, nullptr, m0, R, a.ld), A(D, nullptr, m0 + 16, R, a.ld), B(a.w, nullptr, n0, a.d, V), B(a.w, nullptr, n0 + 16, a.d, V),
                   split * a.h_steps, min((split + 1) * a.h_steps, (V + 15) >> 4), lds);
    if (ri >= R || col >= a.d) return;                     // d is a multiple of 4
    if (a.h_blocks > a.h_tiles) {
      *(f32x4*)(a.slab + ((int64_t)split * R + ri) * a.d + col) = v;
      return;
    }
    v = a.rows[ri].on ? v * a.inv_t : f32x4{0.f, 0.f, 0.f, 0.f};   // whatever the weight holds
    T* y = (T*)a.gh + ri * a.gh_stride + col;
    if constexpr (sizeof(T) == 2) *(uint2*)y = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
    else *(f32x4*)y = v;
    return;
  }
  typedef SmallOperand<float, true, false> A;
  typedef SmallOperand<T, true, true> B;
  v = small_tile(A(D, nullptr, m0, V, R), A(D, nullptr, m0 + 16, V, R), B(a.h, a.rows, n0, a.d, R), B(a.h, a.rows, n0 + 16, a.d, R), 0,
                 (R + 15) >> 4, lds);
  if (ri >= V || col >= a.d) return;
  v *= a.inv_t;
  if (a.gw_f32) {
    f32x4* y = (f32x4*)((float*)a.gw + ri * a.gw_stride + col);
    if (a.add) v += *y;
    *y = v;
  } else {
    u32x2* y = (u32x2*)((uint16_t*)a.gw + ri * a.gw_stride + col);
    if (a.add)
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] += __uint_as_float(q & 1 ? (*y)[q >> 1] & 0xFFFF0000u : (*y)[q >> 1] << 16);
    *y = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
  }
}

// dH from the splits' sums
template <typename T>
__global__ __launch_bounds__(256) void k_head_sum(const float* __restrict__ slab, int splits, int64_t n, int d,
    const HeadRow* __restrict__ rows, float inv_t, T* __restrict__ out, int64_t stride) {
  const int64_t i = 4 * (blockIdx.x * (int64_t)256 + threadIdx.x);
  if (i >= n) return;
  const int64_t r = i / d;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (rows[r].on)
    for (int s = 0; s < splits; ++s) v += *(const f32x4*)(slab + s * n + i);
  v *= inv_t;
  T* y = out + r * stride + (i - r * d);
  if constexpr (sizeof(T) == 2) *(uint2*)y = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
  else *(f32x4*)y = v;
}

// The weight's gradient of no rows
__global__ __launch_bounds__(256) void k_head_zero(uint32_t* __restrict__ out, int64_t stride, int words) {
  for (int i = threadIdx.x; i < words; i += 256) out[blockIdx.x * stride + i] = 0u;
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------
constexpr uint32_t kPairs1 = 0;                            // (0, 0)
constexpr uint32_t kPairs2 = 0x01;                         // a in two parts: (1, 0), (0, 0)
constexpr uint32_t kPairs3 = 0x041852;                     // (2, 0), (1, 1), (0, 2), (1, 0), (0, 1), (0, 0)
constexpr int64_t kPieceBytes = 448 << 20;                 // of D, and of the parts of a piece of an fp32 weight
constexpr int kMaxSteps = 4096;                            // k steps of a block: 64 flags a lane
constexpr int kStatRows = 8192;                            // rows of a launch of the forward tiles
constexpr int kFewRows = 64;
constexpr int kCus = 256;

static int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
static int64_t tiles32(int64_t M, int64_t N) { return (M + 31) / 32 * ((N + 31) / 32); }   // blocks of small tiles

// us of a product of small tiles and of large ones in `pairs` pairs of parts, by rounds of the compute units: 2.4 and 4 us for
// each 256 of k and pair, half of that where a small tile has a compute unit to itself, but 0.75 for a start and its stores
// where many follow each other.  In all (small, large):
//   fp32  509 rows, width 256, 512 ids     forward 12, 53   gradients 18, 186
//         777      1024       4096                132, 133            306, 311
//         1024     1024       8192                302, 143            735, 374
//   bf16  512      512        2048                 31, 31              66, 105
//         1024     512        2048                 54, 31             120, 131
//         1024     1024       8192                297, 41             749, 155
static double small_us(int64_t M, int64_t N, int64_t K, int splits = 1) {
  const int64_t tiles = tiles32(M, N) * splits;
  K = (K + splits - 1) / splits;
  const double tile = 2.4 * K / 256;
  return (splits > 1 ? 10 : 5) + (tiles <= kCus ? 0.5 * tile : (double)(up(tiles, kCus) / kCus) * std::max(tile, 0.75));
}
static double large_us(int64_t M, int64_t N, int64_t K, int pairs) {
  return 14 + (double)(up(((M + 255) / 256) * ((N + 255) / 256), kCus) / kCus) * K * pairs * 4 / 256;
}

HeadPlan head_plan(int dtype, int n_rows, int d, int V, int weight_f32, bool grad) {
  HeadPlan p = {};
  const bool f32 = dtype == SARA_F32;
  const int cols = (V + 255) / 256;
  auto take = [&](int64_t bytes) { const int64_t at = p.bytes; p.bytes += up(bytes, 256); return at; };
  p.width = (int)up(d, 32);
  if (!grad) {
    p.few = n_rows <= kFewRows;
    p.x_tok = take(4 * (int64_t)n_rows);
    if (p.few) {
      p.nt = n_rows <= 16 ? 1 : n_rows <= 32 ? 2 : 4;
      p.few_blocks = (int)std::min<int64_t>((V + 127) / 128, 2 * kCus);
      p.parts = take(16 * (int64_t)16 * p.nt * p.few_blocks);
      return p;
    }
    p.small = small_us(n_rows, V, d) < large_us(n_rows, V, d, f32 ? 6 : 1) + (f32 ? 10 : 5) &&   // and what packing takes
              tiles32(n_rows, V) <= kMaxBlocks;
    if (p.small) {
      p.parts = take(16 * (int64_t)n_rows * ((V + 31) / 32));
      return p;
    }
    p.rows_out = (int)up(n_rows, 256);
    p.parts = take(16 * (int64_t)std::min(p.rows_out, kStatRows) * cols);
    p.h_parts = take((f32 ? 6 : 2) * (int64_t)p.rows_out * p.width);
    p.piece = f32 ? (int)std::min<int64_t>(cols, std::max<int64_t>(1, kPieceBytes / (6 * 256 * (int64_t)p.width))) : cols;
    if (f32) p.w_parts = take(6 * 256 * (int64_t)p.piece * p.width);
    return p;
  }
  const int pairs = f32 ? 6 : 1;
  // Splits of a small dH's contraction, of 1,024 ids or more.  Two fp32 rows of width 256 over 151,936 ids: 238 us
  // for the gradients, 640 in large tiles.
  const int ids16 = (V + 15) / 16;
  const int64_t h_tiles = tiles32(n_rows, d);
  const int h_splits = (int)std::max<int64_t>(1, std::min<int64_t>(2 * kCus / h_tiles, ids16 / 64));
  const double large = large_us(n_rows, V, d, pairs) + large_us(n_rows, d, (V + 63) / 64, pairs) + large_us(V, d, n_rows, pairs);
  // The parts of an fp32 weight are written once and read for each pair, twice over: 34 bytes an element
  const double parts = f32 ? (double)V * d * 34 / 5e6 : 0;
  p.small = small_us(n_rows, V, d) + small_us(n_rows, d, V, h_splits) + small_us(V, d, n_rows) < std::max(large, parts) + (f32 ? 75 : 40) &&
            tiles32(n_rows, V) <= kMaxBlocks && h_splits * h_tiles + tiles32(V, d) <= kMaxBlocks;
  if (p.small) {
    p.width = (int)up(V, 32);
    p.rows = take(sizeof(HeadRow) * up(n_rows, 32));
    p.d = take(4 * up(n_rows, 32) * p.width);
    p.h_steps = (ids16 + h_splits - 1) / h_splits;
    p.splits = (ids16 + p.h_steps - 1) / p.h_steps;
    if (p.splits > 1) p.slab = take(4 * (int64_t)p.splits * n_rows * d);
    return p;
  }
  p.rows_out = (int)up(n_rows, 256);
  p.d_parts = f32 ? 3 : weight_f32 ? 2 : 1;
  const int all_parts = p.d_parts + (f32 ? 0 : 1);
  const int mb = p.rows_out / 256;
  int64_t most = kPieceBytes / (512 * (int64_t)all_parts * p.rows_out);
  if (f32) most = std::min(most, kPieceBytes / (6 * 256 * (int64_t)p.width));
  most = std::min<int64_t>(cols, std::max<int64_t>(1, most));
  // pieces of about the same size; whole rounds of the chip's compute units where that fits
  const int64_t even = (cols + (cols + most - 1) / most - 1) / ((cols + most - 1) / most);
  const int64_t round = up(even * mb, kCus) / mb;
  p.piece = (int)(round <= most ? round : even);
  // Splits of dH's contraction: rounds of blocks, a step of 0.4 us (0.8 where all compute units draw power) and 12 us a
  // block, against the sums' way to memory.  2,048 rows of width 1,536 over 57,344 ids: 317-387 us in 16 splits, which are three
  // whole rounds, and 44 us to add them up; 318 in five, and 13.
  const int64_t tiles = (int64_t)mb * ((d + 255) / 256);
  const int k_steps = (std::min(V, 256 * p.piece) + 31) / 32;
  const int fewest = (k_steps + kMaxSteps - 1) / kMaxSteps;
  double best = INFINITY;
  for (int s = fewest; s <= std::max(64, fewest) && (s == fewest || s * 16 <= k_steps); ++s) {
    const int64_t rounds = up(tiles * s, kCus) / kCus;
    const double busy = (double)(tiles * s) / (double)(rounds * kCus);
    const double us = rounds * ((0.4 + 0.4 * busy) * (double)up((k_steps + s - 1) / s, 16) + 12) + s * (double)n_rows * d * 8 / 4.5e6;
    if (us < best) { best = us; p.splits = s; }
  }
  const int steps = (int)up((k_steps + p.splits - 1) / p.splits, 16);   // the first piece writes every split
  p.splits = (k_steps + steps - 1) / steps;
  p.rows = take(sizeof(HeadRow) * (int64_t)p.rows_out);
  p.d = take(512 * (int64_t)all_parts * p.rows_out * p.piece);
  p.id_flags = take((int64_t)mb * up(8 * p.piece, 64));
  p.row_flags = take((int64_t)p.piece * up(p.rows_out / 32, 64));
  p.slab = take(4 * (int64_t)p.splits * n_rows * d);
  p.h_parts = take(2 * (int64_t)(f32 ? 3 : 1) * p.rows_out * p.width);
  if (f32) p.w_parts = take(6 * 256 * (int64_t)p.piece * p.width);
  return p;
}

static int head_done(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SARA_OK : hip_fail(e, what);
}

static dim3 tile_grid(const HeadTile& t) {
  return dim3(((t.M + 255) / 256) * ((t.N + 255) / 256) * ((((t.K + 31) / 32) + t.steps - 1) / t.steps));
}

// packed into rows_out rows (a multiple of 16) of `width` elements (of 32)
static void pack(bool f32, const void* x, int64_t stride, int n_rows, int d, const HeadRow* rows, uint16_t* y, int rows_out, int width,
                 hipStream_t st) {
  const int tiles = rows_out / 16, blocks = width / 32;
  const dim3 grid(tiles, std::max(1, std::min((blocks + 3) / 4, 2048 / tiles)));
  if (f32) hipLaunchKernelGGL((k_head_pack<float, 3>), grid, dim3(256), 0, st, (const float*)x, stride, n_rows, d, rows, y, tiles, blocks);
  else hipLaunchKernelGGL((k_head_pack<uint16_t, 1>), grid, dim3(256), 0, st, (const uint16_t*)x, stride, n_rows, d, rows, y, tiles, blocks);
}

int launch_head_logprobs(const void* h, int64_t h_stride, const void* w, int64_t w_stride, int dtype, int n_rows, int d, int V,
                         const int32_t* tok, float temp, float* logp, float* entropy, float* stats, void* ws, hipStream_t st) {
  const HeadPlan p = head_plan(dtype, n_rows, d, V, 0, false);
  const float c = (float)(1.4426950408889634 / (double)temp), inv_t = 1.f / temp;
  float* x_tok = (float*)((char*)ws + p.x_tok);
  float4* parts = (float4*)((char*)ws + p.parts);
  if (p.few) {
    const int E = dtype == SARA_BF16 ? 2 : 4;
    const HeadFew f = {(const char*)h, (const char*)w, h_stride * E, w_stride * E, n_rows, d * E / 16, V, tok, c, x_tok, parts};
    auto go = [&](auto k) { hipLaunchKernelGGL(k, dim3(p.few_blocks), dim3(512), 0, st, f); };
    if (dtype == SARA_BF16) {
      if (p.nt == 1) go(k_head_few<uint16_t, 1>);
      else if (p.nt == 2) go(k_head_few<uint16_t, 2>);
      else go(k_head_few<uint16_t, 4>);
    } else {
      if (p.nt == 1) go(k_head_few<float, 1>);
      else if (p.nt == 2) go(k_head_few<float, 2>);
      else go(k_head_few<float, 4>);
    }
    hipLaunchKernelGGL((k_head_join<1>), dim3(n_rows), dim3(256), 0, st, parts, p.few_blocks, 16 * p.nt, 0, n_rows, V, tok, x_tok, c,
                       inv_t, logp, entropy, stats);
    return head_done("head log probabilities launch");
  }
  if (p.small) {
    HeadSmall a = {};
    a.g.n_rows = n_rows;
    a.g.V = V;
    a.g.tok = tok;
    a.h = Rows{h, h_stride};
    a.w = Rows{w, w_stride};
    a.d = d;
    a.m_parts = n_rows;
    a.c = c;
    a.x_tok = x_tok;
    a.parts = parts;
    const dim3 grid((n_rows + 31) / 32 * ((V + 31) / 32));
    if (dtype == SARA_F32) hipLaunchKernelGGL((k_head_small<float, false>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_head_small<uint16_t, false>), grid, dim3(256), 0, st, a);
    hipLaunchKernelGGL((k_head_join<4>), dim3((n_rows + 3) / 4), dim3(256), 0, st, parts, (V + 31) / 32, n_rows, 0, n_rows, V, tok, x_tok, c,
                       inv_t, logp, entropy, stats);
    return head_done("head log probabilities launch");
  }
  const bool f32 = dtype == SARA_F32;
  uint16_t *hp = (uint16_t*)((char*)ws + p.h_parts), *wp = (uint16_t*)((char*)ws + p.w_parts);
  const int h_tiles = p.rows_out / 16, w_tiles = 16 * p.piece;
  pack(f32, h, h_stride, n_rows, d, nullptr, hp, p.rows_out, p.width, st);
  const int cols = (V + 255) / 256;
  for (int row0 = 0; row0 < n_rows; row0 += kStatRows) {
    const int M = std::min(kStatRows, n_rows - row0);
    for (int c0 = 0; c0 < cols; c0 += p.piece) {
      HeadTile t = {};
      t.v0 = 256 * c0;
      t.M = M;
      t.N = std::min(V - t.v0, 256 * p.piece);
      t.a = Mat{hp + (int64_t)row0 / 16 * 512, h_tiles, (int64_t)p.rows_out * p.width};
      t.K = f32 ? p.width : d;
      t.n_pairs = f32 ? 6 : 1;
      t.pairs = f32 ? kPairs3 : kPairs1;
      t.steps = (t.K + 31) / 32;
      t.row0 = row0;
      t.m_parts = std::min(p.rows_out, kStatRows);
      t.c = c;
      t.tok = tok;
      t.x_tok = x_tok;
      t.parts = parts;
      if (f32) {
        if (row0 == 0 || p.piece < cols)
          pack(true, (const float*)w + t.v0 * w_stride, w_stride, t.N, d, nullptr, wp, 256 * p.piece, p.width, st);
        t.b = Mat{wp, w_tiles, 256 * (int64_t)p.piece * p.width};
        hipLaunchKernelGGL((k_head_tile<kPacked, kPacked, kStats>), tile_grid(t), dim3(kTileThreads), 0, st, t);
      } else {
        t.b = Mat{(const uint16_t*)w + t.v0 * w_stride, w_stride, 0};
        hipLaunchKernelGGL((k_head_tile<kPacked, kRowPairs, kStats>), tile_grid(t), dim3(kTileThreads), 0, st, t);
      }
    }
    hipLaunchKernelGGL((k_head_join<4>), dim3((M + 3) / 4), dim3(256), 0, st, parts, cols, std::min(p.rows_out, kStatRows), row0, M, V,
                       tok, x_tok, c, inv_t, logp, entropy, stats);
  }
  return head_done("head log probabilities launch");
}

int launch_head_logprobs_grad(const void* h, int64_t h_stride, const void* w, int64_t w_stride, int dtype, int n_rows, int d, int V,
                              const int32_t* tok, float temp, const float* stats, const float* entropy, const float* g_logp,
                              const float* g_ent, void* gh, int64_t gh_stride, void* gw, int64_t gw_stride, int gw_f32, int accumulate,
                              void* ws, hipStream_t st) {
  const int EW = gw_f32 ? 4 : 2;
  if (n_rows == 0) {
    if (gw && !accumulate)
      hipLaunchKernelGGL(k_head_zero, dim3(V), dim3(256), 0, st, (uint32_t*)gw, gw_stride * EW / 4, d * EW / 4);
    return head_done("head log probabilities gradient launch");
  }
  const HeadPlan p = head_plan(dtype, n_rows, d, V, gw_f32, true);
  const bool f32 = dtype == SARA_F32;
  const float c = (float)(1.4426950408889634 / (double)temp);
  const int half = ilogbf(1.f / temp) / 2;
  const float scale = ldexpf(1.f, half), inv_t = ldexpf(1.f / temp, -half);   // of D, of the results
  auto at = [&](int64_t off) { return (char*)ws + off; };
  HeadRow* rows = (HeadRow*)at(p.rows);
  uint16_t *D = (uint16_t*)at(p.d), *hp = (uint16_t*)at(p.h_parts), *wp = (uint16_t*)at(p.w_parts);
  float* slab = (float*)at(p.slab);
  auto sum = [&]() {
    const int64_t n = (int64_t)n_rows * d;
    const dim3 grid((uint32_t)((n / 4 + 255) / 256));
    if (f32) hipLaunchKernelGGL((k_head_sum<float>), grid, dim3(256), 0, st, slab, p.splits, n, d, rows, inv_t, (float*)gh, gh_stride);
    else hipLaunchKernelGGL((k_head_sum<uint16_t>), grid, dim3(256), 0, st, slab, p.splits, n, d, rows, inv_t, (uint16_t*)gh, gh_stride);
  };
  const HeadGrads g = {n_rows, V, tok, stats, entropy, g_logp, g_ent, scale, 1.f / c};
  if (p.small) {
    HeadSmall a = {};
    a.g = g;
    a.h = Rows{h, h_stride};
    a.w = Rows{w, w_stride};
    a.d = d;
    a.c = c;
    a.inv_t = inv_t;
    a.D = (float*)D;
    a.ld = p.width;
    a.rows = rows;
    a.gh = gh;
    a.gw = gw;
    a.gh_stride = gh_stride;
    a.gw_stride = gw_stride;
    a.gw_f32 = gw_f32;
    a.add = accumulate;
    a.h_tiles = (n_rows + 31) / 32 * ((d + 31) / 32);
    a.h_steps = p.h_steps;
    a.h_blocks = gh ? p.splits * a.h_tiles : 0;
    a.slab = slab;
    const dim3 of_d((n_rows + 31) / 32 * ((V + 31) / 32)), of_grads(a.h_blocks + (gw ? (V + 31) / 32 * ((d + 31) / 32) : 0));
    auto go = [&](auto k, dim3 grid) { hipLaunchKernelGGL(k, grid, dim3(256), 0, st, a); };
    if (dtype == SARA_F32) { go(k_head_small<float, true>, of_d); go(k_head_small_grads<float>, of_grads); }
    else { go(k_head_small<uint16_t, true>, of_d); go(k_head_small_grads<uint16_t>, of_grads); }
    if (gh && p.splits > 1) sum();
    return head_done("head log probabilities gradient launch");
  }
  hipLaunchKernelGGL(k_head_rows, dim3(p.rows_out / 256), dim3(256), 0, st, g, p.rows_out, rows);
  pack(f32, h, h_stride, n_rows, d, rows, hp, p.rows_out, p.width, st);
  const int cols = (V + 255) / 256, tiles = p.rows_out / 16;
  uint8_t *id_flags = (uint8_t*)at(p.id_flags), *row_flags = (uint8_t*)at(p.row_flags);
  const int id_stride = (int)up(8 * p.piece, 64), row_stride = (int)up(p.rows_out / 32, 64);
  const Mat hm = {hp, tiles, (int64_t)p.rows_out * p.width}, dm = {D, tiles, 256 * (int64_t)p.piece * p.rows_out};
  auto go = [&](auto kernel, const HeadTile& t) { hipLaunchKernelGGL(kernel, tile_grid(t), dim3(kTileThreads), 0, st, t); };
  for (int c0 = 0; c0 < cols; c0 += p.piece) {
    const int v0 = 256 * c0, N = std::min(V - v0, 256 * p.piece);
    Mat wm = {(const uint16_t*)w + v0 * w_stride, w_stride, 0};
    if (f32) {
      pack(true, (const float*)w + v0 * w_stride, w_stride, N, d, nullptr, wp, 256 * p.piece, p.width, st);
      wm = Mat{wp, 16 * p.piece, 256 * (int64_t)p.piece * p.width};
    }
    HeadTile t = {};
    t.v0 = v0;
    t.M = n_rows;
    t.N = N;
    t.a = hm;
    t.b = wm;
    t.K = f32 ? p.width : d;
    t.n_pairs = f32 ? 6 : 1;
    t.pairs = f32 ? kPairs3 : kPairs1;
    t.steps = (t.K + 31) / 32;
    t.c = c;
    t.rows = rows;
    t.d = D;
    t.d_tiles = tiles;
    t.d_part = dm.part;
    if (!f32) {
      t.id_flags = id_flags;
      t.row_flags = row_flags;
      t.id_flags_stride = id_stride;
      t.row_flags_stride = row_stride;
    }
    if (f32) go(k_head_tile<kPacked, kPacked, kGradRows + 3>, t);
    else if (p.d_parts == 2) go(k_head_tile<kPacked, kRowPairs, kGradRows + 2>, t);
    else go(k_head_tile<kPacked, kRowPairs, kGradRows + 1>, t);
    if (gh) {
      HeadTile x = {};
      x.a = dm;
      x.b = wm;
      x.M = n_rows;
      x.N = d;
      x.K = N;
      x.n_pairs = f32 ? 6 : 1;
      x.pairs = f32 ? kPairs3 : kPairs1;
      x.steps = (int)up(((N + 31) / 32 + p.splits - 1) / p.splits, 16);
      x.flags = id_flags;
      x.flags_stride = id_stride;
      x.sparse = f32 ? 0 : 1;
      x.slab = slab;
      x.add = c0 > 0;
      if (f32) go(k_head_tile<kPacked, kPackedT, kSlab>, x);
      else go(k_head_tile<kPacked, kCols, kSlab>, x);
    }
    if (gw) {
      HeadTile x = {};
      x.a = dm;
      x.b = hm;
      x.M = N;
      x.N = d;
      x.K = (int)up(n_rows, 32);
      x.n_pairs = f32 ? 6 : p.d_parts;
      x.pairs = f32 ? kPairs3 : p.d_parts == 2 ? kPairs2 : kPairs1;
      x.steps = x.K / 32;
      x.flags = row_flags;
      x.flags_stride = row_stride;
      x.sparse = f32 ? 0 : p.d_parts;
      x.inv_t = inv_t;
      x.out = (char*)gw + v0 * gw_stride * EW;
      x.out_stride = gw_stride;
      x.out_f32 = gw_f32;
      x.add = accumulate;
      go(k_head_tile<kPackedT, kPackedT, kWeight>, x);
    }
  }
  if (gh) sum();
  return head_done("head log probabilities gradient launch");
}

}  // namespace sara
