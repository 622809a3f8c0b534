// Softmax cross entropy of tokens against a vocabulary, z = x w^T, without keeping z:
//
//   lse_i = ln sum_v exp z_iv,   loss_i = lse_i - z_i,label
//   g_iv = (exp(z_iv - lse_i) - [v = label_i]) d_loss_i,   dx = g w,   dw = g^T x
//
// Tokens without a label (negative) take no part: the first launch lists the others (xent_list_kernel), and every product runs
// over that list, whose length stays on the device.  What such a token's features hold, a NaN for instance, reaches nothing.
//
// Forward: the product, whose epilogue leaves the largest logit and the sum of exponentials of every token in a wave's columns,
// and the label's logit; one launch joins them.  Backward: piece by piece of the vocabulary the product again, whose epilogue
// writes g of the piece, then dw of the piece, whole, and the piece's share of dx, which is summed in float32 and rounded behind the
// last piece.  g is bf16 for the matrix cores, one rounding, like a gradient that a layer hands on, and it is kept divided by the
// largest |d_loss|, by which the sums are multiplied in the end: for a mean over the tokens, d_loss = 1 / count everywhere, the label's
// entry p - 1 is then near -1 and next to exact, where -1 / count would carry the same rounding, up to 2^-8, into every gradient.
// No atomics: results repeat bit for bit.
//
// bf16 tiles as in the projections (lvx_project.hip, lvx_project_bwd.hip): a workgroup of 4 waves makes 256 x 256 of a product, a
// wave 128 x 128 of it as 4 x 4 blocks in the accumulation registers, tile pairs of 64 contraction steps go through two
// slots of 64 KB.
#include "lvx_internal.h"
#include "lvx_mfma.h"
#include "lvx_kv_ring.h"

#include <type_traits>

namespace lvx {

namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int T = 256, BK = 64, NSLOT = 2;
constexpr int RK_ROWB = BK * 2;        // [256][64] tile: bytes of a row
constexpr int KR_ROWB = T * 2;         // [64][256] tile
constexpr int TILE_B = BK * KR_ROWB, SLOT_B = 2 * TILE_B, RING_B = NSLOT * SLOT_B;
constexpr int TB_PITCH = 128 * 2 + 16, TB_WAVE = 128 * TB_PITCH;       // epilogue: a wave's rows on their way out
constexpr int SMEM_B = RING_B > 4 * TB_WAVE ? RING_B : 4 * TB_WAVE;
enum { STATS = 0, GRAD = 1, DX = 2, DW = 3 };

__device__ __forceinline__ int perm_of(int r) { return (r & 7) ^ ((r >> 3) & 1); }
template <int J> __device__ __forceinline__ unsigned row_lane(unsigned x) {       // lane J of every 16
  return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x150 + J, 0xf, 0xf, true);
}
// (a value that the compiler works on only where it stands: comparisons with it, made ahead for all row blocks, spill)
__device__ __forceinline__ int opaque(int x) {
  asm volatile("" : "+v"(x));
  return x;
}
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Entry of a list of tiles (a, b), n_a x n_b, in strips of four a: 32 neighbours, what an XCD works on at a time, share four a and
// eight b, and every XCD takes a run of the list.  In rows of the longer dimension they would share one and 32, nearly three times
// the operands.
__device__ __forceinline__ void strip_tile(long entry, int n_a, int n_b, int* ta, int* tb) {
  const int strip = (int)(entry / (4L * n_b)), rest = (int)(entry - strip * (4L * n_b));
  const int w = min(4, n_a - 4 * strip);
  *ta = 4 * strip + rest % w;
  *tb = rest / w;
}
inline long strip_grid(long tiles) { return (tiles + 7) / 8 * 8; }
// The tile (and, DX, the part of the contraction) of workgroup blockIdx.x; false: none.  The grid is made for all tokens, the tiles
// are those of the listed ones.
template <int MODE> __device__ __forceinline__ bool take_tile(int n_rt, int n_ct, int parts, int* rt, int* ct, int* part) {
  const long tiles = (long)n_rt * n_ct;
  long entry;
  if (!xcd_run(blockIdx.x, tiles * parts, &entry)) return false;
  *part = MODE == DX ? (int)(entry / tiles) : 0;
  if (MODE == DX) entry -= *part * tiles;
  if (MODE == STATS || MODE == GRAD) strip_tile(entry, n_ct, n_rt, ct, rt);
  else strip_tile(entry, n_rt, n_ct, rt, ct);
  return true;
}
// Parts that the contraction of dx is cut into, by how many tiles the listed tokens make: as many as make the rounds of workgroups
// shortest, within the room for their sums.
__device__ inline int dx_parts(long tiles, int n_cu, int slots) {
  int best = 1;
  float best_t = 1e30f;
  for (int p = 1; p <= 16 && p * tiles <= slots; ++p) {
    const float t = (float)((tiles * p + n_cu - 1) / n_cu) / (float)p;
    if (t < 0.95f * best_t) {
      best = p;
      best_t = t;
    }
  }
  return best;
}

// ---- the tokens that have a label, in order: tok[i] and its label (-1: not in the vocabulary), and how many they are ----
__global__ void __launch_bounds__(1024) xent_list_kernel(XentArgs a) {
  __shared__ int sums[2][16];
  __shared__ float tops[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int total = 0, turn = 0;
  float top = 0.f;                                   // the largest finite |d_loss|
  for (long base = 0; base < a.n; base += 8192) {
    long lab[8];
    int mine = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const long i = base + 8 * tid + k;
      lab[k] = i < a.n ? a.labels[i] : -1;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) mine += lab[k] >= 0 ? 1 : 0;
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int y = __shfl_up(upto, o);
      upto += lane >= o ? y : 0;
    }
    turn ^= 1;                                       // (who writes a place again has crossed the barrier between)
    if (lane == 63) sums[turn][wave] = upto;
    __syncthreads();
    int at = total + upto - mine;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      at += w < wave ? sums[turn][w] : 0;
      total += sums[turn][w];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const long i = base + 8 * tid + k;
      if (lab[k] >= 0) {
        a.tok[at] = (int)i;
        a.lab[at] = lab[k] < a.V ? (int)lab[k] : -1;
        ++at;
        if (a.d_loss) {
          const float d = fabsf(a.d_loss[i]);
          if (d > top && d < __builtin_inff()) top = d;
        }
      } else if (a.loss && i < a.n) {
        a.loss[i] = 0.f;
        a.lse_out[i] = 0.f;
      }
    }
  }
#pragma unroll
  for (int o = 1; o < 64; o *= 2) top = fmaxf(top, __shfl_xor(top, o));
  if (lane == 0) tops[wave] = top;
  __syncthreads();
  if (tid != 0) return;
  for (int w = 0; w < 16; ++w) top = fmaxf(top, tops[w]);
  a.head->count = total;
  a.head->scale = top > 0.f ? top : 1.f;
  a.head->parts = dx_parts((long)((total + a.tile - 1) / a.tile) * ((a.E + a.tile - 1) / a.tile), a.n_cu, a.slots);
}

// ---- a wave's columns of a logits tile.  z(v, j): the logit in column 32 j + 8 (v / 4) + 4 g + v % 4 of the wave's, JB blocks of 32 ----

// the largest logit (times log2 e) and the sum of exponentials against it
template <int JB, bool WHOLE, class Z> __device__ __forceinline__ void tile_stats_of(int g, int cols, Z&& z, float* m2, float* s) {
  float y[JB][16];
  const int end = opaque(cols - 4 * g);
#pragma unroll
  for (int j = 0; j < JB; ++j)
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      y[j][v] = z(v, j) * LOG2E;
      if (!WHOLE) y[j][v] = 32 * j + 8 * (v / 4) + v % 4 < end ? y[j][v] : -__builtin_inff();
    }
  // (a NaN is dropped here and comes back in the sum)
  float mx = y[0][0];
#pragma unroll
  for (int j = 0; j < JB; ++j)
#pragma unroll
    for (int v = 0; v < 16; v += 2) asm("v_max3_f32 %0, %0, %1, %2" : "+v"(mx) : "v"(y[j][v]), "v"(y[j][v + 1]));
  mx = xhalf_max(mx);
  const float at = mx == -__builtin_inff() ? 0.f : mx;
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < JB; ++j)
#pragma unroll
    for (int v = 0; v < 16; ++v) sum += exp2_fast(y[j][v] - at);
  *m2 = mx;
  *s = xhalf_sum(sum);
}
template <int JB, class Z> __device__ __forceinline__ void tile_stats(int g, int cols, Z&& z, float* m2, float* s) {
  if (cols >= 32 * JB) tile_stats_of<JB, true>(g, cols, z, m2, s);      // (uniform)
  else tile_stats_of<JB, false>(g, cols, z, m2, s);
}
// the logit of column c of the wave's, in the lanes whose half holds it
template <int JB, class Z> __device__ __forceinline__ float tile_pick(int g, int c, Z&& z) {
  float y = 0.f;
  const int at = opaque(c - 4 * g);
#pragma unroll
  for (int j = 0; j < JB; ++j)
#pragma unroll
    for (int v = 0; v < 16; ++v) y = 32 * j + 8 * (v / 4) + v % 4 == at ? z(v, j) : y;
  return y;
}

// lse and loss of the listed tokens from what the tiles' waves left: 8 tokens a workgroup, 32 threads each
__global__ void __launch_bounds__(256) xent_join_kernel(XentArgs a, int n_parts) {
  __shared__ float sm[8][33], ss[8][33];
  const int row_l = threadIdx.x % 8, lane = threadIdx.x / 8, count = a.head->count;
  for (int r0 = blockIdx.x * 8; r0 < count; r0 += gridDim.x * 8) {
    const int r = min(r0 + row_l, count - 1);
    float m = -__builtin_inff(), s = 0.f;
    const auto join = [&](float m1, float s1) {
      const float top = fmaxf(m, m1), at = top == -__builtin_inff() ? 0.f : top;
      s = s * exp2_fast(m - at) + s1 * exp2_fast(m1 - at);
      m = top;
    };
    for (int p0 = lane; p0 < n_parts; p0 += 32 * 8) {
      float2 v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = a.part[(long)min(p0 + 32 * i, n_parts - 1) * a.Mp + r];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (p0 + 32 * i < n_parts) join(v[i].x, v[i].y);
    }
    sm[row_l][lane] = m;
    ss[row_l][lane] = s;
    __syncthreads();
    if (threadIdx.x < 8 && r0 + threadIdx.x < count) {
      m = -__builtin_inff();
      s = 0.f;
      for (int i = 0; i < 32; ++i) join(sm[threadIdx.x][i], ss[threadIdx.x][i]);
      const int row = r0 + threadIdx.x, i = a.tok[row];
      const float bad = a.lab[row] < 0 ? __builtin_nanf("") : 0.f;
      const float lse = (m + __builtin_amdgcn_logf(s)) * LN2 + bad;
      a.lse_out[i] = lse;
      a.loss[i] = lse - a.zlab[row];
    }
    __syncthreads();
  }
}

// ---- bf16 products on the matrix cores ----

// MODE STATS, GRAD: rows = listed tokens, columns = vocabulary, contraction over the features.  Both operands have it contiguous:
//   tiles [rows][64], 128-byte lines, chunks permuted by perm_of.
// MODE DX: rows = listed tokens, columns = features, contraction over the piece's vocabulary; g like x before, w as [64][256 features]
//   with transposing reads.
// MODE DW: rows = vocabulary of the piece, columns = features, contraction over the listed tokens: both as [64 tokens][256].
// Rows of x go by the list; rows behind the last token read the last one again (their g is 0), rows of w behind the vocabulary its last
// (their columns of g are 0).
template <int MODE, int RB>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1)))
xent_bf16_kernel(XentArgs a) {
  constexpr bool LOGITS = MODE == STATS || MODE == GRAD;
  static_assert(RB == 4 || LOGITS, "the low tiles are for logits of few tokens");
  constexpr int TR = 64 * RB;                        // rows of a workgroup's tile
  constexpr int NB = MODE == DW ? 8 : 2 * RB;        // copies per wave and tile pair: B side (rows),
  constexpr int NPART = 8 + NB;                      // and with the 8 of the A side (columns)
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int M = a.head->count, E = a.E;
  const int cols = (int)(a.v1 - a.v0);               // of the piece
  const int n_rt = MODE == DW ? (cols + T - 1) / T : (M + TR - 1) / TR;
  const int n_ct = LOGITS ? (cols + T - 1) / T : (E + T - 1) / T;
  const int parts = MODE == DX ? a.head->parts : 1;
  int rt, ct, part;
  if (!take_tile<MODE>(n_rt, n_ct, parts, &rt, &ct, &part)) return;
  const int r0 = rt * TR, c0 = ct * T;               // (of the list / of the piece / of the features)
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, l31 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int nk_all = LOGITS ? E / BK : MODE == DX ? (cols + BK - 1) / BK : (M + BK - 1) / BK;
  const int k0 = MODE == DX ? (int)((long)part * nk_all / parts) : 0;
  const int nk = MODE == DX ? (int)((long)(part + 1) * nk_all / parts) - k0 : nk_all;
  const unsigned smem_u = lds_base(smem);
  const unsigned xrow_b = (unsigned)(a.ldx * 2), wrow_b = (unsigned)(E * 2);
  const long g_row_b = a.g_pitch * 2L;

  // ---- copies into [rows][64] tiles: one instruction moves 8 rows x 128 bytes, lane l the chunk (l % 8) ^ perm_of(row) of row l / 8
  unsigned bo[LOGITS || MODE == DX ? 2 * RB : 1], ao[LOGITS ? 8 : 1];
  if constexpr (LOGITS || MODE == DX) {
#pragma unroll
    for (int j = 0; j < 2 * RB; ++j) {
      const int r = r0 + 16 * RB * wave + 8 * j + (lane >> 3);
      const unsigned swz = 16u * (unsigned)((lane & 7) ^ perm_of(8 * j + (lane >> 3)));
      if (LOGITS) bo[j] = (unsigned)a.tok[min(r, M - 1)] * xrow_b + swz;
      else bo[j] = (unsigned)((16 * RB * wave + 8 * j + (lane >> 3)) * g_row_b) + swz;
    }
  }
  if constexpr (LOGITS) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int r = 64 * wave + 8 * j + (lane >> 3);
      ao[j] = (unsigned)min((long)r, a.V - 1 - a.v0 - c0) * wrow_b + 16u * (unsigned)((lane & 7) ^ perm_of(8 * j + (lane >> 3)));
    }
  }
  // ---- copies into [64][256] tiles: one instruction moves 2 rows x 512 bytes, lane l position l % 32 of row l / 32, which holds the
  // chunk (l % 32) ^ 4 (row % 4); a wave copies rows 16 wave + 2 j + l / 32.  Features past the last one: the tile's first chunk again.
  const int lh = lane >> 5, pos = lane & 31;
  unsigned kr_a[2], kr_b[2];
#pragma unroll
  for (int par = 0; par < 2; ++par) {
    const int c = pos ^ (4 * ((2 * par + lh) & 3));
    kr_a[par] = LOGITS || c0 + 8 * c >= E ? 0u : 16u * (unsigned)c;
    kr_b[par] = 16u * (unsigned)c + (MODE == DW ? (unsigned)((16 * wave + lh) * g_row_b) : 0u);
  }
  // Where the next pair to go out starts on either side (its copies go out in order, pair by pair).  DX: the rows of w left behind the
  // pair's first, and a lane's row.  DW: the byte offsets of the rows of x that a wave copies, lane l that of row 16 wave + 2 (l % 8) + l / 32.
  const char* ap = LOGITS ? (const char*)a.w + (a.v0 + c0) * wrow_b
                          : MODE == DX ? (const char*)a.w + ((a.v0 + k0 * BK) * E + c0) * 2 : (const char*)a.x + 2L * c0;
  const char* bp = LOGITS ? (const char*)a.x
                          : MODE == DX ? (const char*)a.g + r0 * g_row_b + (long)k0 * RK_ROWB : (const char*)a.g + 2L * r0;
  const unsigned a_lane = (unsigned)(16 * wave + lh) * wrow_b;
  long w_left = a.V - 1 - a.v0 - (long)k0 * BK;
  unsigned w_last = 0u;
  const auto x_rows = [&](int kt) __attribute__((always_inline)) -> int { return a.tok[min(kt * BK + 16 * wave + 2 * (lane & 7) + lh, M - 1)]; };
  unsigned xr = 0u;
  // lane j of every 16 lanes
  const auto lane_of_16 = [&](unsigned x, int j) __attribute__((always_inline)) -> unsigned {
    switch (j) {
      case 0: return row_lane<0>(x);
      case 1: return row_lane<1>(x);
      case 2: return row_lane<2>(x);
      case 3: return row_lane<3>(x);
      case 4: return row_lane<4>(x);
      case 5: return row_lane<5>(x);
      case 6: return row_lane<6>(x);
      default: return row_lane<7>(x);
    }
  };
  auto issue_part = [&](int kt, int p) __attribute__((always_inline)) {
    const unsigned st = smem_u + (unsigned)((kt % NSLOT) * SLOT_B);
    if (p < 8) {                                     // A side
      const int j = p;
      if constexpr (LOGITS) {
        dma16u(ap, ao[j], st + (unsigned)((64 * wave + 8 * j) * RK_ROWB));
      } else if constexpr (MODE == DX) {
        if (j == 0) w_last = (unsigned)min(w_left, 63L) * wrow_b;
        dma16u(ap, min(a_lane + (unsigned)(2 * j) * wrow_b, w_last) + kr_a[j & 1], st + (unsigned)((16 * wave + 2 * j) * KR_ROWB));
      } else {
        dma16u(ap, lane_of_16(xr, j) + kr_a[j & 1], st + (unsigned)((16 * wave + 2 * j) * KR_ROWB));
      }
      if (j == 7) {
        if (LOGITS) ap += RK_ROWB;
        if (MODE == DX) { ap += 64L * wrow_b; w_left -= 64; }
      }
    } else {                                         // B side
      const int j = p - 8;
      if constexpr (MODE != DW) dma16u(bp, bo[j], st + (unsigned)(TILE_B + (16 * RB * wave + 8 * j) * RK_ROWB));
      else dma16u(bp, kr_b[j & 1] + (unsigned)(2 * j) * (unsigned)g_row_b, st + (unsigned)(TILE_B + (16 * wave + 2 * j) * KR_ROWB));
      if (j == NB - 1) bp += MODE == DW ? 64 * g_row_b : RK_ROWB;
    }
  };

  // ---- operands (see lvx_project_bwd.hip): from [rows][64] one 16-byte read; from [64][256] two transposing reads, of rows 8 g ..
  // where the other operand has its eight steps in one chunk (DX), 4 g .. and 8 + 4 g .. where both are such tiles (DW)
  const int j16 = lane & 15, jr = j16 >> 2, tr_col = 32 * ((lane >> 4) & 1) + 8 * (j16 & 3);
  constexpr int KG = MODE == DX ? 8 : 4, KH = MODE == DX ? 4 : 8;
  int rd[4], ka[4], kb[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) rd[q] = l31 * RK_ROWB + 16 * ((2 * q + g) ^ perm_of(l31));
#pragma unroll
  for (int jj = 0; jj < 4; ++jj) {
    ka[jj] = (KG * g + jr) * KR_ROWB + tr_col + 64 * ((4 * wn + jj) ^ jr);
    kb[jj] = TILE_B + (KG * g + jr) * KR_ROWB + tr_col + 64 * ((4 * wm + jj) ^ jr);
  }
  auto tr_op = [&](const char* p) __attribute__((always_inline)) -> bf16x8 {
    const s16x4 lo = lds_read_tr(p), hi = lds_read_tr(p + KH * KR_ROWB);
    typedef __attribute__((ext_vector_type(8))) short s16x8;
    const s16x8 r = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    return __builtin_bit_cast(bf16x8, r);
  };
  auto a_op = [&](const char* st, int q, int j) __attribute__((always_inline)) -> bf16x8 {
    if constexpr (LOGITS) return *(const bf16x8*)(st + (wn * 128 + 32 * j) * RK_ROWB + rd[q]);
    else return tr_op(st + ka[j] + 16 * q * KR_ROWB);
  };
  auto b_op = [&](const char* st, int q, int i) __attribute__((always_inline)) -> bf16x8 {
    if constexpr (MODE != DW) return *(const bf16x8*)(st + TILE_B + (wm * 32 * RB + 32 * i) * RK_ROWB + rd[q]);
    else return tr_op(st + kb[i] + 16 * q * KR_ROWB);
  };

  f32x16 acc[4][RB];                                 // [column block j][row block i]: lane = row, registers = columns
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int i = 0; i < RB; ++i) { acc[j][i] = zero16(); asm volatile("" : "+a"(acc[j][i])); }
  constexpr int NU = 4 * RB;
  auto mma16 = [&](const bf16x8 (&bv)[RB], const bf16x8 (&av)[4], auto&& hook) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < RB; ++i) {
        kvring::mfma_acc(acc[j][i], av[j], bv[i]);
        hook(RB * j + i);
        __builtin_amdgcn_sched_barrier(0);
      }
  };

  if (nk > 0) {
#pragma unroll
    for (int q = 0; q < NSLOT; ++q)
      if (q < nk) {
        if constexpr (MODE == DW) xr = (unsigned)x_rows(q) * xrow_b;
#pragma unroll
        for (int p = 0; p < NPART; ++p) issue_part(q, p);
      }
    if (nk > 1) wait_vmcnt<NPART>();
    else wait_vmcnt<0>();
    wg_barrier();
    bf16x8 ba[RB], aa[4], bb[RB], ab[4];             // operands of even / odd k-steps
#pragma unroll
    for (int i = 0; i < RB; ++i) ba[i] = b_op(smem, 0, i);
#pragma unroll
    for (int i = 0; i < 4; ++i) aa[i] = a_op(smem, 0, i);
    auto fetch = [&](const char* st, int q, int u, bf16x8 (&bv)[RB], bf16x8 (&av)[4]) __attribute__((always_inline)) {
      if (u < RB) bv[u] = b_op(st, q, u);
      else if (u < RB + 4) av[u - RB] = a_op(st, q, u - RB);
    };
    constexpr int EB = NU / NB, EA = NU / 8;         // a copy of one side every so many matrix instructions of a k-step
    auto pair = [&](int P, auto steady, bool send2, bool send1, bool more) __attribute__((always_inline)) {
      constexpr bool STEADY = decltype(steady)::value;
      const char* const st = smem + (P % NSLOT) * SLOT_B;
      const char* const sn = smem + ((P + 1) % NSLOT) * SLOT_B;
      mma16(ba, aa, [&](int u) __attribute__((always_inline)) {
        fetch(st, 1, u, bb, ab);
        if ((STEADY || send2) && u % EB == EB - 1) issue_part(P + 1, 8 + u / EB);
      });
      int next_rows = 0;
      if constexpr (MODE == DW) next_rows = x_rows(P + 2);        // (has come when the wait below is over)
      mma16(bb, ab, [&](int u) __attribute__((always_inline)) { fetch(st, 2, u, ba, aa); });
      mma16(ba, aa, [&](int u) __attribute__((always_inline)) { fetch(st, 3, u, bb, ab); });
      if (STEADY || more) {
        __builtin_amdgcn_s_waitcnt(0x0070);            // vmcnt(0) and lgkmcnt(0)
        wg_barrier();
      }
      if constexpr (MODE == DW) xr = (unsigned)next_rows * xrow_b;
      mma16(bb, ab, [&](int u) __attribute__((always_inline)) {
        if (STEADY || more) fetch(sn, 0, u, ba, aa);
        if ((STEADY || send1) && u % EA == EA - 1) issue_part(P + 2, u / EA);
      });
    };
    int P = 0;
    pair(0, std::false_type{}, false, 2 < nk, 1 < nk);
    P = 1;
    for (; P + 2 < nk; ++P) pair(P, std::true_type{}, true, true, true);
    for (; P < nk; ++P) pair(P, std::false_type{}, P + 1 < nk, false, P + 1 < nk);
  }

  // ---- epilogue: every wave has left the ring, and the last matrix instructions have retired
  wg_barrier();
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int i = 0; i < RB; i += 2) asm volatile("s_nop 15\n\ts_nop 15" : "+a"(acc[j][i]), "+a"(acc[j][i + 1]));
  if constexpr (MODE == STATS) {
    const int left = (int)min((long)T, a.V - c0) - wn * 128;      // columns of this wave
    const int p = 2 * ct + wn;
#pragma unroll
    for (int i = 0; i < RB; ++i) {
      const int r = r0 + wm * 32 * RB + 32 * i + l31;
      const auto z = [&](int v, int j) __attribute__((always_inline)) -> float { return acc[j][i][v]; };
      float m2, s;
      tile_stats<4>(g, left, z, &m2, &s);
      if (g == 0 && r < M) a.part[(long)p * a.Mp + r] = make_float2(m2, s);
      const int c = r < M ? a.lab[r] - c0 - wn * 128 : -1;
      if (__any(c >= 0 && c < 128)) {
        const float y = tile_pick<4>(g, c, z);
        if (c >= 0 && c < 128 && ((c >> 2) & 1) == g) a.zlab[r] = y;
      }
    }
  } else if constexpr (MODE == DX) {
    // in the order of the registers, 16 bytes a lane (xent_dx_kernel reads them so), on top of what the pieces before left
    float* const out = a.dx_part + (((long)part * n_rt + rt) * n_ct + ct) * (T * T) + wave * (T * T / 4) + lane * 4;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f32x4 old[RB][4];
      if (!a.first) {
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q) old[i][q] = *(const f32x4*)(out + ((j * RB + i) * 4 + q) * 256);
      }
#pragma unroll
      for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          f32x4 v = {acc[j][i][4 * q], acc[j][i][4 * q + 1], acc[j][i][4 * q + 2], acc[j][i][4 * q + 3]};
          if (!a.first) v += old[i][q];
          *(f32x4*)(out + ((j * RB + i) * 4 + q) * 256) = v;
        }
    }
  } else {
    // turned around in LDS, rounded to bf16, written in whole 256-byte row segments
    char* const tb = smem + wave * TB_WAVE;
    const float scale = a.head->scale;
    const int left = cols - c0 - wn * 128;           // columns of this wave (GRAD)
#pragma unroll
    for (int i = 0; i < RB; ++i) {
      float lse2 = 0.f, d = 0.f;
      int c = -1;
      if constexpr (MODE == GRAD) {
        const int r = r0 + wm * 32 * RB + 32 * i + l31;
        if (r < M) {
          const int t = a.tok[r];
          lse2 = a.lse[t] * LOG2E;
          d = a.lab[r] < 0 ? __builtin_nanf("") : a.d_loss[t] / scale;
          c = a.lab[r] - (int)a.v0 - c0 - wn * 128;
        }
      }
      const auto put = [&](auto plain) __attribute__((always_inline)) {
        // plain: no label among the wave's columns and rows, all columns are in the piece, all rows have a factor
        constexpr bool PLAIN = decltype(plain)::value;
        const int end = PLAIN ? 0 : opaque(d != 0.f ? left - 4 * g : 0), hot = PLAIN ? 0 : opaque(c - 4 * g);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q) {              // registers 4 q .. 4 q + 3: columns 32 j + 8 q + 4 g + (0..3)
            float y[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              y[k] = acc[j][i][4 * q + k];
              if constexpr (MODE == GRAD) {
                const int at = 32 * j + 8 * q + k;
                y[k] = exp2_fast(fmaf(y[k], LOG2E, -lse2));
                if (!PLAIN) y[k] -= at == hot ? 1.f : 0.f;
                y[k] = PLAIN || at < end ? y[k] * d : 0.f;
              } else {
                y[k] *= scale;
              }
            }
            *(u32x2*)(tb + (32 * i + l31) * TB_PITCH + (32 * j + 8 * q + 4 * g) * 2) = u32x2{pack2_bf16(y[0], y[1]), pack2_bf16(y[2], y[3])};
          }
      };
      if (MODE == DW || (left >= 128 && !__any((c >= 0 && c < 128) || d == 0.f))) put(std::true_type{});
      else put(std::false_type{});
    }
    const int row0 = lane >> 4, ch = lane & 15;
#pragma unroll 4
    for (int it = 0; it < 8 * RB; ++it) {
      const u32x4 y = *(const u32x4*)(tb + (4 * it + row0) * TB_PITCH + ch * 16);
      const int r = r0 + wm * 32 * RB + 4 * it + row0;
      if constexpr (MODE == GRAD) {
        *(u32x4*)((char*)a.g + r * g_row_b + 2L * (c0 + wn * 128 + 8 * ch)) = y;
      } else {
        const int e = c0 + wn * 128 + 8 * ch;
        if (r < cols && e < E) *(u32x4*)((uint16_t*)a.dw + (a.v0 + r) * E + e) = y;
      }
    }
  }
}

// dx of the listed tokens: the parts' sums, 32 tokens x 32 features a workgroup; 0 for the others
__global__ void __launch_bounds__(256) xent_dx_bf16_kernel(XentArgs a, unsigned tiles) {
  const int M = a.head->count, E = a.E, tid = threadIdx.x, n_ec = (E + 31) / 32;
  if (blockIdx.x < tiles) {
    const int r = (int)(blockIdx.x / n_ec) * 32 + tid % 32, c = (int)(blockIdx.x % n_ec) * 32 + 4 * (tid / 32);
    if (r >= M || c >= E) return;
    const int n_ct = (E + T - 1) / T, rl = r % T, cl = c % T;
    const long tile = (long)(r / T) * n_ct + c / T, step = (long)((M + T - 1) / T) * n_ct * T * T;
    const int wave = (rl / 128) * 2 + cl / 128, i = rl % 128 / 32, j = cl % 128 / 32, q = cl % 32 / 8;
    const float* from = a.dx_part + tile * (T * T) + wave * (T * T / 4) + ((j * 4 + i) * 4 + q) * 256 + (rl % 32 + 32 * (cl / 4 % 2)) * 4;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < a.head->parts; ++p) s += *(const f32x4*)(from + p * step);
    s *= a.head->scale;
    *(u32x2*)((uint16_t*)a.dx + a.tok[r] * a.ldx + c) = u32x2{pack2_bf16(s[0], s[1]), pack2_bf16(s[2], s[3])};
    return;
  }
  for (long i = (long)(blockIdx.x - tiles) * 4 + (tid >> 6); i < a.n; i += (long)(gridDim.x - tiles) * 4)
    if (a.labels[i] < 0)
      for (int e = 8 * (tid & 63); e < E; e += 512) *(u32x4*)((uint16_t*)a.dx + i * a.ldx + e) = u32x4{0u, 0u, 0u, 0u};
}

// ---- float32: 128 x 128 tiles, 16 contraction steps at a time through LDS, any width ----

constexpr int FT = 128, FK = 16, FP = FT + 4;
template <int MODE>
__global__ void __launch_bounds__(256) xent_f32_kernel(XentArgs a) {
  constexpr bool LOGITS = MODE == STATS || MODE == GRAD;
  __shared__ float sa[FK][FP], sb[FK][FP];
  const int M = a.head->count, E = a.E, cols = (int)(a.v1 - a.v0);
  const int n_rt = MODE == DW ? (cols + FT - 1) / FT : (M + FT - 1) / FT;
  const int n_ct = LOGITS ? (cols + FT - 1) / FT : (E + FT - 1) / FT;
  const int parts = MODE == DX ? a.head->parts : 1;
  int rt, ct, part;
  if (!take_tile<MODE>(n_rt, n_ct, parts, &rt, &ct, &part)) return;
  const int r0 = rt * FT, c0 = ct * FT;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, l31 = lane & 31, wave = tid >> 6, wm = wave >> 1, wn = wave & 1;
  const int K = LOGITS ? E : MODE == DX ? cols : M;
  const int nk_all = (K + FK - 1) / FK;
  const int k_from = MODE == DX ? (int)((long)part * nk_all / parts) : 0;
  const int k_to = MODE == DX ? (int)((long)(part + 1) * nk_all / parts) : nk_all;
  const float *const x = (const float*)a.x, *const w = (const float*)a.w;
  float* const gg = (float*)a.g;
  // thread's elements of a tile: contraction contiguous: step tid % 16 of rows tid / 16 + 16 i; else row tid % 128 at steps tid / 128 + 2 i
  const int kc = tid % 16, kr = tid / 16, rc = tid % 128, rk = tid / 128;
  const float* brow[8];
  if (LOGITS) {
#pragma unroll
    for (int i = 0; i < 8; ++i) brow[i] = x + a.tok[min(r0 + kr + 16 * i, M - 1)] * a.ldx;
  }
  float va[8], vb[8];
  const auto fetch = [&](int kt) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (LOGITS) {
        const int k = kt * FK + kc;
        va[i] = k < E && c0 + kr + 16 * i < cols ? w[(a.v0 + c0 + kr + 16 * i) * E + k] : 0.f;
        vb[i] = k < E ? brow[i][k] : 0.f;
      } else if constexpr (MODE == DX) {
        const int k = kt * FK + rk + 2 * i, kb = kt * FK + kc;
        va[i] = k < cols && c0 + rc < E ? w[(a.v0 + k) * E + c0 + rc] : 0.f;
        vb[i] = kb < cols ? gg[(r0 + kr + 16 * i) * a.g_pitch + kb] : 0.f;
      } else {
        const int k = kt * FK + rk + 2 * i;
        va[i] = k < M && c0 + rc < E ? x[a.tok[k] * a.ldx + c0 + rc] : 0.f;
        vb[i] = k < M && r0 + rc < cols ? gg[k * a.g_pitch + r0 + rc] : 0.f;
      }
    }
  };
  f32x16 acc[2][2];
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int i = 0; i < 2; ++i) acc[j][i] = zero16();
  if (k_from < k_to) fetch(k_from);
  for (int kt = k_from; kt < k_to; ++kt) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (LOGITS) sa[kc][kr + 16 * i] = va[i];
      else sa[rk + 2 * i][rc] = va[i];
      if (MODE != DW) sb[kc][kr + 16 * i] = vb[i];
      else sb[rk + 2 * i][rc] = vb[i];
    }
    __syncthreads();
    if (kt + 1 < k_to) fetch(kt + 1);
#pragma unroll
    for (int k = 0; k < FK; k += 2) {
      float av[2], bv[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        av[j] = sa[k + g][64 * wn + 32 * j + l31];
        bv[j] = sb[k + g][64 * wm + 32 * j + l31];
      }
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i) acc[j][i] = __builtin_amdgcn_mfma_f32_32x32x2f32(av[j], bv[i], acc[j][i], 0, 0, 0);
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float scale = MODE == STATS ? 1.f : a.head->scale;
    const int r = r0 + 64 * wm + 32 * i + l31, left = cols - c0 - 64 * wn;
    if constexpr (MODE == STATS) {
      const auto z = [&](int v, int j) -> float { return acc[j][i][v]; };
      float m2, s;
      tile_stats<2>(g, left, z, &m2, &s);
      if (g == 0 && r < M) a.part[(2L * ct + wn) * a.Mp + r] = make_float2(m2, s);
      const int c = r < M ? a.lab[r] - c0 - wn * 64 : -1;
      if (c >= 0 && c < 64 && ((c >> 2) & 1) == g) a.zlab[r] = tile_pick<2>(g, c, z);
      continue;
    }
    float lse2 = 0.f, d = 0.f;
    int c = -1;
    if constexpr (MODE == GRAD) {
      if (r < M) {
        const int t = a.tok[r];
        lse2 = a.lse[t] * LOG2E;
        d = a.lab[r] < 0 ? __builtin_nanf("") : a.d_loss[t] / scale;
        c = a.lab[r] - (int)a.v0;
      }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int at = c0 + 64 * wn + 32 * j + 8 * (v / 4) + 4 * g + v % 4;
        float y = acc[j][i][v];
        if constexpr (MODE == GRAD) {
          y = exp2_fast(fmaf(y, LOG2E, -lse2)) - (at == c ? 1.f : 0.f);
          if (at < a.g_pitch) gg[r * a.g_pitch + at] = at < cols && d != 0.f ? y * d : 0.f;
        } else if constexpr (MODE == DX) {
          float* const to = a.dx_part + (((long)part * n_rt + rt) * n_ct + ct) * (FT * FT) + (r - r0) * FT + (at - c0);
          *to = a.first ? y : *to + y;
        } else {
          if (r < cols && at < E) ((float*)a.dw)[(a.v0 + r) * E + at] = y * scale;
        }
      }
  }
}
__global__ void __launch_bounds__(256) xent_dx_f32_kernel(XentArgs a, unsigned rows) {
  const int M = a.head->count, E = a.E;
  if (blockIdx.x < rows) {
    const int r = blockIdx.x;
    if (r >= M) return;
    const int n_ct = (E + FT - 1) / FT, parts = a.head->parts;
    const long step = (long)((M + FT - 1) / FT) * n_ct * (FT * FT);
    for (int e = threadIdx.x; e < E; e += 256) {
      const float* const from = a.dx_part + ((long)(r / FT) * n_ct + e / FT) * (FT * FT) + (r % FT) * FT + e % FT;
      float s = 0.f;
      for (int p = 0; p < parts; ++p) s += from[p * step];
      ((float*)a.dx)[a.tok[r] * a.ldx + e] = s * a.head->scale;
    }
    return;
  }
  for (long i = blockIdx.x - rows; i < a.n; i += gridDim.x - rows)
    if (a.labels[i] < 0)
      for (int e = threadIdx.x; e < E; e += 256) ((float*)a.dx)[i * a.ldx + e] = 0.f;
}

template <int MODE, int RB> hipError_t launch_tiles(const XentArgs& a, long grid, hipStream_t s) {
  static SmemOnce once;
  const hipError_t e = ensure_dynamic_lds((const void*)xent_bf16_kernel<MODE, RB>, SMEM_B, &once);
  if (e != hipSuccess) return e;
  xent_bf16_kernel<MODE, RB><<<(unsigned)grid, 256, SMEM_B, s>>>(a);
  return hipGetLastError();
}
long up(long n, long by) { return (n + by - 1) / by; }
template <int MODE> hipError_t logits(const XentArgs& a, int is_f32, hipStream_t s) {
  const long cols = a.v1 - a.v0;
  if (is_f32) {
    xent_f32_kernel<MODE><<<(unsigned)strip_grid(up(a.n, FT) * up(cols, FT)), 256, 0, s>>>(a);
    return hipGetLastError();
  }
  return a.n <= 128 ? launch_tiles<MODE, 2>(a, strip_grid(up(cols, T)), s) : launch_tiles<MODE, 4>(a, strip_grid(up(a.n, T) * up(cols, T)), s);
}
}  // namespace

bool xent_bf16_supported(int E) { return E % BK == 0; }
int xent_stat_parts(long V, int is_f32) { return (int)(2 * up(V, is_f32 ? FT : T)); }
// one for every tile at least, two for every compute unit where 16 parts of a tile make so many: no more with fewer tokens or features
long xent_dx_slots(long n, int E, int n_cu, int is_f32) {
  const int t = is_f32 ? FT : T;
  const long tiles = up(n, t) * up(E, t), some = 16 * tiles < 2L * n_cu ? 16 * tiles : 2L * n_cu;
  return tiles > some ? tiles : some;
}
size_t xent_dx_slot_bytes(int is_f32) { return sizeof(float) * (is_f32 ? FT * FT : T * T); }

hipError_t launch_xent_fwd(XentArgs a, int is_f32, hipStream_t s) {
  a.tile = is_f32 ? FT : T;
  xent_list_kernel<<<1, 1024, 0, s>>>(a);
  a.v0 = 0;
  a.v1 = a.V;
  const hipError_t e = logits<STATS>(a, is_f32, s);
  if (e != hipSuccess) return e;
  const long wgs = up(a.n, 8);
  xent_join_kernel<<<(unsigned)(wgs < 4096 ? wgs : 4096), 256, 0, s>>>(a, xent_stat_parts(a.V, is_f32));
  return hipGetLastError();
}

hipError_t launch_xent_bwd(XentArgs a, int is_f32, hipStream_t s) {
  const int t = is_f32 ? FT : T;
  a.tile = t;
  xent_list_kernel<<<1, 1024, 0, s>>>(a);
  a.first = 1;
  hipError_t e = hipGetLastError();
  for (a.v0 = 0; a.v0 < a.V && e == hipSuccess; a.v0 = a.v1) {
    a.v1 = a.v0 + a.piece < a.V ? a.v0 + a.piece : a.V;
    e = logits<GRAD>(a, is_f32, s);
    if (e == hipSuccess && a.dw) {
      const long grid = strip_grid(up(a.v1 - a.v0, t) * up(a.E, t));
      if (is_f32) xent_f32_kernel<DW><<<(unsigned)grid, 256, 0, s>>>(a);
      e = is_f32 ? hipGetLastError() : launch_tiles<DW, 4>(a, grid, s);
    }
    if (e == hipSuccess && a.dx) {
      const long grid = strip_grid(a.slots);
      if (is_f32) xent_f32_kernel<DX><<<(unsigned)grid, 256, 0, s>>>(a);
      e = is_f32 ? hipGetLastError() : launch_tiles<DX, 4>(a, grid, s);
      a.first = 0;
    }
  }
  if (e != hipSuccess || !a.dx) return e;
  const long zero = up(a.n, 4) < 1024 ? up(a.n, 4) : 1024;
  if (is_f32) {
    xent_dx_f32_kernel<<<(unsigned)(a.n + zero), 256, 0, s>>>(a, (unsigned)a.n);
  } else {
    const unsigned tiles = (unsigned)(up(a.n, 32) * up(a.E, 32));
    xent_dx_bf16_kernel<<<tiles + (unsigned)zero, 256, 0, s>>>(a, tiles);
  }
  return hipGetLastError();
}

}  // namespace lvx
