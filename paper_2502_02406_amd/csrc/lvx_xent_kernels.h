// Products of the losses against a vocabulary (lvx_xent.hip: softmax cross entropy, lvx_distil.hip: distillation): logits in tiles, whose epilogues leave
// what a softmax needs of them or their gradient, and the products of that gradient.
#pragma once
#include "lvx_internal.h"
#include "lvx_mfma.h"
#include "lvx_kv_ring.h"

#include <algorithm>
#include <type_traits>

namespace lvx {

namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int T = 256, BK = 64, NSLOT = 2;
constexpr int RK_ROWB = BK * 2;        // [256][64] tile: bytes of a row
constexpr int KR_ROWB = T * 2;         // [64][256] tile
constexpr int TILE_B = BK * KR_ROWB, SLOT_B = 2 * TILE_B, RING_B = NSLOT * SLOT_B;
constexpr int NW = 8;                  // waves of a workgroup
constexpr int CB = 16 / NW, WC = 32 * CB;              // a wave's column blocks, and its columns
constexpr int OUT_B = 32 * WC * 2;     // epilogue: 32 rows of a wave on their way out
constexpr int SMEM_B = RING_B + NW * OUT_B;
static_assert(SMEM_B <= 160 * 1024 && NW / 2 * T * 8 + NW * 2048 <= NW * OUT_B, "the layout fits a compute unit, and a tile's statistics and patches the way out");
enum { STATS = 0, GRAD = 1, DX = 2, DW = 3, DW_PARTS = 4 };
// What a token's logits are measured against: its label, or a teacher's logits of some entries of the vocabulary (then z is divided by a
// temperature, and the epilogues of the logits hand out those of the entries; g of these is put right by another launch, behind the epilogues).
enum { LABEL = 0, TEACHER = 1 };

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
// Entries `entry`, `entry` + `step`, .. < `end` of a list of `total` are this workgroup's: every XCD has a run of the list, and its
// workgroups take the next ones of it in turn.  The grid (a multiple of 8) may be made for more entries, or for fewer.
struct Turns { long entry, end, step; };
__device__ __forceinline__ Turns turns_of(long total) {
  const long x = blockIdx.x % 8, wg = (long)blockIdx.y * gridDim.x + blockIdx.x;
  return {total * x / 8 + wg / 8, total * (x + 1) / 8, (long)(gridDim.x / 8) * gridDim.y};
}
// The tile of an entry, and (DX, DW_PARTS) the part of its contraction.
template <int MODE> __device__ __forceinline__ void tile_of(long entry, int n_rt, int n_ct, int* rt, int* ct, int* part) {
  const long tiles = (long)n_rt * n_ct;
  *part = MODE == DX || MODE == DW_PARTS ? (int)(entry / tiles) : 0;
  if (MODE == DX || MODE == DW_PARTS) entry -= *part * tiles;
  if (MODE == STATS || MODE == GRAD) strip_tile(entry, n_ct, n_rt, ct, rt);
  else strip_tile(entry, n_rt, n_ct, rt, ct);
}
// Parts that the contraction of dx is cut into, by how many tiles the listed tokens make: as many as make the rounds of workgroups
// shortest, within the room for their sums, and four tile pairs each (300 tokens x 256 features against 50000, two tiles: 16 parts 61 us, 64
// 30).  A number a lane.
constexpr int MOST_PARTS = 64;
__device__ inline int dx_parts(int tiles, int pairs, int n_cu, int slots) {
  const int p = (threadIdx.x & 63) + 1;
  const float t = p * tiles <= slots && (4 * p <= pairs || p == 1) ? (float)((tiles * p + n_cu - 1) / n_cu) / (float)p : 1e30f;
  float least = t;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) least = fminf(least, __shfl_xor(least, o));
  return __ffsll(__ballot(t <= 1.05f * least));      // (the fewest that come within a twentieth)
}

// The same of up to 64 tokens, by every wave for itself (a.own: there is no list launch, whose 5 us a call of few tokens waits for; loss of 16 x
// 4096 against 32768 56.6 -> 53.1 us, of 2 x 640 against 2560 15.4 -> 12.3, with gradients of 58 x 384 against 5568 47 -> 39): lane i has listed
// token i (i < count) and what belongs to it.
struct Own { int count, tok, lab; float2 row; float scale; long label; };      // (label: of token `lane`)
// Entry k of a teacher's of token i: whether it is there, and its logit
struct Entry { bool there; long id; float t; };
__device__ __forceinline__ Entry entry_of(const XentArgs& a, long i, int k) {
  Entry e;
  e.id = a.ids[i * a.K + k];
  e.there = e.id >= 0;
  e.t = a.teacher_bf16 ? __uint_as_float((unsigned)((const uint16_t*)a.teacher)[i * a.K + k] << 16) : ((const float*)a.teacher)[i * a.K + k];
  return e;
}
// A logit's distance from another one by the temperature (of the difference: the type's lowest value, a mask's, by one below 1 would be -infinity)
__device__ __forceinline__ float apart(const XentArgs& a, float t, float from) { return (t - from) / a.temperature; }
// stat: of a token's entries, the largest logit and the logarithm of the sum of exponentials against it
__device__ __forceinline__ float ln_q_of(const XentArgs& a, const Entry& e, float2 stat) { return apart(a, e.t, stat.x) - stat.y; }
// Whether few tokens' entries (a.own) are looked at where they stand, by every wave and every tile, without launches that prepare them and, for the gradient,
// write them: with both passes of 10 x 256 against 1024 prepared 41.7 us, 33.8 so with one entry a token, 42.7 and 36.4 with 8; of 64 x 64 against 32768 with 8 51.1 and
// 48.8, 65536 with 4 58.7 and 52.2, with 8 59.2 and 59.8, 100000 with one 76.8 and 72.2, with 8 78.7 and 88.0, 300000 with one 165.4 and 165.2; of 32 x 64 float32 against
// 65536 with 4 92.7 and 86.2, with 8 93.1 and 97.9; the loss alone of 64 x 1024 against 32768 with 8 26.0 and 25.1, with 16 26.2 and 31.0.
constexpr int DIRECT_ENTRIES = 8;
constexpr long DIRECT_IN_ALL = 1 << 18;              // entries of a token x the vocabulary's
// Whether a token with these entries takes part: 0, -1 if not, V if an id is outside
__device__ __forceinline__ long label_of(bool any, bool far, long V) { return !any ? -1 : far ? V : 0; }
template <int LOSS = LABEL> __device__ __forceinline__ Own own_list(const XentArgs& a) {
  const int lane = threadIdx.x & 63, n = (int)a.n;
  long label = -1;
  if (LOSS == TEACHER && a.direct) {
    bool any = false, far = false;
    for (int k0 = 0; k0 < a.K; k0 += 4) {
      Entry e[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) e[k] = entry_of(a, min(lane, n - 1), min(k0 + k, a.K - 1));
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        any |= e[k].there && !(e[k].t == -__builtin_inff());
        far |= e[k].there && e[k].id >= a.V;
      }
    }
    if (lane < n) label = label_of(any, far, a.V);
  } else if (lane < n) {
    label = a.labels[lane];
  }
  const float d = a.d_loss && label >= 0 ? a.d_loss[lane] * a.inv_t : 0.f, lse = a.d_loss && label >= 0 ? a.lse[lane] : 0.f;
  const unsigned long long on = __ballot(label >= 0), below = (1ull << lane) - 1;
  Own o;
  o.label = label;
  o.count = __popcll(on);
  // (the others behind them: every lane is written)
  const int to = 4 * (label >= 0 ? __popcll(on & below) : o.count + __popcll(~on & below));
  const auto put = [&](int x) __attribute__((always_inline)) -> int { return __builtin_amdgcn_ds_permute(to, x); };
  o.tok = put(lane);
  o.lab = put(label < a.V ? (int)label : -1);
  o.row = make_float2(__int_as_float(put(__float_as_int(lse * LOG2E))), __int_as_float(put(__float_as_int(label < a.V ? d : __builtin_nanf("")))));
  float top = fabsf(d) < __builtin_inff() ? fabsf(d) : 0.f;
#pragma unroll
  for (int k = 1; k < 64; k *= 2) top = fmaxf(top, __shfl_xor(top, k));
  o.scale = top > 0.f ? top : 1.f;
  return o;
}
// ... for the launches behind: a wave of one workgroup
template <int LOSS> __device__ inline void own_publish(const XentArgs& a, const Own& o) {
  const int lane = threadIdx.x & 63;
  if (LOSS == TEACHER && a.direct && lane < a.n) ((int64_t*)a.labels)[lane] = o.label;
  const int parts = dx_parts((o.count + a.tile_rows - 1) / a.tile_rows * ((a.E + a.tile - 1) / a.tile), (int)(a.piece / BK), a.n_cu, a.slots);
  if (lane < o.count) a.tok[lane] = o.tok;
  if (lane == 0) {
    a.head->count = o.count;
    a.head->scale = o.scale;
    a.head->parts = parts;
  }
}

// ---- a wave's columns of a logits tile.  z(v, j): the logit in column 32 j + 8 (v / 4) + 4 g + v % 4 of the wave's, JB blocks of 32 ----

// log2 e, by the temperature
template <int LOSS> __device__ __forceinline__ float log2_unit(const XentArgs& a) { return LOSS == TEACHER ? a.z2 : LOG2E; }
// the largest logit (times log2 e: z2) and the sum of exponentials against it
template <int JB, bool WHOLE, class Z> __device__ __forceinline__ void tile_stats_of(int g, int cols, float z2, Z&& z, float* m2, float* s) {
  float y[JB][16];
  const int end = WHOLE ? 0 : opaque(cols - 4 * g);
#pragma unroll
  for (int j = 0; j < JB; ++j)
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      y[j][v] = z(v, j);
      if (!WHOLE) y[j][v] = 32 * j + 8 * (v / 4) + v % 4 < end ? y[j][v] : -__builtin_inff();
    }
  // (a NaN is dropped here and comes back in the sum)
  float mx = y[0][0];
#pragma unroll
  for (int j = 0; j < JB; ++j)
#pragma unroll
    for (int v = 0; v < 16; v += 2) asm("v_max3_f32 %0, %0, %1, %2" : "+v"(mx) : "v"(y[j][v]), "v"(y[j][v + 1]));
  mx = xhalf_max(mx) * z2;
  const float at = mx == -__builtin_inff() ? 0.f : mx;
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < JB; ++j)
#pragma unroll
    for (int v = 0; v < 16; ++v) sum[v % 4] += exp2_fast(fmaf(y[j][v], z2, -at));
  *m2 = mx;
  *s = xhalf_sum((sum[0] + sum[1]) + (sum[2] + sum[3]));
}
template <int JB, class Z> __device__ __forceinline__ void tile_stats(int g, int cols, float z2, Z&& z, float* m2, float* s) {
  if (cols >= 32 * JB) tile_stats_of<JB, true>(g, cols, z2, z, m2, s);      // (uniform)
  else tile_stats_of<JB, false>(g, cols, z2, z, m2, s);
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

// The sorted entries of row `row` (a listed token, or where every wave lists for itself a token) that lie in the 64 columns of the vocabulary around
// `col`: the first one's number, and above it the one's behind the last.
typedef unsigned __attribute__((aligned(2))) unsigned_any2;
__device__ __forceinline__ unsigned entries_of(const XentArgs& a, long row, int col) {
  return *(const unsigned_any2*)(a.starts + row * (a.blocks + 1) + min(col / 64, a.blocks - 1));
}
__device__ __forceinline__ int entry_id(const XentArgs& a, long row, unsigned e) { return (e & 0xffffu) < e >> 16 ? a.sorted[row * a.K + (e & 0xffffu)] : -1; }
// The logit of column c of the wave's (0 .. 32 JB - 1), chosen by its bits: right in the half of the wave that has the column
template <int JB, class Z> __device__ __forceinline__ float by_bits(int c, Z&& z) {
  const auto choose = [](int bit, float one, float zero) __attribute__((always_inline)) -> float { return bit ? one : zero; };      // (of values, not of places)
  float y[JB];
#pragma unroll
  for (int j = 0; j < JB; ++j) {
    float t[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) t[q] = choose(c & 2, choose(c & 1, z(4 * q + 3, j), z(4 * q + 2, j)), choose(c & 1, z(4 * q + 1, j), z(4 * q, j)));
    y[j] = choose(c & 16, choose(c & 8, t[3], t[2]), choose(c & 8, t[1], t[0]));
  }
  return JB == 2 ? choose(c & 32, y[JB - 1], y[0]) : y[0];
}
// Of few entries of few tokens (a.direct) all are looked at where they stand: token `row` (`on`: there is one).
template <int JB, class Z> __device__ __forceinline__ void pick_direct(const XentArgs& a, long row, bool on, int cw, int g, Z&& z) {
  for (int k0 = 0; k0 < a.K; k0 += 4) {
    long id[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) id[k] = a.ids[row * a.K + min(k0 + k, a.K - 1)];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const long at = id[k] - cw;
      const int c = on && k0 + k < a.K && at >= 0 && at < 32 * JB ? (int)at : -1;
      if (!__any(c >= 0)) continue;
      const float y = by_bits<JB>(c, z);
      if (c >= 0 && ((c >> 2) & 1) == g) a.z_entry[row * a.K + k0 + k] = y;
    }
  }
}
// ... and of the gradient: takes q off p at the entries of token `row` among 32 columns from `cw` on (KNOWN: its statistics are), where p[v] is that of column 8 (v / 4) + 4 g + v % 4.
// (In a launch of its own, as in the other cases, both passes of 10 x 256 against 1024 with one entry a token take 36.5 us, 33.8 so.)
template <bool KNOWN> __device__ __forceinline__ void subtract_direct(const XentArgs& a, long row, bool on, long cw, int g, float (&p)[16]) {
  Entry e[DIRECT_ENTRIES];
  bool any = false;
#pragma unroll
  for (int k = 0; k < DIRECT_ENTRIES; ++k) {
    e[k] = entry_of(a, row, min(k, a.K - 1));
    e[k].there &= on && k < a.K;
    any |= e[k].there && e[k].id >= cw && e[k].id < cw + 32;
  }
  if (!__any(any)) return;
  float2 stat;
  if constexpr (KNOWN) {
    stat = a.q_stat[row];
  } else {
    float top = -__builtin_inff(), sum = 0.f;
#pragma unroll
    for (int k = 0; k < DIRECT_ENTRIES; ++k) top = e[k].there ? fmaxf(top, e[k].t) : top;
#pragma unroll
    for (int k = 0; k < DIRECT_ENTRIES; ++k) sum += e[k].there ? expf(apart(a, e[k].t, top)) : 0.f;
    stat = make_float2(top, logf(sum));
  }
#pragma unroll
  for (int k = 0; k < DIRECT_ENTRIES; ++k) {
    const int hot = e[k].there && e[k].id >= cw && e[k].id < cw + 32 ? (int)(e[k].id - cw) - 4 * g : -64;
    if (!__any(hot >= -4)) continue;
    const float q = expf(ln_q_of(a, e[k], stat));
#pragma unroll
    for (int v = 0; v < 16; ++v) p[v] -= 8 * (v / 4) + v % 4 == hot ? q : 0.f;
  }
}
// Leaves the logits of those among the wave's 32 JB columns, of which `cw` is the first; z as above, id: that of the first entry, which is chosen by the bits of
// its column.  The others, where a row has more in these columns, through `patch`, 2 KB of LDS of the wave's own: 32 rows x 16 columns at a time, where both halves of the
// wave then look up four entries of a row each (2000 tokens x 256 against 1000, 128 entries: one after the other, by their bits, 40 us, 17 so).
constexpr int PATCH = 32 * 16;
template <int JB, class Z> __device__ __forceinline__ void pick_entries(const XentArgs& a, long row, unsigned e, int id, int cw, int g, float* patch, Z&& z) {
  int at = (int)(e & 0xffffu);
  const int end = (int)(e >> 16);
  {
    const int c = at < end ? id - cw : -1;
    if (__any(c >= 0 && c < 32 * JB)) {
      const float y = by_bits<JB>(c, z);
      if (c >= 0 && c < 32 * JB && ((c >> 2) & 1) == g) a.z_entry[row * a.K + at] = y;
    }
  }
  const int l31 = threadIdx.x & 31;
  for (++at; __any(at < end); at += 8) {
    typedef __attribute__((ext_vector_type(4))) int i32x4;
    typedef i32x4 __attribute__((aligned(4))) i32x4_any;
    const int mine = at + 4 * g;
    i32x4 ids = {0, 0, 0, 0};
    if (mine < end) ids = *(const i32x4_any*)(a.sorted + row * a.K + mine);      // (there is room behind the last one)
    int c[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) c[k] = mine + k < end ? ids[k] - cw : -1;
#pragma unroll
    for (int j = 0; j < JB; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const auto here = [&](int k) __attribute__((always_inline)) -> bool { return (unsigned)(c[k] - (32 * j + 16 * h)) < 16u; };
        if (!__any(here(0) || here(1) || here(2) || here(3))) continue;
        // (the patch is this wave's own: its reads are ordered after its writes, and the next writes after them)
        asm volatile("" ::: "memory");
        *(f32x4*)(patch + 16 * l31 + 4 * g) = f32x4{z(8 * h, j), z(8 * h + 1, j), z(8 * h + 2, j), z(8 * h + 3, j)};
        *(f32x4*)(patch + 16 * l31 + 8 + 4 * g) = f32x4{z(8 * h + 4, j), z(8 * h + 5, j), z(8 * h + 6, j), z(8 * h + 7, j)};
        asm volatile("" ::: "memory");
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (here(k)) a.z_entry[row * a.K + mine + k] = patch[16 * l31 + c[k] - (32 * j + 16 * h)];
        asm volatile("" ::: "memory");
      }
  }
}

__device__ __forceinline__ void join_stats(float* m, float* s, float m1, float s1) {
  const float top = fmaxf(*m, m1), at = top == -__builtin_inff() ? 0.f : top;
  *s = *s * exp2_fast(*m - at) + s1 * exp2_fast(m1 - at);
  *m = top;
}
// ---- bf16 products on the matrix cores ----

// MODE STATS, GRAD: rows = listed tokens, columns = vocabulary, contraction over the features.  Both operands have it contiguous:
//   tiles [rows][64], 128-byte lines, chunks permuted by perm_of.
// MODE DX: rows = listed tokens, columns = features, contraction over the piece's vocabulary; g like x before, w as [64][256 features]
//   with transposing reads.
// MODE DW: rows = vocabulary of the piece, columns = features, contraction over the listed tokens: both as [64 tokens][256].
// MODE DW_PARTS: the same where the tiles are few and the tokens many, the contraction cut like DX's.
// Rows of x go by the list; rows behind the last token read the last one again (their g is 0), rows of w behind the vocabulary its last
// (their columns of g are 0).
//
// A workgroup stays and takes one tile after the other (turns_of).  The first two pairs of the next one go out before the epilogue of a tile,
// which keeps out of the slots, and is over when they have come.  What the epilogue reads of the rows, and the next tile's list, is
// loaded ahead and has come before these copies start: a wait of the compiler's for it would wait for them too, which it does not
// see.  (DX, which reads its sums, starts the next tile behind them; it rarely has one.)
template <int MODE, int RB, int LOSS>
__global__ void __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(NW / 4, NW / 4)))
xent_bf16_kernel(XentArgs a) {
  constexpr bool LOGITS = MODE == STATS || MODE == GRAD, OF_W = MODE == DW || MODE == DW_PARTS, SUMS = MODE == DX || MODE == DW_PARTS;
  static_assert(RB == 4 || RB == 2, "tile heights");
  constexpr int TR = 64 * RB;                        // rows of a workgroup's tile
  constexpr int NA = 32 / NW, NB = 8 * RB / NW;      // copies per wave and tile pair: A side (columns), B side (rows)
  constexpr int NPART = NA + NB;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int M = a.head->count, E = a.E;
  const int cols = (int)(a.v1 - a.v0);               // of the piece
  const int n_rt = ((OF_W ? cols : M) + TR - 1) / TR;
  const int n_ct = LOGITS ? (cols + T - 1) / T : (E + T - 1) / T;
  const int parts = MODE == DX ? a.head->parts : MODE == DW_PARTS ? a.head->dw_parts : 1;
  const int nk_all = LOGITS ? E / BK : MODE == DX ? (cols + BK - 1) / BK : (M + BK - 1) / BK;
  struct Tile { int rt, ct, part, r0, c0, k0, nk; }; // (r0: of the list / of the piece, c0: of the piece / of the features)
  const auto tile_at = [&](long entry) __attribute__((always_inline)) -> Tile {
    Tile t;
    tile_of<MODE>(entry, n_rt, n_ct, &t.rt, &t.ct, &t.part);
    t.r0 = t.rt * TR;
    t.c0 = t.ct * T;
    t.k0 = SUMS ? (int)((long)t.part * nk_all / parts) : 0;
    t.nk = SUMS ? (int)((long)(t.part + 1) * nk_all / parts) - t.k0 : nk_all;
    return t;
  };
  Turns turn = turns_of((long)n_rt * n_ct * parts);
  if (turn.entry >= turn.end) return;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, l31 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / (NW / 2), wn = wave % (NW / 2);
  const unsigned smem_u = lds_base(smem);
  const unsigned xrow_b = (unsigned)(a.ldx * 2), wrow_b = (unsigned)(E * 2);
  const long g_row_b = a.g_pitch * 2L;

  // ---- copies into [rows][64] tiles: one instruction moves 8 rows x 128 bytes, lane l the chunk (l % 8) ^ perm_of(row) of row l / 8;
  // a wave copies rows 8 NA (NB) wave + 8 j + l / 8
  // ---- copies into [64][256] tiles: one instruction moves 2 rows x 512 bytes, lane l position l % 32 of row l / 32, which holds the
  // chunk (l % 32) ^ 4 (row % 4); a wave copies rows 2 NA wave + 2 j + l / 32.  Features past the last one: the tile's first chunk again.
  // (DW's tile of g: [64][TR], an instruction moves BR rows, lane l position l % (64 / BR) of row l / (64 / BR))
  constexpr int BR = 512 / TR, B_ROWB = TR * 2;
  const int lh = lane >> 5, pos = lane & 31, l8 = lane >> 3;
  unsigned bo[OF_W ? 1 : NB], ao[LOGITS ? NA : 1], kr_a[2], kr_b[2];
  if constexpr (MODE == DX) {
#pragma unroll
    for (int j = 0; j < NB; ++j)
      bo[j] = (unsigned)((8 * NB * wave + 8 * j + l8) * g_row_b) + 16u * (unsigned)((lane & 7) ^ perm_of(8 * j + l8));
  }
  if constexpr (OF_W) {
    const int row = lane / (64 / BR);
#pragma unroll
    for (int par = 0; par < 2; ++par)
      kr_b[par] = 16u * (unsigned)((lane % (64 / BR)) ^ (4 * ((BR * par + row) & 3))) + (unsigned)((BR * NB * wave + row) * g_row_b);
  }
  const unsigned a_lane = (unsigned)(2 * NA * wave + lh) * wrow_b;
  // DW: the rows of x that a wave copies of a pair, lane l row 2 NA wave + 2 (l % 8) + l / 32; those of the first two pairs are every tile's
  const auto x_rows = [&](int kt) __attribute__((always_inline)) -> int { return a.tok[min(kt * BK + 2 * NA * wave + 2 * (lane & 7) + lh, M - 1)]; };
  unsigned xr = 0u, xr01[2] = {0u, 0u};              // their byte offsets
  if (OF_W && M > 0) {                               // (DW_PARTS: a workgroup has one tile)
    const int k0 = MODE == DW_PARTS ? tile_at(turn.entry).k0 : 0;
    xr01[0] = (unsigned)x_rows(k0) * xrow_b;
    xr01[1] = (unsigned)x_rows(k0 + 1) * xrow_b;
  }
  // LOGITS: the tokens of a tile that a wave copies
  int tok[NB];
  const auto load_tokens = [&](const Tile& t) __attribute__((always_inline)) {
    if constexpr (LOGITS) {
#pragma unroll
      for (int j = 0; j < NB; ++j) tok[j] = a.tok[min(t.r0 + 8 * NB * wave + 8 * j + l8, M - 1)];
    }
  };
  // Where the next pair to go out starts on either side (its copies go out in order, pair by pair), and what of w is left behind its first row
  const char *ap, *bp;
  long w_left = 0;
  unsigned w_last = 0u;
  const auto point_at = [&](const Tile& t) __attribute__((always_inline)) {
    if constexpr (LOGITS) {
#pragma unroll
      for (int j = 0; j < NB; ++j) bo[j] = (unsigned)tok[j] * xrow_b + 16u * (unsigned)((lane & 7) ^ perm_of(8 * j + l8));
#pragma unroll
      for (int j = 0; j < NA; ++j)
        ao[j] = (unsigned)min((long)(8 * NA * wave + 8 * j + l8), a.V - 1 - a.v0 - t.c0) * wrow_b + 16u * (unsigned)((lane & 7) ^ perm_of(8 * j + l8));
      ap = (const char*)a.w + (a.v0 + t.c0) * wrow_b;
      bp = (const char*)a.x;
    } else {
#pragma unroll
      for (int par = 0; par < 2; ++par) {
        const int c = pos ^ (4 * ((2 * par + lh) & 3));
        kr_a[par] = t.c0 + 8 * c >= E ? 0u : 16u * (unsigned)c;
      }
      ap = MODE == DX ? (const char*)a.w + ((a.v0 + t.k0 * BK) * E + t.c0) * 2 : (const char*)a.x + 2L * t.c0;
      bp = MODE == DX ? (const char*)a.g + t.r0 * g_row_b + (long)t.k0 * RK_ROWB : (const char*)a.g + 2L * t.r0 + (long)t.k0 * BK * g_row_b;
      w_left = a.V - 1 - a.v0 - (long)t.k0 * BK;
    }
  };
  // lane j of every 16 lanes
  const auto lane_of_16 = [&](unsigned x, int j) __attribute__((always_inline)) -> unsigned {
    switch (j) {
      case 0: return row_lane<0>(x);
      case 1: return row_lane<1>(x);
      case 2: return row_lane<2>(x);
      default: return row_lane<3>(x);
    }
  };
  static_assert(NA <= 4, "lane_of_16");
  auto issue_part = [&](int kt, int p) __attribute__((always_inline)) {
    const unsigned st = smem_u + (unsigned)((kt % NSLOT) * SLOT_B);
    if (p < NA) {                                    // A side
      const int j = p;
      if constexpr (LOGITS) {
        dma16u(ap, ao[j], st + (unsigned)((8 * NA * wave + 8 * j) * RK_ROWB));
      } else if constexpr (MODE == DX) {
        if (j == 0) w_last = (unsigned)min(w_left, 63L) * wrow_b;
        dma16u(ap, min(a_lane + (unsigned)(2 * j) * wrow_b, w_last) + kr_a[j & 1], st + (unsigned)((2 * NA * wave + 2 * j) * KR_ROWB));
      } else {
        dma16u(ap, lane_of_16(xr, j) + kr_a[j & 1], st + (unsigned)((2 * NA * wave + 2 * j) * KR_ROWB));
      }
      if (j == NA - 1) {
        if (LOGITS) ap += RK_ROWB;
        if (MODE == DX) { ap += 64L * wrow_b; w_left -= 64; }
      }
    } else {                                         // B side
      const int j = p - NA;
      if constexpr (!OF_W) dma16u(bp, bo[j], st + (unsigned)(TILE_B + (8 * NB * wave + 8 * j) * RK_ROWB));
      else dma16u(bp, kr_b[j & 1] + (unsigned)(BR * j) * (unsigned)g_row_b, st + (unsigned)(TILE_B + BR * (NB * wave + j) * B_ROWB));
      if (j == NB - 1) bp += OF_W ? 64 * g_row_b : RK_ROWB;
    }
  };
  const auto start = [&](const Tile& t) __attribute__((always_inline)) {      // a tile's first two pairs
    point_at(t);
#pragma unroll
    for (int q = 0; q < NSLOT; ++q)
      if (q < t.nk) {
        if (OF_W) xr = xr01[q];
#pragma unroll
        for (int p = 0; p < NPART; ++p) issue_part(q, p);
      }
  };

  // ---- operands (see lvx_project_bwd.hip): from [rows][64] one 16-byte read; from [64][256] two transposing reads, of rows 8 g ..
  // where the other operand has its eight steps in one chunk (DX), 4 g .. and 8 + 4 g .. where both are such tiles (DW)
  const int j16 = lane & 15, jr = j16 >> 2, tr_col = 32 * ((lane >> 4) & 1) + 8 * (j16 & 3);
  constexpr int KG = MODE == DX ? 8 : 4, KH = MODE == DX ? 4 : 8;
  int rd[4], ka[CB], kb[RB];
#pragma unroll
  for (int q = 0; q < 4; ++q) rd[q] = l31 * RK_ROWB + 16 * ((2 * q + g) ^ perm_of(l31));
#pragma unroll
  for (int jj = 0; jj < CB; ++jj) ka[jj] = (KG * g + jr) * KR_ROWB + tr_col + 64 * ((CB * wn + jj) ^ jr);
#pragma unroll
  for (int jj = 0; jj < RB; ++jj) kb[jj] = TILE_B + (KG * g + jr) * B_ROWB + tr_col + 64 * ((RB * wm + jj) ^ jr);
  auto tr_op = [&](const char* p, auto pitch) __attribute__((always_inline)) -> bf16x8 {
    const s16x4 lo = lds_read_tr(p), hi = lds_read_tr(p + KH * decltype(pitch)::value);
    typedef __attribute__((ext_vector_type(8))) short s16x8;
    const s16x8 r = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    return __builtin_bit_cast(bf16x8, r);
  };
  auto a_op = [&](const char* st, int q, int j) __attribute__((always_inline)) -> bf16x8 {
    if constexpr (LOGITS) return *(const bf16x8*)(st + (wn * WC + 32 * j) * RK_ROWB + rd[q]);
    else return tr_op(st + ka[j] + 16 * q * KR_ROWB, std::integral_constant<int, KR_ROWB>{});
  };
  auto b_op = [&](const char* st, int q, int i) __attribute__((always_inline)) -> bf16x8 {
    if constexpr (!OF_W) return *(const bf16x8*)(st + TILE_B + (wm * 32 * RB + 32 * i) * RK_ROWB + rd[q]);
    else return tr_op(st + kb[i] + 16 * q * B_ROWB, std::integral_constant<int, B_ROWB>{});
  };

  f32x16 acc[CB][RB];                                // [column block j][row block i]: lane = row, registers = columns
  constexpr int NU = CB * RB;
  auto mma16 = [&](const bf16x8 (&bv)[RB], const bf16x8 (&av)[CB], auto&& hook) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < CB; ++j)
#pragma unroll
      for (int i = 0; i < RB; ++i) {
        kvring::mfma_acc(acc[j][i], av[j], bv[i]);
        hook(RB * j + i);
        __builtin_amdgcn_sched_barrier(0);
      }
  };
  constexpr int EB = NU / NB, EA = NU / NA;          // a copy of one side every so many matrix instructions of a k-step

  Tile cur = tile_at(turn.entry);
  load_tokens(cur);
  start(cur);
  char* const out = smem + RING_B + wave * OUT_B;
  const float scale = MODE == GRAD || MODE == DW ? a.head->scale : 1.f;
  for (;;) {
    turn.entry += turn.step;
    const bool again = turn.entry < turn.end;
    const Tile nxt = again ? tile_at(turn.entry) : cur;
#pragma unroll
    for (int j = 0; j < CB; ++j)
#pragma unroll
      for (int i = 0; i < RB; ++i) { acc[j][i] = zero16(); asm volatile("" : "+a"(acc[j][i])); }
    // what the epilogue needs of the rows, and the next tile's (lab: TEACHER: the rows' entries)
    int lab[LOGITS ? RB : 1];
    float2 row[MODE == GRAD ? RB : 1];
    constexpr bool PICK = MODE == STATS && LOSS == TEACHER;
    const auto load_rows = [&]() __attribute__((always_inline)) {
      if constexpr (LOGITS) {
#pragma unroll
        for (int i = 0; i < RB; ++i) {
          const int r = min(cur.r0 + wm * 32 * RB + 32 * i + l31, M - 1);
          if (LOSS == LABEL) lab[i] = a.lab[r];
          else if (MODE == STATS) lab[i] = (int)entries_of(a, opaque(r), cur.c0 + wn * WC);
          if constexpr (MODE == GRAD) row[i] = a.row[r];
        }
      }
      load_tokens(nxt);
    };
    if (cur.nk > 0) {
      const int nk = cur.nk;
      if (nk > 1) wait_vmcnt<NPART>();               // (what an epilogue has written since stands behind the copies: it is waited for as well)
      else wait_vmcnt<0>();
      wg_barrier();
      bf16x8 ba[RB], aa[CB], bb[RB], ab[CB];         // operands of even / odd k-steps
#pragma unroll
      for (int i = 0; i < RB; ++i) ba[i] = b_op(smem, 0, i);
#pragma unroll
      for (int i = 0; i < CB; ++i) aa[i] = a_op(smem, 0, i);
      auto fetch = [&](const char* st, int q, int u, bf16x8 (&bv)[RB], bf16x8 (&av)[CB]) __attribute__((always_inline)) {
        if (u < RB) bv[u] = b_op(st, q, u);
        else if (u < RB + CB) av[u - RB] = a_op(st, q, u - RB);
      };
      auto pair = [&](int P, auto steady, bool send2, bool send1, bool more) __attribute__((always_inline)) {
        constexpr bool STEADY = decltype(steady)::value;
        const char* const st = smem + (P % NSLOT) * SLOT_B;
        const char* const sn = smem + ((P + 1) % NSLOT) * SLOT_B;
        mma16(ba, aa, [&](int u) __attribute__((always_inline)) {
          fetch(st, 1, u, bb, ab);
          if ((STEADY || send2) && u % EB == EB - 1) issue_part(P + 1, NA + u / EB);
        });
        int next_rows = 0;
        if constexpr (OF_W) next_rows = x_rows(cur.k0 + P + 2);        // (has come when the wait below is over)
        mma16(bb, ab, [&](int u) __attribute__((always_inline)) { fetch(st, 2, u, ba, aa); });
        mma16(ba, aa, [&](int u) __attribute__((always_inline)) { fetch(st, 3, u, bb, ab); });
        if (STEADY || more) {
          __builtin_amdgcn_s_waitcnt(0x0070);            // vmcnt(0) and lgkmcnt(0)
          wg_barrier();
        }
        if constexpr (OF_W) xr = (unsigned)next_rows * xrow_b;
        mma16(bb, ab, [&](int u) __attribute__((always_inline)) {
          if (STEADY || more) fetch(sn, 0, u, ba, aa);
          if ((STEADY || send1) && u % EA == EA - 1) issue_part(P + 2, u / EA);
        });
      };
      load_rows();
      int P = 0;
      pair(0, std::false_type{}, false, 2 < nk, 1 < nk);
      P = 1;
      for (; P + 2 < nk; ++P) pair(P, std::true_type{}, true, true, true);
      for (; P < nk; ++P) pair(P, std::false_type{}, P + 1 < nk, false, P + 1 < nk);
    }

    // ---- epilogue: every wave has left the slots, what was loaded ahead has come, and the last matrix instructions have retired
    __builtin_amdgcn_s_waitcnt(0x0070);                  // vmcnt(0) and lgkmcnt(0)
    asm volatile("" ::: "memory");
    wg_barrier();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int j = 0; j < CB; ++j)
#pragma unroll
      for (int i = 0; i < RB; i += 2) asm volatile("s_nop 15\n\ts_nop 15" : "+a"(acc[j][i]), "+a"(acc[j][i + 1]));
    int id[PICK ? RB : 1];
    if constexpr (PICK) {                              // the rows' first entries (waited for here: behind the copies they would wait for these)
      const int left = (int)min((long)WC, a.V - cur.c0 - wn * WC);
#pragma unroll
      for (int i = 0; i < RB; ++i) {
        const int r = opaque(cur.r0 + wm * 32 * RB + 32 * i + l31);
        if (r >= M || left <= 0) lab[i] = 0;
        id[i] = entry_id(a, r, (unsigned)lab[i]);
      }
      __builtin_amdgcn_s_waitcnt(0x0070);
    }
    if (MODE != DX && again) start(nxt);
    if constexpr (MODE == STATS) {
      const int cw = cur.c0 + wn * WC, left = (int)min((long)WC, a.V - cw);      // columns of this wave
      float2* const sums = (float2*)(smem + RING_B);  // [NW / 2][TR]
#pragma unroll
      for (int i = 0; i < RB; ++i) {
        const int rl = wm * 32 * RB + 32 * i + l31, r = cur.r0 + rl;
        const auto z = [&](int v, int j) __attribute__((always_inline)) -> float { return acc[j][i][v]; };
        float m2, s;
        tile_stats<CB>(g, left, log2_unit<LOSS>(a), z, &m2, &s);
        if (g == 0) sums[wn * TR + rl] = make_float2(m2, s);
        if constexpr (LOSS == LABEL) {
          const int c = r < M ? lab[i] - cw : -1;
          if (__any(c >= 0 && c < WC)) {
            const float y = tile_pick<CB>(g, c, z);
            if (c >= 0 && c < WC && ((c >> 2) & 1) == g) a.zlab[r] = y;
          }
        }
      }
      if constexpr (PICK) {
#pragma unroll
        for (int i = 0; i < RB; ++i)
          pick_entries<CB>(a, opaque(cur.r0 + wm * 32 * RB + 32 * i + l31), (unsigned)lab[i], id[i], cw, g, (float*)(smem + RING_B + NW / 2 * TR * 8) + wave * PATCH,
                           [&](int v, int j) __attribute__((always_inline)) -> float {      // (read where it stands: all of them, ahead of the loop, spill)
                             float y;
                             asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(y) : "a"(acc[j][i][v]));
                             return y;
                           });
      }
      __builtin_amdgcn_s_waitcnt(0xc07f);              // lgkmcnt(0)
      asm volatile("" ::: "memory");
      wg_barrier();
      asm volatile("" ::: "memory");
      if (tid < TR && cur.r0 + tid < M) {              // one number for all columns of the tile
        float m = -__builtin_inff(), s = 0.f;
#pragma unroll
        for (int w = 0; w < NW / 2; ++w) join_stats(&m, &s, sums[w * TR + tid].x, sums[w * TR + tid].y);
        a.part[(long)cur.ct * a.Mp + cur.r0 + tid] = make_float2(m, s);
      }
    } else if constexpr (SUMS) {
      // in the order of the registers, 16 bytes a lane (xent_sum_bf16_kernel reads them so), on top of what the pieces before left (DX)
      const bool first = MODE == DW_PARTS || a.first;
      float* const to = (MODE == DX ? a.dx_part : a.dw_part) + (((long)cur.part * n_rt + cur.rt) * n_ct + cur.ct) * (TR * T) + wave * (TR * T / NW) + lane * 4;
#pragma unroll
      for (int j = 0; j < CB; ++j)
#pragma unroll
        for (int i0 = 0; i0 < RB; i0 += 2) {             // (eight old values on their way: more would not fit the registers)
          f32x4 old[2][4];
          if (!first) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int q = 0; q < 4; ++q) old[i][q] = *(const f32x4*)(to + ((j * RB + i0 + i) * 4 + q) * 256);
          }
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const f32x16& s = acc[j][i0 + i];
              f32x4 v = {s[4 * q], s[4 * q + 1], s[4 * q + 2], s[4 * q + 3]};
              if (!first) v += old[i][q];
              *(f32x4*)(to + ((j * RB + i0 + i) * 4 + q) * 256) = v;
            }
        }
    } else {
      // 32 rows at a time: turned around in LDS, rounded to bf16, written in whole lines.  (Chunk c of a row lies at c ^ row % 8.)
      const int left = cols - cur.c0 - wn * WC;        // columns of this wave (GRAD)
#pragma unroll
      for (int i = 0; i < RB; ++i) {
        float lse2 = 0.f, d = 0.f;
        int c = -1;
        if constexpr (MODE == GRAD) {
          if (cur.r0 + wm * 32 * RB + 32 * i + l31 < M) {
            lse2 = row[i].x;
            d = row[i].y / scale;
            if (LOSS == LABEL) c = lab[i] - (int)a.v0 - cur.c0 - wn * WC;
          }
        }
        const auto put = [&](auto plain) __attribute__((always_inline)) {
          // plain: no label among the wave's columns and rows, all columns are in the piece, all rows have a factor
          constexpr bool PLAIN = decltype(plain)::value;
          const int end = PLAIN ? 0 : opaque(d != 0.f ? left - 4 * g : 0), hot = PLAIN ? 0 : opaque(c - 4 * g);
#pragma unroll
          for (int j = 0; j < CB; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {              // registers 4 q .. 4 q + 3: columns 32 j + 8 q + 4 g + (0..3)
              float y[4];
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                y[k] = acc[j][i][4 * q + k];
                if constexpr (MODE == GRAD) {
                  const int at = 32 * j + 8 * q + k;
                  y[k] = exp2_fast(fmaf(y[k], log2_unit<LOSS>(a), -lse2));
                  if (!PLAIN && LOSS == LABEL) y[k] -= at == hot ? 1.f : 0.f;
                  y[k] = PLAIN || at < end ? y[k] * d : 0.f;
                } else {
                  y[k] *= scale;
                }
              }
              *(u32x2*)(out + l31 * (2 * WC) + ((4 * j + q) ^ (l31 & 7)) * 16 + 8 * g) = u32x2{pack2_bf16(y[0], y[1]), pack2_bf16(y[2], y[3])};
            }
        };
        if (MODE == DW || (left >= WC && !__any((c >= 0 && c < WC) || d == 0.f))) put(std::true_type{});
        else put(std::false_type{});
        // (the buffer is this wave's own: its reads are ordered after its writes, and the next writes after them)
#pragma unroll
        for (int it = 0; it < 4; ++it) {
          const int rl = 8 * it + l8, ch = lane & 7, r = cur.r0 + wm * 32 * RB + 32 * i + rl, e = cur.c0 + wn * WC + 8 * ch;
          const u32x4 y = *(const u32x4*)(out + rl * (2 * WC) + (ch ^ (rl & 7)) * 16);
          if constexpr (MODE == GRAD) {
            *(u32x4*)((char*)a.g + r * g_row_b + 2L * e) = y;
          } else {
            if (r < cols && e < E) *(u32x4*)((uint16_t*)a.dw + (a.v0 + r) * E + e) = y;
          }
        }
      }
    }
    if (!again) break;
    if (MODE == DX) start(nxt);
    cur = nxt;
  }
}

// Logits of few tokens (few_rows): bound by reading w.  A workgroup takes 128 entries of the vocabulary, a wave 32 of them against 32 RB tokens, and
// NS slots of 64 features are on their way (of w alone, 16 KB each; two-slot tiles of 256 entries kept half of the compute units
// waiting, 16 tokens x 4096 against 32768: 85 -> 66 us).  Six slots (64 tokens) where the workgroups have a compute unit each, three where two share
// one.  Behind the last features the copies go on with these again, so that every step waits for the same number.
template <int MODE, int RB, int NS, bool OWN, int LOSS>
__global__ void __launch_bounds__(256) xent_few_bf16_kernel(XentArgs a) {
  constexpr int CT = 128, A_B = CT * RK_ROWB, B_B = 32 * RB * RK_ROWB, S_B = A_B + B_B, NP = 4 + RB;
  constexpr int W_PITCH = 32 * 2 + 16, W_B = 32 * RB * W_PITCH;      // GRAD: a wave's rows on their way out
  static_assert(4 * W_B <= NS * S_B, "they fit the slots");
  extern __shared__ __attribute__((aligned(16))) char smem[];
  Own own;
  if constexpr (OWN) {
    own = own_list<LOSS>(a);
    if (MODE == GRAD && blockIdx.x == 0 && threadIdx.x < 64) own_publish<LOSS>(a, own);
  }
  const int M = OWN ? own.count : a.head->count, E = a.E, cols = (int)(a.v1 - a.v0), nk = E / BK;
  const int n_rt = (M + 32 * RB - 1) / (32 * RB), n_ct = (cols + CT - 1) / CT;
  const Turns turn = turns_of((long)n_rt * n_ct);
  if (turn.entry >= turn.end) return;
  const int ct = (int)(turn.entry / n_rt), c0 = ct * CT, r0 = (int)(turn.entry % n_rt) * 32 * RB;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, l31 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const unsigned xrow_b = (unsigned)(a.ldx * 2), wrow_b = (unsigned)(E * 2);
  const unsigned smem_u = lds_base(smem);
  unsigned ao[4], bo[RB];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int r = 32 * wave + 8 * j + (lane >> 3);
    ao[j] = (unsigned)min((long)r, a.V - 1 - a.v0 - c0) * wrow_b + 16u * (unsigned)((lane & 7) ^ perm_of(8 * j + (lane >> 3)));
  }
#pragma unroll
  for (int j = 0; j < RB; ++j) {
    const int r = 8 * RB * wave + 8 * j + (lane >> 3);
    bo[j] = (unsigned)(OWN ? __shfl(own.tok, min(r, M - 1)) : a.tok[min(r0 + r, M - 1)]) * xrow_b + 16u * (unsigned)((lane & 7) ^ perm_of(r));
  }
  const char* const wg = (const char*)a.w + (a.v0 + c0) * wrow_b;
  // (every workgroup begins at another feature: at the same one, the lines that all of them ask for lie 2 E bytes apart, in few of the memory's
  // channels; 16 x 4096 against 32768 69 -> 53 us, against 131072 217 -> 186, 5.8 TB/s)
  const int from = (int)(ct * 7u % (unsigned)nk);
  const auto issue = [&](int kt, int slot) __attribute__((always_inline)) {
    const int k = min(kt, nk - 1) + from;
    const long k_b = (long)(k < nk ? k : k - nk) * RK_ROWB;
    const unsigned st = smem_u + (unsigned)(slot * S_B);
#pragma unroll
    for (int j = 0; j < 4; ++j) dma16u(wg + k_b, ao[j], st + (unsigned)((32 * wave + 8 * j) * RK_ROWB));
#pragma unroll
    for (int j = 0; j < RB; ++j) dma16u((const char*)a.x + k_b, bo[j], st + (unsigned)(A_B + (8 * RB * wave + 8 * j) * RK_ROWB));
  };
  f32x16 acc[RB];
#pragma unroll
  for (int i = 0; i < RB; ++i) acc[i] = zero16();
  constexpr bool PICK = MODE == STATS && LOSS == TEACHER;
  int row_e[PICK ? RB : 1];                          // the rows' places among the entries, and those (loaded in front of the copies, which then need not be waited for)
  unsigned en[PICK ? RB : 1];
  if constexpr (PICK) {
#pragma unroll
    for (int i = 0; i < RB; ++i) {
      const int r = 32 * i + l31;
      row_e[i] = OWN ? __shfl(own.tok, min(r, M - 1)) : min(r0 + r, M - 1);
      en[i] = 0u;
      if (!a.direct && r0 + r < M && c0 + 32 * wave < cols) en[i] = entries_of(a, row_e[i], c0 + 32 * wave);
    }
  }
#pragma unroll
  for (int s = 0; s < NS - 1; ++s) issue(s, s);
  int slot = 0, free = NS - 1;
  for (int kt = 0; kt < nk; ++kt) {
    // This step's copies have landed and the reads of the step before have returned; behind the barrier everybody's have, and that step's
    // slot is the next to be filled.
    wait_vmcnt<NP * (NS - 2)>();
    __builtin_amdgcn_s_waitcnt(0xc07f);              // lgkmcnt(0)
    asm volatile("" ::: "memory");
    wg_barrier();
    asm volatile("" ::: "memory");
    issue(kt + NS - 1, free);
    const char* const st = smem + slot * S_B;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int rd = l31 * RK_ROWB + 16 * ((2 * q + g) ^ perm_of(l31));
      const bf16x8 av = *(const bf16x8*)(st + 32 * wave * RK_ROWB + rd);
#pragma unroll
      for (int i = 0; i < RB; ++i) acc[i] = mfma32(av, *(const bf16x8*)(st + A_B + 32 * i * RK_ROWB + rd), acc[i]);
    }
    asm volatile("" ::: "memory");
    free = slot;
    slot = slot + 1 == NS ? 0 : slot + 1;
  }
  wait_vmcnt<0>();
  asm volatile("" ::: "memory");
  wg_barrier();                                      // (the slots are free, and nothing more lands in them)
  asm volatile("" ::: "memory");
  const int cw = 32 * wave, left = cols - c0 - cw;
  if constexpr (MODE == STATS) {
    float2* const sums = (float2*)smem;              // [4][32 RB]
    int id[PICK ? RB : 1];
    if constexpr (PICK) {
#pragma unroll
      for (int i = 0; i < RB; ++i) id[i] = entry_id(a, row_e[i], en[i]);
    }
#pragma unroll
    for (int i = 0; i < RB; ++i) {
      const int r = 32 * i + l31;
      const auto z = [&](int v, int) __attribute__((always_inline)) -> float { return acc[i][v]; };
      float m2, s;
      tile_stats<1>(g, left, log2_unit<LOSS>(a), z, &m2, &s);
      if (g == 0) sums[wave * 32 * RB + r] = make_float2(m2, s);
      if constexpr (LOSS == TEACHER) {
        if (a.direct) pick_direct<1>(a, OWN ? row_e[i] : a.tok[row_e[i]], r0 + r < M, c0 + cw, g, z);
        else pick_entries<1>(a, row_e[i], en[i], id[i], c0 + cw, g, (float*)(smem + 4 * 32 * RB * 8) + wave * PATCH, z);
      } else {
        const int label = OWN ? __shfl(own.lab, r) : r0 + r < M ? a.lab[r0 + r] : -1;
        const int c = r0 + r < M ? label - c0 - cw : -1;
        const float y = tile_pick<1>(g, c, z);
        if (c >= 0 && c < 32 && ((c >> 2) & 1) == g) a.zlab[r0 + r] = y;
      }
    }
    __syncthreads();
    if (tid < 32 * RB && r0 + tid < M) {
      float m = -__builtin_inff(), s = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) join_stats(&m, &s, sums[w * 32 * RB + tid].x, sums[w * 32 * RB + tid].y);
      a.part[(long)ct * a.Mp + r0 + tid] = make_float2(m, s);
    }
  } else {
    const float scale = OWN ? own.scale : a.head->scale;
    char* const tb = smem + wave * W_B;
#pragma unroll
    for (int i = 0; i < RB; ++i) {
      const int r = 32 * i + l31;
      float lse2 = 0.f, d = 0.f;
      int c = -1;
      if constexpr (OWN) {
        const int label = __shfl(own.lab, r);
        const float x = __shfl(own.row.x, r), y = __shfl(own.row.y, r);
        if (r < M) {
          lse2 = x;
          d = y / scale;
          if (LOSS == LABEL) c = label - (int)a.v0 - c0 - cw;
        }
      } else if (r0 + r < M) {
        lse2 = a.row[r0 + r].x;
        d = a.row[r0 + r].y / scale;
        if (LOSS == LABEL) c = a.lab[r0 + r] - (int)a.v0 - c0 - cw;
      }
      const int end = d != 0.f ? left - 4 * g : 0, hot = c - 4 * g;
      float p[16];
#pragma unroll
      for (int v = 0; v < 16; ++v) p[v] = exp2_fast(fmaf(acc[i][v], log2_unit<LOSS>(a), -lse2));
      if constexpr (LOSS == TEACHER) {
        if (a.direct) subtract_direct<!OWN>(a, OWN ? __shfl(own.tok, min(r, M - 1)) : a.tok[min(r0 + r, M - 1)], r0 + r < M, a.v0 + c0 + cw, g, p);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int at = 8 * q + k;
          y[k] = p[4 * q + k];
          if (LOSS == LABEL) y[k] -= at == hot ? 1.f : 0.f;
          y[k] = at < end ? y[k] * d : 0.f;
        }
        *(u32x2*)(tb + r * W_PITCH + (8 * q + 4 * g) * 2) = u32x2{pack2_bf16(y[0], y[1]), pack2_bf16(y[2], y[3])};
      }
    }
    // (the buffer is this wave's own)
#pragma unroll
    for (int it = 0; it < 2 * RB; ++it) {
      const int r = 16 * it + (lane >> 2), ch = lane & 3;
      const u32x4 y = *(const u32x4*)(tb + r * W_PITCH + 16 * ch);
      *(u32x4*)((char*)a.g + (long)(r0 + r) * a.g_pitch * 2 + 2L * (c0 + cw + 8 * ch)) = y;
    }
  }
}

// dx of up to 64 tokens, bound by reading w as well: 128 features and a part of the vocabulary a workgroup, a wave 32 of them against 32 RB tokens,
// NS slots of 64 entries (16 KB of w) on their way.  The parts' sums go out as rows of floats, [part][64][E rounded up to 128].  2 tokens x 640
// against 2560 7.8 -> 4.5 us, 1 x 1664 against 16384 17 -> 11, 64 x 256 against 65536 20 -> 12.5, 16 x 3520 against 131072 230 -> 200 (4.6 TB/s, while
// dw of the launch before is still on its way to memory; 16 x 4096 against 32768 85 in either form).
template <int RB, int NS>
__global__ void __launch_bounds__(256) xent_few_dx_bf16_kernel(XentArgs a) {
  constexpr int CT = 128, PITCH = CT * 2, A_B = BK * PITCH, B_B = 32 * RB * RK_ROWB, S_B = A_B + B_B, NP = 4 + RB;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int M = a.head->count, E = a.E, cols = (int)(a.v1 - a.v0), n_ct = (E + CT - 1) / CT, nk_all = (cols + BK - 1) / BK, parts = a.head->parts;
  const Turns turn = turns_of((long)n_ct * parts);
  if (turn.entry >= turn.end || M == 0) return;
  const int ct = (int)(turn.entry % n_ct), part = (int)(turn.entry / n_ct), e0 = ct * CT;
  const int k0 = (int)((long)part * nk_all / parts), nk = (int)((long)(part + 1) * nk_all / parts) - k0;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, l31 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const unsigned wrow_b = (unsigned)(E * 2), g_row_b = (unsigned)(a.g_pitch * 2);
  const unsigned smem_u = lds_base(smem);
  // copies of w: 4 rows x 256 bytes an instruction, lane l position l % 16 of row l / 16, which holds the chunk (l % 16) ^ 4 (row % 4); features past
  // the last one: the tile's first chunk again
  const int chunk = (lane & 15) ^ (4 * (lane >> 4));
  const unsigned a_chunk = e0 + 8 * chunk >= E ? 0u : 16u * (unsigned)chunk;
  unsigned bo[RB];
#pragma unroll
  for (int j = 0; j < RB; ++j) {
    const int r = 8 * RB * wave + 8 * j + (lane >> 3);
    bo[j] = (unsigned)r * g_row_b + 16u * (unsigned)((lane & 7) ^ perm_of(r));
  }
  const auto issue = [&](int kt, int slot) __attribute__((always_inline)) {
    const int k = k0 + min(kt, nk - 1);              // (behind the last pair that one again, so that every step waits for the same number)
    const unsigned st = smem_u + (unsigned)(slot * S_B);
    const int last = (int)min(63L, a.V - 1 - a.v0 - (long)k * BK);
    const char* const ap = (const char*)a.w + ((a.v0 + (long)k * BK) * E + e0) * 2;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      dma16u(ap, (unsigned)min(16 * wave + 4 * j + (lane >> 4), last) * wrow_b + a_chunk, st + (unsigned)((16 * wave + 4 * j) * PITCH));
#pragma unroll
    for (int j = 0; j < RB; ++j) dma16u((const char*)a.g + (long)k * RK_ROWB, bo[j], st + (unsigned)(A_B + (8 * RB * wave + 8 * j) * RK_ROWB));
  };
  f32x16 acc[RB];
#pragma unroll
  for (int i = 0; i < RB; ++i) acc[i] = zero16();
  const int j16 = lane & 15, jr = j16 >> 2, ka = (8 * g + jr) * PITCH + 32 * ((lane >> 4) & 1) + 8 * (j16 & 3) + 64 * (wave ^ jr);
  if (nk > 0) {                                      // (a short last piece leaves parts without a pair)
#pragma unroll
    for (int s = 0; s < NS - 1; ++s) issue(s, s);
  }
  int slot = 0, free = NS - 1;
  for (int kt = 0; kt < nk; ++kt) {                  // (as in xent_few_bf16_kernel)
    wait_vmcnt<NP * (NS - 2)>();
    __builtin_amdgcn_s_waitcnt(0xc07f);              // lgkmcnt(0)
    asm volatile("" ::: "memory");
    wg_barrier();
    asm volatile("" ::: "memory");
    issue(kt + NS - 1, free);
    const char* const st = smem + slot * S_B;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const char* const p = st + ka + 16 * q * PITCH;
      const s16x4 lo = lds_read_tr(p), hi = lds_read_tr(p + 4 * PITCH);
      typedef __attribute__((ext_vector_type(8))) short s16x8;
      const bf16x8 av = __builtin_bit_cast(bf16x8, s16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
      const int rd = l31 * RK_ROWB + 16 * ((2 * q + g) ^ perm_of(l31));
#pragma unroll
      for (int i = 0; i < RB; ++i) acc[i] = mfma32(av, *(const bf16x8*)(st + A_B + 32 * i * RK_ROWB + rd), acc[i]);
    }
    asm volatile("" ::: "memory");
    free = slot;
    slot = slot + 1 == NS ? 0 : slot + 1;
  }
  wait_vmcnt<0>();
  asm volatile("" ::: "memory");
  const long pitch = (long)n_ct * CT;
#pragma unroll
  for (int i = 0; i < RB; ++i) {
    const int r = 32 * i + l31;
    if (r < M) {
      float* const to = a.dx_part + ((long)part * 64 + r) * pitch + e0 + 32 * wave + 4 * g;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        f32x4 y = {acc[i][4 * q], acc[i][4 * q + 1], acc[i][4 * q + 2], acc[i][4 * q + 3]};
        if (!a.first) y += *(const f32x4*)(to + 8 * q);
        *(f32x4*)(to + 8 * q) = y;
      }
    }
  }
}

// ---- float32: FT x FT tiles (128, or 64 where these are too few), 32 contraction steps at a time through LDS, any width ----
//
// v_mfma_f32_32x32x2_f32 takes two steps at a time, one from each half of the wave.  The lower half takes steps 0 .. 15 of a tile, the
// upper one 16 .. 31, so that of an operand which has the contraction contiguous (LDS [row][32 + 4]) a lane reads four steps at once.
// Operands that have it along their rows lie as [step][FT].  A wave makes FT / 2 x FT / 2.
constexpr int FK = 32, FPK = FK + 4;
typedef f32x4 __attribute__((aligned(4))) f32x4_any;
__device__ __forceinline__ f32x4 load4(const float* p, int there) {      // four floats, of which `there` exist (0 for the others)
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (there >= 4) {
    v = *(const f32x4_any*)p;
  } else {
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (k < there) v[k] = p[k];
  }
  return v;
}
template <int MODE, int FT, int LOSS>
__global__ void __launch_bounds__(256) xent_f32_kernel(XentArgs a) {
  constexpr bool LOGITS = MODE == STATS || MODE == GRAD, OF_W = MODE == DW || MODE == DW_PARTS, SUMS = MODE == DX || MODE == DW_PARTS;
  constexpr bool AK = LOGITS, BK_ = !OF_W;      // whether the operand has the contraction contiguous
  constexpr int NB = FT / 64, NL = FT * FK / 1024;   // 32-blocks of a wave per side; 16-byte loads of a thread per side
  __shared__ __attribute__((aligned(16))) float sa[FT * FPK], sb[FT * FPK];
  const int M = a.head->count, E = a.E, cols = (int)(a.v1 - a.v0);
  const int n_rt = OF_W ? (cols + FT - 1) / FT : (M + FT - 1) / FT;
  const int n_ct = LOGITS ? (cols + FT - 1) / FT : (E + FT - 1) / FT;
  const int parts = MODE == DX ? a.head->parts : MODE == DW_PARTS ? a.head->dw_parts : 1;
  const Turns turn = turns_of((long)n_rt * n_ct * parts);      // (one tile a workgroup: a loop over them costs dw a fifth, in registers)
  if (turn.entry >= turn.end) return;
  int rt, ct, part;
  tile_of<MODE>(turn.entry, n_rt, n_ct, &rt, &ct, &part);
  const int r0 = rt * FT, c0 = ct * FT;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, l31 = lane & 31, wave = tid >> 6, wm = wave >> 1, wn = wave & 1;
  const int K = LOGITS ? E : MODE == DX ? cols : M;
  const int nk_all = (K + FK - 1) / FK;
  const int k_from = SUMS ? (int)((long)part * nk_all / parts) : 0;
  const int k_to = SUMS ? (int)((long)(part + 1) * nk_all / parts) : nk_all;
  const float *const x = (const float*)a.x, *const w = (const float*)a.w;
  float* const gg = (float*)a.g;
  // load i of a thread: contraction contiguous: steps 4 (u % 8) .. of row u / 8; else four columns 4 (u % (FT / 4)) .. of step u / (FT / 4),
  // u = tid + 256 i
  // Steps that are whole, of tiles whose chunks of four columns exist or do not: nothing to ask, and AHEAD of them on their way (700 tokens x
  // 200 against 3000: dw 32.5 -> 23 us; 3000 x 512 against 40000: dw 1160 -> 1050, dx 1125 -> 1070, logits 1100 -> 1060).  Rows and columns
  // past the last one read another one: what becomes of them is not looked at.
  constexpr int AHEAD = FT == 64 ? 3 : 1;
  const int k_whole = LOGITS || E % 4 == 0 || c0 + FT <= E ? max(k_from, min(k_to, K / FK)) : k_from;
  int tok[OF_W ? AHEAD : 1][NL];               // LOGITS: of every step; DW: of the next AHEAD steps to be fetched
  const auto tokens = [&](int kt, int (&t)[NL]) {
#pragma unroll
    for (int i = 0; i < NL; ++i) t[i] = a.tok[min(LOGITS ? r0 + (tid + 256 * i) / 8 : kt * FK + (tid + 256 * i) / (FT / 4), M - 1)];
  };
  if constexpr (LOGITS) tokens(0, tok[0]);
  const auto fetch_whole = [&](int kt_, f32x4 (&va)[NL], f32x4 (&vb)[NL], int (&tok)[NL]) {
    const int kt = min(kt_, k_whole - 1);
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int u = tid + 256 * i;
      const int row = u / 8, kc = kt * FK + 4 * (u % 8), kr = kt * FK + u / (FT / 4), col = 4 * (u % (FT / 4));
      if constexpr (LOGITS) {
        va[i] = *(const f32x4_any*)(w + (a.v0 + min(c0 + row, cols - 1)) * E + kc);
        vb[i] = *(const f32x4_any*)(x + tok[i] * a.ldx + kc);
      } else {
        const int e = c0 + col + 4 <= E ? c0 + col : c0;
        if constexpr (MODE == DX) {
          va[i] = *(const f32x4_any*)(w + (a.v0 + kr) * E + e);
          vb[i] = *(const f32x4*)(gg + (r0 + row) * a.g_pitch + kc);
        } else {
          va[i] = *(const f32x4_any*)(x + tok[i] * a.ldx + e);
          vb[i] = *(const f32x4*)(gg + kr * a.g_pitch + r0 + col);
        }
      }
    }
    if constexpr (OF_W) tokens(kt_ + AHEAD, tok);
  };
  const auto fetch = [&](int kt, f32x4 (&va)[NL], f32x4 (&vb)[NL]) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int u = tid + 256 * i;
      const int row = u / 8, kc = kt * FK + 4 * (u % 8), kr = kt * FK + u / (FT / 4), col = 4 * (u % (FT / 4));
      if constexpr (LOGITS) {
        va[i] = load4(w + (a.v0 + c0 + row) * E + kc, c0 + row < cols ? E - kc : 0);
        vb[i] = load4(x + tok[0][i] * a.ldx + kc, E - kc);
      } else if constexpr (MODE == DX) {
        va[i] = load4(w + (a.v0 + kr) * E + c0 + col, kr < cols ? E - c0 - col : 0);
        vb[i] = load4(gg + (r0 + row) * a.g_pitch + kc, cols - kc);
      } else {
        va[i] = load4(x + (kr < M ? a.tok[kr] * a.ldx : 0) + c0 + col, kr < M ? E - c0 - col : 0);
        vb[i] = load4(gg + kr * a.g_pitch + r0 + col, kr < M ? cols - r0 - col : 0);
      }
    }
  };
  f32x16 acc[NB][NB];
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int i = 0; i < NB; ++i) acc[j][i] = zero16();
  const auto put = [&](const f32x4 (&va)[NL], const f32x4 (&vb)[NL]) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int u = tid + 256 * i, at_k = (u / 8) * FPK + 4 * (u % 8), at_r = (u / (FT / 4)) * FT + 4 * (u % (FT / 4));
      *(f32x4*)(sa + (AK ? at_k : at_r)) = va[i];
      *(f32x4*)(sb + (BK_ ? at_k : at_r)) = vb[i];
    }
  };
  const auto multiply = [&]() {
#pragma unroll
    for (int s = 0; s < FK / 2; s += 4) {
      f32x4 av[NB], bv[NB];
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const int ra = FT / 2 * wn + 32 * j + l31, rb = FT / 2 * wm + 32 * j + l31;
        if constexpr (AK) {
          av[j] = *(const f32x4*)(sa + ra * FPK + FK / 2 * g + s);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) av[j][k] = sa[(FK / 2 * g + s + k) * FT + ra];
        }
        if constexpr (BK_) {
          bv[j] = *(const f32x4*)(sb + rb * FPK + FK / 2 * g + s);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) bv[j][k] = sb[(FK / 2 * g + s + k) * FT + rb];
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
          for (int i = 0; i < NB; ++i) acc[j][i] = __builtin_amdgcn_mfma_f32_32x32x2f32(av[j][k], bv[i][k], acc[j][i], 0, 0, 0);
    }
    __syncthreads();
  };
  f32x4 va[AHEAD][NL], vb[AHEAD][NL];
  const auto whole_steps = [&]() {
#pragma unroll
    for (int d = 0; d < AHEAD; ++d) {
      if constexpr (OF_W) tokens(k_from + d, tok[d]);
      fetch_whole(k_from + d, va[d], vb[d], tok[OF_W ? d : 0]);
    }
    for (int kt = k_from;;) {
#pragma unroll
      for (int d = 0; d < AHEAD; ++d) {
        put(va[d], vb[d]);
        fetch_whole(kt + AHEAD, va[d], vb[d], tok[OF_W ? d : 0]);
        __syncthreads();
        multiply();
        if (++kt == k_whole) return;
      }
    }
  };
  if (k_from < k_whole) whole_steps();
  for (int kt = k_whole; kt < k_to; ++kt) {
    fetch(kt, va[0], vb[0]);
    put(va[0], vb[0]);
    __syncthreads();
    multiply();
  }
  const float scale = MODE == STATS ? 1.f : a.head->scale;
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    const int r = r0 + FT / 2 * wm + 32 * i + l31, cw = c0 + FT / 2 * wn, left = cols - cw;
    if constexpr (MODE == STATS) {
      const auto z = [&](int v, int j) -> float { return acc[j][i][v]; };
      float m2, s;
      tile_stats<NB>(g, left, log2_unit<LOSS>(a), z, &m2, &s);
      if (g == 0 && r < M) a.part[(2L * ct + wn) * a.Mp + r] = make_float2(m2, s);
      if constexpr (LOSS == TEACHER) {
        const int row = min(r, M - 1);
        if (a.direct) {
          pick_direct<NB>(a, a.tok[row], r < M, cw, g, z);
        } else {
          const unsigned e = r < M && left > 0 ? entries_of(a, row, cw) : 0u;
          pick_entries<NB>(a, row, e, entry_id(a, row, e), cw, g, sa + wave * PATCH, z);
        }
      } else {
        const int c = r < M ? a.lab[r] - cw : -1;
        if (__any(c >= 0 && c < FT / 2)) {
          const float y = tile_pick<NB>(g, c, z);
          if (c >= 0 && c < FT / 2 && ((c >> 2) & 1) == g) a.zlab[r] = y;
        }
      }
    } else {
      float lse2 = 0.f, d = 0.f;
      int c = -1;
      if constexpr (MODE == GRAD) {
        if (r < M) {
          lse2 = a.row[r].x;
          d = a.row[r].y / scale;
          if (LOSS == LABEL) c = a.lab[r] - (int)a.v0;
        }
      }
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        float p[MODE == GRAD ? 16 : 1];
        if constexpr (MODE == GRAD) {
#pragma unroll
          for (int v = 0; v < 16; ++v) p[v] = exp2_fast(fmaf(acc[j][i][v], log2_unit<LOSS>(a), -lse2));
          if constexpr (LOSS == TEACHER) {
            if (a.direct) subtract_direct<true>(a, a.tok[min(r, M - 1)], r < M, a.v0 + cw + 32 * j, g, p);
          }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int at = cw + 32 * j + 8 * q + 4 * g;          // four columns from here
          f32x4 y = {acc[j][i][4 * q], acc[j][i][4 * q + 1], acc[j][i][4 * q + 2], acc[j][i][4 * q + 3]};
          if constexpr (MODE == GRAD) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float of_it = p[4 * q + k] - (LOSS == LABEL && at + k == c ? 1.f : 0.f);
              y[k] = at + k < cols && d != 0.f ? of_it * d : 0.f;
            }
            *(f32x4*)(gg + r * a.g_pitch + at) = y;            // (a row of g has room for whole tiles)
          } else if constexpr (SUMS) {
            float* const to = (MODE == DX ? a.dx_part : a.dw_part) + (((long)part * n_rt + rt) * n_ct + ct) * (FT * FT) + (r - r0) * FT + (at - c0);
            if (MODE == DX && !a.first) y += *(const f32x4*)to;
            *(f32x4*)to = y;
          } else if (r < cols) {
            float* const to = (float*)a.dw + (a.v0 + r) * E + at;
            y *= scale;
            if (at + 4 <= E) *(f32x4_any*)to = y;
            else
              for (int k = 0; k < 3; ++k)
                if (at + k < E) to[k] = y[k];
          }
        }
      }
    }
  }
}
// Logits of few tokens (f32_few): 32 x 32 tiles, the features dealt out to the four waves, 32 at a time, which bring their operands straight
// into registers: a lane has 64 bytes of a row of w and of x.
template <int MODE, int LOSS> __global__ void __launch_bounds__(256) xent_few_f32_kernel(XentArgs a) {
  __shared__ __attribute__((aligned(16))) float sums[3][4][256];
  const Own own = own_list<LOSS>(a);
  if (MODE == GRAD && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x < 64) own_publish<LOSS>(a, own);
  const int M = own.count, E = a.E, cols = (int)(a.v1 - a.v0);
  const Turns turn = turns_of((cols + 31) / 32);
  if (turn.entry >= turn.end || M == 0) return;
  const int ct = (int)turn.entry, c0 = ct * 32;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, l31 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const float* const w = (const float*)a.w + (a.v0 + min(c0 + l31, cols - 1)) * E + 16 * g;
  const float* const x = (const float*)a.x + __shfl(own.tok, min(l31, M - 1)) * a.ldx + 16 * g;
  f32x16 acc = zero16();
  const auto multiply = [&](const f32x4 (&av)[4], const f32x4 (&bv)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int k = 0; k < 4; ++k) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(av[j][k], bv[j][k], acc, 0, 0, 0);
  };
  const int whole = E / 32;                          // step s: features 32 s ..; the wave's are wave, wave + 4, ..
  f32x4 av[2][4], bv[2][4];
  const auto fetch = [&](int s, int d) {
    const int at = 32 * min(s, whole - 1);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      av[d][j] = *(const f32x4_any*)(w + at + 4 * j);
      bv[d][j] = *(const f32x4_any*)(x + at + 4 * j);
    }
  };
  if (wave < whole) {
    fetch(wave, 0);
    for (int s = wave; s < whole; s += 8) {
      fetch(s + 4, 1);
      multiply(av[0], bv[0]);
      if (s + 4 >= whole) break;
      fetch(s + 8, 0);
      multiply(av[1], bv[1]);
    }
  }
  if (E % 32 != 0 && wave == whole % 4) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int left = E - 32 * whole - 16 * g - 4 * j;
      av[0][j] = load4(w + 32 * whole + 4 * j, left);
      bv[0][j] = load4(x + 32 * whole + 4 * j, left);
    }
    multiply(av[0], bv[0]);
  }
  if (wave > 0) {
#pragma unroll
    for (int q = 0; q < 4; ++q) *(f32x4*)(&sums[wave - 1][q][4 * lane]) = f32x4{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
  }
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    f32x4 s = *(const f32x4*)(&sums[0][q][4 * lane]);
#pragma unroll
    for (int o = 1; o < 3; ++o) s += *(const f32x4*)(&sums[o][q][4 * lane]);
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[4 * q + k] += s[k];
  }
  const int r = l31, label = __shfl(own.lab, r);
  if constexpr (MODE == STATS) {
    const auto z = [&](int v, int) -> float { return acc[v]; };
    float m2, s;
    tile_stats<1>(g, cols - c0, log2_unit<LOSS>(a), z, &m2, &s);
    if (g == 0 && r < M) a.part[(long)ct * a.Mp + r] = make_float2(m2, s);
    if constexpr (LOSS == TEACHER) {
      const int token = __shfl(own.tok, min(r, M - 1));
      if (a.direct) {
        pick_direct<1>(a, token, r < M, c0, g, z);
      } else {
        const unsigned e = r < M ? entries_of(a, token, c0) : 0u;
        pick_entries<1>(a, token, e, entry_id(a, token, e), c0, g, &sums[0][0][0], z);
      }
    } else {
      const int c = r < M ? label - c0 : -1;
      if (__any(c >= 0 && c < 32)) {
        const float y = tile_pick<1>(g, c, z);
        if (c >= 0 && c < 32 && ((c >> 2) & 1) == g) a.zlab[r] = y;
      }
    }
  } else {
    const float lse2 = __shfl(own.row.x, r), d = __shfl(own.row.y, r) / own.scale;
    const int c = LOSS == LABEL ? label - (int)a.v0 : -1;
    float p[16];
#pragma unroll
    for (int v = 0; v < 16; ++v) p[v] = exp2_fast(fmaf(acc[v], log2_unit<LOSS>(a), -lse2));
    if constexpr (LOSS == TEACHER) {
      if (a.direct) subtract_direct<false>(a, __shfl(own.tok, min(r, M - 1)), r < M, a.v0 + c0, g, p);
    }
    if (r >= M) return;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int at = c0 + 8 * q + 4 * g;
      f32x4 y;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float of_it = p[4 * q + k] - (LOSS == LABEL && at + k == c ? 1.f : 0.f);
        y[k] = at + k < cols && d != 0.f ? of_it * d : 0.f;
      }
      *(f32x4*)((float*)a.g + r * a.g_pitch + at) = y;
    }
  }
}
template <int MODE, int RB, int LOSS = LABEL> hipError_t launch_tiles(const XentArgs& a, long grid, hipStream_t s) {
  static SmemOnce once;
  const hipError_t e = ensure_dynamic_lds((const void*)xent_bf16_kernel<MODE, RB, LOSS>, SMEM_B, &once);
  if (e != hipSuccess) return e;
  const long stay = a.n_cu >= 8 ? a.n_cu / 8 * 8 : 8;
  xent_bf16_kernel<MODE, RB, LOSS><<<(unsigned)(grid < stay ? grid : stay), 64 * NW, SMEM_B, s>>>(a);
  return hipGetLastError();
}
template <int MODE, int RB, int NS, bool OWN, int LOSS> hipError_t launch_few(const XentArgs& a, long wgs, hipStream_t s) {
  constexpr int bytes = NS * (128 + 32 * RB) * RK_ROWB;
  static SmemOnce once;
  const hipError_t e = ensure_dynamic_lds((const void*)xent_few_bf16_kernel<MODE, RB, NS, OWN, LOSS>, bytes, &once);
  if (e != hipSuccess) return e;
  xent_few_bf16_kernel<MODE, RB, NS, OWN, LOSS><<<(unsigned)strip_grid(wgs), 256, bytes, s>>>(a);
  return hipGetLastError();
}
template <int RB, int NS> hipError_t launch_few_dx(const XentArgs& a, hipStream_t s) {
  constexpr int bytes = NS * (BK * 256 + 32 * RB * RK_ROWB);
  static SmemOnce once;
  const hipError_t e = ensure_dynamic_lds((const void*)xent_few_dx_bf16_kernel<RB, NS>, bytes, &once);
  if (e != hipSuccess) return e;
  xent_few_dx_bf16_kernel<RB, NS><<<(unsigned)strip_grid(a.slots), 256, bytes, s>>>(a);
  return hipGetLastError();
}
inline long up(long n, long by) { return (n + by - 1) / by; }
// Whether tiles of 128 rows are the better ones for a product of `rows` x `cols` with `pairs` tile pairs: by the rounds of workgroups, a
// tile's pairs at 1.55 us (128 rows: 0.85, where they take turns 1.05) and what a tile costs beside them, 6 us (3.5).  Statistics and gradient of 300
// tokens x 256 against 50000 26.8 -> 20.8 and 31.5 -> 24.7, x 1024 66 -> 61 and 62 -> 54, 384 x 1024 against 20000 29 -> 23 and 32 -> 22; dw of
// 1261 x 192 against 10305 30 -> 20; where the rule keeps 256 rows, statistics and gradient of 512 x 3840 against 32818 186 -> 216 and 175 -> 194,
// 1000 x 1024 against 30000 60 -> 71 and 66 -> 73; dw of 2206 x 1024 against 50021 298 -> 329, 4000 x 256 against 40000 133 -> 165.
inline bool low_tiles(long rows, long cols, long pairs, int n_cu) {
  const long low = up(rows, 128) * up(cols, T), high = up(rows, T) * up(cols, T);
  return rows <= 128 || up(low, n_cu) * ((low <= n_cu ? 0.85 : 1.05) * pairs + 3.5) < up(high, n_cu) * (1.55 * pairs + 6.0);
}
// Rows of the tiles of logits of xent_few_bf16_kernel; 0: xent_bf16_kernel.  Up to 64 tokens there is one row of tiles.  With more, tiles of 64 x
// 128 where all of them have a place at once: statistics of 664 tokens x 2496 features against 2171 34 -> 20 us, 130 x 3392 against 13376 74 -> 51,
// 922 x 1280 against 3838 22 -> 17.5, 100 x 512 against 4000 10 -> 7.5; where they take turns, 300 x 256 against 20000 9.6 -> 11.5, 1024 x 512
// against 8192 13 -> 17.5.  Up to 128 tokens of many features against a long vocabulary the copies are what counts, and every entry is copied
// once: 128 x 4096 against 32768 91 (xent_bf16_kernel), 68 (64 rows), 54 (128 rows); 100 x 1024 against 30000 20, 16, 17, against 10000 17, 11,
// 16; 95 x 2432 against 4096 19 (64 rows), 29 (128).
// (GRAD: 64 or 128 tokens whatever their number: the contraction of dw runs over g's rows 64 at a time.)
inline int few_rows(long n, long cols, long pairs, int n_cu) {
  const long ct = up(cols, 128);
  if (n > 64 && n <= 128 && ct <= n_cu && 2 * ct > n_cu && pairs >= 32) return 128;
  return n <= 64 || up(n, 64) * ct <= 2L * n_cu ? 64 : 0;
}
template <int MODE, int LOSS = LABEL> hipError_t product(const XentArgs& a, long rows, long cols, long pairs, hipStream_t s) {
  if (low_tiles(rows, cols, pairs, a.n_cu)) return launch_tiles<MODE, 2, LOSS>(a, strip_grid(up(rows, 128) * up(cols, T)), s);
  return launch_tiles<MODE, 4, LOSS>(a, strip_grid(up(rows, T) * up(cols, T)), s);
}
// float32: the edge of the tiles of a product.  64 where 128 makes less than two for every compute unit: 300 tokens x 512 features against 5003,
// the four products 246 -> 112 us
inline int f32_edge(long rows, long cols, int n_cu) { return up(rows, 128) * up(cols, 128) < 2L * n_cu ? 64 : 128; }
// float32: logits by xent_few_f32_kernel.  20 tokens x 512 against 131072 161 -> 99 us, 23 x 1664 against 5347 38 -> 20, 4 x 2048 against 1967 44 -> 20;
// with more tokens rows are brought too often, 300 x 512 against 5003 25 -> 34, 64 x 256 against 65536 42 -> 41
inline bool f32_few(long n) { return n <= 32; }
constexpr long MOST_WGS = 1 << 14;     // along one side of a launch, whose threads may not pass 2^32
inline dim3 grid_of(long wgs) { return dim3((unsigned)std::min(wgs, MOST_WGS), (unsigned)up(wgs, MOST_WGS)); }
template <int MODE, int LOSS = LABEL> hipError_t f32_product(const XentArgs& a, long rows, long cols, int edge, hipStream_t s) {
  const long wgs = strip_grid(MODE == DX ? (long)a.slots : MODE == DW_PARTS ? (long)a.dw_slots : up(rows, edge) * up(cols, edge));
  const dim3 grid = grid_of(wgs);
  if (edge == 64 || MODE == DW_PARTS) xent_f32_kernel<MODE, 64, LOSS><<<grid, 256, 0, s>>>(a);
  else if constexpr (MODE != DW_PARTS) xent_f32_kernel<MODE, 128, LOSS><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}
template <int MODE, int LOSS> hipError_t logits(const XentArgs& a, int is_f32, hipStream_t s) {
  const long cols = a.v1 - a.v0;
  if (is_f32 && f32_few(a.n)) {
    xent_few_f32_kernel<MODE, LOSS><<<grid_of(strip_grid(up(cols, 32))), 256, 0, s>>>(a);
    return hipGetLastError();
  }
  if (is_f32) return f32_product<MODE, LOSS>(a, a.n, cols, f32_edge(a.n, cols, a.n_cu), s);
  const int rows = few_rows(a.n, cols, a.E / BK, a.n_cu);
  const long wgs = rows > 0 ? up(cols, 128) * up(a.n, rows) : 0;
  if (rows == 128) return launch_few<MODE, 4, 4, false, LOSS>(a, wgs, s);
  if (rows > 0 && !a.own) return wgs <= a.n_cu ? launch_few<MODE, 2, 6, false, LOSS>(a, wgs, s) : launch_few<MODE, 2, 3, false, LOSS>(a, wgs, s);
  if (rows > 0) {
    if constexpr (MODE == STATS)
      if (a.n <= 32) return wgs <= a.n_cu ? launch_few<MODE, 1, 6, true, LOSS>(a, wgs, s) : launch_few<MODE, 1, 3, true, LOSS>(a, wgs, s);
    return wgs <= a.n_cu ? launch_few<MODE, 2, 6, true, LOSS>(a, wgs, s) : launch_few<MODE, 2, 3, true, LOSS>(a, wgs, s);
  }
  return product<MODE, LOSS>(a, a.n, cols, a.E / BK, s);
}
// Statistics of a token that logits<STATS> leaves
inline int stat_parts_of(const XentArgs& a, int is_f32) {
  if (is_f32) return (int)(f32_few(a.n) ? up(a.V, 32) : 2 * up(a.V, f32_edge(a.n, a.V, a.n_cu)));
  return (int)(few_rows(a.n, a.V, a.E / BK, a.n_cu) > 0 ? up(a.V, 128) : up(a.V, T));
}
// So few tokens that every wave lists them for itself
inline bool own_of(long n, int is_f32) { return is_f32 ? f32_few(n) : n <= 64; }
// What the launches of a forward pass have in common: the whole vocabulary at once
inline void xent_fwd_sizes(XentArgs* a, int is_f32) {
  a->tile = a->tile_rows = T;
  a->piece = a->V;
  a->own = own_of(a->n, is_f32);
  a->v0 = 0;
  a->v1 = a->V;
}

}  // namespace

}  // namespace lvx
