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
// bf16 tiles of 256 x 256 and tile pairs of 64 contraction steps in two slots of 64 KB, as in the projections (lvx_project.hip,
// lvx_project_bwd.hip), but of 8 waves, two on a SIMD, each 128 x 64 as 4 x 2 blocks in the accumulation registers.  Against 4 waves with
// 128 x 128 each (which read a third less from LDS) this pays where tiles have few pairs, by what stands before and behind their loop, and
// costs where they have many.  A tile with one pair 13.7 -> 10.6 us (statistics), 19.5 -> 16.9 (gradient), 300 tokens x 1024 x 50000, 16 pairs, dw
// 64 -> 57; loss and gradients, in one session: 2206 x 1024 against 50021 (16 pairs) 959 (4 waves), 948 (8), 973 (8 that stay for their tiles,
// as here), 2048 x 4096 against 32768 (64 pairs) 1783, 1802, 1833, 4096 x 4096 against 131072 13200, 13550, 13770.
#include "lvx_xent_kernels.h"

namespace lvx {

namespace {

// ---- the tokens that have a label, in order: tok[i], its label (-1: not in the vocabulary) and (backward) its lse log2 e and d_loss (NaN for
// such a label), and how many they are ----
// 8192 tokens at a time, thread t those with number t modulo 1024, so that a wave's loads and stores are whole lines; every wave sums up the
// 128 counts of 64 tokens for itself.
__global__ void __launch_bounds__(1024) xent_list_kernel(XentArgs a) {
  __shared__ int counts[2][128];
  __shared__ float tops[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int total = 0, turn = 0;
  float top = 0.f;                                   // the largest finite |d_loss|
  for (long base = 0; base < a.n; base += 8192) {
    long lab[8];
    float d[8], lse[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const long i = base + 1024 * k + tid;
      lab[k] = i < a.n ? a.labels[i] : -1;
      d[k] = a.d_loss && i < a.n ? a.d_loss[i] * a.inv_t : 0.f;
      lse[k] = a.d_loss && i < a.n ? a.lse[i] : 0.f;
    }
    turn ^= 1;                                       // (who writes a place again has crossed the barrier between)
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int c = __popcll(__ballot(lab[k] >= 0));
      if (lane == 0) counts[turn][16 * k + wave] = c;
    }
    __syncthreads();
    const int c0 = counts[turn][2 * lane], c1 = counts[turn][2 * lane + 1];
    int upto = c0 + c1;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int y = __shfl_up(upto, o);
      upto += lane >= o ? y : 0;
    }
    const int before = upto - c1 - (wave % 2 == 0 ? c0 : 0);      // of number 2 lane + wave % 2
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const long i = base + 1024 * k + tid;
      const unsigned long long on = __ballot(lab[k] >= 0);
      const int at = total + __shfl(before, 8 * k + wave / 2) + __popcll(on & ((1ull << lane) - 1));
      if (lab[k] >= 0) {
        a.tok[at] = (int)i;
        a.lab[at] = lab[k] < a.V ? (int)lab[k] : -1;
        if (a.d_loss) a.row[at] = make_float2(lse[k] * LOG2E, lab[k] < a.V ? d[k] : __builtin_nanf(""));
        if (fabsf(d[k]) > top && fabsf(d[k]) < __builtin_inff()) top = fabsf(d[k]);
      } else if (a.loss && i < a.n) {
        a.loss[i] = 0.f;
        a.lse_out[i] = 0.f;
      }
    }
    total += __shfl(upto, 63);
  }
#pragma unroll
  for (int o = 1; o < 64; o *= 2) top = fmaxf(top, __shfl_xor(top, o));
  if (lane == 0) tops[wave] = top;
  __syncthreads();
  const int parts = dx_parts((total + a.tile_rows - 1) / a.tile_rows * ((a.E + a.tile - 1) / a.tile), (int)(a.piece / BK), a.n_cu, a.slots);
  const int dw_parts = a.dw_slots > 0 ? dx_parts(a.dw_tiles, (total + BK - 1) / BK, a.n_cu, a.dw_slots) : 1;
  if (tid != 0) return;
  for (int w = 0; w < 16; ++w) top = fmaxf(top, tops[w]);
  a.head->count = total;
  a.head->scale = top > 0.f ? top : 1.f;
  a.head->parts = parts;
  a.head->dw_parts = dw_parts;
}

// lse and loss of the listed tokens from what the tiles' waves left: 8 tokens a workgroup, 32 threads each
__global__ void __launch_bounds__(256) xent_join_kernel(XentArgs a, int n_parts) {
  __shared__ float sm[8][33], ss[8][33];
  const int row_l = threadIdx.x % 8, lane = threadIdx.x / 8;
  const Own own = a.own ? own_list(a) : Own{};
  const int count = a.own ? own.count : a.head->count;
  if (a.own && blockIdx.x == 0 && (int)threadIdx.x >= count && threadIdx.x < a.n) {        // (the tokens that are not listed)
    a.loss[own.tok] = 0.f;
    a.lse_out[own.tok] = 0.f;
  }
  for (int r0 = blockIdx.x * 8; r0 < count; r0 += gridDim.x * 8) {
    const int r = min(r0 + row_l, count - 1);
    const int tok = a.own ? __shfl(own.tok, r) : a.tok[r], lab = a.own ? __shfl(own.lab, r) : a.lab[r];
    float m = -__builtin_inff(), s = 0.f;
    const auto join = [&](float m1, float s1) { join_stats(&m, &s, m1, s1); };
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
      const float bad = lab < 0 ? __builtin_nanf("") : 0.f;
      const float lse = (m + __builtin_amdgcn_logf(s)) * LN2 + bad;
      a.lse_out[tok] = lse;
      a.loss[tok] = lse - a.zlab[r];
    }
    __syncthreads();
  }
}

// Sums of parts, 32 rows x 32 features a workgroup.  DX: of the listed tokens; 0 for the others.  DW_PARTS: of the piece's vocabulary.
template <int MODE> __global__ void __launch_bounds__(256) xent_sum_bf16_kernel(XentArgs a, unsigned tiles) {
  const int M = MODE == DX ? a.head->count : (int)(a.v1 - a.v0), E = a.E, tid = threadIdx.x, n_ec = (E + 31) / 32;
  if (blockIdx.x < tiles) {
    const bool rows = MODE == DX && a.own;             // (what xent_few_dx_bf16_kernel left)
    const int r = (int)(blockIdx.x / n_ec) * 32 + (rows ? tid / 8 : tid % 32), c = (int)(blockIdx.x % n_ec) * 32 + 4 * (rows ? tid % 8 : tid / 32);
    if (r >= M || c >= E) return;
    const int tr = MODE == DX ? a.tile_rows : 128, n_ct = (E + T - 1) / T, rl = r % tr, cl = c % T;
    const long tile = (long)(r / tr) * n_ct + c / T;
    long step = (long)((M + tr - 1) / tr) * n_ct * tr * T;
    const int wave = rl / (tr / 2) * (NW / 2) + cl / WC, i = rl % (tr / 2) / 32, j = cl % WC / 32, q = cl % 32 / 8;
    const float* from = (MODE == DX ? a.dx_part : a.dw_part) + tile * (tr * T) + wave * (tr * T / NW) + ((j * (tr / 64) + i) * 4 + q) * 256 + (rl % 32 + 32 * (cl / 4 % 2)) * 4;
    if (rows) {
      const long pitch = (E + 127) / 128 * 128L;
      from = a.dx_part + r * pitch + c;
      step = 64 * pitch;
    }
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    const int parts = MODE == DX ? a.head->parts : a.head->dw_parts;
    for (int p0 = 0; p0 < parts; p0 += 8) {              // (eight on their way at once)
      f32x4 v[8];
#pragma unroll
      for (int p = 0; p < 8; ++p) v[p] = *(const f32x4*)(from + min(p0 + p, parts - 1) * step);
#pragma unroll
      for (int p = 0; p < 8; ++p)
        if (p0 + p < parts) s += v[p];
    }
    s *= a.head->scale;
    uint16_t* const to = MODE == DX ? (uint16_t*)a.dx + a.tok[r] * a.ldx : (uint16_t*)a.dw + (a.v0 + r) * E;
    *(u32x2*)(to + c) = u32x2{pack2_bf16(s[0], s[1]), pack2_bf16(s[2], s[3])};
    return;
  }
  for (long i = (long)(blockIdx.x - tiles) * 4 + (tid >> 6); i < a.n; i += (long)(gridDim.x - tiles) * 4)
    if (a.labels[i] < 0)
      for (int e = 8 * (tid & 63); e < E; e += 512) *(u32x4*)((uint16_t*)a.dx + i * a.ldx + e) = u32x4{0u, 0u, 0u, 0u};
}

// The same in float32: a row and 256 features (blockIdx.y) a workgroup.
template <int MODE> __global__ void __launch_bounds__(256) xent_sum_f32_kernel(XentArgs a, unsigned rows) {
  const int M = MODE == DX ? a.head->count : (int)(a.v1 - a.v0), E = a.E, e = (int)blockIdx.y * 256 + threadIdx.x;
  if (e >= E) return;
  if (blockIdx.x < rows) {
    const int t = MODE == DX ? a.tile : 64, n_ct = (E + t - 1) / t, parts = MODE == DX ? a.head->parts : a.head->dw_parts;
    const long step = (long)((M + t - 1) / t) * n_ct * (t * t);
    for (int r = blockIdx.x; r < M; r += rows) {
      const float* const from = (MODE == DX ? a.dx_part : a.dw_part) + ((long)(r / t) * n_ct + e / t) * (t * t) + (r % t) * t + e % t;
      float s = 0.f;
      for (int p0 = 0; p0 < parts; p0 += 8) {
        float v[8];
#pragma unroll
        for (int p = 0; p < 8; ++p) v[p] = from[min(p0 + p, parts - 1) * step];
#pragma unroll
        for (int p = 0; p < 8; ++p) s += p0 + p < parts ? v[p] : 0.f;
      }
      (MODE == DX ? (float*)a.dx + a.tok[r] * a.ldx : (float*)a.dw + (a.v0 + r) * E)[e] = s * a.head->scale;
    }
    return;
  }
  for (long i = blockIdx.x - rows; i < a.n; i += gridDim.x - rows)
    if (a.labels[i] < 0) ((float*)a.dx)[i * a.ldx + e] = 0.f;
}

// dx: columns and rows of a tile.  float32: 128 where the parts make one for every compute unit (3000 tokens x 512 features against 40000 1610 -> 1210
// us, 1000 x 512 against 10000 148 -> 118, 2000 x 200 against 3000 53 -> 43; where they do not, 100 x 256 against 30000 32 -> 47, 300 x 1024 against
// 1000 13.6 -> 26) and there is more than half a tile of tokens (20 x 512 against 131072 181 -> 110 with 64, 2 x 640 against 32768 57 -> 35).
int dx_f32_edge(long n, int E, long V, int n_cu) {
  return n <= 64 || up(n, 128) * up(E, 128) * std::max(1L, std::min((long)MOST_PARTS, V / 256)) < n_cu ? 64 : 128;
}
int dx_edge(long n, int E, long V, int n_cu, int is_f32) { return is_f32 ? dx_f32_edge(n, E, V, n_cu) : T; }
int dx_rows(long n, int E, long V, int n_cu, int is_f32) { return is_f32 ? dx_f32_edge(n, E, V, n_cu) : n <= 128 ? 128 : T; }
// dw in parts: its tiles
int dw_rows(int is_f32) { return is_f32 ? 64 : 128; }
int dw_edge(int is_f32) { return is_f32 ? 64 : T; }
long dw_tiles(long cols, int E, int is_f32) { return up(cols, dw_rows(is_f32)) * up(E, dw_edge(is_f32)); }
// Whether the contraction of dw is better cut into parts: a tile pair's time (64 tokens) is 0.85 us, float32 1.6, and writing the parts, reading
// them and the launch cost 12.  dw of 16384 tokens x 128 against 1000 191 -> 25 us, 5000 x 512 against 1500 68 -> 25, 2048 x 512 against 4000
// 30 -> 27, float32 4000 x 256 against 1000 101 -> 37; where the rule keeps one part, 1024 x 1024 against 2000 17 -> 23.
bool dw_parts_pay(long pairs, long parts, int is_f32) { return (is_f32 ? 1.6 : 0.85) * (pairs - pairs / parts) >= 12.0; }
hipError_t dw_in_parts(const XentArgs& a, int is_f32, hipStream_t s) {
  const long cols = a.v1 - a.v0;
  const hipError_t e = is_f32 ? f32_product<DW_PARTS>(a, cols, a.E, 64, s) : launch_tiles<DW_PARTS, 2>(a, strip_grid(a.dw_slots), s);
  if (e != hipSuccess) return e;
  if (is_f32) {
    xent_sum_f32_kernel<DW_PARTS><<<dim3((unsigned)cols, (unsigned)up(a.E, 256)), 256, 0, s>>>(a, (unsigned)cols);
  } else {
    const unsigned tiles = (unsigned)(up(cols, 32) * up(a.E, 32));
    xent_sum_bf16_kernel<DW_PARTS><<<tiles, 256, 0, s>>>(a, tiles);
  }
  return hipGetLastError();
}
}  // namespace

// Tiles of sums of dw that a piece of `cols` columns takes; at most one for a compute unit, so that a workgroup has one.  0: it is not cut.
long xent_dw_slots(long n, int E, long cols, int n_cu, int is_f32) {
  const long tiles = dw_tiles(cols, E, is_f32), pairs = up(n, BK), parts = std::min({(long)MOST_PARTS, pairs / 4, n_cu / 8 * 8 / tiles});
  return parts < 2 || !dw_parts_pay(pairs, parts, is_f32) ? 0 : parts * tiles;
}
size_t xent_dw_bytes(long n, int E, long cols, int n_cu, int is_f32) {
  return sizeof(float) * dw_rows(is_f32) * dw_edge(is_f32) * xent_dw_slots(n, E, cols, n_cu, is_f32);
}
// Room for them, and for those of every problem with fewer tokens, features or entries, which may have parts where this one has none: no more tiles
// than compute units, nor than this one's tiles in the most parts that its tokens allow.
size_t xent_dw_room(long n, int E, long V, int n_cu, int is_f32) {
  const long pairs = up(n, BK), parts = std::min((long)MOST_PARTS, pairs / 4);
  if (parts < 2 || !dw_parts_pay(pairs, parts, is_f32)) return 0;
  return sizeof(float) * dw_rows(is_f32) * dw_edge(is_f32) * std::min((long)(n_cu / 8 * 8), parts * dw_tiles(V, E, is_f32));
}

bool xent_bf16_supported(int E) { return E % BK == 0; }
int xent_stat_parts(long V, int is_f32) { return (int)(2 * up(V, is_f32 ? 64 : T)); }
// Bytes of the tiles of dx's sums, and how many these are: one for every tile at least, two for every compute unit where 64 parts of a tile
// make so many; no more with fewer tokens or features or a smaller vocabulary.
long xent_dx_slots(long n, int E, long V, int n_cu, int is_f32) {
  const long tiles = up(n, dx_rows(n, E, V, n_cu, is_f32)) * up(E, dx_edge(n, E, V, n_cu, is_f32)), some = MOST_PARTS * tiles < 2L * n_cu ? MOST_PARTS * tiles : 2L * n_cu;
  return tiles > some ? tiles : some;
}
size_t xent_dx_bytes(long n, int E, long V, int n_cu, int is_f32) {
  return sizeof(float) * dx_rows(n, E, V, n_cu, is_f32) * dx_edge(n, E, V, n_cu, is_f32) * xent_dx_slots(n, E, V, n_cu, is_f32);
}

hipError_t launch_xent_list(const XentArgs& a, hipStream_t s) {
  xent_list_kernel<<<1, 1024, 0, s>>>(a);
  return hipGetLastError();
}
hipError_t launch_xent_fwd(XentArgs a, int is_f32, hipStream_t s) {
  xent_fwd_sizes(&a, is_f32);
  if (!a.own) xent_list_kernel<<<1, 1024, 0, s>>>(a);
  const hipError_t e = logits<STATS, LABEL>(a, is_f32, s);
  if (e != hipSuccess) return e;
  const long wgs = up(a.n, 8);
  xent_join_kernel<<<(unsigned)(wgs < 4096 ? wgs : 4096), 256, 0, s>>>(a, stat_parts_of(a, is_f32));
  return hipGetLastError();
}

hipError_t launch_xent_bwd(XentArgs a, int is_f32, hipStream_t s) { return launch_xent_products(a, is_f32, s, launch_xent_list, logits<GRAD, LABEL>); }

// list: what xent_list_kernel leaves; gradient: leaves that of a piece's logits
hipError_t launch_xent_products(XentArgs a, int is_f32, hipStream_t s, hipError_t (*list)(const XentArgs&, hipStream_t),
                                hipError_t (*gradient)(const XentArgs&, int, hipStream_t)) {
  a.own = own_of(a.n, is_f32);
  a.dw_tiles = (int)dw_tiles(std::min(a.piece, a.V), a.E, is_f32);
  a.tile = dx_edge(a.n, a.E, a.V, a.n_cu, is_f32);
  a.tile_rows = dx_rows(a.n, a.E, a.V, a.n_cu, is_f32);
  if (a.own && !is_f32) {                            // (tiles of a quarter of the size that there is room for)
    a.tile = 128;
    a.tile_rows = 64;
    a.slots = (int)std::max(up(a.E, 128), std::min(MOST_PARTS * up(a.E, 128), 2L * a.n_cu));
  }
  hipError_t e = a.own ? hipSuccess : list(a, s);
  a.first = 1;
  for (a.v0 = 0; a.v0 < a.V && e == hipSuccess; a.v0 = a.v1) {
    a.v1 = a.v0 + a.piece < a.V ? a.v0 + a.piece : a.V;
    const long cols = a.v1 - a.v0;
    e = gradient(a, is_f32, s);
    if (e == hipSuccess && a.dw && a.dw_slots > 0) e = dw_in_parts(a, is_f32, s);
    else if (e == hipSuccess && a.dw)
      e = is_f32 ? f32_product<DW>(a, cols, a.E, f32_edge(cols, a.E, a.n_cu), s) : product<DW>(a, cols, a.E, up(a.n, BK), s);
    if (e == hipSuccess && a.dx) {
      e = is_f32 ? f32_product<DX>(a, a.n, a.E, a.tile, s)
          : a.own ? a.n <= 32 ? launch_few_dx<1, 6>(a, s) : launch_few_dx<2, 6>(a, s)
                 : a.tile_rows == 128 ? launch_tiles<DX, 2>(a, strip_grid(a.slots), s) : launch_tiles<DX, 4>(a, strip_grid(a.slots), s);
      a.first = 0;
    }
  }
  if (e != hipSuccess || !a.dx) return e;
  const long zero = up(a.n, 4) < 1024 ? up(a.n, 4) : 1024;
  if (is_f32) {
    const unsigned rows = (unsigned)std::min(a.n, MOST_WGS);
    xent_sum_f32_kernel<DX><<<dim3(rows + (unsigned)zero, (unsigned)up(a.E, 256)), 256, 0, s>>>(a, rows);
  } else {
    const unsigned tiles = (unsigned)(up(a.n, 32) * up(a.E, 32));
    xent_sum_bf16_kernel<DX><<<tiles + (unsigned)zero, 256, 0, s>>>(a, tiles);
  }
  return hipGetLastError();
}

}  // namespace lvx
