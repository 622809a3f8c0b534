// Layer norm and root-mean-square norm of token features with their gradients, and the 8-bit checkpoint of what they
// read (lvx_packed.h).
//
//   y = xh gamma + beta,  xh = (x - mu) r,  r = 1 / sqrt(mean((x - mu)^2) + eps)        (rms: mu = 0)
//   dx = r (a - mean(a) - xh mean(a xh)),  a = dy gamma       (rms: without mean(a))
//   dgamma += sum over the rows of dy xh,  dbeta += sum of dy
//
// Sums are float32 throughout; the spread is summed from the differences to the mean, in a second pass over the row, so a large
// mean costs no digits.  The gradients of gamma and beta go through memory as one partial sum per part of the rows and are
// added up in the order of the parts: results repeat bit for bit.
#include "lvx_internal.h"
#include "lvx_mfma.h"
#include "lvx_packed.h"

#include <type_traits>

// What is fused is written out (fmaf): the norm made again from the packed form has to be the first one bit for bit, and the
// compiler's own choice differs from kernel to kernel.
#pragma clang fp contract(off)

namespace lvx {

namespace {

constexpr int WG = 256;

__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const __bf16* p) { return (float)*p; }

// Sums and maxima over 4, 32 or all 64 lanes, in every lane the same: neighbours inside a quad, mirrored halves and rows of 16, then
// rows against each other.  (Both sides of every step add the same two numbers, so the lanes agree to the last bit.)
template <int CTRL> __device__ __forceinline__ unsigned dpp(unsigned x) {
  return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true);
}
template <int W, class F> __device__ __forceinline__ unsigned lanes_join(unsigned x, F&& f) {
  x = f(x, dpp<0xB1>(x));                            // lanes 1 apart
  x = f(x, dpp<0x4E>(x));                            // 2
  if constexpr (W > 4) {
    x = f(x, dpp<0x141>(x));                         // the other quad of 8
    x = f(x, dpp<0x140>(x));                         // the other half of 16
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = f(r[0], r[1]);
  }
  if constexpr (W > 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    x = f(r[0], r[1]);
  }
  return x;
}
template <int W> __device__ __forceinline__ float lanes_sum(float x) {
  return __uint_as_float(lanes_join<W>(__float_as_uint(x), [](unsigned a, unsigned b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}
template <int W> __device__ __forceinline__ unsigned lanes_max(unsigned x) {
  return lanes_join<W>(x, [](unsigned a, unsigned b) { return a > b ? a : b; });
}
// over the workgroup, the same in every thread (`at`: 4 floats of LDS that no wave still reads)
__device__ __forceinline__ float wg_sum(float x, float* at) {
  x = lanes_sum<64>(x);
  if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = x;
  __syncthreads();
  return (at[0] + at[1]) + (at[2] + at[3]);
}

// ---- rows of fewer than 8 features or more than 16384: a workgroup each, an element per thread, the row read again for every sum ----

// Element e of a row as the norm sees it (any e of a group of 32 lanes that asks for a group, E and more: 0).
// SRC 0: x.  1: the packed form of x (which is written where `keep` says so).  2: what was packed before.
template <typename T, int SRC>
__device__ __forceinline__ float norm_in(const T* x, int8_t* q, uint8_t* b, int e, int E, bool keep) {
  if constexpr (SRC == 0) return e < E ? load1(x + e) : 0.f;
  if constexpr (SRC == 2) return e < E ? (float)q[e] * packed::step_of(b[e / packed::GROUP]) : 0.f;
  const float v = e < E ? load1(x + e) : 0.f;
  const unsigned byte = packed::exponent_of(lanes_max<32>(packed::magnitude(v)));
  const float s = packed::steps(v, packed::inverse_step_of(byte));
  if (keep && e < E) {
    q[e] = packed::whole(s);
    if (e % packed::GROUP == 0) b[e / packed::GROUP] = (uint8_t)byte;
  }
  return e < E ? packed::value(s, packed::step_of(byte)) : 0.f;
}

template <typename T, int SRC>
__global__ void __launch_bounds__(WG) norm_fwd_any_kernel(NormArgs a) {
  __shared__ float sums[2][4];
  const int E = a.E, tid = threadIdx.x, E32 = (E + 31) / 32 * 32;
  const float inv = 1.f / (float)E;
  for (long row = blockIdx.x; row < a.n; row += gridDim.x) {
    const T* const x = (const T*)a.x + row * a.x_ss;
    int8_t* const q = a.q + row * E;
    uint8_t* const b = a.b + row * packed::groups(E);
    T* const y = (T*)a.y + row * a.y_ss;
    __syncthreads();                                 // (the sums of the row before have been read)
    float mu = 0.f, s = 0.f;
    if (!a.rms) {
      for (int e = tid; e < E32; e += WG) s += norm_in<T, SRC>(x, q, b, e, E, false);
      mu = wg_sum(s, sums[0]) * inv;
    }
    s = 0.f;
    for (int e = tid; e < E32; e += WG) {
      const float d = norm_in<T, SRC>(x, q, b, e, E, false) - mu;
      s = e < E ? fmaf(d, d, s) : s;
    }
    const float r = 1.f / sqrtf(wg_sum(s, sums[1]) * inv + a.eps);
    for (int e = tid; e < E32; e += WG) {
      const float v = norm_in<T, SRC>(x, q, b, e, E, true);
      if (e < E) {
        y[e] = (T)fmaf((v - mu) * r, load1((const T*)a.gamma + e), a.beta ? load1((const T*)a.beta + e) : 0.f);
      }
    }
    if (tid == 0) {
      a.stats[2 * row] = mu;
      a.stats[2 * row + 1] = r;
    }
  }
}

template <typename T, int SRC>
__global__ void __launch_bounds__(WG) norm_bwd_any_kernel(NormArgs a) {
  __shared__ float sums[2][4];
  const int E = a.E, tid = threadIdx.x;
  const float inv = 1.f / (float)E;
  for (long row = blockIdx.x; row < a.n; row += gridDim.x) {
    const T* const x = (const T*)a.x + row * a.x_ss;
    int8_t* const q = a.q + row * E;
    uint8_t* const b = a.b + row * packed::groups(E);
    const T* const dy = (const T*)a.dy + row * a.y_ss;
    T* const dx = (T*)a.dx + row * a.x_ss;
    const float mu = a.stats_in[2 * row], r = a.stats_in[2 * row + 1];
    float s = 0.f, sx = 0.f;
    for (int e = tid; e < E; e += WG) {
      const float g = load1(dy + e) * load1((const T*)a.gamma + e);
      s += g;
      sx = fmaf(g, (norm_in<T, SRC>(x, q, b, e, E, false) - mu) * r, sx);
    }
    __syncthreads();
    s = a.rms ? 0.f : wg_sum(s, sums[0]) * inv;
    sx = wg_sum(sx, sums[1]) * inv;
    for (int e = tid; e < E; e += WG) {
      const float g = load1(dy + e) * load1((const T*)a.gamma + e);
      const float xh = (norm_in<T, SRC>(x, q, b, e, E, false) - mu) * r;
      dx[e] = (T)(r * fmaf(-xh, sx, g - s));
    }
  }
}

// partial sums of dgamma and dbeta over part blockIdx.y of the rows: [part][2][E]
template <typename T, int SRC>
__global__ void __launch_bounds__(WG) norm_param_any_kernel(NormArgs a) {
  const int E = a.E, e = blockIdx.x * WG + threadIdx.x;
  if (e >= E) return;
  const long r0 = a.n * blockIdx.y / a.parts, r1 = a.n * (blockIdx.y + 1) / a.parts;
  float sg = 0.f, sb = 0.f;
  for (long row = r0; row < r1; ++row) {
    const float dy = load1((const T*)a.dy + row * a.y_ss + e);
    const float xh = (norm_in<T, SRC>((const T*)a.x + row * a.x_ss, a.q + row * E, a.b + row * packed::groups(E), e, E, false) -
                      a.stats_in[2 * row]) * a.stats_in[2 * row + 1];
    sg = fmaf(dy, xh, sg);
    sb += dy;
  }
  a.part[(2L * blockIdx.y) * E + e] = sg;
  a.part[(2L * blockIdx.y + 1) * E + e] = sb;
}

// dgamma += the parts' sums, dbeta likewise, in a fixed order: 32 threads share a column, 8 parts of each are on their way at once
__global__ void __launch_bounds__(WG) norm_param_sum_kernel(NormArgs a) {
  __shared__ float sums[32][33];
  const int col = threadIdx.x % 8, lane = threadIdx.x / 8;
  const long at = (long)blockIdx.x * 32 + 4 * col, n = 2L * a.E;  // dgamma's columns, then dbeta's
  typedef f32x4 __attribute__((aligned(4))) f32x4_any;
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  const int whole = (int)min(n - at, 4L);            // (a place's last columns: fewer, or none)
  for (int p0 = lane; p0 < a.parts; p0 += 256) {
    f32x4 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float* const from = a.part + n * min(p0 + 32 * i, a.parts - 1) + at;
      v[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (whole == 4) v[i] = *(const f32x4_any*)from;
      else
        for (int k = 0; k < 3; ++k)
          if (k < whole) v[i][k] = from[k];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) s[k] += p0 + 32 * i < a.parts ? v[i][k] : 0.f;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) sums[lane][4 * col + k] = s[k];
  __syncthreads();
  const long c = (long)blockIdx.x * 32 + threadIdx.x;
  if (threadIdx.x >= 32 || c >= n) return;
  float x = 0.f;
#pragma unroll
  for (int i = 0; i < 32; ++i) x += sums[i][threadIdx.x];
  float* const to = c < a.E ? a.dgamma : a.dbeta;
  if (to) to[c < a.E ? c : c - a.E] += x;
}

// ---- rows in registers: a team of TPR threads has a row, a thread NV chunks of 8 features of it ----
//
// A chunk is moved at once wherever it lies: the memory instructions take any address that the element type has.  FULL: E is a
// multiple of 8.  Otherwise a row's last chunk is loaded as the row's last 8 features, of which the first skip_of belong to the chunk before and
// are cleared where they are used (not where they are loaded, which would wait for the row while it is on its way), and stored element by
// element.  Which thread has which features goes by E alone, so the norm made again from the packed form is the first one bit for
// bit, whatever x's addresses were.

constexpr int V = 8;
__host__ __device__ constexpr int chunks(int E) { return (E + V - 1) / V; }
typedef u32x4 __attribute__((aligned(2))) u32x4_any2;
typedef u32x4 __attribute__((aligned(4))) u32x4_any4;
typedef u32x2 __attribute__((aligned(1))) u32x2_any;

// where chunk c starts as it is loaded (E >= 8), and how many of its 8 features are not its own
template <bool FULL> __device__ __forceinline__ int start_of(int c, int E) { return FULL ? V * c : min(V * c, E - V); }
template <bool FULL> __device__ __forceinline__ int skip_of(int c, int E) { return FULL || c < chunks(E) - 1 ? 0 : c < chunks(E) ? V * c - (E - V) : V; }

// chunk c of a row of E features as it lies in memory; 0 behind the row's end
template <typename T> struct Chunk;
template <> struct Chunk<__bf16> {
  u32x4 w;
  template <bool FULL> __device__ __forceinline__ void load(const __bf16* row, int c, int E) {
    w = u32x4{0u, 0u, 0u, 0u};
    if (c < chunks(E)) w = *(const u32x4_any2*)(row + start_of<FULL>(c, E));
  }
  __device__ __forceinline__ void keep_from(int skip) {
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] &= (2 * j >= skip ? 0x0000ffffu : 0u) | (2 * j + 1 >= skip ? 0xffff0000u : 0u);
  }
  __device__ __forceinline__ float operator[](int i) const { return __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16); }
  // the largest magnitude, as the bits of a float32
  __device__ __forceinline__ unsigned largest() const {
    typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
    u16x2 m = __builtin_bit_cast(u16x2, w[0] & 0x7fff7fffu);
#pragma unroll
    for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu));
    const unsigned x = (unsigned)m[0] << 16, y = (unsigned)m[1] << 16;
    return x > y ? x : y;
  }
  static __device__ __forceinline__ void store8(__bf16* p, const float (&v)[V]) {
    *(u32x4_any2*)p = u32x4{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7])};
  }
};
template <> struct Chunk<float> {
  u32x4 w[2];
  template <bool FULL> __device__ __forceinline__ void load(const float* row, int c, int E) {
    w[0] = w[1] = u32x4{0u, 0u, 0u, 0u};
    if (c < chunks(E)) {
      const u32x4_any4* const p = (const u32x4_any4*)(row + start_of<FULL>(c, E));
      w[0] = p[0];
      w[1] = p[1];
    }
  }
  __device__ __forceinline__ void keep_from(int skip) {
#pragma unroll
    for (int i = 0; i < V; ++i) w[i / 4][i % 4] = i >= skip ? w[i / 4][i % 4] : 0u;
  }
  __device__ __forceinline__ float operator[](int i) const { return __uint_as_float(w[i / 4][i % 4]); }
  __device__ __forceinline__ unsigned largest() const {
    unsigned m = 0u;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const unsigned x = w[i / 4][i % 4] & 0x7fffffffu;
      m = m > x ? m : x;
    }
    return m;
  }
  static __device__ __forceinline__ void store8(float* p, const float (&v)[V]) {
    *(u32x4_any4*)p = __builtin_bit_cast(u32x4, f32x4{v[0], v[1], v[2], v[3]});
    *(u32x4_any4*)(p + 4) = __builtin_bit_cast(u32x4, f32x4{v[4], v[5], v[6], v[7]});
  }
};
template <bool FULL, typename T> __device__ __forceinline__ void store_chunk(T* row, int c, int E, const float (&v)[V]) {
  if (FULL ? c < chunks(E) : V * c + V <= E) {
    Chunk<T>::store8(row + V * c, v);
  } else if (!FULL && c < chunks(E)) {
    const int skip = skip_of<FULL>(c, E);
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (k >= skip) row[E - V + k] = (T)v[k];
  }
}

// 8 packed features and their exponent byte (behind the row's end: 0 steps)
struct PackedChunk {
  u32x2 w;
  unsigned b;
  template <bool FULL> __device__ __forceinline__ void load(const int8_t* q, const uint8_t* e, int c, int E) {
    w = u32x2{0u, 0u};
    b = 8u;
    if (c < chunks(E)) {
      w = *(const u32x2_any*)(q + start_of<FULL>(c, E));
      b = e[c / (packed::GROUP / V)];
    }
  }
  __device__ __forceinline__ void keep_from(int skip) {
    const unsigned long long m = skip >= V ? 0ull : ~0ull << (8 * skip);
    w[0] &= (unsigned)m;
    w[1] &= (unsigned)(m >> 32);
  }
  __device__ __forceinline__ float step() const { return packed::step_of(b); }
  __device__ __forceinline__ float operator[](int i) const { return (float)(int8_t)(w[i / 4] >> (8 * (i % 4))); }     // in steps
};
// Packs a chunk (all lanes of its group of 32 features take part): its values in steps, and the step.
template <bool FULL, typename T> __device__ __forceinline__ float pack_chunk(const Chunk<T>& x, float (&v)[V], int8_t* q, uint8_t* e, int c, int E) {
  const unsigned b = packed::exponent_of(lanes_max<packed::GROUP / V>(x.largest()));
  const float inverse = packed::inverse_step_of(b);
  unsigned s[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float y = packed::steps(x[i], inverse);
    s[i] = __float_as_uint(y);
    v[i] = y - packed::ROUNDER;
  }
  if (FULL ? c < chunks(E) : V * c + V <= E) {
    const auto four = [](unsigned s0, unsigned s1, unsigned s2, unsigned s3) {          // their low bytes
      return __builtin_amdgcn_perm(__builtin_amdgcn_perm(s3, s2, 0x0c0c0400), __builtin_amdgcn_perm(s1, s0, 0x0c0c0400), 0x05040100);
    };
    *(u32x2_any*)(q + V * c) = u32x2{four(s[0], s[1], s[2], s[3]), four(s[4], s[5], s[6], s[7])};
  } else if (!FULL && c < chunks(E)) {
    const int skip = skip_of<FULL>(c, E);
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (k >= skip) q[E - V + k] = (int8_t)(s[k] & 0xffu);
  }
  if (c < chunks(E) && c % (packed::GROUP / V) == 0) e[c / (packed::GROUP / V)] = (uint8_t)b;
  return packed::step_of(b);
}

// Sums over a team.  One wave: by lanes.  More: through LDS, in two places that take turns, with one barrier each: who writes a
// place again has crossed the barrier of the sum between, which every wave reaches after reading the place.
template <int TPR> struct TeamSum {
  float (*at)[2][16];                                // [turn][which][wave]
  int turn = 0;
  template <int N> __device__ __forceinline__ void operator()(float (&x)[N]) {
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = lanes_sum<64>(x[k]);
    if constexpr (TPR > 64) {
      constexpr int W = TPR / 64;
      turn ^= 1;
      if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int k = 0; k < N; ++k) at[turn][k][threadIdx.x >> 6] = x[k];
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < N; ++k) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) s += at[turn][k][w];
        x[k] = s;
      }
    }
  }
};
constexpr int wg_of(int tpr) { return tpr > WG ? tpr : WG; }

// A team, and the same number in a scalar register (a wave belongs to one team)
template <int TPR> __device__ __forceinline__ int team_of() { return TPR >= WG ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x / TPR); }


// The next row is on its way while one is worked on.  Values are v[i][k] * step[i] (packed features: whole steps; others: step 1).
template <typename T, int SRC, bool FULL, int TPR, int NV>
__global__ void __launch_bounds__(wg_of(TPR), NV > 2 ? 3 : 4) norm_fwd_kernel(NormArgs a) {
  constexpr int TEAMS = wg_of(TPR) / TPR;
  __shared__ float sums[2][2][16];
  TeamSum<TPR> team_sum{sums};
  const int t = threadIdx.x % TPR, E = a.E;
  const float inv = 1.f / (float)E;
  struct Row {
    Chunk<T> x[SRC == 2 ? 1 : NV];
    PackedChunk p[SRC == 2 ? NV : 1];
  };
  auto load = [&](Row& w, long row) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if constexpr (SRC == 2) w.p[i].template load<FULL>(a.q + row * E, a.b + row * packed::groups(E), t + TPR * i, E);
      else w.x[i].template load<FULL>((const T*)a.x + row * a.x_ss, t + TPR * i, E);
    }
  };
  const long by = (long)gridDim.x * TEAMS;
  long row = (long)blockIdx.x * TEAMS + team_of<TPR>();
  Row next;
  if (row < a.n) load(next, row);
  Chunk<T> gamma[NV], beta[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    gamma[i].template load<FULL>((const T*)a.gamma, t + TPR * i, E);
    if (a.beta) beta[i].template load<FULL>((const T*)a.beta, t + TPR * i, E);
    else beta[i] = Chunk<T>{};
  }
  for (; row < a.n; row += by) {
    Row w = next;
    if (row + by < a.n) load(next, row + by);
    if constexpr (!FULL) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if constexpr (SRC == 2) w.p[i].keep_from(skip_of<FULL>(t + TPR * i, E));
        else w.x[i].keep_from(skip_of<FULL>(t + TPR * i, E));
      }
    }
    float v[NV][V], step[NV];
    float s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if constexpr (SRC == 1) {
        step[i] = pack_chunk<FULL>(w.x[i], v[i], a.q + row * E, a.b + row * packed::groups(E), t + TPR * i, E);
      } else {
        if constexpr (SRC == 2) step[i] = w.p[i].step();
#pragma unroll
        for (int k = 0; k < V; ++k) {
          if constexpr (SRC == 2) v[i][k] = w.p[i][k];
          else v[i][k] = w.x[i][k];
        }
      }
      if (SRC == 0) step[i] = 1.f;
      float c = 0.f;
#pragma unroll
      for (int k = 0; k < V; ++k) c += v[i][k];
      s[0] = SRC == 0 ? s[0] + c : fmaf(c, step[i], s[0]);
    }
    float mu = 0.f;
    if (!a.rms) {
      team_sum(s);
      mu = s[0] * inv;
    }
    s[0] = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + TPR * i;
      float z = 0.f;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        v[i][k] = SRC == 0 ? v[i][k] - mu : fmaf(v[i][k], step[i], -mu);
        const float d = FULL || k >= skip_of<FULL>(c, E) ? v[i][k] : 0.f;
        z = fmaf(d, d, z);
      }
      s[0] += c < chunks(E) ? z : 0.f;
    }
    team_sum(s);
    const float r = 1.f / sqrtf(s[0] * inv + a.eps);
    T* const y = (T*)a.y + row * a.y_ss;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float o[V];
#pragma unroll
      for (int k = 0; k < V; ++k) o[k] = fmaf(v[i][k] * r, gamma[i][k], beta[i][k]);
      store_chunk<FULL>(y, t + TPR * i, E, o);
    }
    if (t == 0) {
      a.stats[2 * row] = mu;
      a.stats[2 * row + 1] = r;
    }
  }
}

// waves per SIMD that leave registers for a row, the next one and the columns' sums.  Without spills, but for rows of more than 8192 features with
// the weights' gradients: four chunks a thread of all that, at 256 registers, keep 28 to 140 bytes a lane in scratch memory (bf16; from packed
// features up to 244) or 168 to 232 (float32).  2048 rows, bf16: of 8192 features 24 us (4.1 TB/s), of 12288 34 (4.4), of 16384 46 (4.4);
// float32 38 (5.2), 96 (3.1), 127 (3.2).
constexpr int bwd_waves(int tpr, int nv, bool param) { return nv == 1 || (!param && nv == 2) ? 4 : tpr > WG || nv > 2 ? 2 : 3; }
// dx of the rows, and (PARAM) the part of dgamma and dbeta that these rows make: a thread adds up its own columns over all of
// its rows, the teams of a workgroup are joined in LDS, a workgroup writes one part.  The next row is on its way while one is
// worked on.
template <typename T, int SRC, bool FULL, int TPR, int NV, bool PARAM>
__global__ void __launch_bounds__(wg_of(TPR), bwd_waves(TPR, NV, PARAM)) norm_bwd_kernel(NormArgs a) {
  constexpr int TEAMS = wg_of(TPR) / TPR;
  __shared__ float sums[2][2][16];
  __shared__ float join[PARAM && TEAMS > 1 ? 2 * TPR * NV * V : 1];
  TeamSum<TPR> team_sum{sums};
  const int t = threadIdx.x % TPR, team = team_of<TPR>(), E = a.E;
  const float inv = 1.f / (float)a.E;
  struct Row {
    Chunk<T> x[SRC == 2 ? 1 : NV], dy[NV];
    PackedChunk p[SRC == 2 ? NV : 1];
    float mu, r;
  };
  auto load = [&](Row& w, long row) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + TPR * i;
      w.dy[i].template load<FULL>((const T*)a.dy + row * a.y_ss, c, E);
      if constexpr (SRC == 2) w.p[i].template load<FULL>(a.q + row * E, a.b + row * packed::groups(E), c, E);
      else w.x[i].template load<FULL>((const T*)a.x + row * a.x_ss, c, E);
    }
    w.mu = a.stats_in[2 * row];
    w.r = a.stats_in[2 * row + 1];
  };
  Chunk<T> gamma[NV];
  float pg[PARAM ? NV : 1][V], pb[PARAM ? NV : 1][V];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    gamma[i].template load<FULL>((const T*)a.gamma, t + TPR * i, E);
    if constexpr (PARAM) {
#pragma unroll
      for (int k = 0; k < V; ++k) pg[i][k] = pb[i][k] = 0.f;
    }
  }
  const long step = (long)gridDim.x * TEAMS;
  long row = (long)blockIdx.x * TEAMS + team;
  Row next;
  if (row < a.n) load(next, row);
  for (; row < a.n; row += step) {
    Row w = next;
    if (row + step < a.n) load(next, row + step);
    if constexpr (!FULL) {
#pragma unroll
      for (int i = 0; i < NV; ++i) w.dy[i].keep_from(skip_of<FULL>(t + TPR * i, E));
    }
    // (dy is 0 behind the row's end, and with it all that is summed)
    float s[2] = {0.f, 0.f};
    const float shift = -w.mu * w.r;
    const auto xh = [&](int i, int k) __attribute__((always_inline)) -> float {      // (made twice: kept, they cost more registers than time)
      if constexpr (SRC == 2) return fmaf(w.p[i][k], w.r * w.p[i].step(), shift);
      else return fmaf(w.x[i][k], w.r, shift);
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float x = xh(i, k), dy = w.dy[i][k], g = dy * gamma[i][k];
        s[0] += g;
        s[1] = fmaf(g, x, s[1]);
        if constexpr (PARAM) {
          pg[i][k] = fmaf(dy, x, pg[i][k]);
          pb[i][k] += dy;
        }
      }
    }
    if (a.dx) {                                      // (uniform)
      team_sum(s);
      const float m = a.rms ? 0.f : -s[0] * inv * w.r, mx = -s[1] * inv * w.r;
      T* const dx = (T*)a.dx + row * a.x_ss;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        float o[V];
#pragma unroll
        for (int k = 0; k < V; ++k) o[k] = fmaf(xh(i, k), mx, fmaf(w.dy[i][k] * gamma[i][k], w.r, m));
        store_chunk<FULL>(dx, t + TPR * i, E, o);
      }
    }
  }
  if constexpr (PARAM) {
    if constexpr (TEAMS > 1) {
      for (int k = 0; k < TEAMS; ++k) {
        if (team == k) {
#pragma unroll
          for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int u = 0; u < V; ++u) {
              float* const at = join + 2 * (t + TPR * (V * i + u));
              at[0] = pg[i][u] += k > 0 ? at[0] : 0.f;
              at[1] = pb[i][u] += k > 0 ? at[1] : 0.f;
            }
        }
        __syncthreads();
      }
      if (team != TEAMS - 1) return;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + TPR * i;
      float* const to = a.part + 2L * blockIdx.x * E;
      store_chunk<FULL>(to, c, E, pg[i]);
      store_chunk<FULL>(to + E, c, E, pb[i]);
    }
  }
}

// ---- packing by itself: a thread has 8 features, four chunks of a wave are in flight, a wave takes 2048 features of one row after
// the other ----

template <typename T, bool FULL>
__global__ void __launch_bounds__(WG) pack_kernel(NormArgs a) {
  const int E = a.E, ng = packed::groups(E), c0 = blockIdx.x * 256 + (threadIdx.x & 63);
  for (long row = (long)blockIdx.y * 4 + (threadIdx.x >> 6); row < a.n; row += (long)gridDim.y * 4) {
    Chunk<T> raw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[i].template load<FULL>((const T*)a.x + row * a.x_ss, c0 + 64 * i, E);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float v[V];
      if constexpr (!FULL) raw[i].keep_from(skip_of<FULL>(c0 + 64 * i, E));
      pack_chunk<FULL>(raw[i], v, a.q + row * E, a.b + row * ng, c0 + 64 * i, E);
    }
  }
}
template <typename T, bool FULL>
__global__ void __launch_bounds__(WG) unpack_kernel(NormArgs a) {
  const int E = a.E, ng = packed::groups(E), c0 = blockIdx.x * 256 + (threadIdx.x & 63);
  for (long row = (long)blockIdx.y * 4 + (threadIdx.x >> 6); row < a.n; row += (long)gridDim.y * 4) {
    PackedChunk raw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[i].template load<FULL>(a.q + row * E, a.b + row * ng, c0 + 64 * i, E);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float v[V];
#pragma unroll
      for (int k = 0; k < V; ++k) v[k] = raw[i][k] * raw[i].step();
      store_chunk<FULL>((T*)a.y + row * a.y_ss, c0 + 64 * i, E, v);
    }
  }
}

// ... rows of fewer than 8 features: one group each, 32 lanes
template <typename T>
__global__ void __launch_bounds__(WG) pack_narrow_kernel(NormArgs a, bool back) {
  const int E = a.E, e = threadIdx.x % 32;
  for (long row = (long)blockIdx.x * (WG / 32) + threadIdx.x / 32; row < a.n; row += (long)gridDim.x * (WG / 32)) {
    if (!back) {
      norm_in<T, 1>((const T*)a.x + row * a.x_ss, a.q + row * E, a.b + row, e, E, true);
    } else if (e < E) {
      ((T*)a.y + row * a.y_ss)[e] = (T)norm_in<T, 2>((const T*)nullptr, a.q + row * E, a.b + row, e, E, false);
    }
  }
}

unsigned grid_of(long n, long most) { return (unsigned)(n < most ? n : most); }

template <typename T, bool FULL, int TPR, int NV> void fwd_rows(const NormArgs& a, hipStream_t s) {
  constexpr int W = wg_of(TPR);
  const unsigned grid = grid_of((a.n + W / TPR - 1) / (W / TPR), 8L * a.n_cu);
  if (a.x && a.q) norm_fwd_kernel<T, 1, FULL, TPR, NV><<<grid, W, 0, s>>>(a);
  else if (a.q) norm_fwd_kernel<T, 2, FULL, TPR, NV><<<grid, W, 0, s>>>(a);
  else norm_fwd_kernel<T, 0, FULL, TPR, NV><<<grid, W, 0, s>>>(a);
}
template <typename T, bool FULL, int TPR, int NV> void bwd_rows(const NormArgs& a, hipStream_t s) {
  constexpr int W = wg_of(TPR);
  if (a.dgamma || a.dbeta) {
    if (a.q) norm_bwd_kernel<T, 2, FULL, TPR, NV, true><<<(unsigned)a.parts, W, 0, s>>>(a);
    else norm_bwd_kernel<T, 0, FULL, TPR, NV, true><<<(unsigned)a.parts, W, 0, s>>>(a);
    norm_param_sum_kernel<<<(unsigned)((2L * a.E + 31) / 32), WG, 0, s>>>(a);
    return;
  }
  const unsigned grid = grid_of((a.n + W / TPR - 1) / (W / TPR), 8L * a.n_cu);
  if (a.q) norm_bwd_kernel<T, 2, FULL, TPR, NV, false><<<grid, W, 0, s>>>(a);
  else norm_bwd_kernel<T, 0, FULL, TPR, NV, false><<<grid, W, 0, s>>>(a);
}

// by the width alone (see above)
template <typename T, bool FULL> hipError_t fwd(const NormArgs& a, hipStream_t s) {
  const int E = a.E;
  if (E < V || E > 16384) {
    const unsigned grid = grid_of(a.n, 16L * a.n_cu);
    if (a.x && a.q) norm_fwd_any_kernel<T, 1><<<grid, WG, 0, s>>>(a);
    else if (a.q) norm_fwd_any_kernel<T, 2><<<grid, WG, 0, s>>>(a);
    else norm_fwd_any_kernel<T, 0><<<grid, WG, 0, s>>>(a);
  } else if (E <= 512) fwd_rows<T, FULL, 64, 1>(a, s);
  else if (E <= 1024) fwd_rows<T, FULL, 64, 2>(a, s);
  else if (E <= 1536 && sizeof(T) == 2) fwd_rows<T, FULL, 64, 3>(a, s);       // (7290 x 1152 10.3 -> 8.5 us; float32 12.1 -> 13.0)
  else if (E <= 2048) fwd_rows<T, FULL, 256, 1>(a, s);
  else if (E <= 4096) fwd_rows<T, FULL, 256, 2>(a, s);
  else if (E <= 8192) fwd_rows<T, FULL, 512, 2>(a, s);
  else fwd_rows<T, FULL, 1024, 2>(a, s);
  return hipGetLastError();
}
template <typename T, bool FULL> hipError_t bwd(const NormArgs& a, hipStream_t s) {
  const int E = a.E;
  if (E < V || E > 16384) {
    // (the sums over the rows first: dx may lie where dy does)
    if (a.dgamma || a.dbeta) {
      const dim3 grid((unsigned)((a.E + WG - 1) / WG), (unsigned)a.parts);
      if (a.q) norm_param_any_kernel<T, 2><<<grid, WG, 0, s>>>(a);
      else norm_param_any_kernel<T, 0><<<grid, WG, 0, s>>>(a);
      norm_param_sum_kernel<<<(unsigned)((2L * a.E + 31) / 32), WG, 0, s>>>(a);
    }
    if (a.dx) {
      const unsigned grid = grid_of(a.n, 16L * a.n_cu);
      if (a.q) norm_bwd_any_kernel<T, 2><<<grid, WG, 0, s>>>(a);
      else norm_bwd_any_kernel<T, 0><<<grid, WG, 0, s>>>(a);
    }
  } else if (E <= 512) bwd_rows<T, FULL, 64, 1>(a, s);
  else if (E <= 1024) bwd_rows<T, FULL, 64, 2>(a, s);
  else if (E <= 2048) bwd_rows<T, FULL, 256, 1>(a, s);
  else if (E <= 4096) bwd_rows<T, FULL, 256, 2>(a, s);
  else if (E <= 8192) bwd_rows<T, FULL, 512, 2>(a, s);
  else bwd_rows<T, FULL, 512, 4>(a, s);
  return hipGetLastError();
}
// f(an element, whether E is a multiple of 8)
template <class F> hipError_t by_type(const NormArgs& a, int is_f32, F&& f) {
  using yes = std::true_type;
  using no = std::false_type;
  if (a.E % V == 0) return is_f32 ? f(0.f, yes{}) : f(__bf16{}, yes{});
  return is_f32 ? f(0.f, no{}) : f(__bf16{}, no{});
}
}  // namespace

int norm_parts(long n, int E) {
  (void)E;
  const long parts = (n + 7) / 8, most = 2L * device_cu_count();
  return (int)(parts < most ? parts : most);
}
hipError_t launch_norm_fwd(const NormArgs& a, int is_f32, hipStream_t s) {
  return by_type(a, is_f32, [&](auto t, auto full) { return fwd<decltype(t), decltype(full)::value>(a, s); });
}
hipError_t launch_norm_bwd(const NormArgs& a, int is_f32, hipStream_t s) {
  return by_type(a, is_f32, [&](auto t, auto full) { return bwd<decltype(t), decltype(full)::value>(a, s); });
}
hipError_t launch_pack(const NormArgs& a, int is_f32, hipStream_t s) {
  const dim3 grid((unsigned)((a.E + 2047) / 2048), grid_of((a.n + 3) / 4, 16384));
  return by_type(a, is_f32, [&](auto t, auto full) {
    using E = decltype(t);
    if (a.E < V) pack_narrow_kernel<E><<<grid_of((a.n + 7) / 8, 16384), WG, 0, s>>>(a, false);
    else pack_kernel<E, decltype(full)::value><<<grid, WG, 0, s>>>(a);
    return hipGetLastError();
  });
}
hipError_t launch_unpack(const NormArgs& a, int is_f32, hipStream_t s) {
  const dim3 grid((unsigned)((a.E + 2047) / 2048), grid_of((a.n + 3) / 4, 16384));
  return by_type(a, is_f32, [&](auto t, auto full) {
    using E = decltype(t);
    if (a.E < V) pack_narrow_kernel<E><<<grid_of((a.n + 7) / 8, 16384), WG, 0, s>>>(a, true);
    else unpack_kernel<E, decltype(full)::value><<<grid, WG, 0, s>>>(a);
    return hipGetLastError();
  });
}

}  // namespace lvx
