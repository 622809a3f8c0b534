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

namespace lvx {

namespace {

constexpr int WG = 256;

__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const __bf16* p) { return (float)*p; }

template <int W> __device__ __forceinline__ float lanes_sum(float x) {
#pragma unroll
  for (int o = 1; o < W; o *= 2) x += __shfl_xor(x, o);
  return x;
}
template <int W> __device__ __forceinline__ unsigned lanes_max(unsigned x) {
#pragma unroll
  for (int o = 1; o < W; o *= 2) {
    const unsigned y = (unsigned)__shfl_xor((int)x, o);
    x = x > y ? x : y;
  }
  return x;
}
// over the workgroup, the same in every thread (`at`: 4 floats of LDS that no wave still reads)
__device__ __forceinline__ float wg_sum(float x, float* at) {
  x = lanes_sum<64>(x);
  if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = x;
  __syncthreads();
  return (at[0] + at[1]) + (at[2] + at[3]);
}

// ---- any width: a workgroup per row, an element per thread, the row read again for every sum ----

// Element e of a row as the norm sees it (any e of a group of 32 lanes that asks for a group, E and more: 0).
// SRC 0: x.  1: the packed form of x (which is written where `keep` says so).  2: what was packed before.
template <typename T, int SRC>
__device__ __forceinline__ float norm_in(const T* x, int8_t* q, uint8_t* b, int e, int E, bool keep) {
  if constexpr (SRC == 0) return e < E ? load1(x + e) : 0.f;
  if constexpr (SRC == 2) return e < E ? (float)q[e] * packed::step_of(b[e / packed::GROUP]) : 0.f;
  const float v = e < E ? load1(x + e) : 0.f;
  const unsigned byte = packed::exponent_of(lanes_max<32>(packed::magnitude(v)));
  const float s = packed::steps(byte == 255u ? 0.f : v, packed::inverse_step_of(byte));
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
      s += e < E ? d * d : 0.f;
    }
    const float r = 1.f / sqrtf(wg_sum(s, sums[1]) * inv + a.eps);
    for (int e = tid; e < E32; e += WG) {
      const float v = norm_in<T, SRC>(x, q, b, e, E, true);
      if (e < E) {
        const float yv = (v - mu) * r * load1((const T*)a.gamma + e);
        y[e] = (T)(a.beta ? yv + load1((const T*)a.beta + e) : yv);
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
      sx += g * ((norm_in<T, SRC>(x, q, b, e, E, false) - mu) * r);
    }
    __syncthreads();
    s = a.rms ? 0.f : wg_sum(s, sums[0]) * inv;
    sx = wg_sum(sx, sums[1]) * inv;
    for (int e = tid; e < E; e += WG) {
      const float g = load1(dy + e) * load1((const T*)a.gamma + e);
      const float xh = (norm_in<T, SRC>(x, q, b, e, E, false) - mu) * r;
      dx[e] = (T)(r * (g - s - xh * sx));
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
    sg += dy * xh;
    sb += dy;
  }
  a.part[(2L * blockIdx.y) * E + e] = sg;
  a.part[(2L * blockIdx.y + 1) * E + e] = sb;
}

// dgamma += the parts' sums, dbeta likewise, in a fixed order: 16 threads share a column
__global__ void __launch_bounds__(WG) norm_param_sum_kernel(NormArgs a) {
  __shared__ float sums[16][17];
  const long at = (long)blockIdx.x * 16 + threadIdx.x % 16;      // dgamma's columns, then dbeta's
  const int lane = threadIdx.x / 16;
  float s = 0.f;
  if (at < 2L * a.E)
    for (int p = lane; p < a.parts; p += 16) s += a.part[2L * p * a.E + at];
  sums[lane][threadIdx.x % 16] = s;
  __syncthreads();
  if (threadIdx.x >= 16 || at >= 2L * a.E) return;
  s = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) s += sums[i][threadIdx.x];
  float* const to = at < a.E ? a.dgamma : a.dbeta;
  if (to) to[at < a.E ? at : at - a.E] += s;
}

// ---- packing by itself ----

// 32 lanes per group of a row, any width and alignment
template <typename T>
__global__ void __launch_bounds__(WG) pack_any_kernel(NormArgs a) {
  const int E = a.E, ng = packed::groups(E), l = threadIdx.x % 32;
  const long total = a.n * ng;
  for (long g = (long)blockIdx.x * (WG / 32) + threadIdx.x / 32; g < total; g += (long)gridDim.x * (WG / 32)) {
    const long row = g / ng;
    const int e = (int)(g % ng) * 32 + l;
    norm_in<T, 1>((const T*)a.x + row * a.x_ss, a.q + row * E, a.b + row * ng, e, E, true);
  }
}
template <typename T>
__global__ void __launch_bounds__(WG) unpack_any_kernel(NormArgs a) {
  const int E = a.E, ng = packed::groups(E), l = threadIdx.x % 32;
  const long total = a.n * ng;
  for (long g = (long)blockIdx.x * (WG / 32) + threadIdx.x / 32; g < total; g += (long)gridDim.x * (WG / 32)) {
    const long row = g / ng;
    const int e = (int)(g % ng) * 32 + l;
    const float v = norm_in<T, 2>((const T*)nullptr, a.q + row * E, a.b + row * ng, e, E, false);
    if (e < E) ((T*)a.y + row * a.y_ss)[e] = (T)v;
  }
}

unsigned grid_of(long n, long most) { return (unsigned)(n < most ? n : most); }

template <typename T> hipError_t fwd(const NormArgs& a, hipStream_t s) {
  const unsigned grid = grid_of(a.n, 16L * a.n_cu);
  if (a.x && a.q) norm_fwd_any_kernel<T, 1><<<grid, WG, 0, s>>>(a);
  else if (a.q) norm_fwd_any_kernel<T, 2><<<grid, WG, 0, s>>>(a);
  else norm_fwd_any_kernel<T, 0><<<grid, WG, 0, s>>>(a);
  return hipGetLastError();
}
template <typename T> hipError_t bwd(const NormArgs& a, hipStream_t s) {
  // (the sums over the rows first: dx may lie where dy does)
  if (a.dgamma || a.dbeta) {
    const dim3 grid((unsigned)((a.E + WG - 1) / WG), (unsigned)a.parts);
    if (a.q) norm_param_any_kernel<T, 2><<<grid, WG, 0, s>>>(a);
    else norm_param_any_kernel<T, 0><<<grid, WG, 0, s>>>(a);
    norm_param_sum_kernel<<<(unsigned)((2L * a.E + 15) / 16), WG, 0, s>>>(a);
  }
  if (a.dx) {
    const unsigned grid = grid_of(a.n, 16L * a.n_cu);
    if (a.q) norm_bwd_any_kernel<T, 2><<<grid, WG, 0, s>>>(a);
    else norm_bwd_any_kernel<T, 0><<<grid, WG, 0, s>>>(a);
  }
  return hipGetLastError();
}
}  // namespace

int norm_parts(long n, int E) {
  (void)E;
  const long parts = (n + 15) / 16;
  return (int)(parts < 256 ? parts : 256);
}
hipError_t launch_norm_fwd(const NormArgs& a, int is_f32, hipStream_t s) { return is_f32 ? fwd<float>(a, s) : fwd<__bf16>(a, s); }
hipError_t launch_norm_bwd(const NormArgs& a, int is_f32, hipStream_t s) { return is_f32 ? bwd<float>(a, s) : bwd<__bf16>(a, s); }
hipError_t launch_pack(const NormArgs& a, int is_f32, hipStream_t s) {
  const unsigned grid = grid_of((a.n * packed::groups(a.E) + 7) / 8, 32L * a.n_cu);
  if (is_f32) pack_any_kernel<float><<<grid, WG, 0, s>>>(a);
  else pack_any_kernel<__bf16><<<grid, WG, 0, s>>>(a);
  return hipGetLastError();
}
hipError_t launch_unpack(const NormArgs& a, int is_f32, hipStream_t s) {
  const unsigned grid = grid_of((a.n * packed::groups(a.E) + 7) / 8, 32L * a.n_cu);
  if (is_f32) unpack_any_kernel<float><<<grid, WG, 0, s>>>(a);
  else unpack_any_kernel<__bf16><<<grid, WG, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace lvx
