// Distillation from a teacher's top logits: the divergence of softmax(x w^T / T) from the softmax of K known logits a token, without keeping
// z = x w^T (the products and their tiles: lvx_xent_kernels.h).
//
//   loss_i = sum_k q_k (ln q_k - z_ik / T + lse_i),   lse_i = ln sum_v exp(z_iv / T)
//   g_iv = (exp(z_iv / T - lse_i) - sum over k with id_ik = v of q_k) d_loss_i / T,   dx = g w,   dw = g^T x
//
// What differs from the cross entropy is that a token has K logits to be handed out instead of one.  A launch sorts every listed token's ids
// and counts those below every multiple of 64, so that a tile's epilogue finds the ones among its columns with one lookup a row, and
// leaves their logits in their order (few tokens' few entries stay where they are: direct_of).  The gradient's tiles write exp(z / T - lse) d_loss / T everywhere; at the teacher's entries another launch
// puts exp(ln p) - q in its place, from the ln p of the forward pass, with one rounding like everywhere else: n K values beside the n V.
// (To bf16, which the matrix cores take: dx and dw of 2048 x 4096 against 32768 with 64 entries are off by 0.0023 of their size, by 0.0017 from their own rounding.)
#include "lvx_xent_kernels.h"

namespace lvx {

namespace {

// K entries in LDS, rounded up to four
constexpr int NO_KEY = 0x7ffffffe;
__host__ __device__ constexpr int entries_up(int K) { return (K + 3) / 4 * 4; }
// A token's entries in the order of their ids, as row `row` of what the tiles look them up in, by a workgroup.  keys: filled in by it, NO_KEY behind the last one.
__device__ __forceinline__ void sort_entries(const XentArgs& a, long row, const int* keys, int* sorted) {
  const int tid = threadIdx.x, K = a.K, K4 = entries_up(K);
  __syncthreads();
  for (int k = tid; k < K4; k += 256) {
    const int mine = keys[k];
    int r = 0;
#pragma unroll 4
    for (int j = 0; j < K4; j += 4) {
      const int4 y = *(const int4*)(keys + j);
      const auto before = [&](int y, int j) { return y < mine + (j < k ? 1 : 0) ? 1 : 0; };      // (equal ids: in the order of the entries)
      r += before(y.x, j) + before(y.y, j + 1) + before(y.z, j + 2) + before(y.w, j + 3);
    }
    sorted[r] = mine;                                // (those behind K stay there)
    if (k < K) {
      a.sorted[row * K + r] = mine;
      a.rank[row * K + k] = (uint16_t)r;
    }
  }
  __syncthreads();
  // how many are below 64 b, two b of a thread at a time: steps of powers of two
  int most = 1;
  while (2 * most <= K) most *= 2;
  uint16_t* const starts = a.starts + row * (a.blocks + 1);
  const auto below = [&](auto many, int b0) {
    int at[decltype(many)::value] = {};
    for (int step = most; step > 0; step /= 2)
#pragma unroll
      for (int i = 0; i < decltype(many)::value; ++i) {
        const int to = at[i] + step;
        if (to <= K && sorted[min(to, K) - 1] < 64 * (b0 + 256 * i)) at[i] = to;
      }
#pragma unroll
    for (int i = 0; i < decltype(many)::value; ++i)
      if (b0 + 256 * i <= a.blocks) starts[b0 + 256 * i] = (uint16_t)at[i];
  };
  for (int b0 = tid; b0 < a.blocks; b0 += 2 * 256) below(std::integral_constant<int, 2>{}, b0);
  if (tid == 255) below(std::integral_constant<int, 1>{}, a.blocks);
  __syncthreads();
}
__device__ __forceinline__ int key_of(const XentArgs& a, long id) { return id >= 0 && id < a.V ? (int)id : NO_KEY; }

// A wave a token: whether it takes part (a.labels: 0, -1 if not, V if an id is outside), and the sum of its exponentials.  SORT: and its ids in order, by a workgroup
// a token, whose waves do the rest four times.
template <bool SORT> __global__ void __launch_bounds__(256) distil_prepare_kernel(XentArgs a, bool forward) {
  extern __shared__ __attribute__((aligned(16))) int prepare_mem[];
  constexpr int TOKENS = SORT ? 1 : 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, K = a.K;
  int* const keys = prepare_mem;
  for (long base = blockIdx.x * (long)TOKENS; base < a.n; base += gridDim.x * (long)TOKENS) {
    const long i = SORT ? base : min(base + wave, a.n - 1);      // (the last token again: the same results)
    float top = -__builtin_inff();
    bool any = false, far = false;
    for (int k = lane; k < K; k += 64) {
      const Entry e = entry_of(a, i, k);
      any |= e.there && !(e.t == -__builtin_inff());
      far |= e.there && e.id >= a.V;
      if (e.there) top = fmaxf(top, e.t);            // (a NaN is dropped here and comes back in the sum)
      if (SORT && wave == 0) keys[k] = key_of(a, e.id);
    }
    any = __any(any);
    far = __any(far);
#pragma unroll
    for (int o = 1; o < 64; o *= 2) top = fmaxf(top, __shfl_xor(top, o));
    float sum = 0.f;
    for (int k = lane; k < K; k += 64) {
      const Entry e = entry_of(a, i, k);
      sum += e.there ? expf(apart(a, e.t, top)) : 0.f;
      if (forward && !any) a.ln_p[i * K + k] = 0.f;
    }
#pragma unroll
    for (int o = 1; o < 64; o *= 2) sum += __shfl_xor(sum, o);
    if (lane == 0) {
      ((int64_t*)a.labels)[i] = label_of(any, far, a.V);
      a.q_stat[i] = make_float2(top, logf(sum));
    }
    if constexpr (SORT) {
      if (wave == 0 && lane < 3 && K + lane < entries_up(K)) keys[K + lane] = NO_KEY;
      sort_entries(a, i, keys, keys + entries_up(K));
    }
  }
}
// stat by lanes that share its entries: `lane` of W of them
template <int W> __device__ __forceinline__ float2 stat_of(const XentArgs& a, long tok, int lane) {
  float top = -__builtin_inff(), sum = 0.f;
  for (int k = lane; k < a.K; k += W) {
    const Entry e = entry_of(a, tok, k);
    if (e.there) top = fmaxf(top, e.t);
  }
#pragma unroll
  for (int o = 1; o < W; o *= 2) top = fmaxf(top, __shfl_xor(top, o));
  for (int k = lane; k < a.K; k += W) {
    const Entry e = entry_of(a, tok, k);
    sum += e.there ? expf(apart(a, e.t, top)) : 0.f;
  }
#pragma unroll
  for (int o = 1; o < W; o *= 2) sum += __shfl_xor(sum, o);
  return make_float2(top, logf(sum));
}
// The first two launches of a pass in one, for up to LISTED tokens of few entries: a thread a token, then the list of those that take part
// (xent_list_kernel).  It saves a launch, twice with gradients, but one workgroup's loads have no others beside them (with gradients of n x 512 against 2048,
// two launches and one: 128 with 4 entries 61.6 -> 57.0 us, with 16 63.4 -> 63.9; 512 with 8 74.9 -> 73.9; 768 with 8 79.0 -> 80.1; 1024 with 6 83.3 -> 81.0,
// with 8 83.4 -> 86.7).  (Of these 768 with 8 is within the bound.)
constexpr int LISTED = 1024, LISTED_ENTRIES = 8, LISTED_IN_ALL = 6144;
__global__ void __launch_bounds__(LISTED) distil_list_kernel(XentArgs a, bool forward) {
  __shared__ int counts[16];
  __shared__ float tops[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, K = a.K;
  const long i = min((long)tid, a.n - 1);
  const bool there = tid < a.n;
  float top = -__builtin_inff(), sum = 0.f;
  bool any = false, far = false;
  for (int k0 = 0; k0 < K; k0 += 8) {
    Entry e[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      e[k] = entry_of(a, i, min(k0 + k, K - 1));
      e[k].there &= k0 + k < K;
    }
    // (the sum goes along with the largest so far; one that is still -infinity has none)
    float most = top;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      any |= e[k].there && !(e[k].t == -__builtin_inff());
      far |= e[k].there && e[k].id >= a.V;
      if (e[k].there) most = fmaxf(most, e[k].t);
    }
    sum = top == most || top == -__builtin_inff() ? sum : sum * expf(apart(a, top, most));
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += e[k].there && (most != -__builtin_inff() || e[k].t != most) ? expf(apart(a, e[k].t, most)) : 0.f;
    top = most;
  }
  const long label = there ? label_of(any, far, a.V) : -1;
  const float d = a.d_loss && label >= 0 ? a.d_loss[i] * a.inv_t : 0.f, lse = a.d_loss && label >= 0 ? a.lse[i] : 0.f;
  if (there) {
    ((int64_t*)a.labels)[i] = label;
    a.q_stat[i] = make_float2(top, logf(sum));
  }
  const unsigned long long on = __ballot(label >= 0);
  float largest = fabsf(d) < __builtin_inff() ? fabsf(d) : 0.f;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) largest = fmaxf(largest, __shfl_xor(largest, o));
  if (lane == 0) {
    counts[wave] = __popcll(on);
    tops[wave] = largest;
  }
  __syncthreads();
  int at = __popcll(on & ((1ull << lane) - 1)), total = 0;
#pragma unroll
  for (int w = 0; w < 16; ++w) {
    const int c = counts[w];
    at += w < wave ? c : 0;
    total += c;
    largest = fmaxf(largest, tops[w]);
  }
  if (label >= 0) {
    a.tok[at] = (int)i;
    a.lab[at] = label < a.V ? (int)label : -1;
    if (a.d_loss) a.row[at] = make_float2(lse * LOG2E, label < a.V ? d : __builtin_nanf(""));
  } else if (forward && there) {
    a.loss[i] = 0.f;
    a.lse_out[i] = 0.f;
    for (int k = 0; k < K; ++k) a.ln_p[i * K + k] = 0.f;
  }
  const int parts = dx_parts((total + a.tile_rows - 1) / a.tile_rows * ((a.E + a.tile - 1) / a.tile), (int)(a.piece / BK), a.n_cu, a.slots);
  const int dw_parts = a.dw_slots > 0 ? dx_parts(a.dw_tiles, (total + BK - 1) / BK, a.n_cu, a.dw_slots) : 1;
  if (tid != 0) return;
  a.head->count = total;
  a.head->scale = largest > 0.f ? largest : 1.f;
  a.head->parts = parts;
  a.head->dw_parts = dw_parts;
}
// The listed tokens' ids in order
__global__ void __launch_bounds__(256) distil_sort_kernel(XentArgs a) {
  extern __shared__ __attribute__((aligned(16))) int prepare_mem[];
  const int K = a.K, count = a.head->count;
  int* const keys = prepare_mem;
  for (int r = blockIdx.x; r < count; r += gridDim.x) {
    const long tok = a.tok[r];
    for (int k = threadIdx.x; k < entries_up(K); k += 256) keys[k] = k < K ? key_of(a, a.ids[tok * K + k]) : NO_KEY;
    sort_entries(a, r, keys, keys + entries_up(K));
  }
}

// lse, loss and ln p of the listed tokens from what the tiles left: 8 tokens a workgroup, 32 threads each
__global__ void __launch_bounds__(256) distil_join_kernel(XentArgs a, int n_parts) {
  __shared__ float sm[8][33], ss[8][33], lses[8];
  const int row_l = threadIdx.x % 8, lane = threadIdx.x / 8;
  const Own own = a.own ? own_list<TEACHER>(a) : Own{};
  const int count = a.own ? own.count : a.head->count;
  if (a.own && blockIdx.x == 0 && (int)threadIdx.x >= count && threadIdx.x < a.n) {        // (the tokens that are not listed)
    a.loss[own.tok] = 0.f;
    a.lse_out[own.tok] = 0.f;
    if (a.direct)
      for (int k = 0; k < a.K; ++k) a.ln_p[(long)own.tok * a.K + k] = 0.f;
  }
  for (int r0 = blockIdx.x * 8; r0 < count; r0 += gridDim.x * 8) {
    const int r = min(r0 + row_l, count - 1);
    float m = -__builtin_inff(), s = 0.f;
    for (int p0 = lane; p0 < n_parts; p0 += 32 * 8) {
      float2 v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = a.part[(long)min(p0 + 32 * i, n_parts - 1) * a.Mp + r];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (p0 + 32 * i < n_parts) join_stats(&m, &s, v[i].x, v[i].y);
    }
    sm[row_l][lane] = m;
    ss[row_l][lane] = s;
    __syncthreads();
    if (threadIdx.x < 8) {
      m = -__builtin_inff();
      s = 0.f;
      for (int i = 0; i < 32; ++i) join_stats(&m, &s, sm[threadIdx.x][i], ss[threadIdx.x][i]);
      lses[threadIdx.x] = (m + __builtin_amdgcn_logf(s)) * LN2;
    }
    __syncthreads();
    const int mine = threadIdx.x / 32, r1 = r0 + mine;
    const int listed = min(r1, count - 1), tok = a.own ? __shfl(own.tok, listed) : a.tok[listed];
    const int lab = a.own ? __shfl(own.lab, listed) : a.lab[listed];
    if (r1 < count) {
      const float lse = lab >= 0 ? lses[mine] : __builtin_nanf("");
      const float2 stat = a.own && a.direct ? stat_of<32>(a, tok, threadIdx.x % 32) : a.q_stat[tok];
      const long row = a.own || a.direct ? tok : r1; // among the entries
      float loss = 0.f;
      for (int k = threadIdx.x % 32; k < a.K; k += 32) {
        const Entry e = entry_of(a, tok, k);
        const float z = e.there && e.id < a.V ? a.z_entry[row * a.K + (a.direct ? k : a.rank[row * a.K + k])] : __builtin_nanf("");
        const float ln_p = z * a.inv_t - lse, ln_q = ln_q_of(a, e, stat), q = expf(ln_q);
        a.ln_p[(long)tok * a.K + k] = e.there ? ln_p : 0.f;
        loss += !e.there || q == 0.f ? 0.f : q * (ln_q - ln_p);
      }
#pragma unroll
      for (int o = 1; o < 32; o *= 2) loss += __shfl_xor(loss, o);
      if (threadIdx.x % 32 == 0) {
        a.loss[tok] = loss + 0.f * lse;              // (NaN where an id is outside, also if no entry counts)
        a.lse_out[tok] = lse;
      }
    }
    __syncthreads();
  }
}

// g at the teacher's entries of a piece of the vocabulary: a wave a token
template <typename G> __global__ void __launch_bounds__(256) distil_entries_kernel(XentArgs a) {
  extern __shared__ __attribute__((aligned(16))) int entries_mem[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, K = a.K, count = a.head->count;
  int2* const known = (int2*)entries_mem + wave * entries_up(K);      // id and q
  const float scale = a.head->scale;
  for (int base = blockIdx.x * 4; base < count; base += gridDim.x * 4) {
    const int r = min(base + wave, count - 1);
    const long tok = a.tok[r];
    const float2 stat = a.q_stat[tok];
    const float d = (a.labels[tok] < a.V ? a.d_loss[tok] * a.inv_t : __builtin_nanf("")) / scale;
    __syncthreads();
    for (int k = lane; k < entries_up(K); k += 64) {
      int2 y = {-1, 0};
      if (k < K) {
        const Entry e = entry_of(a, tok, k);
        y = {e.there && e.id < a.V ? (int)e.id : -1, __float_as_int(expf(ln_q_of(a, e, stat)))};
      }
      known[k] = y;
    }
    __syncthreads();
    for (int k = lane; k < K; k += 64) {
      const int id = known[k].x;
      const float p = exp2_fast(a.ln_p[tok * K + k] * LOG2E);
      float q = 0.f;                                 // (every entry of an id writes the same)
#pragma unroll 4
      for (int j = 0; j < entries_up(K); j += 2) {
        const int4 y = *(const int4*)(known + j);
        q += y.x == id ? __int_as_float(y.y) : 0.f;
        q += y.z == id ? __int_as_float(y.w) : 0.f;
      }
      if (id >= a.v0 && id < a.v1) ((G*)a.g)[r * a.g_pitch + (id - a.v0)] = (G)(d != 0.f ? (p - q) * d : 0.f);
    }
  }
}

unsigned waves_for(long n) { return (unsigned)std::min(up(n, 4), 1L << 16); }
unsigned groups_for(long n) { return (unsigned)std::min(n, 1L << 16); }
int entries_lds(const XentArgs& a, int tokens) { return tokens * 2 * entries_up(a.K) * (int)sizeof(int); }
// Whether the launch on `cols` entries of the vocabulary looks at the teacher's entries where they stand (DIRECT_ENTRIES; xent_bf16_kernel does not)
// Of more than 64 tokens it saves the launches of the sort and of g's entries: 128 x 320 against 4096 with one entry 55.8 -> 52.2 us, with 8 57.7 -> 56.9; 300 x 512
// float32 against 5003 with 8 123.8 -> 119.3; 1000 x 128 against 2000 with 4 74.4 -> 69.7, with 8 77.3 -> 75.9; 256 x 1088 against 1024 with 4 72.9 -> 71.2, with 8 74.9 -> 76.1 (within the bound).
bool direct_of(const XentArgs& a, int is_f32, long cols) {
  if (a.K > DIRECT_ENTRIES || a.K * a.V > DIRECT_IN_ALL || a.K * a.V * std::max(a.n, 64L) > 64 * DIRECT_IN_ALL) return false;
  return is_f32 || a.n <= 64 || few_rows(a.n, cols, a.E / BK, a.n_cu) > 0;
}
hipError_t gradient(const XentArgs& all, int is_f32, hipStream_t s) {
  XentArgs a = all;
  a.direct = direct_of(a, is_f32, a.v1 - a.v0);
  const hipError_t e = logits<GRAD, TEACHER>(a, is_f32, s);
  if (e != hipSuccess || a.direct) return e;
  if (is_f32) distil_entries_kernel<float><<<waves_for(a.n), 256, entries_lds(a, 4), s>>>(a);
  else distil_entries_kernel<__bf16><<<waves_for(a.n), 256, entries_lds(a, 4), s>>>(a);
  return hipGetLastError();
}

}  // namespace

// The list of a pass with more tokens than that, and what belongs to each
template <bool FORWARD> static hipError_t list(const XentArgs& a, hipStream_t s) {
  if (a.n <= LISTED && a.K <= LISTED_ENTRIES && a.n * a.K <= LISTED_IN_ALL) {
    distil_list_kernel<<<1, LISTED, 0, s>>>(a, FORWARD);
    return hipGetLastError();
  }
  distil_prepare_kernel<false><<<waves_for(a.n), 256, 0, s>>>(a, FORWARD);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : launch_xent_list(a, s);
}

hipError_t launch_distil_fwd(XentArgs a, int is_f32, hipStream_t s) {
  xent_fwd_sizes(&a, is_f32);
  a.direct = direct_of(a, is_f32, a.V);
  if (a.own && !a.direct) {
    distil_prepare_kernel<true><<<groups_for(a.n), 256, entries_lds(a, 1), s>>>(a, true);
  } else if (!a.own) {
    const hipError_t e = list<true>(a, s);
    if (e != hipSuccess) return e;
    if (!a.direct) distil_sort_kernel<<<groups_for(a.n), 256, entries_lds(a, 1), s>>>(a);
  }
  hipError_t e = hipGetLastError();
  if (e == hipSuccess) e = logits<STATS, TEACHER>(a, is_f32, s);
  if (e != hipSuccess) return e;
  distil_join_kernel<<<(unsigned)std::min(up(a.n, 8), 4096L), 256, 0, s>>>(a, stat_parts_of(a, is_f32));
  return hipGetLastError();
}

hipError_t launch_distil_bwd(XentArgs a, int is_f32, hipStream_t s) {
  if (own_of(a.n, is_f32) && !direct_of(a, is_f32, a.V)) {
    distil_prepare_kernel<false><<<waves_for(a.n), 256, 0, s>>>(a, false);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return launch_xent_products(a, is_f32, s, list<false>, gradient);
}

}  // namespace lvx
