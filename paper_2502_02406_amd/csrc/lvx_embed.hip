// Rows of a table for token ids, scaled, and the table's gradient:
//
//   y_i = scale table[id_i],   d_table[v] = (what is there) + scale sum over i with id_i = v of d_y_i
//
// Both are bound by memory.  Forward: a team of threads for a row, 8 elements each.  Backward: the tokens are sorted by id, equal ids in the
// order of the tokens (a stable sort by digits), and sums run over chunks of the sorted tokens: an id that a chunk has for itself is
// finished there, one that goes on in the next chunk leaves a float32 sum a chunk, which a last launch adds up in the order of the
// chunks.  However often an id occurs, its rows are shared by as many workgroups as there are chunks.  No float atomics: results repeat bit for bit.
#include "lvx_internal.h"
#include "lvx_mfma.h"

#include <algorithm>
#include <type_traits>

namespace lvx {

namespace {

constexpr int V8 = 8;                  // elements a thread takes of a row
typedef u32x4 __attribute__((aligned(2))) u32x4_any2;
typedef u32x4 __attribute__((aligned(4))) u32x4_any4;
constexpr int chunks8(int E) { return (E + V8 - 1) / V8; }
// Threads of a team (a power of two, 256 at most): as many as a row has pieces of 8 elements.
int team_log(int E) {
  int l = 0;
  while (l < 8 && (1 << l) < chunks8(E)) ++l;
  return l;
}

// 16 bytes to memory, PAST the caches: y, and cleared rows that are whole lines (both of 2048 x 4096 bf16, table 32768: 78 -> 70 us
// forward and backward, of 65536 x 4096, table 131072: 522 -> 499).  Of rows that begin anywhere, y: 65536 x 4090, table 50021, forward 203 -> 143 us, with the backward
// pass 458 -> 410, 200000 x 333 59 -> 41, 5514 x 1001 floats 9.3 -> 10.0, with the backward pass 74.7 -> 73.8; but clears of them, the last of these: 74 -> 96.
// A small y that the next launch reads comes from memory then.  Lookup and the norm behind it, through the caches and past them: 2048 x 4096 18.4 and 18.7 us, 20000 x 1024
// 27.5 and 30.6, 5514 x 1001 floats 23.3 and 24.0, 16384 x 4096 97 and 99, 65536 x 4096 409 and 409, 65536 x 4090 444 and 412.
template <bool PAST> __device__ __forceinline__ void put16(void* p, u32x4 v) {
  if constexpr (PAST) __builtin_nontemporal_store(v, (u32x4_any2*)p);
  else *(u32x4_any2*)p = v;
}
bool whole_lines(const void* p, long row_bytes, long pitch_bytes) { return (uintptr_t)p % 64 == 0 && row_bytes % 64 == 0 && pitch_bytes % 64 == 0; }
// 8 elements of a row from element e on, as they lie in memory, of which `there` exist (0 for the others).  load brings the last elements of a row of at least 8
// (`whole`) as its last 8, settle() moves them into place: one wait for several rows, where loads of single elements wait one by one (forward and backward of 31885 x
// 4702, table 8954, 252 -> 200 us).
template <typename T> struct Piece;
template <> struct Piece<__bf16> {
  u32x4 w;
  __device__ __forceinline__ void load(const __bf16* p, int there, bool whole) {
    if (whole) {
      w = *(const u32x4_any2*)(p - max(0, V8 - there));
    } else {
      w = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
      for (int k = 0; k < V8 - 1; ++k)
        if (k < there) w[k / 2] |= (unsigned)((const uint16_t*)p)[k] << (16 * (k % 2));
    }
  }
  __device__ __forceinline__ void settle(int there, bool whole) {
    if (there >= V8 || !whole) return;
    const int over = V8 - there;
    if (over & 4) w = u32x4{w[2], w[3], 0u, 0u};
    if (over & 2) w = u32x4{w[1], w[2], w[3], 0u};
    if (over & 1) w = u32x4{w[0] >> 16 | w[1] << 16, w[1] >> 16 | w[2] << 16, w[2] >> 16 | w[3] << 16, w[3] >> 16};
  }
  __device__ __forceinline__ float operator[](int i) const { return __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16); }
  template <bool PAST = false> static __device__ __forceinline__ void store(__bf16* p, int there, const float (&v)[V8]) {
    if (there >= V8) {
      put16<PAST>(p, u32x4{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7])});
    } else {
#pragma unroll
      for (int k = 0; k < V8 - 1; ++k)
        if (k < there) p[k] = (__bf16)v[k];
    }
  }
};
template <> struct Piece<float> {
  u32x4 w[2];
  __device__ __forceinline__ void load(const float* p, int there, bool whole) {
    if (whole) {
      p -= max(0, V8 - there);
      w[0] = ((const u32x4_any4*)p)[0];
      w[1] = ((const u32x4_any4*)p)[1];
    } else {
      w[0] = w[1] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
      for (int k = 0; k < V8 - 1; ++k)
        if (k < there) w[k / 4][k % 4] = ((const uint32_t*)p)[k];
    }
  }
  __device__ __forceinline__ void settle(int there, bool whole) {
    if (there >= V8 || !whole) return;
    const int over = V8 - there;
    const u32x4 none = {0u, 0u, 0u, 0u};
    if (over & 4) { w[0] = w[1]; w[1] = none; }
    if (over & 2) { w[0] = u32x4{w[0][2], w[0][3], w[1][0], w[1][1]}; w[1] = u32x4{w[1][2], w[1][3], 0u, 0u}; }
    if (over & 1) { w[0] = u32x4{w[0][1], w[0][2], w[0][3], w[1][0]}; w[1] = u32x4{w[1][1], w[1][2], w[1][3], 0u}; }
  }
  __device__ __forceinline__ float operator[](int i) const { return __uint_as_float(w[i / 4][i % 4]); }
  template <bool PAST = false> static __device__ __forceinline__ void store(float* p, int there, const float (&v)[V8]) {
    if (there >= V8) {
      put16<PAST>(p, __builtin_bit_cast(u32x4, f32x4{v[0], v[1], v[2], v[3]}));
      put16<PAST>(p + 4, __builtin_bit_cast(u32x4, f32x4{v[4], v[5], v[6], v[7]}));
    } else {
#pragma unroll
      for (int k = 0; k < V8 - 1; ++k)
        if (k < there) p[k] = v[k];
    }
  }
};

// ---- forward: ROWS rows of a team on their way at once ----
constexpr int ROWS = 4;
template <typename T> __global__ void __launch_bounds__(256) embed_fwd_kernel(EmbedArgs a, int tl) {
  const int E = a.E, e = (((int)blockIdx.y << tl) + (threadIdx.x & ((1 << tl) - 1))) * V8, there = E - e;
  if (there <= 0) return;
  const long teams = 256 >> tl;
  for (long i0 = (long)blockIdx.x * (teams * ROWS) + (threadIdx.x >> tl); i0 < a.n; i0 += (long)gridDim.x * (teams * ROWS)) {
    long id[ROWS];
#pragma unroll
    for (int k = 0; k < ROWS; ++k) id[k] = a.ids[min(i0 + k * teams, a.n - 1)];
    Piece<T> x[ROWS];
#pragma unroll
    for (int k = 0; k < ROWS; ++k) x[k].load((const T*)a.table + min(max(id[k], 0L), a.V - 1) * E + e, there, E >= V8);
#pragma unroll
    for (int k = 0; k < ROWS; ++k) x[k].settle(there, E >= V8);
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      const long i = i0 + k * teams;
      if (i >= a.n) break;
      float v[V8];
#pragma unroll
      for (int j = 0; j < V8; ++j) v[j] = id[k] < 0 ? 0.f : id[k] < a.V ? x[k][j] * a.scale : __builtin_nanf("");
      Piece<T>::template store<true>((T*)a.y + i * a.y_ss + e, there, v);
    }
  }
}

// ---- backward: the sort ----

constexpr int SORT_WG = 1024, SORT_WAVES = SORT_WG / 64;
// Bits of a digit, digits of an id; log2 of the workgroups that share a sort by one launch, by the highest bits of an id, and the bits below these, which the digits are of.
struct Sort { int bits, passes, split, of; };
inline Sort sort_of(long V, int split) {
  int bits = 1;
  while (bits < 62 && (1L << bits) < V) ++bits;
  split = std::min(split, bits - 1);
  const int of = bits - split, passes = (of + EMBED_DIGIT_BITS - 1) / EMBED_DIGIT_BITS;
  return {(of + passes - 1) / passes, passes, split, of};
}

// The rank of every token among those of its wave with the same digit, in order: `rounds` x 64 tokens a wave, `dig` < 0: none.  cnt[digit]: the
// wave's counts, which start at 0.
template <int ROUNDS> __device__ __forceinline__ void rank_in_wave(const int (&dig)[ROUNDS], int (&rank)[ROUNDS], int rounds, int* cnt, int bits) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    if (r >= rounds) break;                          // (uniform)
    unsigned long long same = __ballot(dig[r] >= 0);
    for (int b = 0; b < bits; ++b) {
      const bool one = (dig[r] >> b) & 1;
      const unsigned long long ones = __ballot(one);
      same &= one ? ones : ~ones;
    }
    const int below = __popcll(same & ((1ull << lane) - 1));
    int at = 0;
    if (dig[r] >= 0 && below == 0) at = atomicAdd(&cnt[dig[r]], __popcll(same));
    rank[r] = __shfl(at, dig[r] >= 0 ? __ffsll(same) - 1 : lane) + below;
  }
}
// Exclusive sums of x over the workgroup's threads; *total: of all.  `at`: SORT_WAVES numbers of LDS.
__device__ __forceinline__ int exclusive_sum(int x, int* at, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int upto = x;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const int y = __shfl_up(upto, o);
    upto += lane >= o ? y : 0;
  }
  if (lane == 63) at[wave] = upto;
  __syncthreads();
  int before = 0, all = 0;
  for (int w = 0; w < SORT_WAVES; ++w) {
    const int y = at[w];
    before += w < wave ? y : 0;
    all += y;
  }
  __syncthreads();
  *total = all;
  return before + upto - x;
}
// LDS of the sort: counts [waves][digits] (or two numbers a thread), where every digit starts [digits], exclusive_sum's [waves]
__host__ __device__ constexpr int sort_counts(int digits) { return SORT_WAVES * digits > 2 * SORT_WG ? SORT_WAVES * digits : 2 * SORT_WG; }
inline int sort_lds(int bits) { return (int)sizeof(int) * (sort_counts(1 << bits) + (1 << bits) + SORT_WAVES); }
// Turns the waves' counts of a digit (thread t: digit t) into where the wave's first one stands among all of the workgroup's; returns how many there are.
__device__ __forceinline__ int counts_to_starts(int* cnt, int digits) {
  int run = 0;
  if ((int)threadIdx.x < digits) {
    int c[SORT_WAVES];
#pragma unroll
    for (int w = 0; w < SORT_WAVES; ++w) c[w] = cnt[w * digits + threadIdx.x];
#pragma unroll
    for (int w = 0; w < SORT_WAVES; ++w) {
      cnt[w * digits + threadIdx.x] = run;
      run += c[w];
    }
  }
  return run;
}
__device__ __forceinline__ void clear_counts(int* cnt, int digits) {
  for (int i = threadIdx.x; i < SORT_WAVES * digits; i += SORT_WG) cnt[i] = 0;
}
// Elements of the table's gradient that a launch of the sort sets to 0 beside its own work, by `wgs` further workgroups: the sort keeps few compute units busy, and
// rows that no token has, most of a large table's, have to be written anyway.  (Those that tokens have are written again behind it.)
struct Clear { long from, count; unsigned wgs; };
template <typename T> __device__ __forceinline__ void clear_table(T* p, long elements, long wg, long wgs) {
  // (up to the first 16-byte boundary, and behind the last one, by single elements)
  const long head = min(elements, (long)(((16 - ((uintptr_t)p & 15)) & 15) / sizeof(T))), vecs = (elements - head) * (long)sizeof(T) / 16;
  u32x4* const v = (u32x4*)(p + head);
  for (long i = wg * SORT_WG + threadIdx.x; i < vecs; i += wgs * SORT_WG) __builtin_nontemporal_store(u32x4{0u, 0u, 0u, 0u}, v + i);
  const long tail = head + vecs * (16 / (long)sizeof(T));
  if (wg == 0) {
    if ((long)threadIdx.x < head) p[threadIdx.x] = (T)0.f;
    if (tail + threadIdx.x < elements) p[tail + threadIdx.x] = (T)0.f;
  }
}

// For the lists that the sums leave, by a workgroup
__device__ __forceinline__ void lists_empty(const EmbedArgs& a) {
  if (threadIdx.x <= EMBED_LISTS) a.head->run[threadIdx.x].count = 0;
}
// Up to FEW tokens: every id is compared with all others.  (8 ids 9.6 -> 2.8 us, 64 9.8 -> 3.9, 120 9.9 -> 5.1; 250 of them, in the same way, 13.)
constexpr int FEW = 128;
__device__ __forceinline__ void sort_few(const EmbedArgs& a, const Sort& sort, int* keys) {
  const int tid = threadIdx.x, n = (int)a.n, none = 0x7ffffffe;
  int* const sorted = keys + FEW;
  __shared__ int count[2];
  static_assert(FEW == 128, "two waves");
  const long id = tid < n ? a.ids[tid] : -1;
  const int mine = id >= 0 && id < a.V ? (int)id : none;
  if (tid < FEW) keys[tid] = mine;
  const int on = __popcll(__ballot(mine != none));
  if (tid == 0) count[0] = on;
  if (tid == 64) count[1] = on;
  __syncthreads();
  if (tid < FEW) {
    int r = 0;
    const auto before = [&](int y, int j) { return y < mine + (j < tid ? 1 : 0) ? 1 : 0; };      // (equal ids: in the tokens' order)
    for (int j = 0; j < n; j += 16) {
      int4 y[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) y[k] = *(const int4*)(keys + j + 4 * k);
#pragma unroll
      for (int k = 0; k < 4; ++k) r += before(y[k].x, j + 4 * k) + before(y[k].y, j + 4 * k + 1) + before(y[k].z, j + 4 * k + 2) + before(y[k].w, j + 4 * k + 3);
    }
    if (tid < n) sorted[r] = mine;
    if (mine != none) {
      a.key[0][r] = mine;
      a.tok[0][r] = tid;
    }
  }
  __syncthreads();
  const int low = sort.bits * (sort.passes - 1), tops = 1 << (sort.of - low), m = count[0] + count[1];
  for (int d = tid; d <= tops; d += SORT_WG) {
    int lo = 0, hi = m;                              // the first whose last digit is d or more
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if ((sorted[mid] >> low) < d) lo = mid + 1;
      else hi = mid;
    }
    a.top[d] = lo;
  }
  if (tid == 0) a.head->tokens.count = m;
  lists_empty(a);
}

// Up to ONE_MOST tokens: all digits in one launch, by one workgroup, or by 2^split of them, each of which takes the ids with its value of the highest bits
// and counts those with lower ones.  LDS holds ONE_WG tokens of a workgroup; one that has more of them (most ids alike) sorts in the two lists in memory.
constexpr int ONE_ROUNDS = 8, ONE_WG = SORT_WG * ONE_ROUNDS, ONE_MOST = 32 * SORT_WG;
inline int one_room(long n) { return (int)std::min((long)ONE_WG, (n + SORT_WG - 1) / SORT_WG * SORT_WG); }
inline int one_lds(int bits, long n) { return sort_lds(bits) + 2 * (int)sizeof(int) * one_room(n); }
struct SortMem { int *cnt, *start, *sums, *skey, *stok; };
// The m tokens of group `mine`, in order in skey and stok (ids without the bits of the group), to places `base` and behind
__device__ __forceinline__ void sort_own(const EmbedArgs& a, const Sort& sort, const SortMem& s, int mine, int m, int base) {
  const int bits = sort.bits, digits = 1 << bits, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int rounds = (m + SORT_WG - 1) / SORT_WG, per_wave = 64 * rounds;
  int key[ONE_ROUNDS], tok[ONE_ROUNDS], dig[ONE_ROUNDS], rank[ONE_ROUNDS];
  const auto take = [&]() {
#pragma unroll
    for (int r = 0; r < ONE_ROUNDS; ++r) {
      const int i = wave * per_wave + 64 * r + lane;
      const bool on = r < rounds && i < m;
      key[r] = on ? s.skey[i] : -1;
      tok[r] = on ? s.stok[i] : 0;
    }
  };
  take();
  const int low = bits * (sort.passes - 1), tops = 1 << (sort.of - low);      // (values of the last digit)
  for (int p = 0; p < sort.passes; ++p) {
    clear_counts(s.cnt, digits);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ONE_ROUNDS; ++r) dig[r] = key[r] < 0 ? -1 : (key[r] >> (p * bits)) & (digits - 1);
    rank_in_wave<ONE_ROUNDS>(dig, rank, rounds, s.cnt + wave * digits, bits);
    __syncthreads();
    const int count = counts_to_starts(s.cnt, digits);
    int all;
    const int at = exclusive_sum(count, s.sums, &all);
    if (tid < digits) s.start[tid] = at;
    if (p == sort.passes - 1 && tid < tops) a.top[mine * tops + tid] = base + at;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ONE_ROUNDS; ++r)
      if (dig[r] >= 0) {
        const int to = s.start[dig[r]] + s.cnt[wave * digits + dig[r]] + rank[r];
        s.skey[to] = key[r];
        s.stok[to] = tok[r];
      }
    __syncthreads();
    take();
  }
#pragma unroll
  for (int r = 0; r < ONE_ROUNDS; ++r) {
    const int i = wave * per_wave + 64 * r + lane;
    if (key[r] >= 0) {
      a.key[0][base + i] = key[r] + (mine << sort.of);
      a.tok[0][base + i] = tok[r];
    }
  }
}
// Which list pass p writes; it reads the other one.
__device__ __forceinline__ int list_of(const Sort& sort, int p) { return (sort.passes - 1 - p) & 1; }
// The same of any number of tokens, which stand from `base` on in the list that pass 0 reads
__device__ __forceinline__ void sort_own_in_memory(const EmbedArgs& a, const Sort& sort, const SortMem& s, int mine, int m, int base) {
  constexpr int R = 4;
  const int bits = sort.bits, digits = 1 << bits, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int low = bits * (sort.passes - 1), tops = 1 << (sort.of - low);
  for (int p = 0; p < sort.passes; ++p) {
    const int to = list_of(sort, p), from = 1 - to;
    const bool last = p == sort.passes - 1;
    __syncthreads();
    if (tid < digits) s.start[tid] = 0;
    __syncthreads();
    for (int i = tid; i < m; i += SORT_WG) atomicAdd(&s.start[(a.key[from][base + i] >> (p * bits)) & (digits - 1)], 1);
    __syncthreads();
    const int count = tid < digits ? s.start[tid] : 0;
    int all;
    const int at = exclusive_sum(count, s.sums, &all);
    if (tid < digits) s.start[tid] = at;
    if (last && tid < tops) a.top[mine * tops + tid] = base + at;
    for (int b = 0; b < m; b += SORT_WG * R) {
      int key[R], tok[R], dig[R], rank[R];
      __syncthreads();
      clear_counts(s.cnt, digits);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int i = b + (wave * R + r) * 64 + lane;
        key[r] = i < m ? a.key[from][base + i] : -1;
        tok[r] = i < m ? a.tok[from][base + i] : 0;
        dig[r] = key[r] < 0 ? -1 : (key[r] >> (p * bits)) & (digits - 1);
      }
      __syncthreads();
      rank_in_wave<R>(dig, rank, R, s.cnt + wave * digits, bits);
      __syncthreads();
      const int in_step = counts_to_starts(s.cnt, digits);
      __syncthreads();
#pragma unroll
      for (int r = 0; r < R; ++r)
        if (dig[r] >= 0) {
          const int i = base + s.start[dig[r]] + s.cnt[wave * digits + dig[r]] + rank[r];
          a.key[to][i] = last ? key[r] + (mine << sort.of) : key[r];
          a.tok[to][i] = tok[r];
        }
      __syncthreads();
      if (tid < digits) s.start[tid] += in_step;
    }
    __threadfence_block();                           // (the next pass reads what other waves of this workgroup have written)
  }
}
template <typename T, int ROUNDS> __global__ void __launch_bounds__(SORT_WG) embed_sort_one_kernel(EmbedArgs a, Sort sort, Clear clear, int room) {
  const int groups = 1 << sort.split, mine = blockIdx.x;
  if (mine >= groups) {
    clear_table((T*)a.d_table + clear.from, clear.count, mine - groups, clear.wgs);
    return;
  }
  extern __shared__ __attribute__((aligned(16))) int sort_mem[];
  if (ROUNDS == ONE_ROUNDS && a.n <= FEW) {
    sort_few(a, sort, sort_mem);
    return;
  }
  const int digits = 1 << sort.bits, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  SortMem s;
  s.cnt = sort_mem;
  s.start = s.cnt + sort_counts(digits);
  s.sums = s.start + digits;
  s.skey = s.sums + SORT_WAVES;
  s.stok = s.skey + room;
  const int per_wave = (int)((a.n + SORT_WG - 1) / SORT_WG) * 64, rounds = per_wave / 64;
  // the ids, in order
  int id[ROUNDS];
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const int i = wave * per_wave + 64 * r + lane;
    const long x = r < rounds && i < a.n ? a.ids[i] : -1;
    id[r] = x >= 0 && x < a.V ? (int)x : -1;
  }
  int own = 0, lower = 0;                            // of the wave
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const int group = id[r] >> sort.of;              // (-1: none)
    own += __popcll(__ballot(group == mine));
    lower += __popcll(__ballot(group >= 0 && group < mine));
  }
  if (lane == 0) {
    s.cnt[wave] = own;
    s.cnt[SORT_WAVES + wave] = lower;
  }
  __syncthreads();
  int before = 0, m = 0, base = 0;                   // own ones of the waves before, of all; ids of the groups before
#pragma unroll
  for (int w = 0; w < SORT_WAVES; ++w) {
    const int c = s.cnt[w];
    before += w < wave ? c : 0;
    m += c;
    base += s.cnt[SORT_WAVES + w];
  }
  const bool fits = m <= room;
  int* const far_key = a.key[1 - list_of(sort, 0)] + base;
  int* const far_tok = a.tok[1 - list_of(sort, 0)] + base;
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const bool mine_too = id[r] >> sort.of == mine;
    const unsigned long long on = __ballot(mine_too);
    if (mine_too) {
      const int to = before + __popcll(on & ((1ull << lane) - 1)), key = id[r] & ((1 << sort.of) - 1), tok = wave * per_wave + 64 * r + lane;
      if (fits) {
        s.skey[to] = key;
        s.stok[to] = tok;
      } else {
        far_key[to] = key;
        far_tok[to] = tok;
      }
    }
    before += __popcll(on);
  }
  if (!fits) __threadfence_block();
  __syncthreads();
  if (ROUNDS == ONE_ROUNDS || fits) sort_own(a, sort, s, mine, m, base);
  else sort_own_in_memory(a, sort, s, mine, m, base);
  if (mine == groups - 1) lists_empty(a);
  if (tid == 0 && mine == groups - 1) {
    a.top[groups << (sort.of - sort.bits * (sort.passes - 1))] = base + m;
    a.head->tokens.count = base + m;
  }
}

// More tokens: a pass is two launches of up to EMBED_BLOCKS workgroups, each with a run of the tokens; the first counts the digits of every run, the
// second moves the tokens.  Pass 0 reads the ids and leaves tokens out that have no row.
constexpr int RUN_ROUNDS = 2, RUN_STEP = SORT_WG * RUN_ROUNDS;
inline long run_of(long n) { return std::max((long)RUN_STEP, (n + EMBED_BLOCKS * SORT_WG - 1) / (EMBED_BLOCKS * SORT_WG) * SORT_WG); }
__device__ __forceinline__ int sort_key(const EmbedArgs& a, int p, int from, long i, long n) {
  if (i >= n) return -1;
  if (p > 0) return a.key[from][i];
  const long id = a.ids[i];
  return id >= 0 && id < a.V ? (int)id : -1;
}
// (`from`: which of the two lists a pass reads)
__global__ void __launch_bounds__(SORT_WG) embed_count_kernel(EmbedArgs a, int bits, int p, int from, long run) {
  extern __shared__ __attribute__((aligned(16))) int sort_mem[];
  const int digits = 1 << bits, tid = threadIdx.x;
  for (int i = tid; i < digits; i += SORT_WG) sort_mem[i] = 0;
  __syncthreads();
  const long n = p > 0 ? a.head->tokens.count : a.n, end = min(n, (blockIdx.x + 1) * run);
  for (long i = blockIdx.x * run + tid; i < end; i += SORT_WG) {
    const int key = sort_key(a, p, from, i, n);
    if (key >= 0) atomicAdd(&sort_mem[(key >> (p * bits)) & (digits - 1)], 1);
  }
  __syncthreads();
  for (int i = tid; i < digits; i += SORT_WG) a.hist[(long)blockIdx.x * digits + i] = sort_mem[i];
}
template <typename T> __global__ void __launch_bounds__(SORT_WG) embed_move_kernel(EmbedArgs a, int bits, int p, int from, int to, long run, int blocks, int last, Clear clear) {
  if ((int)blockIdx.x >= blocks) {
    clear_table((T*)a.d_table + clear.from, clear.count, blockIdx.x - blocks, clear.wgs);
    return;
  }
  extern __shared__ __attribute__((aligned(16))) int sort_mem[];
  const int digits = 1 << bits, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int* const cnt = sort_mem;
  int* const start = cnt + sort_counts(digits);
  int* const sums = start + digits;
  const long n = p > 0 ? a.head->tokens.count : a.n, begin = blockIdx.x * run, end = min(n, begin + run);
  // where this run's tokens of every digit go: behind all smaller digits, and behind the runs before.  Several threads add up a digit's counts.
  const int per = SORT_WG / digits, digit = tid & (digits - 1), part = tid / digits;
  int all = 0, before = 0;
  for (int b0 = part; b0 < blocks; b0 += 8 * per) {
    int c[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) c[k] = a.hist[(long)min(b0 + k * per, blocks - 1) * digits + digit];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int b = b0 + k * per;
      all += b < blocks ? c[k] : 0;
      before += b < min(blocks, (int)blockIdx.x) ? c[k] : 0;
    }
  }
  cnt[2 * tid] = all;
  cnt[2 * tid + 1] = before;
  __syncthreads();
  all = before = 0;
  if (tid < digits)
    for (int k = 0; k < per; ++k) {
      all += cnt[2 * (tid + k * digits)];
      before += cnt[2 * (tid + k * digits) + 1];
    }
  int m;
  const int at = exclusive_sum(all, sums, &m);
  if (tid < digits) start[tid] = at + before;
  if (blockIdx.x == 0) {
    if (last) {
      if (tid < digits) a.top[tid] = at;
      if (tid == 0) a.top[digits] = m;
    }
    if (tid == 0 && p == 0) a.head->tokens.count = m;       // (pass 0 does not read it)
    lists_empty(a);
  }
  for (long base = begin; base < end; base += RUN_STEP) {
    int key[RUN_ROUNDS], tok[RUN_ROUNDS], dig[RUN_ROUNDS], rank[RUN_ROUNDS];
    __syncthreads();
    clear_counts(cnt, digits);
#pragma unroll
    for (int r = 0; r < RUN_ROUNDS; ++r) {
      const long i = base + (wave * RUN_ROUNDS + r) * 64 + lane;
      key[r] = sort_key(a, p, from, i, end);
      tok[r] = p == 0 ? (int)i : key[r] >= 0 ? a.tok[from][i] : 0;
      dig[r] = key[r] < 0 ? -1 : (key[r] >> (p * bits)) & (digits - 1);
    }
    __syncthreads();
    rank_in_wave<RUN_ROUNDS>(dig, rank, RUN_ROUNDS, cnt + wave * digits, bits);
    __syncthreads();
    const int count = counts_to_starts(cnt, digits);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < RUN_ROUNDS; ++r)
      if (dig[r] >= 0) {
        const int at = start[dig[r]] + cnt[wave * digits + dig[r]] + rank[r];
        a.key[to][at] = key[r];
        a.tok[to][at] = tok[r];
      }
    __syncthreads();
    if (tid < digits) start[tid] += count;
  }
}

// ---- backward: the sums ----

constexpr int MANY_PARTS = 32;

template <typename T, bool ADD> __device__ __forceinline__ void finish_row(const EmbedArgs& a, int id, int e, int there, const float (&s)[V8], const Piece<T>& old) {
  T* const to = (T*)a.d_table + (long)id * a.E + e;
  float v[V8];
  if constexpr (ADD) {
#pragma unroll
    for (int j = 0; j < V8; ++j) v[j] = fmaf(s[j], a.scale, old[j]);
  } else {
#pragma unroll
    for (int j = 0; j < V8; ++j) v[j] = s[j] * a.scale;
  }
  Piece<T>::store(to, there, v);
}

// Rows that no token has are set to 0: workgroup `wg` takes 2^sub of the ids that share their last digit, finds which of them tokens have (their
// sorted tokens are from top[digit] on) and clears the others.  About 16 KB of rows: many even workgroups (forward and backward of 65536 x
// 4096, table 131072, with 512 KB 500 us, 64 KB 490, 32 KB 480, 16 KB 473, 8 KB 486; of 2048 x 4096, table 32768, 72, 69, 68, 67, 64.  Sums among them instead of in
// front of them: 580 and 65).
constexpr int MOST_ROWS_LOG = 6;
inline int clear_rows_log(long row_bytes, int low) {
  int l = 0;
  while (l < std::min(low, MOST_ROWS_LOG) && (row_bytes << l) < (16 << 10)) ++l;
  return l;
}
template <typename T> __device__ __forceinline__ void clear_rows(const EmbedArgs& a, int tl, long wg, int low, int sub, bool past) {
  __shared__ unsigned has[1 << (MOST_ROWS_LOG - 5)];
  const int tid = threadIdx.x;
  const long v0 = wg << sub, v1 = min(a.V, v0 + (1L << sub));
  if (tid < (1 << (MOST_ROWS_LOG - 5))) has[tid] = 0u;
  __syncthreads();
  const int digit = (int)(v0 >> low);
  for (int i = a.top[digit] + tid; i < a.top[digit + 1]; i += 256) {
    const int r = a.key[0][i] - (int)v0;
    if (r >= 0 && r < (1 << sub)) atomicOr(&has[r / 32], 1u << (r % 32));
  }
  __syncthreads();
  const int per = chunks8(a.E), rows = (int)(v1 - v0);
  const float zero[V8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int r = tid >> tl; r < rows; r += 256 >> tl) {      // (a team a row, as in the sums; by whole workgroups 2000 tokens x 64, table 1000000, took 112 us, 37 so; x 256, 131072 34 and 28)
    if ((has[r / 32] >> (r % 32)) & 1u) continue;
    T* const to = (T*)a.d_table + (v0 + r) * a.E;
    for (int c = tid & ((1 << tl) - 1); c < per; c += 1 << tl) {
      if (past) Piece<T>::template store<true>(to + c * V8, a.E - c * V8, zero);
      else Piece<T>::store(to + c * V8, a.E - c * V8, zero);
    }
  }
}

// Chunks whose last id goes on are listed for the join, in EMBED_LISTS lists: additions to one counter take turns (12945 tokens x 256, added to a table of 3723,
// with one list 12.3 us, 6.0 so).
// Sums over a chunk of the sorted tokens, by a team (ADD: to what is there); workgroups from `sums_x` on clear rows, the first of them piece `early` of the table
// (2^sub rows; low: bits of an id below its last digit)
template <typename T, bool ADD> __global__ void __launch_bounds__(256) embed_sum_kernel(EmbedArgs a, int tl, unsigned sums_x, int n_eb, long early, int low, int sub, bool past) {
  if constexpr (!ADD) {
    if (blockIdx.x >= sums_x) {
      clear_rows<T>(a, tl, early + (blockIdx.x - sums_x), low, sub, past);
      return;
    }
  }
  const int E = a.E, lane = threadIdx.x & ((1 << tl) - 1), eb = (int)(blockIdx.x % n_eb), e = ((eb << tl) + lane) * V8, there = E - e;
  const long c = (long)(blockIdx.x / n_eb) * (256 >> tl) + (threadIdx.x >> tl), p0 = c * a.chunk;
  const int m = a.head->tokens.count;
  if (p0 >= m || there <= 0) return;
  const int first = (int)p0, end = (int)min((long)m, p0 + a.chunk);
  const int *const key = a.key[0], *const tok = a.tok[0];
  const int prev = first > 0 ? key[first - 1] : -1, next = end < m ? key[end] : -1;
  bool before = prev == key[first];
  float s[V8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  constexpr int U = ADD ? 4 : 8;                     // rows on their way at once
  for (int p = first; p < end; p += U) {
    int id[U];
    Piece<T> x[U], old[ADD ? U : 1];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      id[k] = key[min(p + k, end - 1)];
      x[k].load((const T*)a.d_y + tok[min(p + k, end - 1)] * a.y_ss + e, there, E >= V8);
    }
    if constexpr (ADD) {                             // (of an id that is finished here: nobody else writes its row)
#pragma unroll
      for (int k = 0; k < U; ++k) old[k].load((const T*)a.d_table + (long)id[k] * E + e, there, E >= V8);
#pragma unroll
      for (int k = 0; k < U; ++k) old[k].settle(there, E >= V8);
    }
#pragma unroll
    for (int k = 0; k < U; ++k) x[k].settle(there, E >= V8);
#pragma unroll
    for (int k = 0; k < U; ++k)
      if (p + k < end) {
#pragma unroll
        for (int j = 0; j < V8; ++j) s[j] += x[k][j];
        // the last of its id in this chunk?
        const int q = p + k + 1, following = q < end ? (k + 1 < U ? id[min(k + 1, U - 1)] : key[q]) : -1;
        if (following != id[k]) {
          const bool after = q == end && next == id[k];
          if (!before && !after) {
            finish_row<T, ADD>(a, id[k], e, there, s, old[ADD ? k : 0]);
          } else {
            Piece<float>::store(a.part + (2 * c + (before ? 0 : 1)) * E + e, there, s);
            if (after && !before && e == 0) {        // (the lists' order changes no result)
              const long far = (c + MANY_PARTS) * a.chunk;
              const int to = far < m && key[far] == id[k] ? EMBED_LISTS : (int)(c % EMBED_LISTS);
              a.long_list[to * a.list_room + atomicAdd(&a.head->run[to].count, 1)] = make_int2((int)c, id[k]);
            }
          }
#pragma unroll
          for (int j = 0; j < V8; ++j) s[j] = 0.f;
          before = false;
        }
      }
  }
}

// Ids that go over several chunks.
// The chunks that begin with the id follow each other from c0 + 1 on; returns the last of them, by a wave: 64 of them, or 64 that are even over what is left, at once.
__device__ __forceinline__ int last_chunk(const EmbedArgs& a, int c0, int id, int m) {
  const int lane = threadIdx.x & 63;
  long c1 = c0, behind = (m + a.chunk - 1) / a.chunk, stride = 1;
  do {
    const long c = c1 + (lane + 1) * stride;
    const unsigned long long more = __ballot(c < behind && a.key[0][min(c, behind - 1) * a.chunk] == id);
    const int found = more == ~0ull ? 64 : __ffsll(~more) - 1;
    c1 += found * stride;
    if (found < 64) behind = min(behind, c1 + stride);
    stride = (behind - c1 + 63) / 64;
  } while (behind - c1 > 1);
  return (int)c1;
}
// Sums q0 .. q1 - 1 of an id's (the first is the end of chunk c0, the others the beginnings of the chunks behind), four features from e on
__device__ __forceinline__ f32x4 add_parts(const EmbedArgs& a, int c0, int q0, int q1, int e) {
  const int E = a.E;
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  const auto run = [&](auto whole) {
    for (int q = q0; q < q1; q += 8) {
      f32x4 v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int c = min(q + k, q1 - 1);
        const float* const from = a.part + (2L * (c0 + c) + (c == 0 ? 1 : 0)) * E + e;
        if constexpr (decltype(whole)::value) {
          v[k] = __builtin_bit_cast(f32x4, *(const u32x4_any4*)from);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) v[k][j] = e + j < E ? from[j] : 0.f;
        }
      }
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (q + k < q1) s += v[k];
    }
  };
  if (e + 4 <= E) run(std::true_type{});
  else run(std::false_type{});
  return s;
}
// What is there of a row, where it is added to (ahead of the sums), and the row
template <typename T> __device__ __forceinline__ f32x4 joined_to(const EmbedArgs& a, int id, int e) {
  f32x4 old = {0.f, 0.f, 0.f, 0.f};
  if (a.accumulate) {
#pragma unroll
    for (int j = 0; j < 4; ++j) old[j] = (float)((const T*)a.d_table)[(long)id * a.E + min(e + j, a.E - 1)];
  }
  return old;
}
template <typename T> __device__ __forceinline__ void put_joined(const EmbedArgs& a, int id, int e, const f32x4& s, const f32x4& old) {
  T* const to = (T*)a.d_table + (long)id * a.E + e;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (e + j < a.E) to[j] = (T)(a.accumulate ? fmaf(s[j], a.scale, old[j]) : s[j] * a.scale);
}
// An id of more than MANY_PARTS chunks: 256 features a workgroup, whose waves, and in them groups of 2^cl lanes, where a row has no more, take a run of the
// chunks each (the first wgs_many workgroups).  The others, most of them: 256 features a wave.  (131072 tokens x 64, two in three the same id: 928 us with four waves and whole rows, 112 so; x 1024 145 and 124)
constexpr int JOIN_WG = 512, JOIN_WAVES = JOIN_WG / 64;
template <typename T> __global__ void __launch_bounds__(JOIN_WG) embed_join_kernel(EmbedArgs a, int cl, int wgs_many) {
  __shared__ __attribute__((aligned(16))) float sums[JOIN_WAVES][256];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, m = a.head->tokens.count, blocks = (a.E + 255) / 256;
  const int units = JOIN_WAVES << (6 - cl), unit = (wave << (6 - cl)) + (lane >> cl), l = lane & ((1 << cl) - 1);
  if ((int)blockIdx.x >= wgs_many) {
    const int w = ((int)blockIdx.x - wgs_many) * JOIN_WAVES + wave, step = ((int)gridDim.x - wgs_many) * JOIN_WAVES / EMBED_LISTS, list = w % EMBED_LISTS;
    const long n_few = (long)a.head->run[list].count * blocks;
    for (long it = w / EMBED_LISTS; it < n_few; it += step) {
      const int2 run = a.long_list[list * a.list_room + it / blocks];
      const int e = (int)(it % blocks) * 256 + 4 * lane, last = last_chunk(a, run.x, run.y, m);
      if (e < a.E) {
        const f32x4 old = joined_to<T>(a, run.y, e);
        put_joined<T>(a, run.y, e, add_parts(a, run.x, 0, last - run.x + 1, e), old);
      }
    }
    return;
  }
  const long n_many = (long)a.head->run[EMBED_LISTS].count * blocks;
  for (long it = blockIdx.x; it < n_many; it += wgs_many) {
    const int2 run = a.long_list[EMBED_LISTS * a.list_room + it / blocks];
    const int e = (int)(it % blocks) * 256 + 4 * l, parts = last_chunk(a, run.x, run.y, m) - run.x + 1;
    const bool mine = wave == 0 && lane < (1 << cl) && e < a.E;
    const f32x4 old = mine ? joined_to<T>(a, run.y, e) : f32x4{0.f, 0.f, 0.f, 0.f};
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    if (e < a.E) s = add_parts(a, run.x, (int)((long)unit * parts / units), (int)((long)(unit + 1) * parts / units), e);
    for (int o = 1 << cl; o < 64; o *= 2)
#pragma unroll
      for (int j = 0; j < 4; ++j) s[j] += __shfl_xor(s[j], o);
    __syncthreads();                                 // (the sums of the id before have been read)
    if (lane < (1 << cl)) *(f32x4*)&sums[wave][4 * l] = s;
    __syncthreads();
    if (mine) {
      s = *(const f32x4*)&sums[0][4 * l];
      for (int w = 1; w < JOIN_WAVES; ++w) s += *(const f32x4*)&sums[w][4 * l];
      put_joined<T>(a, run.y, e, s, old);
    }
  }
}

long up(long n, long by) { return (n + by - 1) / by; }

// Bytes of the table that a launch of the sort clears: about what goes to memory in its time.  The gradient's us with none of it, half as much, this and twice as much:
// 512 x 1024, table 50000, 31.2, 29.6, 28.3, 24.5; 2048 x 4096, 32768, 65.8, 64.3, 62.3, 57.3; 20000 x 512, 131072, 49.5, 45.2, 40.9, 45.0; 40000 x 1024, 65536, 59.2, 59.3,
// 60.8, 67.9; 65536 x 4096, 131072, 339, 333, 330, 330; 131072 x 256, 131072, 67.6, 62.7, 63.7, 64.0.
constexpr long CLEAR_ONE = 20 << 20, CLEAR_ROUND = 3 << 20, CLEAR_MORE = 1 << 20, CLEAR_MOVE = 48 << 20;

template <typename T> hipError_t embed_fwd(const EmbedArgs& a, hipStream_t s) {
  const int tl = team_log(a.E);
  const dim3 grid((unsigned)std::min(up(a.n, (256 >> tl) * ROWS), 1L << 18), (unsigned)up(a.E, V8 << tl));
  embed_fwd_kernel<T><<<grid, 256, 0, s>>>(a, tl);
  return hipGetLastError();
}

// Workgroups that clear `bytes` of the table, of those that are left from row `*row` on, in whole pieces of `piece` rows
template <typename T> Clear clear_some(const EmbedArgs& a, long bytes, long piece, long* row) {
  const long rows = std::min(a.V - *row, up(bytes, (long)sizeof(T) * a.E * piece) * piece);
  const Clear c = {*row * a.E, rows * a.E, (unsigned)std::min(4L * a.n_cu, up(rows * a.E, SORT_WG * 16))};
  *row += rows;
  return c;
}
template <typename T, int ROUNDS> hipError_t sort_one(const EmbedArgs& a, const Sort& sort, const Clear& clear, hipStream_t s) {
  static SmemOnce once;
  const hipError_t e = ensure_dynamic_lds((const void*)embed_sort_one_kernel<T, ROUNDS>, one_lds(EMBED_DIGIT_BITS, ONE_WG), &once);
  if (e != hipSuccess) return e;
  embed_sort_one_kernel<T, ROUNDS><<<(1 << sort.split) + clear.wgs, SORT_WG, one_lds(sort.bits, a.n), s>>>(a, sort, clear, one_room(a.n));
  return hipGetLastError();
}
// log2 of the workgroups that share a sort (5514 ids: one 17 us, eight 11.5; 20000: 32 workgroups 17.6, the passes over two launches each 26; 65536: 38 and 36)
int split_of(long n) { return n <= SORT_WG || n > ONE_MOST ? 0 : n <= ONE_WG ? 3 : 5; }
template <typename T, bool ADD> hipError_t embed_bwd(const EmbedArgs& a, hipStream_t s) {
  const Sort sort = sort_of(a.V, split_of(a.n));
  const int low = sort.bits * (sort.passes - 1);
  const int sub = clear_rows_log((long)sizeof(T) * a.E, low);
  const long piece = 1L << sub;
  long row = ADD ? a.V : 0;                          // the rows before are cleared already
  hipError_t e;
  if (a.n <= ONE_MOST) {
    const long rounds = up(a.n, SORT_WG);
    const Clear clear = clear_some<T>(a, CLEAR_ONE + CLEAR_ROUND * std::min(rounds, 8L) + CLEAR_MORE * rounds, piece, &row);
    e = a.n <= ONE_WG ? sort_one<T, ONE_ROUNDS>(a, sort, clear, s) : sort_one<T, ONE_MOST / SORT_WG>(a, sort, clear, s);
    if (e != hipSuccess) return e;
  } else {
    static SmemOnce once;
    e = ensure_dynamic_lds((const void*)embed_move_kernel<T>, sort_lds(EMBED_DIGIT_BITS), &once);
    if (e != hipSuccess) return e;
    const long run = run_of(a.n);
    const unsigned blocks = (unsigned)up(a.n, run);
    for (int p = 0; p < sort.passes; ++p) {
      const int to = (sort.passes - 1 - p) % 2, from = 1 - to;
      embed_count_kernel<<<blocks, SORT_WG, (1 << sort.bits) * sizeof(int), s>>>(a, sort.bits, p, from, run);
      const Clear clear = clear_some<T>(a, CLEAR_MOVE, piece, &row);
      embed_move_kernel<T><<<blocks + clear.wgs, SORT_WG, sort_lds(sort.bits), s>>>(a, sort.bits, p, from, to, run, (int)blocks, p == sort.passes - 1, clear);
    }
  }
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int tl = team_log(a.E), n_eb = (int)up(a.E, V8 << tl);
  const long n_chunks = up(a.n, a.chunk), wgs = up(n_chunks, 256 >> tl) * n_eb;
  const bool past = whole_lines(a.d_table, (long)sizeof(T) * a.E, (long)sizeof(T) * a.E);
  embed_sum_kernel<T, ADD><<<(unsigned)(wgs + up(a.V - row, piece)), 256, 0, s>>>(a, tl, (unsigned)wgs, n_eb, row / piece, low, sub, past);
  if (n_chunks > 1) {
    int cl = 0;                                      // lanes for four features each of a row, or of 256 features
    while (cl < 6 && (4 << cl) < a.E) ++cl;
    const long blocks = up(a.E, 256), many = n_chunks > MANY_PARTS ? std::min(n_chunks / MANY_PARTS * blocks, (long)a.n_cu) : 0;
    const long few = up(std::min((n_chunks - 1) * blocks, 3L * a.n_cu * JOIN_WAVES), EMBED_LISTS) * (EMBED_LISTS / JOIN_WAVES);
    embed_join_kernel<T><<<(unsigned)(many + few), JOIN_WG, 0, s>>>(a, cl, (int)many);
  }
  return hipGetLastError();
}

}  // namespace

// Sorted tokens of a chunk: 4 to 64, so that there are threads for about 2^18 pieces of 8 features.  The gradient's us with 2^16, 2^18 and 2^20: 2048 x 4096, table 32768, 56.4,
// 62.3, 62.3, added to what is there 26.1, 24.0, 24.0; 20000 x 512, 131072, 46.1, 40.9, 46.3, added 44.9, 34.7, 36.4; 131072 x 256, 131072, 78.8, 63.7, 86.7; 65536 x 4096, 131072,
// 327, 330, 339, added 250, 251, 238.
constexpr int LEAST_CHUNK = 4;
int embed_chunk(long n, int E) {
  if (n <= 16) return 16;                            // (then nothing is left to join)
  int c = LEAST_CHUNK;
  while (c < 64 && n * chunks8(E) / c > (1L << 18)) c *= 2;
  return c;
}
long embed_list_room(long n) { return n / LEAST_CHUNK / EMBED_LISTS + 1; }
// Chunks are the shorter the less there is: of n E / 8 = P pieces or fewer, no more than min(P / 4, max(2^18, P / 64)) chunk pieces and a row of them.
size_t embed_part_room(long n, int E) {
  const long P = n * chunks8(E);
  return 2 * sizeof(float) * (size_t)V8 * (std::min(P / LEAST_CHUNK, std::max(1L << 18, P / 64)) + chunks8(E) + 1);
}

hipError_t launch_embed_fwd(const EmbedArgs& a, int is_f32, hipStream_t s) { return is_f32 ? embed_fwd<float>(a, s) : embed_fwd<__bf16>(a, s); }
hipError_t launch_embed_bwd(EmbedArgs a, int is_f32, hipStream_t s) {
  a.chunk = embed_chunk(a.n, a.E);
  a.list_room = embed_list_room(a.n);
  if (a.accumulate) return is_f32 ? embed_bwd<float, true>(a, s) : embed_bwd<__bf16, true>(a, s);
  return is_f32 ? embed_bwd<float, false>(a, s) : embed_bwd<__bf16, false>(a, s);
}

}  // namespace lvx
