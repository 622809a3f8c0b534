// Losses of whole sequences from their tokens' negative log likelihoods, and the gradients with respect to these.
//
// Preferences, of a pair (c: the chosen one, r: the rejected one), with t over a sequence's tokens that have a label:
//   margin = sum_t (ref_t - nll_t) of c - the same of r,   h = beta margin
//   logistic  loss = (1 - a) ln(1 + exp(-h)) + a ln(1 + exp(h)),      hinge  max(0, 1 - h),      square  (margin - 1 / (2 beta))^2
//   d_nll_t = -loss'(margin) d_loss on c, +loss'(margin) d_loss on r
// Policies, of a sequence: ratio = exp(old - nll), A its advantage (or the token's), d = nll - ref
//   l_t = -min(ratio A, clamp(ratio, low, high) A) + beta (exp(d) - 1 - d),   loss = mean (or sum) over t of l_t
//   d_nll_t = (ratio A [not clipped] + beta (exp(d) - 1)) d_loss (/ count)
//
// A token is some 20 bytes and, in 64 bits (sums over long sequences of which differences are taken, values next to a bound; the float64 units are as fast
// as the float32 ones here), some hundred instructions: bound by memory, and by launches where there are few.  Few tokens (ONE_TOKENS): a workgroup a pair or
// sequence, in one launch.  More: cut at the multiples of SEQUENCE_BLOCK, a workgroup a piece; the first launch leaves the pieces' sums, the
// second adds up those of its sequence, in order, and does what hangs on them; of very many tokens a launch between the two makes the
// sequences' sums.  No atomics: results repeat bit for bit.
#include "lvx_internal.h"

#include <algorithm>
#include <type_traits>

namespace lvx {

namespace {

__device__ __forceinline__ double other(double x, int o) { return __shfl_xor(x, o); }
__device__ __forceinline__ int other(int x, int o) { return __shfl_xor(x, o); }
struct PrefPart {
  double s;
  __device__ __forceinline__ void add(const PrefPart& o) { s += o.s; }
  __device__ __forceinline__ PrefPart from_lane(int o) const { return {other(s, o)}; }
};
struct PolicyPart {
  double loss, kl;
  int count, clipped;
  __device__ __forceinline__ void add(const PolicyPart& o) { loss += o.loss; kl += o.kl; count += o.count; clipped += o.clipped; }
  __device__ __forceinline__ PolicyPart from_lane(int o) const { return {other(loss, o), other(kl, o), other(count, o), other(clipped, o)}; }
};
// Sums over the workgroup, the same in every thread (`at`: a place a wave in LDS)
template <class P> __device__ __forceinline__ P wg_sum(P x, P* at) {
#pragma unroll
  for (int o = 1; o < 64; o *= 2) x.add(x.from_lane(o));
  const int waves = blockDim.x >> 6;
  if (waves == 1) return x;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = x;
  __syncthreads();
  P y = at[0];
  for (int w = 1; w < waves; ++w) y.add(at[w]);
  return y;
}

// Where a sequence begins and ends, inside the tensors whatever `first` holds
struct Span { long begin, end; };
__device__ __forceinline__ Span span_of(const SequenceArgs& a, long s) {
  const long b = min(max(a.first[s], 0L), a.n), e = min(max(a.first[s + 1], 0L), a.n);
  return {b, max(b, e)};
}

// exp(x) in 64 bits, off by some 1e-14 of itself: 2^k by the exponent, the rest, up to ln 2 / 2, by its series (the first term left out is 6e-15).  The rest is x - k ln 2
// after Cody and Waite: ln 2 as its first 32 bits, whose product with k is exact, and what is left of it.
__device__ __forceinline__ double exp_of(double x) {
  x = x < -800.0 ? -800.0 : x > 800.0 ? 800.0 : x;  // (a NaN stays one)
  const double k = rint(x * 1.4426950408889634);
  double r = fma(k, -0x1.62e42feep-1, x);
  r = fma(k, -0x1.a39ef35793c76p-33, r);
  double p = 1.0 / 39916800.0;
  const double c[11] = {1.0 / 3628800.0, 1.0 / 362880.0, 1.0 / 40320.0, 1.0 / 5040.0, 1.0 / 720.0, 1.0 / 120.0, 1.0 / 24.0, 1.0 / 6.0, 0.5, 1.0, 1.0};
#pragma unroll
  for (int i = 0; i < 11; ++i) p = fma(p, r, c[i]);
  return ldexp(p, (int)k);
}
// exp(x) - 1 - x, which keeps its digits for small x too: x^2 times a series up to 1/2 (the first term left out is 7e-15 of it).  *less_one: exp(x) - 1, which far
// out is not the sum of that and x: -1 for -infinity.
__device__ __forceinline__ double exp_less_line(double x, double* less_one) {
  double p = 1.0 / 6227020800.0;
  const double c[11] = {1.0 / 479001600.0, 1.0 / 39916800.0, 1.0 / 3628800.0, 1.0 / 362880.0, 1.0 / 40320.0, 1.0 / 5040.0, 1.0 / 720.0, 1.0 / 120.0, 1.0 / 24.0, 1.0 / 6.0, 0.5};
#pragma unroll
  for (int i = 0; i < 11; ++i) p = fma(p, x, c[i]);
  const double near = p * x * x, far = exp_of(x) - 1.0;
  const bool small = fabs(x) <= 0.5;
  *less_one = small ? near + x : far;
  return small ? near : far - x;
}

// ---- tokens: U of a thread on their way at once, `wg` apart (behind the last one that one again) ----
constexpr int U = 4;
struct Batch { long label[U]; float nll[U], ref[U], old[U], adv[U]; };
template <bool POLICY> __device__ __forceinline__ void load(const SequenceArgs& a, long t, long end, long wg, Batch* b) {
#pragma unroll
  for (int k = 0; k < U; ++k) {
    const long i = min(t + k * wg, end - 1);
    b->label[k] = a.labels[i];
    b->nll[k] = a.nll[i];
    b->ref[k] = (POLICY ? a.beta != 0.0 : a.ref != nullptr) ? a.ref[i] : 0.f;
    if (POLICY) {
      b->old[k] = a.old[i];
      b->adv[k] = a.per_token ? a.adv[i] : 0.f;
    }
  }
}
__device__ __forceinline__ void sum_pref(const Batch& b, long t, long end, long wg, PrefPart* p) {
#pragma unroll
  for (int k = 0; k < U; ++k) p->s += t + k * wg < end && b.label[k] >= 0 ? (double)b.ref[k] - (double)b.nll[k] : 0.0;
}
// d_nll = d where there is a label
__device__ __forceinline__ void put_pref(const SequenceArgs& a, const long (&label)[U], long t, long end, long wg, float d) {
#pragma unroll
  for (int k = 0; k < U; ++k)
    if (t + k * wg < end) a.d_nll[t + k * wg] = label[k] >= 0 ? d : 0.f;
}
__device__ __forceinline__ void load_labels(const SequenceArgs& a, long t, long end, long wg, long (&label)[U]) {
#pragma unroll
  for (int k = 0; k < U; ++k) label[k] = a.labels[min(t + k * wg, end - 1)];
}
// One token's share of the loss; returns the gradient.  A: its advantage.
__device__ __forceinline__ double token_policy(const SequenceArgs& a, double nll, double old, double ref, double A, PolicyPart* p) {
  const double gone = old - nll;
  const double ratio = exp_of(gone);
  // (by logarithms, of which the difference is exact)
  const bool over = A > 0.0 ? gone > a.ln_high : A < 0.0 && gone < a.ln_low;
  const double high = a.high, low = a.low;
  double loss = over ? -(A > 0.0 ? high : low) * A : -ratio * A, slope = over ? 0.0 : ratio * A;
  if (a.beta != 0.0) {
    const double d = nll - ref;
    double less_one;
    const double more = exp_less_line(d, &less_one);
    loss += a.beta * more;
    slope += a.beta * less_one;
    p->kl += more;
  }
  p->loss += loss;
  p->count += 1;
  p->clipped += over;
  return slope;
}
// adv: the sequence's advantage, d: what the gradients are multiplied by
__device__ __forceinline__ void do_policy(const SequenceArgs& a, Batch& b, long t, long end, long wg, float adv, float d, PolicyPart* p) {
  if (!a.per_token) {
#pragma unroll
    for (int k = 0; k < U; ++k) b.adv[k] = adv;
  }
#pragma unroll
  for (int k = 0; k < U; ++k)
    if (t + k * wg < end) {
      const double slope = b.label[k] >= 0 ? token_policy(a, b.nll[k], b.old[k], b.ref[k], b.adv[k], p) : 0.0;
      if (a.d_nll) a.d_nll[t + k * wg] = b.label[k] >= 0 ? (float)(slope * (double)d) : 0.f;
    }
}
__device__ __forceinline__ void scale_policy(const SequenceArgs& a, long t, long end, long wg, double by) {
  float x[U];
#pragma unroll
  for (int k = 0; k < U; ++k) x[k] = a.d_nll[min(t + k * wg, end - 1)];
#pragma unroll
  for (int k = 0; k < U; ++k)
    if (t + k * wg < end) a.d_nll[t + k * wg] = (float)((double)x[k] * by);
}

// ---- a pair ----
__device__ __forceinline__ double pair_loss(const SequenceArgs& a, double margin, double* slope) {
  const double h = a.beta * margin;
  if (a.form == LVX_PREF_LOGISTIC) {
    const double e = exp(-fabs(h)), soft = log1p(e), q = a.smoothing;
    *slope = a.beta * (q * ((h >= 0.0 ? 1.0 : e) / (1.0 + e)) - (1.0 - q) * ((h < 0.0 ? 1.0 : e) / (1.0 + e)));      // (s(h) - (1 - q) would lose what is left of a sure pair's)
    // (a part of no weight is left out: of an infinite margin it would be 0 times infinity)
    const double won = soft + (h < 0.0 ? -h : 0.0), lost = soft + (h > 0.0 ? h : 0.0);
    return (q < 1.0 ? (1.0 - q) * won : 0.0) + (q > 0.0 ? q * lost : 0.0);
  }
  if (a.form == LVX_PREF_HINGE) {
    *slope = h >= 1.0 ? 0.0 : h < 1.0 ? -a.beta : h;             // (a NaN stays one)
    return h >= 1.0 ? 0.0 : 1.0 - h;
  }
  *slope = 2.0 * (margin - 0.5 / a.beta);
  return (margin - 0.5 / a.beta) * (margin - 0.5 / a.beta);
}
__device__ __forceinline__ void put_stats(const SequenceArgs& a, long s, const PolicyPart& p) {
  const double per = p.count > 0 ? 1.0 / p.count : 0.0;
  a.loss[s] = (float)(a.mean ? p.loss * per : p.loss);
  if (!a.stats) return;
  a.stats[3 * s] = (float)p.count;
  a.stats[3 * s + 1] = (float)(p.clipped * per);
  a.stats[3 * s + 2] = (float)(p.kl * per);
}

// ---- few tokens: a pair or a sequence a workgroup ----
__device__ __forceinline__ PrefPart sum_span(const SequenceArgs& a, const Span& s) {
  PrefPart p{};
  for (long t = s.begin + threadIdx.x; t < s.end; t += U * blockDim.x) {
    Batch b;
    load<false>(a, t, s.end, blockDim.x, &b);
    sum_pref(b, t, s.end, blockDim.x, &p);
  }
  return p;
}
__device__ __forceinline__ void put_span(const SequenceArgs& a, const Span& s, float d) {
  for (long t = s.begin + threadIdx.x; t < s.end; t += U * blockDim.x) {
    long label[U];
    load_labels(a, t, s.end, blockDim.x, label);
    put_pref(a, label, t, s.end, blockDim.x, d);
  }
}
__global__ void __launch_bounds__(1024) preference_one_kernel(SequenceArgs a) {
  __shared__ PrefPart at[16];
  const long pairs = a.count / 2;
  for (long i = blockIdx.x; i < pairs; i += gridDim.x) {
    const Span c = span_of(a, i), r = span_of(a, pairs + i);
    PrefPart p = sum_span(a, c);
    p.s -= sum_span(a, r).s;
    const double margin = wg_sum(p, at).s;
    double slope;
    const double loss = pair_loss(a, margin, &slope);
    if (threadIdx.x == 0) {
      a.loss[i] = (float)loss;
      if (a.margin) a.margin[i] = (float)margin;
    }
    if (!a.d_nll) continue;
    const float d = (float)(slope * (double)a.d_loss[i]);
    put_span(a, c, -d);
    put_span(a, r, d);
  }
}
__global__ void __launch_bounds__(1024) policy_one_kernel(SequenceArgs a) {
  __shared__ PolicyPart at[16];
  const long wg = blockDim.x;
  for (long i = blockIdx.x; i < a.count; i += gridDim.x) {
    const Span c = span_of(a, i);
    const float adv = a.per_token ? 0.f : a.adv[i], d = a.d_nll ? a.d_loss[i] : 0.f;
    PolicyPart p{};
    for (long t = c.begin + threadIdx.x; t < c.end; t += U * wg) {
      Batch b;
      load<true>(a, t, c.end, wg, &b);
      do_policy(a, b, t, c.end, wg, adv, d, &p);
    }
    p = wg_sum(p, at);
    if (threadIdx.x == 0) put_stats(a, i, p);
    if (!a.d_nll || !a.mean || p.count == 0) continue;
    for (long t = c.begin + threadIdx.x; t < c.end; t += U * wg) scale_policy(a, t, c.end, wg, 1.0 / p.count);      // (what this thread has written)
  }
}

// ---- more tokens: a piece of a sequence a workgroup ----

// Workgroups 0 .. count - 1: a sequence up to the first multiple of SEQUENCE_BLOCK behind its start; the others: from a multiple on, where it is inside
// a sequence.  (seq < 0: nothing)
struct Job { long seq, begin, end; };
__device__ __forceinline__ bool is_block(const SequenceArgs& a) { return blockIdx.x >= a.count; }
__device__ __forceinline__ long block_begin(const SequenceArgs& a) { return (blockIdx.x - a.count) * SEQUENCE_BLOCK; }
__device__ __forceinline__ Job job_of(const SequenceArgs& a, int* lds) {
  constexpr long P = SEQUENCE_BLOCK;
  if (!is_block(a)) {
    const Span s = span_of(a, blockIdx.x);
    return {blockIdx.x, s.begin, min(s.end, (s.begin / P + 1) * P)};
  }
  const long x = block_begin(a);
  long lo = 0, hi = a.count + 1;                     // first[lo] <= x < first[hi] (or the ends)
  while (hi - lo > 1) {
    const long step = (hi - lo + 255) / 256, at = lo + (long)threadIdx.x * step;
    const unsigned long long below = __ballot(at < hi && a.first[min(at, a.count)] <= x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = __popcll(below);
    __syncthreads();
    const int found = lds[0] + lds[1] + lds[2] + lds[3];
    if (found == 0) return {-1, 0, 0};               // (in front of the first sequence)
    lo += (found - 1) * step;
    hi = min(hi, lo + step);
  }
  if (lo >= a.count) return {-1, 0, 0};
  const Span s = span_of(a, lo);
  if (s.begin >= x || s.end <= x) return {-1, 0, 0};
  return {lo, x, min(s.end, x + P)};
}
// The sum over a sequence: its first piece and the blocks that go on in it (a thread's share of it)
template <class P> __device__ __forceinline__ P share_of(const SequenceArgs& a, const Span& s, long seq) {
  P p{};
  if (threadIdx.x == 0) p.add(((const P*)a.head)[seq]);
  if (a.totals) return p;
  for (long j = s.begin / SEQUENCE_BLOCK + 1 + threadIdx.x; j * SEQUENCE_BLOCK < s.end; j += blockDim.x) p.add(((const P*)a.block)[j]);
  return p;
}
// Whole sequences' sums in place of their first pieces' (`total`): otherwise every piece's workgroup adds up all pieces of its sequence again, which goes with the
// square of its length
template <class P> __global__ void __launch_bounds__(1024) sequence_total_kernel(SequenceArgs a) {
  __shared__ P at[16];
  for (long i = blockIdx.x; i < a.count; i += gridDim.x) {
    const Span s = span_of(a, i);
    if ((s.begin / SEQUENCE_BLOCK + 1) * SEQUENCE_BLOCK >= s.end) continue;      // (uniform)
    const P p = wg_sum(share_of<P>(a, s, i), at);
    if (threadIdx.x == 0) ((P*)a.head)[i] = p;
  }
}
template <class P> __device__ __forceinline__ void leave(const SequenceArgs& a, const P& p) {
  if (threadIdx.x != 0) return;
  if (!is_block(a)) ((P*)a.head)[blockIdx.x] = p;
  else ((P*)a.block)[blockIdx.x - a.count] = p;
}
static_assert(SEQUENCE_BLOCK == 256 * U, "a piece is one batch of a workgroup");

__global__ void __launch_bounds__(256) preference_sum_kernel(SequenceArgs a) {
  __shared__ PrefPart at[4];
  __shared__ int found[4];
  Batch b;
  if (is_block(a)) load<false>(a, block_begin(a) + threadIdx.x, a.n, 256, &b);       // (ahead of the search for its sequence)
  const Job j = job_of(a, found);
  if (j.seq < 0) return;
  const long t = j.begin + threadIdx.x;
  if (!is_block(a) && j.begin < j.end) load<false>(a, t, j.end, 256, &b);
  PrefPart p{};
  sum_pref(b, t, j.end, 256, &p);
  leave(a, wg_sum(p, at));
}
__global__ void __launch_bounds__(256) preference_grad_kernel(SequenceArgs a) {
  __shared__ PrefPart at[4];
  __shared__ int found[4];
  long label[U];
  if (is_block(a)) load_labels(a, block_begin(a) + threadIdx.x, a.n, 256, label);
  const Job j = job_of(a, found);
  if (j.seq < 0) return;
  const long t = j.begin + threadIdx.x;
  if (!is_block(a) && j.begin < j.end) load_labels(a, t, j.end, 256, label);
  const long pairs = a.count / 2, i = j.seq < pairs ? j.seq : j.seq - pairs;
  PrefPart pc = share_of<PrefPart>(a, span_of(a, i), i);
  pc.s -= share_of<PrefPart>(a, span_of(a, pairs + i), pairs + i).s;
  const double margin = wg_sum(pc, at).s;
  double slope;
  const double loss = pair_loss(a, margin, &slope);
  if (blockIdx.x < pairs && threadIdx.x == 0) {
    a.loss[i] = (float)loss;
    if (a.margin) a.margin[i] = (float)margin;
  }
  if (!a.d_nll) return;
  const float d = (float)(slope * (double)a.d_loss[i]);
  put_pref(a, label, t, j.end, 256, j.seq < pairs ? -d : d);
}
__global__ void __launch_bounds__(256) policy_sum_kernel(SequenceArgs a) {
  __shared__ PolicyPart at[4];
  __shared__ int found[4];
  Batch b;
  if (is_block(a)) load<true>(a, block_begin(a) + threadIdx.x, a.n, 256, &b);
  const Job j = job_of(a, found);
  if (j.seq < 0) return;
  const long t = j.begin + threadIdx.x;
  if (!is_block(a) && j.begin < j.end) load<true>(a, t, j.end, 256, &b);
  const float adv = a.per_token ? 0.f : a.adv[j.seq], d = a.d_nll ? a.d_loss[j.seq] : 0.f;
  PolicyPart p{};
  do_policy(a, b, t, j.end, 256, adv, d, &p);
  leave(a, wg_sum(p, at));
}
// The sequences' losses, and (mean) the gradients divided by the tokens' number
__global__ void __launch_bounds__(256) policy_finish_kernel(SequenceArgs a) {
  __shared__ PolicyPart at[4];
  __shared__ int found[4];
  const Job j = job_of(a, found);
  if (j.seq < 0) return;
  const PolicyPart p = wg_sum(share_of<PolicyPart>(a, span_of(a, j.seq), j.seq), at);
  if (!is_block(a) && threadIdx.x == 0) put_stats(a, j.seq, p);
  if (!a.d_nll || !a.mean || p.count == 0 || j.begin == j.end) return;
  scale_policy(a, j.begin + threadIdx.x, j.end, 256, 1.0 / p.count);
}

// Up to ONE_TOKENS one launch.  us in one launch and in two, preferences / policies: 32768 tokens in 16 sequences alike 7.9 / 7.7 and 7.5 / 9.1, in 512 4.9 / 4.7 and 7.6 / 7.6,
// in 2 17 / 22 and 7.8 / 9.1; 65536 in 16 8.3 / 9.4 and 7.7 / 9.4, in 512 5.1 / 5.0 and 7.7 / 7.7, in 2 29 / 40 and 7.9 / 9.2.  One launch has no bound where
// lengths differ: 32768 tokens in 2048 sequences, of which one has half, 64 / 138 and 15 / 17; 524288 in 512, of which one has half, 104 / 748 and 11 / 13, alike 8.4 / 6.9 and 8.2 / 9.9.
constexpr long ONE_TOKENS = 32768, LONG_TOKENS = 1L << 24;
// Threads for a sequence (or pair) of `per` tokens on average.  us with 64, 256 and 1024, policies of 32768 tokens: per = 16 5.1, 8.9, 36; 64 4.2, 4.7, 10; 256 5.0, 4.8, 5.9; 1024
// 11, 5.8, 7.1; 2048 20, 8.1, 7.7; 8192 70, 22, 14.
unsigned threads_for(long per) { return per >= 2048 ? 1024 : per >= 64 ? 256 : 64; }
// The launch between those of more tokens, where sequences may be long; a piece or more a sequence on average, or so many tokens that one long sequence among
// short ones would cost more than the launch.  us without and with it, preferences / policies, of 2^24 tokens: two sequences 193 / 220 and 87 / 123, 4096 116 / 146 and
// 113 / 155, 4096 of which one has half of the tokens 136 / 188 and 115 / 147, 65536 of these (then it is left out) 354 / 396 and 364 / 460; of 2^26: two 2118 / 2345 and
// 337 / 447, 65536 644 / 668 and 658 / 689, one of them with half 1156 / 1680 and 742 / 869; of 2^27: two 7760 / 8660 and 650 / 870.  (2^22: two 39 / 48 and 34 / 47, 256 36 / 44 and 37 / 47.)
template <class P> void total(SequenceArgs* a, hipStream_t s) {
  if (a->n < LONG_TOKENS || (a->n < 4 * LONG_TOKENS && a->n / a->count < SEQUENCE_BLOCK)) return;
  const unsigned wg = a->n / a->count >= 256 * SEQUENCE_BLOCK ? 1024 : 256;
  sequence_total_kernel<P><<<(unsigned)std::min(a->count, 1L << 16), wg, 0, s>>>(*a);
  a->totals = 1;
}

}  // namespace

size_t sequence_part_bytes() { return sizeof(PolicyPart); }

hipError_t launch_preference(SequenceArgs a, hipStream_t s) {
  const long pairs = a.count / 2;
  if (a.n <= ONE_TOKENS) {
    preference_one_kernel<<<(unsigned)std::min(pairs, 1L << 20), threads_for(a.n / pairs), 0, s>>>(a);
    return hipGetLastError();
  }
  const unsigned all = (unsigned)(a.count + (a.n + SEQUENCE_BLOCK - 1) / SEQUENCE_BLOCK);
  preference_sum_kernel<<<all, 256, 0, s>>>(a);
  total<PrefPart>(&a, s);
  preference_grad_kernel<<<a.d_nll ? all : (unsigned)pairs, 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_policy(SequenceArgs a, hipStream_t s) {
  if (a.n <= ONE_TOKENS) {
    policy_one_kernel<<<(unsigned)std::min(a.count, 1L << 20), threads_for(a.n / a.count), 0, s>>>(a);
    return hipGetLastError();
  }
  const unsigned all = (unsigned)(a.count + (a.n + SEQUENCE_BLOCK - 1) / SEQUENCE_BLOCK);
  policy_sum_kernel<<<all, 256, 0, s>>>(a);
  total<PolicyPart>(&a, s);
  policy_finish_kernel<<<a.d_nll && a.mean ? all : (unsigned)a.count, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace lvx
