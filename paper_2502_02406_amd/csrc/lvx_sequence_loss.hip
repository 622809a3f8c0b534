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
// second adds up those of its sequence, in order, and does what hangs on them.  No atomics: results repeat bit for bit.
#include "lvx_internal.h"

#include <algorithm>
#include <type_traits>

namespace lvx {

namespace {

struct PrefPart {
  double s;
  __device__ void add(const PrefPart& o) { s += o.s; }
};
struct PolicyPart {
  double loss, kl;
  int count, clipped;
  __device__ void add(const PolicyPart& o) { loss += o.loss; kl += o.kl; count += o.count; clipped += o.clipped; }
};
template <class P> __device__ __forceinline__ P from_lane(const P& x, int o) {
  P y;
  const int* const a = (const int*)&x;
  int* const b = (int*)&y;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(P) / 4); ++i) b[i] = __shfl_xor(a[i], o);
  return y;
}
// Sums over the workgroup, the same in every thread (`at`: a place a wave in LDS)
template <class P> __device__ __forceinline__ P wg_sum(P x, P* at) {
#pragma unroll
  for (int o = 1; o < 64; o *= 2) x.add(from_lane(x, o));
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

// ---- a token ----
__device__ __forceinline__ void token_pref(const SequenceArgs& a, long i, PrefPart* p) {
  const bool on = a.labels[i] >= 0;
  const float nll = a.nll[i], ref = a.ref ? a.ref[i] : 0.f;
  p->s += on ? (double)ref - (double)nll : 0.0;
}
// adv: the sequence's advantage.  Returns the gradient of the token's loss (0 without a label).
__device__ __forceinline__ double token_policy(const SequenceArgs& a, long i, float adv, PolicyPart* p) {
  const bool on = a.labels[i] >= 0;
  const double nll = a.nll[i], old = a.old[i], ref = a.beta != 0.0 ? a.ref[i] : 0.f, A = a.per_token ? a.adv[i] : adv;
  if (!on) return 0.0;
  const double gone = old - nll;
  const double ratio = exp(gone);
  // (by logarithms, of which the difference is exact)
  const bool over = A > 0.0 ? gone > a.ln_high : A < 0.0 && gone < a.ln_low;
  double loss = over ? -(A > 0.0 ? a.high : a.low) * A : -ratio * A, slope = over ? 0.0 : ratio * A;
  if (a.beta != 0.0) {
    const double d = nll - ref, up = expm1(d);
    loss += a.beta * (up - d);
    slope += a.beta * up;
    p->kl += up - d;
  }
  p->loss += loss;
  p->count += 1;
  p->clipped += over;
  return slope;
}

// ---- a pair ----
__device__ __forceinline__ double pair_loss(const SequenceArgs& a, double margin, double* slope) {
  const double h = a.beta * margin;
  if (a.form == LVX_PREF_LOGISTIC) {
    const double e = exp(-fabs(h)), soft = log1p(e), q = a.smoothing;
    *slope = a.beta * ((h >= 0.0 ? 1.0 : e) / (1.0 + e) - (1.0 - q));
    return (1.0 - q) * (soft + (h < 0.0 ? -h : 0.0)) + q * (soft + (h > 0.0 ? h : 0.0));
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
__global__ void __launch_bounds__(1024) preference_one_kernel(SequenceArgs a) {
  __shared__ PrefPart at[16];
  const long pairs = a.count / 2, wg = blockDim.x;
  for (long i = blockIdx.x; i < pairs; i += gridDim.x) {
    const Span c = span_of(a, i), r = span_of(a, pairs + i);
    PrefPart pc{}, pr{};
#pragma unroll 4
    for (long t = c.begin + threadIdx.x; t < c.end; t += wg) token_pref(a, t, &pc);
#pragma unroll 4
    for (long t = r.begin + threadIdx.x; t < r.end; t += wg) token_pref(a, t, &pr);
    pc.s -= pr.s;
    const double margin = wg_sum(pc, at).s;
    double slope;
    const double loss = pair_loss(a, margin, &slope);
    if (threadIdx.x == 0) {
      a.loss[i] = (float)loss;
      if (a.margin) a.margin[i] = (float)margin;
    }
    if (!a.d_nll) continue;
    const float d = (float)(slope * (double)a.d_loss[i]);
#pragma unroll 4
    for (long t = c.begin + threadIdx.x; t < c.end; t += wg) a.d_nll[t] = a.labels[t] >= 0 ? -d : 0.f;
#pragma unroll 4
    for (long t = r.begin + threadIdx.x; t < r.end; t += wg) a.d_nll[t] = a.labels[t] >= 0 ? d : 0.f;
  }
}
__global__ void __launch_bounds__(1024) policy_one_kernel(SequenceArgs a) {
  __shared__ PolicyPart at[16];
  const long wg = blockDim.x;
  for (long i = blockIdx.x; i < a.count; i += gridDim.x) {
    const Span c = span_of(a, i);
    const float adv = a.per_token ? 0.f : a.adv[i], d = a.d_nll ? a.d_loss[i] : 0.f;
    PolicyPart p{};
    for (long t = c.begin + threadIdx.x; t < c.end; t += wg) {
      const double slope = token_policy(a, t, adv, &p);
      if (a.d_nll) a.d_nll[t] = (float)(a.labels[t] >= 0 ? slope * (double)d : 0.0);
    }
    p = wg_sum(p, at);
    if (threadIdx.x == 0) put_stats(a, i, p);
    if (!a.d_nll || !a.mean || p.count == 0) continue;
    const float per = (float)(1.0 / p.count);
    for (long t = c.begin + threadIdx.x; t < c.end; t += wg) a.d_nll[t] *= per;      // (what this thread has written)
  }
}

// ---- more tokens: a piece of a sequence a workgroup ----

// Workgroups 0 .. count - 1: a sequence up to the first multiple of SEQUENCE_BLOCK behind its start; the others: from a multiple on, where it is inside
// a sequence.  (seq < 0: nothing)
struct Job { long seq, begin, end; };
__device__ __forceinline__ Job job_of(const SequenceArgs& a, int* lds) {
  constexpr long P = SEQUENCE_BLOCK;
  const long b = blockIdx.x;
  if (b < a.count) {
    const Span s = span_of(a, b);
    return {b, s.begin, min(s.end, (s.begin / P + 1) * P)};
  }
  const long x = (b - a.count) * P;
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
  for (long j = s.begin / SEQUENCE_BLOCK + 1 + threadIdx.x; j * SEQUENCE_BLOCK < s.end; j += 256) p.add(((const P*)a.block)[j]);
  return p;
}
template <class P> __device__ __forceinline__ void leave(const SequenceArgs& a, const P& p) {
  if (threadIdx.x != 0) return;
  if (blockIdx.x < a.count) ((P*)a.head)[blockIdx.x] = p;
  else ((P*)a.block)[blockIdx.x - a.count] = p;
}

__global__ void __launch_bounds__(256) preference_sum_kernel(SequenceArgs a) {
  __shared__ PrefPart at[4];
  __shared__ int found[4];
  const Job j = job_of(a, found);
  if (j.seq < 0) return;
  PrefPart p{};
#pragma unroll 8
  for (long t = j.begin + threadIdx.x; t < j.end; t += 256) token_pref(a, t, &p);
  leave(a, wg_sum(p, at));
}
__global__ void __launch_bounds__(256) preference_grad_kernel(SequenceArgs a) {
  __shared__ PrefPart at[4];
  __shared__ int found[4];
  const Job j = job_of(a, found);
  if (j.seq < 0) return;
  const long pairs = a.count / 2, i = j.seq < pairs ? j.seq : j.seq - pairs;
  if (i >= pairs) return;
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
  float d = (float)(slope * (double)a.d_loss[i]);
  if (j.seq < pairs) d = -d;
#pragma unroll 8
  for (long t = j.begin + threadIdx.x; t < j.end; t += 256) a.d_nll[t] = a.labels[t] >= 0 ? d : 0.f;
}
__global__ void __launch_bounds__(256) policy_sum_kernel(SequenceArgs a) {
  __shared__ PolicyPart at[4];
  __shared__ int found[4];
  const Job j = job_of(a, found);
  if (j.seq < 0) return;
  const float adv = a.per_token ? 0.f : a.adv[j.seq], d = a.d_nll ? a.d_loss[j.seq] : 0.f;
  PolicyPart p{};
  for (long t = j.begin + threadIdx.x; t < j.end; t += 256) {
    const double slope = token_policy(a, t, adv, &p);
    if (a.d_nll) a.d_nll[t] = (float)(a.labels[t] >= 0 ? slope * (double)d : 0.0);
  }
  leave(a, wg_sum(p, at));
}
// The sequences' losses, and (mean) the gradients divided by the tokens' number
__global__ void __launch_bounds__(256) policy_finish_kernel(SequenceArgs a) {
  __shared__ PolicyPart at[4];
  __shared__ int found[4];
  const Job j = job_of(a, found);
  if (j.seq < 0) return;
  const PolicyPart p = wg_sum(share_of<PolicyPart>(a, span_of(a, j.seq), j.seq), at);
  if (blockIdx.x < a.count && threadIdx.x == 0) put_stats(a, j.seq, p);
  if (!a.d_nll || !a.mean || p.count == 0) return;
  const float per = (float)(1.0 / p.count);
#pragma unroll 8
  for (long t = j.begin + threadIdx.x; t < j.end; t += 256) a.d_nll[t] *= per;
}

constexpr long ONE_TOKENS = 32768;
// Threads for a sequence (or pair) of `per` tokens on average
unsigned threads_for(long per) { return per >= 2048 ? 1024 : per >= 64 ? 256 : 64; }

}  // namespace

size_t sequence_part_bytes() { return sizeof(PolicyPart); }

hipError_t launch_preference(const SequenceArgs& a, hipStream_t s) {
  const long pairs = a.count / 2;
  if (a.n <= ONE_TOKENS) {
    preference_one_kernel<<<(unsigned)std::min(pairs, 1L << 20), threads_for(a.n / pairs), 0, s>>>(a);
    return hipGetLastError();
  }
  const unsigned all = (unsigned)(a.count + (a.n + SEQUENCE_BLOCK - 1) / SEQUENCE_BLOCK);
  preference_sum_kernel<<<all, 256, 0, s>>>(a);
  preference_grad_kernel<<<a.d_nll ? all : (unsigned)pairs, 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_policy(const SequenceArgs& a, hipStream_t s) {
  if (a.n <= ONE_TOKENS) {
    policy_one_kernel<<<(unsigned)std::min(a.count, 1L << 20), threads_for(a.n / a.count), 0, s>>>(a);
    return hipGetLastError();
  }
  const unsigned all = (unsigned)(a.count + (a.n + SEQUENCE_BLOCK - 1) / SEQUENCE_BLOCK);
  policy_sum_kernel<<<all, 256, 0, s>>>(a);
  policy_finish_kernel<<<a.d_nll && a.mean ? all : (unsigned)a.count, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace lvx
