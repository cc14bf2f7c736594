// Expert gating: router logits -> scores, choice values, groups, top-k, weights.
//
//   s = softmax(l) or 1 / (1 + exp(-l)),  c = s + bias,
//   ids = top k of c inside the best groups (a group is worth its best 1 or 2 c),
//   w = s[ids] (/ sum) * scale.
//
// One warp per token; lane i holds experts i E .. i E + E - 1 in registers (E =
// 2 .. 32 for N up to 1024, in steps that leave 22 lanes or more in use above N = 64), so
// that among equal values the lowest lane and then its lowest register is the lowest
// index.  The top-k works on order-preserving integer keys: k warp-wide maxima (redux) of
// the lanes' best two give a bound, the few values above it are ranked by counting.  What
// bounds it: latency for few tokens, issue for many; the logits are read once.
//
// fp32 scores carry an error, and two choice values nearer than that would come
// out in an order that depends on the rounding of expf.  Where there is a bias (or
// a group is worth a sum) the kernel looks at the gaps that decided: between
// successive winners, the last winner and the next, any group taken and any left.
// A row with a gap below the error bound is evaluated again in pairs of fp32 values
// (two_float.cuh; fp64 took twice as long on this GPU): the candidates alone where that is enough, else the
// row by way of shared memory.  One such warp sets the time of a small batch (89 rows of 944 experts, softmax
// with a bias, 4 groups: 28 us with one, 11 without).  Without
// a bias s grows with l and the logits themselves are compared, exactly.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cfloat>
#include <cstring>
#include <type_traits>

#include "ops_internal.cuh"
#include "two_float.cuh"

namespace xs {
namespace {

constexpr int kWarps = 4;
constexpr uint32_t kAll = 0xffffffffu;

struct GateParams {
  GateArgs a;
  int dtype;
  int gs;             // experts per group
  uint32_t magic;     // ceil(2^21 / gs): e / gs == (e * magic) >> 21 for e < 1024
  int group_shift;    // 2^group_shift lanes hold a group in their registers; -1: groups are not so many whole lanes
  int scan_shift;     // 2^scan_shift lanes scan a group in shared memory
  bool vec, vec_bias; // rows, the bias are whole words of load_values()
};

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }

// Order-preserving keys; every number but NaN has a key above 0.  -0 is +0.
__device__ __forceinline__ uint32_t key_of(float v) {
  const uint32_t u = __float_as_uint(v + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}
using Key64 = unsigned long long;
__device__ __forceinline__ Key64 key_of(Two v) { return static_cast<Key64>(key_of(v.hi)) << 32 | key_of(v.lo); }
__device__ __forceinline__ Two two_of(Key64 key) {
  return Two{value_of(static_cast<uint32_t>(key >> 32)), value_of(static_cast<uint32_t>(key))};
}
__device__ __forceinline__ uint32_t warp_max(uint32_t k) { return __reduce_max_sync(kAll, k); }
__device__ __forceinline__ Key64 warp_max(Key64 k) {
  const uint32_t hi = static_cast<uint32_t>(k >> 32), top = __reduce_max_sync(kAll, hi);
  const uint32_t lo = __reduce_max_sync(kAll, hi == top ? static_cast<uint32_t>(k) : 0u);
  return static_cast<Key64>(top) << 32 | lo;
}

// What the choice orders: fp32 values, or in the second look the keys of pairs.
__device__ __forceinline__ float shfl_xor(float v, int o) { return __shfl_xor_sync(kAll, v, o); }
__device__ __forceinline__ Key64 shfl_xor(Key64 v, int o) { return __shfl_xor_sync(kAll, v, o); }
template <class V>
__device__ __forceinline__ V lowest();
template <>
__device__ __forceinline__ float lowest<float>() { return -INFINITY; }
template <>
__device__ __forceinline__ Key64 lowest<Key64>() { return 0x007fffff80000000ull; }   // of -infinity and 0
// a + b for choice values: a sum that overflows or has an infinite part is infinite (the
// residuals of a pair would be NaN).
__device__ __forceinline__ Two add_any(Two a, Two b) {
  const float s = a.hi + b.hi;
  return fabsf(s) == INFINITY ? Two{s, 0.f} : a + b;
}
// A group's worth: its best, or the sum of its best two if there are two.
__device__ __forceinline__ float worth_of(float top, float second, bool both) { return both ? top + second : top; }
__device__ __forceinline__ Key64 worth_of(Key64 top, Key64 second, bool both) {
  return both ? key_of(add_any(two_of(top), two_of(second))) : top;
}

template <class V>
__device__ __forceinline__ void take(V x, V *top, V *second) {
  const V less = x < *top ? x : *top;
  *top = x > *top ? x : *top;
  *second = less > *second ? less : *second;
}

// The best two values of the lanes' parts of their group become those of the group.
template <class V>
__device__ __forceinline__ void join_best(int shift, V *top, V *second) {
  for (int o = 1; o < 1 << shift; o <<= 1) {
    const V t2 = shfl_xor(*top, o), s2 = shfl_xor(*second, o);
    take(t2, top, second);
    if (s2 > *second) *second = s2;
  }
}

// The best two of group lane >> scan_shift from the experts' values in shared memory.
template <class V>
__device__ __forceinline__ void scan_group(const GateParams &p, const V *v, V *top, V *second) {
  const int lane = threadIdx.x & 31, shift = p.scan_shift, g = lane >> shift, sub = lane & ((1 << shift) - 1);
  *top = *second = lowest<V>();
  if (g < p.a.prm.n_groups && sub < p.gs) {
    const int n = (p.gs - sub + (1 << shift) - 1) >> shift;
    // Groups start at different places: those of a multiple of 32 values would
    // otherwise all be in the same bank.
    const V *from = v + g * p.gs + sub;
    const int first = min(g, n - 1);
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
      const int at = first + i < n ? first + i : first + i - n;
      take(from[at << shift], top, second);
    }
  }
  join_best(shift, top, second);
}

// The token's best groups (bit g) from the best two values of group lane >> shift, -infinity
// for experts that are not eligible.
__device__ __forceinline__ uint32_t best_groups(const GateParams &p, float top, float second, int shift) {
  const int lane = threadIdx.x & 31;
  const float worth = worth_of(top, second, p.a.prm.group_top == 2 && second > -INFINITY);
  uint32_t key = top > -INFINITY ? key_of(worth) : 0u, taken = 0;
  for (int r = 0; r < p.a.prm.top_groups; ++r) {
    const uint32_t best = warp_max(key);
    if (best == 0) break;
    const int g = (__ffs(__ballot_sync(kAll, key == best)) - 1) >> shift;
    taken |= 1u << g;
    if (lane >> shift == g) key = 0;
  }
  return taken;
}
// Whether fp32 leaves the choice of groups `taken` open: whether some group taken may be worth less
// than some group left.  Each worth is off by what its own values' size gives, which a sum of two does not
// show (s + 1000 and s' - 1000 add up to s + s'), and two groups' scores by `slack` against each
// other.  A value rounds by 2^-24 of itself where the bias is added, a sum of two by 2^-24 of
// at most twice the larger: 2^-23 of the value, 2^-22 of the larger one and, with as much again to spare, 2^-21.
__device__ __forceinline__ bool groups_near(const GateParams &p, float top, float second, int shift, uint32_t taken,
                                            float slack) {
  const int lane = threadIdx.x & 31;
  const bool any = top > -INFINITY, both = p.a.prm.group_top == 2 && second > -INFINITY;
  const bool in = any && (taken >> (lane >> shift)) & 1u;
  const float worth = worth_of(top, second, both);
  const float size = fminf(fmaxf(fabsf(top), both ? fabsf(second) : 0.f), FLT_MAX);
  const float off = size * (both ? 0x1p-21f : 0x1p-23f);
  const uint32_t least = __reduce_min_sync(kAll, in ? key_of(__fsub_rd(worth, off)) : kAll);
  const uint32_t most = __reduce_max_sync(kAll, any && !in ? key_of(__fadd_ru(worth, off)) : 0u);
  // (Infinite worths on both sides leave NaN: near.)
  return most != 0 && !(__fsub_rd(value_of(least), value_of(most)) >= (p.a.prm.group_top == 2 ? 2.f * slack : slack));
}

// Lane r gets the r-th best (r < rounds) of the values c, -1 where none above -infinity is left.
template <int kE>
__device__ __noinline__ int best_experts(const float (&c)[kE], int rounds) {
  const int lane = threadIdx.x & 31;
  const uint32_t none = key_of(-INFINITY);
  uint32_t key[kE], kb = none;
  int jb = 0;
#pragma unroll
  for (int j = 0; j < kE; ++j) {
    key[j] = key_of(c[j]);
    if (key[j] > kb) {
      kb = key[j];
      jb = j;
    }
  }
  int id = -1;
  for (int r = 0; r < rounds; ++r) {
    const uint32_t best = warp_max(kb);
    if (best == none) break;
    const int src = __ffs(__ballot_sync(kAll, kb == best)) - 1;
    const int e = __shfl_sync(kAll, lane * kE + jb, src);
    if (lane == r) id = e;
    if (lane == src) {
      const int out = jb;
      kb = none;
      jb = 0;
#pragma unroll
      for (int j = 0; j < kE; ++j) {
        if (j == out) key[j] = none;
        if (key[j] > kb) {
          kb = key[j];
          jb = j;
        }
      }
    }
  }
  return id;
}

// The same, quicker.  The rounds-th largest of the lanes' best two values each bounds the
// winners from below (as many values are not smaller), so hardly more than `rounds` values are
// candidates; they are gathered in shared memory, one per lane, and each counts who is before
// it.  A round of the loop above costs a rescan of kE registers, here a maximum.  More
// than 32 candidates (many equal values) take the loop.  (With the lanes' maxima alone a third of the rows
// of 944 experts had more than 32 at k = 15.)
struct Candidates {
  uint2 of[32];     // key, expert
  Key64 key[32];    // see rank_keys()
  Key64 tie[32];
  int order[32];
};

// *n: the candidates (above 32: not gathered); *bound: no other value reaches it.
template <int kE>
__device__ __forceinline__ int best_of(const float (&c)[kE], int rounds, Candidates *sh, int *n_out, float *bound) {
  const int lane = threadIdx.x & 31;
  const uint32_t none = key_of(-INFINITY), below = (1u << lane) - 1u;
  uint32_t key[kE], top = none, second = none;
#pragma unroll
  for (int j = 0; j < kE; ++j) {
    key[j] = key_of(c[j]);
    second = max(second, min(top, key[j]));
    top = max(top, key[j]);
  }
  uint32_t least = none + 1;
  for (int r = 0; r < rounds; ++r) {
    const uint32_t best = warp_max(top);
    least = best;
    if (best == none) break;
    // (Equal values of several lanes go in one round: the bound is lower than it has to be.)
    if (top == best) {
      top = second;
      second = none;
    }
  }
  // Fewer values than rounds among the lanes' best two: every one counts.
  *bound = least == none ? -INFINITY : value_of(least);
  least = max(least, none + 1);
  int n = 0;
  __syncwarp();
#pragma unroll
  for (int j = 0; j < kE; ++j) {
    const bool in = key[j] >= least;
    const uint32_t lanes = __ballot_sync(kAll, in);
    const int at = n + __popc(lanes & below);
    if (in && at < 32) sh->of[at] = make_uint2(key[j], lane * kE + j);
    n += __popc(lanes);
  }
  *n_out = n;
  if (n > 32) return best_experts<kE>(c, rounds);
  __syncwarp();
  const uint2 mine = sh->of[lane];
  int rank = 0;
#pragma unroll 4
  for (int r = 0; r < n; ++r) {
    const uint2 o = sh->of[r];
    rank += o.x > mine.x || (o.x == mine.x && o.y < mine.y);
  }
  if (lane < n) sh->order[rank] = mine.y;
  __syncwarp();
  return lane < n && lane < rounds ? sh->order[lane] : -1;
}

// The fp32 score of a logit, given the largest logit and the sum of the row's
// exponentials (softmax).
__device__ __forceinline__ float score_of(bool softmax, float l, float m, float sum) {
  if (softmax) return expf(l - m) * (1.f / sum);
  // e^-|l|, so that no score of a large negative logit is lost to an overflow.  The
  // quick reciprocal of a number between 1 and 2 and one Newton step: 1 ulp, without the
  // division's branches.
  const float e = expf(-fabsf(l)), d = 1.f + e;
  float r = __fdividef(1.f, d);
  r = fmaf(r, fmaf(-d, r, 1.f), r);
  return l >= 0.f ? r : e * r;
}

// A lane's kE values from row[lane kE], as words if the row is whole words (976 experts, 1254 rows:
// 19.4 us element by element, 16 so).
template <int kBytes>
using WordOf = std::conditional_t<kBytes % 16 == 0, uint4, std::conditional_t<kBytes % 8 == 0, uint2,
                                  std::conditional_t<kBytes % 4 == 0, uint32_t, uint16_t>>>;
template <int kE, class T>
__device__ __forceinline__ void load_values(const T *row, int N, bool vec, float (&v)[kE]) {
  const int e0 = (threadIdx.x & 31) * kE;
  T raw[kE];
  if (vec) {
    constexpr int kBytes = kE * sizeof(T);
    using W = WordOf<kBytes>;
    const W *src = reinterpret_cast<const W *>(row + e0);
#pragma unroll
    for (int i = 0; i < kBytes / static_cast<int>(sizeof(W)); ++i)
      if (e0 + i * static_cast<int>(sizeof(W) / sizeof(T)) < N) {   // N is whole words
        const W w = src[i];
        memcpy(reinterpret_cast<char *>(raw) + i * sizeof(W), &w, sizeof(W));
      }
  } else {
#pragma unroll
    for (int j = 0; j < kE; ++j)
      if (e0 + j < N) raw[j] = row[e0 + j];
  }
#pragma unroll
  for (int j = 0; j < kE; ++j) v[j] = e0 + j < N ? to_float(raw[j]) : 0.f;
}

// A lane's logits and biases of row t, 0 where there is none.
template <int kE>
__device__ __forceinline__ void load_row(const GateParams &p, int t, float (&l)[kE], float (&bias)[kE]) {
  const GateArgs &a = p.a;
  const size_t at = static_cast<size_t>(t) * a.N;
  if (p.dtype == XS_F32)
    load_values<kE>(static_cast<const float *>(a.logits) + at, a.N, p.vec, l);
  else if (p.dtype == XS_BF16)
    load_values<kE>(static_cast<const __nv_bfloat16 *>(a.logits) + at, a.N, p.vec, l);
  else
    load_values<kE>(static_cast<const __half *>(a.logits) + at, a.N, p.vec, l);
  if (a.bias != nullptr) {
    load_values<kE>(a.bias, a.N, p.vec_bias, bias);
  } else {
#pragma unroll
    for (int j = 0; j < kE; ++j) bias[j] = 0.f;
  }
}

__device__ __forceinline__ float logit_at(const GateParams &p, int t, int e) {
  const size_t at = static_cast<size_t>(t) * p.a.N + e;
  if (p.dtype == XS_F32) return static_cast<const float *>(p.a.logits)[at];
  if (p.dtype == XS_BF16) return to_float(static_cast<const __nv_bfloat16 *>(p.a.logits)[at]);
  return to_float(static_cast<const __half *>(p.a.logits)[at]);
}
// Whether expert e is eligible for token t, its logit and bias.
__device__ __forceinline__ bool look_up(const GateParams &p, int t, int e, float *l, float *b) {
  const float v = logit_at(p, t, e);
  *l = fminf(v, FLT_MAX);
  *b = p.a.bias != nullptr ? p.a.bias[e] : 0.f;
  return v > -INFINITY && *b > -INFINITY && (p.a.expert_mask == nullptr || p.a.expert_mask[e] != 0);
}

// What decides between equal pairs of choice values with a bias: the larger bias, then the larger
// logit.  A pair loses what lies below its last bit or below fp32's range, of a sigmoid near 0 (e^l), near 1
// (1 - e^-l) or of a softmax; with the same bias the logits tell which lost more, and of
// equal sums the one with the larger bias has the smaller score, which lost more upwards.  So a bias of
// zeros leaves the order of no bias.  Infinite values are equal.
__device__ __forceinline__ Key64 tie_of(const GateParams &p, int t, int e, Key64 key) {
  if (p.a.bias == nullptr || static_cast<uint32_t>(key >> 32) == key_of(INFINITY)) return 0;
  return static_cast<Key64>(key_of(p.a.bias[e])) << 32 | key_of(fminf(logit_at(p, t, e), FLT_MAX));
}

// The order of the n candidates in `sh` by key and tie, in lane i < n those of the i-th: lane r gets the r-th expert.
__device__ __forceinline__ int rank_keys(Candidates *sh, int n, Key64 key, Key64 tie) {
  const int lane = threadIdx.x & 31, id = lane < n ? static_cast<int>(sh->of[lane].y) : 0;
  sh->key[lane] = key;
  sh->tie[lane] = tie;
  __syncwarp();
  int rank = 0;
#pragma unroll 1
  for (int r = 0; r < n; ++r) {
    const Key64 o = sh->key[r], u = sh->tie[r];
    rank += o > key || (o == key && (u > tie || (u == tie && static_cast<int>(sh->of[r].y) < id)));
  }
  if (lane < n) sh->order[rank] = id;
  __syncwarp();
  return lane < n ? sh->order[lane] : -1;
}

// The second look takes kBatch experts of a lane at a time, e, e + 32, ..., looked up before any
// arithmetic: a pair's exponential is a chain of 200 operations, so several run side by side.
constexpr int kBatch = 4;
__device__ __forceinline__ uint32_t look_up_batch(const GateParams &p, int t, int e, float m, float (&l)[kBatch],
                                                  float (&b)[kBatch]) {
  uint32_t ok = 0;
#pragma unroll
  for (int j = 0; j < kBatch; ++j) {
    l[j] = m;
    b[j] = 0.f;
    if (e + 32 * j < p.a.N) {
      float v;
      if (look_up(p, t, e + 32 * j, &v, &b[j])) {
        ok |= 1u << j;
        l[j] = v;
      }
    }
  }
  return ok;
}

// Whether an expert of the groups `taken` comes within `limit` of the choice value v (logit l0, bias b0)
// without being its equal.  For rows where the last winner and the next are equal: the ones behind
// them may still be larger in truth.
__device__ __noinline__ bool border_near(const GateParams &p, int t, float m, float sum, uint32_t taken, float v, float l0,
                                         float b0, float limit) {
  const int lane = threadIdx.x & 31;
  const bool softmax = p.a.prm.scoring == XS_SCORE_SOFTMAX;
  bool near = false;
#pragma unroll 1
  for (int e = lane; e - lane < p.a.N; e += 32 * kBatch) {
    float l[kBatch], b[kBatch];
    const uint32_t ok = look_up_batch(p, t, e, m, l, b);
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const bool in = (ok >> j) & 1u && (taken >> ((static_cast<uint32_t>(e + 32 * j) * p.magic) >> 21)) & 1u;
      near |= in && fabsf(v - (score_of(softmax, l[j], m, sum) + b[j])) < limit && !(l[j] == l0 && b[j] == b0);
    }
  }
  return __any_sync(kAll, near);
}

// 1 / the sum of a row's exponentials, m: the largest logit; sv: nullable, where they are left.
__device__ __noinline__ Two row_scale(const GateParams &p, int t, float m, Two *sv) {
  const int lane = threadIdx.x & 31;
  Two sum{0.f, 0.f};
#pragma unroll 1
  for (int e = lane; e - lane < p.a.N; e += 32 * kBatch) {
    float l[kBatch], b[kBatch];
    const uint32_t ok = look_up_batch(p, t, e, m, l, b);
    Two x[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) x[j] = two_exp_diff(l[j], m);
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const bool in = (ok >> j) & 1u;
      sum = sum + Two{in ? x[j].hi : 0.f, in ? x[j].lo : 0.f};
      if (sv != nullptr && in) sv[e + 32 * j] = x[j];
    }
  }
#pragma unroll 1
  for (int o = 16; o > 0; o >>= 1) sum = sum + Two{shfl_xor(sum.hi, o), shfl_xor(sum.lo, o)};
  return sum.hi > 0.f ? Two{1.f, 0.f} / sum : Two{0.f, 0.f};
}

// The order of the n candidates that best_of() left in `sh`, in pairs.  For choices with
// a bias, among experts whose groups are not in doubt.
__device__ __noinline__ int near_row(const GateParams &p, int t, float m, int n, Candidates *sh) {
  const int lane = threadIdx.x & 31;
  const bool softmax = p.a.prm.scoring == XS_SCORE_SOFTMAX;
  const int id = lane < n ? static_cast<int>(sh->of[lane].y) : 0;
  const float l = lane < n ? fminf(logit_at(p, t, id), FLT_MAX) : m;
  const Two s = softmax ? two_exp_diff(l, m) * row_scale(p, t, m, nullptr) : two_sigmoid(l);
  const Key64 key = key_of(add_any(s, Two{p.a.bias[id], 0.f}));
  return rank_keys(sh, n, key, tie_of(p, t, id, key));
}

// The logits of the best two experts of group lane >> scan_shift by their choice values' pairs, key[e], and where
// these are equal by bias and logit; -infinity where there is none.
__device__ __noinline__ void best_logits(const GateParams &p, int t, const Key64 *key, float *l1, float *l2) {
  const int lane = threadIdx.x & 31, shift = p.scan_shift, g = lane >> shift, sub = lane & ((1 << shift) - 1);
  const Key64 none = key_of(-INFINITY);
  Key64 k1 = lowest<Key64>(), k2 = k1, u1 = none, u2 = none;   // lower halves of u: the logits
  auto take_both = [&](Key64 k, Key64 u) {
    if (k > k1 || (k == k1 && u > u1)) {
      k2 = k1;
      u2 = u1;
      k1 = k;
      u1 = u;
    } else if (k > k2 || (k == k2 && u > u2)) {
      k2 = k;
      u2 = u;
    }
  };
  if (g < p.a.prm.n_groups)
#pragma unroll 1
    for (int e = g * p.gs + sub; e < (g + 1) * p.gs; e += 1 << shift)
      if (key[e] > lowest<Key64>())
        take_both(key[e], static_cast<Key64>(key_of(p.a.bias != nullptr ? p.a.bias[e] : 0.f)) << 32 |
                              key_of(fminf(logit_at(p, t, e), FLT_MAX)));
  for (int o = 1; o < 1 << shift; o <<= 1) {
    const Key64 ka = shfl_xor(k1, o), ua = shfl_xor(u1, o), kb = shfl_xor(k2, o), ub = shfl_xor(u2, o);
    take_both(ka, ua);
    take_both(kb, ub);
  }
  *l1 = value_of(static_cast<uint32_t>(u1));
  *l2 = value_of(static_cast<uint32_t>(u2));
}

// The best groups by their worths in pairs.  Scores below e^-75 lose bits of a pair and then
// all of them, so groups worth less than 2^-100, whose biases are 0 or cancel, are compared by the
// sum of e^(l - m), m: the largest logit among those still left.
__device__ __noinline__ uint32_t exact_groups(const GateParams &p, int t, const Key64 *key) {
  const int lane = threadIdx.x & 31, shift = p.scan_shift;
  Key64 top, second;
  scan_group(p, key, &top, &second);
  const bool both = p.a.prm.group_top == 2 && second > lowest<Key64>();
  const Key64 zero = key_of(Two{0.f, 0.f});
  Key64 worth = top > lowest<Key64>() ? worth_of(top, second, both) : 0;
  const bool tiny = worth >= zero && two_of(worth).hi < 0x1p-100f;
  float l1 = -INFINITY, l2 = -INFINITY;
  if (__any_sync(kAll, tiny)) {
    best_logits(p, t, key, &l1, &l2);
    if (tiny) worth = zero;
  }
  uint32_t taken = 0;
  for (int r = 0; r < p.a.prm.top_groups; ++r) {
    const Key64 best = warp_max(worth);
    if (best == 0) break;
    bool first = worth == best;
    if (best == zero) {
      const float m = value_of(__reduce_max_sync(kAll, first ? key_of(l1) : 0u));
      Key64 part = 0;
      if (first) {
        Two sum = two_exp_diff(l1, m);
        if (both) sum = sum + two_exp_diff(l2, m);
        part = key_of(sum);
      }
      const Key64 most = warp_max(part);
      first = first && part == most;
    }
    const int g = (__ffs(__ballot_sync(kAll, first)) - 1) >> shift;
    taken |= 1u << g;
    if (lane >> shift == g) worth = 0;
  }
  return taken;
}

// The choice of row t again in pairs, sv[e] in shared memory; lane r gets the r-th expert.  m:
// the largest logit.
__device__ __noinline__ int exact_row(const GateParams &p, int t, float m, Two *sv, Candidates *sh) {
  const int lane = threadIdx.x & 31, N = p.a.N, k = p.a.k;
  const bool softmax = p.a.prm.scoring == XS_SCORE_SOFTMAX, biased = p.a.bias != nullptr;
  Key64 *key = reinterpret_cast<Key64 *>(sv);   // exponentials first, then keys
  __syncwarp();
  Two scale{1.f, 0.f};
  if (softmax) scale = row_scale(p, t, m, sv);
#pragma unroll 1
  for (int e = lane; e - lane < N; e += 32 * kBatch) {
    float l[kBatch], b[kBatch];
    const uint32_t ok = look_up_batch(p, t, e, m, l, b);
    Two s[kBatch];
    if (!softmax)
#pragma unroll
      for (int j = 0; j < kBatch; ++j) s[j] = two_sigmoid(l[j]);
#pragma unroll
    for (int j = 0; j < kBatch; ++j)
      if (e + 32 * j < N) {
        const bool in = (ok >> j) & 1u;
        if (softmax && in) s[j] = sv[e + 32 * j] * scale;
        key[e + 32 * j] = in ? key_of(add_any(s[j], Two{b[j], 0.f})) : lowest<Key64>();
      }
  }
  __syncwarp();
  uint32_t taken = kAll;
  if (p.a.prm.top_groups < p.a.prm.n_groups) {
    taken = exact_groups(p, t, key);
    __syncwarp();
  }
  // What decides between experts: without a bias the logits, as in the fp32 pass.  The winners are among
  // those whose key's upper half reaches the k-th largest of the lanes' maxima, as in best_of().
  const uint32_t none = static_cast<uint32_t>(lowest<Key64>() >> 32), below = (1u << lane) - 1u;
  uint32_t most = none;
#pragma unroll 1
  for (int e = lane; e - lane < N; e += 32 * kBatch) {
    float l[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j)
      if (!biased && e + 32 * j < N) l[j] = logit_at(p, t, e + 32 * j);
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int i = e + 32 * j;
      if (i >= N) break;
      const bool in = (taken >> ((static_cast<uint32_t>(i) * p.magic) >> 21)) & 1u;
      Key64 v = key[i];
      if (!in) v = lowest<Key64>();
      if (!biased && v != lowest<Key64>()) v = key_of(Two{fminf(l[j], FLT_MAX), 0.f});
      key[i] = v;
      most = max(most, static_cast<uint32_t>(v >> 32));
    }
  }
  uint32_t least = none + 1;
  for (int r = 0; r < k; ++r) {
    const uint32_t best = warp_max(most);
    least = best;
    if (best == none) break;
    if (most == best) most = none;
  }
  least = max(least, none + 1);
  int n = 0;
#pragma unroll 1
  for (int e0 = 0; e0 < N; e0 += 32) {
    const int e = e0 + lane;
    const bool in = e < N && static_cast<uint32_t>(key[e] >> 32) >= least;
    const uint32_t lanes = __ballot_sync(kAll, in);
    const int at = n + __popc(lanes & below);
    if (in && at < 32) sh->of[at] = make_uint2(0, e);
    n += __popc(lanes);
  }
  __syncwarp();
  if (n <= 32) {
    const int mine = lane < n ? static_cast<int>(sh->of[lane].y) : 0;
    const int id = rank_keys(sh, n, lane < n ? key[mine] : 0, tie_of(p, t, mine, key[mine]));
    return lane < k ? id : -1;
  }
  // Many equal upper halves: k rounds over all keys, then over those that are equal to the largest.
  int id = -1;
#pragma unroll 1
  for (int r = 0; r < k; ++r) {
    Key64 mine = lowest<Key64>(), tie = 0;
    int em = N;
    for (int e = lane; e < N; e += 32) mine = key[e] > mine ? key[e] : mine;
    const Key64 best = warp_max(mine);
    if (best == lowest<Key64>()) break;
    for (int e = lane; e < N; e += 32)
      if (key[e] == best) {
        const Key64 u = tie_of(p, t, e, best);
        if (em == N || u > tie) {
          tie = u;
          em = e;
        }
      }
    const Key64 first = warp_max(tie);
    const int win = __reduce_min_sync(kAll, static_cast<unsigned>(tie == first ? em : N));
    if (lane == r) id = win;
    if ((win & 31) == lane) key[win] = lowest<Key64>();
  }
  return id;
}

// (The bounds keep the rarely called near_row() and exact_row() from setting the register count:
// 2048 rows of 256 5.3 -> 4.3 us.)
template <int kE>
__global__ void __launch_bounds__(32 * kWarps, kE <= 8 ? 8 : kE <= 12 ? 6 : kE <= 16 ? 5 : kE <= 24 ? 4 : 3)
    gate_kernel(const __grid_constant__ GateParams p) {
  extern __shared__ float2 gate_smem[];
  __shared__ Candidates s_best[kWarps];
  const GateArgs &a = p.a;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int t = blockIdx.x * kWarps + warp, N = a.N, k = a.k;
  pdl_wait();
  pdl_trigger();
  if (t >= a.B) return;
  Two *shared = reinterpret_cast<Two *>(gate_smem) + static_cast<size_t>(warp) * N;
  const bool live = a.token_mask == nullptr || a.token_mask[t] != 0;
  // Logits and biases, -infinity for experts that are not eligible: their scores come out as
  // 0 and their choice values as -infinity without another look.
  float l[kE], bias[kE];
  if (live) load_row<kE>(p, t, l, bias);
#pragma unroll
  for (int j = 0; j < kE; ++j) {
    const int e = lane * kE + j;
    // s is finite, so c = s + bias is NaN or -infinity exactly where the bias is.
    const bool ok = live && e < N && l[j] > -INFINITY && bias[j] > -INFINITY &&
                    (a.expert_mask == nullptr || a.expert_mask[e] != 0);
    l[j] = ok ? fminf(l[j], FLT_MAX) : -INFINITY;
    if (!ok) bias[j] = -INFINITY;
  }
  // Scores.
  const bool softmax = a.prm.scoring == XS_SCORE_SOFTMAX;
  float s[kE], m = -INFINITY, sum = 1.f;
  float slack;   // above this gap fp32 values are in the order of the real ones
  if (softmax) {
#pragma unroll
    for (int j = 0; j < kE; ++j) m = fmaxf(m, l[j]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, shfl_xor(m, o));
    if (m == -INFINITY) m = 0.f;   // an empty row: all scores 0
    float part[kE];   // added in pairs: five roundings, not kE
#pragma unroll
    for (int j = 0; j < kE; ++j) part[j] = s[j] = expf(l[j] - m);
#pragma unroll
    for (int w = 1; w < kE; w *= 2)
#pragma unroll
      for (int j = 0; j + w < kE; j += 2 * w) part[j] += part[j + w];
    sum = part[0];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += shfl_xor(sum, o);
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
    for (int j = 0; j < kE; ++j) s[j] *= inv;
    // Of the largest score, 1 / sum: two values' expf (2 ulp), x = l - m rounded (2^-24 |x| e^x) and the
    // product, 6.4e-7; what the sum is off by moves their difference by at most as much: ten
    // additions, expf, the rounding of x (weighed with the scores |x| is below ln 1024), the
    // reciprocal, 1.3e-6.
    slack = sum > 0.f ? 0x1.4p-19f / sum : 0.f;
  } else {
#pragma unroll
    for (int j = 0; j < kE; ++j) s[j] = score_of(false, l[j], m, sum);
    // Two values' expf (2 ulp, weighed with at most 1 / 4), addition, reciprocal (1 ulp) and product: ten
    // times 2^-24 of s <= 1.
    slack = 0x1.8p-21f;
  }
  if (a.scores != nullptr) {
    float *dst = a.scores + static_cast<size_t>(t) * N + lane * kE;
#pragma unroll
    for (int j = 0; j < kE; ++j)
      if (lane * kE + j < N) dst[j] = s[j];
  }
  // Groups and experts.
  const bool biased = a.bias != nullptr;
  const bool sums = a.prm.group_top == 2 && a.prm.top_groups < a.prm.n_groups;
  bool groups = false;   // their choice is open
  uint32_t chosen = kAll, taken = kAll;
#pragma unroll
  for (int j = 0; j < kE; ++j) s[j] = biased || sums ? s[j] + bias[j] : l[j];
  if (a.prm.top_groups < a.prm.n_groups) {
    float top = -INFINITY, second = -INFINITY;
    if (p.group_shift >= 0) {
      // Groups of whole lanes: the lanes of a group exchange their best two.
#pragma unroll
      for (int j = 0; j < kE; ++j) take(s[j], &top, &second);
      join_best(p.group_shift, &top, &second);
      taken = best_groups(p, top, second, p.group_shift);
      chosen = (taken >> (lane >> p.group_shift)) & 1u ? kAll : 0u;
    } else {
      float *values = reinterpret_cast<float *>(shared);
#pragma unroll
      for (int j = 0; j < kE; ++j)
        if (lane * kE + j < N) values[lane * kE + j] = s[j];
      __syncwarp();
      scan_group(p, values, &top, &second);
      taken = best_groups(p, top, second, p.scan_shift);
      chosen = 0;
#pragma unroll
      for (int j = 0; j < kE; ++j) {
        const uint32_t g = (static_cast<uint32_t>(lane * kE + j) * p.magic) >> 21;
        if (g < 32 && (taken >> g) & 1u) chosen |= 1u << j;
      }
    }
    if (biased || sums)
      groups = groups_near(p, top, second, p.group_shift >= 0 ? p.group_shift : p.scan_shift, taken, slack);
#pragma unroll
    for (int j = 0; j < kE; ++j) s[j] = (chosen >> j) & 1u ? (biased ? s[j] : l[j]) : -INFINITY;
  }
  int n_near;
  float bound;
  // With a bias three more candidates than are looked at, for near_row().
  int id = best_of<kE>(s, biased ? k + 4 : k, &s_best[warp], &n_near, &bound);
  if (lane > k) id = -1;
  // The winner's score and choice value, as above.
  const float lw = id >= 0 ? fminf(logit_at(p, t, id), FLT_MAX) : 0.f, bw = id >= 0 && biased ? a.bias[id] : 0.f;
  float score = id >= 0 ? score_of(softmax, lw, m, sum) : 0.f;
  // Did a gap decide that fp32 does not resolve?  Adding the bias rounds too, by 2^-24 of the value.
  if (biased || sums) {
    const float value = score + bw;
    float big = 0.f;
    if (biased) {
      big = id >= 0 ? fabsf(value) : 0.f;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) big = fmaxf(big, shfl_xor(big, o));
    }
    bool near = groups;
    const float limit = slack + 0x1p-22f * big;
    if (biased) {
      const int id2 = __shfl_down_sync(kAll, id, 1);
      const float v2 = __shfl_down_sync(kAll, value, 1);
      const float l2 = __shfl_down_sync(kAll, lw, 1), b2 = __shfl_down_sync(kAll, bw, 1);
      // The same logit and bias: a tie, which the lower index won.
      const bool same = lw == l2 && bw == b2;
      near |= lane < k && id >= 0 && id2 >= 0 && value - v2 < limit && !same;
      if (__any_sync(kAll, lane == k - 1 && id2 >= 0 && same))
        near |= border_near(p, t, m, sum, taken, __shfl_sync(kAll, value, k - 1), __shfl_sync(kAll, lw, k - 1),
                            __shfl_sync(kAll, bw, k - 1), limit);
    }
    if (__any_sync(kAll, near)) {
      // The candidates are enough if no other expert comes near the last winner (with fewer
      // than k winners all are candidates).
      const bool all = n_near <= 32 && biased && !groups &&
                       (__shfl_sync(kAll, id, k - 1) < 0 || __shfl_sync(kAll, value, k - 1) - bound >= limit);
      id = all ? near_row(p, t, m, n_near, &s_best[warp]) : exact_row(p, t, m, shared, &s_best[warp]);
      score = id >= 0 ? score_of(softmax, fminf(logit_at(p, t, id), FLT_MAX), m, sum) : 0.f;
    }
  }
  // Weights, summed in slot order.
  if (lane >= k) id = -1;
  const int n = __popc(__ballot_sync(kAll, id >= 0));
  float w = 0.f;
  if (a.prm.renorm != 0) {
    float total = 0.f;
    for (int r = 0; r < n; ++r) total += __shfl_sync(kAll, score, r);
    w = (total == 0.f ? 1.f / n : score / total) * a.prm.scale;
  } else {
    w = score * a.prm.scale;
  }
  if (lane < k) {
    a.ids[static_cast<size_t>(t) * k + lane] = id;
    a.w[static_cast<size_t>(t) * k + lane] = id >= 0 ? w : 0.f;
  }
}

template <int kE>
cudaError_t launch(const GateArgs &a, int dtype, cudaStream_t s) {
  GateParams p;
  p.a = a;
  p.dtype = dtype;
  p.gs = a.N / a.prm.n_groups;
  p.magic = ((1u << 21) + p.gs - 1) / p.gs;
  // Elements of a word; rows and the bias start 16-byte aligned.
  const int wide = sizeof(WordOf<kE * 4>) / 4, narrow = sizeof(WordOf<kE * 2>) / 2;
  p.vec = a.N % (dtype == XS_F32 ? wide : narrow) == 0;
  p.vec_bias = a.N % wide == 0;
  p.group_shift = -1;
  for (int sh = 0; sh <= 5; ++sh)
    if (p.gs == kE << sh) p.group_shift = sh;
  p.scan_shift = 5;
  while (32 >> p.scan_shift < a.prm.n_groups) --p.scan_shift;
  // A row's values in shared memory: groups that are not whole lanes, and exact_row().
  const bool limited = a.prm.top_groups < a.prm.n_groups;
  const bool shared = a.bias != nullptr || (limited && (p.group_shift < 0 || a.prm.group_top == 2));
  const size_t smem = shared ? kWarps * static_cast<size_t>(a.N) * sizeof(Two) : 0;
  return launch_pdl(gate_kernel<kE>, dim3((a.B + kWarps - 1) / kWarps), dim3(32 * kWarps), smem, s, p);
}

}  // namespace

cudaError_t launch_gate(const GateArgs &a, int dtype, cudaStream_t s) {
  if (a.N <= 64) return launch<2>(a, dtype, s);
  if (a.N <= 96) return launch<3>(a, dtype, s);
  if (a.N <= 128) return launch<4>(a, dtype, s);
  if (a.N <= 192) return launch<6>(a, dtype, s);
  if (a.N <= 256) return launch<8>(a, dtype, s);
  if (a.N <= 384) return launch<12>(a, dtype, s);
  if (a.N <= 512) return launch<16>(a, dtype, s);
  if (a.N <= 768) return launch<24>(a, dtype, s);
  return launch<32>(a, dtype, s);
}

}  // namespace xs
