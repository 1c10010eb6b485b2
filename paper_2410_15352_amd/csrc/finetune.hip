// Losses over the log-probabilities of given tokens.  For a row x of V logits and its target t,
// with m = max x, s = sum exp(x - m):
//
//   l = x_t - m - log s,    dl / dx_v = [v = t] - exp(x_v - m) / s
//
// log-probabilities: l, and dx from a given dl.
// preference: of n pairs of sequences, S = sum over a sequence's rows of (l - reference),
//   D = beta (S_first - S_second),  loss = mean of (1 - e) softplus(-D) + e softplus(D),
//   dloss / dl = +- beta (sigmoid(D) - (1 - e)) / n  in the rows of the first, the second.
// policy: ratio r = exp(l - old), advantage A, bounds lo = 1 - low, hi = 1 + high,
//   loss = mean over the N rows that count of -min(r A, clamp(r, lo, hi) A) + kl (exp(d) - d - 1),
//   d = reference - l;   dl = ((r clamped away ? 0 : -A r) - kl (exp(d) - 1)) / N.
//
// Rows whose target is ignore_index do not count: l = 0, no gradient, and they are not read; a
// target past V makes a row NaN.  A row without a gradient (dl = 0) has zeros, whatever its logits are.
//
// All are bound by HBM: the logits of a row that counts are read once for l, and once more for the
// gradient where that needs sums over other rows first (log-probabilities, preference); the policy
// loss holds a row in registers and forms both.  (Up to 131072 bf16 or 65536 fp32 logits; what a row has
// past them is read for its maximum, its sum and its gradient.)  Measured, of 32000 bf16 logits, 7 of 10 rows counting:
// l of 8192 rows 70 us, 5.3 TB/s, the same right after the gradient of others was written 105 us; the
// gradient 150 us, 5.9 TB/s (some of the logits are still in the cache); the policy loss with its
// gradient 192 us, 4.6 TB/s, and of 4096 rows of 131072 380 us, 4.8 TB/s, where a large copy reaches
// 5.2.  (The rows that count dealt out evenly first: no faster.  Exponents by one fused operation in
// place of two: 1%.)  l is put together in fp64 (a few operations a
// row), what is left of l - reference being a difference of near numbers.
#include <hip/hip_runtime.h>

#include "common.hpp"
#include "functional.hpp"
#include "rows.hpp"

namespace compact {
namespace {

__device__ __forceinline__ double log_prob(float xt, float m, double s) {
  return static_cast<double>(xt) - static_cast<double>(m) - log(s);
}

// e^t for t <= 0.  (The constant's own rounding makes every term too large, by 1.3e-8 |t|, and with it a
// sum of differences l - reference over many rows.)
__device__ __forceinline__ float exp_of(float t) {
  constexpr float kLow = static_cast<float>(1.44269504088896340736 - static_cast<double>(kLog2e));
  return __builtin_amdgcn_exp2f(__builtin_fmaf(t, kLog2e, t * kLow));
}

// ---------------------------- log-probabilities ------------------------------
// A workgroup per row: each thread keeps a running maximum and sum over its chunks, four at a time.  The
// sums of a chunk and of the four are fp32, all longer ones fp64: added one by one in fp32, terms below half a unit
// in the last place of the sum so far are lost (131072 logits, the target's 0 and all others -17.5: l = -0.00329 was
// off by 1.3e-5).
template <bool F32>
__global__ __launch_bounds__(256) void k_token_fwd(TokenArgs a) {
  using R = Row<F32>;
  constexpr int N = R::kN, U = 4;
  __shared__ float red[4];
  __shared__ double sums[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = blockIdx.x, target = a.target[row];
  const float ninf = -__builtin_inff();
  if (target == a.ignore_index) {
    if (tid == 0) a.out[row] = 0.0f;
    return;
  }
  const R r(row, a.V);
  float m = ninf;
  double s = 0.0;
  auto add = [&](float top) {  // a new maximum
    if (top > m) {
      s *= static_cast<double>(exp_of(m - top));
      m = top;
    }
  };
  if (r.end_of(tid) >= 0) {
    const float x = r.one(a.x, r.end_of(tid));
    add(x);
    s += static_cast<double>(exp_of(x - (m == ninf ? 0.0f : m)));
  }
#pragma unroll 1
  for (int c = 0; c + tid < r.chunks; c += 256 * U) {
    u32x4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = r.load(a.x, true, c + 256 * u, tid);
    float top = ninf;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      r.ends(x[u], c + 256 * u + tid);
#pragma unroll
      for (int e = 0; e < N; ++e) top = fmaxf(top, R::value(x[u], e));
    }
    add(top);
    const float shift = m == ninf ? 0.0f : m;
    float four = 0.0f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float one = 0.0f;
#pragma unroll
      for (int e = 0; e < N; ++e) one += exp_of(R::value(x[u], e) - shift);
      four += one;
    }
    s += static_cast<double>(four);
  }
  float top = wave_max(m);
  if (lane == 0) red[wave] = top;
  __syncthreads();
  top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  const float shift = top == ninf ? 0.0f : top;
  // (a thread without a logit above -inf has m = -inf; its sum is 0, or NaN)
  s = wave_sum(s * static_cast<double>(exp_of((m == ninf ? shift : m) - shift)));
  if (lane == 0) sums[wave] = s;
  __syncthreads();
  if (tid == 0) {
    s = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    const bool in = target >= 0 && target < a.V;
    const double l = in ? log_prob(r.one(a.x, static_cast<uint32_t>(target)), shift, s) : __builtin_nan("");
    a.out[row] = static_cast<float>(a.reference != nullptr ? l - static_cast<double>(a.reference[row]) : l);
    if (a.stats != nullptr) {
      a.stats[2 * row] = shift;
      a.stats[2 * row + 1] = static_cast<float>(s);
    }
  }
}

// The logits' gradient: a workgroup per row, four chunks of a thread in flight.
template <bool F32>
__global__ __launch_bounds__(256) void k_token_bwd(TokenArgs a) {
  using R = Row<F32>;
  constexpr int N = R::kN, U = 4;
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x, target = a.target[row];
  const R r(row, a.V);
  float g = 0.0f;
  if (target != a.ignore_index) {
    g = a.grad[row];
    // (of a pair with a target past V the slope is NaN already; in a row of no pair it does not count)
    if (a.dloss != nullptr) g *= a.dloss[0];
    else if (target < 0 || target >= a.V) g = __builtin_nanf("");
  }
  g = uniform(g);
  if (g == 0.0f) {
    const float none[N] = {};
    if (r.end_of(tid) >= 0) r.put(a.dx, r.end_of(tid), 0.0f);
#pragma unroll 4
    for (int c = 0; c + tid < r.chunks; c += 256) r.store(a.dx, c, tid, none);
    return;
  }
  const float m = uniform(a.stats[2 * row]), f = uniform(-g / a.stats[2 * row + 1]);
  auto grad = [&](float v) { return f * __builtin_amdgcn_exp2f((v - m) * kLog2e); };
  const int at = static_cast<int>(target);  // (past V every element is NaN)
  const int end = r.end_of(tid);
  if (end >= 0) r.put(a.dx, end, grad(r.one(a.x, end)) + (end == at ? g : 0.0f));
#pragma unroll 1
  for (int c = 0; c + tid < r.chunks; c += 256 * U) {
    u32x4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = r.load(a.x, true, c + 256 * u, tid);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float v[N];
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = grad(R::value(x[u], e));
      const int k = at - r.head - (c + 256 * u + tid) * N;
      if (static_cast<uint32_t>(k) < static_cast<uint32_t>(N)) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] += e == k ? g : 0.0f;
      }
      r.store(a.dx, c + 256 * u, tid, v);
    }
  }
}

// ---------------------------- preference pairs -------------------------------
// THREADS threads per pair (a wave, or a workgroup of 256): the sums of both sequences (fp64, in a
// fixed order), the pair's loss, and the slope of the mean for each of their rows.  The first and
// the last pair clear the rows before and behind all sequences.  Starts are taken as their running
// maximum within the rows.  lds: room for 4 numbers of 64 bits.
template <int THREADS, typename T, typename F>
__device__ __forceinline__ T joined(T v, T* lds, F join) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = join(v, __shfl_xor(v, d, 64));
  if constexpr (THREADS > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = join(join(lds[0], lds[1]), join(lds[2], lds[3]));
  }
  return v;
}

__device__ __forceinline__ long long start_at(const PairArgs& a, int64_t i) {
  const int64_t x = a.starts64 ? static_cast<const int64_t*>(a.starts)[i * a.stride] : static_cast<const int32_t*>(a.starts)[i * a.stride];
  return x < 0 ? 0 : x > a.rows ? a.rows : x;
}

// The running maximum of the starts, by one workgroup, four to a thread at a time.
__global__ __launch_bounds__(1024) void k_pair_bounds(PairArgs a) {
  constexpr int kOwn = 4;
  __shared__ int lds[2][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t starts = 2 * a.n + 1;
  int carry = 0, turn = 0;
  for (int64_t i0 = 0; i0 < starts; i0 += 1024 * kOwn, turn ^= 1) {
    const int64_t i = i0 + tid * kOwn;
    int v[kOwn];
#pragma unroll
    for (int k = 0; k < kOwn; ++k) v[k] = i + k < starts ? static_cast<int>(start_at(a, i + k)) : 0;
#pragma unroll
    for (int k = 1; k < kOwn; ++k) v[k] = max(v[k], v[k - 1]);
    int upto = v[kOwn - 1];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int w = __shfl_up(upto, d, 64);
      if (lane >= d) upto = max(upto, w);
    }
    if (lane == 63) lds[turn][wave] = upto;
    int before = __shfl_up(upto, 1, 64);
    before = lane > 0 ? max(before, carry) : carry;
    __syncthreads();  // (two sets of numbers: the next but one is written behind the next's barrier)
    for (int w = 0; w < 16; ++w) {
      if (w < wave) before = max(before, lds[turn][w]);
      carry = max(carry, lds[turn][w]);
    }
#pragma unroll
    for (int k = 0; k < kOwn; ++k)
      if (i + k < starts) a.bounds[i + k] = max(v[k], before);
  }
}

template <int THREADS>
__device__ __forceinline__ double pair_loss(const PairArgs& a, int64_t pair, int tid, double* lds) {
  const auto add = [](double x, double y) { return x + y; };
  int64_t e0, e1, e2;
  if (a.bounds != nullptr) {
    e0 = a.bounds[2 * pair], e1 = a.bounds[2 * pair + 1], e2 = a.bounds[2 * pair + 2];
  } else {
    long long first = 0;
    for (int64_t i = tid; i <= 2 * pair; i += THREADS) first = max(first, start_at(a, i));
    e0 = joined<THREADS>(first, reinterpret_cast<long long*>(lds), [](long long x, long long y) { return max(x, y); });
    e1 = max(static_cast<long long>(e0), start_at(a, 2 * pair + 1));
    e2 = max(static_cast<long long>(e1), start_at(a, 2 * pair + 2));
  }
  double s0 = 0.0, s1 = 0.0;
#pragma unroll 4
  for (int64_t i = e0 + tid; i < e1; i += THREADS) s0 += static_cast<double>(a.gain[i]);
#pragma unroll 4
  for (int64_t i = e1 + tid; i < e2; i += THREADS) s1 += static_cast<double>(a.gain[i]);
  s0 = joined<THREADS>(s0, lds, add);
  s1 = joined<THREADS>(s1, lds, add);
  const double beta = a.beta, eps = a.smoothing, delta = beta * (s0 - s1), away = exp(-fabs(delta));
  // sigmoid(D) - (1 - e), of which both parts keep their digits where D is large
  const double up = delta >= 0.0 ? 1.0 / (1.0 + away) : away / (1.0 + away), down = delta >= 0.0 ? away / (1.0 + away) : 1.0 / (1.0 + away);
  const float slope = static_cast<float>(beta / static_cast<double>(a.n) * (eps * up - (1.0 - eps) * down));
  for (int64_t i = e0 + tid; i < e1; i += THREADS) a.slope[i] = slope;
  for (int64_t i = e1 + tid; i < e2; i += THREADS) a.slope[i] = -slope;
  if (pair == 0)
    for (int64_t i = tid; i < e0; i += THREADS) a.slope[i] = 0.0f;
  if (pair == a.n - 1)
    for (int64_t i = e2 + tid; i < a.rows; i += THREADS) a.slope[i] = 0.0f;
  if (tid == 0) {
    a.rewards[2 * pair] = static_cast<float>(beta * s0);
    a.rewards[2 * pair + 1] = static_cast<float>(beta * s1);
  }
  // softplus(-D), softplus(D); of an infinite D times a factor of zero: nothing
  const double soft = log1p(away);
  const double low = (delta < 0.0 ? -delta : delta >= 0.0 ? 0.0 : delta) + soft, high = (delta > 0.0 ? delta : 0.0) + soft;
  return (1.0 - eps) * low + (eps == 0.0 ? 0.0 : eps * high);
}

// Up to kOwnPairs each pair finds its first row by itself, from all starts before it; past that the
// starts' running maximum is formed first, by a launch of its own.  us, without it / with it, 8 rows to a
// pair: 256 pairs 7.3 / 9.7, 2048 13 / 13.6, 4096 24 / 19, 8192 55 / 30, 65536 1890 / 188.  (2^23
// pairs in 2^20 rows, most of them empty: 25 ms with it.)
constexpr int64_t kOwnPairs = 2048;
__global__ __launch_bounds__(256) void k_pairs(PairArgs a) {
  __shared__ double lds[4];
  const double loss = pair_loss<256>(a, blockIdx.x, threadIdx.x, lds);
  if (threadIdx.x == 0) a.loss_pair[blockIdx.x] = static_cast<float>(loss);
}

// A few pairs: a wave each, and their mean, in one workgroup.  us, this / a workgroup per pair and the
// mean's launch (which on the host is 3 more), by rows and pairs:
//             1 pair       2            4           8          16          64
//     200   3.7 / 5.9   3.7 / 6.0   4.1 / 6.1   4.6 / 6.2   5.4 / 6.2
//    2048   5.0 / 6.0   4.3 / 6.2   4.5 / 6.1   4.9 / 6.3   5.6 / 6.2
//    4096   6.8 / 6.3   5.3 / 6.3   4.9 / 6.4   4.7 / 6.2   5.9 / 6.3
//    8192  10.5 / 7.4   7.1 / 6.7   5.8 / 6.4   5.2 / 6.5   5.8 / 6.3    18 / 6.9
//   16384  17.9 / 9.2  10.7 / 7.6   7.6 / 6.8   6.2 / 6.6   6.4 / 6.5
//   32768  32.3 / 12.9 18.2 / 9.4  11.2 / 7.7   8.1 / 6.9   7.6 / 6.5
constexpr int kFewPairs = 16;
constexpr int64_t kFewPairRows = 16384, kFewRowsEach = 4096;
bool few_pairs(int64_t n, int64_t rows) { return n <= kFewPairs && rows <= kFewPairRows && rows <= n * kFewRowsEach; }
__global__ __launch_bounds__(1024) void k_few_pairs(PairArgs a) {
  __shared__ double loss[kFewPairs];
  const int lane = threadIdx.x & 63, pair = threadIdx.x >> 6;
  if (pair < a.n) {
    const double v = pair_loss<64>(a, pair, lane, nullptr);
    if (lane == 0) loss[pair] = v;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    double s = 0.0;
    for (int pair = 0; pair < a.n; ++pair) s += loss[pair];
    a.loss[0] = static_cast<float>(s / static_cast<double>(a.n));
  }
}

// The mean of n values: fp64 sums in a fixed order, by one workgroup of 1024.
__device__ __forceinline__ void store_mean(const float* v, int64_t n, double count, float* out) {
  __shared__ double s[1024];
  double l = 0.0;
#pragma unroll 4
  for (int64_t r = threadIdx.x; r < n; r += 1024) l += static_cast<double>(v[r]);
  s[threadIdx.x] = l;
  __syncthreads();
  for (int d = 512; d > 0; d >>= 1) {
    if (static_cast<int>(threadIdx.x) < d) s[threadIdx.x] += s[threadIdx.x + d];
    __syncthreads();
  }
  if (threadIdx.x == 0) out[0] = static_cast<float>(s[0] / count);
}

__global__ __launch_bounds__(1024) void k_pairs_mean(PairArgs a) { store_mean(a.loss_pair, a.n, static_cast<double>(a.n), a.loss); }

// ------------------------------- policy --------------------------------------
__global__ __launch_bounds__(1024) void k_policy_count(PolicyArgs a) {
  __shared__ int red[16];
  int c = 0;
#pragma unroll 8
  for (int64_t r = threadIdx.x; r < a.rows; r += 1024) c += a.target[r] != a.ignore_index ? 1 : 0;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) c += __shfl_xor(c, d, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = c;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 16; ++w) c += red[w];
    a.count[0] = static_cast<float>(c);
  }
}

// One row per workgroup at a time; NC chunks per thread in registers, any more are read again for
// each walk.
template <bool F32, int THREADS, int NC>
__global__ __launch_bounds__(THREADS, 4) void k_policy(PolicyArgs a) {
  using R = Row<F32>;
  constexpr int N = R::kN, NW = THREADS / 64;
  __shared__ float smax[NW];
  __shared__ double ssum[NW];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float ninf = -__builtin_inff();
  float scale = 1.0f;
  if (a.dloss != nullptr) {
    scale = a.dloss[0];
    if (a.unless_one && scale == 1.0f) return;
  }
  scale = uniform(scale / a.count[0]);

  u32x4 x[NC];
  float xe;   // this thread's single element
  int64_t target;
  bool live;  // else the row has no part: no loss, no gradient, and nothing is read
  auto head_of = [&](int64_t row) {
    target = row < a.rows ? a.target[row] : a.ignore_index;
    live = target != a.ignore_index;
  };
  head_of(blockIdx.x);
  {
    const R r(live ? blockIdx.x : 0, a.V);
    xe = live && r.end_of(tid) >= 0 ? r.one(a.x, r.end_of(tid)) : ninf;
#pragma unroll
    for (int i = 0; i < NC; ++i) x[i] = r.load(a.x, live, THREADS * i, tid);
  }
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const R r(row, a.V);
    const int64_t aim = target;
    float m = live ? xe : 0.0f, g = 0.0f, f = 0.0f;  // the gradient of l, and the factor of the exponentials
    if (live) {
      const bool in = aim >= 0 && aim < a.V;
      const float xt = in ? r.one(a.x, static_cast<uint32_t>(aim)) : __builtin_nanf("");
      const float old = a.old[row], A = a.advantage[row], ref = a.reference != nullptr ? a.reference[row] : 0.0f;
      auto walk = [&](auto f) {
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          f(x[i]);
          asm volatile("" : "+v"(x[i]));
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll 1
        for (int c = THREADS * NC; c + tid < r.chunks; c += THREADS) f(r.load(a.x, true, c, tid));
      };
#pragma unroll
      for (int i = 0; i < NC; ++i) r.ends(x[i], tid + THREADS * i);
      walk([&](const u32x4& c) {
#pragma unroll
        for (int e = 0; e < N; ++e) m = fmaxf(m, R::value(c, e));
      });
      m = wave_max(m);
      if (lane == 0) smax[wave] = m;
      __syncthreads();
      m = wave_max(smax[lane & (NW - 1)]);
      m = uniform(m == ninf ? 0.0f : m);
      double s = static_cast<double>(__builtin_amdgcn_exp2f((xe - m) * kLog2e));
      walk([&](const u32x4& c) {  // (a chunk's sum is fp32, longer ones fp64, as in k_token_fwd)
        float one = 0.0f;
#pragma unroll
        for (int e = 0; e < N; ++e) one += __builtin_amdgcn_exp2f((R::value(c, e) - m) * kLog2e);
        s += static_cast<double>(one);
      });
      s = wave_sum(s);
      if (lane == 0) ssum[wave] = s;
      __syncthreads();
      s = wave_sum(lane < NW ? ssum[lane & (NW - 1)] : 0.0);
      const double l = log_prob(xt, m, s);
      const float lo = 1.0f - a.low, hi = 1.0f + a.high, ratio = expf(static_cast<float>(l - static_cast<double>(old)));
      const bool clamped = (A > 0.0f && ratio > hi) || (A < 0.0f && ratio < lo);
      const bool idle = A == 0.0f && ratio == ratio;  // (a ratio that overflowed must not become 0 x inf)
      const float away = a.reference != nullptr ? static_cast<float>(static_cast<double>(ref) - l) : 0.0f;
      const float odds = a.reference != nullptr ? expm1f(away) : 0.0f;
      g = clamped || idle ? 0.0f : -A * ratio;
      if (a.reference != nullptr) g -= a.kl * odds;
      if (a.loss_row != nullptr && tid == 0) {
        float loss = idle ? 0.0f : -A * (clamped ? (A > 0.0f ? hi : lo) : ratio);
        if (a.reference != nullptr) loss += a.kl * (odds - away);
        a.loss_row[row] = loss;
        a.logp[row] = static_cast<float>(l);
      }
      g = uniform(g * scale);
      f = uniform(g == 0.0f ? 0.0f : -g / static_cast<float>(s));
    } else if (a.loss_row != nullptr && tid == 0) {
      a.loss_row[row] = 0.0f;
      a.logp[row] = 0.0f;
    }
    const bool none = g == 0.0f;
    auto grad = [&](const u32x4& c, int skip) {
      float v[N] = {};
      if (!none) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = f * __builtin_amdgcn_exp2f((R::value(c, e) - m) * kLog2e);
        const int k = static_cast<int>(aim) - r.head - (skip + tid) * N;
        if (static_cast<uint32_t>(k) < static_cast<uint32_t>(N)) {
#pragma unroll
          for (int e = 0; e < N; ++e) v[e] += e == k ? g : 0.0f;
        }
      }
      r.store(a.dx, skip, tid, v);
    };
    if (a.dx != nullptr) {
      const int end = r.end_of(tid);
      if (end >= 0) r.put(a.dx, end, none ? 0.0f : f * __builtin_amdgcn_exp2f((xe - m) * kLog2e) + (end == static_cast<int>(aim) ? g : 0.0f));
#pragma unroll 1
      for (int c = THREADS * NC; c + tid < r.chunks; c += THREADS) grad(r.load(a.x, true, c, tid), c);
    }
    const int64_t next_row = row + gridDim.x;
    head_of(next_row);
    const R next(live ? next_row : row, a.V);
    xe = live && next.end_of(tid) >= 0 ? next.one(a.x, next.end_of(tid)) : ninf;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      if (a.dx != nullptr) grad(x[i], THREADS * i);
      x[i] = next.load(a.x, live, THREADS * i, tid);
      __builtin_amdgcn_sched_barrier(0);  // (all loads at once would want registers of their own)
    }
  }
}

__global__ __launch_bounds__(1024) void k_policy_mean(PolicyArgs a) { store_mean(a.loss_row, a.rows, static_cast<double>(a.count[0]), a.loss); }

template <bool F32, int THREADS, int NC>
void launch_policy(const PolicyArgs& a, hipStream_t s) {
  const int64_t most = 256 * ((NC > 4 ? 1024 : 1536) / THREADS);
  hipLaunchKernelGGL((k_policy<F32, THREADS, NC>), dim3(static_cast<uint32_t>(a.rows < most ? a.rows : most)), dim3(THREADS), 0, s, a);
}

template <bool F32>
void launch_policy(const PolicyArgs& a, hipStream_t s) {
  // The smallest workgroup whose registers hold a row, or all but the last 3% of it.  us by threads x
  // chunks, loss and gradient in bf16, all rows counting (the rule's *):
  //             256 x 1  256 x 4  256 x 16  512 x 16  1024 x 16
  //   16384 x   1000  62*      94      255       507      1015
  //    8192 x   8000  72       60*     136       265       524
  //    8192 x  32001 280      264      227*      300       544
  //    2048 x  65536 181      174      154       121*      171
  //    1024 x 200000 322      317      303       255       225*
  // in fp32, with the launches of the count and the mean:
  //   16384 x   1000  53*      67      148       291       599
  //   16384 x   2000  66       68*     150       291       605
  //    8192 x   4096  55       53*      82       153       309
  //    8192 x   8000 137      122      115*      172       319
  //    8192 x  16384 278      256      218*      227       350
  //    4096 x  32000 316      301      254       210*      245
  //    2048 x  65536 380      369      330       259       228*
  //    1024 x 131072 379      375      362       330       284*  (3.8 TB/s of one read and one write: half of a row in registers)
  const int64_t chunks = a.V / (F32 ? 4 : 8);
  if (chunks <= 256) launch_policy<F32, 256, 1>(a, s);
  else if (chunks <= 1024) launch_policy<F32, 256, 4>(a, s);
  else if (chunks <= 4096 + 128) launch_policy<F32, 256, 16>(a, s);
  else if (chunks <= 8192 + 256) launch_policy<F32, 512, 16>(a, s);
  else launch_policy<F32, 1024, 16>(a, s);
}

bool rows_ok(int64_t rows, int64_t V) { return rows >= 1 && rows < int64_t(1) << 24 && V >= 1 && V <= int64_t(1) << 28; }
int status() { return hipGetLastError() == hipSuccess ? 0 : -5; }

}  // namespace
}  // namespace compact

using namespace compact;

extern "C" {

int compact_token_logprobs(const TokenArgs* a, void* stream) {
  if (!rows_ok(a->rows, a->V)) return -1;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const dim3 grid(static_cast<uint32_t>(a->rows)), block(256);
  if (a->backward) {
    if (a->f32) hipLaunchKernelGGL((k_token_bwd<true>), grid, block, 0, s, *a);
    else hipLaunchKernelGGL((k_token_bwd<false>), grid, block, 0, s, *a);
  } else if (a->f32) {
    hipLaunchKernelGGL((k_token_fwd<true>), grid, block, 0, s, *a);
  } else {
    hipLaunchKernelGGL((k_token_fwd<false>), grid, block, 0, s, *a);
  }
  return status();
}

int compact_preference_pairs(const PairArgs* a, void* stream) {
  if (!rows_ok(a->rows, 1) || a->n < 1 || a->n >= int64_t(1) << 24) return -1;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (few_pairs(a->n, a->rows) && a->bounds == nullptr) {
    hipLaunchKernelGGL(k_few_pairs, dim3(1), dim3(1024), 0, s, *a);
    return status();
  }
  if (a->bounds == nullptr && a->n > kOwnPairs) return -1;
  if (a->bounds != nullptr) hipLaunchKernelGGL(k_pair_bounds, dim3(1), dim3(1024), 0, s, *a);
  hipLaunchKernelGGL(k_pairs, dim3(static_cast<uint32_t>(a->n)), dim3(256), 0, s, *a);
  hipLaunchKernelGGL(k_pairs_mean, dim3(1), dim3(1024), 0, s, *a);
  return status();
}

int compact_policy(const PolicyArgs* a, void* stream) {
  if (!rows_ok(a->rows, a->V) || !(a->low >= 0.0f) || !(a->high >= 0.0f)) return -1;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (!a->ready) hipLaunchKernelGGL(k_policy_count, dim3(1), dim3(1024), 0, s, *a);
  if (a->f32) launch_policy<true>(*a, s);
  else launch_policy<false>(*a, s);
  if (a->loss_row != nullptr) hipLaunchKernelGGL(k_policy_mean, dim3(1), dim3(1024), 0, s, *a);
  return status();
}

}  // extern "C"
