// Distillation from a teacher's top logits.  For a row x of V logits, the teacher's entries
// (t_k, id_k), a temperature T and a weight w, with p = softmax(t / T) over the entries and
// q = softmax(x / T):
//
//   loss_row = w T^2 sum_k p_k (log p_k - log q_id_k) + (1 - w) (lse(x) - x_target)
//   dx_v     = (w T (q_v - sum_{id_k = v} p_k) + (1 - w) (softmax(x)_v - [v = target])) / N
//
// N rows count (all, or those whose target is not ignore_index), the loss is their mean.  An
// entry with a negative id, or a logit of -inf, is none; a row without entries has no first
// part.  Entries with the same id add up.  An id or a target past V makes the row NaN.
//
// Bound by HBM: a row is read once and its gradient written once, by one workgroup that
// holds it in registers: the maximum, the sums of exponentials and the gradient are three
// walks over registers.  The gradient is formed where the loss is, for dloss = 1; the
// backward runs the same kernel again, which ends at once where dloss is 1 indeed.
#include <hip/hip_runtime.h>

#include "common.hpp"
#include "functional.hpp"

namespace compact {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr int kMaxK = 1024;

// a x b for a factor a that may be zero: then nothing, whatever b is.
__device__ __forceinline__ float part(float a, float b) { return a == 0.0f ? 0.0f : a * b; }

template <int NW>
__device__ __forceinline__ float block_max(float v, float* s) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = s[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) v = fmaxf(v, s[w]);
  return v;
}

template <int NW>
__device__ __forceinline__ float block_sum(float v, float* s) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = s[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) v += s[w];
  return v;
}

// The 16-byte chunks of the whole buffer that hold a row: an odd V starts rows anywhere, so
// the first and last chunk have elements of the neighbours.
template <bool F32>
struct Row {
  static constexpr int kN = F32 ? 4 : 8;
  const u32x4* x;
  int64_t begin, end, total, first;
  int chunks;
  __device__ __forceinline__ Row(const void* p, int64_t row, int64_t V, int64_t rows) {
    x = static_cast<const u32x4*>(p);
    begin = row * V;
    end = begin + V;
    total = rows * V;
    first = begin / kN;
    chunks = static_cast<int>((end + kN - 1) / kN - first);
  }
  __device__ __forceinline__ u32x4 load(const void* p, int c) const {
    const int64_t e0 = (first + c) * kN;
    if (e0 + kN <= total) return x[first + c];
    u32x4 w = {0u, 0u, 0u, 0u};  // past the buffer's last whole chunk
#pragma unroll
    for (int e = 0; e < kN; ++e) {
      if (e0 + e >= total) continue;
      if constexpr (F32) w[e] = static_cast<const uint32_t*>(p)[e0 + e];
      else w[e / 2] |= static_cast<uint32_t>(static_cast<const uint16_t*>(p)[e0 + e]) << (16 * (e & 1));
    }
    return w;
  }
  // element e of chunk c is the row's
  __device__ __forceinline__ bool in(int c, int e) const {
    const int64_t at = (first + c) * kN + e;
    return at >= begin && at < end;
  }
  __device__ __forceinline__ bool whole(int c) const {
    const int64_t at = (first + c) * kN;
    return at >= begin && at + kN <= end;
  }
  static __device__ __forceinline__ float value(const u32x4& w, int e) {
    if constexpr (F32) return __uint_as_float(w[e]);
    else return __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
  }
  static __device__ __forceinline__ u32x4 pack(const float (&v)[kN]) {
    u32x4 w;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (F32) w[k] = __float_as_uint(v[k]);
      else w[k] = pack_bf16x2(v[2 * k], v[2 * k + 1]);
    }
    return w;
  }
  static __device__ __forceinline__ float one(const void* p, int64_t at) {
    if constexpr (F32) return static_cast<const float*>(p)[at];
    else return bf16_to_f32(static_cast<const uint16_t*>(p)[at]);
  }
  static __device__ __forceinline__ void put(void* p, int64_t at, float v) {
    if constexpr (F32) static_cast<float*>(p)[at] = v;
    else static_cast<uint16_t*>(p)[at] = f32_to_bf16(v);
  }
};

// One row per workgroup at a time; NC chunks per thread in registers, any more are read again
// for each walk.
template <bool F32, int THREADS, int NC>
__global__ __launch_bounds__(THREADS) void k_distill(DistillArgs a) {
  using R = Row<F32>;
  constexpr int N = R::kN, NW = THREADS / 64;
  __shared__ float red[NW];
  __shared__ float sp[kMaxK];
  __shared__ int sid[kMaxK];
  const int tid = threadIdx.x;
  const float ninf = -__builtin_inff();
  float scale = 1.0f;
  if (a.dloss != nullptr) {
    scale = a.dloss[0];
    if (a.unless_one && scale == 1.0f) return;
  }
  scale /= a.target != nullptr ? a.count[0] : static_cast<float>(a.rows);
  const float T = a.temperature, rT = 1.0f / T, w = a.weight;
  const bool hard = a.target != nullptr && w != 1.0f;
  // one sum serves both where the temperature is 1
  const bool two = hard && T != 1.0f;

  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const R r(a.x, row, a.V, a.rows);
    const int64_t target = a.target != nullptr ? a.target[row] : 0;
    if (a.target != nullptr && target == a.ignore_index) {  // the row has no part: no gradient
      if (a.loss_row != nullptr && tid == 0) a.loss_row[row] = 0.0f;
      if (a.dx != nullptr) {
        for (int c = tid; c < r.chunks; c += THREADS) {
          if (r.whole(c)) {
            static_cast<u32x4*>(a.dx)[r.first + c] = u32x4{0u, 0u, 0u, 0u};
          } else {
#pragma unroll
            for (int e = 0; e < N; ++e)
              if (r.in(c, e)) R::put(a.dx, (r.first + c) * N + e, 0.0f);
          }
        }
      }
      continue;
    }
    u32x4 x[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int c = tid + THREADS * i;
      if (c < r.chunks) x[i] = r.load(a.x, c);
    }
    // f(chunk's words, chunk) over this thread's chunks
    auto walk = [&](auto f) {
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const int c = tid + THREADS * i;
        if (c < r.chunks) f(x[i], c);
      }
      for (int c = tid + THREADS * NC; c < r.chunks; c += THREADS) f(r.load(a.x, c), c);
    };
    // the teacher's entries
    bool bad = hard && (target < 0 || target >= a.V);
    __syncthreads();  // the last row's readers of sp, sid
    float tm = ninf;
    for (int k = tid; k < a.K; k += THREADS) {
      const int64_t id = a.ids32 ? static_cast<const int32_t*>(a.ids)[row * a.ids_ld + k]
                                 : static_cast<const int64_t*>(a.ids)[row * a.ids_ld + k];
      float t = ninf;
      if (id >= 0) t = rT * (a.top32 ? static_cast<const float*>(a.top)[row * a.top_ld + k]
                                     : bf16_to_f32(static_cast<const uint16_t*>(a.top)[row * a.top_ld + k]));
      bad |= id >= a.V;
      sp[k] = t;
      sid[k] = id < 0 || id >= a.V ? -1 : static_cast<int>(id);
      tm = fmaxf(tm, t);
    }
    tm = block_max<NW>(tm, red);
    const float tsh = tm == ninf ? 0.0f : tm;
    float ts = 0.0f;
    for (int k = tid; k < a.K; k += THREADS) ts += expf(sp[k] - tsh);
    ts = block_sum<NW>(ts, red);
    const float tlse = tsh + logf(ts);
    const bool soft = !(ts == 0.0f);  // some entry (a NaN is one)

    float m = ninf;
    walk([&](const u32x4& c, int at) {
      if (r.whole(at)) {
#pragma unroll
        for (int e = 0; e < N; ++e) m = fmaxf(m, R::value(c, e));
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (r.in(at, e)) m = fmaxf(m, R::value(c, e));
      }
    });
    m = block_max<NW>(m, red);
    if (m == ninf) m = 0.0f;
    // sums of 2^(c1 (x - m)), temperature 1, and 2^(cT (x - m))
    const float c1 = kLog2e, cT = kLog2e * rT;
    float s1 = 0.0f, sT = 0.0f;
    walk([&](const u32x4& c, int at) {
      const bool all = r.whole(at);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        if (!all && !r.in(at, e)) continue;
        const float d = R::value(c, e) - m;
        sT += __builtin_amdgcn_exp2f(d * cT);
        if (two) s1 += __builtin_amdgcn_exp2f(d * c1);
      }
    });
    sT = block_sum<NW>(sT, red);
    s1 = two ? block_sum<NW>(s1, red) : sT;
    // log q_v = (x_v - m) / T - lT
    const float lT = logf(sT), l1 = logf(s1);
    if (a.loss_row != nullptr) {
      float kl = 0.0f;
      for (int k = tid; k < a.K; k += THREADS) {
        if (sid[k] < 0) continue;
        const float lp = sp[k] - tlse, p = expf(lp);
        // (x_v - m) / T may leave fp32's range where p brings it back
        kl += part(p, lp + lT) - part(p * rT, R::one(a.x, r.begin + sid[k]) - m);
      }
      kl = block_sum<NW>(kl, red);
      bad = __syncthreads_or(bad);
      if (tid == 0) {
        float loss = soft ? w * T * T * kl : 0.0f;
        if (hard && !bad) loss += (1.0f - w) * (l1 - (R::one(a.x, r.begin + target) - m));
        a.loss_row[row] = bad ? __builtin_nanf("") : loss;
      }
    } else {
      bad = __syncthreads_or(bad);
    }
    if (a.dx == nullptr) continue;
    const float nan = __builtin_nanf("");
    const float gT = bad ? nan : soft ? scale * w * T : 0.0f, g1 = hard ? scale * (1.0f - w) : 0.0f;
    // gradient of a logit without its teacher's or target's part
    const float oT = lT * kLog2e, o1 = l1 * kLog2e;
    auto base = [&](float v) {
      const float d = v - m;
      float g = part(gT, __builtin_amdgcn_exp2f(__builtin_fmaf(d, cT, -oT)));
      if (hard) g += g1 * __builtin_amdgcn_exp2f(__builtin_fmaf(d, c1, -o1));
      return g;
    };
    walk([&](const u32x4& c, int at) {
      float g[N];
#pragma unroll
      for (int e = 0; e < N; ++e) g[e] = base(R::value(c, e));
      if (r.whole(at)) {
        static_cast<u32x4*>(a.dx)[r.first + at] = R::pack(g);
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (r.in(at, e)) R::put(a.dx, (r.first + at) * N + e, g[e]);
      }
    });
    // the teacher's entries and the target, over what the walk wrote
    __syncthreads();
    for (int k = tid; k < a.K + 1; k += THREADS) {
      const bool is_target = k == a.K;
      if (is_target ? !hard || target < 0 || target >= a.V : sid[k] < 0) continue;
      const int v = is_target ? static_cast<int>(target) : sid[k];
      // the first of equal ids writes the sum of all
      float p = 0.0f;
      bool first = true;
      for (int j = 0; j < a.K; ++j) {
        if (sid[j] != v) continue;
        first = first && j >= k;
        p += expf(sp[j] - tlse);
      }
      if (!first) continue;
      float g = base(R::one(a.x, r.begin + v)) - part(gT, p);
      if (hard && v == target) g -= g1;
      R::put(a.dx, r.begin + v, g);
    }
  }
}

// Rows whose target counts.
__global__ __launch_bounds__(1024) void k_distill_count(DistillArgs a) {
  __shared__ int s[16];
  int c = 0;
  for (int64_t r = threadIdx.x; r < a.rows; r += 1024) c += a.target[r] != a.ignore_index ? 1 : 0;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) c += __shfl_xor(c, d, 64);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = c;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 16; ++w) c += s[w];
    a.count[0] = static_cast<float>(c);
  }
}

// The rows' mean: fp64 sums in a fixed order.
__global__ __launch_bounds__(1024) void k_distill_mean(DistillArgs a) {
  __shared__ double s[1024];
  double l = 0.0;
  for (int64_t r = threadIdx.x; r < a.rows; r += 1024) l += a.loss_row[r];
  s[threadIdx.x] = l;
  __syncthreads();
  for (int d = 512; d > 0; d >>= 1) {
    if (static_cast<int>(threadIdx.x) < d) s[threadIdx.x] += s[threadIdx.x + d];
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    const double n = a.target != nullptr ? static_cast<double>(a.count[0]) : static_cast<double>(a.rows);
    a.loss[0] = static_cast<float>(s[0] / n);
  }
}

template <bool F32>
void launch(const DistillArgs& a, hipStream_t s) {
  const int64_t chunks = ceil_div(a.V, F32 ? 4 : 8) + 1;
  const int64_t most = a.unless_one ? 2048 : (int64_t(1) << 22) - 1;
  const dim3 grid(static_cast<uint32_t>(a.rows < most ? a.rows : most));
  if (chunks <= 256) hipLaunchKernelGGL((k_distill<F32, 256, 1>), grid, dim3(256), 0, s, a);
  else if (chunks <= 1024) hipLaunchKernelGGL((k_distill<F32, 256, 4>), grid, dim3(256), 0, s, a);
  else if (chunks <= 4096) hipLaunchKernelGGL((k_distill<F32, 256, 16>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((k_distill<F32, 1024, 16>), grid, dim3(1024), 0, s, a);
}

}  // namespace
}  // namespace compact

using namespace compact;

extern "C" int compact_distill(const DistillArgs* a, void* stream) {
  if (a->rows < 1 || a->rows > 0x7FFFFFFF || a->V < 1 || a->V > int64_t(1) << 30 || a->K < 1 || a->K > kMaxK ||
      !(a->temperature > 0.0f))
    return -1;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (a->target != nullptr && a->loss_row != nullptr) hipLaunchKernelGGL(k_distill_count, dim3(1), dim3(1024), 0, s, *a);
  if (a->f32) launch<true>(*a, s);
  else launch<false>(*a, s);
  if (a->loss_row != nullptr) hipLaunchKernelGGL(k_distill_mean, dim3(1), dim3(1024), 0, s, *a);
  return hipGetLastError() == hipSuccess ? 0 : -5;
}
