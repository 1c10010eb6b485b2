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
// walks over registers, and the next row's loads are issued chunk by chunk behind the
// gradient's.  The gradient is formed where the loss is, for dloss = 1; the backward runs
// the same kernel again, which ends at once where dloss is 1 indeed.
//
// Measured, loss and gradient in bf16 (medians of 100 passes in a row): 8192 rows of 32000 logits
// 235 us, 4.5 TB/s, at T = 2 with targets (two exponentials per logit and walk), 224 us, 4.7 TB/s, at
// T = 1; 4096 rows of 131072 without targets 484 us, 4.4 TB/s; a large copy reaches 5.2 TB/s.  Beside
// them 12 to 15 us of the entries' kernel, 5 of the mean's and 5 of the backward's look at dloss.
// Rows of a thousand logits are bound by a row's chain of walks and barriers: 16384 of them 56 us,
// 1.2 TB/s, and 18 for the entries.
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

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d, 64));
  return v;
}

// A value that every lane holds, as a scalar.
__device__ __forceinline__ float uniform(float v) {
  return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v)));
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
  return v;
}

// A row as the whole 16-byte chunks of the buffer that lie inside it and, an odd V starting
// rows anywhere, up to two ends of single elements, one to a thread.
template <bool F32>
struct Row {
  static constexpr int kN = F32 ? 4 : 8, kSize = F32 ? 4 : 2;
  static constexpr uint32_t kNone = F32 ? 0xFF800000u : 0xFF80FF80u;  // -inf
  int64_t begin;    // the row's first element
  int head, chunks, tail;  // elements before the first whole chunk, whole chunks, elements after
  __device__ __forceinline__ Row(int64_t row, int64_t V) {
    begin = row * V;
    const int off = static_cast<int>(begin % kN), v = static_cast<int>(V);
    head = off == 0 ? 0 : kN - off;
    head = head < v ? head : v;
    chunks = (v - head) / kN;
    tail = v - head - chunks * kN;
  }
  // the element of the ends that is thread t's, or -1
  __device__ __forceinline__ int end_of(int t) const { return t < head ? t : t < head + tail ? chunks * kN + t : -1; }
  // The whole chunks from `skip` on as a buffer: loads past the last give zeros, stores nothing.
  // (`some`: else an empty one, whose loads cost nothing.  A buffer for each of a thread's
  // chunks lets all of them use the same offset: scalars instead of a register each.)
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t from(const void* x, bool some, int skip) const {
    char* at = const_cast<char*>(static_cast<const char*>(x)) + (begin + head) * kSize + skip * 16;
    return __builtin_amdgcn_make_buffer_rsrc(at, static_cast<short>(0), some && skip < chunks ? (chunks - skip) * 16 : 0, 0x00020000);
  }
  __device__ __forceinline__ u32x4 load(const void* x, bool some, int skip, int tid) const {
    return __builtin_amdgcn_raw_buffer_load_b128(from(x, some, skip), tid * 16, 0, 0);
  }
  // -inf for what is past the last chunk.  (Not in load: it would wait there.)
  __device__ __forceinline__ void ends(u32x4& w, int c) const {
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = c < chunks ? w[k] : kNone;
  }
  __device__ __forceinline__ void store(void* x, int skip, int tid, const float (&v)[kN]) const {
    u32x4 w;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (F32) w[k] = __float_as_uint(v[k]);
      else w[k] = pack_bf16x2(v[2 * k], v[2 * k + 1]);
    }
    __builtin_amdgcn_raw_buffer_store_b128(w, from(x, true, skip), tid * 16, 0, 0);
  }
  static __device__ __forceinline__ float value(const u32x4& w, int e) {
    if constexpr (F32) return __uint_as_float(w[e]);
    else return __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
  }
  __device__ __forceinline__ float one(const void* x, uint32_t v) const {
    if constexpr (F32) return (static_cast<const float*>(x) + begin)[v];
    else return bf16_to_f32((static_cast<const uint16_t*>(x) + begin)[v]);
  }
  __device__ __forceinline__ void put(void* x, uint32_t v, float g) const {
    if constexpr (F32) (static_cast<float*>(x) + begin)[v] = g;
    else (static_cast<uint16_t*>(x) + begin)[v] = f32_to_bf16(g);
  }
};

// The teacher's entries of a row as the main kernel wants them, by one wave: distinct ids, each
// with the sum of its p, and behind them the target's, if it is not among them, with p = 0.
// Workgroup 0 counts the rows whose target counts.
__global__ __launch_bounds__(256) void k_distill_entries(DistillArgs a) {
  extern __shared__ __attribute__((aligned(16))) int lds[];  // per wave: K ids and K values, K to a multiple of 4
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, K4 = (a.K + 3) / 4 * 4;
  if (blockIdx.x == 0) {
    if (a.target == nullptr) return;
    int c = 0;
#pragma unroll 8
    for (int64_t r = threadIdx.x; r < a.rows; r += 256) c += a.target[r] != a.ignore_index ? 1 : 0;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) c += __shfl_xor(c, d, 64);
    if (lane == 0) lds[wave] = c;
    __syncthreads();
    if (threadIdx.x == 0) a.count[0] = static_cast<float>(lds[0] + lds[1] + lds[2] + lds[3]);
    return;
  }
  int* sid = lds + wave * 2 * K4;
  float* sp = reinterpret_cast<float*>(sid + K4);
  const int64_t row = (static_cast<int64_t>(blockIdx.x) - 1) * 4 + wave;
  if (row >= a.rows) return;
  const int64_t target = a.target != nullptr ? a.target[row] : a.ignore_index - 1;
  const bool hard = a.target != nullptr && a.weight != 1.0f, aim = hard && target >= 0 && target < a.V;
  const char* ids = static_cast<const char*>(a.ids) + row * a.ids_ld * (a.ids32 ? 4 : 8);
  const char* top = static_cast<const char*>(a.top) + row * a.top_ld * (a.top32 ? 4 : 2);
  const float ninf = -__builtin_inff(), rT = 1.0f / a.temperature;
  bool bad = hard && !aim, among = false;
  float m = ninf;
  for (int k = lane; k < K4; k += 64) {
    int id = -1;
    float t = ninf;
    if (k < a.K) {
      const int64_t given = a.ids32 ? reinterpret_cast<const int32_t*>(ids)[k] : reinterpret_cast<const int64_t*>(ids)[k];
      t = a.top32 ? reinterpret_cast<const float*>(top)[k] : bf16_to_f32(reinterpret_cast<const uint16_t*>(top)[k]);
      t = given < 0 ? ninf : t * rT;
      bad |= given >= a.V;
      id = given < 0 || given >= a.V ? -1 : static_cast<int>(given);
      among |= aim && given == target;
    }
    sid[k] = id;
    sp[k] = t;
    m = fmaxf(m, t);
  }
  if (a.target != nullptr && target == a.ignore_index) return;
  m = wave_max(m);
  if (m == ninf) m = 0.0f;
  float s = 0.0f;
  for (int k = lane; k < K4; k += 64) s += expf(sp[k] - m);
  s = wave_sum(s);
  const float lse = m + logf(s);
  const bool some = !(s == 0.0f);  // (a NaN is an entry)
  float h = 0.0f;
  for (int k = lane; k < K4; k += 64) {
    const float lp = sp[k] - lse, p = some ? expf(lp) : 0.0f;
    h += part(p, lp);
    sp[k] = p;
  }
  h = wave_sum(h);
  int2* out = reinterpret_cast<int2*>(a.entries) + row * (a.K + 1);
  for (int k = lane; k < a.K; k += 64) {
    const int id = sid[k];
    float p = 0.0f;
    int before = 0;  // equal ids before this one: the first has the sum of all
#pragma unroll 4
    for (int j = 0; j < K4; j += 4) {
      const int4 v = *reinterpret_cast<const int4*>(sid + j);
      const float4 q = *reinterpret_cast<const float4*>(sp + j);
      p += (v.x == id ? q.x : 0.0f) + (v.y == id ? q.y : 0.0f) + (v.z == id ? q.z : 0.0f) + (v.w == id ? q.w : 0.0f);
      before |= ((v.x == id) & (j < k)) | ((v.y == id) & (j + 1 < k)) | ((v.z == id) & (j + 2 < k)) | ((v.w == id) & (j + 3 < k));
    }
    const bool one = id >= 0 && !before;
    out[k] = make_int2(one ? id : -1, __float_as_int(one ? p : 0.0f));
  }
  among = __any(among);
  bad = __any(bad);
  if (lane == 0) {
    out[a.K] = make_int2(aim && !among ? static_cast<int>(target) : -1, 0);
    a.stats[2 * row] = bad ? __builtin_nanf("") : h;
    a.stats[2 * row + 1] = some ? 1.0f : 0.0f;
  }
}

// One row per workgroup at a time; NC chunks per thread in registers, any more are read again
// for each walk.  HARD: the targets have a part; TWO: at another temperature than the teacher.
template <bool F32, int THREADS, int NC, bool HARD, bool TWO>
__global__ __launch_bounds__(THREADS, 4) void k_distill(DistillArgs a) {
  using R = Row<F32>;
  constexpr int N = R::kN, NW = THREADS / 64;
  __shared__ float smax[NW], ssum[NW][3];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float ninf = -__builtin_inff(), nan = __builtin_nanf("");
  float scale = 1.0f;
  if (a.dloss != nullptr) {
    scale = a.dloss[0];
    if (a.unless_one && scale == 1.0f) return;
  }
  scale = uniform(scale / (a.target != nullptr ? a.count[0] : static_cast<float>(a.rows)));
  const float T = a.temperature, rT = uniform(1.0f / T), w = a.weight, cT = uniform(kLog2e * rT);
  const int entries = a.K + 1;

  u32x4 x[NC];
  float xe;   // this thread's single element
  int2 entry; // this thread's entry (any more are read where they are used)
  int64_t target;
  bool live;  // else the row has no part: no loss, no gradient, and nothing is read
  auto head_of = [&](int64_t row) {
    target = a.target != nullptr && row < a.rows ? a.target[row] : 0;
    live = row < a.rows && (a.target == nullptr || target != a.ignore_index);
  };
  auto load_ends = [&](const R& r, int64_t row) {
    xe = live && r.end_of(tid) >= 0 ? r.one(a.x, r.end_of(tid)) : ninf;
    entry = make_int2(-1, 0);
    if (live && tid < entries) entry = reinterpret_cast<const int2*>(a.entries)[row * entries + tid];
  };
  head_of(blockIdx.x);
  {
    const R r(live ? blockIdx.x : 0, a.V);
    load_ends(r, blockIdx.x);
#pragma unroll
    for (int i = 0; i < NC; ++i) x[i] = r.load(a.x, live, THREADS * i, tid);
  }
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const R r(row, a.V);
    const bool now = live;
    const int64_t aim = target;
    // gT, g1: the factors of the two softmaxes' gradients, gT / sT and g1 / s1 their exponentials'
    float m = now ? xe : 0.0f, gT = 0.0f, g1 = 0.0f, eT = 0.0f, e1 = 0.0f, xv = 0.0f;
    if (now) {
      // logits that the entries and the target name, on their way while the row is walked
      if (entry.x >= 0) xv = r.one(a.x, entry.x);
      float xt = 0.0f;
      if (HARD && tid == 0 && aim >= 0 && aim < a.V) xt = r.one(a.x, static_cast<uint32_t>(aim));
      const float h = a.stats[2 * row];
      const bool soft = a.stats[2 * row + 1] != 0.0f;
      // f(chunk's words) over this thread's chunks.  (Each walk unpacks the words again: kept from
      // one to the next, the values would take twice the registers.)
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
      // sums of 2^(cT (x - m)), of the same at temperature 1, and of the entries' p (x - m) / T
      float sT = __builtin_amdgcn_exp2f((xe - m) * cT), s1 = __builtin_amdgcn_exp2f((xe - m) * kLog2e), sx = 0.0f;
      walk([&](const u32x4& c) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float d = R::value(c, e) - m;
          sT += __builtin_amdgcn_exp2f(d * cT);
          if constexpr (TWO) s1 += __builtin_amdgcn_exp2f(d * kLog2e);
        }
      });
      if (a.loss_row != nullptr) {
        // (p / T first: (x - m) / T may leave fp32's range where p brings it back)
        sx = part(__int_as_float(entry.y) * rT, xv - m);
#pragma unroll 1
        for (int k = tid + THREADS; k < entries; k += THREADS) {
          const int2 n = reinterpret_cast<const int2*>(a.entries)[row * entries + k];
          if (n.x >= 0) sx += part(__int_as_float(n.y) * rT, r.one(a.x, n.x) - m);
        }
        sx = wave_sum(sx);
      }
      sT = wave_sum(sT);
      if constexpr (TWO) s1 = wave_sum(s1);
      if (lane == 0) {
        ssum[wave][0] = sT;
        ssum[wave][1] = s1;
        ssum[wave][2] = sx;
      }
      __syncthreads();
      // (the waves' sums by lanes: as registers they would be too many beside the row)
      sT = wave_sum(lane < NW ? ssum[lane & (NW - 1)][0] : 0.0f);
      s1 = TWO ? wave_sum(lane < NW ? ssum[lane & (NW - 1)][1] : 0.0f) : sT;
      sx = a.loss_row != nullptr ? wave_sum(lane < NW ? ssum[lane & (NW - 1)][2] : 0.0f) : 0.0f;
      if (a.loss_row != nullptr && tid == 0) {  // log q_v = (x_v - m) / T - log sT
        float loss = soft ? w * T * T * (h + logf(sT) - sx) : 0.0f;
        if (HARD) loss += (1.0f - w) * (logf(TWO ? s1 : sT) - (xt - m));
        a.loss_row[row] = h != h ? nan : loss;
      }
      gT = h != h ? nan : soft ? scale * w * T : 0.0f;
      g1 = HARD ? scale * (1.0f - w) : 0.0f;
      // (not in the exponents: an addition and a selection less for each logit, 275 us for 286)
      eT = uniform(gT == 0.0f ? 0.0f : gT / sT);
      e1 = uniform(g1 == 0.0f ? 0.0f : g1 / (TWO ? s1 : sT));
    } else if (a.loss_row != nullptr && tid == 0) {
      a.loss_row[row] = 0.0f;
    }
    // gradient of a logit without its teacher's or target's part (a row without any part has
    // none, whatever its logits are)
    const bool none = gT == 0.0f && g1 == 0.0f;
    auto base = [&](float v) {
      const float d = v - m, u = __builtin_amdgcn_exp2f(d * cT);
      if constexpr (TWO) return __builtin_fmaf(eT, u, e1 * __builtin_amdgcn_exp2f(d * kLog2e));
      else return u * (eT + e1);
    };
    auto grad = [&](const u32x4& c, int skip) {
      float g[N] = {};
      if (!none) {
#pragma unroll
        for (int e = 0; e < N; ++e) g[e] = base(R::value(c, e));
      }
      r.store(a.dx, skip, tid, g);
    };
    const int2 named = entry;
    if (a.dx != nullptr) {
      if (r.end_of(tid) >= 0) r.put(a.dx, r.end_of(tid), none ? 0.0f : base(xe));
#pragma unroll 1
      for (int c = THREADS * NC; c + tid < r.chunks; c += THREADS) grad(r.load(a.x, true, c, tid), c);
    }
    const int64_t next_row = row + gridDim.x;
    head_of(next_row);
    const R next(live ? next_row : row, a.V);
    load_ends(next, next_row);
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      if (a.dx != nullptr) grad(x[i], THREADS * i);
      x[i] = next.load(a.x, live, THREADS * i, tid);
      __builtin_amdgcn_sched_barrier(0);  // (all loads at once would want registers of their own)
    }
    if (a.dx == nullptr || !now) continue;
    // the entries and the target, over what the walk wrote
    __syncthreads();
    auto fix = [&](const int2& n, float v) {
      float g = (none ? 0.0f : base(v)) - part(gT, __int_as_float(n.y));
      if (HARD && n.x == aim) g -= g1;
      r.put(a.dx, n.x, g);
    };
    if (named.x >= 0) fix(named, xv);
#pragma unroll 1
    for (int k = tid + THREADS; k < entries; k += THREADS) {
      const int2 n = reinterpret_cast<const int2*>(a.entries)[row * entries + k];
      if (n.x >= 0) fix(n, r.one(a.x, n.x));
    }
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

template <bool F32, int THREADS, int NC>
void launch_row(const DistillArgs& a, hipStream_t s) {
  // as many workgroups as the card holds, each with its share of the rows.  (Twice as many are
  // as fast, within 3%; but the loss alone of 4096 fp32 rows of 32000 takes 122 us for 109.)
  const int64_t most = 256 * ((NC > 4 ? 1024 : 1536) / THREADS);
  const dim3 grid(static_cast<uint32_t>(a.rows < most ? a.rows : most)), block(THREADS);
  const bool hard = a.target != nullptr && a.weight != 1.0f;
  if (!hard) hipLaunchKernelGGL((k_distill<F32, THREADS, NC, false, false>), grid, block, 0, s, a);
  else if (a.temperature == 1.0f) hipLaunchKernelGGL((k_distill<F32, THREADS, NC, true, false>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((k_distill<F32, THREADS, NC, true, true>), grid, block, 0, s, a);
}

template <bool F32>
void launch(const DistillArgs& a, hipStream_t s) {
  // The smallest workgroup whose registers hold a row, or all but the last 3% of it.  us of whole calls by
  // threads x chunks, loss and gradient in bf16 at T = 2 (the rule's *):
  //             256 x 1  256 x 4  256 x 16  512 x 16  1024 x 16
  //   16384 x   1000  84*     140      402       784      1540
  //    8192 x   8000 103       89*     211       399       782
  //    8192 x  32001 345      328      275*      419       786
  //    2048 x  65536 197      189      179       150*      224
  //    1024 x 200000 357      352      329       286       260*
  const int64_t chunks = a.V / (F32 ? 4 : 8);
  if (chunks <= 256) launch_row<F32, 256, 1>(a, s);
  else if (chunks <= 1024) launch_row<F32, 256, 4>(a, s);
  else if (chunks <= 4096 + 128) launch_row<F32, 256, 16>(a, s);
  else if (chunks <= 8192 + 256) launch_row<F32, 512, 16>(a, s);
  else launch_row<F32, 1024, 16>(a, s);
}

}  // namespace
}  // namespace compact

using namespace compact;

extern "C" int compact_distill(const DistillArgs* a, void* stream) {
  if (a->rows < 1 || a->rows > 0x7FFFFFFF || a->V < 1 || a->V > int64_t(1) << 28 || a->K < 1 || a->K > kMaxK ||
      !(a->temperature > 0.0f))
    return -1;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (!a->ready)
    hipLaunchKernelGGL(k_distill_entries, dim3(static_cast<uint32_t>(ceil_div(a->rows, 4) + 1)), dim3(256),
                       4 * 2 * sizeof(int) * ((a->K + 3) / 4 * 4), s, *a);
  if (a->f32) launch<true>(*a, s);
  else launch<false>(*a, s);
  if (a->loss_row != nullptr) hipLaunchKernelGGL(k_distill_mean, dim3(1), dim3(1024), 0, s, *a);
  return hipGetLastError() == hipSuccess ? 0 : -5;
}
