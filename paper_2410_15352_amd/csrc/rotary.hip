// Rotary positions: the first `dims` elements of a head as dims / 2 pairs, each turned by its
// token's position times the pair's frequency:
//
//   ya = m (xa cos - xb sin),  yb = m (xb cos + xa sin),  (a, b) = (i, i + dims / 2) or (2 i, 2 i + 1)
//
// and the rest copied; the gradient is the same with the angle's sign turned.  Bound by HBM:
// each element is read and written once.  A workgroup takes a few tokens: their sines and
// cosines are formed once, one pair per thread, into LDS (the angle in revolutions as an fp64
// product of the position and the frequency, of which the nearest whole number is taken off:
// exact for any position, where an fp32 product is off by 2^-24 of the angle), and then serve
// every head of the up to three tensors of a call.
#include <hip/hip_runtime.h>

#include "common.hpp"
#include "functional.hpp"

namespace compact {
namespace {

constexpr int kMaxPairs = 512;  // (cos, sin) of a workgroup's tokens in LDS; a head has at most 1024 elements

struct RotaryPlan {
  int tokens;             // per workgroup
  int per_head;           // items of a head: rotated ones first, then copied chunks
  int rotated;
  int per_token;
  uint32_t div_token, div_head;  // ceil(2^32 / d): n / d = umulhi(n, .) for n < 2^16, d < 2^16
};

__device__ __forceinline__ int div_by(int n, uint32_t magic) { return magic == 0 ? n : static_cast<int>(__umulhi(n, magic)); }

// A 16-byte chunk as fp32 values: 8 of bf16 or 4 of fp32.
template <bool F32>
struct Chunk {
  static constexpr int kN = F32 ? 4 : 8;
  float v[kN];
  __device__ __forceinline__ void load(const char* p) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (F32) {
        v[k] = __uint_as_float(w[k]);
      } else {
        v[2 * k] = __uint_as_float(w[k] << 16);
        v[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
      }
    }
  }
  __device__ __forceinline__ void store(char* p) const {
    u32x4 w;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (F32) w[k] = __float_as_uint(v[k]);
      else w[k] = pack_bf16x2(v[2 * k], v[2 * k + 1]);
    }
    *reinterpret_cast<u32x4*>(p) = w;
  }
};

template <bool F32>
__device__ __forceinline__ float load1(const char* p) {
  if constexpr (F32) return *reinterpret_cast<const float*>(p);
  else return bf16_to_f32(*reinterpret_cast<const uint16_t*>(p));
}
template <bool F32>
__device__ __forceinline__ void store1(char* p, float v) {
  if constexpr (F32) *reinterpret_cast<float*>(p) = v;
  else *reinterpret_cast<uint16_t*>(p) = f32_to_bf16(v);
}

// LAYOUT 0: halves, dims / 2 whole chunks: an item is two chunks; 1: halves, any dims: an item
// is one pair (element by element); 2: neighbours: an item is one chunk.  An item reads all
// that it writes, so dst may be src.
template <bool F32, int LAYOUT>
__global__ __launch_bounds__(256) void k_rotary(RotaryArgs a, RotaryPlan pl) {
  constexpr int N = Chunk<F32>::kN, SZ = F32 ? 4 : 2;
  __shared__ float2 cs[kMaxPairs];
  const int half = a.dims / 2;
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * pl.tokens;
  const int here = static_cast<int>(a.tokens - t0 < pl.tokens ? a.tokens - t0 : pl.tokens);
  for (int u = threadIdx.x; u < here * half; u += 256) {
    const int t = u / half, i = u - t * half;
    const int64_t at = t0 + t, b = at / a.l, x = at - b * a.l;
    int64_t pos = a.offset + x;
    if (a.positions != nullptr) {
      const int64_t o = b * a.pos_b + x * a.pos_l;
      pos = a.pos32 ? static_cast<const int32_t*>(a.positions)[o] : static_cast<const int64_t*>(a.positions)[o];
    }
    const double turn = static_cast<double>(pos) * a.turns[i];
    float s, c;
    sincospif(2.0f * static_cast<float>(turn - rint(turn)), &s, &c);
    cs[u] = make_float2(a.magnitude * c, a.magnitude * (a.inverse ? -s : s));
  }
  __syncthreads();
  for (int u = threadIdx.x; u < here * pl.per_token; u += 256) {
    const int t = div_by(u, pl.div_token), in = u - t * pl.per_token;
    int head = div_by(in, pl.div_head);
    const int item = in - head * pl.per_head;
    int k = 0;
    if (a.count > 1 && head >= a.t[0].heads) {
      head -= a.t[0].heads;
      k = 1;
      if (a.count > 2 && head >= a.t[1].heads) {
        head -= a.t[1].heads;
        k = 2;
      }
    }
    const RotaryTensor& x = a.t[k];
    const int64_t at = t0 + t, b = at / a.l, l = at - b * a.l;
    const char* src = static_cast<const char*>(x.src) + (b * x.src_b + l * x.src_l + head * x.src_h) * SZ;
    char* dst = static_cast<char*>(x.dst) + (b * x.dst_b + l * x.dst_l + head * x.dst_h) * SZ;
    const float2* w = cs + t * half;
    if (item >= pl.rotated) {  // past dims
      const int e = LAYOUT == 0 ? a.dims + (item - pl.rotated) * N : LAYOUT == 1 ? a.dims + (item - pl.rotated) : item * N;
      if (src == dst) continue;
      if constexpr (LAYOUT == 1) store1<F32>(dst + e * SZ, load1<F32>(src + e * SZ));
      else *reinterpret_cast<u32x4*>(dst + e * SZ) = *reinterpret_cast<const u32x4*>(src + e * SZ);
      continue;
    }
    if constexpr (LAYOUT == 0) {
      Chunk<F32> p, q;
      p.load(src + item * 16);
      q.load(src + half * SZ + item * 16);
      if (x.rotate) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float2 r = w[item * N + e];
          const float y = p.v[e] * r.x - q.v[e] * r.y;
          q.v[e] = q.v[e] * r.x + p.v[e] * r.y;
          p.v[e] = y;
        }
      }
      p.store(dst + item * 16);
      q.store(dst + half * SZ + item * 16);
    } else if constexpr (LAYOUT == 1) {
      float p = load1<F32>(src + item * SZ), q = load1<F32>(src + (half + item) * SZ);
      if (x.rotate) {
        const float2 r = w[item];
        const float y = p * r.x - q * r.y;
        q = q * r.x + p * r.y;
        p = y;
      }
      store1<F32>(dst + item * SZ, p);
      store1<F32>(dst + (half + item) * SZ, q);
    } else {
      Chunk<F32> p;
      p.load(src + item * 16);
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        if (item * N + e < a.dims && x.rotate) {  // (dims may end inside a chunk)
          const float2 r = w[item * (N / 2) + e / 2];
          const float y = p.v[e] * r.x - p.v[e + 1] * r.y;
          p.v[e + 1] = p.v[e + 1] * r.x + p.v[e] * r.y;
          p.v[e] = y;
        }
      }
      p.store(dst + item * 16);
    }
  }
}

uint32_t magic_of(int d) { return d == 1 ? 0 : static_cast<uint32_t>(((uint64_t(1) << 32) + d - 1) / d); }

}  // namespace
}  // namespace compact

using namespace compact;

extern "C" int compact_rotary(const RotaryArgs* a, void* stream) {
  const int n = a->f32 ? 4 : 8;
  if (a->count < 1 || a->count > 3 || a->tokens < 1 || a->l < 1 || a->hd < n || a->hd % n != 0 || a->hd > 1024 ||
      a->dims < 2 || a->dims % 2 != 0 || a->dims > a->hd)
    return -1;
  int64_t heads = 0;
  for (int i = 0; i < a->count; ++i) {
    if (a->t[i].heads < 1) return -1;
    heads += a->t[i].heads;
  }
  const int layout = a->interleaved ? 2 : a->dims / 2 % n == 0 ? 0 : 1;
  RotaryPlan p;
  p.rotated = layout == 2 ? static_cast<int>(ceil_div(a->dims, n)) : layout == 0 ? a->dims / 2 / n : a->dims / 2;
  p.per_head = p.rotated + (layout == 2 ? a->hd / n - p.rotated : layout == 0 ? (a->hd - a->dims) / n : a->hd - a->dims);
  if (heads * p.per_head >= 1 << 16) return -1;
  p.per_token = static_cast<int>(heads) * p.per_head;
  // a sine per thread, while that leaves four workgroups for every CU
  int64_t tokens = 512 / a->dims;
  const int64_t most = a->tokens / 1024, fit = ((1 << 16) - 1) / p.per_token;
  tokens = tokens > most ? most : tokens;
  tokens = tokens > fit ? fit : tokens;
  p.tokens = static_cast<int>(tokens < 1 ? 1 : tokens);
  const int64_t grid = ceil_div(a->tokens, p.tokens);
  if (grid >= int64_t(1) << 24) return -1;
  p.div_token = magic_of(p.per_token);
  p.div_head = magic_of(p.per_head);
  const dim3 g(static_cast<uint32_t>(grid)), t(256);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (a->f32) {
    if (layout == 0) hipLaunchKernelGGL((k_rotary<true, 0>), g, t, 0, s, *a, p);
    else if (layout == 1) hipLaunchKernelGGL((k_rotary<true, 1>), g, t, 0, s, *a, p);
    else hipLaunchKernelGGL((k_rotary<true, 2>), g, t, 0, s, *a, p);
  } else {
    if (layout == 0) hipLaunchKernelGGL((k_rotary<false, 0>), g, t, 0, s, *a, p);
    else if (layout == 1) hipLaunchKernelGGL((k_rotary<false, 1>), g, t, 0, s, *a, p);
    else hipLaunchKernelGGL((k_rotary<false, 2>), g, t, 0, s, *a, p);
  }
  return hipGetLastError() == hipSuccess ? 0 : -5;
}
