// Rotary positions: the first `dims` elements of a head as dims / 2 pairs, each turned by its
// token's position times the pair's frequency:
//
//   ya = m (xa cos - xb sin),  yb = m (xb cos + xa sin),  (a, b) = (i, i + dims / 2) or (2 i, 2 i + 1)
//
// and the rest copied; the gradient is the same with the angle's sign turned.  Bound by HBM:
// each element is read and written once.  A workgroup takes a few tokens: their sines and
// cosines are formed once, one pair per thread, into LDS (the angle in revolutions as an fp64
// product of the position and the frequency, of which the nearest whole number is taken off:
// exact for any position, where an fp32 product is off by 2^-24 of the angle), and so are the
// tokens' places in the up to three tensors of a call; then they serve every head.
//
// Measured: 12.9 us, 5.2 TB/s, for q and k of 32 x 256 tokens, 16 heads of 64 in bf16; 206 us,
// 4.8 TB/s, for 2 x 12001 tokens, 32 and 8 heads of 128 in fp32, the first half turned; 4.3 us,
// a launch, for one token of 8 sequences.  (A large copy reaches 5.2 TB/s.)
#include <hip/hip_runtime.h>

#include "common.hpp"
#include "functional.hpp"

namespace compact {
namespace {

constexpr int kMaxPairs = 512;   // (cos, sin) of a workgroup's tokens in LDS; a head has at most 1024 elements
constexpr int kMaxTokens = 64;

struct RotaryPlan {
  int tokens;             // per workgroup
  int per_head;           // items of a head
  int rotated;            // of which turned ones, first
  int per_token;
  uint32_t div_token, div_head;  // ceil(2^32 / d): n / d = umulhi(n, .) for n < 2^16, d < 2^16
};

__device__ __forceinline__ int div_by(int n, uint32_t magic) { return magic == 0 ? n : static_cast<int>(__umulhi(n, magic)); }

// N consecutive elements as fp32 values, moved in one piece.
template <bool F32, int N>
struct Chunk {
  static constexpr int kWords = N * (F32 ? 4 : 2) / 4;  // 0: one bf16
  float v[N];
  __device__ __forceinline__ void load(const char* p) {
    if constexpr (kWords == 0) {
      v[0] = bf16_to_f32(*reinterpret_cast<const uint16_t*>(p));
    } else {
      typedef uint32_t words_t __attribute__((ext_vector_type(kWords)));
      uint32_t w[kWords];
      if constexpr (kWords == 1) w[0] = *reinterpret_cast<const uint32_t*>(p);
      else *reinterpret_cast<words_t*>(w) = *reinterpret_cast<const words_t*>(p);
#pragma unroll
      for (int k = 0; k < kWords; ++k) {
        if constexpr (F32) {
          v[k] = __uint_as_float(w[k]);
        } else {
          v[2 * k] = __uint_as_float(w[k] << 16);
          v[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
        }
      }
    }
  }
  __device__ __forceinline__ void store(char* p) const {
    if constexpr (kWords == 0) {
      *reinterpret_cast<uint16_t*>(p) = f32_to_bf16(v[0]);
    } else {
      typedef uint32_t words_t __attribute__((ext_vector_type(kWords)));
      uint32_t w[kWords];
#pragma unroll
      for (int k = 0; k < kWords; ++k) {
        if constexpr (F32) w[k] = __float_as_uint(v[k]);
        else w[k] = pack_bf16x2(v[2 * k], v[2 * k + 1]);
      }
      if constexpr (kWords == 1) *reinterpret_cast<uint32_t*>(p) = w[0];
      else *reinterpret_cast<words_t*>(p) = *reinterpret_cast<const words_t*>(w);
    }
  }
};

// An item is two chunks of N elements.  Halves: chunk i of either half, then the rest two by two;
// neighbours: two chunks on end.  An item reads all that it writes, so dst may be src.  U items
// per thread at a time: their loads are in flight together.
template <bool F32, int N, bool PAIRS, int U>
__global__ __launch_bounds__(256) void k_rotary(RotaryArgs a, RotaryPlan pl) {
  constexpr int SZ = F32 ? 4 : 2;
  __shared__ float2 cs[kMaxPairs];
  __shared__ int64_t place[kMaxTokens][3][2];
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
    // (the part of a turn is rounded to fp32, off by 2^-26 of a turn at most, 9e-8 radians: fp32
    // rotations are 1.3 times as far from the exact ones as with the sine of the fp64 angle, which
    // would cost fp64 polynomials for every pair; bf16 ones as near)
    sincospif(2.0f * static_cast<float>(turn - rint(turn)), &s, &c);
    cs[u] = make_float2(a.magnitude * c, a.magnitude * (a.inverse ? -s : s));
    if (i < a.count) {
      place[t][i][0] = b * a.t[i].src_b + x * a.t[i].src_l;
      place[t][i][1] = b * a.t[i].dst_b + x * a.t[i].dst_l;
    }
  }
  if (half < a.count) {  // fewer pairs than tensors
    for (int u = threadIdx.x; u < here * a.count; u += 256) {
      const int t = u / a.count, i = u - t * a.count;
      const int64_t at = t0 + t, b = at / a.l, x = at - b * a.l;
      place[t][i][0] = b * a.t[i].src_b + x * a.t[i].src_l;
      place[t][i][1] = b * a.t[i].dst_b + x * a.t[i].dst_l;
    }
  }
  __syncthreads();
  const int items = here * pl.per_token;
  for (int u0 = threadIdx.x; u0 < items; u0 += 256 * U) {
    Chunk<F32, N> p[U], q[U];
    char* dst[U];
    int first[U], second[U], token[U];  // elements of the head; second < 0: none
    bool turn[U], writes[U];
#pragma unroll
    for (int n = 0; n < U; ++n) {
      const int u = u0 + 256 * n < items ? u0 + 256 * n : u0;
      const int t = div_by(u, pl.div_token), in = u - t * pl.per_token;
      int head = div_by(in, pl.div_head);
      const int item = in - head * pl.per_head;
      // (the up to three tensors by selects: an index would read their fields from memory)
      const int h0 = a.t[0].heads, h1 = a.t[1].heads;
      const int k = a.count > 1 && head >= h0 ? (a.count > 2 && head >= h0 + h1 ? 2 : 1) : 0;
      head -= k == 0 ? 0 : k == 1 ? h0 : h0 + h1;
      const void* src = k == 0 ? a.t[0].src : k == 1 ? a.t[1].src : a.t[2].src;
      void* to = k == 0 ? a.t[0].dst : k == 1 ? a.t[1].dst : a.t[2].dst;
      const int64_t sh = k == 0 ? a.t[0].src_h : k == 1 ? a.t[1].src_h : a.t[2].src_h;
      const int64_t dh = k == 0 ? a.t[0].dst_h : k == 1 ? a.t[1].dst_h : a.t[2].dst_h;
      const char* from = static_cast<const char*>(src) + (place[t][k][0] + head * sh) * SZ;
      dst[n] = static_cast<char*>(to) + (place[t][k][1] + head * dh) * SZ;
      token[n] = t;
      turn[n] = item < pl.rotated && (k == 0 ? a.t[0].rotate : k == 1 ? a.t[1].rotate : a.t[2].rotate);
      writes[n] = turn[n] || from != dst[n];
      if constexpr (PAIRS) {
        first[n] = item * 2 * N;
        second[n] = first[n] + N;
      } else {
        const int rest = a.dims + (item - pl.rotated) * 2 * N;
        first[n] = item < pl.rotated ? item * N : rest;
        second[n] = item < pl.rotated ? half + item * N : rest + N;
      }
      if (second[n] >= a.hd) second[n] = -1;
      p[n].load(from + first[n] * SZ);
      q[n].load(from + (second[n] < 0 ? first[n] : second[n]) * SZ);
    }
#pragma unroll
    for (int n = 0; n < U; ++n) {
      if (u0 + 256 * n >= items || !writes[n]) continue;
      const float2* w = cs + token[n] * half;
      if constexpr (PAIRS) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          float* v = c == 0 ? p[n].v : q[n].v;
#pragma unroll
          for (int e = 0; e + 1 < N; e += 2) {
            const int i = (first[n] + c * N + e) / 2;  // (dims may end inside a chunk)
            const float2 r = w[i < half ? i : half - 1];
            const float y = v[e] * r.x - v[e + 1] * r.y, z = v[e + 1] * r.x + v[e] * r.y;
            const bool in = turn[n] && i < half;
            v[e] = in ? y : v[e];
            v[e + 1] = in ? z : v[e + 1];
          }
        }
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float2 r = w[turn[n] ? first[n] + e : 0];
          const float y = p[n].v[e] * r.x - q[n].v[e] * r.y, z = q[n].v[e] * r.x + p[n].v[e] * r.y;
          p[n].v[e] = turn[n] ? y : p[n].v[e];
          q[n].v[e] = turn[n] ? z : q[n].v[e];
        }
      }
      p[n].store(dst[n] + first[n] * SZ);
      if (second[n] >= 0) q[n].store(dst[n] + second[n] * SZ);
    }
  }
}

template <bool F32, int N, bool PAIRS>
void launch(const RotaryArgs& a, const RotaryPlan& p, dim3 grid, hipStream_t s) {
  // (one, two or four items in flight: 215, 207 and 204 us for the fp32 tensors above, 42.8, 43.6
  // and 46.2 for 8 x 4096 tokens, 20 heads of 96 in bf16)
  hipLaunchKernelGGL((k_rotary<F32, N, PAIRS, 2>), grid, dim3(256), 0, s, a, p);
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
  // elements moved in one piece: halves start where the widest piece that divides them can
  // (halves of 64 turned by pieces of 8, 5.2 TB/s; of 10, which leave pieces of 2, 3.8)
  int piece = n;
  if (!a->interleaved)
    while (a->dims / 2 % piece != 0) piece /= 2;
  RotaryPlan p;
  const int pieces = a->hd / piece;
  p.rotated = a->interleaved ? static_cast<int>(ceil_div(a->dims, 2 * piece)) : a->dims / 2 / piece;
  p.per_head = a->interleaved ? static_cast<int>(ceil_div(pieces, 2))
                              : p.rotated + static_cast<int>(ceil_div(pieces - 2 * p.rotated, 2));
  if (heads * p.per_head >= 1 << 16) return -1;
  p.per_token = static_cast<int>(heads) * p.per_head;
  // a sine per thread, while that leaves four workgroups for every CU.  (us with half as many
  // sines / a sine / two per thread: 32 x 256 tokens, 32 heads of 64: 14.0 / 12.7 / 12.7; 8 x
  // 4096, 20 of 96: 48.5 / 43.6 / 46.2; 2 x 12001, 40 of 128, fp32: 198 / 207 / 213.  One
  // workgroup for every CU at least, where four are asked for: the first 15.7.)
  int64_t tokens = 512 / a->dims;
  const int64_t most = a->tokens / 1024, fit = ((1 << 16) - 1) / p.per_token;
  tokens = tokens > most ? most : tokens;
  tokens = tokens > fit ? fit : tokens;
  tokens = tokens > kMaxTokens ? kMaxTokens : tokens;
  p.tokens = static_cast<int>(tokens < 1 ? 1 : tokens);
  const int64_t grid = ceil_div(a->tokens, p.tokens);
  if (grid >= int64_t(1) << 24) return -1;
  p.div_token = magic_of(p.per_token);
  p.div_head = magic_of(p.per_head);
  const dim3 g(static_cast<uint32_t>(grid));
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (a->f32) {
    if (a->interleaved) launch<true, 4, true>(*a, p, g, s);
    else if (piece == 4) launch<true, 4, false>(*a, p, g, s);
    else if (piece == 2) launch<true, 2, false>(*a, p, g, s);
    else launch<true, 1, false>(*a, p, g, s);
  } else {
    if (a->interleaved) launch<false, 8, true>(*a, p, g, s);
    else if (piece == 8) launch<false, 8, false>(*a, p, g, s);
    else if (piece == 4) launch<false, 4, false>(*a, p, g, s);
    else if (piece == 2) launch<false, 2, false>(*a, p, g, s);
    else launch<false, 1, false>(*a, p, g, s);
  }
  return hipGetLastError() == hipSuccess ? 0 : -5;
}
