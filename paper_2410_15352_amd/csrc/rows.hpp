// Rows of logits: bf16 or fp32, of any length, read and written in 16-byte chunks; sums and maxima
// over a wave.
#pragma once
#include <hip/hip_runtime.h>

#include "common.hpp"

namespace compact {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;

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

template <typename T>
__device__ __forceinline__ T wave_sum(T v) {
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

}  // namespace
}  // namespace compact
