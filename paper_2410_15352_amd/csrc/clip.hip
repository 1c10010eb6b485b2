// The global norm of many tensors, n = sqrt(sum g^2), and g *= min(1, max / (n + 1e-6)).
//
// Bound by HBM: every element is read once for the norm, and, where it passes the bound, read and
// written once more.  Squares are added in fp64: their sum neither overflows nor vanishes for any
// bf16 or fp32 gradient, and costs less than the reading.  A tensor is cut into pieces of whole
// 16-byte chunks from its first 16-byte boundary on (up to two ends of single elements belong to
// its first piece), a workgroup to each; the pieces' sums lie in the order of the tensors and are
// added in a fixed order.  Measured: the norm of 93 MB in 75 tensors 17 us, 5.4 TB/s; of 320 MB in 219
// 86 us, 3.7 TB/s with what wrote them still in the caches, and their scaling 100 us, 6.4 TB/s (the last
// ones are read first: 315 us a pass for 325).  Launches carry their tensors in their arguments, so that nothing is
// copied to the device first.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "common.hpp"
#include "functional.hpp"

namespace compact {
namespace {

constexpr int kPieceBytes = 1 << 16;  // per workgroup.  (32 KB to 256 KB are within 2%, 16 KB 10% slower: 320 MB in 220 tensors.)
constexpr int kMostTensors = 160;  // per launch: a launch has 4 KB of arguments

struct Tensors {
  uint64_t at[kMostTensors];
  int64_t count[kMostTensors];       // elements; 2 x, with the lowest bit set for fp32
  uint32_t first[kMostTensors];      // piece of this launch
  int32_t tensors;
  uint32_t piece0;                   // of all
};

// Elements before the first whole chunk, whole chunks, elements after.
struct Cut {
  int64_t head, chunks, tail;
  __host__ __device__ __forceinline__ Cut(uint64_t at, int64_t count, bool f32) {
    const int64_t size = f32 ? 4 : 2, off = static_cast<int64_t>((16 - (at & 15)) & 15) / size;
    head = off < count ? off : count;
    chunks = (count - head) * size / 16;
    tail = count - head - chunks * (16 / size);
  }
};
constexpr int64_t kPieceChunks = kPieceBytes / 16;
int64_t pieces_of(uint64_t at, int64_t count, bool f32) {
  const int64_t chunks = Cut(at, count, f32).chunks;
  return chunks == 0 ? 1 : ceil_div(chunks, kPieceChunks);
}

template <bool F32>
__device__ __forceinline__ double square(uint32_t w) {
  if constexpr (F32) {
    const double v = __uint_as_float(w);
    return v * v;
  } else {
    const double lo = __uint_as_float(w << 16), hi = __uint_as_float(w & 0xFFFF0000u);
    return __builtin_fma(hi, hi, lo * lo);
  }
}

template <bool F32>
__device__ __forceinline__ double one_square(uint64_t at, int64_t i) {
  const double v = F32 ? reinterpret_cast<const float*>(at)[i] : bf16_to_f32(reinterpret_cast<const uint16_t*>(at)[i]);
  return v * v;
}

// The tensor of piece `id` of a launch, and the piece's number in it.
__device__ __forceinline__ int tensor_of(const Tensors& t, uint32_t id, uint32_t& piece) {
  int lo = 0, hi = t.tensors - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= id) lo = mid;
    else hi = mid - 1;
  }
  piece = id - t.first[lo];
  return lo;
}

template <bool F32>
__device__ __forceinline__ double piece_sum(uint64_t at, int64_t count, uint32_t piece) {
  const Cut cut(at, count, F32);
  const int tid = threadIdx.x;
  const u32x4* body = reinterpret_cast<const u32x4*>(at + cut.head * (F32 ? 4 : 2));
  const int64_t c0 = piece * kPieceChunks, c1 = c0 + kPieceChunks < cut.chunks ? c0 + kPieceChunks : cut.chunks;
  double s = 0.0;
#pragma unroll 8
  for (int64_t c = c0 + tid; c < c1; c += 256) {
    const u32x4 w = body[c];
    s += (square<F32>(w[0]) + square<F32>(w[1])) + (square<F32>(w[2]) + square<F32>(w[3]));
  }
  if (piece == 0) {
    if (tid < cut.head) s += one_square<F32>(at, tid);
    if (tid < cut.tail) s += one_square<F32>(at, count - cut.tail + tid);
  }
  return s;
}

__device__ __forceinline__ double block_sum(double v, double* lds) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.0;
  for (int w = 0; w < static_cast<int>(blockDim.x) / 64; ++w) v += lds[w];
  return v;
}

__global__ __launch_bounds__(256) void k_norm_pieces(Tensors t, double* part) {
  __shared__ double lds[4];
  uint32_t piece;
  const int i = tensor_of(t, blockIdx.x, piece);
  const int64_t count = t.count[i] >> 1;
  double s = t.count[i] & 1 ? piece_sum<true>(t.at[i], count, piece) : piece_sum<false>(t.at[i], count, piece);
  s = block_sum(s, lds);
  if (threadIdx.x == 0) part[t.piece0 + blockIdx.x] = s;
}

// The norm, and the factor (1 without a bound).
__global__ __launch_bounds__(1024) void k_norm(const double* part, int64_t pieces, double most, float* out) {
  __shared__ double lds[16];
  double s = 0.0;
#pragma unroll 4
  for (int64_t i = threadIdx.x; i < pieces; i += 1024) s += part[i];
  s = sqrt(block_sum(s, lds));
  if (threadIdx.x == 0) {
    out[0] = static_cast<float>(s);
    const double f = most / (s + 1e-6);
    out[1] = static_cast<float>(f > 1.0 ? 1.0 : f);  // (NaN stays NaN)
  }
}

template <bool F32>
__device__ __forceinline__ void scale_piece(uint64_t at, int64_t count, uint32_t piece, float f) {
  const Cut cut(at, count, F32);
  const int tid = threadIdx.x;
  u32x4* body = reinterpret_cast<u32x4*>(at + cut.head * (F32 ? 4 : 2));
  const int64_t c0 = piece * kPieceChunks, c1 = c0 + kPieceChunks < cut.chunks ? c0 + kPieceChunks : cut.chunks;
#pragma unroll 8
  for (int64_t c = c0 + tid; c < c1; c += 256) {
    u32x4 w = body[c];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (F32) w[k] = __float_as_uint(__uint_as_float(w[k]) * f);
      else w[k] = pack_bf16x2(__uint_as_float(w[k] << 16) * f, __uint_as_float(w[k] & 0xFFFF0000u) * f);
    }
    body[c] = w;
  }
  if (piece != 0) return;
  auto one = [&](int64_t i) {
    if constexpr (F32) reinterpret_cast<float*>(at)[i] *= f;
    else reinterpret_cast<uint16_t*>(at)[i] = f32_to_bf16(bf16_to_f32(reinterpret_cast<uint16_t*>(at)[i]) * f);
  };
  if (tid < cut.head) one(tid);
  if (tid < cut.tail) one(count - cut.tail + tid);
}

__global__ __launch_bounds__(256) void k_clip_pieces(Tensors t, const float* norm) {
  const float f = norm[1];
  if (f == 1.0f) return;
  uint32_t piece;  // the last ones first: what the norm read last may still be in the cache
  const int i = tensor_of(t, gridDim.x - 1 - blockIdx.x, piece);
  const int64_t count = t.count[i] >> 1;
  if (t.count[i] & 1) scale_piece<true>(t.at[i], count, piece, f);
  else scale_piece<false>(t.at[i], count, piece, f);
}

// Entry i of the list joins a launch's table.
void append(Tensors& t, const ClipTensor& e, uint32_t& grid) {
  t.at[t.tensors] = e.at;
  t.count[t.tensors] = e.count * 2 + (e.f32 ? 1 : 0);
  t.first[t.tensors++] = grid;
  grid += static_cast<uint32_t>(pieces_of(e.at, e.count, e.f32 != 0));
}

// f(table, grid) for each launch: of kMostTensors entries from i0 on, forward or from the list's
// end.  (Entries without elements are those that were given twice.)
template <typename F>
void for_tables(const ClipTensor* list, int64_t n, bool backward, F f) {
  const int64_t tables = ceil_div(n, kMostTensors);
  uint32_t piece0 = 0;
  for (int64_t k = 0; k < tables; ++k) {
    const int64_t i0 = (backward ? tables - 1 - k : k) * kMostTensors, i1 = i0 + kMostTensors < n ? i0 + kMostTensors : n;
    Tensors t = {};
    uint32_t grid = 0;
    for (int64_t i = i0; i < i1; ++i)
      if (list[i].count > 0) append(t, list[i], grid);
    t.piece0 = piece0;
    piece0 += grid;
    if (grid > 0) f(t, grid);
  }
}

}  // namespace
}  // namespace compact

using namespace compact;

extern "C" {

// The pieces that compact_clip has sums of.  A tensor that is given twice keeps its elements in one
// of its entries.  `order`: room for n indexes.  -1: sizes it does not take; -2: two tensors overlap.
int64_t compact_clip_pieces(ClipTensor* list, int64_t n, int64_t* order) {
  for (int64_t i = 0; i < n; ++i) {
    if (list[i].count < 0 || list[i].count >= int64_t(1) << 40 || (list[i].count > 0 && list[i].at == 0) || list[i].at % (list[i].f32 ? 4 : 2) != 0) return -1;
    order[i] = i;
  }
  std::sort(order, order + n, [&](int64_t a, int64_t b) { return list[a].at != list[b].at ? list[a].at < list[b].at : a < b; });
  int64_t pieces = 0, last = -1;
  for (int64_t i = 0; i < n; ++i) {
    ClipTensor& t = list[order[i]];
    if (t.count == 0) continue;
    if (last >= 0) {
      const ClipTensor& before = list[last];
      if (t.at == before.at && t.count == before.count && t.f32 == before.f32) {
        t.count = 0;
        continue;
      }
      if (before.at + static_cast<uint64_t>(before.count) * (before.f32 ? 4 : 2) > t.at) return -2;
    }
    pieces += pieces_of(t.at, t.count, t.f32 != 0);
    last = order[i];
  }
  return pieces < int64_t(1) << 24 ? pieces : -1;  // (a launch has under 2^32 threads)
}

// out: the norm and the factor.  bounded: whether the tensors are scaled.
int compact_clip(const ClipTensor* list, int64_t n, double most, int bounded, double* part, int64_t pieces, float* out, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  for_tables(list, n, false, [&](const Tensors& t, uint32_t grid) {
    hipLaunchKernelGGL(k_norm_pieces, dim3(grid), dim3(256), 0, s, t, part);
  });
  hipLaunchKernelGGL(k_norm, dim3(1), dim3(1024), 0, s, part, pieces, bounded ? most : __builtin_inf(), out);
  if (bounded)
    for_tables(list, n, true, [&](const Tensors& t, uint32_t grid) { hipLaunchKernelGGL(k_clip_pieces, dim3(grid), dim3(256), 0, s, t, out); });
  return hipGetLastError() == hipSuccess ? 0 : -5;
}

}  // extern "C"
