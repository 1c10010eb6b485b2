// Attention with a sliding window and sinks, bf16, grouped heads, any row strides:
//
//   row i of a sequence of L keys stands at position p = i + L - lq and sees key j when
//   0 <= j <= p and (p - j < window or j < sinks);
//   s = scale q.k,  P = softmax of s over the keys seen,  o = P v  (0 where none is seen);
//   D = sum(do o),  dS = P (do.v - D),  dq = scale dS k,  dk = scale dS^T q,  dv = P^T do.
//
// All products run as 32x32x16 bf16 MFMAs with fp32 sums; P and dS are rounded to bf16 as
// their operands, statistics, sums and accumulators are fp32.  P in one bf16 part leaves o and dv,
// rounded themselves, 1.2 to 1.42 times as far from the exact ones as their own rounding; a second
// part would cost a third product beside the forward's two.
//
// Kernel times below are medians of 100 passes in a row (the first dozen run 10 to 15% longer);
// comparisons of two forms were timed alone, one after the other.
//
// Every product is laid out so that what the softmax yields is the next product's operand
// as it stands: with keys as rows and queries as columns (S^T = K Q^T) a lane holds 16 of
// 32 keys of one query, its other half-wave the other 16; the row sums of the softmax are
// sums over a lane's registers and one exchange between the halves, and the packed values
// are the B operand of O^T = V^T P^T with the keys in the order
//   slot (half h, element e) of a 16-key step  =  key 4 h + e mod 4 + 8 (e / 4),
// in which the A operand V^T is read (transposing LDS reads).  The gradients of k and v
// have queries as rows and keys as columns, with dO^T and Q^T read that way.
#pragma once
#include <hip/hip_runtime.h>

#include "common.hpp"
#include "functional.hpp"

namespace compact {
namespace {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
typedef __attribute__((address_space(3))) void lds_void;

constexpr float kLog2e = 1.44269504088896340736f;
// Rows that see this many keys at most have dS in two bf16 parts in the gradients' products.
// dS rounded to bf16 alone leaves dq and dk, rounded themselves, 1.42 times as far from the
// exact gradients as their own rounding; with few keys to a row the error of o in D comes on
// top (1.49 at windows of 16 and 20).  In two parts: 1.02 to 1.08.  Two more products of nine:
// where windows are long 10% of the backward's time with heads of 64 (325 to 357 us at 4 x 4096
// rows, window 1024) and 19% with heads of 128 (1723 to 2048 us at 16384, window 4096).
constexpr int kFineKeys = 512;
constexpr int kBN = 64;  // keys (or queries) per staged tile

// A tile of rows of HD bf16 in LDS, 16-byte chunk c of row r at chunk c ^ swz(r): the 16
// lanes of a row read (one chunk of 16 consecutive rows) and the 32 lanes of a transposing
// read (64 bytes of 4 consecutive rows) then touch every bank once.
template <int HD>
struct Tile {
  static constexpr int kChunks = HD / 8;
  static constexpr int kBytes = kBN * HD * 2;
  static __device__ __forceinline__ int swz(int r) {
    if constexpr (HD == 128) return ((r & 3) << 2) | ((r >> 2) & 3);
    else if constexpr (HD == 64) return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
    else return (r >> 2) & 3;
  }
  static __device__ __forceinline__ int at(int r, int c) { return r * (HD * 2) + ((c ^ swz(r)) * 16); }
  // rows r0 + lane mod 32, the 8 columns 16 s + 8 (lane / 32).  (Here and below r0 is a multiple of 16,
  // which swz does not see: added behind it, it is a constant of the reading instruction and wants
  // no register.)
  static __device__ __forceinline__ u32x4 row_frag(const char* t, int r0, int s, int lane) {
    return *reinterpret_cast<const u32x4*>(t + at(lane & 31, 2 * s + (lane >> 5)) + r0 * (HD * 2));
  }
  // column 32 d + lane mod 32 of the rows r0 + 4 h + (0..3), r0 + 8 + 4 h + (0..3), h = lane / 32.
  // In a 16-lane group the transposing read hands output lane t, element j, the element
  // t mod 4 of source lane 4 j + t / 4.
  static __device__ __forceinline__ u32x4 col_frag(const char* t, int r0, int d, int lane) {
    const int g = lane >> 4, j = (lane >> 2) & 3, q = lane & 3;
    const int c = 4 * d + 2 * (g & 1) + (q >> 1);
    u32x4 out;
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      const int r = 4 * (g >> 1) + 8 * hh + j;
      const bf16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
          (lds_bf16x4*)(const_cast<char*>(t) + at(r, c) + 8 * (q & 1) + r0 * (HD * 2)));
      const u32x2 w = __builtin_bit_cast(u32x2, v);
      out[2 * hh] = w.x;
      out[2 * hh + 1] = w.y;
    }
    return out;
  }
};

// What a tile's values become on their way into LDS.  A value that is infinite or NaN meets
// factors of zero in the rows that do not see it, and 0 x inf must stay 0 there.  The kernels
// form their products plainly and look at their sums at the end, where such a NaN cannot
// hide; only then they do their work again:
//   kClean     such values as zeros
//   kPos, kNeg 1 where the value is +inf or NaN, -inf or NaN, else 0; with them the forward reads
//              keys of zeros, so that it counts those a row sees (a softmax's weights may
//              underflow, and would lose them)
enum Values { kPlain, kClean, kPos, kNeg };

__device__ __forceinline__ uint32_t value_pair(uint32_t w, int mode) {
  uint32_t out = 0;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t x = (w >> (16 * h)) & 0xFFFFu;
    const bool bad = (x & 0x7F80u) == 0x7F80u, nan = bad && (x & 0x7Fu) != 0;
    const bool one = nan || x == (mode == kPos ? 0x7F80u : 0xFF80u);
    out |= (mode == kClean ? (bad ? 0u : x) : one ? 0x3F80u : 0u) << (16 * h);
  }
  return out;
}

// A tile's way into LDS without registers: each wave copies kN blocks of 1 KB, lane after lane
// 16 bytes, fetching for each place of the tile the chunk that belongs there.  Rows at or past
// `rows` and columns at or past hd read as zeros (the buffer's range check).  A tile's bytes
// lie within 2^31 (row strides below kMaxStride), the tile's own start is a 64-bit address.
constexpr int64_t kMaxStride = (int64_t(1) << 24) - 512;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t tile_rows(const uint16_t* base, int64_t stride, int j0, int n, int hd) {
  const int bytes = n > 0 ? ((n - 1) * static_cast<int>(stride) + hd) * 2 : 0;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(base + j0 * stride), static_cast<short>(0), bytes, 0x00020000);
}

template <int HD, int ROWS = kBN, int WAVES = 4>
struct Copy {
  static constexpr int kN = ROWS * HD * 2 / 1024 / WAVES;
  int off[kN];
  __device__ __forceinline__ void init(int64_t stride, int hd, int tid) {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int idx = ((tid >> 6) * kN + i) * 64 + (tid & 63), r = idx / (HD / 8), c = (idx % (HD / 8)) ^ Tile<HD>::swz(r);
      off[i] = c * 8 < hd ? r * static_cast<int>(stride) * 2 + c * 16 : 0x7FFFFFF0;
    }
  }
  __device__ __forceinline__ void issue(const uint16_t* base, int64_t stride, int j0, int rows, int hd, char* t, int wave) const {
    const __amdgpu_buffer_rsrc_t rs = tile_rows(base, stride, j0, min(rows - j0, ROWS), hd);
#pragma unroll
    for (int i = 0; i < kN; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)(t + (wave * kN + i) * 1024), 16, off[i], 0, 0, 0);
  }
};

// kBN fp32 values v[r0 ..] of `rows`, by one wave.
__device__ __forceinline__ void copy_row_values(const float* v, int r0, int rows, char* t, int lane) {
  const int n = min(rows - r0, kBN);
  const __amdgpu_buffer_rsrc_t rs =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(v + r0), static_cast<short>(0), n > 0 ? n * 4 : 0, 0x00020000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)t, 4, lane * 4, 0, 0, 0);
}

// This wave's copies have arrived and its reads are done, and every wave's.
__device__ __forceinline__ void copies_done() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" : : : "memory"); }

// A tile's values converted where they are; bad[r] = 1 for a row r with an infinity or NaN.
template <int HD, int ROWS = kBN, int THREADS = 256>
__device__ __forceinline__ void convert_tile(char* t, int mode, int* bad, int tid) {
#pragma unroll 1
  for (int idx = tid; idx < ROWS * (HD / 8); idx += THREADS) {
    u32x4* at = reinterpret_cast<u32x4*>(t + Tile<HD>::at(idx / (HD / 8), idx % (HD / 8)));
    u32x4 w = *at;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t x = value_pair(w[e], mode);
      if (bad != nullptr && x != w[e]) bad[idx / (HD / 8)] = 1;
      w[e] = x;
    }
    *at = w;
  }
}

// B operand straight from memory: column (row of the matrix) `row`, 8 values 16 s + 8 (lane / 32).
template <int HD>
__device__ __forceinline__ void load_frags(u32x4 (&f)[HD / 16], const uint16_t* base, int64_t stride, int row, int rows,
                                           int hd, int lane) {
#pragma unroll
  for (int s = 0; s < HD / 16; ++s) {
    const int c = 16 * s + 8 * (lane >> 5);
    f[s] = u32x4{0u, 0u, 0u, 0u};
    if (row < rows && c < hd) f[s] = *reinterpret_cast<const u32x4*>(base + int64_t(row) * stride + c);
  }
}

// v of this lane and of the lane in the other half-wave: (lower half's, upper half's).
__device__ __forceinline__ void both_halves(float v, float& lo, float& hi) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  lo = __uint_as_float(r[0]);
  hi = __uint_as_float(r[1]);
}
// The maximum that keeps a NaN: one instruction for three values, where fmaxf has each quieted first.
__device__ __forceinline__ float max_of(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float halves_max(float v) {
  float lo, hi;
  both_halves(v, lo, hi);
  return max_of(lo, hi);
}
__device__ __forceinline__ float halves_sum(float v) {
  float lo, hi;
  both_halves(v, lo, hi);
  return lo + hi;
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int v = 0; v < 16; ++v) z[v] = 0.0f;
  return z;
}

// N products in order, use(i, factor), of factors that are read from LDS, AHEAD of them on their
// way.  (Left alone the compiler reads each factor right before its product, which then waits for
// LDS every time: 4 documents in 32768 rows, 16 heads on 4 of 128, window 4096, forward and backward
// 4229 us, so 3839.)  Only vector and scalar arithmetic may be moved across a product's place.
template <int N, int AHEAD, typename Read, typename Use>
__device__ __forceinline__ void products(Read read, Use use) {
  constexpr int kArithmetic = 0x2 | 0x4 | 0x400;
  decltype(read(0)) f[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) f[i] = read(i);
  __builtin_amdgcn_sched_barrier(kArithmetic);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    use(i, f[i % AHEAD]);
    if (i + AHEAD < N) f[i % AHEAD] = read(i + AHEAD);
    __builtin_amdgcn_sched_barrier(kArithmetic);
  }
}

// Row (of 32) of element v of a result: 8 (v / 4) + 4 (lane / 32) + v mod 4.
__device__ __forceinline__ int acc_row(int v, int lane) { return 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3); }

// Two 16-row steps of a 32x32 result as bf16 B operands.
__device__ __forceinline__ void pack_steps(const f32x16& p, u32x4 (&out)[2]) {
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int w = 0; w < 4; ++w) out[t][w] = pack_bf16x2(p[8 * t + 2 * w], p[8 * t + 2 * w + 1]);
}

// A sum that met an infinity or NaN.
template <int N>
__device__ __forceinline__ bool not_finite(const f32x16 (&acc)[N]) {
  float z = 0.0f;
#pragma unroll
  for (int d = 0; d < N; ++d)
#pragma unroll
    for (int v = 0; v < 16; ++v) z = __builtin_fmaf(acc[d][v], 0.0f, z);
  return !(z == 0.0f);
}

// What pack_steps' rounding took off, as operands of their own.
__device__ __forceinline__ void pack_rest(const f32x16& p, const u32x4 (&hi)[2], u32x4 (&out)[2]) {
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int w = 0; w < 4; ++w)
      out[t][w] = pack_bf16x2(p[8 * t + 2 * w] - __uint_as_float(hi[t][w] << 16),
                              p[8 * t + 2 * w + 1] - __uint_as_float(hi[t][w] & 0xFFFF0000u));
}

// The tiles of TN keys that rows at positions pmin .. pmax (of L keys) see: the sinks' tiles
// before the window's, then the window's.
template <int TN>
struct Walk {
  int sink_tiles, first, count;
  __device__ __forceinline__ Walk(int pmin, int pmax, int L, int window, int sinks) {
    if (pmax > L - 1) pmax = L - 1;
    int lo = pmin - window + 1;
    lo = lo < 0 ? 0 : lo;
    first = lo / TN;
    int st = (sinks + TN - 1) / TN;
    st = st < first ? st : first;
    sink_tiles = st;
    count = pmax < 0 ? 0 : st + (pmax / TN - first + 1);
    if (count < 0) count = 0;
  }
  __device__ __forceinline__ int key(int t) const { return (t < sink_tiles ? t : first + t - sink_tiles) * TN; }
};

__device__ __forceinline__ bool seen(int j, int p, int window, int sinks) {
  // (no short cuts: element by element they would become branches)
  return (j <= p) & ((p - j < window) | (j < sinks));
}

// Elements 32 kb + 8 (e / 4) + e mod 4 behind a lane's first: hidden where past(that number).  (Numbers
// that the compare holds as a constant: differences of them would each want a register, and the
// gradient of q at heads of 64 its third wave: 123 us, so 107, for 24 documents in 16384 rows.)
template <int NB, typename F>
__device__ __forceinline__ void hide(f32x16 (&s)[NB], float hidden, F past) {
#pragma unroll
  for (int kb = 0; kb < NB; ++kb)
#pragma unroll
    for (int e = 0; e < 16; ++e) s[kb][e] = past(32 * kb + 8 * (e >> 2) + (e & 3)) ? hidden : s[kb][e];
}

// What a lane's row p does not see of the 32 NB keys from j0 on.
template <int NB>
__device__ __forceinline__ void hide_unseen(f32x16 (&s)[NB], float hidden, int j0, int p, int window, int sinks, int lane) {
  const int first = j0 + 4 * (lane >> 5), last = p - first, before = last - window, behind = sinks - first;
  hide(s, hidden, [&](int k) { return (k > last) | ((k <= before) & (k >= behind)); });
}

// No key of j0 .. j0 + n - 1 is seen from a position in pmin .. pmax / all are from all of them.
__device__ __forceinline__ bool none_seen(int j0, int n, int pmin, int pmax, int window, int sinks) {
  return j0 > pmax || (pmin - (j0 + n - 1) >= window && j0 >= sinks);
}
__device__ __forceinline__ bool all_seen(int j0, int n, int pmin, int pmax, int window, int sinks) {
  return j0 + n - 1 <= pmin && (pmax - j0 < window || j0 + n - 1 < sinks);
}

__device__ __forceinline__ int length_of(const AttnArgs& a, int b) {
  if (a.lengths == nullptr) return a.lk;
  const int L = a.lengths[b];
  return L < 0 ? 0 : L > a.lk ? a.lk : L;
}

// The rows that a workgroup's tiles lie in: `rows` rows of which the sequence has its last, over L
// keys.  A padded batch (window_attention): those of batch entry b, at the strides of the batch.
// PACKED (packed_attention): the rows first .. first + rows - 1 of all of them, over as many keys,
// or over none (rows of no sequence: zeros).  Statistics lie by head, then by row.
template <bool PACKED>
struct Span {
  int b, rows, L;
  __device__ __forceinline__ Span(const AttnArgs& a, int b) : b(b), rows(a.lq), L(length_of(a, b)) {}
  __device__ __forceinline__ const uint16_t* at(const uint16_t* x, const int64_t (&s)[3], int h) const { return x + b * s[0] + h * s[1]; }
  __device__ __forceinline__ uint16_t* at(uint16_t* x, const int64_t (&s)[3], int h) const { return x + b * s[0] + h * s[1]; }
  __device__ __forceinline__ int64_t row_of(const AttnArgs& a, int h) const { return (int64_t(b) * a.heads + h) * a.lq; }
};
template <>
struct Span<true> {
  int b, rows, L, first, seq;  // seq: which sequence
  __device__ __forceinline__ Span(int first, int rows, int seq) : b(0), rows(rows), L(seq < 0 ? 0 : rows), first(first), seq(seq) {}
  __device__ __forceinline__ const uint16_t* at(const uint16_t* x, const int64_t (&s)[3], int h) const { return x + h * s[1] + first * s[2]; }
  __device__ __forceinline__ uint16_t* at(uint16_t* x, const int64_t (&s)[3], int h) const { return x + h * s[1] + first * s[2]; }
  __device__ __forceinline__ int64_t row_of(const AttnArgs& a, int h) const { return int64_t(h) * a.lq + first; }
};

// What rounding to bf16 took off a value, as a byte: in 127ths of half a unit in the last place
// of the rounded value (bits r; none for the smallest numbers, infinities and NaN).
__device__ __forceinline__ float half_place(uint32_t r, int sign) {
  const int e = static_cast<int>((r >> 7) & 0xFFu);
  return e > 16 && e < 255 ? __uint_as_float(static_cast<uint32_t>(127 + sign * (e - 127 - 8)) << 23) : 0.0f;
}
__device__ __forceinline__ uint32_t low_byte(float v, uint32_t r) {
  const float left = (v - __uint_as_float(r << 16)) * half_place(r, -1) * 127.0f;
  return static_cast<uint32_t>(static_cast<int>(rintf(half_place(r, -1) == 0.0f ? 0.0f : left))) & 0xFFu;
}
__device__ __forceinline__ float low_value(uint32_t byte, uint32_t r) {
  return static_cast<float>(static_cast<int8_t>(byte)) * half_place(r, 1) * (1.0f / 127.0f);
}
__device__ __forceinline__ uint32_t low_bytes(const float (&v)[4], const u32x2& w) {
  uint32_t out = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) out |= low_byte(v[e], (w[e / 2] >> (16 * (e & 1))) & 0xFFFFu) << (8 * e);
  return out;
}

// This wave's writes to LDS before its reads of them, and the other way round.  (LDS serves a wave in
// order; the compiler must not change it.)
__device__ __forceinline__ void in_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Columns of a transposed result (lane mod 32: the row of the output) as rows of bf16: those from
// `begin` up to `end` of 32.  A lane holds four values of its row here and there; they go through a
// wave's own 64 HD bytes of LDS (its rows as in a tile), so that neighbouring lanes store a row's
// neighbouring chunks.  (Stored as they stand, 8 bytes at a time to 32 rows, they are four times as
// many requests to L2: 24 documents in 16384 rows, 16 heads of 64, forward and backward 324 us, so 313.)
// low: also what the rounding took off, in rows of hd bytes that follow one another, by way of
// 32 HD bytes at t_low.
template <int HD>
__device__ __forceinline__ void store_rows(const f32x16 (&acc)[HD / 32], float f, uint16_t* rows, int64_t stride, int begin, int end,
                                           int hd, char* t, int lane, int8_t* low = nullptr, char* t_low = nullptr) {
  asm volatile("" : "+v"(lane));  // (places formed here: hoisted to the kernel's beginning, they spill)
  auto low_at = [](int r, int c) { return r * HD + ((c ^ (r & (HD == 96 ? 3 : HD / 8 - 1))) * 8); };  // chunk c of 8 bytes
  in_order();
#pragma unroll
  for (int d = 0; d < HD / 32; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const float v[4] = {acc[d][4 * g] * f, acc[d][4 * g + 1] * f, acc[d][4 * g + 2] * f, acc[d][4 * g + 3] * f};
      const u32x2 w = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
      *reinterpret_cast<u32x2*>(t + Tile<HD>::at(lane & 31, 4 * d + g) + 8 * (lane >> 5)) = w;
      if (low != nullptr) *reinterpret_cast<uint32_t*>(t_low + low_at(lane & 31, 4 * d + g) + 4 * (lane >> 5)) = low_bytes(v, w);
    }
  in_order();
#pragma unroll
  for (int i = 0; i < HD / 16; ++i) {
    const int idx = i * 64 + lane, r = idx / (HD / 8), c = idx % (HD / 8);
    if (r >= begin && r < end && c * 8 < hd) {
      *reinterpret_cast<u32x4*>(rows + r * stride + c * 8) = *reinterpret_cast<const u32x4*>(t + Tile<HD>::at(r, c));
      if (low != nullptr) *reinterpret_cast<u32x2*>(low + int64_t(r) * hd + c * 8) = *reinterpret_cast<const u32x2*>(t_low + low_at(r, c));
    }
  }
}

template <int HD>
__device__ __forceinline__ void store_row_values(const f32x16 (&acc)[HD / 32], float f, float* row, int hd, int lane) {
#pragma unroll
  for (int d = 0; d < HD / 32; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int c = 32 * d + 8 * g + 4 * (lane >> 5);
      if (c < hd) {
        const f32x4 w = {acc[d][4 * g] * f, acc[d][4 * g + 1] * f, acc[d][4 * g + 2] * f, acc[d][4 * g + 3] * f};
        *reinterpret_cast<f32x4*>(row + c) = w;
      }
    }
}

// Columns of a transposed sum of products with kPos or kNeg values: the rows' elements where it
// is not zero become what they are with an infinity (of that sign) or NaN in their sum.
template <int HD, typename T>
__device__ __forceinline__ void mark_rows(const f32x16 (&acc)[HD / 32], int mode, T* row, int hd, int lane) {
#pragma unroll
  for (int d = 0; d < HD / 32; ++d)
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int c = 32 * d + acc_row(v, lane);
      if (c >= hd || acc[d][v] == 0.0f) continue;
      const float inf = mode == kPos ? __builtin_inff() : -__builtin_inff();
      if constexpr (sizeof(T) == 2) row[c] = f32_to_bf16(bf16_to_f32(row[c]) + inf);
      else row[c] += inf;
    }
}

// Running maximum (in units of log2, scaled) and sum of one query column, with its rows of O^T.
template <int HD>
struct Softmax {
  f32x16 o[HD / 32];
  float m, l;
  __device__ __forceinline__ void init() {
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) o[d] = zero16();
    m = -__builtin_inff();
    l = 0.0f;
  }
  // A new maximum of scaled scores `top` (both halves' own): what was summed so far is scaled.
  // (A NaN moves nothing: its row is NaN whatever the reference.)
  // The reference of a row moves only when a score lies more than 2^8 above it: P <= 256 costs
  // no accuracy in fp32 sums and bf16 factors, and most tiles leave O alone.
  __device__ __forceinline__ void raise(float top) {
    top = halves_max(top);
    const bool up = top > m + 8.0f;
    if (__any(up)) {
      const float f = up ? exp2_fast(m - top) : 1.0f;
      m = up ? top : m;
      l *= f;
#pragma unroll
      for (int d = 0; d < HD / 32; ++d)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[d][v] *= f;
    }
  }
  __device__ __forceinline__ float shift() const { return m == -__builtin_inff() ? 0.0f : m; }
};

// ------------------------------- forward ------------------------------------
// A workgroup of four waves takes 128 queries of one head, 32 columns per wave, and walks the
// keys they see in tiles of 64, the next tile's copies in flight under the work on one.  (Each
// of the two buffers is a variable of its own: so the compiler knows which reads a copy in
// flight has nothing to do with.)  The work with V's values of `mode`; false: not finite, to be
// done by modes.
//
// Bound by a wave's own chain (scores, maximum, exponentials, P V) with two or three waves on a
// SIMD; LDS has no bank conflicts.  Tried and slower: the next tile's scores among this one's
// exponentials (heads of 64: 125-145 us for 105, alone, at 4 x 4096, 16 heads, window 1024; heads
// of 128: 3-7 % faster, but its two tiles of scores do not fit the registers), 64 columns per wave
// (no longer two workgroups per CU), tiles of 32 keys and a wave more on a SIMD (heads of 64: 382
// us for 358 at 12288 rows, all earlier keys; heads of 128 spill), a wave's priority raised for its
// products (no difference).
// Measured: there 115 us, 526 TFLOP/s over the pairs that are seen; 513 us, 940 TFLOP/s, at
// 16384 rows, 16 heads on 4 of 128, window 4096; 28 us at 3 x 1531 rows, 10 on 2 of 80, window
// 301; 19 us at 32 x 256 rows, 8 heads, window 128.  A large matrix product: 1223 TFLOP/s.
template <int HD>
struct TilePair {
  char k[Tile<HD>::kBytes], v[Tile<HD>::kBytes];
};

template <int HD, bool PACKED>
__device__ __forceinline__ bool attn_fwd(const AttnArgs& a, const Span<PACKED>& sp, TilePair<HD>& even, TilePair<HD>& odd, int h,
                                         int q0, int split, int mode) {
  constexpr int KS = HD / 16;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), w0 = q0 + wave * 32;
  const int hk = h / (a.heads / a.kv), lq = sp.rows, L = sp.L, off = L - lq;
  const uint16_t* q = sp.at(a.q, a.qs, h);
  const uint16_t* k = sp.at(a.k, a.ks, hk);
  const uint16_t* v = sp.at(a.v, a.vs, hk);
  const float c = a.scale * kLog2e;

  const int last = min(lq, q0 + 128) - 1;
  const Walk<kBN> walk(q0 + off, last + off, L, a.window, a.sinks);
  const int row = w0 + (lane & 31), p = row + off, pmin = w0 + off, pmax = min(w0 + 31, last) + off;
  Copy<HD> ck, cv;
  ck.init(a.ks[2], a.hd, tid);
  cv.init(a.vs[2], a.hd, tid);
  const int Lk = mode >= kPos ? 0 : L;
  auto fetch = [&](int t, TilePair<HD>& to) {
    ck.issue(k, a.ks[2], walk.key(t), Lk, a.hd, to.k, wave);
    cv.issue(v, a.vs[2], walk.key(t), L, a.hd, to.v, wave);
  };
  // the tiles of this split (all of them without splits)
  const int per = a.splits > 0 ? (walk.count + a.splits - 1) / a.splits : walk.count;
  const int t0 = split * per, t1 = min(walk.count, t0 + per);
  if (t0 < t1) fetch(t0, even);
  u32x4 qf[KS];
  Softmax<HD> sm;
  load_frags<HD>(qf, q, a.qs[2], row, lq, a.hd, lane);
  sm.init();

  auto step = [&](int t, TilePair<HD>& now, TilePair<HD>& next) {
    copies_done();
    if (t + 1 < t1) fetch(t + 1, next);
    if (mode != kPlain) {
      convert_tile<HD>(now.v, mode, nullptr, tid);
      __syncthreads();
    }
    const int j0 = walk.key(t);
    if (w0 > last || none_seen(j0, kBN, pmin, pmax, a.window, a.sinks)) return;
    f32x16 s[2];
    s[0] = s[1] = zero16();
    products<2 * KS, 4>([&](int i) { return Tile<HD>::row_frag(now.k, 32 * (i & 1), i >> 1, lane); },
                        [&](int i, const u32x4& f) { s[i & 1] = mfma32x32x16(f, qf[i >> 1], s[i & 1]); });
    if (!all_seen(j0, kBN, pmin, pmax, a.window, a.sinks)) hide_unseen(s, -__builtin_inff(), j0, p, a.window, a.sinks, lane);
    float top = max_of(s[0][0], s[1][0]);
#pragma unroll
    for (int e = 1; e < 16; ++e) top = max_of(max_of(top, s[0][e]), s[1][e]);
    sm.raise(top * c);
    const float sh = sm.shift();
    u32x4 pf[4];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[kb][e] = exp2_fast(__builtin_fmaf(s[kb][e], c, -sh));
        sm.l += s[kb][e];
      }
      u32x4 two[2];
      pack_steps(s[kb], two);
      pf[2 * kb] = two[0];
      pf[2 * kb + 1] = two[1];
    }
    constexpr int ND = HD / 32;
    products<4 * ND, 4>([&](int i) { return Tile<HD>::col_frag(now.v, 16 * (i / ND), i % ND, lane); },
                        [&](int i, const u32x4& f) { sm.o[i % ND] = mfma32x32x16(f, pf[i / ND], sm.o[i % ND]); });
  };
  for (int t = t0; t < t1; t += 2) {
    step(t, even, odd);
    if (t + 1 < t1) step(t + 1, odd, even);
  }
  if (mode == kPlain) {
    if (__syncthreads_or(not_finite(sm.o))) return false;
  } else {
    __syncthreads();
  }
  const float l = halves_sum(sm.l);
  const int64_t at_row = sp.row_of(a, h) + row;
  // no key in this split, which weighs nothing then; without splits: none for the row, which is
  // before its sequence (of scores that are all -inf the softmax is NaN)
  const bool empty = a.splits > 0 ? sm.m == -__builtin_inff() && l == 0.0f : p < 0;
  const float f = empty ? 0.0f : 1.0f / l;
  if (a.splits > 0) {
    if (row >= lq) return true;
    const int64_t rows = int64_t(a.b) * a.heads * a.lq, at = split * rows + at_row;
    if (mode >= kPos) {
      mark_rows<HD>(sm.o, mode, a.part_o + at * a.hd, a.hd, lane);
      return true;
    }
    store_row_values<HD>(sm.o, f, a.part_o + at * a.hd, a.hd, lane);
    if (lane < 32) a.part_lse[at] = empty ? -__builtin_inff() : sm.m + log2f(l);
    return true;
  }
  uint16_t* out = sp.at(a.o, a.os, h) + w0 * a.os[2];
  if (mode >= kPos) {
    if (row < lq) mark_rows<HD>(sm.o, mode, out + (lane & 31) * a.os[2], a.hd, lane);
    return true;
  }
  store_rows<HD>(sm.o, f, out, a.os[2], 0, lq - w0, a.hd, reinterpret_cast<char*>(&even) + wave * 64 * HD, lane,
                 a.o_low == nullptr ? nullptr : a.o_low + (sp.row_of(a, h) + w0) * a.hd, reinterpret_cast<char*>(&odd) + wave * 32 * HD);
  if (row < lq && lane < 32) a.lse[at_row] = empty ? __builtin_inff() : sm.m + log2f(l);
  return true;
}

// ------------------------------ gradient of q --------------------------------
// As the forward, with S^T and dP^T = V dO^T; D = sum(dO o) on the way, for the other kernel
// too.  Where the sums are not finite the work is done again with clean values, and NaN in the
// rows that see a key that had others.
//
// Bound as the forward, with three waves to a SIMD at heads of 64.  Measured: 133 us at 4 x 4096
// rows, 16 heads of 64, window 1024; 691 us, 1044 TFLOP/s of its three products, at 16384 rows, 16
// heads on 4 of 128, window 4096; 23 us at 32 x 256 rows, 8 heads of 64, window 128.
constexpr int kDqAhead = 4, kDkvAhead = 2;

template <int HD, bool FINE, bool PACKED>
__device__ __forceinline__ bool attn_dq(const AttnGradArgs& ga, const Span<PACKED>& sp, TilePair<HD>& even, TilePair<HD>& odd,
                                        int* bad_key, int h, int q0, int mode) {
  constexpr int KS = HD / 16;
  const AttnArgs& a = ga.f;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), w0 = q0 + wave * 32;
  const int hk = h / (a.heads / a.kv), lq = sp.rows, L = sp.L, off = L - lq;
  const uint16_t* k = sp.at(a.k, a.ks, hk);
  const uint16_t* v = sp.at(a.v, a.vs, hk);
  const int64_t stat = sp.row_of(a, h);
  const float c = a.scale * kLog2e;

  const int last = min(lq, q0 + 128) - 1;
  const Walk<kBN> walk(q0 + off, last + off, L, a.window, a.sinks);
  const int row = w0 + (lane & 31), p = row + off, pmin = w0 + off, pmax = min(w0 + 31, last) + off;
  Copy<HD> ck, cv;
  ck.init(a.ks[2], a.hd, tid);
  cv.init(a.vs[2], a.hd, tid);
  auto fetch = [&](int t, TilePair<HD>& to) {
    ck.issue(k, a.ks[2], walk.key(t), L, a.hd, to.k, wave);
    cv.issue(v, a.vs[2], walk.key(t), L, a.hd, to.v, wave);
  };
  if (walk.count > 0) fetch(0, even);
  u32x4 qf[KS], gf[KS];
  load_frags<HD>(qf, sp.at(a.o, a.os, h), a.os[2], row, lq, a.hd, lane);
  load_frags<HD>(gf, sp.at(ga.go, ga.gs, h), ga.gs[2], row, lq, a.hd, lane);
  // sum(do o), o with what its rounding took off: where a row sees few keys dS is a difference
  // of near numbers, and a rounded o would cost it digits
  float sum = 0.0f;
#pragma unroll
  for (int st = 0; st < KS; ++st) {
    u32x2 low = {0u, 0u};
    if (row < lq && 16 * st + 8 * (lane >> 5) < a.hd)
      low = *reinterpret_cast<const u32x2*>(a.o_low + (stat + row) * a.hd + 16 * st + 8 * (lane >> 5));
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t r = (qf[st][e / 2] >> (16 * (e & 1))) & 0xFFFFu, g = (gf[st][e / 2] >> (16 * (e & 1))) & 0xFFFFu;
      const float o = __uint_as_float(r << 16) + low_value((low[e / 4] >> (8 * (e & 3))) & 0xFFu, r);
      sum = __builtin_fmaf(o, __uint_as_float(g << 16), sum);
    }
  }
  const float delta = halves_sum(sum);
  const float lse = row < lq ? a.lse[stat + row] : __builtin_inff();
  if (row < lq && lane < 32) ga.delta[stat + row] = delta;
  load_frags<HD>(qf, sp.at(a.q, a.qs, h), a.qs[2], row, lq, a.hd, lane);
  f32x16 dq[HD / 32];
#pragma unroll
  for (int d = 0; d < HD / 32; ++d) dq[d] = zero16();

  auto step = [&](int t, TilePair<HD>& now, TilePair<HD>& next) {
    copies_done();
    if (t + 1 < walk.count) fetch(t + 1, next);
    if (mode != kPlain) {
      if (tid < kBN) bad_key[tid] = 0;
      __syncthreads();
      convert_tile<HD>(now.k, mode, bad_key, tid);
      convert_tile<HD>(now.v, mode, bad_key, tid);
      __syncthreads();
    }
    const int j0 = walk.key(t);
    if (w0 > last || none_seen(j0, kBN, pmin, pmax, a.window, a.sinks)) return;
    const bool edge = mode != kPlain || !all_seen(j0, kBN, pmin, pmax, a.window, a.sinks);
    constexpr int kUnroll = HD == 64 ? 2 : 1;
#pragma unroll kUnroll
    for (int kb = 0; kb < 2; ++kb) {
      f32x16 one[1] = {zero16()}, &s = one[0], dp = zero16();
      products<2 * KS, kDqAhead>([&](int i) { return Tile<HD>::row_frag(i & 1 ? now.v : now.k, 32 * kb, i >> 1, lane); },
                                 [&](int i, const u32x4& f) {
                                   if (i & 1) dp = mfma32x32x16(f, gf[i >> 1], dp);
                                   else s = mfma32x32x16(f, qf[i >> 1], s);
                                 });
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = exp2_fast(__builtin_fmaf(s[e], c, -lse)) * (dp[e] - delta);
      if (edge) {
        if (mode != kPlain) {
#pragma unroll
          for (int e = 0; e < 16; ++e) s[e] = bad_key[32 * kb + acc_row(e, lane)] ? __builtin_nanf("") : s[e];
        }
        hide_unseen(one, 0.0f, j0 + 32 * kb, p, a.window, a.sinks, lane);
      }
      u32x4 ds[2], dr[2];
      pack_steps(s, ds);
      if constexpr (FINE) pack_rest(s, ds, dr);
      constexpr int ND = HD / 32;
      products<2 * ND, kDqAhead>([&](int i) { return Tile<HD>::col_frag(now.k, 32 * kb + 16 * (i / ND), i % ND, lane); },
                                 [&](int i, const u32x4& f) {
                                   dq[i % ND] = mfma32x32x16(f, ds[i / ND], dq[i % ND]);
                                   if constexpr (FINE) dq[i % ND] = mfma32x32x16(f, dr[i / ND], dq[i % ND]);
                                 });
    }
  };
  for (int t = 0; t < walk.count; t += 2) {
    step(t, even, odd);
    if (t + 1 < walk.count) step(t + 1, odd, even);
  }
  if (mode == kPlain) {
    if (__syncthreads_or(not_finite(dq))) return false;
  } else {
    __syncthreads();
  }
  store_rows<HD>(dq, a.scale, sp.at(ga.dq, ga.dqs, h) + w0 * ga.dqs[2], ga.dqs[2], 0, lq - w0, a.hd,
                 reinterpret_cast<char*>(&even) + wave * 64 * HD, lane);
  return true;
}

// --------------------------- gradients of k and v ----------------------------
// A workgroup takes 128 keys and walks the query tiles of the heads that share them in order: no
// atomics, the same sums every time.  Two things would leave the card to a few long workgroups:
// few keys and heads (then `parts` workgroups share a block's tiles), and the sinks, which every
// row sees.  Pairs beyond the window ("far") are a work of their own: 64 (128) of the sinks, 32
// to a pair of waves that share a tile's rows, in `chunks` of the tiles.  What several workgroups
// form lies in fp32 in slots of `part`, and k_attn_dkv_sum adds the slots in order:
//   near [parts][b kv][near_keys][2][hd], then far [chunks, each far_slots times][b kv][far_keys][2][hd].
//
// Bound by the chain of one wave (products, exponentials, products) with two to a SIMD, and with
// 128 columns by LDS too: a step's fragments take 1.5 times as long to read as its products.
// Measured: 180 us at 4 x 4096 rows, 16 heads of 64, window 1024; 1078 us, 892 TFLOP/s of its four
// products, at 16384 rows, 16 heads on 4 of 128, window 4096; 25 us at 32 x 256 rows, 8 heads of
// 64, window 128.  Both halves of a tile in one stretch of code spill, or leave one wave to a SIMD.
template <int HD>
struct RowPair {
  char q[Tile<HD>::kBytes], g[Tile<HD>::kBytes];
  float lse[kBN], delta[kBN];
};

struct DkvJob {
  int bk, k0, slot, far;  // bk: of the batch's heads of k; PACKED: the head of k
};

// Heads over 96: eight waves, of which two share 32 keys, each with half of a tile's rows; the
// block's k and v lie in LDS, and at the end the one half's sums are added to the other's.
// Else four waves with both halves, k and v in registers.  With 128 columns of dk and dv the
// latter is one wave to a SIMD, with nothing to run while it waits; 64 columns leave room for
// two anyway, and the reads of k and v cost them more.  The whole backward, us, with eight / four
// waves: 16384 rows, 16 heads on 4 of 128, window 4096: 1723 / 2346; 2 x 4096, 16 of 128, all
// keys: 530 / 663; 4 x 4096, 16 of 64, window 1024: 382 / 325; 1000, 16 on 2 of 96: 60 / 61.
__host__ __device__ constexpr bool shared_keys(int hd) { return hd > 96; }
__host__ __device__ constexpr int far_block(int hd) { return shared_keys(hd) ? 128 : 64; }
__host__ __device__ constexpr int far_slots(int hd) { return shared_keys(hd) ? 1 : 2; }

template <int HD, bool SHARED>
struct KeyBlock {
  char k[2][Tile<HD>::kBytes], v[2][Tile<HD>::kBytes];
};
template <int HD>
struct KeyBlock<HD, false> {};

// Packed: what several workgroups form, or far work adds to, in fp32 rows of 2 hd values in `part`:
// near [parts][kv][T], or without parts [kv][packed_far_rows], then far [chunks, each far_slots
// times][kv][packed_far_rows], where row x of a head is key j of sequence x / far_keys, or, where
// those would be more than the rows, row x of all.
__host__ __device__ __forceinline__ bool packed_by_row(const AttnGradArgs& ga) { return int64_t(ga.sequences) * ga.far_keys >= ga.f.lk; }
__host__ __device__ __forceinline__ int64_t packed_far_rows(const AttnGradArgs& ga) {
  return packed_by_row(ga) ? ga.f.lk : int64_t(ga.sequences) * ga.far_keys;
}
__host__ __device__ __forceinline__ int64_t packed_near_rows(const AttnGradArgs& ga) {
  return ga.f.kv * (ga.parts > 1 ? ga.parts * int64_t(ga.f.lk) : packed_far_rows(ga));
}

template <int HD, bool FINE, bool PACKED>
__device__ __forceinline__ bool attn_dkv(const AttnGradArgs& ga, const Span<PACKED>& sp, KeyBlock<HD, shared_keys(HD)>& keys,
                                         RowPair<HD>& even, RowPair<HD>& odd, int* bad_row, const DkvJob& job, int mode) {
  constexpr int KS = HD / 16;
  constexpr bool SHARED = shared_keys(HD);
  const AttnArgs& a = ga.f;
  int tid = threadIdx.x;  // (places formed anew for each walk: kept for the second, which hardly ever comes, they spill)
  asm volatile("" : "+v"(tid));
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), G = a.heads / a.kv;
  const int hk = job.bk % a.kv, lq = sp.rows, L = sp.L, off = L - lq;
  const bool far = job.far != 0, halves = SHARED || far;  // a wave has one half of each tile's rows
  const int kw = halves ? wave >> 1 : wave, w0 = job.k0 + 32 * kw, j = w0 + (lane & 31);
  const float c = a.scale * kLog2e;

  // the rows that see some key of the block
  const int kl = min(job.k0 + (far ? far_block(HD) : 128), far ? min(L, a.sinks) : L) - 1;
  int i0 = max(0, job.k0 + (far ? a.window : 0) - off), i1 = lq;
  if (!far && int64_t(kl) + a.window - off < i1) i1 = kl + a.window - off;
  i0 = i0 / kBN;
  // a pair is this work's when apart <= p - j < apart + span; a key that is not, far ahead
  const int apart = far ? a.window : 0, jj = j <= kl ? j : 1 << 30;
  const uint32_t span = far ? 1u << 30 : static_cast<uint32_t>(a.window);
  const int tiles = kl < job.k0 || i1 <= i0 * kBN ? 0 : (i1 + kBN - 1) / kBN - i0;
  const int per = (tiles * G + (far ? ga.chunks : ga.parts) - 1) / (far ? ga.chunks : ga.parts);
  const int first = job.slot * per, steps = max(0, min(tiles * G, first + per) - first);

  const uint16_t* k = sp.at(a.k, a.ks, hk);
  const uint16_t* v = sp.at(a.v, a.vs, hk);
  Copy<HD> cq, cg;  // SHARED: the first four waves copy q and k, the others do and v, all with cq
  const bool of_g = SHARED && wave >= 4;
  u32x4 kf[KS], vf[KS];
  if constexpr (SHARED) {
    if (steps > 0) {
      const int64_t stride = of_g ? a.vs[2] : a.ks[2];
      cq.init(stride, a.hd, tid & 255);
#pragma unroll
      for (int i = 0; i < 2; ++i)
        cq.issue(of_g ? v : k, stride, job.k0 + i * kBN, L, a.hd, of_g ? keys.v[i] : keys.k[i], wave & 3);
    }
    cq.init(of_g ? ga.gs[2] : a.qs[2], a.hd, tid & 255);
  } else {
    cq.init(a.qs[2], a.hd, tid);
    cg.init(ga.gs[2], a.hd, tid);
  }
  auto fetch = [&](int t, RowPair<HD>& to) {
    const int h = hk * G + (first + t) / tiles, r0 = (i0 + (first + t) % tiles) * kBN;
    const uint16_t* q = sp.at(a.q, a.qs, h);
    const uint16_t* g = sp.at(ga.go, ga.gs, h);
    if constexpr (SHARED) {
      cq.issue(of_g ? g : q, of_g ? ga.gs[2] : a.qs[2], r0, lq, a.hd, of_g ? to.g : to.q, wave & 3);
    } else {
      cq.issue(q, a.qs[2], r0, lq, a.hd, to.q, wave);
      cg.issue(g, ga.gs[2], r0, lq, a.hd, to.g, wave);
    }
    const int64_t row = sp.row_of(a, h);
    if (wave == 0) copy_row_values(a.lse + row, r0, lq, reinterpret_cast<char*>(to.lse), lane);
    if (wave == 1) copy_row_values(ga.delta + row, r0, lq, reinterpret_cast<char*>(to.delta), lane);
  };
  if (steps > 0) fetch(0, even);
  if constexpr (!SHARED) {
    load_frags<HD>(kf, k, a.ks[2], j, L, a.hd, lane);
    load_frags<HD>(vf, v, a.vs[2], j, L, a.hd, lane);
  }
  f32x16 dk[HD / 32], dv[HD / 32];
#pragma unroll
  for (int d = 0; d < HD / 32; ++d) dk[d] = dv[d] = zero16();

  auto step = [&](int t, RowPair<HD>& now, RowPair<HD>& next) {
    copies_done();
    if (t + 1 < steps) fetch(t + 1, next);
    if (mode != kPlain) {
      if (tid < kBN) bad_row[tid] = 0;
      __syncthreads();
      convert_tile<HD, kBN, SHARED ? 512 : 256>(now.q, mode, bad_row, tid);
      convert_tile<HD, kBN, SHARED ? 512 : 256>(now.g, mode, bad_row, tid);
      __syncthreads();
    }
    const int r0 = (i0 + (first + t) % tiles) * kBN;
    // (Where registers are short most places in LDS are formed anew for each tile: kept, they spill.)
    int ln = lane;
    if constexpr (SHARED) asm volatile("" : "+v"(ln));
    constexpr int kUnroll = HD == 64 ? 2 : 1;
#pragma unroll kUnroll
    for (int n = 0; n < (SHARED ? 1 : 2); ++n) {
      const int qb = SHARED ? wave & 1 : n, i1st = r0 + 32 * qb, pmin = i1st + off, pmax = pmin + 31;
      if (w0 > kl || i1st >= lq) continue;
      if (far ? (wave & 1) != qb || pmax - w0 < a.window : w0 > pmax || pmin - (w0 + 31) >= a.window) continue;
      const bool all = far ? w0 + 31 < a.sinks && pmin - (w0 + 31) >= a.window : w0 + 31 <= pmin && pmax - w0 < a.window;
      const bool edge = mode != kPlain || i1st + 31 >= lq || w0 + 31 > kl || !all;
      f32x16 s = zero16(), dp = zero16();
      if constexpr (SHARED) {
        struct Pair {
          u32x4 row, key;
        };
        products<2 * KS, kDkvAhead>(
            [&](int i) {
              return Pair{Tile<HD>::row_frag(i & 1 ? now.g : now.q, 32 * qb, i >> 1, ln),
                          Tile<HD>::row_frag(i & 1 ? keys.v[kw >> 1] : keys.k[kw >> 1], 32 * (kw & 1), i >> 1, lane)};
            },
            [&](int i, const Pair& f) {
              if (i & 1) dp = mfma32x32x16(f.row, f.key, dp);
              else s = mfma32x32x16(f.row, f.key, s);
            });
      } else {
        products<2 * KS, 2 * kDkvAhead>([&](int i) { return Tile<HD>::row_frag(i & 1 ? now.g : now.q, 32 * qb, i >> 1, ln); },
                                        [&](int i, const u32x4& f) {
                                          if (i & 1) dp = mfma32x32x16(f, vf[i >> 1], dp);
                                          else s = mfma32x32x16(f, kf[i >> 1], s);
                                        });
      }
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 l4 = *reinterpret_cast<const f32x4*>(now.lse + 32 * qb + 8 * g + 4 * (ln >> 5));
        const f32x4 d4 = *reinterpret_cast<const f32x4*>(now.delta + 32 * qb + 8 * g + 4 * (ln >> 5));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float pr = exp2_fast(__builtin_fmaf(s[4 * g + e], c, -l4[e]));
          dp[4 * g + e] = pr * (dp[4 * g + e] - d4[e]);
          s[4 * g + e] = pr;
        }
      }
      if (edge) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int r = 32 * qb + acc_row(e, ln), p = r0 + r + off;
          const bool in = (static_cast<uint32_t>(p - jj - apart) < span) & (p < L), nan = mode != kPlain && bad_row[r];
          s[e] = in ? (nan ? __builtin_nanf("") : s[e]) : 0.0f;
          dp[e] = in ? (nan ? __builtin_nanf("") : dp[e]) : 0.0f;
        }
      }
      u32x4 pf[2], df[2];
      pack_steps(s, pf);
      pack_steps(dp, df);
      u32x4 dr[2];
      if constexpr (FINE) pack_rest(dp, df, dr);
      constexpr int ND = HD / 32;
      products<4 * ND, 2 * kDkvAhead>(
          [&](int i) { return Tile<HD>::col_frag(i & 1 ? now.q : now.g, 32 * qb + 16 * (i / (2 * ND)), i / 2 % ND, ln); },
          [&](int i, const u32x4& f) {
            const int st = i / (2 * ND), d = i / 2 % ND;
            if (!(i & 1)) {
              dv[d] = mfma32x32x16(f, pf[st], dv[d]);
            } else {
              dk[d] = mfma32x32x16(f, df[st], dk[d]);
              if constexpr (FINE) dk[d] = mfma32x32x16(f, dr[st], dk[d]);
            }
          });
    }
  };
  for (int t = 0; t < steps; t += 2) {
    step(t, even, odd);
    if (t + 1 < steps) step(t + 1, odd, even);
  }
  if (mode == kPlain) {
    if (__syncthreads_or(not_finite(dk) || not_finite(dv))) return false;
  } else {
    __syncthreads();
  }
  if constexpr (SHARED) {
    // (128 columns of four waves: in fp32 as much as the block's k and v in bf16)
    f32x4* at = reinterpret_cast<f32x4*>(&keys) + kw * (HD / 8) * 64 + lane;
    auto join = [&](f32x16 (&x)[HD / 32]) {
      if (wave & 1) {
#pragma unroll
        for (int i = 0; i < HD / 8; ++i) {
          const f32x16& y = x[i / 4];
          at[i * 64] = f32x4{y[4 * (i % 4)], y[4 * (i % 4) + 1], y[4 * (i % 4) + 2], y[4 * (i % 4) + 3]};
        }
      }
      __syncthreads();
      if (!(wave & 1)) {
#pragma unroll
        for (int i = 0; i < HD / 8; ++i) {
          const f32x4 y = at[i * 64];
#pragma unroll
          for (int e = 0; e < 4; ++e) x[i / 4][4 * (i % 4) + e] += y[e];
        }
      }
      __syncthreads();
    };
    join(dk);
    join(dv);
    if (wave & 1) return true;
  }
  // keys below `slots` go to slots of `part`, the others to their places
  const int keys_here = PACKED ? lq : a.lk, slots = far ? keys_here : PACKED ? (L == 0 ? 0 : ga.parts > 1 ? L : ga.far_keys) : ga.near_keys;
  if (!far && w0 < keys_here && w0 + 32 > slots) {
    store_rows<HD>(dk, a.scale, sp.at(ga.dk, ga.dks, hk) + w0 * ga.dks[2], ga.dks[2], slots - w0, keys_here - w0, a.hd,
                   reinterpret_cast<char*>(&even) + kw * 64 * HD, lane);
    store_rows<HD>(dv, 1.0f, sp.at(ga.dv, ga.dvs, hk) + w0 * ga.dvs[2], ga.dvs[2], slots - w0, keys_here - w0, a.hd,
                   reinterpret_cast<char*>(&odd) + kw * 64 * HD, lane);
  }
  if (far || j < slots) {
    const int slot = far ? far_slots(HD) * job.slot + (SHARED ? 0 : wave & 1) : job.slot;
    int64_t at;
    if constexpr (PACKED) {
      if (j >= (far ? min(ga.far_keys, L) : L)) return true;
      const int64_t row = packed_by_row(ga) ? sp.first : int64_t(sp.seq) * ga.far_keys;
      int64_t base;
      if (far) base = packed_near_rows(ga) + (slot * int64_t(a.kv) + hk) * packed_far_rows(ga) + row;
      else base = ga.parts > 1 ? (slot * int64_t(a.kv) + hk) * a.lk + sp.first : hk * packed_far_rows(ga) + row;
      at = base + j;
    } else {
      const int64_t bk_all = int64_t(a.b) * a.kv;
      if (j >= (far ? ga.far_keys : ga.near_keys)) return true;
      if (far) at = ga.parts * bk_all * ga.near_keys + (slot * bk_all + job.bk) * ga.far_keys + j;
      else at = (slot * bk_all + job.bk) * ga.near_keys + j;
    }
    float* out = ga.part + at * 2 * a.hd;
    store_row_values<HD>(dk, a.scale, out, a.hd, lane);
    store_row_values<HD>(dv, 1.0f, out + a.hd, a.hd, lane);
  }
  return true;
}

// Far workgroups are 1024 at most, or one to a block of sinks: a chunk costs a slot in fp32 for each
// sink.  us (MB of scratch beside the gradients) without a limit / 2048 / 1024 / 512: 4 x 16384 rows, 16
// heads of 64, window 1024, 4 sinks 1294 (6) / 1295 (6) / 1287 (2) / 1290; 1024 sinks 2862 (2046) /
// 2243 (167) / 2236 (100) / 2242; 16384 rows, window 128, 4096 sinks 1858 (2183) / 1076 (168) / 1114
// (101) / 1109; 16 heads on 4 of 128, window 4096, 4096 sinks 2920 (220) / 2925 / 2872 (153) / 2944.
constexpr int64_t kFarWork = 1024;

constexpr int64_t kSumGrid = int64_t(1) << 20;  // workgroups that add slots

inline bool args_ok(const AttnArgs& a) {
  constexpr int64_t most = int64_t(1) << 30;
  if (a.b < 1 || a.heads < 1 || a.kv < 1 || a.heads % a.kv != 0 || a.lq < 1 || a.lk < 1 || a.hd < 8 || a.hd % 8 != 0 ||
      a.hd > 128 || a.window < 1 || a.sinks < 0 || a.lq > most || a.lk > most || a.window > most || a.sinks > most ||
      !(a.scale > 0.0f))
    return false;
  for (const int64_t* s : {a.qs, a.ks, a.vs, a.os})
    if (s[0] < 0 || s[1] < 0 || s[2] < 0 || s[2] > kMaxStride) return false;
  if ((a.lq > 1 && a.qs[2] < a.hd) || (a.lk > 1 && (a.ks[2] < a.hd || a.vs[2] < a.hd))) return false;
  return int64_t(a.b) * a.heads * ceil_div(a.lq, 32) < (int64_t(1) << 24) &&
         int64_t(a.b) * a.kv * ceil_div(a.lk, 32) < (int64_t(1) << 24);
}

inline int status() { return hipGetLastError() == hipSuccess ? 0 : -5; }

}  // namespace
}  // namespace compact
