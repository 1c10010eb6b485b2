// Attention with a sliding window and sinks, bf16, grouped heads, any row strides:
//
//   row i of a sequence of L keys stands at position p = i + L - lq and sees key j when
//   0 <= j <= p and (p - j < window or j < sinks);
//   s = scale q.k,  P = softmax of s over the keys seen,  o = P v  (0 where none is seen);
//   D = sum(do o),  dS = P (do.v - D),  dq = scale dS k,  dk = scale dS^T q,  dv = P^T do.
//
// All products run as 32x32x16 bf16 MFMAs with fp32 sums; P and dS are rounded to bf16 as
// their operands, statistics, sums and accumulators are fp32.
//
// Every product is laid out so that what the softmax yields is the next product's operand
// as it stands: with keys as rows and queries as columns (S^T = K Q^T) a lane holds 16 of
// 32 keys of one query, its other half-wave the other 16; the row sums of the softmax are
// sums over a lane's registers and one exchange between the halves, and the packed values
// are the B operand of O^T = V^T P^T with the keys in the order
//   slot (half h, element e) of a 16-key step  =  key 4 h + e mod 4 + 8 (e / 4),
// in which the A operand V^T is read (transposing LDS reads).  The gradients of k and v
// have queries as rows and keys as columns, with dO^T and Q^T read that way.
#include <hip/hip_runtime.h>

#include "common.hpp"
#include "functional.hpp"

namespace compact {
namespace {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;

constexpr float kLog2e = 1.44269504088896340736f;
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
  // rows r0 + lane mod 32, the 8 columns 16 s + 8 (lane / 32)
  static __device__ __forceinline__ u32x4 row_frag(const char* t, int r0, int s, int lane) {
    return *reinterpret_cast<const u32x4*>(t + at(r0 + (lane & 31), 2 * s + (lane >> 5)));
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
      const int r = r0 + 4 * (g >> 1) + 8 * hh + j;
      const bf16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
          (lds_bf16x4*)(const_cast<char*>(t) + at(r, c) + 8 * (q & 1)));
      const u32x2 w = __builtin_bit_cast(u32x2, v);
      out[2 * hh] = w.x;
      out[2 * hh + 1] = w.y;
    }
    return out;
  }
};

// This thread's chunks of a tile on their way from memory to LDS: rows j0 .. j0 + ROWS - 1 of
// a matrix, rows at or past `rows` and columns at or past hd as zeros.
template <int HD, int ROWS, int THREADS>
struct Stage {
  static constexpr int kN = ROWS * (HD / 8) / THREADS;
  u32x4 w[kN];
  __device__ __forceinline__ void load(const uint16_t* base, int64_t stride, int j0, int rows, int hd, int tid) {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int idx = tid + THREADS * i, r = idx / (HD / 8), c = idx % (HD / 8);
      w[i] = u32x4{0u, 0u, 0u, 0u};
      if (j0 + r < rows && c * 8 < hd) w[i] = *reinterpret_cast<const u32x4*>(base + (int64_t(j0) + r) * stride + c * 8);
    }
  }
  __device__ __forceinline__ void store(char* t, int tid) const {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int idx = tid + THREADS * i;
      *reinterpret_cast<u32x4*>(t + Tile<HD>::at(idx / (HD / 8), idx % (HD / 8))) = w[i];
    }
  }
};

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

__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32, 64); }

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int v = 0; v < 16; ++v) z[v] = 0.0f;
  return z;
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

__device__ __forceinline__ bool not_finite(const u32x4& a) {
  bool bad = false;
#pragma unroll
  for (int w = 0; w < 4; ++w) bad |= (a[w] & 0x7F80u) == 0x7F80u || (a[w] & 0x7F800000u) == 0x7F800000u;
  return bad;
}

// acc + A B where a value of A may be infinite or NaN beside rows whose factor in B is zero
// because they do not see it: 0 x inf must stay 0 there.  Such values enter as 1 in products
// of their own, and wherever those are not zero the result is what the sum would be (`grad`:
// NaN, as B's sign is not looked at; else the infinity or NaN).
template <bool GRAD>
__device__ __forceinline__ f32x16 mfma_seen(const u32x4& a, const u32x4& b, f32x16 acc) {
  if (!__any(not_finite(a))) return mfma32x32x16(a, b, acc);
  u32x4 clean, pos, neg, mag;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    uint32_t cl = 0, po = 0, ne = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t x = (a[w] >> (16 * h)) & 0xFFFFu;
      const bool bad = (x & 0x7F80u) == 0x7F80u, nan = bad && (x & 0x7Fu) != 0;
      if (!bad) cl |= x << (16 * h);
      if (nan || x == 0x7F80u) po |= 0x3F80u << (16 * h);
      if (nan || x == 0xFF80u) ne |= 0x3F80u << (16 * h);
    }
    clean[w] = cl;
    pos[w] = po;
    neg[w] = ne;
    mag[w] = b[w] & 0x7FFF7FFFu;
  }
  acc = mfma32x32x16(clean, b, acc);
  const f32x16 up = mfma32x32x16(pos, mag, zero16()), down = mfma32x32x16(neg, mag, zero16());
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    // (a NaN in B is a NaN in both)
    if (!(up[v] == 0.0f)) acc[v] += GRAD ? __builtin_nanf("") : __builtin_inff();
    if (!(down[v] == 0.0f)) acc[v] += GRAD ? __builtin_nanf("") : -__builtin_inff();
  }
  return acc;
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
  return j <= p && (p - j < window || j < sinks);
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

// Columns of a transposed result (lane mod 32: the row of the output) as rows of bf16.
template <int HD>
__device__ __forceinline__ void store_rows(const f32x16 (&acc)[HD / 32], float f, uint16_t* row, int hd, int lane) {
#pragma unroll
  for (int d = 0; d < HD / 32; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int c = 32 * d + 8 * g + 4 * (lane >> 5);
      if (c < hd) {
        u32x2 w = {pack_bf16x2(acc[d][4 * g] * f, acc[d][4 * g + 1] * f),
                   pack_bf16x2(acc[d][4 * g + 2] * f, acc[d][4 * g + 3] * f)};
        *reinterpret_cast<u32x2*>(row + c) = w;
      }
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
  // The reference moves only when a score lies more than 2^8 above it: P <= 256 costs no
  // accuracy in fp32 sums and bf16 factors, and most tiles leave O alone.
  __device__ __forceinline__ void raise(float top) {
    top = fmaxf(top, other_half(top));
    if (__any(top > m + 8.0f)) {
      const float nm = fmaxf(m, top);
      const float f = nm == -__builtin_inff() ? 1.0f : exp2_fast(m - nm);
      m = nm;
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
// A workgroup of four waves takes 128 NQ queries of one head, NQ columns of 32 per wave.
template <int HD, int NQ>
__global__ __launch_bounds__(256, 2) void k_attn_fwd(AttnArgs a) {
  constexpr int BM = 128 * NQ, KS = HD / 16;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int nqb = (a.lq + BM - 1) / BM;
  const uint32_t id = xcd_remap(blockIdx.x, gridDim.x);
  const int bh = static_cast<int>(id / nqb), qb = nqb - 1 - static_cast<int>(id % nqb);
  const int b = bh / a.heads, h = bh % a.heads, hk = h / (a.heads / a.kv);
  const int L = length_of(a, b), off = L - a.lq;
  const uint16_t* q = a.q + b * a.qs[0] + h * a.qs[1];
  const uint16_t* k = a.k + b * a.ks[0] + hk * a.ks[1];
  const uint16_t* v = a.v + b * a.vs[0] + hk * a.vs[1];
  const float c = a.scale * kLog2e;

  const int q0 = qb * BM, last = min(a.lq, q0 + BM) - 1;
  const Walk<kBN> walk(q0 + off, last + off, L, a.window, a.sinks);
  const int w0 = q0 + wave * 32 * NQ;
  u32x4 qf[NQ][KS];
  Softmax<HD> sm[NQ];
  int p[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int row = w0 + 32 * n + (lane & 31);
    load_frags<HD>(qf[n], q, a.qs[2], row, a.lq, a.hd, lane);
    sm[n].init();
    p[n] = row + off;
  }
  const int pmin = w0 + off, pmax = min(w0 + 32 * NQ - 1, last) + off;

  Stage<HD, kBN, 256> sk, sv;
  if (walk.count > 0) {
    sk.load(k, a.ks[2], walk.key(0), L, a.hd, tid);
    sv.load(v, a.vs[2], walk.key(0), L, a.hd, tid);
  }
  for (int t = 0; t < walk.count; ++t) {
    char* tk = lds + (t & 1) * 2 * Tile<HD>::kBytes;
    char* tv = tk + Tile<HD>::kBytes;
    sk.store(tk, tid);
    sv.store(tv, tid);
    __syncthreads();
    if (t + 1 < walk.count) {
      sk.load(k, a.ks[2], walk.key(t + 1), L, a.hd, tid);
      sv.load(v, a.vs[2], walk.key(t + 1), L, a.hd, tid);
    }
    const int j0 = walk.key(t);
    if (w0 > last || none_seen(j0, kBN, pmin, pmax, a.window, a.sinks)) continue;
    f32x16 s[NQ][2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) s[n][kb] = zero16();
#pragma unroll
      for (int st = 0; st < KS; ++st) {
        const u32x4 kf = Tile<HD>::row_frag(tk, 32 * kb, st, lane);
#pragma unroll
        for (int n = 0; n < NQ; ++n) s[n][kb] = mfma32x32x16(kf, qf[n][st], s[n][kb]);
      }
    }
    const bool edge = !all_seen(j0, kBN, pmin, pmax, a.window, a.sinks);
    if (edge) {
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (!seen(j0 + 32 * kb + acc_row(e, lane), p[n], a.window, a.sinks)) s[n][kb][e] = -__builtin_inff();
    }
    u32x4 pf[NQ][4];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      float top = s[n][0][0];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, s[n][kb][e]);
      sm[n].raise(top * c);
      const float sh = sm[n].shift();
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          s[n][kb][e] = exp2_fast(__builtin_fmaf(s[n][kb][e], c, -sh));
          sm[n].l += s[n][kb][e];
        }
        u32x4 two[2];
        pack_steps(s[n][kb], two);
        pf[n][2 * kb] = two[0];
        pf[n][2 * kb + 1] = two[1];
      }
    }
#pragma unroll
    for (int st = 0; st < 4; ++st)
#pragma unroll
      for (int d = 0; d < HD / 32; ++d) {
        const u32x4 vf = Tile<HD>::col_frag(tv, 16 * st, d, lane);
        if (edge) {
#pragma unroll
          for (int n = 0; n < NQ; ++n) sm[n].o[d] = mfma_seen<false>(vf, pf[n][st], sm[n].o[d]);
        } else {
#pragma unroll
          for (int n = 0; n < NQ; ++n) sm[n].o[d] = mfma32x32x16(vf, pf[n][st], sm[n].o[d]);
        }
      }
  }
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int row = w0 + 32 * n + (lane & 31);
    const float l = sm[n].l + other_half(sm[n].l);
    if (row >= a.lq) continue;
    const bool empty = sm[n].m == -__builtin_inff() && l == 0.0f;
    store_rows<HD>(sm[n].o, empty ? 0.0f : 1.0f / l, a.o + b * a.os[0] + h * a.os[1] + row * a.os[2], a.hd, lane);
    if (lane < 32) a.lse[int64_t(bh) * a.lq + row] = empty ? __builtin_inff() : sm[n].m + log2f(l);
  }
}

// ------------------------- forward, split over the keys ----------------------
// Few rows over many keys: the rows of the heads that share keys (32 of the G lq at a time)
// are the columns of one wave, and each wave takes a range of the keys on its own, K straight
// from memory as the A operand, V through its own part of LDS.
template <int HD>
__global__ __launch_bounds__(256) void k_attn_split(AttnArgs a) {
  constexpr int KS = HD / 16, TN = 32;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int G = a.heads / a.kv, R = G * a.lq;
  const int split = static_cast<int>(blockIdx.x) * 4 + wave, r0 = static_cast<int>(blockIdx.y) * 32;
  const int b = static_cast<int>(blockIdx.z) / a.kv, hk = static_cast<int>(blockIdx.z) % a.kv;
  if (split >= a.splits) return;
  const int L = length_of(a, b), off = L - a.lq;
  const uint16_t* k = a.k + b * a.ks[0] + hk * a.ks[1];
  const uint16_t* v = a.v + b * a.vs[0] + hk * a.vs[1];
  const float c = a.scale * kLog2e;
  const int r = r0 + (lane & 31), g = min(r, R - 1) / a.lq, i = min(r, R - 1) - g * a.lq;
  const int p = i + off;
  // rows of one head: a range of positions; of several: all of them
  const int rl = min(r0 + 31, R - 1);
  const bool one = r0 / a.lq == rl / a.lq;
  const int pmin = (one ? r0 % a.lq : 0) + off, pmax = (one ? rl % a.lq : a.lq - 1) + off;
  const Walk<TN> walk(pmin, pmax, L, a.window, a.sinks);
  const int per = (walk.count + a.splits - 1) / a.splits;
  const int t0 = split * per, t1 = min(walk.count, t0 + per);

  u32x4 qf[KS];
  load_frags<HD>(qf, a.q + b * a.qs[0] + (hk * G + g) * a.qs[1], a.qs[2], r < R ? i : a.lq, a.lq, a.hd, lane);
  Softmax<HD> sm;
  sm.init();
  char* tv = lds + wave * (TN * HD * 2);
  u32x4 kf[KS], kn[KS];
  Stage<HD, TN, 64> sv;
  if (t0 < t1) {
    load_frags<HD>(kn, k, a.ks[2], walk.key(t0) + (lane & 31), L, a.hd, lane);
    sv.load(v, a.vs[2], walk.key(t0), L, a.hd, lane);
  }
  for (int t = t0; t < t1; ++t) {
    const int j0 = walk.key(t);
#pragma unroll
    for (int s = 0; s < KS; ++s) kf[s] = kn[s];
    sv.store(tv, lane);
    if (t + 1 < t1) {
      load_frags<HD>(kn, k, a.ks[2], walk.key(t + 1) + (lane & 31), L, a.hd, lane);
      sv.load(v, a.vs[2], walk.key(t + 1), L, a.hd, lane);
    }
    f32x16 s = zero16();
#pragma unroll
    for (int st = 0; st < KS; ++st) s = mfma32x32x16(kf[st], qf[st], s);
    const bool edge = !all_seen(j0, TN, pmin, pmax, a.window, a.sinks);
    if (edge) {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (!seen(j0 + acc_row(e, lane), p, a.window, a.sinks)) s[e] = -__builtin_inff();
    }
    float top = s[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) top = fmaxf(top, s[e]);
    sm.raise(top * c);
    const float sh = sm.shift();
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[e] = exp2_fast(__builtin_fmaf(s[e], c, -sh));
      sm.l += s[e];
    }
    u32x4 pf[2];
    pack_steps(s, pf);
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int d = 0; d < HD / 32; ++d) {
        const u32x4 vf = Tile<HD>::col_frag(tv, 16 * st, d, lane);
        sm.o[d] = edge ? mfma_seen<false>(vf, pf[st], sm.o[d]) : mfma32x32x16(vf, pf[st], sm.o[d]);
      }
  }
  const float l = sm.l + other_half(sm.l);
  if (r >= R) return;
  const int64_t row = (int64_t(b) * a.heads + hk * G + g) * a.lq + i, rows = int64_t(a.b) * a.heads * a.lq;
  const bool empty = sm.m == -__builtin_inff() && l == 0.0f;
  if (lane < 32) a.part_lse[split * rows + row] = empty ? -__builtin_inff() : sm.m + log2f(l);
  const float f = empty ? 0.0f : 1.0f / l;
  float* out = a.part_o + (split * rows + row) * a.hd;
#pragma unroll
  for (int d = 0; d < HD / 32; ++d)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int cc = 32 * d + 8 * e + 4 * (lane >> 5);
      if (cc < a.hd) {
        f32x4 w = {sm.o[d][4 * e] * f, sm.o[d][4 * e + 1] * f, sm.o[d][4 * e + 2] * f, sm.o[d][4 * e + 3] * f};
        *reinterpret_cast<f32x4*>(out + cc) = w;
      }
    }
}

// The splits' rows joined: o = sum 2^(lse_i - lse) o_i; a wave per row, two columns per lane.
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t rows = int64_t(a.b) * a.heads * a.lq, row = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (row >= rows) return;
  float m = -__builtin_inff();
  for (int s = lane; s < a.splits; s += 64) {
    const float x = a.part_lse[s * rows + row];
    m = x > m || x != x ? x : m;
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const float x = __shfl_xor(m, d, 64);
    m = x > m || x != x ? x : m;
  }
  const bool empty = m == -__builtin_inff();
  float l = 0.0f, o0 = 0.0f, o1 = 0.0f;
  const int c = 2 * lane;
  for (int s = 0; s < a.splits; ++s) {
    const float x = a.part_lse[s * rows + row];
    if (x == -__builtin_inff()) continue;
    const float f = exp2_fast(x - m);
    l += f;
    if (c < a.hd) {
      const float2 w = *reinterpret_cast<const float2*>(a.part_o + (s * rows + row) * a.hd + c);
      o0 += f * w.x;
      o1 += f * w.y;
    }
  }
  const float f = empty ? 0.0f : 1.0f / l;
  const int bh = static_cast<int>(row / a.lq), i = static_cast<int>(row % a.lq);
  if (c < a.hd)
    *reinterpret_cast<uint32_t*>(a.o + (bh / a.heads) * a.os[0] + (bh % a.heads) * a.os[1] + i * a.os[2] + c) =
        pack_bf16x2(o0 * f, o1 * f);
  if (lane == 0) a.lse[row] = empty ? __builtin_inff() : m + log2f(l);
}

// ------------------------------ gradient of q --------------------------------
// As the forward, with S^T and dP^T = V dO^T; D = sum(dO o) on the way (o as it was rounded),
// for the other kernel too.
template <int HD, int NQ>
__global__ __launch_bounds__(256, 2) void k_attn_dq(AttnGradArgs ga) {
  constexpr int BM = 128 * NQ, KS = HD / 16;
  const AttnArgs& a = ga.f;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int nqb = (a.lq + BM - 1) / BM;
  const uint32_t id = xcd_remap(blockIdx.x, gridDim.x);
  const int bh = static_cast<int>(id / nqb), qb = nqb - 1 - static_cast<int>(id % nqb);
  const int b = bh / a.heads, h = bh % a.heads, hk = h / (a.heads / a.kv);
  const int L = length_of(a, b), off = L - a.lq;
  const uint16_t* k = a.k + b * a.ks[0] + hk * a.ks[1];
  const uint16_t* v = a.v + b * a.vs[0] + hk * a.vs[1];
  const float c = a.scale * kLog2e;

  const int q0 = qb * BM, last = min(a.lq, q0 + BM) - 1;
  const Walk<kBN> walk(q0 + off, last + off, L, a.window, a.sinks);
  const int w0 = q0 + wave * 32 * NQ;
  u32x4 qf[NQ][KS], gf[NQ][KS];
  f32x16 dq[NQ][HD / 32];
  float lse[NQ], delta[NQ];
  int p[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int row = w0 + 32 * n + (lane & 31);
    load_frags<HD>(qf[n], a.o + b * a.os[0] + h * a.os[1], a.os[2], row, a.lq, a.hd, lane);
    load_frags<HD>(gf[n], ga.go + b * ga.gs[0] + h * ga.gs[1], ga.gs[2], row, a.lq, a.hd, lane);
    float s = 0.0f;
#pragma unroll
    for (int st = 0; st < KS; ++st)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        s = __builtin_fmaf(__uint_as_float(qf[n][st][w] << 16), __uint_as_float(gf[n][st][w] << 16), s);
        s = __builtin_fmaf(__uint_as_float(qf[n][st][w] & 0xFFFF0000u), __uint_as_float(gf[n][st][w] & 0xFFFF0000u), s);
      }
    delta[n] = s + other_half(s);
    lse[n] = row < a.lq ? a.lse[int64_t(bh) * a.lq + row] : __builtin_inff();
    if (row < a.lq && lane < 32) ga.delta[int64_t(bh) * a.lq + row] = delta[n];
    load_frags<HD>(qf[n], a.q + b * a.qs[0] + h * a.qs[1], a.qs[2], row, a.lq, a.hd, lane);
    p[n] = row + off;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) dq[n][d] = zero16();
  }
  const int pmin = w0 + off, pmax = min(w0 + 32 * NQ - 1, last) + off;

  Stage<HD, kBN, 256> sk, sv;
  if (walk.count > 0) {
    sk.load(k, a.ks[2], walk.key(0), L, a.hd, tid);
    sv.load(v, a.vs[2], walk.key(0), L, a.hd, tid);
  }
  for (int t = 0; t < walk.count; ++t) {
    char* tk = lds + (t & 1) * 2 * Tile<HD>::kBytes;
    char* tv = tk + Tile<HD>::kBytes;
    sk.store(tk, tid);
    sv.store(tv, tid);
    __syncthreads();
    if (t + 1 < walk.count) {
      sk.load(k, a.ks[2], walk.key(t + 1), L, a.hd, tid);
      sv.load(v, a.vs[2], walk.key(t + 1), L, a.hd, tid);
    }
    const int j0 = walk.key(t);
    if (w0 > last || none_seen(j0, kBN, pmin, pmax, a.window, a.sinks)) continue;
    const bool edge = !all_seen(j0, kBN, pmin, pmax, a.window, a.sinks);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      f32x16 s[NQ], dp[NQ];
#pragma unroll
      for (int n = 0; n < NQ; ++n) s[n] = dp[n] = zero16();
#pragma unroll
      for (int st = 0; st < KS; ++st) {
        const u32x4 kf = Tile<HD>::row_frag(tk, 32 * kb, st, lane), vf = Tile<HD>::row_frag(tv, 32 * kb, st, lane);
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          s[n] = mfma32x32x16(kf, qf[n][st], s[n]);
          dp[n] = mfma32x32x16(vf, gf[n][st], dp[n]);
        }
      }
      u32x4 ds[NQ][2];
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          s[n][e] = exp2_fast(__builtin_fmaf(s[n][e], c, -lse[n])) * (dp[n][e] - delta[n]);
        if (edge) {
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (!seen(j0 + 32 * kb + acc_row(e, lane), p[n], a.window, a.sinks)) s[n][e] = 0.0f;
        }
        pack_steps(s[n], ds[n]);
      }
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int d = 0; d < HD / 32; ++d) {
          const u32x4 kf = Tile<HD>::col_frag(tk, 32 * kb + 16 * st, d, lane);
          if (edge) {
#pragma unroll
            for (int n = 0; n < NQ; ++n) dq[n][d] = mfma_seen<true>(kf, ds[n][st], dq[n][d]);
          } else {
#pragma unroll
            for (int n = 0; n < NQ; ++n) dq[n][d] = mfma32x32x16(kf, ds[n][st], dq[n][d]);
          }
        }
    }
  }
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int row = w0 + 32 * n + (lane & 31);
    if (row < a.lq)
      store_rows<HD>(dq[n], a.scale, ga.dq + b * ga.dqs[0] + h * ga.dqs[1] + row * ga.dqs[2], a.hd, lane);
  }
}

// --------------------------- gradients of k and v ----------------------------
// A workgroup takes 128 keys, 32 per wave, and walks the query tiles of every head that
// shares them (their sum is formed here, in order).
template <int HD>
__global__ __launch_bounds__(256, 2) void k_attn_dkv(AttnGradArgs ga) {
  constexpr int BK = 128, KS = HD / 16;
  const AttnArgs& a = ga.f;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int nkb = (a.lk + BK - 1) / BK, G = a.heads / a.kv;
  const uint32_t id = xcd_remap(blockIdx.x, gridDim.x);
  const int bk = static_cast<int>(id / nkb), kb = static_cast<int>(id % nkb);
  const int b = bk / a.kv, hk = bk % a.kv;
  const int L = length_of(a, b), off = L - a.lq;
  const int k0 = kb * BK, w0 = k0 + wave * 32, j = w0 + (lane & 31);
  const float c = a.scale * kLog2e;

  u32x4 kf[KS], vf[KS];
  load_frags<HD>(kf, a.k + b * a.ks[0] + hk * a.ks[1], a.ks[2], j, L, a.hd, lane);
  load_frags<HD>(vf, a.v + b * a.vs[0] + hk * a.vs[1], a.vs[2], j, L, a.hd, lane);
  f32x16 dk[HD / 32], dv[HD / 32];
#pragma unroll
  for (int d = 0; d < HD / 32; ++d) dk[d] = dv[d] = zero16();

  // the rows that see some key of the block
  const int kl = min(k0 + BK, L) - 1;
  int i0 = max(0, k0 - off), i1 = a.lq;
  if (k0 >= a.sinks && int64_t(kl) + a.window - off < i1) i1 = kl + a.window - off;
  i0 = i0 / kBN;
  const int tiles = kl < k0 || i1 <= i0 * kBN ? 0 : (i1 + kBN - 1) / kBN - i0;
  const int steps = tiles * G;

  Stage<HD, kBN, 256> sq, sg;
  float rl = 0.0f, rd = 0.0f;  // thread 0 .. 63: lse and D of a row
  auto fetch = [&](int t) {
    const int h = hk * G + t / tiles, r0 = (i0 + t % tiles) * kBN;
    sq.load(a.q + b * a.qs[0] + h * a.qs[1], a.qs[2], r0, a.lq, a.hd, tid);
    sg.load(ga.go + b * ga.gs[0] + h * ga.gs[1], ga.gs[2], r0, a.lq, a.hd, tid);
    if (tid < kBN) {
      const int64_t at = (int64_t(b) * a.heads + h) * a.lq + r0 + tid;
      const bool in = r0 + tid < a.lq;
      rl = in ? a.lse[at] : __builtin_inff();
      rd = in ? ga.delta[at] : 0.0f;
    }
  };
  if (steps > 0) fetch(0);
  for (int t = 0; t < steps; ++t) {
    char* tq = lds + (t & 1) * (2 * Tile<HD>::kBytes + 2 * kBN * 4);
    char* tg = tq + Tile<HD>::kBytes;
    float* sl = reinterpret_cast<float*>(tg + Tile<HD>::kBytes);
    sq.store(tq, tid);
    sg.store(tg, tid);
    if (tid < kBN) {
      sl[tid] = rl;
      sl[kBN + tid] = rd;
    }
    __syncthreads();
    if (t + 1 < steps) fetch(t + 1);
    const int r0 = (i0 + t % tiles) * kBN;
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
      const int pmin = r0 + 32 * qb + off, pmax = pmin + 31;
      if (w0 >= L || none_seen(w0, 32, pmin, pmax, a.window, a.sinks)) continue;
      const bool edge = r0 + 32 * qb + 31 >= a.lq || w0 + 31 >= L || !all_seen(w0, 32, pmin, pmax, a.window, a.sinks);
      f32x16 s = zero16(), dp = zero16();
#pragma unroll
      for (int st = 0; st < KS; ++st) {
        s = mfma32x32x16(Tile<HD>::row_frag(tq, 32 * qb, st, lane), kf[st], s);
        dp = mfma32x32x16(Tile<HD>::row_frag(tg, 32 * qb, st, lane), vf[st], dp);
      }
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 l4 = *reinterpret_cast<const f32x4*>(sl + 32 * qb + 8 * g + 4 * (lane >> 5));
        const f32x4 d4 = *reinterpret_cast<const f32x4*>(sl + kBN + 32 * qb + 8 * g + 4 * (lane >> 5));
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
          const int i = r0 + 32 * qb + acc_row(e, lane);
          if (i >= a.lq || j >= L || !seen(j, i + off, a.window, a.sinks)) s[e] = dp[e] = 0.0f;
        }
      }
      u32x4 pf[2], df[2];
      pack_steps(s, pf);
      pack_steps(dp, df);
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int d = 0; d < HD / 32; ++d) {
          const u32x4 gt = Tile<HD>::col_frag(tg, 32 * qb + 16 * st, d, lane);
          const u32x4 qt = Tile<HD>::col_frag(tq, 32 * qb + 16 * st, d, lane);
          if (edge) {
            dv[d] = mfma_seen<true>(gt, pf[st], dv[d]);
            dk[d] = mfma_seen<true>(qt, df[st], dk[d]);
          } else {
            dv[d] = mfma32x32x16(gt, pf[st], dv[d]);
            dk[d] = mfma32x32x16(qt, df[st], dk[d]);
          }
        }
    }
  }
  if (j < a.lk) {
    store_rows<HD>(dk, a.scale, ga.dk + b * ga.dks[0] + hk * ga.dks[1] + j * ga.dks[2], a.hd, lane);
    store_rows<HD>(dv, 1.0f, ga.dv + b * ga.dvs[0] + hk * ga.dvs[1] + j * ga.dvs[2], a.hd, lane);
  }
}

bool args_ok(const AttnArgs& a) {
  constexpr int64_t most = int64_t(1) << 30;
  if (a.b < 1 || a.heads < 1 || a.kv < 1 || a.heads % a.kv != 0 || a.lq < 1 || a.lk < 1 || a.hd < 8 || a.hd % 8 != 0 ||
      a.hd > 128 || a.window < 1 || a.sinks < 0 || a.lq > most || a.lk > most || a.window > most || a.sinks > most ||
      !(a.scale > 0.0f))
    return false;
  return int64_t(a.b) * a.heads * ceil_div(a.lq, 32) < (int64_t(1) << 24) &&
         int64_t(a.b) * a.kv * ceil_div(a.lk, 32) < (int64_t(1) << 24);
}

template <int HD, int NQ>
void launch_fwd(const AttnArgs& a, hipStream_t s) {
  const int grid = a.b * a.heads * static_cast<int>(ceil_div(a.lq, 128 * NQ));
  hipLaunchKernelGGL((k_attn_fwd<HD, NQ>), dim3(grid), dim3(256), 4 * Tile<HD>::kBytes, s, a);
}

template <int HD>
void launch_split(const AttnArgs& a, hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>(ceil_div(a.splits, 4)),
                  static_cast<uint32_t>(ceil_div(int64_t(a.heads / a.kv) * a.lq, 32)), static_cast<uint32_t>(a.b * a.kv));
  hipLaunchKernelGGL((k_attn_split<HD>), grid, dim3(256), 4 * 32 * HD * 2, s, a);
  const int64_t rows = int64_t(a.b) * a.heads * a.lq;
  hipLaunchKernelGGL(k_attn_join, dim3(static_cast<uint32_t>(ceil_div(rows, 4))), dim3(256), 0, s, a);
}

template <int HD, int NQ>
void launch_bwd(const AttnGradArgs& a, bool kv, hipStream_t s) {
  const int grid = a.f.b * a.f.heads * static_cast<int>(ceil_div(a.f.lq, 128 * NQ));
  hipLaunchKernelGGL((k_attn_dq<HD, NQ>), dim3(grid), dim3(256), 4 * Tile<HD>::kBytes, s, a);
  if (!kv) return;
  const int keys = a.f.b * a.f.kv * static_cast<int>(ceil_div(a.f.lk, 128));
  hipLaunchKernelGGL((k_attn_dkv<HD>), dim3(keys), dim3(256), 2 * (2 * Tile<HD>::kBytes + 2 * kBN * 4), s, a);
}

int status() { return hipGetLastError() == hipSuccess ? 0 : -5; }

}  // namespace
}  // namespace compact

using namespace compact;

extern "C" {

int compact_attention_fwd(const AttnArgs* a, void* stream) {
  if (!args_ok(*a)) return -1;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (a->splits > 0) {
    if (int64_t(a->b) * a->kv > 65535 || ceil_div(int64_t(a->heads / a->kv) * a->lq, 32) > 65535) return -1;
    if (a->hd <= 64) launch_split<64>(*a, s);
    else if (a->hd <= 96) launch_split<96>(*a, s);
    else launch_split<128>(*a, s);
  } else if (a->hd <= 64) launch_fwd<64, 2>(*a, s);
  else if (a->hd <= 96) launch_fwd<96, 1>(*a, s);
  else launch_fwd<128, 1>(*a, s);
  return status();
}

// dk and dv are left out where dk is NULL.
int compact_attention_bwd(const AttnGradArgs* a, void* stream) {
  if (!args_ok(a->f)) return -1;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool kv = a->dk != nullptr;
  if (a->f.hd <= 64) launch_bwd<64, 1>(*a, kv, s);
  else if (a->f.hd <= 96) launch_bwd<96, 1>(*a, kv, s);
  else launch_bwd<128, 1>(*a, kv, s);
  return status();
}

}  // extern "C"
