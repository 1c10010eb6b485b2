// Attention over padded batches: the kernels and entry points of window_attention, around the
// tiles of attention_tiles.hpp, which has the mathematics; and the forward of few rows over many
// keys, split over the keys.
#include "attention_tiles.hpp"

namespace compact {
namespace {

template <int HD>
__global__ __launch_bounds__(256, 2) void k_attn_fwd(AttnArgs a) {
  __shared__ __attribute__((aligned(16))) TilePair<HD> even, odd;
  const int nqb = (a.lq + 127) / 128, splits = a.splits > 0 ? a.splits : 1;
  const uint32_t id0 = xcd_remap(blockIdx.x, gridDim.x), id = id0 / splits;
  const int split = static_cast<int>(id0 % splits);
  const int bh = static_cast<int>(id / nqb), q0 = (nqb - 1 - static_cast<int>(id % nqb)) * 128;
#pragma unroll 1
  for (int mode = kPlain; mode <= kNeg; ++mode) {
    if (attn_fwd<HD, false>(a, Span<false>(a, bh / a.heads), even, odd, bh % a.heads, q0, split, mode) && mode == kPlain) break;
    __syncthreads();
  }
}

// ------------------------- forward, split over the keys ----------------------
// Few rows over many keys: the rows of the heads that share keys (32 of the G lq at a time)
// are the columns of one wave, and each wave takes a range of the keys on its own: K straight
// from memory as the A operand, V by copies into its own part of LDS, both a tile of 32 keys
// ahead.  Bound by HBM where there are keys enough: 157 us, 5.5 TB/s, for one token of 4
// sequences of up to 70000 keys, 32 heads on 8 of 128 (with the join 167 us), as a large copy;
// 15 us and the join's 4 for 16 sequences, 16 heads of 64, 1028 keys seen (4.3 TB/s over both
// would be 13 us), where each wave's few tiles in a row are what counts.
template <int HD>
struct WaveTiles {
  char v[4][32 * HD * 2];
};

template <int HD>
__device__ __forceinline__ bool attn_split(const AttnArgs& a, WaveTiles<HD>& even, WaveTiles<HD>& odd, int split, int r0, int b,
                                           int hk, int mode) {
  constexpr int KS = HD / 16, TN = 32;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int G = a.heads / a.kv, R = G * a.lq;
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

  u32x4 qf[KS], kf[KS];
  Copy<HD, TN, 1> cv;
  cv.init(a.vs[2], a.hd, lane);
  const int koff = (lane & 31) * static_cast<int>(a.ks[2]) * 2 + 16 * (lane >> 5);
  // always issued, past the last tile with no rows: a wait then counts the loads behind it
  auto rows_of = [&](int t) { return t < t1 ? min(L - walk.key(t), TN) : 0; };
  auto fetch_v = [&](int t, WaveTiles<HD>& to) {
    cv.issue(v, a.vs[2], walk.key(t), walk.key(t) + rows_of(t), a.hd, to.v[wave], 0);
  };
  auto fetch_k = [&](int t) {
    const __amdgpu_buffer_rsrc_t rs = tile_rows(k, a.ks[2], walk.key(t), mode >= kPos ? 0 : rows_of(t), a.hd);
#pragma unroll
    for (int s = 0; s < KS; ++s)
      kf[s] = __builtin_amdgcn_raw_buffer_load_b128(rs, 16 * s + 8 * (lane >> 5) < a.hd ? koff + 32 * s : 0x7FFFFFF0, 0, 0);
  };
  fetch_v(t0, even);
  fetch_k(t0);
  load_frags<HD>(qf, a.q + b * a.qs[0] + (hk * G + g) * a.qs[1], a.qs[2], r < R ? i : a.lq, a.lq, a.hd, lane);
  Softmax<HD> sm;
  sm.init();
  auto step = [&](int t, WaveTiles<HD>& now, WaveTiles<HD>& next) {
    const int j0 = walk.key(t);
    fetch_v(t + 1, next);
    if (mode != kPlain) convert_tile<HD, TN, 64>(now.v[wave], mode, nullptr, lane);
    f32x16 one[1] = {zero16()}, &s = one[0];
#pragma unroll
    for (int st = 0; st < KS; ++st) s = mfma32x32x16(kf[st], qf[st], s);
    fetch_k(t + 1);
    if (!all_seen(j0, TN, pmin, pmax, a.window, a.sinks)) hide_unseen(one, -__builtin_inff(), j0, p, a.window, a.sinks, lane);
    float top = s[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) top = max_of(top, s[e]);
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
      for (int d = 0; d < HD / 32; ++d)
        sm.o[d] = mfma32x32x16(Tile<HD>::col_frag(now.v[wave], 16 * st, d, lane), pf[st], sm.o[d]);
  };
  for (int t = t0; t < t1; t += 2) {
    step(t, even, odd);
    if (t + 1 < t1) step(t + 1, odd, even);
  }
  if (mode == kPlain && __any(not_finite(sm.o))) return false;
  const float l = halves_sum(sm.l);
  if (r >= R) return true;
  const int64_t row = (int64_t(b) * a.heads + hk * G + g) * a.lq + i, rows = int64_t(a.b) * a.heads * a.lq;
  float* out = a.part_o + (split * rows + row) * a.hd;
  if (mode >= kPos) {
    mark_rows<HD>(sm.o, mode, out, a.hd, lane);
    return true;
  }
  const bool empty = sm.m == -__builtin_inff() && l == 0.0f;
  if (lane < 32) a.part_lse[split * rows + row] = empty ? -__builtin_inff() : sm.m + log2f(l);
  store_row_values<HD>(sm.o, empty ? 0.0f : 1.0f / l, out, a.hd, lane);
  return true;
}

template <int HD>
__global__ __launch_bounds__(256, 2) void k_attn_split(AttnArgs a) {
  __shared__ __attribute__((aligned(16))) WaveTiles<HD> even, odd;
  const int split = static_cast<int>(blockIdx.x) * 4 + static_cast<int>(threadIdx.x >> 6), r0 = static_cast<int>(blockIdx.y) * 32;
  const int b = static_cast<int>(blockIdx.z) / a.kv, hk = static_cast<int>(blockIdx.z) % a.kv;
  if (split >= a.splits) return;
#pragma unroll 1
  for (int mode = kPlain; mode <= kNeg; ++mode)
    if (attn_split<HD>(a, even, odd, __builtin_amdgcn_readfirstlane(split), r0, b, hk, mode) && mode == kPlain) break;
}

// The splits' rows joined: o = sum 2^(lse_i - lse) o_i.  A workgroup per row, 32 lanes over
// its columns, the splits dealt to 8 such groups: few loads one after another.
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs a) {
  __shared__ float red[4];
  __shared__ f32x4 sums[8][32];
  __shared__ float weights[8];
  const int tid = threadIdx.x, lane = tid & 31, group = tid >> 5;
  const int64_t rows = int64_t(a.b) * a.heads * a.lq, row = blockIdx.x;
  float m = -__builtin_inff();
  for (int s = tid; s < a.splits; s += 256) {
    const float x = a.part_lse[s * rows + row];
    m = x > m || x != x ? x : m;
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const float x = __shfl_xor(m, d, 64);
    m = x > m || x != x ? x : m;
  }
  if ((tid & 63) == 0) red[tid >> 6] = m;
  __syncthreads();
  m = red[0];
  for (int w = 1; w < 4; ++w) m = red[w] > m || red[w] != red[w] ? red[w] : m;
  const int bh = static_cast<int>(row / a.lq), i = static_cast<int>(row % a.lq);
  const bool empty = i + length_of(a, bh / a.heads) - a.lq < 0;  // (of scores that are all -inf the softmax is NaN)
  const float shift = m == -__builtin_inff() ? 0.0f : m;
  float l = 0.0f;
  f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
  const int c = 4 * lane;
  for (int s = group; s < a.splits; s += 8) {
    const float f = exp2_fast(a.part_lse[s * rows + row] - shift);
    l += f;
    if (c < a.hd) {
      const f32x4 w = *reinterpret_cast<const f32x4*>(a.part_o + (s * rows + row) * a.hd + c);
      // (a split without keys holds zeros)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(f, w[e], o[e]);
    }
  }
  sums[group][lane] = o;
  if (lane == 0) weights[group] = l;
  __syncthreads();
  if (group != 0) return;
  for (int g = 1; g < 8; ++g) {
    o += sums[g][lane];
    l += weights[g];
  }
  const float f = empty ? 0.0f : 1.0f / l;
  if (c < a.hd) {
    const float v[4] = {o[0] * f, o[1] * f, o[2] * f, o[3] * f};
    const u32x2 w = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    *reinterpret_cast<u32x2*>(a.o + (bh / a.heads) * a.os[0] + (bh % a.heads) * a.os[1] + i * a.os[2] + c) = w;
    if (a.o_low != nullptr) *reinterpret_cast<uint32_t*>(a.o_low + row * a.hd + c) = low_bytes(v, w);
  }
  if (lane == 0) a.lse[row] = empty ? __builtin_inff() : m + log2f(l);
}

template <int HD, bool FINE>
__global__ __launch_bounds__(256, 2) void k_attn_dq(AttnGradArgs ga) {
  __shared__ __attribute__((aligned(16))) TilePair<HD> even, odd;
  __shared__ int bad_key[kBN];
  const int nqb = (ga.f.lq + 127) / 128;
  const uint32_t id = xcd_remap(blockIdx.x, gridDim.x);
  const int bh = static_cast<int>(id / nqb), q0 = (nqb - 1 - static_cast<int>(id % nqb)) * 128;
#pragma unroll 1
  for (int mode = kPlain; mode <= kClean; ++mode) {
    if (attn_dq<HD, FINE, false>(ga, Span<false>(ga.f, bh / ga.f.heads), even, odd, bad_key, bh % ga.f.heads, q0, mode)) break;
    __syncthreads();
  }
}

template <int HD, bool FINE>
__global__ __launch_bounds__(shared_keys(HD) ? 512 : 256, 2) void k_attn_dkv(AttnGradArgs ga) {
  __shared__ __attribute__((aligned(16))) KeyBlock<HD, shared_keys(HD)> keys;
  __shared__ __attribute__((aligned(16))) RowPair<HD> even, odd;
  __shared__ int bad_row[kBN];
  // A head's blocks stay on one XCD where the heads are a multiple of 8 (on two, where 4): what
  // its workgroups walk at a time is rows that an L2 holds.  (Runs of 8 or of 32 neighbouring
  // blocks, for fewer heads, were no faster, within 0 and 5%, at 16384 rows, 4 heads of k, with
  // the gradient of q.)  The first keys' blocks, whose windows are whole, go first, and
  // the far work, in shorter pieces, last: with a workgroup or two to a CU a long one that
  // starts late is all that runs at the end.
  const int nkb = (ga.f.lk + 127) / 128, nfb = (ga.far_keys + far_block(HD) - 1) / far_block(HD), bk_all = ga.f.b * ga.f.kv;
  const int blocks = nkb * bk_all, near = (blocks + kNumXcd - 1) / kNumXcd * kNumXcd * ga.parts;
  DkvJob job;
  if (static_cast<int>(blockIdx.x) < near) {
    const int k = blockIdx.x / kNumXcd, r = k / ga.parts * kNumXcd + blockIdx.x % kNumXcd;
    if (r >= blocks) return;
    job = {r % bk_all, r / bk_all * 128, k % ga.parts, 0};
  } else {
    const int id = blockIdx.x - near;
    job = {id / (ga.chunks * nfb), id / ga.chunks % nfb * far_block(HD), id % ga.chunks, 1};
  }
#pragma unroll 1
  for (int mode = kPlain; mode <= kClean; ++mode) {
    if (attn_dkv<HD, FINE, false>(ga, Span<false>(ga.f, job.bk / ga.f.kv), keys, even, odd, bad_row, job, mode)) break;
    __syncthreads();
  }
}

// The slots' sum of the first near_keys (or, without near parts, far_keys) keys: four columns
// of dk or dv per thread at a time.
__host__ __device__ inline int64_t dkv_sum_work(const AttnGradArgs& a) { return int64_t(a.f.b) * a.f.kv * a.near_keys * (a.f.hd / 2); }

__global__ __launch_bounds__(256) void k_attn_dkv_sum(AttnGradArgs ga) {
  const AttnArgs& a = ga.f;
  const int cols = 2 * a.hd / 4;
  const int64_t work = dkv_sum_work(ga), bk_all = int64_t(a.b) * a.kv;
  for (int64_t u = int64_t(blockIdx.x) * 256 + threadIdx.x; u < work; u += int64_t(gridDim.x) * 256) {
    const int64_t row = u / cols, bk = row / ga.near_keys;
    const int col = static_cast<int>(u % cols) * 4, j = static_cast<int>(row % ga.near_keys);
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int p = 0; p < ga.parts; ++p)
      s += *reinterpret_cast<const f32x4*>(ga.part + ((p * bk_all + bk) * ga.near_keys + j) * 2 * a.hd + col);
    if (j < ga.far_keys) {
      const float* far = ga.part + ga.parts * bk_all * ga.near_keys * 2 * a.hd;
      for (int p = 0; p < far_slots(a.hd) * ga.chunks; ++p)
        s += *reinterpret_cast<const f32x4*>(far + ((p * bk_all + bk) * ga.far_keys + j) * 2 * a.hd + col);
    }
    const int b = static_cast<int>(bk / a.kv), hk = static_cast<int>(bk % a.kv);
    uint16_t* out = col < a.hd ? ga.dk + b * ga.dks[0] + hk * ga.dks[1] + j * ga.dks[2] + col
                               : ga.dv + b * ga.dvs[0] + hk * ga.dvs[1] + j * ga.dvs[2] + col - a.hd;
    const u32x2 w = {pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3])};
    *reinterpret_cast<u32x2*>(out) = w;
  }
}

// How the gradients of k and v are split (AttnGradArgs), and the floats of `part`.
// parts: 512 workgroups (two per CU) of at least 8 tiles where the blocks of keys are fewer.
// chunks: a far workgroup walks a quarter of a near one's tiles, at least 8.
// The whole backward, us, with at least 4 / 8 tiles: 3 x 1531 rows, 10 heads on 2 of 80, window
// 301: 97 / 83; 2 x 5000, 4 on 1 of 64, window 700: 75 / 71; 1000, 16 on 2 of 96: 62 / 61.
// Far work of at least 16 / 8 tiles: 4 x 4096, 16 heads of 64, window 1024: 326 / 325.
int64_t plan_dkv(AttnGradArgs* g) {
  const AttnArgs& a = g->f;
  const int64_t bk = int64_t(a.b) * a.kv, G = a.heads / a.kv;
  const int64_t blocks = bk * ceil_div(a.lk, 128);
  const int64_t rows = a.window < a.lk ? (int64_t(a.window) + 127 < a.lq ? int64_t(a.window) + 127 : a.lq) : a.lq;
  const int64_t tiles = G * ceil_div(rows, kBN);
  int64_t parts = ceil_div(512, blocks);
  if (parts > tiles / 8) parts = tiles / 8;
  if (parts < 1) parts = 1;
  g->parts = static_cast<int>(parts);
  const bool far = a.sinks > 0 && a.window < a.lk;
  g->far_keys = far ? (a.sinks < a.lk ? a.sinks : a.lk) : 0;
  g->near_keys = parts > 1 ? a.lk : g->far_keys;
  g->fine = (a.window < a.lk ? a.window + a.sinks : a.lk) <= kFineKeys;
  g->chunks = 0;
  if (far) {
    const int64_t far_rows = a.lk - a.window < a.lq ? a.lk - a.window : a.lq, far_tiles = G * ceil_div(far_rows, kBN);
    const int64_t own = ceil_div(tiles, 4 * parts), most = ceil_div(kFarWork, bk * ceil_div(g->far_keys, far_block(a.hd)));
    int64_t chunks = ceil_div(far_tiles, own < 8 ? 8 : own);
    chunks = chunks > 64 ? 64 : chunks;
    g->chunks = static_cast<int>(chunks > most ? most : chunks);
  }
  return 2 * a.hd * bk * (parts * g->near_keys + far_slots(a.hd) * int64_t(g->chunks) * g->far_keys);
}

int64_t dkv_grid(const AttnGradArgs& a) {
  const int64_t bk = int64_t(a.f.b) * a.f.kv;
  return round_up(bk * ceil_div(a.f.lk, 128), kNumXcd) * a.parts + bk * ceil_div(a.far_keys, far_block(a.f.hd)) * a.chunks;
}
// A launch has under 2^32 threads.
bool plan_fits(const AttnGradArgs& a) { return dkv_grid(a) * (shared_keys(a.f.hd) ? 512 : 256) < int64_t(1) << 32; }

void launch_join(const AttnArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(k_attn_join, dim3(static_cast<uint32_t>(int64_t(a.b) * a.heads * a.lq)), dim3(256), 0, s, a);
}

template <int HD>
void launch_fwd(const AttnArgs& a, hipStream_t s) {
  const int grid = a.b * a.heads * static_cast<int>(ceil_div(a.lq, 128)) * (a.splits > 0 ? a.splits : 1);
  hipLaunchKernelGGL((k_attn_fwd<HD>), dim3(grid), dim3(256), 0, s, a);
  if (a.splits > 0) launch_join(a, s);
}

template <int HD>
void launch_waves(const AttnArgs& a, hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>(ceil_div(a.splits, 4)),
                  static_cast<uint32_t>(ceil_div(int64_t(a.heads / a.kv) * a.lq, 32)), static_cast<uint32_t>(a.b * a.kv));
  hipLaunchKernelGGL((k_attn_split<HD>), grid, dim3(256), 0, s, a);
  launch_join(a, s);
}

template <int HD, bool FINE>
void launch_grads(const AttnGradArgs& a, bool kv, hipStream_t s) {
  const int grid = a.f.b * a.f.heads * static_cast<int>(ceil_div(a.f.lq, 128));
  hipLaunchKernelGGL((k_attn_dq<HD, FINE>), dim3(grid), dim3(256), 0, s, a);
  if (!kv) return;
  hipLaunchKernelGGL((k_attn_dkv<HD, FINE>), dim3(static_cast<uint32_t>(dkv_grid(a))), dim3(shared_keys(HD) ? 512 : 256), 0, s, a);
  const int64_t sums = ceil_div(dkv_sum_work(a), 256);
  if (sums > 0) hipLaunchKernelGGL(k_attn_dkv_sum, dim3(static_cast<uint32_t>(sums < kSumGrid ? sums : kSumGrid)), dim3(256), 0, s, a);
}

template <int HD>
void launch_bwd(const AttnGradArgs& a, bool kv, hipStream_t s) {
  if (a.fine) launch_grads<HD, true>(a, kv, s);
  else launch_grads<HD, false>(a, kv, s);
}

}  // namespace
}  // namespace compact

using namespace compact;

extern "C" {

int compact_attention_fwd(const AttnArgs* a, void* stream) {
  if (!args_ok(*a)) return -1;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (a->splits > 0 &&
      (a->splits > 4096 || int64_t(a->b) * a->heads * a->lq >= int64_t(1) << 24 || a->part_o == nullptr ||
       int64_t(a->b) * a->heads * ceil_div(a->lq, 128) * a->splits >= int64_t(1) << 31))
    return -1;
  if (a->splits > 0 && a->waves) {
    if (int64_t(a->b) * a->kv > 65535 || ceil_div(int64_t(a->heads / a->kv) * a->lq, 32) > 65535) return -1;
    if (a->hd <= 64) launch_waves<64>(*a, s);
    else if (a->hd <= 96) launch_waves<96>(*a, s);
    else launch_waves<128>(*a, s);
  } else if (a->hd <= 64) launch_fwd<64>(*a, s);
  else if (a->hd <= 96) launch_fwd<96>(*a, s);
  else launch_fwd<128>(*a, s);
  return status();
}

// The floats of scratch (`part`) that the backward needs; -1: sizes it does not take.
int64_t compact_attention_bwd_scratch(const AttnArgs* a) {
  if (!args_ok(*a)) return -1;
  AttnGradArgs g = {};
  g.f = *a;
  const int64_t floats = plan_dkv(&g);
  return plan_fits(g) ? floats : -1;
}

// dk and dv are left out where dk is NULL.
int compact_attention_bwd(const AttnGradArgs* args, void* stream) {
  AttnGradArgs plan = *args;
  const AttnGradArgs* a = &plan;
  if (!args_ok(a->f) || a->f.o_low == nullptr || a->gs[2] < 0 || a->gs[2] > kMaxStride || (a->f.lq > 1 && a->gs[2] < a->f.hd)) return -1;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool kv = a->dk != nullptr;
  const bool parts = plan_dkv(&plan) > 0;
  if (kv && ((parts && a->part == nullptr) || !plan_fits(plan))) return -1;
  if (a->f.hd <= 64) launch_bwd<64>(*a, kv, s);
  else if (a->f.hd <= 96) launch_bwd<96>(*a, kv, s);
  else launch_bwd<128>(*a, kv, s);
  return status();
}

}  // extern "C"
