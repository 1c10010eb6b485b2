// Attention inside each of n sequences that lie end to end in T rows: the tiles of
// attention_tiles.hpp, with the rows that each workgroup takes from a table which the call's
// first launch writes.
//
// Sequence s holds the rows e_s .. e_{s+1} - 1, with e the running maximum of the given starts,
// each within 0 .. T: whatever they hold, sequences lie inside the rows and apart.  Rows of no
// sequence (before the first, behind the last) are two spans of their own, over no keys: zeros.
//
// Long sequences are bound as padded batches are: 870 us forward, 950 TFLOP/s over the pairs that
// are seen, 1164 us for the gradient of q, 1992 for those of k and v, at 4 documents in 32768 rows,
// 16 heads on 4 of 128, window 4096.  Short ones by a workgroup's life: of 10 us besides its tiles'
// 2 us each, most is waiting for its first loads, which all workgroups make at about the same time:
// 149 us for 31 prompts of 39 to 1367 rows, 32 heads on 8 of 128 (7 tiles to a workgroup); 86, 101
// and 133 us for 24 documents of 87 to 2237 rows, 16 heads of 64 (11 tiles).  Tried and no faster:
// workgroups that stay and fetch the next item's first tile under the last tile of the one before
// (169 us for 152 at the prompts); 32 rows of four heads that share keys to a workgroup (147 for 147).
#include "attention_tiles.hpp"

namespace compact {
namespace {

// The table (int32): the number of items (and three words of nothing), the n + 3 bounds of the
// spans (0, e_0 .. e_n, T), the spans' first items by span (n + 3, scratch), the items.  Each
// of those three starts on a multiple of four words.
struct Plan {
  int32_t* base;
  int spans;  // n + 2
  __host__ __device__ Plan(int32_t* base, int n) : base(base), spans(n + 2) {}
  __host__ __device__ __forceinline__ int64_t words() const { return (int64_t(spans) + 1 + 3) / 4 * 4; }
  __host__ __device__ __forceinline__ int32_t* bounds() const { return base + 4; }
  __host__ __device__ __forceinline__ int32_t* firsts() const { return bounds() + words(); }
  __host__ __device__ __forceinline__ int4* items() const { return reinterpret_cast<int4*>(firsts() + words()); }
};

// Every span begins a tile of 128 rows of its own.
__host__ __device__ inline int64_t most_items(int64_t n, int64_t T) { return T / 128 + (n + 2 < T ? n + 2 : T); }

constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64;
constexpr int kLevels = 4096;  // items are ordered by their tile's number, up to this

// The values of the threads up to this one joined.
template <typename F>
__device__ __forceinline__ int block_scan(int v, int* lds, F join) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int w = __shfl_up(v, d, 64);
    if (lane >= d) v = join(v, w);
  }
  __syncthreads();
  if (lane == 63) lds[wave] = v;
  __syncthreads();
  for (int w = 0; w < wave; ++w) v = join(v, lds[w]);
  return v;
}

__device__ __forceinline__ int start_at(const void* starts, int starts64, int64_t stride, int i, int T) {
  const int64_t x = starts64 ? static_cast<const int64_t*>(starts)[i * stride] : static_cast<const int32_t*>(starts)[i * stride];
  return x < 0 ? 0 : x > T ? T : static_cast<int>(x);
}

__device__ __forceinline__ int upper_span(const int32_t* x, int spans, int i) {  // the last span s with x[s] <= i
  int lo = 0, hi = spans - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (x[mid] <= i) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// One workgroup: two scans over the sequences, then the items, those with the most keys to see
// first (by a count of each tile number and places handed out in its range; the order among
// equals is left open, no result depends on it).  7 us: a launch and some twenty barriers.  (With the
// spans in LDS in place of the table 6.4.)
__global__ __launch_bounds__(kPlanThreads) void k_packed_plan(const void* starts, int starts64, int64_t stride, int n, int T,
                                                              int32_t* base) {
  __shared__ int lds[kPlanWaves], level[kLevels];
  const Plan plan(base, n);
  const int tid = threadIdx.x, spans = plan.spans;
  const auto larger = [](int a, int b) { return a > b ? a : b; };
  const auto sum = [](int a, int b) { return a + b; };
  int32_t *bounds = plan.bounds(), *firsts = plan.firsts();
  int carry = 0;
  for (int i0 = 0; i0 <= spans; i0 += kPlanThreads) {
    const int i = i0 + tid;
    int v = 0;
    if (i >= 1 && i <= n + 1) v = start_at(starts, starts64, stride, i - 1, T);
    else if (i > n + 1) v = T;
    v = larger(block_scan(v, lds, larger), carry);
    if (i <= spans) bounds[i] = v;
    __syncthreads();
    if (tid == kPlanThreads - 1) lds[0] = v;
    __syncthreads();
    carry = lds[0];
    __syncthreads();
  }
  for (int i = tid; i < kLevels; i += kPlanThreads) level[i] = 0;
  carry = 0;
  for (int i0 = 0; i0 < spans; i0 += kPlanThreads) {
    const int i = i0 + tid, tiles = i < spans ? (bounds[i + 1] - bounds[i] + 127) / 128 : 0;
    const int v = block_scan(tiles, lds, sum) + carry;
    if (i < spans) firsts[i] = v - tiles;
    __syncthreads();
    if (tid == kPlanThreads - 1) lds[0] = v;
    __syncthreads();
    carry = lds[0];
    __syncthreads();
  }
  const int count = carry;
  if (tid == 0) base[0] = count;
  for (int i = tid; i < count; i += kPlanThreads) {
    const int s = upper_span(firsts, spans, i), t = i - firsts[s];
    atomicAdd(&level[t < kLevels ? t : kLevels - 1], 1);
  }
  __syncthreads();
  // each level's first place, the highest level first: four to a thread
  constexpr int kOwn = kLevels / kPlanThreads;
  int own[kOwn], all = 0;
#pragma unroll
  for (int k = 0; k < kOwn; ++k) {
    own[k] = level[kLevels - 1 - (tid * kOwn + k)];
    all += own[k];
  }
  int at = block_scan(all, lds, sum) - all;
#pragma unroll
  for (int k = 0; k < kOwn; ++k) {
    level[kLevels - 1 - (tid * kOwn + k)] = at;
    at += own[k];
  }
  __syncthreads();
  for (int i = tid; i < count; i += kPlanThreads) {
    const int s = upper_span(firsts, spans, i), t = i - firsts[s];
    const int place = atomicAdd(&level[t < kLevels ? t : kLevels - 1], 1);
    plan.items()[place] = make_int4(bounds[s], bounds[s + 1] - bounds[s], t, s >= 1 && s <= n ? s - 1 : -1);
  }
}

__device__ __forceinline__ int scalar(int v) { return __builtin_amdgcn_readfirstlane(v); }
// Item i, in scalar registers.
__device__ __forceinline__ int4 item_at(const int4* items, uint32_t i) {
  const int4 v = items[i];
  return make_int4(scalar(v.x), scalar(v.y), scalar(v.z), scalar(v.w));
}

// Workgroups go to the XCDs in turn: with a multiple of 8 heads each XCD keeps its own, in an
// order in which those that share keys are one XCD's.
__device__ __forceinline__ int head_of(uint32_t i, int heads) {
  return heads % kNumXcd == 0 ? static_cast<int>(i % kNumXcd) * (heads / kNumXcd) + static_cast<int>(i / kNumXcd) : static_cast<int>(i);
}

// The starts as the caller gave them.
struct Starts {
  const void* at;
  int64_t stride;
  int32_t is64, n;
};

// Few sequences and few workgroups want no table: each wave finds item `at` of the spans in their
// own order by itself, a span to a lane.  false: there is none.
// us of a forward in a replayed graph, without / with the table: 1 sequence of 8 rows, 8 heads of 64, 24
// workgroups: 6.8 / 11.7; 6 in 6000 rows, 8 of 64, 432: 34.5 / 39.0; 61 in 1952, 8 of 64, 624: 9.4 / 15.1; 20 in
// 6000, 16 of 128, 1088: 35.1 / 40.6; 61 in 18300, 16 of 128, 3280: 102 / 105; 61 in 61000, 8 of 64, 4312: 144 /
// 137, where the table's order, longest first, counts.  (The limit, two workgroups to a CU, is well before that.)
constexpr int kOwnSequences = 61, kOwnGrid = 512;
__device__ __forceinline__ bool own_item(const Starts& s, int T, int at, int4& item) {
  const int lane = threadIdx.x & 63;
  int bound = lane == 0 ? 0 : lane <= s.n + 1 ? start_at(s.at, s.is64, s.stride, lane - 1, T) : T;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int w = __shfl_up(bound, d, 64);
    if (lane >= d) bound = bound > w ? bound : w;
  }
  const int next = __shfl_down(bound, 1, 64);  // (asked of every lane: one that does not ask does not answer)
  const int rows = lane < s.n + 2 ? next - bound : 0, tiles = (rows + 127) / 128;
  int upto = tiles;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int w = __shfl_up(upto, d, 64);
    if (lane >= d) upto += w;
  }
  const uint64_t behind = __ballot(at < upto);
  if (behind == 0) return false;
  const int span = __ffsll(static_cast<unsigned long long>(behind)) - 1;
  item = make_int4(__builtin_amdgcn_readlane(bound, span), __builtin_amdgcn_readlane(rows, span),
                   at - __builtin_amdgcn_readlane(upto - tiles, span), span >= 1 && span <= s.n ? span - 1 : -1);
  return true;
}

template <int HD, bool OWN>
__global__ __launch_bounds__(256, 2) void k_packed_fwd(AttnArgs a, const int32_t* count, const int4* items, Starts starts) {
  __shared__ __attribute__((aligned(16))) TilePair<HD> even, odd;
  const uint32_t id = blockIdx.x, at = id / a.heads;
  int4 item;
  if constexpr (OWN) {
    if (!own_item(starts, a.lq, scalar(static_cast<int>(at)), item)) return;
  } else {
    item = item_at(items, at);  // (read beside the count, not behind it: past it is room, too)
    if (static_cast<int>(at) >= scalar(count[0])) return;
  }
  const Span<true> sp(item.x, item.y, item.w);
#pragma unroll 1
  for (int mode = kPlain; mode <= kNeg; ++mode) {
    if (attn_fwd<HD, true>(a, sp, even, odd, head_of(id % a.heads, a.heads), item.z * 128, 0, mode) && mode == kPlain) break;
    __syncthreads();
  }
}

template <int HD, bool FINE>
__global__ __launch_bounds__(256, 2) void k_packed_dq(AttnGradArgs ga, const int32_t* count, const int4* items) {
  __shared__ __attribute__((aligned(16))) TilePair<HD> even, odd;
  __shared__ int bad_key[kBN];
  const int heads = ga.f.heads;
  const uint32_t id = blockIdx.x, at = id / heads;
  const int4 item = item_at(items, at);
  if (static_cast<int>(at) >= scalar(count[0])) return;
  const Span<true> sp(item.x, item.y, item.w);
  const int h = head_of(id % heads, heads);
#pragma unroll 1
  for (int mode = kPlain; mode <= kClean; ++mode) {
    if (attn_dq<HD, FINE, true>(ga, sp, even, odd, bad_key, h, item.z * 128, mode)) break;
    __syncthreads();
  }
}

__host__ __device__ inline int far_blocks(const AttnGradArgs& a) { return (a.far_keys + far_block(a.f.hd) - 1) / far_block(a.f.hd); }

// A block of keys is seen by the rows behind it: the table's order, read from a sequence's other end.
template <int HD, bool FINE>
__global__ __launch_bounds__(shared_keys(HD) ? 512 : 256, 2) void k_packed_dkv(AttnGradArgs ga, const int32_t* count,
                                                                               const int4* items, const int32_t* bounds,
                                                                               uint32_t near) {
  __shared__ __attribute__((aligned(16))) KeyBlock<HD, shared_keys(HD)> keys;
  __shared__ __attribute__((aligned(16))) RowPair<HD> even, odd;
  __shared__ int bad_row[kBN];
  const int kv = ga.f.kv;
  int4 item;
  DkvJob job;
  if (blockIdx.x < near) {
    const uint32_t r = blockIdx.x / kv, at = r / ga.parts;
    item = item_at(items, at);
    if (static_cast<int>(at) >= scalar(count[0])) return;
    job = {static_cast<int>(blockIdx.x % kv), ((item.y + 127) / 128 - 1 - item.z) * 128, static_cast<int>(r % ga.parts), 0};
    if (item.w < 0 && job.slot > 0) return;  // (rows of no sequence: zeros, written once)
  } else {
    // the sinks' blocks by sequence, or those of the table's blocks that hold sinks
    const uint32_t id = blockIdx.x - near, blocks = packed_by_row(ga) ? 128 / far_block(HD) : far_blocks(ga);
    const uint32_t at = id / (ga.chunks * blocks * kv), block = id / (ga.chunks * kv) % blocks;
    job = {static_cast<int>(id % kv), static_cast<int>(block) * far_block(HD), static_cast<int>(id / kv) % ga.chunks, 1};
    if (packed_by_row(ga)) {
      if (static_cast<int>(at) >= count[0]) return;
      item = item_at(items, at);
      job.k0 += item.z * 128;
      if (job.k0 >= ga.far_keys || item.w < 0) return;
    } else {
      const int first = scalar(bounds[at + 1]);
      item = make_int4(first, scalar(bounds[at + 2]) - first, 0, static_cast<int>(at));
    }
  }
#pragma unroll 1
  for (int mode = kPlain; mode <= kClean; ++mode) {
    // (what a walk forms from the item is formed anew for each: kept for the second, which hardly
    // ever comes, it takes registers that the first lacks)
    asm volatile("" : "+s"(item.x), "+s"(item.y), "+s"(item.w), "+s"(job.k0), "+s"(job.bk), "+s"(job.slot), "+s"(job.far));
    if (attn_dkv<HD, FINE, true>(ga, Span<true>(item.x, item.y, item.w), keys, even, odd, bad_row, job, mode)) break;
    __syncthreads();
  }
}

// The slots' sums, four columns of dk or dv per thread at a time: in parts, of every row of a
// sequence; else of the sequences' first far_keys.
__host__ __device__ inline int64_t packed_sum_work(const AttnGradArgs& a) { return packed_near_rows(a) / a.parts * (a.f.hd / 2); }

__global__ __launch_bounds__(256) void k_packed_sum(AttnGradArgs ga, const int32_t* bounds) {
  const AttnArgs& a = ga.f;
  const int cols = 2 * a.hd / 4, n = ga.sequences;
  const bool by_row = packed_by_row(ga);
  const int64_t far_rows = packed_far_rows(ga), head_rows = ga.parts > 1 ? a.lk : far_rows, work = packed_sum_work(ga);
  for (int64_t u = int64_t(blockIdx.x) * 256 + threadIdx.x; u < work; u += int64_t(gridDim.x) * 256) {
    const int64_t r = u / cols, x = r % head_rows;
    const int col = static_cast<int>(u % cols) * 4, hk = static_cast<int>(r / head_rows);
    const int seq = ga.parts > 1 || by_row ? upper_span(bounds, n + 2, static_cast<int>(x)) - 1 : static_cast<int>(x / ga.far_keys);
    if (seq < 0 || seq >= n) continue;
    const int first = bounds[seq + 1];
    const int j = static_cast<int>(ga.parts > 1 || by_row ? x - first : x - int64_t(seq) * ga.far_keys);
    if (j >= bounds[seq + 2] - first || (ga.parts == 1 && j >= ga.far_keys)) continue;
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int p = 0; p < ga.parts; ++p)
      s += *reinterpret_cast<const f32x4*>(ga.part + (p * a.kv * head_rows + r) * 2 * a.hd + col);
    if (j < ga.far_keys) {
      const int64_t at = packed_near_rows(ga) + hk * far_rows + (by_row ? first : int64_t(seq) * ga.far_keys) + j;
      for (int p = 0; p < far_slots(a.hd) * ga.chunks; ++p)
        s += *reinterpret_cast<const f32x4*>(ga.part + (at + p * a.kv * far_rows) * 2 * a.hd + col);
    }
    uint16_t* out = col < a.hd ? ga.dk + hk * ga.dks[1] + (int64_t(first) + j) * ga.dks[2] + col
                               : ga.dv + hk * ga.dvs[1] + (int64_t(first) + j) * ga.dvs[2] + col - a.hd;
    const u32x2 w = {pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3])};
    *reinterpret_cast<u32x2*>(out) = w;
  }
}

// How the gradients of k and v are split, and the floats of `part`: as in a padded batch, with
// the sequences' mean length, which is all that the host knows, for their own.  So is the choice
// of dS in two parts: sequences of up to kFineKeys rows beside long ones have theirs in one, as
// the long ones.  (Both forms in a kernel, by the workgroup's own sequence, spill 20 to 430
// registers; a launch of each would have half of its workgroups leave at once.)
int64_t far_jobs(const AttnGradArgs& a) {
  return a.f.kv * (packed_by_row(a) ? most_items(a.sequences, a.f.lk) * (128 / far_block(a.f.hd)) : int64_t(a.sequences) * far_blocks(a));
}
int64_t near_grid(const AttnGradArgs& a) { return most_items(a.sequences, a.f.lk) * a.parts * a.f.kv; }
int64_t far_grid(const AttnGradArgs& a) { return a.far_keys > 0 ? far_jobs(a) * a.chunks : 0; }

int64_t plan_packed(AttnGradArgs* g) {
  const AttnArgs& a = g->f;
  const int64_t kv = a.kv, n = g->sequences, G = a.heads / a.kv, mean = ceil_div(a.lk, n);
  const int64_t rows = int64_t(a.window) + 127 < mean ? int64_t(a.window) + 127 : mean;
  const int64_t tiles = G * ceil_div(rows, kBN);
  int64_t parts = ceil_div(512, kv * ceil_div(a.lk, 128));
  if (parts > tiles / 8) parts = tiles / 8;
  if (parts < 1 || most_items(n, a.lk) * kv * parts >= 1 << 20) parts = 1;
  g->parts = static_cast<int>(parts);
  const bool far = a.sinks > 0 && a.window < a.lk;
  g->far_keys = far ? (a.sinks < a.lk ? a.sinks : a.lk) : 0;
  g->near_keys = 0;
  g->fine = (int64_t(a.window) + a.sinks < mean ? int64_t(a.window) + a.sinks : mean) <= kFineKeys;
  g->chunks = 0;
  if (far) {
    const int64_t far_tiles = G * ceil_div(a.lk - a.window, kBN);
    const int64_t own = ceil_div(tiles, 4 * parts), most = ceil_div(kFarWork, far_jobs(*g));
    int64_t chunks = ceil_div(far_tiles, own < 8 ? 8 : own);
    chunks = chunks > 64 ? 64 : chunks;
    g->chunks = static_cast<int>(chunks > most ? most : chunks);
  }
  const int64_t near = parts > 1 || far ? packed_near_rows(*g) : 0;
  return 2 * a.hd * (near + far_slots(a.hd) * int64_t(g->chunks) * kv * packed_far_rows(*g));
}

// A launch has under 2^32 threads.
bool packed_ok(const AttnArgs& a, int n) {
  return args_ok(a) && a.b == 1 && a.lq == a.lk && n >= 1 && n < 1 << 24 && most_items(n, a.lk) * a.heads < int64_t(1) << 24;
}
bool grads_fit(const AttnGradArgs& a) {
  return (near_grid(a) + far_grid(a)) * (shared_keys(a.f.hd) ? 512 : 256) < int64_t(1) << 32;
}

template <int HD>
void launch_fwd(const AttnArgs& a, const Plan& plan, const Starts& starts, hipStream_t s) {
  const int grid = static_cast<int>(most_items(starts.n, a.lk) * a.heads);
  if (plan.base == nullptr)
    hipLaunchKernelGGL((k_packed_fwd<HD, true>), dim3(grid), dim3(256), 0, s, a, nullptr, nullptr, starts);
  else
    hipLaunchKernelGGL((k_packed_fwd<HD, false>), dim3(grid), dim3(256), 0, s, a, plan.base, plan.items(), starts);
}

template <int HD, bool FINE>
void launch_grads(const AttnGradArgs& a, const Plan& plan, bool kv, hipStream_t s) {
  const int grid = static_cast<int>(most_items(a.sequences, a.f.lk) * a.f.heads);
  hipLaunchKernelGGL((k_packed_dq<HD, FINE>), dim3(grid), dim3(256), 0, s, a, plan.base, plan.items());
  if (!kv) return;
  const uint32_t near = static_cast<uint32_t>(near_grid(a));
  hipLaunchKernelGGL((k_packed_dkv<HD, FINE>), dim3(near + static_cast<uint32_t>(far_grid(a))), dim3(shared_keys(HD) ? 512 : 256), 0, s, a,
                     plan.base, plan.items(), plan.bounds(), near);
  if (a.parts == 1 && a.far_keys == 0) return;
  const int64_t sums = ceil_div(packed_sum_work(a), 256);
  hipLaunchKernelGGL(k_packed_sum, dim3(static_cast<uint32_t>(sums < kSumGrid ? sums : kSumGrid)), dim3(256), 0, s, a, plan.bounds());
}

template <int HD>
void launch_bwd(const AttnGradArgs& a, const Plan& plan, bool kv, hipStream_t s) {
  if (a.fine) launch_grads<HD, true>(a, plan, kv, s);
  else launch_grads<HD, false>(a, plan, kv, s);
}

}  // namespace
}  // namespace compact

using namespace compact;

extern "C" {

// q, k, v and o as a padded batch of one: (1, heads, T, hd).  plan: 4 + 2 round4(n + 3) + 4
// (T / 128 + min(n + 2, T)) int32, which the backward reads too; NULL where kOwnSequences and kOwnGrid
// allow it.
int compact_packed_fwd(const AttnArgs* a, const void* starts, int starts64, int64_t stride, int n, int32_t* table, void* stream) {
  if (!packed_ok(*a, n)) return -1;
  if (table == nullptr && (n > kOwnSequences || most_items(n, a->lk) * a->heads > kOwnGrid)) return -1;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const Plan plan(table, n);
  const Starts given = {starts, stride, starts64, n};
  if (table != nullptr) hipLaunchKernelGGL(k_packed_plan, dim3(1), dim3(kPlanThreads), 0, s, starts, starts64, stride, n, a->lk, table);
  if (a->hd <= 64) launch_fwd<64>(*a, plan, given, s);
  else if (a->hd <= 96) launch_fwd<96>(*a, plan, given, s);
  else launch_fwd<128>(*a, plan, given, s);
  return status();
}

// The floats of scratch (`part`) that the backward needs; -1: sizes it does not take.
int64_t compact_packed_bwd_scratch(const AttnArgs* a, int n) {
  if (!packed_ok(*a, n)) return -1;
  AttnGradArgs g = {};
  g.f = *a;
  g.sequences = n;
  const int64_t floats = plan_packed(&g);
  return grads_fit(g) ? floats : -1;
}

// dk and dv are left out where dk is NULL.
int compact_packed_bwd(const AttnGradArgs* args, int n, int32_t* table, void* stream) {
  AttnGradArgs a = *args;
  a.sequences = n;
  if (table == nullptr || !packed_ok(a.f, n) || a.f.o_low == nullptr || a.gs[2] < 0 || a.gs[2] > kMaxStride || (a.f.lq > 1 && a.gs[2] < a.f.hd)) return -1;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool kv = a.dk != nullptr;
  const bool parts = plan_packed(&a) > 0;
  if (kv && ((parts && a.part == nullptr) || !grads_fit(a))) return -1;
  const Plan plan(table, n);
  if (a.f.hd <= 64) launch_bwd<64>(a, plan, kv, s);
  else if (a.f.hd <= 96) launch_bwd<96>(a, plan, kv, s);
  else launch_bwd<128>(a, plan, kv, s);
  return status();
}

}  // extern "C"
