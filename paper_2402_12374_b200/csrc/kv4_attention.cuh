// What the kernels of seq_tree_kv4_attention share: their arguments, how the work is laid out and cut, and the pieces that
// CTAs leave for one another.
//
// A unit is (request, kv head, tile of query rows); a row is a (node, head in group) pair.  A unit's keys come in steps: those of the prefix that
// some row can see (the sinks, then the window: the steps in between are left out), then the tree's.  The steps of all
// units are laid end to end and cut into equal ranges, one a CTA, whatever lengths the requests have.  A unit inside one range is
// finished there; the pieces of one that is cut go to the workspace, and a second kernel adds them, in the order of their CTAs.
#pragma once

#include "kv4.cuh"

namespace seqtree {

// A score's unit at the least, the smallest normal number: hidden scores, -inf, times zero would be NaN.  (Sums of products are below
// 2^9 * 65504 * 128: what units below it stand for rounds to zero.)
constexpr float kLeastUnit = 1.17549435e-38f;
// A score less the reference is one fused operation, whose product is not rounded, while the reference is a rounded one: the largest
// exponent is off by up to 2^-24 of its score, and beyond 2^31 no probability would be left, or all be infinite.  Scores beyond this are
// rounded first.
constexpr float kWideScore = 4194304.f;
constexpr int kKv4TreeSteps = SEQ_MAX_TREE / 32;  // steps of the tree, at most

struct Kv4Args {
  int32_t batch, n, max_len, Hq, Hkv, group, rows;  // rows: n * group
  int32_t window, sinks;
  int32_t num_pages, page_size, page_shift;
  int32_t row_tile, tiles, ctas, min_steps, cluster;
  int32_t unit_cost;   // positions at a unit's start that stand for what a unit costs,
  int32_t tree_cost;   // ... and as many for each of its steps of the tree, for what these take longer
  int32_t tree_steps;  // of the last tile of rows; a tile has those up to its last node
  int32_t tree_from[kKv4TreeSteps];  // the first tile with more than k steps of the tree
  int32_t tree_total;  // positions of all tiles' steps of the tree, with what they take longer
  const uint8_t* q; int64_t q_req, q_tok, q_head;  // all strides in bytes
  const uint8_t* kt; const uint8_t* vt; int64_t t_req, t_tok, t_head;
  const uint8_t* pages; int64_t page_stride;
  const int32_t* table; int64_t table_stride;
  const int32_t* lengths;
  const uint32_t* mask; int32_t mask_wpr; int64_t mask_req;
  uint8_t* out; int64_t o_req, o_tok, o_head;
  float* lse;
  int4* ws_cut;       // [ctas] the unit that begins in the CTA's range and is cut: (unit or -1, its first piece's slot, its last CTA)
  float2* ws_ml;      // [2 * ctas][row_tile] (m, l): reference maximum (log2 units) and sum of a piece
  float* ws_o;        // [2 * ctas][row_tile][128] its unnormalised rows
  float scale_log2;
  int32_t* status;
};

struct Kv4Plan {
  int32_t start[SEQ_MAX_BATCH + 1];  // steps before each request's
  int32_t warp_sum[32];
};

// The prefix steps of kStep keys that a request's rows can see: step t holds the keys from key_step(t) * kStep on.
struct Kv4Prefix {
  int32_t steps, split, gap;
  __device__ __forceinline__ int key_step(int t) const { return t < split ? t : t + gap; }
};
template <int kStep>
__device__ __forceinline__ Kv4Prefix kv4_prefix(const Kv4Args& a, int L) {
  const int all = (L + kStep - 1) / kStep;
  if (a.window == 0) return {all, all, 0};
  const int first = max(0, L + 1 - a.window);  // what the root's window begins with; a deeper node's begins later
  const int sink_steps = (min(a.sinks, L) + kStep - 1) / kStep, window_step = first / kStep;
  if (window_step <= sink_steps) return {all, all, 0};
  return {sink_steps + max(all - window_step, 0), sink_steps, window_step - sink_steps};
}

// Request r's prefix; -1: idle
__device__ __forceinline__ int kv4_len(const Kv4Args& a, int r) { return min(max(a.lengths[r], -1), a.max_len); }

__host__ __device__ __forceinline__ int kv4_tree_positions(const Kv4Args& a, int steps) { return steps * (1 + a.tree_cost); }

// Positions of a request
template <int kStep>
__device__ __forceinline__ int kv4_positions(const Kv4Args& a, int L) { return a.Hkv * (a.tiles * (a.unit_cost + kv4_prefix<kStep>(a, L).steps) + a.tree_total); }

// Every thread of the CTA calls it; the plan is there behind the next barrier that it ends with.
template <int kStep, int kThreads>
__device__ __forceinline__ void kv4_plan(Kv4Plan* plan, const Kv4Args& a) {
  const int per = (a.batch + kThreads - 1) / kThreads, first = threadIdx.x * per;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int sum = 0;
  for (int j = first; j < first + per && j < a.batch; ++j) {
    const int L = kv4_len(a, j);
    if (blockIdx.x == 0 && a.lengths[j] > a.max_len) dev_flag(a.status, SEQ_DEV_BAD_LENGTH);
    if (L >= 0) sum += kv4_positions<kStep>(a, L);
  }
  int incl = sum;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, incl, d);
    if (lane >= d) incl += v;
  }
  if (lane == 31) plan->warp_sum[warp] = incl;
  __syncthreads();
  int at = incl - sum;
  for (int w = 0; w < warp; ++w) at += plan->warp_sum[w];
  for (int j = first; j < first + per && j < a.batch; ++j) {
    plan->start[j] = at;
    const int L = kv4_len(a, j);
    if (L >= 0) at += kv4_positions<kStep>(a, L);
    if (j == a.batch - 1) plan->start[a.batch] = at;
  }
  __syncthreads();
}

// The ranges: no more than one for every min_steps steps.
struct Kv4Ranges {
  int32_t total, ctas, base, extra;  // base positions each, one more in the first `extra`
  __device__ __forceinline__ int lo(int c) const { return c * base + min(c, extra); }
  __device__ __forceinline__ int at(int pos) const {  // the CTA that has pos
    const int longer = extra * (base + 1);
    return pos < longer ? pos / (base + 1) : extra + (pos - longer) / base;
  }
};
__device__ __forceinline__ Kv4Ranges kv4_ranges(const Kv4Plan* plan, const Kv4Args& a) {
  const int total = plan->start[a.batch], ctas = max(1, min(a.ctas, (total + a.min_steps - 1) / a.min_steps));
  return {total, ctas, total / ctas, total % ctas};
}

struct Kv4Unit {
  int32_t r, g, m, L;
  int32_t begin, work, end;  // positions: what stands for costs, the steps
  Kv4Prefix prefix;
};
template <int kStep>
__device__ __forceinline__ Kv4Unit kv4_unit(const Kv4Plan* plan, const Kv4Args& a, int pos) {
  int lo = 0, hi = a.batch - 1;  // the last request that starts at or before pos and has steps
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (plan->start[mid] <= pos) lo = mid; else hi = mid - 1;
  }
  Kv4Unit u;
  u.r = lo;
  u.L = max(kv4_len(a, lo), 0);
  u.prefix = kv4_prefix<kStep>(a, u.L);
  const int fixed = a.unit_cost + u.prefix.steps, head = a.tiles * fixed + a.tree_total;
  int rem = pos - plan->start[lo];
  u.g = rem / head;
  rem -= u.g * head;
  // tiles [tree_from[k], tree_from[k + 1]) have k + 1 steps of the tree
  int k = 0, at = 0;
#pragma unroll 1
  for (; k + 1 < a.tree_steps; ++k) {
    const int next = at + (a.tree_from[k + 1] - a.tree_from[k]) * (fixed + kv4_tree_positions(a, k + 1));
    if (rem < next) break;
    at = next;
  }
  const int steps = fixed + kv4_tree_positions(a, k + 1), x = (rem - at) / steps;
  u.m = a.tree_from[k] + x;
  u.begin = pos - (rem - at - x * steps);
  u.end = u.begin + steps;
  u.work = u.end - (k + 1) - u.prefix.steps;
  return u;
}
// Where CTA c leaves its piece of a unit that begins at `begin`: the piece that opens its range, or the one that closes it.
__device__ __forceinline__ int kv4_slot(const Kv4Ranges& ranges, int c, int begin) { return 2 * c + (begin <= ranges.lo(c) ? 0 : 1); }

// The unit that a CTA's last segment begins and that goes on behind its range (the merge's later pieces are in slots 2 c)
__device__ __forceinline__ int4 kv4_cut(const Kv4Args& a, const Kv4Ranges& ranges, const Kv4Unit& u) {
  return make_int4((u.r * a.Hkv + u.g) * a.tiles + u.m, kv4_slot(ranges, blockIdx.x, u.begin), ranges.at(u.end - 1), 0);
}

__device__ __forceinline__ const uint32_t* kv4_mask_row(const Kv4Args& a, int r, int node) {
  return a.mask != nullptr ? a.mask + r * a.mask_req + (int64_t)node * a.mask_wpr : nullptr;
}
// Bits of the tree rows [32 w, 32 w + 32) that `node` sees, the window aside
__device__ __forceinline__ uint32_t kv4_mask_word(const Kv4Args& a, const uint32_t* row, int node, int w) {
  const int left = a.n - 32 * w;
  if (left <= 0) return 0u;
  uint32_t bits;
  if (row != nullptr) bits = row[w];
  else bits = node >= 32 * w + 31 ? 0xffffffffu : (node < 32 * w ? 0u : (2u << (node - 32 * w)) - 1u);
  return left < 32 ? bits & ((1u << left) - 1u) : bits;
}
__device__ __forceinline__ int kv4_depth(const Kv4Args& a, int r, int node) {
  const uint32_t* row = kv4_mask_row(a, r, node);
  if (row == nullptr) return node;
  int c = 0;
#pragma unroll 1
  for (int w = 0; w < (a.n + 31) >> 5; ++w) c += __popc(kv4_mask_word(a, row, node, w));
  return max(c - 1, 0);
}
// ... with the window: rows a of the tree at L + depth(a)
__device__ __forceinline__ uint32_t kv4_window_word(const Kv4Args& a, int r, int L, int depth, int w, uint32_t bits) {
  if (a.window == 0 || depth < a.window) return bits;  // (no ancestor is further away than the root)
#pragma unroll 1
  for (uint32_t left = bits; left != 0; left &= left - 1) {
    const int b = __ffs(left) - 1, d = kv4_depth(a, r, 32 * w + b);
    if (d <= depth - a.window && L + d >= a.sinks) bits &= ~(1u << b);
  }
  return bits;
}

// Whether the kernel for few rows takes it
bool kv4_few_rows(const seq_tree_kv4_attention_params& p);
size_t kv4_rows_workspace_bytes(const seq_tree_kv4_attention_params& p);
int launch_kv4_rows(const seq_tree_kv4_attention_params& p, cudaStream_t stream);
size_t kv4_tiles_workspace_bytes();
int launch_kv4_tiles(const seq_tree_kv4_attention_params& p, cudaStream_t stream);
// Arguments, for tiles of so many query rows and steps of so many keys of the tree
Kv4Args kv4_args(const seq_tree_kv4_attention_params& p, int row_tile, int step, int unit_cost, int tree_cost);
// Adds the pieces of the units that are cut.  tiles: which kernel left them.
int launch_kv4_merge(const Kv4Args& a, bool bf16, bool tiles, cudaStream_t stream);
// The workspace's parts: ws_o, ws_ml, ws_cut
inline size_t kv4_ranges_bytes(size_t ctas, size_t row_tile) { return ctas * (2 * row_tile * (kHeadDim * sizeof(float) + sizeof(float2)) + sizeof(int4)); }
inline void kv4_ranges_place(Kv4Args& a, size_t ctas, void* workspace) {
  a.ws_o = static_cast<float*>(workspace);
  a.ws_ml = reinterpret_cast<float2*>(a.ws_o + 2 * ctas * a.row_tile * kHeadDim);
  a.ws_cut = reinterpret_cast<int4*>(a.ws_ml + 2 * ctas * a.row_tile);
}

}  // namespace seqtree
