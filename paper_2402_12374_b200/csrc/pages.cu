// seq_tree_pages_resize, _fork, _compact: the page tables of a paged cache (include/seq_tree.h states what they do).
//
// Which page goes where is a chain of counts over all slots and all pages, so one cluster of up to 16 CTAs plans a call: each CTA
// owns a share of the pages, counts its free (or held) ones, reads the other CTAs' counts from their shared memory, and
// from then on knows the number of every page in its share among all of them.  No order of atomics enters a result: counts
// are sums, and a page's rank says who gets it.  What is only moved - rows of the table, contents of pages - goes over the
// whole device: further clusters of the planning launch copy the table's rows, a second launch behind it the pages.
// Bound by latency for small states (a plan is four exchanges across the cluster), by HBM where pages move.
#include "common.cuh"

namespace seqtree {

constexpr int kPlanCtas = 16;           // CTAs that plan, at most
constexpr int kPagesPerCta = 4096;      // ... one for each so many pages
constexpr int kPlanThreads = 1024;
constexpr int kMoveThreads = 256;
constexpr int kInFlight = 16;  // loads of a lane before the first is used
constexpr int kSlotsPerThread = SEQ_MAX_SLOTS / kPlanThreads;

struct PagesArgs {
  int32_t slots, max_pages, num_pages, page_size;
  const int32_t* table; int64_t table_stride;
  const int32_t* count; const int32_t* refs; const int32_t* lengths;
  int32_t* table_out; int64_t table_out_stride;
  int32_t* count_out; int32_t* refs_out; int32_t* lengths_out;
  const int32_t* tokens; const int32_t* source;
  int32_t* live;
  int32_t* ws;  // resize: free pages in order; fork, compact: [0] how many pages move, then from[], to[] (fork: slots each, compact: num_pages each), map[num_pages] (compact)
  int32_t* status;
};

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
// Also orders the CTAs' global memory accesses: what one wrote before it, every other one reads behind it.
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ int peer_word(const int* p, uint32_t cta) {
  uint32_t at;
  int v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(cta));
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}

struct PlanSmem {
  int32_t before[SEQ_MAX_SLOTS + 1];  // pages that the slots before need
  int32_t source[SEQ_MAX_SLOTS];      // fork: a slot's source, -1 for none, and the source's length
  int32_t length[SEQ_MAX_SLOTS];      // (resize: the pages a slot holds)
  int32_t warp_sum[kPlanThreads / 32];
  int32_t total;
  int32_t mine;  // what this CTA counted; read by the others
  int32_t base, all;
};

// Exclusive sum of v over the CTA's threads; sm->total is the sum of all.  All threads call it.
__device__ __forceinline__ int block_scan(PlanSmem* sm, int v) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int incl = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, incl, d);
    if (lane >= d) incl += u;
  }
  __syncthreads();  // (the last scan's results are out of use)
  if (lane == 31) sm->warp_sum[warp] = incl;
  __syncthreads();
  if (warp == 0) {
    const int s = sm->warp_sum[lane];
    int t = s;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, t, d);
      if (lane >= d) t += u;
    }
    sm->warp_sum[lane] = t - s;
    if (lane == 31) sm->total = t;
  }
  __syncthreads();
  return sm->warp_sum[warp] + incl - v;
}

// The CTAs' counts `mine` become sm->base (those of the CTAs before this one) and sm->all.
__device__ __forceinline__ void cluster_count(PlanSmem* sm, uint32_t rank, int mine) {
  if (threadIdx.x == 0) sm->mine = mine;
  cluster_sync();
  if (threadIdx.x < 32) {
    const int v = threadIdx.x < cluster_size() ? peer_word(&sm->mine, threadIdx.x) : 0;
    const int before = __reduce_add_sync(0xffffffffu, threadIdx.x < rank ? v : 0);
    const int all = __reduce_add_sync(0xffffffffu, v);
    if (threadIdx.x == 0) { sm->base = before; sm->all = all; }
  }
  cluster_sync();  // (nobody's count is read any more)
}

// The slot whose pages hold number k: the last with before[slot] <= k
__device__ __forceinline__ int slot_of(const PlanSmem* sm, int slots, int k) {
  int lo = 0, hi = slots - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (sm->before[mid] <= k) lo = mid; else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ int ceil_pages(int tokens, int page_size) { return tokens / page_size + (tokens % page_size != 0); }

// One CTA's share of the pages, a multiple of four (16-byte loads; only the last share's end is ragged)
struct Share { int lo, hi; };
__device__ __forceinline__ Share share_of(int num_pages, uint32_t rank) {
  const int ctas = cluster_size(), per = ((num_pages + ctas - 1) / ctas + 3) & ~3;
  const int64_t lo = (int64_t)per * rank;
  return {(int)min(lo, (int64_t)num_pages), (int)min(lo + per, (int64_t)num_pages)};
}

// Entries of slot r's row that are its own; all of them where its count cannot be: such a row stays as it is.
__device__ __forceinline__ int held_of(const PagesArgs& a, int r, bool tell) {
  const int have = a.count[r];
  if (have >= 0 && have <= a.max_pages) return have;
  if (tell) dev_flag(a.status, SEQ_DEV_BAD_SLOT);
  return a.max_pages;
}

// How slot r is resized: pages before and after
__device__ __forceinline__ bool wanted_of(const PagesArgs& a, int r, int& have, int& want, bool tell) {
  have = want = held_of(a, r, tell);
  if (have != a.count[r]) return false;
  const int t = a.tokens[r];
  if (t < 0) return false;
  const int w = ceil_pages(t, a.page_size);
  if (w > a.max_pages) {
    if (tell) dev_flag(a.status, SEQ_DEV_BAD_SLOT);
    return false;
  }
  want = w;
  return true;
}

// Slot r's source if it becomes a fork, else -1
__device__ __forceinline__ int fork_source(const PagesArgs& a, int r, bool tell) {
  const int s = a.source[r];
  if (s < 0) return -1;
  int ok = s < a.slots && s != r && a.count[r] == 0;
  if (ok) {
    const int n = a.lengths[s], have = a.count[s];
    ok = n >= 0 && have >= 0 && have <= a.max_pages && ceil_pages(n, a.page_size) <= have;
  }
  if (!ok && tell) dev_flag(a.status, SEQ_DEV_BAD_SLOT);
  return ok ? s : -1;
}

// Rows of a table that is not written in place, by the clusters behind the planning one: a warp a row.  `Mode` 0 resize: the
// plan writes what lies between the old and the new count.  1 fork: rows of slots that do not become forks.
template <int kMode>
__device__ void copy_rows(const PagesArgs& a) {
  const int lane = threadIdx.x & 31;
  const int ctas = gridDim.x - cluster_size(), cta = blockIdx.x - cluster_size();  // (a slot's neighbours go to other CTAs)
  for (int r = (threadIdx.x >> 5) * ctas + cta; r < a.slots; r += ctas * (kPlanThreads / 32)) {
    int have, want;
    if (kMode == 0) {
      wanted_of(a, r, have, want, false);
    } else {
      if (fork_source(a, r, false) >= 0) continue;
      have = want = held_of(a, r, false);
    }
    const int keep = min(have, want), end = max(have, want);
    const int32_t* from = a.table + r * a.table_stride;
    int32_t* to = a.table_out + r * a.table_out_stride;
    for (int i0 = lane; i0 < keep; i0 += 32 * kInFlight) {
      int v[kInFlight];
#pragma unroll
      for (int y = 0; y < kInFlight; ++y) v[y] = i0 + 32 * y < keep ? from[i0 + 32 * y] : 0;
#pragma unroll
      for (int y = 0; y < kInFlight; ++y)
        if (i0 + 32 * y < keep) to[i0 + 32 * y] = v[y];
    }
    for (int i = end + lane; i < a.max_pages; i += 32) to[i] = -1;
  }
}

// The reference counts of this CTA's share into the output
__device__ __forceinline__ void copy_refs(const PagesArgs& a, Share s) {
  if (a.refs == a.refs_out) return;
  if (((reinterpret_cast<uintptr_t>(a.refs) | reinterpret_cast<uintptr_t>(a.refs_out)) & 15) == 0) {
    const int n4 = (s.hi - s.lo) >> 2;
    const int4* from = reinterpret_cast<const int4*>(a.refs + s.lo);
    int4* to = reinterpret_cast<int4*>(a.refs_out + s.lo);
    for (int i0 = threadIdx.x; i0 < n4; i0 += 8 * kPlanThreads) {
      int4 v[8];
#pragma unroll
      for (int y = 0; y < 8; ++y)
        if (i0 + y * kPlanThreads < n4) v[y] = from[i0 + y * kPlanThreads];
#pragma unroll
      for (int y = 0; y < 8; ++y)
        if (i0 + y * kPlanThreads < n4) to[i0 + y * kPlanThreads] = v[y];
    }
    for (int i = s.lo + 4 * n4 + threadIdx.x; i < s.hi; i += kPlanThreads) a.refs_out[i] = a.refs[i];
  } else {
    for (int i = s.lo + threadIdx.x; i < s.hi; i += kPlanThreads) a.refs_out[i] = a.refs[i];
  }
}

// Calls visit(i, v) for a warp's run of pages [lo, hi): a lane has four neighbours i .. i + 3 at a time (i >= hi
// for lanes behind the end), v their counts.  Four loads of a lane are in flight before the first is used.
template <typename Visit>
__device__ __forceinline__ void for_run(const int32_t* refs, int lo, int hi, Visit visit) {
  constexpr int kBatch = 4;
  const int lane = threadIdx.x & 31;
  const bool aligned = ((reinterpret_cast<uintptr_t>(refs) | (uintptr_t)lo << 2) & 15) == 0;  // (i - lo is a multiple of four)
  for (int i0 = lo; i0 < hi; i0 += 128 * kBatch) {
    int4 v[kBatch];
#pragma unroll
    for (int y = 0; y < kBatch; ++y) {
      const int i = i0 + 128 * y + 4 * lane;
      v[y] = make_int4(0, 0, 0, 0);
      if (aligned && i + 4 <= hi) {
        v[y] = __ldcg(reinterpret_cast<const int4*>(refs + i));
      } else {
        if (i < hi) v[y].x = __ldcg(refs + i);
        if (i + 1 < hi) v[y].y = __ldcg(refs + i + 1);
        if (i + 2 < hi) v[y].z = __ldcg(refs + i + 2);
        if (i + 3 < hi) v[y].w = __ldcg(refs + i + 3);
      }
    }
#pragma unroll
    for (int y = 0; y < kBatch; ++y)
      if (i0 + 128 * y < hi) visit(i0 + 128 * y + 4 * lane, v[y]);
  }
}

// Calls take(number, page) for the pages of this CTA's share that chosen(page, refs[page]) holds for: their numbers among all CTAs',
// in order, below `limit`.  A warp has a run of neighbours; a lane's pages, four at a time, have numbers in a row.
template <typename Chosen, typename Take>
__device__ __forceinline__ void number_pages(PlanSmem* sm, uint32_t rank, Share s, const int32_t* refs, int limit, Chosen chosen, Take take, int& total) {
  const int warps = kPlanThreads / 32, lane = threadIdx.x & 31;
  const int per = ((s.hi - s.lo + warps - 1) / warps + 3) & ~3;
  const int lo = min(s.lo + (int)(threadIdx.x >> 5) * per, s.hi), hi = min(lo + per, s.hi);
  auto bits = [&](int i, int4 v) -> int {
    return (int)(i < hi && chosen(i, v.x)) | (int)(i + 1 < hi && chosen(i + 1, v.y)) << 1 | (int)(i + 2 < hi && chosen(i + 2, v.z)) << 2 |
           (int)(i + 3 < hi && chosen(i + 3, v.w)) << 3;
  };
  // (what was chosen is kept where 64 bits hold it: up to 2048 pages a warp)
  int mine = 0, turn = 0;
  uint64_t kept = 0;
  for_run(refs, lo, hi, [&](int i, int4 v) {
    const int b = bits(i, v);
    mine += __popc(b);
    kept |= turn < 16 ? (uint64_t)b << (4 * turn) : 0ull;
    ++turn;
  });
  const int before = block_scan(sm, mine);
  cluster_count(sm, rank, sm->total);
  total = sm->all;
  int at = sm->base + __shfl_sync(0xffffffffu, before, 0);  // of the warp's first page
  const int found = __reduce_add_sync(0xffffffffu, mine);
  if (found == 0 || at >= limit) return;
  auto number = [&](int i, int b) {
    const int n = __popc(b);
    int incl = n;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += u;
    }
    int k = at + incl - n;
    at += __shfl_sync(0xffffffffu, incl, 31);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if ((b >> e) & 1) {
        if (k < limit) take(k, i + e);
        ++k;
      }
  };
  if (turn <= 16) {
    for (int y = 0; y < turn; ++y) number(lo + 128 * y + 4 * lane, (int)(kept >> (4 * y)) & 15);
  } else {
    for_run(refs, lo, hi, [&](int i, int4 v) { number(i, bits(i, v)); });
  }
}

__global__ void __launch_bounds__(kPlanThreads, 1) pages_resize_kernel(const PagesArgs a) {
  __shared__ PlanSmem smem;
  PlanSmem* sm = &smem;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (blockIdx.x >= cluster_size()) {
    copy_rows<0>(a);
    return;
  }
  const uint32_t rank = cluster_rank();
  const Share share = share_of(a.num_pages, rank);
  copy_refs(a, share);
  cluster_sync();

  // What is given up.  A warp a slot.
  const int lane = threadIdx.x & 31;
  const uint32_t ctas = cluster_size();
  for (int r = (threadIdx.x >> 5) * ctas + rank; r < a.slots; r += ctas * (kPlanThreads / 32)) {
    int have, want;
    wanted_of(a, r, have, want, lane == 0);
    const int32_t* row = a.table + r * a.table_stride;
    int32_t* out = a.table_out + r * a.table_out_stride;
    for (int i0 = want + lane; i0 < have; i0 += 32 * kInFlight) {
      int page[kInFlight];
#pragma unroll
      for (int y = 0; y < kInFlight; ++y) page[y] = i0 + 32 * y < have ? row[i0 + 32 * y] : 0;
#pragma unroll
      for (int y = 0; y < kInFlight; ++y) {
        if (i0 + 32 * y >= have) break;
        out[i0 + 32 * y] = -1;
        if (page[y] < 0 || page[y] >= a.num_pages) dev_flag(a.status, SEQ_DEV_BAD_PAGE);
        else atomicSub(a.refs_out + page[y], 1);
      }
    }
  }
  // Meanwhile, every CTA for itself: how many pages the slots before each one need
  const int first = threadIdx.x * kSlotsPerThread;
  int need[kSlotsPerThread], sum = 0;
#pragma unroll
  for (int j = 0; j < kSlotsPerThread; ++j) {
    int have, want;
    need[j] = 0;
    if (first + j < a.slots) {
      wanted_of(a, first + j, have, want, false);
      need[j] = max(want - have, 0);
      sm->length[first + j] = have;  // (kept: in place, the counts change below)
    }
    sum += need[j];
  }
  int at = block_scan(sm, sum);
#pragma unroll
  for (int j = 0; j < kSlotsPerThread; ++j) {
    if (first + j < a.slots) sm->before[first + j] = at;
    at += need[j];
  }
  if (threadIdx.x == 0) sm->before[a.slots] = sm->total;
  cluster_sync();

  // The free pages, lowest first: number k goes to the slot whose growth holds it, if that fits as a whole.
  const int needed = sm->before[a.slots];
  int free_pages = 0;
  const auto is_free = [&](int page, int v) -> bool {
    if (v < 0) {  // a reference too many was given up
      dev_flag(a.status, SEQ_DEV_BAD_SLOT);
      a.refs_out[page] = 0;
    }
    return v <= 0;
  };
  number_pages(sm, rank, share, a.refs_out, needed, is_free, [&](int k, int page) { a.ws[k] = page; }, free_pages);
  cluster_sync();  // the list is there
  for (int k = rank * kPlanThreads + threadIdx.x; k < min(needed, free_pages); k += ctas * kPlanThreads) {
    const int r = slot_of(sm, a.slots, k);
    if (sm->before[r + 1] > free_pages) continue;
    const int page = __ldcg(a.ws + k);
    a.table_out[r * a.table_out_stride + sm->length[r] + k - sm->before[r]] = page;
    a.refs_out[page] = 1;
  }
  // the slots' counts, and what is not there for those that do not grow
  for (int r = rank * kPlanThreads + threadIdx.x; r < a.slots; r += ctas * kPlanThreads) {
    int have, want;
    wanted_of(a, r, have, want, false);
    const bool grows = want > have;
    const bool fits = !grows || sm->before[r + 1] <= free_pages;
    if (!fits) {
      dev_flag(a.status, SEQ_DEV_NO_PAGES);
      for (int i = have; i < want; ++i) a.table_out[r * a.table_out_stride + i] = -1;
    }
    const int was = a.count[r], c = have != was ? was : fits ? want : have;
    if (a.count_out != a.count || c != was) a.count_out[r] = c;
  }
}

__global__ void __launch_bounds__(kPlanThreads, 1) pages_fork_kernel(const PagesArgs a) {
  __shared__ PlanSmem smem;
  PlanSmem* sm = &smem;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (blockIdx.x >= cluster_size()) {
    copy_rows<1>(a);
    return;
  }
  const uint32_t rank = cluster_rank();
  const Share share = share_of(a.num_pages, rank);
  copy_refs(a, share);
  const int first = threadIdx.x * kSlotsPerThread;
  int need[kSlotsPerThread], sum = 0;
#pragma unroll
  for (int j = 0; j < kSlotsPerThread; ++j) {
    need[j] = 0;
    if (first + j < a.slots) {
      held_of(a, first + j, rank == 0);
      const int s = fork_source(a, first + j, rank == 0);
      const int n = s >= 0 ? a.lengths[s] : 0;
      sm->source[first + j] = s;  // (kept: in place, counts and lengths change below)
      sm->length[first + j] = n;
      need[j] = n % a.page_size != 0;
    }
    sum += need[j];
  }
  int at = block_scan(sm, sum);
#pragma unroll
  for (int j = 0; j < kSlotsPerThread; ++j) {
    if (first + j < a.slots) sm->before[first + j] = at;
    at += need[j];
  }
  if (threadIdx.x == 0) sm->before[a.slots] = sm->total;
  cluster_sync();

  const int needed = sm->before[a.slots];
  int32_t* from = a.ws + 1;
  int32_t* to = from + a.slots;
  const uint32_t ctas = cluster_size();
  int free_pages = 0;
  // The open pages that are copied: asked for here, looked at below
  int open[kSlotsPerThread];
#pragma unroll
  for (int j = 0; j < kSlotsPerThread; ++j) {
    const int k = (j * ctas + rank) * kPlanThreads + threadIdx.x;
    open[j] = -1;
    if (k < needed) {
      const int r = slot_of(sm, a.slots, k);
      open[j] = a.table[sm->source[r] * a.table_stride + sm->length[r] / a.page_size];
    }
  }
  const auto give = [&](int k, int page) {
    const int r = slot_of(sm, a.slots, k);
    to[k] = page;
    a.table_out[r * a.table_out_stride + sm->length[r] / a.page_size] = page;
  };
  const auto is_free = [&](int page, int v) -> bool {
    if (v < 0) {
      dev_flag(a.status, SEQ_DEV_BAD_SLOT);
      a.refs_out[page] = 0;
    }
    return v <= 0;
  };
  number_pages(sm, rank, share, a.refs_out, needed, is_free, give, free_pages);
  const int given = min(needed, free_pages);
  if (rank == 0 && threadIdx.x == 0) a.ws[0] = given;
#pragma unroll
  for (int j = 0; j < kSlotsPerThread; ++j) {
    const int k = (j * ctas + rank) * kPlanThreads + threadIdx.x;
    if (k >= given) continue;
    int page = open[j];
    if (page < 0 || page >= a.num_pages) {
      dev_flag(a.status, SEQ_DEV_BAD_PAGE);
      page = -1;
    } else if (__ldcg(a.refs_out + page) <= 0) {  // held, but counted as free: it may be written in this call
      dev_flag(a.status, SEQ_DEV_BAD_SLOT);
      page = -1;
    }
    from[k] = page;  // (-1: nothing is copied)
  }
  cluster_sync();  // every free page is numbered: from here on counts change
  // The forks' rows, a warp each.  (The pages of their own are counted by the launch that fills them: what is counted here, references to
  // pages that are shared, finds 0 where a page is held but counted as free, whatever runs first.)
  const int lane = threadIdx.x & 31;
  for (int r = (threadIdx.x >> 5) * ctas + rank; r < a.slots; r += ctas * (kPlanThreads / 32)) {
    const int s = sm->source[r], n = sm->length[r];
    const bool copied = sm->before[r + 1] > sm->before[r];
    const bool fits = s >= 0 && (!copied || sm->before[r + 1] <= free_pages);
    if (s >= 0) {
      const int full = fits ? n / a.page_size : 0, held = fits ? full + copied : 0;
      int32_t* row = a.table_out + r * a.table_out_stride;
      const int32_t* from_row = a.table + s * a.table_stride;
      for (int i0 = lane; i0 < full; i0 += 32 * kInFlight) {
        int page[kInFlight];
#pragma unroll
        for (int y = 0; y < kInFlight; ++y) page[y] = i0 + 32 * y < full ? from_row[i0 + 32 * y] : 0;
#pragma unroll
        for (int y = 0; y < kInFlight; ++y) {
          if (i0 + 32 * y >= full) break;
          const bool good = page[y] >= 0 && page[y] < a.num_pages;
          row[i0 + 32 * y] = good ? page[y] : -1;
          if (!good) dev_flag(a.status, SEQ_DEV_BAD_PAGE);
          else if (atomicAdd(a.refs_out + page[y], 1) <= 0) dev_flag(a.status, SEQ_DEV_BAD_SLOT);
        }
      }
      for (int i = held + lane; i < a.max_pages; i += 32) row[i] = -1;
      if (!fits && lane == 0) dev_flag(a.status, SEQ_DEV_NO_PAGES);
      if (lane == 0) {
        if (fits || a.count_out != a.count) a.count_out[r] = held;
        if (fits) a.lengths_out[r] = n;
        else if (a.lengths_out != a.lengths) a.lengths_out[r] = a.lengths[r];
      }
    } else if (lane == 0) {
      if (a.count_out != a.count) a.count_out[r] = a.count[r];
      if (a.lengths_out != a.lengths) a.lengths_out[r] = a.lengths[r];
    }
  }
}

__global__ void __launch_bounds__(kPlanThreads, 1) pages_compact_kernel(const PagesArgs a) {
  __shared__ PlanSmem smem;
  PlanSmem* sm = &smem;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const uint32_t rank = cluster_rank();
  const Share share = share_of(a.num_pages, rank);
  int32_t* from = a.ws + 1;
  int32_t* to = from + a.num_pages;
  int32_t* map = to + a.num_pages;
  int mine = 0;
  for (int i = share.lo + threadIdx.x; i < share.hi; i += kPlanThreads) {
    const int v = a.refs[i];
    mine += v > 0;
    if (v < 0) dev_flag(a.status, SEQ_DEV_BAD_SLOT);
  }
  block_scan(sm, mine);
  cluster_count(sm, rank, sm->total);
  const int live = sm->all;
  // far = held pages from `live` on, holes = free ones below it: as many of the one as of the other
  const Share below = {min(share.lo, live), min(share.hi, live)}, above = {max(share.lo, live), max(share.hi, live)};
  int holes = 0, far = 0;
  number_pages(sm, rank, share, a.refs, 0x7fffffff, [&](int page, int v) { return page < live && v <= 0; }, [&](int k, int page) { to[k] = page; }, holes);
  number_pages(sm, rank, share, a.refs, 0x7fffffff, [&](int page, int v) { return page >= live && v > 0; }, [&](int k, int page) { from[k] = page; }, far);
  if (rank == 0 && threadIdx.x == 0) {
    a.ws[0] = far;
    if (a.live != nullptr) *a.live = live;
  }
  cluster_sync();  // both lists are there
  // Where each held page is found (the table is rewritten by it), and the counts.  A page that moves is written by the holder
  // of its number in the lists, the others by the holder of their share.
  for (int i = below.lo + threadIdx.x; i < below.hi; i += kPlanThreads) {
    const int v = a.refs[i];
    map[i] = v > 0 ? i : -1;
    if (a.refs_out != a.refs && v > 0) a.refs_out[i] = v;
  }
  for (int i = above.lo + threadIdx.x; i < above.hi; i += kPlanThreads)
    if (a.refs[i] <= 0) {
      map[i] = -1;
      if (a.refs_out != a.refs || a.refs[i] < 0) a.refs_out[i] = 0;
    }
  cluster_sync();  // (in place: what is moved below was free above)
  for (int k = rank * kPlanThreads + threadIdx.x; k < far; k += cluster_size() * kPlanThreads) {
    const int p = __ldcg(from + k), q = __ldcg(to + k);
    const int v = a.refs[p];
    map[p] = q;
    a.refs_out[q] = v;
    a.refs_out[p] = 0;
  }
}

struct MoveArgs {
  const int32_t* list;  // [0] how many, then from[stride], to[stride]
  int32_t list_stride, num_pages;
  uint8_t* pages; int32_t planes; int64_t plane_stride, page_stride; int32_t chunks;  // pieces of a plane's page
  int64_t page_bytes;
  int32_t* refs;  // where the pages that are filled get a reference (fork)
  // the table, rewritten by `map` where there is one
  const int32_t* map; int32_t slots, max_pages;
  const int32_t* table; int64_t table_stride; const int32_t* count;
  int32_t* table_out; int64_t table_out_stride;
  int32_t* status;
};

constexpr int kMoveUnroll = 8;
constexpr int kMoveChunk = kMoveThreads * kMoveUnroll * 16;  // bytes a CTA moves at a time

__global__ void __launch_bounds__(kMoveThreads) pages_move_kernel(const MoveArgs a) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (a.map != nullptr) {
    for (int r = blockIdx.x; r < a.slots; r += gridDim.x) {
      const int have = a.count[r];
      const bool bad = have < 0 || have > a.max_pages;
      if (bad && threadIdx.x == 0) dev_flag(a.status, SEQ_DEV_BAD_SLOT);
      if (bad && a.table == a.table_out) continue;
      for (int i = threadIdx.x; i < a.max_pages; i += kMoveThreads) {
        if (i >= have && a.table == a.table_out) break;
        int page = -1;
        if (bad) {  // such a row stays as it is
          page = a.table[r * a.table_stride + i];
        } else if (i < have) {
          page = a.table[r * a.table_stride + i];
          if (page < 0 || page >= a.num_pages) {
            dev_flag(a.status, SEQ_DEV_BAD_PAGE);
            page = -1;
          } else {
            page = a.map[page];
            if (page < 0) dev_flag(a.status, SEQ_DEV_BAD_SLOT);  // held, but counted as free
          }
        }
        a.table_out[r * a.table_out_stride + i] = page;
      }
    }
  }
  const int64_t per_page = (int64_t)a.planes * a.chunks;
  const int64_t total = a.list[0] * per_page;
  for (int64_t w = blockIdx.x; w < total; w += gridDim.x) {
    const int k = (int)(w / per_page);
    const int rest = (int)(w - k * per_page), x = rest / a.chunks, c = rest - x * a.chunks;
    const int src = a.list[1 + k], dst = a.list[1 + a.list_stride + k];
    if (a.refs != nullptr && rest == 0 && threadIdx.x == 0) atomicAdd(a.refs + dst, 1);
    if (src < 0) continue;
    const int64_t at = (int64_t)c * kMoveChunk + threadIdx.x * 16;
    const uint8_t* from = a.pages + src * a.page_stride + x * a.plane_stride + at;
    uint8_t* to = a.pages + dst * a.page_stride + x * a.plane_stride + at;
    const int64_t left = a.page_bytes - at;
    uint4 v[kMoveUnroll];
#pragma unroll
    for (int u = 0; u < kMoveUnroll; ++u)
      if (u * kMoveThreads * 16 < left) v[u] = __ldcs(reinterpret_cast<const uint4*>(from + u * kMoveThreads * 16));
#pragma unroll
    for (int u = 0; u < kMoveUnroll; ++u)
      if (u * kMoveThreads * 16 < left) __stcs(reinterpret_cast<uint4*>(to + u * kMoveThreads * 16), v[u]);
  }
}

// ---------------------------------------------------------------- host side ---------------------
static int check_pages(const seq_tree_pages_params* p) {
  if (p == nullptr || p->page_table == nullptr || p->page_count == nullptr || p->ref_count == nullptr || p->table_out == nullptr ||
      p->refs_out == nullptr)
    return SEQ_ERR_INVALID_ARG;
  if (p->slots < 1 || p->slots > SEQ_MAX_SLOTS || p->max_pages < 1 || p->max_pages >= (1 << 30) || p->num_pages < 1 || p->num_pages >= (1 << 30) ||
      p->table_stride < p->max_pages || p->table_out_stride < p->max_pages)
    return SEQ_ERR_INVALID_ARG;
  if ((int64_t)p->slots * p->max_pages > 0x7fffffff) return SEQ_ERR_INVALID_ARG;  // what slots need is summed in 32 bits
  // all arrays in place, or none: what copies rows of the one reads the others while the plan writes them
  const bool in_place = p->table_out == p->page_table;
  if (in_place != (p->refs_out == p->ref_count) || (in_place && p->table_out_stride != p->table_stride)) return SEQ_ERR_INVALID_ARG;
  return SEQ_OK;
}
static int check_pool(const seq_tree_pages_params* p) {
  if (p->pages == nullptr || reinterpret_cast<uintptr_t>(p->pages) % 16 != 0 || p->num_planes < 1) return SEQ_ERR_INVALID_ARG;
  if (p->page_bytes < 16 || p->page_bytes % 16 != 0 || p->page_stride_bytes < p->page_bytes || p->page_stride_bytes % 16 != 0) return SEQ_ERR_INVALID_ARG;
  if (p->num_planes > 1 && (p->plane_stride_bytes < p->page_bytes || p->plane_stride_bytes % 16 != 0)) return SEQ_ERR_INVALID_ARG;
  if (p->page_bytes / kMoveChunk > (1 << 24) || p->num_planes * (p->page_bytes / kMoveChunk + 1) > 0x7fffffff) return SEQ_ERR_INVALID_ARG;
  return SEQ_OK;
}
static int check_workspace(const seq_tree_pages_params* p) {
  if (p->workspace == nullptr || p->workspace_bytes < seq_tree_pages_workspace_bytes(p)) return SEQ_ERR_WORKSPACE;
  return reinterpret_cast<uintptr_t>(p->workspace) % 16 != 0 ? SEQ_ERR_INVALID_ARG : SEQ_OK;
}

static PagesArgs pages_args(const seq_tree_pages_params* p) {
  PagesArgs a;
  a.slots = p->slots; a.max_pages = p->max_pages; a.num_pages = p->num_pages; a.page_size = p->page_size;
  a.table = p->page_table; a.table_stride = p->table_stride; a.count = p->page_count; a.refs = p->ref_count; a.lengths = p->lengths;
  a.table_out = p->table_out; a.table_out_stride = p->table_out_stride;
  a.count_out = p->count_out; a.refs_out = p->refs_out; a.lengths_out = p->lengths_out;
  a.tokens = p->tokens; a.source = p->source; a.live = p->live;
  a.ws = static_cast<int32_t*>(p->workspace); a.status = p->dev_status;
  return a;
}

// CTAs of a planning cluster at most: kPlanCtas where the device can place such a cluster (a partition may not have as many SMs side by side), the
// portable 8 otherwise.  `known` keeps the answer per device.
template <typename Kernel>
static int most_plan_ctas(Kernel kernel, int* known) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 8;
  int most = __atomic_load_n(&known[dev], __ATOMIC_ACQUIRE);
  if (most == 0) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(kPlanCtas);
    cfg.blockDim = dim3(kPlanThreads);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = kPlanCtas; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int clusters = 0;
    most = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
           cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg) == cudaSuccess && clusters > 0 ? kPlanCtas : 8;
    if (most != kPlanCtas) cudaGetLastError();
    __atomic_store_n(&known[dev], most, __ATOMIC_RELEASE);
  }
  return most;
}

template <typename Kernel>
static int launch_plan(Kernel kernel, int* known, const seq_tree_pages_params* p, bool rows_are_copied, void* stream) {
  const int most = most_plan_ctas(kernel, known);
  // A cluster plans: a CTA for every kPagesPerCta pages or table entries (exchanges between CTAs cost more than a few loads), a power of two.
  int ctas = 1;
  const int64_t entries = (int64_t)p->slots * p->max_pages;
  while (ctas < most && (int64_t)ctas * kPagesPerCta < (p->num_pages > entries ? p->num_pages : entries)) ctas *= 2;
  // CTAs that copy the table, in clusters of the same size: one for every 8 Ki entries, up to 96
  int copiers = 0;
  if (rows_are_copied) {
    const int64_t want = (entries + 8191) / 8192;
    copiers = (int)((want < 96 ? want : 96) + ctas - 1) / ctas;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas * (1 + copiers));
  cfg.blockDim = dim3(kPlanThreads);
  cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = ctas; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  SEQ_CUDA_OK(cudaLaunchKernelEx(&cfg, kernel, pages_args(p)));
  return SEQ_OK;
}

static int launch_move(const seq_tree_pages_params* p, int list_stride, int32_t* refs, const int32_t* map, int64_t most_pages, void* stream) {
  MoveArgs a;
  a.list = static_cast<const int32_t*>(p->workspace); a.list_stride = list_stride; a.num_pages = p->num_pages;
  a.pages = static_cast<uint8_t*>(p->pages); a.planes = p->num_planes; a.plane_stride = p->plane_stride_bytes; a.page_stride = p->page_stride_bytes;
  a.chunks = (int)((p->page_bytes + kMoveChunk - 1) / kMoveChunk);
  a.page_bytes = p->page_bytes;
  a.refs = refs;
  a.map = map; a.slots = p->slots; a.max_pages = p->max_pages;
  a.table = p->page_table; a.table_stride = p->table_stride; a.count = p->page_count;
  a.table_out = p->table_out; a.table_out_stride = p->table_out_stride;
  a.status = p->dev_status;
  int64_t want = most_pages * a.planes * a.chunks;
  if (map != nullptr && want < p->slots) want = p->slots;
  const int64_t cap = (int64_t)device_sm_count() * 8;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(want < cap ? want : cap));
  cfg.blockDim = dim3(kMoveThreads);
  cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute early[1];
  early[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = early;
  cfg.numAttrs = 1;
  SEQ_CUDA_OK(cudaLaunchKernelEx(&cfg, pages_move_kernel, a));
  return SEQ_OK;
}

}  // namespace seqtree

using namespace seqtree;

extern "C" size_t seq_tree_pages_workspace_bytes(const seq_tree_pages_params* p) {
  if (p == nullptr || p->slots < 1 || p->num_pages < 1) return 0;
  const size_t fork = 1 + 2 * (size_t)p->slots, compact = 1 + 3 * (size_t)p->num_pages;
  return (fork > compact ? fork : compact) * sizeof(int32_t);
}

extern "C" int seq_tree_pages_resize(const seq_tree_pages_params* p, void* stream) {
  int rc = check_pages(p);
  if (rc != SEQ_OK) return rc;
  if (p->tokens == nullptr || p->count_out == nullptr || p->page_size < 1) return SEQ_ERR_INVALID_ARG;
  if ((p->count_out == p->page_count) != (p->table_out == p->page_table)) return SEQ_ERR_INVALID_ARG;
  rc = check_workspace(p);
  if (rc != SEQ_OK) return rc;
  static int known[64];
  return launch_plan(pages_resize_kernel, known, p, p->table_out != p->page_table, stream);
}

extern "C" int seq_tree_pages_fork(const seq_tree_pages_params* p, void* stream) {
  int rc = check_pages(p);
  if (rc != SEQ_OK) return rc;
  if (p->source == nullptr || p->lengths == nullptr || p->lengths_out == nullptr || p->count_out == nullptr || p->page_size < 1) return SEQ_ERR_INVALID_ARG;
  const bool in_place = p->table_out == p->page_table;
  if ((p->count_out == p->page_count) != in_place || (p->lengths_out == p->lengths) != in_place) return SEQ_ERR_INVALID_ARG;
  rc = check_pool(p);
  if (rc == SEQ_OK) rc = check_workspace(p);
  if (rc != SEQ_OK) return rc;
  static int known[64];
  rc = launch_plan(pages_fork_kernel, known, p, p->table_out != p->page_table, stream);
  if (rc != SEQ_OK) return rc;
  return launch_move(p, p->slots, p->refs_out, nullptr, p->slots, stream);
}

extern "C" int seq_tree_pages_compact(const seq_tree_pages_params* p, void* stream) {
  int rc = check_pages(p);
  if (rc != SEQ_OK) return rc;
  rc = check_pool(p);
  if (rc == SEQ_OK) rc = check_workspace(p);
  if (rc != SEQ_OK) return rc;
  static int known[64];
  rc = launch_plan(pages_compact_kernel, known, p, false, stream);
  if (rc != SEQ_OK) return rc;
  const int32_t* map = static_cast<const int32_t*>(p->workspace) + 1 + 2 * (size_t)p->num_pages;
  return launch_move(p, p->num_pages, nullptr, map, p->num_pages, stream);
}
