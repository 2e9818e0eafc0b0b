// Attention over the 4-bit pages on the 5th-generation tensor cores: tiles of 128 query rows against 128 keys.
//
//     S = Q K^T   128x128x128, both operands in shared memory
//     P = 2^(scale*S - m), masked, a thread a row, half precision, over S in tensor memory
//     O += P V    128x128x128, P from tensor memory, V from shared memory
//
// What is special is where K and V come from.  Bulk copies bring granules (16 tokens, 2176 bytes) of 4-bit codes into a ring;
// eight warps turn them into half-precision tiles in the layout that the tensor core reads (128-byte swizzle).  For bfloat16 rows
// a tile holds scale * (code - 8) + mid, one rounding, an eighth of out's.  For half-precision rows it holds code - 8, and the
// scales and mids are applied in fp32: a score is s * (q . code) + m * sum(q), P is scale * probability (the rows' reference counts the
// tile's largest scale, so that it fits), and the sum of m * probability is added to all channels of O.  One rounding instead of three,
// 3.0e-4 instead of 4.6e-4 of the output (2.1e-4 are out's own), and scores as exact as fp32 is, for 20 % of the time (64 nodes of
// 32/32 heads over a window of 4096: 59 -> 71 us; 72 now).  Eight channels leave a code word in the order 0,4,1,5,2,6,3,7 (two nibbles of a 32-bit word per instruction);
// Q's channels are stored in that order too, and O's columns are put back when the rows are written.  The tree's 16-bit rows go
// through the same warps.
//
// Two groups of 128 threads, a thread a row, have the even and the odd key tiles, three S/P buffers let the next tiles' scores be
// computed meanwhile.  Both add to one accumulator and share the rows' reference maxima, which they settle in the keys' order (see
// the groups).  A group reads a tile's scores twice, 32 at a time, for the maximum and for the exponentials: the second reading costs
// less than the registers and the code that keep them.  While a segment's results are written the next one's Q is in place already
// and its first scores are computed.
//
// What bounds it: instructions, 1700 a scheduler and key tile (600 to unpack K and V, 500 for the 128 x 128 scores, the rest
// waits, hand-overs, the tree's tiles and the segments' ends), of which 0.61 are issued a cycle; and that they have to be in the
// instruction caches: five warps of a scheduler run four different loops.  So loops are rolled and there is one copy of each: a
// third of the code less gave 203 -> 188 us (768 nodes on 4096 tokens of 64/8 heads, 64 us at the tensor cores' rate; 172 now, 163 with the
// same inputs in a graph).
// Without effect or slower, for that reason or another: three groups (182 us against 180), sixteen unpacking warps (185), 16 scores
// at a time (186 against 181), the ancestor words fetched ahead (181 against 171), and two tiles of 128 rows that shared the unpacked keys.
// Faster here and slower there: 16 rows of the tree in flight (these 168 against 171, but 64 nodes of 32/32 heads 63 against 59).
//
// Every mbarrier wait is bounded; one that runs out raises SEQ_DEV_TIMEOUT and the CTA drains.
#include "kv4_attention.cuh"
#include "umma.cuh"

namespace seqtree {

constexpr int kTilesThreads = 640;  // warps: loader, two issuers, one idle; four that unpack K, four V; two groups of four for the rows
constexpr int kUnpackWarp = 4, kGroupWarp = 12, kGroups = 2, kSBufs = 3;
constexpr int kTilesStep = 128;     // keys
constexpr int kRegsIssue = 40, kRegsUnpack = 56, kRegsGroup = 160;  // 128 * 40 + 256 * 56 + 256 * 160 <= 640 * 96
constexpr int kHalfKeys = 64;       // keys of a ring stage
constexpr float kLargestHalf = 65504.f;
constexpr int kStageBytes = kHalfKeys / kGranule * kGranuleBytes;
constexpr int kTreeTiles = SEQ_MAX_TREE / kTilesStep;

constexpr int kParamTiles = 5;  // tiles of scales and mids: one is written again behind the scores that follow its own three tiles later
// What a unit's start and end take, and what a step of the tree takes longer than one of the prefix, in steps.  Chosen on 768 nodes of 64/8 heads on
// 4096 tokens; us in a graph there and on batches of trees with short prefixes, where the constants are near the best but not always it:
//                                             2, 1 (these)   tree 0   tree 2   unit 0   unit 4
//   768 nodes on 4096 tokens, 64/8 heads          162.8       168.8    170.6    164.3    162.9
//   768 nodes on 300 tokens, 64/8 heads            67.7        63.0     76.7     74.1     66.1
//   16 x 64 nodes on 300 tokens, 32/32 heads       49.9        51.3     51.6     52.9     52.5
//   32 x 64 nodes on 100 tokens, 32/32 heads       67.2        65.5     65.2     67.0     66.6
//   16 x 128 nodes on 200 tokens, 40/40 heads      73.5        67.8     74.5     69.8     76.8
constexpr int kUnitCost = 2;
constexpr int kTreeCost = 1;
constexpr uint32_t kTmemS = 128;  // tensor memory: O in columns 0..127, then the S/P buffers

template <bool kExact>
struct TilesSmem {
  static constexpr int kStages = kExact ? 5 : 6;
  uint8_t q[kTileBytes];     // tiles: 1024-byte aligned
  uint8_t k[2][kTileBytes];  // [key tile parity]
  uint8_t v[2][kTileBytes];
  uint8_t ring[kStages][kStageBytes];
  uint64_t raw_full[kStages], raw_empty[kStages];
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2];
  uint64_t q_full;
  uint64_t s_full[kSBufs], p_full[kSBufs], pv_done[kSBufs];
  uint64_t settled[kGroups][4];  // [group][lane quarter]: the reference of the quarter's rows is settled for the group's tile
  uint64_t drained[2];
  float ref[kTileM];             // the rows' reference maximum, handed on in the keys' order
  float sum[kGroups][kTileM];
  uint32_t top[kGroups][kTileM]; // q's largest magnitudes
  uint32_t bad[2][4][kTreeTiles][4];  // [K, V][segment mod 4]: tree rows that are not finite in half precision
  uint32_t tmem_base;
  volatile int abort_flag;
  Kv4Plan plan;
  // exact codes: scales and mids of the tiles' keys and values (two keys' scales, their mids), the largest scale's bits of 32 values, the
  // rows' sums of q, and of mid * probability
  float ref_scale[kExact ? kTileM : 1];  // exact codes: ref is for ref + ref_scale
  float4 key_params[kExact ? kParamTiles : 1][kTilesStep / 2], value_params[kExact ? kParamTiles : 1][kTilesStep / 2];
  int4 largest[kExact ? kParamTiles : 1];
  float q_sum[kExact ? kGroups : 1][kTileM], mids[kExact ? kGroups : 1][kTileM];
};
template <bool kExact>
constexpr size_t kTilesSmemBytes = sizeof(TilesSmem<kExact>) + 1024;
static_assert(kTilesSmemBytes<false> <= 227 * 1024 && kTilesSmemBytes<true> <= 227 * 1024, "one CTA's shared memory");

// mbar_wait, rolled: what the warps run has to stay in the instruction caches
template <typename Smem>
__device__ __forceinline__ bool kv4_wait(Smem* sm, uint64_t* bar, uint32_t parity, int32_t* status) {
#pragma unroll 1
  for (uint32_t it = 0; it < kSpinLimit; ++it) {
    if (mbar_try_wait(bar, parity)) return true;
    if ((it & 1023u) == 1023u && sm->abort_flag) return false;
  }
  sm->abort_flag = 1;
  dev_flag(status, SEQ_DEV_TIMEOUT);
  return false;
}

__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(smem_u32(dst)), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void sts128(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
#define SEQ_R16(a, o) \
  "=r"(a[o]), "=r"(a[o + 1]), "=r"(a[o + 2]), "=r"(a[o + 3]), "=r"(a[o + 4]), "=r"(a[o + 5]), "=r"(a[o + 6]), "=r"(a[o + 7]), "=r"(a[o + 8]), \
  "=r"(a[o + 9]), "=r"(a[o + 10]), "=r"(a[o + 11]), "=r"(a[o + 12]), "=r"(a[o + 13]), "=r"(a[o + 14]), "=r"(a[o + 15])
// Consecutive fp32 columns of this thread's tensor-memory lane, there when it returns
__device__ __forceinline__ void tmem_get16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : SEQ_R16(r, 0) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_get32(uint32_t taddr, uint32_t (&r)[32]) {
  tmem_ld32(taddr, r, 0);
  tc_wait_ld();
#pragma unroll
  for (int e = 0; e < 32; ++e) asm volatile("" : "+r"(r[e]));  // (nothing of it moves ahead of the wait)
}
__device__ __forceinline__ uint32_t bits_below(int x) { return x <= 0 ? 0u : (x >= 32 ? 0xffffffffu : (1u << x) - 1u); }

// The steps of a unit that fall into a CTA's range: none, if that is only what stands for its cost
struct TilesSeg {
  Kv4Unit u;
  int32_t next, t0, steps;  // the next segment's position, first step, how many
  bool whole;
};
__device__ __forceinline__ TilesSeg tiles_seg(const Kv4Plan* plan, const Kv4Args& a, int pos, int range_hi) {
  TilesSeg s;
  s.u = kv4_unit<kTilesStep>(plan, a, pos);
  s.next = min(s.u.end, range_hi);
  s.whole = pos == s.u.begin && s.next == s.u.end;
  s.t0 = max(pos - s.u.work, 0);
  s.steps = max(s.next - s.u.work, 0) - s.t0;
  return s;
}

template <bool kBf16>
__global__ void __launch_bounds__(kTilesThreads, 1) kv4_tiles_kernel(const Kv4Args a) {
  // Half-precision rows: codes enter as they are, see the head.  (For bfloat16 ones out's rounding is 8 times as coarse as a value's.)
  constexpr bool kExact = !kBf16;
  using Smem = TilesSmem<kExact>;
  constexpr int kStages = Smem::kStages;
  extern __shared__ uint8_t smem_raw[];
  Smem* sm = reinterpret_cast<Smem*>(smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u));
  const int warp = uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) { mbar_init(&sm->raw_full[s], 1); mbar_init(&sm->raw_empty[s], 8); }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&sm->k_full[b], 4); mbar_init(&sm->k_empty[b], 1);
      mbar_init(&sm->v_full[b], 4); mbar_init(&sm->v_empty[b], 1);
      mbar_init(&sm->drained[b], 1);
    }
    mbar_init(&sm->q_full, 4 * kGroups);
    for (int b = 0; b < kSBufs; ++b) { mbar_init(&sm->s_full[b], 1); mbar_init(&sm->p_full[b], 4); mbar_init(&sm->pv_done[b], 1); }
    for (int x = 0; x < 4 * kGroups; ++x) mbar_init(&sm->settled[x >> 2][x & 3], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    sm->abort_flag = 0;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (warp == 1) {  // all 512 tensor-memory columns
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&sm->tmem_base)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  kv4_plan<kTilesStep, kTilesThreads>(&sm->plan, a);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = uniform(sm->tmem_base);
  const Kv4Ranges ranges = kv4_ranges(&sm->plan, a);
  const bool works = (int)blockIdx.x < ranges.ctas && ranges.total > 0;
  if (warp == 3 && lane == 0 && (int)blockIdx.x < a.ctas) {
    int4 cut = make_int4(-1, 0, 0, 0);
    if (works) {
      const Kv4Unit u = kv4_unit<kTilesStep>(&sm->plan, a, ranges.lo(blockIdx.x + 1) - 1);
      if (u.begin >= ranges.lo(blockIdx.x) && u.end > ranges.lo(blockIdx.x + 1)) cut = kv4_cut(a, ranges, u);
    }
    a.ws_cut[blockIdx.x] = cut;
  }
  const int range_lo = works ? ranges.lo(blockIdx.x) : 0, range_hi = works ? ranges.lo(blockIdx.x + 1) : 0;

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsIssue));
    if (warp == 0) {
      // ============================ loader: 64 keys a stage ============================
      int issued = 0;
      int r_known = -1, page0 = 0, id = 0;  // lane x holds the number of request r_known's page page0 + x
      bool ok = true;
      for (int pos = range_lo; pos < range_hi && ok;) {
        const TilesSeg sg = tiles_seg(&sm->plan, a, pos, range_hi);
        for (int i = 0; i < sg.steps && ok; ++i) {
          if (sg.t0 + i >= sg.u.prefix.steps) break;  // the tree's
          for (int h = 0; h < 2; ++h) {
            const int key = sg.u.prefix.key_step(sg.t0 + i) * kTilesStep + h * kHalfKeys;
            if (key >= sg.u.L) break;
            const int granules = min(kHalfKeys / kGranule, (sg.u.L - key + kGranule - 1) / kGranule);
            const int st = issued % kStages, w = issued / kStages;
            const int first = key >> a.page_shift, last = (key + granules * kGranule - 1) >> a.page_shift;
            if (r_known != sg.u.r || first < page0 || last >= page0 + 32) {
              r_known = sg.u.r;
              page0 = first;
              const int x = first + lane;
              id = 0;
              if ((int64_t)x * a.page_size < sg.u.L) {
                id = a.table[sg.u.r * a.table_stride + x];
                if ((unsigned)id >= (unsigned)a.num_pages) {
                  dev_flag(a.status, SEQ_DEV_BAD_PAGE);
                  id = 0;
                }
              }
            }
            if (w > 0 && !kv4_wait(sm, &sm->raw_empty[st], (w - 1) & 1, a.status)) { ok = false; break; }
            if (lane == 0) mbar_expect_tx(&sm->raw_full[st], granules * kGranuleBytes);
            __syncwarp();
            // lane x: the x-th page's part
            const int per = min(kHalfKeys, a.page_size) / kGranule;  // granules of a page in the stage
            const int mine = __shfl_sync(0xffffffffu, id, (first - page0 + lane) & 31);
            if (lane * per < granules) {
              const uint8_t* src = a.pages + mine * a.page_stride + (int64_t)sg.u.g * a.page_size * 136 + (key & (a.page_size - 1)) / kGranule * kGranuleBytes;
              bulk_load(sm->ring[st] + lane * per * kGranuleBytes, src, min(per, granules - lane * per) * kGranuleBytes, &sm->raw_full[st]);
            }
            __syncwarp();
            ++issued;
          }
        }
        pos = sg.next;
      }
      // (after a wait that ran out: nobody leaves while a copy into its shared memory is under way)
      if (sm->abort_flag)
        for (int x = max(issued - kStages, 0); x < issued; ++x)
          for (uint32_t it = 0; it < (1u << 16); ++it)
            if (mbar_try_wait(&sm->raw_full[x % kStages], (x / kStages) & 1)) break;
    } else if (warp < 3) {
      // ============================ issuers: S (warp 1), P V (warp 2) ============================
      const uint32_t idesc = (1u << 4) | ((uint32_t)(kTileM >> 4) << 24) | ((uint32_t)(kTilesStep >> 3) << 17);  // fp16, sums fp32, N = 128
      const uint32_t idesc_pv = idesc | (1u << 16);                                                             // V is MN-major
      const uint32_t q_lo = desc_lo(smem_u32(sm->q), 16);
      int step = 0, seg = 0, sb = 0, u = 0;  // key tiles before this segment, segments with steps, the next tile's buffer and how often that was used
      bool ok = true;
      for (int pos = range_lo; pos < range_hi && ok;) {
        const TilesSeg sg = tiles_seg(&sm->plan, a, pos, range_hi);
        if (warp == 1 && sg.steps > 0) ok = kv4_wait(sm, &sm->q_full, seg & 1, a.status);
        for (int i = 0; i < sg.steps && ok; ++i) {
          const int x = step + i, b = x & 1;
          const uint32_t sp = tmem + kTmemS + 128u * sb;
          if (warp == 1) {
            // S goes where the P of three tiles ago was: its product has completed
            ok = kv4_wait(sm, &sm->k_full[b], (x >> 1) & 1, a.status) && (u == 0 || kv4_wait(sm, &sm->pv_done[sb], (u - 1) & 1, a.status));
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
              mma_qk<kHalfBytes, kHalfBytes>(sp, q_lo, desc_lo(smem_u32(sm->k[b]), 16), idesc);
              tc_commit(&sm->s_full[sb]);
              tc_commit(&sm->k_empty[b]);
            }
          } else {
            const uint32_t v_lo = desc_lo(smem_u32(sm->v[b]), kHalfBytes);
            ok = kv4_wait(sm, &sm->v_full[b], (x >> 1) & 1, a.status) && kv4_wait(sm, &sm->p_full[sb], u & 1, a.status);
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {  // (P of each half of the keys is where its scores were)
              mma_pv(tmem, sp, v_lo, idesc_pv, i > 0 ? 1u : 0u);
              mma_pv(tmem, sp + 64u, v_lo + (kHalfKeys * 128 >> 4), idesc_pv, 1u);
              tc_commit(&sm->pv_done[sb]);
              tc_commit(&sm->v_empty[b]);
            }
          }
          __syncwarp();
          if (++sb == kSBufs) { sb = 0; ++u; }
        }
        step += sg.steps;
        seg += sg.steps > 0;
        pos = sg.next;
      }
      if (!ok) {  // what has been issued reads shared and tensor memory
        if (elect_one()) tc_commit(&sm->drained[warp - 1]);
        __syncwarp();
        for (uint32_t it = 0; it < (1u << 16); ++it)
          if (mbar_try_wait(&sm->drained[warp - 1], 0)) break;
      }
    }
  } else if (warp < kGroupWarp) {
    // ============================ codes, and the tree's rows, to half-precision tiles: 32 rows of K or of V a warp ============================
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsUnpack));
    const int which = (warp - kUnpackWarp) >> 2, w4 = warp & 3, quad = lane & 3, r8 = lane >> 2;
    uint64_t* const full = which ? sm->v_full : sm->k_full;
    uint64_t* const empty = which ? sm->v_empty : sm->k_empty;
    int step = 0, taken = 0, seg = 0;  // (segments with steps)
    bool ok = true;
    // A thread's 32 channels of a row are four 16-byte pieces.  Quads 2, 3 write to the tile's second half, 16 KiB on, that is, to the same
    // banks: they go through their pieces in another order.  (A thread's rows are alike modulo 8: the pieces' places are the same.)
    const uint32_t swap = quad >= 2 ? 2u : 0u;
    uint32_t place[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) place[p] = (quad >> 1) * kHalfBytes + r8 * 128 + ((((quad & 1) * 4 + (p ^ swap)) ^ r8) << 4);
    for (int pos = range_lo; pos < range_hi && ok;) {
      const TilesSeg sg = tiles_seg(&sm->plan, a, pos, range_hi);
      for (int i = 0; i < sg.steps && ok; ++i) {
        const int x = step + i, b = x & 1, w = x >> 1, t = sg.t0 + i;
        const bool tree = t >= sg.u.prefix.steps;
        const int key0 = tree ? (t - sg.u.prefix.steps) * kTilesStep : sg.u.prefix.key_step(t) * kTilesStep;
        const int left = (tree ? a.n : sg.u.L) - key0;  // keys of the tile that there are
        if (w > 0) ok = kv4_wait(sm, &empty[b], (w - 1) & 1, a.status);
        const uint32_t tile = smem_u32(which ? sm->v[b] : sm->k[b]);
        const int slot = kExact ? x % kParamTiles : 0;
        uint32_t largest = 0;  // exact codes: the warps of K leave the scales and mids of both, as they are ahead
        if (!tree) {
#pragma unroll 1
          for (int h = 0; h < 2 && ok; ++h) {
            const int st = taken % kStages;
            if (h * kHalfKeys < left) ok = kv4_wait(sm, &sm->raw_full[st], (taken / kStages) & 1, a.status);
            __syncwarp();
            if (!ok) break;
            const uint32_t granule = smem_u32(sm->ring[st]) + w4 * kGranuleBytes;
            uint4 cd[2];
            uint32_t params[2];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              cd[y] = make_uint4(0u, 0u, 0u, 0u);
              params[y] = 0;  // a key behind the prefix: zeros
              if (h * kHalfKeys + w4 * kGranule + 8 * y + r8 < left) {
                asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(cd[y].x), "=r"(cd[y].y), "=r"(cd[y].z), "=r"(cd[y].w)
                             : "r"(granule + which * kGranuleV + (8 * y + r8) * kCodeBytes + quad * 16));
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(params[y]) : "r"(granule + kGranuleParams + which * (kGranule * 4) + (8 * y + r8) * 4));
              }
            }
            if (!kExact) {
              // A row's largest value can be past the largest half (65504 comes back as 65536), and an infinity in a tile of V gets
              // into rows that do not see it: where 8 scale + |mid| is, the scale is cut to what fits, by a step of half's at most.
              const uint32_t most = hfma2_bits(__byte_perm(params[0], params[1], 0x5410) & 0x7fff7fffu, 0x48004800u, __byte_perm(params[0], params[1], 0x7632) & 0x7fff7fffu);
              if (__any_sync(0xffffffffu, (((most & 0x7fff7fffu) + 0x04000400u) & 0x80008000u) != 0)) {
#pragma unroll 1
                for (int y = 0; y < 2; ++y) {
                  const uint32_t one = y == 0 ? params[0] : params[1];
                  const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&one));
                  const __half fits = __float2half_rz(fminf(v.x, fminf((kLargestHalf - v.y) * (1.f / 7.f), (kLargestHalf + v.y) * 0.125f)));
                  const uint32_t now = (one & 0xffff0000u) | __half_as_ushort(fits);
                  if (y == 0) params[0] = now; else params[1] = now;
                }
              }
            }
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const uint32_t scale = __byte_perm(params[y], 0u, 0x1010), mid = __byte_perm(params[y], 0u, 0x3232);
              const uint32_t words[4] = {swap ? cd[y].z : cd[y].x, swap ? cd[y].w : cd[y].y, swap ? cd[y].x : cd[y].z, swap ? cd[y].y : cd[y].w};
              const uint32_t line = tile + (h * kHalfKeys + w4 * kGranule + 8 * y) * 128;
              if (kExact && which == 0) {
                const int key = h * kHalfKeys + w4 * kGranule + 8 * y + r8;
                uint32_t values = 0;
                if (key < left) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(values) : "r"(granule + kGranuleParams + kGranule * 4 + (8 * y + r8) * 4));
                largest = max(largest, values & 0x7fffu);
                const float2 sm2 = __half22float2(*reinterpret_cast<const __half2*>(quad == 0 ? &params[y] : &values));
                float* to = reinterpret_cast<float*>(quad == 0 ? sm->key_params[slot] : sm->value_params[slot]) + 4 * (key >> 1) + (key & 1);
                if (quad < 2) {
                  to[0] = sm2.x;
                  to[2] = sm2.y;
                }
              }
#pragma unroll
              for (int p = 0; p < 4; ++p) {
                uint32_t v[4];
                unpack4(words[p], v);
                if (kExact) sts128(line + place[p], v[0], v[1], v[2], v[3]);
                else sts128(line + place[p], hfma2_bits(v[0], scale, mid), hfma2_bits(v[1], scale, mid), hfma2_bits(v[2], scale, mid), hfma2_bits(v[3], scale, mid));
              }
            }
            if (h * kHalfKeys < left) {
              __syncwarp();
              if (lane == 0) mbar_arrive(&sm->raw_empty[st]);
              ++taken;
            }
          }
        } else if (ok) {
          if (kExact && which == 0) {  // (the tree's rows are what they are)
            largest = 0x3c00u;
            const int at = 4 * (w4 * 16 + (lane >> 1)) + (lane & 1);
            float* to = reinterpret_cast<float*>(sm->key_params[slot]) + at;
            to[0] = 1.f;
            to[2] = 0.f;
            to = reinterpret_cast<float*>(sm->value_params[slot]) + at;
            to[0] = 1.f;
            to[2] = 0.f;
          }
          uint32_t bad = 0;  // of the warp's 32 rows
          const uint8_t* rows = (which ? a.vt : a.kt) + sg.u.r * a.t_req + sg.u.g * a.t_head + quad * 64;
#pragma unroll 1
          for (int y = 0; y < 4; ++y) {
            const int key = w4 * 32 + 8 * y + r8;
            uint4 in[4];
#pragma unroll
            for (int p = 0; p < 4; ++p) {
              in[p] = make_uint4(0u, 0u, 0u, 0u);
              if (key < left) in[p] = reinterpret_cast<const uint4*>(rows + (int64_t)(key0 + key) * a.t_tok)[p ^ swap];
            }
            uint32_t big = 0;
#pragma unroll
            for (int p = 0; p < 4; ++p) {
              if (kBf16) {
                in[p].x = pack2<false>(__uint_as_float(in[p].x << 16), __uint_as_float(in[p].x & 0xffff0000u));
                in[p].y = pack2<false>(__uint_as_float(in[p].y << 16), __uint_as_float(in[p].y & 0xffff0000u));
                in[p].z = pack2<false>(__uint_as_float(in[p].z << 16), __uint_as_float(in[p].z & 0xffff0000u));
                in[p].w = pack2<false>(__uint_as_float(in[p].w << 16), __uint_as_float(in[p].w & 0xffff0000u));
              }
              big = __vmaxu2(__vmaxu2(big, in[p].x & 0x7c007c00u), __vmaxu2(in[p].y & 0x7c007c00u, __vmaxu2(in[p].z & 0x7c007c00u, in[p].w & 0x7c007c00u)));
            }
            // a row that is not finite counts as zeros, so that it stays out of the rows that do not see it; those that do become
            // NaN when they are written.  (A key's infinity could make its score -inf, which is what a hidden key has.)
            uint32_t keep = 0xffffffffu;
            const uint32_t b4 = __ballot_sync(0xffffffffu, (big & 0xffffu) == 0x7c00u || (big >> 16) == 0x7c00u);
            if ((b4 >> (lane & 28)) & 15u) keep = 0u;
            if (b4 != 0)
#pragma unroll 1
              for (int z = 0; z < 8; ++z) bad |= (b4 >> (4 * z)) & 15u ? 1u << (8 * y + z) : 0u;
            const uint32_t line = tile + (w4 * 32 + 8 * y) * 128;
#pragma unroll
            for (int p = 0; p < 4; ++p)
              sts128(line + place[p], __byte_perm(in[p].x, in[p].z, 0x5410) & keep, __byte_perm(in[p].x, in[p].z, 0x7632) & keep,
                     __byte_perm(in[p].y, in[p].w, 0x5410) & keep, __byte_perm(in[p].y, in[p].w, 0x7632) & keep);
          }
          // Four segments' words: the rows look at a segment's when it is through.  The warps of V are two tiles ahead of that at most;
          // those of K two ahead of the scores, which do not go beyond the segment whose q the rows have brought: the next one.
          if (lane == 0) sm->bad[which][seg & 3][key0 / kTilesStep][w4] = bad;
        }
        if (!ok) break;
        if (kExact && which == 0) {
          largest = __reduce_max_sync(0xffffffffu, largest);
          if (lane == 0) reinterpret_cast<int*>(&sm->largest[slot])[w4] = (int)largest;
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&full[b]);
      }
      step += sg.steps;
      seg += sg.steps > 0;
      pos = sg.next;
    }
  } else {
    // ============================ groups: one thread a row ============================
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsGroup));
    const int grp = (warp - kGroupWarp) >> 2;  // even or odd tiles
    const int quarter = warp & 3, row = quarter * 32 + lane;
    const uint32_t lane_sel = (uint32_t)(quarter * 32) << 16;
    const uint32_t tmem_o = tmem + lane_sel;
    auto rows_sync = [&]() { asm volatile("bar.sync 1, 256;" ::: "memory"); };
    int step = 0, seg = 0, own = 0;  // key tiles before this segment, segments with steps, tiles of this group
    bool ok = true;
    // The thread's row of a segment
    struct Row {
      TilesSeg sg;
      int node, h, depth, begin, latest;  // (begin: where the row's window begins)
      float rs, q_sum;
      bool valid, warp_live;              // a warp of padding rows only keeps in step
      const uint32_t* mask;
    };
    Row cur;
    bool have = false;
    float m_used = -INFINITY, m_scale = 0.f, l = 0.f, mids = 0.f;
    for (int pos = range_lo;;) {
      // ---- the next segment's rows; its first scores are computed while the last segment's results are written
      Row next;
      const bool more = pos < range_hi;
      if (more) {
        next.sg = tiles_seg(&sm->plan, a, pos, range_hi);
        const int r = next.sg.u.r, rw = next.sg.u.m * kTileM + row;
        const int node = next.node = min(rw, a.rows - 1) / a.group, h = next.h = next.sg.u.g * a.group + min(rw, a.rows - 1) % a.group;
        const bool valid = next.valid = rw < a.rows;
        next.warp_live = rw - lane < a.rows;
        // q: half precision (a bfloat16 row scaled by a power of two, exactly), channels in the codes' order
        float rs = a.scale_log2;
        if (next.sg.steps > 0) {
          // each group brings every other piece of eight channels
          const uint4* src = reinterpret_cast<const uint4*>(a.q + r * a.q_req + node * a.q_tok + h * a.q_head) + grp;
          uint4 x[8];
#pragma unroll
          for (int p = 0; p < 8; ++p) x[p] = valid ? src[p * kGroups] : make_uint4(0u, 0u, 0u, 0u);
          // The scores of the segment before are complete: its q is read, and, as they took all warps' q, every row is through with what
          // the groups exchanged for it (behind the CTA's first segment no barrier says so, and a group without a tile in it would be ahead).
          if (have && cur.sg.steps > 0) {
            const int x = step - 1, u = x / kSBufs;
            ok = kv4_wait(sm, &sm->s_full[x - u * kSBufs], u & 1, a.status);
            __syncwarp();
          }
          float f = 1.f;
          if (kBf16) {
            uint32_t top = 0;
#pragma unroll
            for (int p = 0; p < 8; ++p) top = __vmaxu2(__vmaxu2(top, __vmaxu2(x[p].x & 0x7fff7fffu, x[p].y & 0x7fff7fffu)), __vmaxu2(x[p].z & 0x7fff7fffu, x[p].w & 0x7fff7fffu));
            sm->top[grp][row] = top = max(top & 0xffffu, top >> 16);
            rows_sync();
            const int e = (int)(max(top, sm->top[grp ^ 1][row]) >> 7);
            if (e > 8 && e < 255) {  // the largest magnitude into [2^8, 2^9)
              const int up = 8 + 127 - e;  // -119..126
              f = __uint_as_float((uint32_t)(127 + up) << 23);
              rs *= __uint_as_float((uint32_t)(127 - up) << 23);
            }
          }
          if (kExact) {
            float sum = 0.f;
#pragma unroll
            for (int p = 0; p < 8; ++p) {
              const uint32_t y[4] = {x[p].x, x[p].y, x[p].z, x[p].w};
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float2 two = __half22float2(*reinterpret_cast<const __half2*>(&y[e]));
                sum += two.x + two.y;
              }
            }
            sm->q_sum[grp][row] = sum;
            rows_sync();
            next.q_sum = sm->q_sum[0][row] + sm->q_sum[1][row];
          }
          const uint32_t line = smem_u32(sm->q) + row * 128;
#pragma unroll
          for (int p = 0; p < 8; ++p) {
            if (kBf16) {
              x[p].x = pack2<false>(__uint_as_float(x[p].x << 16) * f, __uint_as_float(x[p].x & 0xffff0000u) * f);
              x[p].y = pack2<false>(__uint_as_float(x[p].y << 16) * f, __uint_as_float(x[p].y & 0xffff0000u) * f);
              x[p].z = pack2<false>(__uint_as_float(x[p].z << 16) * f, __uint_as_float(x[p].z & 0xffff0000u) * f);
              x[p].w = pack2<false>(__uint_as_float(x[p].w << 16) * f, __uint_as_float(x[p].w & 0xffff0000u) * f);
            }
            sts128(line + (p >> 2) * kHalfBytes + ((((p & 3) * kGroups + grp) ^ (row & 7)) << 4), __byte_perm(x[p].x, x[p].z, 0x5410), __byte_perm(x[p].x, x[p].z, 0x7632),
                   __byte_perm(x[p].y, x[p].w, 0x5410), __byte_perm(x[p].y, x[p].w, 0x7632));
          }
          fence_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(&sm->q_full);
        }
        next.rs = fmaxf(rs, kLeastUnit);
        next.mask = kv4_mask_row(a, r, node);
        next.depth = a.window > 0 ? kv4_depth(a, r, node) : 0;
        next.begin = a.window > 0 ? next.sg.u.L + next.depth + 1 - a.window : 0;
        next.latest = __reduce_max_sync(0xffffffffu, next.begin);
        pos = next.sg.next;
      }
      if (have) {
        const TilesSeg& sg = cur.sg;
        const int L = sg.u.L, r = sg.u.r, node = cur.node, h = cur.h, depth = cur.depth;
        const uint32_t* mask_row = cur.mask;
        const bool valid = cur.valid;
        // ---- the last product.  Its tile may be the other group's, and this one be here before that tile's scores are: the barrier would then
        // still wait for the product of three tiles ago, and its parity look like that of the one after.  The scores come behind that product, so
        // they are waited for: above, where a next segment's q is brought, and here where none is.  (Behind the next q they could be two
        // phases on.)
        if (sg.steps > 0 && ok) {
          const int x = step - 1, u = x / kSBufs;
          if (!more || next.sg.steps == 0) ok = kv4_wait(sm, &sm->s_full[x - u * kSBufs], u & 1, a.status);
          if (ok) ok = kv4_wait(sm, &sm->pv_done[x - u * kSBufs], u & 1, a.status);
        }
        __syncwarp();
        tc_fence_after();
        const bool any = sg.steps > 0 && ok;
        uint32_t poison = 0;  // tree rows that are not finite and that the row sees
#pragma unroll 1
        for (int i = max(sg.u.prefix.steps - sg.t0, 0); i < sg.steps; ++i) {
          const int tt = sg.t0 + i - sg.u.prefix.steps;
#pragma unroll 1
          for (int w = 0; w < 4; ++w) {
            const uint32_t bad = sm->bad[0][(seg - 1) & 3][tt][w] | sm->bad[1][(seg - 1) & 3][tt][w];
            if (bad != 0) poison |= bad & kv4_window_word(a, r, L, depth, 4 * tt + w, kv4_mask_word(a, mask_row, node, 4 * tt + w));
          }
        }
        // ---- the groups' sums, against the reference that O ended in: the last one settled
        const float M = any ? sm->ref[row] : -INFINITY, M_scale = kExact && any ? sm->ref_scale[row] : 0.f;
        const float behind = m_used == -INFINITY ? 0.f : ex2((m_used - M) + (kExact ? m_scale - M_scale : 0.f));
        sm->sum[grp][row] = poison != 0 ? NAN : m_used == -INFINITY ? l : l * behind;
        if (kExact) sm->mids[grp][row] = mids * behind;
        rows_sync();
        const float unit = kExact ? __uint_as_float((uint32_t)(127 + (int)M_scale) << 23) : 1.f;  // (-15..16: what a piece leaves is for M)
        const float own_sum = sm->sum[0][row] + sm->sum[1][row], sum = own_sum * unit;
        const float all_mids = kExact ? (sm->mids[0][row] + sm->mids[1][row]) * unit : 0.f;
        const float inv = 1.f / sum;
        const int64_t mine = (int64_t)kv4_slot(ranges, blockIdx.x, sg.u.begin) * kTileM;
#pragma unroll 1
        for (int c = grp; c < 4; c += kGroups) {  // 32 columns
          uint32_t o[32];
          tmem_get32(tmem_o + 32u * c, o);
          if (kExact) {
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(fmaf(__uint_as_float(o[e]), unit, all_mids));
          }
          if (!sg.whole) {  // a piece, unnormalised
            uint4* to = reinterpret_cast<uint4*>(a.ws_o + mine * kHeadDim) + 8 * c * kTileM + row;  // [channel / 4][row]
#pragma unroll
            for (int e = 0; e < 32; e += 4) to[(e >> 2) * kTileM] = any ? make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]) : make_uint4(0u, 0u, 0u, 0u);
          } else if (valid) {
            uint8_t* out = a.out + r * a.o_req + node * a.o_tok + h * a.o_head + 64 * c;
#pragma unroll
            for (int e = 0; e < 32; e += 8) {  // columns 0,2,4,6,1,3,5,7 are channels 0..7
              float y[8];
#pragma unroll
              for (int z = 0; z < 8; ++z) y[z] = __uint_as_float(o[e + z]) * inv;
              *reinterpret_cast<uint4*>(out + 2 * e) =
                  make_uint4(pack2<kBf16>(y[0], y[2]), pack2<kBf16>(y[4], y[6]), pack2<kBf16>(y[1], y[3]), pack2<kBf16>(y[5], y[7]));
            }
          }
          __syncwarp();
        }
        tc_fence_before();
        rows_sync();  // the accumulator is read, the rows are through with what they exchanged
        if (grp == 0) {
          if (!sg.whole) a.ws_ml[mine + row] = make_float2(M, sum);
          else if (valid && a.lse != nullptr) a.lse[((int64_t)r * a.Hq + h) * a.n + node] = (M + log2f(sum)) * kLn2;
        }
      }
      if (!more) break;
      cur = next;
      have = true;
      const TilesSeg& sg = cur.sg;
      const int L = sg.u.L, r = sg.u.r, node = cur.node, depth = cur.depth, begin = cur.begin, latest = cur.latest;
      const uint32_t* mask_row = cur.mask;
      const float rs = cur.rs;
      const bool warp_live = cur.warp_live;
      m_used = -INFINITY;
      m_scale = l = mids = 0.f;
      for (int i = (grp ^ step) & 1; i < sg.steps; i += kGroups, ++own) {
        const int t = sg.t0 + i, x = step + i, u = x / kSBufs, sb = x - u * kSBufs;
        const uint32_t tmem_s = tmem + kTmemS + 128u * sb + lane_sel;
        const int slot = kExact ? x % kParamTiles : 0;
        const bool tree = t >= sg.u.prefix.steps;
        const int key0 = (tree ? t - sg.u.prefix.steps : sg.u.prefix.key_step(t)) * kTilesStep;
        const bool masked = tree || key0 + kTilesStep > L || key0 < latest;  // some keys are not there, or not every row's
        auto hide = [&](int c, uint32_t (&s)[32]) {  // masked scores become -inf
          const int k = key0 + 32 * c;
          uint32_t bits;
          if (tree) bits = kv4_window_word(a, r, L, depth, k >> 5, kv4_mask_word(a, mask_row, node, k >> 5));
          else bits = bits_below(L - k) & (~bits_below(begin - k) | bits_below(a.sinks - k));
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (!((bits >> e) & 1u)) s[e] = __float_as_uint(-INFINITY);
        };
        ok = kv4_wait(sm, &sm->s_full[sb], u & 1, a.status);
        __syncwarp();
        if (!ok) break;
        if (warp_live) {
          tc_fence_after();
          uint32_t s[32];
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll 1
          for (int c = 0; c < 4; ++c) {
            tmem_get32(tmem_s + 32u * c, s);
            if (kExact) {
              const uint64_t q_sum2 = pair_of(cur.q_sum, cur.q_sum);
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const float4 kp = sm->key_params[slot][16 * c + e];
                float y0, y1;
                unpair(fma2(pair_of(__uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1])), pair_of(kp.x, kp.y), mul2(pair_of(kp.z, kp.w), q_sum2)), y0, y1);
                s[2 * e] = __float_as_uint(y0);
                s[2 * e + 1] = __float_as_uint(y1);
              }
            }
            if (masked) hide(c, s);
            if (masked || kExact) tmem_st32(tmem_s + 32u * c, s, 0);
#pragma unroll
            for (int e = 0; e < 32; e += 2) mx[(e >> 1) & 3] = max3(mx[(e >> 1) & 3], __uint_as_float(s[e]), __uint_as_float(s[e + 1]));
          }
          if (masked || kExact) tc_wait_st();
          float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * rs;  // rs > 0
          // Scale * probability is what is rounded: the reference counts the tile's largest scale, apart from the scores where their last bits
          // are too coarse for it.
          float top_scale = 0.f;
          if (kExact) {
            const int4 big = sm->largest[slot];
            top_scale = (float)((max(max(big.x, big.y), max(big.z, big.w)) >> 10) - 15);
            if (!(fabsf(top) > kWideScore)) {
              top += top_scale;
              top_scale = 0.f;
            }
          }
          // All groups add to one accumulator, so they share the rows' reference: it is settled tile by tile, in order, before the
          // exponentials.  It moves only when a score exceeds it by more than the threshold, or with the first score.
          float ref = -INFINITY, ref_scale = 0.f;
          if (i > 0) {
            ok = kv4_wait(sm, &sm->settled[grp ^ 1][quarter], (own - (grp == 0)) & 1, a.status);
            __syncwarp();
            if (!ok) break;
            ref = sm->ref[row];
            if (kExact) ref_scale = sm->ref_scale[row];
          }
          const float above = (top - ref) + (kExact ? top_scale - ref_scale : 0.f);
          const bool move = above > kRescaleThreshold;  // (of two that are -inf: NaN)
          const float now = move ? top : ref, now_scale = move ? top_scale : ref_scale;
          if (__any_sync(0xffffffffu, move) || i == 0) {
            const float alpha = move && ref != -INFINITY ? ex2(-above) : 1.f;
            if (i > 0) {
              // O may still be taking the tile before
              ok = kv4_wait(sm, &sm->pv_done[sb == 0 ? kSBufs - 1 : sb - 1], (u - (sb == 0)) & 1, a.status);
              __syncwarp();
              if (!ok) break;
              tc_fence_after();
#pragma unroll 1
              for (int x8 = 0; x8 < 8; ++x8) {
                uint32_t o[16];
                tmem_get16(tmem_o + 16u * x8, o);
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
                tmem_st16(tmem_o + 16u * x8, o);
              }
              tc_wait_st();
              tc_fence_before();
            }
            sm->ref[row] = now;
            if (kExact) sm->ref_scale[row] = now_scale;
            __syncwarp();
          }
          if (lane == 0) mbar_arrive(&sm->settled[grp][quarter]);
          if (now != m_used || (kExact && now_scale != m_scale)) {
            const float f = m_used == -INFINITY ? 0.f : ex2((m_used - now) + (kExact ? m_scale - now_scale : 0.f));
            l *= f;
            mids *= f;
            m_used = now;
            m_scale = now_scale;
          }
          const float neg_m = now == -INFINITY ? 0.f : -now;
          const bool wide = __any_sync(0xffffffffu, fabsf(neg_m) > kWideScore);
          const float less = wide ? -now_scale : neg_m;  // (not wide: no scale apart)
          const uint64_t rs2 = pair_of(rs, rs), unit2 = wide ? pair_of(1.f, 1.f) : rs2, less2 = pair_of(less, less);
          if (wide) {  // scores in units of 1, less the reference.  (A packed product and sum would be made one operation by the assembler.)
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
              tmem_get32(tmem_s + 32u * c, s);
#pragma unroll
              for (int e = 0; e < 32; ++e) s[e] = __float_as_uint(__fadd_rn(__fmul_rn(__uint_as_float(s[e]), rs), neg_m));
              tmem_st32(tmem_s + 32u * c, s, 0);
            }
            tc_wait_st();
          }
          uint64_t sums[2] = {pair_of(0.f, 0.f), pair_of(0.f, 0.f)}, mids2 = pair_of(0.f, 0.f);
#pragma unroll 1
          for (int c = 0; c < 4; ++c) {
            tmem_get32(tmem_s + 32u * c, s);
            uint32_t packed[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              float y0, y1;
              unpair(fma2(pair_of(__uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1])), unit2, less2), y0, y1);
              float p0 = ex2(y0), p1 = ex2(y1);
              sums[e & 1] = add2(sums[e & 1], pair_of(p0, p1));
              if (kExact) {
                const float4 vp = sm->value_params[slot][16 * c + e];
                const uint64_t p = pair_of(p0, p1);
                mids2 = fma2(p, pair_of(vp.z, vp.w), mids2);
                unpair(mul2(p, pair_of(vp.x, vp.y)), p0, p1);
              }
              packed[e] = pack2<false>(p0, p1);
            }
            tmem_st16(tmem_s + 64u * (c >> 1) + 16u * (c & 1), packed);  // over scores that have been read
          }
          float s0, s1, s2, s3;
          unpair(sums[0], s0, s1);
          unpair(sums[1], s2, s3);
          l += (s0 + s1) + (s2 + s3);
          if (kExact) {
            unpair(mids2, s0, s1);
            mids += s0 + s1;
          }
          tc_wait_st();
          tc_fence_before();
        } else if (lane == 0) {
          mbar_arrive(&sm->settled[grp][quarter]);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm->p_full[sb]);
      }
      step += sg.steps;
      seg += sg.steps > 0;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

// ---------------------------------------------------------------- host side ---------------------
size_t kv4_tiles_workspace_bytes() {
  const size_t sms = device_sm_count();
  return kv4_ranges_bytes(sms, kTileM);
}

int launch_kv4_tiles(const seq_tree_kv4_attention_params& p, cudaStream_t stream) {
  const int sms = device_sm_count();
  Kv4Args a = kv4_args(p, kTileM, kTilesStep, kUnitCost, kTreeCost);
  a.min_steps = 2 + kUnitCost;
  const int64_t most = (int64_t)a.batch * a.Hkv * a.tiles * ((p.max_len + kTilesStep - 1) / kTilesStep + 1 + a.unit_cost + kv4_tree_positions(a, a.tree_steps));
  if (most > 0x7fffffff) return SEQ_ERR_UNSUPPORTED;
  const int64_t want = (most + a.min_steps - 1) / a.min_steps;
  a.ctas = want < sms ? (int)want : sms;
  kv4_ranges_place(a, sms, p.workspace);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(a.ctas);
  cfg.blockDim = dim3(kTilesThreads);
  cfg.stream = stream;
  cudaLaunchAttribute early[1];
  early[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = early;
  cfg.numAttrs = 1;
  auto launch = [&](auto kernel, int which, size_t smem) -> int {
    static int done[2][64];
    const int rc = once_per_device(done[which], [&]() -> int {
      SEQ_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
      return SEQ_OK;
    });
    if (rc != SEQ_OK) return rc;
    cfg.dynamicSmemBytes = smem;
    SEQ_CUDA_OK(cudaLaunchKernelEx(&cfg, kernel, a));
    return SEQ_OK;
  };
  const bool bf16 = p.dtype == SEQ_BF16;
  const int rc = bf16 ? launch(kv4_tiles_kernel<true>, 0, kTilesSmemBytes<false>) : launch(kv4_tiles_kernel<false>, 1, kTilesSmemBytes<true>);
  return rc != SEQ_OK ? rc : launch_kv4_merge(a, bf16, true, stream);
}

}  // namespace seqtree
