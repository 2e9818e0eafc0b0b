// Attention over the 4-bit pages for few query rows: the codes go from shared memory into mma fragments in registers.
//
// A warp works on 32 keys at a time, S^T = K Q^T with the keys in the 16-row operand and 8 query rows in the 8-column one, so that
// a single token's eight grouped heads fill the tile.  What bounds such a kernel before HBM does is instructions, so codes are not
// converted at all: four bits at the bottom of a half-precision word are the subnormal number code * 2^-24, four bits above
// them code * 2^-20, and the tensor core takes subnormals exactly.  One AND makes two operand values, a shift serves four.
//     S^T  keys x rows:     A = codes of K; q's channels that meet codes of 2^-20 are sixteen times smaller.  With s, m a key's scale and mid,
//                           s * (q . code) + (m - 8 s) * sum(q) is put together in fp32.
//     O^T  channels x rows: A = V^T, codes as they are (ldmatrix transposes 16-bit units, four channels of a key); B = P^T, a
//                           movmatrix of S^T's layout, P = s * probability in half precision; m * probability and -8 P are summed beside it.
// Scales are divided by a power of two not far from the largest met so far, so that P neither overflows nor becomes subnormal.
// Each warp has a ring of steps in shared memory, filled by bulk copies (granules are contiguous in a page), its own maxima and
// sums, and takes every fourth step of the CTA's range; the four meet at the end of each unit.
//
// Two ways to cut the work.  Few units: a cluster of CTAs each, which meet in shared memory, one launch without a workspace.  Many:
// the ranges of kv4_attention.cuh, equal whatever the requests' lengths are.
//
// What bounds it: HBM while it streams (6.0 of 6.5 TB/s: 17.8 us for each 107 MB), and 17 us of a call with ranges that are the start (lengths, plan,
// page numbers and the first codes are loads that wait for one another), the pieces and the kernel that adds them: 32 requests of 4096 to
// 8192 tokens, 32/8 heads, in 53 us.  A single token on 500 of one request takes 6.0 us, a launch's latency and one meeting of a cluster.
// Three stages of 32 keys a warp: more of them, or 64 keys, cost the registers or the shared memory of a third CTA on an SM (89 us then).
#include "kv4_attention.cuh"
#include "umma.cuh"

namespace seqtree {

constexpr int kRowsWarps = 4;
constexpr int kTreeStep = 32;  // rows of the tree in a step
constexpr int kRowsCluster = 8;  // CTAs of a cluster, at most
constexpr float kNoRef = -3e38f;  // a row that has seen no key yet

constexpr int kKeys = 32;    // of a step
constexpr int kStages = 3;
constexpr int kBytes = kKeys / kGranule * kGranuleBytes;

template <int NT>
struct RowsSmem {
  uint8_t ring[kRowsWarps][kStages][kBytes];
  float o[kRowsWarps][8 * NT][kHeadDim + 4];
  float2 ml[kRowsWarps][8 * NT];
  uint64_t full[kRowsWarps][kStages];
  volatile int abort_flag;
  int32_t begin[8 * NT];  // where the rows' windows begin
  Kv4Plan plan;
};

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ uint32_t lds32(uint32_t at) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ uint4 lds128(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void mma16816(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// eight 8x8 blocks of 16-bit units in two instructions: thread (g, t) gets unit g of rows 2t, 2t + 1, transposed
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t at, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
// 16-bit pairs as half precision pairs
template <bool kBf16>
__device__ __forceinline__ uint32_t to_half2(uint32_t x) {
  if (!kBf16) return x;
  return pack2<false>(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
}
// channels (0,4), (1,5), (2,6), (3,7) of eight: the order that a code word's come in
__device__ __forceinline__ void pairs_of_8(uint4 x, uint32_t* out) {
  out[0] = __byte_perm(x.x, x.z, 0x5410);
  out[1] = __byte_perm(x.x, x.z, 0x7632);
  out[2] = __byte_perm(x.y, x.w, 0x5410);
  out[3] = __byte_perm(x.y, x.w, 0x7632);
}
// Four codes of two words' halves each, as subnormal halves: x[0], x[2] code * 2^-24, x[1], x[3] code * 2^-20
__device__ __forceinline__ void codes4(uint32_t w, uint32_t* x) {
  const uint32_t v = w >> 8;
  x[0] = w & 0x000f000fu;
  x[1] = w & 0x00f000f0u;
  x[2] = v & 0x000f000fu;
  x[3] = v & 0x00f000f0u;
}
constexpr float k2p24 = 16777216.f, k2p20 = 1048576.f;
__device__ __forceinline__ float2 halves(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2*>(&x)); }

__device__ __forceinline__ void rows_cluster_sync() { asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ uint32_t peer_address(uint32_t at, uint32_t cta) {
  uint32_t p;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(p) : "r"(at), "r"(cta));
  return p;
}

// What a warp knows of its rows 2 t4 and 2 t4 + 1 (of each group of eight)
template <int NT>
struct RowsState {
  float rs[NT][2];             // a score's unit, log2
  float m[NT][2], l[NT][2];    // reference maximum (log2 units), sum of probabilities
  float pm[NT][2], pr[NT][2];  // sums of mid * probability and of P as rounded, over the thread's keys
  float o[NT][8][4];           // codes x P; or, once finished, values x probabilities
  int e;                       // P holds scale * probability / 2^e
  bool wide;                   // scores of the warp's rows may be beyond kWideScore
};

// Scores a (-inf where masked) become exponents y against the reference, which follows scores that exceed it by more than the
// threshold, as the exponent e does larger scales.
template <int NG, int NT>
__device__ __forceinline__ void follow(const float (&a)[NG][NT][4], float (&y)[NG][NT][4], int e, RowsState<NT>& st) {
  auto exponents = [&]() {
#pragma unroll
    for (int gr = 0; gr < NG; ++gr)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int v = 0; v < 4; ++v) y[gr][nt][v] = fmaf(a[gr][nt][v], st.rs[nt][v & 1], -st.m[nt][v & 1]);
    if (!st.wide) return;
#pragma unroll
    for (int gr = 0; gr < NG; ++gr)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int v = 0; v < 4; ++v) y[gr][nt][v] = __fadd_rn(__fmul_rn(a[gr][nt][v], st.rs[nt][v & 1]), -st.m[nt][v & 1]);
  };
  exponents();
  bool move = e > st.e;
#pragma unroll
  for (int gr = 0; gr < NG; ++gr)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int v = 0; v < 4; ++v) move |= y[gr][nt][v] > kRescaleThreshold;
  if (!__any_sync(0xffffffffu, move)) return;
  const float shrink = e > st.e ? (st.e - e < -126 ? 0.f : __uint_as_float((uint32_t)(127 + st.e - e) << 23)) : 1.f;
  st.e = max(st.e, e);
  bool wide = false;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float top = -INFINITY;
#pragma unroll
      for (int gr = 0; gr < NG; ++gr) top = max3(top, a[gr][nt][i], a[gr][nt][i + 2]);
      top *= st.rs[nt][i];  // (rs > 0)
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
      top = fmaxf(top, st.m[nt][i]);
      const float alpha = ex2(st.m[nt][i] - top);
      st.m[nt][i] = top;
      wide |= fabsf(top) > kWideScore && top != kNoRef;
      st.l[nt][i] *= alpha;
      st.pm[nt][i] *= alpha;
      st.pr[nt][i] *= alpha * shrink;
#pragma unroll
      for (int mt = 0; mt < 8; ++mt) {
        st.o[nt][mt][i] *= alpha * shrink;
        st.o[nt][mt][i + 2] *= alpha * shrink;
      }
    }
  st.wide = __any_sync(0xffffffffu, wide);
  exponents();
}

// The sums over the thread's keys become the warp's, and o what it stands for.  O's tile 4 j + k, rows 0..7, 8..15: channels
// 4 * (16 j + g8) + k, 4 * (16 j + 8 + g8) + k.
template <int NT>
__device__ __forceinline__ void finish(RowsState<NT>& st) {
  const int e = min(max(st.e, -126), 126);
  const float unit = __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float pm = st.pm[nt][i], pr = st.pr[nt][i];
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) {
        pm += __shfl_xor_sync(0xffffffffu, pm, d);
        pr += __shfl_xor_sync(0xffffffffu, pr, d);
      }
#pragma unroll
      for (int mt = 0; mt < 8; ++mt) {
        const float c = mt & 1 ? k2p20 : k2p24;
        st.o[nt][mt][i] = fmaf(unit, fmaf(st.o[nt][mt][i], c, -8.f * pr), pm);
        st.o[nt][mt][i + 2] = fmaf(unit, fmaf(st.o[nt][mt][i + 2], c, -8.f * pr), pm);
      }
    }
}

template <int NT, bool kBf16, bool kCluster>
__global__ void __launch_bounds__(32 * kRowsWarps, NT == 1 ? 3 : 2) kv4_rows_kernel(const Kv4Args a) {
  extern __shared__ __align__(128) uint8_t smem_raw[];
  RowsSmem<NT>* sm = reinterpret_cast<RowsSmem<NT>*>(smem_raw);
  const int warp = uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31, g8 = lane >> 2, t4 = lane & 3;
  if (threadIdx.x == 0) {
    for (int w = 0; w < kRowsWarps; ++w)
      for (int s = 0; s < kStages; ++s) mbar_init(&sm->full[w][s], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    sm->abort_flag = 0;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // The CTA's range of positions: of all units', or of its cluster's unit, which starts at 0.
  Kv4Ranges ranges = {0, 1, 0, 0};
  Kv4Unit own = {};
  int range_lo, range_hi;
  if (kCluster) {
    const int unit = blockIdx.x / a.cluster, rank = blockIdx.x - unit * a.cluster, x = unit / a.tiles;
    own.m = unit - x * a.tiles;
    own.r = x / a.Hkv;
    own.g = x - own.r * a.Hkv;
    own.L = kv4_len(a, own.r);
    if (a.lengths[own.r] > a.max_len && threadIdx.x == 0) dev_flag(a.status, SEQ_DEV_BAD_LENGTH);
    if (own.L < 0) return;  // (the whole cluster)
    own.prefix = kv4_prefix<kKeys>(a, own.L);
    own.end = own.prefix.steps + (min(a.n, ((own.m + 1) * a.row_tile + a.group - 1) / a.group) + kTreeStep - 1) / kTreeStep;
    range_lo = own.end * rank / a.cluster;
    range_hi = own.end * (rank + 1) / a.cluster;
    __syncthreads();
  } else {
    kv4_plan<kKeys, 32 * kRowsWarps>(&sm->plan, a);
    ranges = kv4_ranges(&sm->plan, a);
    if (threadIdx.x == 0) a.ws_cut[blockIdx.x] = make_int4(-1, 0, 0, 0);
    if ((int)blockIdx.x >= ranges.ctas || ranges.total == 0) return;
    range_lo = ranges.lo(blockIdx.x);
    range_hi = ranges.lo(blockIdx.x + 1);
  }
  auto unit_at = [&](int pos) -> Kv4Unit {
    if (kCluster) return own;
    return kv4_unit<kKeys>(&sm->plan, a, pos);
  };

  // ---- the loader: every warp's lane 0 asks for its steps, kStages of them ahead.  Page numbers are looked up 32 steps at a time,
  // a lane each.
  const uint32_t ring = smem_u32(sm->ring[warp][0]), bars = smem_u32(&sm->full[warp][0]);
  int load_pos = range_lo + warp, load_stage = 0, loaded = 0;
  int lt = 0, lt_end = 0;  // the step of the unit at load_pos, where the unit's prefix (or the range) ends
  int l_unit_end = 0, l_len = 0, l_split = 0, l_gap = 0, l_r = 0, l_g = 0;
  int id0 = 0, id1 = 0, ids = 32;  // lane x: the pages of the step x steps ahead of where they were looked up, ids steps ago
  auto load_next = [&]() {
    while (lt >= lt_end) {  // (a unit's prefix is through; its tree's steps are read where they are used)
      if (kCluster && lt_end > 0) return;
      const int from = loaded == 0 ? load_pos : max(load_pos, l_unit_end + ((warp - (l_unit_end - range_lo)) & (kRowsWarps - 1)));
      if (from >= range_hi) return;
      load_pos = from;
      const Kv4Unit lu = unit_at(load_pos);
      l_unit_end = lu.end; l_len = lu.L; l_split = lu.prefix.split; l_gap = lu.prefix.gap; l_r = lu.r; l_g = lu.g;
      lt = load_pos - lu.begin;
      lt_end = min(lu.prefix.steps, range_hi - lu.begin);
      ids = 32;
      if (lt >= lt_end) {  // nothing of this unit to load
        if (kCluster) {
          lt = lt_end = 1;
          return;
        }
        load_pos = l_unit_end + ((warp - (l_unit_end - range_lo)) & (kRowsWarps - 1));
        lt = lt_end = 0;
      }
    }
    if (ids == 32) {
      const int ahead = lt + lane * kRowsWarps, key = (ahead < l_split ? ahead : ahead + l_gap) * kKeys;
      id0 = id1 = 0;
      if (ahead < lt_end) {
        const int32_t* row = a.table + l_r * a.table_stride + (key >> a.page_shift);
        id0 = row[0];
        if (a.page_size == kGranule && key + kGranule < l_len) id1 = row[1];
        if ((unsigned)id0 >= (unsigned)a.num_pages || (unsigned)id1 >= (unsigned)a.num_pages) {
          dev_flag(a.status, SEQ_DEV_BAD_PAGE);
          if ((unsigned)id0 >= (unsigned)a.num_pages) id0 = 0;
          if ((unsigned)id1 >= (unsigned)a.num_pages) id1 = 0;
        }
      }
      ids = 0;
    }
    const int p0 = __shfl_sync(0xffffffffu, id0, ids), p1 = __shfl_sync(0xffffffffu, id1, ids);
    if (lane == 0) {
      const int key = (lt < l_split ? lt : lt + l_gap) * kKeys;
      const uint32_t dst = ring + load_stage * kBytes, bar = bars + 8 * load_stage;
      const uint8_t* head = a.pages + l_g * (a.page_size * 136);  // (4096 heads of 17408 bytes at most)
      const bool all = a.page_size > kGranule || key + kGranule < l_len;
      asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(all ? kBytes : kGranuleBytes) : "memory");
      if (a.page_size > kGranule) {
        bulk_load(dst, head + p0 * a.page_stride + (key & (a.page_size - 1)) * 136, kBytes, bar);
      } else {
        bulk_load(dst, head + p0 * a.page_stride, kGranuleBytes, bar);
        if (all) bulk_load(dst + kGranuleBytes, head + p1 * a.page_stride, kGranuleBytes, bar);
      }
    }
    __syncwarp();
    ++ids;
    ++loaded;
    load_stage = load_stage + 1 == kStages ? 0 : load_stage + 1;
    lt += kRowsWarps;
    load_pos += kRowsWarps;
  };
  for (int s = 0; s < kStages; ++s) load_next();

  bool ok = true;
  int used = 0, stage = 0, phase = 0;
  for (int pos = range_lo; pos < range_hi || kCluster;) {
    const Kv4Unit u = unit_at(pos);
    const int seg_end = min(u.end, range_hi);
    const int row0 = u.m * 8 * NT, live_rows = min(8 * NT, a.rows - row0);

    // ---- the unit's rows: q as half precision (scaled by a power of two), its sum, what it sees
    uint32_t qc[NT][16];
    float sq[NT][2];
    RowsState<NT> st;
    st.e = -1000;
    st.wide = false;
    int latest = 0;  // the last begin of a row's window
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int row = min(row0 + nt * 8 + g8, a.rows - 1);
      const int nd = row / a.group, h = u.g * a.group + row - nd * a.group;
      const uint4* src = reinterpret_cast<const uint4*>(a.q + u.r * a.q_req + nd * a.q_tok + h * a.q_head) + 4 * t4;
      uint4 x[4];
#pragma unroll
      for (int w = 0; w < 4; ++w) x[w] = src[w];
      float v[4][8], top = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t y[4] = {x[w].x, x[w].y, x[w].z, x[w].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (kBf16) {
            v[w][2 * i] = __uint_as_float(y[i] << 16);
            v[w][2 * i + 1] = __uint_as_float(y[i] & 0xffff0000u);
          } else {
            const float2 f2 = halves(y[i]);
            v[w][2 * i] = f2.x;
            v[w][2 * i + 1] = f2.y;
          }
          top = max3(top, fabsf(v[w][2 * i]), fabsf(v[w][2 * i + 1]));
        }
      }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      // the row's largest magnitude into [2^8, 2^9); a row of zeros, or one that is not finite, as it is
      const int e = (int)(__float_as_uint(top) >> 23);
      float f = 1.f, inv_f = 1.f;
      if (e > 8 && e < 255) {
        const int up = 8 + 127 - e;  // -119..126
        f = __uint_as_float((uint32_t)(127 + up) << 23);
        inv_f = __uint_as_float((uint32_t)(127 - up) << 23);
      }
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          y[i] = pack2<false>(v[w][2 * i] * f, v[w][2 * i + 1] * f);
          const float2 z = halves(y[i]);
          sum += z.x + z.y;
        }
        pairs_of_8(make_uint4(y[0], y[1], y[2], y[3]), &qc[nt][4 * w]);
        // channels 1, 3, 5, 7 meet codes of 2^-20
        qc[nt][4 * w + 1] = hmul2_bits(qc[nt][4 * w + 1], 0x2c002c00u);
        qc[nt][4 * w + 3] = hmul2_bits(qc[nt][4 * w + 3], 0x2c002c00u);
      }
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        sq[nt][i] = __shfl_sync(0xffffffffu, sum, (2 * t4 + i) * 4);
        st.rs[nt][i] = fmaxf(a.scale_log2 * __shfl_sync(0xffffffffu, inv_f, (2 * t4 + i) * 4), kLeastUnit);
        if (a.window > 0) {  // (every warp finds the same)
          const int begin = u.L + 1 - a.window + kv4_depth(a, u.r, min(row0 + nt * 8 + 2 * t4 + i, a.rows - 1) / a.group);
          sm->begin[nt * 8 + 2 * t4 + i] = begin;
          latest = max(latest, begin);
        }
        st.m[nt][i] = kNoRef;
        st.l[nt][i] = st.pm[nt][i] = st.pr[nt][i] = 0.f;
      }
#pragma unroll
      for (int mt = 0; mt < 8; ++mt)
#pragma unroll
        for (int e2 = 0; e2 < 4; ++e2) st.o[nt][mt][e2] = 0.f;
    }
    latest = __reduce_max_sync(0xffffffffu, latest);
    __syncwarp();

    int t = pos - u.begin + ((warp - (pos - range_lo)) & (kRowsWarps - 1));
    const int t_end = seg_end - u.begin;
    for (; t < min(u.prefix.steps, t_end); t += kRowsWarps) {
      if (ok) ok = mbar_wait(sm, &sm->full[warp][stage], phase, a.status);
      if (!ok) break;
      const int key0 = u.prefix.key_step(t) * kKeys;
      const uint32_t at = ring + stage * kBytes;
      const bool ends = key0 + kKeys > u.L;
      // the step's largest scale of V, a lane a key: the exponent of a half, rounded up (of zero and of subnormals: -14)
      uint32_t vp = lds32(at + (lane >> 4) * kGranuleBytes + kGranuleParams + kGranule * 4 + (lane & 15) * 4);
      if (ends && key0 + lane >= u.L) vp = 0u;
      const int e = __reduce_max_sync(0xffffffffu, (int)((vp >> 10) & 31u)) - 14;
      float x[2][NT][4], y[2][NT][4];
#pragma unroll
      for (int gr = 0; gr < 2; ++gr) {
        const uint32_t k_at = at + gr * kGranuleBytes + g8 * kCodeBytes + t4 * 16;
        const uint4 ka = lds128(k_at), kb = lds128(k_at + 8 * kCodeBytes);
        const uint32_t p_at = at + gr * kGranuleBytes + kGranuleParams + g8 * 4;
        const float2 fa = halves(lds32(p_at)), fb = halves(lds32(p_at + 32));
        float s[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int v = 0; v < 4; ++v) s[nt][v] = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          uint32_t a0[4], a1[4];
          codes4(w == 0 ? ka.x : w == 1 ? ka.y : w == 2 ? ka.z : ka.w, a0);
          codes4(w == 0 ? kb.x : w == 1 ? kb.y : w == 2 ? kb.z : kb.w, a1);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            mma16816(s[nt], a0[0], a1[0], a0[1], a1[1], qc[nt][4 * w], qc[nt][4 * w + 1]);
            mma16816(s[nt], a0[2], a1[2], a0[3], a1[3], qc[nt][4 * w + 2], qc[nt][4 * w + 3]);
          }
        }
        const float sa = fa.x * k2p24, sb = fb.x * k2p24, ma = fmaf(fa.x, -8.f, fa.y), mb = fmaf(fb.x, -8.f, fb.y);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            x[gr][nt][i] = fmaf(sa, s[nt][i], ma * sq[nt][i]);
            x[gr][nt][i + 2] = fmaf(sb, s[nt][i + 2], mb * sq[nt][i]);
          }
      }
      if (ends || key0 < latest) {  // some keys are not there, or not every row's
#pragma unroll
        for (int gr = 0; gr < 2; ++gr)
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            const int j = key0 + gr * kGranule + g8 + 8 * v;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int i = 0; i < 2; ++i)
                if (j >= u.L || (latest > 0 && j < sm->begin[nt * 8 + 2 * t4 + i] && j >= a.sinks)) x[gr][nt][2 * v + i] = -INFINITY;
          }
      }
      follow<2, NT>(x, y, e, st);
      const float per_unit = __uint_as_float((uint32_t)(127 - st.e) << 23);  // (-14 <= e <= 17)
      uint32_t pf[2][NT][2];
#pragma unroll
      for (int gr = 0; gr < 2; ++gr)
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          // V's scale and mid of key g8 + 8 v; what lies behind the prefix may be anything: zeros
          uint32_t vb = lds32(at + gr * kGranuleBytes + kGranuleParams + kGranule * 4 + g8 * 4 + 32 * v);
          if (ends && key0 + gr * kGranule + g8 + 8 * v >= u.L) vb = 0u;
          const float2 sm2 = halves(vb);
          const float sc = sm2.x * per_unit;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            const float p0 = ex2(y[gr][nt][2 * v]), p1 = ex2(y[gr][nt][2 * v + 1]);
            const uint32_t packed = pack2<false>(p0 * sc, p1 * sc);
            const float2 back = halves(packed);
            st.l[nt][0] += p0;
            st.l[nt][1] += p1;
            st.pm[nt][0] = fmaf(p0, sm2.y, st.pm[nt][0]);
            st.pm[nt][1] = fmaf(p1, sm2.y, st.pm[nt][1]);
            st.pr[nt][0] += back.x;
            st.pr[nt][1] += back.y;
            pf[gr][nt][v] = transpose8x8(packed);
          }
        }
#pragma unroll
      for (int gr = 0; gr < 2; ++gr) {
        // lane: a row of the four blocks (keys 0..7 and 8..15 of 16-byte columns 2 c and 2 c + 1)
        const uint32_t v_at = at + gr * kGranuleBytes + kGranuleV + (lane & 15) * kCodeBytes + (lane >> 4) * 16;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          uint32_t w[4], b[4][4];  // blocks: (column 2c, keys 0..7), (2c, 8..15), (2c + 1, 0..7), (2c + 1, 8..15)
          ldmatrix_x4_trans(v_at + 32 * c, w);
#pragma unroll
          for (int z = 0; z < 4; ++z) codes4(w[z], b[z]);
#pragma unroll
          for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma16816(st.o[nt][4 * c + k], b[0][k], b[2][k], b[1][k], b[3][k], pf[gr][nt][0], pf[gr][nt][1]);
        }
      }
      __syncwarp();  // every lane has read the stage
      ++used;
      if (++stage == kStages) { stage = 0; phase ^= 1; }
      load_next();
    }
    finish(st);
    // ---- the tree's rows, 16 at a time, from global memory.  (They come last: o is now what it stands for.)
    for (; t < t_end; t += kRowsWarps) {
      if (t < u.prefix.steps) continue;  // (only after a wait that ran out)
      const int w = t - u.prefix.steps;
      const uint8_t* k_rows = a.kt + u.r * a.t_req + u.g * a.t_head;
      const uint8_t* v_rows = a.vt + u.r * a.t_req + u.g * a.t_head;
#pragma unroll 1
      for (int gr = 0; gr < 2 && 32 * w + 16 * gr < a.n; ++gr) {
        const int n0 = 32 * w + 16 * gr;
        uint4 kx[2][4];
        uint2 vx[2][2][4];
#pragma unroll
        for (int z = 0; z < 2; ++z)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int j = n0 + g8 + 8 * z;
            kx[z][c] = make_uint4(0u, 0u, 0u, 0u);
            if (j < a.n) kx[z][c] = reinterpret_cast<const uint4*>(k_rows + j * a.t_tok)[4 * t4 + c];
          }
        // V in pairs of rows (2 t4, 2 t4 + 1 and eight more), channels 4 * (8 c + g8) and the three behind.  A cluster asks for it before anything
        // is used, where latency counts; the ranges do without the registers.
        auto load_v = [&]() {
#pragma unroll
          for (int z = 0; z < 2; ++z)
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
              for (int c = 0; c < 4; ++c) {
                const int j = n0 + 2 * t4 + 8 * z + y;
                vx[z][y][c] = make_uint2(0u, 0u);
                if (j < a.n) vx[z][y][c] = reinterpret_cast<const uint2*>(v_rows + j * a.t_tok)[8 * c + g8];
              }
        };
        if (kCluster) load_v();
        uint32_t seen[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int node = min(row0 + nt * 8 + 2 * t4 + i, a.rows - 1) / a.group;
            const uint32_t bits = kv4_mask_word(a, kv4_mask_row(a, u.r, node), node, w);
            seen[nt][i] = kv4_window_word(a, u.r, u.L, a.window > 0 ? sm->begin[nt * 8 + 2 * t4 + i] + a.window - 1 - u.L : 0, w, bits);
          }
        float s[1][NT][4], y[1][NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[0][nt][e] = 0.f;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t f[2][4];
#pragma unroll
          for (int z = 0; z < 2; ++z)
            pairs_of_8(make_uint4(to_half2<kBf16>(kx[z][c].x), to_half2<kBf16>(kx[z][c].y), to_half2<kBf16>(kx[z][c].z), to_half2<kBf16>(kx[z][c].w)), f[z]);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            mma16816(s[0][nt], f[0][0], f[1][0], f[0][1], f[1][1], qc[nt][4 * c], hmul2_bits(qc[nt][4 * c + 1], 0x4c004c00u));
            mma16816(s[0][nt], f[0][2], f[1][2], f[0][3], f[1][3], qc[nt][4 * c + 2], hmul2_bits(qc[nt][4 * c + 3], 0x4c004c00u));
          }
        }
        if (!kCluster) load_v();
        // A row of V with a value that is not finite in half precision counts as zeros, so that it stays out of the rows that do not see
        // it; those that do become NaN.
        uint32_t v[2][16], not_finite = 0;
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          uint32_t big = 0;  // the largest exponents of the two rows
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const uint32_t h0 = to_half2<kBf16>(i ? vx[z][0][c].y : vx[z][0][c].x), h1 = to_half2<kBf16>(i ? vx[z][1][c].y : vx[z][1][c].x);
              v[z][4 * c + 2 * i] = __byte_perm(h0, h1, 0x5410);
              v[z][4 * c + 2 * i + 1] = __byte_perm(h0, h1, 0x7632);
              big = __vmaxu2(big, __vmaxu2(v[z][4 * c + 2 * i] & 0x7c007c00u, v[z][4 * c + 2 * i + 1] & 0x7c007c00u));
            }
          if ((big & 0xffffu) == 0x7c00u) not_finite |= 1u << (16 * gr + 2 * t4 + 8 * z);
          if ((big >> 16) == 0x7c00u) not_finite |= 2u << (16 * gr + 2 * t4 + 8 * z);
        }
        not_finite = __reduce_or_sync(0xffffffffu, not_finite);
        if (not_finite != 0) {
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            const uint32_t two = not_finite >> (16 * gr + 2 * t4 + 8 * z);
            const uint32_t keep = (two & 1u ? 0u : 0xffffu) | (two & 2u ? 0u : 0xffff0000u);
#pragma unroll
            for (int i = 0; i < 16; ++i) v[z][i] &= keep;
          }
        }
        // A key that is not finite in half precision has no finite score (q is finite, or its row NaN anyway), and could have that of a hidden
        // one, -inf: rows that see it become NaN.
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool hidden = !((seen[nt][e & 1] >> (16 * gr + g8 + 8 * (e >> 1))) & 1u), finite = fabsf(s[0][nt][e]) < INFINITY;
            if (!hidden && !finite) st.l[nt][e & 1] = NAN;
            if (hidden || !finite) s[0][nt][e] = -INFINITY;
          }
        follow<1, NT>(s, y, st.e, st);
        uint32_t pf[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            const float p0 = ex2(y[0][nt][2 * z]), p1 = ex2(y[0][nt][2 * z + 1]);
            st.l[nt][0] += p0;
            st.l[nt][1] += p1;
            pf[nt][z] = transpose8x8(pack2<false>(p0, p1));
          }
        if (not_finite != 0) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 2; ++i)
              if (seen[nt][i] & not_finite) st.l[nt][i] = NAN;
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int k = 0; k < 4; ++k)
              mma16816(st.o[nt][4 * c + k], v[0][8 * c + k], v[0][8 * c + 4 + k], v[1][8 * c + k], v[1][8 * c + 4 + k], pf[nt][0], pf[nt][1]);
      }
    }

    // ---- the four warps' rows meet
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float l = st.l[nt][i];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
        const int row = nt * 8 + 2 * t4 + i;
        if (g8 == 0) sm->ml[warp][row] = make_float2(st.m[nt][i] > 0.5f * kNoRef || st.m[nt][i] != st.m[nt][i] ? st.m[nt][i] : -INFINITY, l);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int mt = 4 * (c >> 1), v = i + 2 * (c & 1);
          *reinterpret_cast<float4*>(&sm->o[warp][row][4 * (8 * c + g8)]) = make_float4(st.o[nt][mt][v], st.o[nt][mt + 1][v], st.o[nt][mt + 2][v], st.o[nt][mt + 3][v]);
        }
      }
    __syncthreads();
    const bool whole = !kCluster && pos == u.begin && seg_end == u.end;
    const int64_t slot = kCluster ? 0 : (int64_t)kv4_slot(ranges, blockIdx.x, u.begin) * a.row_tile;
    // Warp w: rows w, w + 4, ...; a lane has four channels of a row.
    auto write_row = [&](int row, float M, float sum, float4 acc) {
      const int rw = row0 + row, nd = rw / a.group, h = u.g * a.group + rw - nd * a.group;
      const float inv = 1.f / sum;
      *reinterpret_cast<uint2*>(a.out + u.r * a.o_req + nd * a.o_tok + h * a.o_head + 8 * lane) =
          make_uint2(pack2<kBf16>(acc.x * inv, acc.y * inv), pack2<kBf16>(acc.z * inv, acc.w * inv));
      if (a.lse != nullptr && lane == 0) a.lse[((int64_t)u.r * a.Hq + h) * a.n + nd] = (M + log2f(sum)) * kLn2;
    };
#pragma unroll
    for (int z = 0; z < 2 * NT; ++z) {
      const int row = warp + kRowsWarps * z;
      if (row >= live_rows) continue;
      float M = -INFINITY, sum = 0.f;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kRowsWarps; ++w) M = fmaxf(M, sm->ml[w][row].x);
#pragma unroll
      for (int w = 0; w < kRowsWarps; ++w) {
        const float2 ml = sm->ml[w][row];
        const float f = ml.x == -INFINITY ? 0.f : ex2(ml.x - M);
        const float4 v = *reinterpret_cast<const float4*>(&sm->o[w][row][4 * lane]);
        sum = fmaf(ml.y, f, sum);
        acc.x = fmaf(v.x, f, acc.x); acc.y = fmaf(v.y, f, acc.y); acc.z = fmaf(v.z, f, acc.z); acc.w = fmaf(v.w, f, acc.w);
      }
      if (kCluster) {  // (a row is its warp's own)
        __syncwarp();
        *reinterpret_cast<float4*>(&sm->o[0][row][4 * lane]) = acc;
        if (lane == 0) sm->ml[0][row] = make_float2(M, sum);
      } else if (whole) {
        write_row(row, M, sum, acc);
      } else {
        reinterpret_cast<float4*>(a.ws_o + (slot + row) * kHeadDim)[lane] = acc;
        if (lane == 0) a.ws_ml[slot + row] = make_float2(M, sum);
      }
    }
    if (kCluster) {
      // ---- the cluster's CTAs meet: each writes some of the rows
      rows_cluster_sync();
      const int rank = blockIdx.x % a.cluster;
      for (int row = rank + a.cluster * warp; row < live_rows; row += a.cluster * kRowsWarps) {
        float2 ml = make_float2(-INFINITY, 0.f);
        if (lane < a.cluster) {
          const uint32_t at = peer_address(smem_u32(&sm->ml[0][row]), lane);
          asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(ml.x), "=f"(ml.y) : "r"(at) : "memory");
        }
        const float M = warp_max(ml.x), f = ml.x == -INFINITY ? 0.f : ex2(ml.x - M), sum = warp_sum(ml.y * f);
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f), v[kRowsCluster];
#pragma unroll
        for (int p = 0; p < kRowsCluster; ++p) {
          v[p] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (p < a.cluster) {
            const uint32_t at = peer_address(smem_u32(&sm->o[0][row][4 * lane]), p);
            asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[p].x), "=f"(v[p].y), "=f"(v[p].z), "=f"(v[p].w) : "r"(at) : "memory");
          }
        }
#pragma unroll
        for (int p = 0; p < kRowsCluster; ++p) {
          const float w = __shfl_sync(0xffffffffu, f, p);
          acc.x = fmaf(v[p].x, w, acc.x); acc.y = fmaf(v[p].y, w, acc.y); acc.z = fmaf(v[p].z, w, acc.z); acc.w = fmaf(v[p].w, w, acc.w);
        }
        write_row(row, M, sum, acc);
      }
      rows_cluster_sync();  // nobody's rows are read any more
      break;
    }
    if (threadIdx.x == 0 && seg_end < u.end && pos == u.begin) a.ws_cut[blockIdx.x] = kv4_cut(a, ranges, u);
    __syncthreads();
    pos = seg_end;
  }
  // Nobody leaves while a copy into its shared memory is under way (only after a wait that ran out).
  for (; used < loaded; ++used) {
    for (uint32_t it = 0; it < (1u << 16); ++it)
      if (mbar_try_wait(&sm->full[warp][stage], phase)) break;
    if (++stage == kStages) { stage = 0; phase ^= 1; }
  }
}

// ---------------------------------------------------------------- host side ---------------------
static int rows_nt(const seq_tree_kv4_attention_params& p) { return p.n_tree * (p.num_q_heads / p.num_kv_heads) <= 8 ? 1 : 2; }
static int rows_ctas(int nt) { return device_sm_count() * (nt == 1 ? 3 : 2); }
static int64_t rows_units(const seq_tree_kv4_attention_params& p) {
  const int tile = 8 * rows_nt(p);
  return (int64_t)p.batch * p.num_kv_heads * ((p.n_tree * (p.num_q_heads / p.num_kv_heads) + tile - 1) / tile);
}
// Steps of 32 keys, of the longest prefix
static int rows_steps(const seq_tree_kv4_attention_params& p) {
  int L = p.max_len;
  if (p.window > 0 && (int64_t)p.window + p.sinks < L) L = p.window + p.sinks;
  return (L + 31) / 32 + (p.n_tree + kTreeStep - 1) / kTreeStep;
}
// CTAs of a unit's cluster, 0 for ranges.
static int rows_cluster(const seq_tree_kv4_attention_params& p) {
  const int64_t units = rows_units(p);
  const int steps = rows_steps(p);
  int c = 1;
  while (c < kRowsCluster && c * kRowsWarps < steps) c *= 2;
  while (c > 1 && units * c > rows_ctas(rows_nt(p))) c /= 2;
  if (units * c > rows_ctas(rows_nt(p)) || steps > 24 * c * kRowsWarps) return 0;
  return c;
}

// This kernel takes 16 query rows of a kv head at a time, the one of tiles 128 and 15 us for its start and its last pieces.  So up to 16 rows are
// this one's.  More rows, each pair the time of this kernel and of the tiles' (us, bfloat16 where nothing is said):
//   clusters, more than two tiles of rows: this one where a warp has at most 9 steps.
//     8 steps   12 nodes of 64/8 heads on 4096 tokens   19, 19        64 nodes of 32/32 heads on 1024 tokens   17, 19
//     16 steps  12 nodes of 64/8 heads on 8192 tokens   29, 22        more: 64 nodes of 32/32 heads on 4096    32, 26
//   clusters, two tiles of rows: always this one (16 steps: 18 to 31 against 21 to 34).
//   ranges, two tiles of rows: this one up to 20 steps a warp, and at any number for half-precision rows, whose tiles take longer.
//     4 requests of 2048 tokens, 32 nodes of 32/32 heads   32, 36     16 of them                                131, 98; fp16 122, 112
//     16 requests of 4096, 24 nodes of 32/32 heads         167, 147; fp16 161, 177
bool kv4_few_rows(const seq_tree_kv4_attention_params& p) {
  const int rows = p.n_tree * (p.num_q_heads / p.num_kv_heads), c = rows_cluster(p);
  if (rows <= 16) return true;
  if (c != 0) return rows <= 32 || rows_steps(p) <= 9 * c * kRowsWarps;
  return rows <= 32 && (p.dtype == SEQ_F16 || rows_units(p) * rows_steps(p) <= (int64_t)20 * kRowsWarps * rows_ctas(rows_nt(p)));
}

size_t kv4_rows_workspace_bytes(const seq_tree_kv4_attention_params& p) {
  if (rows_cluster(p) != 0) return 0;
  const int nt = rows_nt(p);
  return kv4_ranges_bytes(rows_ctas(nt), 8 * nt);
}

int launch_kv4_rows(const seq_tree_kv4_attention_params& p, cudaStream_t stream) {
  const int nt = rows_nt(p);
  Kv4Args a = kv4_args(p, 8 * nt, kTreeStep, 0, 0);
  a.min_steps = kRowsWarps;
  a.cluster = rows_cluster(p);
  const bool bf16 = p.dtype == SEQ_BF16;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(32 * kRowsWarps);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (a.cluster != 0) {
    cfg.gridDim = dim3((unsigned)(rows_units(p) * a.cluster));
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = a.cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.numAttrs = 2;
  } else {
    const int64_t most = (int64_t)a.batch * a.Hkv * a.tiles * ((p.max_len + kKeys - 1) / kKeys + 1 + a.tree_steps);
    if (most > 0x7fffffff) return SEQ_ERR_UNSUPPORTED;
    const int64_t want = (most + a.min_steps - 1) / a.min_steps;
    a.ctas = want < rows_ctas(nt) ? (int)want : rows_ctas(nt);
    kv4_ranges_place(a, rows_ctas(nt), p.workspace);
    cfg.gridDim = dim3(a.ctas);
  }
  auto launch = [&](auto kernel, int which, size_t smem) -> int {
    static int done[8][64];
    const int rc = once_per_device(done[which], [&]() -> int {
      SEQ_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
      return SEQ_OK;
    });
    if (rc != SEQ_OK) return rc;
    cfg.dynamicSmemBytes = smem;
    SEQ_CUDA_OK(cudaLaunchKernelEx(&cfg, kernel, a));
    return SEQ_OK;
  };
  constexpr size_t s1 = sizeof(RowsSmem<1>), s2 = sizeof(RowsSmem<2>);
  if (a.cluster != 0) {
    if (nt == 1) return bf16 ? launch(kv4_rows_kernel<1, true, true>, 0, s1) : launch(kv4_rows_kernel<1, false, true>, 1, s1);
    return bf16 ? launch(kv4_rows_kernel<2, true, true>, 2, s2) : launch(kv4_rows_kernel<2, false, true>, 3, s2);
  }
  int rc;
  if (nt == 1) rc = bf16 ? launch(kv4_rows_kernel<1, true, false>, 4, s1) : launch(kv4_rows_kernel<1, false, false>, 5, s1);
  else rc = bf16 ? launch(kv4_rows_kernel<2, true, false>, 6, s2) : launch(kv4_rows_kernel<2, false, false>, 7, s2);
  return rc != SEQ_OK ? rc : launch_kv4_merge(a, bf16, false, stream);
}

}  // namespace seqtree
