// Attention over the 4-bit pages for few query rows: the codes go from shared memory into mma fragments in registers.
//
// A warp takes 32 keys at a time, S^T = K Q^T with the keys in the 16-row operand and 8 query rows in the 8-column one, so that
// a single token's eight grouped heads fill the tile.  What bounds such a kernel before HBM does is instructions, so codes are not
// converted at all: four bits at the bottom of a half-precision word are the subnormal number code * 2^-24, four bits above
// them code * 2^-20, and the tensor core takes subnormals exactly.  One AND makes two operand values, a shift serves four.
//     S^T  keys x rows:     A = codes of K; q's channels that meet codes of 2^-20 are sixteen times smaller.  With s, m a key's scale and mid,
//                           s * (q . code) + (m - 8 s) * sum(q) is put together in fp32.
//     O^T  channels x rows: A = V^T, codes as they are (ldmatrix transposes 16-bit units, four channels of a key); B = P^T, a
//                           movmatrix of S^T's layout, P = s * probability in half precision; m * probability and -8 P are summed beside it.
// Scales are divided by a power of two not far from the largest met so far, so that P neither overflows nor becomes subnormal.
// Each warp has a ring of steps in shared memory, filled by bulk copies (a step is two granules, contiguous in a page), its
// own maxima and sums, and takes every fourth step of the CTA's range; the four meet at the end of each unit.
#include "kv4_attention.cuh"
#include "umma.cuh"

namespace seqtree {

constexpr int kRowsWarps = 4;
constexpr int kRowsStep = 32;  // keys
constexpr int kRowsStepBytes = kRowsStep / kGranule * kGranuleBytes;
constexpr int kOPad = kHeadDim + 4;

template <int NT>
struct RowsSmem {
  static constexpr int kStages = 3;
  uint8_t ring[kRowsWarps][kStages][kRowsStepBytes];
  float o[kRowsWarps][8 * NT][kOPad];
  float2 ml[kRowsWarps][8 * NT];
  uint64_t full[kRowsWarps][kStages];
  Kv4Plan plan;
  volatile int abort_flag;
  int32_t last;  // this CTA completes the unit
};

__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(smem_u32(dst)), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ uint32_t lds32(uint32_t at) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t at) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at) : "memory");
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
// 16-bit pairs as half precision pairs
template <bool kBf16>
__device__ __forceinline__ uint32_t to_half2(uint32_t x) {
  if (!kBf16) return x;
  return pack2<false>(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
}
// channels (0,4), (1,5), (2,6), (3,7) of eight: the order that unpack4 gives a code word's in
__device__ __forceinline__ void pairs_of_8(uint4 x, uint32_t* out) {
  out[0] = __byte_perm(x.x, x.z, 0x5410);
  out[1] = __byte_perm(x.x, x.z, 0x7632);
  out[2] = __byte_perm(x.y, x.w, 0x5410);
  out[3] = __byte_perm(x.y, x.w, 0x7632);
}

// eight 8x8 blocks of 16-bit units in two instructions: thread (g, t) gets unit g of rows 2t, 2t + 1, transposed
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t at, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
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

// What a warp knows of its rows 2 t4 and 2 t4 + 1 (of each group of eight)
template <int NT>
struct RowsState {
  float m[NT][2], l[NT][2];    // reference maximum (log2 units), sum of probabilities
  float pm[NT][2], pr[NT][2];  // sums of mid * probability and of P as rounded, over the thread's keys
  float o[NT][8][4];           // codes x P; or, once finished(), values x probabilities
  int e;                       // P holds scale * probability / 2^e
};

// The reference follows scores that exceed it by more than the threshold, the exponent larger scales.
template <int NG, int NT>
__device__ __forceinline__ void follow(const float (&x)[NG][NT][4], int e, RowsState<NT>& st) {
  bool move = e > st.e;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int v = 0; v < 4; ++v)
#pragma unroll
      for (int gr = 0; gr < NG; ++gr) move |= x[gr][nt][v] > st.m[nt][v & 1] + kRescaleThreshold;  // (also the first score: m = -inf)
  if (!__any_sync(0xffffffffu, move)) return;
  const float shrink = e > st.e ? (st.e - e < -126 ? 0.f : __uint_as_float((uint32_t)(127 + st.e - e) << 23)) : 1.f;
  st.e = max(st.e, e);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float mx = st.m[nt][i];
#pragma unroll
      for (int gr = 0; gr < NG; ++gr) mx = max3(mx, x[gr][nt][i], x[gr][nt][i + 2]);
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
      const float alpha = st.m[nt][i] == -INFINITY ? 0.f : ex2(st.m[nt][i] - mx);
      st.m[nt][i] = mx;
      st.l[nt][i] *= alpha;
      st.pm[nt][i] *= alpha;
      st.pr[nt][i] *= alpha * shrink;
#pragma unroll
      for (int mt = 0; mt < 8; ++mt) {
        st.o[nt][mt][i] *= alpha * shrink;
        st.o[nt][mt][i + 2] *= alpha * shrink;
      }
    }
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

template <int NT, bool kBf16>
__global__ void __launch_bounds__(32 * kRowsWarps, NT == 1 ? 3 : 2) kv4_rows_kernel(const Kv4Args a) {
  extern __shared__ __align__(128) uint8_t smem_raw[];
  using Smem = RowsSmem<NT>;
  Smem* sm = reinterpret_cast<Smem*>(smem_raw);
  constexpr int kStages = Smem::kStages;
  const int warp = uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31, g8 = lane >> 2, t4 = lane & 3;
  if (threadIdx.x == 0) {
    for (int w = 0; w < kRowsWarps; ++w)
      for (int s = 0; s < kStages; ++s) mbar_init(&sm->full[w][s], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    sm->abort_flag = 0;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  kv4_plan<kRowsStep, 32 * kRowsWarps>(&sm->plan, a);
  const Kv4Ranges ranges = kv4_ranges(&sm->plan, a);
  if ((int)blockIdx.x >= ranges.ctas || ranges.total == 0) return;
  const int range_lo = ranges.lo(blockIdx.x), range_hi = ranges.lo(blockIdx.x + 1);

  // ---- the loader: every warp's lane 0 asks for its steps, kStages of them ahead.  Page numbers are looked up 32 steps at a
  // time, a lane each.
  int load_pos = range_lo + warp, loaded = 0, used = 0;  // steps asked for, steps taken
  Kv4Unit lu;
  lu.end = -1;
  int id0 = 0, id1 = 0, ids_at = 0, ids_left = 0;
  auto load_next = [&]() {
    while (load_pos < range_hi) {
      if (load_pos >= lu.end) {
        lu = kv4_unit<kRowsStep>(&sm->plan, a, load_pos);
        ids_left = 0;
      }
      const int t = load_pos - lu.begin;
      if (t < lu.prefix.steps) break;
      load_pos += kRowsWarps;  // (a step of the tree: read where it is used)
    }
    if (load_pos >= range_hi) return;
    const int t = load_pos - lu.begin;
    if (ids_left == 0) {
      const int tt = t + lane * kRowsWarps;
      if (tt < lu.prefix.steps) {
        const int key = lu.prefix.key_step(tt) * kRowsStep;
        const int32_t* row = a.table + lu.r * a.table_stride;
        id0 = row[key >> a.page_shift];
        id1 = a.page_size == kGranule && key + kGranule < lu.L ? row[(key >> a.page_shift) + 1] : id0;
        if ((unsigned)id0 >= (unsigned)a.num_pages || (unsigned)id1 >= (unsigned)a.num_pages) {
          dev_flag(a.status, SEQ_DEV_BAD_PAGE);
          id0 = (unsigned)id0 < (unsigned)a.num_pages ? id0 : 0;
          id1 = (unsigned)id1 < (unsigned)a.num_pages ? id1 : 0;
        }
      }
      ids_at = 0;
      ids_left = 32;
    }
    const int p0 = __shfl_sync(0xffffffffu, id0, ids_at), p1 = __shfl_sync(0xffffffffu, id1, ids_at);
    ++ids_at;
    --ids_left;
    const int stage = loaded % kStages;
    if (lane == 0) {
      const int key = lu.prefix.key_step(t) * kRowsStep;
      uint8_t* dst = sm->ring[warp][stage];
      uint64_t* bar = &sm->full[warp][stage];
      const uint8_t* head = a.pages + (int64_t)lu.g * a.page_size * 136;
      if (a.page_size == kGranule) {
        const bool both = key + kGranule < lu.L;
        mbar_expect_tx(bar, both ? kRowsStepBytes : kGranuleBytes);
        bulk_load(dst, head + p0 * a.page_stride, kGranuleBytes, bar);
        if (both) bulk_load(dst + kGranuleBytes, head + p1 * a.page_stride, kGranuleBytes, bar);
      } else {
        mbar_expect_tx(bar, kRowsStepBytes);
        bulk_load(dst, head + p0 * a.page_stride + (key & (a.page_size - 1)) / kGranule * kGranuleBytes, kRowsStepBytes, bar);
      }
    }
    __syncwarp();
    ++loaded;
    load_pos += kRowsWarps;
  };
  for (int s = 0; s < kStages; ++s) load_next();

  bool ok = true;
  for (int pos = range_lo; pos < range_hi;) {
    const Kv4Unit u = kv4_unit<kRowsStep>(&sm->plan, a, pos);
    const int seg_end = min(u.end, range_hi);
    const int row0 = u.m * 8 * NT, live_rows = min(8 * NT, a.rows - row0);

    // ---- the unit's rows: q as half precision (bf16 rows scaled by a power of two, exactly), its sum, what it sees
    uint32_t qc[NT][16];
    float rs[NT][2], sq[NT][2];
    RowsState<NT> st;
    st.e = -1000;
    bool finished = false;
    int node[NT][2], begin[NT][2], depth[NT][2];
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
            const float2 f2 = __half22float2(*reinterpret_cast<const __half2*>(&y[i]));
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
        const int up = min(max(8 + 127 - e, -100), 100);
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
          const float2 z = __half22float2(*reinterpret_cast<const __half2*>(&y[i]));
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
        rs[nt][i] = a.scale_log2 * __shfl_sync(0xffffffffu, inv_f, (2 * t4 + i) * 4);
        const int rw = min(row0 + nt * 8 + 2 * t4 + i, a.rows - 1);
        node[nt][i] = rw / a.group;
        depth[nt][i] = a.window > 0 ? kv4_depth(a, u.r, node[nt][i]) : 0;
        begin[nt][i] = a.window > 0 ? u.L + depth[nt][i] + 1 - a.window : 0;
        latest = max(latest, begin[nt][i]);
        st.m[nt][i] = -INFINITY;
        st.l[nt][i] = st.pm[nt][i] = st.pr[nt][i] = 0.f;
      }
#pragma unroll
      for (int mt = 0; mt < 8; ++mt)
#pragma unroll
        for (int e2 = 0; e2 < 4; ++e2) st.o[nt][mt][e2] = 0.f;
    }
    latest = __reduce_max_sync(0xffffffffu, latest);

    const int seg_first = pos + ((warp - (pos - range_lo)) & (kRowsWarps - 1));
    for (int p = seg_first; p < seg_end; p += kRowsWarps) {
      const int t = p - u.begin;
      if (t < u.prefix.steps) {
        const int stage = used % kStages, key0 = u.prefix.key_step(t) * kRowsStep;
        if (ok) ok = mbar_wait(sm, &sm->full[warp][stage], (used / kStages) & 1, a.status);
        if (!ok) break;
        const uint32_t at = smem_u32(sm->ring[warp][stage]);
        const bool ends = key0 + kRowsStep > u.L;
        // the step's largest scale of V: a lane a key
        uint32_t vp = lds32(at + (lane >> 4) * kGranuleBytes + kGranuleParams + kGranule * 4 + (lane & 15) * 4);
        if (ends && key0 + lane >= u.L) vp = 0u;
        // (the exponent of a half, rounded up; of zero and of subnormals: -14)
        const int e = __reduce_max_sync(0xffffffffu, (int)((vp >> 10) & 31u)) - 14;
        float x[2][NT][4];
        float vs[2][2], vm[2][2];  // V's scale and mid of the thread's keys g8, g8 + 8
#pragma unroll
        for (int gr = 0; gr < 2; ++gr) {
          const uint32_t k_at = at + gr * kGranuleBytes + g8 * kCodeBytes + t4 * 16;
          const uint4 ka = lds128(k_at), kb = lds128(k_at + 8 * kCodeBytes);
          const uint32_t p_at = at + gr * kGranuleBytes + kGranuleParams + g8 * 4;
          const uint32_t pa = lds32(p_at), pb = lds32(p_at + 32);
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
          const float2 fa = __half22float2(*reinterpret_cast<const __half2*>(&pa)), fb = __half22float2(*reinterpret_cast<const __half2*>(&pb));
          const float sa = fa.x * k2p24, sb = fb.x * k2p24, ma = fmaf(fa.x, -8.f, fa.y), mb = fmaf(fb.x, -8.f, fb.y);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              x[gr][nt][i] = rs[nt][i] * fmaf(sa, s[nt][i], ma * sq[nt][i]);
              x[gr][nt][i + 2] = rs[nt][i] * fmaf(sb, s[nt][i + 2], mb * sq[nt][i]);
            }
          uint32_t va = lds32(p_at + kGranule * 4), vb = lds32(p_at + kGranule * 4 + 32);
          if (ends) {  // what lies behind the prefix may be anything: zeros
            if (key0 + gr * kGranule + g8 >= u.L) va = 0u;
            if (key0 + gr * kGranule + g8 + 8 >= u.L) vb = 0u;
          }
          const float2 ga = __half22float2(*reinterpret_cast<const __half2*>(&va)), gb = __half22float2(*reinterpret_cast<const __half2*>(&vb));
          vs[gr][0] = ga.x; vm[gr][0] = ga.y;
          vs[gr][1] = gb.x; vm[gr][1] = gb.y;
        }
        if (ends || (a.window > 0 && key0 < latest)) {  // some keys are not there, or not every row's
#pragma unroll
          for (int gr = 0; gr < 2; ++gr)
#pragma unroll
            for (int v = 0; v < 2; ++v) {
              const int j = key0 + gr * kGranule + g8 + 8 * v;
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                  if (j >= u.L || (j < begin[nt][i] && j >= a.sinks)) x[gr][nt][2 * v + i] = -INFINITY;
            }
        }
        follow<2, NT>(x, e, st);
        const float per_unit = __uint_as_float((uint32_t)(127 - st.e) << 23);  // (-14 <= e <= 17)
        uint32_t pf[2][NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const float n0 = st.m[nt][0] == -INFINITY ? 0.f : st.m[nt][0], n1 = st.m[nt][1] == -INFINITY ? 0.f : st.m[nt][1];
#pragma unroll
          for (int gr = 0; gr < 2; ++gr)
#pragma unroll
            for (int v = 0; v < 2; ++v) {
              const float p0 = ex2(x[gr][nt][2 * v] - n0), p1 = ex2(x[gr][nt][2 * v + 1] - n1);
              const float sc = vs[gr][v] * per_unit;
              const uint32_t packed = pack2<false>(p0 * sc, p1 * sc);
              const float2 back = __half22float2(*reinterpret_cast<const __half2*>(&packed));
              st.l[nt][0] += p0;
              st.l[nt][1] += p1;
              st.pm[nt][0] = fmaf(p0, vm[gr][v], st.pm[nt][0]);
              st.pm[nt][1] = fmaf(p1, vm[gr][v], st.pm[nt][1]);
              st.pr[nt][0] += back.x;
              st.pr[nt][1] += back.y;
              pf[gr][nt][v] = transpose8x8(packed);
            }
        }
#pragma unroll
        for (int gr = 0; gr < 2; ++gr) {
          // lane: a row of the four blocks (keys 0..7 and 8..15 of 16-byte columns 2 c and 2 c + 1)
          const uint32_t v_at = at + gr * kGranuleBytes + kGranuleV + ((lane & 7) + 8 * ((lane >> 3) & 1)) * kCodeBytes + (lane >> 4) * 16;
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint32_t w[4], b[4][4];  // blocks: (column 2c, keys 0..7), (2c, 8..15), (2c + 1, 0..7), (2c + 1, 8..15)
            ldmatrix_x4_trans(v_at + 32 * c, w);
#pragma unroll
            for (int y = 0; y < 4; ++y) codes4(w[y], b[y]);
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) mma16816(st.o[nt][4 * c + k], b[0][k], b[2][k], b[1][k], b[3][k], pf[gr][nt][0], pf[gr][nt][1]);
          }
        }
        __syncwarp();  // every lane has read the stage
        ++used;
        load_next();
        continue;
      }
      // ---- 32 rows of the tree, from global memory: 16 at a time.  (The last steps of a unit: o becomes what it stands for.)
      if (!finished) {
        finish(st);
        finished = true;
      }
      const int w = t - u.prefix.steps;
      uint32_t seen[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t bits = kv4_mask_word(a, kv4_mask_row(a, u.r, node[nt][i]), node[nt][i], w);
          seen[nt][i] = kv4_window_word(a, u.r, u.L, depth[nt][i], w, bits);
        }
      const uint8_t* k_rows = a.kt + u.r * a.t_req + u.g * a.t_head;
      const uint8_t* v_rows = a.vt + u.r * a.t_req + u.g * a.t_head;
#pragma unroll 1
      for (int gr = 0; gr < 2 && 32 * w + 16 * gr < a.n; ++gr) {
        const int n0 = 32 * w + 16 * gr;
        float s[1][NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[0][nt][e] = 0.f;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t f0[4], f1[4];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int j = n0 + g8 + 8 * e;
            uint4 x = make_uint4(0u, 0u, 0u, 0u);
            if (j < a.n) x = reinterpret_cast<const uint4*>(k_rows + j * a.t_tok)[4 * t4 + c];
            x = make_uint4(to_half2<kBf16>(x.x), to_half2<kBf16>(x.y), to_half2<kBf16>(x.z), to_half2<kBf16>(x.w));
            pairs_of_8(x, e ? f1 : f0);
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            mma16816(s[0][nt], f0[0], f1[0], f0[1], f1[1], qc[nt][4 * c], hmul2_bits(qc[nt][4 * c + 1], 0x4c004c00u));
            mma16816(s[0][nt], f0[2], f1[2], f0[3], f1[3], qc[nt][4 * c + 2], hmul2_bits(qc[nt][4 * c + 3], 0x4c004c00u));
          }
        }
        // V, in pairs of rows (2 t4, 2 t4 + 1 and eight more).  A row with a value that is not finite in half precision counts as zeros, so that
        // it stays out of the rows that do not see it; those that do become NaN.
        uint32_t v[2][16], not_finite = 0;
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const int j = n0 + 2 * t4 + 8 * y;
          uint32_t big = 0;  // the largest exponents of the two rows
#pragma unroll
          for (int c = 0; c < 4; ++c) {  // channels 4 * (8 c + g8) and the three behind
            uint2 x0 = make_uint2(0u, 0u), x1 = make_uint2(0u, 0u);
            if (j < a.n) x0 = reinterpret_cast<const uint2*>(v_rows + j * a.t_tok)[8 * c + g8];
            if (j + 1 < a.n) x1 = reinterpret_cast<const uint2*>(v_rows + (j + 1) * a.t_tok)[8 * c + g8];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const uint32_t h0 = to_half2<kBf16>(i ? x0.y : x0.x), h1 = to_half2<kBf16>(i ? x1.y : x1.x);
              v[y][4 * c + 2 * i] = __byte_perm(h0, h1, 0x5410);
              v[y][4 * c + 2 * i + 1] = __byte_perm(h0, h1, 0x7632);
              big = __vmaxu2(big, __vmaxu2(v[y][4 * c + 2 * i] & 0x7c007c00u, v[y][4 * c + 2 * i + 1] & 0x7c007c00u));
            }
          }
          if ((big & 0xffffu) == 0x7c00u) not_finite |= 1u << (16 * gr + 2 * t4 + 8 * y);
          if ((big >> 16) == 0x7c00u) not_finite |= 2u << (16 * gr + 2 * t4 + 8 * y);
        }
        not_finite = __reduce_or_sync(0xffffffffu, not_finite);
        if (not_finite != 0) {
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const uint32_t two = not_finite >> (16 * gr + 2 * t4 + 8 * y);
            const uint32_t keep = (two & 1u ? 0u : 0xffffu) | (two & 2u ? 0u : 0xffff0000u);
#pragma unroll
            for (int i = 0; i < 16; ++i) v[y][i] &= keep;
          }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool visible = (seen[nt][e & 1] >> (16 * gr + g8 + 8 * (e >> 1))) & 1u;
            s[0][nt][e] = visible ? s[0][nt][e] * rs[nt][e & 1] : -INFINITY;
          }
        follow<1, NT>(s, st.e, st);
        uint32_t pf[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const float n0 = st.m[nt][0] == -INFINITY ? 0.f : st.m[nt][0], n1 = st.m[nt][1] == -INFINITY ? 0.f : st.m[nt][1];
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const float p0 = ex2(s[0][nt][2 * y] - n0), p1 = ex2(s[0][nt][2 * y + 1] - n1);
            st.l[nt][0] += p0;
            st.l[nt][1] += p1;
            pf[nt][y] = transpose8x8(pack2<false>(p0, p1));
          }
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
    if (!finished) finish(st);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float l = st.l[nt][i];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
        const int row = nt * 8 + 2 * t4 + i;
        if (g8 == 0) sm->ml[warp][row] = make_float2(st.m[nt][i], l);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int mt = 4 * (c >> 1), v = i + 2 * (c & 1);
          *reinterpret_cast<float4*>(&sm->o[warp][row][4 * (8 * c + g8)]) = make_float4(st.o[nt][mt][v], st.o[nt][mt + 1][v], st.o[nt][mt + 2][v], st.o[nt][mt + 3][v]);
        }
      }
    __syncthreads();
    const bool whole = pos == u.begin && seg_end == u.end;
    const int64_t slot = (int64_t)kv4_slot(ranges, blockIdx.x, u.begin) * a.row_tile;
    // Warp w: rows w, w + 4, ...; a lane has four channels of a row.
    using T = typename std::conditional<kBf16, __nv_bfloat16, __half>::type;
    auto write_row = [&](int row, float M, float sum, float4 acc) {
      const int rw = row0 + row, nd = rw / a.group, h = u.g * a.group + rw - nd * a.group;
      const float inv = 1.f / sum;
      *reinterpret_cast<uint2*>(a.out + u.r * a.o_req + nd * a.o_tok + h * a.o_head + 8 * lane) =
          make_uint2(pack2<kBf16>(acc.x * inv, acc.y * inv), pack2<kBf16>(acc.z * inv, acc.w * inv));
      if (a.lse != nullptr && lane == 0) a.lse[((int64_t)u.r * a.Hq + h) * a.n + nd] = (M + log2f(sum)) * kLn2;
    };
#pragma unroll
    for (int y = 0; y < 2 * NT; ++y) {
      const int row = warp + kRowsWarps * y;
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
      if (row >= live_rows) continue;
      if (whole) {
        write_row(row, M, sum, acc);
      } else {
        reinterpret_cast<float4*>(a.ws_o + (slot + row) * kHeadDim)[lane] = acc;
        if (lane == 0) a.ws_ml[slot + row] = make_float2(M, sum);
      }
    }
    if (!whole) {
      // The piece is counted; the CTA that counts the last one adds them all, in the order of their CTAs.  Nobody waits.
      const Kv4Pieces pieces = kv4_pieces(ranges, u);
      __threadfence();
      __syncthreads();
      if (threadIdx.x == 0) sm->last = atomicAdd(a.ws_count + 2 * pieces.first, 1) == pieces.last - pieces.first;
      __syncthreads();
      if (sm->last) {
        __threadfence();
#pragma unroll
        for (int y = 0; y < 2 * NT; ++y) {
          const int row = warp + kRowsWarps * y;
          if (row >= live_rows) continue;
          // 32 pieces at a time: a lane looks one's (m, l) up, then all add its rows
          float M = -INFINITY, sum = 0.f;
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
          for (int p0 = pieces.first; p0 <= pieces.last; p0 += 32) {
            const int n = min(32, pieces.last - p0 + 1);
            float2 ml = make_float2(-INFINITY, 0.f);
            if (lane < n) ml = __ldcg(a.ws_ml + (int64_t)kv4_slot(ranges, p0 + lane, u.begin) * a.row_tile + row);
            const float now = fmaxf(M, warp_max(ml.x)), old = M == -INFINITY ? 0.f : ex2(M - now);
            M = now;
            const float f = ml.x == -INFINITY ? 0.f : ex2(ml.x - M);
            sum = sum * old + warp_sum(ml.y * f);
            acc.x *= old; acc.y *= old; acc.z *= old; acc.w *= old;
#pragma unroll 4
            for (int p = 0; p < n; ++p) {
              const float4 v = __ldcg(reinterpret_cast<const float4*>(a.ws_o + ((int64_t)kv4_slot(ranges, p0 + p, u.begin) * a.row_tile + row) * kHeadDim) + lane);
              const float w = __shfl_sync(0xffffffffu, f, p);
              acc.x = fmaf(v.x, w, acc.x); acc.y = fmaf(v.y, w, acc.y); acc.z = fmaf(v.z, w, acc.z); acc.w = fmaf(v.w, w, acc.w);
            }
          }
          write_row(row, M, sum, acc);
        }
      }
    }
    __syncthreads();
    pos = seg_end;
  }
  // Nobody leaves while a copy into its shared memory is under way (only after a wait that ran out).
  for (; used < loaded; ++used)
    for (uint32_t it = 0; it < (1u << 16); ++it)
      if (mbar_try_wait(&sm->full[warp][used % kStages], (used / kStages) & 1)) break;
}

// ---------------------------------------------------------------- host side ---------------------
static int rows_nt(const seq_tree_kv4_attention_params& p) { return p.n_tree * (p.num_q_heads / p.num_kv_heads) <= 8 ? 1 : 2; }
static int rows_ctas(int nt) { return device_sm_count() * (nt == 1 ? 3 : 2); }

size_t kv4_rows_workspace_bytes(const seq_tree_kv4_attention_params& p) {
  const int nt = rows_nt(p);
  return kv4_count_bytes(rows_ctas(nt)) + (size_t)2 * rows_ctas(nt) * 8 * nt * (kHeadDim * sizeof(float) + sizeof(float2));
}

int launch_kv4_rows(const seq_tree_kv4_attention_params& p, cudaStream_t stream) {
  const int nt = rows_nt(p);
  Kv4Args a = kv4_args(p);
  a.row_tile = 8 * nt;
  a.tiles = (a.rows + a.row_tile - 1) / a.row_tile;
  a.tree_steps = (a.n + kRowsStep - 1) / kRowsStep;
  a.min_steps = kRowsWarps;
  const int64_t most = (int64_t)a.batch * a.Hkv * a.tiles * ((p.max_len + kRowsStep - 1) / kRowsStep + 1 + a.tree_steps);
  if (most > 0x7fffffff) return SEQ_ERR_UNSUPPORTED;
  const int64_t want = (most + a.min_steps - 1) / a.min_steps;
  a.ctas = want < rows_ctas(nt) ? (int)want : rows_ctas(nt);
  a.ws_count = static_cast<int32_t*>(p.workspace);
  a.ws_o = reinterpret_cast<float*>(static_cast<uint8_t*>(p.workspace) + kv4_count_bytes(rows_ctas(nt)));
  a.ws_ml = reinterpret_cast<float2*>(a.ws_o + (size_t)2 * rows_ctas(nt) * a.row_tile * kHeadDim);
  const int rc0 = launch_kv4_zero(a, stream);
  if (rc0 != SEQ_OK) return rc0;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(a.ctas);
  cfg.blockDim = dim3(32 * kRowsWarps);
  cfg.stream = stream;
  cudaLaunchAttribute early[1];
  early[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = early;
  cfg.numAttrs = 1;
  auto launch = [&](auto kernel, int which, size_t smem) -> int {
    static int done[4][64];
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
  int rc;
  if (nt == 1) rc = bf16 ? launch(kv4_rows_kernel<1, true>, 0, sizeof(RowsSmem<1>)) : launch(kv4_rows_kernel<1, false>, 1, sizeof(RowsSmem<1>));
  else rc = bf16 ? launch(kv4_rows_kernel<2, true>, 2, sizeof(RowsSmem<2>)) : launch(kv4_rows_kernel<2, false>, 3, sizeof(RowsSmem<2>));
  return rc;
}

}  // namespace seqtree
