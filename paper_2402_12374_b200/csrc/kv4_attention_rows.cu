// Attention over the 4-bit pages for few query rows: the codes go from shared memory into mma fragments in registers.
//
// A warp takes 32 keys at a time, S^T = K Q^T with the keys in the 16-row operand and 8 query rows in the 8-column one, so that
// a single token's eight grouped heads fill the tile:
//     S^T  keys x rows:    A = codes less 8 of K, exact in half precision; scale and mid of a key are applied to the fp32 sums,
//                          scale * (q . (code - 8)) + mid * sum(q)
//     O^T  channels x rows: A = V^T, the values scale * (code - 8) + mid rounded to half; B = P^T, a movmatrix of S^T's layout
// A thread's code words hold channels of one key (K) or, two words interleaved, of a pair of keys (V); the contraction's order
// is free, so neither needs a transposition.  Each warp has a ring of steps in shared memory, filled by bulk copies (a step is
// two granules, contiguous in a page), its own maxima and sums, and takes every fourth step of the CTA's range; the four meet
// at the end of each unit.
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

// A step's scores x (log2 units, -inf where masked) become probabilities of half precision in P^T's layout, against reference
// maxima that only move when a score exceeds them by more than the threshold.
template <int NG, int NT>
__device__ __forceinline__ void softmax_step(float (&x)[NG][NT][4], float (&m)[NT][2], float (&l)[NT][2], float (&o)[NT][8][4], uint32_t (&p)[NG][NT][2]) {
  bool move = false;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int gr = 0; gr < NG; ++gr) move |= x[gr][nt][e] > m[nt][e & 1] + kRescaleThreshold;  // (also the first score: m = -inf)
  if (__any_sync(0xffffffffu, move)) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float mx = m[nt][i];
#pragma unroll
        for (int gr = 0; gr < NG; ++gr) mx = max3(mx, x[gr][nt][i], x[gr][nt][i + 2]);
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
        const float alpha = m[nt][i] == -INFINITY ? 0.f : ex2(m[nt][i] - mx);
        m[nt][i] = mx;
        l[nt][i] *= alpha;
#pragma unroll
        for (int mt = 0; mt < 8; ++mt) {
          o[nt][mt][i] *= alpha;
          o[nt][mt][i + 2] *= alpha;
        }
      }
  }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const float n0 = m[nt][0] == -INFINITY ? 0.f : m[nt][0], n1 = m[nt][1] == -INFINITY ? 0.f : m[nt][1];
#pragma unroll
    for (int gr = 0; gr < NG; ++gr) {
      const float p0 = ex2(x[gr][nt][0] - n0), p1 = ex2(x[gr][nt][1] - n1), p2 = ex2(x[gr][nt][2] - n0), p3 = ex2(x[gr][nt][3] - n1);
      l[nt][0] += p0 + p2;
      l[nt][1] += p1 + p3;
      p[gr][nt][0] = transpose8x8(pack2<false>(p0, p1));
      p[gr][nt][1] = transpose8x8(pack2<false>(p2, p3));
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
  const int kappa = (g8 & 1) ? 4 + ((g8 >> 1) ^ 1) : g8 >> 1;  // the key in the granule of operand row g8 (row g8 + 8: 8 more)
  for (int pos = range_lo; pos < range_hi;) {
    const Kv4Unit u = kv4_unit<kRowsStep>(&sm->plan, a, pos);
    const int seg_end = min(u.end, range_hi);
    const int row0 = u.m * 8 * NT, live_rows = min(8 * NT, a.rows - row0);

    // ---- the unit's rows: q as half precision (bf16 rows scaled by a power of two, exactly), its sum, what it sees
    uint32_t qf[NT][16];
    float rs[NT][2], sq[NT][2], m[NT][2], l[NT][2], o[NT][8][4];
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
      float f = 1.f, inv_f = 1.f;
      if (kBf16) {  // the row's largest magnitude into [2^8, 2^9); a row of zeros, or one that is not finite, as it is
        uint32_t top = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t v = i == 0 ? x[w].x : i == 1 ? x[w].y : i == 2 ? x[w].z : x[w].w;
            top = max(top, max((v << 16) & 0x7fffffffu, v & 0x7fff0000u));
          }
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int e = (int)(top >> 23);
        if (e > 8 && e < 255) {
          const int up = min(max(8 + 127 - e, -100), 100);
          f = __uint_as_float((uint32_t)(127 + up) << 23);
          inv_f = __uint_as_float((uint32_t)(127 - up) << 23);
        }
      }
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t v[4] = {x[w].x, x[w].y, x[w].z, x[w].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (kBf16) v[i] = pack2<false>(__uint_as_float(v[i] << 16) * f, __uint_as_float(v[i] & 0xffff0000u) * f);
          const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&v[i]));
          sum += y.x + y.y;
        }
        pairs_of_8(make_uint4(v[0], v[1], v[2], v[3]), &qf[nt][4 * w]);
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
        m[nt][i] = -INFINITY;
        l[nt][i] = 0.f;
      }
#pragma unroll
      for (int mt = 0; mt < 8; ++mt)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[nt][mt][e] = 0.f;
    }
    latest = __reduce_max_sync(0xffffffffu, latest);

    const int seg_first = pos + ((warp - (pos - range_lo)) & (kRowsWarps - 1));
    for (int p = seg_first; p < seg_end; p += kRowsWarps) {
      const int t = p - u.begin;
      if (t < u.prefix.steps) {
        const int stage = used % kStages, key0 = u.prefix.key_step(t) * kRowsStep;
        if (ok) ok = mbar_wait(sm, &sm->full[warp][stage], (used / kStages) & 1, a.status);
        if (!ok) break;
        const uint32_t st = smem_u32(sm->ring[warp][stage]);
        float x[2][NT][4];
#pragma unroll
        for (int gr = 0; gr < 2; ++gr) {
          const uint32_t k_at = st + gr * kGranuleBytes + kappa * kCodeBytes + t4 * 16;
          const uint4 ka = lds128(k_at), kb = lds128(k_at + 8 * kCodeBytes);
          const uint32_t p_at = st + gr * kGranuleBytes + kGranuleParams + kappa * 4;
          const uint32_t pa = lds32(p_at), pb = lds32(p_at + 32);
          float s[NT][4];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[nt][e] = 0.f;
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            uint32_t a0[4], a1[4];
            unpack4(w == 0 ? ka.x : w == 1 ? ka.y : w == 2 ? ka.z : ka.w, a0);
            unpack4(w == 0 ? kb.x : w == 1 ? kb.y : w == 2 ? kb.z : kb.w, a1);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              mma16816(s[nt], a0[0], a1[0], a0[1], a1[1], qf[nt][4 * w], qf[nt][4 * w + 1]);
              mma16816(s[nt], a0[2], a1[2], a0[3], a1[3], qf[nt][4 * w + 2], qf[nt][4 * w + 3]);
            }
          }
          const float2 fa = __half22float2(*reinterpret_cast<const __half2*>(&pa)), fb = __half22float2(*reinterpret_cast<const __half2*>(&pb));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              x[gr][nt][i] = rs[nt][i] * fmaf(fa.x, s[nt][i], fa.y * sq[nt][i]);
              x[gr][nt][i + 2] = rs[nt][i] * fmaf(fb.x, s[nt][i + 2], fb.y * sq[nt][i]);
            }
        }
        const bool ends = key0 + kRowsStep > u.L;
        if (ends || (a.window > 0 && key0 < latest)) {  // some keys are not there, or not every row's
#pragma unroll
          for (int gr = 0; gr < 2; ++gr)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int j = key0 + gr * kGranule + kappa + 8 * e;
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                  if (j >= u.L || (j < begin[nt][i] && j >= a.sinks)) x[gr][nt][2 * e + i] = -INFINITY;
            }
        }
        uint32_t pf[2][NT][2];
        softmax_step<2, NT>(x, m, l, o, pf);
#pragma unroll
        for (int gr = 0; gr < 2; ++gr) {
          // the thread's four keys of the granule, in two pairs: operand columns 2 t4, 2 t4 + 1 and eight more
          const int ja = t4, jb = 4 + (t4 ^ 1);
          const uint32_t v_at = st + gr * kGranuleBytes + kGranuleV + g8 * 8;
          const uint32_t q_at = st + gr * kGranuleBytes + kGranuleParams + kGranule * 4;
          const uint2 wa = lds64(v_at + ja * kCodeBytes), wb = lds64(v_at + jb * kCodeBytes);
          const uint2 wc = lds64(v_at + (ja + 8) * kCodeBytes), wd = lds64(v_at + (jb + 8) * kCodeBytes);
          uint32_t pa = lds32(q_at + ja * 4), pb = lds32(q_at + jb * 4), pc = lds32(q_at + ja * 4 + 32), pd = lds32(q_at + jb * 4 + 32);
          if (ends) {  // what lies behind the prefix may be anything: zeros
            const int j = key0 + gr * kGranule;
            pa = j + ja < u.L ? pa : 0u;
            pb = j + jb < u.L ? pb : 0u;
            pc = j + ja + 8 < u.L ? pc : 0u;
            pd = j + jb + 8 < u.L ? pd : 0u;
          }
          const uint32_t s_ab = __byte_perm(pa, pb, 0x5410), m_ab = __byte_perm(pa, pb, 0x7632);
          const uint32_t s_cd = __byte_perm(pc, pd, 0x5410), m_cd = __byte_perm(pc, pd, 0x7632);
#pragma unroll
          for (int half = 0; half < 2; ++half) {  // channels 4 half .. 4 half + 3 of the thread's two words
            const int sel = half ? 0x7632 : 0x5410;
            uint32_t v0[4], v1[4], v2[4], v3[4];
            unpack4(__byte_perm(wa.x, wb.x, sel), v0);
            unpack4(__byte_perm(wa.y, wb.y, sel), v1);
            unpack4(__byte_perm(wc.x, wd.x, sel), v2);
            unpack4(__byte_perm(wc.y, wd.y, sel), v3);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const uint32_t b0 = hfma2_bits(v0[c], s_ab, m_ab), b1 = hfma2_bits(v1[c], s_ab, m_ab);
              const uint32_t b2 = hfma2_bits(v2[c], s_cd, m_cd), b3 = hfma2_bits(v3[c], s_cd, m_cd);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) mma16816(o[nt][4 * half + c], b0, b1, b2, b3, pf[gr][nt][0], pf[gr][nt][1]);
            }
          }
        }
        __syncwarp();  // every lane has read the stage
        ++used;
        load_next();
        continue;
      }
      // ---- 32 rows of the tree, from global memory: 16 at a time
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
            mma16816(s[0][nt], f0[0], f1[0], f0[1], f1[1], qf[nt][4 * c], qf[nt][4 * c + 1]);
            mma16816(s[0][nt], f0[2], f1[2], f0[3], f1[3], qf[nt][4 * c + 2], qf[nt][4 * c + 3]);
          }
        }
        // V, in pairs of rows (2 t4, 2 t4 + 1 and eight more).  A row with a value that is not finite in half precision counts as zeros, so that
        // it stays out of the rows that do not see it; those that do become NaN.
        uint32_t v[2][16], not_finite = 0;
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const int j = n0 + 2 * t4 + 8 * y;
          uint4 x0[2], x1[2];
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            x0[z] = x1[z] = make_uint4(0u, 0u, 0u, 0u);
            if (j < a.n) x0[z] = reinterpret_cast<const uint4*>(v_rows + j * a.t_tok)[2 * g8 + z];
            if (j + 1 < a.n) x1[z] = reinterpret_cast<const uint4*>(v_rows + (j + 1) * a.t_tok)[2 * g8 + z];
          }
          uint32_t big = 0;  // the largest exponents of the two rows
#pragma unroll
          for (int z = 0; z < 2; ++z)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t h0 = to_half2<kBf16>(i == 0 ? x0[z].x : i == 1 ? x0[z].y : i == 2 ? x0[z].z : x0[z].w);
              const uint32_t h1 = to_half2<kBf16>(i == 0 ? x1[z].x : i == 1 ? x1[z].y : i == 2 ? x1[z].z : x1[z].w);
              v[y][8 * z + 2 * i] = __byte_perm(h0, h1, 0x5410);
              v[y][8 * z + 2 * i + 1] = __byte_perm(h0, h1, 0x7632);
              big = __vmaxu2(big, __vmaxu2(v[y][8 * z + 2 * i] & 0x7c007c00u, v[y][8 * z + 2 * i + 1] & 0x7c007c00u));
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
        uint32_t pf[1][NT][2];
        softmax_step<1, NT>(s, m, l, o, pf);
        if (not_finite != 0) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 2; ++i)
              if (seen[nt][i] & not_finite) l[nt][i] = NAN;
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int mt = 0; mt < 8; ++mt) mma16816(o[nt][mt], v[0][mt], v[0][8 + mt], v[1][mt], v[1][8 + mt], pf[0][nt][0], pf[0][nt][1]);
      }
    }

    // ---- the four warps' rows meet
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) l[nt][i] += __shfl_xor_sync(0xffffffffu, l[nt][i], d);
        const int row = nt * 8 + 2 * t4 + i;
        if (g8 == 0) sm->ml[warp][row] = make_float2(m[nt][i], l[nt][i]);
        float4* to = reinterpret_cast<float4*>(&sm->o[warp][row][16 * g8]);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          to[c] = make_float4(o[nt][4 * c][i], o[nt][4 * c + 1][i], o[nt][4 * c + 2][i], o[nt][4 * c + 3][i]);
          to[c + 2] = make_float4(o[nt][4 * c][i + 2], o[nt][4 * c + 1][i + 2], o[nt][4 * c + 2][i + 2], o[nt][4 * c + 3][i + 2]);
        }
      }
    __syncthreads();
    const bool whole = pos == u.begin && seg_end == u.end;
    const int c = threadIdx.x;
    using T = typename std::conditional<kBf16, __nv_bfloat16, __half>::type;
    auto write_row = [&](int row, float M, float sum, float acc) {
      const int rw = row0 + row, nd = rw / a.group, h = u.g * a.group + rw - nd * a.group;
      reinterpret_cast<T*>(a.out + u.r * a.o_req + nd * a.o_tok + h * a.o_head)[c] = from_float<T>(acc / sum);
      if (a.lse != nullptr && c == 0) a.lse[((int64_t)u.r * a.Hq + h) * a.n + nd] = (M + log2f(sum)) * kLn2;
    };
    const int64_t slot = (int64_t)kv4_slot(ranges, blockIdx.x, u.begin) * a.row_tile;
    for (int row = 0; row < live_rows; ++row) {
      float M = -INFINITY;
#pragma unroll
      for (int w = 0; w < kRowsWarps; ++w) M = fmaxf(M, sm->ml[w][row].x);
      float sum = 0.f, acc = 0.f;
#pragma unroll
      for (int w = 0; w < kRowsWarps; ++w) {
        const float2 ml = sm->ml[w][row];
        const float f = ml.x == -INFINITY ? 0.f : ex2(ml.x - M);
        sum = fmaf(ml.y, f, sum);
        acc = fmaf(sm->o[w][row][c], f, acc);
      }
      if (whole) {
        write_row(row, M, sum, acc);
      } else {
        a.ws_o[(slot + row) * kHeadDim + c] = acc;
        if (c == 0) a.ws_ml[slot + row] = make_float2(M, sum);
      }
    }
    if (!whole) {
      // The piece is counted; the CTA that counts the last one adds them all, in the order of their CTAs.  Nobody waits.
      const Kv4Pieces pieces = kv4_pieces(ranges, u);
      __threadfence();
      __syncthreads();
      if (c == 0) sm->last = atomicAdd(a.ws_count + 2 * pieces.first, 1) == pieces.last - pieces.first;
      __syncthreads();
      if (sm->last) {
        __threadfence();
        for (int row = 0; row < live_rows; ++row) {
          float M = -INFINITY;
          for (int x = pieces.first; x <= pieces.last; ++x) M = fmaxf(M, __ldcg(a.ws_ml + (int64_t)kv4_slot(ranges, x, u.begin) * a.row_tile + row).x);
          float sum = 0.f, acc = 0.f;
          for (int x = pieces.first; x <= pieces.last; ++x) {
            const int64_t s = (int64_t)kv4_slot(ranges, x, u.begin) * a.row_tile + row;
            const float2 ml = __ldcg(a.ws_ml + s);
            const float f = ml.x == -INFINITY ? 0.f : ex2(ml.x - M);
            sum = fmaf(ml.y, f, sum);
            acc = fmaf(__ldcg(a.ws_o + s * kHeadDim + c), f, acc);
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
