// seq_tree_kv4_append, seq_tree_kv4_read: rows of 16 bits to and from the 4-bit pages (the format: include/seq_tree.h).
//
// Half a warp has a row (128 channels, 16 bytes a lane): its maximum and minimum as one packed pair (max, -min) by four shuffles, the
// codes of a lane's eight channels are one 32-bit word, the row's 64 bytes one store.  A half-warp walks 16 consecutive rows of
// one (layer, request, kv head, K or V); the 16 rows' places are looked up at once, a lane each, and their (scale, mid) worked out
// and stored by a lane each, four rows at a time: done by every lane for every row, that and the addresses were half of the
// instructions, which bind the kernel before HBM does (two prompts of up to 4001 rows, 4 layers of 32 heads: append 346 -> 175 us,
// still at three quarters of the issue slots; read 146 -> 107, at two thirds of HBM).
// Paths are bound by latency.  Blocks are in the order (16-row chunk, layer, request, heads), so those behind a
// request's count, which have nothing to do, come last.
#include "kv4.cuh"
#include "umma.cuh"

namespace seqtree {

constexpr int kRowThreads = 256;
constexpr int kChunkRows = 16;
constexpr float kLargest = 65504.f;  // of half precision

struct RowsArgs {
  int32_t layers, batch, n_rows, heads, max_pages, num_pages, page_size;
  int32_t groups;  // blocks for the (kv head, K or V) pairs of a (layer, request)
  const uint8_t* k; const uint8_t* v;  // (written by the read)
  int64_t s_layer, s_req, s_tok, s_head;  // bytes
  uint8_t* pages; int64_t page_stride, layer_stride;
  const int32_t* table; int64_t table_stride;
  const int32_t* lengths; const int32_t* count; const int32_t* path; int64_t path_stride;
  int32_t* new_lengths; int32_t* status;
};

template <typename T>
__device__ __forceinline__ void widen8(uint4 x, float* v) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (sizeof(T) == 2 && std::is_same<T, __nv_bfloat16>::value) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    } else {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      v[2 * i] = f.x;
      v[2 * i + 1] = f.y;
    }
  }
}

// (a, b) -> (max, max), NaN if either is one
template <typename T>
__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b) {
  uint32_t d;
  if (std::is_same<T, __nv_bfloat16>::value) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  else asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// The largest of a lane's eight channels and the largest of their negatives, as a pair
template <typename T>
__device__ __forceinline__ uint32_t extremes(uint4 x) {
  const uint32_t hi = max_pair<T>(max_pair<T>(x.x, x.y), max_pair<T>(x.z, x.w));
  const uint32_t n = 0x80008000u;
  const uint32_t lo = max_pair<T>(max_pair<T>(x.x ^ n, x.y ^ n), max_pair<T>(x.z ^ n, x.w ^ n));
  return max_pair<T>(__byte_perm(hi, lo, 0x5410), __byte_perm(hi, lo, 0x7632));
}

// The eight codes of a lane's channels.  Quotients are taken as products with the reciprocal (off by less than 3e-6 at +-8); `near`: one
// lies so near the middle between two codes that this could decide, or outside the codes (where a row's mid is large against its
// scale, so that mid's rounding counts): such lanes divide and clamp.
constexpr float kMagic = 12582920.f;  // 1.5 * 2^23 + 8: adding it rounds to a whole number, even in the middle, 8 more in the last bits
__device__ __forceinline__ uint32_t join8(const float* c, uint32_t& outside) {
  // the last bits of each, four apart; what else the numbers hold is the same and taken off
  uint32_t word = 0, rest = 0;
  outside = 0;
#pragma unroll
  for (int i = 7; i >= 0; --i) {
    const uint32_t bits = __float_as_uint(c[i]);
    word = word * 16u + bits;
    rest = rest * 16u + 0x4b400000u;
    outside |= bits ^ 0x4b400000u;  // (above 15: not a code)
  }
  return word - rest;
}
__device__ __forceinline__ uint32_t quantise8(const float* v, float inv, float mid, bool& near) {
  const uint64_t inv2 = pair_of(inv, inv), mid2 = pair_of(-mid, -mid), magic = pair_of(kMagic, kMagic), minus = pair_of(-1.f, -1.f);
  float off = 0.f, c[8];
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const uint64_t d = add2(pair_of(v[i], v[i + 1]), mid2), y = fma2(d, inv2, magic);
    float a, b;
    unpair(fma2(d, inv2, fma2(y, minus, magic)), a, b);  // how far from the whole number
    off = max3(off, fabsf(a), fabsf(b));
    unpair(y, c[i], c[i + 1]);
  }
  uint32_t outside;
  const uint32_t word = join8(c, outside);
  near = off > 0.499995f || outside > 15u;
  return word;
}
__device__ __forceinline__ uint32_t divide8(const float* v, float scale, float mid) {
  float c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = fminf(fmaxf((scale > 0.f ? __fdiv_rn(v[i] - mid, scale) : 0.f) + kMagic, kMagic - 8.f), kMagic + 7.f);
  uint32_t outside;
  return join8(c, outside);
}
__device__ __forceinline__ uint64_t shfl64(uint64_t x, int from) {
  const uint32_t lo = __shfl_sync(0xffffffffu, (uint32_t)x, from, 16), hi = __shfl_sync(0xffffffffu, (uint32_t)(x >> 32), from, 16);
  return (uint64_t)hi << 32 | lo;
}

// How many rows of request r there are; -1: none, for a reason that is told once per call
__device__ __forceinline__ int rows_of(const RowsArgs& a, int r, int len, bool tell) {
  if (len < 0) return -1;
  const int m = a.count != nullptr ? a.count[r] : a.n_rows;
  if (m < 0 || m > a.n_rows) {
    if (tell) dev_flag(a.status, SEQ_DEV_BAD_PATH);
    return -1;
  }
  if ((int64_t)len + m > (int64_t)a.max_pages * a.page_size) {
    if (tell) dev_flag(a.status, SEQ_DEV_BAD_LENGTH);
    return -1;
  }
  return m;
}

template <typename T, bool kAppend>
__global__ void __launch_bounds__(kRowThreads) kv4_rows_copy_kernel(const RowsArgs a) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int chunk = blockIdx.y;
  const int lr = blockIdx.x / a.groups, l = lr / a.batch, r = lr - l * a.batch;
  const int item = (blockIdx.x - lr * a.groups) * (kRowThreads / 16) + (threadIdx.x >> 4);  // (kv head, K or V)
  const int lane = threadIdx.x & 15;
  const bool first_block = chunk == 0 && blockIdx.x - lr * a.groups == 0 && l == 0;
  const int len = a.lengths != nullptr ? a.lengths[r] : 0;
  int m = rows_of(a, r, len, first_block && threadIdx.x == 0);
  // a path entry outside the rows: the whole request is left alone, so every block looks at all of it
  if (kAppend && a.path != nullptr && m > 0) {
    int bad = 0;
    for (int i = threadIdx.x; i < m; i += kRowThreads) {
      const int node = a.path[r * a.path_stride + i];
      bad |= node < 0 || node >= a.n_rows;
    }
    if (__syncthreads_or(bad)) {
      if (first_block && threadIdx.x == 0) dev_flag(a.status, SEQ_DEV_BAD_PATH);
      m = -1;
    }
  }
  if (kAppend && first_block && threadIdx.x == 0 && a.new_lengths != nullptr) a.new_lengths[r] = len + max(m, 0);
  const int i0 = chunk * kChunkRows;
  if (i0 >= m) return;
  const bool live = item < 2 * a.heads;  // (both halves of a warp go through everything)
  const int g = min(item >> 1, a.heads - 1), which = item & 1;

  // lane j: where row i0 + j's codes and its (scale, mid) are (0: nowhere), and where the row is
  uint64_t codes = 0;
  uint32_t* params = nullptr;
  uint64_t row = 0;
  if (i0 + lane < m) {
    const int t = len + i0 + lane, in_page = t & (a.page_size - 1), line = in_page & (kGranule - 1);
    const int page = a.table[r * a.table_stride + t / a.page_size];
    if (page < 0 || page >= a.num_pages) {
      if (l == 0 && item == 0) dev_flag(a.status, SEQ_DEV_BAD_PAGE);
    } else if (live) {
      uint8_t* granule = a.pages + l * a.layer_stride + page * a.page_stride + (int64_t)g * a.page_size * 136 + in_page / kGranule * kGranuleBytes;
      codes = reinterpret_cast<uint64_t>(granule + which * kGranuleV + line * kCodeBytes);
      params = reinterpret_cast<uint32_t*>(granule + kGranuleParams + which * (kGranule * 4) + line * 4);
    }
    row = (uint64_t)((kAppend && a.path != nullptr ? a.path[r * a.path_stride + i0 + lane] : i0 + lane) * a.s_tok);
  }
  const uint8_t* rows = (which ? a.v : a.k) + l * a.s_layer + r * a.s_req + g * a.s_head + 16 * lane;
  const int rows_here = min(kChunkRows, m - i0);
  if (kAppend) {
    uint32_t mine = 0;  // lane j: row j's (scale, mid)
#pragma unroll 1
    for (int j0 = 0; j0 < rows_here; j0 += 4) {
      uint4 x[4];
      uint32_t both[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) x[u] = *reinterpret_cast<const uint4*>(rows + shfl64(row, j0 + u));  // (rows behind the last: row 0)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        both[u] = extremes<T>(x[u]);
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) both[u] = max_pair<T>(both[u], __shfl_xor_sync(0xffffffffu, both[u], o, 16));
      }
      // lane j works out row j0 + (j & 3)'s scale and mid
      const uint32_t b = (lane & 2) ? ((lane & 1) ? both[3] : both[2]) : ((lane & 1) ? both[1] : both[0]);
      float hi, lo;
      if (std::is_same<T, __nv_bfloat16>::value) {
        hi = __uint_as_float(b << 16);
        lo = -__uint_as_float(b & 0xffff0000u);
      } else {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&b));
        hi = f.x;
        lo = -f.y;
      }
      const bool fine = fabsf(hi) <= kLargest && fabsf(lo) <= kLargest;  // (false for a NaN)
      // halves, so that the difference cannot overflow; it is exact in fp32 but for magnitudes far apart
      __half2 sm = __floats2half2_rn(__fdiv_rn(hi * 0.5f - lo * 0.5f, 7.5f), 0.f);
      const float scale = __low2float(sm);
      sm.y = __float2half_rn(scale * 8.f + lo);
      const float mid = __high2float(sm);
      float inv;
      asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(scale));
      inv = scale > 0.f ? inv : 0.f;
      const bool some_bad = __any_sync(0xffffffffu, !fine);
      if ((lane >> 2) == (j0 >> 2)) {
        mine = fine ? *reinterpret_cast<uint32_t*>(&sm) : 0u;
        if (!fine && params != nullptr) dev_flag(a.status, SEQ_DEV_NONFINITE);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float iu = __shfl_sync(0xffffffffu, inv, u, 16), mu = __shfl_sync(0xffffffffu, mid, u, 16);
        float v[8];
        widen8<T>(x[u], v);
        bool near;
        uint32_t word = quantise8(v, iu, mu, near);
        if (__any_sync(0xffffffffu, near)) {
          const float su = __shfl_sync(0xffffffffu, scale, u, 16);
          if (near) word = divide8(v, su, mu);
        }
        if (some_bad && !__shfl_sync(0xffffffffu, (int)fine, u, 16)) word = 0x88888888u;
        const uint64_t to = shfl64(codes, j0 + u);
        if (to != 0) *reinterpret_cast<uint32_t*>(to + 4 * lane) = word;
      }
    }
    if (params != nullptr) *params = mine;
  } else {
    const uint32_t sm = params != nullptr ? *params : 0u;
    uint8_t* out = const_cast<uint8_t*>(rows);
#pragma unroll 1
    for (int j0 = 0; j0 < rows_here; j0 += 8) {
      uint32_t x[8];
      uint64_t from[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        from[u] = shfl64(codes, j0 + u);
        x[u] = from[u] != 0 ? *reinterpret_cast<const uint32_t*>(from[u] + 4 * lane) : 0u;
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const uint32_t p = __shfl_sync(0xffffffffu, sm, j0 + u, 16);
        uint32_t c[4];  // channels (0, 4), (1, 5), (2, 6), (3, 7), less 8
        unpack4(x[u], c);
        uint4 o;
        if (std::is_same<T, __nv_bfloat16>::value) {
          const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&p));
          float2 y[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            y[i] = __half22float2(*reinterpret_cast<const __half2*>(&c[i]));
            y[i].x = fmaf(f.x, y[i].x, f.y);
            y[i].y = fmaf(f.x, y[i].y, f.y);
          }
          o = make_uint4(pack2<true>(y[0].x, y[1].x), pack2<true>(y[2].x, y[3].x), pack2<true>(y[0].y, y[1].y), pack2<true>(y[2].y, y[3].y));
        } else {  // (the fused multiply-add of halves rounds once, too)
          const uint32_t s = __byte_perm(p, 0u, 0x1010), m2 = __byte_perm(p, 0u, 0x3232);
#pragma unroll
          for (int i = 0; i < 4; ++i) c[i] = hfma2_bits(c[i], s, m2);
          o = make_uint4(__byte_perm(c[0], c[1], 0x5410), __byte_perm(c[2], c[3], 0x5410), __byte_perm(c[0], c[1], 0x7632), __byte_perm(c[2], c[3], 0x7632));
        }
        if (from[u] != 0) *reinterpret_cast<uint4*>(out + (int64_t)(i0 + j0 + u) * a.s_tok) = o;
      }
    }
  }
}

static int check_rows(const seq_tree_kv4_append_params* p) {
  if (p == nullptr || p->k == nullptr || p->v == nullptr || p->pages == nullptr || p->page_table == nullptr) return SEQ_ERR_INVALID_ARG;
  if (p->num_layers < 1 || p->batch < 1 || p->batch > SEQ_MAX_BATCH || p->n_rows < 1 || p->num_kv_heads < 1 || p->num_pages < 1 || p->max_pages < 1)
    return SEQ_ERR_INVALID_ARG;
  if (p->head_dim != kHeadDim || !kv4_page_size_ok(p->page_size) || (p->dtype != SEQ_F16 && p->dtype != SEQ_BF16)) return SEQ_ERR_UNSUPPORTED;
  // a request's tokens and a launch's blocks are counted in 32 bits
  if (p->n_rows > (1 << 20) || p->num_layers > 1024 || p->num_kv_heads > 1024 || (int64_t)p->max_pages * p->page_size > (1 << 30))
    return SEQ_ERR_INVALID_ARG;
  const int64_t part = (int64_t)p->num_kv_heads * p->page_size * 136;
  if (p->page_stride_bytes < part || p->page_stride_bytes % 16 != 0 || p->table_stride < p->max_pages) return SEQ_ERR_INVALID_ARG;
  if (p->num_layers > 1 && (p->layer_stride_bytes < part || p->layer_stride_bytes % 16 != 0)) return SEQ_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(p->k) % 16 != 0 || reinterpret_cast<uintptr_t>(p->v) % 16 != 0 || reinterpret_cast<uintptr_t>(p->pages) % 16 != 0)
    return SEQ_ERR_INVALID_ARG;
  for (int64_t s : {p->stride_layer, p->stride_req, p->stride_tok, p->stride_head})
    if (s < 0 || s % 8 != 0) return SEQ_ERR_INVALID_ARG;
  if (p->path != nullptr && p->path_stride < p->n_rows) return SEQ_ERR_INVALID_ARG;
  return SEQ_OK;
}

template <bool kAppend>
static int launch_rows(const seq_tree_kv4_append_params* p, void* stream) {
  RowsArgs a;
  a.layers = p->num_layers; a.batch = p->batch; a.n_rows = p->n_rows; a.heads = p->num_kv_heads;
  a.max_pages = p->max_pages; a.num_pages = p->num_pages; a.page_size = p->page_size;
  a.groups = (2 * p->num_kv_heads + kRowThreads / 16 - 1) / (kRowThreads / 16);
  a.k = static_cast<const uint8_t*>(p->k); a.v = static_cast<const uint8_t*>(p->v);
  a.s_layer = 2 * p->stride_layer; a.s_req = 2 * p->stride_req; a.s_tok = 2 * p->stride_tok; a.s_head = 2 * p->stride_head;
  a.pages = static_cast<uint8_t*>(p->pages); a.page_stride = p->page_stride_bytes; a.layer_stride = p->layer_stride_bytes;
  a.table = p->page_table; a.table_stride = p->table_stride;
  a.lengths = p->lengths; a.count = p->count; a.path = p->path; a.path_stride = p->path_stride;
  a.new_lengths = p->new_lengths; a.status = p->dev_status;
  const int64_t blocks = (int64_t)p->num_layers * p->batch * a.groups;
  const int chunks = (p->n_rows + kChunkRows - 1) / kChunkRows;
  if (blocks > 0x7fffffff || chunks > 65535) return SEQ_ERR_INVALID_ARG;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks, chunks);
  cfg.blockDim = dim3(kRowThreads);
  cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute early[1];
  early[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = early;
  cfg.numAttrs = 1;
  if (p->dtype == SEQ_BF16) SEQ_CUDA_OK(cudaLaunchKernelEx(&cfg, kv4_rows_copy_kernel<__nv_bfloat16, kAppend>, a));
  else SEQ_CUDA_OK(cudaLaunchKernelEx(&cfg, kv4_rows_copy_kernel<__half, kAppend>, a));
  return SEQ_OK;
}

}  // namespace seqtree

using namespace seqtree;

extern "C" int seq_tree_kv4_append(const seq_tree_kv4_append_params* p, void* stream) {
  const int rc = check_rows(p);
  if (rc != SEQ_OK) return rc;
  if (p->lengths == nullptr || p->lengths == p->new_lengths) return SEQ_ERR_INVALID_ARG;
  return launch_rows<true>(p, stream);
}

extern "C" int seq_tree_kv4_read(const seq_tree_kv4_append_params* p, void* stream) {
  const int rc = check_rows(p);
  if (rc != SEQ_OK) return rc;
  if (p->path != nullptr || p->new_lengths != nullptr) return SEQ_ERR_INVALID_ARG;
  if ((p->num_layers > 1 && p->stride_layer == 0) || (p->batch > 1 && p->stride_req == 0) || (p->n_rows > 1 && p->stride_tok == 0) ||
      (p->num_kv_heads > 1 && p->stride_head == 0))
    return SEQ_ERR_INVALID_ARG;  // rows over one another
  return launch_rows<false>(p, stream);
}
