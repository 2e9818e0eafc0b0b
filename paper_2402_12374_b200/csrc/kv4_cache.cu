// seq_tree_kv4_append, seq_tree_kv4_read: rows of 16 bits to and from the 4-bit pages (the format: include/seq_tree.h).
//
// Half a warp has a row (128 channels, 16 bytes a lane): its maximum and minimum as one packed pair (max, -min) by four shuffles, the
// codes of a lane's eight channels are one 32-bit word, the row's 64 bytes one store.  A half-warp walks 16 consecutive rows of
// one (layer, request, kv head, K or V) with the 16 page numbers (and path entries) looked up at once, a lane each; the append has
// four rows in flight, the read, whose loads are smaller, eight.
// Bound by HBM for prompts, by latency for paths.  Blocks are in the order (16-row chunk, layer, request, heads), so those behind a
// request's count, which have nothing to do, come last.
#include "kv4.cuh"

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

// The eight codes of a lane's channels.  Quotients are taken as products with the reciprocal (off by less than 3e-6 at +-8); where
// one lies so near the middle between two codes that this could decide, they are divided.
__device__ __forceinline__ uint32_t quantise8(const float* v, float scale, float mid) {
  constexpr float kMagic = 12582920.f;  // 1.5 * 2^23 + 8: adding it rounds to a whole number, even in the middle, 8 more in the last bits
  float inv;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(scale));
  inv = scale > 0.f ? inv : 0.f;
  float off = 0.f;
  float c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float d = v[i] - mid;
    c[i] = fmaf(d, inv, kMagic);
    off = fmaxf(off, fabsf(fmaf(d, inv, kMagic - c[i])));
    c[i] = fminf(fmaxf(c[i], kMagic - 8.f), kMagic + 7.f);
  }
  if (off > 0.499995f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = fminf(fmaxf(scale > 0.f ? __fdiv_rn(v[i] - mid, scale) : 0.f, -8.f), 7.f) + kMagic;
  }
  // the last bits of each, four apart; what else the numbers hold is the same and taken off
  uint32_t word = 0, rest = 0;
#pragma unroll
  for (int i = 7; i >= 0; --i) {
    word = word * 16u + __float_as_uint(c[i]);
    rest = rest * 16u + 0x4b400000u;
  }
  return word - rest;
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
  const unsigned half = 0xffffu << (threadIdx.x & 16);
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
  if (i0 >= m || item >= 2 * a.heads) return;
  const int g = item >> 1, which = item & 1;

  // lane j: row i0 + j's page, its place there and its row
  int page = -1, node = 0;
  if (i0 + lane < m) {
    const int t = len + i0 + lane;
    page = a.table[r * a.table_stride + t / a.page_size];
    if (page < 0 || page >= a.num_pages) {
      if (l == 0 && item == 0) dev_flag(a.status, SEQ_DEV_BAD_PAGE);
      page = -1;
    }
    node = kAppend && a.path != nullptr ? a.path[r * a.path_stride + i0 + lane] : i0 + lane;
  }
  const uint8_t* rows = (which ? a.v : a.k) + l * a.s_layer + r * a.s_req + g * a.s_head + 16 * lane;
  uint8_t* pool = a.pages + l * a.layer_stride + (int64_t)g * a.page_size * 136;
  const int rows_here = min(kChunkRows, m - i0);
  constexpr int kRowsInFlight = kAppend ? 4 : 8;
  for (int j0 = 0; j0 < rows_here; j0 += kRowsInFlight) {
    uint4 x[kRowsInFlight];
    uint8_t* at[kRowsInFlight];  // the row's codes; the row's (scale, mid) at `params`
    int params[kRowsInFlight];
#pragma unroll
    for (int u = 0; u < kRowsInFlight; ++u) {
      const int j = j0 + u;
      const int p = __shfl_sync(half, page, j, 16), nd = __shfl_sync(half, node, j, 16);
      const int t = len + i0 + j, in_page = t & (a.page_size - 1), row = in_page & (kGranule - 1);
      at[u] = p < 0 ? nullptr : pool + p * a.page_stride + (int64_t)(in_page / kGranule) * kGranuleBytes + which * kGranuleV + row * kCodeBytes;
      params[u] = kGranuleParams + which * (kGranule * 4) - which * kGranuleV - row * kCodeBytes + row * 4;
      x[u] = make_uint4(0u, 0u, 0u, 0u);
      if (at[u] == nullptr) continue;
      if (kAppend) {
        x[u] = *reinterpret_cast<const uint4*>(rows + nd * a.s_tok);
      } else {
        x[u].x = *reinterpret_cast<const uint32_t*>(at[u] + 4 * lane);
        x[u].y = *reinterpret_cast<const uint32_t*>(at[u] + params[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < kRowsInFlight; ++u) {
      if (at[u] == nullptr) continue;  // (the same for the whole half)
      if (kAppend) {
        float v[8];
        widen8<T>(x[u], v);
        uint32_t both = extremes<T>(x[u]);
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) both = max_pair<T>(both, __shfl_xor_sync(half, both, o, 16));
        float hi, lo;
        if (std::is_same<T, __nv_bfloat16>::value) {
          hi = __uint_as_float(both << 16);
          lo = -__uint_as_float(both & 0xffff0000u);
        } else {
          const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&both));
          hi = f.x;
          lo = -f.y;
        }
        const bool fine = fabsf(hi) <= kLargest && fabsf(lo) <= kLargest;  // (false for a NaN)
        // halves, so that the difference cannot overflow; it is exact in fp32 but for magnitudes far apart
        __half2 sm = __floats2half2_rn(__fdiv_rn(hi * 0.5f - lo * 0.5f, 7.5f), 0.f);
        sm.y = __float2half_rn(__low2float(sm) * 8.f + lo);
        if (!fine) {
          sm = __floats2half2_rn(0.f, 0.f);
          if (lane == 0) dev_flag(a.status, SEQ_DEV_NONFINITE);
        }
        const uint32_t word = fine ? quantise8(v, __low2float(sm), __high2float(sm)) : 0x88888888u;
        *reinterpret_cast<uint32_t*>(at[u] + 4 * lane) = word;
        if (lane == 0) *reinterpret_cast<__half2*>(at[u] + params[u]) = sm;
      } else {
        const float2 sm = __half22float2(*reinterpret_cast<const __half2*>(&x[u].y));
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float c0 = __uint_as_float(((x[u].x >> (8 * i)) & 15u) | 0x4b000000u) - 8388616.f;  // the nibble less 8
          const float c1 = __uint_as_float(((x[u].x >> (8 * i + 4)) & 15u) | 0x4b000000u) - 8388616.f;
          const T lo = from_float<T>(fmaf(sm.x, c0, sm.y)), hi = from_float<T>(fmaf(sm.x, c1, sm.y));
          o[i] = (uint32_t)*reinterpret_cast<const uint16_t*>(&lo) | ((uint32_t)*reinterpret_cast<const uint16_t*>(&hi) << 16);
        }
        *reinterpret_cast<uint4*>(const_cast<uint8_t*>(rows) + (int64_t)(i0 + j0 + u) * a.s_tok) = make_uint4(o[0], o[1], o[2], o[3]);
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
  return launch_rows<false>(p, stream);
}
