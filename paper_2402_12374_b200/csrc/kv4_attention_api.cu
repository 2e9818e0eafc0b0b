// seq_tree_kv4_attention: checks and the choice of kernel.
#include "kv4_attention.cuh"
#include "umma.cuh"

#include <algorithm>

namespace seqtree {

// The pieces of the units that are cut.  A CTA has some rows of one unit (16 of the tiles kernel's, whose pieces are [channel / 4][row], 8 of the
// other's, [row][channel]), a thread eight channels of a row, or twice eight; four pieces, (m, l) and rows, are on their way at once (32 requests 54 -> 52 us against (m, l) first).
// The launch behind it is not let in early: its CTAs took the places that these leave first and were spread unevenly (32 requests of 8192
// tokens, launch after launch: 54 us, 74 with it).
template <bool kBf16, bool kTiles>
__global__ void __launch_bounds__(128) kv4_merge_kernel(const Kv4Args a) {
  constexpr int kRows = kTiles ? 16 : 8, kSets = kTiles ? 2 : 1, kFlight = 4;
  const int slices = a.row_tile / kRows, c = blockIdx.x / slices;
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4;
  const int row = (blockIdx.x - c * slices) * kRows + (kTiles ? x : y), set = kTiles ? y : x;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int4 cut = a.ws_cut[c];
  const int rg = cut.x / a.tiles, rw = (cut.x - rg * a.tiles) * a.row_tile + row;
  if (cut.x < 0 || rw >= a.rows) return;
  const int pieces = cut.z - c + 1;
  auto piece = [&](int p) -> int64_t { return (int64_t)(p == 0 ? cut.y : 2 * (c + p)) * a.row_tile; };
  float M = -INFINITY, sum = 0.f;
  float o[kSets][8];
#pragma unroll
  for (int s = 0; s < kSets; ++s)
#pragma unroll
    for (int e = 0; e < 8; ++e) o[s][e] = 0.f;
  for (int p0 = 0; p0 < pieces; p0 += kFlight) {
    float2 ml[kFlight];
    float4 v[kFlight][kSets][2];
#pragma unroll
    for (int p = 0; p < kFlight; ++p) {
      ml[p] = make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int s = 0; s < kSets; ++s) v[p][s][0] = v[p][s][1] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (p0 + p < pieces) {
        ml[p] = a.ws_ml[piece(p0 + p) + row];
        const float4* from = reinterpret_cast<const float4*>(a.ws_o + piece(p0 + p) * kHeadDim);
#pragma unroll
        for (int s = 0; s < kSets; ++s)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int quad = 2 * (set + 8 * s) + e;
            v[p][s][e] = from[kTiles ? quad * a.row_tile + row : row * (kHeadDim / 4) + quad];
          }
      }
    }
    float now = M;
#pragma unroll
    for (int p = 0; p < kFlight; ++p) now = fmaxf(now, ml[p].x);
    const float old = M == -INFINITY ? 0.f : ex2(M - now);
    M = now;
    sum *= old;
#pragma unroll
    for (int s = 0; s < kSets; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e) o[s][e] *= old;
#pragma unroll
    for (int p = 0; p < kFlight; ++p) {
      const float f = ml[p].x == -INFINITY ? 0.f : ex2(ml[p].x - M);
      sum = fmaf(ml[p].y, f, sum);
#pragma unroll
      for (int s = 0; s < kSets; ++s)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          o[s][4 * e] = fmaf(v[p][s][e].x, f, o[s][4 * e]);
          o[s][4 * e + 1] = fmaf(v[p][s][e].y, f, o[s][4 * e + 1]);
          o[s][4 * e + 2] = fmaf(v[p][s][e].z, f, o[s][4 * e + 2]);
          o[s][4 * e + 3] = fmaf(v[p][s][e].w, f, o[s][4 * e + 3]);
        }
    }
  }
  const float inv = 1.f / sum;
  const int r = rg / a.Hkv, nd = rw / a.group, h = (rg - r * a.Hkv) * a.group + rw - nd * a.group;
  uint8_t* out = a.out + r * a.o_req + nd * a.o_tok + h * a.o_head;
#pragma unroll
  for (int s = 0; s < kSets; ++s) {
    float z[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = o[s][kTiles ? ((e & 3) << 1) + (e >> 2) : e] * inv;  // (the tiles' columns are channels 0,4,1,5,2,6,3,7)
    *reinterpret_cast<uint4*>(out + 16 * (set + 8 * s)) = make_uint4(pack2<kBf16>(z[0], z[1]), pack2<kBf16>(z[2], z[3]), pack2<kBf16>(z[4], z[5]), pack2<kBf16>(z[6], z[7]));
  }
  if (a.lse != nullptr && set == 0) a.lse[((int64_t)r * a.Hq + h) * a.n + nd] = (M + log2f(sum)) * kLn2;
}

int launch_kv4_merge(const Kv4Args& a, bool bf16, bool tiles, cudaStream_t stream) {
  if (a.ctas < 2) return SEQ_OK;  // nothing is cut
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((a.ctas - 1) * (a.row_tile / (tiles ? 16 : 8)));  // (nothing that begins in the last range is)
  cfg.blockDim = dim3(128);
  cfg.stream = stream;
  cudaLaunchAttribute early[1];
  early[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = early;
  cfg.numAttrs = 1;
  SEQ_CUDA_OK(cudaLaunchKernelEx(&cfg, bf16 ? (tiles ? kv4_merge_kernel<true, true> : kv4_merge_kernel<true, false>)
                                            : (tiles ? kv4_merge_kernel<false, true> : kv4_merge_kernel<false, false>), a));
  return SEQ_OK;
}

Kv4Args kv4_args(const seq_tree_kv4_attention_params& p, int row_tile, int step, int unit_cost, int tree_cost) {
  Kv4Args a = {};
  a.batch = p.batch; a.n = p.n_tree; a.max_len = p.max_len; a.Hq = p.num_q_heads; a.Hkv = p.num_kv_heads;
  a.group = p.num_q_heads / p.num_kv_heads;
  a.rows = a.n * a.group;
  a.window = p.window; a.sinks = p.sinks;
  a.num_pages = p.num_pages; a.page_size = p.page_size;
  a.page_shift = p.page_size == 16 ? 4 : p.page_size == 32 ? 5 : p.page_size == 64 ? 6 : 7;
  a.q = static_cast<const uint8_t*>(p.q); a.q_req = 2 * p.q_stride_req; a.q_tok = 2 * p.q_stride_tok; a.q_head = 2 * p.q_stride_head;
  a.kt = static_cast<const uint8_t*>(p.k_tree); a.vt = static_cast<const uint8_t*>(p.v_tree);
  a.t_req = 2 * p.t_stride_req; a.t_tok = 2 * p.t_stride_tok; a.t_head = 2 * p.t_stride_head;
  a.pages = static_cast<const uint8_t*>(p.pages); a.page_stride = p.page_stride_bytes;
  a.table = p.page_table; a.table_stride = p.table_stride; a.lengths = p.lengths;
  a.mask = p.mask_bits; a.mask_wpr = p.mask_words_per_row; a.mask_req = p.mask_stride_req;
  a.out = static_cast<uint8_t*>(p.out); a.o_req = 2 * p.o_stride_req; a.o_tok = 2 * p.o_stride_tok; a.o_head = 2 * p.o_stride_head;
  a.lse = p.lse;
  a.scale_log2 = (p.softmax_scale > 0.f ? p.softmax_scale : 0.08838834764831845f) * kLog2e;
  a.status = p.dev_status;
  a.row_tile = row_tile;
  a.unit_cost = unit_cost;
  a.tree_cost = tree_cost;
  a.tiles = (a.rows + row_tile - 1) / row_tile;
  for (int m = 0; m < a.tiles; ++m) {
    const int nodes = std::min(a.n, ((m + 1) * row_tile + a.group - 1) / a.group), steps = (nodes + step - 1) / step;
    while (a.tree_steps < steps) a.tree_from[a.tree_steps++] = m;
    a.tree_total += kv4_tree_positions(a, steps);
  }
  return a;
}

static int check_kv4_attention(const seq_tree_kv4_attention_params* p) {
  if (p == nullptr || p->q == nullptr || p->k_tree == nullptr || p->v_tree == nullptr || p->pages == nullptr || p->page_table == nullptr ||
      p->lengths == nullptr || p->out == nullptr)
    return SEQ_ERR_INVALID_ARG;
  if (p->batch < 1 || p->batch > SEQ_MAX_BATCH || p->n_tree < 1 || p->n_tree > SEQ_MAX_TREE || p->max_len < 0 || p->num_kv_heads < 1 ||
      p->num_q_heads < 1 || p->num_q_heads % p->num_kv_heads != 0 || p->num_q_heads > 4096 || p->window < 0 || p->window > (1 << 30) || p->sinks < 0 ||
      p->sinks > (1 << 30) || p->num_pages < 1 || p->max_pages < 1)
    return SEQ_ERR_INVALID_ARG;
  if (p->head_dim != kHeadDim || !kv4_page_size_ok(p->page_size) || (p->dtype != SEQ_F16 && p->dtype != SEQ_BF16)) return SEQ_ERR_UNSUPPORTED;
  if (!(p->softmax_scale >= 0.f || p->softmax_scale < 0.f) || p->softmax_scale > 1e30f) return SEQ_ERR_INVALID_ARG;  // NaN, inf
  if (p->max_len > (1 << 30) || p->max_len > (int64_t)p->max_pages * p->page_size || p->table_stride < p->max_pages) return SEQ_ERR_INVALID_ARG;
  if (p->page_stride_bytes < (int64_t)p->num_kv_heads * p->page_size * 136 || p->page_stride_bytes % 16 != 0) return SEQ_ERR_INVALID_ARG;
  for (const void* x : {p->q, p->k_tree, p->v_tree, p->pages, static_cast<const void*>(p->out)})
    if (reinterpret_cast<uintptr_t>(x) % 16 != 0) return SEQ_ERR_INVALID_ARG;
  for (int64_t s : {p->q_stride_req, p->q_stride_tok, p->q_stride_head, p->t_stride_req, p->t_stride_tok, p->t_stride_head, p->o_stride_req,
                    p->o_stride_tok, p->o_stride_head})
    if (s < 0 || s % 8 != 0) return SEQ_ERR_INVALID_ARG;
  if ((p->batch > 1 && p->o_stride_req == 0) || (p->n_tree > 1 && p->o_stride_tok == 0) || (p->num_q_heads > 1 && p->o_stride_head == 0))
    return SEQ_ERR_INVALID_ARG;  // rows of out over one another
  if (p->mask_bits != nullptr && (p->mask_words_per_row < (p->n_tree + 31) / 32 || p->mask_stride_req < 0)) return SEQ_ERR_INVALID_ARG;
  return SEQ_OK;
}

}  // namespace seqtree

using namespace seqtree;

extern "C" size_t seq_tree_kv4_attention_workspace_bytes(const seq_tree_kv4_attention_params* p) {
  if (p == nullptr || p->num_kv_heads < 1 || p->num_q_heads < 1 || p->n_tree < 1) return 0;
  return kv4_few_rows(*p) ? kv4_rows_workspace_bytes(*p) : kv4_tiles_workspace_bytes();
}

extern "C" int seq_tree_kv4_attention(const seq_tree_kv4_attention_params* p, void* stream) {
  const int rc = check_kv4_attention(p);
  if (rc != SEQ_OK) return rc;
  const size_t need = seq_tree_kv4_attention_workspace_bytes(p);
  if (need > 0 && (p->workspace == nullptr || p->workspace_bytes < need)) return SEQ_ERR_WORKSPACE;
  if (need > 0 && reinterpret_cast<uintptr_t>(p->workspace) % 256 != 0) return SEQ_ERR_INVALID_ARG;
  return kv4_few_rows(*p) ? launch_kv4_rows(*p, static_cast<cudaStream_t>(stream)) : launch_kv4_tiles(*p, static_cast<cudaStream_t>(stream));
}
