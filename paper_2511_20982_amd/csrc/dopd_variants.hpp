// C ABI of the windowed and tree attention over the paged cache and of the calls
// that rearrange its pages (declarations and contracts in include/dopd_attn.h).
// Host side, as in dopd_attn.hip, whose helpers it uses: argument validation before
// any HIP call, planning from the host copies of the lengths, launches on the
// caller's stream.  No allocation, no synchronisation, no state.
#include "kernels/kv_pages.hpp"
#include "kernels/masked_common.hpp"
#include "kernels/masked_f32.hpp"
#include "kernels/masked_few.hpp"
#include "kernels/masked_mid.hpp"
#include "kernels/masked_rows.hpp"
#include "plan_masked.hpp"

namespace {

constexpr int kMaMaxWords = 32;  // of a draft's mask: trees of up to 1024 drafts

int elem_bytes_of(int32_t dtype) { return dtype == DOPD_FP32 ? 4 : dtype == DOPD_BF16 ? 2 : 1; }

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Lengths of a windowed or tree call; words: 32-bit words of a mask row (trees).
dopd_status check_masked_lens(const dopd_attn_shape* s, const int32_t* cu_host, const int32_t* prefix_host,
                              int32_t nreq, const dopd::MaskRule& rule, int32_t words) {
  if (nreq < 0) return DOPD_ERR_INVALID_SHAPE;
  if (rule.tree ? words < 1 || words > kMaMaxWords : rule.window < 1 || rule.sinks < 0) return DOPD_ERR_INVALID_SHAPE;
  if (nreq == 0) return DOPD_OK;
  if (!cu_host || !prefix_host) return DOPD_ERR_NULL_POINTER;
  if (cu_host[0] != 0) return DOPD_ERR_INVALID_SHAPE;
  const int64_t g = s->num_q_heads / s->num_kv_heads;
  for (int32_t r = 0; r < nreq; ++r) {
    const int64_t n = (int64_t)cu_host[r + 1] - cu_host[r];
    if (n < 0 || prefix_host[r] < 0 || prefix_host[r] + n > dopd::kMaMaxPos) return DOPD_ERR_INVALID_SHAPE;
    if (rule.tree && n > 32 * (int64_t)words) return DOPD_ERR_INVALID_SHAPE;
    if (n * g * g >= ((int64_t)1 << 32) || n * g > INT32_MAX / 2) return DOPD_ERR_INVALID_SHAPE;
  }
  return DOPD_OK;
}

// A window or a count of sinks beyond every position is as good as that.
dopd::MaskRule window_rule(int32_t window, int32_t sinks) {
  return dopd::MaskRule{0, std::min(window, dopd::kMaMaxPos), std::min(sinks, dopd::kMaMaxPos)};
}
dopd::MaskRule tree_rule() { return dopd::MaskRule{1, 0, 0}; }

dopd::MaPlan masked_plan(const dopd::MaKind& k, const dopd_attn_shape* s, const dopd::MaskRule& rule,
                         const int32_t* cu_host, const int32_t* prefix_host, int32_t nreq) {
  const dopd::MaCosts cost = k.which == dopd::kMaMany ? dopd::MaCosts{20, 12, 6}
                                                      : dopd::MaCosts{s->dtype == DOPD_FP8_E4M3 ? 12 : 8, 16, 4};
  const int g = s->num_q_heads / s->num_kv_heads;
  return dopd::ma_plan(rule, k, cu_host, prefix_host, nreq, g, s->num_kv_heads, machine_shape(), cost);
}

size_t masked_ws_bytes(const dopd_attn_shape* s, const dopd::MaskRule& rule, const int32_t* cu_host,
                       const int32_t* prefix_host, int32_t nreq) {
  if (s->dtype == DOPD_FP32) return 0;
  const dopd::MaSplit split = dopd::ma_split(rule, cu_host, prefix_host, nreq, s->num_q_heads / s->num_kv_heads, s->num_kv_heads,
                                              dopd::ma_mid(s->dtype == DOPD_FP8_E4M3, s->head_dim), machine_shape());
  size_t bytes = 0;
  for (int i = 0; i < 3; ++i) {
    const dopd::MaKind k = dopd::ma_kernel(split, i);
    bytes += dopd::ma_ws_bytes(masked_plan(k, s, rule, cu_host, prefix_host, nreq), k, s->head_dim);
  }
  return bytes;
}

size_t masked_workspace_size(const dopd_attn_shape* s, const dopd::MaskRule& rule, const int32_t* cu_host,
                             const int32_t* prefix_host, int32_t nreq) {
  // (any number of mask words: a call checks its own)
  if (check_shape(s) != DOPD_OK || check_masked_lens(s, cu_host, prefix_host, nreq, rule, kMaMaxWords) != DOPD_OK) return 0;
  return std::max<size_t>(256, masked_ws_bytes(s, rule, cu_host, prefix_host, nreq));
}

template <int D, bool KV8, bool TREE>
dopd_status launch_masked(const dopd::MaKind& k, const dopd::MaskedArgs& a, const dopd::MaPlan& p, hipStream_t strm) {
  const dim3 grid = grid_of(p.blocks), block(256), merge((unsigned)((p.nwg - 1) * (k.rows / dopd::merge_rows(k.which))));
  switch (k.which) {
    case dopd::kMaFew: hipLaunchKernelGGL((dopd::masked_few_kernel<D, KV8, TREE>), grid, block, 0, strm, a); break;
    case dopd::kMaMid:
      if constexpr (dopd::ma_mid(KV8, D)) hipLaunchKernelGGL((dopd::masked_mid_kernel<D, KV8, TREE>), grid, block, 0, strm, a);
      break;
    default: hipLaunchKernelGGL((dopd::masked_rows_kernel<D, KV8, TREE>), grid, block, 0, strm, a);
  }
  const dopd_status st = launch_status();
  if (st != DOPD_OK || p.nwg <= 1) return st;
  switch (k.which) {
    case dopd::kMaFew: hipLaunchKernelGGL((dopd::masked_merge_kernel<D, dopd::kMaFew>), merge, block, 0, strm, a); break;
    case dopd::kMaMid: hipLaunchKernelGGL((dopd::masked_merge_kernel<D, dopd::kMaMid>), merge, block, 0, strm, a); break;
    default: hipLaunchKernelGGL((dopd::masked_merge_kernel<D, dopd::kMaMany>), merge, block, 0, strm, a);
  }
  return launch_status();
}

template <bool KV8, bool TREE>
dopd_status launch_masked_d(const dopd::MaKind& k, const dopd::MaskedArgs& a, const dopd::MaPlan& p, int d, hipStream_t strm) {
  return d == 64 ? launch_masked<64, KV8, TREE>(k, a, p, strm) : launch_masked<128, KV8, TREE>(k, a, p, strm);
}

dopd_status masked_impl(const dopd_attn_shape* s, bool kv8, const void* q, const void* k_pool, const void* v_pool,
                        const float* k_scale, const float* v_scale, int32_t num_pages, const int32_t* page_table,
                        int32_t pt_stride, const int32_t* cu, const int32_t* cu_host, const int32_t* prefix,
                        const int32_t* prefix_host, int32_t nreq, const dopd::MaskRule& rule, const uint32_t* mask,
                        int32_t words, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  dopd_status st = kv8 ? check_shape(s) : check_shape_no_fp8(s);
  if (st != DOPD_OK) return st;
  if (kv8 && s->dtype != DOPD_FP8_E4M3) return DOPD_ERR_UNSUPPORTED;
  if (num_pages < 0 || pt_stride < 0) return DOPD_ERR_INVALID_SHAPE;
  st = check_masked_lens(s, cu_host, prefix_host, nreq, rule, words);
  if (st != DOPD_OK) return st;
  if (nreq == 0 || cu_host[nreq] == 0) return DOPD_OK;
  if (!q || !k_pool || !v_pool || !page_table || !cu || !prefix || !out || (rule.tree && !mask) ||
      (kv8 && (!k_scale || !v_scale)))
    return DOPD_ERR_NULL_POINTER;
  for (int32_t r = 0; r < nreq; ++r) {  // every page the request's keys touch has a column
    const int64_t n = cu_host[r + 1] - cu_host[r];
    if (n > 0 && (prefix_host[r] + n + dopd::kPage - 1) / dopd::kPage > pt_stride) return DOPD_ERR_INVALID_SHAPE;
  }
  if (!aligned16(q) || !aligned16(k_pool) || !aligned16(v_pool) || !aligned16(out)) return DOPD_ERR_INVALID_SHAPE;

  const int hq = s->num_q_heads, hkv = s->num_kv_heads, d = s->head_dim;
  dopd::MaskedArgs a;
  std::memset(&a, 0, sizeof(a));
  a.q = q;
  a.k_pool = k_pool;
  a.v_pool = v_pool;
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.page_table = page_table;
  a.cu = cu;
  a.prefix = prefix;
  a.mask = mask;
  a.out = out;
  a.lse = lse;
  a.rule = rule;
  a.deal = dopd::ma_deal(hkv, std::max(1, machine_shape().xcds));
  a.by_g = dopd::fast_div((uint32_t)(hq / hkv));
  a.pt_stride = pt_stride;
  a.nreq = nreq;
  a.hq = hq;
  a.hkv = hkv;
  a.words = words;
  hipStream_t strm = as_stream(stream);

  if (s->dtype == DOPD_FP32) {
    const dopd::MaKind kind = dopd::ma_kind(dopd::kMaF32);
    a.scale = s->softmax_scale;
    a.hi = INT32_MAX;
    const dopd::MaPlan p = dopd::ma_plan(rule, kind, cu_host, prefix_host, nreq, hq / hkv, hkv, machine_shape(), dopd::MaCosts{});
    if (!p.fits) return DOPD_ERR_INVALID_SHAPE;
    const dim3 grid = grid_of(p.blocks);
    if (d == 64) {
      const dim3 block(64 * dopd::f32_waves<64>());
      if (rule.tree) hipLaunchKernelGGL((dopd::masked_f32_kernel<64, true>), grid, block, 0, strm, a);
      else hipLaunchKernelGGL((dopd::masked_f32_kernel<64, false>), grid, block, 0, strm, a);
    } else {
      const dim3 block(64 * dopd::f32_waves<128>());
      if (rule.tree) hipLaunchKernelGGL((dopd::masked_f32_kernel<128, true>), grid, block, 0, strm, a);
      else hipLaunchKernelGGL((dopd::masked_f32_kernel<128, false>), grid, block, 0, strm, a);
    }
    return launch_status();
  }

  a.scale = s->softmax_scale * dopd::kLog2e;
  const dopd::MaSplit split = dopd::ma_split(rule, cu_host, prefix_host, nreq, hq / hkv, hkv,
                                              dopd::ma_mid(s->dtype == DOPD_FP8_E4M3, d), machine_shape());
  dopd::MaPlan plans[3];
  size_t need = 0;
  for (int i = 0; i < 3; ++i) {
    const dopd::MaKind k = dopd::ma_kernel(split, i);
    plans[i] = masked_plan(k, s, rule, cu_host, prefix_host, nreq);
    if (!plans[i].fits) return DOPD_ERR_INVALID_SHAPE;
    need += dopd::ma_ws_bytes(plans[i], k, d);
  }
  if (need > 0) {
    if (!workspace) return DOPD_ERR_NULL_POINTER;
    if (workspace_bytes < need) return DOPD_ERR_WORKSPACE_TOO_SMALL;
  }
  if ((reinterpret_cast<uintptr_t>(workspace) & 255) != 0) return DOPD_ERR_INVALID_SHAPE;
  char* ws = static_cast<char*>(workspace);
  for (int i = 2; i >= 0; --i) {  // (the longest kernel first)
    const dopd::MaPlan& p = plans[i];
    if (p.blocks == 0) continue;
    const dopd::MaKind k = dopd::ma_kernel(split, i);
    a.lo = k.lo;
    a.hi = k.hi;
    a.nwg = p.nwg;
    a.seg = p.seg;
    a.total = (int)p.total;
    a.slices = dopd::ma_slices(p.total, p.nwg);
    a.part_o = reinterpret_cast<float*>(ws);
    a.part_ml = reinterpret_cast<float*>(ws + dopd::ma_part_ml_off(p, k, d));
    ws += dopd::ma_ws_bytes(p, k, d);
    if (kv8) st = rule.tree ? launch_masked_d<true, true>(k, a, p, d, strm) : launch_masked_d<true, false>(k, a, p, d, strm);
    else st = rule.tree ? launch_masked_d<false, true>(k, a, p, d, strm) : launch_masked_d<false, false>(k, a, p, d, strm);
    if (st != DOPD_OK) return st;
  }
  return DOPD_OK;
}

}  // namespace

extern "C" {

size_t dopd_window_workspace_size(const dopd_attn_shape* s, const int32_t* cu_host, const int32_t* prefix_host,
                                  int32_t nreq, int32_t window, int32_t num_sinks) {
  return masked_workspace_size(s, window_rule(window, num_sinks), cu_host, prefix_host, nreq);
}

dopd_status dopd_window_attn(const dopd_attn_shape* s, const void* q, const void* k_pool, const void* v_pool,
                             int32_t num_pages, const int32_t* page_table, int32_t pt_stride, const int32_t* cu,
                             const int32_t* cu_host, const int32_t* prefix, const int32_t* prefix_host, int32_t nreq,
                             int32_t window, int32_t num_sinks, void* out, float* lse, void* workspace,
                             size_t workspace_bytes, void* stream) {
  return masked_impl(s, false, q, k_pool, v_pool, nullptr, nullptr, num_pages, page_table, pt_stride, cu, cu_host,
                     prefix, prefix_host, nreq, window_rule(window, num_sinks), nullptr, 0, out, lse, workspace,
                     workspace_bytes, stream);
}

dopd_status dopd_window_attn_fp8(const dopd_attn_shape* s, const void* q, const void* k_pool, const void* v_pool,
                                 const float* k_scale, const float* v_scale, int32_t num_pages,
                                 const int32_t* page_table, int32_t pt_stride, const int32_t* cu,
                                 const int32_t* cu_host, const int32_t* prefix, const int32_t* prefix_host,
                                 int32_t nreq, int32_t window, int32_t num_sinks, void* out, float* lse,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  return masked_impl(s, true, q, k_pool, v_pool, k_scale, v_scale, num_pages, page_table, pt_stride, cu, cu_host,
                     prefix, prefix_host, nreq, window_rule(window, num_sinks), nullptr, 0, out, lse, workspace,
                     workspace_bytes, stream);
}

size_t dopd_tree_workspace_size(const dopd_attn_shape* s, const int32_t* cu_host, const int32_t* prefix_host,
                                int32_t nreq) {
  return masked_workspace_size(s, tree_rule(), cu_host, prefix_host, nreq);
}

dopd_status dopd_tree_attn(const dopd_attn_shape* s, const void* q, const void* k_pool, const void* v_pool,
                           int32_t num_pages, const int32_t* page_table, int32_t pt_stride, const int32_t* cu,
                           const int32_t* cu_host, const int32_t* prefix, const int32_t* prefix_host, int32_t nreq,
                           const uint32_t* tree_mask, int32_t mask_words, void* out, float* lse, void* workspace,
                           size_t workspace_bytes, void* stream) {
  return masked_impl(s, false, q, k_pool, v_pool, nullptr, nullptr, num_pages, page_table, pt_stride, cu, cu_host,
                     prefix, prefix_host, nreq, tree_rule(), tree_mask, mask_words, out, lse, workspace,
                     workspace_bytes, stream);
}

dopd_status dopd_tree_attn_fp8(const dopd_attn_shape* s, const void* q, const void* k_pool, const void* v_pool,
                               const float* k_scale, const float* v_scale, int32_t num_pages,
                               const int32_t* page_table, int32_t pt_stride, const int32_t* cu, const int32_t* cu_host,
                               const int32_t* prefix, const int32_t* prefix_host, int32_t nreq,
                               const uint32_t* tree_mask, int32_t mask_words, void* out, float* lse, void* workspace,
                               size_t workspace_bytes, void* stream) {
  return masked_impl(s, true, q, k_pool, v_pool, k_scale, v_scale, num_pages, page_table, pt_stride, cu, cu_host,
                     prefix, prefix_host, nreq, tree_rule(), tree_mask, mask_words, out, lse, workspace,
                     workspace_bytes, stream);
}

dopd_status dopd_kv_copy_pages(const dopd_attn_shape* s, int32_t num_layers, void* k_pool, void* v_pool,
                               int32_t num_pages, const int32_t* src_pages, const int32_t* dst_pages,
                               int32_t num_copies, void* stream) {
  const dopd_status st = check_shape(s);
  if (st != DOPD_OK) return st;
  if (num_layers < 0 || num_pages < 0 || num_copies < 0) return DOPD_ERR_INVALID_SHAPE;
  if (num_layers == 0 || num_copies == 0) return DOPD_OK;
  if (!k_pool || !v_pool || !src_pages || !dst_pages) return DOPD_ERR_NULL_POINTER;
  if (!aligned16(k_pool) || !aligned16(v_pool)) return DOPD_ERR_INVALID_SHAPE;
  const int64_t bytes = (int64_t)s->num_kv_heads * dopd::kPage * s->head_dim * elem_bytes_of(s->dtype);
  if (bytes > INT32_MAX / 2) return DOPD_ERR_INVALID_SHAPE;
  dopd::CopyPagesArgs a;
  a.k_pool = static_cast<char*>(k_pool);
  a.v_pool = static_cast<char*>(v_pool);
  a.src = src_pages;
  a.dst = dst_pages;
  a.num_pages = num_pages;
  a.copies = num_copies;
  a.page_bytes = (int)bytes;
  a.pieces = (int)((bytes + dopd::kCopyPiece - 1) / dopd::kCopyPiece);
  if ((int64_t)num_layers * num_copies > dopd::kGridMaxBlocks / 2 / a.pieces) return DOPD_ERR_INVALID_SHAPE;
  a.blocks = (int64_t)2 * num_layers * num_copies * a.pieces;
  hipLaunchKernelGGL(dopd::kv_copy_pages_kernel, grid_of(a.blocks), dim3(dopd::kCopyThreads), 0, as_stream(stream), a);
  return launch_status();
}

dopd_status dopd_kv_compact(const dopd_attn_shape* s, int32_t num_layers, void* k_pool, void* v_pool,
                            int32_t num_pages, const int32_t* page_table, int32_t page_table_stride,
                            const int32_t* prefix_lens, const int32_t* accepted, const int32_t* num_accepted,
                            int32_t max_accepted, int32_t num_reqs, void* stream) {
  const dopd_status st = check_shape(s);
  if (st != DOPD_OK) return st;
  if (num_layers < 0 || num_pages < 0 || page_table_stride < 0 || max_accepted < 0 || num_reqs < 0)
    return DOPD_ERR_INVALID_SHAPE;
  if (num_layers == 0 || max_accepted == 0 || num_reqs == 0) return DOPD_OK;
  if (!k_pool || !v_pool || !page_table || !prefix_lens || !accepted || !num_accepted) return DOPD_ERR_NULL_POINTER;
  if (!aligned16(k_pool) || !aligned16(v_pool)) return DOPD_ERR_INVALID_SHAPE;
  const int d = s->head_dim, es = elem_bytes_of(s->dtype);
  const int64_t units = (int64_t)s->num_kv_heads * (d + d * es / 16);
  if (units > INT32_MAX / 2) return DOPD_ERR_INVALID_SHAPE;
  dopd::CompactArgs a;
  a.k_pool = static_cast<char*>(k_pool);
  a.v_pool = static_cast<char*>(v_pool);
  a.page_table = page_table;
  a.prefix = prefix_lens;
  a.path = accepted;
  a.count = num_accepted;
  a.num_pages = num_pages;
  a.pt_stride = page_table_stride;
  a.hkv = s->num_kv_heads;
  a.most = max_accepted;
  a.nreq = num_reqs;
  a.per = (int)((units + dopd::kCompactThreads - 1) / dopd::kCompactThreads);
  if ((int64_t)num_layers * num_reqs > dopd::kGridMaxBlocks / a.per) return DOPD_ERR_INVALID_SHAPE;
  a.blocks = (int64_t)num_layers * num_reqs * a.per;
  const dim3 grid = grid_of(a.blocks), block(dopd::kCompactThreads);
  hipStream_t strm = as_stream(stream);
  auto launch = [&](auto elem) {
    using T = decltype(elem);
    if (d == 64) hipLaunchKernelGGL((dopd::kv_compact_kernel<T, 64>), grid, block, 0, strm, a);
    else hipLaunchKernelGGL((dopd::kv_compact_kernel<T, 128>), grid, block, 0, strm, a);
  };
  if (es == 4) launch(uint32_t{});
  else if (es == 2) launch(uint16_t{});
  else launch(uint8_t{});
  return launch_status();
}

}  // extern "C"
