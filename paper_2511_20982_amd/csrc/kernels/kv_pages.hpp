// Calls that rearrange the pages of a cache in place, in every layer: whole pages
// copied to other pages, and the accepted tokens of a drafted tree moved to the
// places right behind their request's prefix.  Bit copies of any element type.
#pragma once
#include <type_traits>

#include "../plan_masked.hpp"
#include "common.hpp"

namespace dopd {

// ---- page copies --------------------------------------------------------------
// A page of one layer's K (or V) pool is one run of Hkv * 16 * D elements.  Workgroup
// = one piece of up to 16 KiB of one (layer, K/V, copy), four 16-byte loads a thread
// in flight before its stores.  HBM-bound at size.
struct CopyPagesArgs {
  char* k_pool;         // [layers][num_pages][page_bytes]
  char* v_pool;
  const int32_t* src;   // [copies]
  const int32_t* dst;
  int num_pages, copies, pieces;
  int page_bytes;       // (a multiple of 1024)
  int64_t blocks;
};
constexpr int kCopyPiece = 16384, kCopyThreads = 256;

__global__ __launch_bounds__(kCopyThreads) void kv_copy_pages_kernel(CopyPagesArgs a) {
  const int64_t b = grid_block(blockIdx.x, blockIdx.y);
  if (b >= a.blocks) return;
  const int piece = (int)(b % a.pieces);
  int64_t rest = b / a.pieces;
  const int i = (int)(rest % a.copies);
  rest /= a.copies;  // layer * 2 + K/V
  const int64_t layer = rest >> 1;
  const int s = a.src[i], d = a.dst[i];
  if ((unsigned)s >= (unsigned)a.num_pages || (unsigned)d >= (unsigned)a.num_pages || s == d) return;
  char* pool = (rest & 1 ? a.v_pool : a.k_pool) + layer * a.num_pages * (int64_t)a.page_bytes;
  const u32x4* from = reinterpret_cast<const u32x4*>(pool + (int64_t)s * a.page_bytes);
  u32x4* to = reinterpret_cast<u32x4*>(pool + (int64_t)d * a.page_bytes);
  const int first = piece * (kCopyPiece / 16) + (int)threadIdx.x, last = a.page_bytes / 16;
  u32x4 x[kCopyPiece / 16 / kCopyThreads];
#pragma unroll
  for (int u = 0; u < kCopyPiece / 16 / kCopyThreads; ++u)
    if (first + u * kCopyThreads < last) x[u] = from[first + u * kCopyThreads];
#pragma unroll
  for (int u = 0; u < kCopyPiece / 16 / kCopyThreads; ++u)
    if (first + u * kCopyThreads < last) to[first + u * kCopyThreads] = x[u];
}

// ---- accepted tokens ------------------------------------------------------------
// Request r: position prefix[r] + i takes what position prefix[r] + path[r][i] held,
// i < count[r], path strictly increasing (so path[i] >= i, and what a later move
// reads no earlier one has written).  A thread moves one dim row of V or one 16-byte
// chunk of K rows for all tokens of a request, loads before stores: it touches nothing
// another thread does, so the moves need no barrier.  A token of V is one element of
// each dim row, and a row is written whole: element by element, every token writes
// parts of the same 32-byte sectors again (28 layers x 192 requests: 77 us, and 62 this way).
// Places are uniform and come by scalar loads.  Bound by the sectors of V's rows.
struct CompactArgs {
  char* k_pool;               // [layers][num_pages][Hkv][16][D]
  char* v_pool;               // [layers][num_pages][Hkv][D][16]
  const int32_t* page_table;  // [nreq][pt_stride]
  const int32_t* prefix;      // [nreq]
  const int32_t* path;        // [nreq][most]
  const int32_t* count;       // [nreq]
  int num_pages, pt_stride, hkv, most, nreq;
  int per;                    // workgroups of one (request, layer)
  int64_t blocks;
};
constexpr int kCompactThreads = 256, kCompactTokens = 8;

template <typename T, int D>
__global__ __launch_bounds__(kCompactThreads) void kv_compact_kernel(CompactArgs a) {
  constexpr int CPR = D * (int)sizeof(T) / 16;  // chunks of a K row
  const int64_t b = grid_block(blockIdx.x, blockIdx.y);
  if (b >= a.blocks) return;
  const int part = (int)(b % a.per);
  const int64_t rest = b / a.per;
  const int r = (int)(rest % a.nreq);
  const int64_t layer = rest / a.nreq;
  typedef const __attribute__((address_space(4))) int32_t* ScalarPtr;
  const ScalarPtr count = (ScalarPtr)(uintptr_t)a.count, prefix = (ScalarPtr)(uintptr_t)a.prefix;
  const ScalarPtr pt = (ScalarPtr)(uintptr_t)(a.page_table + (int64_t)r * a.pt_stride);
  const ScalarPtr path = (ScalarPtr)(uintptr_t)(a.path + (int64_t)r * a.most);
  const int pre = prefix[r];
  if (pre < 0 || pre >= kMaMaxPos) return;
  const int m = compact_tokens(count[r], a.most, pre, (int64_t)a.pt_stride * kPage);
  if (m <= 0) return;
  const int unit = part * kCompactThreads + (int)threadIdx.x;
  const int nv = a.hkv * D;
  const int64_t page_elems = (int64_t)a.hkv * kPage * D, base = layer * a.num_pages * page_elems;

  // Page of a position; a negative one where the table has none.
  auto page_of = [&](int pos) {
    if (pos / kPage >= a.pt_stride) return -1;
    const int p = pt[pos / kPage];
    return p < a.num_pages ? p : -1;
  };
  // Where token i comes from: its position, and its page (-1: it stays, or has no path).
  auto source = [&](int i, int& pos) {
    const int from = path[i];
    if (from <= i || from >= kMaMaxPos) return -1;
    pos = pre + from;
    return page_of(pos);
  };
  if (unit < nv) {
    T* at = reinterpret_cast<T*>(a.v_pool) + base + (int64_t)unit * kPage;  // this thread's row of page 0
    for (int t = pre / kPage; t <= (pre + m - 1) / kPage; ++t) {
      const int pd = page_of(t * kPage);
      if (pd < 0) continue;
      typedef T Row __attribute__((ext_vector_type(kPage)));
      Row* to = reinterpret_cast<Row*>(at + pd * page_elems);
      Row x = *to;
      bool any = false;
#pragma unroll
      for (int s = 0; s < kPage; ++s) {
        const int i = t * kPage + s - pre;
        if (i < 0 || i >= m) continue;
        int pos = 0;
        const int ps = source(i, pos);
        if (ps < 0) continue;
        x[s] = at[ps * page_elems + pos % kPage];
        any = true;
      }
      if (any) *to = x;
    }
  } else if (unit < nv + a.hkv * CPR) {
    const int k = unit - nv, h = k / CPR, q = k % CPR;
    u32x4* at = reinterpret_cast<u32x4*>(reinterpret_cast<T*>(a.k_pool) + base + (int64_t)h * kPage * D) + q;
    constexpr int ratio = 16 / sizeof(T);
    for (int i0 = 0; i0 < m; i0 += kCompactTokens) {
      u32x4 x[kCompactTokens];
      int64_t to[kCompactTokens];
#pragma unroll
      for (int u = 0; u < kCompactTokens; ++u) {
        to[u] = -1;
        if (i0 + u >= m) continue;
        int pos = 0;
        const int ps = source(i0 + u, pos), pd = page_of(pre + i0 + u);
        if (ps < 0 || pd < 0) continue;
        x[u] = at[(ps * page_elems + (pos % kPage) * D) / ratio];
        to[u] = (pd * page_elems + ((pre + i0 + u) % kPage) * D) / ratio;
      }
#pragma unroll
      for (int u = 0; u < kCompactTokens; ++u)
        if (to[u] >= 0) at[to[u]] = x[u];
    }
  }
}

}  // namespace dopd
