// What the kernels of the windowed and the tree attention share: their
// arguments, the visibility of keys, the item of a workgroup and the merge of
// items whose keys were split.
//
//   out[t][h] = sum_{j in V(t)} p_j v_j / sum p_j,  p_j = 2^(c q.k_j - m),
// with V(t) the cached positions row t sees: the window and the sinks, or the
// prefix and the drafts its mask names.  A row that sees nothing has out = 0
// and lse = -inf.
//
// Non-finite values at positions a row does not see never reach it: scores of
// unseen keys are replaced by a select, V of positions that no row of an item sees
// is cleared, and where a tile is seen by some rows only and a V in it is not
// finite, each row's product is formed with V cleared where that row sees
// nothing (0 * inf is NaN).
#pragma once
#include "../plan_masked.hpp"
#include "common.hpp"

namespace dopd {

struct MaskedArgs {
  const void* q;              // [T][Hq][D] bf16 or fp32
  const void* k_pool;         // [P][Hkv][16][D]
  const void* v_pool;         // [P][Hkv][D][16]
  const float* k_scale;       // [Hkv], E4M3 pools only
  const float* v_scale;
  const int32_t* page_table;  // [nreq][pt_stride]
  const int32_t* cu;          // [nreq + 1]
  const int32_t* prefix;      // [nreq]
  const uint32_t* mask;       // [T][words], tree calls only
  void* out;                  // [T][Hq][D]
  float* lse;                 // [T][Hq] or null
  float* part_o;              // [slots][rows][D]
  float* part_ml;             // [slots][rows][2]
  MaskRule rule;
  MaDeal deal;
  FastDiv by_g;               // (packed rows of a call stay below 2^32 / g: host check)
  int pt_stride, nreq, hq, hkv, words;
  int target;                 // tiles of a part
  float scale;                // softmax scale, times log2(e) but for fp32
};

// Bits t of [0, n) of a 32-bit word, n of any sign.
__device__ __forceinline__ uint32_t bits_below(int n) {
  return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u;
}

// Which of the keys base .. base + 31 the row at position `pos` (draft i of the
// request, mask row `mrow`) sees.  `pre`: cached tokens, `end`: keys of the request.
template <bool TREE>
__device__ __forceinline__ uint32_t row_sees(const MaskedArgs& a, int base, int pre, int end, int pos,
                                             const uint32_t* mrow) {
  if constexpr (TREE) {
    const int j = base - pre, w = j >> 5, s = j & 31;  // (draft index of the first key)
    auto word = [&](int i) { return i < 0 ? ~0u : i < a.words ? mrow[i] : 0u; };
    const uint64_t both = (uint64_t)word(w + 1) << 32 | word(w);
    return (uint32_t)(both >> s) & bits_below(end - base);
  } else {
    return bits_below(pos + 1 - base) & (~bits_below(pos - a.rule.window + 1 - base) | bits_below(a.rule.sinks - base));
  }
}
// Which of them some row at position p0 or later sees (a draft: whatever its mask).
template <bool TREE>
__device__ __forceinline__ uint32_t any_sees(const MaskedArgs& a, int base, int p0, int end) {
  const uint32_t below = bits_below(end - base);
  return TREE ? below : below & (~bits_below(ma_low_key(a.rule, p0) - base) | bits_below(a.rule.sinks - base));
}
// Do all rows at positions p0 .. p1 see all keys of [base, base + keys)?
template <bool TREE>
__device__ __forceinline__ bool all_see(const MaskedArgs& a, int base, int keys, int pre, int p0, int p1) {
  if constexpr (TREE) return base + keys <= pre;
  else return base + keys - 1 <= p0 && (base > p1 - a.rule.window || base + keys <= a.rule.sinks);
}
// The page read for page t of a request: t, or, where no row at position p0 or
// later sees any of it (its table entry may be stale), a page that one does.
__device__ __forceinline__ int seen_page(const MaskedArgs& a, int t, int low_key, int end) {
  const int low = low_key / kPage;
  return t * kPage >= a.rule.sinks && t < low ? low : min(t, (end - 1) / kPage);
}

// A workgroup's part of a call.
struct MaItem {
  int req, c, rt, split, nsplit;
  int row0, n, pre;  // the request's rows of q, its tokens, its cached tokens
  int64_t slot;      // of its partial result
};

// Part of workgroup b (the same in every lane of every wave); false: none.
template <int KIND>
__device__ __forceinline__ bool ma_find(const MaskedArgs& a, int b, MaItem& it) {
  constexpr MaKind kind = ma_kind(KIND);
  constexpr int ROWS = kind.rows;
  const int l = lane_id(), g = (int)a.by_g.d;
  int base = 0;
  int64_t slots = 0;
  for (int r0 = 0; r0 < a.nreq; r0 += 64) {
    const int r = min(r0 + l, a.nreq - 1);
    const int row0 = a.cu[r], n = a.cu[r + 1] - row0, pre = a.prefix[r];
    int blocks = 0, s = 1, rt = 0;
    if (r0 + l < a.nreq && ma_mine(kind, n, g)) {
      rt = ma_row_tiles(n, g, ROWS);
      s = ma_splits(ma_most_tiles(a.rule, pre, n, g, kind), a.target);
      blocks = (int)ma_blocks(a.deal, a.hkv, (int64_t)rt * s);
    }
    const int sl = s > 1 ? a.hkv * rt * s : 0;
    const int incl = wave_inclusive_scan(blocks), incl_s = wave_inclusive_scan(sl);
    const int total = __builtin_amdgcn_readlane(incl, 63);
    if (b < base + total) {
      const int o = __ffsll((long long)__ballot(b - base < incl)) - 1;
      auto of = [&](int v) { return __builtin_amdgcn_readlane(v, o); };
      const int local = b - base - of(incl - blocks);
      const int parts = of(rt) * of(s);
      it.req = r0 + o;
      it.nsplit = of(s);
      it.row0 = of(row0);
      it.n = of(n);
      it.pre = of(pre);
      int idx;
      if (!ma_part(a.deal, a.hkv, parts, local, it.c, idx)) return false;
      it.split = idx / of(rt);
      it.rt = idx - it.split * of(rt);
      it.slot = slots + of(incl_s - sl) + (int64_t)it.c * parts + idx;
      return true;
    }
    base += total;
    slots += __builtin_amdgcn_readlane(incl_s, 63);
  }
  return false;
}

// The merge of the split items: workgroup = 16 packed rows of one item, thread = a
// 4-dim chunk of a row, the item's partials folded in key order:
//   M = max_s m_s,  L = sum_s 2^(m_s - M) l_s,  o = sum_s 2^(m_s - M) o~_s / L.
// Bound by the partials' bytes (HBM or the caches); several workgroups an item,
// since one alone reads 16 partials of 64 KiB in about 15 us.
template <int D, int KIND>
__global__ __launch_bounds__(256) void masked_merge_kernel(MaskedArgs a) {
  constexpr MaKind kind = ma_kind(KIND);
  constexpr int ROWS = kind.rows;
  constexpr int kGroup = 16;
  const int l = lane_id(), g = (int)a.by_g.d;
  const int item = (int)blockIdx.x / (ROWS / kGroup), part = (int)blockIdx.x % (ROWS / kGroup);
  int rt_l = 0, s_l = 1, row0_l = 0, n_l = 0, slots_l = 0;
  int64_t slots = 0;
  int base = 0, r = -1, local = 0;
  for (int r0 = 0; r0 < a.nreq; r0 += 64) {
    const int rr = min(r0 + l, a.nreq - 1);
    row0_l = a.cu[rr];
    n_l = a.cu[rr + 1] - row0_l;
    rt_l = 0;
    s_l = 1;
    if (r0 + l < a.nreq && ma_mine(kind, n_l, g)) {
      rt_l = ma_row_tiles(n_l, g, ROWS);
      s_l = ma_splits(ma_most_tiles(a.rule, a.prefix[rr], n_l, g, kind), a.target);
    }
    const int items = s_l > 1 ? a.hkv * rt_l : 0;
    slots_l = items * s_l;
    const int incl = wave_inclusive_scan(items), incl_s = wave_inclusive_scan(slots_l);
    const int total = __builtin_amdgcn_readlane(incl, 63);
    if (item < base + total) {
      const int o = __ffsll((long long)__ballot(item - base < incl)) - 1;
      r = o;
      local = item - base - __builtin_amdgcn_readlane(incl - items, o);
      slots += __builtin_amdgcn_readlane(incl_s - slots_l, o);
      break;
    }
    base += total;
    slots += __builtin_amdgcn_readlane(incl_s, 63);
  }
  if (r < 0) return;
  const int rt = __builtin_amdgcn_readlane(rt_l, r), s = __builtin_amdgcn_readlane(s_l, r);
  const int row0 = __builtin_amdgcn_readlane(row0_l, r), n = __builtin_amdgcn_readlane(n_l, r);
  const int c = local / rt, tile = local - c * rt;
  const int64_t slot0 = slots + (int64_t)c * rt * s + tile;  // of split u: slot0 + u * rt
  const int live = min(ROWS, n * g - tile * ROWS);
  constexpr int CH = D / 4;
  for (int i = (int)threadIdx.x; i < kGroup * CH; i += 256) {
    const int row = kGroup * part + i / CH, e0 = 4 * (i % CH);
    if (row >= live) break;
    float M = -INFINITY;
    for (int u = 0; u < s; ++u) M = fmaxf(M, a.part_ml[((slot0 + (int64_t)u * rt) * ROWS + row) * 2]);
    float L = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int u = 0; u < s; ++u) {
      const int64_t at = (slot0 + (int64_t)u * rt) * ROWS + row;
      const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + at * 2);
      const f32x4 o = *reinterpret_cast<const f32x4*>(a.part_o + at * D + e0);
      const float w = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - M);  // (a part that saw nothing)
      L += w * ml.y;
      acc += o * w;
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
    const int x = tile * ROWS + row, tok = fast_quot(x, a.by_g);
    const int64_t at = (int64_t)(row0 + tok) * a.hq + c * g + (x - tok * g);
    u32x2 w2;
    w2[0] = pack_bf16x2(acc[0] * inv, acc[1] * inv);
    w2[1] = pack_bf16x2(acc[2] * inv, acc[3] * inv);
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + at * D + e0) = w2;
    if (a.lse && e0 == 0) a.lse[at] = (M + __log2f(L)) * kLn2;
  }
}

}  // namespace dopd
