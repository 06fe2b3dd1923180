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
  float* part_o;              // [2 nwg][rows][D]
  float* part_ml;             // [2 nwg][rows][2]
  MaskRule rule;
  MaDeal deal;
  FastDiv by_g;               // (packed rows of a call stay below 2^32 / g: host check)
  int pt_stride, nreq, hq, hkv, words;
  int nwg, seg, total;        // slices (nwg 0: whole items), see the plan
  MaSlices slices;
  int lo, hi;                 // packed rows of the requests that this kernel takes: in (lo, hi]
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

// Eight bf16 (or E4M3 codes), of which those with a set bit are kept.
__device__ __forceinline__ u32x4 keep_of(u32x4 x, uint32_t bits) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    x[i] &= (bits >> (2 * i) & 1u ? 0xffffu : 0u) | (bits >> (2 * i) & 2u ? 0xffff0000u : 0u);
  return x;
}
__device__ __forceinline__ u32x2 keep_of(u32x2 x, uint32_t bits) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t b = bits >> (4 * i);
    x[i] &= (b & 1u ? 0xffu : 0u) | (b & 2u ? 0xff00u : 0u) | (b & 4u ? 0xff0000u : 0u) | (b & 8u ? 0xff000000u : 0u);
  }
  return x;
}

// Over the four lanes l % 16 + 0, 16, 32, 48 (on the vector unit: through LDS each of
// the two exchanges takes some 100 cycles).
__device__ __forceinline__ float quad_max(float x) {
  const uint32_t b = __float_as_uint(x);
  const auto h = __builtin_amdgcn_permlane16_swap(b, b, false, false);
  const uint32_t y = __float_as_uint(fmaxf(__uint_as_float(h[0]), __uint_as_float(h[1])));
  const auto f = __builtin_amdgcn_permlane32_swap(y, y, false, false);
  return fmaxf(__uint_as_float(f[0]), __uint_as_float(f[1]));
}
__device__ __forceinline__ float quad_sum(float x) {
  const uint32_t b = __float_as_uint(x);
  const auto h = __builtin_amdgcn_permlane16_swap(b, b, false, false);
  const uint32_t y = __float_as_uint(__uint_as_float(h[0]) + __uint_as_float(h[1]));
  const auto f = __builtin_amdgcn_permlane32_swap(y, y, false, false);
  return __uint_as_float(f[0]) + __uint_as_float(f[1]);
}

// Eight keys of a V row as a bf16 operand.
__device__ __forceinline__ bf16x8 v_operand(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }
__device__ __forceinline__ bf16x8 v_operand(u32x2 v) {
  const u32x2 lo = bf16x4_from_e4m3x4(v[0]), hi = bf16x4_from_e4m3x4(v[1]);
  return __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
}

__device__ __forceinline__ void store_bf16x4(void* out, int64_t at, f32x4 o) {
  u32x2 w;
  w[0] = pack_bf16x2(o[0], o[1]);
  w[1] = pack_bf16x2(o[2], o[3]);
  *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(out) + at) = w;
}
template <int N, class V>
__device__ __forceinline__ bool any_not_finite(const V (&o)[N]) {  // in the wave
  float top = 0.f;
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (unsigned j = 0; j < sizeof(V) / 4; ++j) top = __builtin_elementwise_maximum(top, __builtin_fabsf(o[n][j]));
  return __ballot(!(top < INFINITY)) != 0;
}

// A workgroup's item, or the part of one that lies in its slice.
struct MaItem {
  int req, c, rt;
  int row0, n, pre;  // the request's rows of q, its tokens, its cached tokens
  int u0, u1;        // units of the item's span [u0, u1) in the slice (whole items: all)
  int slot;          // of a partial result
};

// The request that unit (or block) x of the call lies in, and x's offset in it;
// count(r, n, pre): the units of request r.  The same in every lane; every wave takes
// part.  false: past the last one.
template <int KIND, class Count>
__device__ __forceinline__ bool ma_find(const MaskedArgs& a, int x, Count count, MaItem& it, int& local) {
  const MaKind kind = ma_kind(KIND, a.lo, a.hi);
  const int l = lane_id(), g = (int)a.by_g.d;
  int base = 0;
  for (int r0 = 0; r0 < a.nreq; r0 += 64) {
    const int r = min(r0 + l, a.nreq - 1);
    const int row0 = a.cu[r], n = a.cu[r + 1] - row0, pre = a.prefix[r];
    const int mine = r0 + l < a.nreq && ma_mine(kind, n, g) ? count(n, pre) : 0;
    const int incl = wave_inclusive_scan(mine);
    const int total = __builtin_amdgcn_readlane(incl, 63);
    if (x < base + total) {
      const int o = __ffsll((long long)__ballot(x - base < incl)) - 1;
      local = x - base - __builtin_amdgcn_readlane(incl - mine, o);
      it.req = r0 + o;
      it.row0 = __builtin_amdgcn_readlane(row0, o);
      it.n = __builtin_amdgcn_readlane(n, o);
      it.pre = __builtin_amdgcn_readlane(pre, o);
      return true;
    }
    base += total;
  }
  return false;
}

// Calls body(item) for each item of workgroup b (uniform).
template <int KIND, class Body>
__device__ __forceinline__ void ma_items(const MaskedArgs& a, int b, Body body) {
  const MaKind kind = ma_kind(KIND, a.lo, a.hi);
  const int g = (int)a.by_g.d;
  MaItem it;
  int local, begin = 0, pos = 0, end = 0, slice = 0;
  auto units = [&](int n, int pre) {
    return a.hkv * ma_row_tiles(n, g, kind.rows) * (int)ma_span_units(a.rule, pre, n, g, kind, a.seg);
  };
  if (a.nwg == 0) {
    auto blocks = [&](int n, int) { return (int)ma_blocks(a.deal, a.hkv, ma_row_tiles(n, g, kind.rows)); };
    if (!ma_find<KIND>(a, b, blocks, it, local)) return;
    if (!ma_part(a.deal, a.hkv, ma_row_tiles(it.n, g, kind.rows), local, it.c, it.rt)) return;
  } else {
    slice = ma_slice_index(b, a.nwg, a.deal.xcds);
    begin = pos = ma_slice_begin(slice, a.slices);
    end = ma_slice_begin(slice + 1, a.slices);
    if (pos >= end || !ma_find<KIND>(a, pos, units, it, local)) return;
  }
  while (true) {  // slices: one item, or part of one, at a time
    if (a.nwg != 0) {
      const int span = (int)ma_span_units(a.rule, it.pre, it.n, g, kind, a.seg), rts = ma_row_tiles(it.n, g, kind.rows);
      const int index = local / span;
      it.u0 = local - index * span;
      it.u1 = min(span, it.u0 + end - pos);
      it.c = index / rts;
      it.rt = index - it.c * rts;
      it.slot = 2 * slice + (pos == begin ? 0 : 1);
      pos += it.u1 - it.u0;
      local += it.u1 - it.u0;
    }
    if (a.nwg == 0 || it.u1 > a.seg) body(it);  // (else only units of the start)
    if (pos >= end) return;
    if (local == units(it.n, it.pre)) {  // the next request of this kernel
      do {
        ++it.req;
        it.row0 = __builtin_amdgcn_readfirstlane(a.cu[it.req]);
        it.n = __builtin_amdgcn_readfirstlane(a.cu[it.req + 1]) - it.row0;
      } while (!ma_mine(kind, it.n, g));
      it.pre = __builtin_amdgcn_readfirstlane(a.prefix[it.req]);
      local = 0;
    }
  }
}

// Tiles [v0, v1) of an item of n tiles that its units cover, and whether that is all
// of it.  (A span can be longer than the item: ma_most_tiles is a bound.)
__device__ __forceinline__ bool ma_tiles_of(const MaskedArgs& a, const MaItem& it, int n, int& v0, int& v1) {
  v0 = a.nwg == 0 ? 0 : min(n, max(0, it.u0 - a.seg));
  v1 = a.nwg == 0 ? n : min(n, it.u1 - a.seg);
  return v0 == 0 && v1 == n;
}

// A part's sum may hold weights far above 1 where they were formed against a maximum that
// stayed behind: its binary exponent moves from the sum (which becomes 0.5 .. 1; 0, inf and
// NaN stay) and the part's O, whose factor is returned, to the maximum.  Both factors are
// powers of two, so only the maximum's sum rounds; parts of large V then add up as they do
// under their true maxima.
__device__ __forceinline__ float part_to_unit_sum(float& m, float& l) {
  const int e = __builtin_amdgcn_frexp_expf(l);
  m += (float)e;
  l = __builtin_amdgcn_ldexpf(l, -e);
  return __builtin_amdgcn_ldexpf(1.f, -e);
}

// The merge of the items that lie in several slices: workgroup = merge_rows packed
// rows of the item that a slice continues, if that slice is the first to continue it;
// thread = a 4-dim chunk of up to four rows, the partials folded in key order:
//   M = max_s m_s,  L = sum_s 2^(m_s - M) l_s,  o = sum_s 2^(m_s - M) o~_s / L.
// Bound by the partials' bytes and the start of a kernel.
constexpr int merge_rows(int kind) { return ma_kind(kind).rows < 32 ? ma_kind(kind).rows : 32; }
template <int D, int KIND>
__global__ __launch_bounds__(256) void masked_merge_kernel(MaskedArgs a) {
  const MaKind kind = ma_kind(KIND, a.lo, a.hi);
  constexpr int ROWS = ma_kind(KIND).rows, kGroup = merge_rows(KIND), CH = D / 4;
  constexpr int STEP = 256 / CH, R = kGroup / STEP;  // rows that the threads cover at once; rows of a thread
  const int g = (int)a.by_g.d;
  const int slice = 1 + (int)blockIdx.x / (ROWS / kGroup), group = (int)blockIdx.x % (ROWS / kGroup);
  MaItem it;
  int local;
  const int at = ma_slice_begin(slice, a.slices);
  auto units = [&](int n, int pre) {
    return a.hkv * ma_row_tiles(n, g, ROWS) * (int)ma_span_units(a.rule, pre, n, g, kind, a.seg);
  };
  if (at >= a.total || !ma_find<KIND>(a, at, units, it, local)) return;
  const int span = (int)ma_span_units(a.rule, it.pre, it.n, g, kind, a.seg), rts = ma_row_tiles(it.n, g, ROWS);
  const int index = local / span, c = index / rts, rt = index - c * rts;
  const int x0 = rt * ROWS, live = min(ROWS, it.n * g - x0);
  if (group * kGroup >= live) return;
  const int p0 = it.pre + fast_quot(x0, a.by_g), p1 = it.pre + fast_quot(x0 + live - 1, a.by_g);
  const int tiles = ma_key_tiles(a.rule, p0, a.rule.tree ? it.pre + it.n - 1 : p1, kind.keys).n;
  const int first = at - (local - index * span);  // the item's first unit
  const int b0 = ma_slice_of(first + a.seg, a.slices), b1 = ma_slice_of(first + a.seg + tiles - 1, a.slices);
  if (b0 == b1 || slice != b0 + 1) return;
  const int slot0 = 2 * b0 + (ma_slice_begin(b0, a.slices) >= first ? 0 : 1);
  const int row0 = kGroup * group + (int)threadIdx.x / CH, e0 = 4 * ((int)threadIdx.x % CH);
  float M[R], L[R];
  f32x4 acc[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    M[r] = -INFINITY;
    L[r] = 0.f;
    acc[r] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  constexpr int P = R > 2 ? 2 : 4;  // partials in flight
  for (int b = b0; b <= b1; b += P) {
    float2 ml[P][R];
    f32x4 o[P][R];
#pragma unroll
    for (int u = 0; u < P; ++u) {
      if (b + u > b1) break;
      const int64_t slot = b + u == b0 ? slot0 : 2 * (b + u);
#pragma unroll
      for (int r = 0; r < R; ++r) {  // (rows past the last: the last again)
        const int64_t from = slot * ROWS + min(row0 + r * STEP, live - 1);
        ml[u][r] = *reinterpret_cast<const float2*>(a.part_ml + from * 2);
        o[u][r] = *reinterpret_cast<const f32x4*>(a.part_o + from * D + e0);
      }
    }
#pragma unroll
    for (int u = 0; u < P; ++u) {
      if (b + u > b1) break;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        // A part that saw nothing of the row.  (One whose scores are all NaN has the same
        // maximum, and a sum of NaN: 0 times that makes the row NaN, in any order of parts.)
        if (ml[u][r].x == -INFINITY && ml[u][r].y == 0.f) continue;
        const float m = fmaxf(M[r], ml[u][r].x);
        const float old = M[r] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M[r] - m);
        const float now = __builtin_amdgcn_exp2f(ml[u][r].x - m);
        L[r] = L[r] * old + ml[u][r].y * now;
        acc[r] = acc[r] * old + o[u][r] * now;
        M[r] = m;
      }
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = row0 + r * STEP;
    if (row >= live) break;
    const float inv = L[r] == 0.f ? 0.f : 1.f / L[r];
    const int x = x0 + row, tok = fast_quot(x, a.by_g);
    const int64_t to = (int64_t)(it.row0 + tok) * a.hq + c * g + (x - tok * g);
    store_bf16x4(a.out, to * D + e0, acc[r] * inv);
    if (a.lse && e0 == 0) a.lse[to] = (M[r] + __log2f(L[r])) * kLn2;
  }
}

}  // namespace dopd
