// Launch planning of the windowed and the tree attention over the paged cache:
// which keys the rows of a request can see, in tiles, and how the work items of
// a call are dealt to workgroups.  Integer arithmetic only, shared by the host,
// the kernels and the CPU tests.
#pragma once
#include "plan.hpp"

namespace dopd {

// Positions stay below this, so that sums and differences of two fit an int.
constexpr int kMaMaxPos = 1 << 30;

// What a row at position p of a request sees of the cached positions j.
//   window: j <= p and (j > p - window or j < sinks)
//   tree:   every j before the drafts, and the drafts its mask names
struct MaskRule {
  int tree;
  int window, sinks;  // (window calls)
};

// First position that some row at p0 or later sees through the window.
constexpr int ma_low_key(const MaskRule& m, int p0) {
  return m.tree ? 0 : (p0 - m.window + 1 > 0 ? p0 - m.window + 1 : 0);
}

// Tiles of `keys` keys that rows at positions p0 .. p1 see: those of the sinks,
// then those of the windows.  Visited tile v is tile ma_tile(t, v).
struct KeyTiles {
  int nsink;  // tiles of sinks in front of a gap (0: no gap)
  int low;    // first tile behind the gap
  int n;
};
constexpr int ma_tile(const KeyTiles& t, int v) { return v < t.nsink ? v : v - t.nsink + t.low; }

constexpr KeyTiles ma_key_tiles(const MaskRule& m, int p0, int p1, int keys) {
  const int all = p1 / keys + 1;  // ceil((p1 + 1) / keys)
  const int low = ma_low_key(m, p0) / keys;
  if (low == 0) return KeyTiles{0, 0, all};
  const int ns = (m.sinks + keys - 1) / keys;  // (sinks before low: all of them exist)
  return ns >= low ? KeyTiles{0, 0, all} : KeyTiles{ns, low, ns + all - low};
}

// ---- work items ---------------------------------------------------------------
// Request r's chunk of n rows, packed with the g query heads of a KV head: packed
// row x is token x / g, query head c * g + x % g.  An item is (request, KV head c,
// `rows` packed rows).
//
// Kernels, by the packed rows of a request: one for up to 16, one for up to 64, a
// many-row kernel with items of 128, the fp32 kernel for any.  A kernel of a call
// takes the requests whose rows lie in (lo, hi].
enum { kMaFew = 0, kMaMid = 1, kMaMany = 2, kMaF32 = 3, kMaKinds = 4 };
struct MaKind {
  int which, rows, keys;  // packed rows of an item, keys of a tile
  int lo, hi;
};
constexpr MaKind ma_kind(int which, int lo = 0, int hi = INT32_MAX) {
  return which == kMaFew    ? MaKind{kMaFew, 16, 32, lo, hi}
         : which == kMaMid  ? MaKind{kMaMid, 64, 32, lo, hi}
         : which == kMaMany ? MaKind{kMaMany, 128, 32, lo, hi}
                            : MaKind{kMaF32, 16, 16, lo, hi};
}
constexpr bool ma_mine(const MaKind& k, int n, int g) { return n > 0 && (int64_t)n * g > k.lo && (int64_t)n * g <= k.hi; }
constexpr int ma_row_tiles(int n, int g, int rows) { return (n * g + rows - 1) / rows; }

// A bound of an item's tiles that depends on the request alone (rows at positions
// pre .. pre + n - 1, at most ceil(rows / g) + 1 tokens of them in one item).
constexpr int ma_most_tiles(const MaskRule& m, int pre, int n, int g, const MaKind& k) {
  const int tokens = (k.rows + g - 1) / g + 1;
  const KeyTiles whole = ma_key_tiles(m, pre, pre + n - 1, k.keys);
  if (m.tree || tokens >= n) return whole.n;
  const int ns = (m.sinks < pre + n ? m.sinks : pre + n);
  const int64_t some = (int64_t)(ns + k.keys - 1) / k.keys + ((int64_t)m.window + tokens - 1 + k.keys - 1) / k.keys + 1;
  return some < whole.n ? (int)some : whole.n;
}

// Two ways to deal a call's items to workgroups.
//
// Whole items: one workgroup each, the row tiles of one KV head, which read the
// same pages, on one XCD (or on `share` of them; workgroup b is on XCD b % xcds).
struct MaDeal {
  int xcds, share;  // share 0: in order
};
constexpr MaDeal ma_deal(int hkv, int xcds) {
  return hkv % xcds == 0 ? MaDeal{xcds, 1} : xcds % hkv == 0 ? MaDeal{xcds, xcds / hkv} : MaDeal{xcds, 0};
}
constexpr int64_t ma_blocks(const MaDeal& d, int hkv, int64_t parts) {  // of a request of `parts` row tiles
  return d.share == 0 ? hkv * parts : hkv * ((parts + d.share - 1) / d.share) * d.share;
}
// KV head and row tile of block `local` of a request; false where there is none.
constexpr bool ma_part(const MaDeal& d, int hkv, int parts, int local, int& c, int& rt) {
  if (d.share == 0) {
    c = local / parts;
    rt = local - c * parts;
    return c < hkv;
  }
  const int x = local % d.xcds, k = local / d.xcds;
  if (d.share == 1) {
    c = x + d.xcds * (k / parts);
    rt = k % parts;
    return c < hkv;
  }
  c = x % hkv;
  rt = k * d.share + x / hkv;
  return rt < parts;
}

// Slices: an item is a span of `seg` units (the fixed cost of starting it) and one
// per tile (ma_most_tiles of its request), the spans lie one after the other (by
// request, KV head, row tile), and every workgroup takes a slice of as many units:
// equal work whatever the lengths, one round over the machine.  An item whose tiles lie in several slices leaves a
// partial result in each: in slot 2 i where its part starts with the slice (or
// earlier), else in slot 2 i + 1.  Consecutive slices run on one XCD.
// (32-bit arithmetic: the first total % nwg slices are a unit longer.)
struct MaSlices {
  int per, longer;  // units of a slice; slices of one more
};
constexpr MaSlices ma_slices(int64_t total, int nwg) {
  return nwg > 0 ? MaSlices{(int)(total / nwg), (int)(total % nwg)} : MaSlices{0, 0};
}
constexpr int ma_slice_begin(int i, const MaSlices& s) { return i * s.per + (i < s.longer ? i : s.longer); }
constexpr int ma_slice_of(int unit, const MaSlices& s) {
  const int head = s.longer * (s.per + 1);
  return unit < head ? unit / (s.per + 1) : s.longer + (unit - head) / s.per;  // (per 0: every unit is in the head)
}
constexpr int ma_slice_index(int b, int nwg, int xcds) {
  return nwg % xcds == 0 ? b % xcds * (nwg / xcds) + b / xcds : b;
}
constexpr int64_t ma_span_units(const MaskRule& m, int pre, int n, int g, const MaKind& k, int seg) {
  return seg + ma_most_tiles(m, pre, n, g, k);
}
constexpr int64_t kMaMaxUnits = INT32_MAX / 2;

// ---- a call's plan --------------------------------------------------------------
struct MaPlan {
  int64_t blocks;  // workgroups (0: no item)
  int nwg;         // slices (0: whole items)
  int seg;
  int64_t total;   // units
  bool fits;       // the count fits the kernels' integers
};

struct MaCosts {
  int seg;         // start of an item, in tiles
  int merge;       // of a sliced call, in tiles: the partials and the kernel that merges them
  int min_tiles;   // fewest units of a slice
};

// Tiles that a request's items have on average (windows: the first rows of a
// context see less than the others).
inline double ma_mean_tiles(const MaskRule& m, int pre, int n, int g, const MaKind& k) {
  const double most = ma_most_tiles(m, pre, n, g, k);
  if (m.tree || pre + 1 >= m.window) return most;
  const double first = (pre + 1 + k.keys - 1) / k.keys;
  const double grow = std::min<double>(n, m.window - pre);  // rows until the window is full
  return most - (most - std::min(first, most)) * 0.5 * grow / n;
}

// Whole items where they fill the machine evenly enough, else slices: with R
// workgroups resident, whole items take about their tiles and starts over R plus
// half the longest item (the last round), and at least the longest; slices take the
// same over R and the merge.
inline MaPlan ma_plan(const MaskRule& m, const MaKind& k, const int32_t* cu, const int32_t* pre, int nreq, int g,
                      int hkv, const MachineShape& mach, const MaCosts& cost) {
  const int xcds = std::max(1, mach.xcds);
  const MaDeal d = ma_deal(hkv, xcds);
  const double resident = (double)kWgPerCu * std::max(1, mach.cus);
  MaPlan p{0, 0, cost.seg, 0, true};
  double items = 0, work = 0, bound = 0, longest = 0;
  for (int r = 0; r < nreq; ++r) {
    const int n = cu[r + 1] - cu[r];
    if (!ma_mine(k, n, g)) continue;
    const int rt = ma_row_tiles(n, g, k.rows);
    const double most = ma_most_tiles(m, pre[r], n, g, k), all = (double)hkv * rt;
    p.blocks += ma_blocks(d, hkv, rt);
    p.total += (int64_t)hkv * rt * ma_span_units(m, pre[r], n, g, k, cost.seg);
    items += all;
    work += all * (ma_mean_tiles(m, pre[r], n, g, k) + cost.seg);
    bound += all * (most + cost.seg);
    longest = std::max(longest, most + cost.seg);
  }
  if (p.blocks == 0) return p;
  const double whole = items <= resident ? longest : std::max(longest, work / resident + 0.5 * longest);
  const double slices = std::min(resident, std::max(1.0, bound / cost.min_tiles));
  const double sliced = (bound + slices * cost.seg) / slices + cost.merge;
  p.fits = p.blocks <= kMaMaxUnits;
  if (k.which == kMaF32 || whole <= sliced || p.total > kMaMaxUnits) return p;
  p.nwg = (int)slices;
  if (p.nwg > xcds) p.nwg -= p.nwg % xcds;
  p.blocks = p.nwg;
  return p;
}

// The kernels of a call.  A class of fewer rows can go with the next (whose kernel
// takes it, less efficiently) rather than to a launch of its own behind the others.
// mid: is the kernel of up to 64 rows the better one for them?  Its waves read and
// convert every tile for 16 rows each, the many-row kernel's for 32.  bf16 at d = 128:
// 115 us against 129 (48 rows over 3000 keys, 32 requests x 8 KV heads), d = 64 106
// against 106; E4M3, where that work counts, at d = 128 138 us against 117 (24 rows, 64
// requests), 94 against 90 (64 rows), at d = 64, whose tiles are too small for the
// many-row kernel's steps, 86 against 97 (32 rows).
constexpr bool ma_mid(bool fp8, int d) { return !(fp8 && d == 128); }
struct MaSplit {
  int hi16, hi64;  // the first kernel takes rows up to hi16, the second up to hi64, the third the rest
};
inline MaSplit ma_split(const MaskRule& m, const int32_t* cu, const int32_t* pre, int nreq, int g, int hkv, bool mid,
                        const MachineShape& mach = kDefaultMachine) {
  double tiles[3] = {0, 0, 0};  // of 32 keys
  for (int r = 0; r < nreq; ++r) {
    const int n = cu[r + 1] - cu[r];
    if (n == 0) continue;
    const int64_t rows = (int64_t)n * g;
    const int c = rows <= 16 ? 0 : rows <= 64 ? 1 : 2;
    tiles[c] += ma_most_tiles(m, pre[r], n, g, ma_kind(kMaMid)) * (c == 2 ? (double)ma_row_tiles(n, g, 128) : 1.);
  }
  // Few-row requests beside those of the middle kernel, which reads a tile once for up
  // to 64 rows, go with them unless they are most of the work: 32 trees of 8 drafts and
  // 32 decodes 98 us against 135 as two launches, 64 decodes 175 against 172.  The
  // many-row kernel takes a class whose tiles are few: 8 a workgroup or less (2 chunks of
  // 256 and 8 decodes over 1000 keys 68 us against 83; 8 chunks and 16 decodes over 2000
  // keys, 64/8 heads, 354 against 319).
  const double few = 8. * kWgPerCu * std::max(1, mach.cus) / hkv;
  MaSplit s{16, 64};
  const bool beside = mid && tiles[1] > 0;
  if (tiles[1] + tiles[2] > 0 && tiles[0] < (beside ? 2 * tiles[1] : few)) {
    s.hi16 = 0;
    tiles[1] += tiles[0];
  }
  if (!mid || (tiles[2] > 0 && tiles[1] < few)) s.hi64 = s.hi16;
  return s;
}
// Kernel i (0, 1, 2) of a call.
constexpr MaKind ma_kernel(const MaSplit& s, int i) {
  return i == 0 ? ma_kind(kMaFew, 0, s.hi16) : i == 1 ? ma_kind(kMaMid, s.hi16, s.hi64) : ma_kind(kMaMany, s.hi64);
}

// Workspace of one kernel's plan: [2 nwg][rows][D] partial outputs, then
// [2 nwg][rows][2] (m, l), each at a multiple of 256 bytes.
inline size_t ma_part_ml_off(const MaPlan& p, const MaKind& k, int d) {
  return align256((size_t)2 * p.nwg * k.rows * d * sizeof(float));
}
inline size_t ma_ws_bytes(const MaPlan& p, const MaKind& k, int d) {
  return p.nwg <= 1 ? 0 : ma_part_ml_off(p, k, d) + align256((size_t)2 * p.nwg * k.rows * 2 * sizeof(float));
}

// ---- compaction of accepted drafts ------------------------------------------------
// Tokens of a request to look at: of the accepted ones those whose place is among the
// `slots` of its row of the page table, and at most kMaMaxPos, so that places and loop
// counters fit an int whatever the lists hold.
constexpr int compact_tokens(int count, int most, int pre, int64_t slots) {
  const int64_t room = slots - pre;
  const int64_t m = count < most ? count : most;
  const int64_t top = room < kMaMaxPos ? room : kMaMaxPos;
  return (int)(m < top ? m : top);
}

}  // namespace dopd
