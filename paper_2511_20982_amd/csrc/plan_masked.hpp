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
// `rows` packed rows); its tiles of keys are cut into ma_splits parts, computed by
// different workgroups and merged exactly by log-sum-exp rescaling.
//
// The few-row kernel takes requests of at most kMaFewRows packed rows, the
// many-row kernel the others; a call with both launches both.  The fp32 kernel
// takes all and splits none.
constexpr int kMaFewRows = 16;
constexpr int kMaMaxSplits = 64;

enum { kMaFew = 0, kMaMany = 1, kMaF32 = 2 };
struct MaKind {  // of a kernel: packed rows of an item, keys of a tile
  int which, rows, keys;
};
constexpr MaKind ma_kind(int which) {
  return which == kMaFew ? MaKind{kMaFew, kMaFewRows, 32} : which == kMaMany ? MaKind{kMaMany, 128, 64} : MaKind{kMaF32, 16, 16};
}
constexpr bool ma_mine(const MaKind& k, int n, int g) {
  return n > 0 && (k.which == kMaF32 || ((int64_t)n * g <= kMaFewRows) == (k.which == kMaFew));
}
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
constexpr int ma_splits(int tiles, int target) {
  return tiles <= target ? 1 : (tiles + target - 1) / target;
}

// Blocks of a request: its (KV head, split, row tile) parts, dealt so that the row
// tiles and splits of one KV head, which read the same pages, run on one XCD (or on
// `share` of them), with workgroup b on XCD b % xcds.  idx = split * row_tiles +
// row tile of the part.
struct MaDeal {
  int xcds, share;  // share 0: in order
};
constexpr MaDeal ma_deal(int hkv, int xcds) {
  return hkv % xcds == 0 ? MaDeal{xcds, 1} : xcds % hkv == 0 ? MaDeal{xcds, xcds / hkv} : MaDeal{xcds, 0};
}
constexpr int64_t ma_blocks(const MaDeal& d, int hkv, int64_t parts) {
  return d.share == 0 ? hkv * parts : hkv * ((parts + d.share - 1) / d.share) * d.share;
}
// KV head and part of block `local` of a request; false where there is none.
constexpr bool ma_part(const MaDeal& d, int hkv, int parts, int local, int& c, int& idx) {
  if (d.share == 0) {
    c = local / parts;
    idx = local - c * parts;
    return c < hkv;
  }
  const int x = local % d.xcds, k = local / d.xcds;
  if (d.share == 1) {
    c = x + d.xcds * (k / parts);
    idx = k % parts;
    return c < hkv;
  }
  c = x % hkv;
  idx = k * d.share + x / hkv;
  return idx < parts;
}

// ---- a call's plan --------------------------------------------------------------
struct MaPlan {
  int target;          // tiles of a part
  int64_t blocks;      // workgroups
  int64_t slots;       // partial results (0: nothing is split)
  int64_t merges;      // items that are merged
};

// The target that a simple model of the call makes fastest: with as many resident
// workgroups as `resident`, parts of at most `target` tiles that each cost `start`
// tiles more to begin and to merge, all rounds but the last full.
inline MaPlan ma_plan_of(const MaskRule& m, const MaKind& k, const int32_t* cu, const int32_t* pre, int nreq, int g,
                         int hkv, const MaDeal& d, int target) {
  MaPlan p{target, 0, 0, 0};
  for (int r = 0; r < nreq; ++r) {
    const int n = cu[r + 1] - cu[r];
    if (!ma_mine(k, n, g)) continue;
    const int rt = ma_row_tiles(n, g, k.rows), s = ma_splits(ma_most_tiles(m, pre[r], n, g, k), target);
    p.blocks += ma_blocks(d, hkv, (int64_t)rt * s);
    if (s > 1) {
      p.slots += (int64_t)hkv * rt * s;
      p.merges += (int64_t)hkv * rt;
    }
  }
  return p;
}

inline MaPlan ma_plan(const MaskRule& m, const MaKind& k, const int32_t* cu, const int32_t* pre, int nreq, int g,
                      int hkv, const MachineShape& mach, int min_tiles, int start) {
  const MaDeal d = ma_deal(hkv, std::max(1, mach.xcds));
  int most = 0;
  for (int r = 0; r < nreq; ++r)
    if (ma_mine(k, cu[r + 1] - cu[r], g)) most = std::max(most, ma_most_tiles(m, pre[r], cu[r + 1] - cu[r], g, k));
  if (most == 0) return MaPlan{1, 0, 0, 0};
  const int64_t resident = (int64_t)kWgPerCu * std::max(1, mach.cus);
  int best = most;
  double least = -1;
  for (int s = 1; s <= kMaMaxSplits; s = s < 4 ? s + 1 : s + s / 2) {
    const int target = (most + s - 1) / s;
    if (s > 1 && target < min_tiles) break;
    double items = 0, tiles = 0;
    for (int r = 0; r < nreq; ++r) {
      const int n = cu[r + 1] - cu[r];
      if (!ma_mine(k, n, g)) continue;
      const int t = ma_most_tiles(m, pre[r], n, g, k);
      const double it = (double)hkv * ma_row_tiles(n, g, k.rows);
      items += it * ma_splits(t, target);
      tiles += it * t;
    }
    const double longest = target + start;
    const double each = (tiles + items * start) / (double)resident;
    const double time = items <= (double)resident ? longest : each + 0.5 * longest;
    if (least < 0 || time < least) {
      least = time;
      best = target;
    }
  }
  return ma_plan_of(m, k, cu, pre, nreq, g, hkv, d, best);
}

// Workspace of one kernel's plan: [slots][rows][D] partial outputs, then
// [slots][rows][2] (m, l), each at a multiple of 256 bytes.
inline size_t ma_part_ml_off(const MaPlan& p, const MaKind& k, int d) {
  return align256((size_t)p.slots * k.rows * d * sizeof(float));
}
inline size_t ma_ws_bytes(const MaPlan& p, const MaKind& k, int d) {
  return p.slots == 0 ? 0 : ma_part_ml_off(p, k, d) + align256((size_t)p.slots * k.rows * 2 * sizeof(float));
}

}  // namespace dopd
