// CPU check of the planning of the windowed and the tree attention
// (paper_2511_20982_amd/csrc/plan_masked.hpp): the visited tiles hold every position
// a row sees, the pages read are pages that some row sees, the workgroups of a plan
// take every tile of every item once, and the merge reads the partials they leave.
// Usage: masked_harness <cus> <xcds> <cases>; prints "ok" or the first failure.
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <set>
#include <utility>
#include <vector>

#include "../paper_2511_20982_amd/csrc/plan_masked.hpp"

using namespace dopd;

static int fail(const char* what, long a, long b) {
  std::printf("FAIL %s (%ld, %ld)\n", what, a, b);
  return 1;
}

static bool sees(const MaskRule& m, int pre, int n, int p, int j) {
  if (m.tree) return j < pre + n;  // (any mask)
  return j <= p && (j > p - m.window || j < m.sinks);
}

// seen_page of the kernels.
static int page_read(const MaskRule& m, int t, int low_key, int end) {
  const int low = low_key / 16;
  return t * 16 >= m.sinks && t < low ? low : std::min(t, (end - 1) / 16);
}

static int check_tiles(const MaskRule& m, int pre, int n, int g, const MaKind& k) {
  const int rows = n * g, rt = ma_row_tiles(n, g, k.rows);
  for (int i = 0; i < rt; ++i) {
    const int p0 = pre + i * k.rows / g, p1 = pre + (std::min(rows, (i + 1) * k.rows) - 1) / g;
    const int end = m.tree ? pre + n : p1 + 1;
    const KeyTiles t = ma_key_tiles(m, p0, end - 1, k.keys);
    if (t.n < 1 || t.n > ma_most_tiles(m, pre, n, g, k)) return fail("tiles above their bound", t.n, ma_most_tiles(m, pre, n, g, k));
    std::set<int> visited;
    for (int v = 0; v < t.n; ++v) {
      const int tile = ma_tile(t, v);
      if (!visited.insert(tile).second) return fail("tile visited twice", v, tile);
      if (v > 0 && tile <= ma_tile(t, v - 1)) return fail("tiles not ascending", v, tile);
      bool any = false;
      for (int pg = tile * (k.keys / 16); pg < (tile + 1) * (k.keys / 16); ++pg) {
        const int read = page_read(m, pg, ma_low_key(m, p0), end);
        bool seen = false;
        for (int j = 16 * read; j < 16 * read + 16; ++j)
          for (int p = p0; p <= p1; ++p) seen |= sees(m, pre, n, p, j);
        if (!seen) return fail("a page that nobody sees is read", pg, read);
        bool here = false;
        for (int j = 16 * pg; j < 16 * pg + 16; ++j)
          for (int p = p0; p <= p1; ++p) here |= sees(m, pre, n, p, j);
        if (here && read != pg) return fail("a seen page is not read", pg, read);
        any |= here;
      }
      if (!any) return fail("a tile that nobody sees is visited", v, tile);
    }
    for (int p = p0; p <= p1; ++p)
      for (int j = 0; j < end; ++j)
        if (sees(m, pre, n, p, j) && !visited.count(j / k.keys)) return fail("a seen position is not visited", p, j);
  }
  return 0;
}

// Walks the workgroups of a plan as the kernels do: every tile of every item is taken
// once, partial results lie in slots of their own, and the merge finds each split
// item once, with the slots that were written.
static int check_plan(const MaskRule& m, const std::vector<int32_t>& cu, const std::vector<int32_t>& pre, int g,
                      int hkv, const MaKind& k, const MachineShape& mach, const MaCosts& cost, bool slices) {
  const int n = (int)pre.size();
  const MaDeal d = ma_deal(hkv, mach.xcds);
  MaPlan p = ma_plan(m, k, cu.data(), pre.data(), n, g, hkv, mach, cost);
  if (!p.fits) return fail("does not fit", p.blocks, p.total);
  if (slices && p.nwg == 0 && p.blocks > 0 && p.total <= kMaMaxUnits) p.blocks = p.nwg = 1 + (int)(p.total % 97);  // (any count has to work)
  struct Item {
    int r, c, rt, tiles;
    int64_t first;
  };
  std::vector<Item> items;
  int64_t units = 0, base = 0;
  for (int r = 0; r < n; ++r) {
    const int len = cu[r + 1] - cu[r];
    if (!ma_mine(k, len, g)) continue;
    const int rts = ma_row_tiles(len, g, k.rows);
    for (int c = 0; c < hkv; ++c)
      for (int rt = 0; rt < rts; ++rt) {
        const int p0 = pre[r] + rt * k.rows / g, p1 = pre[r] + (std::min(len * g, (rt + 1) * k.rows) - 1) / g;
        items.push_back({r, c, rt, ma_key_tiles(m, p0, m.tree ? pre[r] + len - 1 : p1, k.keys).n, units});
        units += ma_span_units(m, pre[r], len, g, k, p.seg);
      }
    const int64_t blocks = ma_blocks(d, hkv, rts);
    if (p.nwg == 0) {
      if (d.share && (blocks % mach.xcds || base % mach.xcds)) return fail("XCD phase", blocks, base);
      std::set<std::pair<int, int>> seen;
      for (int64_t b = 0; b < blocks; ++b) {
        int c, rt;
        if (!ma_part(d, hkv, rts, (int)b, c, rt)) continue;
        if (c < 0 || c >= hkv || rt < 0 || rt >= rts) return fail("item out of range", c, rt);
        if (!seen.insert({c, rt}).second) return fail("item dealt twice", r, rt);
      }
      if ((int)seen.size() != hkv * rts) return fail("items missing", (long)seen.size(), hkv * rts);
    }
    base += blocks;
  }
  if (units != p.total) return fail("units", units, p.total);
  if (p.nwg == 0) return base == p.blocks ? 0 : fail("blocks", base, p.blocks);
  const MaSlices sl = ma_slices(p.total, p.nwg);
  std::set<int> order;
  for (int b = 0; b < p.nwg; ++b) order.insert(ma_slice_index(b, p.nwg, mach.xcds));
  if ((int)order.size() != p.nwg || *order.begin() != 0 || *order.rbegin() != p.nwg - 1) return fail("slice order", p.nwg, 0);
  std::map<std::pair<size_t, int>, int> written;  // (item, slice) -> slot
  std::set<int> slots;
  std::vector<int> taken(items.size(), 0);
  size_t at = 0;
  for (int i = 0; i < p.nwg; ++i) {
    const int64_t begin = ma_slice_begin(i, sl), end = ma_slice_begin(i + 1, sl);
    if (begin > end || (i == 0 && begin != 0) || (i == p.nwg - 1 && end != p.total)) return fail("slices", begin, end);
    int64_t pos = begin;
    while (at > 0 && items[at].first > pos) --at;
    while (at + 1 < items.size() && items[at + 1].first <= pos) ++at;
    while (pos < end) {
      const Item& it = items[at];
      const int len = cu[it.r + 1] - cu[it.r];
      const int span = (int)ma_span_units(m, pre[it.r], len, g, k, p.seg), u0 = (int)(pos - it.first);
      const int u1 = (int)std::min<int64_t>(span, u0 + end - pos);
      const int v0 = std::min(it.tiles, std::max(0, u0 - p.seg)), v1 = std::min(it.tiles, u1 - p.seg);
      if (u1 > p.seg && v0 < v1) {
        if (v0 != taken[at]) return fail("tiles out of order", v0, taken[at]);
        taken[at] = v1;
        if (!(v0 == 0 && v1 == it.tiles)) {
          const int slot = 2 * i + (pos == begin ? 0 : 1);
          if (!slots.insert(slot).second || slot >= 2 * p.nwg) return fail("slot", slot, p.nwg);
          written[{at, i}] = slot;
        }
      }
      pos += u1 - u0;
      if (pos < end || pos == it.first + span) {
        if (pos == it.first + span && at + 1 < items.size()) ++at;
      }
    }
  }
  for (size_t i = 0; i < items.size(); ++i)
    if (taken[i] != items[i].tiles) return fail("tiles missing", taken[i], items[i].tiles);
  std::set<size_t> merged;
  size_t found = 0;
  for (int slice = 1; slice < p.nwg; ++slice) {
    const int64_t unit = ma_slice_begin(slice, sl);
    if (unit >= p.total) continue;
    size_t i = 0;
    while (i + 1 < items.size() && items[i + 1].first <= unit) ++i;
    const Item& it = items[i];
    const int b0 = ma_slice_of((int)it.first + p.seg, sl);
    const int b1 = ma_slice_of((int)it.first + p.seg + it.tiles - 1, sl);
    if (b0 == b1 || slice != b0 + 1) continue;
    if (!merged.insert(i).second) return fail("merged twice", i, slice);
    for (int b = b0; b <= b1; ++b) {
      const int slot = b == b0 ? 2 * b0 + (ma_slice_begin(b0, sl) >= it.first ? 0 : 1) : 2 * b;
      auto w = written.find({i, b});
      if (w == written.end() || w->second != slot) return fail("merge reads a slot that was not written", b, slot);
      ++found;
    }
  }
  if (found != written.size()) return fail("partials not merged", found, (long)written.size());
  return 0;
}

int main(int argc, char** argv) {
  if (argc < 4) return 2;
  const MachineShape mach{std::atoi(argv[1]), std::atoi(argv[2])};
  const int cases = std::atoi(argv[3]);
  std::mt19937 rng(17);
  auto pick = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
  auto log = [&](int lo, int hi) { return std::min(hi, lo + (int)(rng() % (1u << pick(0, 10))) % (hi - lo + 1)); };
  for (int i = 0; i < cases; ++i) {
    const MaskRule m{pick(0, 2) == 0, log(1, 700), pick(0, 3) ? log(0, 90) : 0};
    const int g = (const int[]){1, 2, 3, 7, 8, 16, 32, 130}[pick(0, 7)];
    for (int which = 0; which < kMaKinds; ++which) {
      const MaKind k = ma_kind(which, 0, which <= kMaMid ? ma_kind(which).rows : INT32_MAX);
      const int n = which <= kMaMid ? pick(1, std::max(1, k.rows / g)) : log(1, 200);
      if (!ma_mine(k, n, g)) continue;
      if (int rc = check_tiles(m, log(0, 900), n, g, k)) return rc;
    }
    const int reqs = pick(1, 150), hkv = (const int[]){1, 2, 3, 4, 5, 8, 16, 32}[pick(0, 7)];
    std::vector<int32_t> cu{0}, pre;
    for (int r = 0; r < reqs; ++r) {
      cu.push_back(cu.back() + (pick(0, 3) ? log(0, 300) : pick(0, 2)));
      pre.push_back(pick(0, 4) ? log(0, 900) : pick(0, 100000));
    }
    const MaCosts cost{pick(0, 12), pick(0, 20), pick(1, 6)};
    const MaSplit split = ma_split(m, cu.data(), pre.data(), reqs, g, hkv, pick(0, 1) != 0);
    std::vector<int> taken(reqs, 0);
    for (int j = 0; j < 4; ++j) {
      const MaKind k = j < 3 ? ma_kernel(split, j) : ma_kind(kMaF32);
      for (int r = 0; j < 3 && r < reqs; ++r) {
        const int len = cu[r + 1] - cu[r];
        taken[r] += ma_mine(k, len, g);
        if (ma_mine(k, len, g) && k.which <= kMaMid && len * g > k.rows) return fail("rows above the kernel's", len * g, k.rows);
      }
      for (bool slices : {false, true})
        if (int rc = check_plan(m, cu, pre, g, hkv, k, mach, cost, slices && j < 3)) return rc;
    }
    for (int r = 0; r < reqs; ++r)
      if (taken[r] != (cu[r + 1] > cu[r])) return fail("a request is not taken once", r, taken[r]);
  }
  // Positions and windows at their limits do not overflow.
  for (int which = 0; which < kMaKinds; ++which) {
    const MaKind k = ma_kind(which);
    const int32_t cu[2] = {0, which <= kMaMid ? 1 : 17}, pre[1] = {kMaMaxPos - 17};
    for (const MaskRule m : {MaskRule{1, 0, 0}, MaskRule{0, kMaMaxPos, kMaMaxPos}, MaskRule{0, 1, 0}}) {
      const MaPlan p = ma_plan(m, k, cu, pre, 1, 1, 8, mach, MaCosts{3, 6, 3});
      if (p.blocks < 8 || p.total < 8) return fail("largest positions", p.blocks, p.total);
    }
  }
  std::printf("ok\n");
  return 0;
}
