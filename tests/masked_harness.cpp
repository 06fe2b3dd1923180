// CPU check of the planning of the windowed and the tree attention
// (paper_2511_20982_amd/csrc/plan_masked.hpp): the visited tiles hold every position
// a row sees, the pages read are pages that some row sees, the workgroups of a plan
// cover every part of every item once, and their partial slots are distinct.
// Usage: masked_harness <cus> <xcds> <cases>; prints "ok" or the first failure.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <set>
#include <tuple>
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

static int check_plan(const MaskRule& m, const std::vector<int32_t>& cu, const std::vector<int32_t>& pre, int g,
                      int hkv, const MaKind& k, const MachineShape& mach) {
  const int n = (int)pre.size();
  const MaDeal d = ma_deal(hkv, mach.xcds);
  const MaPlan p = ma_plan(m, k, cu.data(), pre.data(), n, g, hkv, mach, 4, 3);
  int64_t base = 0, slot0 = 0, merges = 0;
  std::set<std::tuple<int, int, int>> seen;
  std::set<int64_t> slots;
  for (int r = 0; r < n; ++r) {
    const int len = cu[r + 1] - cu[r];
    if (!ma_mine(k, len, g)) continue;
    const int rt = ma_row_tiles(len, g, k.rows), s = ma_splits(ma_most_tiles(m, pre[r], len, g, k), p.target);
    if (s > kMaMaxSplits * 2) return fail("splits", s, p.target);
    const int parts = rt * s;
    const int64_t blocks = ma_blocks(d, hkv, parts);
    if (d.share && (blocks % mach.xcds || base % mach.xcds)) return fail("XCD phase", blocks, base);
    for (int64_t b = 0; b < blocks; ++b) {
      int c, idx;
      if (!ma_part(d, hkv, parts, (int)b, c, idx)) continue;
      if (c < 0 || c >= hkv || idx < 0 || idx >= parts) return fail("part out of range", c, idx);
      if (!seen.insert({r, c, idx}).second) return fail("part dealt twice", r, idx);
      if (s > 1 && !slots.insert(slot0 + (int64_t)c * parts + idx).second) return fail("slot used twice", r, idx);
    }
    if ((int64_t)seen.size() == 0) return fail("no part", r, parts);
    base += blocks;
    if (s > 1) {
      slot0 += (int64_t)hkv * parts;
      merges += (int64_t)hkv * rt;
    }
  }
  int64_t want = 0;
  for (int r = 0; r < n; ++r) {
    const int len = cu[r + 1] - cu[r];
    if (ma_mine(k, len, g))
      want += (int64_t)hkv * ma_row_tiles(len, g, k.rows) * ma_splits(ma_most_tiles(m, pre[r], len, g, k), p.target);
  }
  if ((int64_t)seen.size() != want) return fail("parts missing", (long)seen.size(), want);
  if (base != p.blocks || slot0 != p.slots || merges != p.merges) return fail("totals", base, p.blocks);
  if (!slots.empty() && *slots.rbegin() >= p.slots) return fail("slot past the workspace", *slots.rbegin(), p.slots);
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
    for (int which : {(int)kMaFew, (int)kMaMany, (int)kMaF32}) {
      const MaKind k = ma_kind(which);
      const int n = which == kMaFew ? pick(1, std::max(1, 16 / g)) : log(1, 200);
      if (!ma_mine(k, n, g)) continue;
      if (int rc = check_tiles(m, log(0, 900), n, g, k)) return rc;
    }
    const int reqs = pick(1, 150), hkv = (const int[]){1, 2, 3, 4, 5, 8, 16, 32}[pick(0, 7)];
    std::vector<int32_t> cu{0}, pre;
    for (int r = 0; r < reqs; ++r) {
      cu.push_back(cu.back() + (pick(0, 3) ? log(0, 300) : pick(0, 2)));
      pre.push_back(pick(0, 4) ? log(0, 900) : pick(0, 100000));
    }
    for (int which : {(int)kMaFew, (int)kMaMany})
      if (int rc = check_plan(m, cu, pre, g, hkv, ma_kind(which), mach)) return rc;
  }
  // Positions and windows at their limits do not overflow.
  for (int which : {(int)kMaFew, (int)kMaMany, (int)kMaF32}) {
    const MaKind k = ma_kind(which);
    const int32_t cu[2] = {0, which == kMaFew ? 1 : 17}, pre[1] = {kMaMaxPos - 17};
    for (const MaskRule m : {MaskRule{1, 0, 0}, MaskRule{0, kMaMaxPos, kMaMaxPos}, MaskRule{0, 1, 0}}) {
      const MaPlan p = ma_plan(m, k, cu, pre, 1, 1, 8, mach, 4, 3);
      if (which != kMaF32 && (p.blocks < 8 || p.slots < 0)) return fail("largest positions", p.blocks, p.slots);
    }
  }
  std::printf("ok\n");
  return 0;
}
