// Windowed and tree attention for requests of at most 16 packed rows (decode steps,
// small trees), bf16 in / fp32 accumulate, over bf16 or E4M3 pages.
//
// Workgroup = 4 waves = one (request, KV head), or a slice of the call's items: the
// visited pairs of pages (32 keys) are taken by the waves in turn and merged through
// LDS.  Per pair and wave, the packed rows being the 16 MFMA columns,
//   S^T[32 keys][16] = K[32][d] . Q^T[d][16]     2 x (d / 32) v_mfma_f32_16x16x32_bf16
//   O^T[d][16]      += V^T[d][32] . P^T[32][16]  (d / 16) of them
// with an online softmax in the exp2 domain.  Every K and V operand is one 16-byte
// load (E4M3: 16 bytes of K, 8 of V) straight from the pages; the key order inside a
// pair makes the S^T accumulator the P^T operand.
//
// HBM-bound: each page that some row sees is read once for all rows of the group.
// Two workgroups a CU, two pairs in flight a wave.
// The row sums add the unrounded weights, so that lse keeps fp32 precision; P is
// rounded to bf16 for the MFMA only, half a step of 2^-8 a weight.
#pragma once
#include <type_traits>

#include "masked_common.hpp"

namespace dopd {

constexpr int kFewWaves = 4;

template <int D, bool KV8>
struct FewPair {
  u32x4 k1[D / 32], k2[D / 32];  // K rows of the two QK MFMAs
  u32x4 v[D / 16];               // V^T rows, one per 16-dim tile
};
template <int D>
struct FewPair<D, true> {  // raw E4M3 codes
  u32x4 k1[D / 64], k2[D / 64];
  u32x2 v[D / 16];
};

// bf16 operand i of a K run.
template <bool KV8>
__device__ __forceinline__ bf16x8 few_k_operand(const u32x4* k, int i) {
  if constexpr (KV8) {
    const u32x4 w = k[i >> 1];
    const u32x2 lo = bf16x4_from_e4m3x4(w[2 * (i & 1)]), hi = bf16x4_from_e4m3x4(w[2 * (i & 1) + 1]);
    return __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
  } else {
    return __builtin_bit_cast(bf16x8, k[i]);
  }
}
template <int D, bool KV8, bool TREE>
__global__ __launch_bounds__(64 * kFewWaves, 2) void masked_few_kernel(MaskedArgs a) {
  using KT = std::conditional_t<KV8, uint8_t, uint16_t>;
  using VT = std::conditional_t<KV8, u32x2, u32x4>;  // eight keys of a V row
  constexpr int ROWS = ma_kind(kMaFew).rows, KEYS = ma_kind(kMaFew).keys;
  constexpr int NQK = D / 32, NT = D / 16, W = kFewWaves;
  constexpr int kChunk = 32 * W;  // pairs whose page ids a workgroup's lanes hold at once
  __shared__ __attribute__((aligned(16))) f32x4 s_o[W][NT * 64];
  __shared__ float s_m[W][ROWS], s_l[W][ROWS];
  __shared__ uint32_t s_bad[W];

  ma_items<kMaFew>(a, grid_block(blockIdx.x, blockIdx.y), [&](const MaItem& it) {
  const int l = lane_id(), w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int g = (int)a.by_g.d, c = it.c, hkv = a.hkv;
  const int rows = it.n * g;
  const int pre = it.pre, end = pre + it.n, p1 = end - 1;
  const KeyTiles kt = ma_key_tiles(a.rule, pre, p1, KEYS);
  int v0, v1;
  const bool whole = ma_tiles_of(a, it, kt.n, v0, v1);
  if (v0 >= v1) return;
  const int low_key = ma_low_key(a.rule, pre);

  const int col = l & 15, qg = l >> 4;  // MFMA column = packed row; lane group = k-slot group
  const int x = min(col, rows - 1), tok = fast_quot(x, a.by_g);  // (past the end: the last row, not stored)
  const int64_t qrow = (int64_t)(it.row0 + tok) * a.hq + c * g + (x - tok * g);
  const int tq1 = 8 * (col >> 2) + (col & 3);  // MFMA #1 rows: pair keys 0-3, 8-11, 16-19, 24-27; #2: +4
  const int64_t page_elems = (int64_t)hkv * kPage * D;

  // Q^T operand i holds the dims its K operand holds: load n of a K row gives lane
  // group qg the elements KST n + KEL qg + 0 .. KEL-1.
  constexpr int KEL = 16 / (int)sizeof(KT), KST = 4 * KEL;
  bf16x8 qop[NQK];
  {
    const uint16_t* qp = static_cast<const uint16_t*>(a.q) + qrow * D + KEL * qg;
#pragma unroll
    for (int i = 0; i < NQK; ++i)
      qop[i] = __builtin_bit_cast(
          bf16x8, *reinterpret_cast<const u32x4*>(qp + (KV8 ? KST * (i / 2) + 8 * (i % 2) : KST * i)));
  }
  f32x4 oacc[NT];
  float m_run, l_run;
  auto clear = [&] {
    m_run = -INFINITY;
    l_run = 0.f;
#pragma unroll
    for (int n = 0; n < NT; ++n) oacc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
  };
  clear();
  const float sl2 = KV8 ? a.scale * a.k_scale[c] : a.scale;

  const KT* kbase = static_cast<const KT*>(a.k_pool) + (int64_t)c * kPage * D + (tq1 & 15) * D + KEL * qg;
  const KT* vbase = static_cast<const KT*>(a.v_pool) + (int64_t)c * D * kPage + col * kPage + 8 * (qg & 1);
  const int32_t* pt = a.page_table + (int64_t)it.req * a.pt_stride;

  // One pass over the wave's pairs.  careful: V is cleared, row by row, where the row
  // sees nothing.
  auto pass = [&](auto careful) {
  for (int cb = v0; cb < v1; cb += kChunk) {
    const int npairs = min(v1 - cb, kChunk);
    const int mine = npairs > w ? (npairs - w + W - 1) / W : 0;
    // Lane j holds the id of page j & 1 of the wave's pair j / 2 of the chunk.
    const int pv = min(cb + w + W * (l >> 1), v1 - 1);
    const int pid = pt[seen_page(a, 2 * ma_tile(kt, pv) + (l & 1), low_key, end)];

    auto load = [&](FewPair<D, KV8>& buf, int k) {
      const int64_t pa = __builtin_amdgcn_readlane(pid, 2 * k), pb = __builtin_amdgcn_readlane(pid, 2 * k + 1);
      const KT* kp = kbase + (tq1 < kPage ? pa : pb) * page_elems;  // (tq1 and tq1 + 4: one page)
#pragma unroll
      for (int i = 0; i < D / KST; ++i) {
        buf.k1[i] = *reinterpret_cast<const u32x4*>(kp + KST * i);
        buf.k2[i] = *reinterpret_cast<const u32x4*>(kp + 4 * D + KST * i);
      }
      const KT* vp = vbase + (qg < 2 ? pa : pb) * page_elems;
#pragma unroll
      for (int n = 0; n < NT; ++n) buf.v[n] = *reinterpret_cast<const VT*>(vp + 16 * n * kPage);
    };

    auto compute = [&](FewPair<D, KV8>& buf, int k) {
      const int base = KEYS * ma_tile(kt, cb + w + W * k);  // first key of the pair
      f32x4 s1 = {0.f, 0.f, 0.f, 0.f}, s2 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NQK; ++i) {
        s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(few_k_operand<KV8>(buf.k1, i), qop[i], s1, 0, 0, 0);
        s2 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(few_k_operand<KV8>(buf.k2, i), qop[i], s2, 0, 0, 0);
      }
      float s[8];  // keys base + 8 qg + 0 .. 7 of this lane's row
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[j] = s1[j] * sl2;
        s[4 + j] = s2[j] * sl2;
      }
      uint32_t sees = 0;
      if (careful() || !all_see<TREE>(a, base, KEYS, pre, pre, p1)) {  // uniform
        const uint32_t* mrow = TREE ? a.mask + (int64_t)(it.row0 + tok) * a.words : nullptr;
        sees = row_sees<TREE>(a, base, pre, end, pre + tok, mrow) >> (8 * qg);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (!(sees >> j & 1)) s[j] = -INFINITY;
        // V that no row sees (slots that may hold anything)
        const uint32_t live = any_sees<TREE>(a, base, pre, end);  // uniform
        if (live != ~0u) {
#pragma unroll
          for (int n = 0; n < NT; ++n) buf.v[n] = keep_of(buf.v[n], live >> (8 * qg));
        }
      }
      float mx = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
      mx = quad_max(mx);
      const float m_new = fmaxf(m_run, mx);
      const float m_use = m_new == -INFINITY ? 0.f : m_new;  // (no key seen so far: weights 0)
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_use);
      m_run = m_new;
      bf16x8 p;
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float e = __builtin_amdgcn_exp2f(s[j] - m_use);
        sum += e;
        p[j] = (__bf16)e;
      }
      l_run = l_run * alpha + sum;
#pragma unroll
      for (int n = 0; n < NT; ++n) oacc[n] *= alpha;
      if constexpr (!careful()) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
          oacc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v_operand(buf.v[n]), p, oacc[n], 0, 0, 0);
      } else {
#pragma unroll 1
        for (int r = 0; r < ROWS; ++r) {
          const uint32_t see = (uint32_t)__shfl((int)sees, (l & 48) + r, 64);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            const f32x4 o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v_operand(keep_of(buf.v[n], see)), p, oacc[n], 0, 0, 0);
            if (col == r) oacc[n] = o;
          }
        }
      }
    };

    if (mine > 0) {
      const int last = mine - 1;
      if constexpr (careful()) {
        FewPair<D, KV8> b;
#pragma unroll 1
        for (int k = 0; k < mine; ++k) {
          load(b, k);
          compute(b, k);
        }
      } else {
        // Loads past the end re-read the last pair (a cache hit), so that the wait is
        // for the buffer being computed alone.
        FewPair<D, KV8> b0, b1;
        load(b0, 0);
        for (int k = 0; k < mine; k += 2) {
          load(b1, min(k + 1, last));
          compute(b0, k);
          load(b0, min(k + 2, last));
          if (k + 1 < mine) compute(b1, k + 1);
        }
      }
    }
  }
  };
  pass(std::false_type{});

  // A value that is not finite, in a pair that only some rows see, has reached rows
  // that do not see it (0 * inf is NaN): then the part is computed again.
  if (l == 0) s_bad[w] = 0;
  if (any_not_finite<NT>(oacc) && l == 0) s_bad[w] = 1;
  __syncthreads();
  if (s_bad[0] | s_bad[1] | s_bad[2] | s_bad[3]) {
    clear();
    pass(std::true_type{});
  }

  // Row sums over the lane groups, then the merge of the waves.
  l_run = quad_sum(l_run);
  if (qg == 0) {
    s_m[w][col] = m_run;
    s_l[w][col] = l_run;
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) s_o[w][n * 64 + l] = oacc[n];
  __syncthreads();
  float M = -INFINITY, L = 0.f, f[W];
#pragma unroll
  for (int u = 0; u < W; ++u) M = fmaxf(M, s_m[u][col]);
#pragma unroll
  for (int u = 0; u < W; ++u) {
    f[u] = s_m[u][col] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s_m[u][col] - M);
    L += f[u] * s_l[u][col];
  }
  const float vsc = KV8 ? a.v_scale[c] : 1.f;
  const float fac = !whole ? vsc : L == 0.f ? 0.f : vsc / L;
#pragma unroll
  for (int n0 = 0; n0 < NT; n0 += W) {
    const int n = n0 + w;
    f32x4 o = s_o[0][n * 64 + l] * f[0];
#pragma unroll
    for (int u = 1; u < W; ++u) o += s_o[u][n * 64 + l] * f[u];
    o *= fac;
    if (col >= rows) continue;
    if (whole) store_bf16x4(a.out, qrow * D + 16 * n + 4 * qg, o);
    else *reinterpret_cast<f32x4*>(a.part_o + ((int64_t)it.slot * ROWS + col) * D + 16 * n + 4 * qg) = o;
  }
  if (w == 0 && qg == 0 && col < rows) {
    if (!whole) *reinterpret_cast<float2*>(a.part_ml + ((int64_t)it.slot * ROWS + col) * 2) = float2{M, L};
    else if (a.lse) a.lse[qrow] = (M + __log2f(L)) * kLn2;
  }
  __syncthreads();  // the next item reuses the buffers
  });
}

}  // namespace dopd
