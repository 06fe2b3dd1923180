// Windowed and tree attention in fp32: fp32 operands, products and sums
// throughout, on v_mfma_f32_16x16x4_f32.
//
// Workgroup = W waves = 16 packed rows of one (request, KV head); its waves take the
// visited 16-key tiles (one page) in turn and merge through LDS.  Per tile and wave
//   S^T[16 keys][16] = K[16][d] . Q^T[d][16]     d / 4 MFMAs
//   O^T[d][16]      += V^T[d][16] . P^T[16][16]  (d / 16) x 4 of them
// A lane reads a run of d / 4 elements of one K row, and the S^T accumulator is the
// P^T operand as it stands.  A score's products are added eight at a time and then
// pair by pair, and the division by the row sum rounds once: a few 1e-7 from 64
// bits.  Bound by latency at small sizes.
#pragma once
#include "attn_f32.hpp"
#include "masked_common.hpp"

namespace dopd {

template <int D, bool TREE, int W = f32_waves<D>()>
__global__ __launch_bounds__(64 * W, 8 / W) void masked_f32_kernel(MaskedArgs a) {
  constexpr int ROWS = ma_kind(kMaF32).rows, KEYS = ma_kind(kMaF32).keys;
  constexpr int KR = D / 4;   // elements of a K row one lane holds
  constexpr int NT = D / 16;  // O^T tiles of 16 dims
  constexpr int OP = D + 4;   // padded row of the merge buffer
  __shared__ float s_o[W][ROWS][OP];
  __shared__ float s_m[W][ROWS], s_l[W][ROWS];

  ma_items<kMaF32>(a, grid_block(blockIdx.x, blockIdx.y), [&](const MaItem& it) {
  const int l = lane_id(), w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int g = (int)a.by_g.d, c = it.c, hkv = a.hkv;
  const int rows = it.n * g, x0 = it.rt * ROWS, last_row = min(rows, x0 + ROWS) - 1;
  const int pre = it.pre, p0 = pre + fast_quot(x0, a.by_g), p1 = pre + fast_quot(last_row, a.by_g);
  const int end = TREE ? pre + it.n : p1 + 1;
  const KeyTiles kt = ma_key_tiles(a.rule, p0, end - 1, KEYS);
  const int low_key = ma_low_key(a.rule, p0);

  const int col = l & 15, qg = l >> 4;
  const int x = min(x0 + col, rows - 1), tok = fast_quot(x, a.by_g);  // (rows past the end repeat the last)
  const int64_t qrow = (int64_t)(it.row0 + tok) * a.hq + c * g + (x - tok * g);
  const uint32_t* mrow = TREE ? a.mask + (int64_t)(it.row0 + tok) * a.words : nullptr;
  float qv[KR];
  {
    const float* qp = static_cast<const float*>(a.q) + qrow * D + KR * qg;
#pragma unroll
    for (int i = 0; i < KR; i += 4) load_to(qv + i, qp + i);
  }
  const int32_t* pt = a.page_table + (int64_t)it.req * a.pt_stride;
  struct Tile {
    float k[KR];     // K[key l % 16][KR qg + 0 ..]
    float v[NT][4];  // v[n][j] = V[key 4 qg + j][dim 16 n + l % 16]
  };
  auto load = [&](Tile& t, int v) {
    const int64_t blk = ((int64_t)pt[seen_page(a, ma_tile(kt, v), low_key, end)] * hkv + c) * (kPage * D);
    const float* kp = static_cast<const float*>(a.k_pool) + blk + col * D + KR * qg;
#pragma unroll
    for (int i = 0; i < KR; i += 4) load_to(t.k + i, kp + i);
    const float* vp = static_cast<const float*>(a.v_pool) + blk + 4 * qg;
#pragma unroll
    for (int n = 0; n < NT; ++n) load_to(t.v[n], vp + (16 * n + col) * kPage);
  };

  f32x4 o[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) o[n] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, lsum = 0.f;  // of this lane's row; lsum of its own keys only

  auto compute = [&](Tile& t, int v) {
    const int base = KEYS * ma_tile(kt, v);
    f32x4 sum[KR / 2];  // of eight products each, then added pair by pair
#pragma unroll
    for (int i = 0; i < KR / 2; ++i) {
      sum[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(t.k[2 * i], qv[2 * i], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
      sum[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(t.k[2 * i + 1], qv[2 * i + 1], sum[i], 0, 0, 0);
#pragma unroll
      for (int b = 1; (i + 1) % (2 * b) == 0; b *= 2) sum[i + 1 - 2 * b] += sum[i + 1 - b];
    }
    f32x4 s = sum[0] * a.scale;
    const bool full = all_see<TREE>(a, base, KEYS, pre, p0, p1);  // uniform
    uint32_t sees = 0xf;
    bool odd = false;
    if (!full) {
      sees = row_sees<TREE>(a, base, pre, end, pre + tok, mrow) >> (4 * qg);
      const uint32_t live = any_sees<TREE>(a, base, p0, end) >> (4 * qg);
      bool bad = false;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (!(sees >> j & 1)) s[j] = -INFINITY;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          if (!(live >> j & 1)) t.v[n][j] = 0.f;
          bad |= !(fabsf(t.v[n][j]) < INFINITY);
        }
      }
      odd = __ballot(bad) != 0;
    }
    float mx = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
    mx = quad_max(mx);
    const float m_new = fmaxf(m, mx);
    const float m_use = m_new == -INFINITY ? 0.f : m_new;  // (no key seen so far: weights 0)
    const float alpha = expf(m - m_use);
    f32x4 p;
#pragma unroll
    for (int j = 0; j < 4; ++j) p[j] = expf(s[j] - m_use);
    lsum = lsum * alpha + ((p[0] + p[1]) + (p[2] + p[3]));
    m = m_new;
#pragma unroll
    for (int n = 0; n < NT; ++n) o[n] *= alpha;
    if (!odd) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int n = 0; n < NT; ++n) o[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(t.v[n][j], p[j], o[n], 0, 0, 0);
    } else {
      for (int r = 0; r < ROWS; ++r) {  // row r alone, V cleared where it sees nothing
        const uint32_t see = (uint32_t)__shfl((int)sees, (l & 48) + r, 64);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          f32x4 on = o[n];
#pragma unroll
          for (int j = 0; j < 4; ++j)
            on = __builtin_amdgcn_mfma_f32_16x16x4f32(see >> j & 1 ? t.v[n][j] : 0.f, p[j], on, 0, 0, 0);
          if (col == r) o[n] = on;
        }
      }
    }
  };

  if (w < kt.n) {
    Tile t0, t1;
    load(t0, w);
    for (int v = w; v < kt.n; v += 2 * W) {
      if (v + W < kt.n) load(t1, v + W);
      compute(t0, v);
      if (v + W >= kt.n) break;
      if (v + 2 * W < kt.n) load(t0, v + 2 * W);
      compute(t1, v + W);
    }
  }
  lsum = quad_sum(lsum);
  if (qg == 0) {
    s_m[w][col] = m;
    s_l[w][col] = lsum;
  }
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int j = 0; j < 4; ++j) s_o[w][col][16 * n + 4 * qg + j] = o[n][j];
  __syncthreads();
  const int live = last_row + 1 - x0;
  for (int i = (int)threadIdx.x; i < live * D; i += 64 * W) {
    const int y = i / D, e = i % D, ty = fast_quot(x0 + y, a.by_g);
    float M = -INFINITY;
#pragma unroll
    for (int u = 0; u < W; ++u) M = fmaxf(M, s_m[u][y]);
    float sum = 0.f, acc = 0.f;
#pragma unroll
    for (int u = 0; u < W; ++u) {
      const float f = s_m[u][y] == -INFINITY ? 0.f : expf(s_m[u][y] - M);  // (a wave that saw nothing of the row)
      sum += f * s_l[u][y];
      acc += f * s_o[u][y][e];
    }
    const int64_t at = (int64_t)(it.row0 + ty) * a.hq + c * g + (x0 + y - ty * g);
    static_cast<float*>(a.out)[at * D + e] = sum == 0.f ? 0.f : F32Quot(sum)(acc);
    if (a.lse && e == 0) a.lse[at] = M + logf(sum);
  }
  });
}

}  // namespace dopd
