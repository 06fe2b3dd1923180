// Windowed and tree attention for requests of more than 16 packed rows (chunks,
// larger trees), bf16 in / fp32 accumulate, over bf16 or E4M3 pages.
//
// Workgroup = 4 waves = one part of an item of 128 packed rows of one (request, KV
// head), 32 rows a wave; two workgroups share a CU.  Packing the g query heads of a
// KV head into the rows lets 128 / g tokens share a tile, so that a window's
// ragged ends take few masked tiles and a small tree fills the matrix units.  Per
// visited tile of 64 keys and wave
//   S^T[64 keys][32] = K[64][d] . Q^T[d][32]      2 x (d / 16) v_mfma_f32_32x32x16_bf16
//   O^T[d][32]      += V^T[d][64] . P^T[64][32]   (d / 32) x 4 of them
// so that a row lives in one lane pair and the S^T accumulator is the P^T operand.
// The tile's four pages go straight into LDS (a page a wave), double-buffered.
// Bound by the matrix units and the softmax for wide items, by HBM for few rows.
#pragma once
#include "masked_few.hpp"

namespace dopd {

constexpr int kRowsThreads = 256;
// bf16 elements of one K or V tile buffer.
template <int D, bool KV8>
constexpr int rows_tile_elems() { return ma_kind(kMaMany).keys * D / (KV8 ? 2 : 1); }

template <int D, bool KV8, bool TREE>
__global__ __launch_bounds__(kRowsThreads, 2) void masked_rows_kernel(MaskedArgs a) {
  constexpr int ROWS = ma_kind(kMaMany).rows, KEYS = ma_kind(kMaMany).keys;
  constexpr int KS = D / 16;    // k-steps of the QK MFMA
  constexpr int ET = D / 32;    // O^T tiles of 32 dims
  constexpr int NCH8 = D / 16;  // E4M3: 16-byte chunks of a K row
  constexpr int TE = rows_tile_elems<D, KV8>();
  constexpr int RS = D + 8;     // padded row of the output staging
  constexpr int kStage = 32 * RS > TE ? 32 * RS : TE;  // (a wave's output block reuses a tile buffer)
  __shared__ __attribute__((aligned(16))) uint16_t sK0[kStage], sK1[kStage], sV0[kStage], sV1[kStage];

  MaItem it;
  if (!ma_find<kMaMany>(a, (int)blockIdx.x, it)) return;  // uniform
  const int tid = (int)threadIdx.x, l = lane_id();
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = (int)a.by_g.d, c = it.c, hkv = a.hkv;
  const int rows = it.n * g;               // packed rows of the request
  const int x0 = it.rt * ROWS;             // first of this item
  const int pre = it.pre;
  const int last_row = min(rows, x0 + ROWS) - 1;
  const int p0 = pre + fast_quot(x0, a.by_g), p1 = pre + fast_quot(last_row, a.by_g);
  const int end = TREE ? pre + it.n : p1 + 1;  // keys of the item: below this
  const KeyTiles kt = ma_key_tiles(a.rule, p0, end - 1, KEYS);
  const int v0 = (int)((int64_t)it.split * kt.n / it.nsplit), v1 = (int)((int64_t)(it.split + 1) * kt.n / it.nsplit);
  const int low_key = ma_low_key(a.rule, p0);

  const int hi = l >> 5;
  const int xw = x0 + 32 * w;              // first packed row of this wave
  const bool active = xw < rows;           // uniform
  const int x = min(xw + (l & 31), rows - 1);  // (rows past the end repeat the last; not stored)
  const int tok = fast_quot(x, a.by_g);
  const int64_t qrow = (int64_t)(it.row0 + tok) * a.hq + c * g + (x - tok * g);
  const uint32_t* mrow = TREE ? a.mask + (int64_t)(it.row0 + tok) * a.words : nullptr;

  // Q^T operand: Q[row][16 ks + 8 hi + 0..7] (E4M3: the dims a 16-byte read of a K
  // row gives a lane over two k-steps).
  bf16x8 qop[KS];
  {
    const uint16_t* qp = static_cast<const uint16_t*>(a.q) + qrow * D + (KV8 ? 16 : 8) * hi;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      qop[ks] = __builtin_bit_cast(
          bf16x8, *reinterpret_cast<const u32x4*>(qp + (KV8 ? 32 * (ks / 2) + 8 * (ks % 2) : 16 * ks)));
  }
  f32x16 oacc[ET];
#pragma unroll
  for (int et = 0; et < ET; ++et)
#pragma unroll
    for (int i = 0; i < 16; ++i) oacc[et][i] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  const float c_in = KV8 ? a.scale * a.k_scale[c] : a.scale;
  const bool pos = c_in > 0.f;  // else scores are scaled before their maximum is taken
  const float c_eff = pos ? c_in : 1.f;

  // ---- tiles: wave w brings page w of a tile.  K (bf16) in 16-byte chunks,
  // [D / 32 chunk groups][64 rows][4 slots], chunk ch of row t in slot (ch % 4) ^
  // ((t / 4) % 4), rows in the order pi (bits 2 and 3 of a page slot swapped) that
  // makes a lane's weights 8 consecutive keys per P.V k-step; V [D / 32 dim
  // groups][8 key chunks][32 dims][8 keys].  E4M3: the page blocks as they are, K
  // rows in the order pi with their chunks swizzled by row.
  const int32_t* pt = a.page_table + (int64_t)it.req * a.pt_stride;
  auto page_of = [&](int v) {  // (a vector load, made uniform where it is used)
    return pt[seen_page(a, (KEYS / kPage) * ma_tile(kt, min(v, v1 - 1)) + w, low_key, end)];
  };
  const int k_t = 16 * w + (l >> 2);
  const int pk_slot = ((l >> 2) & 3) | ((l >> 3) & 4) | ((l >> 1) & 8);
  const int lane_k = KV8 ? [&] {
    const int s8 = l / NCH8, pc = l % NCH8;
    return ((s8 & 3) | ((s8 & 4) << 1) | ((s8 & 8) >> 1)) * D + 16 * (pc ^ (s8 % NCH8));
  }() : pk_slot * (2 * D) + 16 * ((l & 3) ^ ((k_t >> 2) & 3));
  const int lane_v = KV8 ? 16 * l : (l & 31) * (2 * kPage) + 16 * (l >> 5);
  constexpr int kPageBytes = kPage * D * (KV8 ? 1 : 2);
  auto stage = [&](const void* pool, uint16_t* lds, int page, int lane_off, int step) {
    const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(
        (void*)(static_cast<const char*>(pool) + ((int64_t)page * hkv + c) * kPageBytes), (short)0, kPageBytes,
        0x00020000);
#pragma unroll
    for (int u = 0; u < kPageBytes / 1024; ++u)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rsrc, (__attribute__((address_space(3))) void*)(lds + (KV8 ? (w * kPageBytes + 1024 * u) / 2 : (4 * u + w) * 512)),
          16, lane_off, step * u, 0, 0);
  };
  // (E4M3 K: rows s and s + 8 of a page block are page slots pi(s) and pi(s) + 4.)
  auto load_tile = [&](uint16_t* k, uint16_t* v, int page) {
    stage(a.k_pool, k, page, lane_k, KV8 ? 4 * D : 64);
    stage(a.v_pool, v, page, lane_v, KV8 ? 1024 : 64 * kPage);
  };

  // A operands of the QK MFMA: K[32 tt + l % 32][16 ks + 8 hi + 0..7].
  const int kr_m = hi ^ ((l >> 2) & 3);
  const int kr_even = (l & 31) * 32 + 8 * kr_m, kr_odd = (l & 31) * 32 + 8 * (kr_m ^ 2);
  auto kread = [&](const uint16_t* sk, int tt, bf16x8 (&ka)[KS]) {
    if constexpr (KV8) {
      const int row = 32 * tt + (l & 31);
#pragma unroll
      for (int p = 0; p < KS / 2; ++p) {
        const u32x4 q = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint8_t*>(sk) + row * D +
                                                        16 * ((2 * p + hi) ^ (row % NCH8)));
        ka[2 * p] = __builtin_bit_cast(bf16x8, few_v_operand(u32x2{q[0], q[1]}));
        ka[2 * p + 1] = __builtin_bit_cast(bf16x8, few_v_operand(u32x2{q[2], q[3]}));
      }
    } else {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        ka[ks] = *reinterpret_cast<const bf16x8*>(sk + (ks >> 1) * (KEYS * 32) + tt * 1024 + ((ks & 1) ? kr_odd : kr_even));
    }
  };
  // A operand of P.V k-step kk: V^T[32 et + l % 32][keys 16 kk + 8 hi + 0..7].
  auto vread = [&](const uint16_t* sv, int kk, int et) {
    if constexpr (KV8)
      return few_v_operand(*reinterpret_cast<const u32x2*>(reinterpret_cast<const uint8_t*>(sv) + kk * (kPage * D) +
                                                           (32 * et + (l & 31)) * kPage + 8 * hi));
    else
      return *reinterpret_cast<const u32x4*>(sv + ((et * 8 + 2 * kk + hi) * 32 + (l & 31)) * 8);
  };

  bf16x8 p[4];  // P^T: B operands of the four P.V k-steps
  // Weights against m_use; returns this lane's half of the row sum.
  auto weights = [&](const f32x16 (&s)[2], float m_use) {
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[tt][i], c_eff, -m_use));
        sum[i & 3] += e;
        p[2 * tt + (i >> 3)][i & 7] = (__bf16)e;
      }
    return (sum[0] + sum[1]) + (sum[2] + sum[3]);
  };
  auto raise_max = [&](const f32x16 (&s)[2]) {
    float mx = __builtin_elementwise_maximum(s[0][0], s[1][0]);
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = __builtin_elementwise_maximum(mx, __builtin_elementwise_maximum(s[0][i], s[1][i]));
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
    mx = __builtin_elementwise_maximum(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * c_eff;
    // The running maximum moves only where a tile raises it by more than 8 (log2), so
    // that most tiles rescale nothing; the weights then stay below 2^8.
    if (__ballot(!(mx <= m_run + 8.f)) == 0) return;  // (a NaN moves it too; -inf: stays)
    const float m_new = fmaxf(m_run, mx);
    const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
    m_run = m_new;
    l_run *= alpha;
#pragma unroll
    for (int et = 0; et < ET; ++et) oacc[et] *= alpha;
  };

  auto step = [&](const uint16_t* sk, const uint16_t* sv, int v) {
    const int base = KEYS * ma_tile(kt, v);
    f32x16 s[2];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[tt][i] = 0.f;
      bf16x8 ka[KS];
      kread(sk, tt, ka);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) s[tt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[ks], qop[ks], s[tt], 0, 0, 0);
    }
    const bool full = all_see<TREE>(a, base, KEYS, pre, p0, p1);  // uniform
    if (full && pos) {
      // No maximum is taken: the weights are formed against the running one, and only
      // a sum beyond 2^20 (a tile far above it; the first one seen) takes it.
      float sum = weights(s, m_run);
      if (__ballot(!(sum <= 1048576.f))) {
        raise_max(s);
        sum = weights(s, m_run);
      }
      l_run += sum;
#pragma unroll
      for (int kk = 0; kk < 4; ++kk)
#pragma unroll
        for (int et = 0; et < ET; ++et)
          oacc[et] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vread(sv, kk, et)), p[kk],
                                                             oacc[et], 0, 0, 0);
      return;
    }
    uint32_t sees[2], live[2];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      if (!pos) s[tt] *= c_in;
      sees[tt] = row_sees<TREE>(a, base + 32 * tt, pre, end, pre + tok, mrow);
      live[tt] = any_sees<TREE>(a, base + 32 * tt, p0, end) >> (8 * hi);
#pragma unroll
      for (int i = 0; i < 16; ++i)  // accumulator row i is key 16 (i / 8) + 8 hi + i % 8
        if (!(sees[tt] >> (16 * (i >> 3) + 8 * hi + (i & 7)) & 1)) s[tt][i] = -INFINITY;
    }
    raise_max(s);
    l_run += weights(s, m_run == -INFINITY ? 0.f : m_run);  // (nothing seen so far: weights 0)
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      const uint32_t keep = live[kk >> 1] >> (16 * (kk & 1));
      u32x4 va[ET];
      u16x2 top = {0, 0};
#pragma unroll
      for (int et = 0; et < ET; ++et) {
        va[et] = keep_bf16x8(vread(sv, kk, et), keep);
        top = max_magnitude(va[et], top);
      }
      if (!any_non_finite(top)) {
#pragma unroll
        for (int et = 0; et < ET; ++et)
          oacc[et] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, va[et]), p[kk], oacc[et], 0, 0, 0);
      } else {
        for (int r = 0; r < 32; ++r) {  // row r alone, V cleared where it sees nothing
          const uint32_t see = (uint32_t)__builtin_amdgcn_readlane((int)sees[kk >> 1], r) >> (16 * (kk & 1) + 8 * hi);
#pragma unroll
          for (int et = 0; et < ET; ++et) {
            const f32x16 o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                __builtin_bit_cast(bf16x8, keep_bf16x8(va[et], see)), p[kk], oacc[et], 0, 0, 0);
            if ((l & 31) == r) oacc[et] = o;
          }
        }
      }
    }
  };

  // Tile v sits in buffer (v - v0) % 2.  One barrier a step: it waits for the tile's
  // loads and for the waves that still read the buffer the next loads go into.
  if (v0 < v1) {
    load_tile(sK0, sV0, __builtin_amdgcn_readfirstlane(page_of(v0)));
    int ahead = page_of(v0 + 1);
    int v = v0;
    while (true) {
      __syncthreads();
      if (v + 1 < v1) load_tile(sK1, sV1, __builtin_amdgcn_readfirstlane(ahead));
      ahead = page_of(v + 2);
      if (active) step(sK0, sV0, v);
      if (++v >= v1) break;
      __syncthreads();
      if (v + 1 < v1) load_tile(sK0, sV0, __builtin_amdgcn_readfirstlane(ahead));
      ahead = page_of(v + 2);
      if (active) step(sK1, sV1, v);
      if (++v >= v1) break;
    }
  }
  __syncthreads();  // the tile buffers become the waves' output staging
  if (!active) return;

  const float L = l_run + __shfl_xor(l_run, 32, 64);
  const float vsc = KV8 ? a.v_scale[c] : 1.f;
  const bool mine = xw + (l & 31) < rows;
  if (it.nsplit > 1) {
    const int64_t at = it.slot * ROWS + 32 * w + (l & 31);
    if (mine) {
      float* po = a.part_o + at * D + 4 * hi;
#pragma unroll
      for (int et = 0; et < ET; ++et)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<f32x4*>(po + 32 * et + 8 * q) =
              f32x4{oacc[et][4 * q], oacc[et][4 * q + 1], oacc[et][4 * q + 2], oacc[et][4 * q + 3]} * vsc;
      if (hi == 0) *reinterpret_cast<float2*>(a.part_ml + at * 2) = float2{m_run, L};
    }
    return;
  }
  const float inv = L == 0.f ? 0.f : vsc / L;
  // Through LDS, so that 16 lanes store one 256-byte row.
  uint16_t* so = w == 0 ? sK0 : w == 1 ? sK1 : w == 2 ? sV0 : sV1;
#pragma unroll
  for (int et = 0; et < ET; ++et)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      u32x2 o2;
      o2[0] = pack_bf16x2(oacc[et][4 * q] * inv, oacc[et][4 * q + 1] * inv);
      o2[1] = pack_bf16x2(oacc[et][4 * q + 2] * inv, oacc[et][4 * q + 3] * inv);
      *reinterpret_cast<u32x2*>(so + (l & 31) * RS + 32 * et + 8 * q + 4 * hi) = o2;
    }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  constexpr int CH = D / 8;
#pragma unroll
  for (int u = 0; u < 32 * CH / 64; ++u) {
    const int i = l + 64 * u, rr = i / CH, ch = i % CH;
    const u32x4 o4 = *reinterpret_cast<const u32x4*>(so + rr * RS + 8 * ch);
    const int y = xw + rr, ty = fast_quot(y, a.by_g);
    if (y < rows)
      __builtin_nontemporal_store(
          o4, reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.out) +
                                       ((int64_t)(it.row0 + ty) * a.hq + c * g + (y - ty * g)) * D + 8 * ch));
  }
  if (a.lse && hi == 0 && mine) a.lse[qrow] = (m_run + __log2f(L)) * kLn2;
}

}  // namespace dopd
