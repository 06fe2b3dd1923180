// Windowed and tree attention for requests of more than 64 packed rows (chunks,
// larger trees), bf16 in / fp32 accumulate, over bf16 or E4M3 pages.
//
// Workgroup = 4 waves = an item of 128 packed rows of one (request, KV head), 32 rows
// a wave, or a slice of the call's items; two workgroups share a CU.  Packing the g query heads of a
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
  constexpr int kStage = 32 * RS + 8 > TE ? 32 * RS + 8 : TE;  // (a wave's output block reuses a tile buffer)
  __shared__ __attribute__((aligned(16))) uint16_t sK0[kStage], sK1[kStage], sV0[kStage], sV1[kStage];
  // Q operands KS / 2 .. of every lane, read from here by every step but a tree's full
  // ones: held in registers there too, some were spilled, and a reload waits for the
  // tiles in flight (16 chunks of 512 x 32 heads, window 1024, bf16: 298 us, and 264 this way).
  __shared__ __attribute__((aligned(16))) uint16_t sQ[KS / 2 * kRowsThreads * 8];

  ma_items<kMaMany>(a, grid_block(blockIdx.x, blockIdx.y), [&](const MaItem& it) {
  const int l = lane_id(), hi = l >> 5;
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int g = (int)a.by_g.d, c = it.c, hkv = a.hkv;
  const int rows = it.n * g;               // packed rows of the request
  const int x0 = it.rt * ROWS;             // first of this item
  const int pre = it.pre;
  const int last_row = min(rows, x0 + ROWS) - 1;
  const int p0 = pre + fast_quot(x0, a.by_g), p1 = pre + fast_quot(last_row, a.by_g);
  const int end = TREE ? pre + it.n : p1 + 1;  // keys of the item: below this
  const KeyTiles kt = ma_key_tiles(a.rule, p0, end - 1, KEYS);
  int v0, v1;
  const bool whole = ma_tiles_of(a, it, kt.n, v0, v1);
  if (v0 >= v1) return;
  const int low_key = ma_low_key(a.rule, p0);

  const int xw = x0 + 32 * w;              // first packed row of this wave
  const bool active = xw < rows;           // uniform
  // Lane l's packed row (past the end: the last, not stored), token and row of Q.
  auto row_of = [&](int l) { return min(xw + (l & 31), rows - 1); };
  auto token_of = [&](int l) { return fast_quot(row_of(l), a.by_g); };
  auto q_row = [&](int l) {
    const int x = row_of(l), tok = fast_quot(x, a.by_g);
    return (int64_t)(it.row0 + tok) * a.hq + c * g + (x - tok * g);
  };
  // Scores are c_in > 0 times K . Q: the scale's sign goes to Q, and so does a scale of
  // 0 (inf becomes NaN there, as it would).
  const float scale = KV8 ? a.scale * a.k_scale[c] : a.scale;
  const float c_in = scale == 0.f ? 1.f : __builtin_fabsf(scale);
  auto signed_q = [&](u32x4 q) {
    if (!(scale > 0.f)) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (scale < 0.f) {
          q[i] ^= 0x80008000u;
        } else if (scale == 0.f) {
          const uint32_t lo = q[i] & 0x7f80, top = q[i] & 0x7f800000;
          q[i] = (lo == 0x7f80 ? 0x7fc0u : 0u) | (top == 0x7f800000 ? 0x7fc00000u : 0u);
        }
    }
    return q;
  };

  // Q^T operand: Q[row][16 ks + 8 hi + 0..7] (E4M3: the dims a 16-byte read of a K
  // row gives a lane over two k-steps).  The upper half stays in LDS (this lane's own
  // slots: no barrier needed) and comes to registers for runs of full tiles.
  constexpr int KH = KS / 2;
  bf16x8 qlo[KH];
  {
    const uint16_t* qp = static_cast<const uint16_t*>(a.q) + q_row(l) * D + (KV8 ? 16 : 8) * hi;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const u32x4 q = signed_q(*reinterpret_cast<const u32x4*>(qp + (KV8 ? 32 * (ks / 2) + 8 * (ks % 2) : 16 * ks)));
      if (ks < KH) qlo[ks] = __builtin_bit_cast(bf16x8, q);
      else *reinterpret_cast<u32x4*>(sQ + ((ks - KH) * kRowsThreads + 64 * w + l) * 8) = q;
    }
  }
  auto qhi_lds = [&](int i) { return *reinterpret_cast<const bf16x8*>(sQ + (i * kRowsThreads + 64 * w + l) * 8); };
  f32x16 oacc[ET];
#pragma unroll
  for (int et = 0; et < ET; ++et)
#pragma unroll
    for (int i = 0; i < 16; ++i) oacc[et][i] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;

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
  auto lane_k = [&] {
    if constexpr (KV8) {
      const int s8 = l / NCH8, pc = l % NCH8;
      return ((s8 & 3) | ((s8 & 4) << 1) | ((s8 & 8) >> 1)) * D + 16 * (pc ^ (s8 % NCH8));
    }
    const int k_t = 16 * w + (l >> 2), slot = ((l >> 2) & 3) | ((l >> 3) & 4) | ((l >> 1) & 8);
    return slot * (2 * D) + 16 * ((l & 3) ^ ((k_t >> 2) & 3));
  };
  auto lane_v = [&] { return KV8 ? 16 * l : (l & 31) * (2 * kPage) + 16 * (l >> 5); };
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
  constexpr int kStepK = KV8 ? 4 * D : 64, kStepV = KV8 ? 1024 : 64 * kPage;

  // A operands of the QK MFMA: K[32 tt + l % 32][16 ks + 8 hi + 0..7].
  auto kread = [&](const uint16_t* sk, int tt, bf16x8 (&ka)[KS]) {
    if constexpr (KV8) {
      const int row = 32 * tt + (l & 31);
#pragma unroll
      for (int p = 0; p < KS / 2; ++p) {
        const u32x4 q = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint8_t*>(sk) + row * D +
                                                        16 * ((2 * p + hi) ^ (row % NCH8)));
        ka[2 * p] = v_operand(u32x2{q[0], q[1]});
        ka[2 * p + 1] = v_operand(u32x2{q[2], q[3]});
      }
    } else {
      const int kr_m = hi ^ ((l >> 2) & 3);
      const int kr_even = (l & 31) * 32 + 8 * kr_m, kr_odd = (l & 31) * 32 + 8 * (kr_m ^ 2);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        ka[ks] = *reinterpret_cast<const bf16x8*>(sk + (ks >> 1) * (KEYS * 32) + tt * 1024 + ((ks & 1) ? kr_odd : kr_even));
    }
  };
  // A operand of P.V k-step kk: V^T[32 et + l % 32][keys 16 kk + 8 hi + 0..7].
  auto vread = [&](const uint16_t* sv, int kk, int et) {
    if constexpr (KV8)
      return *reinterpret_cast<const u32x2*>(reinterpret_cast<const uint8_t*>(sv) + kk * (kPage * D) +
                                             (32 * et + (l & 31)) * kPage + 8 * hi);
    else
      return *reinterpret_cast<const u32x4*>(sv + ((et * 8 + 2 * kk + hi) * 32 + (l & 31)) * 8);
  };

  bf16x8 p[4];  // P^T: B operands of the four P.V k-steps
  // Weights 2^(c s - m_use); returns this lane's half of the row sum.
  auto weights = [&](const f32x16 (&s)[2], float c, float m_use) {
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[tt][i], c, -m_use));
        sum[i & 3] += e;
        p[2 * tt + (i >> 3)][i & 7] = (__bf16)e;
      }
    return (sum[0] + sum[1]) + (sum[2] + sum[3]);
  };
  auto row_max = [&](const f32x16 (&s)[2]) {
    float mx = __builtin_elementwise_maximum(s[0][0], s[1][0]);
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = __builtin_elementwise_maximum(mx, __builtin_elementwise_maximum(s[0][i], s[1][i]));
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
    return __builtin_elementwise_maximum(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
  };
  // The running maximum becomes m_new; O and the row sum follow.
  auto rescale = [&](float m_new) {
    const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
    m_run = m_new;
    l_run *= alpha;
#pragma unroll
    for (int et = 0; et < ET; ++et) oacc[et] *= alpha;
  };
  // S^T of a tile; qhi(i): Q operand KH + i.
  auto qk = [&](const uint16_t* sk, f32x16 (&s)[2], auto qhi) {
    bf16x8 ka[2][KS];
    kread(sk, 0, ka[0]);
    kread(sk, 1, ka[1]);
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[tt][i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const bf16x8 qv = ks < KH ? qlo[ks < KH ? ks : 0] : qhi(ks - KH);
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) s[tt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[tt][ks], qv, s[tt], 0, 0, 0);
    }
  };
  auto pv = [&](const uint16_t* sv) {
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int et = 0; et < ET; ++et)
        oacc[et] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_operand(vread(sv, kk, et)), p[kk], oacc[et], 0,
                                                           0, 0);
  };
  // Makes the scores of what a row does not see -inf; sees: by 32 keys of the tile.  The
  // lane is found anew, so that nothing for it is held (and spilled) over other steps.
  auto hide = [&](f32x16 (&s)[2], int base, uint32_t (&sees)[2]) {
    int l;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=&v"(l));
    const int tok = token_of(l);
    const uint32_t* mrow = TREE ? a.mask + (int64_t)(it.row0 + tok) * a.words : nullptr;
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      sees[tt] = row_sees<TREE>(a, base + 32 * tt, pre, end, pre + tok, mrow) >> (8 * (l >> 5));
#pragma unroll
      for (int i = 0; i < 16; ++i)  // accumulator row i is key 16 (i / 8) + 8 hi + i % 8
        s[tt][i] = sees[tt] >> (16 * (i >> 3) + (i & 7)) & 1 ? s[tt][i] : -INFINITY;
    }
  };
  // V of positions of visited tile v that no row of the item sees (slots that may hold
  // anything: 0 * NaN is NaN) is cleared in LDS by the wave that brought its page, once
  // that has landed; the barrier that ends the step publishes it.
  auto clear_dead = [&](uint16_t* sv, int v) {
    if (v >= v1) return;
    const uint32_t live = any_sees<TREE>(a, KEYS * ma_tile(kt, v) + kPage * w, p0, end) & 0xffff;  // uniform
    if (live == 0xffff) return;
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
    if constexpr (KV8) {  // [D dim rows][16 key bytes]: two halves a row
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        const int j = l + 64 * i;
        u32x2* x = reinterpret_cast<u32x2*>(reinterpret_cast<uint8_t*>(sv) + w * (kPage * D) + j * 8);
        *x = keep_of(*x, live >> (8 * (j & 1)));
      }
    } else {
#pragma unroll
      for (int et = 0; et < ET; ++et) {
        u32x4* x = reinterpret_cast<u32x4*>(sv + ((et * 8 + 2 * w + hi) * 32 + (l & 31)) * 8);
        *x = keep_of(*x, live >> (8 * hi));
      }
    }
  };
  // What this wave (positions pw0 .. pw1) has to do, by wave and not by item, because of
  // the few tiles at a window's two ends a wave finds most either whole or empty: tiles
  // va .. ve - 1 are seen in full by its rows (full tiles of sinks go with the masked),
  // none from vl on.
  const int pw0 = pre + fast_quot(min(xw, rows - 1), a.by_g), pw1 = pre + fast_quot(min(xw + 31, rows - 1), a.by_g);
  auto none = [&](int v) {
    if constexpr (TREE) return false;
    const int base = KEYS * ma_tile(kt, v);
    return base + KEYS <= pw0 - a.rule.window + 1 && base >= a.rule.sinks;
  };
  int va = v0, ve, vl;
  if constexpr (TREE) {
    ve = min(v1, pre / KEYS);
    vl = active ? v1 : v0;
  } else {
    const int low = (max(pw1 - a.rule.window + 1, 0) + KEYS - 1) / KEYS;
    va = max(v0, low - kt.low + kt.nsink);
    ve = min(v1, (pw0 + 1) / KEYS - kt.low + kt.nsink);
    vl = active ? min(v1, max(v0, pw1 / KEYS + 1 - kt.low + kt.nsink)) : v0;
  }

  // K tile i (of v0 + i) sits in K buffer i % 2, V tile i in V buffer i % 2, K a tile
  // ahead.  Step i loads K tile i + 2 and V tile i + 1 and, after (or while) it forms
  // the weights of tile i, computes S^T of tile i + 1; the barrier that ends it waits
  // for the loads and for the waves that read what the next ones replace.
  int pid_k, pid_v, ahead;
  auto kbuf = [&](int b) { return b ? sK1 : sK0; };
  auto vbuf = [&](int b) { return b ? sV1 : sV0; };
  auto prefetch = [&](int par, int v) {
    if (v + 2 < v1) stage(a.k_pool, kbuf(par), pid_k, lane_k(), kStepK);
    if (v + 1 < v1) stage(a.v_pool, vbuf(par ^ 1), pid_v, lane_v(), kStepV);
    pid_v = pid_k;
    pid_k = __builtin_amdgcn_readfirstlane(ahead);  // (landed at the last barrier)
    ahead = page_of(v + 4);
  };
  {
    const int first = __builtin_amdgcn_readfirstlane(page_of(v0));
    pid_v = __builtin_amdgcn_readfirstlane(page_of(v0 + 1));
    stage(a.k_pool, sK0, first, lane_k(), kStepK);
    if (v0 + 1 < v1) stage(a.k_pool, sK1, pid_v, lane_k(), kStepK);
    stage(a.v_pool, sV0, first, lane_v(), kStepV);
    pid_k = __builtin_amdgcn_readfirstlane(page_of(v0 + 2));
    ahead = page_of(v0 + 3);
    clear_dead(sV0, v0);
  }
  __syncthreads();
  f32x16 sa[2], sb[2];  // S^T of two consecutive tiles
  qk(sK0, sa, qhi_lds);
  if (va == v0 && v0 < ve) m_run = row_max(sa) * c_in;
  __syncthreads();  // (K tile 2 goes where tile 0 was)

  // A tile's maximum is taken where it is masked.  A full one's weights are formed
  // against the running maximum, and only a sum beyond 2^20 (a tile far above it, the
  // first one seen) takes it.
  int v = v0;
  auto step = [&](f32x16 (&sc)[2], f32x16 (&sn)[2], auto par) {
    prefetch(par(), v);
    if (none(v)) {
      qk(kbuf(par() ^ 1), sn, qhi_lds);
    } else {
      float m_use = m_run;
      if (v < va || v >= ve) {
        uint32_t sees[2];
        hide(sc, KEYS * ma_tile(kt, v), sees);
        rescale(fmaxf(m_run, row_max(sc) * c_in));
        m_use = m_run == -INFINITY ? 0.f : m_run;  // (nothing seen so far: weights 0)
      }
      qk(kbuf(par() ^ 1), sn, qhi_lds);
      if constexpr (!KV8) {
        // The K reads spread over the products: all of them ahead, Q operands are
        // spilled, and a reload waits for the tiles in flight.
        constexpr int kMfma = 0x008, kDsRead = 0x100, kAhead = 6;
        __builtin_amdgcn_sched_group_barrier(kDsRead, kAhead, 0);
#pragma unroll
        for (int i = 0; i < (2 * KS - kAhead + 1) / 2; ++i) {
          __builtin_amdgcn_sched_group_barrier(kMfma, 2, 0);
          __builtin_amdgcn_sched_group_barrier(kDsRead, 2, 0);
        }
      }
      float sum = weights(sc, c_in, m_use);
      if (__ballot(!(sum <= 1048576.f))) {
        rescale(fmaxf(m_run, row_max(sc) * c_in));
        sum = weights(sc, c_in, m_run == -INFINITY ? 0.f : m_run);
      }
      l_run += sum;
      pv(vbuf(par()));
    }
    clear_dead(vbuf(par() ^ 1), v + 1);
    __syncthreads();
    ++v;
  };
  while (v < vl) {
    step(sa, sb, [] { return 0; });
    if (v >= vl) break;
    step(sb, sa, [] { return 1; });
  }
  for (; v < v1; ++v) {  // (the others' tiles: brings its pages)
    prefetch((v - v0) & 1, v);
    clear_dead(vbuf((v - v0 + 1) & 1), v + 1);
    __syncthreads();
  }

  // A value that is not finite, in a tile that only some rows see, has reached rows
  // that do not see it (0 * inf): then the item is computed again, row by row there.
  uint32_t* flags = reinterpret_cast<uint32_t*>(sK1 + kStage - 8);  // (behind the output staging)
  const bool wave_bad = active && any_not_finite<ET>(oacc);
  if (l == 0) flags[w] = wave_bad;
  __syncthreads();
  if (flags[0] | flags[1] | flags[2] | flags[3]) {
    m_run = -INFINITY;
    l_run = 0.f;
#pragma unroll
    for (int et = 0; et < ET; ++et)
#pragma unroll
      for (int i = 0; i < 16; ++i) oacc[et][i] = 0.f;
#pragma unroll 1
    for (int v = v0; v < v1; ++v) {
      const int page = __builtin_amdgcn_readfirstlane(page_of(v));
      stage(a.k_pool, sK0, page, lane_k(), kStepK);
      stage(a.v_pool, sV0, page, lane_v(), kStepV);
      __syncthreads();
      if (active) {
        uint32_t sees[2];
        qk(sK0, sa, qhi_lds);
        hide(sa, KEYS * ma_tile(kt, v), sees);
        rescale(fmaxf(m_run, row_max(sa) * c_in));
        l_run += weights(sa, c_in, m_run == -INFINITY ? 0.f : m_run);
#pragma unroll 1
        for (int r = 0; r < 32; ++r)  // row r alone, V cleared where it sees nothing
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {
            const int lane = (l & 32) + r;
            const uint32_t see = (uint32_t)__shfl((int)sees[kk >> 1], lane, 64) >> (16 * (kk & 1));
#pragma unroll
            for (int et = 0; et < ET; ++et) {
              const f32x16 o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                  v_operand(keep_of(vread(sV0, kk, et), see)), p[kk], oacc[et], 0, 0, 0);
              if ((l & 31) == r) oacc[et] = o;
            }
          }
      }
      __syncthreads();
    }
  }

  // The tile buffers become the waves' output staging.
  if (active) {
  const float L = l_run + __shfl_xor(l_run, 32, 64);
  const float vsc = KV8 ? a.v_scale[c] : 1.f;
  const bool mine = xw + (l & 31) < rows;
  if (!whole) {
    const int64_t at = (int64_t)it.slot * ROWS + 32 * w + (l & 31);
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
  } else {
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
  if (a.lse && hi == 0 && mine) a.lse[q_row(l)] = (m_run + __log2f(L)) * kLn2;
  }
  }
  __syncthreads();  // (the next item's tiles)
  });
}

}  // namespace dopd
