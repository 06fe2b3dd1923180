// Windowed and tree attention for requests of more than 64 packed rows (chunks,
// larger trees), bf16 in / fp32 accumulate, over bf16 or E4M3 pages.
//
// Workgroup = 4 waves = an item of 128 packed rows of one (request, KV head), 32 rows
// a wave, or a slice of the call's items; two workgroups share a CU.  Packing the g query
// heads of a KV head into the rows lets 128 / g tokens share a tile, so that a window's
// ragged ends take few masked tiles and a small tree fills the matrix units.  Per
// visited tile of 32 keys and wave
//   S^T[32 keys][32] = K[32][d] . Q^T[d][32]        d / 16 v_mfma_f32_32x32x16_bf16
//   O^T[d][32]      += V^T[d][32] . P^T[32][32]     (d / 32) x 2 of them
// so that a row lives in one lane pair and the S^T accumulator is the P^T operand.
// K and V go straight into LDS, each through a ring of five tiles of which four are in
// flight: the time such a load takes under traffic is several times a tile's work.
// (Double-buffered 64-key tiles: 16 chunks of 512 x 32 heads, window 1024, 243 us;
// without their loads 168, without the work 158.)
// Bound by the matrix units and the softmax for wide items (two chunks of 1021 over
// E4M3, window 4001: 285 us, 940 TFLOP/s; those 16 chunks: 203 us, 602 TFLOP/s of
// visible keys, their loads alone 134, their work alone 157), by HBM for few rows.
#pragma once
#include "masked_few.hpp"

namespace dopd {

constexpr int kRowsThreads = 256;
template <int N>
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
// For all waves' writes and reads of LDS; nothing else is exchanged.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// bf16 elements of one K or V tile buffer.
template <int D, bool KV8>
constexpr int rows_tile_elems() { return ma_kind(kMaMany).keys * D / (KV8 ? 2 : 1); }

template <int D, bool KV8, bool TREE>
__global__ __launch_bounds__(kRowsThreads, 2) void masked_rows_kernel(MaskedArgs a) {
  constexpr int ROWS = ma_kind(kMaMany).rows, KEYS = ma_kind(kMaMany).keys;
  constexpr int KS = D / 16;    // k-steps of the QK MFMA
  constexpr int ET = D / 32;    // O^T tiles of 32 dims
  constexpr int TE = rows_tile_elems<D, KV8>();
  // Stage i: what step i, i + 5, .. reads, K of the tile behind and V of the one before.
  // (Arrays of their own, so that the compiler sees that a read does not wait for the
  // loads of other stages.)
  __shared__ __attribute__((aligned(16))) uint16_t st0[2 * TE], st1[2 * TE], st2[2 * TE], st3[2 * TE], st4[2 * TE];
  static_assert(2 * TE >= 32 * D);  // (a stage takes a wave's output)

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
  // 0 (inf becomes NaN there, as it would) or NaN (so that what a row does not see stays
  // -inf).
  const float scale = KV8 ? a.scale * a.k_scale[c] : a.scale;
  const float c_in = scale > 0.f || scale < 0.f ? __builtin_fabsf(scale) : 1.f;
  auto signed_q = [&](u32x4 q) {
    if (!(scale > 0.f)) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (scale < 0.f) {
          q[i] ^= 0x80008000u;
        } else if (scale == 0.f) {
          const uint32_t lo = q[i] & 0x7f80, top = q[i] & 0x7f800000;
          q[i] = (lo == 0x7f80 ? 0x7fc0u : 0u) | (top == 0x7f800000 ? 0x7fc00000u : 0u);
        } else {
          q[i] = 0x7fc07fc0u;
        }
    }
    return q;
  };

  // Q^T operand: Q[row][16 ks + 8 hi + 0..7] (E4M3: the dims a 16-byte read of a K
  // row gives a lane over two k-steps).
  bf16x8 qreg[KS];
  {
    const uint16_t* qp = static_cast<const uint16_t*>(a.q) + q_row(l) * D + (KV8 ? 16 : 8) * hi;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const u32x4 q = signed_q(*reinterpret_cast<const u32x4*>(qp + (KV8 ? 32 * (ks / 2) + 8 * (ks % 2) : 16 * ks)));
      qreg[ks] = __builtin_bit_cast(bf16x8, q);
    }
  }
  f32x16 oacc[ET];
#pragma unroll
  for (int et = 0; et < ET; ++et)
#pragma unroll
    for (int i = 0; i < 16; ++i) oacc[et][i] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;

  // ---- tiles, loaded in pieces of 1 KiB: of a tile's two pages wave w brings half of
  // page w / 2 of K and V (E4M3 at d = 64: waves 0, 1 the K, waves 2, 3 the V of page
  // w % 2).  LDS layouts:
  //   K, bf16: [D / 32 chunk groups][32 rows][4 slots of 16 bytes], E4M3: [32 rows][D],
  //     chunks of a row swizzled so that 16 lanes' reads fall into different banks;
  //   V, bf16: [D / 32 dim groups][4 key chunks][32 dims][8 keys], E4M3: [2 pages][D][16].
  // MFMA row m of S^T is key 16 (m / 4 % 2) + 4 (m / 8) + m % 4 of the tile, so that a
  // lane's 16 accumulators are the 16 keys of page hi: a whole V row of it.
  constexpr bool kByPool = KV8 && D == 64;
  constexpr int kPageBytes = kPage * D * (KV8 ? 1 : 2);
  constexpr int NL = kByPool ? 1 : kPageBytes / 2048;  // loads of K (and of V) of a wave and tile
  constexpr int kPerStep = kByPool ? 1 : 2 * NL;
  const int wp = kByPool ? w & 1 : w >> 1;             // its page of a tile
  typedef const __attribute__((address_space(4))) int32_t* ScalarPtr;  // (scalar loads: the wait
  const ScalarPtr pt = (ScalarPtr)(uintptr_t)(a.page_table + (int64_t)it.req * a.pt_stride);  // for one is not for tiles)
  auto page_of = [&](int v) {
    return pt[__builtin_amdgcn_readfirstlane(seen_page(a, 2 * ma_tile(kt, min(v, v1 - 1)) + wp, low_key, end))];
  };
  auto swizzle = [&](int r, int page) {  // of row r of a page
    return KV8 && D == 128 ? ((r >> 1) & 3) | page << 2 : ((r >> 2) & 1) | page << 1;
  };
  auto place = [&](int u) { return kByPool ? wp : (KV8 ? wp * (2 * NL) + NL * (w & 1) + u : 2 * (NL * (w & 1) + u) + wp); };
  auto stage = [&](const void* pool, uint16_t* lds, int page, int lane_off, int step, bool any) {
    const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(
        (void*)(static_cast<const char*>(pool) + ((int64_t)page * hkv + c) * kPageBytes), (short)0,
        any ? kPageBytes : 0, 0x00020000);
#pragma unroll
    for (int u = 0; u < NL; ++u)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)(lds + 512 * place(u)), 16,
                                               lane_off, step * (kByPool ? 0 : NL * (w & 1) + u), 0, 0);
  };
  const int lane_k = [&] {
    constexpr int NCH = KV8 ? D / 16 : 4;  // 16-byte chunks of a row in a piece
    const int r = l / NCH;
    return r * (KV8 ? D : 2 * D) + 16 * ((l % NCH) ^ swizzle(r, wp));
  }();
  const int lane_v = KV8 ? 16 * l : (l & 31) * (2 * kPage) + 16 * (l >> 5);
  // K (if any_k) from page pk and V (if any_v) from page pv into a stage.  A load of what
  // there is none of is out of its buffer's range, moves nothing and counts like the
  // others: which loads are in flight is then known wherever a stage is read.
  auto load = [&](uint16_t* st, int pk, bool any_k, int pv, bool any_v) {
    if constexpr (kByPool) {
      const bool k = w < 2;
      stage(k ? a.k_pool : a.v_pool, k ? st : st + TE, k ? pk : pv, k ? lane_k : lane_v, 0, k ? any_k : any_v);
    } else {
      stage(a.k_pool, st, pk, lane_k, KV8 ? 1024 : 64, any_k);
      stage(a.v_pool, st + TE, pv, lane_v, 1024, any_v);
    }
  };

  // A operands of the QK MFMA, K[key of row l % 32][16 ks + 8 hi + 0..7], k-step by
  // k-step (E4M3: two to a read) ..
  const int kr = 4 * ((l >> 3) & 3) + (l & 3), kr_page = (l >> 2) & 1, kr_sw = swizzle(kr, kr_page);
  auto read_k = [&](const uint16_t* st, int i) {
    if constexpr (KV8)
      return *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint8_t*>(st) + (16 * kr_page + kr) * D +
                                             16 * ((2 * i + hi) ^ kr_sw));
    else
      return *reinterpret_cast<const u32x4*>(st + (i >> 1) * (KEYS * 32) + (16 * kr_page + kr) * 32 +
                                             ((8 * (hi ^ kr_sw)) ^ (16 * (i & 1))));
  };
  // .. and of the P.V MFMA, V^T[32 et + l % 32][keys 16 hi + 8 kk + 0..7]: et = i % ET,
  // kk = i / ET (E4M3: et = i, both kk).
  auto read_v = [&](const uint16_t* st, int i) {
    if constexpr (KV8)
      return *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint8_t*>(st + TE) + (hi * D + 32 * i + (l & 31)) * kPage);
    else
      return *reinterpret_cast<const u32x4*>(st + TE + (((i % ET) * 4 + 2 * hi + i / ET) * 32 + (l & 31)) * 8);
  };
  constexpr int PER = KV8 ? 2 : 1;  // operands of a read
  using Half = std::conditional_t<KV8, u32x2, u32x4>;
  auto half_of = [&](u32x4 x, int h) {
    if constexpr (KV8) return h ? u32x2{x[2], x[3]} : u32x2{x[0], x[1]};
    else return x;
  };

  bf16x8 p[2];  // P^T: B operands of the two P.V k-steps
  float sum[4];
  auto weight = [&](const f32x16& s, int i, float c, float m_use, bf16x8 (&p)[2]) {  // 2^(c s - m_use)
    const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c, -m_use));
    sum[i & 3] = i < 4 ? e : sum[i & 3] + e;
    p[i >> 3][i & 7] = (__bf16)e;
  };
  auto total = [&] { return (sum[0] + sum[1]) + (sum[2] + sum[3]); };  // this lane's half of the row sum
  auto weights = [&](const f32x16& s, float c, float m_use) {
#pragma unroll
    for (int i = 0; i < 16; ++i) weight(s, i, c, m_use, p);
    return total();
  };
  auto row_max = [&](const f32x16& s) {
    float mx = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = __builtin_elementwise_maximum(mx, s[i]);
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
  auto qk = [&](const uint16_t* st, f32x16& s) {  // S^T of a tile
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_operand(half_of(read_k(st, ks / PER), ks % PER)), qreg[ks], s, 0, 0, 0);
  };
  // What this wave (positions pw0 .. pw1) has to do, by wave and not by item, because of
  // the few tiles at a window's two ends a wave finds most either whole or empty: tiles
  // va .. ve - 1 are seen in full by its rows (full tiles of sinks go with the masked),
  // none from vl on.
  const int pw0 = pre + fast_quot(min(xw, rows - 1), a.by_g), pw1 = pre + fast_quot(min(xw + 31, rows - 1), a.by_g);
  int va = v0, ve, vl;
  if constexpr (TREE) {
    ve = min(v1, pre / KEYS);
    vl = active ? v1 : v0 - 1;
  } else {
    const int low = (max(pw1 - a.rule.window + 1, 0) + KEYS - 1) / KEYS;
    va = max(v0, low - kt.low + kt.nsink);
    ve = min(v1, (pw0 + 1) / KEYS - kt.low + kt.nsink);
    vl = active ? min(v1, max(v0, pw1 / KEYS + 1 - kt.low + kt.nsink)) : v0 - 1;
  }

  // Makes the scores of what a row does not see -inf; returns which of its 16 keys of
  // the tile it sees.  The lane is found anew, so that nothing for it is held (and
  // spilled) over other steps.
  auto hide = [&](f32x16& s, int v) {
    int l;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=&v"(l));
    const int tok = token_of(l);
    const uint32_t* mrow = TREE ? a.mask + (int64_t)(it.row0 + tok) * a.words : nullptr;
    const uint32_t sees = v < vl ? row_sees<TREE>(a, KEYS * ma_tile(kt, v), pre, end, pre + tok, mrow) >> (16 * (l >> 5)) : 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = sees >> i & 1 ? s[i] : -INFINITY;
    return sees;
  };
  // V of positions of visited tile v that no row of the item sees (slots that may hold
  // anything: 0 * NaN is NaN) is cleared in LDS by the wave that brought it, once it has
  // landed and before the barrier that publishes it.
  auto clear_dead = [&](uint16_t* sv, int v) {
    if (v < v0 || v >= v1 || (kByPool && w < 2)) return;
    const uint32_t live = any_sees<TREE>(a, KEYS * ma_tile(kt, v) + kPage * wp, p0, end) & 0xffff;  // uniform
    if (live == 0xffff) return;
#pragma unroll
    for (int u = 0; u < NL; ++u) {
      u32x4* at = reinterpret_cast<u32x4*>(sv + 512 * place(u)) + l;
      const u32x4 x = *at;
      if constexpr (KV8) {  // a dim's 16 keys
        const u32x2 lo = keep_of(u32x2{x[0], x[1]}, live), top = keep_of(u32x2{x[2], x[3]}, live >> 8);
        *at = u32x4{lo[0], lo[1], top[0], top[1]};
      } else {
        *at = keep_of(x, live >> (8 * hi));
      }
    }
  };
  // Step i (of tile v0 + i) loads K of tile i + 5 and V of tile i + 3 into the stage that
  // step i - 1 read, and does three things that do not wait for each other: S^T of tile
  // i + 1, the weights of tile i, and the product of the weights of tile i - 1 with V.
  // It ends when what step i + 1 reads has landed: this wave's loads of the three steps
  // before may be in flight then.
  int id[6];  // (all at once: one after the other, an item began with five trips to memory)
#pragma unroll
  for (int i = 0; i < 6; ++i) id[i] = page_of(v0 + i);
  int pid_k = id[5], pid_k1 = id[4], pid_v = id[3];
  auto issue = [&](int v, uint16_t* st) {
    const int next = page_of(v + 6);
    load(st, pid_k, v + 5 < v1, pid_v, v + 3 < v1);
    pid_v = pid_k1;
    pid_k1 = pid_k;
    pid_k = next;
  };
  auto finish = [&](int v, uint16_t* next) {
    wait_loads<3 * kPerStep>();
    clear_dead(next + TE, v);
    lds_barrier();
  };
  for (int i = (int)threadIdx.x; i < TE / 8; i += kRowsThreads)  // (step 0: weights 0 and no V)
    reinterpret_cast<u32x4*>(st0 + TE)[i] = u32x4{0, 0, 0, 0};
  load(st4, id[0], true, id[0], false);
  load(st0, id[1], v0 + 1 < v1, id[0], false);
  load(st1, id[2], v0 + 2 < v1, id[0], true);
  load(st2, id[3], v0 + 3 < v1, id[1], v0 + 1 < v1);
  load(st3, id[4], v0 + 4 < v1, id[2], v0 + 2 < v1);
  finish(v0 - 1, st0);
  f32x16 sa, sb;  // S^T of two consecutive tiles
  qk(st4, sa);
  lds_barrier();  // (step 0 loads into st4)

  // Weights are formed against the running maximum, and only a sum beyond 2^20 (a tile
  // far above it, the first one seen: NaN) takes the tile's own.
  int v = v0;
  p[0] = p[1] = bf16x8{};
  auto step = [&](f32x16& sc, f32x16& sn, uint16_t* before, const uint16_t* now, uint16_t* next) {
    issue(v, before);
    if (v < va || v >= ve) hide(sc, v);
    // The matrix products of S^T and O^T in turn, so that none waits for the one before,
    // and between two of them what the compiler would otherwise put in front or behind:
    // the conversion of the next operand, a read of one further on, weights.
    constexpr int NM = KS + 2 * ET, NR = NM / PER, AHEAD = KV8 ? NR : 6;
    u32x4 raw[NR];
    auto read = [&](int i) { raw[i] = i % 2 == 0 ? read_k(now, i / 2) : read_v(now, i / 2); };
    auto operand = [&](int i) {  // of product i
      return v_operand(half_of(raw[2 * (i / (2 * PER)) + i % 2], (i / 2) % PER));
    };
    bf16x8 p_now[2];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) read(i);
#pragma unroll
    for (int i = 0; i < 16; ++i) sn[i] = 0.f;
    bf16x8 op = operand(0);
#pragma unroll
    for (int i = 0; i < NM; ++i) {
      const int j = i / 2, et = KV8 ? j / 2 : j % ET, kk = KV8 ? j % 2 : j / ET;
      if (i + AHEAD < NR) read(i + AHEAD);
      if (i % 2 == 0) sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op, qreg[j], sn, 0, 0, 0);
      else oacc[et] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op, p[kk], oacc[et], 0, 0, 0);
      if (i + 1 < NM) op = operand(i + 1);
#pragma unroll
      for (int e = 16 * i / NM; e < 16 * (i + 1) / NM; ++e) weight(sc, e, c_in, m_run, p_now);
      __builtin_amdgcn_sched_barrier(0);
    }
    float sum = total();
    p[0] = p_now[0];
    p[1] = p_now[1];
    if (__ballot(!(sum <= 1048576.f))) {
      rescale(fmaxf(m_run, row_max(sc) * c_in));
      sum = weights(sc, c_in, m_run == -INFINITY ? 0.f : m_run);  // (nothing seen so far: weights 0)
    }
    l_run += sum;
    finish(v, next);
    ++v;
  };
  while (v <= vl) {
    step(sa, sb, st4, st0, st1);
    if (v > vl) break;
    step(sb, sa, st0, st1, st2);
    if (v > vl) break;
    step(sa, sb, st1, st2, st3);
    if (v > vl) break;
    step(sb, sa, st2, st3, st4);
    if (v > vl) break;
    step(sa, sb, st3, st4, st0);
    sa = sb;
  }
  int i = (v - v0) % 5;
  for (; v <= v1; ++v) {  // (the others' tiles: brings its part)
    issue(v, i == 0 ? st4 : i == 1 ? st0 : i == 2 ? st1 : i == 3 ? st2 : st3);
    finish(v, i == 0 ? st1 : i == 1 ? st2 : i == 2 ? st3 : i == 3 ? st4 : st0);
    i = i == 4 ? 0 : i + 1;
  }
  wait_loads<0>();  // (the last steps' loads of nothing)
  lds_barrier();

  // A value that is not finite, in a tile that only some rows see, has reached rows
  // that do not see it (0 * inf): then the item is computed again, row by row there.
  uint32_t* flags = reinterpret_cast<uint32_t*>(st4);
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
      const int page = page_of(v);
      load(st0, page, true, page, true);
      wait_loads<0>();
      __syncthreads();
      if (active) {
        qk(st0, sa);
        const uint32_t sees = hide(sa, v);
        rescale(fmaxf(m_run, row_max(sa) * c_in));
        l_run += weights(sa, c_in, m_run == -INFINITY ? 0.f : m_run);
#pragma unroll 1
        for (int r = 0; r < 32; ++r)  // row r alone, V cleared where it sees nothing
#pragma unroll
          for (int kk = 0; kk < 2; ++kk) {
            const uint32_t see = (uint32_t)__shfl((int)sees, (l & 32) + r, 64) >> (8 * kk);
#pragma unroll
            for (int et = 0; et < ET; ++et) {
              const Half x = half_of(read_v(st0, KV8 ? et : kk * ET + et), kk);
              const f32x16 o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_operand(keep_of(x, see)), p[kk], oacc[et], 0, 0, 0);
              if ((l & 31) == r) oacc[et] = o;
            }
          }
      }
      __syncthreads();
    }
  }

  // Stages become the waves' output staging, 16-byte chunks swizzled by row.
  if (active) {
  float L = l_run + __shfl_xor(l_run, 32, 64);
  const float vsc = KV8 ? a.v_scale[c] : 1.f;
  const bool mine = xw + (l & 31) < rows;
  if (!whole) {
    const float fac = vsc * part_to_unit_sum(m_run, L);
    const int64_t at = (int64_t)it.slot * ROWS + 32 * w + (l & 31);
    if (mine) {
      float* po = a.part_o + at * D + 4 * hi;
#pragma unroll
      for (int et = 0; et < ET; ++et)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<f32x4*>(po + 32 * et + 8 * q) =
              f32x4{oacc[et][4 * q], oacc[et][4 * q + 1], oacc[et][4 * q + 2], oacc[et][4 * q + 3]} * fac;
      if (hi == 0) *reinterpret_cast<float2*>(a.part_ml + at * 2) = float2{m_run, L};
    }
  } else {
  const float inv = L == 0.f ? 0.f : vsc / L;
  // Through LDS, so that 16 lanes store one 256-byte row.
  uint16_t* so = w == 0 ? st0 : w == 1 ? st1 : w == 2 ? st2 : st3;
  constexpr int CH = D / 8;
#pragma unroll
  for (int et = 0; et < ET; ++et)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      u32x2 o2;
      o2[0] = pack_bf16x2(oacc[et][4 * q] * inv, oacc[et][4 * q + 1] * inv);
      o2[1] = pack_bf16x2(oacc[et][4 * q + 2] * inv, oacc[et][4 * q + 3] * inv);
      *reinterpret_cast<u32x2*>(so + (l & 31) * D + 8 * ((4 * et + q) ^ (l & (CH - 1))) + 4 * hi) = o2;
    }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
  for (int u = 0; u < 32 * CH / 64; ++u) {
    const int i = l + 64 * u, rr = i / CH, ch = i % CH;
    const u32x4 o4 = *reinterpret_cast<const u32x4*>(so + rr * D + 8 * (ch ^ (rr & (CH - 1))));
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
