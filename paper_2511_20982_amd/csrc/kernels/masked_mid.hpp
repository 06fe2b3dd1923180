// Windowed and tree attention for requests of 17 to 64 packed rows (ordinary trees,
// short chunks), bf16 in / fp32 accumulate, over bf16 pages, or E4M3 at d = 64.
//
// Workgroup = 4 waves = one (request, KV head), or a slice of the call's items; wave w
// holds rows 16 w .. 16 w + 15 and goes through all visited pairs of pages (32 keys),
//   S^T[32 keys][16] = K[32][d] . Q^T[d][16]     2 x (d / 32) v_mfma_f32_16x16x32_bf16
//   O^T[d][16]      += V^T[d][32] . P^T[32][16]  (d / 16) of them
// with operands from LDS, where the pages go straight from memory.
//
// HBM-bound: up to 64 rows share each byte read, which is 64 flop a byte against a
// ridge of about 300.  What counts is bytes in flight: a ring of four 16 KiB stages a
// workgroup, two workgroups a CU, three stages of each on their way while one is
// computed (64-key tiles in two buffers, one on its way, ran 64 rows at 3.7 TB/s; this,
// 8 drafts x 64 requests of some 2000 keys, at 4.6, and with the merge at 4.2).
// Waits count the loads still allowed in flight, so that a step waits for its own
// stage alone.
#pragma once
#include "masked_few.hpp"

namespace dopd {

constexpr int kMidStages = 4, kMidStageBytes = 16384;

// Waits until at most N of this wave's loads are in flight, then for the workgroup's
// other waves.  (No fence: nothing but the loads into LDS is exchanged here.)
template <int N>
__device__ __forceinline__ void wait_loads_and_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

template <int D, bool KV8, bool TREE>
__global__ __launch_bounds__(256, 2) void masked_mid_kernel(MaskedArgs a) {
  constexpr int ROWS = ma_kind(kMaMid).rows, KEYS = ma_kind(kMaMid).keys;
  constexpr int NQK = D / 32, NT = D / 16;
  constexpr int PB = kPage * D * (KV8 ? 1 : 2);        // bytes of a page's K (or V) of one head
  constexpr int NI = PB / 1024;                        // loads of one
  constexpr int PG = kMidStageBytes / (2 * PB);        // pages of a stage
  constexpr int PPS = PG / 2;                          // pairs of a stage
  constexpr int kPerWave = kMidStageBytes / 1024 / 4;  // loads of a stage by one wave
  // A stage: for each of its pages, K then V.  K: [64-byte groups of a row][16 rows][4
  // chunks of 16 bytes], rows in the order pi (bits 2 and 3 of the slot swapped), chunk
  // ch of row r of page pg in slot ch ^ ((r / 4) % 2 + 2 (pg % 2)), so that 16 lanes
  // reading 16 rows hit 16 bank groups.  V bf16: [dims][2 halves of 8 keys], the halves
  // swapped in every second eight dims; E4M3: [dims][16 keys].
  __shared__ __attribute__((aligned(16))) uint8_t st0[kMidStageBytes], st1[kMidStageBytes], st2[kMidStageBytes],
      st3[kMidStageBytes];
  __shared__ uint32_t s_bad[4];

  ma_items<kMaMid>(a, grid_block(blockIdx.x, blockIdx.y), [&](const MaItem& it) {
  const int l = lane_id(), w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int g = (int)a.by_g.d, c = it.c, hkv = a.hkv;
  const int rows = it.n * g;
  const int pre = it.pre, end = pre + it.n, p1 = end - 1;
  const KeyTiles kt = ma_key_tiles(a.rule, pre, p1, KEYS);
  int v0, v1;
  const bool whole = ma_tiles_of(a, it, kt.n, v0, v1);
  if (v0 >= v1) return;
  const int low_key = ma_low_key(a.rule, pre);
  const int nst = (v1 - v0 + PPS - 1) / PPS;  // stages

  const int col = l & 15, qg = l >> 4;
  const bool active = 16 * w < rows;                   // uniform
  const int x = min(16 * w + col, rows - 1), tok = fast_quot(x, a.by_g);  // (past the end: the last row, not stored)
  const int64_t qrow = (int64_t)(it.row0 + tok) * a.hq + c * g + (x - tok * g);
  constexpr int KEL = KV8 ? 16 : 8, KST = 4 * KEL;     // elements of a chunk, of a group
  bf16x8 qop[NQK];
  {
    const uint16_t* qp = static_cast<const uint16_t*>(a.q) + qrow * D + KEL * qg;
#pragma unroll
    for (int i = 0; i < NQK; ++i)
      qop[i] = __builtin_bit_cast(
          bf16x8, *reinterpret_cast<const u32x4*>(qp + (KV8 ? KST * (i / 2) + 8 * (i % 2) : KST * i)));
  }
#pragma unroll
  for (int i = 0; i < NQK; ++i) asm volatile("" : "+v"(qop[i]));  // (here now, so that no step waits for it)
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

  // ---- loads.  A wave brings the K or V of one page, or both of PG / 4 pages.  Page
  // ids come by scalar loads, a stage ahead: a vector load among the others would make
  // the wait for it a wait for the stages before it.
  constexpr int NP = PG == 2 ? 1 : PG / 4;  // pages of a stage that this wave brings
  typedef const __attribute__((address_space(4))) int32_t* ScalarPtr;
  const ScalarPtr pt = (ScalarPtr)(uintptr_t)(a.page_table + (int64_t)it.req * a.pt_stride);
  int ids[NP];  // of the next stage to bring
  auto read_ids = [&](int s) {
#pragma unroll
    for (int u = 0; u < NP; ++u) {
      const int q = s * PG + (PG == 2 ? (w & 1) : NP * w + u);  // visited page, from v0's
      ids[u] = pt[__builtin_amdgcn_readfirstlane(
          seen_page(a, 2 * ma_tile(kt, min(v0 + (q >> 1), v1 - 1)) + (q & 1), low_key, end))];
    }
  };
  // This lane's place in a K (V) load: row l / 4, slot l % 4 of a group; two halves of
  // 32 dims (E4M3: 64 dims).
  const int r4 = l >> 2, pi_r = (r4 & 3) | ((r4 & 4) << 1) | ((r4 & 8) >> 1);
  constexpr int kRowBytes = D * (KV8 ? 1 : 2);
  const int lane_k0 = pi_r * kRowBytes + 16 * ((l & 3) ^ ((r4 >> 2) & 1));
  const int lane_k1 = pi_r * kRowBytes + 16 * ((l & 3) ^ (((r4 >> 2) & 1) | 2));
  const int lane_v = KV8 ? 16 * l : (l >> 1) * 32 + 16 * ((l & 1) ^ ((l >> 4) & 1));
  auto copy = [&](const void* pool, uint8_t* to, int page, int lane_off, int step) {
    const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(
        (void*)(static_cast<const char*>(pool) + ((int64_t)page * hkv + c) * PB), (short)0, PB, 0x00020000);
#pragma unroll
    for (int u = 0; u < NI; ++u)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)(to + 1024 * u), 16, lane_off,
                                               step * u, 0, 0);
  };
  // Stage s into `st` (its ids are there), and the ids of the next.
  auto issue = [&](int s, uint8_t* st) {
    if constexpr (PG == 2) {
      if (w < 2) copy(a.k_pool, st + 2 * PB * w, ids[0], w & 1 ? lane_k1 : lane_k0, 64);
      else copy(a.v_pool, st + 2 * PB * (w - 2) + PB, ids[0], lane_v, 1024);
    } else {
#pragma unroll
      for (int u = 0; u < NP; ++u) {
        const int q = NP * w + u;
        copy(a.k_pool, st + 2 * PB * q, ids[u], q & 1 ? lane_k1 : lane_k0, 64);
        copy(a.v_pool, st + 2 * PB * q + PB, ids[u], lane_v, 1024);
      }
    }
    read_ids(s + 1);
  };

  // ---- a pair of pages at `st`, keys base ..
  const int kr = 64 * (col & 7);  // (MFMA #1: row col % 8 of page col / 8; #2: 8 rows on)
  const int ksl0 = 16 * (qg ^ ((col >> 2) & 1)), ksl1 = 16 * (qg ^ (((col >> 2) & 1) | 2));
  auto compute = [&](const uint8_t* st, int pair, int v, auto careful) {
    const int base = KEYS * ma_tile(kt, v);
    const uint8_t* pages = st + 4 * PB * pair;
    const uint8_t* krow = pages + (col >> 3 ? 2 * PB + ksl1 : ksl0) + kr;
    f32x4 s1 = {0.f, 0.f, 0.f, 0.f}, s2 = {0.f, 0.f, 0.f, 0.f};
    u32x4 k1[NI], k2[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      k1[i] = *reinterpret_cast<const u32x4*>(krow + 1024 * i);
      k2[i] = *reinterpret_cast<const u32x4*>(krow + 1024 * i + 512);
    }
#pragma unroll
    for (int i = 0; i < NQK; ++i) {
      s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(few_k_operand<KV8>(k1, i), qop[i], s1, 0, 0, 0);
      s2 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(few_k_operand<KV8>(k2, i), qop[i], s2, 0, 0, 0);
    }
    float s[8];  // keys base + 8 qg + 0 .. 7 of this lane's row
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      s[j] = s1[j] * sl2;
      s[4 + j] = s2[j] * sl2;
    }
    uint32_t sees = 0, live = ~0u;
    const bool part = careful() || !all_see<TREE>(a, base, KEYS, pre, pre, p1);  // uniform
    if (part) {
      const uint32_t* mrow = TREE ? a.mask + (int64_t)(it.row0 + tok) * a.words : nullptr;
      sees = row_sees<TREE>(a, base, pre, end, pre + tok, mrow) >> (8 * qg);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (!(sees >> j & 1)) s[j] = -INFINITY;
      live = any_sees<TREE>(a, base, pre, end);  // uniform
    }
    // Weights are formed against the running maximum; only a sum beyond 2^20 (keys far
    // above it, the first ones seen: inf or NaN) takes the maximum of these.  The careful
    // pass always does: weights of 2^20 times large V may have been what was not finite.
    bf16x8 p;
    float sum;
    auto weights = [&](float m) {
      float part[2] = {0.f, 0.f};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float e = __builtin_amdgcn_exp2f(s[j] - m);
        part[j & 1] += e;
        p[j] = (__bf16)e;
      }
      sum = part[0] + part[1];
    };
    weights(m_run);
    if (careful() || __ballot(!(sum <= 1048576.f))) {
      const float mx = quad_max(fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7]))));
      const float m_new = fmaxf(m_run, mx);
      const float m_use = m_new == -INFINITY ? 0.f : m_new;  // (no key seen so far: weights 0)
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_use);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int n = 0; n < NT; ++n) oacc[n] *= alpha;
      weights(m_use);
    }
    l_run += sum;
    // V^T operand n: dims 16 n + col, keys 8 qg + 0 .. 7 (page qg / 2, half qg % 2).
    using VT = std::conditional_t<KV8, u32x2, u32x4>;
    const uint8_t* vrow = pages + (qg >> 1) * 2 * PB + PB + (KV8 ? 16 * col : 32 * col + 16 * ((qg & 1) ^ (col >> 3)));
    VT vv[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(vrow + (KV8 ? 256 : 512) * n);
      // (E4M3: a dim's 16 keys, of which the half is taken.  Two 8-byte reads would be
      // paired, and for a paired read the compiler loses which buffer it reads and waits
      // for every load in flight.)
      if constexpr (KV8) vv[n] = qg & 1 ? u32x2{v[2], v[3]} : u32x2{v[0], v[1]};
      else vv[n] = v;
    }
    if (live != ~0u) {  // V that no row sees (slots that may hold anything)
#pragma unroll
      for (int n = 0; n < NT; ++n) vv[n] = keep_of(vv[n], live >> (8 * qg));
    }
    if constexpr (!careful()) {
#pragma unroll
      for (int n = 0; n < NT; ++n) oacc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v_operand(vv[n]), p, oacc[n], 0, 0, 0);
    } else {
#pragma unroll 1
      for (int r = 0; r < 16; ++r) {
        const uint32_t see = (uint32_t)__shfl((int)sees, (l & 48) + r, 64);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const f32x4 o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v_operand(keep_of(vv[n], see)), p, oacc[n], 0, 0, 0);
          if (col == r) oacc[n] = o;
        }
      }
    }
  };

  // ---- the ring: stage s in buffer s % 4.  A step waits for its stage (this wave's
  // loads of the two behind it may be in flight), and its barrier, which every wave
  // passes once it has read the stage before, frees that one's buffer for stage s + 3.
  auto pass = [&](auto careful) {
    read_ids(0);
    issue(0, st0);
    if (nst > 1) issue(1, st1);
    if (nst > 2) issue(2, st2);
    auto step = [&](int s, const uint8_t* now, uint8_t* free_) {
      if (s + 2 < nst) wait_loads_and_barrier<2 * kPerWave>();
      else if (s + 1 < nst) wait_loads_and_barrier<kPerWave>();
      else wait_loads_and_barrier<0>();
      if (s + 3 < nst) issue(s + 3, free_);
      if (active) {
#pragma unroll
        for (int i = 0; i < PPS; ++i)
          if (i == 0 || v0 + s * PPS + i < v1) compute(now, i, v0 + s * PPS + i, careful);
      }
    };
    for (int s = 0; s < nst; s += 4) {
      step(s, st0, st3);
      if (s + 1 < nst) step(s + 1, st1, st0);
      if (s + 2 < nst) step(s + 2, st2, st1);
      if (s + 3 < nst) step(s + 3, st3, st2);
    }
    __syncthreads();  // (what comes next reuses the buffers)
  };
  pass(std::false_type{});
  // A value that is not finite, in a pair that only some rows see, has reached rows
  // that do not see it (0 * inf is NaN): then the part is computed again.
  const bool bad = active && any_not_finite<NT>(oacc);
  if (l == 0) s_bad[w] = bad;
  __syncthreads();
  const bool again = (s_bad[0] | s_bad[1] | s_bad[2] | s_bad[3]) != 0;
  __syncthreads();  // (the next item's flags)
  if (again) {
    clear();
    pass(std::true_type{});
  }
  if (!active) return;

  l_run = quad_sum(l_run);
  const float vsc = KV8 ? a.v_scale[c] : 1.f;
  const float fac = !whole ? vsc * part_to_unit_sum(m_run, l_run) : l_run == 0.f ? 0.f : vsc / l_run;
  const int row = 16 * w + col;
  if (row >= rows) return;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    if (whole) store_bf16x4(a.out, qrow * D + 16 * n + 4 * qg, oacc[n] * fac);
    else *reinterpret_cast<f32x4*>(a.part_o + ((int64_t)it.slot * ROWS + row) * D + 16 * n + 4 * qg) = oacc[n] * fac;
  }
  if (qg == 0) {
    if (!whole) *reinterpret_cast<float2*>(a.part_ml + ((int64_t)it.slot * ROWS + row) * 2) = float2{m_run, l_run};
    else if (a.lse) a.lse[qrow] = (m_run + __log2f(l_run)) * kLn2;
  }
  });
}

}  // namespace dopd
