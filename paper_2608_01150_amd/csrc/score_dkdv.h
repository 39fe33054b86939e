// Scored attention: dK and dV, bf16 inputs, gfx950 MFMA.
//
// The plan is that of the plain dK/dV (bwd_bf16.hip): an item is up to 128 keys of one
// K/V head, run by one workgroup per CU; four producer waves hold 32 keys each and four
// consumer waves the dV or dK accumulators of half of d for all 128.  Queries come in
// 64-row tiles, of every head that shares the K/V head one after another, as one sequence
// of 32-row sub-blocks k:
//   A(k)  producer: S = Q K^T, dP - D = dO V^T - D (MFMA, K and V in registers)
//   B(k)  producer: P = exp(A - LSE), dS = P (dP - D) f' (VALU), to LDS as bf16
//   C(k)  consumers: dV^T += dO^T P, dK^T += Q^T dS (MFMA, transpose reads)
// P and dS are rounded to bf16, the type of what they meet, which also halves the exchange:
// 0.26% of the gradients against 0.17% of rounding them alone, with D from the O in bf16.
// Phase j runs A(j) with B(j-1) on the producers and C(j-2) on the consumers.
//
// Where a segment has few key tiles and its K/V heads serve several query heads, an item
// takes some of those heads (score_splits in zl_host.cpp), and score_sum_kernel adds the
// items' fp32 partials.
//
// Rows from the first to the last tile that see a key of the item are run.  Per
// sub-block a producer knows from the rows' intervals and positions (wave-uniform)
// that no row sees its keys (their weights are zero), that all rows see all of
// them at one side of slope or table (one fma per score and, with a slope, two more
// adds), or that it has to work scores out one by one (`exactly`); it looks in the phase in
// front of the one that needs it, or the look stands in front of every phase's products
// (8192 rows in documents of 1900, 16 heads of 128: 421 -> 321 us, with the rows' intervals
// made ready by score_pre_kernel).
//
// Bound by the producers' chain, about 1.1 us per phase: 8192 unmasked tokens, 16 heads of
// 128, 1030 us, 1070 TFLOP/s of the 8 d flop a pair that it runs.

#pragma once

#include "zl_score_device.h"

namespace zl {
namespace {
namespace dkdv {

constexpr int NT = 512;
constexpr int BQ = 64;              // queries per tile
constexpr int NBUF = 3;

// Position in the sequence of query tiles: head of the group, tile.
struct Cursor {
  int g, t;
};

template <int D>
struct Lds {
  static constexpr int TILE = BQ * Pad<D>::PITCH;
  __attribute__((aligned(16))) char qs[NBUF][TILE], dos[NBUF][TILE];
  __attribute__((aligned(16))) float lss[NBUF][BQ], dss[NBUF][BQ];
  __attribute__((aligned(16))) int los[NBUF][BQ], lens[NBUF][BQ];
  u32x4 xch[2][4][4][64];   // [k%2][key group][word: P h0, P h1, dS h0, dS h1][lane]
  int s_mask[2][4], s_first[8], s_last[8];
};

// Item `item`, by a workgroup of NT threads.  tables: room for those of a group's even and odd heads.
template <int D, bool CAP, int BIAS>
__device__ __forceinline__ void run(const ScoreBwdParams& p, int item, Lds<D>& lds, float* tables) {
  constexpr int PITCH = Pad<D>::PITCH;
  constexpr int NM = D / 8;         // MFMAs per sub-block and role
  auto &qs = lds.qs, &dos = lds.dos;
  auto &lss = lds.lss, &dss = lds.dss;
  auto &los = lds.los, &lens = lds.lens;
  auto& xch = lds.xch;
  auto& s_mask = lds.s_mask;
  auto &s_first = lds.s_first, &s_last = lds.s_last;
  const int bins = 2 * (p.fn.reach + kScoreBinMargin) + 1;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool producer = wave < 4;
  const int kw = wave & 3;
  const int ln = lane & 31, g = lane >> 5;
  const int H = p.num_heads, Hk = H / p.group;
  const int key = kw * 32 + ln;
  const uint32_t a_off = poff<D>(perm32(ln), g * 8), t_off = tr_lane_off<D>(lane);
  const float coef = CAP ? -2.f * p.fn.cap_log2 : p.fn.scale_log2;
  const bool plain_rows = !p.fn.key_lo && !p.fn.key_hi;

  using Dma = TileDma<D, BQ>;
  const uint32_t row_bytes = (uint32_t)H * D * 2u, stat_bytes = (uint32_t)H * 4u;
  Dma dma;
  dma.init(kw, lane, row_bytes);

  // Tiles [t0, t1) hold every row that sees a key of the item.
  auto tiles_of = [&](const ScoreKeyItem& it, int& t0, int& t1) __attribute__((always_inline)) {
    const int k_last = it.k_pos + it.k_len - 1;
    t0 = 0;
    t1 = (it.q_len + BQ - 1) / BQ;
    if (plain_rows) {
      if (p.fn.causal) t0 = min(max(it.k_pos - it.q_pos, 0) / BQ, t1);
    } else {
      int first = INT32_MAX, last = -1;
      for (int t = tid; t < t1; t += NT) {
        const int2 see = p.tile_see[it.tile0 + t];
        if (see.x <= k_last && see.y > it.k_pos) {
          first = min(first, t);
          last = t;
        }
      }
#pragma unroll
      for (int m = 32; m; m >>= 1) {
        first = min(first, __shfl_xor(first, m));
        last = max(last, __shfl_xor(last, m));
      }
      if (lane == 0) {
        s_first[wave] = first;
        s_last[wave] = last;
      }
      __syncthreads();
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        first = min(first, s_first[w]);
        last = max(last, s_last[w]);
      }
      const int f = __builtin_amdgcn_readfirstlane(first), l = __builtin_amdgcn_readfirstlane(last);
      t0 = l < 0 ? 0 : f;
      t1 = l + 1;
    }
  };

  // Tile `c` to buffer b: producers load Q and, one wave each, LSE, -D and what
  // the rows see; consumers load dO.  Rows past the segment read as zero, tiles past the
  // last one are all zero and never used.
  auto fetch = [&](const ScoreKeyItem& it, int nt, int G, Cursor c, int b) __attribute__((always_inline)) {
    c = {__builtin_amdgcn_readfirstlane(c.g), __builtin_amdgcn_readfirstlane(c.t)};
    const int q0 = c.t * BQ, nq = c.g < G && nt > 0 ? it.q_len - q0 : 0;
    const int64_t row0 = (int64_t)(it.q_start + q0) * H + it.kv_head * p.group + it.g0 + c.g;
    if (producer) {
      dma.issue(qs[b], static_cast<const uint16_t*>(p.q) + row0 * D, nq, row_bytes);
      const int nv = min(nq, BQ);
      const char* src = reinterpret_cast<const char*>(kw == 0 ? p.lse2 : p.dsum) + row0 * 4;
      uint32_t pitch = stat_bytes;
      void* to = kw == 0 ? (void*)lss[b] : (void*)dss[b];
      if (kw >= 2) {
        src = reinterpret_cast<const char*>((kw == 2 ? p.row_lo : p.row_len) + it.q_start + q0);
        pitch = 4;
        to = kw == 2 ? (void*)los[b] : (void*)lens[b];
      }
      const i32x4 rsrc = buf_rsrc(src, nv > 0 ? (nv - 1) * pitch + 4u : 0u);
      dma4(rsrc, lane * pitch, __builtin_amdgcn_readfirstlane(lds_addr(to)));
    } else {
      dma.issue(dos[b], static_cast<const uint16_t*>(p.dout) + row0 * D, nq, row_bytes);
    }
  };

  const ScoreKeyItem it = p.kv_items[item];
  const int head0 = it.kv_head * p.group + it.g0, G = it.gn;  // the item's query heads
  int t0, t1;
  tiles_of(it, t0, t1);
  const int nt = t1 - t0, total = nt * G;
  auto next = [&](Cursor c) { return c.t + 1 < t1 ? Cursor{c.g, c.t + 1} : Cursor{c.g + 1, t0}; };

  if (producer) {
    // ---------------------------------------------------------- producer
    Cursor cur{0, t0}, ahead{0, t0};
    fetch(it, nt, G, ahead, 0);
    ahead = next(ahead);
    const bool k_ok = key < it.k_len;
    const int64_t krow = ((int64_t)(it.k_start + key) * Hk + it.kv_head) * D;
    u32x4 kf[D / 16], vf[D / 16];
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      kf[kk] = vf[kk] = u32x4{0, 0, 0, 0};
      if (k_ok) {
        kf[kk] = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p.k) + krow + kk * 16 + g * 8);
        vf[kk] = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p.v) + krow + kk * 16 + g * 8);
      }
    }
    // The loop carries no pending register loads.
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();  // tile 0 published

    const bool live = kw * 32 < it.k_len;
    const int kp = it.k_pos + key;                                   // this lane's key
    const int kp0 = it.k_pos + kw * 32, kp1 = it.k_pos + min(kw * 32 + 32, it.k_len) - 1;   // the wave's
    f32x16 sc[2], dp[2];
    float slope2 = 0.f, far_lo = 0.f, far_hi = 0.f;
    auto of_head = [&](int gh) {
      if constexpr (BIAS == kBiasSlope) slope2 = p.fn.slope[head0 + gh] * 1.4426950408889634f;
      if constexpr (BIAS == kBiasTable) {
        far_lo = bias_at(p.fn, -p.fn.reach, head0 + gh, H) * 1.4426950408889634f;
        far_hi = bias_at(p.fn, p.fn.reach, head0 + gh, H) * 1.4426950408889634f;
      }
      __builtin_amdgcn_s_waitcnt(0);
    };

    // What the rows of half h of tile t in buffer b see of the wave's keys: some row some key,
    // every row every key.  Taken in the phase in front of the one that needs it.
    // A row without a weight (a table of -inf) sees nothing, whatever its interval.
    bool see_any = false, see_all = false;
    struct Row {
      float lse2;
      int lo, len;
    };
    auto row_of = [&](int b, int h) __attribute__((always_inline)) -> Row {
      if (plain_rows) return {lss[b][32 * h + ln], 0, 0};
      return {lss[b][32 * h + ln], los[b][32 * h + ln], lens[b][32 * h + ln]};
    };
    auto look = [&](const Row& r, int h, int t) __attribute__((always_inline)) {
      const int q0 = t * BQ + 32 * h, nrow = min(it.q_len - q0, 32), p0 = it.q_pos + q0;
      const bool none = r.lse2 == kScoreNoKey;  // not behind the segment: zero there
      see_any = nrow > 0;
      see_all = true;
      if (plain_rows) {
        if (p.fn.causal) {
          see_any &= p0 + nrow - 1 >= kp0;
          see_all = p0 >= kp1;
        }
      } else {
        see_any &= __any((ln < nrow) & (r.len > 0) & (r.lo <= kp1) & (r.lo + r.len > kp0)) != 0;
        see_all = __all((ln >= nrow) | ((r.lo <= kp0) & (r.lo + r.len > kp1))) != 0;
      }
      see_all &= !__any(none);
    };

    // A of half ka of tile ta in buffer b, with B (has_b) of half sb of tile `cur` in buffer bb.
    auto phase = [&](int ka, int b, int ta, int sb, int bb, bool has_b, int xb) __attribute__((always_inline)) {
      const int kb = 1 - ka;
      // What B's rows see of the wave's keys.
      const int q0 = cur.t * BQ + 32 * sb, nrow = min(it.q_len - q0, 32), p0 = it.q_pos + q0;
      const bool any = live && see_any, all = see_all;
      bool near = false;
      float cf = coef, sl = 0.f, add = 0.f;
      if (has_b) {
        if constexpr (BIAS == kBiasSlope) {
          const bool behind = kp0 >= p0 + nrow - 1;  // the keys, of all rows
          near = !behind && kp1 > p0;
          sl = behind ? slope2 : -slope2;
          add = sl * (float)(p0 + 8 * g - kp);
        }
        if constexpr (BIAS == kBiasTable) {
          const bool behind = kp0 - (p0 + nrow - 1) >= p.fn.reach;
          near = !behind && kp1 - p0 > -p.fn.reach;
          add = behind ? far_hi : far_lo;
        }
        if (lane == 0) s_mask[xb][kw] = live && !(any && all);
      }
      if (!live) return;
      if (has_b && !any) {
#pragma unroll
        for (int w = 0; w < 4; ++w) xch[xb][kw][w][lane] = u32x4{0, 0, 0, 0};
        has_b = false;
      }
      const char* qa = qs[b] + a_off + 32 * ka * PITCH;
      const char* oa = dos[b] + a_off + 32 * ka * PITCH;
      auto a_op = [&](int j) {
        return *reinterpret_cast<const u32x4*>(((j & 1) ? oa : qa) + poff<D>(0, (j >> 1) * 16));
      };
      auto squash = [&](int i) __attribute__((always_inline)) {
        if constexpr (CAP) {
          const float r = __builtin_amdgcn_rcpf(1.f + fast_exp2(sc[kb][i] * p.fn.cap_in));
          sc[kb][i] = r;
          dp[kb][i] *= fmaf(-r, r, r);  // f' / 4
        }
      };
      f32x4 nd[2][2], lsv[2][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          nd[h][e] = *reinterpret_cast<const f32x4*>(&dss[b][ka * 32 + 16 * h + 8 * g + 4 * e]);
          lsv[h][e] = *reinterpret_cast<const f32x4*>(&lss[bb][sb * 32 + 16 * h + 8 * g + 4 * e]);
        }
      }
      auto exactly = [&]() __attribute__((always_inline)) {
        // This lane's key from its first row; pinned, or what follows from it per score is
        // worked out ahead of the loop and spilled.
        int rel0 = kp - p0 - 8 * g;
        asm volatile("" : "+v"(rel0));
        if (BIAS != kBiasNone && near) {
          const float* t = tables + (cur.g & 1) * bins + (BIAS == kBiasTable ? rel0 + p.fn.reach + kScoreBinMargin : 0);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int off = 16 * (i >> 3) + (i & 7);
            if constexpr (BIAS == kBiasSlope) sc[kb][i] = fmaf(-slope2, fabsf((float)(rel0 - off)), sc[kb][i] * coef);
            else sc[kb][i] = fmaf(sc[kb][i], coef, t[-off]);
            if (BIAS == kBiasTable && (i & 7) == 7) __builtin_amdgcn_sched_barrier(0);  // registers
          }
          cf = 1.f;
          sl = add = 0.f;
        }
        if (!all || nrow < 32) {
          const float none = cf < 0.f ? INFINITY : -INFINITY;  // exponent -inf either way
          // the rows' intervals, in the order of the registers; in halves of eight
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            i32x4 lo[2], len[2];  // rows behind the segment: none
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              lo[e] = *reinterpret_cast<const i32x4*>(&los[bb][32 * sb + 16 * h + 8 * g + 4 * e]);
              len[e] = *reinterpret_cast<const i32x4*>(&lens[bb][32 * sb + 16 * h + 8 * g + 4 * e]);
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
              const int i = 8 * h + u;
              const bool seen = (uint32_t)(kp - lo[u >> 2][u & 3]) < (uint32_t)len[u >> 2][u & 3] && lsv[h][u >> 2][u & 3] != kScoreNoKey;
              sc[kb][i] = seen ? sc[kb][i] : none;
              dp[kb][i] = seen ? dp[kb][i] : 0.f;
            }
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      };
      const Row row = row_of(b, ka);  // read ahead of its use by half of the products
      u32x4 pp[2], pds[2];
      constexpr int PFA = 4;
      u32x4 ring[PFA];
#pragma unroll
      for (int j = 0; j < PFA; ++j) ring[j] = a_op(j);
      if (!CAP && has_b) exactly();
      __builtin_amdgcn_sched_barrier(0);
      f32x16 s = f32x16{}, d_;
#pragma unroll
      for (int i = 0; i < 16; ++i) d_[i] = nd[i >> 3][(i >> 2) & 1][i & 3];
      auto weights = [&](int c) __attribute__((always_inline)) {  // elements 2c, 2c+1 of B
        const int h = c >> 2, t2 = c & 3;
        float pv[2], dv_[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int tt = 2 * t2 + e, i = 8 * h + tt;
          float t = -lsv[h][tt >> 2][tt & 3];
          if constexpr (BIAS != kBiasNone) t += add;
          if constexpr (BIAS == kBiasSlope) t = fmaf(sl, (float)(16 * h + tt), t);
          pv[e] = fast_exp2(fmaf(sc[kb][i], cf, t));
          dv_[e] = pv[e] * dp[kb][i];
        }
        pp[h][t2] = pack_bf16(pv[0], pv[1]);
        pds[h][t2] = pack_bf16(dv_[0], dv_[1]);
      };
#pragma unroll
      for (int j = 0; j < NM; ++j) {
        const u32x4 a = ring[j % PFA];
        if (j + PFA < NM) ring[j % PFA] = a_op(j + PFA);
        if (j & 1) d_ = mfma32(a, vf[j >> 1], d_);
        else s = mfma32(a, kf[j >> 1], s);
        if (has_b) {
          if constexpr (CAP) {
            // first half of the slots: the cap of all scores; second half: their weights
            constexpr int PER = 8 / (NM / 2);  // pairs per slot
#pragma unroll
            for (int e = 0; e < PER; ++e) {
              const int c = (j % (NM / 2)) * PER + e;
              if (j < NM / 2) {
                squash(2 * c);
                squash(2 * c + 1);
              } else {
                weights(c);
              }
            }
            if (j == NM / 2 - 1) exactly();
          } else if (j % (NM / 8) == NM / 8 - 1) {
            weights(j / (NM / 8));
          }
        }
        if (j == NM / 2 - 1) look(row, ka, ta);
        __builtin_amdgcn_sched_barrier(0);
      }
      asm volatile("" : "+v"(s), "+v"(d_));
      sc[ka] = s;
      dp[ka] = d_;
      if (has_b) {
        xch[xb][kw][0][lane] = pp[0];
        xch[xb][kw][1][lane] = pp[1];
        xch[xb][kw][2][lane] = pds[0];
        xch[xb][kw][3][lane] = pds[1];
      }
    };

    fetch(it, nt, G, ahead, 1);
    ahead = next(ahead);
    phase(0, 0, t0, 0, 0, false, 0);
    __syncthreads();
    // The buffers of tiles t, t+1, t+2 in turn.  They are numbers at run time: unrolled by three,
    // with what masked blocks need in every phase, the loop's code outgrew the instruction cache.
    int b0 = 0, b1 = 1, b2 = 2;
#pragma unroll 1
    for (int t = 0; t < total; ++t) {
      if (BIAS != kBiasNone && cur.t == t0) of_head(cur.g);
      phase(1, b0, cur.t, 0, b0, true, 0);
      wait_vmem();  // own loads of tile t+1 landed
      __syncthreads();
      fetch(it, nt, G, ahead, b2);
      ahead = next(ahead);
      phase(0, b1, next(cur).t, 1, b0, true, 1);
      __syncthreads();
      cur = next(cur);
      const int b = b0;
      b0 = b1;
      b1 = b2;
      b2 = b;
    }
    __syncthreads();
    wait_vmem();  // the lookahead loads must land before the LDS is released
  } else {
    // ---------------------------------------------------------- consumer
    // A head's table, in log2 units, by the consumers in the phase in front of its first use.
    auto table = [&](int gh) {
      if constexpr (BIAS == kBiasTable) {
        BiasFill<256> fill;
        fill.start(p.fn, tid - 256);
        fill.finish(tables + (gh & 1) * bins, p.fn, head0 + gh, H, tid - 256);
      }
    };

    // Consumer wave 4 + ci: dV (ci < 2) or dK (ci >= 2) of all 128 keys, half dh = ci % 2 of d.
    const int ci = wave - 4;
    const bool is_dk = ci >= 2;
    const int dh = ci & 1;
    constexpr int NDT = D / 64;
    Cursor cur{0, t0}, ahead{0, t0};
    fetch(it, nt, G, ahead, 0);
    ahead = next(ahead);
    f32x16 acc[4][NDT];
#pragma unroll
    for (int kg = 0; kg < 4; ++kg) {
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) acc[kg][dt] = f32x16{};
    }
    wait_vmem();
    __syncthreads();  // tile 0 published

    auto phaseC = [&](int r, int sb, int xb) __attribute__((always_inline)) {
      const char* tbuf = (is_dk ? qs[r] : dos[r]) + t_off;
      u32x4 a[2][NDT], w[4][2];
      const int m0 = s_mask[xb][0], m1 = s_mask[xb][1], m2 = s_mask[xb][2], m3 = s_mask[xb][3];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) a[h][dt] = tr_operand<D>(tbuf, sb * 32 + 16 * h, (dh * NDT + dt) * 32);
#pragma unroll
        for (int kg = 0; kg < 4; ++kg) w[kg][h] = xch[xb][kg][(is_dk ? 2 : 0) + h][lane];
      }
      // A mask runs through a block: its weights of zero must meet finite values.  What a row
      // sees that is not finite is in its weights already (score_pre_kernel).
      if (__builtin_amdgcn_readfirstlane(m0 | m1 | m2 | m3)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt) a[h][dt] = finite_only(a[h][dt]);
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) {
#pragma unroll
          for (int kg = 0; kg < 4; ++kg) acc[kg][dt] = mfma32(a[h][dt], w[kg][h], acc[kg][dt]);
        }
      }
    };
    fetch(it, nt, G, ahead, 1);
    ahead = next(ahead);
    if (total > 0) table(0);
    __syncthreads();
    wait_vmem();  // own loads of tile 1 landed
    __syncthreads();
    // Phases 2t+2, 2t+3: C(2t), C(2t+1).
    int b0 = 0, b1 = 1, b2 = 2;
#pragma unroll 1
    for (int t = 0; t < total; ++t) {
      fetch(it, nt, G, ahead, b2);
      ahead = next(ahead);
      cur = next(cur);
      if (cur.t == t0 && cur.g < G) table(cur.g);
      phaseC(b0, 0, 0);
      __syncthreads();
      phaseC(b0, 1, 1);
      wait_vmem();  // own loads of tile t+2 landed
      __syncthreads();
#pragma unroll
      for (int kg = 0; kg < 4; ++kg) {
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) asm volatile("" : "+v"(acc[kg][dt]));
      }
      const int b = b0;
      b0 = b1;
      b1 = b2;
      b2 = b;
    }

    // dK = scale * dK^T (and the 4 of f') or dV = dV^T: register i <-> d = (dh*NDT + dt)*32 + 16*(i/8) + 8g + i%8.
    // An item of some of the heads leaves fp32 partials: [part][dK, dV][128 keys][d].
    const float osc = is_dk ? p.scale * (CAP ? 4.f : 1.f) : 1.f;
    uint16_t* og = static_cast<uint16_t*>(is_dk ? p.dk : p.dv);
#pragma unroll
    for (int kg = 0; kg < 4; ++kg) {
      const int okey = kg * 32 + ln;
      if (okey >= it.k_len) continue;
      uint16_t* dst = og + ((int64_t)(it.k_start + okey) * Hk + it.kv_head) * D;
      float* part = p.kv_part + (((int64_t)it.part * 2 + (is_dk ? 0 : 1)) * kScoreKvTileN + okey) * D;
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (it.part >= 0) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
              *reinterpret_cast<f32x4*>(part + (dh * NDT + dt) * 32 + 16 * h + 8 * g + 4 * t) =
                  f32x4{acc[kg][dt][8 * h + 4 * t] * osc, acc[kg][dt][8 * h + 4 * t + 1] * osc,
                        acc[kg][dt][8 * h + 4 * t + 2] * osc, acc[kg][dt][8 * h + 4 * t + 3] * osc};
            continue;
          }
          u32x4 wo;
#pragma unroll
          for (int t = 0; t < 4; ++t)
            wo[t] = pack_bf16(acc[kg][dt][8 * h + 2 * t] * osc, acc[kg][dt][8 * h + 2 * t + 1] * osc);
          *reinterpret_cast<u32x4*>(dst + (dh * NDT + dt) * 32 + 16 * h + 8 * g) = wo;
        }
      }
    }
  }
}

}  // namespace dkdv
}  // namespace
}  // namespace zl
