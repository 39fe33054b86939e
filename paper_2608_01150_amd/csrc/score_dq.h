// Scored attention: dQ and the sums for the bias table's gradient, bf16 inputs,
// gfx950 MFMA.
//
// An item is up to 128 query rows of one head (4 waves x 32) against the key ranges of its
// segment, one per workgroup, two workgroups on a CU (see score_fwd.hip; 10920 tokens of
// frames, 12 heads of 128: 762 us against 884 with 256 rows and eight waves; in the order of
// their keys 626, 1000 TFLOP/s of the 6 d flop a pair that it runs).  As in the
// plain dQ (bwd_bf16.hip), per step of 64 keys
//   S^T = K Q^T,  dP^T - D = V dO^T - D   MFMA (Q, dO in registers, one query per lane)
//   dS^T = P^T (dP^T - D) f'              VALU
//   dQ^T += K^T dS^T                      MFMA, K^T by transpose reads, dS rounded to bf16 as K is
// with K and V staged one tile ahead.  Blocks of 32 keys that no row of the wave sees
// are left out, and those that all rows see at one side of slope or table cost one or
// two fma per score, as in the forward.  Other blocks are worked out score by score
// (`exactly`), which leaves dS itself in the place of dP - D and a weight of one.
//
// The table's gradient: dA = P (dP - D) of a pair goes to the sum of its relative
// position.  A block beyond the table's reach has one sum per lane, which goes to a bin of
// the margins (they join the table's ends): sums kept in registers made the joint launch of
// short calls spill (2 x 512 tokens, 12 heads of 128, 85 us; 53 with the bins).
// In the others a wave sums the block's diagonals across its lanes (one permute per
// register) and adds them to bins in LDS, a row of bins per half of a wave: no two lanes
// add to one bin, and the order of every sum is fixed.  (LDS atomics, one per score,
// took 80 ns per wave instruction, the permute takes 3.)  An item writes its sums per
// relative position; score_dbias_kernel adds the items' and then the positions of each
// bucket.

#pragma once

#include "zl_score_device.h"

namespace zl {
namespace {
namespace dq {

constexpr int BN = 64;            // keys per step
constexpr int NW = 4;             // waves that share the item's rows

// Keys per staged tile; the bins need the LDS of a second step (and, with d = 128, leave room
// for one workgroup per CU: 2 x 2048 tokens, 16 heads, 178 us with the gradient, 110 without).
template <int D, bool TABLE_GRAD>
constexpr int kTileN = D == 128 || TABLE_GRAD ? BN : 2 * BN;

template <int D, bool TABLE_GRAD, bool SPLIT>
struct Lds {
  static constexpr int BUFS = (SPLIT ? 2 : 1) * 2 * kTileN<D, TABLE_GRAD> * Pad<D>::PITCH;
  __attribute__((aligned(16))) char k_lds[BUFS], v_lds[BUFS];
  float s_bins[TABLE_GRAD ? 2 * NW : 1][TABLE_GRAD ? kScoreBins : 1];
  float s_ends[2];
  int s_lo[NW], s_hi[NW];
};

// Item `item`, by a workgroup of four waves, or eight with SPLIT (no table gradient): two groups
// of waves, each with every other tile of the keys, as in the forward.  s_bias: room for a table.
template <int D, bool CAP, int BIAS, bool TABLE_GRAD, bool SPLIT>
__device__ __forceinline__ void run(const ScoreBwdParams& p, int item, Lds<D, TABLE_GRAD, SPLIT>& lds, float* s_bias) {
  static_assert(!(SPLIT && TABLE_GRAD), "the bins leave no LDS for a second group's tiles");
  constexpr int NG = SPLIT ? 2 : 1, NT = 64 * NW * NG;
  constexpr int PITCH = Pad<D>::PITCH;
  constexpr int TN = kTileN<D, TABLE_GRAD>;
  constexpr int STRIDE = NG * TN;      // from one of a group's tiles to the next
  constexpr int TILE = TN * PITCH, HALF = BN * PITCH;
  using Dma = TileDma<D, BN, NW / 2>;  // half of a group's waves load K tiles, the others V tiles
  constexpr int DMA_PER_STEP = Dma::PER_WAVE;
  auto &k_lds = lds.k_lds, &v_lds = lds.v_lds;
  auto& s_bins = lds.s_bins;
  auto& s_ends = lds.s_ends;
  auto &s_lo = lds.s_lo, &s_hi = lds.s_hi;

  const int tid = threadIdx.x, lane = tid & 63;
  const int group = SPLIT ? __builtin_amdgcn_readfirstlane(tid >> 8) : 0;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6) & (NW - 1);  // of its group
  char *const ks = k_lds + group * 2 * TILE, *const vs = v_lds + group * 2 * TILE;
  const int ln = lane & 31, g = lane >> 5;
  const uint32_t a_off = poff<D>(perm32(ln), g * 8), t_off = tr_lane_off<D>(lane);
  const int H = p.num_heads, Hk = H / p.group;
  const float coef = CAP ? -2.f * p.fn.cap_log2 : p.fn.scale_log2;
  const bool plain_rows = !p.fn.key_lo && !p.fn.key_hi;
  const int reach = p.fn.reach, mid = reach + kScoreBinMargin;  // bin of relative position 0

  const ScoreItem it = p.q_items[item];
  const int kvh = it.head / p.group;
  const int64_t rs = (int64_t)Hk * D;
  const uint32_t row_bytes = (uint32_t)rs * 2u;

  const int qr = wave * 32 + ln;
  const bool q_ok = qr < it.q_len;
  const bool wave_live = wave * 32 < it.q_len;
  const int64_t qrow = (int64_t)(it.q_start + qr) * H + it.head;
  u32x4 qf[D / 16], of[D / 16];
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) {
    qf[kk] = of[kk] = u32x4{0, 0, 0, 0};
    if (q_ok) {
      qf[kk] = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p.q) + qrow * D + kk * 16 + g * 8);
      of[kk] = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p.dout) + qrow * D + kk * 16 + g * 8);
    }
  }
  float lse2 = q_ok ? p.lse2[qrow] : kScoreNoKey;
  float nd = q_ok ? p.dsum[qrow] : 0.f;  // -D of this lane's query, where every dP^T block starts
  if (lse2 == kScoreNoGrad) {
    lse2 = 0.f;
    nd = __builtin_nanf("");
  }
  RowSee see{it.q_pos + qr, 0, 0};
  if (q_ok) see = row_see(p.fn, it.q_start + qr, it.q_pos + qr);
  // a row without a weight (a table of -inf) sees nothing either: 0 * NaN in what it holds
  const bool none = q_ok && lse2 == kScoreNoKey;
  if (none) see.lo = see.hi = 0;
  float slope2 = 0.f;
  if constexpr (BIAS == kBiasSlope) slope2 = p.fn.slope[it.head] * 1.4426950408889634f;
  BiasFill<NT> fill;
  if constexpr (BIAS == kBiasTable) fill.start(p.fn, tid);
  // Sums of a row's P: beyond the table's reach before and behind it, and in the other blocks; and of all its dA.
  float weight[2] = {0.f, 0.f}, within = 0.f, rest = 0.f;
  if constexpr (TABLE_GRAD) {
    for (int i = tid; i <= 2 * mid; i += NT) {
#pragma unroll
      for (int r = 0; r < 2 * NW; ++r) s_bins[r][i] = 0.f;
    }
  }

  WaveSee ws;
  int i_lo = 0, i_hi = INT32_MAX;
  if (plain_rows) {
    const int first = it.q_pos + wave * 32, last = it.q_pos + min(wave * 32 + 31, it.q_len - 1);
    ws = {first, last, 0, 0, p.fn.causal ? first + 1 : INT32_MAX, p.fn.causal ? last + 1 : INT32_MAX};
    if (p.fn.causal) i_hi = it.q_pos + it.q_len;
    if (__any(none)) ws.hi_min = 0;  // no block that all rows see
  } else {
    ws = wave_see(see, q_ok);
    if (lane == 0) {
      s_lo[wave] = ws.lo_min < ws.hi_max ? ws.lo_min : INT32_MAX;
      s_hi[wave] = ws.hi_max;
    }
    __syncthreads();
    i_lo = INT32_MAX;
    i_hi = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      i_lo = min(i_lo, s_lo[w]);
      i_hi = max(i_hi, s_hi[w]);
    }
    i_lo = __builtin_amdgcn_readfirstlane(i_lo);
    i_hi = __builtin_amdgcn_readfirstlane(i_hi);
  }
  // Keys [k0, k1) of a range that some row of the item sees, from a whole tile on, so that a
  // row meets its keys in the same steps in every item.
  auto visible = [&](const ScoreRange& rg, int& k0, int& k1) {
    k1 = min(rg.k_len, max(i_hi - rg.k_pos, 0));
    k0 = max(i_lo - rg.k_pos, 0) & ~((SPLIT ? TN : BN) - 1);
  };
  // This group's first key from k0 on.
  auto first_key = [&](int k0) { return SPLIT && ((k0 / TN) & 1) != group ? k0 + TN : k0; };
  const bool loads_k = wave < NW / 2;
  char* const dst = loads_k ? ks : vs;
  Dma dma;
  dma.init(wave & (NW / 2 - 1), lane, row_bytes);
  auto source = [&](const ScoreRange& rg) {
    return static_cast<const uint16_t*>(loads_k ? p.k : p.v) + ((int64_t)rg.k_start * Hk + kvh) * D;
  };
  auto fetch = [&](const ScoreRange& rg, int k0, int k1) {
    const uint16_t* src = source(rg) + (int64_t)k0 * rs;
    dma.issue(dst, src, k1 - k0, row_bytes);
    if constexpr (TN > BN) dma.issue(dst + HALF, src + (int64_t)BN * rs, k1 - k0 - BN, row_bytes);
  };
  {  // the first tile, under way with the rows' own loads
    const ScoreRange rg = uniform(it.range);
    int k0, k1;
    visible(rg, k0, k1);
    if (k0 < k1) fetch(rg, first_key(k0), k1);
  }
  float far_lo = 0.f, far_hi = 0.f;  // the table's ends
  if constexpr (BIAS == kBiasTable) {
    fill.finish(s_bias, p.fn, it.head, H, tid);
    __syncthreads();
    far_lo = s_bias[0];
    far_hi = s_bias[2 * mid];
  }
  f32x16 dq[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db) dq[db] = f32x16{};
  __builtin_amdgcn_s_waitcnt(0);  // no pending register loads in the step loop

  for (int ri = 0; ri < it.range_count; ++ri) {
    ScoreRange rg = uniform(it.range);
    if (ri > 0) rg = uniform(p.ranges[it.range_next + ri - 1]);
    int k0, k1;
    visible(rg, k0, k1);
    if (k0 >= k1) continue;
    const uint16_t* src = source(rg);
    auto resource = [&](int kt) { return Dma::resource(src + (int64_t)kt * rs, k1 - kt, row_bytes); };

    // One 64-key step as two 32-key blocks kb, pipelined inside the wave:
    //   S/dP of kb 0; S/dP of kb 1 with the scores of kb 0; dQ of kb 0 with those of kb 1; dQ of kb 1.
    auto step = [&](int buf, int kt, const i32x4& rsrc, uint32_t lds) __attribute__((always_inline)) {
      const char *ka = ks + buf + a_off, *va = vs + buf + a_off, *kt_ = ks + buf + t_off;
      constexpr int NSD = 2 * (D / 16) * 2, NQ = 2 * (D / 32) * 2, PF = D == 128 ? 2 : 6, PFC = D == 128 ? 2 : 3;
      constexpr int DMA_GAP = NSD / DMA_PER_STEP;
      static_assert(DMA_GAP >= 1 && (DMA_PER_STEP - 1) * DMA_GAP < NSD, "spread fetch must fit the S/dP MFMAs");
      auto a_op = [&](int j) {
        return *reinterpret_cast<const u32x4*>(((j & 1) ? va : ka) +
                                               poff<D>((j / (NSD / 2)) * 32, ((j % (NSD / 2)) >> 1) * 16));
      };
      auto c_op = [&](int m) {
        return tr_operand<D>(kt_, (m / (NQ / 2)) * 32 + 16 * (m & 1), ((m % (NQ / 2)) >> 1) * 32);
      };
      const int kp = rg.k_pos + kt, nvalid = k1 - kt;
      f32x16 sc[2], dpc[2];
      u32x4 pds[2][2];
      float cf[2], sl[2], tb[2];
      // masked: a mask runs through the block.  near: the diagonal or the table's reach does.
      bool masked[2], cut[2], near[2];
      int side[2];  // table: -1 or 1 beyond its reach before or behind the rows, 0 within
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const int b0 = kp + 32 * kb;
        masked[kb] = !ws.sees_all(b0, min(32, max(nvalid - 32 * kb, 0)));
        cut[kb] = masked[kb] || nvalid < 32 * kb + 32;
        near[kb] = false;
        cf[kb] = coef;
        sl[kb] = 0.f;
        tb[kb] = -lse2;
        side[kb] = 0;
        if constexpr (BIAS == kBiasSlope) {
          const bool behind = b0 >= ws.pos_max;
          near[kb] = !behind && b0 + 31 > ws.pos_min;
          sl[kb] = behind ? -slope2 : slope2;
          tb[kb] = fmaf(-sl[kb], (float)(see.pos - b0 - 8 * g), -lse2);
        }
        if constexpr (BIAS == kBiasTable) {
          const bool behind = b0 - ws.pos_max >= reach;
          side[kb] = behind ? 1 : b0 + 31 - ws.pos_min <= -reach ? -1 : 0;
          near[kb] = side[kb] == 0;
          tb[kb] += behind ? far_hi : far_lo;
        }
      }
      auto squash = [&](int kb, int i) __attribute__((always_inline)) {
        if constexpr (CAP) sc[kb][i] = __builtin_amdgcn_rcpf(1.f + fast_exp2(sc[kb][i] * p.fn.cap_in));
      };
      // What of a block is worked out score by score.  A mask takes scores to an exponent of -inf
      // and dP - D to zero; the diagonal or the table leave dS itself in the place of dP - D and
      // an exponent of zero.
      auto exactly = [&](int kb) __attribute__((always_inline)) {
        const int b0 = kp + 32 * kb + 8 * g;  // position of this lane's first key
        if (cut[kb]) {
          const int end = min(see.hi, kp + nvalid);
          const uint32_t len = (uint32_t)max(end - see.lo, 0);
          // pinned, or what follows from it per score is worked out ahead of the loop and spilled
          int from_lo = b0 - see.lo;
          asm volatile("" : "+v"(from_lo));
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const bool seen = (uint32_t)(from_lo + 16 * (i >> 3) + (i & 7)) < len;
            sc[kb][i] = seen ? sc[kb][i] : CAP ? 1e18f : -INFINITY;  // CAP: r (1 - r) stays finite
            dpc[kb][i] = seen ? dpc[kb][i] : 0.f;
          }
        }
        if (BIAS != kBiasNone && near[kb]) {
          int rel0 = b0 - see.pos;
          asm volatile("" : "+v"(rel0));
          const float* t = s_bias + (BIAS == kBiasTable ? rel0 + mid : 0);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int off = 16 * (i >> 3) + (i & 7);
            float a = fmaf(sc[kb][i], coef, -lse2);
            if constexpr (BIAS == kBiasSlope) a = fmaf(-slope2, fabsf((float)(rel0 + off)), a);
            else a += t[off];
            const float w = fast_exp2(a);
            dpc[kb][i] *= w;
            if constexpr (TABLE_GRAD) within += w;
          }
          if constexpr (TABLE_GRAD) {
#pragma unroll
            for (int i = 0; i < 16; ++i) rest += dpc[kb][i];
            // The sums of the block's 63 diagonals.  At register i (offset off of both halves' keys,
            // which are 8 apart) lane p of half g takes the value that is off - p lanes on from its
            // half's first: with off >= p row off - p of its own half, diagonal p + 8 g; otherwise
            // row 32 + off - p of the other half, diagonal p - 24 - 8 g.
            const int from = (32 * g - ln) * 4;
            float own = 0.f, other = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int off = 16 * (i >> 3) + (i & 7);
              const float x = __int_as_float(__builtin_amdgcn_ds_bpermute(from + 4 * off, __float_as_int(dpc[kb][i])));
              own += off >= ln ? x : 0.f;
              other += off >= ln ? 0.f : x;
            }
            float* bin = s_bins[2 * wave + g] + b0 + ln - ws.pos_min + mid;
            // One lane's second bin is another's first: the adds stay in this order (LDS runs a
            // wave's accesses in order; the compiler must keep them so).
            asm volatile("" ::: "memory");
            bin[0] += own;
            asm volatile("" ::: "memory");
            bin[g ? -40 : -24] += other;
            asm volatile("" ::: "memory");
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            // CAP: r = 1/2 leaves a factor of 1/4, as every r (1 - r) stands for f' / 4
            if constexpr (CAP) dpc[kb][i] *= 4.f * fmaf(-sc[kb][i], sc[kb][i], sc[kb][i]);
            sc[kb][i] = CAP ? 0.5f : 0.f;
          }
          cf[kb] = sl[kb] = tb[kb] = 0.f;
        }
        // What follows is one path for every block: without the pins the compiler splits it into
        // one with these constants and one without, score by score.
        if constexpr (BIAS != kBiasNone) asm volatile("" : "+v"(sc[kb]), "+v"(cf[kb]), "+v"(tb[kb]), "+v"(sl[kb]));
      };
      float total[2] = {0.f, 0.f}, psum[2] = {0.f, 0.f};
      auto softmax2 = [&](int kb, int i) __attribute__((always_inline)) {  // elements i, i+1 -> one packed dS word
        float e[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int x = i + u;
          const float t = BIAS == kBiasSlope ? fmaf(sl[kb], (float)(16 * (x >> 3) + (x & 7)), tb[kb]) : tb[kb];
          const float w = fast_exp2(fmaf(sc[kb][x], cf[kb], t));
          e[u] = w * dpc[kb][x];
          if constexpr (TABLE_GRAD) {
            total[kb] += e[u];
            psum[kb] += w;
          }
          if constexpr (CAP) e[u] *= fmaf(-sc[kb][x], sc[kb][x], sc[kb][x]);
        }
        pds[kb][i >> 3][(i & 7) >> 1] = pack_bf16(e[0], e[1]);
      };
      u32x4 ring[PF];
#pragma unroll
      for (int j = 0; j < PF; ++j) ring[j] = a_op(j);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) sc[kb] = f32x16{};
      // Not held as a vector across the loop: sixteen registers.
      asm volatile("" : "+v"(nd));
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < NSD; ++j) {
        const u32x4 a = ring[j % PF];
        if (j + PF < NSD) ring[j % PF] = a_op(j + PF);
        const int kb = j / (NSD / 2), kk = (j % (NSD / 2)) >> 1;
        if (j % (NSD / 2) == 0) {
#pragma unroll
          for (int i = 0; i < 16; ++i) dpc[kb][i] = nd;
        }
        if (j & 1) dpc[kb] = mfma32(a, of[kk], dpc[kb]);
        else sc[kb] = mfma32(a, qf[kk], sc[kb]);
        if (j % DMA_GAP == (DMA_GAP > 1 ? 1 : 0) && j / DMA_GAP < DMA_PER_STEP) dma.issue_one(rsrc, lds, j / DMA_GAP);
        // kb 1's MFMAs carry kb 0's scores: 16 elements over NSD/2 MFMAs.
        if (j >= NSD / 2) {
          constexpr int SLOTS = NSD / 2;
          const int x = j - NSD / 2;
          if constexpr (CAP) {
            constexpr int PER = 16 / (SLOTS / 2);  // elements per slot: caps in the first half, weights in the second
#pragma unroll
            for (int u = 0; u < PER; u += 2) {
              const int i = (x % (SLOTS / 2)) * PER + u;
              if (x < SLOTS / 2) {
                squash(0, i);
                squash(0, i + 1);
              } else {
                softmax2(0, i);
              }
            }
            if (x == SLOTS / 2 - 1) exactly(0);
          } else {
            if (x == 0) exactly(0);
            if (x % (SLOTS / 8) == SLOTS / 8 - 1) softmax2(0, 2 * (x / (SLOTS / 8)));
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      u32x4 cring[PFC];
#pragma unroll
      for (int m = 0; m < PFC; ++m) {
        cring[m] = c_op(m);
        if (masked[m / (NQ / 2)]) cring[m] = finite_only(cring[m]);
      }
      if (!CAP) exactly(1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int m = 0; m < NQ; ++m) {
        const u32x4 a = cring[m % PFC];
        if (m + PFC < NQ) {
          u32x4 c = c_op(m + PFC);
          // a mask runs through the block: its weights of zero must meet finite keys
          if (masked[(m + PFC) / (NQ / 2)]) c = finite_only(c);
          cring[m % PFC] = c;
        }
        if (m < NQ / 2) {
          constexpr int SLOTS = NQ / 2;
          if constexpr (CAP) {
            constexpr int PER = 16 / (SLOTS / 2);
#pragma unroll
            for (int u = 0; u < PER; u += 2) {
              const int i = (m % (SLOTS / 2)) * PER + u;
              if (m < SLOTS / 2) {
                squash(1, i);
                squash(1, i + 1);
              } else {
                softmax2(1, i);
              }
            }
            if (m == SLOTS / 2 - 1) exactly(1);
          } else {
            softmax2(1, (16 / SLOTS) * m);
            if (16 / SLOTS == 4) softmax2(1, (16 / SLOTS) * m + 2);
          }
        }
        const int kb = m / (NQ / 2), db = (m % (NQ / 2)) >> 1, s2 = m & 1;
        dq[db] = mfma32(a, pds[kb][s2], dq[db]);
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (TABLE_GRAD) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          if (side[kb] == 0) continue;
          // to bins of the margins, which belong to the table's ends: a bin of its own per lane
          s_bins[2 * wave + g][side[kb] < 0 ? ln : 2 * mid - ln] += total[kb];
          asm volatile("" ::: "memory");
          rest += total[kb];
          if (side[kb] < 0) weight[0] += psum[kb];
          else weight[1] += psum[kb];
        }
      }
    };

    if (ri > 0) {
      __syncthreads();  // the last range's tiles are no longer read
      fetch(rg, first_key(k0), k1);
    }
    // Steps that the wave sees nothing of only fetch, in a loop of their own (see the forward).
    int kt = first_key(k0), buf = 0, half = 0;
    const int end = SPLIT ? kt + (k1 - k0 + STRIDE - 1) / STRIDE * STRIDE : k1;  // as many tiles in both groups
    auto advance = [&]() __attribute__((always_inline)) {
      kt += BN;
      half += HALF;
      if (half == TILE) {
        half = 0;
        buf = TILE - buf;
        kt += STRIDE - TN;
        asm volatile("" : "+s"(buf));
      }
    };
#pragma unroll 1
    for (;;) {
      i32x4 rsrc = {};
      uint32_t lds = 0;
      bool live = false;
#pragma unroll 1
      while (kt < end) {
        if (half == 0) {
          wait_vmem();
          __syncthreads();  // this tile complete; the other buffer no longer read
        }
        rsrc = resource(kt + STRIDE);
        lds = lds_addr(dst + (TILE - buf) + half);
        const int kp = rg.k_pos + kt;
        live = wave_live && (!SPLIT || kt < k1) && kp < ws.hi_max && kp + BN > ws.lo_min;
        if (live) break;
#pragma unroll
        for (int jj = 0; jj < DMA_PER_STEP; ++jj) dma.issue_one(rsrc, lds, jj);
        advance();
      }
      if (!live) break;
      step(buf + half, kt, rsrc, lds);
      advance();
    }
    wait_vmem();  // the lookahead loads must land before the LDS is used again
  }

  if constexpr (SPLIT) {  // the second group's part, through LDS
    constexpr int NR = D / 32 * 4;
    static_assert(NR * NW * 64 * 16 <= NG * 2 * TILE, "the part must fit the K tiles");
    f32x4* x = reinterpret_cast<f32x4*>(k_lds) + wave * NR * 64 + lane;
    __syncthreads();  // tiles no longer read
    if (group == 1) {
#pragma unroll
      for (int r = 0; r < NR; ++r)
        x[r * 64] = f32x4{dq[r / 4][4 * (r % 4)], dq[r / 4][4 * (r % 4) + 1], dq[r / 4][4 * (r % 4) + 2], dq[r / 4][4 * (r % 4) + 3]};
    }
    __syncthreads();
    if (group == 1) return;
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      const f32x4 y = x[r * 64];
#pragma unroll
      for (int e = 0; e < 4; ++e) dq[r / 4][4 * (r % 4) + e] += y[e];
    }
  }

  if (q_ok) {
    const auto* pp = kernargs<ScoreBwdParams>();
    const float osc = pp->scale * (CAP ? 4.f : 1.f);
    uint16_t* dqg = static_cast<uint16_t*>(pp->dq) + qrow * D;
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        u32x4 w;
#pragma unroll
        for (int t = 0; t < 4; ++t) w[t] = pack_bf16(dq[db][8 * h + 2 * t] * osc, dq[db][8 * h + 2 * t + 1] * osc);
        *reinterpret_cast<u32x4*>(dqg + db * 32 + 16 * h + 8 * g) = w;
      }
    }
  }
  if constexpr (TABLE_GRAD) {
    // What lies beyond the reach joins its ends: the margins of all rows of bins, by one wave each.
    __syncthreads();  // bins complete
    // A row's dA add up to zero over all of its keys.  What they add up to here is D's error then,
    // mostly that of the rounding of the O it comes from, and the buckets of the table's ends, with
    // most of a long row's weight, would take most of it: they are relieved of their share (198 rows
    // of 994 keys, one head: the gradient's error 0.76% -> 0.1%).  The row's weights tell whether the
    // call holds all of its keys: they add up to one then.  Within 2^-12, where keys elsewhere have
    // less of the row than an eighth of what a rounding of O to bf16 may take from it.
    const float mass = xor32_sum(within + weight[0] + weight[1]), all = xor32_sum(rest);
    const float off = fabsf(mass - 1.f) <= 0x1p-12f ? all : 0.f;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float x = weight[e] == 0.f ? 0.f : -off * weight[e];
#pragma unroll
      for (int m = 32; m; m >>= 1) x += __shfl_xor(x, m);
      if (lane == 0) s_bins[2 * wave][e ? 2 * mid : 0] += x;  // bins that no pair reaches
    }
    __syncthreads();
    if (wave < 2) {
      float x = 0.f;
      for (int i = lane; i <= kScoreBinMargin; i += 64) {
        const int at = wave ? mid + reach + i : i;
#pragma unroll
        for (int r = 0; r < 2 * NW; ++r) x += s_bins[r][at];
      }
#pragma unroll
      for (int m = 32; m; m >>= 1) x += __shfl_xor(x, m);
      if (lane == 0) s_ends[wave] = x;
    }
    __syncthreads();
    float* part = p.dbias_part + (int64_t)it.part * (2 * reach + 1);
    for (int i = tid; i <= 2 * reach; i += NT) {
      float x = 0.f;
      if (i == 0 || i == 2 * reach) {
        x = s_ends[i != 0];
      } else {
#pragma unroll
        for (int r = 0; r < 2 * NW; ++r) x += s_bins[r][i + kScoreBinMargin];
      }
      part[i] = x;
    }
  }
}

}  // namespace dq
}  // namespace
}  // namespace zl
