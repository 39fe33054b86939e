// Scored attention forward, bf16 inputs, gfx950 MFMA.
//
// An item is up to 128 query rows of one head against its key ranges, run by a workgroup
// of four waves of 32 rows each.  As in the plain forward (fwd_bf16.hip), per step of 64
// keys
//   S^T = K Q^T      MFMA 32x32x16 bf16, one query per lane (two lanes share it)
//   A                cap, bias and mask, in log2 units
//   online softmax   against the running maximum as it stands (kSumBound)
//   O^T += V^T P^T   MFMA, V^T by transpose reads, P rounded to bf16 (as V is: a product of
//                    fp32 weights would take three of these)
// with K and V staged by direct global-to-LDS loads ahead of use (two waves load K, two
// V).  The row is normalised by the sum of the rounded weights, so that they sum to one
// exactly; the LSE takes the unrounded sum.
//
// Workgroups share a CU (two with d = 128, three or four with 64), so that one's prologue, epilogue and waits lie under the
// other's products, and masks that leave items unequal are evened out at 128 rows.
// Against one workgroup of eight waves and 256 rows: 10920 tokens of 7 frames, 12 heads
// of 128, 654 -> 611 us; 2048 causal tokens, 16 heads, 59 -> 49; 8192 unmasked tokens, 16
// heads, 536 -> 552.  One item per workgroup: the work queues of the plain kernels cost
// launches of short items more than they even out (16 captions 87 us with them, 43
// without) and long ones nothing (8192 tokens 543 and 535).  Shards of few items have two
// groups of four waves share an item's keys instead (SPLIT).
//
// Bounds.  8192 unmasked tokens, 16 heads of 128, run at 980 TFLOP/s of the 1207 that a
// large product reaches: the softmax's instructions between the MFMAs.  A step takes a
// wave 1.1 us beside another and 1.75 alone, so short launches go by their longest item
// (2048 causal tokens, 16 heads: 56 us, 310 TFLOP/s) and a cap by its transcendentals
// (6000 causal tokens, 32 heads: 730 TFLOP/s).
//
// What a score passes costs nothing where it need not.  Per 32-key block a wave knows
// from its rows' extremes of [lo, hi) and position (wave-uniform)
//   - that none of its rows sees the block: the step is left out, and keys that no row
//     of the item sees are not even loaded;
//   - that all of them see all of it, and all its keys are on one side of the rows
//     (slope) or beyond the table's reach (table): exponent = fma(s, coef, t), with
//     t = fma(slope, key offset, base) for a slope (one more instruction per score)
//     and t = base, the table's end and the maximum in it, otherwise;
//   - otherwise the block's bias, its mask or both are worked out score by score
//     (`exactly`): about two of a row's blocks under a causal mask, those within reach
//     of the diagonal with a table.
// A cap is r = 1 / (1 + exp2(2 s log2(e) / cap)), f = cap - 2 cap r: two more
// transcendentals per score, run under the S and PV MFMAs.

#include "zl_score_device.h"

namespace zl {
namespace {

constexpr int BN = 64;            // keys per step
constexpr int NW = 4;             // waves that share the item's rows
constexpr float kSumBound = 0x1p64f;  // see fwd_bf16.hip

// Epilogue: o[db][i] is (d = db*32 + 16*(i/8) + 8*g + i%8, this lane's query).
template <int D>
__device__ __forceinline__ void score_store(const __attribute__((address_space(4))) ScoreFwdParams* pp,
                                            const ScoreItem& it, int qr, bool q_ok, int g, const f32x16 (&o)[D / 32],
                                            float m_run, float l_part, float lr) {
  const auto& p = *pp;
  const float l = xor32_sum(l_part);
  const float inv = l != l ? l : lr == 0.f ? 0.f : 1.f / lr;
  const bool none = l == 0.f;  // weights of zero alone: O = 0, whatever they met in V
  const float lse = l == 0.f ? -INFINITY : (m_run + __log2f(l)) * kLn2;
  if (!q_ok) return;
  const int64_t row = (int64_t)(it.q_start + qr) * p.num_heads + it.head;
#pragma unroll
  for (int db = 0; db < D / 32; ++db) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int c0 = db * 32 + 16 * h + 8 * g;
      float x[8];
#pragma unroll
      for (int t = 0; t < 8; ++t) x[t] = none ? 0.f : o[db][8 * h + t] * inv;
      if (it.slot < 0) {
        const u32x4 w = {pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
        *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p.out) + row * D + c0) = w;
      } else {
        float* og = p.o_part + it.slot * p.slot_stride + row * D + c0;
        *reinterpret_cast<f32x4*>(og) = f32x4{x[0], x[1], x[2], x[3]};
        *reinterpret_cast<f32x4*>(og + 4) = f32x4{x[4], x[5], x[6], x[7]};
      }
    }
  }
  if (g == 0) {
    if (it.slot < 0) p.lse[row] = lse;
    else p.lse_part[it.slot * p.lse_slot_stride + row] = lse;
  }
}

// Waves per SIMD.  d = 64 leaves registers and, with tiles of one step, LDS for three workgroups
// per CU, and for four where nothing is added to a score: 16 captions of up to 512 tokens, 32
// heads, with a table 43 -> 36 us, without 35 -> 30; 8192 tokens, 16 heads, 421 -> 347.  Four
// with a table, a slope or a cap spill (83 us) or gain nothing (cap: 42 us, three 38).
template <int D, bool CAP, int BIAS, bool SPLIT>
constexpr int kOccupancy = D == 128 || SPLIT ? 2 : CAP || BIAS != kBiasNone ? 3 : 4;

// SPLIT: two groups of four waves, of which the first takes every other tile of the keys from
// the range's start on and the second the ones between, each with a maximum, sums and tiles of
// its own, joined at the end; one workgroup per CU.
template <int D, bool CAP, int BIAS, bool SPLIT>
__global__ __launch_bounds__(SPLIT ? 128 * NW : 64 * NW, (kOccupancy<D, CAP, BIAS, SPLIT>)) void score_fwd_kernel(ScoreFwdParams p) {
  constexpr int NG = SPLIT ? 2 : 1, NT = 64 * NW * NG;
  constexpr int PITCH = Pad<D>::PITCH;
  constexpr int TN = D == 64 && SPLIT ? 2 * BN : BN;  // keys per staged tile
  constexpr int TILE = TN * PITCH, HALF = BN * PITCH;
  constexpr int STRIDE = NG * TN;      // from one of a group's tiles to the next
  using Dma = TileDma<D, BN, NW / 2>;  // half of a group's waves load K tiles, the others V tiles
  constexpr int DMA_PER_STEP = Dma::PER_WAVE;
  __shared__ __attribute__((aligned(16))) char k_lds[NG * 2 * TILE], v_lds[NG * 2 * TILE];
  extern __shared__ float s_bias[];  // the table (dynamic: with a reach of up to 400 two workgroups fit)
  __shared__ int s_lo[NW], s_hi[NW];
  __shared__ uint64_t s_low[NG][NW];

  const int tid = threadIdx.x, lane = tid & 63;
  const int group = SPLIT ? __builtin_amdgcn_readfirstlane(tid >> 8) : 0;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6) & (NW - 1);  // of its group
  char *const ks = k_lds + group * 2 * TILE, *const vs = v_lds + group * 2 * TILE;
  const int ln = lane & 31, g = lane >> 5;
  const uint32_t a_off = poff<D>(perm32(ln), g * 8), t_off = tr_lane_off<D>(lane);
  const int Hk = p.num_heads / p.group;
  const float coef = CAP ? -2.f * p.fn.cap_log2 : p.fn.scale_log2;
  const float capc = CAP ? p.fn.cap_log2 : 0.f;
  // rows that are masked and placed by their positions alone
  const bool plain_rows = !p.fn.key_lo && !p.fn.key_hi && !p.fn.q_pos;

  const ScoreItem it = p.items[blockIdx.x];
  const int kvh = it.head / p.group;
  const int64_t rs = (int64_t)Hk * D;  // elements between consecutive keys
  const uint32_t row_bytes = (uint32_t)rs * 2u;

  const int qr = wave * 32 + ln;
  const bool q_ok = qr < it.q_len;
  const bool wave_live = wave * 32 < it.q_len;
  RowSee see{it.q_pos + qr, 0, 0};
  if (q_ok) see = row_see(p.fn, it.q_start + qr, it.q_pos + qr);
  const uint16_t* qg = static_cast<const uint16_t*>(p.q) + ((int64_t)(it.q_start + qr) * p.num_heads + it.head) * D;
  u32x4 qf[D / 16];
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk)
    qf[kk] = q_ok ? *reinterpret_cast<const u32x4*>(qg + kk * 16 + g * 8) : u32x4{0, 0, 0, 0};
  float slope2 = 0.f;
  if constexpr (BIAS == kBiasSlope) slope2 = p.fn.slope[it.head] * 1.4426950408889634f;
  // What a slope takes from a lane's keys of a block in front of the rows, from the last and nearest
  // on (so that it is never more than what it takes in all), in units of S: the S products start
  // from it, and the exponent costs no more than without a slope.
  constexpr bool LEAN = BIAS == kBiasSlope && !CAP;
  const float lean1 = slope2 / p.fn.scale_log2;
  f32x16 lean;
  if constexpr (LEAN) {
#pragma unroll
    for (int i = 0; i < 16; ++i) lean[i] = lean1 * (float)(16 * (i >> 3) + (i & 7) - 23);
  }
  BiasFill<NT> fill;
  if constexpr (BIAS == kBiasTable) fill.start(p.fn, tid);

  // Extremes over the wave's rows, and over the item's.
  WaveSee ws;
  int i_lo = 0, i_hi = INT32_MAX;
  if (plain_rows) {
    const int first = it.q_pos + wave * 32, last = it.q_pos + min(wave * 32 + 31, it.q_len - 1);
    ws = {first, last, 0, 0, p.fn.causal ? first + 1 : INT32_MAX, p.fn.causal ? last + 1 : INT32_MAX};
    if (p.fn.causal) i_hi = it.q_pos + it.q_len;
  } else {
    ws = wave_see(see, q_ok);
    if (!q_ok) see.pos = ws.pos_min;  // look-ups of lanes without a row stay beside the others
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
    fill.finish(s_bias, p.fn, it.head, p.num_heads, tid);
    __syncthreads();
    far_lo = s_bias[0];
    far_hi = s_bias[2 * (p.fn.reach + kScoreBinMargin)];
  }
  // The step loop carries no pending register loads (see fwd_bf16.hip).
  __builtin_amdgcn_s_waitcnt(0);

  float m_run, l_part;
  f32x4 racc;  // sums of the rounded weights (see fwd_bf16.hip)
  const uint32_t selw = ((lane >> 4) & 1) == ((lane >> 2) & 1) ? 0x3F803F80u : 0u;
  const u32x4 rsel = {selw, selw, selw, selw};
  f32x16 o[D / 32];
  bool infinite;  // some step kept infinities off (wave-uniform)

  // With a slope the scores grow towards the row, their weights by up to 2^65 a step, and a
  // maximum that starts at the first step's is moved in every other one.  So it starts at the
  // slope's share of the nearest key that the row sees (2048 causal rows, 16 heads of 64, 57 -> 46
  // us, 41 without a slope; 4096 and 1777 behind a prefix, 16 heads of 128, 147 -> 127).  Where
  // that turns out too high for a row's weights, the item is run again without.
  float m_start = kNegBig;
  bool sees = false;
  if constexpr (BIAS == kBiasSlope) {
    int dist = INT32_MAX;
    for (int ri = 0; ri < it.range_count; ++ri) {
      ScoreRange rg = uniform(it.range);
      if (ri > 0) rg = uniform(p.ranges[it.range_next + ri - 1]);
      const int a = max(see.lo, rg.k_pos), b = min(see.hi, rg.k_pos + rg.k_len);
      if (a < b) dist = min(dist, max(max(a - see.pos, see.pos - (b - 1)), 0));
    }
    sees = q_ok && dist < INT32_MAX;
    m_start = sees ? -slope2 * (float)dist : 0.f;
  }
  for (bool again = false;; again = true) {
    m_run = again ? kNegBig : m_start;
    l_part = 0.f;
    racc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int db = 0; db < D / 32; ++db) o[db] = f32x16{};
    infinite = false;
    for (int ri = 0; ri < it.range_count; ++ri) {
      ScoreRange rg = uniform(it.range);
      if (ri > 0) rg = uniform(p.ranges[it.range_next + ri - 1]);
      int k0, k1;
      visible(rg, k0, k1);
      if (k0 >= k1) continue;
      const uint16_t* src = source(rg);
      auto resource = [&](int kt) { return Dma::resource(src + (int64_t)kt * rs, k1 - kt, row_bytes); };

      // One 64-key step from LDS byte offset `buf` of both tiles; `rsrc` and `lds` take the
      // next tile's half.  keep_off: a mask runs through the step and V is not finite in it.
      // Blocks kb of 32 keys, pipelined inside the wave:
      //   S of kb 0;  S of kb 1 with the scores of kb 0;  PV of kb 0 with those of kb 1;  PV of kb 1.
      auto step = [&](int buf, int kt, const i32x4& rsrc, uint32_t lds, bool keep_off) __attribute__((always_inline)) {
        const char *ka = ks + buf + a_off, *vt = vs + buf + t_off;
        constexpr int NS = 2 * (D / 16), NP = 2 * (D / 32) * 2, PF = 6, PFC = 3;
        constexpr int DMA_GAP = NS / DMA_PER_STEP;
        static_assert(DMA_GAP >= 1 && (DMA_PER_STEP - 1) * DMA_GAP < NS, "spread fetch must fit the S MFMAs");
        auto a_op = [&](int j) {
          return *reinterpret_cast<const u32x4*>(ka + poff<D>((j / (NS / 2)) * 32, (j % (NS / 2)) * 16));
        };
        auto c_op = [&](int m) {
          return tr_operand<D>(vt, (m / (NP / 2)) * 32 + 16 * (m & 1), ((m % (NP / 2)) >> 1) * 32);
        };
        const int kp = rg.k_pos + kt, nvalid = k1 - kt;
        // The exponent of score i of block kb is fma(s, cf, fma(sl, offset of key i, tb)).
        f32x16 s[2];
        u32x4 pb[2][2];
        float lsum[2][2] = {};
        float cf[2], sl[2], tb[2];
        float rel[2];    // slope: this lane's position minus that of its first key of the block (LEAN: nearest)
        float add[2];    // what belongs to the exponent beside the maximum
        bool masked[2], near[2];  // a mask or the range's end, the diagonal or the table's reach runs through it
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          const int b0 = kp + 32 * kb;
          masked[kb] = !ws.sees_all(b0, 32) || nvalid < 32 * kb + 32;
          near[kb] = false;
          cf[kb] = coef;
          sl[kb] = 0.f;
          rel[kb] = 0.f;
          add[kb] = capc;
          if constexpr (BIAS == kBiasSlope) {
            const bool behind = b0 >= ws.pos_max;
            near[kb] = !behind && b0 + 31 > ws.pos_min;
            sl[kb] = behind ? -slope2 : slope2;
            rel[kb] = (float)(see.pos - b0 - 8 * g - (LEAN && !behind ? 23 : 0));
          }
          if constexpr (BIAS == kBiasTable) {
            const bool behind = b0 - ws.pos_max >= p.fn.reach;
            near[kb] = !behind && b0 + 31 - ws.pos_min > -p.fn.reach;
            add[kb] += behind ? far_hi : far_lo;
          }
        }
        auto base = [&](int kb, float m) { return BIAS == kBiasSlope ? fmaf(-sl[kb], rel[kb], add[kb] - m) : add[kb] - m; };
        auto offset = [](int i) { return (float)(16 * (i >> 3) + (i & 7)); };
        auto expnt = [&](int kb, int i, float t) {
          return fmaf(s[kb][i], cf[kb], BIAS == kBiasSlope && !LEAN ? fmaf(sl[kb], offset(i), t) : t);
        };
        auto squash = [&](int kb, int i) {
          if constexpr (CAP) s[kb][i] = __builtin_amdgcn_rcpf(1.f + fast_exp2(s[kb][i] * p.fn.cap_in));
        };
        // Scores of such a block, one by one.  What each follows from is pinned, or it is worked
        // out ahead of the loop for all sixteen and spilled.
        auto exactly = [&](int kb) {
          const int b0 = kp + 32 * kb + 8 * g;  // position of this lane's first key
          if (BIAS != kBiasNone && near[kb]) {
            int rel0 = b0 - see.pos;
            asm volatile("" : "+v"(rel0));
            if (BIAS == kBiasSlope) {
#pragma unroll
              for (int i = 0; i < 16; ++i)
                s[kb][i] = fmaf(-slope2, fabsf((float)(rel0 + 16 * (i >> 3) + (i & 7))), fmaf(s[kb][i], coef, capc));
            } else if (ws.pos_max - ws.pos_min < 32) {
              const float* t = s_bias + rel0 + p.fn.reach + kScoreBinMargin;
#pragma unroll
              for (int i = 0; i < 16; ++i) s[kb][i] = fmaf(s[kb][i], coef, capc) + t[16 * (i >> 3) + (i & 7)];
            } else {  // rows at positions apart (q_pos)
              const int mid = p.fn.reach + kScoreBinMargin;
#pragma unroll
              for (int i = 0; i < 16; ++i)
                s[kb][i] = fmaf(s[kb][i], coef, capc) + s_bias[min(max(rel0 + 16 * (i >> 3) + (i & 7) + mid, 0), 2 * mid)];
            }
            cf[kb] = 1.f;
            sl[kb] = add[kb] = 0.f;
          }
          if (masked[kb]) {
            const int end = min(see.hi, kp + nvalid);
            const uint32_t len = (uint32_t)max(end - see.lo, 0);
            int from_lo = b0 - see.lo;
            asm volatile("" : "+v"(from_lo));
            const float none = cf[kb] < 0.f ? INFINITY : -INFINITY;  // exponent -inf either way
#pragma unroll
            for (int i = 0; i < 16; ++i) s[kb][i] = (uint32_t)(from_lo + 16 * (i >> 3) + (i & 7)) < len ? s[kb][i] : none;
          }
        };
        auto expo = [&](int kb, int c) {
          const float e0 = fast_exp2(expnt(kb, 2 * c, tb[kb])), e1 = fast_exp2(expnt(kb, 2 * c + 1, tb[kb]));
          lsum[kb][c & 1] += e0 + e1;
          pb[kb][c >> 2][c & 3] = pack_bf16(e0, e1);
        };
        auto block_fix = [&](int kb) {
          const float t0 = base(kb, 0.f);
          float mt = -INFINITY;
#pragma unroll
          for (int i = 0; i < 16; ++i) mt = fmaxf(mt, expnt(kb, i, t0));
          const float m_new = fmaxf(m_run, xor32_max(mt));
          const float alpha = fast_exp2(m_run - m_new);
          m_run = m_new;
          l_part *= alpha;
          racc *= alpha;
#pragma unroll
          for (int db = 0; db < D / 32; ++db) {
#pragma unroll
            for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
          }
          lsum[kb][0] = lsum[kb][1] = 0.f;
          tb[kb] = base(kb, m_run);
#pragma unroll
          for (int c = 0; c < 8; ++c) expo(kb, c);
          // A row whose weights are no numbers keeps that in its sum alone: the rounded
          // sums of two rows share a product.
          if (lsum[kb][0] + lsum[kb][1] != lsum[kb][0] + lsum[kb][1]) pb[kb][0] = pb[kb][1] = u32x4{0, 0, 0, 0};
        };
        auto block_done = [&](int kb) {
          if (__any(!(lsum[kb][0] + lsum[kb][1] <= kSumBound))) block_fix(kb);
          l_part += lsum[kb][0] + lsum[kb][1];
        };

        u32x4 ring[PF];
#pragma unroll
        for (int j = 0; j < PF; ++j) ring[j] = a_op(j);
        s[0] = s[1] = f32x16{};
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int j = 0; j < NS; ++j) {
          const u32x4 a = ring[j % PF];
          if (j + PF < NS) ring[j % PF] = a_op(j + PF);
          const int kb = j / (NS / 2);
          if (LEAN && j % (NS / 2) == 0) {
            if (kp + 32 * kb + 31 <= ws.pos_min) {
              s[kb] = mfma32(a, qf[0], lean);
            } else {  // keys behind the rows, or on both sides of them (`exactly`)
              const float l1 = near[kb] ? 0.f : lean1;
#pragma unroll
              for (int i = 0; i < 16; ++i) s[kb][i] = l1 * -(float)(16 * (i >> 3) + (i & 7));
              s[kb] = mfma32(a, qf[0], s[kb]);
            }
          } else {
            s[kb] = mfma32(a, qf[j % (NS / 2)], s[kb]);
          }
          if (j % DMA_GAP == (DMA_GAP > 1 ? 1 : 0) && j / DMA_GAP < DMA_PER_STEP) dma.issue_one(rsrc, lds, j / DMA_GAP);
          if (!CAP && j == NS / 2) {
            exactly(0);
            tb[0] = base(0, m_run);
          }
          if (j > NS / 2) {
            constexpr int SLOTS = NS / 2 - 1;
            const int c0 = (j - NS / 2 - 1) * 8 / SLOTS, c1 = (j - NS / 2) * 8 / SLOTS;
#pragma unroll
            for (int c = c0; c < c1; ++c) {
              if constexpr (CAP) {
                squash(0, 2 * c);
                squash(0, 2 * c + 1);
              } else {
                expo(0, c);
                asm volatile("" : "+v"(pb[0][c >> 2][c & 3]), "+v"(lsum[0][c & 1]));
              }
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        u32x4 cring[PFC];
#pragma unroll
        for (int m = 0; m < PFC; ++m) {
          cring[m] = c_op(m);
          if (keep_off) cring[m] = finite_only(cring[m]);
        }
        if constexpr (CAP) {
          exactly(0);
          tb[0] = base(0, m_run);
#pragma unroll
          for (int c = 0; c < 8; ++c) expo(0, c);
        }
        block_done(0);
        if (!CAP) {
          exactly(1);
          tb[1] = base(1, m_run);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int m = 0; m < NP; ++m) {
          const u32x4 a = cring[m % PFC];
          if (m + PFC < NP) {
            u32x4 c = c_op(m + PFC);
            if (keep_off) c = finite_only(c);
            cring[m % PFC] = c;
          }
          if (m < NP / 2) {
#pragma unroll
            for (int c = m * 8 / (NP / 2); c < (m + 1) * 8 / (NP / 2); ++c) {
              if constexpr (CAP) {
                squash(1, 2 * c);
                squash(1, 2 * c + 1);
              } else {
                expo(1, c);
                asm volatile("" : "+v"(pb[1][c >> 2][c & 3]), "+v"(lsum[1][c & 1]));
              }
            }
          }
          if (m == NP / 2) {
            if constexpr (CAP) {
              exactly(1);
              tb[1] = base(1, m_run);
#pragma unroll
              for (int c = 0; c < 8; ++c) expo(1, c);
            }
            block_done(1);
          }
          const int kb = m / (NP / 2), db = (m % (NP / 2)) >> 1, s2 = m & 1;
          o[db] = mfma32(a, pb[kb][s2], o[db]);
          if ((m % (NP / 2)) % (NP / 4) == 1) racc = mfma16(rsel, pb[kb][(m % (NP / 2)) / (NP / 4)], racc);
          __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
      };

      // Two buffers in rotation: tile t+1 is fetched during tile t, half by half; a fetch past the
      // range has an empty resource and reads nothing.  Steps that the wave sees nothing of only
      // fetch, in a loop of their own: as a branch around the step they made the compiler move the
      // accumulators three times a step.
      if (ri > 0 || again) {
        __syncthreads();  // the last range's tiles are no longer read
        fetch(rg, first_key(k0), k1);
      }
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
        const bool keep_off = !ws.sees_all(rg.k_pos + kt, min(BN, k1 - kt)) && !all_finite<D>(vs + buf + half, lane);
        infinite |= keep_off;
        step(buf + half, kt, rsrc, lds, keep_off);
        advance();
      }
      wait_vmem();  // the lookahead loads must land before the LDS is used again
    }
    if constexpr (BIAS != kBiasSlope) break;
    if (again) break;
    const uint64_t low = __ballot(sees && xor32_sum(l_part) < 0x1p-64f);
    if (lane == 0) s_low[group][wave] = low;
    __syncthreads();
    bool any = false;
#pragma unroll
    for (int w = 0; w < NW; ++w) any |= (s_low[0][w] & s_low[NG - 1][w]) != 0;
    if (!any) break;
  }

  if constexpr (SPLIT) {
    // The second group's part through LDS.  A group without keys has a maximum that makes its
    // factor zero, both without any leave sums of zero.
    constexpr int NR = D / 32 * 4;
    static_assert((NR + 1) * NW * 64 * 16 <= NG * 2 * TILE, "the part must fit the K tiles");
    f32x4* x = reinterpret_cast<f32x4*>(k_lds) + wave * (NR + 1) * 64 + lane;
    __syncthreads();  // tiles no longer read
    if (group == 1) {
#pragma unroll
      for (int r = 0; r < NR; ++r)
        x[r * 64] = f32x4{o[r / 4][4 * (r % 4)], o[r / 4][4 * (r % 4) + 1], o[r / 4][4 * (r % 4) + 2], o[r / 4][4 * (r % 4) + 3]};
      x[NR * 64] = f32x4{m_run, l_part, racc[0], infinite ? 1.f : 0.f};
    }
    __syncthreads();
    if (group == 1) return;
    const f32x4 other = x[NR * 64];
    const float m_new = fmaxf(m_run, other[0]);
    const float a0 = fast_exp2(m_run - m_new), a1 = fast_exp2(other[0] - m_new);
    m_run = m_new;
    l_part = l_part * a0 + other[1] * a1;
    racc[0] = racc[0] * a0 + other[2] * a1;
    infinite |= __any(other[3] != 0.f);
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      const f32x4 y = x[r * 64];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[r / 4][4 * (r % 4) + e] = fmaf(o[r / 4][4 * (r % 4) + e], a0, y[e] * a1);
    }
  }

  // Where a mask runs through a step whose V holds infinities or NaN, the product took zeros in
  // their place, so that they do not reach rows that do not see them (0 * inf); the rows that do
  // get them here, from memory.  A weight that underflows makes no difference to an infinity.
  if (infinite) {
    for (int ri = 0; ri < it.range_count; ++ri) {
      ScoreRange rg = uniform(it.range);
      if (ri > 0) rg = uniform(p.ranges[it.range_next + ri - 1]);
      int k0, k1;
      visible(rg, k0, k1);
      for (int key = k0; key < k1; ++key) {
        const int at = rg.k_pos + (key & ~(BN - 1)), pos = rg.k_pos + key;
        if (at >= ws.hi_max || at + BN <= ws.lo_min || ws.sees_all(at, min(BN, k1 - (key & ~(BN - 1))))) continue;
        const bool seen = pos >= see.lo && pos < see.hi;
        const uint16_t* row = static_cast<const uint16_t*>(p.v) + ((int64_t)(rg.k_start + key) * Hk + kvh) * D + 8 * g;
#pragma unroll
        for (int db = 0; db < D / 32; ++db) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const u32x4 w = *reinterpret_cast<const u32x4*>(row + db * 32 + 16 * h);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              if (!not_finite(w[t]) || !seen) continue;
              const float lo = bf16_lo(w[t]), hi = bf16_hi(w[t]);
              if (lo - lo != 0.f) o[db][8 * h + 2 * t] += lo;
              if (hi - hi != 0.f) o[db][8 * h + 2 * t + 1] += hi;
            }
          }
        }
      }
    }
  }
  score_store<D>(kernargs<ScoreFwdParams>(), it, qr, q_ok, g, o, m_run, l_part, racc[0]);
}

template <int D, bool CAP, int BIAS>
hipError_t launch(const ScoreFwdParams& p, hipStream_t s) {
  const size_t lds = BIAS == kBiasTable ? score_bins(p.fn) * sizeof(float) : 0;
  ScoreFwdParams part = p;
  const hipError_t e = in_grids(p.n_split, 128 * NW, [&](int64_t first, dim3 grid) {
    part.items = p.items + first;
    hipLaunchKernelGGL((score_fwd_kernel<D, CAP, BIAS, true>), grid, dim3(128 * NW), lds, s, part);
  });
  if (e != hipSuccess) return e;
  return in_grids(p.n_items - p.n_split, 64 * NW, [&](int64_t first, dim3 grid) {
    part.items = p.items + p.n_split + first;
    hipLaunchKernelGGL((score_fwd_kernel<D, CAP, BIAS, false>), grid, dim3(64 * NW), lds, s, part);
  });
}

template <int D, bool CAP>
hipError_t launch_cap(const ScoreFwdParams& p, hipStream_t s) {
  if (p.fn.slope) return launch<D, CAP, kBiasSlope>(p, s);
  if (p.fn.bias) return launch<D, CAP, kBiasTable>(p, s);
  return launch<D, CAP, kBiasNone>(p, s);
}

template <int D>
hipError_t launch_d(const ScoreFwdParams& p, hipStream_t s) {
  return p.fn.cap_log2 != 0.f ? launch_cap<D, true>(p, s) : launch_cap<D, false>(p, s);
}

}  // namespace

hipError_t launch_score_fwd(const ScoreFwdParams& p, int head_dim, hipStream_t s) {
  if (p.n_items == 0) return hipSuccess;
  return head_dim == 128 ? launch_d<128>(p, s) : launch_d<64>(p, s);
}

}  // namespace zl
