// Scored attention forward of few rows (single tokens against a cache), gfx950.
//
// With few rows the K/V stream is everything: the work is divided along the keys.  An
// item is up to 32 rows of one K/V head (a row: a query token and one of the heads that
// share the K/V head, so K and V are read once for the group) against up to a chunk of
// keys; each of its four waves takes every fourth tile of 64 keys, on its own: K comes
// straight to registers as the A operand of S^T = K Q^T, V by direct loads to the
// wave's own LDS for the transpose reads of O^T += V^T P^T, and nothing waits for
// another wave until the end.  There the waves' sums are joined, and score_join_kernel
// joins the items of a row.  Keys past the last one that a row sees (the unfilled part
// of a cache) are not read.
//
// P is rounded to bf16 where it meets V, as in score_fwd.hip, and the row divided by the sum
// of the rounded weights; all else is fp32.
//
// Bound by HBM where there are many items, by the latency of two launches and one
// tile's loads where there are few.  The chunk goes by the segment's own key count
// (score_chunk in zl_host.cpp), so a segment's results do not depend on the batch.

#include "zl_score_device.h"

namespace zl {
namespace {

constexpr int NW = 4;             // waves per workgroup
constexpr int NT = 64 * NW;
constexpr int BN = 64;            // keys per tile

// Eight values of a row: the final output (slot < 0), or a block's partial.
template <int D>
__device__ __forceinline__ void few_store(const ScoreFewParams& p, int64_t row, int c, int slot, const float (&x)[8], float lse) {
  if (slot < 0) {
    const u32x4 w = {pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
    *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p.out) + row * D + c) = w;
    if (c == 0) p.lse[row] = lse;
  } else {
    float* og = p.o_part + slot * p.slot_stride + row * D + c;
    *reinterpret_cast<f32x4*>(og) = f32x4{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4*>(og + 4) = f32x4{x[4], x[5], x[6], x[7]};
    if (c == 0) p.lse_part[slot * p.lse_slot_stride + row] = lse;
  }
}

template <int D, bool CAP, int BIAS>
__global__ __launch_bounds__(NT, 2) void score_few_kernel(ScoreFewParams p) {
  constexpr int PITCH = Pad<D>::PITCH;
  constexpr int TILE = BN * PITCH;
  constexpr int OPITCH = D + 4;   // floats between the rows of a wave's result, in its V tile
  static_assert(32 * OPITCH * 4 <= TILE, "a wave's result fits its V tile");
  using Dma = TileDma<D, BN, 1>;
  __shared__ __attribute__((aligned(16))) char vs[NW][TILE];
  __shared__ float s_m[NW][32], s_l[NW][32], s_r[NW][32];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int ln = lane & 31, g = lane >> 5;
  const ScoreFewItem it = p.items[blockIdx.x];
  const int H = p.num_heads, G = p.group, Hk = H / G;
  const int64_t rs = (int64_t)Hk * D;
  const float coef = CAP ? -2.f * p.fn.cap_log2 : p.fn.scale_log2;
  const float capc = CAP ? p.fn.cap_log2 : 0.f;

  const bool q_ok = ln < it.rows;
  const int m = it.row0 + ln, r = m / G, head = it.kv_head * G + m % G;
  RowSee see{0, 0, 0};
  u32x4 qf[D / 16];
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) qf[kk] = u32x4{0, 0, 0, 0};
  float slope2 = 0.f, far_lo = 0.f, far_hi = 0.f;
  if (q_ok) {
    see = row_see(p.fn, it.q_start + r, it.q_pos + r);
    const uint16_t* qg = static_cast<const uint16_t*>(p.q) + ((int64_t)(it.q_start + r) * H + head) * D;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) qf[kk] = *reinterpret_cast<const u32x4*>(qg + kk * 16 + g * 8);
    if constexpr (BIAS == kBiasSlope) slope2 = p.fn.slope[head] * 1.4426950408889634f;
    if constexpr (BIAS == kBiasTable) {
      far_lo = bias_at(p.fn, -p.fn.reach, head, H) * 1.4426950408889634f;
      far_hi = bias_at(p.fn, p.fn.reach, head, H) * 1.4426950408889634f;
    }
  }
  const WaveSee ws = wave_see(see, q_ok);
  const int k1 = min(it.k_len, max(ws.hi_max - it.k_pos, 0)), k0 = max(ws.lo_min - it.k_pos, 0) & ~(BN - 1);

  float m_run = kNegBig, l = 0.f, lr = 0.f;
  f32x16 o[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db) o[db] = f32x16{};
  const uint16_t* kg = static_cast<const uint16_t*>(p.k) + ((int64_t)it.k_start * Hk + it.kv_head) * D + g * 8;
  const uint16_t* vg = static_cast<const uint16_t*>(p.v) + ((int64_t)it.k_start * Hk + it.kv_head) * D;
  Dma dma;
  dma.init(0, lane, (uint32_t)rs * 2u);
  const char* vt = vs[wave] + tr_lane_off<D>(lane);

  for (int kt = k0 + wave * BN; kt < k1; kt += NW * BN) {
    const int kp = it.k_pos + kt, nvalid = k1 - kt;
    dma.issue(vs[wave], vg + (int64_t)kt * rs, nvalid, (uint32_t)rs * 2u);
    u32x4 kf[2][D / 16];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const uint16_t* kr = kg + (int64_t)(kt + min(32 * kb + perm32(ln), nvalid - 1)) * rs;
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) kf[kb][kk] = *reinterpret_cast<const u32x4*>(kr + kk * 16);
    }
    // Loads land in the order of their issue: with K in registers, V is in the LDS.
    __builtin_amdgcn_s_waitcnt(0);
    wait_vmem();
    const bool masked = !ws.sees_all(kp, min(BN, nvalid));
    const bool keep_off = masked && !all_finite<D>(vs[wave], lane);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      if (32 * kb >= nvalid) break;
      f32x16 s = f32x16{};
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) s = mfma32(kf[kb][kk], qf[kk], s);
      const int b0 = kp + 32 * kb;
      bool special = masked || nvalid < 32 * kb + 32;
      float sl = 0.f, base = capc;
      if constexpr (BIAS == kBiasSlope) {
        const bool behind = b0 >= ws.pos_max;
        special |= !behind && b0 + 31 > ws.pos_min;
        sl = behind ? -slope2 : slope2;
        base = fmaf(-sl, (float)(see.pos - b0 - 8 * g), capc);
      }
      if constexpr (BIAS == kBiasTable) {
        const bool behind = b0 - ws.pos_max >= p.fn.reach;
        special |= !behind && b0 + 31 - ws.pos_min > -p.fn.reach;
        base += behind ? far_hi : far_lo;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if constexpr (CAP) s[i] = __builtin_amdgcn_rcpf(1.f + fast_exp2(s[i] * p.fn.cap_in));
      }
      if (special) {
        const int f0 = b0 + 8 * g, end = min(see.hi, kp + nvalid);
        const uint32_t len = (uint32_t)max(end - see.lo, 0);
        float bias[16];
        if constexpr (BIAS == kBiasTable) bias_of_block(bias, p.fn, f0 - see.pos, head, H);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int pos = f0 + 16 * (i >> 3) + (i & 7);
          float a = fmaf(s[i], coef, capc);
          if constexpr (BIAS == kBiasSlope) a = fmaf(-slope2, fabsf((float)(pos - see.pos)), a);
          if constexpr (BIAS == kBiasTable) a = fmaf(bias[i], 1.4426950408889634f, a);
          s[i] = (uint32_t)(pos - see.lo) < len ? a : -INFINITY;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float t = BIAS == kBiasSlope ? fmaf(sl, (float)(16 * (i >> 3) + (i & 7)), base) : base;
          s[i] = fmaf(s[i], coef, t);
        }
      }
      float mt = s[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) mt = fmaxf(mt, s[i]);
      const float m_new = fmaxf(m_run, xor32_max(mt));
      if (__any(m_new > m_run)) {
        const float alpha = fast_exp2(m_run - m_new);
        m_run = m_new;
        l *= alpha;
        lr *= alpha;
#pragma unroll
        for (int db = 0; db < D / 32; ++db) {
#pragma unroll
          for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
        }
      }
      u32x4 pb[2];
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const float e0 = fast_exp2(s[2 * c] - m_run), e1 = fast_exp2(s[2 * c + 1] - m_run);
        const uint32_t w = pack_bf16(e0, e1);
        l += e0 + e1;
        lr += bf16_lo(w) + bf16_hi(w);
        pb[c >> 2][c & 3] = w;
      }
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const u32x4 a = tr_operand<D>(vt, 32 * kb + 16 * h, db * 32);
          if (keep_off) mfma32_masked(a, pb[h], o[db]);
          else o[db] = mfma32(a, pb[h], o[db]);
        }
      }
    }
    // The tile's transpose reads end before the next tile's loads may write over it.
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }

  // The waves' sums, each in its own V tile, joined row by row.
  float* const ow = reinterpret_cast<float*>(vs[wave]);
  if (g == 0) s_m[wave][ln] = m_run;
  const float lw = xor32_sum(l), rw = xor32_sum(lr);
  if (g == 0) {
    s_l[wave][ln] = lw;
    s_r[wave][ln] = rw;
  }
#pragma unroll
  for (int db = 0; db < D / 32; ++db) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float* at = ow + ln * OPITCH + db * 32 + 16 * h + 8 * g;
      *reinterpret_cast<f32x4*>(at) = f32x4{o[db][8 * h], o[db][8 * h + 1], o[db][8 * h + 2], o[db][8 * h + 3]};
      *reinterpret_cast<f32x4*>(at + 4) = f32x4{o[db][8 * h + 4], o[db][8 * h + 5], o[db][8 * h + 6], o[db][8 * h + 7]};
    }
  }
  __syncthreads();
  constexpr int TPR = D / 8;      // threads per row, 8 values each
  for (int row = tid / TPR; row < it.rows; row += NT / TPR) {
    const int c = tid % TPR * 8;
    float top = kNegBig, sum = 0.f, rsum = 0.f, x[8] = {};
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, s_m[w][row]);
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = fast_exp2(s_m[w][row] - top);
      sum += f * s_l[w][row];
      rsum += f * s_r[w][row];
      const float* at = reinterpret_cast<const float*>(vs[w]) + row * OPITCH + c;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = fmaf(f, at[e], x[e]);
    }
    const float inv = sum != sum ? sum : rsum == 0.f ? 0.f : 1.f / rsum;
    const float lse = sum == 0.f ? -INFINITY : (top + __log2f(sum)) * kLn2;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = sum == 0.f ? 0.f : x[e] * inv;  // weights of zero alone: whatever they met in V
    if (it.part >= 0) {
      if (sum != 0.f) {  // a chunk that the row sees nothing of is left out by the join
        float* og = p.part_o + (int64_t)(it.part + row) * D + c;
        *reinterpret_cast<f32x4*>(og) = f32x4{x[0], x[1], x[2], x[3]};
        *reinterpret_cast<f32x4*>(og + 4) = f32x4{x[4], x[5], x[6], x[7]};
      }
      if (c == 0) p.part_lse[it.part + row] = lse;
    } else {
      const int mm = it.row0 + row;
      few_store<D>(p, (int64_t)(it.q_start + mm / G) * H + it.kv_head * G + mm % G, c, it.slot, x, lse);
    }
  }
}

// Rows of items over several chunks: O = sum_c exp(LSE_c - LSE) O_c, as zl_lse_merge.  D/8
// lanes per row and slice: with fewer rows than a workgroup has room for, each slice takes
// every so many'th chunk, four at a time, and the slices are joined in their order.  A chunk
// that the row sees nothing of has LSE_c = -inf and no O_c.  Latency: 48 tokens of 32 heads
// of 128 over 16 chunks 9 -> 6 us by slices.
template <int D>
__global__ __launch_bounds__(NT) void score_join_kernel(ScoreFewParams p) {
  constexpr int TPR = D / 8, UNITS = NT / TPR, U = 4;
  __shared__ float s_x[UNITS][D + 4], s_top[UNITS], s_sum[UNITS];
  const ScoreJoin it = p.joins[blockIdx.x];
  const int c = threadIdx.x % TPR * 8, unit = threadIdx.x / TPR;
  const int rows = min(it.rows, UNITS), slices = UNITS / rows, slice = unit / rows;
  for (int row0 = 0; row0 < it.rows; row0 += rows) {
    const int row = row0 + unit % rows;
    const bool on = row < it.rows && slice < slices;
    float top = -INFINITY, sum = 0.f, x[8] = {};
    for (int i0 = slice; on && i0 < it.parts; i0 += U * slices) {
      float z[U];
      f32x4 a[U], b[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int at = it.part + min(i0 + u * slices, it.parts - 1) * it.rows + row;
        z[u] = i0 + u * slices < it.parts ? p.part_lse[at] * 1.4426950408889634f : -INFINITY;
        a[u] = *reinterpret_cast<const f32x4*>(p.part_o + (int64_t)at * D + c);
        b[u] = *reinterpret_cast<const f32x4*>(p.part_o + (int64_t)at * D + c + 4);
      }
      float top1 = top;
#pragma unroll
      for (int u = 0; u < U; ++u) top1 = fmaxf(top1, z[u]);
      if (top1 != top) {
        const float f = fast_exp2(top - top1);
        sum *= f;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= f;
        top = top1;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool part = z[u] != -INFINITY;
        const float w = part ? fast_exp2(z[u] - top) : 0.f;
        sum += w;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] = fmaf(w, part ? a[u][e] : 0.f, x[e]);
          x[4 + e] = fmaf(w, part ? b[u][e] : 0.f, x[4 + e]);
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) s_x[unit][c + e] = x[e];
    if (c == 0) {
      s_top[unit] = top;
      s_sum[unit] = sum;
    }
    __syncthreads();
    if (on && slice == 0) {
      for (int k = 1; k < slices; ++k) top = fmaxf(top, s_top[unit + k * rows]);
      float all = 0.f, y[8] = {};
      for (int k = 0; k < slices; ++k) {
        const int at = unit + k * rows;
        const float f = s_sum[at] == 0.f ? 0.f : fast_exp2(s_top[at] - top);
        all = fmaf(f, s_sum[at], all);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = fmaf(f, s_x[at][c + e], y[e]);
      }
      const float inv = all != all ? all : all == 0.f ? 0.f : 1.f / all;
      const float lse = all == 0.f ? -INFINITY : (top + __log2f(all)) * kLn2;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] *= inv;
      const int mm = it.row0 + row, G = p.group;
      few_store<D>(p, (int64_t)(it.q_start + mm / G) * p.num_heads + it.kv_head * G + mm % G, c, it.slot, y, lse);
    }
    __syncthreads();
  }
}

template <int D, bool CAP, int BIAS>
hipError_t launch(const ScoreFewParams& p, hipStream_t s) {
  ScoreFewParams part = p;
  return in_grids(p.n_items, NT, [&](int64_t first, dim3 grid) {
    part.items = p.items + first;
    hipLaunchKernelGGL((score_few_kernel<D, CAP, BIAS>), grid, dim3(NT), 0, s, part);
  });
}

template <int D, bool CAP>
hipError_t launch_cap(const ScoreFewParams& p, hipStream_t s) {
  if (p.fn.slope) return launch<D, CAP, kBiasSlope>(p, s);
  if (p.fn.bias) return launch<D, CAP, kBiasTable>(p, s);
  return launch<D, CAP, kBiasNone>(p, s);
}

template <int D>
hipError_t launch_d(const ScoreFewParams& p, hipStream_t s) {
  const hipError_t e = p.fn.cap_log2 != 0.f ? launch_cap<D, true>(p, s) : launch_cap<D, false>(p, s);
  if (e != hipSuccess) return e;
  ScoreFewParams part = p;
  return in_grids(p.n_joins, NT, [&](int64_t first, dim3 grid) {
    part.joins = p.joins + first;
    hipLaunchKernelGGL(score_join_kernel<D>, grid, dim3(NT), 0, s, part);
  });
}

}  // namespace

hipError_t launch_score_few(const ScoreFewParams& p, int head_dim, hipStream_t s) {
  if (p.n_items == 0) return hipSuccess;
  return head_dim == 128 ? launch_d<128>(p, s) : launch_d<64>(p, s);
}

}  // namespace zl
