// Scored attention: dQ and dK/dV in one launch, for calls whose items do not fill the chip
// in two.  The dQ items come first, the dK/dV items behind them; a workgroup has the eight
// waves of a dK/dV item, of which a dQ item that no two groups share uses four.  One
// workgroup per CU, so it pays where the items of both come to at most two per CU
// (one_launch in zl_host.cpp): 226 rows of 905 keys, 8 heads of 128, 74 -> 52 us with the
// forward; 1001 causal rows of 3003 keys, 12 heads of 64, capped, 127 -> 93.  With the table's
// gradient, dQ and dK/dV alone: 2 x 512 tokens, 12 heads, d = 64, 53 -> 31 us, 4 x 512 58 -> 52.
// With d = 128 its dQ takes some 370 registers when launched apart, with four waves a CU, and has
// 256 here (80 spilled), so this pays in one round only: 192 items (2 x 512 tokens, 12 heads)
// 65 -> 54 us, capped 72 -> 72, but 384 (4 x 512) 69 -> 78, capped 77 -> 91, and 512 (2 x 1024, 16
// heads) 106 -> 127, capped 120 -> 160.  Results are those of two launches.

#include "score_dkdv.h"
#include "score_dq.h"

namespace zl {
namespace {

constexpr size_t larger(size_t a, size_t b) { return a > b ? a : b; }

template <int D, bool TABLE_GRAD>
constexpr size_t kLds = larger(larger(sizeof(dkdv::Lds<D>), sizeof(dq::Lds<D, TABLE_GRAD, false>)),
                               TABLE_GRAD ? 0 : sizeof(dq::Lds<D, false, true>));

size_t tables_lds(const ScoreBwdParams& p) { return p.fn.bias ? 2 * score_bins(p.fn) * sizeof(float) : 0; }

template <int D, bool CAP, int BIAS, bool TABLE_GRAD>
__global__ __launch_bounds__(dkdv::NT, 2) void score_both_kernel(ScoreBwdParams p) {
  using Keys = dkdv::Lds<D>;
  using Shared = dq::Lds<D, false, true>;
  using Rows = dq::Lds<D, TABLE_GRAD, false>;
  static_assert(dkdv::NT == 128 * dq::NW, "a workgroup runs any of the three");
  __shared__ __attribute__((aligned(16))) char lds[kLds<D, TABLE_GRAD>];
  extern __shared__ float tables[];
  const int b = blockIdx.x;
  if (b >= p.n_q_items) {
    dkdv::run<D, CAP, BIAS>(p, b - p.n_q_items, *reinterpret_cast<Keys*>(lds), tables);
    return;
  }
  if constexpr (!TABLE_GRAD) {
    if (b < p.n_split) {
      dq::run<D, CAP, BIAS, false, true>(p, b, *reinterpret_cast<Shared*>(lds), tables);
      return;
    }
  }
  // waves that have ended take no part in barriers
  if (threadIdx.x < 64 * dq::NW) dq::run<D, CAP, BIAS, TABLE_GRAD, false>(p, b, *reinterpret_cast<Rows*>(lds), tables);
}

template <int D, bool CAP, int BIAS, bool TABLE_GRAD>
hipError_t launch(const ScoreBwdParams& p, hipStream_t s) {
  hipLaunchKernelGGL((score_both_kernel<D, CAP, BIAS, TABLE_GRAD>), dim3(p.n_q_items + p.n_kv_items), dim3(dkdv::NT),
                     tables_lds(p), s, p);
  return hipGetLastError();
}

template <int D, bool CAP>
hipError_t launch_cap(const ScoreBwdParams& p, hipStream_t s) {
  if (p.fn.slope) return launch<D, CAP, kBiasSlope, false>(p, s);
  if (p.dbias) return launch<D, CAP, kBiasTable, true>(p, s);
  if (p.fn.bias) return launch<D, CAP, kBiasTable, false>(p, s);
  return launch<D, CAP, kBiasNone, false>(p, s);
}

template <int D>
hipError_t launch_d(const ScoreBwdParams& p, hipStream_t s) {
  return p.fn.cap_log2 != 0.f ? launch_cap<D, true>(p, s) : launch_cap<D, false>(p, s);
}

}  // namespace

bool score_both_fits(const ScoreBwdParams& p, int head_dim) {
  const size_t lds = head_dim == 128 ? p.dbias ? kLds<128, true> : kLds<128, false> : p.dbias ? kLds<64, true> : kLds<64, false>;
  return lds + tables_lds(p) <= 160 * 1024;
}

hipError_t launch_score_both(const ScoreBwdParams& p, int head_dim, hipStream_t s) {
  return head_dim == 128 ? launch_d<128>(p, s) : launch_d<64>(p, s);
}

}  // namespace zl
