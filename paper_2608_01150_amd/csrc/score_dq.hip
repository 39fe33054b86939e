// Scored attention: the dQ launch (score_dq.h).

#include "score_dq.h"

namespace zl {
namespace {

template <int D, bool CAP, int BIAS, bool TABLE_GRAD, bool SPLIT>
__global__ __launch_bounds__(SPLIT ? 128 * dq::NW : 64 * dq::NW, 2) void score_dq_kernel(ScoreBwdParams p) {
  __shared__ dq::Lds<D, TABLE_GRAD, SPLIT> lds;
  extern __shared__ float table[];
  dq::run<D, CAP, BIAS, TABLE_GRAD, SPLIT>(p, blockIdx.x, lds, table);
}

template <int D, bool CAP, int BIAS, bool TABLE_GRAD>
hipError_t launch(const ScoreBwdParams& p, hipStream_t s) {
  const size_t lds = BIAS == kBiasTable ? score_bins(p.fn) * sizeof(float) : 0;
  ScoreBwdParams part = p;
  if constexpr (!TABLE_GRAD) {
    const hipError_t e = in_grids(p.n_split, 128 * dq::NW, [&](int64_t first, dim3 grid) {
      part.q_items = p.q_items + first;
      hipLaunchKernelGGL((score_dq_kernel<D, CAP, BIAS, false, true>), grid, dim3(128 * dq::NW), lds, s, part);
    });
    if (e != hipSuccess) return e;
  }
  return in_grids(p.n_q_items - p.n_split, 64 * dq::NW, [&](int64_t first, dim3 grid) {
    part.q_items = p.q_items + p.n_split + first;
    hipLaunchKernelGGL((score_dq_kernel<D, CAP, BIAS, TABLE_GRAD, false>), grid, dim3(64 * dq::NW), lds, s, part);
  });
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

hipError_t launch_score_dq(const ScoreBwdParams& p, int head_dim, hipStream_t s) {
  if (p.n_q_items == 0) return hipSuccess;
  return head_dim == 128 ? launch_d<128>(p, s) : launch_d<64>(p, s);
}

}  // namespace zl
