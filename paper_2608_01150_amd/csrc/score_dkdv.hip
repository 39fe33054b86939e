// Scored attention: the dK/dV launch (score_dkdv.h).

#include "score_dkdv.h"

namespace zl {
namespace {

template <int D, bool CAP, int BIAS>
__global__ __launch_bounds__(dkdv::NT, 1) void score_dkdv_kernel(ScoreBwdParams p) {
  __shared__ dkdv::Lds<D> lds;
  extern __shared__ float tables[];
  dkdv::run<D, CAP, BIAS>(p, blockIdx.x, lds, tables);
}

template <int D, bool CAP, int BIAS>
hipError_t launch(const ScoreBwdParams& p, hipStream_t s) {
  const size_t lds = BIAS == kBiasTable ? 2 * score_bins(p.fn) * sizeof(float) : 0;
  ScoreBwdParams part = p;
  return in_grids(p.n_kv_items, dkdv::NT, [&](int64_t first, dim3 grid) {
    part.kv_items = p.kv_items + first;
    hipLaunchKernelGGL((score_dkdv_kernel<D, CAP, BIAS>), grid, dim3(dkdv::NT), lds, s, part);
  });
}

template <int D, bool CAP>
hipError_t launch_cap(const ScoreBwdParams& p, hipStream_t s) {
  if (p.fn.slope) return launch<D, CAP, kBiasSlope>(p, s);
  if (p.fn.bias) return launch<D, CAP, kBiasTable>(p, s);
  return launch<D, CAP, kBiasNone>(p, s);
}

template <int D>
hipError_t launch_d(const ScoreBwdParams& p, hipStream_t s) {
  return p.fn.cap_log2 != 0.f ? launch_cap<D, true>(p, s) : launch_cap<D, false>(p, s);
}

}  // namespace

hipError_t launch_score_dkdv(const ScoreBwdParams& p, int head_dim, hipStream_t s) {
  if (p.n_kv_items == 0) return hipSuccess;
  return head_dim == 128 ? launch_d<128>(p, s) : launch_d<64>(p, s);
}

}  // namespace zl
