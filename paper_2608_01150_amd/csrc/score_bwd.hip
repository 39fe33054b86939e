// Scored attention backward: the kernels around dK/dV (score_dkdv.hip) and dQ
// (score_dq.hip).  No atomics on memory; every sum has a fixed order.

#include "zl_score_device.h"

namespace zl {
namespace {

constexpr int NT = 256;

// -D_i = -dO_i . O_i and LSE_i in log2 units, less the cap's constant, fp32 per (row,
// head).  HBM-bound: reads O and dO once.  The workgroups behind those, a wave per 64-row
// tile, write what its rows see, each (first position and how many) and together.
template <int D>
__global__ __launch_bounds__(NT) void score_pre_kernel(ScoreBwdParams p, int64_t first, int64_t unit_blocks) {
  const int64_t block = first + blockIdx.x;
  if (block >= unit_blocks) {
    const int64_t t = (block - unit_blocks) * (NT / 64) + (int)threadIdx.x / 64;
    const int lane = threadIdx.x & 63;
    if (t >= p.n_tiles) return;
    const ScoreTile tile = p.tiles[t];
    int lo = INT32_MAX, hi = 0;
    if (lane < tile.rows) {
      const RowSee see = row_see(p.fn, tile.row + lane, tile.pos + lane);
      p.row_lo[tile.row + lane] = see.lo;
      p.row_len[tile.row + lane] = see.hi - see.lo;
      if (see.lo < see.hi) {
        lo = see.lo;
        hi = see.hi;
      }
    }
#pragma unroll
    for (int m = 32; m; m >>= 1) {
      lo = min(lo, __shfl_xor(lo, m));
      hi = max(hi, __shfl_xor(hi, m));
    }
    if (lane == 0) p.tile_see[t] = int2{lo, hi};
    return;
  }
  constexpr int LPU = D / 8;  // lanes per (row, head), 8 bf16 each
  const int sub = threadIdx.x % LPU;
  const int64_t u = block * (NT / LPU) + threadIdx.x / LPU;
  const bool live = u < p.total_q * p.num_heads;
  float acc = 0.f;
  if (live) {
    const u32x4 a =
        __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p.out) + u * D + sub * 8));
    const u32x4 b = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p.dout) + u * D + sub * 8);
#pragma unroll
    for (int t = 0; t < 4; ++t) acc += bf16_lo(a[t]) * bf16_lo(b[t]) + bf16_hi(a[t]) * bf16_hi(b[t]);
  }
  acc = lanes_sum<LPU>(acc);
  if (live && sub == 0) {
    const float lse = p.lse[u];
    p.dsum[u] = -acc;
    // a row that sees nothing has weights of zero; one whose LSE or dO . O is no number has no
    // gradient that is one
    p.lse2[u] = lse == -INFINITY                          ? kScoreNoKey
                : acc - acc == 0.f && lse - lse == 0.f ? fmaf(lse, 1.4426950408889634f, -p.fn.cap_log2)
                                                       : kScoreNoGrad;
  }
}

// dK (blockIdx.y 0) or dV of a key tile whose items took some heads each: their partials
// added in order, rounded once.
template <int D>
__global__ __launch_bounds__(NT) void score_sum_kernel(ScoreBwdParams p) {
  const ScoreSum it = p.sums[blockIdx.x];
  const int Hk = p.num_heads / p.group;
  constexpr int64_t kPart = 2 * kScoreKvTileN * D;
  const float* from = p.kv_part + it.part * kPart + (int64_t)blockIdx.y * kScoreKvTileN * D;
  uint16_t* to = static_cast<uint16_t*>(blockIdx.y ? p.dv : p.dk);
  for (int i = threadIdx.x; i < it.k_len * (D / 8); i += NT) {
    const int row = i / (D / 8), c = i % (D / 8) * 8;
    f32x4 a = {0.f, 0.f, 0.f, 0.f}, b = a;
    for (int x = 0; x < it.parts; ++x) {
      const f32x4* at = reinterpret_cast<const f32x4*>(from + x * kPart + row * D + c);
      a += at[0];
      b += at[1];
    }
    *reinterpret_cast<u32x4*>(to + ((int64_t)(it.k_start + row) * Hk + it.kv_head) * D + c) =
        u32x4{pack_bf16(a[0], a[1]), pack_bf16(a[2], a[3]), pack_bf16(b[0], b[1]), pack_bf16(b[2], b[3])};
  }
}

// The bias table's gradient, one workgroup per head.  Eight threads per relative
// position add every eighth item's sums, the eight are added in order, and a wave adds
// the positions of a bucket: every 64th per lane, then a butterfly.
constexpr int NTB = 1024;
__global__ __launch_bounds__(NTB) void score_dbias_kernel(ScoreBwdParams p) {
  constexpr int N = 2 * kScoreMaxReach + 1;
  __shared__ float sums[8][N];
  __shared__ int16_t of[N];
  const int head = blockIdx.x, n = 2 * p.fn.reach + 1;
  const int first = p.head_first[head], last = p.head_first[head + 1];
  const int sub = threadIdx.x / (NTB / 8);
  for (int i = threadIdx.x % (NTB / 8); i < n; i += NTB / 8) {
    float x = 0.f;
    for (int j = first + sub; j < last; j += 8) x += p.dbias_part[(int64_t)j * n + i];
    sums[sub][i] = x;
    if (sub == 0) of[i] = p.fn.bucket[i];
  }
  __syncthreads();
  const int lane = threadIdx.x & 63;
  for (int b = threadIdx.x >> 6; b < p.fn.n_buckets; b += NTB / 64) {
    float x = 0.f;
    for (int i = lane; i < n; i += 64) {
      if (of[i] != b) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) x += sums[e][i];
    }
#pragma unroll
    for (int m = 32; m; m >>= 1) x += __shfl_xor(x, m);
    if (lane) continue;
    const int64_t at = (int64_t)b * p.num_heads + head;
    if (p.fn.bias_bf16) static_cast<uint16_t*>(p.dbias)[at] = (uint16_t)pack_bf16(x, 0.f);
    else static_cast<float*>(p.dbias)[at] = x;
  }
}

}  // namespace

hipError_t launch_score_pre(const ScoreBwdParams& p, int head_dim, hipStream_t s) {
  const int64_t units = p.total_q * p.num_heads;
  if (units == 0) return hipSuccess;
  const int upb = NT / (head_dim / 8);
  const int64_t unit_blocks = (units + upb - 1) / upb;
  return in_grids(unit_blocks + (p.n_tiles + NT / 64 - 1) / (NT / 64), NT, [&](int64_t first, dim3 grid) {
    if (head_dim == 128) hipLaunchKernelGGL(score_pre_kernel<128>, grid, dim3(NT), 0, s, p, first, unit_blocks);
    else hipLaunchKernelGGL(score_pre_kernel<64>, grid, dim3(NT), 0, s, p, first, unit_blocks);
  });
}

hipError_t launch_score_sum(const ScoreBwdParams& p, int head_dim, hipStream_t s) {
  ScoreBwdParams part = p;
  return in_grids(p.n_sums, NT, [&](int64_t first, dim3 grid) {
    part.sums = p.sums + first;
    grid.y = 2;
    if (head_dim == 128) hipLaunchKernelGGL(score_sum_kernel<128>, grid, dim3(NT), 0, s, part);
    else hipLaunchKernelGGL(score_sum_kernel<64>, grid, dim3(NT), 0, s, part);
  });
}

hipError_t launch_score_dbias(const ScoreBwdParams& p, hipStream_t s) {
  hipLaunchKernelGGL(score_dbias_kernel, dim3(p.num_heads), dim3(NTB), 0, s, p);
  return hipGetLastError();
}

}  // namespace zl
