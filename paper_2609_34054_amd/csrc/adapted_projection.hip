// Projection of hidden states with the low-rank adapter of each row's agent
// (Eq. 1 for many agents at once):
//     Y[i] = X[i] W + (X[i] A_a) B_a,   a = agent[i]   (no such agent: X[i] W)
// in bf16, or with X and W in e4m3 (X = x_scale[i] X8, W = w_scale[j] W8).
// The rank-r rows X A_a are formed first (fp32 sums, then bf16, as the LR
// caches hold them) and added, expanded by B_a, as Y is written.
#include "common.hpp"
#include "kernels.hpp"

namespace prc {
namespace {

__device__ __forceinline__ u32x2 lds_read_tr(const uint16_t* p) {
  typedef short v4s __attribute__((ext_vector_type(4)));
  v4s v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((v4s __attribute__((address_space(3)))*)(p));
  return __builtin_bit_cast(u32x2, v);
}

// Eight e4m3 values as bf16 (exact).
__device__ __forceinline__ u32x4 bf16_of_e4m3(u32x2 v) {
  u32x4 o;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[h], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[h], true);
    o[2 * h] = pack_bf16(lo[0], lo[1]);
    o[2 * h + 1] = pack_bf16(hi[0], hi[1]);
  }
  return o;
}

// Eight consecutive elements of X or W as bf16, or zeros.
template <bool FP8>
__device__ __forceinline__ u32x4 load8(const void* p, int64_t i, bool ok) {
  if constexpr (FP8) {
    const u32x2 z = {0u, 0u};
    return bf16_of_e4m3(ok ? *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(p) + i) : z);
  } else {
    return ld16(static_cast<const uint16_t*>(p) + i, ok);
  }
}

// H[i] = X[i] A_a (times x_scale[i]): a workgroup per row.
template <bool FP8, int R>
__global__ void __launch_bounds__(256) shrink_kernel(const ProjectArgs a) {
  __shared__ float part[4][R];
  const int64_t row = blockIdx.x;
  const int ag = a.agent[row];
  if (ag < 0 || ag >= a.n_agents) return;  // uniform over the workgroup
  const int tid = threadIdx.x;
  const int64_t ldA = (int64_t)a.n_agents * R;
  float acc[R];
#pragma unroll
  for (int j = 0; j < R; ++j) acc[j] = 0.f;
  for (int64_t k = tid * 8; k < a.d_in; k += 2048) {
    const u32x4 xv = load8<FP8>(a.X, row * a.ld_x + k, true);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = i % 2 ? bf_hi(xv[i / 2]) : bf_lo(xv[i / 2]);
      const uint16_t* ap = a.A + (k + i) * ldA + (int64_t)ag * R;
#pragma unroll
      for (int j = 0; j < R; j += 8) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(ap + j);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          acc[j + 2 * e] += x * bf_lo(w[e]);
          acc[j + 2 * e + 1] += x * bf_hi(w[e]);
        }
      }
    }
  }
#pragma unroll
  for (int j = 0; j < R; ++j) {
#pragma unroll
    for (int m = 1; m < 64; m *= 2) acc[j] += shfl_xor(acc[j], m);
    if (tid % 64 == 0) part[tid / 64][j] = acc[j];
  }
  __syncthreads();
  if (tid < R) {
    float v = part[0][tid] + part[1][tid] + part[2][tid] + part[3][tid];
    if (FP8) v *= a.x_scale[row];
    static_cast<uint16_t*>(a.ws)[row * R + tid] = (uint16_t)(pack_bf16(v, 0.f) & 0xffffu);
  }
}

// 64 tokens x 64 columns a workgroup, 32 k a step; wave w owns 16 columns.
template <bool FP8>
__global__ void __launch_bounds__(256) project_kernel(const ProjectArgs a) {
  __shared__ __attribute__((aligned(16))) uint16_t xt[64][40], wt[32][72];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, q = lane >> 4, c16 = lane & 15;
  const int64_t t0 = (int64_t)blockIdx.y * 64, c0 = (int64_t)blockIdx.x * 64;
  f32x4 acc[4] = {};
  const int xr = tid / 4, xk = tid % 4 * 8, wr = tid / 8, wc = tid % 8 * 8;
  for (int64_t k0 = 0; k0 < a.d_in; k0 += 32) {
    const u32x4 xv = load8<FP8>(a.X, (t0 + xr) * a.ld_x + k0 + xk, t0 + xr < a.T && k0 + xk < a.d_in);
    const u32x4 wv = load8<FP8>(a.W, (k0 + wr) * a.d_out + c0 + wc, k0 + wr < a.d_in && c0 + wc < a.d_out);
    __syncthreads();
    *reinterpret_cast<u32x4*>(&xt[xr][xk]) = xv;
    *reinterpret_cast<u32x4*>(&wt[wr][wc]) = wv;
    __syncthreads();
    const u32x2 lo = lds_read_tr(&wt[8 * q + c16 / 4][16 * w + 4 * (c16 % 4)]);
    const u32x2 hi = lds_read_tr(&wt[8 * q + 4 + c16 / 4][16 * w + 4 * (c16 % 4)]);
#pragma unroll
    for (int m = 0; m < 4; ++m)
      acc[m] = mfma16x16x32(as_bf16x8(u32x4{lo[0], lo[1], hi[0], hi[1]}),
                            as_bf16x8(*reinterpret_cast<const u32x4*>(&xt[16 * m + c16][8 * q])), acc[m]);
  }
  const int64_t c = c0 + 16 * w + 4 * q;  // this lane's four columns
  if (c >= a.d_out) return;
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    const int64_t t = t0 + 16 * m + c16;
    if (t >= a.T) continue;
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = FP8 ? acc[m][i] * (a.x_scale[t] * a.w_scale[c + i]) : acc[m][i];
    const int ag = a.n_agents > 0 ? a.agent[t] : -1;
    if (ag >= 0 && ag < a.n_agents) {
      const uint16_t* h = static_cast<const uint16_t*>(a.ws) + t * a.rank;
      for (int j = 0; j < a.rank; ++j) {
        const float hj = bf_lo(h[j]);
        const u32x2 b = *reinterpret_cast<const u32x2*>(a.B + ((int64_t)ag * a.rank + j) * a.d_out + c);
        v[0] += hj * bf_lo(b[0]);
        v[1] += hj * bf_hi(b[0]);
        v[2] += hj * bf_lo(b[1]);
        v[3] += hj * bf_hi(b[1]);
      }
    }
    *reinterpret_cast<u32x2*>(a.Y + t * a.ld_y + c) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
  }
}

template <bool FP8>
hipError_t launch(const ProjectArgs& a, hipStream_t st) {
  if (a.n_agents > 0) {
    const dim3 grid((unsigned)a.T);
    switch (a.rank) {
      case 8: hipLaunchKernelGGL((shrink_kernel<FP8, 8>), grid, dim3(256), 0, st, a); break;
      case 16: hipLaunchKernelGGL((shrink_kernel<FP8, 16>), grid, dim3(256), 0, st, a); break;
      case 32: hipLaunchKernelGGL((shrink_kernel<FP8, 32>), grid, dim3(256), 0, st, a); break;
      default: hipLaunchKernelGGL((shrink_kernel<FP8, 64>), grid, dim3(256), 0, st, a); break;
    }
    if (const hipError_t e = hipGetLastError()) return e;
  }
  const dim3 grid((unsigned)((a.d_out + 63) / 64), (unsigned)((a.T + 63) / 64));
  hipLaunchKernelGGL((project_kernel<FP8>), grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace

size_t adapted_projection_bytes(int64_t T, int64_t d_in, int64_t d_out, int n_agents, int rank, int cus) {
  return n_agents > 0 ? (size_t)T * (size_t)rank * 2 : 0;
}

hipError_t launch_adapted_projection(const ProjectArgs& a, hipStream_t st) {
  return a.x_scale != nullptr ? launch<true>(a, st) : launch<false>(a, st);
}

}  // namespace prc
