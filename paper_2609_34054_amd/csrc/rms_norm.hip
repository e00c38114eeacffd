// The layer input: residual sum and root-mean-square norm, written in bf16 or
// in 8 bits (e4m3) with one scale a row.
//     s = x + residual,   y = s / sqrt(mean(s^2) + eps) * weight
// A row is read once and stays in the registers of the threads that share it
// (fp32, 8 elements a chunk) until its mean of squares, and for e4m3 its
// largest |y|, are known; so every byte moves once and memory bounds it: 4096
// rows of 4096 with a residual take 25.3 us in bf16, 5.3 TB/s, the rate of a
// copy.  Small calls take a launch, 4.5 us.
#include "common.hpp"
#include "kernels.hpp"

namespace prc {
namespace {

constexpr float kE4m3Max = 448.f;
constexpr float kLeastMax = 0x1p-100f;  // rows below it: the scale stays a normal number

// TPR threads share a row (64: a wave each, four rows a workgroup), NCH chunks
// of 8 elements a thread.
template <int TPR, int NCH, bool FP8>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) rms_norm_kernel(const NormArgs a) {
  constexpr int RPW = TPR < 256 ? 256 / TPR : 1, NW = TPR / 64;
  __shared__ float part[NW];
  __shared__ uint32_t pmax[NW];
  const int tid = threadIdx.x, l = tid % TPR;
  const int64_t row = (int64_t)blockIdx.x * RPW + tid / TPR;
  if (row >= a.T) return;  // whole waves, or no one
  const uint16_t* x = a.x + row * a.ld_x;
  const uint16_t* res = a.residual == nullptr ? nullptr : a.residual + row * a.ld_res;
  const int d = a.d;
  u32x4 xv[NCH], rv[NCH];
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int c = (i * TPR + l) * 8;
    xv[i] = ld16(x + c, c < d);
  }
  if (res != nullptr) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = (i * TPR + l) * 8;
      rv[i] = ld16(res + c, c < d);
    }
  }
  float s[NCH][8];
  float sq = 0.f;
#pragma unroll
  for (int i = 0; i < NCH; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s[i][2 * e] = bf_lo(xv[i][e]);
      s[i][2 * e + 1] = bf_hi(xv[i][e]);
      if (res != nullptr) {
        s[i][2 * e] += bf_lo(rv[i][e]);
        s[i][2 * e + 1] += bf_hi(rv[i][e]);
      }
      sq += s[i][2 * e] * s[i][2 * e];
      sq += s[i][2 * e + 1] * s[i][2 * e + 1];
    }
  if (a.residual_out != nullptr) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = (i * TPR + l) * 8;
      if (c < d)
        *reinterpret_cast<u32x4*>(a.residual_out + row * a.ld_ro + c) =
            u32x4{pack_bf16(s[i][0], s[i][1]), pack_bf16(s[i][2], s[i][3]), pack_bf16(s[i][4], s[i][5]), pack_bf16(s[i][6], s[i][7])};
    }
  }
#pragma unroll
  for (int m = 1; m < 64; m *= 2) sq += shfl_xor(sq, m);
  if constexpr (NW > 1) {
    if (tid % 64 == 0) part[tid / 64] = sq;
    __syncthreads();
    sq = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) sq += part[w];
  }
  const float rs = 1.f / sqrtf(sq / (float)d + a.eps);
  // |y| as bits orders like |y|, infinities and NaN above all numbers.
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int c = (i * TPR + l) * 8;
    const u32x4 wv = ld16(a.weight + c, c < d);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s[i][2 * e] = s[i][2 * e] * rs * bf_lo(wv[e]);
      s[i][2 * e + 1] = s[i][2 * e + 1] * rs * bf_hi(wv[e]);
    }
    if constexpr (!FP8) {
      if (c < d)
        *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.y) + row * a.ld_y + c) =
            u32x4{pack_bf16(s[i][0], s[i][1]), pack_bf16(s[i][2], s[i][3]), pack_bf16(s[i][4], s[i][5]), pack_bf16(s[i][6], s[i][7])};
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t m = c < d ? __float_as_uint(s[i][e]) & 0x7fffffffu : 0u;  // past the row: 0 * inf may be NaN
        top = m > top ? m : top;
      }
    }
  }
  if constexpr (FP8) {
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
      const uint32_t o = __shfl_xor(top, m, kWave);
      top = o > top ? o : top;
    }
    if constexpr (NW > 1) {
      if (tid % 64 == 0) pmax[tid / 64] = top;
      __syncthreads();
      top = 0;
#pragma unroll
      for (int w = 0; w < NW; ++w) top = pmax[w] > top ? pmax[w] : top;
    }
    const float least = kLeastMax;
    const float scale = __uint_as_float(top > __float_as_uint(least) ? top : __float_as_uint(least)) / kE4m3Max;
    // One division a row: y * (1 / scale) is within 1.5 units in the last place
    // of y / scale, 2^-19 of an e4m3 step.
    const float inv = 1.f / scale;
    if (l == 0) a.y_scale[row] = scale;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = (i * TPR + l) * 8;
      uint32_t o[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float q = s[i][4 * h + e] * inv;  // NaN passes both comparisons
          v[e] = q > kE4m3Max ? kE4m3Max : (q < -kE4m3Max ? -kE4m3Max : q);
        }
        int p = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
        p = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], p, true);
        o[h] = (uint32_t)p;
      }
      if (c < d) *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(a.y) + row * a.ld_y + c) = u32x2{o[0], o[1]};
    }
  }
}

// A grid holds fewer than 2^32 threads: what is longer goes in launches of 2^31
// (2^25 rows up to 512 wide, 2^23 to 4096, 2^21 past 8192).
template <int TPR, int NCH>
hipError_t launch(const NormArgs& a, hipStream_t st) {
  constexpr int rpw = TPR < 256 ? 256 / TPR : 1, threads = TPR < 256 ? 256 : TPR;
  constexpr int64_t most = (1LL << 31) / threads * rpw;
  for (int64_t r = 0; r < a.T; r += most) {
    NormArgs p = a;
    p.T = a.T - r < most ? a.T - r : most;
    p.x = a.x + r * a.ld_x;
    if (a.residual != nullptr) p.residual = a.residual + r * a.ld_res;
    if (a.residual_out != nullptr) p.residual_out = a.residual_out + r * a.ld_ro;
    p.y = static_cast<char*>(a.y) + r * a.ld_y * (a.y_scale != nullptr ? 1 : 2);
    if (a.y_scale != nullptr) p.y_scale = a.y_scale + r;
    const dim3 grid((unsigned)((p.T + rpw - 1) / rpw));
    if (a.y_scale != nullptr) hipLaunchKernelGGL((rms_norm_kernel<TPR, NCH, true>), grid, dim3(threads), 0, st, p);
    else hipLaunchKernelGGL((rms_norm_kernel<TPR, NCH, false>), grid, dim3(threads), 0, st, p);
    if (const hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_rms_norm(const NormArgs& a, hipStream_t st) {
  // As few threads a row as keep its chunks in registers: more wait for each
  // other, and stand idle in short rows.  16384 rows in bf16 and e4m3, against
  // 1024 threads a row: 512 wide 46.1 -> 12.7 and 83.9 -> 12.8 us, 1024 wide 65.2
  // -> 25.0 and 87.4 -> 23.9, 2048 wide 75.4 -> 48.3 and 92.2 -> 44.1, 4096 wide
  // 95.7 -> 93.0 and 111 -> 81, 8192 wide no change and 175 -> 161; against waves
  // of their own 4096 wide 102 -> 93.  2048 rows of 16384, two chunks a
  // thread against eight: 57 -> 51 and 69 -> 46.
  if (a.d <= 64 * 8) return launch<64, 1>(a, st);
  if (a.d <= 64 * 16) return launch<64, 2>(a, st);
  if (a.d <= 256 * 8) return launch<256, 1>(a, st);
  if (a.d <= 256 * 16) return launch<256, 2>(a, st);
  if (a.d <= 512 * 16) return launch<512, 2>(a, st);
  if (a.d <= 1024 * 16) return launch<1024, 2>(a, st);
  if (a.d <= 1024 * 32) return launch<1024, 4>(a, st);
  return launch<1024, 8>(a, st);
}

}  // namespace prc
