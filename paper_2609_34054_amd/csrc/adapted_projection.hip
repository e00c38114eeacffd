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

// Transposing LDS reads.  16-bit: lane j of a 16-lane group points at 4
// elements, lane i receives element i % 4 of lanes i / 4, i / 4 + 4, ... + 12.
// 8-bit: lane j points at 8 elements, lane i receives element i % 8 of lanes
// i / 8, i / 8 + 2, ... + 14.
__device__ __forceinline__ u32x2 lds_read_tr16(const void* p) {
  typedef short v4s __attribute__((ext_vector_type(4)));
  v4s v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((v4s __attribute__((address_space(3)))*)(p));
  return __builtin_bit_cast(u32x2, v);
}
__device__ __forceinline__ u32x2 lds_read_tr8(const void* p) {
  typedef int v2i __attribute__((ext_vector_type(2)));
  v2i v = __builtin_amdgcn_ds_read_tr8_b64_v2i32((v2i __attribute__((address_space(3)))*)(p));
  return __builtin_bit_cast(u32x2, v);
}

// Waits until at most N of this wave's loads are in flight, or for its LDS
// reads; memory accesses stay on their side.
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

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

// ---------------------------------------------------------------------------
// Few rows (T <= 64): the weights are streamed once, so memory bounds it.  A
// workgroup takes a column tile (128 bytes of each weight row) and a slice of
// k, its eight waves an eighth of that each; a wave brings its own 32-k steps
// (weights and the rows of X) through a private ring in LDS with direct loads,
// several steps ahead and without barriers.  Weight rows lie in LDS as in
// memory, their 16-column units XOR-swizzled by row so that the rows which a
// transposing read takes together hit different banks.  The same kernel forms
// the rows X A_a: a workgroup per distinct agent (and k slice).  The waves'
// sums are added through LDS in a fixed order and go to the workspace; a
// second kernel adds the k slices and the expanded adapter rows.
constexpr int ST_W = 8;   // waves
constexpr int ST_T = 64;  // most rows

template <bool FP8, int TB>  // TB blocks of 16 rows
struct Stream {
  static constexpr int CW = FP8 ? 128 : 64, NB = CW / 16;     // columns and 16-column blocks of a tile
  static constexpr int XI = FP8 ? (TB + 1) / 2 : TB;          // 1 KB loads of X per step
  static constexpr int NI = 4 + XI, STEP = NI * 1024;         // loads and bytes of a step
  static constexpr int RING = 20 / NI;                        // steps in flight: 16 to 20 KB a wave
  static constexpr int G = NB * TB > 16 ? 16 / TB : NB;       // column blocks summed at a time (LDS)
  static_assert(ST_W * G * TB * 1024 <= ST_W * RING * STEP, "partials fit the ring");
  static_assert(ST_W * RING * STEP <= 160 * 1024, "LDS");
};

// Unit (16 columns) of weight row r is stored at unit ^ swz(r).
template <bool FP8>
__device__ __forceinline__ int swz(int r) {
  return FP8 ? ((r >> 1) & 3) + 4 * ((r >> 3) & 1) : ((r >> 1) & 1) + 2 * ((r >> 3) & 1);
}

// One pass over this wave's steps [s_lo, s_hi): acc[nb][tb] += W^T X^T for the
// 16-column blocks nb.  AD: the weights are `rank` columns of A from column
// col0 (bf16, NBA blocks), else a tile of W.
template <bool FP8, int TB, bool AD, typename Acc>
__device__ __forceinline__ void stream_steps(const ProjectArgs& a, char* ring, int64_t t0, int toks, int64_t col0, int s_lo,
                                             int s_hi, Acc& acc) {
  using C = Stream<FP8, TB>;
  constexpr int XE = FP8 ? 1 : 2, WE = AD ? 2 : XE;  // bytes of an element
  const int lane = threadIdx.x & 63, q = lane >> 4, c16 = lane & 15;
  const int d_in = (int)a.d_in, R = a.rank;
  const int32_t ldw = (int32_t)((AD ? (int64_t)a.n_agents * R : a.d_out) * WE), ldx = (int32_t)(a.ld_x * XE);
  const i32x4 rw = buffer_rsrc(AD ? static_cast<const void*>(a.A) : a.W, d_in * ldw);
  const i32x4 rx = buffer_rsrc(static_cast<const char*>(a.X) + t0 * ldx, (toks - 1) * ldx + d_in * XE);
  // Each lane's k within a step and byte offset at k = 0, for every load.
  int32_t kw[4], ow[4], kx[C::XI], ox[C::XI];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (AD) {
      const int b = j * 1024 + lane * 16, rb = 2 * R;
      kw[j] = b / rb;
      ow[j] = b < 32 * rb ? kw[j] * ldw + (int32_t)col0 * 2 + b % rb : INT32_MIN;
    } else {
      kw[j] = j * 8 + lane / 8;
      const int p = lane % 8;
      const int64_t c = col0 + (FP8 ? (p ^ swz<true>(kw[j])) * 16 : ((p / 2) ^ swz<false>(kw[j])) * 16 + p % 2 * 8);
      ow[j] = c < a.d_out ? kw[j] * ldw + (int32_t)c * WE : INT32_MIN;
    }
  }
#pragma unroll
  for (int j = 0; j < C::XI; ++j) {
    const int t = FP8 ? j * 32 + lane / 2 : j * 16 + lane / 4;
    kx[j] = FP8 ? lane % 2 * 16 : lane % 4 * 8;
    ox[j] = t < toks && t < 16 * TB ? t * ldx + kx[j] * XE : INT32_MIN;
  }
  auto issue = [&](int s) {
    char* st = ring + (s % C::RING) * C::STEP;
    const int k0 = s * 32;
    const int left = s < s_hi ? d_in - k0 : 0;  // steps past the slice load zeros
#pragma unroll
    for (int j = 0; j < 4; ++j)
      lds_dma16(rw, st + j * 1024, kw[j] < left && ow[j] != INT32_MIN ? (int32_t)(ow[j] + (uint32_t)k0 * (uint32_t)ldw) : INT32_MIN, 0);
#pragma unroll
    for (int j = 0; j < C::XI; ++j)
      lds_dma16(rx, st + 4096 + j * 1024, kx[j] < left && ox[j] != INT32_MIN ? ox[j] + k0 * XE : INT32_MIN, 0);
  };
  for (int i = 0; i < C::RING; ++i) issue(s_lo + i);
  for (int s = s_lo; s < s_hi; ++s) {
    wait_loads<(C::RING - 1) * C::NI>();
    const char* st = ring + (s % C::RING) * C::STEP;
    const char* xp = st + 4096;
    if constexpr (FP8 && !AD) {
      long x[TB];
#pragma unroll
      for (int tb = 0; tb < TB; ++tb) x[tb] = *reinterpret_cast<const long*>(xp + tb * 512 + c16 * 32 + q * 8);
      const int kr = 8 * q + c16 / 2;
#pragma unroll
      for (int nb = 0; nb < C::NB; ++nb) {
        const long w = __builtin_bit_cast(long, lds_read_tr8(st + kr * 128 + (nb ^ swz<true>(kr)) * 16 + c16 % 2 * 8));
#pragma unroll
        for (int tb = 0; tb < TB; ++tb) acc[nb][tb] = __builtin_amdgcn_mfma_f32_16x16x32_fp8_fp8(w, x[tb], acc[nb][tb], 0, 0, 0);
      }
    } else {
      bf16x8 x[TB];
#pragma unroll
      for (int tb = 0; tb < TB; ++tb) {
        if constexpr (FP8)
          x[tb] = as_bf16x8(bf16_of_e4m3(*reinterpret_cast<const u32x2*>(xp + tb * 512 + c16 * 32 + q * 8)));
        else
          x[tb] = as_bf16x8(*reinterpret_cast<const u32x4*>(xp + tb * 1024 + c16 * 64 + q * 16));
      }
      const int kr = 8 * q + c16 / 4, rb = AD ? 2 * R : 128;
#pragma unroll
      for (int nb = 0; nb < 4; ++nb) {
        if (AD && nb * 16 >= R) break;  // uniform (rank 8: one block, its upper columns dropped)
        const char* p = st + kr * rb + (AD ? nb : nb ^ swz<false>(kr)) * 32 + c16 % 4 * 8;
        const u32x2 lo = lds_read_tr16(p), hi = lds_read_tr16(p + 4 * rb);
#pragma unroll
        for (int tb = 0; tb < TB; ++tb)
          acc[nb][tb] = mfma16x16x32(as_bf16x8(u32x4{lo[0], lo[1], hi[0], hi[1]}), x[tb], acc[nb][tb]);
      }
    }
    wait_lds();  // this step's slot is free
    issue(s + C::RING);
  }
  wait_loads<0>();
}

// Sums the waves' acc[g0 + g][tb] (g < n) through LDS in a fixed order and
// hands out the sums of block g, row t, columns 4 q ..: put(g, t, q, sum).
template <int TB, int G, int NB, typename Put>
__device__ __forceinline__ void sum_waves(f32x4 (&acc)[NB][TB], char* lds, int g0, int n, Put put) {
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  f32x4* part = reinterpret_cast<f32x4*>(lds);  // [wave][G][TB][64]
  __syncthreads();  // the ring, or the sums before, are no longer read
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int tb = 0; tb < TB; ++tb) part[((w * G + g) * TB + tb) * 64 + lane] = acc[g0 + g][tb];
  __syncthreads();
  for (int u = tid; u < n * TB * 64; u += ST_W * 64) {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < ST_W; ++v) s += part[v * G * TB * 64 + u];
    put(u / (TB * 64), u / 64 % TB * 16 + u % 16, u / 16 % 4, s);
  }
}

// Workspace of the two kernels: sums of W [ks][T][d_out], then of the adapters
// [ksa][T][rank], fp32.
struct StreamPlan {
  int n_ct, ks, ksa;
};

template <bool FP8, int TB>
__global__ void __launch_bounds__(ST_W * 64) stream_kernel(const ProjectArgs a, const StreamPlan p) {
  using C = Stream<FP8, TB>;
  __shared__ __attribute__((aligned(1024))) char lds[ST_W * C::RING * C::STEP];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int T = (int)a.T, nk = (int)((a.d_in + 31) / 32);
  char* ring = lds + w * C::RING * C::STEP;
  const int n_main = p.n_ct * p.ks;
  f32x4 acc[C::NB][TB];
#pragma unroll
  for (int i = 0; i < C::NB; ++i)
#pragma unroll
    for (int j = 0; j < TB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  if ((int)blockIdx.x < n_main) {
    const int ct = blockIdx.x % p.n_ct, ki = blockIdx.x / p.n_ct, parts = p.ks * ST_W, part = ki * ST_W + w;
    const int64_t c0 = (int64_t)ct * C::CW;
    stream_steps<FP8, TB, false>(a, ring, 0, T, c0, (int)((int64_t)nk * part / parts), (int)((int64_t)nk * (part + 1) / parts), acc);
    float* out = static_cast<float*>(a.ws) + (int64_t)ki * T * a.d_out;
#pragma unroll
    for (int g0 = 0; g0 < C::NB; g0 += C::G)
      sum_waves<TB, C::G>(acc, lds, g0, C::G, [&](int g, int t, int q, f32x4 s) {
        const int64_t c = c0 + (g0 + g) * 16 + 4 * q;
        if (t < T && c < a.d_out) *reinterpret_cast<f32x4*>(out + t * a.d_out + c) = s;
      });
    return;
  }
  // Adapter rows: workgroup i works for row i's agent if no earlier row has it.
  const int i = (blockIdx.x - n_main) % T, ki = (blockIdx.x - n_main) / T, parts = p.ksa * ST_W, part = ki * ST_W + w;
  const int ag = a.agent[i], lane = threadIdx.x & 63;
  if (ag < 0 || ag >= a.n_agents) return;
  const bool same = lane < T && a.agent[lane < T ? lane : 0] == ag;
  const uint64_t mine = __ballot(same);
  if (mine & ((1ull << i) - 1)) return;  // uniform: every wave sees the same rows
  f32x4 (&acc4)[C::NB][TB] = acc;
  stream_steps<FP8, TB, true>(a, ring, 0, T, (int64_t)ag * a.rank, (int)((int64_t)nk * part / parts),
                              (int)((int64_t)nk * (part + 1) / parts), acc4);
  float* out = static_cast<float*>(a.ws) + (int64_t)p.ks * T * a.d_out + (int64_t)ki * T * a.rank;
  constexpr int G = 4;
  static_assert(C::NB >= G, "blocks of rank 64");
  sum_waves<TB, G>(acc, lds, 0, (a.rank + 15) / 16, [&](int g, int t, int q, f32x4 s) {
    const int j = g * 16 + 4 * q;
    if (j < a.rank && (mine >> t & 1)) *reinterpret_cast<f32x4*>(out + t * a.rank + j) = s;
  });
}

// Y of 256 columns of a row: a wave, four columns a lane.
template <int R>
__global__ void __launch_bounds__(64) join_kernel(const ProjectArgs a, const StreamPlan p) {
  const int lane = threadIdx.x;
  const int64_t t = blockIdx.y, c = (int64_t)blockIdx.x * 256 + lane * 4, T = a.T;
  const float* P = static_cast<const float*>(a.ws);
  const bool ok = c < a.d_out;
  const int ag = a.n_agents > 0 ? a.agent[t] : -1;
  const bool lr = ag >= 0 && ag < a.n_agents;  // uniform
  const float xs = a.x_scale != nullptr ? a.x_scale[t] : 1.f;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  u32x2 b[R];
  float h = 0.f;
  if (lr) {
    const uint16_t* B = a.B + (int64_t)ag * R * a.d_out + c;
#pragma unroll
    for (int j = 0; j < R; ++j) b[j] = ld8(B + j * a.d_out, ok);
    const float* H = P + p.ks * T * a.d_out + t * R;
    if (lane < R)
      for (int k = 0; k < p.ksa; ++k) h += H[k * T * R + lane];
  }
  if (ok) {
    for (int k = 0; k < p.ks; ++k) v += *reinterpret_cast<const f32x4*>(P + (k * T + t) * a.d_out + c);
    if (a.x_scale != nullptr) {
      const f32x4 wsc = *reinterpret_cast<const f32x4*>(a.w_scale + c);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] *= xs * wsc[i];
    }
  }
  if (lr) {
    const float hb = bf_lo(pack_bf16(h * xs, 0.f));
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const float hj = readlane_f(hb, j);
      v[0] += hj * bf_lo(b[j][0]);
      v[1] += hj * bf_hi(b[j][0]);
      v[2] += hj * bf_lo(b[j][1]);
      v[3] += hj * bf_hi(b[j][1]);
    }
  }
  if (ok) *reinterpret_cast<u32x2*>(a.Y + t * a.ld_y + c) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
}

// Column tiles, and k slices so that all workgroups of W and of the adapters
// (each no longer than one of W) run at once, one a CU.
StreamPlan stream_plan(int64_t T, int64_t d_in, int64_t d_out, int n_agents, int rank, bool fp8, int cus) {
  StreamPlan p;
  const int cw = fp8 ? 128 : 64, ad = (int)(T < n_agents ? T : n_agents);
  p.n_ct = (int)((d_out + cw - 1) / cw);
  const int64_t steps = (d_in + 31) / 32;
  int most = (int)(steps / ST_W);  // a step a wave at least
  if (most < 1) most = 1;
  p.ks = cus / p.n_ct;
  p.ks = p.ks < 1 ? 1 : (p.ks > most ? most : p.ks);
  auto slices = [&](int ks) { return (ks * rank + 63) / 64; };
  while (p.ks > 1 && p.n_ct * p.ks + ad * slices(p.ks) > cus) --p.ks;
  p.ksa = ad > 0 ? slices(p.ks) : 0;
  return p;
}
size_t stream_bytes(int64_t T, int64_t d_out, int rank, const StreamPlan& p) {
  return ((size_t)p.ks * (size_t)T * (size_t)d_out + (size_t)p.ksa * (size_t)T * (size_t)rank) * 4;
}

template <bool FP8, int TB>
hipError_t launch_stream_tb(const ProjectArgs& a, const StreamPlan& p, hipStream_t st) {
  const unsigned grid = (unsigned)(p.n_ct * p.ks + p.ksa * (int)a.T);
  hipLaunchKernelGGL((stream_kernel<FP8, TB>), dim3(grid), dim3(ST_W * 64), 0, st, a, p);
  return hipGetLastError();
}

template <bool FP8>
hipError_t launch_stream(const ProjectArgs& a, hipStream_t st) {
  const StreamPlan p = stream_plan(a.T, a.d_in, a.d_out, a.n_agents, a.rank, FP8, a.cus);
  hipError_t e = a.T <= 16 ? launch_stream_tb<FP8, 1>(a, p, st)
                           : (a.T <= 32 ? launch_stream_tb<FP8, 2>(a, p, st) : launch_stream_tb<FP8, 4>(a, p, st));
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)((a.d_out + 255) / 256), (unsigned)a.T);
  switch (a.rank) {
    case 8: hipLaunchKernelGGL((join_kernel<8>), grid, dim3(64), 0, st, a, p); break;
    case 16: hipLaunchKernelGGL((join_kernel<16>), grid, dim3(64), 0, st, a, p); break;
    case 32: hipLaunchKernelGGL((join_kernel<32>), grid, dim3(64), 0, st, a, p); break;
    default: hipLaunchKernelGGL((join_kernel<64>), grid, dim3(64), 0, st, a, p); break;
  }
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
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
    const u32x2 lo = lds_read_tr16(&wt[8 * q + c16 / 4][16 * w + 4 * (c16 % 4)]);
    const u32x2 hi = lds_read_tr16(&wt[8 * q + 4 + c16 / 4][16 * w + 4 * (c16 % 4)]);
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
  if (a.T <= ST_T) return launch_stream<FP8>(a, st);
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
  if (n_agents == 0) rank = 8;
  if (T <= ST_T) {
    const size_t a = stream_bytes(T, d_out, rank, stream_plan(T, d_in, d_out, n_agents, rank, false, cus));
    const size_t b = stream_bytes(T, d_out, rank, stream_plan(T, d_in, d_out, n_agents, rank, true, cus));
    return a > b ? a : b;
  }
  return n_agents > 0 ? (size_t)T * (size_t)rank * 2 : 0;
}

hipError_t launch_adapted_projection(const ProjectArgs& a, hipStream_t st) {
  return a.x_scale != nullptr ? launch<true>(a, st) : launch<false>(a, st);
}

}  // namespace prc
