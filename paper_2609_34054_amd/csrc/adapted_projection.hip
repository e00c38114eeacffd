// Projection of hidden states with the low-rank adapter of each row's agent
// (Eq. 1 for many agents at once):
//     Y[i] = X[i] W + (X[i] A_a) B_a,   a = agent[i]   (no such agent: X[i] W)
// in bf16, or with X and W in e4m3 (X = x_scale[i] X8, W = w_scale[j] W8).
// The rank-r rows X A_a are formed first (fp32 sums, then bf16, as the LR
// caches hold them) and added, expanded by B_a, as Y is written.
#include "common.hpp"
#include "kernels.hpp"

#include <type_traits>
#include <cstdlib>

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
// Many rows: X A_a of every row first (a workgroup per 16 rows, its agents in
// turn), then X W in 256 x 256 tiles with the expanded adapter rows added as
// each tile is written.
template <bool FP8>
__global__ void __launch_bounds__(ST_W * 64) shrink_kernel(const ProjectArgs a) {
  using C = Stream<FP8, 1>;
  __shared__ __attribute__((aligned(1024))) char lds[ST_W * C::RING * C::STEP];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t t0 = (int64_t)blockIdx.x * 16;
  const int toks = (int)(a.T - t0 < 16 ? a.T - t0 : (int64_t)16), nk = (int)((a.d_in + 31) / 32);
  const int ag = lane < toks ? a.agent[t0 + lane] : -1;
  uint64_t todo = __ballot(ag >= 0 && ag < a.n_agents);  // the same in every wave
  uint16_t* H = static_cast<uint16_t*>(a.ws) + t0 * a.rank;
  while (todo != 0) {
    const int cur = __builtin_amdgcn_readlane(ag, __builtin_ctzll(todo));
    const uint64_t mine = __ballot(ag == cur);
    todo &= ~mine;
    f32x4 acc[4][1] = {};
    __syncthreads();  // the sums before are read
    stream_steps<FP8, 1, true>(a, lds + w * C::RING * C::STEP, t0, toks, (int64_t)cur * a.rank, nk * w / ST_W,
                               nk * (w + 1) / ST_W, acc);
    sum_waves<1, 4>(acc, lds, 0, (a.rank + 15) / 16, [&](int g, int t, int q, f32x4 s) {
      const int j = g * 16 + 4 * q;
      if (j >= a.rank || !(mine >> t & 1)) return;
      if (FP8) s *= a.x_scale[t0 + t];
      *reinterpret_cast<u32x2*>(H + t * a.rank + j) = u32x2{pack_bf16(s[0], s[1]), pack_bf16(s[2], s[3])};
    });
  }
}

typedef int i32x8 __attribute__((ext_vector_type(8)));

// Tiles of 256 tokens x 32 (C0 + C1) columns: eight waves, four by tokens (64
// each) and two by columns (32 C0 and 32 C1 of them), on 32x32 MFMAs.  Waves w
// and w + 4 share a SIMD, so an uneven pair loads all SIMDs alike.  The operands
// come through a ring of stages (64 bytes of k of each row and column) with
// direct loads that all waves issue; a wave reads the fragments of its next
// step between the MFMAs of this one.  X rows are XOR-swizzled in 16-byte
// chunks, weight rows (as in memory) in blocks of 32 columns, so that the rows
// which one read takes together hit different banks.
constexpr int TL_T = 256;

template <bool FP8, int NP>  // NP = C0 + C1 column blocks
struct Tile {
  static constexpr int E = FP8 ? 1 : 2, KS = 64 / E, KK = FP8 ? 1 : 2;  // bytes, k and MFMA steps of a stage
  static constexpr int CT = 32 * NP, WRB = CT * E;                      // columns; bytes of a weight row
  static constexpr int XB = TL_T * 64, SB = XB + CT * 64;               // bytes of X and of a stage
  static constexpr int RING = 160 * 1024 / SB < 6 ? 160 * 1024 / SB : 6;
  static constexpr int NL = SB / 1024, NI = (NL + 7) / 8;               // 1 KB loads of a stage; of a wave, at most
  // Column block b of weight row k is stored at b ^ swz(k): bf16 reads take 4
  // rows of 64 bytes together, e4m3 reads 8 rows of 32.
  static __device__ __forceinline__ int swz(int k) {
    if (NP % 2 != 0) return 0;  // odd row strides do it
    if (FP8) return NP % 8 == 0 ? k & 7 : (NP % 4 == 0 ? (k >> 1) & 3 : (k >> 2) & 1);
    return NP % 4 == 0 ? k & 3 : (k >> 1) & 1;
  }
};

// One wave's part of a tile: tokens t0 + 64 wt .., columns c0 + 32 cb0 .. of CB blocks.
template <bool FP8, int NP, int CB>
__device__ __forceinline__ void tile_wave(const ProjectArgs& a, char* ring, int64_t t0, int64_t c0, int cb0) {
  using C = Tile<FP8, NP>;
  constexpr int E = C::E, FR = FP8 ? 8 : 4;  // registers of a fragment
  typedef uint32_t Frag __attribute__((ext_vector_type(FR)));
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wt = wv & 3;
  const int toks = (int)(a.T - t0 < TL_T ? a.T - t0 : (int64_t)TL_T), d_in = (int)a.d_in;
  const int32_t ldw = (int32_t)(a.d_out * E), ldx = (int32_t)(a.ld_x * E);
  const i32x4 rx = buffer_rsrc(static_cast<const char*>(a.X) + t0 * ldx, (toks - 1) * ldx + d_in * E);
  const i32x4 rw = buffer_rsrc(a.W, d_in * ldw);
  // Load j of this wave is load 8 j + wv of the stage, X rows first.
  const bool full = 8 * (C::NI - 1) + wv < C::NL;  // this wave has NI loads a stage, or one less
  int32_t off[C::NI], kof[C::NI];
#pragma unroll
  for (int j = 0; j < C::NI; ++j) {
    const int b = (8 * j + wv) * 1024 + lane * 16;
    if (j < C::XB / 8192) {
      const int r = b / 64, c = (lane % 4) ^ ((r >> 2) & 3);
      kof[j] = c * 16 / E;
      off[j] = r < toks ? r * ldx + c * 16 : INT32_MIN;
    } else {
      const int k = (b - C::XB) / C::WRB, p = (b - C::XB) % C::WRB / (32 * E), in = (b - C::XB) % (32 * E) / E;
      const int64_t col = c0 + (p ^ C::swz(k)) * 32 + in;
      kof[j] = k;
      off[j] = col < a.d_out ? k * ldw + (int32_t)col * E : INT32_MIN;
    }
  }
  static_assert(C::XB % 8192 == 0 && C::WRB % 16 == 0 && C::NL % 2 == 0, "X and weight loads are separate instructions");
  auto issue = [&](int s, int slot) {
    char* st = ring + slot * C::SB;
    const int k0 = s * C::KS;
    const bool whole = k0 + C::KS <= d_in;  // the k offset is scalar
#pragma unroll
    for (int j = 0; j < C::NI; ++j) {
      if (j == C::NI - 1 && !full) break;
      const bool x = j < C::XB / 8192;
      const uint32_t ks = (uint32_t)k0 * (uint32_t)(x ? E : ldw);
      if (whole) {
        lds_dma16(x ? rx : rw, st + (8 * j + wv) * 1024, off[j], (int32_t)ks);
      } else {
        const bool ok = k0 + kof[j] < d_in && off[j] != INT32_MIN;
        lds_dma16(x ? rx : rw, st + (8 * j + wv) * 1024, ok ? (int32_t)((uint32_t)off[j] + ks) : INT32_MIN, 0);
      }
    }
  };
  // Waits until only `n` stages of this wave's loads are in flight.
  auto wait_stages = [&](auto n) {
    if (full) wait_loads<decltype(n)::value * C::NI>();
    else wait_loads<decltype(n)::value * (C::NI - 1)>();
  };

  const int l32 = lane & 31, h = lane >> 5, grp = lane >> 4, i16 = lane & 15;
  f32x16 acc[CB][2];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
      for (int j = 0; j < 16; ++j) acc[cb][tb][j] = 0.f;
  const int xrow = 64 * wt + l32, xs = (xrow >> 2) & 3;  // rows 32 further swizzle alike
  auto read_x = [&](int tb, const char* st, int kk) -> Frag {
    const char* p = st + (xrow + 32 * tb) * 64;
    if constexpr (FP8) {
      const u32x4 lo = *reinterpret_cast<const u32x4*>(p + ((2 * h) ^ xs) * 16);
      const u32x4 hi = *reinterpret_cast<const u32x4*>(p + ((2 * h + 1) ^ xs) * 16);
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      return *reinterpret_cast<const u32x4*>(p + ((2 * kk + h) ^ xs) * 16);
    }
  };
  // First weight row of this lane; the rows it reads besides swizzle alike.
  const int wk = FP8 ? 32 * h + i16 / 2 : 8 * h + i16 / 4, ws = C::swz(wk);
  const int wo = C::XB + wk * C::WRB + (grp & 1) * 16 * E + (FP8 ? i16 % 2 : i16 % 4) * 8;
  auto read_w = [&](int cb, const char* st, int kk) -> Frag {
    const char* p = st + wo + ((cb0 + cb) ^ ws) * (32 * E) + 16 * kk * C::WRB;
    if constexpr (FP8) {
      const u32x2 v0 = lds_read_tr8(p), v1 = lds_read_tr8(p + 8 * C::WRB), v2 = lds_read_tr8(p + 16 * C::WRB),
                  v3 = lds_read_tr8(p + 24 * C::WRB);
      return Frag{v0[0], v0[1], v1[0], v1[1], v2[0], v2[1], v3[0], v3[1]};
    } else {
      const u32x2 lo = lds_read_tr16(p), hi = lds_read_tr16(p + 4 * C::WRB);
      return Frag{lo[0], lo[1], hi[0], hi[1]};
    }
  };
  auto mma = [&](Frag w, Frag x, f32x16 c) -> f32x16 {
    if constexpr (FP8)
      return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(__builtin_bit_cast(i32x8, w), __builtin_bit_cast(i32x8, x), c, 0, 0, 0,
                                                             0, 0, 0);
    else
      return mfma32x32x16(as_bf16x8(w), as_bf16x8(x), c);
  };

  const int ns = (d_in + C::KS - 1) / C::KS;
#pragma unroll
  for (int s = 0; s < C::RING - 1; ++s) issue(s, s);
  wait_stages(std::integral_constant<int, C::RING - 2>{});
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  Frag fw[CB], fx[2][2];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) fw[cb] = read_w(cb, ring, 0);
#pragma unroll
  for (int tb = 0; tb < 2; ++tb) fx[0][tb] = read_x(tb, ring, 0);
  int slot = 0, last = C::RING - 1;  // slots of stage s and of stage s - 1
  // Stage s, its first X fragments in set p0.  A weight fragment is read again
  // (of the next step) as soon as its last MFMA is issued.
  auto stage = [&](int s, auto P0) {
    constexpr int p0 = decltype(P0)::value;
    const int next = slot + 1 == C::RING ? 0 : slot + 1;
    const char* st = ring + slot * C::SB;
    const char* stn = ring + next * C::SB;
#pragma unroll
    for (int kk = 0; kk < C::KK; ++kk) {
      const int cur = (p0 + kk) & 1, nxt = cur ^ 1;
      if (kk == C::KK - 1) {
        // Stage s + 1 has landed, and every wave has used what it read of stage
        // s - 1, whose slot is filled again.
        wait_stages(std::integral_constant<int, C::RING - 3>{});
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        issue(s + C::RING - 1, last);  // past the end: zeros
      }
      const char* sn = kk == C::KK - 1 ? stn : st;
      const int kn = kk == C::KK - 1 ? 0 : kk + 1;
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        if (cb < 2) fx[nxt][cb] = read_x(cb, sn, kn);
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) acc[cb][tb] = mma(fw[cb], fx[cur][tb], acc[cb][tb]);
        fw[cb] = read_w(cb, sn, kn);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    last = slot;
    slot = next;
  };
  static_assert(CB >= 2, "both X fragments are read");
  if constexpr (C::KK == 2) {
    for (int s = 0; s < ns; ++s) stage(s, std::integral_constant<int, 0>{});
  } else {
    int s = 0;
    for (; s + 1 < ns; s += 2) {
      stage(s, std::integral_constant<int, 0>{});
      stage(s + 1, std::integral_constant<int, 1>{});
    }
    if (s < ns) stage(s, std::integral_constant<int, 0>{});
  }
  wait_loads<0>();
  wait_lds();
  __builtin_amdgcn_s_barrier();  // the ring is free
  asm volatile("" ::: "memory");

  // acc[cb][tb][j]: column cw + 32 cb + (j / 4) * 8 + 4 h + j % 4, token
  // tw + 32 tb.
  const int64_t cw = c0 + 32 * cb0, tw = t0 + 64 * wt + l32;
  if constexpr (FP8) {
    float xsc[2];
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) xsc[tb] = tw + 32 * tb < a.T ? a.x_scale[tw + 32 * tb] : 0.f;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int jg = 0; jg < 4; ++jg) {
        const int64_t c = cw + 32 * cb + jg * 8 + 4 * h;
        f32x4 wsc = {0.f, 0.f, 0.f, 0.f};
        if (c < a.d_out) wsc = *reinterpret_cast<const f32x4*>(a.w_scale + c);
#pragma unroll
        for (int tb = 0; tb < 2; ++tb)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[cb][tb][4 * jg + i] *= xsc[tb] * wsc[i];
      }
  }
  if (a.n_agents > 0) {
    // Agents of the wave's tokens in turn.  Where a block of 32 tokens has one
    // agent (tokens past T go with any), its product is summed in place, else it
    // is added to that agent's tokens alone, so that what is infinite or NaN in
    // an adapter stays in the rows that use it.
    int ag[2];
    uint64_t todo[2];
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
      ag[tb] = tw + 32 * tb < a.T ? a.agent[tw + 32 * tb] : -1;
      todo[tb] = __ballot(ag[tb] >= 0 && ag[tb] < a.n_agents);
    }
    const int R = a.rank, nr = (R + 15) / 16;
    while ((todo[0] | todo[1]) != 0) {
      const int cur = todo[0] != 0 ? __builtin_amdgcn_readlane(ag[0], __builtin_ctzll(todo[0]))
                                   : __builtin_amdgcn_readlane(ag[1], __builtin_ctzll(todo[1]));
      u32x4 fh[2][4];  // ranks 16 kk + 8 h .. of token l32 of each block
      bool mine[2], whole[2], some[2];
#pragma unroll
      for (int tb = 0; tb < 2; ++tb) {
        const int64_t t = tw + 32 * tb;
        mine[tb] = ag[tb] == cur;
        const uint64_t m = __ballot(mine[tb]);
        some[tb] = m != 0;
        todo[tb] &= ~m;
        whole[tb] = __ballot(mine[tb] || t >= a.T) == ~0ull;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
          fh[tb][kk] = ld16(static_cast<const uint16_t*>(a.ws) + t * R + 16 * kk + 8 * h, mine[tb] && 16 * kk + 8 * h < R);
      }
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        const int64_t c = cw + 32 * cb + l32;
        u32x4 fb[4];  // B_a^T: the same ranks of column l32
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          if (kk >= nr) break;  // uniform
          const bool ok = c < a.d_out && 16 * kk + 8 * h < R;
          const uint16_t* bp = a.B + ((int64_t)cur * R + 16 * kk + 8 * h) * a.d_out + c;
          uint32_t v[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = ok ? bp[i * a.d_out] : 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) fb[kk][i] = v[2 * i] | v[2 * i + 1] << 16;
        }
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) {
          if (!some[tb]) continue;  // uniform, as the next
          f32x16 sum;
#pragma unroll
          for (int j = 0; j < 16; ++j) sum[j] = whole[tb] ? acc[cb][tb][j] : 0.f;
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {
            if (kk >= nr) break;
            sum = mfma32x32x16(as_bf16x8(fb[kk]), as_bf16x8(fh[tb][kk]), sum);
          }
#pragma unroll
          for (int j = 0; j < 16; ++j) acc[cb][tb][j] = whole[tb] ? sum[j] : (mine[tb] ? acc[cb][tb][j] + sum[j] : acc[cb][tb][j]);
        }
      }
    }
  }
  // Out through LDS (rows padded by 16 bytes), so that each row is written in
  // one piece of 64 CB bytes.
  constexpr int RB = 64 * CB + 16;
  static_assert(8 * 64 * (64 * ((NP + 1) / 2) + 16) <= C::RING * C::SB, "the waves' results fit the ring");
  char* mineb = ring + wv * 64 * (64 * ((NP + 1) / 2) + 16);
#pragma unroll
  for (int tb = 0; tb < 2; ++tb)
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int jg = 0; jg < 4; ++jg) {
        const f32x16& v = acc[cb][tb];
        *reinterpret_cast<u32x2*>(mineb + (32 * tb + l32) * RB + cb * 64 + jg * 16 + h * 8) =
            u32x2{pack_bf16(v[4 * jg], v[4 * jg + 1]), pack_bf16(v[4 * jg + 2], v[4 * jg + 3])};
      }
  wait_lds();
#pragma unroll
  for (int i = 0; i < 4 * CB; ++i) {
    const int u = i * 64 + lane, r = u / (4 * CB), ch = u % (4 * CB);
    const int64_t t = t0 + 64 * wt + r, c = cw + ch * 8;
    const u32x4 v = *reinterpret_cast<const u32x4*>(mineb + r * RB + ch * 16);
    if (t < a.T && c < a.d_out) *reinterpret_cast<u32x4*>(a.Y + t * a.ld_y + c) = v;
  }
}

template <bool FP8, int C0, int C1>
__global__ void __launch_bounds__(512, 2) tile_kernel(const ProjectArgs a, int n_tt, int n_ct) {
  using C = Tile<FP8, C0 + C1>;
  __shared__ __attribute__((aligned(1024))) char ring[C::RING * C::SB];
  // Workgroup L runs on XCD L % 8; each XCD takes a contiguous eighth of the
  // tiles, in bands of four token tiles, whose rows of X and columns of W its
  // L2 then serves several times.
  const int n_tiles = n_tt * n_ct, per = (n_tiles + 7) / 8;
  const int tile = (int)(blockIdx.x % 8) * per + (int)(blockIdx.x / 8);
  if ((int)(blockIdx.x / 8) >= per || tile >= n_tiles) return;  // uniform over the workgroup
  const int band = tile / (4 * n_ct), in = tile - band * 4 * n_ct, bh = n_tt - 4 * band < 4 ? n_tt - 4 * band : 4;
  const int ct = __builtin_amdgcn_readfirstlane(in / bh), tt = __builtin_amdgcn_readfirstlane(4 * band + in % bh);
  const int64_t t0 = (int64_t)tt * TL_T, c0 = (int64_t)ct * C::CT;
  if (__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) < 4) tile_wave<FP8, C0 + C1, C0>(a, ring, t0, c0, 0);
  else tile_wave<FP8, C0 + C1, C1>(a, ring, t0, c0, C0);
}

template <bool FP8, int C0, int C1>
hipError_t launch_tiles(const ProjectArgs& a, hipStream_t st) {
  const int64_t n_tt = (a.T + TL_T - 1) / TL_T, n_ct = (a.d_out + 32 * (C0 + C1) - 1) / (32 * (C0 + C1));
  hipLaunchKernelGGL((tile_kernel<FP8, C0, C1>), dim3((unsigned)((n_tt * n_ct + 7) / 8 * 8)), dim3(512), 0, st, a, (int)n_tt,
                     (int)n_ct);
  return hipGetLastError();
}

template <bool FP8>
hipError_t launch(const ProjectArgs& a, hipStream_t st) {
  if (a.T <= ST_T) return launch_stream<FP8>(a, st);
  if (a.n_agents > 0) {
    hipLaunchKernelGGL((shrink_kernel<FP8>), dim3((unsigned)((a.T + 15) / 16)), dim3(ST_W * 64), 0, st, a);
    if (const hipError_t e = hipGetLastError()) return e;
  }
  // The width that takes the least time by rounds of the CUs.
  int best = 8;
  double least = 1e300;
  for (int np : {8, 6, 5, 4}) {
    const int64_t tiles = ((a.T + TL_T - 1) / TL_T) * ((a.d_out + 32 * np - 1) / (32 * np));
    const double t = (double)((tiles + a.cus - 1) / a.cus) * (np + 0.5);
    if (t < least) {
      least = t;
      best = np;
    }
  }
  if (const char* f = getenv("TL_NP")) best = atoi(f);
  switch (best) {
    case 8: return launch_tiles<FP8, 4, 4>(a, st);
    case 6: return launch_tiles<FP8, 3, 3>(a, st);
    case 5: return launch_tiles<FP8, 3, 2>(a, st);
    default: return launch_tiles<FP8, 2, 2>(a, st);
  }
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
