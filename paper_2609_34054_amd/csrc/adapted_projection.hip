// Projection of hidden states with the low-rank adapter of each row's agent
// (Eq. 1 for many agents at once):
//     Y[i] = X[i] W + (X[i] A_a) B_a,   a = agent[i]   (no such agent: X[i] W)
// in bf16, or with X and W in e4m3 (X = x_scale[i] X8, W = w_scale[j] W8).
// The rank-r rows X A_a are formed first, in fp32, and added, expanded by B_a, as
// Y is written: by fp32 products for few rows, for tiles by matrix instructions
// that take each row as the sum of two bf16 ones, 16 bits of it (one alone made
// the error of Y 6 to 11% larger at ranks 8 and 16 and 25 to 28% at rank 64).
#include "common.hpp"
#include "kernels.hpp"

#include <type_traits>

namespace prc {
namespace {

// LDS pointers that stay 32 bits wide, and accesses through them.
typedef __attribute__((address_space(3))) char lds_char;
__device__ __forceinline__ u32x4 lds_read16(const lds_char* p) { return *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(p); }
// Transposing LDS reads.  16-bit: lane j of a 16-lane group points at 4
// elements, lane i receives element i % 4 of lanes i / 4, i / 4 + 4, ... + 12.
// 8-bit: lane j points at 8 elements, lane i receives element i % 8 of lanes
// i / 8, i / 8 + 2, ... + 14.
__device__ __forceinline__ u32x2 lds_tr16(const lds_char* p) {
  typedef short v4s __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((v4s __attribute__((address_space(3)))*)(p)));
}
__device__ __forceinline__ u32x2 lds_tr8(const lds_char* p) {
  typedef int v2i __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((v2i __attribute__((address_space(3)))*)(p)));
}
__device__ __forceinline__ u32x2 lds_read_tr16(const void* p) { return lds_tr16((const lds_char*)p); }
__device__ __forceinline__ u32x2 lds_read_tr8(const void* p) { return lds_tr8((const lds_char*)p); }
// lds_dma16 with the (wave-uniform) LDS address as a number.
__device__ __forceinline__ void lds_dma16_at(i32x4 rsrc, uint32_t to, int32_t voff, int32_t soff) {
  asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(voff), "s"(rsrc), "s"(soff)
               : "memory", "m0");
}

// Waits until at most N of this wave's loads are in flight, or for its LDS
// reads; memory accesses stay on their side.
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Four column scales, which need not lie at a multiple of 16 bytes.
__device__ __forceinline__ f32x4 ld_scales(const float* p) {
  typedef f32x4 f32x4_at4 __attribute__((aligned(4)));
  return *reinterpret_cast<const f32x4_at4*>(p);
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

// ---------------------------------------------------------------------------
// Few rows (T <= 16): the weights are streamed once, so memory bounds it.  A
// workgroup takes a column tile (128 bytes of each weight row) and a slice of
// k, its eight waves an eighth of that each; a wave brings its own 32-k steps
// (weights and the rows of X) through a private ring in LDS with direct loads,
// several steps ahead and without barriers.  Weight rows lie in LDS as in
// memory, their 16-column units XOR-swizzled by row so that the rows which a
// transposing read takes together hit different banks.  The same kernel forms
// the rows X A_a: a workgroup per distinct agent (and k slice).  The waves'
// sums are added through LDS in a fixed order and go to the workspace; a
// second kernel adds the k slices and the expanded adapter rows.
//
// 4096 x 4096 in bf16, one row: 11.0 us for both kernels, of which the weights
// (32 MB) take 6.7 at the rate of a copy; the rest is two launches and the start
// and end of the ring.  With more than 16 rows their loads and MFMAs, repeated
// for each distinct agent, outweigh the barriers saved (see the slabs below).
constexpr int ST_W = 8;   // waves
constexpr int ST_T = 16;  // most rows

template <bool FP8>
struct Stream {
  static constexpr int CW = FP8 ? 128 : 64, NB = CW / 16;  // columns and 16-column blocks of a tile
  static constexpr int NI = 5, STEP = NI * 1024;           // 1 KB loads (4 of weights, 1 of X) and bytes of a step
  // Steps in flight: 10 KB a wave, so that a CU holds two workgroups and those
  // of the adapters run beside the others'.
  static constexpr int RING = 2;
  static_assert(NB <= RING * NI, "partials fit the ring");
  static_assert(ST_W * RING * STEP <= 80 * 1024, "LDS");
};

// Unit (16 columns) of weight row r is stored at unit ^ swz(r).
template <bool FP8>
__device__ __forceinline__ int swz(int r) {
  return FP8 ? ((r >> 1) & 3) + 4 * ((r >> 3) & 1) : ((r >> 1) & 1) + 2 * ((r >> 3) & 1);
}

// One pass over this wave's steps [s_lo, s_hi): acc[nb] += W^T X^T for the
// 16-column blocks nb.  AD: the weights are `rank` columns of A from column
// col0 (bf16, NBA blocks), else a tile of W.
template <bool FP8, bool AD>
__device__ __forceinline__ void stream_steps(const ProjectArgs& a, char* ring, int toks, int64_t col0, int s_lo,
                                             int s_hi, f32x4 (&acc)[Stream<FP8>::NB]) {
  using C = Stream<FP8>;
  constexpr int XE = FP8 ? 1 : 2, WE = AD ? 2 : XE;  // bytes of an element
  const int lane = threadIdx.x & 63, q = lane >> 4, c16 = lane & 15;
  const int d_in = (int)a.d_in, R = a.rank;
  const int32_t ldw = (int32_t)((AD ? (int64_t)a.n_agents * R : a.d_out) * WE), ldx = (int32_t)(a.ld_x * XE);
  const i32x4 rw = buffer_rsrc(AD ? static_cast<const void*>(a.A) : a.W, d_in * ldw);
  const i32x4 rx = buffer_rsrc(a.X, (toks - 1) * ldx + d_in * XE);
  // Each lane's k within a step and byte offset at k = 0, for every load.
  int32_t kw[4], ow[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (AD) {
      const int b = j * 1024 + lane * 16, rb = 2 * R;
      kw[j] = b / rb;
      ow[j] = b < 32 * rb ? (int32_t)((uint32_t)kw[j] * (uint32_t)ldw + (uint32_t)(col0 * 2 + b % rb)) : INT32_MIN;  // (past d_in: wraps, unread)
    } else {
      kw[j] = j * 8 + lane / 8;
      const int p = lane % 8;
      const int64_t c = col0 + (FP8 ? (p ^ swz<true>(kw[j])) * 16 : ((p / 2) ^ swz<false>(kw[j])) * 16 + p % 2 * 8);
      ow[j] = c < a.d_out ? kw[j] * ldw + (int32_t)c * WE : INT32_MIN;
    }
  }
  const int tx = FP8 ? lane / 2 : lane / 4, kx = FP8 ? lane % 2 * 16 : lane % 4 * 8;
  const int32_t ox = tx < toks ? tx * ldx + kx * XE : INT32_MIN;
  auto issue = [&](int s) {
    char* st = ring + (s % C::RING) * C::STEP;
    const int k0 = s * 32;
    const int left = s < s_hi ? d_in - k0 : 0;  // steps past the slice load zeros
#pragma unroll
    for (int j = 0; j < 4; ++j)
      lds_dma16(rw, st + j * 1024, kw[j] < left && ow[j] != INT32_MIN ? (int32_t)(ow[j] + (uint32_t)k0 * (uint32_t)ldw) : INT32_MIN, 0);
    lds_dma16(rx, st + 4096, kx < left && ox != INT32_MIN ? ox + k0 * XE : INT32_MIN, 0);
  };
  for (int i = 0; i < C::RING; ++i) issue(s_lo + i);
  for (int s = s_lo; s < s_hi; ++s) {
    wait_loads<(C::RING - 1) * C::NI>();
    const char* st = ring + (s % C::RING) * C::STEP;
    const char* xp = st + 4096;
    if constexpr (FP8 && !AD) {
      const long x = *reinterpret_cast<const long*>(xp + c16 * 32 + q * 8);
      const int kr = 8 * q + c16 / 2;
#pragma unroll
      for (int nb = 0; nb < C::NB; ++nb) {
        const long w = __builtin_bit_cast(long, lds_read_tr8(st + kr * 128 + (nb ^ swz<true>(kr)) * 16 + c16 % 2 * 8));
        acc[nb] = __builtin_amdgcn_mfma_f32_16x16x32_fp8_fp8(w, x, acc[nb], 0, 0, 0);
      }
    } else {
      bf16x8 x;
      if constexpr (FP8)
        x = as_bf16x8(bf16_of_e4m3(*reinterpret_cast<const u32x2*>(xp + c16 * 32 + q * 8)));
      else
        x = as_bf16x8(*reinterpret_cast<const u32x4*>(xp + c16 * 64 + q * 16));
      const int kr = 8 * q + c16 / 4, rb = AD ? 2 * R : 128;
#pragma unroll
      for (int nb = 0; nb < 4; ++nb) {
        if (AD && nb * 16 >= R) break;  // uniform (rank 8: one block, its upper columns dropped)
        const char* p = st + kr * rb + (AD ? nb : nb ^ swz<false>(kr)) * 32 + c16 % 4 * 8;
        const u32x2 lo = lds_read_tr16(p), hi = lds_read_tr16(p + 4 * rb);
        acc[nb] = mfma16x16x32(as_bf16x8(u32x4{lo[0], lo[1], hi[0], hi[1]}), x, acc[nb]);
      }
    }
    wait_lds();  // this step's slot is free
    issue(s + C::RING);
  }
  wait_loads<0>();
}

// Sums the waves' acc[g] (g < n <= G) through LDS in a fixed order and hands out
// the sums of block g, row t, columns 4 q ..: put(g, t, q, sum).
template <int G, int NB, typename Put>
__device__ __forceinline__ void sum_waves(f32x4 (&acc)[NB], char* lds, int n, Put put) {
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  f32x4* part = reinterpret_cast<f32x4*>(lds);  // [wave][G][64]
  __syncthreads();  // the ring is no longer read
#pragma unroll
  for (int g = 0; g < G; ++g) part[(w * G + g) * 64 + lane] = acc[g];
  __syncthreads();
  for (int u = tid; u < n * 64; u += ST_W * 64) {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < ST_W; ++v) s += part[v * G * 64 + u];
    put(u / 64, u % 16, u / 16 % 4, s);
  }
}

// Workspace of a product over k slices: sums of W [ks][T][d_out], then of the
// adapters [ksa][T][rank], fp32.
struct SlabPlan {
  int n_ct, n_tt, ks;  // column tiles of W (0: the adapter rows alone), row tiles, k slices
  int ksa;             // k slices of the adapter rows (0: none)
  int turns;           // slabs that share the agents of a row tile and slice
  int64_t h_at;        // fp32 words before their sums
};

template <bool FP8>
__global__ void __launch_bounds__(ST_W * 64) stream_kernel(const ProjectArgs a, const SlabPlan p) {
  using C = Stream<FP8>;
  __shared__ __attribute__((aligned(1024))) char lds[ST_W * C::RING * C::STEP];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int T = (int)a.T, nk = (int)((a.d_in + 31) / 32);
  char* ring = lds + w * C::RING * C::STEP;
  const int n_main = p.n_ct * p.ks;
  f32x4 acc[C::NB];
#pragma unroll
  for (int i = 0; i < C::NB; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  if ((int)blockIdx.x < n_main) {
    const int ct = blockIdx.x % p.n_ct, ki = blockIdx.x / p.n_ct, parts = p.ks * ST_W, part = ki * ST_W + w;
    const int64_t c0 = (int64_t)ct * C::CW;
    stream_steps<FP8, false>(a, ring, T, c0, (int)((int64_t)nk * part / parts), (int)((int64_t)nk * (part + 1) / parts), acc);
    float* out = static_cast<float*>(a.ws) + (int64_t)ki * T * a.d_out;
    sum_waves<C::NB>(acc, lds, C::NB, [&](int g, int t, int q, f32x4 s) {
      const int64_t c = c0 + g * 16 + 4 * q;
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
  stream_steps<FP8, true>(a, ring, T, (int64_t)ag * a.rank, (int)((int64_t)nk * part / parts),
                          (int)((int64_t)nk * (part + 1) / parts), acc);
  float* out = static_cast<float*>(a.ws) + p.h_at + (int64_t)ki * T * a.rank;
  sum_waves<4>(acc, lds, (a.rank + 15) / 16, [&](int g, int t, int q, f32x4 s) {
    const int j = g * 16 + 4 * q;
    if (j < a.rank && (mine >> t & 1)) *reinterpret_cast<f32x4*>(out + t * a.rank + j) = s;
  });
}

// Y of 256 columns of a row, four columns a lane: each of four waves takes a
// quarter of the ranks and every fourth k slice, its loads in flight together (8 x
// 5120 x 5120 in e4m3, rank 64: 14.6 -> 13.8 us for the two kernels)
// (lanes past the last column read the row's first ones); their sums are added
// in a fixed order.
template <int R>
__global__ void __launch_bounds__(256) join_kernel(const ProjectArgs a, const SlabPlan p) {
  constexpr int RW = R / 4;
  __shared__ f32x4 part[3][64];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t t = blockIdx.y, c0 = (int64_t)blockIdx.x * 256 + lane * 4, T = a.T;
  const float* P = static_cast<const float*>(a.ws);
  const bool ok = c0 < a.d_out;
  const int64_t c = ok ? c0 : 0;
  const int ag = a.n_agents > 0 ? a.agent[t] : -1;
  const bool lr = ag >= 0 && ag < a.n_agents;  // uniform
  const float xs = a.x_scale != nullptr ? a.x_scale[t] : 1.f;
  f32x4 wsc = {1.f, 1.f, 1.f, 1.f};
  if (a.x_scale != nullptr) wsc = ld_scales(a.w_scale + c) * xs;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  for (int k = w; k < p.ks; k += 16) {
    f32x4 u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (k + 4 * i < p.ks) u[i] = *reinterpret_cast<const f32x4*>(P + ((k + 4 * i) * T + t) * a.d_out + c);
    }
    v += (u[0] + u[1]) + (u[2] + u[3]);
  }
  v *= wsc;
  if (lr) {
    u32x2 b[RW];
    const uint16_t* B = a.B + ((int64_t)ag * R + w * RW) * a.d_out + c;
#pragma unroll
    for (int j = 0; j < RW; ++j) b[j] = *reinterpret_cast<const u32x2*>(B + j * a.d_out);
    const float* H = P + p.h_at + t * R + w * RW + lane % RW;
    float h = 0.f;
    for (int k = 0; k < p.ksa; k += 8) {
      float u[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = k + i < p.ksa ? H[(k + i) * T * R] : 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) h += u[i];
    }
    h *= xs;
#pragma unroll
    for (int j = 0; j < RW; ++j) {
      const float hj = readlane_f(h, j);
      v[0] += hj * bf_lo(b[j][0]);
      v[1] += hj * bf_hi(b[j][0]);
      v[2] += hj * bf_lo(b[j][1]);
      v[3] += hj * bf_hi(b[j][1]);
    }
  }
  if (w > 0) part[w - 1][lane] = v;
  __syncthreads();
  if (w > 0 || !ok) return;
#pragma unroll
  for (int i = 0; i < 3; ++i) v += part[i][lane];
  *reinterpret_cast<u32x2*>(a.Y + t * a.ld_y + c) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
}

// Column tiles, and k slices so that all workgroups run at once: those of W one
// a CU, those of the adapters (as long as W's at most) beside them.  Up to 4 rows
// two a CU (4096 x 4096: 11.3 us against 12.3 for one row, 15.2 against 13.5 for
// 16: the slices' sums are written and read again).
SlabPlan stream_plan(int64_t T, int64_t d_in, int64_t d_out, int n_agents, bool fp8, int cus) {
  SlabPlan p{};
  const int cw = fp8 ? 128 : 64, ad = (int)(T < n_agents ? T : n_agents);
  p.n_ct = (int)((d_out + cw - 1) / cw);
  const int64_t steps = (d_in + 31) / 32;
  int most = (int)(steps / ST_W);  // a step a wave at least
  if (most < 1) most = 1;
  p.ks = (T <= 4 ? 2 * cus : cus) / p.n_ct;
  p.ks = p.ks < 1 ? 1 : (p.ks > most ? most : p.ks);
  while (p.ks > 1 && (p.n_ct + ad) * p.ks > 2 * cus) --p.ks;
  p.ksa = ad > 0 ? p.ks : 0;
  p.n_tt = 1;
  p.h_at = (int64_t)p.ks * T * d_out;
  return p;
}
size_t plan_bytes(int64_t T, int rank, const SlabPlan& p) {
  return ((size_t)p.h_at + (size_t)p.ksa * (size_t)T * (size_t)rank) * 4;
}

hipError_t launch_join(const ProjectArgs& a, const SlabPlan& p, hipStream_t st) {
  const dim3 grid((unsigned)((a.d_out + 255) / 256), (unsigned)a.T);
  switch (a.rank) {
    case 8: hipLaunchKernelGGL((join_kernel<8>), grid, dim3(256), 0, st, a, p); break;
    case 16: hipLaunchKernelGGL((join_kernel<16>), grid, dim3(256), 0, st, a, p); break;
    case 32: hipLaunchKernelGGL((join_kernel<32>), grid, dim3(256), 0, st, a, p); break;
    default: hipLaunchKernelGGL((join_kernel<64>), grid, dim3(256), 0, st, a, p); break;
  }
  return hipGetLastError();
}

template <bool FP8>
hipError_t launch_stream(const ProjectArgs& a, hipStream_t st) {
  const SlabPlan p = stream_plan(a.T, a.d_in, a.d_out, a.n_agents, FP8, a.cus);
  const int64_t blocks = (int64_t)p.n_ct * p.ks + (int64_t)p.ksa * a.T;
  hipLaunchKernelGGL((stream_kernel<FP8>), dim3((unsigned)blocks), dim3(ST_W * 64), 0, st, a, p);
  if (const hipError_t e = hipGetLastError()) return e;
  return launch_join(a, p, st);
}

// ---------------------------------------------------------------------------
// Many rows: X A_a of every row first, then X W in tiles with the expanded
// adapter rows added as each tile is written.
//
// Slabs: 64 rows x 128 bytes of weight columns x a slice of k, summed in fp32 in
// the workspace.  They form the adapter rows X A_a for the tiles, and for calls
// of a few hundred rows X W beside them, joined by the kernel above.  Stages (128
// bytes of k) come through a ring in LDS with direct loads that all waves issue;
// weight rows lie in 16-column units XOR-swizzled by row.
//
// Of A a workgroup takes as many of its rows' agents at a time as 64 columns
// hold; rows with more take turns, several workgroups at once.  A's rows are
// short (2 r bytes, and a CU takes one request of up to 128 bytes every other
// cycle), so A bounds it: 64 rows share each of them.
constexpr int SL_T = 64, SL_NB = 4;  // rows; 16-column blocks of A


template <bool FP8>
struct Slab {
  static constexpr int E = FP8 ? 1 : 2, KS = 128 / E, KK = KS / 32;  // bytes of an element; k and MFMA steps of a stage
  static constexpr int CW = FP8 ? 128 : 64;                          // columns of W
  static constexpr int XB = SL_T * 128, AB = KS * 128;               // bytes of X and of weights
  static constexpr int NA = AB / 8192, NI = 1 + NA;                  // a wave's loads of weights, and all
  // Two workgroups a CU: one's start and end beside the other's loads (adapter
  // rows of 4096: 11.3 us against 14.1 with one and twice the stages).
  static constexpr int STEP = XB + AB, RING = FP8 ? 3 : 5;
  static_assert(RING * STEP <= 80 * 1024, "LDS");
};

// A slab's stages s_lo .. s_hi of this wave: load(s) issues stage s's X, then its
// weights; use(stage) multiplies.
template <bool FP8, typename IssueX, typename IssueW, typename Use>
__device__ __forceinline__ void slab_stages(int s_lo, int s_hi, IssueX issue_x, IssueW issue_w, Use use) {
  using C = Slab<FP8>;
  __syncthreads();  // the stages of the agents before are read
  for (int i = 0; i < C::RING - 1; ++i) issue_x(s_lo + i, i);
  for (int i = 0; i < C::RING - 1; ++i) issue_w(s_lo + i, i);
  int slot = 0, last = C::RING - 1;
  for (int s = s_lo; s < s_hi; ++s) {
    // After stage s came the weights of the RING - 2 first stages, or all of as many.
    if (s < s_lo + C::RING - 1) wait_loads<(C::RING - 2) * C::NA>();
    else wait_loads<(C::RING - 2) * C::NI>();
    wait_lds();
    __builtin_amdgcn_s_barrier();  // stage s has landed, stage s - 1 is read
    asm volatile("" ::: "memory");
    issue_x(s + C::RING - 1, last);
    issue_w(s + C::RING - 1, last);
    use(slot);
    last = slot;
    slot = slot + 1 == C::RING ? 0 : slot + 1;
  }
  wait_loads<0>();
}

template <bool FP8>
__global__ void __launch_bounds__(512, 4) slab_kernel(const ProjectArgs a, const SlabPlan p) {
  using C = Slab<FP8>;
  constexpr int E = C::E;
  __shared__ __attribute__((aligned(1024))) char ring[C::RING * C::STEP];
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, q = lane >> 4, c16 = lane & 15;
  // Workgroup L runs on XCD L % 8: each takes an eighth of the slabs of W, row
  // tiles fastest (they share columns), then those of the adapters follow.
  const int n_main = p.n_ct * p.n_tt * p.ks, per = (n_main + 7) / 8, L = (int)blockIdx.x;
  const bool ad = L >= 8 * per;
  const int m = ad ? L - 8 * per : L % 8 * per + L / 8;
  if (!ad && m >= n_main) return;  // uniform over the workgroup
  const int ks = ad ? p.ksa : p.ks;
  // First turns first, so that those of workgroups without an agent delay none
  // (2048 rows of 5120 x 5120 in e4m3, rank 64: 75.8 us turns inside, 70.7).
  const int n_rt = (int)((a.T + SL_T - 1) / SL_T) * p.ksa, mt = ad ? m % n_rt : 0;
  const int tt = __builtin_amdgcn_readfirstlane(ad ? mt / p.ksa : m % p.n_tt), ct = ad ? 0 : m / p.n_tt % p.n_ct;
  const int ki = __builtin_amdgcn_readfirstlane(ad ? mt % p.ksa : m / p.n_tt / p.n_ct);
  const int64_t t0 = (int64_t)tt * SL_T;
  const int toks = (int)(a.T - t0 < SL_T ? a.T - t0 : (int64_t)SL_T), d_in = (int)a.d_in;
  const int nk = (d_in + C::KS - 1) / C::KS;
  const int s_lo = (int)((int64_t)nk * ki / ks), s_hi = (int)((int64_t)nk * (ki + 1) / ks);
  const int32_t ldx = (int32_t)(a.ld_x * E);
  const i32x4 rx = buffer_rsrc(static_cast<const char*>(a.X) + t0 * ldx, (toks - 1) * ldx + d_in * E);
  // X: rows 8 wv .. of this wave, 16-byte chunks XOR-swizzled by row.
  const int xr = 8 * wv + lane / 8, kx = ((lane % 8) ^ ((xr >> 1) & 7)) * 16 / E;
  const int32_t ox = xr < toks ? xr * ldx + kx * E : INT32_MIN;
  auto issue_x = [&](int s, int slot) {
    const int k0 = s * C::KS, left = s < s_hi ? d_in - k0 : 0;
    lds_dma16(rx, ring + slot * C::STEP + wv * 1024, kx < left && ox != INT32_MIN ? ox + k0 * E : INT32_MIN, 0);
  };
  // Weights: rows 8 (8 j + wv) .. of 128 bytes, from byte offsets ow of rows kw.
  int32_t kw[C::NA], ow[C::NA];
  auto issue_w = [&](i32x4 r, int32_t ld, int s, int slot) {
    const int k0 = s * C::KS, left = s < s_hi ? d_in - k0 : 0;
#pragma unroll
    for (int j = 0; j < C::NA; ++j)
      lds_dma16(r, ring + slot * C::STEP + C::XB + (8 * j + wv) * 1024,
                kw[j] < left && ow[j] != INT32_MIN ? (int32_t)((uint32_t)ow[j] + (uint32_t)k0 * (uint32_t)ld) : INT32_MIN, 0);
  };
  // This wave's rows 16 tb ..; of bf16 weights blocks cb and cb + 2, of e4m3 four from 4 cb.
  const int tb = wv & 3, cb = wv >> 2, row = 16 * tb + c16, xs = (row >> 1) & 7;
  const int64_t t = t0 + row;
  // The MFMAs of a stage with bf16 weights: all fragments first, one wait for them.
  auto use16 = [&](int slot, f32x4 (&acc)[2]) {
    const char* st = ring + slot * C::STEP;
    bf16x8 x[C::KK], w[C::KK][2];
#pragma unroll
    for (int kk = 0; kk < C::KK; ++kk) {
      const char* xp = st + row * 128;
      if constexpr (FP8)
        x[kk] = as_bf16x8(bf16_of_e4m3(*reinterpret_cast<const u32x2*>(xp + ((2 * kk + q / 2) ^ xs) * 16 + q % 2 * 8)));
      else
        x[kk] = as_bf16x8(*reinterpret_cast<const u32x4*>(xp + ((4 * kk + q) ^ xs) * 16));
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = 8 * q + c16 / 4;  // row r + 4 and those 32 further swizzle alike
        const char* wp = st + C::XB + (32 * kk + r) * 128 + ((cb + 2 * i) ^ swz<false>(r)) * 32 + c16 % 4 * 8;
        const u32x2 lo = lds_read_tr16(wp), hi = lds_read_tr16(wp + 512);
        w[kk][i] = as_bf16x8(u32x4{lo[0], lo[1], hi[0], hi[1]});
      }
    }
#pragma unroll
    for (int kk = 0; kk < C::KK; ++kk)
#pragma unroll
      for (int i = 0; i < 2; ++i) acc[i] = mfma16x16x32(w[kk][i], x[kk], acc[i]);
  };

  if (!ad) {
    const int64_t c0 = (int64_t)ct * C::CW;
    const int32_t ldw = (int32_t)(a.d_out * E);
    const i32x4 rw = buffer_rsrc(a.W, d_in * ldw);
#pragma unroll
    for (int j = 0; j < C::NA; ++j) {
      const int k = (8 * j + wv) * 8 + lane / 8, c = FP8 ? ((lane % 8) ^ swz<true>(k)) * 16 : ((lane % 8 / 2) ^ swz<false>(k)) * 16 + lane % 2 * 8;
      kw[j] = k;
      ow[j] = c0 + c < a.d_out ? k * ldw + (int32_t)(c0 + c) * E : INT32_MIN;
    }
    auto issue = [&](int s, int slot) { issue_w(rw, ldw, s, slot); };
    float* out = static_cast<float*>(a.ws) + ((int64_t)ki * a.T + t) * a.d_out + c0;
    if constexpr (!FP8) {
      f32x4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
      slab_stages<FP8>(s_lo, s_hi, issue_x, issue, [&](int slot) { use16(slot, acc); });
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int c = (cb + 2 * i) * 16 + 4 * q;
        if (row < toks && c0 + c < a.d_out) *reinterpret_cast<f32x4*>(out + c) = acc[i];
      }
    } else {
      f32x4 acc[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      slab_stages<FP8>(s_lo, s_hi, issue_x, issue, [&](int slot) {
        const char* st = ring + slot * C::STEP;
        long x[C::KK], w[C::KK][4];
#pragma unroll
        for (int kk = 0; kk < C::KK; ++kk) {
          x[kk] = *reinterpret_cast<const long*>(st + row * 128 + ((2 * kk + q / 2) ^ xs) * 16 + q % 2 * 8);
          const int r = 32 * kk + 8 * q + c16 / 2;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            w[kk][i] = __builtin_bit_cast(long, lds_read_tr8(st + C::XB + r * 128 + ((4 * cb + i) ^ swz<true>(r)) * 16 + c16 % 2 * 8));
        }
#pragma unroll
        for (int kk = 0; kk < C::KK; ++kk)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_fp8_fp8(w[kk][i], x[kk], acc[i], 0, 0, 0);
      });
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = (4 * cb + i) * 16 + 4 * q;
        if (row < toks && c0 + c < a.d_out) *reinterpret_cast<f32x4*>(out + c) = acc[i];
      }
    }
    return;
  }

  // ---- adapter rows ------------------------------------------------------------
  const int R = a.rank, rp = R < 16 ? 16 : R;
  const int ag = lane < toks ? a.agent[t0 + lane] : -1, own = row < toks ? a.agent[t] : -1;
  uint64_t todo = __ballot(ag >= 0 && ag < a.n_agents);  // the same in every wave
  float* H = static_cast<float*>(a.ws) + p.h_at + ((int64_t)ki * a.T + t0) * R;
  const int32_t lda = (int32_t)((int64_t)a.n_agents * R * 2);
  const i32x4 ra = buffer_rsrc(a.A, d_in * lda);
  for (int turn = 0; todo != 0; ++turn) {
    // The agents of blocks 0 .. 3 (-1: none).
    int id[SL_NB];
#pragma unroll
    for (int b = 0; b < SL_NB; ++b) {
      if (b * 16 % rp != 0) {  // another block of the same agent
        id[b] = b > 0 ? id[b - 1] : -1;
        continue;
      }
      id[b] = todo != 0 ? __builtin_amdgcn_readlane(ag, __builtin_ctzll(todo)) : -1;
      if (todo != 0) todo &= ~__ballot(ag == id[b]);
    }
    if (turn % p.turns != m / n_rt) continue;  // uniform
#pragma unroll
    for (int j = 0; j < C::NA; ++j) {
      const int k = (8 * j + wv) * 8 + lane / 8, blk = (lane % 8 / 2) ^ swz<false>(k), c = blk * 16 % rp + lane % 2 * 8;
      int mine = id[0];
#pragma unroll
      for (int i = 1; i < SL_NB; ++i) mine = blk == i ? id[i] : mine;
      kw[j] = k;
      ow[j] = mine >= 0 && c < R ? (int32_t)((uint32_t)k * (uint32_t)lda + (uint32_t)((mine * R + c) * 2)) : INT32_MIN;  // (past d_in: wraps, unread)
    }
    f32x4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    slab_stages<FP8>(s_lo, s_hi, issue_x, [&](int s, int slot) { issue_w(ra, lda, s, slot); }, [&](int slot) { use16(slot, acc); });
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int j = (cb + 2 * i) * 16 % rp + 4 * q;
      if (id[cb + 2 * i] >= 0 && own == id[cb + 2 * i] && j < R) *reinterpret_cast<f32x4*>(H + row * R + j) = acc[i];
    }
  }
}

template <bool FP8>
hipError_t launch_slabs(const ProjectArgs& a, const SlabPlan& p, hipStream_t st) {
  const int64_t n_main = (int64_t)p.n_ct * p.n_tt * p.ks, n_ad = (a.T + SL_T - 1) / SL_T * p.ksa * p.turns;
  hipLaunchKernelGGL((slab_kernel<FP8>), dim3((unsigned)((n_main + 7) / 8 * 8 + n_ad)), dim3(512), 0, st, a, p);
  return hipGetLastError();
}

// k slices of the adapter rows alone: enough workgroups for the CUs, two stages
// each at least; no more than 256 sums a row, which every tile of the row adds.
int shrink_slices(int64_t T, int64_t d_in, int rank, int cus) {
  const int64_t rows = (T + SL_T - 1) / SL_T, most = d_in / 256, sums = 256 / rank;
  int64_t k = cus / rows;
  k = k > most ? most : k;
  k = k > sums ? sums : k;
  return (int)(k < 1 ? 1 : (k > 8 ? 8 : k));
}

// Turns: as many as 64 rows' agents may need and as `room` workgroups, which run
// at once anyhow, hold for `each` row tile and slice.  (24 rows of 4096 x 4096 in
// e4m3 of as many agents of rank 64: two turns 19.9 us, eight 15.8; 256 rows 64.6
// and 27.7.  Workgroups without a turn that do not fit cost: 4096 rows with eight
// 157 us against 127.)
int slab_turns(int n_agents, int rank, int64_t room, int64_t each) {
  const int64_t own = SL_NB * 16 / (rank < 16 ? 16 : rank), need = ((n_agents < SL_T ? n_agents : SL_T) + own - 1) / own;
  int64_t n = room / each;
  n = n > need ? need : n;
  return (int)(n < 1 ? 1 : (n > 8 ? 8 : n));
}

typedef int i32x8 __attribute__((ext_vector_type(8)));

template <bool FP8>
struct Mma {
  static constexpr int FR = FP8 ? 8 : 4;  // registers of an operand
  typedef uint32_t Frag __attribute__((ext_vector_type(FR)));
  // 32x32 outputs over 16 k (bf16) or 64 (e4m3: sums of eight products cut what
  // is below 2^-13 of the largest, then fp32).
  static __device__ __forceinline__ f32x16 mma(Frag w, Frag x, f32x16 c) {
    if constexpr (FP8)
      return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(__builtin_bit_cast(i32x8, w), __builtin_bit_cast(i32x8, x), c, 0, 0, 0,
                                                             0, 0, 0);
    else
      return mfma32x32x16(as_bf16x8(w), as_bf16x8(x), c);
  }
};

// Column block b of weight row k is stored at b ^ swz(k), of NP blocks a row:
// bf16 reads take 4 rows of 64 bytes together, e4m3 reads 8 rows of 32; odd
// rows of blocks spread over the banks by themselves.
template <bool FP8, int NP>
__device__ __forceinline__ int swz_blocks(int k) {
  if (NP % 2 != 0) return 0;
  if (FP8) return NP % 8 == 0 ? k & 7 : (NP % 4 == 0 ? (k >> 1) & 3 : (k >> 2) & 1);
  return NP % 4 == 0 ? k & 3 : (k >> 1) & 1;
}

// What a wave does with its sums acc[cb][tb][j]: column cw + 32 cb + (j / 4) * 8
// + 4 h + j % 4, token tw + 32 tb + l32.
//
// The scales of e4m3.
template <int CB, int TB>
__device__ __forceinline__ void scale_tile(const ProjectArgs& a, f32x16 (&acc)[CB][TB], int64_t tw, int64_t cw) {
  const int lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5;
  float xsc[TB];
#pragma unroll
  for (int tb = 0; tb < TB; ++tb) xsc[tb] = tw + 32 * tb + l32 < a.T ? a.x_scale[tw + 32 * tb + l32] : 1.f;
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int jg = 0; jg < 4; ++jg) {
      const int64_t c = cw + 32 * cb + jg * 8 + 4 * h;
      f32x4 wsc = {0.f, 0.f, 0.f, 0.f};
      if (c < a.d_out) wsc = ld_scales(a.w_scale + c);
#pragma unroll
      for (int tb = 0; tb < TB; ++tb)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[cb][tb][4 * jg + i] *= xsc[tb] * wsc[i];
    }
}

// The expanded adapter rows: all waves of the tile (TT tokens from t0, NP column
// blocks from c0) together, four of its agents at a time (three where LDS holds no
// more).  The tile's rows X A_a are summed over the k slices, split into two bf16
// parts and put into LDS, and each agent's rows of B_a beside them, laid out as
// the weights are.  A product is added to the tokens of its agent alone, so that
// what is infinite or NaN in an adapter stays in the rows that use it.  The second
// part costs 4096 x 4096 x 4096 in bf16 nothing at rank 16 and 3 of 146 us at rank
// 64 where rows come in runs, 16 of 263 at rank 16 where 32 agents mix; 2048 x 5120 x
// 5120 in e4m3, rank 64, 0.5 of 67.
constexpr int EX_A = 4;  // agents at a time
constexpr int EX_LDS = 160 * 1024;

template <int NP, int TT>
constexpr int expand_agents(int rp) {  // of (padded) rank rp
  return (EX_LDS - TT * 256) / (rp * NP * 64) < EX_A ? (EX_LDS - TT * 256) / (rp * NP * 64) : EX_A;
}
template <int NP, int TT>
constexpr int expand_bytes = TT * 256 + expand_agents<NP, TT>(64) * 64 * NP * 64;

// v = hi + lo as bf16, to 2^-17 of it.  An infinity (or NaN) is hi's alone.
__device__ __forceinline__ void split_bf16(f32x4 v0, f32x4 v1, u32x4& hi, u32x4& lo) {
  hi = u32x4{pack_bf16(v0[0], v0[1]), pack_bf16(v0[2], v0[3]), pack_bf16(v1[0], v1[1]), pack_bf16(v1[2], v1[3])};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float a = j < 2 ? v0[2 * j] : v1[2 * j - 4], b = j < 2 ? v0[2 * j + 1] : v1[2 * j - 3];
    const uint32_t ha = hi[j] << 16, hb = hi[j] & 0xffff0000u;
    lo[j] = pack_bf16((ha & 0x7f800000u) == 0x7f800000u ? 0.f : a - __uint_as_float(ha),
                      (hb & 0x7f800000u) == 0x7f800000u ? 0.f : b - __uint_as_float(hb));
  }
}

template <bool FP8, int NP, int TT, int CB, int TB>
__device__ __forceinline__ void expand_tile(const ProjectArgs& a, int ksa, f32x16 (&acc)[CB][TB], char* lds, int64_t t0, int tw,
                                            int64_t c0, int cb0) {
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31;
  const int R = a.rank, rp = R < 16 ? 16 : R, nc = rp / 8;  // ranks with padding; 16-byte chunks of a row
  // Agents of the tile's tokens (four or two a lane) and of this wave's.
  constexpr int NT = TT / 64;
  int all[NT], ag[TB];
  uint64_t todo[NT], any = 0;  // tokens whose agent is still to come, the same in every wave
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int64_t t = t0 + 64 * i + lane;
    all[i] = t < a.T ? a.agent[t] : -1;
    todo[i] = __ballot(all[i] >= 0 && all[i] < a.n_agents);
    any |= todo[i];
  }
  if (any == 0) return;
#pragma unroll
  for (int tb = 0; tb < TB; ++tb) ag[tb] = t0 + tw + 32 * tb + l32 < a.T ? a.agent[t0 + tw + 32 * tb + l32] : -1;
  auto chunk = [&](int r, int c) {  // where chunk c of row r lies
    return r * rp * 2 + (nc == 2 ? c : (nc == 4 ? c ^ ((r >> 2) & 3) : c ^ ((r >> 1) & 7))) * 16;
  };
  constexpr int part = TT * 128;  // the rows' low parts lie this far behind (room for rank 64)
  auto rows_to_lds = [&]() {
    // 16-byte chunk u of the tile's rows is thread u % 512's, two at a time.
    const float* H = static_cast<const float*>(a.ws) + t0 * R;
    for (int u0 = tid; u0 < TT * nc; u0 += 1024) {
      f32x4 v[2][2];
      bool ok[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int u = u0 + 512 * i, r = u / nc;
        const int own = u < TT * nc && t0 + r < a.T ? a.agent[t0 + r] : -1;
        ok[i] = own >= 0 && own < a.n_agents && u % nc * 8 < R;
        v[i][0] = v[i][1] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
#pragma unroll 4
      for (int k = 0; k < ksa; ++k)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (ok[i]) {
            const int u = u0 + 512 * i;
            const f32x4* p = reinterpret_cast<const f32x4*>(H + k * a.T * R + (u / nc) * R + u % nc * 8);
            v[i][0] += p[0];
            v[i][1] += p[1];
          }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int u = u0 + 512 * i;
        if (u >= TT * nc) break;
        if constexpr (FP8) {
          const float xsc = ok[i] ? a.x_scale[t0 + u / nc] : 1.f;
          v[i][0] *= xsc;
          v[i][1] *= xsc;
        }
        u32x4 hi, lo;
        split_bf16(v[i][0], v[i][1], hi, lo);
        *reinterpret_cast<u32x4*>(lds + chunk(u / nc, u % nc)) = hi;
        *reinterpret_cast<u32x4*>(lds + part + chunk(u / nc, u % nc)) = lo;
      }
    }
  };
  constexpr int WRB = NP * 64;  // bytes of a row of B
  char* bs = lds + 2 * part;
  static_assert(expand_agents<NP, TT>(32) == EX_A, "fewer at rank 64 alone");
  const int most = rp == 64 ? expand_agents<NP, TT>(64) : EX_A;
  for (bool first = true; any != 0; first = false) {
    int id[EX_A] = {-1, -1, -1, -1};
#pragma unroll
    for (int g = 0; g < EX_A; ++g) {
      if (g >= most) break;
#pragma unroll
      for (int i = NT - 1; i >= 0; --i)
        if (todo[i] != 0) id[g] = __builtin_amdgcn_readlane(all[i], __builtin_ctzll(todo[i]));
      any = 0;
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        todo[i] &= ~__ballot(all[i] == id[g]);
        any |= todo[i];
      }
    }
#pragma unroll
    for (int g = 0; g < EX_A; ++g) {
      if (id[g] < 0) break;
      const i32x4 rb = buffer_rsrc(a.B + (int64_t)id[g] * R * a.d_out, (int32_t)(R * a.d_out * 2));
      int ln = lane;  // (as below)
      asm volatile("" : "+v"(ln));
      for (int i = wv; i < rp * NP / 16; i += 8) {
        const int b = i * 1024 + ln * 16, k = b / WRB, p = b % WRB / 64, in = b % 64 / 2;
        const int64_t col = c0 + (p ^ swz_blocks<false, NP>(k)) * 32 + in;
        lds_dma16(rb, bs + g * rp * WRB + i * 1024, k < R && col < a.d_out ? (int32_t)((k * a.d_out + col) * 2) : INT32_MIN, 0);
      }
    }
    if (first) rows_to_lds();
    wait_loads<0>();
    __syncthreads();  // the rows and these agents are in LDS
#pragma unroll
    for (int g = 0; g < EX_A; ++g) {
      if (id[g] < 0) break;
      // Addresses formed anew for each agent: those of all, kept, spill.
      int ln = lane;
      asm volatile("" : "+v"(ln));
      const int r0 = tw + (ln & 31), hn = ln >> 5, wk = 8 * hn + (ln & 15) / 4, ws = swz_blocks<false, NP>(wk);
      const int wo = wk * WRB + (ln >> 4 & 1) * 32 + (ln & 3) * 8;
      if constexpr (CB * TB >= 8) {
        // 128 sums a lane leave room for one block's fragments at a time (more
        // spills: 34 us against 23 at 4096 x 256 x 4096).
#pragma unroll
        for (int tb = 0; tb < TB; ++tb) {
          const bool mine = ag[tb] == id[g];
          if (__ballot(mine) == 0) continue;
          const bool whole = __ballot(mine || t0 + tw + 32 * tb + l32 >= a.T) == ~0ull;
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) {
            f32x16 sum;
#pragma unroll
            for (int j = 0; j < 16; ++j) sum[j] = whole ? acc[cb][tb][j] : 0.f;
            for (int kk = 0; kk < rp / 16; ++kk) {
              const char* p = bs + g * rp * WRB + wo + ((cb0 + cb) ^ ws) * 64 + 16 * kk * WRB;
              const u32x2 lo = lds_read_tr16(p), hi = lds_read_tr16(p + 4 * WRB);
              const char* hp = lds + chunk(r0 + 32 * tb, 2 * kk + hn);
              u32x4 fh = *reinterpret_cast<const u32x4*>(hp), fl = *reinterpret_cast<const u32x4*>(hp + part);
              if (!mine) fh = fl = u32x4{0u, 0u, 0u, 0u};
              const bf16x8 fb = as_bf16x8(u32x4{lo[0], lo[1], hi[0], hi[1]});
              sum = mfma32x32x16(fb, as_bf16x8(fl), sum);
              sum = mfma32x32x16(fb, as_bf16x8(fh), sum);
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) acc[cb][tb][j] = whole ? sum[j] : (mine ? acc[cb][tb][j] + sum[j] : acc[cb][tb][j]);
          }
        }
        continue;
      }
      auto add = [&](auto KR) {  // KR steps of 16 ranks
        constexpr int kr = decltype(KR)::value;
        const char* rows = lds + r0 * kr * 32;  // rows 32 further swizzle alike
        const int hs = (kr == 1 ? hn : (kr == 2 ? hn ^ ((r0 >> 2) & 3) : hn ^ ((r0 >> 1) & 7))) * 16;
        // Both parts of one token block at a time: those of all spill.
#pragma unroll
        for (int tb = 0; tb < TB; ++tb) {
          const bool mine = ag[tb] == id[g];
          if (__ballot(mine) == 0) continue;  // uniform
          bf16x8 fh[kr], fl[kr];
#pragma unroll
          for (int kk = 0; kk < kr; ++kk) {
            const char* p = rows + 32 * tb * kr * 32 + (hs ^ (32 * kk));  // chunk 2 kk + h
            fh[kk] = as_bf16x8(*reinterpret_cast<const u32x4*>(p));
            fl[kk] = as_bf16x8(*reinterpret_cast<const u32x4*>(p + part));
          }
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) {
            const char* p = bs + g * rp * WRB + wo + ((cb0 + cb) ^ ws) * 64;
            bf16x8 fb[kr];
#pragma unroll
            for (int kk = 0; kk < kr; ++kk) {
              const u32x2 lo = lds_read_tr16(p + 16 * kk * WRB), hi = lds_read_tr16(p + (16 * kk + 4) * WRB);
              fb[kk] = as_bf16x8(u32x4{lo[0], lo[1], hi[0], hi[1]});
            }
            f32x16 sum;
#pragma unroll
            for (int j = 0; j < 16; ++j) sum[j] = 0.f;
#pragma unroll
            for (int kk = 0; kk < kr; ++kk) sum = mfma32x32x16(fb[kk], fl[kk], sum);
#pragma unroll
            for (int kk = 0; kk < kr; ++kk) sum = mfma32x32x16(fb[kk], fh[kk], sum);
#pragma unroll
            for (int j = 0; j < 16; ++j) acc[cb][tb][j] += mine ? sum[j] : 0.f;
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      };
      if (rp == 16) add(std::integral_constant<int, 1>{});
      else if (rp == 32) add(std::integral_constant<int, 2>{});
      else add(std::integral_constant<int, 4>{});
    }
    __syncthreads();  // all is read
  }
}

// Y, by way of `lds` (this wave's, rows padded by 16 bytes), so that each row is
// written in one piece of 64 CB bytes.
template <int CB, int TB>
constexpr int store_bytes = 32 * TB * (64 * CB + 16);

template <int CB, int TB>
__device__ __forceinline__ void store_tile(const ProjectArgs& a, f32x16 (&acc)[CB][TB], char* lds, int64_t tw, int64_t cw) {
  const int lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5;
  constexpr int RB = 64 * CB + 16;
#pragma unroll
  for (int tb = 0; tb < TB; ++tb)
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int jg = 0; jg < 4; ++jg) {
        const f32x16& v = acc[cb][tb];
        *reinterpret_cast<u32x2*>(lds + (32 * tb + l32) * RB + cb * 64 + jg * 16 + h * 8) =
            u32x2{pack_bf16(v[4 * jg], v[4 * jg + 1]), pack_bf16(v[4 * jg + 2], v[4 * jg + 3])};
      }
  wait_lds();
#pragma unroll
  for (int i = 0; i < 2 * TB * CB; ++i) {
    const int u = i * 64 + lane, r = u / (4 * CB), ch = u % (4 * CB);
    const int64_t t = tw + r, c = cw + ch * 8;
    const u32x4 v = *reinterpret_cast<const u32x4*>(lds + r * RB + ch * 16);
    if (t < a.T && c < a.d_out) *reinterpret_cast<u32x4*>(a.Y + t * a.ld_y + c) = v;
  }
}

// Tiles of 256 tokens x 32 (C0 + C1) columns: eight waves, four by tokens (64
// each) and two by columns (32 C0 and 32 C1 of them), on 32x32 MFMAs.  Waves w
// and w + 4 share a SIMD, so an uneven pair loads all SIMDs alike.  The operands
// come through rings in LDS with direct loads that all waves issue: X in three
// blocks of 128 bytes of k a row (half a line costs a CU as much as a whole one:
// with 64 bytes a row the loads ran at 31 bytes a clock and bounded the kernel,
// whole lines run at 63), the weights in four half-blocks.  A wave reads the
// fragments of its next step between the MFMAs of this one.  X rows are
// XOR-swizzled in 16-byte chunks, weight rows (as in memory) in blocks of 32
// columns, so that the rows which one read takes together hit different banks.
// MFMAs bound it: 4096 x 4096 x 4096 without adapters 106 us in bf16 (1.29
// PFLOP/s) and 55 in e4m3.
constexpr int TL_T = 256;

template <bool FP8, int NP>  // NP = C0 + C1 column blocks
struct Tile {
  static constexpr int E = FP8 ? 1 : 2, KS = 64 / E, KK = FP8 ? 1 : 2;  // bytes; k and MFMA steps of a half-block
  static constexpr int CT = 32 * NP, WRB = CT * E;                      // columns; bytes of a weight row
  static constexpr int XB = TL_T * 128, WB = CT * 64;                   // bytes of a block of X, of a half-block of W
  // 1 KB loads of W of a half-block: N0 by each of waves 0 .. 3, N1 by each of
  // the others, so that every wave's count is known to the compiler (what
  // exceeds NW loads zeros past the rings).
  static constexpr int NW = WB / 1024, N0 = (NW + 7) / 8, N1 = (NW - 4 * N0 + 3) / 4;
  static constexpr int RINGS = 3 * XB + 4 * WB, LOADS = RINGS + (4 * (N0 + N1) > NW ? 1024 : 0);
  static constexpr int BYTES = LOADS > expand_bytes<NP, TL_T> ? LOADS : expand_bytes<NP, TL_T>;
};

// One wave's part of a tile: tokens t0 + 64 wt .., columns c0 + 32 cb0 .. of CB
// blocks; GRP: waves 0 .. 3 or the others.
template <bool FP8, int NP, int CB, int GRP>
__device__ __forceinline__ void tile_wave(const ProjectArgs& a, int ksa, char* lds, int64_t t0, int64_t c0, int cb0) {
  using C = Tile<FP8, NP>;
  using M = Mma<FP8>;
  using Frag = typename M::Frag;
  constexpr int E = C::E, NWL = GRP == 0 ? C::N0 : C::N1, NI = 2 + NWL;  // loads of W and of all, of this wave and half-block
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wt = wv & 3;
  const int toks = (int)(a.T - t0 < TL_T ? a.T - t0 : (int64_t)TL_T), d_in = (int)a.d_in;
  const int32_t ldw = (int32_t)(a.d_out * E), ldx = (int32_t)(a.ld_x * E);
  const i32x4 rx = buffer_rsrc(static_cast<const char*>(a.X) + t0 * ldx, (toks - 1) * ldx + d_in * E);
  const i32x4 rw = buffer_rsrc(a.W, d_in * ldw);
  lds_char* const ring = (lds_char*)lds;
  lds_char* const ringw = ring + 3 * C::XB;
  const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)ring);
  // A wave's loads of a half-block: two of the 32 of the block of X (8 rows
  // each), the other two come with the other half; and its loads of W.
  int32_t offx[4], kx, offw[NWL], kw[NWL];
  uint32_t tow[NWL];  // LDS address in slot 0
  bool in_ring[NWL];
  kx = ((lane % 8) ^ (lane / 16 + 4 * (wv & 1))) * 16 / E;  // rows 8 i + lane / 8 swizzle by (row / 2) % 8, i = wv (mod 2)
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int r = (8 * j + wv) * 8 + lane / 8;
    offx[j] = r < toks ? r * ldx + kx * E : INT32_MIN;
  }
#pragma unroll
  for (int j = 0; j < NWL; ++j) {
    const int i = (GRP == 0 ? 0 : 4 * C::N0) + 4 * j + wt, b = i * 1024 + lane * 16, k = b / C::WRB, p = b % C::WRB / (32 * E),
              in = b % (32 * E) / E;
    const int64_t col = c0 + (p ^ swz_blocks<FP8, NP>(k)) * 32 + in;
    kw[j] = k;
    in_ring[j] = i < C::NW;
    offw[j] = i < C::NW && col < a.d_out ? k * ldw + (int32_t)col * E : INT32_MIN;
    tow[j] = at + (i < C::NW ? 3 * C::XB + i * 1024 : C::RINGS);
  }
  static_assert(C::WRB % 32 == 0 && C::BYTES <= 160 * 1024 && 4 * (C::N0 + C::N1) >= C::NW, "loads, LDS");
  // Load j (0, 1) of part `part` of block `blk` of X; load j of half-block hb of
  // W.  WHOLE: all of its k are below d_in, and the k offset is scalar.
  auto issue_x = [&](auto WHOLE, int blk, int slot, int part, int j) {
    const int k0 = blk * 2 * C::KS;
    const int32_t off = part ? offx[2 + j] : offx[j];
    const uint32_t to = at + slot * C::XB + (8 * (2 * part + j) + wv) * 1024;
    if constexpr (decltype(WHOLE)::value) lds_dma16_at(rx, to, off, k0 * E);
    else lds_dma16_at(rx, to, k0 + kx < d_in && off != INT32_MIN ? off + k0 * E : INT32_MIN, 0);
  };
  auto issue_w = [&](auto WHOLE, int hb, int slot, int j) {
    if (j >= NWL) return;
    const int k0 = hb * C::KS;
    const uint32_t ks = (uint32_t)k0 * (uint32_t)ldw, to = tow[j] + (in_ring[j] ? slot * C::WB : 0);
    if constexpr (decltype(WHOLE)::value) lds_dma16_at(rw, to, offw[j], (int32_t)ks);
    else lds_dma16_at(rw, to, k0 + kw[j] < d_in && offw[j] != INT32_MIN ? (int32_t)((uint32_t)offw[j] + ks) : INT32_MIN, 0);
  };

  const int l32 = lane & 31, h = lane >> 5, grp = lane >> 4, i16 = lane & 15;
  f32x16 acc[CB][2];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
      for (int j = 0; j < 16; ++j) acc[cb][tb][j] = 0.f;
  const int xrow = 64 * wt + l32, xs = (xrow >> 1) & 7;  // rows 32 further swizzle alike
  const int xo = xrow * 128 + ((FP8 ? 2 * h : h) ^ xs) * 16;  // chunk c + i of the row lies at (xo ^ 16 c) ^ 16 i
  auto read_x = [&](int tb, const lds_char* st, int c) -> Frag {  // from chunk c of the row's block on
    const lds_char* p = st + (xo ^ (c * 16)) + 32 * tb * 128;
    if constexpr (FP8) {
      const u32x4 lo = lds_read16(p), hi = lds_read16(st + (xo ^ (c * 16 + 16)) + 32 * tb * 128);
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      return lds_read16(p);
    }
  };
  // First weight row of this lane; the rows it reads besides swizzle alike.
  const int wk = FP8 ? 32 * h + i16 / 2 : 8 * h + i16 / 4, ws = swz_blocks<FP8, NP>(wk);
  int wo[CB];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) wo[cb] = wk * C::WRB + (grp & 1) * 16 * E + (FP8 ? i16 % 2 : i16 % 4) * 8 + ((cb0 + cb) ^ ws) * (32 * E);
  auto read_w = [&](int cb, const lds_char* st, int kk) -> Frag {
    const lds_char* p = st + wo[cb] + 16 * kk * C::WRB;
    if constexpr (FP8) {
      const u32x2 v0 = lds_tr8(p), v1 = lds_tr8(p + 8 * C::WRB), v2 = lds_tr8(p + 16 * C::WRB), v3 = lds_tr8(p + 24 * C::WRB);
      return Frag{v0[0], v0[1], v1[0], v1[1], v2[0], v2[1], v3[0], v3[1]};
    } else {
      const u32x2 lo = lds_tr16(p), hi = lds_tr16(p + 4 * C::WRB);
      return Frag{lo[0], lo[1], hi[0], hi[1]};
    }
  };

  // Half-block s's turn issues half of block s / 2 + 2 of X and half-block s + 3
  // of W, one load at a time between its MFMAs (a CU takes 16 cycles for each,
  // and a wave that waits for its turn issues nothing else).  With two steps a
  // half-block the loads of W come in the first step of the next one.
  using T1 = std::true_type;
  using T0 = std::false_type;
  const int nh = (d_in + C::KS - 1) / C::KS;
#pragma unroll
  for (int j = 0; j < 2; ++j) issue_x(T0{}, 0, 0, 0, j);
#pragma unroll
  for (int j = 0; j < 2; ++j) issue_x(T0{}, 0, 0, 1, j);
#pragma unroll
  for (int j = 0; j < 2; ++j) issue_w(T0{}, 0, 0, j);
#pragma unroll
  for (int j = 0; j < 2; ++j) issue_x(T0{}, 1, 1, 0, j);
#pragma unroll
  for (int j = 0; j < 2; ++j) issue_w(T0{}, 1, 1, j);
#pragma unroll
  for (int j = 0; j < 2; ++j) issue_x(T0{}, 1, 1, 1, j);
  if constexpr (C::KK == 1) {
#pragma unroll
    for (int j = 0; j < 2; ++j) issue_w(T0{}, 2, 2, j);
  }
  wait_loads<C::KK == 1 ? 2 * NI : NI + 2>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  Frag fw[CB], fx[2][2];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) fw[cb] = read_w(cb, ringw, 0);
#pragma unroll
  for (int tb = 0; tb < 2; ++tb) fx[0][tb] = read_x(tb, ring, 0);
  int xsl = 0, wsl = 0;  // slots of the block of X and half-block of W in use
  // Half-block s = 2 b + HALF, its first X fragments in set P0.  A weight
  // fragment is read again (of the next step) as soon as its last MFMA is issued.
  auto half = [&](int s, auto HALF, auto P0, auto WHOLE) {
    constexpr int hf = decltype(HALF)::value, p0 = decltype(P0)::value;
    const int wn = (wsl + 1) & 3, xn = xsl == 2 ? 0 : xsl + 1, xl = xsl == 0 ? 2 : xsl - 1, wl = (wsl + 3) & 3;
    const lds_char* sx = ring + xsl * C::XB;
    const lds_char* sxn = hf ? ring + xn * C::XB : sx;
    const lds_char* sw = ringw + wsl * C::WB;
    const lds_char* swn = ringw + wn * C::WB;
#pragma unroll
    for (int kk = 0; kk < C::KK; ++kk) {
      const int cur = (p0 + kk) & 1, nxt = cur ^ 1;
      const bool end = kk == C::KK - 1;
      if (end) {
        // What half-block s + 1 needs was issued two turns ago or earlier and
        // has landed; every wave has used what it read of half-block s - 1, so
        // its slot of W, and the slot of X before this one, are filled again.
        wait_loads<NI>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
      }
      const lds_char* rx_ = end ? sxn : sx;
      const lds_char* rw_ = end ? swn : sw;
      const int kn = end ? 0 : kk + 1;
      const int cn = end ? (hf ? 0 : 4) : 4 * hf + 2 * (kk + 1);  // chunk of the next step
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        if (cb == 0) {
          fx[nxt][0] = read_x(0, rx_, cn);
          fx[nxt][1] = read_x(1, rx_, cn);
        }
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) acc[cb][tb] = M::mma(fw[cb], fx[cur][tb], acc[cb][tb]);
        fw[cb] = read_w(cb, rw_, kn);
        // Past the end the loads bring zeros.
        if constexpr (C::KK == 1) {
          if (cb == 0) issue_x(WHOLE, s / 2 + 2, xl, hf, 0);
          if (cb == CB / 2) issue_x(WHOLE, s / 2 + 2, xl, hf, 1);
          if (cb == 1) issue_w(WHOLE, s + 3, wl, 0);
          if (cb == CB - 1) issue_w(WHOLE, s + 3, wl, 1);
        } else if (end) {
          if (cb == 0) issue_x(WHOLE, s / 2 + 2, xl, hf, 0);
          if (cb == CB / 2) issue_x(WHOLE, s / 2 + 2, xl, hf, 1);
        } else {
          if (cb == 0) issue_w(WHOLE, s + 2, (wsl + 2) & 3, 0);
          if (cb == CB / 2) issue_w(WHOLE, s + 2, (wsl + 2) & 3, 1);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    wsl = wn;
    if (hf) xsl = xn;
  };
  using I0 = std::integral_constant<int, 0>;
  using I1 = std::integral_constant<int, 1>;
  using IP = std::integral_constant<int, C::KK & 1>;  // the set after one half-block
  int s = 0;
  // Half-blocks s and s + 1 issue X up to k = (s + 6) KS and W up to (s + 5) KS.
  for (; (s + 6) * C::KS <= d_in; s += 2) {
    half(s, I0{}, I0{}, T1{});
    half(s + 1, I1{}, IP{}, T1{});
  }
  for (; s + 1 < nh; s += 2) {
    half(s, I0{}, I0{}, T0{});
    half(s + 1, I1{}, IP{}, T0{});
  }
  if (s < nh) half(s, I0{}, I0{}, T0{});
  wait_loads<0>();
  wait_lds();
  __builtin_amdgcn_s_barrier();  // the rings are free
  asm volatile("" ::: "memory");
  static_assert(8 * store_bytes<(NP + 1) / 2, 2> <= C::BYTES && expand_bytes<NP, TL_T> <= C::BYTES, "the rings hold these");
  if constexpr (FP8) scale_tile<CB, 2>(a, acc, t0 + 64 * wt, c0 + 32 * cb0);
  if (a.n_agents > 0) expand_tile<FP8, NP, TL_T, CB, 2>(a, ksa, acc, lds, t0, 64 * wt, c0, cb0);
  store_tile<CB, 2>(a, acc, lds + wv * store_bytes<(NP + 1) / 2, 2>, t0 + 64 * wt, c0 + 32 * cb0);
}

// Workgroup L runs on XCD L % 8; each XCD takes a contiguous eighth of the
// tiles, in bands of four token tiles, whose rows of X and columns of W its L2
// then serves several times.  False: past the last tile.
__device__ __forceinline__ bool my_tile(int n_tt, int n_ct, int& tt, int& ct) {
  const int n_tiles = n_tt * n_ct, per = (n_tiles + 7) / 8;
  const int tile = (int)(blockIdx.x % 8) * per + (int)(blockIdx.x / 8);
  if ((int)(blockIdx.x / 8) >= per || tile >= n_tiles) return false;
  const int band = tile / (4 * n_ct), in = tile - band * 4 * n_ct, bh = n_tt - 4 * band < 4 ? n_tt - 4 * band : 4;
  ct = __builtin_amdgcn_readfirstlane(in / bh);
  tt = __builtin_amdgcn_readfirstlane(4 * band + in % bh);
  return true;
}

template <bool FP8, int C0, int C1>
__global__ void __launch_bounds__(512, 2) tile_kernel(const ProjectArgs a, int ksa, int n_tt, int n_ct) {
  using C = Tile<FP8, C0 + C1>;
  __shared__ __attribute__((aligned(1024))) char ring[C::BYTES];
  int tt, ct;
  if (!my_tile(n_tt, n_ct, tt, ct)) return;  // uniform over the workgroup
  const int64_t t0 = (int64_t)tt * TL_T, c0 = (int64_t)ct * C::CT;
  if (__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) < 4) tile_wave<FP8, C0 + C1, C0, 0>(a, ksa, ring, t0, c0, 0);
  else tile_wave<FP8, C0 + C1, C1, 1>(a, ksa, ring, t0, c0, C0);
}

template <bool FP8, int C0, int C1>
hipError_t launch_tiles(const ProjectArgs& a, int ksa, hipStream_t st) {
  const int64_t n_tt = (a.T + TL_T - 1) / TL_T, n_ct = (a.d_out + 32 * (C0 + C1) - 1) / (32 * (C0 + C1));
  hipLaunchKernelGGL((tile_kernel<FP8, C0, C1>), dim3((unsigned)((n_tt * n_ct + 7) / 8 * 8)), dim3(512), 0, st, a, ksa, (int)n_tt,
                     (int)n_ct);
  return hipGetLastError();
}

// Tiles of 128 tokens x 32 NP columns, for calls whose larger tiles would leave
// CUs idle: eight waves, two by tokens (64 each), two by columns, and two by k
// (each stage's first and second half; waves w and w + 4 share a SIMD, one's
// reads beside the other's MFMAs).  Stages of 128 bytes of k a row come through
// one ring.  At the end the two waves of a k pair exchange halves of their sums.
// 512 x 4096 x 4096 in bf16 takes 27.5 us, 25 without the MFMAs: its loads, their
// waits and barriers bound it, at half the 64 bytes a clock that a CU takes of whole
// lines in the tiles above (24 KB a stage would be 12 us; why is not known).
constexpr int MD_T = 128;

template <bool FP8, int NP>
struct Mid {
  static constexpr int E = FP8 ? 1 : 2, KS = 128 / E, KK = FP8 ? 1 : 2;  // bytes; k of a stage; MFMA steps of a wave's half
  static constexpr int CT = 32 * NP, WRB = CT * E, CB = NP / 2;          // columns; bytes of a weight row; blocks of a wave
  static constexpr int XB = MD_T * 128, SB = XB + CT * 128;              // bytes of X and of a stage
  static constexpr int NI = SB / 8192;                                   // 1 KB loads of a wave
  static constexpr int RING = 160 * 1024 / SB < 6 ? 160 * 1024 / SB : 6;
  static constexpr int BYTES = RING * SB;
};

template <bool FP8, int NP>
__global__ void __launch_bounds__(512, 2) mid_kernel(const ProjectArgs a, int ksa, int n_tt, int n_ct) {
  using C = Mid<FP8, NP>;
  using M = Mma<FP8>;
  using Frag = typename M::Frag;
  constexpr int E = C::E, CB = C::CB;
  __shared__ __attribute__((aligned(1024))) char ring[C::BYTES];
  int tt, ct;
  if (!my_tile(n_tt, n_ct, tt, ct)) return;  // uniform over the workgroup
  const int64_t t0 = (int64_t)tt * MD_T, c0 = (int64_t)ct * C::CT;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wt = wv & 1, wc = (wv >> 1) & 1, g = wv >> 2;
  const int toks = (int)(a.T - t0 < MD_T ? a.T - t0 : (int64_t)MD_T), d_in = (int)a.d_in;
  const int32_t ldw = (int32_t)(a.d_out * E), ldx = (int32_t)(a.ld_x * E);
  const i32x4 rx = buffer_rsrc(static_cast<const char*>(a.X) + t0 * ldx, (toks - 1) * ldx + d_in * E);
  const i32x4 rw = buffer_rsrc(a.W, d_in * ldw);
  // Load j of this wave is load 8 j + wv of the stage, X rows first.
  int32_t off[C::NI], kof[C::NI];
#pragma unroll
  for (int j = 0; j < C::NI; ++j) {
    const int b = (8 * j + wv) * 1024 + lane * 16;
    if (j < C::XB / 8192) {
      const int r = b / 128, c = (lane % 8) ^ ((r >> 1) & 7);
      kof[j] = c * 16 / E;
      off[j] = r < toks ? r * ldx + c * 16 : INT32_MIN;
    } else {
      const int k = (b - C::XB) / C::WRB, p = (b - C::XB) % C::WRB / (32 * E), in = b % (32 * E) / E;
      const int64_t col = c0 + (p ^ swz_blocks<FP8, NP>(k)) * 32 + in;
      kof[j] = k;
      off[j] = col < a.d_out ? k * ldw + (int32_t)col * E : INT32_MIN;
    }
  }
  lds_char* const lds = (lds_char*)ring;
  const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)lds);
  // WHOLE: all k of the stage are below d_in, and the k offset is scalar.
  auto issue = [&](auto WHOLE, int s, int slot, int j) {
    const uint32_t to = at + slot * C::SB + (8 * j + wv) * 1024;
    const int k0 = s * C::KS;
    const bool x = j < C::XB / 8192;
    const uint32_t ks = (uint32_t)k0 * (uint32_t)(x ? E : ldw);
    if constexpr (decltype(WHOLE)::value) lds_dma16_at(x ? rx : rw, to, off[j], (int32_t)ks);
    else lds_dma16_at(x ? rx : rw, to, k0 + kof[j] < d_in && off[j] != INT32_MIN ? (int32_t)((uint32_t)off[j] + ks) : INT32_MIN, 0);
  };
  const int l32 = lane & 31, h = lane >> 5, grp = lane >> 4, i16 = lane & 15;
  f32x16 acc[CB][2];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
      for (int j = 0; j < 16; ++j) acc[cb][tb][j] = 0.f;
  const int xrow = 64 * wt + l32, xs = (xrow >> 1) & 7;  // rows 32 further swizzle alike
  const int xo = xrow * 128 + ((4 * g + (FP8 ? 2 * h : h)) ^ xs) * 16;  // chunk c further on lies at xo ^ 16 c
  auto read_x = [&](int tb, const lds_char* st, int kk) -> Frag {
    if constexpr (FP8) {
      const u32x4 lo = lds_read16(st + xo + 32 * tb * 128), hi = lds_read16(st + (xo ^ 16) + 32 * tb * 128);
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      return lds_read16(st + (xo ^ (32 * kk)) + 32 * tb * 128);
    }
  };
  const int wk = (FP8 ? 32 * h + i16 / 2 : 8 * h + i16 / 4), ws = swz_blocks<FP8, NP>(wk);
  int wo[CB];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
    wo[cb] = C::XB + (wk + g * C::KS / 2) * C::WRB + (grp & 1) * 16 * E + (FP8 ? i16 % 2 : i16 % 4) * 8 + ((CB * wc + cb) ^ ws) * (32 * E);
  auto read_w = [&](int cb, const lds_char* st, int kk) -> Frag {
    const lds_char* p = st + wo[cb] + 16 * kk * C::WRB;
    if constexpr (FP8) {
      const u32x2 v0 = lds_tr8(p), v1 = lds_tr8(p + 8 * C::WRB), v2 = lds_tr8(p + 16 * C::WRB), v3 = lds_tr8(p + 24 * C::WRB);
      return Frag{v0[0], v0[1], v1[0], v1[1], v2[0], v2[1], v3[0], v3[1]};
    } else {
      const u32x2 lo = lds_tr16(p), hi = lds_tr16(p + 4 * C::WRB);
      return Frag{lo[0], lo[1], hi[0], hi[1]};
    }
  };
  const int ns = (d_in + C::KS - 1) / C::KS;
  for (int s = 0; s < C::RING - 1; ++s)
#pragma unroll
    for (int j = 0; j < C::NI; ++j) issue(std::false_type{}, s, s, j);
  wait_loads<(C::RING - 2) * C::NI>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  Frag fw[2][CB], fx[2][2];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) fw[0][cb] = read_w(cb, lds, 0);
#pragma unroll
  for (int tb = 0; tb < 2; ++tb) fx[0][tb] = read_x(tb, lds, 0);
  int slot = 0, last = C::RING - 1;  // slots of stage s and of stage s - 1
  auto stage = [&](int s, auto P0, auto WHOLE) {
    constexpr int p0 = decltype(P0)::value;
    const int next = slot + 1 == C::RING ? 0 : slot + 1;
    const lds_char* st = lds + slot * C::SB;
    const lds_char* stn = lds + next * C::SB;
#pragma unroll
    for (int kk = 0; kk < C::KK; ++kk) {
      const int cur = (p0 + kk) & 1, nxt = cur ^ 1;
      const bool end = kk == C::KK - 1;
      if (end) {
        // Stage s + 1 has landed, and every wave has used what it read of stage
        // s - 1, whose slot is filled again.
        wait_loads<(C::RING - 3) * C::NI>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
      }
      const lds_char* sn = end ? stn : st;
      const int kn = end ? 0 : kk + 1;
#pragma unroll
      for (int tb = 0; tb < 2; ++tb) {
        if (tb == 0) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (i < CB) fw[nxt][i] = read_w(i, sn, kn);
            fx[nxt][i] = read_x(i, sn, kn);
          }
        }
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) acc[cb][tb] = M::mma(fw[cur][cb], fx[cur][tb], acc[cb][tb]);
        if (end) {  // past the end: zeros
#pragma unroll
          for (int j = tb * ((C::NI + 1) / 2); j < (tb ? C::NI : (C::NI + 1) / 2); ++j) issue(WHOLE, s + C::RING - 1, last, j);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    last = slot;
    slot = next;
  };
  using I0 = std::integral_constant<int, 0>;
  using IP = std::integral_constant<int, C::KK & 1>;
  int s = 0;
  for (; (s + 1 + C::RING) * C::KS <= d_in; s += 2) {
    stage(s, I0{}, std::true_type{});
    stage(s + 1, IP{}, std::true_type{});
  }
  for (; s + 1 < ns; s += 2) {
    stage(s, I0{}, std::false_type{});
    stage(s + 1, IP{}, std::false_type{});
  }
  if (s < ns) stage(s, I0{}, std::false_type{});
  wait_loads<0>();
  wait_lds();
  __builtin_amdgcn_s_barrier();  // the ring is free
  asm volatile("" ::: "memory");
  // Waves w and w + 4 hold the two halves of k: the first takes the sums of
  // token block 0, the second those of block 1.
  f32x4* ex = reinterpret_cast<f32x4*>(ring);  // [wave][CB][4][64]
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f32x4 v;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = g ? acc[cb][0][4 * j + i] : acc[cb][1][4 * j + i];
      ex[((wv * CB + cb) * 4 + j) * 64 + lane] = v;
    }
  __syncthreads();
  f32x16 out[CB][1];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x4 v = ex[(((wv ^ 4) * CB + cb) * 4 + j) * 64 + lane];
#pragma unroll
      for (int i = 0; i < 4; ++i) out[cb][0][4 * j + i] = (g ? acc[cb][1][4 * j + i] : acc[cb][0][4 * j + i]) + v[i];
    }
  __syncthreads();  // the ring is free again
  static_assert(8 * store_bytes<CB, 1> <= C::BYTES && expand_bytes<NP, MD_T> <= C::BYTES && 8 * CB * 4096 <= C::BYTES, "the ring holds these");
  const int tw = 64 * wt + 32 * g;
  const int64_t cw = c0 + 32 * CB * wc;
  if constexpr (FP8) scale_tile<CB, 1>(a, out, t0 + tw, cw);
  if (a.n_agents > 0) expand_tile<FP8, NP, MD_T, CB, 1>(a, ksa, out, ring, t0, tw, c0, CB * wc);
  store_tile<CB, 1>(a, out, ring + wv * store_bytes<CB, 1>, t0 + tw, cw);
}

template <bool FP8, int NP>
hipError_t launch_mid(const ProjectArgs& a, int ksa, hipStream_t st) {
  const int64_t n_tt = (a.T + MD_T - 1) / MD_T, n_ct = (a.d_out + 32 * NP - 1) / (32 * NP);
  hipLaunchKernelGGL((mid_kernel<FP8, NP>), dim3((unsigned)((n_tt * n_ct + 7) / 8 * 8)), dim3(512), 0, st, a, ksa, (int)n_tt,
                     (int)n_ct);
  return hipGetLastError();
}

// The time of slabs in `ks` slices, in microseconds: a stage takes 0.29 while a CU
// has one workgroup and 0.56 with two (96 rows of 4096 x 4096 in bf16: one slice,
// on half the CUs, 28.0 us, two 22.7, three 19.4; four, which do not run at once,
// 23.9), twice that in e4m3, whose stages bring 24 KB instead of 16 (320 rows of
// 5120 x 7168, rank 16: 47 us, as tiles 35; 20 rows of 14336 x 4096, where it adds
// slices, 26.8 -> 18.7), the
// stages together no less than W takes at the rate of a copy (24 rows of 4096 x
// 14336: one slice 30.5 us, two 36.7); sums are written and read at 3.5 TB/s (256
// rows of 1024 x 1024: three slices 10.8 us, seven 13.9), each row's B at 11.
// A few CUs with two workgroups delay all, so those count as 1.3 at least (two
// slices of the 96 rows are 260 workgroups; 256 rows in one slice are as many, 35.6
// us, as tiles 31.9).  Counting two always as 1.5 times one leaves no room for the
// turns of rows of many agents (160 rows of 14336 x 4096 in bf16, rank 64, eight
// agents: 77 -> 163 us).
double slab_time(int64_t T, int64_t d_in, int64_t d_out, int rank, bool fp8, int cus, int ks) {
  const int64_t cw = fp8 ? 128 : 64, n = ((d_out + cw - 1) / cw + 1) * ((T + SL_T - 1) / SL_T) * ks, nk = (d_in + cw - 1) / cw;
  const int64_t rounds = (n + 2 * cus - 1) / (2 * cus);
  const double fill = n <= cus ? 1.0 : (rounds > 1 ? 2.0 : ((double)n / cus > 1.3 ? (double)n / cus : 1.3)), out = (double)T * (double)d_out;
  const double stages = (double)(rounds * ((nk + ks - 1) / ks)) * (0.29 + 0.27 * (fill - 1.0)) * (fp8 ? 2.0 : 1.0);
  const double once = (double)d_in * (double)d_out * (fp8 ? 1.0 : 2.0) / 5e6;
  return 7.5 + (stages > once ? stages : once) + out * 8.0 * ks / 3.5e6 + out * 2.0 * rank / 11e6;
}

// The same k slices of W and of the adapters.
SlabPlan slab_plan(int64_t T, int64_t d_in, int64_t d_out, int n_agents, int rank, bool fp8, int cus) {
  SlabPlan p{};
  const int cw = fp8 ? 128 : 64;
  p.n_ct = (int)((d_out + cw - 1) / cw);
  p.n_tt = (int)((T + SL_T - 1) / SL_T);
  p.ks = 1;
  for (int k = 2; k <= 8 && k <= (d_in + 127) / 128; ++k)
    if (slab_time(T, d_in, d_out, rank, fp8, cus, k) < slab_time(T, d_in, d_out, rank, fp8, cus, p.ks)) p.ks = k;
  p.ksa = n_agents > 0 ? p.ks : 0;
  p.turns = n_agents > 0 ? slab_turns(n_agents, rank, 2 * cus - (int64_t)p.n_ct * p.n_tt * p.ks, (int64_t)p.n_tt * p.ks) : 1;
  p.h_at = (int64_t)p.ks * T * d_out;
  return p;
}

// The tile shape that takes the least time.  A CU holds one tile at a time, so a
// launch takes as many rounds as its tiles fill the CUs; a round takes a fixed
// time and one that goes with d_in (microseconds, the latter at 4096), less in a
// round that leaves CUs idle (down to about 0.6 of it: the clock rises), and
// more where adapter rows are added.  Measured with 256 tiles at d_in 1024 and
// 4096, bf16 and e4m3.
int tile_form(int64_t T, int64_t d_in, int64_t d_out, int n_agents, bool fp8, int cus, double* us) {
  struct Form {
    int toks, cols;
    double fixed[2], per[2], lr;
  };
  static constexpr Form forms[6] = {
      {128, 64, {4.8, 4.9}, {20.0, 12.3}, 3.0},    {128, 128, {6.7, 6.9}, {29.2, 14.1}, 3.0},
      {256, 128, {6.1, 8.0}, {55.8, 28.1}, 6.0},   {256, 160, {6.2, 8.4}, {73.3, 31.9}, 6.0},
      {256, 192, {6.9, 8.9}, {78.3, 36.4}, 6.0},   {256, 256, {7.6, 11.6}, {105.0, 46.4}, 6.0},
  };
  int best = 0;
  double least = 1e300;
  for (int i = 0; i < 6; ++i) {
    const Form& f = forms[i];
    const int64_t tiles = ((T + f.toks - 1) / f.toks) * ((d_out + f.cols - 1) / f.cols), rounds = tiles / cus,
                  rest = tiles % cus;
    const double fixed = f.fixed[fp8] + (n_agents > 0 ? f.lr : 0.0), per = f.per[fp8] * (double)d_in / 4096.0;
    const double t = (double)rounds * (fixed + per) + (rest > 0 ? fixed + per * (0.6 + 0.4 * (double)rest / cus) : 0.0);
    if (t < least) {
      least = t;
      best = i;
    }
  }
  *us = least;
  return best;
}

// Slabs or tiles.  Slabs fill the CUs where tiles would leave most idle, and form
// the adapter rows beside the others, but read X and W more often and their sums
// once more.  Measured for 96 to 480 rows of 1024 x 8192 to 14336 x 4096 and up to
// 4000 of 4096 x 256, in both types with ranks 8 to 64: 4096 x 4096 in bf16, rank
// 16, 96 rows 19.3 us as slabs against 30.1, 192 rows 25.8 against 30.0, 320 rows
// 38.1 against 30.7, 512 rows 55.9 against 35.5; 14336 x 4096 in e4m3, 160 rows 42.8
// against 65.8; 1100 rows of 4096 x 256 18.9 against 33.7.  Up to 64 rows always:
// less than a tile's.  Without adapters (n_agents 0) it goes as with some of rank 16.
constexpr int SL_MOST = 4096;  // bounds the workspace

bool slabs_pay(int64_t T, int64_t d_in, int64_t d_out, int n_agents, int rank, bool fp8, int cus) {
  if (T <= SL_T || T > SL_MOST) return T <= SL_T;
  if (n_agents == 0) rank = 16;
  const SlabPlan p = slab_plan(T, d_in, d_out, n_agents, rank, fp8, cus);
  double us;
  tile_form(T, d_in, d_out, 1, fp8, cus, &us);
  // The adapter rows' launch, and their longer expansion past rank 16 (320 rows of
  // 2048 x 2048, rank 64: 18.8 us as slabs, 25.2 as tiles).
  us += 6.0 + 5.0 * (double)d_in / 4096.0 + (rank > 16 ? (rank - 16) / 12.0 : 0.0);
  return slab_time(T, d_in, d_out, rank, fp8, cus, p.ks) < us;
}

template <bool FP8>
hipError_t launch(const ProjectArgs& a, hipStream_t st) {
  if (a.T <= ST_T) return launch_stream<FP8>(a, st);
  if (slabs_pay(a.T, a.d_in, a.d_out, a.n_agents, a.rank, FP8, a.cus)) {
    const SlabPlan p = slab_plan(a.T, a.d_in, a.d_out, a.n_agents, a.rank, FP8, a.cus);
    if (const hipError_t e = launch_slabs<FP8>(a, p, st)) return e;
    return launch_join(a, p, st);
  }
  const int ksa = shrink_slices(a.T, a.d_in, a.rank, a.cus);
  if (a.n_agents > 0) {
    SlabPlan p{};
    p.n_tt = 1;
    p.ksa = ksa;
    p.turns = slab_turns(a.n_agents, a.rank, 2 * a.cus, (a.T + SL_T - 1) / SL_T * ksa);
    if (const hipError_t e = launch_slabs<FP8>(a, p, st)) return e;
  }
  double us;
  switch (tile_form(a.T, a.d_in, a.d_out, a.n_agents, FP8, a.cus, &us)) {
    case 0: return launch_mid<FP8, 2>(a, ksa, st);
    case 1: return launch_mid<FP8, 4>(a, ksa, st);
    case 2: return launch_tiles<FP8, 2, 2>(a, ksa, st);
    case 3: return launch_tiles<FP8, 3, 2>(a, ksa, st);
    case 4: return launch_tiles<FP8, 3, 3>(a, ksa, st);
    default: return launch_tiles<FP8, 4, 4>(a, ksa, st);
  }
}

}  // namespace

// A grid holds fewer than 2^32 threads, 2^23 workgroups here.  Tiles of 128 x 64 are
// the most, the adapters' slabs one per 64 rows when rows are many; so a call goes
// in parts of rows that have about 2^22 such tiles and 2^28 rows at most (64 GB of Y).
static int64_t rows_at_once(int64_t T, int64_t d_out) {
  const int64_t across = (d_out + 63) / 64, tiles = (1 << 22) / across;
  const int64_t most = tiles * 128 < (1LL << 28) ? tiles * 128 : (1LL << 28), parts = (T + most - 1) / most;
  return parts == 1 ? T : ((T + parts - 1) / parts + 255) / 256 * 256;
}

static size_t part_bytes(int64_t T, int64_t d_in, int64_t d_out, int n_agents, int rank, int cus) {
  size_t most = 0;
  for (const bool fp8 : {false, true}) {
    size_t b = n_agents > 0 ? (size_t)shrink_slices(T, d_in, rank, cus) * (size_t)T * (size_t)rank * 4 : 0;
    if (T <= ST_T)
      b = plan_bytes(T, rank, stream_plan(T, d_in, d_out, n_agents, fp8, cus));
    else if (slabs_pay(T, d_in, d_out, n_agents, rank, fp8, cus))
      b = plan_bytes(T, rank, slab_plan(T, d_in, d_out, n_agents, rank, fp8, cus));
    most = b > most ? b : most;
  }
  return most;
}

size_t adapted_projection_bytes(int64_t T, int64_t d_in, int64_t d_out, int n_agents, int rank, int cus) {
  if (n_agents == 0) rank = 8;
  const int64_t part = rows_at_once(T, d_out), last = T - (T - 1) / part * part;
  const size_t a = part_bytes(part, d_in, d_out, n_agents, rank, cus);
  const size_t b = last == part ? a : part_bytes(last, d_in, d_out, n_agents, rank, cus);
  return a > b ? a : b;
}

hipError_t launch_adapted_projection(const ProjectArgs& a, hipStream_t st) {
  const int64_t part = rows_at_once(a.T, a.d_out);
  for (int64_t r = 0; r < a.T; r += part) {
    ProjectArgs p = a;
    p.T = a.T - r < part ? a.T - r : part;
    p.X = static_cast<const char*>(a.X) + r * a.ld_x * (a.x_scale != nullptr ? 1 : 2);
    if (a.x_scale != nullptr) p.x_scale = a.x_scale + r;
    if (a.agent != nullptr) p.agent = a.agent + r;
    p.Y = a.Y + r * a.ld_y;
    if (const hipError_t e = a.x_scale != nullptr ? launch<true>(p, st) : launch<false>(p, st)) return e;
  }
  return hipSuccess;
}

}  // namespace prc
