// The head's three products in fp32, on the fp32 matrix cores: the forms of
// kernels_headgemm.hip on 128 x 128 tiles of four waves (64 x 64 each,
// v_mfma_f32_32x32x2_f32; 128 x 64 for logits and dh of few rows), 16 of k in an LDS stage [k][x], whatever way an
// operand lies in memory; the next stage's values wait in registers, and four
// workgroups to a CU cover each other's barriers. Logits are
// stored as they are (in units of log 2), their statistics are a pass of their
// own (kernels_head.hip). 2560 rows of width 2048 over 50304 classes: 119 TFLOP/s
// over the whole call (library products 146), 630 of 768: 100 (85 to 109); the
// matrix cores are busy 75 % of the clocks.
#include <algorithm>

#include "dsf_device.h"
#include "head.h"

namespace dsf {

namespace {
constexpr int kT = 128, kBK = 16;

// Value (x, k) of a stage of X values x. Odd k have the halves of their 64 banks swapped: a
// read's two k then cover all banks.
template <int X>
__device__ __forceinline__ int f32_at(int x, int k) { return k * X + (x ^ ((k & 1) << 5)); }

// COL false: element (x, k) at p[x ld + k]; COL true: at p[k ld + x]. Outside
// [0, nx) x [0, nk) zeros (nx, nk, ld multiples of 4 on the contiguous side).
template <bool COL, int X>
struct F32Op {
  static constexpr int kVecs = X * kBK / 4 / 256;  // 16-byte vectors a thread brings
  const float* p;
  int64_t ld;
  int nx, nk;
  f32x4 r[kVecs];
  // values of k0 .. k0 + 15, x0 .. x0 + X - 1
  __device__ __forceinline__ void load(int64_t x0, int k0, int tid) {
#pragma unroll
    for (int u = 0; u < kVecs; ++u) {
      const int64_t x = COL ? x0 + 4 * (tid % (X / 4)) : x0 + (tid & 63) + 64 * u;
      const int k = COL ? k0 + tid / (X / 4) + 1024 / X * u : k0 + 4 * (tid >> 6);
      r[u] = x < nx && k < nk ? *reinterpret_cast<const f32x4*>(p + (COL ? k * ld + x : x * ld + k))
                              : f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  __device__ __forceinline__ void store(float* lds, int tid) const {
#pragma unroll
    for (int u = 0; u < kVecs; ++u) {
      if constexpr (COL) {
        *reinterpret_cast<f32x4*>(lds + f32_at<X>(4 * (tid % (X / 4)), tid / (X / 4) + 1024 / X * u)) = r[u];
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) lds[f32_at<X>((tid & 63) + 64 * u, 4 * (tid >> 6) + i)] = r[u][i];
      }
    }
  }
};
}  // namespace

// A workgroup's tile: 128 m by TN n (two waves by two, of 64 m by TN / 2 n).
template <int MODE, int TN>
__device__ __forceinline__ void head_f32_tile(const HeadGemmArgs& g, int rows, float* smem) {
  constexpr bool ACOL = MODE != kHeadLogits, BCOL = MODE == kHeadDw;
  constexpr int NJ = TN / 64, kStage = kBK * (kT + TN);  // floats of a stage: A, then B
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave >> 1, wn = wave & 1, r32 = lane & 31, hi = lane >> 5;
  // (logits: all columns of ldz are written)
  const int tr = (rows + TN - 1) / TN, tv = (MODE == kHeadLogits ? g.ldz : g.V + kT - 1) / kT, td = (g.d + kT - 1) / kT;
  const int outer = MODE == kHeadDw ? tv : tr, inner = MODE == kHeadLogits ? tv : td;
  const int nt = outer * inner;
  const int splits = MODE == kHeadDh ? *g.splits : 1;
  if (int(blockIdx.x) >= nt * splits) return;  // (the grid is for all rows and the most shares)
  const int w = xcd_remap(int(blockIdx.x), nt * splits);
  const int sp = w / nt, tn = (w - sp * nt) / inner, tm = (w - sp * nt) - tn * inner;

  const int K = MODE == kHeadLogits ? g.d : MODE == kHeadDh ? g.ldz : rows;
  F32Op<ACOL, kT> A{(const float*)(MODE == kHeadDw ? g.h : g.w), g.d, MODE == kHeadLogits ? g.V : g.d,
                MODE == kHeadDh ? g.V : K};
  F32Op<BCOL, TN> B{(const float*)(MODE == kHeadLogits ? g.h : g.z), MODE == kHeadLogits ? g.d : g.ldz,
                MODE == kHeadDw ? g.ldz : rows, K};
  const int nk = (K + kBK - 1) / kBK;
  const int kb = int(int64_t(nk) * sp / splits), ke = int(int64_t(nk) * (sp + 1) / splits);
  const int64_t xm = int64_t(tm) * kT, xn = int64_t(tn) * TN;

  f32x16 acc[2][NJ];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
  if (kb < ke) {
    A.load(xm, kb * kBK, tid);
    B.load(xn, kb * kBK, tid);
    A.store(smem, tid);
    B.store(smem + kBK * kT, tid);
  }
  for (int kt = kb; kt < ke; ++kt) {
    const int s = (kt - kb) & 1;
    __syncthreads();
    if (kt + 1 < ke) {
      A.load(xm, (kt + 1) * kBK, tid);
      B.load(xn, (kt + 1) * kBK, tid);
    }
    const float *at[2], *bt[NJ];
#pragma unroll
    for (int i = 0; i < 2; ++i) at[i] = smem + s * kStage + f32_at<kT>(wm * 64 + 32 * i + r32, hi);
#pragma unroll
    for (int j = 0; j < NJ; ++j) bt[j] = smem + s * kStage + kBK * kT + f32_at<TN>(wn * (TN / 2) + 32 * j + r32, hi);
    // the fragments of two k are read while the two before them are multiplied
    float af[2][2], bf[2][NJ];
    auto read = [&](int set, int k) {
#pragma unroll
      for (int i = 0; i < 2; ++i) af[set][i] = at[i][k * kT];
#pragma unroll
      for (int j = 0; j < NJ; ++j) bf[set][j] = bt[j][k * TN];
    };
    read(0, 0);
#pragma unroll
    for (int k = 0; k < kBK; k += 2) {
      const int set = (k >> 1) & 1;
      if (k + 2 < kBK) read(set ^ 1, k + 2);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(af[set][i], bf[set][j], acc[i][j], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (kt + 1 < ke) {  // the other stage was read before this iteration's barrier
      A.store(smem + (s ^ 1) * kStage, tid);
      B.store(smem + (s ^ 1) * kStage + kBK * kT, tid);
    }
  }
  // lane holds out[n = 32 j + r32][m = 32 i + 8 q + 4 hi + e], e < 4
  const float scale = MODE == kHeadDw ? *g.scale : 1.f;
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int n = tn * TN + wn * (TN / 2) + 32 * j + r32;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int m = tm * kT + wm * 64 + 32 * i + 8 * q + 4 * hi;
        f32x4 v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        if constexpr (MODE == kHeadLogits) {
          // columns past the last class (ldz is a multiple of 128) weigh nothing
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = m + e < g.V ? v[e] * g.z_scale : -INFINITY;
          if (n < rows) *reinterpret_cast<f32x4*>((float*)g.zout + int64_t(n) * g.ldz + m) = v;
        } else if constexpr (MODE == kHeadDh) {
          if (n < rows && m < g.d)
            *reinterpret_cast<f32x4*>(g.part + (int64_t(sp) * g.rows_ld + n) * g.d + m) = v;
        } else if (n < g.V && m < g.d) {
          v *= scale;
          if (g.prev) v += *reinterpret_cast<const f32x4*>(g.prev + int64_t(n) * g.d + m);
          *reinterpret_cast<f32x4*>(g.out32 + int64_t(n) * g.d + m) = v;
        }
      }
  }
}

template <int MODE>
__global__ __launch_bounds__(256, 4) void head_f32_kernel(HeadGemmArgs g) {
  __shared__ __attribute__((aligned(16))) float smem[2 * kBK * 2 * kT];
  int rows = *g.n_active - g.row0;
  rows = rows < 0 ? 0 : rows > g.rows ? g.rows : rows;
  if (MODE != kHeadDw && head_f32_rows(rows) == 64) head_f32_tile<MODE, 64>(g, rows, smem);
  else head_f32_tile<MODE, kT>(g, rows, smem);
}

hipError_t launch_head_gemm_f32(int mode, const HeadGemmArgs& g, hipStream_t s) {
  // (tiles of 64 rows are taken up to kHeadF32Few rows)
  const int tr = std::max((g.rows + kT - 1) / kT, (std::min(g.rows, kHeadF32Few) + 63) / 64), tv = (g.V + kT - 1) / kT, td = (g.d + kT - 1) / kT;
  if (mode == kHeadLogits) head_f32_kernel<kHeadLogits><<<tr * (g.ldz / kT), 256, 0, s>>>(g);
  else if (mode == kHeadDh) head_f32_kernel<kHeadDh><<<tr * td * g.most, 256, 0, s>>>(g);
  else head_f32_kernel<kHeadDw><<<tv * td, 256, 0, s>>>(g);
  return hipGetLastError();
}

}  // namespace dsf
