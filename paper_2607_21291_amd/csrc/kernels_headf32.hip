// The head's three products in fp32, on the fp32 matrix cores: the forms of
// kernels_headgemm.hip on 128 x 128 tiles of four waves (64 x 64 each,
// v_mfma_f32_32x32x2_f32), 16 of k in an LDS stage [k][x], whatever way an
// operand lies in memory; the next stage's values wait in registers, and four
// workgroups to a CU cover each other's barriers. Logits are
// stored as they are (in units of log 2), their statistics are a pass of their
// own (kernels_head.hip).
#include "dsf_device.h"
#include "head.h"

namespace dsf {

namespace {
constexpr int kT = 128, kBK = 16;
constexpr int kVecs = kT * kBK / 4 / 256;  // 16-byte vectors of an operand a thread brings

// Value (x, k) of a stage. Odd k have the halves of their 64 banks swapped: a read's two k
// then cover all banks.
__device__ __forceinline__ int f32_at(int x, int k) { return k * kT + (x ^ ((k & 1) << 5)); }

// COL false: element (x, k) at p[x ld + k]; COL true: at p[k ld + x]. Outside
// [0, nx) x [0, nk) zeros (nx, nk, ld multiples of 4 on the contiguous side).
template <bool COL>
struct F32Op {
  const float* p;
  int64_t ld;
  int nx, nk;
  f32x4 r[kVecs];
  // values of k0 .. k0 + 15, x0 .. x0 + 127
  __device__ __forceinline__ void load(int64_t x0, int k0, int tid) {
#pragma unroll
    for (int u = 0; u < kVecs; ++u) {
      const int64_t x = COL ? x0 + 4 * (tid & 31) : x0 + (tid & 63) + 64 * (u & 1);
      const int k = COL ? k0 + (tid >> 5) + 8 * u : k0 + 4 * (tid >> 6) + 16 * (u >> 1);
      r[u] = x < nx && k < nk ? *reinterpret_cast<const f32x4*>(p + (COL ? k * ld + x : x * ld + k))
                              : f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  __device__ __forceinline__ void store(float* lds, int tid) const {
#pragma unroll
    for (int u = 0; u < kVecs; ++u) {
      if constexpr (COL) {
        *reinterpret_cast<f32x4*>(lds + f32_at(4 * (tid & 31), (tid >> 5) + 8 * u)) = r[u];
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) lds[f32_at((tid & 63) + 64 * (u & 1), 4 * (tid >> 6) + 16 * (u >> 1) + i)] = r[u][i];
      }
    }
  }
};
}  // namespace

template <int MODE>
__global__ __launch_bounds__(256, 4) void head_f32_kernel(HeadGemmArgs g) {
  constexpr bool ACOL = MODE != kHeadLogits, BCOL = MODE == kHeadDw;
  __shared__ __attribute__((aligned(16))) float smem[2][2][kBK * kT];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave >> 1, wn = wave & 1, r32 = lane & 31, hi = lane >> 5;
  int rows = *g.n_active - g.row0;
  rows = rows < 0 ? 0 : rows > g.rows ? g.rows : rows;
  // (logits: all columns of ldz are written)
  const int tr = (rows + kT - 1) / kT, tv = (MODE == kHeadLogits ? g.ldz : g.V + kT - 1) / kT, td = (g.d + kT - 1) / kT;
  const int outer = MODE == kHeadDw ? tv : tr, inner = MODE == kHeadLogits ? tv : td;
  const int nt = outer * inner;
  const int splits = MODE == kHeadDh ? *g.splits : 1;
  if (int(blockIdx.x) >= nt * splits) return;  // (the grid is for all rows and the most shares)
  const int w = xcd_remap(int(blockIdx.x), nt * splits);
  const int sp = w / nt, tn = (w - sp * nt) / inner, tm = (w - sp * nt) - tn * inner;

  const int K = MODE == kHeadLogits ? g.d : MODE == kHeadDh ? g.ldz : rows;
  F32Op<ACOL> A{(const float*)(MODE == kHeadDw ? g.h : g.w), g.d, MODE == kHeadLogits ? g.V : g.d,
                MODE == kHeadDh ? g.V : K};
  F32Op<BCOL> B{(const float*)(MODE == kHeadLogits ? g.h : g.z), MODE == kHeadLogits ? g.d : g.ldz,
                MODE == kHeadDw ? g.ldz : rows, K};
  const int nk = (K + kBK - 1) / kBK;
  const int kb = int(int64_t(nk) * sp / splits), ke = int(int64_t(nk) * (sp + 1) / splits);
  const int64_t xm = int64_t(tm) * kT, xn = int64_t(tn) * kT;

  f32x16 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
  if (kb < ke) {
    A.load(xm, kb * kBK, tid);
    B.load(xn, kb * kBK, tid);
    A.store(smem[0][0], tid);
    B.store(smem[0][1], tid);
  }
  for (int kt = kb; kt < ke; ++kt) {
    const int s = (kt - kb) & 1;
    __syncthreads();
    if (kt + 1 < ke) {
      A.load(xm, (kt + 1) * kBK, tid);
      B.load(xn, (kt + 1) * kBK, tid);
    }
    const float* at[2] = {smem[s][0] + f32_at(wm * 64 + r32, hi), smem[s][0] + f32_at(wm * 64 + 32 + r32, hi)};
    const float* bt[2] = {smem[s][1] + f32_at(wn * 64 + r32, hi), smem[s][1] + f32_at(wn * 64 + 32 + r32, hi)};
    // the fragments of two k are read while the two before them are multiplied
    float af[2][2], bf[2][2];
    auto read = [&](int set, int k) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        af[set][i] = at[i][k * kT];
        bf[set][i] = bt[i][k * kT];
      }
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
        for (int j = 0; j < 2; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(af[set][i], bf[set][j], acc[i][j], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (kt + 1 < ke) {  // the other stage was read before this iteration's barrier
      A.store(smem[s ^ 1][0], tid);
      B.store(smem[s ^ 1][1], tid);
    }
  }
  // lane holds out[n = 32 j + r32][m = 32 i + 8 q + 4 hi + e], e < 4
  const float scale = MODE == kHeadDw ? *g.scale : 1.f;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int n = tn * kT + wn * 64 + 32 * j + r32;
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

hipError_t launch_head_gemm_f32(int mode, const HeadGemmArgs& g, hipStream_t s) {
  const int tr = (g.rows + kT - 1) / kT, tv = (g.V + kT - 1) / kT, td = (g.d + kT - 1) / kT;
  if (mode == kHeadLogits) head_f32_kernel<kHeadLogits><<<tr * (g.ldz / kT), 256, 0, s>>>(g);
  else if (mode == kHeadDh) head_f32_kernel<kHeadDh><<<tr * td * g.most, 256, 0, s>>>(g);
  else head_f32_kernel<kHeadDw><<<tv * td, 256, 0, s>>>(g);
  return hipGetLastError();
}

}  // namespace dsf
