// The three products of the head's losses on the matrix cores (bf16), for h
// [rows, d] and the head's weights W [V, d]:
//   logits   z = h W^T, never stored: a tile leaves each row's maximum and
//            sum of exponentials over its 256 classes and, for gradients, a
//            16-bit code of every logit relative to that maximum;
//   dh       = dz W,    a reduction over classes, cut along them;
//   dW       = dz^T h,  a reduction over rows.
//
// One kernel: out[n][m] = sum_k A[k, m] B[k, n] on 256 x 256 tiles of eight
// waves (64 m by 128 n each), 64 of k per LDS stage, two stages filled by
// buffer DMA. An operand lies in memory along k (rows of 64 k go to LDS, read
// as 16-byte fragments) or along m or n (64 rows of 256 columns, read with the
// LDS transpose load), so nothing is transposed in memory. A's index m is the
// one that is contiguous in the output: an MFMA leaves four consecutive m in a
// lane, eight after a swap between 16-lane rows.
#include <type_traits>

#include "dsf_device.h"
#include "gemm_sched.h"
#include "head.h"

namespace dsf {

namespace {
constexpr int kT = 256, kBK = 64, kThreads = 512;
constexpr int kOpBytes = kT * kBK * 2;   // one operand of a stage
constexpr int kStage = 2 * kOpBytes;     // the other stage's addresses differ in this bit
constexpr int kSubBytes = kBK * 128 * 2; // 128 columns of an operand stored by rows of k

typedef short s16x4 __attribute__((ext_vector_type(4)));
#define DSF_LDS __attribute__((address_space(3)))
typedef DSF_LDS char LdsChar;

// Two loads of 1 KiB (16 bytes a lane) into LDS at at0 and at1 (addresses of the
// wave; lane l's go to + 16 l). Inline assembly, as the compiler would wait for
// all of them before the next transpose load, which it cannot tell apart from
// them; the callers wait and meet at a barrier. The assembly brings the wait
// states that a scalar operand just written by a vector instruction needs. (M0
// is reserved: the compiler keeps nothing in it.)
__device__ __forceinline__ void head_dma2(__amdgpu_buffer_rsrc_t ra, uint32_t va, uint32_t at0,
                                          __amdgpu_buffer_rsrc_t rb, uint32_t vb, uint32_t at1) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 4\n\t"
      "buffer_load_dwordx4 %1, %2, 0 offen lds\n\t"
      "s_mov_b32 m0, %3\n\t"
      "s_nop 4\n\t"
      "buffer_load_dwordx4 %4, %5, 0 offen lds" ::"s"(at0),
      "v"(va), "s"(ra), "s"(at1), "v"(vb), "s"(rb)
      : "memory");
}

// An operand in global memory and its share of a stage. The lane's part of an
// offset is the same for every load; load u of a wave is load l = 8 u + wave of
// the operand's 32 (1 KiB each).
// COL false: element (x, k) at p[x ld + k]; load l fills tile rows 8 l .. + 7, 128 bytes
//   each, 16-byte chunk c of row r at c ^ (r & 7).
// COL true: element (x, k) at p[k ld + x]; subtile l / 16 (128 columns) rows 4 (l % 16) .. + 3
//   of k, 256 bytes each, chunk c of row r at c ^ key(r), key(r) = 2 ((r & 3) + 4 (r >> 3 & 1)): the
//   sixteen rows of a transpose load, 32 bytes each, then cover the 64 banks twice, the minimum.
template <bool COL>
struct HeadOp {
  const uint16_t* base;  // at the tile's first x
  int64_t bytes;         // from there to the end of the operand
  int ld, kmax;
  uint32_t voff;
  int chunk_k;           // COL false: first k of the lane's chunk within a tile
  __device__ __forceinline__ HeadOp(const uint16_t* p, int ld_, int64_t nx, int64_t nk, int64_t x0, int wave, int lane)
      : ld(ld_), kmax(int(nk)) {
    if constexpr (COL) {
      base = p + x0;
      bytes = (nk * ld - x0) * 2;
      const int key = ((lane >> 4) + 4 * ((wave >> 1) & 1)) << 1;
      voff = uint32_t(lane >> 4) * uint32_t(ld) * 2u + uint32_t(((lane & 15) ^ key) * 16);
      chunk_k = 0;
    } else {
      base = p + x0 * ld;
      bytes = (nx - x0) * ld * 2;
      const int c = (lane & 7) ^ (lane >> 3);
      voff = uint32_t(lane >> 3) * uint32_t(ld) * 2u + uint32_t(c * 16);
      chunk_k = 8 * c;
    }
  }
  // resource and offset of load l of k-tile kt. The resource ends with the
  // operand: what lies past it reads as zeros.
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t source(int kt, int l, uint32_t& v) const {
    const int64_t at = COL ? int64_t(kt) * kBK * ld : int64_t(kt) * kBK, left = bytes - at * 2;
    if constexpr (COL) {
      v = voff + uint32_t(4 * (l & 15)) * uint32_t(ld) * 2u + uint32_t(l >> 4) * 256u;
    } else {
      // chunks past the end of a row (a reduction that is no multiple of 64), too
      v = kt * kBK + chunk_k < kmax ? voff + uint32_t(8 * l) * uint32_t(ld) * 2u : 0x80000000u;
    }
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(base + at), (short)0,
                                             int(left < 0 ? 0 : left > 0x7fffffff ? 0x7fffffff : left), 0x00020000);
  }
};

// LDS addresses of an operand's fragments: lane (r16, grp) of block b (16 of x)
// and substep ks (32 of k) gets x = 16 b + r16, k = 32 ks + 8 grp .. + 7.
template <bool COL>
struct HeadFrag {
  uint32_t at;
  __device__ __forceinline__ HeadFrag(uint32_t op, int lane, int x0) {
    const int r16 = lane & 15, grp = lane >> 4;
    if constexpr (COL) {
      // lane 16 G + a + 4 j addresses row j (of the four of a load), columns 4 a .. 4 a + 3
      const int a = lane & 3, row = 8 * grp + ((lane >> 2) & 3);
      const int key = ((row & 3) + 4 * ((row >> 3) & 1)) << 1;
      const int c = (x0 & 127) / 8 + (a >> 1);
      at = op + uint32_t((x0 >> 7) * kSubBytes + row * 256 + ((c ^ key) * 16) + (a & 1) * 8);
    } else {
      at = op + uint32_t((x0 + r16) * 128 + ((grp ^ (r16 & 7)) * 16));
    }
  }
  // block b counts from x0 (COL: x0 a multiple of 64, blocks within its 128 columns)
  __device__ __forceinline__ bf16x8 read(int ks, int b) const {
    if constexpr (COL) {
      typedef DSF_LDS s16x4* P;
      const uint32_t p = (at ^ uint32_t(b * 32)) + uint32_t(ks * 8192);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)p);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)(p + 1024));
      struct { s16x4 a, b; } v{lo, hi};
      return __builtin_bit_cast(bf16x8, v);
    } else {  // substep 1: chunk 4 + grp
      return *(DSF_LDS const bf16x8*)(uintptr_t)((at ^ uint32_t(ks * 64)) + b * 2048);
    }
  }
};

__device__ __forceinline__ u32x4 swap_rows8(uint32_t a0, uint32_t a1, uint32_t b0, uint32_t b1) {
  // a: four 16-bit values of block i, b: of block i + 1. After the swap of odd with even
  // 16-lane rows a lane holds eight consecutive values: columns 16 (i + (grp & 1)) + 8 (grp >> 1).
  const auto x = __builtin_amdgcn_permlane16_swap(a0, b0, false, false);
  const auto y = __builtin_amdgcn_permlane16_swap(a1, b1, false, false);
  return u32x4{x[0], y[0], x[1], y[1]};
}
}  // namespace

// MODE 0: logits (A = W along k, B = h along k); 1: dh (A = W by rows of k, B = dz along k);
// 2: dW (A = h by rows of k, B = dz by rows of k).
template <int MODE>
__global__ __launch_bounds__(kThreads) void head_gemm_kernel(HeadGemmArgs g) {
  constexpr bool ACOL = MODE != kHeadLogits, BCOL = MODE == kHeadDw;
  constexpr int MI = 4, NI = 8;
  __shared__ __attribute__((aligned(65536))) char smem[2 * kStage];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1, r16 = lane & 15, grp = lane >> 4;
  // rows of this piece that take part
  int rows = *g.n_active - g.row0;
  rows = rows < 0 ? 0 : rows > g.rows ? g.rows : rows;

  // the tiles of the rows that take part; a grid for more has workgroups that end here
  const int tr = (rows + kT - 1) / kT, tv = (g.V + kT - 1) / kT, td = (g.d + kT - 1) / kT;
  const int outer = MODE == kHeadDw ? tv : tr, inner = MODE == kHeadLogits ? tv : td;
  const int nt = outer * inner;
  if (int(blockIdx.x) >= nt * g.splits) return;
  const int w = xcd_remap(int(blockIdx.x), nt * g.splits);
  const int sp = w / nt;
  const GemmTile t = gemm_tile(w - sp * nt, outer, inner, MODE == kHeadLogits ? 4 : 0);
  const int tm = t.tn, tn = t.tm;  // out[n][m]: rows of tiles are n

  const int64_t nm = MODE == kHeadLogits ? g.V : g.d;
  const int64_t nn = MODE == kHeadDw ? g.ldz : rows;
  const int K = MODE == kHeadLogits ? g.d : MODE == kHeadDh ? g.ldz : rows;
  const HeadOp<ACOL> A((const uint16_t*)(MODE == kHeadDw ? g.h : g.w), g.d, nm, MODE == kHeadDh ? g.V : K, int64_t(tm) * kT, wave, lane);
  const HeadOp<BCOL> B((const uint16_t*)(MODE == kHeadLogits ? g.h : g.z), MODE == kHeadLogits ? g.d : g.ldz, nn, K, int64_t(tn) * kT, wave,
                       lane);
  const uint32_t lds = uint32_t(__builtin_amdgcn_readfirstlane(int(uint32_t(uintptr_t((DSF_LDS char*)smem)))));
  HeadFrag<ACOL> fa(lds, lane, wm * 64);
  HeadFrag<BCOL> fb(lds + kOpBytes, lane, wn * 128);
  const int nk = (K + kBK - 1) / kBK;
  const int kb = int(int64_t(nk) * sp / g.splits), ke = int(int64_t(nk) * (sp + 1) / g.splits);

  f32x4 acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

#define DSF_INLINE __attribute__((always_inline))
  // the wave's loads u of A and B of k-tile kt, into the stage at st
  auto issue = [&](int kt, uint32_t st, int u) DSF_INLINE {
    const int l = 8 * u + wave;
    uint32_t va, vb;
    const auto ra = A.source(kt, l, va);
    const auto rb = B.source(kt, l, vb);
    head_dma2(ra, va, st + 1024 * l, rb, vb, st + kOpBytes + 1024 * l);
  };
  bf16x8 af[2][MI], bq[2][NI];
  // read n of a fragment set, in the order of their use: A 0, B 0 .. NI - 1, A 1 .. MI - 1
  auto read_n = [&](int set, int ks, int n) DSF_INLINE {
    if (n == 0) af[set][0] = fa.read(ks, 0);
    else if (n <= NI) bq[set][n - 1] = fb.read(ks, n - 1);
    else af[set][n - NI] = fa.read(ks, n - NI);
  };
  constexpr int R = MI + NI;
  // One substep: the products of fragment set S, and between them the reads of
  // the other set (substep ks) and the loads of tile kn into the stage at dma.
  auto substep = [&](auto Sc, int ks, bool do_issue, int kn, uint32_t dma) DSF_INLINE {
    constexpr int S = decltype(Sc)::value;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      acc[i][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(af[S][i], bq[S][0], acc[i][0], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      if (i < MI - 1) {
#pragma unroll
        for (int n = i * R / (MI - 1); n < (i + 1) * R / (MI - 1); ++n) read_n(1 - S, ks, n);
      }
      if (S == 1 && do_issue) issue(kn, dma, i);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 1; j < NI; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(af[S][i], bq[S][j], acc[i][j], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  if (kb < ke) {
#pragma unroll
    for (int u = 0; u < 4; ++u) issue(kb, lds, u);
    if (kb + 1 < ke) {
#pragma unroll
      for (int u = 0; u < 4; ++u) issue(kb + 1, lds ^ kStage, u);
      asm volatile("s_waitcnt vmcnt(8)\n\ts_barrier" ::: "memory");
    } else {
      asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
    }
#pragma unroll
    for (int n = 0; n < R; ++n) read_n(0, 0, n);
    uint32_t cur = lds;
    // One k-tile. All its fragments are in registers by the middle, where the
    // barrier publishes the next tile and frees this one's stage. (The last
    // tile reads stale LDS there; nothing uses it.)
    for (int kt = kb; kt < ke; ++kt) {
      substep(std::integral_constant<int, 0>(), 1, false, 0, 0);
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      fa.at ^= kStage;
      fb.at ^= kStage;
      substep(std::integral_constant<int, 1>(), 0, kt + 2 < ke, kt + 2, cur);
      cur ^= kStage;
    }
  }

  // lane holds out[n = 16 j + r16][m = 16 i + 4 grp + e] of its wave's part
  const int m0 = tm * kT + wm * 64, n0 = tn * kT + wn * 128 + r16;
  if constexpr (MODE == kHeadLogits) {
    // per row: the maximum over the tile's classes (in units of log 2, at the
    // temperature), the sum of 2^(z - max), codes (max - z) * kHeadSteps
    float* red = reinterpret_cast<float*>(smem);  // [2][4][256]
    const float c = g.z_scale;
    const bool ragged = (tm + 1) * kT > g.V;
    float mx[NI];
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      mx[j] = -INFINITY;
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float z = acc[i][j][e] * c;
          if (ragged && m0 + 16 * i + 4 * grp + e >= g.V) z = -INFINITY;
          acc[i][j][e] = z;
          mx[j] = fmaxf(mx[j], z);
        }
      mx[j] = rows4_max(mx[j]);
    }
    __syncthreads();  // every wave has read the last tile
    if (grp == 0)
#pragma unroll
      for (int j = 0; j < NI; ++j) red[wm * kT + wn * 128 + 16 * j + r16] = mx[j];
    __syncthreads();
    float sum[NI];
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const float* r = red + wn * 128 + 16 * j + r16;
      const float m = fmaxf(fmaxf(r[0], r[kT]), fmaxf(r[2 * kT], r[3 * kT]));
      const float ref = m == -INFINITY ? 0.f : m;
      mx[j] = m;
      sum[j] = 0.f;
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float below = ref - acc[i][j][e];
          sum[j] += __builtin_amdgcn_exp2f(-below);
          acc[i][j][e] = below;
        }
      sum[j] = rows4_sum(sum[j]);
    }
    float* red2 = red + 4 * kT;
    if (grp == 0)
#pragma unroll
      for (int j = 0; j < NI; ++j) red2[wm * kT + wn * 128 + 16 * j + r16] = sum[j];
    __syncthreads();
    if (wm == 0 && grp == 0)
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int n = n0 + 16 * j;
        const float* r = red2 + wn * 128 + 16 * j + r16;
        if (n < rows) g.stats[int64_t(tm) * g.rows_ld + n] = float2{mx[j], (r[0] + r[kT]) + (r[2 * kT] + r[3 * kT])};
      }
    if (!g.zout) return;
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int n = n0 + 16 * j;
#pragma unroll
      for (int i = 0; i < MI; i += 2) {
        uint32_t pk[2][2];
#pragma unroll
        for (int ii = 0; ii < 2; ++ii)
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const uint32_t lo = uint32_t(fminf(fmaf(acc[i + ii][j][2 * q], kHeadSteps, 0.5f), 65535.f));
            const uint32_t hi = uint32_t(fminf(fmaf(acc[i + ii][j][2 * q + 1], kHeadSteps, 0.5f), 65535.f));
            pk[ii][q] = lo | hi << 16;
          }
        const u32x4 v = swap_rows8(pk[0][0], pk[0][1], pk[1][0], pk[1][1]);
        if (n < rows)
          *reinterpret_cast<u32x4*>((uint16_t*)g.zout + int64_t(n) * g.ldz + m0 + 16 * (i + (grp & 1)) + 8 * (grp >> 1)) = v;
      }
    }
  } else if constexpr (MODE == kHeadDh) {
    float* out = g.part + int64_t(sp) * g.rows_ld * g.d;
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int n = n0 + 16 * j;
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        const int m = m0 + 16 * i + 4 * grp;
        if (n < rows && m < g.d) *reinterpret_cast<f32x4*>(out + int64_t(n) * g.d + m) = acc[i][j];
      }
    }
  } else {
    const float scale = *g.scale;
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int n = n0 + 16 * j;
      const bool in = n < g.V;
      const int64_t row = int64_t(n) * g.d;
#pragma unroll
      for (int i = 0; i < MI; i += 2) {
        f32x4 v[2];
#pragma unroll
        for (int ii = 0; ii < 2; ++ii) {
          const int m = m0 + 16 * (i + ii) + 4 * grp;
          v[ii] = acc[i + ii][j] * scale;
          if (g.prev && in && m < g.d) v[ii] += *reinterpret_cast<const f32x4*>(g.prev + row + m);
          if (g.out32 && in && m < g.d) *reinterpret_cast<f32x4*>(g.out32 + row + m) = v[ii];
        }
        if (!g.out16) continue;
        uint32_t pk[2][2];
#pragma unroll
        for (int ii = 0; ii < 2; ++ii)
#pragma unroll
          for (int q = 0; q < 2; ++q)
            pk[ii][q] = uint32_t(f2bf(v[ii][2 * q])) | uint32_t(f2bf(v[ii][2 * q + 1])) << 16;
        const u32x4 u = swap_rows8(pk[0][0], pk[0][1], pk[1][0], pk[1][1]);
        const int m = m0 + 16 * (i + (grp & 1)) + 8 * (grp >> 1);
        if (in && m < g.d) *reinterpret_cast<u32x4*>(g.out16 + row + m) = u;
      }
    }
  }
}

hipError_t launch_head_gemm(int mode, const HeadGemmArgs& g, hipStream_t s) {
  const int tr = (g.rows + kT - 1) / kT, tv = (g.V + kT - 1) / kT, td = (g.d + kT - 1) / kT;
  if (mode == kHeadLogits) head_gemm_kernel<kHeadLogits><<<tr * tv, kThreads, 0, s>>>(g);
  else if (mode == kHeadDh) head_gemm_kernel<kHeadDh><<<tr * td * g.splits, kThreads, 0, s>>>(g);
  else head_gemm_kernel<kHeadDw><<<tv * td, kThreads, 0, s>>>(g);
  return hipGetLastError();
}

}  // namespace dsf
