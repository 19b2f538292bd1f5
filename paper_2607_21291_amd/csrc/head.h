// Shared by the head's losses: the plan of a call, and the arguments of its
// products and of the kernels between them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dsf {

// A logit is held as its distance below its tile's row maximum, in 65535 steps of
// kHeadReach factors of two (1024 steps to a factor; what lies lower counts as 0).
// Half a step changes a probability by 3.4e-4 relative, a tenth of the rounding
// to bf16 that the product with it needs anyway.
constexpr float kHeadReach = 64.f;
constexpr int kHeadGrid = 256;  // workgroups of a product: one per CU
constexpr int kHeadTile = 256;  // classes of a tile of the logits
constexpr int kHeadMaxTop = 1024;

// The codes, and dz after them (bf16), lie in blocks of 256 rows by 64 classes, rows of
// 128 bytes: a block is what a product reads of them for one of its k-tiles (by
// rows: four quarters of blocks), and an eighth of a wave's tile of logits. Rows
// of all classes, 300 KB apart, had a CU read from 40 pages of 2 MB at a time.
constexpr int kZRows = 256, kZClasses = 64, kZBlock = kZRows * kZClasses;
__host__ __device__ inline int64_t head_z_at(int row, int c, int ldz) {
  return (int64_t(row / kZRows) * (ldz / kZClasses) + c / kZClasses) * kZBlock + (row % kZRows) * kZClasses + c % kZClasses;
}

// dz is rounded to bf16. Over many rows that adds as much to the gradients' error as their own
// rounding; in a call of few the errors of some large entries (a target's p - q) do not
// average out, up to 2^-8 of a row's gradient. There are few rows' tiles to spare then: up to
// kHeadTwin rows (that take part) have dz in two terms, what the first of row s leaves in row
// n_active + s (2 rows of width 3584 over 151936 classes: relative error 0.0034 -> 0.0016, the
// results' own rounding, for 791 -> 797 us; 64 of width 896: dh 66 -> 72 us, dW 85 -> 102).
constexpr int kHeadTwin = 128;
__host__ __device__ inline int head_dz_rows(int n_active, int rows) { return n_active <= kHeadTwin ? 2 * rows : rows; }

// fp32: rows of a tile of the logits and of dh. Of few rows 64 where that pads them less
// (64 rows of width 768 over 50304 classes: logits 117 -> 79 us, dh 96 -> 59).
constexpr int kHeadF32Few = 320;
__host__ __device__ inline int head_f32_rows(int rows) {
  return rows <= kHeadF32Few && (rows + 127) / 128 * 128 - rows >= 64 ? 64 : 128;
}

enum HeadMode { kHeadLogits = 0, kHeadDh = 1, kHeadDw = 2 };

// One of a call's three products, over a piece of its active rows (bf16; fp32
// the same with float operands).
struct HeadGemmArgs {
  const void* h;        // active rows of this piece [rows, d]
  const void* w;        // [V, d]
  const void* z;        // dz of rows x ldz classes, in blocks (fp32: [rows, ldz])
  void* zout;           // codes, in blocks (fp32: logits in units of log 2, [rows, ldz]); null: statistics alone
  float2* stats;        // bf16: [classes / 256][rows_ld] (maximum, sum)
  float* part;          // partial sums: of dh [splits][rows_ld][d], of dW's last round [kHeadGrid][256][256]
  const float* prev;    // dW so far, fp32 (nullable)
  float* out32;         // dW in fp32 (nullable)
  uint16_t* out16;      // dW in bf16 (nullable)
  const float* scale;   // factor of dW (device)
  const int32_t* n_active;  // active rows of the call (device)
  float z_scale;        // log2(e) / temperature
  int row0, rows, rows_ld;  // the piece: its first active row, its rows at most, leading dimension of the above
  int V, d, ldz;
  const int32_t* splits;  // dh: shares of the classes (device), at most `most`
  int most;
};
hipError_t launch_head_gemm(int mode, const HeadGemmArgs& g, hipStream_t s);      // kernels_headgemm.hip
hipError_t launch_head_gemm_f32(int mode, const HeadGemmArgs& g, hipStream_t s);  // kernels_headf32.hip

}  // namespace dsf
