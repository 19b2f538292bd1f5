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
//
// A workgroup per CU walks its tiles with one stream of k-tiles: the loads run
// two k-tiles ahead, into the next tile while this one ends, so that only its
// epilogue is between two tiles' products.
//
// 8192 rows of width 3584 over 151936 classes: logits 7.1 ms, dh 6.6-6.9, dW 6.7-6.95
// (1.25-1.35 PFLOP/s), at the card's power limit: the clock falls to 1.8 GHz, of
// which the matrix cores are busy 63-68 %. Width 768 over 50304: 740, 590, 540 us, the
// logits' epilogue (two reductions over the tile's rows, an exponential and a code a logit)
// being a quarter of theirs: accumulators fill the registers, so it stands alone. (Logits spill
// 6 registers, dW of half-full tiles 7, between the products' loops and a few times a tile;
// none in a loop over k.)
#include <algorithm>
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
#define DSF_INLINE __attribute__((always_inline))  // for lambdas over register arrays
#define DSF_LDS __attribute__((address_space(3)))
typedef DSF_LDS char LdsChar;

// Two loads of 1 KiB (16 bytes a lane) into LDS at at0 and at1 (addresses of the
// wave; lane l's go to + 16 l). Inline assembly, as the compiler would wait for
// all of them before the next transpose load, which it cannot tell apart from
// them; the callers wait and meet at a barrier. The assembly brings the wait
// states that a scalar operand just written by a vector instruction needs. (M0
// is reserved: the compiler keeps nothing in it.)
__device__ __forceinline__ void head_dma2(u32x4 ra, uint32_t va, uint32_t at0, u32x4 rb, uint32_t vb, uint32_t at1) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 4\n\t"
      "buffer_load_dwordx4 %1, %2, 0 offen lds\n\t"
      "s_mov_b32 m0, %3\n\t"
      "s_nop 0\n\t"
      "buffer_load_dwordx4 %4, %5, 0 offen lds" ::"s"(at0),
      "v"(va), "s"(ra), "s"(at1), "v"(vb), "s"(rb)
      : "memory");
}

// An operand in global memory and its share of a stage: 32 loads of 1 KiB, load
// l = 8 u + wave the wave's u-th. The lane's part of an offset is the same for
// every load.
// COL false: element (x, k) at p[x ld + k]; load l fills tile rows 8 l .. + 7, 128 bytes
//   each, 16-byte chunk c of row r at c ^ (r & 7).
// COL true: element (x, k) at p[k ld + x]; subtile l / 16 (128 columns) rows 4 (l % 16) .. + 3
//   of k, 256 bytes each, chunk c of row r at c ^ key(r), key(r) = 2 ((r & 3) + 4 (r >> 3 & 1)): the
//   sixteen rows of a transpose load, 32 bytes each, then cover the 64 banks twice, the minimum.
// BLOCKS: dz in its blocks, rows being x (COL false) or k (COL true).
// What lies past the operand's last row reads as zeros (the resource ends there);
// of dz by rows of k the rows to the next multiple of 64 are zeros in memory.
template <bool COL, bool BLOCKS>
struct HeadOp {
  const char* base = nullptr;  // of the next k-tile to load
  uint32_t ld2 = 0;            // bytes of a row
  int rows = 0;                // COL: rows of k left; else rows of the tile
  uint32_t voff = 0;
  int64_t step = 0;            // BLOCKS by rows of k: from a quarter of blocks to the next row of blocks
  int quarter = 0;
  __device__ __forceinline__ void set(const void* p, int ld, int64_t nx, int64_t nk, int64_t x0, int kt, int wave,
                                      int lane) {
    ld2 = BLOCKS ? uint32_t(kZClasses) * 2u : uint32_t(ld) * 2u;
    if constexpr (COL) {
      const int c = (lane & 15) ^ (((lane >> 4) + 4 * ((wave >> 1) & 1)) << 1);
      if constexpr (BLOCKS) {
        step = int64_t(ld / kZClasses) * (kZBlock * 2);
        quarter = kt & 3;
        base = (const char*)p + (kt >> 2) * step + (x0 / kZClasses) * (kZBlock * 2) + quarter * (kBK * kZClasses * 2);
        rows = kBK;
        voff = uint32_t(4 * wave + (lane >> 4)) * ld2 + uint32_t(c >> 3) * (kZBlock * 2u) + uint32_t((c & 7) * 16);
      } else {
        base = (const char*)p + int64_t(kt) * kBK * ld2;
        rows = int(nk - int64_t(kt) * kBK);
        voff = uint32_t(4 * wave + (lane >> 4)) * ld2 + uint32_t(x0) * 2u + uint32_t(c * 16);
      }
    } else {
      base = BLOCKS ? (const char*)p + ((x0 / kZRows) * (ld / kZClasses) + kt) * (kZBlock * 2)
                    : (const char*)p + x0 * ld2 + int64_t(kt) * (kBK * 2);
      rows = int(nx - x0 < kT ? nx - x0 : kT);
      voff = uint32_t(8 * wave + (lane >> 3)) * ld2 + uint32_t(((lane & 7) ^ (lane >> 3)) * 16);
    }
  }
  // resource of the next k-tile (none: zeros), which is then the one after. Rows
  // are counted from the k-tile's first byte: an offset past them is one past the
  // operand (COL false: or in its last row, past the k-tiles of this call).
  __device__ __forceinline__ u32x4 next(bool any) {
    const uint64_t b = reinterpret_cast<uint64_t>(base);
    const int n = COL && rows > kBK ? kBK : rows;
    auto uniform = [](uint32_t x) { return uint32_t(__builtin_amdgcn_readfirstlane(int(x))); };
    // (blocks by rows of k: four blocks' quarters)
    const uint32_t bytes = COL && BLOCKS ? uint32_t(3 * kZBlock * 2 + kBK * kZClasses * 2) : uint32_t(n) * ld2;
    const u32x4 r = {uniform(uint32_t(b)), uniform(uint32_t(b >> 32) & 0xffffu), uniform(any && n > 0 ? bytes : 0u),
                     0x00020000u};
    if constexpr (COL && BLOCKS) {
      base += quarter == 3 ? step - 3 * (kBK * kZClasses * 2) : kBK * kZClasses * 2;
      quarter = (quarter + 1) & 3;
    } else if constexpr (BLOCKS) {
      base += kZBlock * 2;
    } else {
      base += COL ? int64_t(kBK) * ld2 : kBK * 2;
      if (COL) rows -= kBK;
    }
    return r;
  }
  __device__ __forceinline__ uint32_t offset(int u) const {
    if constexpr (COL)
      return voff + uint32_t(32 * (u & 1)) * ld2 + uint32_t(u >> 1) * (BLOCKS ? 2u * kZBlock * 2u : 256u);
    return voff + uint32_t(64 * u) * ld2;
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

// A barrier that leaves loads into LDS and stores in flight.
__device__ __forceinline__ void ring_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Two values of [0, 1] as 16-bit fractions of 65535, clamped.
__device__ __forceinline__ uint32_t pack_unit(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pknorm_u16(a, b));
}

// Rows of a piece that take part (dz: and their second terms).
__device__ __forceinline__ int head_piece_rows(const HeadGemmArgs& g, bool dz) {
  const int active = *g.n_active, rows = active - g.row0;
  const int n = rows < 0 ? 0 : rows > g.rows ? g.rows : rows;
  return dz ? head_dz_rows(active, n) : n;
}

// Shares of a tile of dW in the last round, of `left` tiles: as many as fill the grid, each at least
// eight k-tiles long.
__device__ __forceinline__ int head_dw_cut(int left, int nk, int grid) {
  if (left == 0) return 1;
  const int most = nk / 8, fit = grid / left;
  return most < 1 ? 1 : most < fit ? most : fit;
}

__device__ __forceinline__ u32x4 swap_rows8(uint32_t a0, uint32_t a1, uint32_t b0, uint32_t b1) {
  // a: four 16-bit values of block i, b: of block i + 1. After the swap of odd with even
  // 16-lane rows a lane holds eight consecutive values: columns 16 (i + (grp & 1)) + 8 (grp >> 1).
  const auto x = __builtin_amdgcn_permlane16_swap(a0, b0, false, false);
  const auto y = __builtin_amdgcn_permlane16_swap(a1, b1, false, false);
  return u32x4{x[0], y[0], x[1], y[1]};
}
// a and b: 64 bytes of a row (16 a lane, the row's four lanes r16 + 16 grp) each, a row
// to an r16. Lanes of the upper eight rows swap their a with the b of those
// eight rows below: then a holds rows 0-7 and b rows 8-15, 128 bytes of a row
// over eight lanes (r16 < 8 what was a, else what was b), and a store of them
// writes whole lines. They are written past the L2, which holds the operands: a
// round of tiles, 4 MB an XCD, would push all of them out (8192 rows of width 768
// over 50304 classes: logits 807 -> 638 us; dW of 256 rows of width 1536 over 151936
// classes 195 -> 157 us; half lines 4 % slower).
__device__ __forceinline__ void whole_lines(u32x4& a, u32x4& b, bool low) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const uint32_t t = uint32_t(__builtin_amdgcn_mov_dpp(int(low ? b[q] : a[q]), 0x128, 0xF, 0xF, false));  // row_ror:8
    a[q] = low ? a[q] : t;
    b[q] = low ? t : b[q];
  }
}
}  // namespace

// MODE 0: logits (A = W along k, B = h along k); 1: dh (A = W by rows of k, B = dz along k);
// 2: dW (A = h by rows of k, B = dz by rows of k).
// HALF: the last tile of m is at most half full.
template <int MODE, bool HALF>
__global__ __launch_bounds__(kThreads) void head_gemm_kernel(HeadGemmArgs g) {
  constexpr bool ACOL = MODE != kHeadLogits, BCOL = MODE == kHeadDw;
  constexpr int MI = 4, NI = 8;
  __shared__ __attribute__((aligned(65536))) char smem[2 * kStage];
  __shared__ float red[MODE == kHeadLogits ? 8 * kT : 1];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1, r16 = lane & 15, grp = lane >> 4;
  const int rows = head_piece_rows(g, MODE != kHeadLogits);
  const int K = MODE == kHeadLogits ? g.d : MODE == kHeadDh ? g.ldz : rows;
  const int nk = (K + kBK - 1) / kBK;

  // This workgroup's items (a tile, or a share of a tile's k-tiles): as many whole rounds
  // of the grid as there are, each XCD a contiguous range of the tile order in which its
  // workgroups take one item after another; then one of what is left, if it gets one.
  const int tr = (rows + kT - 1) / kT, tv = (g.V + kT - 1) / kT, td = (g.d + kT - 1) / kT;
  const int outer = MODE == kHeadDw ? tv : tr, inner = MODE == kHeadLogits ? tv : td;
  const int nt = outer * inner, per = int(gridDim.x) / kXcds;
  const int splits = MODE == kHeadDh ? *g.splits : 1;
  const int xcd = int(blockIdx.x) % kXcds, place = int(blockIdx.x) / kXcds;
  const int rounds = nt * splits / int(gridDim.x), full = rounds * int(gridDim.x);
  const int cut = MODE == kHeadDw ? head_dw_cut(nt - full, nk, int(gridDim.x)) : 1;
  const int left = (nt * splits - full) * cut, lq = left / kXcds, lr = left % kXcds;
  const int items = rounds + (place < lq + (xcd < lr) ? 1 : 0);
  if (items == 0) return;
  struct Item {
    int tm, tn, kb, ke, split;  // split < 0: a whole tile; else its partial sum's slot
  };
  auto item_of = [&](int i) {
    Item it;
    int tile, share, shares;
    if (i < rounds) {
      const int w = xcd * (full / kXcds) + i * per + place;
      share = w / nt;
      tile = w - share * nt;
      shares = splits;
      it.split = MODE == kHeadDh ? share : -1;
    } else {
      const int w = xcd * lq + (xcd < lr ? xcd : lr) + place;
      if (MODE == kHeadDw) {
        tile = full + w / cut;
        share = w % cut;
        shares = cut;
        it.split = cut > 1 ? w : -1;
      } else {
        share = (full + w) / nt;
        tile = full + w - share * nt;
        shares = splits;
        it.split = MODE == kHeadDh ? share : -1;
      }
    }
    // bands of four tile rows, column by column, share both operands in the L2s (row by
    // row: dW of 4096 rows of width 3584 over 151936 classes 3597 us, so 3474)
    const GemmTile t = gemm_tile(tile, outer, inner, 4);
    it.tm = t.tn;
    it.tn = t.tm;  // out[n][m]: rows of the tile order are n
    it.kb = int(int64_t(nk) * share / shares);
    it.ke = int(int64_t(nk) * (share + 1) / shares);
    return it;
  };

  const uint32_t lds = uint32_t(__builtin_amdgcn_readfirstlane(int(uint32_t(uintptr_t((DSF_LDS char*)smem)))));
  HeadFrag<ACOL> fa(lds, lane, wm * 64);
  HeadFrag<BCOL> fb(lds + kOpBytes, lane, wn * 128);
  f32x4 acc[MI][NI];

  // The stream of loads: k-tile lk of item li, two k-tiles ahead of the products.
  HeadOp<ACOL, false> A;
  HeadOp<BCOL, MODE != kHeadLogits> B;
  int li = -1, lk = 0, lke = 0;
  u32x4 ra, rb;
  const int chunk_k = 8 * ((lane & 7) ^ (lane >> 3));
  // Sets the next k-tile's resources; returns what moves the chunks past the end of
  // a row (logits of a width that is no multiple of 64) out of range.
  auto start = [&]() DSF_INLINE {
    if (lk == lke && li < items) {
      if (++li < items) {
        const Item it = item_of(li);
        lk = it.kb;
        lke = it.ke;
        A.set(MODE == kHeadDw ? g.h : g.w, g.d, MODE == kHeadLogits ? g.V : g.d, MODE == kHeadDh ? g.V : K,
              int64_t(it.tm) * kT, lk, wave, lane);
        B.set(MODE == kHeadLogits ? g.h : g.z, MODE == kHeadLogits ? g.d : g.ldz, MODE == kHeadDw ? g.ldz : rows, K,
              int64_t(it.tn) * kT, lk, wave, lane);
      }
    }
    const bool any = li < items;
    ra = A.next(any);
    rb = B.next(any);
    const uint32_t past = MODE == kHeadLogits && lk * kBK + chunk_k >= K ? 0x80000000u : 0u;
    lk += any;
    return past;
  };
  // The wave's loads u of A and B, into the stage at st.
  auto issue = [&](uint32_t st, int u, uint32_t past) DSF_INLINE {
    head_dma2(ra, A.offset(u) + past, st + 1024u * uint32_t(8 * u + wave), rb, B.offset(u) + past,
              st + kOpBytes + 1024u * uint32_t(8 * u + wave));
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
  // the other set (substep ks) and (S = 1) a tile's loads into the stage at dma.
  // (dW, whose reads are all transpose loads, two to a fragment: one fragment at a
  // time, 8192 x 151936 x 3584: +3 %; the others lose as much by it.)
  auto substep = [&](auto Sc, int ks, uint32_t dma, uint32_t past) DSF_INLINE {
    constexpr int S = decltype(Sc)::value;
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(af[S][i], bq[S][j], acc[i][j], 0, 0, 0);
        if constexpr (MODE == kHeadDw) {
          const int x = i * NI + j;
          __builtin_amdgcn_sched_barrier(0);
          if (x % 2 == 1 && x / 2 < R) read_n(1 - S, ks, x / 2);
          if (S == 1 && j == 5) issue(dma, i, past);
          __builtin_amdgcn_sched_barrier(0);
        } else if (j == 0) {
          __builtin_amdgcn_sched_barrier(0);
          if (i < MI - 1) {
#pragma unroll
            for (int n = i * R / (MI - 1); n < (i + 1) * R / (MI - 1); ++n) read_n(1 - S, ks, n);
          }
          if (S == 1) issue(dma, i, past);
          __builtin_amdgcn_sched_barrier(0);
        } else if (j == NI - 1) {
          __builtin_amdgcn_sched_barrier(0);
        }
      }
  };
  if (nk > 0) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint32_t past = start();
#pragma unroll
      for (int u = 0; u < 4; ++u) issue(lds ^ (t * kStage), u, past);
    }
    asm volatile("s_waitcnt vmcnt(8)\n\ts_barrier" ::: "memory");
#pragma unroll
    for (int n = 0; n < R; ++n) read_n(0, 0, n);
  }
  uint32_t cur = lds;
  for (int item = 0; item < items; ++item) {
    const Item it = item_of(item);
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // One k-tile. All its fragments are in registers by the middle, where the
    // barrier publishes the next k-tile and frees this one's stage. (Past the
    // stream's end zeros are loaded and read; nothing uses them.)
    auto middle = [&]() DSF_INLINE {
      const uint32_t past = start();
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      fa.at ^= kStage;
      fb.at ^= kStage;
      return past;
    };
    if (!HALF || it.tm * kT + wm * 64 < g.d) {
      for (int kt = it.kb; kt < it.ke; ++kt) {
        substep(std::integral_constant<int, 0>(), 1, 0, 0);
        const uint32_t past = middle();
        substep(std::integral_constant<int, 1>(), 0, cur, past);
        cur ^= kStage;
      }
    } else {
      // No column for this wave, one of a SIMD's two: its loads alone, and the next
      // item's first fragments.
      for (int kt = it.kb; kt < it.ke; ++kt) {
        const uint32_t past = middle();
#pragma unroll
        for (int u = 0; u < 4; ++u) issue(cur, u, past);
        cur ^= kStage;
      }
#pragma unroll
      for (int n = 0; n < R; ++n) read_n(0, 0, n);
    }
    // lane holds out[n = 16 j + r16][m = 16 i + 4 grp + e] of its wave's part
    const int m0 = it.tm * kT + wm * 64, n0 = it.tn * kT + wn * 128 + r16;
    if constexpr (MODE == kHeadLogits) {
      // per row: the maximum over the tile's classes (in units of log 2, at the
      // temperature), the sum of 2^(z - max), and codes of max - z
      const float c = g.z_scale;
      if ((it.tm + 1) * kT > g.V) {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (m0 + 16 * i + 4 * grp + e >= g.V)
#pragma unroll
              for (int j = 0; j < NI; ++j) acc[i][j][e] = -INFINITY;
      }
      float mx[NI];
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        mx[j] = acc[0][j][0];
#pragma unroll
        for (int x = 1; x < 16; ++x) mx[j] = fmaxf(mx[j], acc[x >> 2][j][x & 3]);
        mx[j] = rows4_max(mx[j]);
      }
      if (grp == 0)
#pragma unroll
        for (int j = 0; j < NI; ++j) red[wm * kT + wn * 128 + 16 * j + r16] = mx[j];
      ring_barrier();
      float* const red2 = red + 4 * kT;
      float top[NI];
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        if (j % 2 == 0 && rows - it.tn * kT <= wn * 128 + 16 * j) break;  // no row that takes part (one row, 594 tiles: 77 -> 72 us)
        const float* r = red + wn * 128 + 16 * j + r16;
        top[j] = c * fmaxf(fmaxf(r[0], r[kT]), fmaxf(r[2 * kT], r[3 * kT]));
        const float ref = top[j] == -INFINITY ? 0.f : top[j];
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float below = fmaf(-c, acc[i][j][e], ref);
            sum += __builtin_amdgcn_exp2f(-below);
            acc[i][j][e] = below * (1.f / kHeadReach);
          }
        sum = rows4_sum(sum);
        if (grp == 0) red2[wm * kT + wn * 128 + 16 * j + r16] = sum;
      }
      ring_barrier();
      if (wm == 0 && grp == 0)
#pragma unroll
        for (int j = 0; j < NI; ++j) {
          const int n = n0 + 16 * j;
          const float* r = red2 + wn * 128 + 16 * j + r16;
          if (n < rows)
            g.stats[int64_t(it.tm) * g.rows_ld + n] = float2{top[j], (r[0] + r[kT]) + (r[2 * kT] + r[3 * kT])};
        }
      if (g.zout) {
        const bool low = r16 < 8;
        uint16_t* to = (uint16_t*)g.zout + head_z_at(it.tn * kT + wn * 128, it.tm * kT + wm * 64, g.ldz) +
                       (r16 & 7) * kZClasses + 16 * (grp & 1) + 8 * (grp >> 1) + (low ? 0 : 32);
        int left = rows - (n0 - r16) - (r16 & 7);
#pragma unroll
        for (int j = 0; j < NI; ++j) {
          u32x4 v[2];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const f32x4 x = acc[2 * h][j], y = acc[2 * h + 1][j];
            v[h] = swap_rows8(pack_unit(x[0], x[1]), pack_unit(x[2], x[3]), pack_unit(y[0], y[1]), pack_unit(y[2], y[3]));
          }
          whole_lines(v[0], v[1], low);
#pragma unroll
          for (int h = 0; h < 2; ++h)
            if (left > 8 * h) __builtin_nontemporal_store(v[h], reinterpret_cast<u32x4*>(to + 8 * h * kZClasses));
          to += 16 * kZClasses;
          left -= 16;
          asm volatile("" : "+v"(to), "+v"(left));  // one address at a time: all of them together spill
        }
      }
    } else if (MODE == kHeadDh || it.split >= 0) {
      // a partial sum: dh [split][n][m]; dW [slot][256][256]
      float* out = MODE == kHeadDh ? g.part + int64_t(it.split) * g.rows_ld * g.d + int64_t(n0) * g.d + m0
                                   : g.part + (int64_t(it.split) * kT + wn * 128 + r16) * kT + wm * 64;
      const int ld = MODE == kHeadDh ? g.d : kT;
#pragma unroll
      for (int j = 0; j < NI; ++j)
#pragma unroll
        for (int i = 0; i < MI; ++i)
          if (MODE == kHeadDw || (n0 + 16 * j < rows && m0 + 16 * i + 4 * grp < g.d))
            *reinterpret_cast<f32x4*>(out + int64_t(16 * j) * ld + 16 * i + 4 * grp) = acc[i][j];
    } else {
      const float scale = *g.scale;
      const bool low = r16 < 8;
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int n = n0 + 16 * j;
        const bool in = n < g.V;
        const int64_t row = int64_t(n) * g.d;
        u32x4 v16[2];
#pragma unroll
        for (int i = 0; i < MI; i += 2) {
          f32x4 v[2];
#pragma unroll
          for (int ii = 0; ii < 2; ++ii) {
            const int m = m0 + 16 * (i + ii) + 4 * grp;
            v[ii] = acc[i + ii][j] * scale;
            if (g.prev && in && m < g.d) v[ii] += *reinterpret_cast<const f32x4*>(g.prev + row + m);
            if (g.out32 && in && m < g.d) __builtin_nontemporal_store(v[ii], reinterpret_cast<f32x4*>(g.out32 + row + m));
          }
          uint32_t pk[2][2];
#pragma unroll
          for (int ii = 0; ii < 2; ++ii)
#pragma unroll
            for (int q = 0; q < 2; ++q)
              pk[ii][q] = uint32_t(f2bf(v[ii][2 * q])) | uint32_t(f2bf(v[ii][2 * q + 1])) << 16;
          v16[i >> 1] = swap_rows8(pk[0][0], pk[0][1], pk[1][0], pk[1][1]);
        }
        if (!g.out16) continue;
        whole_lines(v16[0], v16[1], low);
        const int m = m0 + 16 * (grp & 1) + 8 * (grp >> 1) + (low ? 0 : 32);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int to = n - r16 + 8 * h + (r16 & 7);
          if (to < g.V && m < g.d) __builtin_nontemporal_store(v16[h], reinterpret_cast<u32x4*>(g.out16 + int64_t(to) * g.d + m));
          __builtin_amdgcn_sched_barrier(0);  // one address after another
        }
      }
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // loads past the stream's end write LDS
}

// dW of the tiles that the last, incomplete round cut along the rows: their partial sums
// added in order, then as in the kernel above. A workgroup takes 32 rows of a tile.
__global__ __launch_bounds__(256) void head_dw_join_kernel(HeadGemmArgs g, int grid) {
  const int rows = head_piece_rows(g, true), nk = (rows + kBK - 1) / kBK;
  const int tv = (g.V + kT - 1) / kT, td = (g.d + kT - 1) / kT, nt = tv * td, full = nt / grid * grid;
  const int cut = head_dw_cut(nt - full, nk, grid);
  if (cut <= 1) return;
  const int t = int(blockIdx.x) >> 3;
  const GemmTile gt = gemm_tile(full + t, tv, td, 4);
  const int n = gt.tm * kT + (int(blockIdx.x) & 7) * 32 + int(threadIdx.x >> 3);
  const float scale = *g.scale;
  if (n >= g.V) return;
  const float* src = g.part + (int64_t(t) * cut * kT + (n & (kT - 1))) * kT;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int mc = 8 * (int(threadIdx.x & 7) + 8 * u), m = gt.tn * kT + mc;
    if (m >= g.d) continue;
    float v[8], x[8];
    load8(src + mc, v);
    for (int s = 1; s < cut; ++s) {
      load8(src + int64_t(s) * kT * kT + mc, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += x[e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= scale;
    const int64_t at = int64_t(n) * g.d + m;
    if (g.prev) {
      load8(g.prev + at, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += x[e];
    }
    if (g.out32) store8(g.out32 + at, v);
    if (g.out16) store8(g.out16 + at, v);
  }
}

hipError_t launch_head_gemm(int mode, const HeadGemmArgs& g, hipStream_t s) {
  const int64_t tr = (g.rows + kT - 1) / kT, tv = (g.V + kT - 1) / kT, td = (g.d + kT - 1) / kT;
  auto grid = [](int64_t items) { return dim3(uint32_t(std::min<int64_t>(kHeadGrid, (items + kXcds - 1) / kXcds * kXcds))); };
  if (mode == kHeadLogits) {
    head_gemm_kernel<kHeadLogits, false><<<grid(tr * tv), kThreads, 0, s>>>(g);
  } else if (mode == kHeadDh) {
    head_gemm_kernel<kHeadDh, false><<<kHeadGrid, kThreads, 0, s>>>(g);
  } else {
    const int nt = int(tv * td), left = nt % kHeadGrid;
    // Leaving out the products past a width like 896 takes registers, 3 % of whole tiles' time, and
    // is worth it where a workgroup has some of either kind (6554 rows, 151936 classes: dW 1648 ->
    // 1560 us; dh, whose workgroups have few, gains nothing).
    if ((g.d - 1) % kT < kT / 2) head_gemm_kernel<kHeadDw, true><<<kHeadGrid, kThreads, 0, s>>>(g);
    else head_gemm_kernel<kHeadDw, false><<<kHeadGrid, kThreads, 0, s>>>(g);
    if (left && 2 * left <= kHeadGrid) head_dw_join_kernel<<<left * 8, 256, 0, s>>>(g, kHeadGrid);
  }
  return hipGetLastError();
}

}  // namespace dsf
