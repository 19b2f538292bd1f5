// Attention of each sequence's new tokens over its pages (gfx950).
//
// The query heads of a kv head and a sequence's new tokens are the rows of
// one problem, token-major (row m = token * G + head), so that a tile of rows
// reads a key or value once for all of them. Rows are cut into tiles of BM,
// a sequence's slots into splits of equal length where there are too few
// tiles for the chip (paged_item); a workgroup takes one (tile, split, kv
// head), keeps the running maximum and sum of the softmax in fp32, and writes
// the result, or its share of it, which paged_join_kernel adds up in the order of the splits.
#include <algorithm>

#include "paged.h"

namespace dsf {

struct PagedKernelArgs {
  PagedPool pool;
  PagedBatch pb;
  const void* q; int64_t q_row, q_head;
  void* out; int64_t o_row, o_head;
  int G, window;
  int bm_shift;    // log2 of the rows per tile
  int m_lo, m_hi;  // sequences with m_lo < rows * G <= m_hi take part
  int items;       // per kv head: the grid's, and no more than that have a place in part_o
  int target;      // of them to cut the work into (0: no splits)
  int split_min;   // least blocks of 64 slots per split
  float* part_o;   // [item][kv head][BM][HD]
  float2* part_ml; // [item][kv head][BM]: maximum (log2 units), sum
};

// ------------------------------------------------------------ work items

// Sum and inclusive prefix sum of a small number over the wave.
__device__ __forceinline__ int wave_prefix(int v) {
#define DSF_SCAN(ctrl, rows) v += __builtin_amdgcn_update_dpp(0, v, ctrl, rows, 0xf, false)
  DSF_SCAN(0x111, 0xf);  // row_shr 1, 2, 4, 8: within 16 lanes
  DSF_SCAN(0x112, 0xf);
  DSF_SCAN(0x114, 0xf);
  DSF_SCAN(0x118, 0xf);
  DSF_SCAN(0x142, 0xa);  // lane 15 of each row to the next row (rows 1 and 3)
  DSF_SCAN(0x143, 0xc);  // lane 31 to rows 2 and 3
#undef DSF_SCAN
  return v;
}

// How sequence b's work is cut: `tiles` tiles of BM rows, slots from `lo` (a
// multiple of 64) to kv in splits of `len`.
struct PagedShape {
  int n, row0, kv;  // rows, first row, slots
  int M;            // rows * G that take part
  int tiles, lo, blocks;
};
__device__ __forceinline__ PagedShape paged_shape(const PagedKernelArgs& a, int b) {
  const PagedSeq s = paged_seq(a.pb, b);
  PagedShape w;
  w.n = s.n;
  w.row0 = s.row0;
  w.kv = s.kv;
  w.M = min(s.n, a.pb.max_rows) * a.G;
  // (row_start that does not ascend may claim more tiles than there are items; the minimum keeps the sums of them small)
  w.tiles = w.M > a.m_lo && w.M <= a.m_hi ? min((w.M + (1 << a.bm_shift) - 1) >> a.bm_shift, a.items) : 0;
  w.lo = a.window ? max(s.kv - s.n - a.window + 1, 0) & ~63 : 0;
  w.blocks = (max(s.kv - w.lo, 0) + 63) >> 6;
  return w;
}
struct PagedItem {
  int b;       // -1: none
  int first;   // the sequence's first item
  int local;   // this one's number among them
  int len;     // slots per split
  int splits;  // of the sequence
};
constexpr int kNoSplit = 1 << 19;  // blocks: more slots than a sequence may have
// Blocks of 64 slots per split: all the work (tiles times blocks) over the
// number of items aimed at, so that items are alike whatever the sequences'
// lengths. Sequences in lanes: b = lane of the first 64 in w.
__device__ __forceinline__ int paged_split_blocks(const PagedKernelArgs& a, const PagedShape& w, int lane) {
  if (a.target == 0) return kNoSplit;
  int sum = w.tiles * w.blocks;
  for (int b0 = 64; b0 < a.pb.B; b0 += 64) {
    if (b0 + lane < a.pb.B) {
      const PagedShape x = paged_shape(a, b0 + lane);
      sum += x.tiles * x.blocks;
    }
  }
  sum = __builtin_amdgcn_readlane(wave_prefix(sum), 63);
  return max((sum + a.target - 1) / a.target, a.split_min);
}
__device__ __forceinline__ int paged_splits(const PagedShape& w, int per) { return max((w.blocks + per - 1) / per, 1); }

// The sequence that item `item` (of one kv head) belongs to.
__device__ __forceinline__ PagedItem paged_item(const PagedKernelArgs& a, int item, int lane) {
  PagedShape w = {};
  if (lane < a.pb.B) w = paged_shape(a, lane);
  const int per = paged_split_blocks(a, w, lane);
  PagedItem it = {-1, 0, 0, 0, 0};
  int first = 0;
  for (int b0 = 0; b0 < a.pb.B; b0 += 64) {
    if (b0) {
      w = PagedShape{};
      if (b0 + lane < a.pb.B) w = paged_shape(a, b0 + lane);
    }
    const int splits = paged_splits(w, per), c = min(w.tiles * splits, a.items);
    const int end = wave_prefix(c);
    const uint64_t over = __builtin_amdgcn_ballot_w64(first + end > item);
    if (over) {
      const int l = __builtin_ctzll(over);
      it.b = b0 + l;
      it.first = first + __builtin_amdgcn_readlane(end, l) - __builtin_amdgcn_readlane(c, l);
      it.local = item - it.first;
      it.len = per << 6;
      it.splits = __builtin_amdgcn_readlane(splits, l);
      return it;
    }
    first += __builtin_amdgcn_readlane(end, 63);
  }
  return it;
}

// One item's tile and slots. Splits outermost: the tiles of one split read
// the same slots at the same time; within a split the last tile, which sees
// the most, is the first.
struct PagedWork {
  int b, n, row0, kv, M, lo;
  int tile;            // of BM rows
  int p0;              // slot of the sequence's first row (may be negative)
  int begin, end;      // slots of this item that some row of the tile sees
  int splits;
};
__device__ __forceinline__ void paged_range(const PagedKernelArgs& a, const PagedShape& w, int tile, int split, int len,
                                            int* begin, int* end) {
  const int p0 = w.kv - w.n;
  const int m0 = tile << a.bm_shift, m1 = min(m0 + (1 << a.bm_shift), w.M) - 1;
  int e = p0 + m1 / a.G + 1, s = a.window ? max(p0 + m0 / a.G - a.window + 1, 0) : 0;
  s = max(s & ~63, w.lo + split * len);
  e = min(e, min(w.kv, w.lo + (split + 1) * len));
  *begin = s;
  *end = max(e, s);
}
__device__ __forceinline__ PagedWork paged_work(const PagedKernelArgs& a, const PagedItem& it) {
  PagedWork k;
  const PagedShape w = paged_shape(a, it.b);
  k.b = it.b;
  k.n = w.n;
  k.row0 = w.row0;
  k.kv = w.kv;
  k.M = w.M;
  k.lo = w.lo;
  k.p0 = w.kv - w.n;
  const int split = it.local / w.tiles;
  k.tile = w.tiles - 1 - (it.local - split * w.tiles);
  k.splits = it.splits;
  paged_range(a, w, k.tile, split, it.len, &k.begin, &k.end);
  return k;
}

// Pages of a sequence, 64 at a time in a register of the wave: lane i holds
// page `base + i`.
struct PagedTable {
  int ids, base;
  __device__ __forceinline__ void load(const PagedKernelArgs& a, int b, int from, int lane) {
    base = from;
    ids = paged_page(a.pb, b, from + lane, a.pool.n_pages);
  }
  __device__ __forceinline__ int at(const PagedKernelArgs& a, int b, int i, int lane) {
    if (i >= base + 64) load(a, b, i, lane);
    return __builtin_amdgcn_readlane(ids, i - base);
  }
};

// Maximum and sum over a lane and the lane 32 beside it.
__device__ __forceinline__ float pair32_max(float v) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float pair32_sum(float v) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// ------------------------------------------------------- LDS tiles of slots

// R slots of HD bf16, row-major; 16-byte chunk c of row r lies at chunk
// c ^ swz(r). swz spreads over the banks both the fragments of 8 consecutive
// rows at one chunk and the transpose loads' four consecutive rows at four
// consecutive chunks.
template <int HD>
struct SlotTile {
  static constexpr int kRowBytes = 2 * HD;
  static constexpr int kChunks = HD / 8;
  __device__ static __forceinline__ int swz(int r) {
    if constexpr (HD == 128) return ((r & 3) << 2) | ((r >> 2) & 3);
    else if constexpr (HD == 64) return ((r & 2) << 1) | ((r >> 2) & 3);
    else return (r >> 2) & 3;
  }
};

// 16 slots from `slot` on of one kv head to LDS at `lds` (a tile's row 16 i):
// bf16 by DMA, each lane 16 bytes at a time; slots at or past `end` become
// zeros. All 16 lie in one page.
template <int HD>
struct DmaSlots {
  __device__ static __forceinline__ void load(const void* pool, const PagedKernelArgs& a, int page, int kvh, int slot,
                                              int end, char* lds, int lane) {
    using S = SlotTile<HD>;
    const int mask = (1 << a.pb.page_shift) - 1;
    const int64_t row = ((int64_t(page) * a.pool.Hkv + kvh) << a.pb.page_shift) + (slot & mask);
    const int bytes = min(max(end - slot, 0), 16) * S::kRowBytes;
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<char*>(static_cast<const char*>(pool)) + row * S::kRowBytes, (short)0, bytes, 0x00020000);
#pragma unroll
    for (int e = 0; e < 16 * S::kRowBytes / 1024; ++e) {
      const int byte = 1024 * e + 16 * lane;
      const int r = byte / S::kRowBytes, c = byte % S::kRowBytes / 16;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)(lds + 1024 * e), 16,
                                               r * S::kRowBytes + ((c ^ S::swz(r)) << 4), 0, 0, 0);
    }
  }
};

// The same of e4m3 codes: loaded into registers, 16 codes of a slot at a
// time, and later widened into the tile.
template <int HD>
struct CodeSlots {
  static constexpr int kCpr = HD / 16;                       // 16-byte loads per slot
  static constexpr int kLoads = kCpr >= 4 ? 16 * kCpr / 64 : 1;
  u32x4 c[kLoads];
  uint32_t e[kLoads];
  __device__ __forceinline__ void load(const void* pool, const uint8_t* exps, const PagedKernelArgs& a, int page, int kvh,
                                       int slot, int end, int lane) {
    const int mask = (1 << a.pb.page_shift) - 1;
    const int64_t row = ((int64_t(page) * a.pool.Hkv + kvh) << a.pb.page_shift) + (slot & mask);
    const int rows = min(max(end - slot, 0), 16);
    // slots at or past `end` load as zeros, their exponents too: code 0 times 0
    const auto rc = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<char*>(static_cast<const char*>(pool)) + row * HD, (short)0, rows * HD, 0x00020000);
    const auto re = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(exps) + row, (short)0, rows, 0x00020000);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      c[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rc, 1024 * i + 16 * lane, 0, 0));
      e[i] = __builtin_amdgcn_raw_buffer_load_b8(re, 64 / kCpr * i + lane / kCpr, 0, 0);
    }
  }
  __device__ __forceinline__ void store(char* lds, int lane) const {
    using S = SlotTile<HD>;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = 64 / kCpr * i + lane / kCpr, ch = 2 * (lane % kCpr);
      const float s = paged_scale(e[i]);
      if (r < 16) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const u32x2 x = paged_widen4(c[i][2 * h], s), y = paged_widen4(c[i][2 * h + 1], s);
          *reinterpret_cast<u32x4*>(lds + r * S::kRowBytes + (((ch + h) ^ S::swz(r)) << 4)) =
              u32x4{x[0], x[1], y[0], y[1]};
        }
      }
    }
  }
};

// A masked slot weighs nothing, but 0 times an infinite or NaN value is NaN.
// Where a tile hides slots from some of its rows, such values are therefore
// taken out of the product (finite_or_zero) and counted in a second one of
// codes (1: inf, 256: -inf, 65536: NaN, exact sums of at most 64) with ones
// at the slots that a row sees, and what a row saw is added to its sum.
//
// Bits 15 and 31 of the result: whether a half of some word has an exponent
// field of ones (adding one to that field carries into them then).
__device__ __forceinline__ uint32_t not_finite_bits(bf16x8 v) {
  const u32x4 w = __builtin_bit_cast(u32x4, v);
  uint32_t r = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) r |= (w[i] & 0x7f807f80u) + 0x00800080u;
  return r & 0x80008000u;
}
__device__ __forceinline__ bf16x8 finite_or_zero(bf16x8 v) {
  bf16x8 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = fabsf(float(v[i])) < INFINITY ? v[i] : (__bf16)0.0f;
  return r;
}
__device__ __forceinline__ bf16x8 not_finite_codes(bf16x8 v) {
  bf16x8 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = float(v[i]);
    r[i] = (__bf16)(x != x ? 65536.0f : x == INFINITY ? 1.0f : x == -INFINITY ? 256.0f : 0.0f);
  }
  return r;
}
// what a sum of codes adds to an accumulator
__device__ __forceinline__ float not_finite_sum(float c) {
  const float low = c - 256.0f * floorf(c / 256.0f);  // infinities
  if (c == 0.f) return 0.f;
  if (c >= 65536.0f || (low > 0.f && c > low)) return NAN;
  return low > 0.f ? INFINITY : -INFINITY;
}

// ---------------------------------------------------------- chunks of tokens

// Eight transpose loads: for four steps of 16 slots (two of `steps` 16-slot
// halves each) the V^T operand of v_mfma_f32_32x32x16_bf16 for 32 dims. Issue
// and wait in one statement; the DMA in flight fills the other stage.
template <int ROW>
__device__ __forceinline__ void lds_read_tr8(uint32_t addr0, uint32_t addr1, u32x2 (&v)[8]) {
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8\n\t"
      "ds_read_b64_tr_b16 %1, %9\n\t"
      "ds_read_b64_tr_b16 %2, %8 offset:%10\n\t"
      "ds_read_b64_tr_b16 %3, %9 offset:%10\n\t"
      "ds_read_b64_tr_b16 %4, %8 offset:%11\n\t"
      "ds_read_b64_tr_b16 %5, %9 offset:%11\n\t"
      "ds_read_b64_tr_b16 %6, %8 offset:%12\n\t"
      "ds_read_b64_tr_b16 %7, %9 offset:%12\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7])
      : "v"(addr0), "v"(addr1), "n"(16 * ROW), "n"(32 * ROW), "n"(48 * ROW)
      : "memory");
}

// A workgroup of four waves takes 128 NQ rows, a wave 32 NQ of them, and 64
// slots at a time, staged by all four (two stages).
//
// S^T = K Q^T with v_mfma_f32_32x32x16_bf16: lane (r32, hi) holds of row r32
// the scores of slots 32 kb + 8 (i / 4) + 4 hi + i % 4, i < 16, so a row's
// maximum needs one exchange between two lanes, and its probabilities lie as
// the B operand of O^T += V^T P^T wants them if the product takes the slots
// in that order: step s covers 16 slots, element j of lane (., hi) being slot
// 16 s + 4 hi + j % 4 + 8 (j / 4). Probabilities are rounded to bf16 for that
// product (off by 2^-8 at most each, and the row's sum is of the rounded
// ones); maximum, sum and accumulators are fp32.
template <int HD, bool E8, int NQ>
__global__ __launch_bounds__(256) void paged_chunk_kernel(PagedKernelArgs a) {
  using S = SlotTile<HD>;
  constexpr int BM = 128 * NQ, NS = HD / 16, ND = HD / 32;
  constexpr int kTile = 64 * S::kRowBytes, kStage = 2 * kTile;
  __shared__ __attribute__((aligned(16))) char smem[2 * kStage];
  const int tid = threadIdx.x, lane = tid & 63, r32 = lane & 31, hi = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // kv head innermost: consecutive workgroups go to different XCDs, so that
  // (with 8 heads or a divisor of 8) an XCD's L2 sees the slots of few heads
  const int item = int(blockIdx.x) / a.pool.Hkv, kvh = int(blockIdx.x) - item * a.pool.Hkv;
  const PagedItem it = paged_item(a, item, lane);
  if (it.b < 0) return;
  const PagedWork w = paged_work(a, it);
  if (w.splits > 1 && w.begin >= w.end) return;  // a split that none of the tile's rows sees

  // this wave's rows: row m of the sequence, its token's slot
  int slot_of[NQ];
  bool live[NQ];
  bf16x8 qf[NQ][NS];
  const int m0 = w.tile * BM + wave * 32 * NQ;
#pragma unroll
  for (int qi = 0; qi < NQ; ++qi) {
    const int m = m0 + 32 * qi + r32, mc = min(m, w.M - 1);
    const int tok = mc / a.G, g = mc - tok * a.G;
    live[qi] = m < w.M;
    slot_of[qi] = w.p0 + tok;
    const uint16_t* qp = static_cast<const uint16_t*>(a.q) + int64_t(w.row0 + tok) * a.q_row + int64_t(kvh * a.G + g) * a.q_head;
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[qi][s] = *reinterpret_cast<const bf16x8*>(qp + 16 * s + 8 * hi);
  }
  // slots that every row of the wave sees: [see_lo, see_hi)
  const int see_hi = w.p0 + min(m0, w.M - 1) / a.G + 1;
  const int see_lo = a.window ? w.p0 + min(m0 + 32 * NQ - 1, w.M - 1) / a.G - a.window + 1 : 0;
  // and that some row sees
  const int any_hi = m0 < w.M ? w.p0 + min(m0 + 32 * NQ - 1, w.M - 1) / a.G + 1 : 0;

  f32x16 o[NQ][ND];
  float m_run[NQ], l_run[NQ];
#pragma unroll
  for (int qi = 0; qi < NQ; ++qi) {
    m_run[qi] = -INFINITY;
    l_run[qi] = 0.f;
#pragma unroll
    for (int db = 0; db < ND; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[qi][db][i] = 0.f;
  }
  const float sc = 1.4426950408889634f / sqrtf(float(HD));  // log2(e) / sqrt(hd)

  // staging: this wave brings slots 16 wave .. + 15 of every tile
  PagedTable tab;
  const int ntiles = (w.end - w.begin + 63) >> 6;
  CodeSlots<HD> kc, vc;
  const int s0 = w.begin + 16 * wave;
  tab.load(a, w.b, w.begin >> a.pb.page_shift, lane);
  auto fetch = [&](int t) {
    const int slot = s0 + 64 * t;
    const int page = tab.at(a, w.b, slot >> a.pb.page_shift, lane);
    char* st = smem + (t & 1) * kStage + 16 * wave * S::kRowBytes;
    if constexpr (E8) {
      kc.load(a.pool.k, a.pool.ke, a, page, kvh, slot, w.end, lane);
      vc.load(a.pool.v, a.pool.ve, a, page, kvh, slot, w.end, lane);
    } else {
      DmaSlots<HD>::load(a.pool.k, a, page, kvh, slot, w.end, st, lane);
      DmaSlots<HD>::load(a.pool.v, a, page, kvh, slot, w.end, st + kTile, lane);
    }
  };
  auto settle = [&](int t) {  // e4m3: the fetched codes into their stage
    if constexpr (E8) {
      char* st = smem + (t & 1) * kStage + 16 * wave * S::kRowBytes;
      kc.store(st, lane);
      vc.store(st + kTile, lane);
    }
  };

  // V^T reads: lane (group of 16 G, a4 = lane & 3, j = lane / 4 & 3) addresses slot 4 hi + j at dims 16 (G & 1) + 4 a4
  const int tj = (lane >> 2) & 3, vrow = 4 * hi + tj;
  const int vch = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), vbyte = (lane & 1) * 8;

  auto tile = [&](int t) {
    const int kb0 = w.begin + 64 * t;
    const char* Ks = smem + (t & 1) * kStage;
    const char* Vs = Ks + kTile;
    if (kb0 >= any_hi) return;  // in the future of every row of this wave
    f32x16 s[NQ][2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const int row = 32 * kb + r32;
#pragma unroll
      for (int qi = 0; qi < NQ; ++qi)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[qi][kb][i] = 0.f;
#pragma unroll
      for (int st = 0; st < NS; ++st) {
        const bf16x8 kf = *reinterpret_cast<const bf16x8*>(Ks + row * S::kRowBytes + (((2 * st + hi) ^ S::swz(row)) << 4));
#pragma unroll
        for (int qi = 0; qi < NQ; ++qi)
          s[qi][kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[qi][st], s[qi][kb], 0, 0, 0);
      }
    }
    const bool masked = kb0 + 64 > min(see_hi, w.end) || kb0 < see_lo;  // wave-uniform
    bf16x8 pb[NQ][4];
#pragma unroll
    for (int qi = 0; qi < NQ; ++qi) {
      if (masked) {
        // slot kb0 + x is seen iff lo <= x <= top
        const int top = min(slot_of[qi], w.end - 1) - kb0 - 4 * hi;
        const int lo = a.window ? slot_of[qi] - a.window + 1 - kb0 - 4 * hi : -64;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int x = 32 * kb + 8 * (i / 4) + i % 4;
            s[qi][kb][i] = x > top || x < lo ? -INFINITY : s[qi][kb][i];
          }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[qi][kb][i]);
      const float m_new = fmaxf(m_run[qi], pair32_max(mx) * sc);
      const float base = m_new == -INFINITY ? 0.f : m_new;
      if (__builtin_amdgcn_ballot_w64(m_new != m_run[qi])) {
        const float alpha = __builtin_amdgcn_exp2f(m_run[qi] - base);
        l_run[qi] *= alpha;
#pragma unroll
        for (int db = 0; db < ND; ++db) o[qi][db] *= alpha;
      }
      m_run[qi] = m_new;
#pragma unroll
      for (int st = 0; st < 4; ++st)
#pragma unroll
        for (int j = 0; j < 8; ++j)
          pb[qi][st][j] = (__bf16)__builtin_amdgcn_exp2f(fmaf(s[qi][st / 2][8 * (st & 1) + j], sc, -base));
      float sum = l_run[qi];
#pragma unroll
      for (int st = 0; st < 4; ++st)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
          const bf16x2 one = {(__bf16)1.0f, (__bf16)1.0f}, p2 = {pb[qi][st][2 * j], pb[qi][st][2 * j + 1]};
          sum = __builtin_amdgcn_fdot2_f32_bf16(p2, one, sum, false);
        }
      l_run[qi] = sum;
    }
    const uint32_t vs = uint32_t(size_t((__attribute__((address_space(3))) const char*)Vs)) + vrow * S::kRowBytes + vbyte;
#pragma unroll
    for (int db = 0; db < ND; ++db) {
      u32x2 v[8];
      lds_read_tr8<S::kRowBytes>(vs + (((4 * db + vch) ^ S::swz(vrow)) << 4),
                                 vs + 8 * S::kRowBytes + (((4 * db + vch) ^ S::swz(vrow + 8)) << 4), v);
      bf16x8 vf[4];
#pragma unroll
      for (int st = 0; st < 4; ++st) {
        const u32x4 raw = {v[2 * st][0], v[2 * st][1], v[2 * st + 1][0], v[2 * st + 1][1]};
        vf[st] = __builtin_bit_cast(bf16x8, raw);
      }
      if (masked) {
        uint32_t bad = 0;
#pragma unroll
        for (int st = 0; st < 4; ++st) bad |= not_finite_bits(vf[st]);
        if (__builtin_amdgcn_ballot_w64(bad != 0)) {
#pragma unroll
          for (int qi = 0; qi < NQ; ++qi) {
            const int top = min(slot_of[qi], w.end - 1) - kb0 - 4 * hi;
            const int lo = a.window ? slot_of[qi] - a.window + 1 - kb0 - 4 * hi : -64;
            f32x16 c;
#pragma unroll
            for (int i = 0; i < 16; ++i) c[i] = 0.f;
#pragma unroll
            for (int st = 0; st < 4; ++st) {
              bf16x8 one;
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                const int x = 16 * st + j % 4 + 8 * (j / 4);
                one[j] = (__bf16)(x > top || x < lo ? 0.f : 1.f);
              }
              c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(not_finite_codes(vf[st]), one, c, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) o[qi][db][i] += not_finite_sum(c[i]);
          }
#pragma unroll
          for (int st = 0; st < 4; ++st) vf[st] = finite_or_zero(vf[st]);
        }
      }
#pragma unroll
      for (int st = 0; st < 4; ++st)
#pragma unroll
        for (int qi = 0; qi < NQ; ++qi)
          o[qi][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[st], pb[qi][st], o[qi][db], 0, 0, 0);
    }
  };

  if (ntiles > 0) fetch(0);
  if constexpr (E8) {
    if (ntiles > 0) settle(0);
  }
  for (int t = 0; t < ntiles; ++t) {
    // tile t is in LDS for every wave, and every wave is done with tile t - 1, whose stage is filled next
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __syncthreads();
    if (t + 1 < ntiles) fetch(t + 1);
    tile(t);
    if (t + 1 < ntiles) settle(t + 1);
  }

  // lane holds O^T[dim 32 db + 8 (i / 4) + 4 hi + i % 4][row r32]
#pragma unroll
  for (int qi = 0; qi < NQ; ++qi) {
    const float l = pair32_sum(l_run[qi]);
    if (!live[qi]) continue;
    const int m = m0 + 32 * qi + r32;
    if (w.splits > 1) {
      const int64_t slot = int64_t(blockIdx.x) * BM + (m - w.tile * BM);
      float* po = a.part_o + slot * HD;
#pragma unroll
      for (int db = 0; db < ND; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<f32x4*>(po + 32 * db + 8 * i + 4 * hi) =
              f32x4{o[qi][db][4 * i], o[qi][db][4 * i + 1], o[qi][db][4 * i + 2], o[qi][db][4 * i + 3]};
      if (hi == 0) a.part_ml[slot] = make_float2(m_run[qi], l);
    } else {
      const float inv = l == 0.f ? 0.f : 1.0f / l;  // a row that sees nothing: zeros
      const int tok = m / a.G, g = m - tok * a.G;
      uint16_t* op = static_cast<uint16_t*>(a.out) + int64_t(w.row0 + tok) * a.o_row + int64_t(kvh * a.G + g) * a.o_head;
#pragma unroll
      for (int db = 0; db < ND; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          u32x2 pk;
          pk[0] = uint32_t(f2bf(o[qi][db][4 * i] * inv)) | uint32_t(f2bf(o[qi][db][4 * i + 1] * inv)) << 16;
          pk[1] = uint32_t(f2bf(o[qi][db][4 * i + 2] * inv)) | uint32_t(f2bf(o[qi][db][4 * i + 3] * inv)) << 16;
          *reinterpret_cast<u32x2*>(op + 32 * db + 8 * i + 4 * hi) = pk;
        }
    }
  }
}

// ------------------------------------------------------------ a few tokens

// R transpose loads and their wait: for the steps of 32 slots of a tile (two
// 16-slot halves each) the V^T operand of v_mfma_f32_16x16x32_bf16 for 16 dims.
template <int ROW>
__device__ __forceinline__ void lds_read_tr2(uint32_t addr, u32x2 (&v)[2]) {
  asm volatile(
      "ds_read_b64_tr_b16 %0, %2\n\t"
      "ds_read_b64_tr_b16 %1, %2 offset:%3\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(v[0]), "=&v"(v[1])
      : "v"(addr), "n"(16 * ROW)
      : "memory");
}

// A workgroup of four waves takes 16 NR rows; each wave runs through every
// fourth piece of TK slots by itself, from its own LDS, with a softmax of its
// own, and the four are joined in wave order at the end: nothing waits for
// another wave while slots stream in (memory bound: the rows of one token of
// a few heads are far too few for the matrix cores to matter).
//
// S^T = K Q^T with v_mfma_f32_16x16x32_bf16: lane (r16, grp) holds of row r16
// the scores of slots 16 kb + 4 grp + i, which is the B operand of
// O^T += V^T P^T when step ks takes slots 32 ks + 16 (j / 4) + 4 grp + j % 4.
// A probability goes into that product as two bf16 numbers (its rounding and
// what that leaves), so it counts with 16 bits: the second product costs
// nothing here.
template <int HD, bool E8, int NR>
__global__ __launch_bounds__(256) void paged_token_kernel(PagedKernelArgs a) {
  using S = SlotTile<HD>;
  constexpr int BM = 16 * NR, TK = 4096 / HD, NS = HD / 32, ND = HD / 16, KB = TK / 16;
  constexpr int kTile = TK * S::kRowBytes, kStages = E8 ? 1 : 2, kRing = 2 * kTile * kStages;
  constexpr int kDma = 2 * kTile / 1024;  // DMA instructions per piece
  constexpr int OS = HD + 4;              // floats per row of the join, so that 16 rows spread over the banks
  static_assert(4 * kRing >= 4 * 16 * OS * 4, "the join reuses the ring");
  __shared__ __attribute__((aligned(16))) char smem[4 * kRing];
  __shared__ float ms[4][BM], ls[4][BM];
  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int item = int(blockIdx.x) / a.pool.Hkv, kvh = int(blockIdx.x) - item * a.pool.Hkv;
  const PagedItem it = paged_item(a, item, lane);
  if (it.b < 0) return;
  const PagedWork w = paged_work(a, it);
  if (w.splits > 1 && w.begin >= w.end) return;

  int slot_of[NR];
  bf16x8 qf[NR][NS];
  const int m0 = w.tile * BM;
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    const int mc = min(m0 + 16 * r + r16, w.M - 1);
    const int tok = mc / a.G, g = mc - tok * a.G;
    slot_of[r] = w.p0 + tok;
    const uint16_t* qp = static_cast<const uint16_t*>(a.q) + int64_t(w.row0 + tok) * a.q_row + int64_t(kvh * a.G + g) * a.q_head;
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[r][s] = *reinterpret_cast<const bf16x8*>(qp + 32 * s + 8 * grp);
  }
  const int see_hi = w.p0 + m0 / a.G + 1, last = w.p0 + min(m0 + BM - 1, w.M - 1) / a.G;
  const int see_lo = a.window ? last - a.window + 1 : 0;
  f32x4 o[NR][ND];
  float m_run[NR], l_run[NR];
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    m_run[r] = -INFINITY;
    l_run[r] = 0.f;
#pragma unroll
    for (int db = 0; db < ND; ++db) o[r][db] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float sc = 1.4426950408889634f / sqrtf(float(HD));

  char* ring = smem + wave * kRing;
  const int s0 = w.begin + TK * wave;
  const int nt = w.end > s0 ? (w.end - s0 + 4 * TK - 1) / (4 * TK) : 0;
  PagedTable tab;
  tab.load(a, w.b, w.begin >> a.pb.page_shift, lane);
  CodeSlots<HD> kc[KB], vc[KB];
  auto fetch = [&](int t) {
    const int slot = s0 + 4 * TK * t;
    char* st = ring + (t & (kStages - 1)) * 2 * kTile;
#pragma unroll
    for (int i = 0; i < KB; ++i) {
      const int page = tab.at(a, w.b, (slot + 16 * i) >> a.pb.page_shift, lane);
      if constexpr (E8) {
        kc[i].load(a.pool.k, a.pool.ke, a, page, kvh, slot + 16 * i, w.end, lane);
        vc[i].load(a.pool.v, a.pool.ve, a, page, kvh, slot + 16 * i, w.end, lane);
      } else {
        DmaSlots<HD>::load(a.pool.k, a, page, kvh, slot + 16 * i, w.end, st + 16 * i * S::kRowBytes, lane);
        DmaSlots<HD>::load(a.pool.v, a, page, kvh, slot + 16 * i, w.end, st + kTile + 16 * i * S::kRowBytes, lane);
      }
    }
  };
  const int tj = (lane >> 2) & 3, vrow = 4 * grp + tj, vch = (lane & 3) >> 1, vbyte = (lane & 1) * 8;
  auto piece = [&](int t) {
    const int kb0 = s0 + 4 * TK * t;
    const char* Ks = ring + (t & (kStages - 1)) * 2 * kTile;
    f32x4 s[NR][KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const int row = 16 * kb + r16;
#pragma unroll
      for (int r = 0; r < NR; ++r) s[r][kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < NS; ++st) {
        const bf16x8 kf = *reinterpret_cast<const bf16x8*>(Ks + row * S::kRowBytes + (((4 * st + grp) ^ S::swz(row)) << 4));
#pragma unroll
        for (int r = 0; r < NR; ++r) s[r][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[r][st], s[r][kb], 0, 0, 0);
      }
    }
    const bool masked = kb0 + TK > min(see_hi, w.end) || kb0 < see_lo;
    bf16x8 ph[NR][KB / 2], pl[NR][KB / 2];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      if (masked) {
        const int top = min(slot_of[r], w.end - 1) - kb0 - 4 * grp;
        const int lo = a.window ? slot_of[r] - a.window + 1 - kb0 - 4 * grp : -TK;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[r][kb][i] = 16 * kb + i > top || 16 * kb + i < lo ? -INFINITY : s[r][kb][i];
      }
      float mx = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[r][kb][i]);
      const float m_new = fmaxf(m_run[r], rows4_max(mx) * sc);
      const float base = m_new == -INFINITY ? 0.f : m_new;
      if (__builtin_amdgcn_ballot_w64(m_new != m_run[r])) {
        const float alpha = __builtin_amdgcn_exp2f(m_run[r] - base);
        l_run[r] *= alpha;
#pragma unroll
        for (int db = 0; db < ND; ++db) o[r][db] *= alpha;
      }
      m_run[r] = m_new;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p = __builtin_amdgcn_exp2f(fmaf(s[r][kb][i], sc, -base));
          l_run[r] += p;
          const __bf16 h = (__bf16)p;
          ph[r][kb / 2][4 * (kb & 1) + i] = h;
          pl[r][kb / 2][4 * (kb & 1) + i] = (__bf16)(p - float(h));
        }
    }
    const uint32_t vs = uint32_t(size_t((__attribute__((address_space(3))) const char*)(Ks + kTile))) + vrow * S::kRowBytes + vbyte;
#pragma unroll
    for (int db = 0; db < ND; ++db) {
      const uint32_t vc0 = vs + (((2 * db + vch) ^ S::swz(vrow)) << 4);
#pragma unroll
      for (int ks = 0; ks < KB / 2; ++ks) {
        u32x2 v[2];
        lds_read_tr2<S::kRowBytes>(vc0 + 32 * ks * S::kRowBytes, v);
        const u32x4 raw = {v[0][0], v[0][1], v[1][0], v[1][1]};
        bf16x8 vf = __builtin_bit_cast(bf16x8, raw);
        if (masked) {
          if (__builtin_amdgcn_ballot_w64(not_finite_bits(vf) != 0)) {
#pragma unroll
            for (int r = 0; r < NR; ++r) {
              const int top = min(slot_of[r], w.end - 1) - kb0 - 4 * grp - 32 * ks;
              const int lo = a.window ? slot_of[r] - a.window + 1 - kb0 - 4 * grp - 32 * ks : -TK;
              bf16x8 one;
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                const int x = 16 * (j / 4) + j % 4;
                one[j] = (__bf16)(x > top || x < lo ? 0.f : 1.f);
              }
              const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
              const f32x4 c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(not_finite_codes(vf), one, zero, 0, 0, 0);
#pragma unroll
              for (int i = 0; i < 4; ++i) o[r][db][i] += not_finite_sum(c[i]);
            }
            vf = finite_or_zero(vf);
          }
        }
#pragma unroll
        for (int r = 0; r < NR; ++r) {
          o[r][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, ph[r][ks], o[r][db], 0, 0, 0);
          o[r][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pl[r][ks], o[r][db], 0, 0, 0);
        }
      }
    }
  };
  if (nt > 0) fetch(0);
  for (int t = 0; t < nt; ++t) {
    if constexpr (E8) {
      // the codes of this piece into LDS (the wave is done with the last one's), then the next ones' loads
      char* st = ring;
#pragma unroll
      for (int i = 0; i < KB; ++i) {
        kc[i].store(st + 16 * i * S::kRowBytes, lane);
        vc[i].store(st + kTile + 16 * i * S::kRowBytes, lane);
      }
      if (t + 1 < nt) fetch(t + 1);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    } else {
      if (t + 1 < nt) {
        fetch(t + 1);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kDma) : "memory");  // all but the next piece's
      } else {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      }
    }
    __builtin_amdgcn_wave_barrier();
    piece(t);
    __builtin_amdgcn_wave_barrier();
  }

  // the four waves' shares, in wave order; 16 rows at a time through the ring
  float* os = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    const float l = rows4_sum(l_run[r]);
    if (grp == 0) {
      ms[wave][16 * r + r16] = m_run[r];
      ls[wave][16 * r + r16] = l;
    }
    __syncthreads();  // every wave is done with the ring, and with the last 16 rows
#pragma unroll
    for (int db = 0; db < ND; ++db) *reinterpret_cast<f32x4*>(os + (wave * 16 + r16) * OS + 16 * db + 4 * grp) = o[r][db];
    __syncthreads();
    for (int e = tid; e < 16 * HD / 4; e += 256) {
      const int q = e / (HD / 4), d = e % (HD / 4) * 4, m = m0 + 16 * r + q;
      if (m >= w.M) break;
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) M = fmaxf(M, ms[i][16 * r + q]);
      f32x4 O = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float mi = ms[i][16 * r + q], f = mi == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mi - M);
        // a wave whose slots are all hidden (maximum -inf) has a sum of 0, or of NaN where a score is NaN
        L += mi == -INFINITY ? ls[i][16 * r + q] : ls[i][16 * r + q] * f;
        const f32x4 oi = *reinterpret_cast<const f32x4*>(os + (i * 16 + q) * OS + d);
        O += mi == -INFINITY ? oi : oi * f;
      }
      if (w.splits > 1) {
        const int64_t slot = int64_t(blockIdx.x) * BM + 16 * r + q;
        *reinterpret_cast<f32x4*>(a.part_o + slot * HD + d) = O;
        if (d == 0) a.part_ml[slot] = make_float2(M, L);
      } else {
        const float inv = L == 0.f ? 0.f : 1.0f / L;
        const int tok = m / a.G, g = m - tok * a.G;
        u32x2 pk;
        pk[0] = uint32_t(f2bf(O[0] * inv)) | uint32_t(f2bf(O[1] * inv)) << 16;
        pk[1] = uint32_t(f2bf(O[2] * inv)) | uint32_t(f2bf(O[3] * inv)) << 16;
        *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + int64_t(w.row0 + tok) * a.o_row +
                                  int64_t(kvh * a.G + g) * a.o_head + d) = pk;
      }
    }
  }
}

// -------------------------------------------------------------------- fp32

// fp32 on the fp32 matrix cores: a workgroup takes 16 rows, its four waves
// every fourth piece of 32 slots, each with a softmax of its own, joined
// through LDS in wave order. Rows and slots are the two operands' rows, 16
// bytes of a row per lane, element e of the vectors forming one 4-deep
// product; the probabilities go through a per-wave LDS tile into the A
// operand of P V, whose B operand is HD / 16 neighbouring dims of slot
// 4 s + grp as they come from memory.
template <int HD, bool E8>
__global__ __launch_bounds__(256) void paged_f32_kernel(PagedKernelArgs a) {
  constexpr int NK = HD / 16, DPL = HD / 16, KV = 32;
  __shared__ float ps[4][16][KV + 4];
  __shared__ float osum[4][16][HD];
  __shared__ float ms[4][16], ls[4][16];
  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, grp = lane >> 4;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int item = int(blockIdx.x) / a.pool.Hkv, kvh = int(blockIdx.x) - item * a.pool.Hkv;
  const PagedItem it = paged_item(a, item, lane);
  if (it.b < 0) return;
  const PagedWork w = paged_work(a, it);
  if (w.splits > 1 && w.begin >= w.end) return;
  const int m0 = w.tile * 16;
  f32x4 qf[NK];
  {
    const int mc = min(m0 + r16, w.M - 1), tok = mc / a.G, g = mc - tok * a.G;
    const float* qp = static_cast<const float*>(a.q) + int64_t(w.row0 + tok) * a.q_row + int64_t(kvh * a.G + g) * a.q_head;
#pragma unroll
    for (int s = 0; s < NK; ++s) qf[s] = *reinterpret_cast<const f32x4*>(qp + 16 * s + 4 * grp);
  }
  int slot_of[4];  // of rows m0 + 4 grp + i
#pragma unroll
  for (int i = 0; i < 4; ++i) slot_of[i] = w.p0 + min(m0 + 4 * grp + i, w.M - 1) / a.G;
  const int see_hi = w.p0 + m0 / a.G + 1;
  const int see_lo = a.window ? w.p0 + min(m0 + 15, w.M - 1) / a.G - a.window + 1 : 0;
  const float scale = 1.0f / sqrtf(float(HD));
  float m[4], l[4];
  f32x4 o[DPL];  // o[e][i]: row m0 + 4 grp + i, dim DPL r16 + e
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
  }
#pragma unroll
  for (int e = 0; e < DPL; ++e) o[e] = f32x4{0.f, 0.f, 0.f, 0.f};
  PagedTable tab;
  tab.load(a, w.b, w.begin >> a.pb.page_shift, lane);
  const int mask = (1 << a.pb.page_shift) - 1;
  for (int key0 = w.begin + KV * wv; key0 < w.end; key0 += 4 * KV) {
    f32x4 kf[2][NK];
    float vf[KV / 4][DPL];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      // slots past the end are read where the page has them, and not used
      const int page = tab.at(a, w.b, (key0 + 16 * kb) >> a.pb.page_shift, lane);
      const int64_t row = ((int64_t(page) * a.pool.Hkv + kvh) << a.pb.page_shift) + ((key0 + 16 * kb) & mask);
      if constexpr (E8) {
        const float s = paged_scale(a.pool.ke[row + r16]);
        const uint8_t* kp = static_cast<const uint8_t*>(a.pool.k) + (row + r16) * HD + 4 * grp;
#pragma unroll
        for (int st = 0; st < NK; ++st) kf[kb][st] = paged_widen4_f32(*reinterpret_cast<const uint32_t*>(kp + 16 * st), s);
      } else {
        const float* kp = static_cast<const float*>(a.pool.k) + (row + r16) * HD + 4 * grp;
#pragma unroll
        for (int st = 0; st < NK; ++st) kf[kb][st] = *reinterpret_cast<const f32x4*>(kp + 16 * st);
      }
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int64_t vr = row + 4 * s + grp;
        float* v = vf[4 * kb + s];
        if constexpr (E8) {
          const float sv = paged_scale(a.pool.ve[vr]);
          const uint8_t* vp = static_cast<const uint8_t*>(a.pool.v) + vr * HD + DPL * r16;
          if constexpr (DPL == 2) {
            const f32x4 t = paged_widen4_f32(*reinterpret_cast<const uint16_t*>(vp), sv);
            v[0] = t[0];
            v[1] = t[1];
          } else {
#pragma unroll
            for (int j = 0; j < DPL / 4; ++j) {
              const f32x4 t = paged_widen4_f32(reinterpret_cast<const uint32_t*>(vp)[j], sv);
#pragma unroll
              for (int i = 0; i < 4; ++i) v[4 * j + i] = t[i];
            }
          }
        } else {
          const float* vp = static_cast<const float*>(a.pool.v) + vr * HD + DPL * r16;
          if constexpr (DPL == 2) {
            const float2 t = *reinterpret_cast<const float2*>(vp);
            v[0] = t.x;
            v[1] = t.y;
          } else {
#pragma unroll
            for (int j = 0; j < DPL / 4; ++j) {
              const f32x4 t = reinterpret_cast<const f32x4*>(vp)[j];
#pragma unroll
              for (int i = 0; i < 4; ++i) v[4 * j + i] = t[i];
            }
          }
        }
        // whatever lies behind the sequence's last slot is none of its values
        if (key0 + 16 * kb + 4 * s + grp >= w.end) {
#pragma unroll
          for (int e = 0; e < DPL; ++e) v[e] = 0.f;
        }
      }
    }
    float sc[2][4];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      f32x4 acc[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < NK; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(qf[s][e], kf[kb][s][e], acc[e], 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = key0 + 16 * kb + r16;
        const bool in = key <= slot_of[i] && key < w.end && (!a.window || key > slot_of[i] - a.window);
        sc[kb][i] = in ? ((acc[0][i] + acc[1][i]) + (acc[2][i] + acc[3][i])) * scale : -INFINITY;
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float mx = fmaxf(sc[0][i], sc[1][i]);
      mx = fmaxf(mx, DSF_DPP(mx, 0xB1));  // over the 16 lanes of the row: quads, half rows, rows
      mx = fmaxf(mx, DSF_DPP(mx, 0x4E));
      mx = fmaxf(mx, DSF_DPP(mx, 0x141));
      mx = fmaxf(mx, DSF_DPP(mx, 0x140));
      const float mn = fmaxf(m[i], mx);
      const float c = mn == -INFINITY ? 1.f : expf(m[i] - mn);
      float sum = 0.f;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const float p = sc[kb][i] == -INFINITY ? 0.f : expf(sc[kb][i] - mn);
        sum += p;
        ps[wv][4 * grp + i][16 * kb + r16] = p;
      }
      l[i] = l[i] * c + row16_sum(sum);
#pragma unroll
      for (int e = 0; e < DPL; ++e) o[e][i] *= c;
      m[i] = mn;
    }
    // a wave reads back only its own probabilities
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
    __builtin_amdgcn_wave_barrier();
    // where slots are hidden from some rows, infinite and NaN values are left
    // out of the product (0 times them is NaN) and added to the rows that see them
    bool bad = false;
    if (key0 + KV > min(see_hi, w.end) || key0 < see_lo) {
#pragma unroll
      for (int s = 0; s < KV / 4; ++s)
#pragma unroll
        for (int e = 0; e < DPL; ++e) bad = bad || !(fabsf(vf[s][e]) < INFINITY);
    }
    const bool fix = __ballot(bad) != 0;
#pragma unroll
    for (int s = 0; s < KV / 4; ++s) {
      const float pa = ps[wv][r16][4 * s + grp];
#pragma unroll
      for (int e = 0; e < DPL; ++e)
        o[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(pa, fix && !(fabsf(vf[s][e]) < INFINITY) ? 0.f : vf[s][e], o[e], 0,
                                                    0, 0);
    }
    if (fix) {
#pragma unroll
      for (int s = 0; s < KV / 4; ++s)
        for (int g = 0; g < 4; ++g) {
          const int key = key0 + 4 * s + g;
#pragma unroll
          for (int e = 0; e < DPL; ++e) {
            const float v = __shfl(vf[s][e], r16 + 16 * g, 64);
            if (!(fabsf(v) < INFINITY))
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (key <= slot_of[i] && (!a.window || key > slot_of[i] - a.window)) o[e][i] += v;
          }
        }
    }
    __builtin_amdgcn_s_waitcnt(0xc07f);  // read before the next piece's overwrite them
    __builtin_amdgcn_wave_barrier();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int e = 0; e < DPL; ++e) osum[wv][4 * grp + i][DPL * r16 + e] = o[e][i];
    if (r16 == 0) {
      ms[wv][4 * grp + i] = m[i];
      ls[wv][4 * grp + i] = l[i];
    }
  }
  __syncthreads();
  for (int e = tid; e < 16 * HD; e += 256) {
    const int q = e / HD, d = e - q * HD, mr = m0 + q;
    if (mr >= w.M) break;
    const float M = fmaxf(fmaxf(ms[0][q], ms[1][q]), fmaxf(ms[2][q], ms[3][q]));
    float O = 0.f, L = 0.f;
#pragma unroll
    for (int ww = 0; ww < 4; ++ww) {
      // a wave that saw nothing has zeros (NaN where a score was)
      const float c = ms[ww][q] == -INFINITY ? 1.f : expf(ms[ww][q] - M);
      O = fmaf(osum[ww][q][d], c, O);
      L = fmaf(ls[ww][q], c, L);
    }
    if (w.splits > 1) {
      const int64_t slot = int64_t(blockIdx.x) * 16 + q;
      a.part_o[slot * HD + d] = O;
      if (d == 0) a.part_ml[slot] = make_float2(M, L);
    } else {
      const int tok = mr / a.G, g = mr - tok * a.G;
      static_cast<float*>(a.out)[int64_t(w.row0 + tok) * a.o_row + int64_t(kvh * a.G + g) * a.o_head + d] =
          L == 0.f ? 0.f : O / L;
    }
  }
}

// ---------------------------------------------------- joining the splits

// One workgroup per (row, kv head): every split's share of the row, in the
// splits' order. Rows of sequences that were not split are done already.
// LOG2: the maxima are in log2 units.
template <int HD, typename T>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedKernelArgs a) {
  constexpr bool LOG2 = sizeof(T) == 2;
  const int r = blockIdx.x, kvh = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  PagedShape w = {};
  if (lane < a.pb.B) w = paged_shape(a, lane);
  const int per = paged_split_blocks(a, w, lane);
  int first = 0;
  for (int b0 = 0; b0 < a.pb.B; b0 += 64) {
    if (b0) {
      w = PagedShape{};
      if (b0 + lane < a.pb.B) w = paged_shape(a, b0 + lane);
    }
    const int splits = paged_splits(w, per), c = min(w.tiles * splits, a.items);
    const int end = wave_prefix(c);
    const uint64_t here = __builtin_amdgcn_ballot_w64(w.tiles > 0 && r >= w.row0 && r < w.row0 + min(w.n, a.pb.max_rows));
    if (here) {
      const int ln = __builtin_ctzll(here), ns = __builtin_amdgcn_readlane(splits, ln);
      if (ns == 1) return;
      first += __builtin_amdgcn_readlane(end, ln) - __builtin_amdgcn_readlane(c, ln);
      const PagedShape s = paged_shape(a, b0 + ln);
      const int tok = r - s.row0;
      for (int e = tid; e < a.G * (HD / 4); e += 256) {
        const int g = e / (HD / 4), d = e % (HD / 4) * 4, m = tok * a.G + g;
        const int tile = m >> a.bm_shift, row = m & ((1 << a.bm_shift) - 1);
        float M = -INFINITY, L = 0.f;
        f32x4 O = {0.f, 0.f, 0.f, 0.f};
        for (int i = 0; i < ns; ++i) {
          int begin, stop;
          paged_range(a, s, tile, i, per << 6, &begin, &stop);
          if (begin >= stop) continue;
          const int64_t item = min(first + i * s.tiles + max(s.tiles - 1 - tile, 0), a.items - 1);
          const int64_t slot = ((item * a.pool.Hkv + kvh) << a.bm_shift) + row;
          const float2 ml = a.part_ml[slot];
          const f32x4 oi = *reinterpret_cast<const f32x4*>(a.part_o + slot * HD + d);
          const float mn = fmaxf(M, ml.x);
          // nothing seen so far, or nothing in this split: zeros (NaN where a score was)
          const float f0 = M == -INFINITY ? 1.f : LOG2 ? __builtin_amdgcn_exp2f(M - mn) : expf(M - mn);
          const float f1 = ml.x == -INFINITY ? 1.f : LOG2 ? __builtin_amdgcn_exp2f(ml.x - mn) : expf(ml.x - mn);
          O = O * f0 + oi * f1;
          L = L * f0 + ml.y * f1;
          M = mn;
        }
        const float inv = L == 0.f ? 0.f : 1.0f / L;
        T* op = static_cast<T*>(a.out) + int64_t(r) * a.o_row + int64_t(kvh * a.G + g) * a.o_head + d;
        if constexpr (sizeof(T) == 2) {
          u32x2 pk;
          pk[0] = uint32_t(f2bf(O[0] * inv)) | uint32_t(f2bf(O[1] * inv)) << 16;
          pk[1] = uint32_t(f2bf(O[2] * inv)) | uint32_t(f2bf(O[3] * inv)) << 16;
          *reinterpret_cast<u32x2*>(op) = pk;
        } else {
          *reinterpret_cast<f32x4*>(op) = O * inv;
        }
      }
      return;
    }
    first = min(first + __builtin_amdgcn_readlane(end, 63), a.items);
  }
}

// ------------------------------------------------------------------ launch

namespace {

// One launch over the sequences of m_lo < rows * G <= m_hi.
struct PagedPlan {
  bool on;
  int bm_shift, m_lo, m_hi;
  int items;   // per kv head, at most
  int target;  // per kv head (0: no splits)
  size_t bytes;
};

constexpr int kTokenRows = 64;        // rows of a sequence (tokens times heads) the token kernel takes
constexpr int kTokenItems = 1024;     // items aimed at, of all kv heads
constexpr int kChunkItems = 512;
constexpr int kF32Items = 1024;
constexpr int kSplitMinBlocks = 8;    // 512 slots

size_t align256(size_t n) { return (n + 255) & ~size_t(255); }

PagedPlan make_plan(const PagedBatch& pb, int G, int Hkv, int hd, int bm_shift, int m_lo, int m_hi, int total) {
  PagedPlan p = {true, bm_shift, m_lo, m_hi, 0, 0, 0};
  // tiles: full ones, and a part of one per sequence that takes part
  const int64_t rows = int64_t(pb.n_rows) * G;
  const int64_t seqs = std::min<int64_t>(std::min(pb.B, pb.n_rows), rows / (m_lo + 1));
  const int64_t tiles = (rows >> bm_shift) + seqs;
  const int64_t blocks = (int64_t(pb.max_pages) << pb.page_shift) / 64;
  if (blocks > kSplitMinBlocks && tiles <= 4096 && tiles * Hkv < 2 * total) p.target = std::max(total / Hkv, 1);
  p.items = int(tiles + p.target);
  if (p.target)
    p.bytes = align256((size_t(p.items) * Hkv << bm_shift) * hd * 4) + align256((size_t(p.items) * Hkv << bm_shift) * 8);
  return p;
}

// The launches of a call: [0] sequences of few rows, [1] the others.
void paged_plans(int dtype, int Hq, const PagedPool& pool, const PagedBatch& pb, PagedPlan (&p)[2]) {
  const int G = Hq / pool.Hkv;
  p[0] = p[1] = PagedPlan{};
  if (dtype == DSF_F32) {
    p[0] = make_plan(pb, G, pool.Hkv, pool.hd, 4, 0, 0x7fffffff, kF32Items);
    return;
  }
  const int64_t most = int64_t(std::min(pb.max_rows, pb.n_rows)) * G;
  // sequences of one token stay with the token kernel beside ones with chunks
  const int few = most <= kTokenRows ? int(most) : std::min((G + 15) / 16 * 16, kTokenRows);
  if (most <= kTokenRows || pb.B > 1)
    p[0] = make_plan(pb, G, pool.Hkv, pool.hd, few <= 16 ? 4 : few <= 32 ? 5 : 6, 0, few, kTokenItems);
  if (most > kTokenRows) p[1] = make_plan(pb, G, pool.Hkv, pool.hd, 7, pb.B > 1 ? few : 0, 0x7fffffff, kChunkItems);
}

}  // namespace

size_t paged_attention_workspace_bytes(int dtype, int Hq, const PagedPool& pool, const PagedBatch& pb) {
  PagedPlan p[2];
  paged_plans(dtype, Hq, pool, pb, p);
  return std::max<size_t>(p[0].bytes + p[1].bytes, 256);
}

hipError_t launch_paged_attention(const PagedAttnArgs& a, hipStream_t s) {
  if (a.pb.B == 0 || a.pb.n_rows == 0 || a.pb.max_rows == 0) return hipSuccess;
  TimedScope ts(DSF_KIND_ATTN, s);
  PagedPlan p[2];
  paged_plans(a.dtype, a.Hq, a.pool, a.pb, p);
  char* ws = static_cast<char*>(a.workspace);
  const bool e8 = a.pool.codes;
  for (int i = 0; i < 2; ++i) {
    if (!p[i].on) continue;
    PagedKernelArgs k;
    k.pool = a.pool;
    k.pb = a.pb;
    k.q = a.q;
    k.q_row = a.q_row;
    k.q_head = a.q_head;
    k.out = a.out;
    k.o_row = a.o_row;
    k.o_head = a.o_head;
    k.G = a.Hq / a.pool.Hkv;
    k.window = a.window;
    k.bm_shift = p[i].bm_shift;
    k.m_lo = p[i].m_lo;
    k.m_hi = p[i].m_hi;
    k.items = p[i].items;
    k.target = p[i].target;
    k.split_min = kSplitMinBlocks;
    const size_t rows = size_t(p[i].items) * a.pool.Hkv << p[i].bm_shift;
    k.part_o = reinterpret_cast<float*>(ws);
    k.part_ml = reinterpret_cast<float2*>(ws + align256(rows * a.pool.hd * 4));
    ws += p[i].bytes;
    const unsigned grid = unsigned(p[i].items) * a.pool.Hkv;
    auto run = [&](auto hdc, auto e8c) -> hipError_t {
      constexpr int HD = decltype(hdc)::value;
      constexpr bool E8 = decltype(e8c)::value;
      if (a.dtype == DSF_F32) paged_f32_kernel<HD, E8><<<grid, 256, 0, s>>>(k);
      else if (i == 1) paged_chunk_kernel<HD, E8, 1><<<grid, 256, 0, s>>>(k);
      else if (k.bm_shift == 4) paged_token_kernel<HD, E8, 1><<<grid, 256, 0, s>>>(k);
      else if (k.bm_shift == 5) paged_token_kernel<HD, E8, 2><<<grid, 256, 0, s>>>(k);
      else paged_token_kernel<HD, E8, 4><<<grid, 256, 0, s>>>(k);
      hipError_t e = hipGetLastError();
      if (e != hipSuccess || !k.target) return e;
      const dim3 jg(a.pb.n_rows, a.pool.Hkv);
      if (a.dtype == DSF_F32) paged_join_kernel<HD, float><<<jg, 256, 0, s>>>(k);
      else paged_join_kernel<HD, uint16_t><<<jg, 256, 0, s>>>(k);
      return hipGetLastError();
    };
    auto run_h = [&](auto e8c) -> hipError_t {
      switch (a.pool.hd) {
        case 32: return run(std::integral_constant<int, 32>(), e8c);
        case 64: return run(std::integral_constant<int, 64>(), e8c);
        case 128: return run(std::integral_constant<int, 128>(), e8c);
        default: return hipErrorInvalidValue;
      }
    };
    const hipError_t e = e8 ? run_h(std::true_type()) : run_h(std::false_type());
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace dsf
