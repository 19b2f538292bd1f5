// Attention of each sequence's new tokens over its pages (gfx950).
//
// The query heads of a kv head and a sequence's new tokens are the rows of
// one problem, token-major (row m = token * G + head), so that a tile of rows
// reads a key or value once for all of them. A workgroup keeps the running
// maximum and sum of the softmax of a tile's rows in fp32. Where there are
// too few tiles for the chip the slots are divided too, by rules that every
// workgroup works out for itself from the sequences' lengths on the device
// (the host knows only bounds): chunks of tokens and fp32 in even splits of
// each tile (paged_item), sequences of few rows in equal shares of all the
// slots (paged_flat). The shares of a tile go to the workspace and
// paged_join_kernel adds them up in their order.
//
// Times in this file are of whole calls with their join, in turn over three
// sets of inputs, unless a kernel's is meant. A call of few tokens is a chain
// of waits: 2.4 us until a workgroup knows its share (lengths, a scan), 1.5 to
// its pages and queries, then 2.2 per turn of a wave.
#include <algorithm>
#include <type_traits>

#include "paged.h"

namespace dsf {

struct PagedKernelArgs {
  PagedPool pool;
  PagedBatch pb;
  const void* q; int64_t q_row, q_head;
  void* out; int64_t o_row, o_head;
  int G, window;
  Divisor by_G, by_Hkv;
  int bm_shift;    // log2 of the rows per tile
  int m_lo, m_hi;  // sequences with m_lo < rows * G <= m_hi take part
  int items;       // per kv head: the grid's, and no more than that have a place in part_o
  int target;      // of them to cut the work into (0: no splits)
  int split_min;   // least blocks of 64 slots per split
  int split_gain;  // least blocks that the longest tile has to be cut by
  int unit_shift;  // paged_flat: log2 of the slots per unit
  float* part_o;   // [item][kv head][BM][HD]
  float2* part_ml; // [item][kv head][BM]: maximum (log2 units), sum
};

// Rows of a sequence (tokens times heads of a kv head) up to which its weights
// have 16 bits, whatever else is in the batch and whichever kernel takes it:
// the token kernel where no sequence may have more by the batch's bounds, else
// the chunk kernel (but for the sequences of one token). A choice for what a
// decoding step answers, not for time: 16 sequences of 49 rows over 500 to
// 6000 slots take 44.1 us, as chunks with 8 bits 33.1; 64 of 28 rows 112.5 and
// 114.8; those 16 beside a chunk of 512 over 4096 slots 75, with 8 bits 67.
constexpr int kTokenRows = 64;

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

// Largest of the wave's numbers (none negative), in every lane.
__device__ __forceinline__ int wave_most(int v) {
#define DSF_SCAN(ctrl, rows) v = max(v, __builtin_amdgcn_update_dpp(0, v, ctrl, rows, 0xf, false))
  DSF_SCAN(0x111, 0xf);
  DSF_SCAN(0x112, 0xf);
  DSF_SCAN(0x114, 0xf);
  DSF_SCAN(0x118, 0xf);
  DSF_SCAN(0x142, 0xa);
  DSF_SCAN(0x143, 0xc);
#undef DSF_SCAN
  return __builtin_amdgcn_readlane(v, 63);
}

// A sequence's work: `tiles` tiles of BM rows, slots from `lo` (a multiple of
// 64) to kv, of which a tile sees no more than `blocks` blocks of 64.
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
  if (a.window) w.blocks = min(w.blocks, (min(a.window, w.kv) + ((1 << a.bm_shift) - 1) / a.by_G + 64 + 63) >> 6);
  return w;
}
// Lane l's shape, in every lane.
__device__ __forceinline__ PagedShape shape_of(const PagedShape& w, int l) {
  auto at = [l](int v) { return __builtin_amdgcn_readlane(v, l); };
  return PagedShape{at(w.n), at(w.row0), at(w.kv), at(w.M), at(w.tiles), at(w.lo), at(w.blocks)};
}
struct PagedItem {
  PagedShape w;
  int b;       // -1: none
  int first;   // the sequence's first item
  int local;   // this one's number among them
  int splits;  // of each of the sequence's tiles
};
constexpr int kNoSplit = 1 << 19;  // blocks: more slots than a sequence may have
// A tile's blocks go to its splits evenly, so that they end at the same time.
__device__ __forceinline__ int paged_splits(const PagedShape& w, int per) { return max((w.blocks + per - 1) / per, 1); }
// Blocks of 64 slots per split, at most. All the work (tiles times blocks)
// over the number of items aimed at: a longer item would outlast the others.
// Where there are fewer tiles than that, so many longer that the items are no
// more: one round of workgroups, and a few in a second would double the time.
// No splits where they would shorten the longest tile by a.split_gain or less.
// w: shapes of the first 64 sequences, in lanes. Batches of more are only cut
// by the share: the two rules after it need the sequences several times over
// (60 tokens and 4 chunks of 300, 64 sequences: 39.8 us; with one token more
// 44.6).
// (Even splits of what a tile sees, not of its sequence: 24 sequences with six
// chunks 60.2 -> 57.1 us, chunks with a window 56.7 -> 55.5. Splits of one
// place kept on one XCD, for its L2: 2 to 15 % slower, the XCDs' loads differ.)
__device__ __forceinline__ int paged_split_blocks(const PagedKernelArgs& a, const PagedShape& w, int lane) {
  if (a.target == 0) return kNoSplit;
  // sum over the sequences of what f says of them
  auto total = [&](auto f) {
    int n = f(w);
    for (int b0 = 64; b0 < a.pb.B; b0 += 64)
      if (b0 + lane < a.pb.B) n += f(paged_shape(a, b0 + lane));
    return __builtin_amdgcn_readlane(wave_prefix(n), 63);
  };
  const int sum = total([](const PagedShape& x) { return x.tiles * x.blocks; });
  int per = max((sum + a.target - 1) / a.target, a.split_min);
  if (a.pb.B <= 64 && total([](const PagedShape& x) { return x.tiles; }) < a.target) {
    for (int i = 0; i < 4; ++i) {
      const int items = total([per](const PagedShape& x) { return x.tiles * paged_splits(x, per); });
      if (items <= a.target) break;
      // (a row_start that does not ascend may claim any number of items)
      per = int(min((unsigned(per) * unsigned(min(items, 4096)) + a.target - 1) / unsigned(a.target), unsigned(kNoSplit)));
    }
    if (wave_most(w.tiles ? w.blocks : 0) <= per + a.split_gain) per = kNoSplit;
  }
  return per;
}

// The sequence that item `item` (of one kv head) belongs to.
__device__ __forceinline__ PagedItem paged_item(const PagedKernelArgs& a, int item, int lane) {
  PagedShape w = {};
  if (lane < a.pb.B) w = paged_shape(a, lane);
  const int per = paged_split_blocks(a, w, lane);
  PagedItem it = {};
  it.b = -1;
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
      it.splits = __builtin_amdgcn_readlane(splits, l);
      it.w = shape_of(w, l);
      return it;
    }
    first += __builtin_amdgcn_readlane(end, 63);
  }
  return it;
}

// Sequences of few rows: the slots of all tiles, in units of 64 (more where
// their number could pass 2^30), as one line that a kv head's workgroups
// share evenly. Workgroup j has the units from start(j) to start(j + 1), so
// at most its first and its last tile are shared with others; it leaves the
// share of a tile that began before it at place 2 j, of one that goes on
// behind it at place 2 j + 1. Short work is not cut up: with tiles for
// everybody, none longer than kWholeUnits, each workgroup has whole tiles.
// kWholeUnits: whole, 900 slots of one sequence take 9.7 us, cut up 10.8, and
// 513 slots 8.3 and 11.0; but 2000 slots 14.4 and 10.5.
// kLeastUnits: 2000 slots of four sequences take 10.6 us; with 2, for more
// shares to join, 11.4, with 8, for fewer workgroups, 11.8.
constexpr int kWholeUnits = 16;  // 1024 slots
constexpr int kLeastUnits = 4;   // of a share
struct PagedFlat {
  int wgs;    // with work
  int q, r;   // units each, and one more for the first r
  bool whole; // workgroup j has tile j
  __device__ __forceinline__ int start(int j) const { return j * q + min(j, r); }
  __device__ __forceinline__ int of(int u) const { return u < r * (q + 1) ? u / (q + 1) : r + (u - r * (q + 1)) / q; }
};
__device__ __forceinline__ int paged_units(const PagedKernelArgs& a, const PagedShape& w) {  // of a tile
  return max((max(w.kv - w.lo, 0) + (1 << a.unit_shift) - 1) >> a.unit_shift, 1);
}
__device__ __forceinline__ PagedFlat paged_flat(const PagedKernelArgs& a, const PagedShape& w, int lane) {
  int units = w.tiles ? w.tiles * paged_units(a, w) : 0, tiles = w.tiles, most = w.tiles ? paged_units(a, w) : 0;
  for (int b0 = 64; b0 < a.pb.B; b0 += 64) {
    if (b0 + lane < a.pb.B) {
      const PagedShape x = paged_shape(a, b0 + lane);
      if (x.tiles) {
        const int n = paged_units(a, x);
        units += x.tiles * n;
        tiles += x.tiles;
        most = max(most, n);
      }
    }
  }
  units = __builtin_amdgcn_readlane(wave_prefix(units), 63);
  tiles = __builtin_amdgcn_readlane(wave_prefix(tiles), 63);
  most = wave_most(most);
  PagedFlat f;
  f.whole = most << a.unit_shift <= kWholeUnits << 6 && tiles <= a.items;
  f.wgs = f.whole ? tiles : min(max(units / kLeastUnits, 1), a.items);
  if (units == 0) f.wgs = 0;
  f.q = f.wgs ? units / f.wgs : 0;
  f.r = units - f.q * f.wgs;
  return f;
}
// The sequence and tile of position `pos`, a unit or (whole) a tile.
struct PagedSpot {
  PagedShape w;
  int b;           // -1: none
  int tile;        // of the sequence
  int from, until; // units (whole: tiles) that the tile spans, on the line
};
__device__ __forceinline__ PagedSpot paged_spot(const PagedKernelArgs& a, PagedShape w, bool whole, int pos, int lane) {
  int base = 0;
  for (int b0 = 0; b0 < a.pb.B; b0 += 64) {
    if (b0) {
      w = PagedShape{};
      if (b0 + lane < a.pb.B) w = paged_shape(a, b0 + lane);
    }
    const int each = whole ? 1 : paged_units(a, w), c = w.tiles * each, end = wave_prefix(c);
    const uint64_t over = __builtin_amdgcn_ballot_w64(base + end > pos);
    if (over) {
      const int l = __builtin_ctzll(over), n = __builtin_amdgcn_readlane(each, l);
      const int first = base + __builtin_amdgcn_readlane(end, l) - __builtin_amdgcn_readlane(c, l);
      const int t = (pos - first) / n;
      return PagedSpot{shape_of(w, l), b0 + l, t, first + t * n, first + t * n + n};
    }
    base += __builtin_amdgcn_readlane(end, 63);
  }
  return PagedSpot{PagedShape{}, -1, 0, 0, 0};
}

// One item's tile and slots. Splits outermost: neighbouring tiles read about
// the same slots at the same time; within a split the last tile, which sees
// the most, is the first.
struct PagedWork {
  int b, n, row0, kv, M;
  int tile;            // of BM rows
  int p0;              // slot of the sequence's first row (may be negative)
  int begin, end;      // slots of this item that some row of the tile sees
  int splits;
};
// Slots that some row of the tile sees: from a multiple of 64.
__device__ __forceinline__ void paged_range(const PagedKernelArgs& a, const PagedShape& w, int tile, int* begin, int* end) {
  const int p0 = w.kv - w.n;
  const int m0 = tile << a.bm_shift, m1 = min(m0 + (1 << a.bm_shift), w.M) - 1;
  const int s = a.window ? max(p0 + m0 / a.by_G - a.window + 1, 0) & ~63 : 0;
  *begin = s;
  *end = max(min(p0 + m1 / a.by_G + 1, w.kv), s);
}
// Slots per split of such a range (0: there are none).
__device__ __forceinline__ int paged_split_len(int begin, int end, int splits) {
  return (((end - begin + 63) >> 6) + splits - 1) / splits << 6;
}
__device__ __forceinline__ PagedWork paged_work(const PagedKernelArgs& a, const PagedItem& it) {
  PagedWork k;
  const PagedShape& w = it.w;
  k.b = it.b;
  k.n = w.n;
  k.row0 = w.row0;
  k.kv = w.kv;
  k.M = w.M;
  k.p0 = w.kv - w.n;
  const int split = it.local / w.tiles;
  k.tile = w.tiles - 1 - (it.local - split * w.tiles);
  k.splits = it.splits;
  paged_range(a, w, k.tile, &k.begin, &k.end);
  const int len = paged_split_len(k.begin, k.end, it.splits);
  k.begin = min(k.begin + split * len, k.end);
  k.end = min(k.begin + len, k.end);
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

// LDS transpose load: within each 16-lane group G, lane 16 G + 4 a + b
// receives element b of the 8-byte rows addressed by lanes 16 G + a + 4 j,
// j = 0..3.
__device__ __forceinline__ bf16x4 lds_read_tr(const char* p) {
  typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
  return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(__attribute__((address_space(3))) const char*)p);
}

// Maximum and sum over a lane and the lane 32 beside it.
__device__ __forceinline__ float pair32_max(float v) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  float r;  // (fmaxf would first quiet what it cannot see to be a number already)
  asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a[0]), "v"(a[1]));
  return r;
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

#define DSF_INLINE __attribute__((always_inline))  // for lambdas over register arrays

// N DMA instructions of a wave: lane l of the e-th brings the 16 bytes at
// offset(e) of `src` to lds + 1024 e + 16 l, zeros for those past `bytes`.
// A scalar register that a vector instruction (v_readfirstlane, a spill's
// v_readlane) writes may be an operand of a memory instruction five wait
// states later, M0 one state after it is written; the compiler does not count
// for inline assembly, so each of these brings its own six. (M0 is reserved:
// the compiler keeps nothing in it, and nothing else here uses it.)
template <int N, typename F>
__device__ __forceinline__ void lds_dma(const char* src, int bytes, char* lds, F offset) {
  auto uniform = [](uint32_t x) { return uint32_t(__builtin_amdgcn_readfirstlane(int(x))); };
  const uint64_t base = reinterpret_cast<uint64_t>(src);
  // buffer resource: base, no stride, size, raw 32-bit format
  const u32x4 rsrc = {uniform(uint32_t(base)), uniform(uint32_t(base >> 32) & 0xffffu), uniform(uint32_t(bytes)),
                      0x00020000u};
  const uint32_t at = uniform(uint32_t(size_t((__attribute__((address_space(3))) char*)lds)));
#pragma unroll
  for (int e = 0; e < N; ++e)
    asm volatile(
        "s_mov_b32 m0, %0\n\t"
        "s_nop 4\n\t"
        "buffer_load_dwordx4 %1, %2, 0 offen lds"
        :
        : "s"(at + 1024 * e), "v"(offset(e)), "s"(rsrc)
        : "memory");
}

// 16 slots from `slot` on of one kv head to LDS at `lds` (a tile's row 16 i):
// bf16 by DMA, each lane 16 bytes at a time; slots at or past `end` become
// zeros. All 16 lie in one page.
template <int HD>
struct DmaSlots {
  __device__ static __forceinline__ void load(const void* pool, const PagedKernelArgs& a, int page, int kvh, int slot,
                                              int end, char* lds, int lane) {
    using S = SlotTile<HD>;
    const int64_t row = ((int64_t(page) * a.pool.Hkv + kvh) << a.pb.page_shift) + (slot & ((1 << a.pb.page_shift) - 1));
    lds_dma<16 * S::kRowBytes / 1024>(static_cast<const char*>(pool) + row * S::kRowBytes,
                                      min(max(end - slot, 0), 16) * S::kRowBytes, lds, [lane](int e) {
                                        const int byte = 1024 * e + 16 * lane;
                                        const int r = byte / S::kRowBytes, c = byte % S::kRowBytes / 16;
                                        return r * S::kRowBytes + ((c ^ S::swz(r)) << 4);
                                      });
  }
};

// 16 slots of e4m3 codes as they are, to `lds` (at least 1 KB).
template <int HD>
__device__ __forceinline__ void codes16_dma(const void* pool, const PagedKernelArgs& a, int page, int kvh, int slot, int end,
                                            char* lds, int lane) {
  const int64_t row = ((int64_t(page) * a.pool.Hkv + kvh) << a.pb.page_shift) + (slot & ((1 << a.pb.page_shift) - 1));
  lds_dma<(16 * HD + 1023) / 1024>(static_cast<const char*>(pool) + row * HD, min(max(end - slot, 0), 16) * HD, lds,
                                   [lane](int e) { return 1024 * e + 16 * lane; });
}

// e4m3 codes in registers, 16 of a slot at a time, and their widening into
// the tile.
template <int HD>
struct CodeSlots {
  static constexpr int kCpr = HD / 16;                       // 16-byte loads per slot
  static constexpr int kLoads = kCpr >= 4 ? 16 * kCpr / 64 : 1;
  u32x4 c[kLoads];
  uint32_t e;  // exponent byte of slot lane & 15
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
    for (int i = 0; i < kLoads; ++i)
      c[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rc, 1024 * i + 16 * lane, 0, 0));
    e = __builtin_amdgcn_raw_buffer_load_b8(re, lane & 15, 0, 0);
  }
  // what codes16_dma brought; `exps`: the exponent byte of slot lane & 15
  __device__ __forceinline__ void read(const char* lds, uint32_t exps, int lane) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) c[i] = *reinterpret_cast<const u32x4*>(lds + 1024 * i + 16 * lane);
    e = exps;
  }
  __device__ __forceinline__ void store(char* lds, int lane) const {
    using S = SlotTile<HD>;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = 64 / kCpr * i + lane / kCpr, ch = 2 * (lane % kCpr);
      const float s = paged_scale(__builtin_amdgcn_ds_bpermute((r & 15) << 2, int(e)));
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
// Where a tile hides slots from some of its rows (bf16 tokens: everywhere),
// such values are therefore taken out of the product (finite_or_zero) and
// counted in a second one of codes (1: inf, 256: -inf, 65536: NaN, exact sums
// of at most 64) with ones at the slots that a row sees, and what a row saw is
// added to its sum.
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

// A workgroup of four waves takes 128 rows, a wave 32 of them, and 64 slots
// at a time, staged by all four.
//
// S^T = K Q^T with v_mfma_f32_32x32x16_bf16: lane (r32, hi) holds of row r32
// the scores of slots 8 (i / 4) + 4 hi + i % 4 of 32, i < 16, so a row's
// maximum needs one exchange between two lanes, and its probabilities lie as
// the B operand of O^T += V^T P^T wants them if the product takes the slots
// in that order: step s covers 16 slots, element j of lane (., hi) being slot
// 16 s + 4 hi + j % 4 + 8 (j / 4). Probabilities are rounded to bf16 for that
// product (off by 2^-8 at most each, and the row's sum is of the rounded
// ones); maximum, sum and accumulators are fp32. The maximum a row is scaled
// by follows the true one at a distance: it moves when a tile's is over 2^8
// times it, so weights stay below 2^8 and the accumulators are rarely
// rescaled.
//
// The matrix cores and the vector units of a SIMD overlap only within a wave
// (a probe: 4 FMAs and an exponential beside each 32 x 32 MFMA cost nothing),
// so each half turn, of 32 slots, does three things that do not depend on
// each other: the scores of half u + 1, the softmax of half u and the product
// of half u - 1 with its values. Turn t has the product of tile t's two halves
// and the scores of tile t + 1's, so of keys and of values one tile each is
// in use and one on its way. Turns with hidden slots and the last run in a
// general form of the same.
//
// PRECISE, for sequences of up to kTokenRows rows: two waves' rows are all, so
// a wave takes one half of every tile, with a second bf16 part of the weights
// in the product (the sum is of the fp32 ones), and at the end the second
// halves' results go to the first ones' waves. Scores, softmax and product
// follow each other. (Both halves by one wave: 16 sequences of 49 rows beside
// a chunk 90 us where weights of 8 bits took 64, with 60 to 120 bytes of
// spills; this way 75 and 67. A function of its own, so that neither form's
// registers count for the other.)
//
// DMA into LDS is issued in inline assembly: the compiler, which cannot tell
// the stages apart, would wait for it before every transpose load. e4m3 codes
// come as they are and are widened on their way to the stage a turn later.
//
// Bound by LDS reads at head dim 128: 32 keys and 32 values of 128 are 16 KB
// for a wave and half turn. A loop of nothing else reads 124 bytes a clock and
// CU with the keys' loads and 67 with the values' (transpose loads, in either
// case from these addresses), so the 6.8e7 loads of the batch below, a third of
// them keys', take 5.3e8 of the CUs' 6.8e8 clocks; matrix products take 53 % of
// the SIMDs'. (SQ_LDS_IDX_ACTIVE counts 4 clocks for a load of keys that takes
// 8, and 2 for one of values.) Two chunks of some 4000 tokens over 12000 to
// 20000 slots (28 heads over 4, 1.48 TFLOP): 1360 us, 1.09 PFLOP/s (a large
// library product of the same type: 1.61); 1420 to 1680 on some hosts. Slower,
// where this took 1405: 64 rows a wave, for half the reads, 1595 us (one wave
// to a SIMD issues a vector instruction every 7 clocks); eight waves with 256
// rows and four stages 1430; LDS addresses that move with the turn instead of
// constant ones 1412 against 1377.
// One chunk of 512 over 8192 slots (12 heads over 2): 44 us, the kernel 38: 5
// us to the first scores, 13 turns of 1.8 us, 6 us for 29 MB of shares.
// LDS: two tiles of keys, two of values; e4m3: each wave's codes of a tile of
// either. Four stages at head dim 64 gained nothing.
template <int HD>
constexpr int kCodeBytes = 16 * HD > 1024 ? 16 * HD : 1024;
template <int HD, bool E8>
constexpr int kChunkLds = 4 * 64 * SlotTile<HD>::kRowBytes + (E8 ? 8 * kCodeBytes<HD> : 0);
template <int HD, bool E8, bool PRECISE>
__device__ __forceinline__ void paged_chunk_tile(const PagedKernelArgs& a, const PagedItem& it, int block, int kvh,
                                                 char* smem) {
  using S = SlotTile<HD>;
  constexpr int BM = 128, NS = HD / 16, ND = HD / 32;
  constexpr int kTile = 64 * S::kRowBytes;
  constexpr float kLag = 8.f;           // log2 units
  constexpr float kNothing = -3.0e38f;  // the maximum of nothing: finite, so that -inf less it is -inf
  const int tid = threadIdx.x, lane = tid & 63, r32 = lane & 31, hi = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = wave >> 1;  // PRECISE
  const PagedWork w = paged_work(a, it);
  if (w.splits > 1 && w.begin >= w.end) return;  // a split that none of the tile's rows sees

  // this wave's rows: row m of the sequence, its token's slot
  const int m0 = w.tile * BM + (PRECISE ? wave & 1 : wave) * 32, m = m0 + r32, mc = min(m, w.M - 1);
  const int tok = mc / a.by_G, g = mc - tok * a.G, my_slot = w.p0 + tok;
  bf16x8 qf[NS];
  {
    const uint16_t* qp =
        static_cast<const uint16_t*>(a.q) + int64_t(w.row0 + tok) * a.q_row + int64_t(kvh * a.G + g) * a.q_head;
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(qp + 16 * s + 8 * hi);
  }
  // slots that every row of the wave sees: [see_lo, see_hi)
  const int see_hi = min(w.p0 + min(m0, w.M - 1) / a.by_G + 1, w.end);
  const int see_lo = a.window ? w.p0 + min(m0 + 31, w.M - 1) / a.by_G - a.window + 1 : 0;

  // tiles up to the last one that some row sees
  const int any_hi = m0 < w.M ? w.p0 + min(m0 + 31, w.M - 1) / a.by_G + 1 : 0;
  const int my_nt = max(min(any_hi, w.end) - w.begin + 63, 0) >> 6;

  const float sc = 1.4426950408889634f / sqrtf(float(HD));  // log2(e) / sqrt(hd)
  f32x16 o[ND];
  float m_run = kNothing, l_run = 0.f;
#pragma unroll
  for (int db = 0; db < ND; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.f;

  // staging: this wave brings slots 16 wave .. + 15 of every tile
  const int nt = (w.end - w.begin + 63) >> 6, s0 = w.begin + 16 * wave;
  PagedTable tab;
  tab.load(a, w.b, w.begin >> a.pb.page_shift, lane);
  PagedTable vtab = tab;  // values are a tile behind
  char* const mine = smem + 16 * wave * S::kRowBytes;
  char* const raw = smem + 4 * kTile + 2 * wave * kCodeBytes<HD>;  // keys' codes, then values'
  uint32_t ke = 0, ve = 0;  // exponent bytes of the codes there, of slot lane & 15
  auto exponents = [&](const uint8_t* exps, int page, int slot) DSF_INLINE {
    const int64_t row = ((int64_t(page) * a.pool.Hkv + kvh) << a.pb.page_shift) + (slot & ((1 << a.pb.page_shift) - 1));
    return uint32_t(slot + (lane & 15) < w.end ? exps[row + (lane & 15)] : 0);
  };
  auto fetch_k = [&](int t) DSF_INLINE {
    const int slot = s0 + 64 * t, page = tab.at(a, w.b, slot >> a.pb.page_shift, lane);
    if constexpr (E8) {
      ke = exponents(a.pool.ke, page, slot);
      codes16_dma<HD>(a.pool.k, a, page, kvh, slot, w.end, raw, lane);
    } else {
      DmaSlots<HD>::load(a.pool.k, a, page, kvh, slot, w.end, mine + (t & 1) * kTile, lane);
    }
  };
  auto fetch_v = [&](int t) DSF_INLINE {
    const int slot = s0 + 64 * t, page = vtab.at(a, w.b, slot >> a.pb.page_shift, lane);
    if constexpr (E8) {
      ve = exponents(a.pool.ve, page, slot);
      codes16_dma<HD>(a.pool.v, a, page, kvh, slot, w.end, raw + kCodeBytes<HD>, lane);
    } else {
      DmaSlots<HD>::load(a.pool.v, a, page, kvh, slot, w.end, mine + (2 + (t & 1)) * kTile, lane);
    }
  };
  // e4m3: the codes fetched last, widened into tile t's stage
  auto widen = [&](int t, bool values) DSF_INLINE {
    CodeSlots<HD> x;
    x.read(raw + (values ? kCodeBytes<HD> : 0), values ? ve : ke, lane);
    x.store(mine + ((values ? 2 : 0) + (t & 1)) * kTile, lane);
  };
  constexpr int kTileDma = 16 * S::kRowBytes / 1024;  // DMA instructions of fetch_k, of fetch_v (bf16)
  auto meet = [&]() DSF_INLINE {                      // what every wave has written to LDS is there for all
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  auto landed = [&]() DSF_INLINE {  // and what every wave has fetched
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    meet();
  };

  // LDS addresses: rows r32 (+ 32 half) of a key tile, chunk 2 st + hi; of a value tile lane (group of 16 G, a4 =
  // lane & 3, j = lane / 4 & 3) reads slots 4 hi + j (+ 8) (+ 16 st) at dims 32 db + 16 (G & 1) + 4 a4
  const int vrow = 4 * hi + ((lane >> 2) & 3), vch = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
  const char *ka[NS], *va[ND], *vb[ND];
#pragma unroll
  for (int st = 0; st < NS; ++st) ka[st] = smem + r32 * S::kRowBytes + (((2 * st + hi) ^ S::swz(r32)) << 4);
#pragma unroll
  for (int db = 0; db < ND; ++db) {
    const char* v = smem + 2 * kTile + vrow * S::kRowBytes + (lane & 1) * 8;
    va[db] = v + (((4 * db + vch) ^ S::swz(vrow)) << 4);
    vb[db] = v + 8 * S::kRowBytes + (((4 * db + vch) ^ S::swz(vrow + 8)) << 4);
  }
  // step st of a half of a key tile, and 32 dims of 16 slots of a value tile, at byte `at` of the stages
  auto read_k = [&](int at, int st) DSF_INLINE { return *reinterpret_cast<const bf16x8*>(ka[st] + at); };
  auto read_v = [&](int at, int db) DSF_INLINE {
    return __builtin_shufflevector(lds_read_tr(va[db] + at), lds_read_tr(vb[db] + at), 0, 1, 2, 3, 4, 5, 6, 7);
  };

  // scores of one half of tile t
  auto scores = [&](int t, int half, f32x16& s) DSF_INLINE {
    const int at = (t & 1) * kTile + 32 * half * S::kRowBytes;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int st = 0; st < NS; ++st) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_k(at, st), qf[st], s, 0, 0, 0);
  };
  // the slots of a half of tile t that this lane's row sees, relative to the lane's first
  auto bounds = [&](int t, int half, int* lo, int* top) DSF_INLINE {
    const int kb0 = w.begin + 64 * t + 32 * half + 4 * hi;
    *top = min(my_slot, w.end - 1) - kb0;
    *lo = a.window ? my_slot - a.window + 1 - kb0 : -64;
  };
  // The softmax of a half's scores in twelve steps of about the same work: the maximum in 0 to 3, then two of a lane's
  // 16 weights in each. `sum` is of this half's, m_new what they are scaled by.
  struct Soft {
    float mx, m_new, sum;
  };
  auto soft = [&](int step, Soft& f, f32x16& s, bf16x8 (&p)[2]) DSF_INLINE {
    if (step == 0) {
      f.mx = fmaxf(s[0], s[1]);
#pragma unroll
      for (int i = 2; i < 8; ++i) f.mx = fmaxf(f.mx, s[i]);
    } else if (step == 1) {
#pragma unroll
      for (int i = 8; i < 16; ++i) f.mx = fmaxf(f.mx, s[i]);
    } else if (step == 2) {
      f.mx = pair32_max(f.mx) * sc;
    } else if (step == 3) {
      f.m_new = f.mx > m_run + kLag ? f.mx : m_run;
      f.sum = 0.f;
    } else {
      const int e = 2 * (step - 4);
      typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
      const bf16x2 one = {(__bf16)1.0f, (__bf16)1.0f};
      const bf16x2 p2 = {(__bf16)__builtin_amdgcn_exp2f(fmaf(s[e], sc, -f.m_new)),
                         (__bf16)__builtin_amdgcn_exp2f(fmaf(s[e + 1], sc, -f.m_new))};
      p[e / 8][e % 8] = p2[0];
      p[e / 8][e % 8 + 1] = p2[1];
      f.sum = __builtin_amdgcn_fdot2_f32_bf16(p2, one, f.sum, false);
    }
  };
  // after it, and after the product that the accumulators had still to get with the old maximum
  auto settle = [&](const Soft& f) DSF_INLINE {
    if (__builtin_amdgcn_ballot_w64(f.m_new != m_run)) {
      const float alpha = __builtin_amdgcn_exp2f(m_run - f.m_new);  // 1 where it did not move
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < ND; ++db) o[db] *= alpha;
    }
    l_run += f.sum;
    m_run = f.m_new;
  };
  // product of a half of tile t, where some row may not see some slot; `low`: the weights' second parts, or none
  auto product = [&](int t, int half, const bf16x8 (&p)[2], const bf16x8* low) DSF_INLINE {
    const int at = (t & 1) * kTile + 32 * half * S::kRowBytes;
#pragma unroll
    for (int db = 0; db < ND; ++db) {
      bf16x8 vf[2];
#pragma unroll
      for (int st = 0; st < 2; ++st) vf[st] = read_v(at + 16 * st * S::kRowBytes, db);
      if (__builtin_amdgcn_ballot_w64((not_finite_bits(vf[0]) | not_finite_bits(vf[1])) != 0)) {
        int lo, top;
        bounds(t, half, &lo, &top);
        f32x16 c;
#pragma unroll
        for (int i = 0; i < 16; ++i) c[i] = 0.f;
#pragma unroll
        for (int st = 0; st < 2; ++st) {
          bf16x8 one;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int x = 16 * st + j % 4 + 8 * (j / 4);
            one[j] = (__bf16)(x > top || x < lo ? 0.f : 1.f);
          }
          c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(not_finite_codes(vf[st]), one, c, 0, 0, 0);
          vf[st] = finite_or_zero(vf[st]);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] += not_finite_sum(c[i]);
      }
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[st], p[st], o[db], 0, 0, 0);
        if (low) o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[st], low[st], o[db], 0, 0, 0);
      }
    }
  };
  auto hide = [&](int t, int half, f32x16& s) DSF_INLINE {
    int lo, top;
    bounds(t, half, &lo, &top);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int x = 8 * (i / 4) + i % 4;
      s[i] = x > top || x < lo ? -INFINITY : s[i];
    }
  };
  // A half turn without hidden slots: s_next of the half at byte `kat` of the key stages, the softmax of s_now into
  // p_now, the product of the half at byte `vat` of the value stages with p_last. The instructions stand in the order
  // they are to be issued in: a matrix product, of the scores and of the values in turn, then a part of the softmax;
  // operands are read kAhead products of a kind ahead.
  auto half_turn = [&](int kat, f32x16& s_next, f32x16& s_now, bf16x8 (&p_now)[2], int vat,
                       const bf16x8 (&p_last)[2]) DSF_INLINE {
    constexpr int kPairs = NS, kSteps = 12, kAhead = 2;  // NS == 2 ND: as many products of either kind
    Soft f = {};
    bf16x8 kf[kAhead + 1], vf[kAhead + 1];
    auto next_k = [&](int i) DSF_INLINE { kf[i % (kAhead + 1)] = read_k(kat, i); };
    auto next_v = [&](int i) DSF_INLINE { vf[i % (kAhead + 1)] = read_v(vat + 16 * (i / ND) * S::kRowBytes, i % ND); };
#pragma unroll
    for (int i = 0; i < kAhead && i < kPairs; ++i) {
      next_k(i);
      next_v(i);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) s_next[i] = 0.f;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 2 * kPairs; ++i) {
      const int j = i / 2;
      if (i % 2 == 0) {
        if (j + kAhead < kPairs) next_k(j + kAhead);
        s_next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[j % (kAhead + 1)], qf[j], s_next, 0, 0, 0);
      } else {
        if (j + kAhead < kPairs) next_v(j + kAhead);
        o[j % ND] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[j % (kAhead + 1)], p_last[j / ND], o[j % ND], 0, 0, 0);
      }
#pragma unroll
      for (int step = i * kSteps / (2 * kPairs); step < (i + 1) * kSteps / (2 * kPairs); ++step) soft(step, f, s_now, p_now);
      __builtin_amdgcn_sched_barrier(0);
    }
    // the weights are wanted in the next half turn only: keep them from moving there
    asm volatile("" : "+v"(p_now[0]), "+v"(p_now[1]), "+v"(f.sum));
    settle(f);
  };
  // PRECISE: a half's scores to weights of 16 bits, as two bf16 numbers, and their product with its values
  auto precise_half = [&](int t, int half, f32x16& s) DSF_INLINE {
    hide(t, half, s);
    float mx = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
    Soft f;
    f.m_new = fmaxf(pair32_max(mx) * sc, m_run);
    f.sum = 0.f;
    bf16x8 high[2], low[2];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float x = __builtin_amdgcn_exp2f(fmaf(s[i], sc, -f.m_new));
      f.sum += x;
      high[i / 8][i % 8] = (__bf16)x;
      low[i / 8][i % 8] = (__bf16)(x - float((__bf16)x));
    }
    settle(f);
    product(t, half, high, low);
  };
  auto soft_all = [&](Soft& f, f32x16& s, bf16x8 (&p)[2]) DSF_INLINE {
#pragma unroll
    for (int step = 0; step < 12; ++step) soft(step, f, s, p);
  };

  if (nt > 0) {
    f32x16 s0x, s1;  // scores of a tile's halves
    bf16x8 p0[2], p1[2];
    Soft f = {};
    fetch_k(0);
    if constexpr (E8) {
      fetch_v(0);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      widen(0, false);
      widen(0, true);
      if (nt > 1) {
        fetch_k(1);
        fetch_v(1);
      }
    } else {
      fetch_v(0);
      if (nt > 1) fetch_k(1);
      // the first keys
      if (nt > 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * kTileDma) : "memory");
      else asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kTileDma) : "memory");
    }
    meet();
    if constexpr (PRECISE) {
      scores(0, half, s0x);
    } else {
      scores(0, 0, s0x);
      scores(0, 1, s1);
      hide(0, 0, s0x);
      soft_all(f, s0x, p0);
      settle(f);
    }
    if constexpr (E8) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      if (nt > 1) widen(1, false);
      if (nt > 2) fetch_k(2);
    }
    // At the start of turn t: p0 and s1 of tile t. Keys of tile t + 1 and values of tile t are in LDS then, and the
    // other stages are free: for what comes by DMA in this turn, or (e4m3) for the codes that came in the last one.
    auto open = [&](int t) DSF_INLINE {
      landed();
      if constexpr (E8) {
        if (t + 2 < nt) widen(t + 2, false);
        if (t + 1 < nt) widen(t + 1, true);
        if (t + 3 < nt) fetch_k(t + 3);
        if (t + 2 < nt) fetch_v(t + 2);
      } else {
        if (t + 2 < nt) fetch_k(t + 2);
        if (t + 1 < nt) fetch_v(t + 1);
      }
    };
    // turns [t0, t1) have no hidden slot in tiles t and t + 1; they go in pairs from an even one, so that the stages'
    // addresses are constants
    const int t0 = min(max(see_lo - w.begin + 63, 0) >> 6, nt);
    const int t1 = max((see_hi - w.begin) / 64 - 1, t0);
    constexpr int kHalf = 32 * S::kRowBytes;
    int t = 0;
    if constexpr (PRECISE) {
      // (scores of tile t before its turn, in which its keys' stage is filled again)
      for (; t < my_nt; ++t) {
        open(t);
        precise_half(t, half, s0x);
        if (t + 1 < my_nt) scores(t + 1, half, s0x);
      }
    } else {
      while (t < my_nt) {
        if (t >= t0 && !(t & 1)) {
          for (; t + 1 < t1; t += 2) {
            open(t);
            half_turn(kTile, s0x, s1, p1, 0, p0);
            half_turn(kTile + kHalf, s1, s0x, p0, kHalf, p1);
            open(t + 1);
            half_turn(0, s0x, s1, p1, kTile, p0);
            half_turn(kHalf, s1, s0x, p0, kTile + kHalf, p1);
          }
          if (t >= my_nt) break;
        }
        open(t);
        const bool more = t + 1 < my_nt;
        if (more) scores(t + 1, 0, s0x);
        hide(t, 1, s1);
        soft_all(f, s1, p1);
        product(t, 0, p0, nullptr);
        settle(f);
        if (more) {
          scores(t + 1, 1, s1);
          hide(t + 1, 0, s0x);
          soft_all(f, s0x, p0);
        }
        product(t, 1, p1, nullptr);
        if (more) settle(f);
        ++t;
      }
    }
    for (; t < nt; ++t) open(t);  // for the other waves
    if constexpr (PRECISE) {
      // the second halves' results to the waves that have the first ones'
      meet();  // every wave is done with the stages
      f32x4* os = reinterpret_cast<f32x4*>(smem) + (wave & 1) * 8 * HD + lane;
      float2* mls = reinterpret_cast<float2*>(smem + 256 * HD) + (wave & 1) * 64 + lane;
      if (half) {
#pragma unroll
        for (int db = 0; db < ND; ++db)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            os[64 * (4 * db + i)] = f32x4{o[db][4 * i], o[db][4 * i + 1], o[db][4 * i + 2], o[db][4 * i + 3]};
        *mls = make_float2(m_run, l_run);
      }
      meet();
      if (half) return;
      const float2 ml = *mls;
      const float top = fmaxf(m_run, ml.x);
      const float f0 = __builtin_amdgcn_exp2f(m_run - top), f1 = __builtin_amdgcn_exp2f(ml.x - top);
#pragma unroll
      for (int db = 0; db < ND; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x4 x = os[64 * (4 * db + i)];
#pragma unroll
          for (int j = 0; j < 4; ++j) o[db][4 * i + j] = o[db][4 * i + j] * f0 + x[j] * f1;
        }
      l_run = l_run * f0 + ml.y * f1;
      m_run = top;
    }
  }
  if (PRECISE && half) return;

  // lane holds O^T[dim 32 db + 8 (i / 4) + 4 hi + i % 4][row r32]
  const float l = pair32_sum(l_run);
  if (m >= w.M) return;
  if (w.splits > 1) {
    const int64_t at = int64_t(block) * BM + (m - w.tile * BM);
    float* po = a.part_o + at * HD;
#pragma unroll
    for (int db = 0; db < ND; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4*>(po + 32 * db + 8 * i + 4 * hi) =
            f32x4{o[db][4 * i], o[db][4 * i + 1], o[db][4 * i + 2], o[db][4 * i + 3]};
    if (hi == 0) a.part_ml[at] = make_float2(m_run == kNothing ? -INFINITY : m_run, l);
  } else {
    const float inv = l == 0.f ? 0.f : 1.0f / l;  // a row that sees nothing: zeros
    uint16_t* op = static_cast<uint16_t*>(a.out) + int64_t(w.row0 + tok) * a.o_row + int64_t(kvh * a.G + g) * a.o_head;
#pragma unroll
    for (int db = 0; db < ND; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u32x2 pk;
        pk[0] = uint32_t(f2bf(o[db][4 * i] * inv)) | uint32_t(f2bf(o[db][4 * i + 1] * inv)) << 16;
        pk[1] = uint32_t(f2bf(o[db][4 * i + 2] * inv)) | uint32_t(f2bf(o[db][4 * i + 3] * inv)) << 16;
        *reinterpret_cast<u32x2*>(op + 32 * db + 8 * i + 4 * hi) = pk;
      }
  }
}

template <int HD, bool E8>
__device__ __forceinline__ void paged_chunk(const PagedKernelArgs& a, int block, char* smem) {
  // kv head innermost: consecutive workgroups go to different XCDs, so that
  // (with 8 heads or a divisor of 8) an XCD's L2 sees the slots of few heads
  const int item = block / a.by_Hkv, kvh = block - item * a.pool.Hkv;
  const PagedItem it = paged_item(a, item, threadIdx.x & 63);
  if (it.b < 0) return;
  if (it.w.M > kTokenRows) paged_chunk_tile<HD, E8, false>(a, it, block, kvh, smem);
  else paged_chunk_tile<HD, E8, true>(a, it, block, kvh, smem);
}

// ------------------------------------------------------------ a few tokens

// Two transpose loads at each of four addresses and their wait: the V^T
// operands of v_mfma_f32_16x16x32_bf16 for four (16 dims, 32 slots).
template <int ROW>
__device__ __forceinline__ void lds_read_tr4x2(const uint32_t (&at)[4], u32x2 (&v)[8]) {
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8\n\t"
      "ds_read_b64_tr_b16 %1, %8 offset:%12\n\t"
      "ds_read_b64_tr_b16 %2, %9\n\t"
      "ds_read_b64_tr_b16 %3, %9 offset:%12\n\t"
      "ds_read_b64_tr_b16 %4, %10\n\t"
      "ds_read_b64_tr_b16 %5, %10 offset:%12\n\t"
      "ds_read_b64_tr_b16 %6, %11\n\t"
      "ds_read_b64_tr_b16 %7, %11 offset:%12\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7])
      : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "n"(16 * ROW)
      : "memory");
}

// 16 slots of keys as the A operands of S^T = K Q^T: lane (r16, grp) has dims
// dim(st, grp) .. + 7 of slot r16 for step st. The dims may be taken in any
// order that Q is taken in too, so e4m3 codes are loaded 16 at a time, half
// of them for the next step.
template <int HD, bool E8>
struct KeySlots {
  static constexpr int NS = HD / 32;
  static constexpr bool kWide = E8 && HD >= 64;
  static constexpr int kWords = E8 ? HD / 16 : HD / 8;  // of a lane
  uint32_t c[kWords];
  uint32_t e;
  __device__ static __forceinline__ int dim(int st, int grp) {
    return kWide ? 64 * (st >> 1) + 16 * grp + 8 * (st & 1) : 32 * st + 8 * grp;
  }
  __device__ __forceinline__ void load(const PagedKernelArgs& a, int page, int kvh, int slot, int end, int lane) {
    const int r16 = lane & 15, grp = lane >> 4, eb = E8 ? 1 : 2;
    const int64_t row = ((int64_t(page) * a.pool.Hkv + kvh) << a.pb.page_shift) + (slot & ((1 << a.pb.page_shift) - 1));
    const int rows = min(max(end - slot, 0), 16);
    const auto rc = __builtin_amdgcn_make_buffer_rsrc(static_cast<char*>(a.pool.k) + row * HD * eb, (short)0,
                                                      rows * HD * eb, 0x00020000);
    if constexpr (E8 && !kWide) {
      const u32x2 t = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rc, r16 * HD + 8 * grp, 0, 0));
      c[0] = t[0];
      c[1] = t[1];
    } else {
#pragma unroll
      for (int i = 0; i < kWords / 4; ++i) {
        const u32x4 t =
            __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rc, r16 * HD * eb + 16 * grp + 64 * i, 0, 0));
#pragma unroll
        for (int j = 0; j < 4; ++j) c[4 * i + j] = t[j];
      }
    }
    if constexpr (E8) {
      const auto re = __builtin_amdgcn_make_buffer_rsrc(a.pool.ke + row, (short)0, rows, 0x00020000);
      e = __builtin_amdgcn_raw_buffer_load_b8(re, r16, 0, 0);
    }
  }
  __device__ __forceinline__ bf16x8 at(int st) const {
    if constexpr (E8) {
      const float s = paged_scale(e);
      const u32x2 x = paged_widen4(c[2 * st], s), y = paged_widen4(c[2 * st + 1], s);
      return __builtin_bit_cast(bf16x8, u32x4{x[0], x[1], y[0], y[1]});
    } else {
      return __builtin_bit_cast(bf16x8, u32x4{c[4 * st], c[4 * st + 1], c[4 * st + 2], c[4 * st + 3]});
    }
  }
};

// 16 slots of values, 16 bytes a lane, for LDS.
template <int HD>
struct ValueSlots {
  static constexpr int kLoads = HD / 32;
  u32x4 c[kLoads];
  __device__ __forceinline__ void load(const PagedKernelArgs& a, int page, int kvh, int slot, int end, int lane) {
    const int64_t row = ((int64_t(page) * a.pool.Hkv + kvh) << a.pb.page_shift) + (slot & ((1 << a.pb.page_shift) - 1));
    const int rows = min(max(end - slot, 0), 16);  // the others load as zeros
    const auto rc = __builtin_amdgcn_make_buffer_rsrc(static_cast<char*>(a.pool.v) + row * HD * 2, (short)0, rows * HD * 2,
                                                      0x00020000);
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      c[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rc, 1024 * i + 16 * lane, 0, 0));
  }
  __device__ __forceinline__ void store(char* lds, int lane) const {
    using S = SlotTile<HD>;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int byte = 1024 * i + 16 * lane, r = byte / S::kRowBytes, ch = byte % S::kRowBytes / 16;
      *reinterpret_cast<u32x4*>(lds + r * S::kRowBytes + ((ch ^ S::swz(r)) << 4)) = c[i];
    }
  }
};

// A workgroup of W waves takes its share of the line (paged_flat), one
// tile of 16 NR rows after the other; of a tile's slots each wave runs through
// every W-th piece of TK by itself, with a softmax of its own, and they are
// joined in wave order. Memory bound (the rows of one token of a few
// heads are far too few for the matrix cores to matter), so what counts is
// bytes on the way: keys are loaded as the matrix operand they will be,
// straight into registers, values into registers and on through LDS, which
// transposes them; the next piece's loads are issued as soon as this one's
// registers are free. 16 rows leave registers for two waves to a SIMD: eight
// waves, one workgroup to a CU, so that short sequences take fewer turns and
// long ones have half the shares to join (two workgroups of four waves: one
// token over 513 slots 9.0 us for 8.1, 64 tokens 99.5 for 97.2, 9 long e4m3
// sequences 55.2 for 53.5; two of eight, in two rounds: 101.6 and 59.2). More
// rows have four (32 rows by eight waves spill: 112 -> 151 us).
//
// S^T = K Q^T with v_mfma_f32_16x16x32_bf16: lane (r16, grp) holds of row r16
// the scores of slots 16 kb + 4 grp + i, which is the B operand of
// O^T += V^T P^T when step ks takes slots 32 ks + 16 (j / 4) + 4 grp + j % 4.
// A probability goes into that product as two bf16 numbers (its rounding and
// what that leaves), so it counts with 16 bits: the second product costs
// nothing here.
//
// 64 tokens over 60 to 8100 slots each (28 heads over 4 of 128, bf16, 516 MB):
// 99 us, 5.2 TB/s with the join (a large copy: 5.4). 9 tokens over 20000 to
// 33000 slots, e4m3 (235 MB): 53.4 us. One token over 513 slots, 14 heads over
// 2 of 64: 8.3 us, all of it waits. Every workgroup reads all sequences'
// lengths, and the line again for each tile it begins, so batches of very many
// cost more than their bytes: 256 tokens over 60 to 1000 slots (14 heads over 2
// of 64, 70 MB) 38 us, 1024 (282 MB) 153, 4096 (1.13 GB) 1095. With four
// waves, two pieces on their way instead of one: 105 us in place of 100, for
// registers.
//
// LDS: the waves' values, or 16 rows of all the waves (rows HD + 4 floats
// apart, so that they spread over the banks); then maxima and sums.
template <int HD, int W>
constexpr int kTokenShare = W * (8192 > 16 * (HD + 4) * 4 ? 8192 : 16 * (HD + 4) * 4);
template <int HD, int NR, int W>
constexpr int kTokenLds = kTokenShare<HD, W> + 2 * W * 16 * NR * 4;
template <int HD, bool E8, int NR, int W>
__device__ __forceinline__ void paged_token(const PagedKernelArgs& a, int block, char* smem) {
  using S = SlotTile<HD>;
  using K = KeySlots<HD, E8>;
  using V = std::conditional_t<E8, CodeSlots<HD>, ValueSlots<HD>>;
  constexpr int BM = 16 * NR, TK = 4096 / HD, NS = HD / 32, ND = HD / 16, KB = TK / 16;
  constexpr int kTile = TK * S::kRowBytes;  // values of a piece
  constexpr int OS = HD + 4;                // floats per row of the join
  static_assert(kTile == 8192, "values of a piece");
  auto ms = reinterpret_cast<float(*)[BM]>(smem + kTokenShare<HD, W>);  // [W][BM]
  auto ls = ms + W;
  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wg = block / a.by_Hkv, kvh = block - wg * a.pool.Hkv;
  PagedShape shapes = {};
  if (lane < a.pb.B) shapes = paged_shape(a, lane);
  const PagedFlat flat = paged_flat(a, shapes, lane);
  if (wg >= flat.wgs) return;
  int pos = flat.whole ? wg : flat.start(wg);
  const int stop = flat.whole ? wg + 1 : flat.start(wg + 1);
  const float sc = 1.4426950408889634f / sqrtf(float(HD));
  char* vt = smem + wave * kTile;
  const int tj = (lane >> 2) & 3, vrow = 4 * grp + tj, vch = (lane & 3) >> 1, vbyte = (lane & 1) * 8;
  const uint32_t vs = uint32_t(size_t((__attribute__((address_space(3))) const char*)vt)) + vrow * S::kRowBytes + vbyte;

  while (pos < stop) {
    const PagedSpot spot = paged_spot(a, shapes, flat.whole, pos, lane);
    if (spot.b < 0) return;
    const int until = min(spot.until, stop);
    const bool before = pos > spot.from, after = until < spot.until;  // shared with the last, the next workgroup
    const PagedShape& w = spot.w;
    int begin, end;
    paged_range(a, w, spot.tile, &begin, &end);
    if (!flat.whole) {
      begin = max(begin, w.lo + ((pos - spot.from) << a.unit_shift));
      end = max(min(end, w.lo + ((until - spot.from) << a.unit_shift)), begin);
    }
    pos = until;
    const int p0 = w.kv - w.n, m0 = spot.tile * BM;

    int slot_of[NR];
    bf16x8 qf[NR][NS];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      const int mc = min(m0 + 16 * r + r16, w.M - 1);
      const int tok = mc / a.by_G, g = mc - tok * a.G;
      slot_of[r] = p0 + tok;
      const uint16_t* qp =
          static_cast<const uint16_t*>(a.q) + int64_t(w.row0 + tok) * a.q_row + int64_t(kvh * a.G + g) * a.q_head;
#pragma unroll
      for (int s = 0; s < NS; ++s) qf[r][s] = *reinterpret_cast<const bf16x8*>(qp + K::dim(s, grp));
    }
    const int see_hi = p0 + m0 / a.by_G + 1, last = p0 + min(m0 + BM - 1, w.M - 1) / a.by_G;
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

    const int s0 = begin + TK * wave;
    const int nt = end > s0 ? (end - s0 + W * TK - 1) / (W * TK) : 0;
    PagedTable tab;
    tab.load(a, spot.b, begin >> a.pb.page_shift, lane);
    K kx[KB];
    V vx[KB];
    auto fetch = [&](int slot) {
#pragma unroll
      for (int i = 0; i < KB; ++i) {
        const int page = tab.at(a, spot.b, (slot + 16 * i) >> a.pb.page_shift, lane);
        kx[i].load(a, page, kvh, slot + 16 * i, end, lane);
        if constexpr (E8) vx[i].load(a.pool.v, a.pool.ve, a, page, kvh, slot + 16 * i, end, lane);
        else vx[i].load(a, page, kvh, slot + 16 * i, end, lane);
      }
    };
    if (nt > 0) fetch(s0);
    for (int t = 0; t < nt; ++t) {
      const int kb0 = s0 + W * TK * t;
      f32x4 s[NR][KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
        for (int r = 0; r < NR; ++r) s[r][kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < NS; ++st) {
          const bf16x8 kf = kx[kb].at(st);
#pragma unroll
          for (int r = 0; r < NR; ++r)
            s[r][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[r][st], s[r][kb], 0, 0, 0);
        }
      }
      // the values into LDS (this wave has read the last piece's), and the next piece's loads
#pragma unroll
      for (int i = 0; i < KB; ++i) vx[i].store(vt + 16 * i * S::kRowBytes, lane);
      if (t + 1 < nt) fetch(kb0 + W * TK);
      const bool masked = kb0 + TK > min(see_hi, end) || kb0 < see_lo;
      bf16x8 ph[NR][KB / 2], pl[NR][KB / 2];
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        if (masked) {
          const int top = min(slot_of[r], end - 1) - kb0 - 4 * grp;
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
      // products four (16 dims, 32 slots) at a time
#pragma unroll
      for (int c0 = 0; c0 < ND * KB / 2; c0 += 4) {
        uint32_t at[4];
        u32x2 v[8];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int db = (c0 + c) % ND, ks = (c0 + c) / ND;
          at[c] = vs + (((2 * db + vch) ^ S::swz(vrow)) << 4) + 32 * ks * S::kRowBytes;
        }
        lds_read_tr4x2<S::kRowBytes>(at, v);
        auto values = [&v](int c) DSF_INLINE {
          return __builtin_bit_cast(bf16x8, u32x4{v[2 * c][0], v[2 * c][1], v[2 * c + 1][0], v[2 * c + 1][1]});
        };
        // bf16 also where every row sees every slot: infinity times a weight's second part, which is 0 or below, would
        // make it NaN. Codes are finite or NaN.
        bool fix = false;
        if (!E8 || masked) {
          uint32_t odd = 0;
#pragma unroll
          for (int c = 0; c < 4; ++c) odd |= not_finite_bits(values(c));
          fix = __builtin_amdgcn_ballot_w64(odd != 0) != 0;
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int db = (c0 + c) % ND, ks = (c0 + c) / ND;
          bf16x8 vf = values(c);
          if (fix) {
#pragma unroll
            for (int r = 0; r < NR; ++r) {
              const int top = min(slot_of[r], end - 1) - kb0 - 4 * grp - 32 * ks;
              const int lo = a.window ? slot_of[r] - a.window + 1 - kb0 - 4 * grp - 32 * ks : -TK;
              bf16x8 one;
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                const int x = 16 * (j / 4) + j % 4;
                one[j] = (__bf16)(x > top || x < lo ? 0.f : 1.f);
              }
              const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
              const f32x4 n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(not_finite_codes(vf), one, zero, 0, 0, 0);
#pragma unroll
              for (int i = 0; i < 4; ++i) o[r][db][i] += not_finite_sum(n[i]);
            }
            vf = finite_or_zero(vf);
          }
#pragma unroll
          for (int r = 0; r < NR; ++r) {
            o[r][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, ph[r][ks], o[r][db], 0, 0, 0);
            o[r][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pl[r][ks], o[r][db], 0, 0, 0);
          }
        }
      }
    }

    // the waves' results, in wave order; 16 rows at a time
    float* os = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      const float l = rows4_sum(l_run[r]);
      __syncthreads();  // every wave is done with its values, or with the last 16 rows
      if (grp == 0) {
        ms[wave][16 * r + r16] = m_run[r];
        ls[wave][16 * r + r16] = l;
      }
#pragma unroll
      for (int db = 0; db < ND; ++db) *reinterpret_cast<f32x4*>(os + (wave * 16 + r16) * OS + 16 * db + 4 * grp) = o[r][db];
      __syncthreads();
      for (int e = tid; e < 16 * HD / 4; e += 64 * W) {
        const int q = e / (HD / 4), d = e % (HD / 4) * 4, m = m0 + 16 * r + q;
        if (m >= w.M) break;
        float M = -INFINITY, L = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) M = fmaxf(M, ms[i][16 * r + q]);
        f32x4 O = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < W; ++i) {
          // a wave whose slots are all hidden (maximum -inf) has zeros (NaN where a score was)
          const float mi = ms[i][16 * r + q], f = mi == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mi - M);
          L += ls[i][16 * r + q] * f;
          O += *reinterpret_cast<const f32x4*>(os + (i * 16 + q) * OS + d) * f;
        }
        if (before || after) {
          const int64_t slot = (int64_t(2 * wg + (before ? 0 : 1)) * a.pool.Hkv + kvh) * BM + 16 * r + q;
          *reinterpret_cast<f32x4*>(a.part_o + slot * HD + d) = O;
          if (d == 0) a.part_ml[slot] = make_float2(M, L);
        } else {
          const float inv = L == 0.f ? 0.f : 1.0f / L;
          const int tok = m / a.by_G, g = m - tok * a.G;
          u32x2 pk;
          pk[0] = uint32_t(f2bf(O[0] * inv)) | uint32_t(f2bf(O[1] * inv)) << 16;
          pk[1] = uint32_t(f2bf(O[2] * inv)) | uint32_t(f2bf(O[3] * inv)) << 16;
          *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + int64_t(w.row0 + tok) * a.o_row +
                                    int64_t(kvh * a.G + g) * a.o_head + d) = pk;
        }
      }
    }
    __syncthreads();  // the next tile's values go where these were
  }
}

// --------------------------------------------------------------- kernels

template <int HD, bool E8>
__global__ __launch_bounds__(256, 2) void paged_chunk_kernel(PagedKernelArgs a) {
  __shared__ __attribute__((aligned(16))) char smem[kChunkLds<HD, E8>];
  paged_chunk<HD, E8>(a, blockIdx.x, smem);
}
template <int HD, bool E8, int NR, int W>
__global__ __launch_bounds__(64 * W) void paged_token_kernel(PagedKernelArgs a) {
  __shared__ __attribute__((aligned(16))) char smem[kTokenLds<HD, NR, W>];
  paged_token<HD, E8, NR, W>(a, blockIdx.x, smem);
}
// Both, for batches that may have either: the chunks' workgroups first (their
// work is longer), the tokens' where those leave places, which chunks cut for
// the whole chip do only as they end. 24 sequences, six of them with chunks of
// 158 to 616 tokens (14 heads over 2 of 64, e4m3): 55.4 us (as two launches
// 72.2, where one took 57.7); five chunks with a window 55.9 (58.6 and 55.5);
// two long chunks the same either way. What bounds the first is its longest
// items (26 turns of 64 slots at 1.5 us, the average is 18) after 5.5 us to the
// first scores.
template <int HD, bool E8>
__global__ __launch_bounds__(256, 2) void paged_mixed_kernel(PagedKernelArgs chunks, PagedKernelArgs tokens) {
  constexpr int kLds = kChunkLds<HD, E8> > kTokenLds<HD, 1, 4> ? kChunkLds<HD, E8> : kTokenLds<HD, 1, 4>;
  __shared__ __attribute__((aligned(16))) char smem[kLds];
  const int first = chunks.items * chunks.pool.Hkv;
  if (int(blockIdx.x) < first) paged_chunk<HD, E8>(chunks, blockIdx.x, smem);
  else paged_token<HD, E8, 1, 4>(tokens, int(blockIdx.x) - first, smem);
}

// -------------------------------------------------------------------- fp32

// fp32 on the fp32 matrix cores: a workgroup takes 16 rows, its four waves
// every fourth piece of 32 slots, each with a softmax of its own, joined
// through LDS in wave order. Rows and slots are the two operands' rows, 16
// bytes of a row per lane, element e of the vectors forming one 4-deep
// product; the probabilities go through a per-wave LDS tile into the A
// operand of P V, whose B operand is HD / 16 neighbouring dims of slot
// 4 s + grp as they come from memory. Loads of the next piece during this
// one's product cost more in registers than they hid (21.0 -> 24.1 us): other
// waves hide them. Two chunks of 77 to 200 tokens over 350 to 1000 slots, 12
// heads of 64 (0.39 GFLOP): 21.5 us, the kernel 17; at head dim 128 47 us. 900
// over 3900 slots and 500 over 2000 (12.2 GFLOP): 213 us, 57 TFLOP/s, 229 from
// e4m3 pages. 16 tokens over 500 to 6000 slots, 12 heads over 2 of 128: 33.1
// us (91 MB), from e4m3 29.5 (23 MB).
template <int HD, bool E8>
__global__ __launch_bounds__(256) void paged_f32_kernel(PagedKernelArgs a) {
  constexpr int NK = HD / 16, DPL = HD / 16, KV = 32;
  __shared__ float ps[4][16][KV + 4];
  __shared__ float osum[4][16][HD];
  __shared__ float ms[4][16], ls[4][16];
  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, grp = lane >> 4;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int item = int(blockIdx.x) / a.by_Hkv, kvh = int(blockIdx.x) - item * a.pool.Hkv;
  const PagedItem it = paged_item(a, item, lane);
  if (it.b < 0) return;
  const PagedWork w = paged_work(a, it);
  if (w.splits > 1 && w.begin >= w.end) return;
  const int m0 = w.tile * 16;
  f32x4 qf[NK];
  {
    const int mc = min(m0 + r16, w.M - 1), tok = mc / a.by_G, g = mc - tok * a.G;
    const float* qp = static_cast<const float*>(a.q) + int64_t(w.row0 + tok) * a.q_row + int64_t(kvh * a.G + g) * a.q_head;
#pragma unroll
    for (int s = 0; s < NK; ++s) qf[s] = *reinterpret_cast<const f32x4*>(qp + 16 * s + 4 * grp);
  }
  int slot_of[4];  // of rows m0 + 4 grp + i
#pragma unroll
  for (int i = 0; i < 4; ++i) slot_of[i] = w.p0 + min(m0 + 4 * grp + i, w.M - 1) / a.by_G;
  const int see_hi = w.p0 + m0 / a.by_G + 1;
  const int see_lo = a.window ? w.p0 + min(m0 + 15, w.M - 1) / a.by_G - a.window + 1 : 0;
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
        float v[DPL];
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
        const bool mine = key0 + 16 * kb + 4 * s + grp < w.end;
#pragma unroll
        for (int e = 0; e < DPL; ++e) vf[4 * kb + s][e] = mine ? v[e] : 0.f;
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
#pragma unroll 1
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int s = 0; s < KV / 4; ++s) {
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
      const int tok = mr / a.by_G, g = mr - tok * a.G;
      static_cast<float*>(a.out)[int64_t(w.row0 + tok) * a.o_row + int64_t(kvh * a.G + g) * a.o_head + d] =
          L == 0.f ? 0.f : O / L;
    }
  }
}

// ---------------------------------------------------- joining the shares

// Shares 0 .. n - 1 of a row of a tile, in their order, eight of them on the
// way at a time, with a running maximum. Share i lies at place
// i ? at1 + i * step : at0 of the workspace. The maxima are in log2 units for
// bf16, natural ones for fp32.
template <int HD, typename T>
__device__ __forceinline__ void paged_join_row(const PagedKernelArgs& a, int64_t at0, int64_t at1, int64_t step, int n,
                                               int d, T* op) {
  constexpr bool LOG2 = sizeof(T) == 2;
  constexpr int U = 8;
  float M = -INFINITY, L = 0.f;
  f32x4 O = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = 0; i0 < n; i0 += U) {
    float2 x[U];
    f32x4 v[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int i = min(i0 + j, n - 1);
      const int64_t at = i ? at1 + i * step : at0;
      x[j] = a.part_ml[at];
      v[j] = *reinterpret_cast<const f32x4*>(a.part_o + at * HD + d);
    }
    float mx = M;
#pragma unroll
    for (int j = 0; j < U; ++j) mx = fmaxf(mx, x[j].x);
    // a share that saw nothing has zeros (NaN where a score was), as has the start
    auto factor = [mx](float m) { return m == -INFINITY ? 1.f : LOG2 ? __builtin_amdgcn_exp2f(m - mx) : expf(m - mx); };
    const float f0 = factor(M);
    O *= f0;
    L *= f0;
#pragma unroll
    for (int j = 0; j < U; ++j)
      if (i0 + j < n) {
        const float f = factor(x[j].x);
        O += v[j] * f;
        L += x[j].y * f;
      }
    M = mx;
  }
  const float inv = L == 0.f ? 0.f : 1.0f / L;
  if constexpr (sizeof(T) == 2) {
    u32x2 pk;
    pk[0] = uint32_t(f2bf(O[0] * inv)) | uint32_t(f2bf(O[1] * inv)) << 16;
    pk[1] = uint32_t(f2bf(O[2] * inv)) | uint32_t(f2bf(O[3] * inv)) << 16;
    *reinterpret_cast<u32x2*>(op) = pk;
  } else {
    *reinterpret_cast<f32x4*>(op) = O * inv;
  }
}

// A workgroup takes kJoinRows rows of one tile and kv head at a time, a
// thread four dims of a row, and goes on to every blocks-th such part. Tiles
// that one workgroup had to itself are done already. FLAT: shares of the
// line, else splits. Four to ten us, half of it until the first share is there
// (four or sixteen of them on the way instead of eight: within 1 us); 1024
// workgroups: two chunks of 900 tokens 35.4 us, with 512 38.3, with 4096 35.7,
// but then the mixed batch 59.7 for 56.9, by workgroups without work.
constexpr int kJoinRows = 16;
constexpr int kJoinBlocks = 1024;
template <int HD, typename T, bool FLAT>
__device__ __forceinline__ void paged_join(const PagedKernelArgs& a, int block, int blocks) {
  const int tid = threadIdx.x, lane = tid & 63;
  PagedShape w0 = {};
  if (lane < a.pb.B) w0 = paged_shape(a, lane);
  PagedFlat flat = {};
  int per = 0;
  if constexpr (FLAT) {
    flat = paged_flat(a, w0, lane);
    if (flat.whole) return;
  } else {
    per = paged_split_blocks(a, w0, lane);
    // no sequence is split
    if (a.pb.B <= 64 && !__builtin_amdgcn_ballot_w64(w0.tiles > 0 && paged_splits(w0, per) > 1)) return;
  }
  const int parts = (1 << a.bm_shift) / kJoinRows;
  for (int unit = block;; unit += blocks) {
    int tile = unit / parts / a.by_Hkv;
    const int part = unit % parts, kvh = unit / parts - tile * a.pool.Hkv;
    // the sequence that has the tile, and where its items (FLAT: units) begin
    PagedShape w = w0, s = {};
    int first = 0, b = -1, each = 0;
    for (int b0 = 0; b0 < a.pb.B; b0 += 64) {
      if (b0) {
        w = PagedShape{};
        if (b0 + lane < a.pb.B) w = paged_shape(a, b0 + lane);
      }
      const int n = FLAT ? paged_units(a, w) : paged_splits(w, per);
      const int c = FLAT ? w.tiles * n : min(w.tiles * n, a.items);
      const int tend = wave_prefix(w.tiles), end = wave_prefix(c);
      const uint64_t over = __builtin_amdgcn_ballot_w64(tend > tile);
      if (over) {
        const int l = __builtin_ctzll(over);
        b = b0 + l;
        s = shape_of(w, l);
        each = __builtin_amdgcn_readlane(n, l);
        tile -= __builtin_amdgcn_readlane(tend, l) - __builtin_amdgcn_readlane(w.tiles, l);
        first += __builtin_amdgcn_readlane(end, l) - __builtin_amdgcn_readlane(c, l);
        break;
      }
      tile -= __builtin_amdgcn_readlane(tend, 63);
      first += __builtin_amdgcn_readlane(end, 63);
      if (!FLAT) first = min(first, a.items);
    }
    if (b < 0) return;  // past the last tile
    int n;
    int64_t at0, at1, step;  // places, in tiles
    if constexpr (FLAT) {
      const int j0 = flat.of(first + tile * each), j1 = flat.of(first + tile * each + each - 1);
      n = j1 - j0 + 1;
      if (n <= 1 || j0 < 0 || j1 >= a.items) continue;
      at0 = int64_t(2 * j0 + 1) * a.pool.Hkv + kvh;
      at1 = int64_t(2 * j0) * a.pool.Hkv + kvh;
      step = 2 * a.pool.Hkv;
    } else {
      if (each == 1) continue;
      int begin, stop;
      paged_range(a, s, tile, &begin, &stop);
      const int len = paged_split_len(begin, stop, each);
      n = len ? (stop - begin + len - 1) / len : 0;
      const int item = first + (s.tiles - 1 - tile);
      // tables that claim more items than the launch has (row_start not ascending) end here
      if (item < 0 || item + int64_t(max(n - 1, 0)) * s.tiles >= a.items) continue;
      at0 = at1 = int64_t(item) * a.pool.Hkv + kvh;
      step = int64_t(s.tiles) * a.pool.Hkv;
    }
    for (int e = tid; e < kJoinRows * (HD / 4); e += 256) {
      const int row = part * kJoinRows + e / (HD / 4), d = e % (HD / 4) * 4, m = (tile << a.bm_shift) + row;
      if (m >= s.M) break;
      const int tok = m / a.by_G, g = m - tok * a.G;
      paged_join_row<HD, T>(a, (at0 << a.bm_shift) + row, (at1 << a.bm_shift) + row, step << a.bm_shift, n, d,
                            static_cast<T*>(a.out) + int64_t(s.row0 + tok) * a.o_row + int64_t(kvh * a.G + g) * a.o_head + d);
    }
  }
}

template <int HD, typename T, bool FLAT>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedKernelArgs a) {
  paged_join<HD, T, FLAT>(a, blockIdx.x, gridDim.x);
}
// The chunks' tiles by `first` workgroups, the tokens' by the others.
template <int HD>
__global__ __launch_bounds__(256) void paged_mixed_join_kernel(PagedKernelArgs chunks, PagedKernelArgs tokens, int first) {
  if (int(blockIdx.x) < first) paged_join<HD, uint16_t, false>(chunks, blockIdx.x, first);
  else paged_join<HD, uint16_t, true>(tokens, int(blockIdx.x) - first, int(gridDim.x) - first);
}

// ------------------------------------------------------------------ launch

namespace {

// One launch over the sequences of m_lo < rows * G <= m_hi.
struct PagedPlan {
  bool on;
  int bm_shift, m_lo, m_hi;
  int items;       // workgroups per kv head, at most
  int tiles;       // of rows, the same
  int target;      // splits: items aimed at (0: none)
  int unit_shift;
  bool join;       // whether tiles may have shares
  size_t places;   // of shares, per kv head
};

// Workgroups aimed at with splits, of all kv heads: two to a CU. A chunk of
// 512 over 8192 slots took 45.5 us (256: 46.6, 1024: 60.2), the mixed batch
// 57 (59.2, 58.5), a window 55.5 (55.5, 78.5), each in one comparison.
constexpr int kChunkItems = 512;
// fp32: three to a CU. Short chunks 20.9 us (512: 22.1, 1536: 20.9), 500 to
// 900 tokens over 2000 to 4000 slots 314.5 (314.1, 317.4).
constexpr int kF32Items = 768;
// 256 slots. A chunk of 256 over 2048 slots takes 20.9 us (128 slots: 24.3,
// 512: 23.7), short ones in fp32 20.9 (22.4, 22.2).
constexpr int kSplitMinBlocks = 4;
// What a split's way through memory and the join cost, in a chunk's turns: two
// chunks of 900 tokens on their own context take 27.9 us, with 4 (so that they
// are split) 35.7; two of 300 over 1000 slots 24.1, with 12 (so that they are
// not) 29.9. fp32 turns are longer: short chunks 20.9 with 0, 26.6 with 8.
constexpr int kSplitGain = 8;

size_t align256(size_t n) { return (n + 255) & ~size_t(255); }

PagedPlan tiles_plan(const PagedBatch& pb, int G, int bm_shift, int m_lo, int m_hi) {
  PagedPlan p = {};
  p.on = true;
  p.bm_shift = bm_shift;
  p.m_lo = m_lo;
  p.m_hi = m_hi;
  p.unit_shift = 6;
  // tiles: full ones, and a part of one per sequence that takes part
  const int64_t rows = int64_t(pb.n_rows) * G;
  const int64_t seqs = std::min<int64_t>(std::min(pb.B, pb.n_rows), rows / (m_lo + 1));
  int64_t tiles = (rows >> bm_shift) + seqs;
  if (m_hi < 1 << 20) tiles = std::min<int64_t>(tiles, seqs * (((m_hi - 1) >> bm_shift) + 1));
  p.tiles = int(tiles);
  return p;
}

PagedPlan split_plan(const PagedBatch& pb, int G, int Hkv, int bm_shift, int m_lo, int m_hi, int total) {
  PagedPlan p = tiles_plan(pb, G, bm_shift, m_lo, m_hi);
  const int64_t blocks = (int64_t(pb.max_pages) << pb.page_shift) / 64;
  // (with two rounds of tiles and more nothing is split: the last round is a small part then, and 4 chunks of 500 to 900
  // tokens over 3000 to 9000 slots, 1.1 rounds, are split and take 104 us. Tiles are counted by n_rows, so a captured
  // step should not have room for many more rows than it brings: a chunk of 512 over 8192 slots, 44 us, takes 146 in a
  // batch with room for 11000)
  if (blocks > kSplitMinBlocks && p.tiles <= 4096 && int64_t(p.tiles) * Hkv < 2 * total) p.target = std::max(total / Hkv, 1);
  p.items = p.tiles + p.target;
  p.join = p.target != 0;
  p.places = p.join ? p.items : 0;
  return p;
}

// per_cu: workgroups to a CU, for one round of equal shares: eight waves of 16
// rows (comment at paged_token), or four of more rows, fill it; beside chunks 16
// rows have four, two to a CU. One to a CU there: 9 tokens over long e4m3
// sequences in a batch with room for chunks 83.2 us for 57.5, 64 bf16 tokens
// 137 for 102; with a chunk of 512 over 4096 slots 129 for 110 and 188 for 164.
// (32 sequences of 14 rows with a chunk of 256: 25.4 for 26.4.)
PagedPlan flat_plan(const PagedBatch& pb, int G, int Hkv, int bm_shift, int m_hi, int per_cu) {
  PagedPlan p = tiles_plan(pb, G, bm_shift, 0, m_hi);
  p.items = std::max(256 * per_cu / Hkv, 1);
  const int64_t slots = int64_t(pb.max_pages) << pb.page_shift;
  // (row_start that does not ascend may claim all tiles of every sequence)
  const int64_t most = int64_t(pb.B) * (((m_hi - 1) >> bm_shift) + 1);
  while (most * ((slots >> p.unit_shift) + 1) > int64_t(1) << 30) ++p.unit_shift;
  p.join = slots > kWholeUnits << 6 || most > p.items;
  p.places = p.join ? 2 * size_t(p.items) : 0;
  return p;
}

// The launches of a call: [0] sequences of few rows, [1] the others.
void paged_plans(int dtype, int Hq, const PagedPool& pool, const PagedBatch& pb, PagedPlan (&p)[2]) {
  const int G = Hq / pool.Hkv;
  p[0] = p[1] = PagedPlan{};
  if (dtype == DSF_F32) {
    p[1] = split_plan(pb, G, pool.Hkv, 4, 0, 0x7fffffff, kF32Items);
    return;
  }
  const int64_t most = int64_t(std::min(pb.max_rows, pb.n_rows)) * G;
  // sequences of one token stay with the token kernel beside ones with chunks
  const int few = most <= kTokenRows ? int(most) : std::min((G + 15) / 16 * 16, kTokenRows);
  const int shift = few <= 16 ? 4 : few <= 32 ? 5 : 6;
  if (most <= kTokenRows || pb.B > 1) p[0] = flat_plan(pb, G, pool.Hkv, shift, few, most > kTokenRows && shift == 4 ? 2 : 1);
  if (most > kTokenRows) p[1] = split_plan(pb, G, pool.Hkv, 7, pb.B > 1 ? few : 0, 0x7fffffff, kChunkItems);
}

size_t plan_rows(const PagedPlan& p, int Hkv) { return p.places * Hkv << p.bm_shift; }
size_t plan_bytes(const PagedPlan& p, const PagedPool& pool) {
  const size_t rows = plan_rows(p, pool.Hkv);
  return align256(rows * pool.hd * 4) + align256(rows * 8);
}

}  // namespace

size_t paged_attention_workspace_bytes(int dtype, int Hq, const PagedPool& pool, const PagedBatch& pb) {
  PagedPlan p[2];
  paged_plans(dtype, Hq, pool, pb, p);
  return std::max<size_t>(plan_bytes(p[0], pool) + plan_bytes(p[1], pool), 256);
}

hipError_t launch_paged_attention(const PagedAttnArgs& a, hipStream_t s) {
  if (a.pb.B == 0 || a.pb.n_rows == 0 || a.pb.max_rows == 0) return hipSuccess;
  TimedScope ts(DSF_KIND_ATTN, s);
  PagedPlan p[2];
  paged_plans(a.dtype, a.Hq, a.pool, a.pb, p);
  char* ws = static_cast<char*>(a.workspace);
  PagedKernelArgs k[2];
  unsigned grid[2] = {}, joins[2] = {};
  for (int i = 0; i < 2; ++i) {
    if (!p[i].on) continue;
    k[i].pool = a.pool;
    k[i].pb = a.pb;
    k[i].q = a.q;
    k[i].q_row = a.q_row;
    k[i].q_head = a.q_head;
    k[i].out = a.out;
    k[i].o_row = a.o_row;
    k[i].o_head = a.o_head;
    k[i].G = a.Hq / a.pool.Hkv;
    k[i].by_G = divisor(k[i].G);
    k[i].by_Hkv = divisor(a.pool.Hkv);
    k[i].window = a.window;
    k[i].bm_shift = p[i].bm_shift;
    k[i].m_lo = p[i].m_lo;
    k[i].m_hi = p[i].m_hi;
    k[i].items = p[i].items;
    k[i].target = p[i].target;
    k[i].split_min = kSplitMinBlocks;
    k[i].split_gain = a.dtype == DSF_F32 ? 0 : kSplitGain;
    k[i].unit_shift = p[i].unit_shift;
    k[i].part_o = reinterpret_cast<float*>(ws);
    k[i].part_ml = reinterpret_cast<float2*>(ws + align256(plan_rows(p[i], a.pool.Hkv) * a.pool.hd * 4));
    ws += plan_bytes(p[i], a.pool);
    grid[i] = unsigned(p[i].items) * a.pool.Hkv;
    const int64_t parts = int64_t(p[i].tiles) * a.pool.Hkv * ((1 << p[i].bm_shift) / kJoinRows);
    joins[i] = p[i].join ? unsigned(std::min<int64_t>(parts, kJoinBlocks)) : 0;
  }
  auto run = [&](auto hdc, auto e8c) -> hipError_t {
    constexpr int HD = decltype(hdc)::value;
    constexpr bool E8 = decltype(e8c)::value;
    if (a.dtype == DSF_F32) {
      paged_f32_kernel<HD, E8><<<grid[1], 256, 0, s>>>(k[1]);
      if (joins[1]) paged_join_kernel<HD, float, false><<<joins[1], 256, 0, s>>>(k[1]);
      return hipGetLastError();
    }
    if (p[0].on && p[1].on && p[0].bm_shift == 4) {
      paged_mixed_kernel<HD, E8><<<grid[0] + grid[1], 256, 0, s>>>(k[1], k[0]);
      if (joins[0] + joins[1]) paged_mixed_join_kernel<HD><<<joins[0] + joins[1], 256, 0, s>>>(k[1], k[0], int(joins[1]));
      return hipGetLastError();
    }
    if (p[1].on) {
      paged_chunk_kernel<HD, E8><<<grid[1], 256, 0, s>>>(k[1]);
      if (joins[1]) paged_join_kernel<HD, uint16_t, false><<<joins[1], 256, 0, s>>>(k[1]);
    }
    if (p[0].on) {
      if (p[0].bm_shift == 4) paged_token_kernel<HD, E8, 1, 8><<<grid[0], 512, 0, s>>>(k[0]);
      else if (p[0].bm_shift == 5) paged_token_kernel<HD, E8, 2, 4><<<grid[0], 256, 0, s>>>(k[0]);
      else paged_token_kernel<HD, E8, 4, 4><<<grid[0], 256, 0, s>>>(k[0]);
      if (joins[0]) paged_join_kernel<HD, uint16_t, true><<<joins[0], 256, 0, s>>>(k[0]);
    }
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
  return a.pool.codes ? run_h(std::true_type()) : run_h(std::false_type());
}

}  // namespace dsf
