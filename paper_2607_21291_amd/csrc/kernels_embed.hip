// Embedding lookup with scaling, and its gradient by sorted tokens.
//
// The gradient's row of a token sums the rows of dy where it stands, in fp32
// and in the order of the positions, without atomics: embed_order_kernel sorts
// the positions by token, embed_sum_kernel sums each token's. Sequences of one
// token that are longer than kLong positions are cut into pieces of the sorted
// list (kLong positions each, wherever tokens begin and end), whose sums
// embed_join_kernel adds in order and in 64 bits: text's commonest tokens take several percent
// of a batch, padding most of it.
//
// Memory bounds both. Lookup: 20000 rows of width 2048 21 us, 7.6 TB/s with what the
// caches hold of common rows. Gradient: 16384 positions, table 151936 x 896, bf16: sort
// and zero rows 50 us (245 MB, 4.9 TB/s), sums 15, join 5; of 6001 positions added to
// a table of 50304 x 768 in fp32 20 us, three chains of dependent loads; 40000 positions
// of one token 221 us, 115 of them the join (a wave to 512 columns).
#include <algorithm>

#include "dsf_device.h"
#include "dsf_internal.h"

namespace dsf {

namespace {
constexpr int kRange = 256;  // table rows of a workgroup of the sort
constexpr int kWaves = 16;
constexpr int kLong = 32;  // (16384 positions of text over 151936 tokens: 16 68.0 us, 32 66.8)
}  // namespace

// out[i] = scale * table[tokens[i]], zeros for a token outside [0, V). A
// workgroup takes 1024 consecutive 16-byte vectors of out.
template <typename T>
__global__ __launch_bounds__(256) void embed_kernel(const int32_t* __restrict__ tokens, const T* __restrict__ table,
                                                    int n, int V, int d, float scale, T* __restrict__ out) {
  constexpr int VEC = Elem<T>::kVec;
  const uint32_t nv = uint32_t(d) / VEC;
  const int64_t base = wide_index() * 1024, all = int64_t(n) * nv;
  const int64_t row0 = base / nv;
  const uint32_t rem = uint32_t(base - row0 * nv);
  u32x4 raw[4];
  int64_t at[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const uint32_t o = rem + threadIdx.x + 256 * u;
    const uint32_t r = o / nv, c = o - r * nv;
    at[u] = base + threadIdx.x + 256 * u;
    raw[u] = u32x4{0, 0, 0, 0};
    if (at[u] >= all) continue;
    const int t = tokens[row0 + r];
    if (uint32_t(t) < uint32_t(V)) raw[u] = reinterpret_cast<const u32x4*>(table + int64_t(t) * d)[c];
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    if (at[u] >= all) continue;
    if (scale != 1.f) {
      float v[VEC];
      load_vec(reinterpret_cast<const T*>(&raw[u]), v);
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[i] *= scale;
      store_vec(reinterpret_cast<T*>(&raw[u]), v);
    }
    reinterpret_cast<u32x4*>(out)[at[u]] = raw[u];
  }
}

// Positions sorted by token (order, and the tokens in key), those of one token
// ascending (and, for a gradient written whole, the rows of absent tokens: zeros,
// `row_vecs` vectors of 16 bytes); start[v] = number of positions whose token is
// in [0, v). A workgroup sorts the positions of
// kRange tokens: it reads all tokens twice (they stay in L2), counts those
// before its range, and each wave places the positions of its stretch, 64 at
// a time, ranked among equals by ballots over the bits of the token.
__global__ __launch_bounds__(64 * kWaves) void embed_order_kernel(const int32_t* __restrict__ tokens, int n, int V,
                                                                  int32_t* __restrict__ order,
                                                                  int32_t* __restrict__ key,
                                                                  int32_t* __restrict__ start,
                                                                  u32x4* __restrict__ out, int row_vecs) {
  __shared__ int hist[kWaves][kRange];
  __shared__ int part[kWaves];
  __shared__ uint64_t absent[kRange / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t lo = wide_index() * kRange;
  if (lo >= V) return;
  const int size = int(std::min<int64_t>(kRange, V - lo));
  const int seg = ((n + kWaves - 1) / kWaves + 63) / 64 * 64;
  const int b = std::min(int64_t(n), int64_t(wave) * seg), e = std::min(int64_t(n), int64_t(b) + seg);
  for (int i = tid; i < kWaves * kRange; i += 64 * kWaves) (&hist[0][0])[i] = 0;
  __syncthreads();
  int less = 0;
  for (int i = b; i < e; i += 512) {
    int t[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) t[u] = i + 64 * u + lane < e ? tokens[i + 64 * u + lane] : -1;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int64_t r = int64_t(t[u]) - lo;
      less += t[u] >= 0 && r < 0;
      if (r >= 0 && r < size) atomicAdd(&hist[wave][r], 1);
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) less += __shfl_xor(less, o, 64);
  if (lane == 0) part[wave] = less;
  __syncthreads();
  int base = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) base += part[w];
  // exclusive sums over the range's tokens, then over the waves of a token
  int c[kWaves], all = 0;
  if (tid < kRange) {
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      c[w] = hist[w][tid];
      all += c[w];
    }
  }
  int incl = all;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(incl, o, 64);
    if (lane >= o) incl += v;
  }
  __syncthreads();
  if (lane == 63) part[wave] = incl;
  __syncthreads();
  if (tid < kRange) {
    const uint64_t none = __ballot(tid < size && all == 0);
    if (lane == 0) absent[wave] = none;
    int at = base + incl - all;
    for (int w = 0; w < wave; ++w) at += part[w];
    if (tid < size) start[lo + tid] = at;
    if (lo + tid == V - 1) start[V] = at + all;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      hist[w][tid] = at;
      at += c[w];
    }
  }
  __syncthreads();
  for (int i = b; i < e; i += 512) {
    int t[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) t[u] = i + 64 * u + lane < e ? tokens[i + 64 * u + lane] : -1;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int64_t r64 = int64_t(t[u]) - lo;
      const bool in = r64 >= 0 && r64 < size;
      uint64_t same = __ballot(in);
      if (same == 0) continue;
      const int r = in ? int(r64) : 0;
#pragma unroll
      for (int bit = 0; bit < 8; ++bit) {
        const uint64_t m = __ballot((r >> bit) & 1);
        same &= (r >> bit) & 1 ? m : ~m;
      }
      if (in) {
        const int rank = __popcll(same & ((uint64_t(1) << lane) - 1));
        const int at = hist[wave][r];
        order[at + rank] = i + 64 * u + lane;
        key[at + rank] = t[u];
        if (rank == 0) hist[wave][r] = at + __popcll(same);
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
  if (!out) return;
  constexpr int kRows = kRange / kWaves;
  uint32_t rows = uint32_t(absent[wave * kRows / 64] >> (wave * kRows % 64)) & ((1u << kRows) - 1u);
  u32x4* p = out + (lo + wave * kRows) * row_vecs;
  for (; rows; rows >>= 1, p += row_vecs)
    if (rows & 1)
      for (int c = lane; c < row_vecs; c += 64) p[c] = u32x4{0, 0, 0, 0};
}

struct EmbedSumArgs {
  const int32_t* order; const int32_t* key; const int32_t* start;
  const void* dy; void* out;
  float* part;  // [pieces][2][d]: sums of a piece's positions for the token it goes on with, and for the one it begins
  int n, V, d, accumulate;
  float scale;
  int long_wgs, slabs;
};

constexpr int kSlab = 512;  // columns a wave sums at a time (8 a lane)

template <typename TO>
__device__ __forceinline__ void embed_store(TO* p, const float* v, float scale, bool add) {
  float o[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] = 0.f;
  if (add) load8(p, o);
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] += v[i] * scale;
  store8(p, o);
}

// v = columns c .. c + 7 summed over the rows pos[first .. first + count) of dy, pos
// lane by lane. Called by whole waves: a row's number comes from another lane,
// which must be running; `in` (c < d) covers the loads alone.
template <typename TI>
__device__ __forceinline__ void embed_rows(const TI* dy, int d, int pos, int first, int count, int c, bool in, float* v) {
  constexpr int U = 8;  // rows in flight
  const int end = first + count;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = 0.f;
  for (int j = first; j < end; j += U) {
    int64_t at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) at[u] = int64_t(__builtin_amdgcn_readlane(pos, std::min(j + u, end - 1))) * d;
    if (in) {
      Raw8<TI> x[U];
      // (past the end the last row again, which is not added)
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (u < 2 || j + u < end) x[u] = load_raw8(dy + at[u] + c);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (j + u < end) {
          float f[8];
          unpack8(x[u], f);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] += f[e];
        }
    }
  }
}

// Workgroups [0, long_wgs): a wave to a piece and slab, the sums of tokens of more
// than kLong positions. The others: a wave to a slab and a sorted place that begins
// a token of fewer.
template <typename TI, typename TO>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedSumArgs a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6));
  const TI* dy = (const TI*)a.dy;
  TO* out = (TO*)a.out;
  const int n = a.start[a.V];  // positions that have a token (from there on order and key hold nothing)
  const int64_t wg = wide_index();
  if (wg < a.long_wgs) {
    const int task = int(wg) * 4 + wave, piece = task / a.slabs, c = (task - piece * a.slabs) * kSlab + lane * 8;
    const int i0 = piece * kLong;
    if (i0 >= n) return;
    const int m = std::min(kLong, n - i0);
    const int pos = a.order[i0 + std::min(lane, m - 1)];
    const int t = a.key[i0 + std::min(lane, m - 1)];
    const int s = a.start[t];
    const bool is_long = a.start[t + 1] - s > kLong;
    // lanes of the long token that began before the piece, and of one that begins in it
    const uint64_t in[2] = {__ballot(lane < m && is_long && s < i0), __ballot(lane < m && is_long && s >= i0)};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (in[k] == 0) continue;
      float v[8];
      embed_rows(dy, a.d, pos, __builtin_ctzll(in[k]), __popcll(in[k]), c, c < a.d, v);  // consecutive lanes
      if (c < a.d) store8(a.part + (int64_t(piece) * 2 + k) * a.d + c, v);
    }
    return;
  }
  const int64_t task = (wg - a.long_wgs) * 4 + wave;
  const int i = int(task / a.slabs), c = int(task - int64_t(i) * a.slabs) * kSlab + lane * 8;
  // the places from i - 1 on, a lane to each: the token's are those from i to the next other's
  // (read beside n, not after it)
  const int here = a.key[std::max(0, std::min(i - 1 + lane, a.n - 1))], pos = a.order[std::min(i + lane, a.n - 1)];
  if (i >= n) return;
  const int last = std::min(i + kLong, n - 1);
  const int t = __builtin_amdgcn_readlane(here, 1);
  const int m = __popcll(__ballot(here == t && lane >= 1 && i - 1 + lane <= last));
  if ((i > 0 && __builtin_amdgcn_readfirstlane(here) == t) || m > kLong) return;
  float v[8];
  embed_rows(dy, a.d, pos, 0, m, c, c < a.d, v);
  if (c < a.d) embed_store(out + int64_t(t) * a.d + c, v, a.scale, a.accumulate);
}

// The rows of tokens of more than kLong positions: a wave to the piece that a
// token begins in, and a slab. The pieces' sums are added by eights, and these in 64 bits: a
// token may have 2^25 pieces, and equal ones round the same way (2^17 of 3.2 in fp32: 0.2 %
// off). (Each in 64 bits: 40000 positions of one token 240 us; so 221.)
template <typename TO>
__global__ __launch_bounds__(256) void embed_join_kernel(EmbedSumArgs a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6));
  const int task = int(wide_index()) * 4 + wave, piece = task / a.slabs;
  const int c = (task - piece * a.slabs) * kSlab + lane * 8;
  const int n = a.start[a.V], i0 = piece * kLong;
  if (i0 >= n) return;
  const int m = std::min(kLong, n - i0);
  const int t = a.key[i0 + std::min(lane, m - 1)];
  const int s = a.start[t], e1 = a.start[t + 1];
  const uint64_t begins = __ballot(lane < m && e1 - s > kLong && s >= i0);
  if (begins == 0) return;
  const int src = __builtin_ctzll(begins);  // one such token at most fits a piece
  const int tok = __builtin_amdgcn_readlane(t, src), end = __builtin_amdgcn_readlane(e1, src);
  if (c >= a.d) return;
  float v[8];
  double sum[8];
  load8(a.part + (int64_t(piece) * 2 + 1) * a.d + c, v);
#pragma unroll
  for (int e = 0; e < 8; ++e) sum[e] = v[e];
  const int last = (end - 1) / kLong;
  for (int p = piece + 1; p <= last; p += 8) {
    float x[8][8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[u][e] = 0.f;
      if (p + u <= last) load8(a.part + int64_t(p + u) * 2 * a.d + c, x[u]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
      sum[e] += double(((x[0][e] + x[1][e]) + (x[2][e] + x[3][e])) + ((x[4][e] + x[5][e]) + (x[6][e] + x[7][e])));
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = float(sum[e]);
  embed_store((TO*)a.out + int64_t(tok) * a.d + c, v, a.scale, a.accumulate);
}

hipError_t launch_embed(int dtype, const int32_t* tokens, const void* table, int n, int V, int d, float scale, void* out,
                        hipStream_t s) {
  const int64_t nv = int64_t(n) * d / (dtype == DSF_F32 ? 4 : 8);
  const dim3 grid = wide_grid((nv + 1023) / 1024);
  if (dtype == DSF_F32)
    embed_kernel<float><<<grid, 256, 0, s>>>(tokens, (const float*)table, n, V, d, scale, (float*)out);
  else
    embed_kernel<uint16_t><<<grid, 256, 0, s>>>(tokens, (const uint16_t*)table, n, V, d, scale, (uint16_t*)out);
  return hipGetLastError();
}

static size_t up256b(size_t v) { return (v + 255) & ~size_t(255); }

size_t embed_backward_workspace_bytes(int n, int d, int V) {
  const size_t pieces = n > kLong ? size_t(n + kLong - 1) / kLong : 0;
  return 2 * up256b(size_t(n) * 4) + up256b((size_t(V) + 1) * 4) + up256b(pieces * 2 * d * 4);
}

hipError_t launch_embed_backward(const EmbedBackwardArgs& b, hipStream_t s) {
  char* ws = (char*)b.workspace;
  EmbedSumArgs a{};
  int32_t* order = (int32_t*)ws;
  int32_t* key = (int32_t*)(ws + up256b(size_t(b.n) * 4));
  int32_t* start = (int32_t*)(ws + 2 * up256b(size_t(b.n) * 4));
  a.part = (float*)(ws + 2 * up256b(size_t(b.n) * 4) + up256b((size_t(b.V) + 1) * 4));
  a.key = key;
  a.order = order;
  a.start = start;
  a.dy = b.dy;
  a.out = b.dtable;
  a.n = b.n;
  a.V = b.V;
  a.d = b.d;
  a.accumulate = b.accumulate;
  a.scale = b.scale;
  a.slabs = (b.d + kSlab - 1) / kSlab;
  const int64_t tasks = b.n > kLong ? int64_t((b.n + kLong - 1) / kLong) * a.slabs : 0;
  a.long_wgs = int((tasks + 3) / 4);
  const int row_vecs = b.d * (b.dtable_type == DSF_F32 ? 4 : 2) / 16;
  embed_order_kernel<<<wide_grid((int64_t(b.V) + kRange - 1) / kRange), 64 * kWaves, 0, s>>>(
      b.tokens, b.n, b.V, order, key, start, b.accumulate ? nullptr : (u32x4*)b.dtable, row_vecs);
  const dim3 grid = wide_grid(a.long_wgs + (int64_t(b.n) * a.slabs + 3) / 4);
  const bool in32 = b.dtype == DSF_F32, out32 = b.dtable_type == DSF_F32;
  if (grid.x) {
    if (in32) embed_sum_kernel<float, float><<<grid, 256, 0, s>>>(a);
    else if (out32) embed_sum_kernel<uint16_t, float><<<grid, 256, 0, s>>>(a);
    else embed_sum_kernel<uint16_t, uint16_t><<<grid, 256, 0, s>>>(a);
  }
  if (a.long_wgs) {
    if (out32) embed_join_kernel<float><<<wide_grid(a.long_wgs), 256, 0, s>>>(a);
    else embed_join_kernel<uint16_t><<<wide_grid(a.long_wgs), 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace dsf
