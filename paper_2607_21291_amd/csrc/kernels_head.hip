// The head's losses (cross entropy, distillation from a teacher's top logits)
// around their three products (kernels_headgemm.hip, kernels_headf32.hip).
//
// A row's target is a list of k classes with probabilities q (cross entropy:
// one class, q = 1). With z = h W^T / T, in units of log 2, lse = log2 sum 2^z:
//   loss = T^2 sum_j q_j (log q_j - ln 2 (z_j - lse)),  dz = T (p - q).
// Steps: the teacher's q; the rows that take part (a target, a weight), counted
// and listed in order; their h, gathered; z at the targets; then for pieces of
// those rows the logits' tiles, lse and losses, dz in place of the logits' codes,
// dh and dW. Only the listed rows cost products, and what lies in the others (NaN
// too) has no effect.
//
// A row that is sure of its target has z = lse but for e^-z: both have to come from the
// same sums, or the loss and p - 1 are a logit's rounding (1e-4 at 45 and width 3584).
// z at the targets is the product's own, bit by bit (bf16: the same matrix
// instructions in the same order; fp32: read back), and lse stays in two terms, the
// greatest logit and log2 of the sum relative to it: z - maximum is taken first.
//
// 16 bits per logit of a piece are all that is kept: with them the backward
// needs no second product for the logits (three products, not four; 25 % of the
// large call), at 6 bytes moved per logit, which cost a tenth of that product.
#include <algorithm>

#include "dsf_device.h"
#include "dsf_internal.h"
#include "head.h"

namespace dsf {

namespace {
constexpr float kLn2 = 0.6931471805599453f, kLog2e = 1.4426950408889634f;
constexpr int kLseRows = 16;  // rows of a workgroup of the lse kernel

__device__ __forceinline__ double block_sum(double v, double* lds, int tid, int nt) {
  v = wave_sum(v);
  if ((tid & 63) == 0) lds[tid >> 6] = v;
  __syncthreads();
  double t = 0.0;
  for (int i = 0; i < nt / 64; ++i) t += lds[i];
  __syncthreads();
  return t;
}
}  // namespace

// q[r][j], and plogp[r] = sum_j q_j log q_j; a row without an entry: live[r] = 0.
// An entry counts if its class is in [0, V) and its logit is over -inf; c is
// log2(e) / T (for differences of logits: the lowest finite one, which masks
// use, times c would be -inf).
// qsum[r][j]: the sum of the q of entry j's class where j is the first entry of
// that class, -1 where it is not or its class is none. A wave to a row.
__global__ __launch_bounds__(256) void head_teacher_kernel(const int32_t* __restrict__ top, const float* __restrict__ value,
                                                           int n, int k, int V, float c, float* __restrict__ q,
                                                           float* __restrict__ qsum, float* __restrict__ plogp,
                                                           int32_t* __restrict__ live) {
  extern __shared__ float list[];  // k classes and k probabilities a wave
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = blockIdx.x * 4 + wave;
  int32_t* cls = reinterpret_cast<int32_t*>(list) + wave * 2 * k;
  float* prob = list + wave * 2 * k + k;
  const int64_t at = int64_t(r) * k;
  float m = -INFINITY, sum = 0.f, h = 0.f;
  int any = 0;
  if (r < n) {
    for (int j = lane; j < k; j += 64) {
      const int t = top[at + j];
      const float v = uint32_t(t) < uint32_t(V) ? value[at + j] : -INFINITY;
      cls[j] = uint32_t(t) < uint32_t(V) ? t : -1;
      prob[j] = v;
      any |= !(v == -INFINITY);
      m = fmaxf(m, v);
    }
    any = __any(any);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    for (int j = lane; j < k; j += 64) sum += prob[j] == -INFINITY ? 0.f : exp2f((prob[j] - m) * c);
    sum = wave_sum(sum);
    for (int j = lane; j < k; j += 64) {
      const float v = prob[j];
      const float p = v == -INFINITY ? 0.f : exp2f((v - m) * c) / sum;
      q[at + j] = p;
      prob[j] = p;
      if (!(p == 0.f)) h += p * ((v - m) * c - log2f(sum));
    }
    h = wave_sum(h);
    if (lane == 0) {
      plogp[r] = h * kLn2;
      live[r] = any;
    }
  }
  __syncthreads();
  if (r >= n) return;
  for (int j = lane; j < k; j += 64) {
    const int t = cls[j];
    float s = 0.f;
    bool first = t >= 0;
    for (int i = 0; i < k; ++i)
      if (cls[i] == t) {
        s += prob[i];
        first = first && i >= j;
      }
    qsum[at + j] = first ? s : -1.f;
  }
}

// Shares of the classes for dh, by a whole wave: each round of the grid costs its
// k-tiles and about eight more, each share a partial sum written and read again
// (at some 3 MB a k-tile). The fewest of the cheapest.
__device__ __forceinline__ int head_dh_splits(int rows, int d, int ldz, bool f32, int most, int lane) {
  const int t = f32 ? 128 : 256, tr = f32 ? head_f32_rows(rows) : 256, slots = f32 ? 512 : kHeadGrid;
  const int tiles = ((rows + tr - 1) / tr) * ((d + t - 1) / t);
  const float nk = float(ldz) / 64.f, join = float(rows) * float(d) * 8.f / (f32 ? 4e6f : 3e6f);
  int got = 1;
  float best = INFINITY;
  for (int s = 1 + lane; s <= most; s += 64) {
    const float cost = float((tiles * s + slots - 1) / slots) * (nk / float(s) + 8.f) + float(s) * join;
    if (cost < best) {
      best = cost;
      got = s;
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const float c = __shfl_xor(best, o, 64);
    const int g = __shfl_xor(got, o, 64);
    if (c < best || (c == best && g < got)) {
      best = c;
      got = g;
    }
  }
  return got;
}

struct HeadRowsArgs {
  const int32_t* targets; const int32_t* live; const float* weight;
  int n, V;
  float factor;
  int mean;
  int32_t* act; int32_t* slot; int32_t* n_active;
  double* wsum; float* scale; uint32_t* count;
  float* row_loss;
  int32_t* splits;  // of each piece (null: not wanted)
  int pieces, rows, d, ldz, most, f32;
};
// The rows that take part, in order: act[slot] = row, slot[row] = slot or -1;
// n_active; wsum = sum of their weights; scale = factor / wsum (mean; 0 for a
// sum of 0) or factor. Rows that do not take part get a loss of 0. One
// workgroup: each wave counts its stretch of the rows, then places it.
__global__ __launch_bounds__(1024) void head_rows_kernel(HeadRowsArgs a) {
  __shared__ int part[16];
  __shared__ double red[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int seg = ((a.n + 15) / 16 + 63) / 64 * 64;
  const int b = std::min(int64_t(a.n), int64_t(wave) * seg), e = std::min(int64_t(a.n), int64_t(b) + seg);
  constexpr int U = 8;
  // rows i .. i + 64 U: whether the lane's take part, and their weights
  auto look = [&](int i, bool (&in)[U], float (&w)[U]) {
    int t[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = i + 64 * u + lane;
      t[u] = r < e ? (a.targets ? a.targets[r] : a.live[r]) : -1;
      w[u] = a.weight && r < e ? a.weight[r] : 1.f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      in[u] = (a.targets ? uint32_t(t[u]) < uint32_t(a.V) : t[u] > 0) && !(w[u] == 0.f);
  };
  int c = 0;
  double sum = 0.0;
  for (int i = b; i < e; i += 64 * U) {
    bool in[U];
    float w[U];
    look(i, in, w);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      c += __popcll(__ballot(in[u]));
      sum += in[u] ? double(w[u]) : 0.0;
    }
  }
  if (lane == 0) part[wave] = c;
  sum = block_sum(sum, red, tid, 1024);  // (its barriers publish part, too)
  int at = 0, all = 0;
  for (int i = 0; i < 16; ++i) {
    if (i < wave) at += part[i];
    all += part[i];
  }
  for (int i = b; i < e; i += 64 * U) {
    bool in[U];
    float w[U];
    look(i, in, w);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = i + 64 * u + lane;
      const uint64_t m = __ballot(in[u]);
      const int here = at + __popcll(m & ((uint64_t(1) << lane) - 1));
      at += __popcll(m);
      if (r >= e) continue;
      a.slot[r] = in[u] ? here : -1;
      if (in[u]) a.act[here] = r;
      else if (a.row_loss) a.row_loss[r] = 0.f;
    }
  }
  if (a.splits)
    for (int p = wave; p < a.pieces; p += 16) {
      const int here = std::max(0, std::min(all - p * a.rows, a.rows));
      const int n = head_dh_splits(a.f32 ? here : head_dz_rows(all, here), a.d, a.ldz, a.f32 != 0, a.most, lane);
      if (lane == 0) a.splits[p] = n;
    }
  if (tid == 0) {
    *a.n_active = all;
    *a.wsum = sum;
    *a.scale = a.mean ? (sum == 0.0 ? 0.f : float(double(a.factor) / sum)) : a.factor;
    *a.count = 0u;
  }
}

// The rows that take part, and (bf16) their logits at their lists' classes:
// hc[slot] = h[act[slot]] (few rows: again for dz's second terms), z2[slot][j] = <h, W[class j]>,
// 0 for a class outside [0, V).
//
// bf16: a wave to sixteen entries of the lists one after another, entry x being list place
// x % k of slot x / k: A's rows are the entries' rows of W, B's their rows of h, and
// the products' diagonal is z2. k goes up by the 32 of an instruction, from the same zeros and in
// the same lanes as in a tile of logits, so that the sums have the same bits. A slot's first
// entry copies its row. (One wave a workgroup: 8192 rows of one class are 512, 34 us at width
// 3584, eight operands in flight 37; 6554 rows of width 896 with lists of 64 124 us, 6.1 TB/s
// with what the caches hold.)
constexpr int kDots = 16;
__global__ __launch_bounds__(64) void head_gather_kernel(const uint16_t* __restrict__ h, const uint16_t* __restrict__ w,
                                                         const int32_t* __restrict__ classes, int k, int V, int d,
                                                         const int32_t* __restrict__ act,
                                                         const int32_t* __restrict__ n_active, uint16_t* __restrict__ hc,
                                                         float* __restrict__ z2) {
  constexpr int U = 16;  // products whose operands are in flight
  const int lane = threadIdx.x & 63, r16 = lane & 15, grp = lane >> 4;
  const int n = *n_active;
  const int64_t x0 = wide_index() * kDots, all = int64_t(n) * k, x = x0 + r16;
  if (x0 >= all) return;
  const bool in = x < all;
  const int s = in ? int(x / k) : 0, j = in ? int(x - int64_t(s) * k) : 0, row = act[s];
  const int c = in ? classes[int64_t(row) * k + j] : -1;
  const bool some = uint32_t(c) < uint32_t(V), first = in && j == 0;
  const bool twin = first && head_dz_rows(n, n) > n;
  const uint16_t* const hr = h + int64_t(row) * d;
  const uint16_t* const wr = w + int64_t(some ? c : 0) * d;
  uint16_t* const to = hc + int64_t(s) * d;
  uint16_t* const to2 = hc + int64_t(n + s) * d;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = 0; k0 < d; k0 += 32 * U) {
    u32x4 a[U], b[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = k0 + 32 * u + 8 * grp;
      a[u] = b[u] = u32x4{0, 0, 0, 0};
      if (in && at < d) b[u] = *reinterpret_cast<const u32x4*>(hr + at);
      if (some && at < d) a[u] = *reinterpret_cast<const u32x4*>(wr + at);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = k0 + 32 * u + 8 * grp;
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[u]), __builtin_bit_cast(bf16x8, b[u]), acc,
                                                    0, 0, 0);
      if (first && at < d) *reinterpret_cast<u32x4*>(to + at) = b[u];
      if (twin && at < d) *reinterpret_cast<u32x4*>(to2 + at) = b[u];
    }
  }
  // lane holds out[n = r16][m = 4 grp + e]
  const float v = r16 & 2 ? (r16 & 1 ? acc[3] : acc[2]) : (r16 & 1 ? acc[1] : acc[0]);
  if (in && grp == r16 >> 2) z2[x] = some ? v : 0.f;
}

// fp32: the rows alone, a wave to a row (z at the targets is read back from the product).
__global__ __launch_bounds__(256) void head_rows_f32_kernel(const float* __restrict__ h, int d,
                                                            const int32_t* __restrict__ act,
                                                            const int32_t* __restrict__ n_active, float* __restrict__ hc) {
  const int lane = threadIdx.x & 63;
  const int64_t s = wide_index() * 4 + (threadIdx.x >> 6);
  if (s >= *n_active) return;
  const u32x4* src = reinterpret_cast<const u32x4*>(h + int64_t(act[s]) * d);
  u32x4* to = reinterpret_cast<u32x4*>(hc + s * d);
  for (int c = lane; c < d / 4; c += 64) to[c] = src[c];
}

// fp32: (maximum, sum of 2^(z - maximum)) of kStatCols of a row's logits, which stay in
// registers between the two. (a workgroup to a whole row, read twice: 63 rows of 151936
// logits 33 -> 11 us, 700 of 50304 40 -> 28, 4.9 TB/s.)
constexpr int kStatCols = 16384;
__global__ __launch_bounds__(1024) void head_stats_f32_kernel(const float* __restrict__ z, int ldz, int row0, int rows_max,
                                                             const int32_t* __restrict__ n_active, int rows_ld, int tiles,
                                                             float2* __restrict__ stats) {
  __shared__ float red[2][16];
  const int64_t wg = wide_index();
  const int rows = std::min(*n_active - row0, rows_max), s = int(wg / tiles), t = int(wg - int64_t(s) * tiles);
  if (s >= rows) return;
  const float* p = z + int64_t(s) * ldz;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float v[4][4], m = -INFINITY;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int c = t * kStatCols + 4096 * u + int(threadIdx.x) * 4;
    v[u][0] = v[u][1] = v[u][2] = v[u][3] = -INFINITY;
    if (c < ldz) load_vec(p + c, v[u]);
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) m = fmaxf(fmaxf(fmaxf(m, v[u][0]), fmaxf(v[u][1], v[u][2])), v[u][3]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  if (lane == 0) red[0][wave] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 16; ++i) m = fmaxf(m, red[0][i]);
  const float ref = m == -INFINITY ? 0.f : m;
  float sum = 0.f;
#pragma unroll
  for (int u = 0; u < 4; ++u)
    sum += (exp2f(v[u][0] - ref) + exp2f(v[u][1] - ref)) + (exp2f(v[u][2] - ref) + exp2f(v[u][3] - ref));
  sum = wave_sum(sum);
  if (lane == 0) red[1][wave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = 0.f;
    for (int i = 0; i < 16; ++i) sum += red[1][i];
    stats[int64_t(t) * rows_ld + s] = float2{m, sum};
  }
}

// lse[s] = (greatest logit, log2 of the sum of 2^(z - greatest)) from the tiles'
// statistics, the row's loss, and the sum of weight x
// loss: a partial sum of each workgroup, added in order by the last of the
// call's to finish. 16 rows by 64 groups of tiles; then a wave to a row's list.
// fp32: z at the list's classes comes from the logits, and goes to z2.
struct HeadLseArgs {
  const float2* stats; int tiles, rows_ld;
  float* z2; const float* q; const float* plogp;  // q null: one class, q = 1
  float z_scale;  // of z2: to units of log 2
  const float* z; int ldz; const int32_t* classes; int V;  // z: fp32 logits, or null
  const float* weight;
  const int32_t* act; const int32_t* n_active;
  const double* wsum;
  float2* lse; float* row_loss; float* total; double* partial; uint32_t* count;
  int row0, rows, k, first, workgroups;  // first: index of this launch's first partial sum; workgroups of the call
  float T;
};
__global__ __launch_bounds__(1024) void head_lse_kernel(HeadLseArgs a) {
  __shared__ float2 st[64][kLseRows];
  __shared__ double red[16];
  __shared__ int last;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int rows = std::min(*a.n_active - a.row0, a.rows), s0 = blockIdx.x * kLseRows;
  {
    const int rl = tid & 15, grp = tid >> 4, s = s0 + rl;
    float M = -INFINITY, S = 0.f;
    if (s < rows)
      for (int t = grp; t < a.tiles; t += 4 * 64) {
        float2 v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
          v[u] = t + 64 * u < a.tiles ? a.stats[int64_t(t + 64 * u) * a.rows_ld + s] : float2{-INFINITY, 0.f};
        const float m = fmaxf(fmaxf(fmaxf(M, v[0].x), fmaxf(v[1].x, v[2].x)), v[3].x), ref = m == -INFINITY ? 0.f : m;
        S *= exp2f(M - ref);
#pragma unroll
        for (int u = 0; u < 4; ++u) S += v[u].y * exp2f(v[u].x - ref);
        M = m;
      }
    st[grp][rl] = float2{M, S};
  }
  __syncthreads();
  // wave w: row w of the workgroup
  const int s = s0 + wave, g = a.row0 + s;  // slot in the piece, in the call
  const bool in = s < rows;
  const float2 mine = st[lane][wave];
  float M = mine.x;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
  const float ref = M == -INFINITY ? 0.f : M;
  const float logs = log2f(wave_sum(mine.y * exp2f(mine.x - ref)));
  const int row = in ? a.act[g] : 0;
  // sum_j q_j (lse - z_j)
  float x = 0.f;
  if (in)
    for (int j = lane; j < a.k; j += 64) {
      const float q = a.q ? a.q[int64_t(row) * a.k + j] : 1.f;
      float z;
      if (a.z) {
        const int c = a.classes[int64_t(row) * a.k + j];
        a.z2[int64_t(g) * a.k + j] = z = uint32_t(c) < uint32_t(a.V) ? a.z[int64_t(s) * a.ldz + c] : 0.f;
      } else {
        z = a.z2[int64_t(g) * a.k + j];
      }
      // (a probability is at most 1: what the sum's rounding leaves below 0 is 0; NaN stays)
      const float below = fmaf(-a.z_scale, z, ref) + logs;
      if (!(q == 0.f)) x += q * (below < 0.f ? 0.f : below);
    }
  x = wave_sum(x);
  if (lane == 0) {
    double wl = 0.0;
    if (in) {
      a.lse[s] = float2{ref, logs};
      const float loss = a.T * a.T * ((a.q ? a.plogp[row] : 0.f) + kLn2 * x);
      if (a.row_loss) a.row_loss[row] = loss;
      wl = (a.weight ? double(a.weight[row]) : 1.0) * double(loss);
    }
    red[wave] = wl;
  }
  if (!a.total) return;
  __syncthreads();
  if (tid == 0) {
    double t = 0.0;
    for (int i = 0; i < 16; ++i) t += red[i];
    __hip_atomic_store(a.partial + a.first + blockIdx.x, t, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    last = __hip_atomic_fetch_add(a.count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == uint32_t(a.workgroups - 1);
  }
  __syncthreads();
  if (!last) return;
  double t = 0.0;
  for (int i = tid; i < a.workgroups; i += 1024)
    t += __hip_atomic_load(a.partial + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  t = block_sum(t, red, tid, 1024);
  if (tid == 0) {
    a.total[0] = float(t);
    a.total[1] = float(*a.wsum);
  }
}

// dz / T in place of the logits: weight (p - q). A workgroup takes some rows and
// a range of their classes: p from all codes (fp32: logits), then the target
// classes' entries from their fp32 logits (p - sum of the q of a class, also
// where a list names it twice).
struct HeadProbsArgs {
  void* z; int ldz;
  const float2* stats; int rows_ld;  // bf16: the tiles' maxima
  const float2* lse; const float* z2; float z_scale;  // as above
  const float* qsum;  // null: cross entropy
  const float* weight; const int32_t* classes;
  const int32_t* act; const int32_t* n_active;
  int row0, rows, k, V, cuts, cols;  // cols: classes of a range, a multiple of 2048 (bf16: 256)
};
// The entry of list place j of slot s, if its class lies in [c0, c1) and is not named before.
template <typename F>
__device__ __forceinline__ void head_probs_entry(const HeadProbsArgs& a, int s, int j, int c0, int c1, F store) {
  const int g = a.row0 + s, row = a.act[g];
  const int64_t at = int64_t(row) * a.k + j;
  const int c = a.classes[at];
  if (c < c0 || c >= std::min(c1, a.V)) return;
  const float sum = a.qsum ? a.qsum[at] : 1.f;
  if (sum == -1.f) return;
  const float2 lse = a.lse[s];
  const float z = fmaf(a.z_scale, a.z2[int64_t(g) * a.k + j], -lse.x) - lse.y;
  store(c, (a.weight ? a.weight[row] : 1.f) * (exp2f(z > 0.f ? 0.f : z) - sum));
}

// bf16, in blocks: 32 rows, a thread to 16 bytes of a row of a block, then the
// same of the next; few rows' second terms with the first. Rows from the last to
// the next multiple of 64 become zeros. Memory bounds it (8192 x 151936: 970 us,
// 5.1 TB/s for a read and a write).
constexpr int kProbsRows = 32;
__global__ __launch_bounds__(256) void head_probs_kernel(HeadProbsArgs a) {
  // the last rows first: their logits were written last
  const int active = *a.n_active, rows = std::min(active - a.row0, a.rows), r = int(blockIdx.x) / a.cuts;
  if (rows <= 0) return;
  const int all = head_dz_rows(active, rows);
  const int s0 = ((all + 63) / 64 * 64 / kProbsRows - 1 - r) * kProbsRows, c0 = (int(blockIdx.x) - r * a.cuts) * a.cols;
  if (s0 < 0) return;
  const int c1 = std::min(a.ldz, c0 + a.cols), s = s0 + int(threadIdx.x >> 3);
  const bool live = s < rows, twin = live && all > rows;
  const float2 lse = live ? a.lse[s] : float2{0.f, 0.f};
  const float wt = !live ? 0.f : a.weight ? a.weight[a.act[a.row0 + s]] : 1.f;
  u32x4* p = reinterpret_cast<u32x4*>((uint16_t*)a.z + head_z_at(s, c0, a.ldz) + (threadIdx.x & 7) * 8);
  // (the second terms' rows lie in the same blocks of 256)
  u32x4* const p2 = p + int64_t(rows) * (kZClasses / 8);
  constexpr int kStep = kZBlock / 8;  // vectors of a block
  auto probs = [&](u32x4& raw, u32x4& rest, float top) {
    float v[8], w[8];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t code = e ? raw[i] >> 16 : raw[i] & 0xffffu;
        const float x = __builtin_amdgcn_exp2f(fmaf(float(code), -kHeadReach / 65535.f, top));
        v[2 * i + e] = !live || code == 0xffffu ? 0.f : wt * x;
      }
    store_vec(reinterpret_cast<uint16_t*>(&raw), v);
    if (twin) {
      load_vec(reinterpret_cast<const uint16_t*>(&raw), w);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] -= w[i];
      store_vec(reinterpret_cast<uint16_t*>(&rest), v);
    }
  };
  if (live || s >= all)  // (the others are second terms)
    for (int c = c0, at = 0; c < c1; c += kHeadTile, at += 4 * kStep) {
      const float top = live ? (a.stats[int64_t(c / kHeadTile) * a.rows_ld + s].x - lse.x) - lse.y : 0.f;
      u32x4 raw[4], rest;
#pragma unroll
      for (int u = 0; u < 4; ++u) raw[u] = p[at + u * kStep];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        probs(raw[u], rest, top);
        p[at + u * kStep] = raw[u];
        if (twin) p2[at + u * kStep] = rest;
      }
    }
  __syncthreads();  // (the stores below come after those above)
  for (int i = threadIdx.x; i < kProbsRows * a.k; i += 256) {
    const int si = s0 + i / a.k;
    if (si < rows)
      head_probs_entry(a, si, i % a.k, c0, c1, [&](int c, float v) {
        const uint16_t first = f2bf(v);
        ((uint16_t*)a.z)[head_z_at(si, c, a.ldz)] = first;
        if (all > rows) ((uint16_t*)a.z)[head_z_at(rows + si, c, a.ldz)] = f2bf(v - bf2f(first));
      });
  }
}

// fp32, a row.
__global__ __launch_bounds__(256) void head_probs_f32_kernel(HeadProbsArgs a) {
  const int s = int(blockIdx.x) / a.cuts, c0 = (int(blockIdx.x) - s * a.cuts) * a.cols;
  if (s >= std::min(*a.n_active - a.row0, a.rows)) return;
  const int c1 = std::min(a.ldz, c0 + a.cols);
  const float2 lse = a.lse[s];
  const float wt = a.weight ? a.weight[a.act[a.row0 + s]] : 1.f;
  float* z = (float*)a.z + int64_t(s) * a.ldz;
  for (int c = c0 + int(threadIdx.x) * 4; c < c1; c += 1024) {
    float p[4];
    load_vec(z + c, p);
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = p[i] == -INFINITY ? 0.f : wt * exp2f((p[i] - lse.x) - lse.y);
    store_vec(z + c, p);
  }
  __syncthreads();
  for (int j = threadIdx.x; j < a.k; j += 256) head_probs_entry(a, s, j, c0, c1, [&](int c, float v) { z[c] = v; });
}

// dh of every row: scale times the sum of its partial sums, zeros for rows that
// do not take part (written with the first piece). `groups` lanes of a wave (a
// power of two) share a vector's partial sums, which are then added in order: 64
// rows of width 896, 64 shares of two terms, one lane 18 us, eight 8.3.
template <typename T>
__global__ __launch_bounds__(256) void head_dh_kernel(const float* __restrict__ part, const int32_t* __restrict__ n_splits,
                                                      const int32_t* __restrict__ n_active, int rows_ld, int d,
                                                      const int32_t* __restrict__ slot, int n, int row0, int rows,
                                                      const float* __restrict__ scale, T* __restrict__ dh, int groups) {
  constexpr int VEC = Elem<T>::kVec, kPart = 16;  // partial sums in flight
  const int nv = d / VEC, splits = *n_splits, active = *n_active;
  // (few rows: dz's second terms' sums lie `active` rows on)
  const int terms = sizeof(T) == 2 && head_dz_rows(active, 1) == 2 ? 2 : 1, sums = splits * terms;
  const int lane = threadIdx.x & 63, per = 64 / groups, grp = lane / per;
  const int64_t wave = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
  for (int64_t i = wave * per + lane % per; i < int64_t(n) * nv; i += int64_t(gridDim.x) * 4 * per) {
    const int r = int(i / nv), c = int(i - int64_t(r) * nv) * VEC;
    const int s = slot[r] - row0;
    float v[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = 0.f;
    if (slot[r] < 0) {
      if (row0 != 0) continue;
    } else {
      if (s < 0 || s >= rows) continue;
      const float* p = part + int64_t(s) * d + c;
      for (int q = grp * kPart; q < sums; q += groups * kPart) {
        float x[kPart][VEC];
#pragma unroll
        for (int u = 0; u < kPart; ++u)
          if (q + u < sums) {
            const int sp = (q + u) / terms, row = (q + u) % terms * active;
#pragma unroll
            for (int e = 0; e < VEC; e += 4) load_vec(p + (int64_t(sp) * rows_ld + row) * d + e, &x[u][e]);
          }
#pragma unroll
        for (int u = 0; u < kPart; ++u)
          if (q + u < sums)
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[e] += x[u][e];
      }
      // (a vector's lanes have come the same way)
      for (int o = per; o < 64; o <<= 1)
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] += __shfl_xor(v[e], o, 64);
      const float f = *scale;
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[e] *= f;
    }
    if (grp == 0) store_vec(dh + int64_t(r) * d + c, v);
  }
}

// ------------------------------------------------------------------- host

namespace {
struct HeadPlan {
  int ldz, rows, pieces, tiles, most, dz_rows, cuts, cols;  // dz_rows: of dz (with second terms), at most
  size_t splits, act, slot, live, scalars, q, qsum, plogp, z2, hc, lse, stats, partial, z, part, acc, total;
};

size_t up(size_t v) { return (v + 255) & ~size_t(255); }

// Bytes of a piece's logits (codes), and of one share of its rows' dh (which is more where
// classes are few and rows wide), at most: a piece more is a pass over dW more (in fp32, read
// and written), so pieces are large; 4 GiB are 14000 rows of 151936 classes.
constexpr size_t kPieceBytes = size_t(4) << 30;
constexpr size_t kDhPartBytes = size_t(1) << 29;

HeadPlan head_plan(int dtype, int n, int d, int V, int k, bool grads) {
  HeadPlan p{};
  const bool f32 = dtype == DSF_F32;
  const size_t eb = f32 ? 4 : 2;
  p.ldz = (V + kHeadTile - 1) / kHeadTile * kHeadTile;
  p.tiles = f32 ? (p.ldz + kStatCols - 1) / kStatCols : p.ldz / kHeadTile;
  const int64_t n256 = (int64_t(n) + 255) / 256 * 256;
  // statistics alone (bf16): no logits are kept, a piece is bounded by its statistics
  size_t per_row = (grads || f32) ? size_t(p.ldz) * eb : size_t(p.tiles) * sizeof(float2);
  if (grads) per_row = std::max(per_row, size_t(d) * 4);
  const int64_t most = std::max<int64_t>(256, int64_t(kPieceBytes / per_row) / 256 * 256);
  p.pieces = int((n256 + most - 1) / most);
  // (rows <= most, so that the pieces before the last leave it at least one row)
  p.rows = int(((n256 + p.pieces - 1) / p.pieces + 255) / 256 * 256);
  // shares of the classes for dh, at most
  const int64_t fit = int64_t(kDhPartBytes / (size_t(p.rows) * d * 4));
  p.most = int(std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(128, p.ldz / 256), fit)));
  // ranges of the classes for dz: some workgroups for each CU
  p.dz_rows = std::min(p.rows, n);
  if (!f32) p.dz_rows = (std::max(p.dz_rows, 2 * std::min(n, kHeadTwin)) + 63) / 64 * 64;
  const int unit = f32 ? 2048 : kHeadTile, groups = f32 ? p.dz_rows : p.dz_rows / kProbsRows;
  p.cuts = std::max(1, std::min(p.ldz / unit, (2048 + groups - 1) / groups));
  p.cols = ((p.ldz + p.cuts - 1) / p.cuts + unit - 1) / unit * unit;
  p.cuts = (p.ldz + p.cols - 1) / p.cols;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += up(bytes);
    return here;
  };
  p.scalars = take(256);
  p.splits = take(size_t(p.pieces) * 4);
  p.act = take(size_t(n) * 4);
  p.slot = take(size_t(n) * 4);
  p.live = take(size_t(n) * 4);
  p.plogp = take(size_t(n) * 4);
  p.q = take(size_t(n) * k * 4);
  p.qsum = take(size_t(n) * k * 4);
  p.z2 = take(size_t(n) * std::max(k, 1) * 4);
  p.lse = take(size_t(p.rows) * sizeof(float2));
  p.partial = take(size_t(p.pieces) * ((p.rows + kLseRows - 1) / kLseRows) * 8);
  p.stats = take(size_t(p.tiles) * p.rows * sizeof(float2));
  p.hc = take(size_t(f32 ? n : std::max(n, 2 * std::min(n, kHeadTwin))) * d * eb);
  if (grads || f32) p.z = take(size_t(p.rows) * p.ldz * eb);
  if (grads) {
    p.part = take(std::max(size_t(p.most) * p.rows * d * 4, size_t(kHeadGrid) * kHeadTile * kHeadTile * 4));
    if (!f32 && p.pieces > 1) p.acc = take(size_t(V) * d * 4);
  }
  p.total = at;
  return p;
}
}  // namespace

// (for gradients: also enough without, where a piece has more rows: of 15 M rows over 700000
// classes their statistics are 1 % more than the logits of a piece with gradients)
size_t head_workspace_bytes(int dtype, int n, int d, int V, int k, bool grads) {
  const size_t alone = head_plan(dtype, n, d, V, k, false).total;
  return grads ? std::max(alone, head_plan(dtype, n, d, V, k, true).total) : alone;
}

hipError_t launch_head_loss(const HeadLossArgs& a, hipStream_t s) {
  const bool grads = a.dh || a.dw, f32 = a.dtype == DSF_F32, distill = a.value != nullptr;
  const int k = distill ? a.k : 1;
  const HeadPlan p = head_plan(a.dtype, a.n, a.d, a.V, distill ? a.k : 0, grads);
  char* ws = (char*)a.workspace;
  int32_t* n_active = (int32_t*)(ws + p.scalars);
  float* scale = (float*)(ws + p.scalars + 8);
  uint32_t* count = (uint32_t*)(ws + p.scalars + 16);
  double* wsum = (double*)(ws + p.scalars + 24);
  int32_t* act = (int32_t*)(ws + p.act);
  int32_t* slot = (int32_t*)(ws + p.slot);
  float* q = distill ? (float*)(ws + p.q) : nullptr;
  float* z2 = (float*)(ws + p.z2);
  float2* lse = (float2*)(ws + p.lse);
  float2* stats = (float2*)(ws + p.stats);
  const float z_scale = kLog2e / a.temperature;
  hipError_t e;
#define DSF_TRY(x) do { if ((e = (x)) != hipSuccess) return e; } while (0)
  if (distill) {
    head_teacher_kernel<<<(a.n + 3) / 4, 256, 8 * k * sizeof(float), s>>>(a.classes, a.value, a.n, k, a.V, z_scale, q,
                                                                          (float*)(ws + p.qsum), (float*)(ws + p.plogp),
                                                                          (int32_t*)(ws + p.live));
    DSF_TRY(hipGetLastError());
  }
  int32_t* splits = (int32_t*)(ws + p.splits);
  const HeadRowsArgs r{distill ? nullptr : a.classes, (const int32_t*)(ws + p.live), a.weight, a.n, a.V,
                       a.grad_scale * a.temperature, a.mean, act, slot, n_active, wsum, scale, count, a.row_loss,
                       a.dh ? splits : nullptr, p.pieces, p.rows, a.d, p.ldz, p.most, f32};
  head_rows_kernel<<<1, 1024, 0, s>>>(r);
  DSF_TRY(hipGetLastError());
  if (f32)
    head_rows_f32_kernel<<<wide_grid((int64_t(a.n) + 3) / 4), 256, 0, s>>>((const float*)a.h, a.d, act, n_active,
                                                                           (float*)(ws + p.hc));
  else
    head_gather_kernel<<<wide_grid((int64_t(a.n) * k + kDots - 1) / kDots), 64, 0, s>>>(
        (const uint16_t*)a.h, (const uint16_t*)a.w, a.classes, k, a.V, a.d, act, n_active, (uint16_t*)(ws + p.hc), z2);
  DSF_TRY(hipGetLastError());
  const int lse_wgs = p.rows / kLseRows, last_rows = a.n - (p.pieces - 1) * p.rows;
  const int workgroups = (p.pieces - 1) * lse_wgs + (last_rows + kLseRows - 1) / kLseRows;
  for (int i = 0; i < p.pieces; ++i) {
    HeadGemmArgs g{};
    g.row0 = i * p.rows;
    g.rows = std::min(p.rows, a.n - g.row0);
    g.rows_ld = p.rows;
    g.h = ws + p.hc + size_t(g.row0) * a.d * (f32 ? 4 : 2);
    g.w = a.w;
    g.V = a.V;
    g.d = a.d;
    g.ldz = p.ldz;
    g.z = ws + p.z;
    g.zout = grads || f32 ? ws + p.z : nullptr;
    g.stats = stats;
    g.part = (float*)(ws + p.part);
    g.scale = scale;
    g.n_active = n_active;
    g.z_scale = z_scale;
    g.splits = splits + i;
    g.most = p.most;
    auto product = [&](int mode) { return f32 ? launch_head_gemm_f32(mode, g, s) : launch_head_gemm(mode, g, s); };
    DSF_TRY(product(kHeadLogits));
    if (f32) {
      head_stats_f32_kernel<<<wide_grid(int64_t(g.rows) * p.tiles), 1024, 0, s>>>((const float*)g.z, p.ldz, g.row0, g.rows,
                                                                                  n_active, p.rows, p.tiles, stats);
      DSF_TRY(hipGetLastError());
    }
    HeadLseArgs l{};
    l.stats = stats;
    l.tiles = p.tiles;
    l.rows_ld = p.rows;
    l.z2 = z2;
    l.z_scale = f32 ? 1.f : z_scale;
    l.z = f32 ? (const float*)g.z : nullptr;
    l.ldz = p.ldz;
    l.classes = a.classes;
    l.V = a.V;
    l.q = q;
    l.plogp = (const float*)(ws + p.plogp);
    l.weight = a.weight;
    l.act = act;
    l.n_active = n_active;
    l.wsum = wsum;
    l.lse = lse;
    l.row_loss = a.row_loss;
    l.total = a.total;
    l.partial = (double*)(ws + p.partial);
    l.count = count;
    l.row0 = g.row0;
    l.rows = g.rows;
    l.k = k;
    l.first = i * lse_wgs;
    l.workgroups = workgroups;
    l.T = a.temperature;
    head_lse_kernel<<<(g.rows + kLseRows - 1) / kLseRows, 1024, 0, s>>>(l);
    DSF_TRY(hipGetLastError());
    if (!grads) continue;
    HeadProbsArgs b{};
    b.z = ws + p.z;
    b.ldz = p.ldz;
    b.stats = stats;
    b.rows_ld = p.rows;
    b.lse = lse;
    b.z2 = z2;
    b.z_scale = l.z_scale;
    b.qsum = distill ? (const float*)(ws + p.qsum) : nullptr;
    b.weight = a.weight;
    b.classes = a.classes;
    b.act = act;
    b.n_active = n_active;
    b.row0 = g.row0;
    b.rows = g.rows;
    b.k = k;
    b.V = a.V;
    b.cuts = p.cuts;
    b.cols = p.cols;
    if (f32) head_probs_f32_kernel<<<g.rows * p.cuts, 256, 0, s>>>(b);
    else head_probs_kernel<<<p.dz_rows / kProbsRows * p.cuts, 256, 0, s>>>(b);
    DSF_TRY(hipGetLastError());
    if (a.dh) {
      DSF_TRY(product(kHeadDh));
      const int64_t nv = int64_t(a.n) * a.d / (f32 ? 4 : 8);
      int groups = 1;  // lanes of a vector: some workgroups for each CU
      while (groups < 8 && nv * groups < (1 << 17)) groups *= 2;
      const dim3 grid(uint32_t(std::min<int64_t>((nv * groups + 255) / 256, 8192)));
      if (f32)
        head_dh_kernel<float><<<grid, 256, 0, s>>>(g.part, g.splits, n_active, p.rows, a.d, slot, a.n, g.row0, g.rows, scale,
                                                   (float*)a.dh, groups);
      else
        head_dh_kernel<uint16_t><<<grid, 256, 0, s>>>(g.part, g.splits, n_active, p.rows, a.d, slot, a.n, g.row0, g.rows, scale,
                                                      (uint16_t*)a.dh, groups);
      DSF_TRY(hipGetLastError());
    }
    if (a.dw) {
      const bool last = i + 1 == p.pieces;
      float* sum = a.dw_f32 ? (float*)a.dw : (float*)(ws + p.acc);
      g.prev = i > 0 ? sum : nullptr;
      g.out32 = a.dw_f32 || !last ? sum : nullptr;
      g.out16 = !a.dw_f32 && last ? (uint16_t*)a.dw : nullptr;
      DSF_TRY(product(kHeadDw));
    }
  }
#undef DSF_TRY
  return hipSuccess;
}

}  // namespace dsf
