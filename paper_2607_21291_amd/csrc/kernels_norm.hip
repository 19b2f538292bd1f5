// LayerNorm / RMSNorm of dense rows and the adjoint with the gradients of gain
// and bias, for the norms outside the layers (the final one before the head).
// With xh = (x - m) r, r = (mean (x - m)^2 + eps)^-1/2 (RMSNorm: m = 0):
//   y = xh w + b;  g = dy w,  dx = r (g - mean g - xh mean(g xh)) (+ add)
//   (RMSNorm: without mean g),  dw = sum dy xh,  db = sum dy.
// Rows stay in registers between their one read and their write; one wave or
// one workgroup to a row. The adjoint's workgroups walk the rows with the
// gradients of gain and bias in registers; their partial sums are added in a
// second launch, in an order that the number of rows fixes. Memory bounds both:
// 8192 rows of width 2048 (bf16) 14 us, 4.8 TB/s, what a copy reaches; the adjoint
// of 32768 of width 3584 170 us, 4.1 TB/s of three streams, and 6 for the sums.
#include <algorithm>
#include <type_traits>

#include "dsf_device.h"
#include "dsf_internal.h"

namespace dsf {

namespace {
constexpr int kBwdWgs = 1024;

// Sum over the WAVES waves of a row; red: WAVES values of LDS that no other
// sum in flight uses.
template <int WAVES>
__device__ __forceinline__ float row_sum(float v, float* red) {
  v = wave_sum_fast(v);
  if constexpr (WAVES > 1) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) v += red[i];
  }
  return v;
}
// Outputs larger than the L2s together go past them (8192 x 2048 bf16 15.9 -> 14.5 us, the adjoint of
// 32768 x 3584 171 -> 165); smaller ones stay for the next call.
constexpr int64_t kPastL2 = int64_t(32) << 20;
template <typename T>
__device__ __forceinline__ void put_vec(T* p, const float* v, bool past) {
  u32x4 raw;
  store_vec(reinterpret_cast<T*>(&raw), v);
  if (past) __builtin_nontemporal_store(raw, reinterpret_cast<u32x4*>(p));
  else *reinterpret_cast<u32x4*>(p) = raw;
}
}  // namespace

// C vectors of 16 bytes a lane. WAVES 1: four rows a workgroup; 4: one. out may be x.
template <typename T, int C, int WAVES, bool RMS>
__global__ __launch_bounds__(256) void norm_rows_kernel(const T* x, const T* __restrict__ w, const T* __restrict__ b,
                                                        int64_t n, int d, float eps, T* out) {
  constexpr int V = Elem<T>::kVec, L = 64 * WAVES;
  __shared__ float red[2][4];
  const int l = WAVES == 1 ? int(threadIdx.x & 63) : int(threadIdx.x);
  const int64_t r = WAVES == 1 ? wide_index() * 4 + (threadIdx.x >> 6) : wide_index();
  if (r >= n) return;
  float v[C][V];
  float s = 0.f;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int at = (l + L * c) * V;
#pragma unroll
    for (int i = 0; i < V; ++i) v[c][i] = 0.f;
    if (at < d) load_vec(x + r * d + at, v[c]);
  }
  float m = 0.f;
  if constexpr (!RMS) {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i) s += v[c][i];
    m = row_sum<WAVES>(s, red[0]) / float(d);
  }
  float q = 0.f;
#pragma unroll
  for (int c = 0; c < C; ++c)
    if ((l + L * c) * V < d)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        v[c][i] -= m;
        q += v[c][i] * v[c][i];
      }
  const float rstd = 1.0f / sqrtf(row_sum<WAVES>(q, red[1]) / float(d) + eps);
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int at = (l + L * c) * V;
    if (at >= d) continue;
    float wv[V], bv[V];
    load_vec(w + at, wv);
#pragma unroll
    for (int i = 0; i < V; ++i) bv[i] = 0.f;
    if (b) load_vec(b + at, bv);
#pragma unroll
    for (int i = 0; i < V; ++i) v[c][i] = v[c][i] * rstd * wv[i] + bv[i];
    put_vec(out + r * d + at, v[c], n * d * int64_t(sizeof(T)) > kPastL2);
  }
}

// A workgroup to a row. SUMS: also partial[workgroup][0] = sum dy xh, [1] = sum dy over its rows.
// dx may be x, dy or add: a row's are read before it is written, by the threads that write it.
template <typename T, int C, bool RMS, bool SUMS>
__global__ __launch_bounds__(256) void norm_grad_kernel(const T* x, const T* dy,
                                                        const T* __restrict__ w, const T* add, int64_t n, int d,
                                                        float eps, T* dx, float* __restrict__ partial) {
  constexpr int V = Elem<T>::kVec, WAVES = 4, L = 64 * WAVES;
  __shared__ float red[2][4][4];
  const int l = int(threadIdx.x);
  float dw[SUMS ? C : 1][V], db[SUMS && !RMS ? C : 1][V];
#pragma unroll
  for (int c = 0; c < (SUMS ? C : 1); ++c)
#pragma unroll
    for (int i = 0; i < V; ++i) dw[c][i] = 0.f;
#pragma unroll
  for (int c = 0; c < (SUMS && !RMS ? C : 1); ++c)
#pragma unroll
    for (int i = 0; i < V; ++i) db[c][i] = 0.f;
  const float rd = 1.0f / float(d);
  int turn = 0;
  // a row's vectors are asked for while the row before it is worked on (in
  // registers as they are; rows of many vectors have no room for it)
  constexpr bool kAhead = C <= 4;
  u32x4 xr[kAhead ? C : 1], gr[kAhead ? C : 1];
  auto ask = [&](int64_t r) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = (l + L * c) * V;
      if (at < d && r < n) {
        xr[c] = *reinterpret_cast<const u32x4*>(x + r * d + at);
        gr[c] = *reinterpret_cast<const u32x4*>(dy + r * d + at);
      }
    }
  };
  if constexpr (kAhead) ask(blockIdx.x);
  for (int64_t r = blockIdx.x; r < n; r += gridDim.x, turn ^= 1) {
    float xv[C][V], gv[C][V];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = (l + L * c) * V;
#pragma unroll
      for (int i = 0; i < V; ++i) xv[c][i] = gv[c][i] = 0.f;
      if (at >= d) continue;
      if constexpr (kAhead) {
        load_vec(reinterpret_cast<const T*>(&xr[c]), xv[c]);
        load_vec(reinterpret_cast<const T*>(&gr[c]), gv[c]);
      } else {
        load_vec(x + r * d + at, xv[c]);
        load_vec(dy + r * d + at, gv[c]);
      }
    }
    if constexpr (kAhead) ask(r + gridDim.x);
    float m = 0.f;
    if constexpr (!RMS) {
      float s = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) s += xv[c][i];
      m = row_sum<WAVES>(s, red[turn][0]) * rd;
    }
    float q = 0.f, sg = 0.f, sgx = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = (l + L * c) * V;
      if (at >= d) continue;
      float wv[V];
      load_vec(w + at, wv);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        xv[c][i] -= m;
        q += xv[c][i] * xv[c][i];
        const float g = gv[c][i] * wv[i];
        sg += g;
        sgx += g * xv[c][i];
      }
    }
    // three sums, one barrier
    q = wave_sum_fast(q);
    sgx = wave_sum_fast(sgx);
    if constexpr (!RMS) sg = wave_sum_fast(sg);
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
      red[turn][1][wave] = q;
      red[turn][2][wave] = sgx;
      red[turn][3][wave] = sg;
    }
    __syncthreads();
    q = red[turn][1][0];
    sgx = red[turn][2][0];
    sg = red[turn][3][0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) {
      q += red[turn][1][i];
      sgx += red[turn][2][i];
      sg += red[turn][3][i];
    }
    const float rstd = 1.0f / sqrtf(q * rd + eps);
    const float mgx = sgx * rd * rstd * rstd, mg = RMS ? 0.f : sg * rd;  // mean(g xh) r, mean g
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = (l + L * c) * V;
      if (at >= d) continue;
      float wv[V], o[V];
      load_vec(w + at, wv);
#pragma unroll
      for (int i = 0; i < V; ++i) o[i] = 0.f;
      if (add) load_vec(add + r * d + at, o);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        o[i] += rstd * (gv[c][i] * wv[i] - mg - xv[c][i] * mgx);
        if constexpr (SUMS) {
          dw[c][i] += gv[c][i] * (xv[c][i] * rstd);
          if constexpr (!RMS) db[c][i] += gv[c][i];
        }
      }
      if (dx) put_vec(dx + r * d + at, o, n * d * int64_t(sizeof(T)) > kPastL2);
    }
  }
  if constexpr (SUMS) {
    float* p = partial + int64_t(blockIdx.x) * (RMS ? 1 : 2) * d;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = (l + L * c) * V;
      if (at >= d) continue;
#pragma unroll
      for (int i = 0; i < V; i += 4) {
        store_vec(p + at + i, &dw[c][i]);
        if constexpr (!RMS) store_vec(p + d + at + i, &db[c][i]);
      }
    }
  }
}

// dw[c] (and db[c]) = sum over the partial sums: 64 columns of a workgroup, a
// column's partial sums in 16 groups, then the groups in order.
__global__ __launch_bounds__(1024) void norm_grad_sums_kernel(const float* __restrict__ partial, int slots, int d, int two,
                                                              float* __restrict__ dw, float* __restrict__ db) {
  __shared__ float red[16][64];
  const int col = threadIdx.x & 63, grp = threadIdx.x >> 6;
  const int c = blockIdx.x * 64 + col, width = d << two;
  float v = 0.f;
  if (c < width)
    for (int i = grp; i < slots; i += 16 * 16) {
      float x[16];
#pragma unroll
      for (int u = 0; u < 16; ++u) x[u] = i + 16 * u < slots ? partial[int64_t(i + 16 * u) * width + c] : 0.f;
#pragma unroll
      for (int u = 0; u < 16; ++u) v += x[u];
    }
  red[grp][col] = v;
  __syncthreads();
  if (grp != 0 || c >= width) return;
  v = 0.f;
  for (int i = 0; i < 16; ++i) v += red[i][col];
  float* out = c < d ? dw : db;
  if (out) out[c < d ? c : c - d] = v;
}

namespace {
// vectors a lane of four waves to a row, by the row's 16-byte vectors (sixteen: fp32 alone,
// the widest rows of bf16 have 2048)
template <typename T, typename F>
void norm_shape(int nv, F f) {
  if (nv <= 256) f(std::integral_constant<int, 1>());
  else if (nv <= 512) f(std::integral_constant<int, 2>());
  else if (nv <= 1024) f(std::integral_constant<int, 4>());
  else if (sizeof(T) == 2 || nv <= 2048) f(std::integral_constant<int, 8>());
  else if constexpr (sizeof(T) == 4) f(std::integral_constant<int, 16>());
}
}  // namespace

int norm_rows_max_d() { return 16384; }

hipError_t launch_norm_rows(int dtype, bool rms, const void* x, const void* w, const void* b, int64_t n, int d, float eps,
                            void* out, hipStream_t s) {
  auto run = [&](auto Tz) {
    using T = decltype(Tz);
    const int nv = d / Elem<T>::kVec;
    auto go = [&](auto Cc, auto Wc) {
      constexpr int C = decltype(Cc)::value, W = decltype(Wc)::value;
      const dim3 grid = wide_grid(W == 1 ? (n + 3) / 4 : n);
      if (rms) norm_rows_kernel<T, C, W, true><<<grid, 256, 0, s>>>((const T*)x, (const T*)w, (const T*)b, n, d, eps, (T*)out);
      else norm_rows_kernel<T, C, W, false><<<grid, 256, 0, s>>>((const T*)x, (const T*)w, (const T*)b, n, d, eps, (T*)out);
    };
    // Many narrow rows: a wave to a row, so that its lanes have loads enough (width 768, bf16: 16384 rows
    // 12.6 -> 9.7 us, 4096 4.5 -> 3.9; 1024 2.3 -> 2.7).
    using One = std::integral_constant<int, 1>;
    if (n >= 2048 && nv <= 64) go(One(), One());
    else if (n >= 2048 && nv <= 128) go(std::integral_constant<int, 2>(), One());
    else norm_shape<T>(nv, [&](auto Cc) { go(Cc, std::integral_constant<int, 4>()); });
  };
  if (dtype == DSF_F32) run(float());
  else run(uint16_t());
  return hipGetLastError();
}

// partial sums: one a workgroup at most
size_t norm_backward_workspace_bytes(int64_t n, int d) {
  return size_t(std::min<int64_t>(n, kBwdWgs)) * 2 * d * sizeof(float);
}

hipError_t launch_norm_backward(const NormBackwardArgs& a, hipStream_t s) {
  auto run = [&](auto Tz) {
    using T = decltype(Tz);
    // (a workgroup to a row also where rows are narrow: a wave to each leaves four times the partial
    // sums, 4096 rows of width 768 14.1 -> 27.3 us, 16384 29.4 -> 35.0)
    norm_shape<T>(a.d / Elem<T>::kVec, [&](auto Cc) {
      constexpr int C = decltype(Cc)::value;
      // two rows or more for each partial sum once every CU has a workgroup (1024 rows of width 3584 on 1024
      // workgroups 16.9 us, on 512 13.1); up to 1024 (16384 rows: on 512 125 us, 1024 91, 2048 97)
      const int wgs = int(std::min<int64_t>(a.n, std::min<int64_t>(kBwdWgs, std::max<int64_t>(256, (a.n + 1) / 2))));
      const bool sums = a.dw || a.db;
      auto go = [&](auto R, auto S) {
        norm_grad_kernel<T, C, decltype(R)::value, decltype(S)::value><<<wgs, 256, 0, s>>>(
            (const T*)a.x, (const T*)a.dy, (const T*)a.w, (const T*)a.add, a.n, a.d, a.eps, (T*)a.dx, (float*)a.workspace);
      };
      using Y = std::true_type;
      using N = std::false_type;
      if (a.rms && sums) go(Y(), Y());
      else if (a.rms) go(Y(), N());
      else if (sums) go(N(), Y());
      else go(N(), N());
      if (!sums) return;
      const int width = a.d * (a.rms ? 1 : 2);
      norm_grad_sums_kernel<<<(width + 63) / 64, 1024, 0, s>>>((const float*)a.workspace, wgs, a.d, a.rms ? 0 : 1, a.dw, a.db);
    });
  };
  if (a.dtype == DSF_F32) run(float());
  else run(uint16_t());
  return hipGetLastError();
}

}  // namespace dsf
