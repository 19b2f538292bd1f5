// Writing keys and values into a paged cache and reading them back (gfx950).
//
// Both are copies: HD / 8 lanes take a (row, kv head), eight elements each,
// its key and its value, so that a wave's loads and stores are whole rows.
// With e4m3 codes a row's power of two is a maximum over those lanes, found
// with DPP moves, and everything else about the code is exact or one
// rounding. The sequence of a row is found by bisection in row_start, which
// the workgroup keeps in LDS.
#include <algorithm>

#include "paged.h"

namespace dsf {

constexpr int kPagedLdsSeqs = 1024;  // row_start is bisected in LDS up to this many sequences

// Maximum over the L neighbouring lanes (4, 8 or 16) of a row's share.
template <int L>
__device__ __forceinline__ float lanes_max(float v) {
  v = fmaxf(v, DSF_DPP(v, 0xB1));                    // lane ^ 1
  v = fmaxf(v, DSF_DPP(v, 0x4E));                    // lane ^ 2
  if constexpr (L >= 8) v = fmaxf(v, DSF_DPP(v, 0x141));   // the other quad of 8 lanes
  if constexpr (L >= 16) v = fmaxf(v, DSF_DPP(v, 0x140));  // the other half of 16
  return v;
}

// Eight elements of a row to the cache: copied, or as codes (its exponent by
// the row's first lane).
template <typename T, bool E8, int HD>
__device__ __forceinline__ void paged_put(const Raw8<T>& raw, void* pool, uint8_t* exps, int64_t slot_row, int part) {
  if constexpr (!E8) {
    u32x4* dst = reinterpret_cast<u32x4*>(static_cast<T*>(pool) + slot_row * HD + 8 * part);
#pragma unroll
    for (int i = 0; i < int(sizeof(T)) / 2; ++i) dst[i] = raw.v[i];
  } else {
    float x[8];
    unpack8<T>(raw, x);
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float a = fabsf(x[i]);
      top = fmaxf(top, a < INFINITY ? a : 0.f);  // NaN compares false
    }
    const uint32_t e = paged_exponent(lanes_max<HD / 8>(top));
    const float inv = paged_scale(254 - e);
    *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(pool) + slot_row * HD + 8 * part) =
        u32x2{paged_codes4(x, inv), paged_codes4(x + 4, inv)};
    if (part == 0) exps[slot_row] = uint8_t(e);
  }
}
// and back
template <typename T, bool E8, int HD>
__device__ __forceinline__ Raw8<T> paged_get(const void* pool, const uint8_t* exps, int64_t slot_row, int part) {
  if constexpr (!E8) {
    return load_raw8<T>(static_cast<const T*>(pool) + slot_row * HD + 8 * part);
  } else {
    const u32x2 c = *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(pool) + slot_row * HD + 8 * part);
    const float s = paged_scale(exps[slot_row]);
    Raw8<T> r;
    if constexpr (sizeof(T) == 2) {
      const u32x2 a = paged_widen4(c[0], s), b = paged_widen4(c[1], s);
      r.v[0] = u32x4{a[0], a[1], b[0], b[1]};
    } else {
      r.v[0] = __builtin_bit_cast(u32x4, paged_widen4_f32(c[0], s));
      r.v[1] = __builtin_bit_cast(u32x4, paged_widen4_f32(c[1], s));
    }
    return r;
  }
}

template <typename T, bool E8, int HD, bool WRITE>
__global__ __launch_bounds__(256) void paged_copy_kernel(PagedPool pool, PagedBatch pb, T* __restrict__ k,
                                                         int64_t k_row, int64_t k_head, T* __restrict__ v,
                                                         int64_t v_row, int64_t v_head) {
  constexpr int L = HD / 8, RPB = 256 / L;  // lanes per (row, head), and those per workgroup
  __shared__ int starts[kPagedLdsSeqs + 1];
  const int tid = threadIdx.x;
  const bool in_lds = pb.B <= kPagedLdsSeqs;
  if (in_lds) {
    for (int i = tid; i <= pb.B; i += 256) starts[i] = pb.row_start[i];
    __syncthreads();
  }
  const int part = tid % L;
  const int64_t pairs = int64_t(pb.n_rows) * pool.Hkv;
  // every lane of a (row, head) leaves or stays together, so the maximum over them is whole
  for (int64_t p = int64_t(blockIdx.x) * RPB + tid / L; p < pairs; p += int64_t(gridDim.x) * RPB) {
    const int r = int(p / pool.Hkv), h = int(p - int64_t(r) * pool.Hkv);
    int lo = 0, hi = pb.B;  // the last b with row_start[b] <= r
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if ((in_lds ? starts[mid] : pb.row_start[mid]) <= r) lo = mid;
      else hi = mid;
    }
    const PagedSeq s = paged_seq(pb, lo);
    const int i = r - s.row0;
    if (i < 0 || i >= min(s.n, pb.max_rows)) continue;  // no sequence's row
    const int slot = s.kv - s.n + i;
    T* kp = k + r * k_row + h * k_head + 8 * part;
    T* vp = v + r * v_row + h * v_head + 8 * part;
    if (slot < 0) {  // before the first slot: nothing to write, zeros to read
      if constexpr (!WRITE) {
        const float zero[8] = {};
        store8<T>(kp, zero);
        store8<T>(vp, zero);
      }
      continue;
    }
    const int page = paged_page(pb, lo, slot >> pb.page_shift, pool.n_pages);
    const int64_t slot_row =
        ((int64_t(page) * pool.Hkv + h) << pb.page_shift) + (slot & ((1 << pb.page_shift) - 1));
    if constexpr (WRITE) {
      const Raw8<T> kx = load_raw8<T>(kp), vx = load_raw8<T>(vp);
      paged_put<T, E8, HD>(kx, pool.k, pool.ke, slot_row, part);
      paged_put<T, E8, HD>(vx, pool.v, pool.ve, slot_row, part);
    } else {
      const Raw8<T> kx = paged_get<T, E8, HD>(pool.k, pool.ke, slot_row, part);
      const Raw8<T> vx = paged_get<T, E8, HD>(pool.v, pool.ve, slot_row, part);
#pragma unroll
      for (int j = 0; j < int(sizeof(T)) / 2; ++j) {
        reinterpret_cast<u32x4*>(kp)[j] = kx.v[j];
        reinterpret_cast<u32x4*>(vp)[j] = vx.v[j];
      }
    }
  }
}

hipError_t launch_paged_copy(int dtype, bool write, const PagedPool& pool, const PagedBatch& pb, void* k, int64_t k_row,
                             int64_t k_head, void* v, int64_t v_row, int64_t v_head, hipStream_t s) {
  if (pb.B == 0 || pb.n_rows == 0 || pb.max_rows == 0) return hipSuccess;
  TimedScope ts(DSF_KIND_OTHER, s);
  auto run = [&](auto tag, auto e8c, auto hdc, auto wc) -> hipError_t {
    using T = decltype(tag);
    constexpr int HD = decltype(hdc)::value, RPB = 256 / (HD / 8);
    const int64_t pairs = int64_t(pb.n_rows) * pool.Hkv;
    const int grid = int(std::min<int64_t>((pairs + RPB - 1) / RPB, 8192));
    paged_copy_kernel<T, decltype(e8c)::value, HD, decltype(wc)::value>
        <<<grid, 256, 0, s>>>(pool, pb, (T*)k, k_row, k_head, (T*)v, v_row, v_head);
    return hipGetLastError();
  };
  auto run_w = [&](auto tag, auto e8c, auto hdc) {
    return write ? run(tag, e8c, hdc, std::true_type()) : run(tag, e8c, hdc, std::false_type());
  };
  auto run_h = [&](auto tag, auto e8c) -> hipError_t {
    switch (pool.hd) {
      case 32: return run_w(tag, e8c, std::integral_constant<int, 32>());
      case 64: return run_w(tag, e8c, std::integral_constant<int, 64>());
      case 128: return run_w(tag, e8c, std::integral_constant<int, 128>());
      default: return hipErrorInvalidValue;
    }
  };
  auto run_e = [&](auto tag) { return pool.codes ? run_h(tag, std::true_type()) : run_h(tag, std::false_type()); };
  return dtype == DSF_BF16 ? run_e(uint16_t()) : run_e(float());
}

}  // namespace dsf
