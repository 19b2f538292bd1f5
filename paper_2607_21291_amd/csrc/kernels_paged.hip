// Writing keys and values into a paged cache and reading them back (gfx950).
//
// Both are copies: HD / 8 lanes take a (row, kv head), eight elements each,
// its key and its value, so that a wave's loads and stores are whole rows.
// With e4m3 codes a row's power of two is a maximum over those lanes, found
// with DPP moves, and everything else about the code is exact or one
// rounding. The sequence of a row is found by bisection in row_start, which
// the workgroup keeps in LDS.
//
// Bound by memory, once each wave's chain of loads (page, codes) is hidden: 8
// workgroups to a CU (2048 in all) go through the pairs together, each finds
// its next pair's page while this one's data is on its way. Reading 34352 rows
// of 4 heads of 128 from e4m3 to bf16 (106 MB): 25.0 us, 4.2 TB/s (a copy of
// as many bytes: 21.5 us), to fp32 (176 MB) 53.2; where the first took 25.3:
// with a workgroup for every 16 pairs, up to 8192, and one pair after the other
// 28.4 us, with 1024 workgroups 34.5, with a contiguous share for each 26.6,
// with two pairs at a time 30.0. Writing 11861 rows as e4m3 takes 10.9 us from
// bf16 (37 MB), 13.0 from fp32 (61 MB); copying 8 tokens of 12 heads 2.8 us on
// the GPU.
#include <algorithm>

#include "paged.h"

namespace dsf {

constexpr int kPagedCopyBlocks = 2048;  // all that fit on 256 CUs
constexpr int kPagedLdsSeqs = 1024;  // the batch's arrays are taken into LDS up to this many sequences

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
    const float inv = paged_scale(254 - e), limit = paged_code_limit(e);
    *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(pool) + slot_row * HD + 8 * part) =
        u32x2{paged_codes4(x, inv, limit), paged_codes4(x + 4, inv, limit)};
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
__global__ __launch_bounds__(256) void paged_copy_kernel(PagedPool pool, PagedBatch pb, Divisor by_Hkv, T* __restrict__ k,
                                                         int64_t k_row, int64_t k_head, T* __restrict__ v,
                                                         int64_t v_row, int64_t v_head) {
  constexpr int L = HD / 8, RPB = 256 / L;  // lanes per (row, head), and those per workgroup
  __shared__ int starts[kPagedLdsSeqs + 1], lens[kPagedLdsSeqs];
  const int tid = threadIdx.x;
  const bool in_lds = pb.B <= kPagedLdsSeqs;
  if (in_lds) {
    for (int i = tid; i <= pb.B; i += 256) starts[i] = pb.row_start[i];
    for (int i = tid; i < pb.B; i += 256) lens[i] = pb.kv_len[i];
    __syncthreads();
  }
  const int part = tid % L;
  const int pairs = pb.n_rows * pool.Hkv, stride = gridDim.x * RPB;  // (pairs: below 2^31)
  // The slot's row in the pool that (row, head) p has; -1 before the first slot, -2 if it is no sequence's row.
  auto locate = [&](int p) -> int64_t {
    const int r = p / by_Hkv, h = p - r * pool.Hkv;
    int lo = 0, hi = pb.B;  // the last b with row_start[b] <= r
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if ((in_lds ? starts[mid] : pb.row_start[mid]) <= r) lo = mid;
      else hi = mid;
    }
    const PagedSeq s = in_lds ? paged_seq(pb, starts[lo], starts[lo + 1], lens[lo]) : paged_seq(pb, lo);
    const int i = r - s.row0, slot = s.kv - s.n + i;
    if (i < 0 || i >= min(s.n, pb.max_rows)) return -2;
    if (slot < 0) return -1;
    const int page = paged_page(pb, lo, slot >> pb.page_shift, pool.n_pages);
    return ((int64_t(page) * pool.Hkv + h) << pb.page_shift) + (slot & ((1 << pb.page_shift) - 1));
  };
  // every lane of a (row, head) goes the same way, so the maximum over them is whole
  int p = blockIdx.x * RPB + tid / L;
  if (p >= pairs) return;
  int64_t at = locate(p);
  while (true) {
    const int r = p / by_Hkv, h = p - r * pool.Hkv;
    T* kp = k + r * k_row + h * k_head + 8 * part;
    T* vp = v + r * v_row + h * v_head + 8 * part;
    Raw8<T> kx = {}, vx = {};
    if (at >= 0) {
      if constexpr (WRITE) {
        kx = load_raw8<T>(kp);
        vx = load_raw8<T>(vp);
      } else {
        kx = paged_get<T, E8, HD>(pool.k, pool.ke, at, part);
        vx = paged_get<T, E8, HD>(pool.v, pool.ve, at, part);
      }
    }
    const int64_t here = at;
    const bool more = p < pairs - stride;
    if (more) at = locate(p += stride);  // while the loads are on their way
    if constexpr (WRITE) {
      if (here >= 0) {
        paged_put<T, E8, HD>(kx, pool.k, pool.ke, here, part);
        paged_put<T, E8, HD>(vx, pool.v, pool.ve, here, part);
      }
    } else if (here != -2) {  // (zeros before the first slot)
#pragma unroll
      for (int j = 0; j < int(sizeof(T)) / 2; ++j) {
        reinterpret_cast<u32x4*>(kp)[j] = kx.v[j];
        reinterpret_cast<u32x4*>(vp)[j] = vx.v[j];
      }
    }
    if (!more) return;
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
    const int grid = int(std::min<int64_t>((pairs + RPB - 1) / RPB, kPagedCopyBlocks));
    paged_copy_kernel<T, decltype(e8c)::value, HD, decltype(wc)::value>
        <<<grid, 256, 0, s>>>(pool, pb, divisor(pool.Hkv), (T*)k, k_row, k_head, (T*)v, v_row, v_head);
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
