// Paged caches on the device: what a launch knows about the pages and the
// batch, where a slot lies, e4m3 codes with a power of two per row, and how
// the work of an attention launch is cut into items.
#pragma once

#include "dsf_device.h"
#include "dsf_internal.h"

namespace dsf {

// A number known before the launch to divide by, 1 <= n < 2^31. With 2^(l - 1)
// < n <= 2^l and mul the next whole number over 2^(31 + l) / n, which is below
// 2^32, m * mul / 2^(31 + l) is over m / n by at most m / 2^(31 + l), for m <
// 2^31 less than 1 / n: its whole part is m / n's.
struct Divisor {
  uint32_t mul;
  int l;
};
inline Divisor divisor(int n) {
  Divisor d = {0, 0};
  while ((int64_t(1) << d.l) < n) ++d.l;
  d.mul = uint32_t((uint64_t(1) << (31 + d.l)) / uint64_t(n) + 1);
  return d;
}
__device__ __forceinline__ int operator/(int m, const Divisor& d) { return int(__umulhi(2u * uint32_t(m), d.mul) >> d.l); }

// Sequence b of the batch: rows [row0, row0 + n) of the step, at slots
// kv - n .. kv - 1. Whatever the arrays hold, rows stay within the launch's
// n_rows and slots within the page table.
struct PagedSeq {
  int row0, n, kv;
};
__device__ __forceinline__ PagedSeq paged_seq(const PagedBatch& pb, int r0, int r1, int kv) {
  PagedSeq s;
  s.row0 = min(max(r0, 0), pb.n_rows);
  s.n = min(max(r1, s.row0), pb.n_rows) - s.row0;
  s.kv = min(max(kv, 0), pb.max_pages << pb.page_shift);
  return s;
}
__device__ __forceinline__ PagedSeq paged_seq(const PagedBatch& pb, int b) {
  return paged_seq(pb, pb.row_start[b], pb.row_start[b + 1], pb.kv_len[b]);
}
// Page that holds page index i (>= 0) of sequence b.
__device__ __forceinline__ int paged_page(const PagedBatch& pb, int b, int i, int n_pages) {
  const int p = pb.pages[int64_t(b) * pb.max_pages + min(i, pb.max_pages - 1)];
  return min(max(p, 0), n_pages - 1);
}

// ---- e4m3 codes: x ~ code * 2^e, e = byte - 127 ----
// The power of two is the fp32 number whose exponent field is the byte.
__device__ __forceinline__ float paged_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Exponent byte of a row whose largest finite magnitude is `top`: the least e
// with top <= 448 * 2^e (448 = 1.75 * 2^8, the largest e4m3 number), so e is
// top's own exponent less 8, one more where top's significand is over 1.75.
// Never below -126, where 2^e and 2^-e are both normal numbers.
__device__ __forceinline__ uint32_t paged_exponent(float top) {
  const uint32_t u = __float_as_uint(top);
  const int e = int(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return uint32_t(max(e, 1));
}
// The largest code of a row with that byte: 448, and 240 where e is 120, its
// greatest value: 256 * 2^120, the next code, is past fp32's and bf16's numbers.
__device__ __forceinline__ float paged_code_limit(uint32_t byte) { return byte >= 247 ? 240.f : 448.f; }
// Four numbers times inv (2^-e: exact) to four codes, round to nearest even.
// Infinities become the largest code, NaN the NaN code.
__device__ __forceinline__ uint32_t paged_codes4(const float* x, float inv, float limit) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float t = x[i] * inv;
    y[i] = t != t ? t : fminf(fmaxf(t, -limit), limit);
  }
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], r, true);
  return uint32_t(r);
}
// Four codes times 2^e as bf16: exact (four significant bits, and bf16 has
// fp32's exponents) down to 2^-126, below it to the nearest multiple of
// 2^-133.
__device__ __forceinline__ u32x2 paged_widen4(uint32_t c, float scale) {
  u32x2 r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, scale, false));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, scale, true));
  return r;
}
// and as fp32 (exact)
__device__ __forceinline__ f32x4 paged_widen4_f32(uint32_t c, float scale) {
  const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, scale, false);
  const auto b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, scale, true);
  return f32x4{a[0], a[1], b[0], b[1]};
}

}  // namespace dsf
