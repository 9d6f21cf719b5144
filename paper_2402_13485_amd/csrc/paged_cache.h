// What the calls of a paged cache share: where a row lies, and rows held in 8 bits.
#pragma once

#include <math.h>

#include "common.h"

namespace propd {

constexpr int kLeastPageRows = 16, kMostPageRows = 1024;

// propd_paged_cache for kernels
struct Pages {
  unsigned char *k, *v;
  uint8_t *k_scale, *v_scale;
  const int32_t *table;
  int n_pages, table_pages, shift;  // page_rows = 1 << shift
  int capacity;                     // rows of a sequence, at most
};

inline Pages pages_of(const propd_paged_cache *c) {
  Pages p;
  p.k = reinterpret_cast<unsigned char *>(c->k_pages);
  p.v = reinterpret_cast<unsigned char *>(c->v_pages);
  p.k_scale = c->k_scale;
  p.v_scale = c->v_scale;
  p.table = c->page_table;
  p.n_pages = c->n_pages;
  p.table_pages = c->table_pages;
  p.shift = __builtin_ctz((unsigned)c->page_rows);
  p.capacity = c->table_pages * c->page_rows;
  return p;
}

// PROPD_OK if the cache can be used by a call of this type
inline propd_status paged_cache_check(const propd_paged_cache *c, propd_dtype dt) {
  if (!c || !c->k_pages || !c->v_pages || !c->page_table || c->n_pages < 1 || c->table_pages < 1) return PROPD_ERR_INVALID_ARG;
  if (c->dt != dt && c->dt != PROPD_E4M3) return PROPD_ERR_INVALID_ARG;
  if (c->dt == PROPD_E4M3 && (!c->k_scale || !c->v_scale)) return PROPD_ERR_INVALID_ARG;
  if (c->page_rows < kLeastPageRows || c->page_rows > kMostPageRows || (c->page_rows & (c->page_rows - 1)) != 0) return PROPD_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(c->k_pages) % 16 != 0 || reinterpret_cast<uintptr_t>(c->v_pages) % 16 != 0) return PROPD_ERR_INVALID_ARG;
  if ((long long)c->table_pages * c->page_rows > (1ll << 30)) return PROPD_ERR_UNSUPPORTED;
  return PROPD_OK;
}

// The page of row `row` of sequence b, -1 if there is none; 0 <= row < capacity
__device__ __forceinline__ int page_of(const Pages &p, int b, int row) {
  const int page = p.table[(size_t)b * p.table_pages + (row >> p.shift)];
  return (unsigned)page < (unsigned)p.n_pages ? page : -1;
}

// where row `row` of K/V head h lies in its page, in rows
__device__ __forceinline__ size_t row_in_pool(const Pages &p, int page, int h, int H_kv, int row) {
  return (((size_t)page * H_kv + h) << p.shift) + (row & ((1 << p.shift) - 1));
}

__device__ __forceinline__ int clamped(int v, int most) { return v < 0 ? 0 : (v > most ? most : v); }

// ---- rows in 8 bits
constexpr int kLeastPower = -117, kMostPower = 119;  // code and scale of such rows make a value that bf16 holds exactly
constexpr float kMostCode = 448.f;

// 2^e by its bits
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// The exponent of a row's scale from its largest finite magnitude m = f * 2^x, 1 <= f < 2: 448 = 1.75 * 2^8.
__device__ __forceinline__ int scale_power(float most) {
  const uint32_t bits = __float_as_uint(most);
  if (bits < 0x00800000u) return kLeastPower;  // zero, or too small for the exponent to matter
  const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return e < kLeastPower ? kLeastPower : (e > kMostPower ? kMostPower : e);
}

// Two values over the scale as codes (low 16 bits): v_cvt_pk_fp8_f32 rounds to nearest even, and what is not finite becomes NaN.
__device__ __forceinline__ float to_code_range(float x, float inv) {
  const float y = fminf(fmaxf(x * inv, -kMostCode), kMostCode);
  return fabsf(x) < INFINITY ? y : __uint_as_float(0x7fc00000u);
}
__device__ __forceinline__ u32x2 codes_of(const float (&x)[8], float inv) {
  uint32_t lo = 0, hi = 0;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(to_code_range(x[0], inv), to_code_range(x[1], inv), lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(to_code_range(x[2], inv), to_code_range(x[3], inv), lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(to_code_range(x[4], inv), to_code_range(x[5], inv), hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(to_code_range(x[6], inv), to_code_range(x[7], inv), hi, true);
  return u32x2{lo, hi};
}

// Four codes as values, exact: as two bf16 pairs, or as four fp32 numbers.
typedef __bf16 bf16_pair __attribute__((ext_vector_type(2)));
typedef float f32_pair __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u32x2 codes_to_bf16(uint32_t codes, float scale) {
  const bf16_pair lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true);
  return u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}
__device__ __forceinline__ f32x4 codes_to_f32(uint32_t codes, float scale) {
  const f32_pair lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, scale, true);
  return f32x4{lo.x, lo.y, hi.x, hi.y};
}

// A scale's byte as a number.  Bytes that no row of propd_paged_commit or propd_paged_prompt has count as the nearest that one can have.
__device__ __forceinline__ float scale_of(uint32_t byte) {
  const int e = (int)byte - 127;
  return power_of_two(e < kLeastPower ? kLeastPower : (e > kMostPower ? kMostPower : e));
}

}  // namespace propd
