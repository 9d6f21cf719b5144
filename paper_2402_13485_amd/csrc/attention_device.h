// What the attention kernels share: geometry of a stage of K/V rows in LDS, loads and LDS reads that are
// waited for by hand, the layout of results and partial results, values that are not finite.
#pragma once

#include <type_traits>
#include <utility>

#include "common.h"

namespace propd {

constexpr int kStageRows = 32;   // K/V rows per ring stage

// What depends on the head size D.
template <int D>
struct Geo {
  static constexpr int kRowBytes = D * 2;                     // one bf16 row
  static constexpr int kHalfStage = kStageRows * kRowBytes;   // K part of a stage; the V part follows
  static constexpr int kStageBytes = 2 * kHalfStage;          // 16 KB (D = 128) or 8 KB
  static constexpr int kChunks = kRowBytes / 16;              // 16-byte chunks of a row
  static constexpr int kLdRows = 1024 / kRowBytes;            // rows that one direct load of a wave fills
  static constexpr int kLoads = kHalfStage / 4096;            // direct loads of a wave per half stage
  static constexpr int kMb = D / 32;                          // 32-wide blocks of d of PV
  // Workgroups resident on a compute unit: what LDS (two rings of 80 KB) and registers (one wave per 32 queries 253
  // or, with kAnew, all 256; two 215 to 218) allow at D = 128, and registers at D = 64 with one wave (208).  With two it
  // takes 165 and 41 KB of LDS, and a third workgroup would fit (not measured).  A bound of four spilled at D = 64, which this
  // kernel must not: loads that it waits for by hand would land in registers given away meanwhile.
  static constexpr int kPerCu = 2;
  // Chunk c of row r of a stage lies at chunk position c ^ key(r).
  //   K: the 16 rows x 16 bytes that one pass of a fragment read takes (one chunk column) fall
  //      into 16 different bank groups (rows of 128 bytes: two rows share a 256-byte bank line)
  //   V: so do the 4 rows x 64 bytes of one transposing read
  static __device__ __forceinline__ int k_key(int r) { return D == 128 ? r & 15 : (r >> 1) & 7; }
  static __device__ __forceinline__ int v_key(int r) {
    return D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : ((r >> 1) & 1) << 2;
  }
};

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// two floats -> packed bf16 pair (round to nearest even), one v_cvt_pk_bf16_f32
__device__ __forceinline__ uint32_t cvt_pk_bf16(float lo, float hi) {
  const f32x2 f = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
}

// Transposing LDS read (ds_read_b64_tr_b16), issued as assembly so that the compiler does
// not fence it against the ring's direct loads in flight (the builtin counts as a possible
// LDS write, which would drain them).  The result is valid only after wait_lds<>().
template <int OFFSET>
__device__ __forceinline__ u32x2 lds_read_tr16(uint32_t addr) {
  u32x2 r;
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(r) : "v"(addr), "n"(OFFSET));
  return r;
}

// LDS traffic between the waves of a workgroup, for the same reason as assembly.
template <int OFFSET>
__device__ __forceinline__ void lds_write16(uint32_t addr, f32x4 v) {
  asm volatile("ds_write_b128 %0, %1 offset:%2" ::"v"(addr), "v"(v), "n"(OFFSET) : "memory");
}
__device__ __forceinline__ void lds_write8(uint32_t addr, u32x2 v) {
  asm volatile("ds_write_b64 %0, %1" ::"v"(addr), "v"(v) : "memory");
}
template <class F, int... I>
__device__ __forceinline__ void static_for_i_impl(F &&f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void static_for_i(F &&f) {
  static_for_i_impl(f, std::make_integer_sequence<int, N>{});
}

// wait until at most N LDS operations of this wave are outstanding; the registers named
// are the results being waited for, so that their uses cannot be scheduled above the wait
template <int N>
__device__ __forceinline__ void wait_lds(u32x2 (&a)[4]) {
  asm volatile("s_waitcnt lgkmcnt(%4)" : "+v"(a[0]), "+v"(a[1]), "+v"(a[2]), "+v"(a[3]) : "n"(N));
}
template <int N>
__device__ __forceinline__ void wait_lds(u32x2 (&a)[8]) {
  asm volatile("s_waitcnt lgkmcnt(%8)"
               : "+v"(a[0]), "+v"(a[1]), "+v"(a[2]), "+v"(a[3]), "+v"(a[4]), "+v"(a[5]), "+v"(a[6]),
                 "+v"(a[7])
               : "n"(N));
}

// wait until at most N of this wave's vector memory operations are outstanding
template <int N>
__device__ __forceinline__ void wait_vmem() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Global loads and stores issued as assembly.  The main kernel waits for its vector memory
// operations itself, with explicit counts; the compiler's own bookkeeping would fence the
// ring's loads in flight at every use of a loaded register.  The compiler's hazard
// recognizer does not look inside assembly either: the stores carry their own wait states
// for data registers written just before by vector or cross-lane instructions, and after
// themselves, because a store wider than 8 bytes still reads its data registers when the
// next instruction issues.
__device__ __forceinline__ u32x4 global_load16_untracked(const void *ptr) {
  u32x4 r;
  asm volatile("s_nop 3\n\tglobal_load_dwordx4 %0, %1, off" : "=v"(r) : "v"(ptr) : "memory");
  return r;
}
__device__ __forceinline__ void global_store16_untracked(void *ptr, u32x4 v) {
  asm volatile("s_nop 7\n\tglobal_store_dwordx4 %0, %1, off sc1\n\ts_nop 3" ::"v"(ptr), "v"(v) : "memory");
}
__device__ __forceinline__ void global_store4_untracked(void *ptr, float v) {
  asm volatile("s_nop 7\n\tglobal_store_dword %0, %1, off sc1\n\ts_nop 3" ::"v"(ptr), "v"(v) : "memory");
}

// Exchange between the two 32-lane halves of a wave (v_permlane32_swap): afterwards lane
// l < 32 holds (a[l], a[l+32]) and lane l >= 32 holds (b[l-32], b[l]) in (a, b).
__device__ __forceinline__ void swap_halves(uint32_t &a, uint32_t &b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}

// A lane of the main kernel holds, for its query t = 32*wave + lane%32, the 64 values
// d = 32*mb + 8*q4 + 4*(lane/32) + j of O^T in o_acc[mb][4*q4 + j].
// Output rows: neighbouring q4 of the two lane halves are exchanged so that every lane
// writes 8 consecutive bf16 values (16 bytes) per store.
template <bool kUntracked>
__device__ __forceinline__ void store_out_block(uint16_t *orow, const f32x16 &o, float inv, int g, int mb) {
#pragma unroll
  for (int jp = 0; jp < 2; ++jp) {
    const int e = 8 * jp, od = 8 * jp + 4;  // first register of the even / odd q4 of the pair
    uint32_t a0 = cvt_pk_bf16(o[e] * inv, o[e + 1] * inv);
    uint32_t a1 = cvt_pk_bf16(o[e + 2] * inv, o[e + 3] * inv);
    uint32_t b0 = cvt_pk_bf16(o[od] * inv, o[od + 1] * inv);
    uint32_t b1 = cvt_pk_bf16(o[od + 2] * inv, o[od + 3] * inv);
    swap_halves(a0, b0);
    swap_halves(a1, b1);
    // lower half: d = 32*mb + 16*jp + 0..7, upper half: the 8 values after those
    const u32x4 w4 = {a0, a1, b0, b1};
    if (kUntracked) global_store16_untracked(orow + mb * 32 + 16 * jp + 8 * g, w4);
    else *reinterpret_cast<u32x4 *>(orow + mb * 32 + 16 * jp + 8 * g) = w4;
  }
}

// Partial results keep the register layout, so that a wave writes and reads them as
// contiguous 1 KB blocks: part_o[slot][wave][4*mb + q4][lane][j], part_ml[slot][wave][m|l][lane].
constexpr size_t kPartOFloats = 4 * 16 * 64 * 4;  // floats of part_o per slot
constexpr size_t kPartMlFloats = 4 * 2 * 64;     // floats of part_ml per slot
__device__ __forceinline__ size_t part_o_index(size_t slot, int wave, int blk, int lane) {
  return (((slot * 4 + wave) * 16 + blk) * 64 + lane) * 4;
}
__device__ __forceinline__ size_t part_ml_index(size_t slot, int wave, int which, int lane) {
  return ((slot * 4 + wave) * 2 + which) * 64 + lane;
}

// A wave-uniform 32-bit load on the scalar path.  Issued as assembly: the compiler would
// use a vector load here and wait for it with vmcnt(0), which drains the ring.  The
// scalar cache is invalidated when a kernel starts, like the vector caches, so values
// that an earlier kernel or the caller rewrote in place are seen.
__device__ __forceinline__ int32_t uniform_load_i32(const int32_t *ptr) {
  const uint64_t a = (uint64_t)(uintptr_t)ptr;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
  const uint64_t sa = ((uint64_t)hi << 32) | lo;  // in scalar registers
  int32_t v;
  asm volatile("s_load_dword %0, %1, 0x0\n\ts_waitcnt lgkmcnt(0)" : "=s"(v) : "s"(sa) : "memory");
  return v;
}

// Sums and extremes over the lanes by data-parallel moves between registers (a few cycles per step, a
// tenth of what a step through LDS takes).  `idle` fills the lanes that a step does not reach.
template <class F>
__device__ __forceinline__ int wave_scan_i32(int v, int idle, F &&join) {
  v = join(v, __builtin_amdgcn_update_dpp(idle, v, 0x111, 0xf, 0xf, false));  // row_shr:1
  v = join(v, __builtin_amdgcn_update_dpp(idle, v, 0x112, 0xf, 0xf, false));  // row_shr:2
  v = join(v, __builtin_amdgcn_update_dpp(idle, v, 0x114, 0xf, 0xf, false));  // row_shr:4
  v = join(v, __builtin_amdgcn_update_dpp(idle, v, 0x118, 0xf, 0xf, false));  // row_shr:8
  v = join(v, __builtin_amdgcn_update_dpp(idle, v, 0x142, 0xa, 0xf, false));  // row_bcast:15 into rows 1 and 3
  v = join(v, __builtin_amdgcn_update_dpp(idle, v, 0x143, 0xc, 0xf, false));  // row_bcast:31 into rows 2 and 3
  return v;
}

// Values of V that are not finite.  The tiled kernels multiply every row of a tile by a weight,
// zero for the rows that a query does not see (or that weigh less than the smallest number), and zero
// times such a value is NaN.  D = 64 and fp32 operands keep these values to the queries that give them
// weight: a tile is multiplied with zeros in the place of such values, and with a code in their place and
// zero for all others by weights of 0 and 1.  The sum of the codes tells how many +inf, -inf and NaN
// (at most 32 of each) the query sees in that column, and what to add to its result.
//   fp32: tiles that have weights of zero (tree rows; hardly any other) and such a value.  With a NaN in
//     every unit 2 x 16 units of 48 queries x 1024 keys take 31 us instead of 28, by HIP events.
//   D = 64: a weight of three parts has zeros among them in any tile, and looking through every
//     tile costs 1 us of 34, so a piece whose results hold a NaN is done once more: 83 us instead
//     of 38 where every unit of 8 x 16 has one (64 queries x 2048 keys; 0.6 us for the question).
constexpr float kCodePlus = 1.f, kCodeMinus = 64.f, kCodeNan = 4096.f;  // exact in bf16, sums exact in fp32
__device__ __forceinline__ float not_finite_sum(float codes) {
  const int n = (int)codes;
  float x = (n & 63) != 0 ? INFINITY : 0.f;
  x -= ((n >> 6) & 63) != 0 ? INFINITY : 0.f;
  return (n >> 12) != 0 ? __uint_as_float(0x7fc00000u) : x;
}
// the code of a value, 0 for a finite one
__device__ __forceinline__ float not_finite_code(uint32_t bits) {
  const uint32_t mag = bits & 0x7fffffffu;
  return mag < 0x7f800000u ? 0.f : mag > 0x7f800000u ? kCodeNan : bits >> 31 ? kCodeMinus : kCodePlus;
}
// both halves of a bf16 pair: their codes as a pair; the halves that have one become zero
__device__ __forceinline__ uint32_t take_not_finite(uint32_t &pair) {
  const uint32_t lo = __float_as_uint(not_finite_code(pair << 16)) >> 16;
  const uint32_t hi = __float_as_uint(not_finite_code(pair & 0xffff0000u)) & 0xffff0000u;
  pair &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
  return lo | hi;
}

template <int MB>
__device__ __forceinline__ bool has_nan(const f32x16 (&o)[MB]) {
  float sum = 0.f;  // NaN as soon as a term is (and for +inf - inf)
#pragma unroll
  for (int mb = 0; mb < MB; ++mb)
#pragma unroll
    for (int r = 0; r < 16; ++r) sum += o[mb][r];
  return sum != sum;
}

}  // namespace propd
