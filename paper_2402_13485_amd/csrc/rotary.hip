// Rotary positions of one or several axes: pair c of every head is turned by (start + offset of the pair's axis) * inv_freq[c].
//
// Bound by the bytes of q and k, once in and once out.  What could cost more is the angles: a position may be
// far (2^31 radians and more), so they are made and reduced in 64 bits, and sine and cosine of the remainder in 32.  A
// thread makes them for the pairs of one 16-byte piece of a row once and turns that piece of every head of its share.
#include "common.h"

namespace propd {

constexpr int kRotaryThreads = 256;

struct RotaryParams {
  const int32_t *axis_of, *start, *offset, *n_rows;
  const float *inv_freq;
  const unsigned char *q, *k;
  unsigned char *q_out, *k_out;
  int B, S, H, H_kv, d, rot, n_axes, offset_axes;
  int per_thread;     // heads of a thread
  int pieces;         // items of a row: pairs of pieces that turn, and pieces that are copied
  int turning;        // of these, the first so many turn
};

// cos and sin of a number of radians: the nearest multiple of pi/2 is taken
// off in two parts (pi/2 to 2 x 53 bits), |rest| <= pi/4 then; Taylor polynomials up to x^9 and x^10, cut 2e-9 off at most, 6e-8
// with their roundings.
__device__ __forceinline__ void cos_sin(double angle, float &c, float &s) {
  const double turns = rint(angle * 0.63661977236758134308);
  const double rest = fma(-turns, 6.123233995736766e-17, fma(-turns, 1.5707963267948966, angle));
  const float x = (float)rest, x2 = x * x;
  const float sn = x * fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -1.6666667e-1f), 1.f);
  const float cs = fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f), 4.1666667e-2f), -.5f), 1.f);
  const int quarter = (int)(turns - 4.0 * floor(turns * 0.25));
  const float a = quarter & 1 ? sn : cs, b = quarter & 1 ? cs : sn;  // |cos|, |sin| of the angle up to their signs
  c = quarter == 1 || quarter == 2 ? -a : a;
  s = quarter >= 2 ? -b : b;
}

template <class E>
struct Piece {  // 16 bytes
  static constexpr int N = 16 / (int)sizeof(E);
  float v[N];
  __device__ __forceinline__ void load(const unsigned char *at) {
    const u32x4 w = *reinterpret_cast<const u32x4 *>(at);
    if constexpr (N == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    }
  }
  __device__ __forceinline__ void store(unsigned char *at) const {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (N == 4) w[i] = __float_as_uint(v[i]);
      else w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
    }
    *reinterpret_cast<u32x4 *>(at) = w;
  }
};

// One thread per (row, item, share of the heads).  kAdjacent: an item is one piece, whose neighbours are pairs; otherwise
// it is a piece of the first half of the turning channels and the one opposite.
template <class E, bool kAdjacent>
__global__ __launch_bounds__(kRotaryThreads) void rotary_kernel(RotaryParams p) {
  constexpr int N = Piece<E>::N, kPairs = kAdjacent ? N / 2 : N;
  const long long rows = (long long)p.B * p.S;
  const long long at = (long long)blockIdx.x * kRotaryThreads + threadIdx.x;
  const long long row = at / p.pieces;
  if (row >= rows) return;
  const int item = (int)(at - row * p.pieces), b = (int)(row / p.S), s = (int)(row - (long long)b * p.S);
  if (p.n_rows && s >= p.n_rows[b]) return;
  const int head0 = blockIdx.y * p.per_thread, heads = p.H + p.H_kv;
  const int head_end = head0 + p.per_thread < heads ? head0 + p.per_thread : heads;
  const size_t row_bytes = (size_t)p.d * sizeof(E), head_bytes = row_bytes * p.S;
  const size_t q_at = ((size_t)b * p.H * p.S + s) * row_bytes, k_at = ((size_t)b * p.H_kv * p.S + s) * row_bytes;
  const size_t opposite = (size_t)(p.rot / 2) * sizeof(E);
  if (item >= p.turning) {  // copied
    const size_t in_row = (size_t)p.rot * sizeof(E) + 16 * (size_t)(item - p.turning);
    for (int h = head0; h < head_end; ++h) {
      const bool key = h >= p.H;
      const size_t x = (key ? k_at + (size_t)(h - p.H) * head_bytes : q_at + (size_t)h * head_bytes) + in_row;
      *reinterpret_cast<u32x4 *>((key ? p.k_out : p.q_out) + x) = *reinterpret_cast<const u32x4 *>((key ? p.k : p.q) + x);
    }
    return;
  }
  float c[kPairs], sn[kPairs];
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    const int pair = item * kPairs + i;
    int axis = p.axis_of ? p.axis_of[pair] : 0;
    axis = axis < 0 ? 0 : (axis >= p.n_axes ? p.n_axes - 1 : axis);
    const long long position = (p.start ? (long long)p.start[(size_t)b * p.n_axes + axis] : 0ll) +
                               p.offset[((size_t)b * p.offset_axes + (p.offset_axes > 1 ? axis : 0)) * p.S + s];
    cos_sin((double)position * (double)p.inv_freq[pair], c[i], sn[i]);
  }
  const size_t in_row = 16 * (size_t)item;
  for (int h = head0; h < head_end; ++h) {
    const bool key = h >= p.H;
    const size_t x = (key ? k_at + (size_t)(h - p.H) * head_bytes : q_at + (size_t)h * head_bytes) + in_row;
    const unsigned char *src = (key ? p.k : p.q) + x;
    unsigned char *dst = (key ? p.k_out : p.q_out) + x;
    Piece<E> u;
    u.load(src);
    if constexpr (kAdjacent) {
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        const float a = u.v[2 * i], o = u.v[2 * i + 1];
        u.v[2 * i] = fmaf(a, c[i], -(o * sn[i]));
        u.v[2 * i + 1] = fmaf(o, c[i], a * sn[i]);
      }
      u.store(dst);
    } else {
      Piece<E> w;
      w.load(src + opposite);
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        const float a = u.v[i], o = w.v[i];
        u.v[i] = fmaf(a, c[i], -(o * sn[i]));
        w.v[i] = fmaf(o, c[i], a * sn[i]);
      }
      u.store(dst);
      w.store(dst + opposite);
    }
  }
}

template <class E>
static bool launch_rotary(RotaryParams p, bool adjacent, hipStream_t st) {
  constexpr int N = Piece<E>::N;
  p.turning = p.rot / (adjacent ? N : 2 * N);
  p.pieces = p.turning + (p.d - p.rot) / N;
  const long long threads = (long long)p.B * p.S * p.pieces;
  const int heads = p.H + p.H_kv;
  // The angles are made once per share of the heads, and fewer threads walk fewer streams of memory at a time: as few shares as keep
  // 4 MB requested, of rows that are there (of trees of different sizes about half).  4 x 4096 rows of 40 heads, 1 / 2 / 4 shares: 66 / 72 /
  // 78 us; 16 x 128 rows of 48 heads, fp32, ragged, 2 / 4 / 8 / 24 shares: 33 / 24 / 20 / 23; 64 rows, 1 / 20 shares: 23 / 5.6.
  // Prompts with n_rows count as whole: taken for half, 4 x 4096 rows of which all / two thirds are there take 65 / 52 us instead of
  // 61 / 58, 4 x 1000 21 / 19 instead of 20 / 17.  Trees taken for whole, 32 x 128 rows of which a tenth is there: 14.5 instead of 11.2.
  const long long requested = threads * (adjacent ? 16 : 32) / (p.n_rows && p.S <= PROPD_MAX_TREE ? 2 : 1);
  int per = heads;
  while (per > 2 && requested * ((heads + per - 1) / per) < (4ll << 20)) per = (per + 1) / 2;
  p.per_thread = per;
  const dim3 grid((unsigned)((threads + kRotaryThreads - 1) / kRotaryThreads), (unsigned)((heads + per - 1) / per));
  if (adjacent) hipLaunchKernelGGL((rotary_kernel<E, true>), grid, dim3(kRotaryThreads), 0, st, p);
  else hipLaunchKernelGGL((rotary_kernel<E, false>), grid, dim3(kRotaryThreads), 0, st, p);
  return launch_ok();
}

}  // namespace propd

extern "C" propd_status propd_rotary(propd_dtype dt, int32_t B, int32_t S, int32_t H, int32_t H_kv, int32_t d, int32_t rot,
                                     int32_t adjacent, int32_t n_axes, const int32_t *axis_of, const float *inv_freq,
                                     const int32_t *start, const int32_t *offset, int32_t offset_axes, const int32_t *n_rows,
                                     const void *q, const void *k, void *q_out, void *k_out, void *hip_stream) {
  using namespace propd;
  if (B < 1 || S < 1 || H < 1 || H_kv < 0 || d < 1 || rot < 1 || rot > d || n_axes < 1 || (offset_axes != 1 && offset_axes != n_axes) ||
      !inv_freq || !offset || !q || !q_out || (H_kv > 0 && (!k || !k_out)))
    return PROPD_ERR_INVALID_ARG;
  if (dt != PROPD_BF16 && dt != PROPD_F32) return PROPD_ERR_INVALID_ARG;
  if (d % 8 != 0 || rot % 16 != 0) return PROPD_ERR_UNSUPPORTED;
  for (const void *ptr : {q, k, (const void *)q_out, (const void *)k_out})
    if (reinterpret_cast<uintptr_t>(ptr) % 16 != 0) return PROPD_ERR_INVALID_ARG;
  const long long heads = (long long)H + H_kv;
  if (heads > 65535 || (long long)B * S * (d / 4) > (1ll << 31)) return PROPD_ERR_UNSUPPORTED;
  RotaryParams p;
  p.axis_of = axis_of;
  p.start = start;
  p.offset = offset;
  p.n_rows = n_rows;
  p.inv_freq = inv_freq;
  p.q = reinterpret_cast<const unsigned char *>(q);
  p.k = reinterpret_cast<const unsigned char *>(k);
  p.q_out = reinterpret_cast<unsigned char *>(q_out);
  p.k_out = reinterpret_cast<unsigned char *>(k_out);
  p.B = B;
  p.S = S;
  p.H = H;
  p.H_kv = H_kv;
  p.d = d;
  p.rot = rot;
  p.n_axes = n_axes;
  p.offset_axes = offset_axes;
  hipStream_t st = as_stream(hip_stream);
  return (dt == PROPD_BF16 ? launch_rotary<uint16_t>(p, adjacent != 0, st) : launch_rotary<float>(p, adjacent != 0, st))
             ? PROPD_OK
             : PROPD_ERR_DEVICE;
}
