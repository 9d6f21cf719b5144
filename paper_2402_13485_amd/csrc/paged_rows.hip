// Rows in and out of the pages of a paged cache: the accepted nodes' rows after a step, prompts, and back to dense tensors.
// Bytes are what these calls cost: every row is read once and written once, its scale found in between by the lanes
// that hold the row (d / 8 of them, 8 values each).  4 x 4096 rows of 8 heads to pages in 8 bits take 20.9 us (4.8 TB/s), 8 sequences of up to 4096
// rows back 22.8 (6.4 TB/s, some of it from the memory-side cache), the rows of a step one launch.
#include "paged_cache.h"

namespace propd {

constexpr int kRowThreads = 256;
// Rows of a group of lanes requested together.  1 / 2 / 4 / 8, us: 4 x 4096 rows to pages in 8 bits 22.2 / 21.2 / 23.2 / 26.2, 8 sequences of up
// to 4096 rows from pages (stored the usual way) 31.4 / 32.5 / 34.8 / 36.4.
constexpr int kRowItems = 2;

struct WriteParams {
  Pages pages;
  const unsigned char *k, *v;                           // [B,H_kv,S,d]
  const int32_t *n_append, *index, *n_nodes, *seq_lens;  // index NULL: row j is row j; n_append NULL: S
  int32_t *seq_lens_out;                                // NULL: written by another kernel
  const int32_t *token, *next_token;
  int32_t *out_tokens;
  int out_stride, stride;  // of index
  int B, S, H_kv;
};

struct Append {
  int L, a, rows;  // rows in use, rows to append, those of them that fit
};
__device__ __forceinline__ Append append_of(const WriteParams &p, int b) {
  Append x;
  x.L = clamped(p.seq_lens[b], p.pages.capacity);
  x.a = p.n_append ? clamped(p.n_append[b], p.index ? p.stride : p.S) : p.S;
  x.rows = x.a > p.pages.capacity - x.L ? p.pages.capacity - x.L : x.a;
  return x;
}

// The 8 values of a lane, as they are held by the caller.
template <bool kBf16>
struct Eight {
  u32x4 raw[kBf16 ? 1 : 2];
  __device__ __forceinline__ void load(const unsigned char *p) {
#pragma unroll
    for (int i = 0; i < (kBf16 ? 1 : 2); ++i) raw[i] = reinterpret_cast<const u32x4 *>(p)[i];
  }
  // What is read or written once need not stay in the caches: 4 x 4096 rows to pages 21.4 -> 20.9 us by its loads, 8 sequences of up to 4096
  // rows from pages 32.5 -> 22.7 by its stores (26.6 by its loads; a copy of as many bytes takes 28.6).
  __device__ __forceinline__ void load_once(const unsigned char *p) {
#pragma unroll
    for (int i = 0; i < (kBf16 ? 1 : 2); ++i) raw[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p) + i);
  }
  __device__ __forceinline__ void store_once(unsigned char *p) const {
#pragma unroll
    for (int i = 0; i < (kBf16 ? 1 : 2); ++i) __builtin_nontemporal_store(raw[i], reinterpret_cast<u32x4 *>(p) + i);
  }
  __device__ __forceinline__ void store(unsigned char *p) const {
#pragma unroll
    for (int i = 0; i < (kBf16 ? 1 : 2); ++i) reinterpret_cast<u32x4 *>(p)[i] = raw[i];
  }
  __device__ __forceinline__ void values(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (kBf16) {
        x[2 * i] = __uint_as_float(raw[0][i] << 16);
        x[2 * i + 1] = __uint_as_float(raw[0][i] & 0xffff0000u);
      } else {
        x[i] = __uint_as_float(raw[0][i]);
        x[4 + i] = __uint_as_float(raw[kBf16 ? 0 : 1][i]);
      }
    }
  }
  __device__ __forceinline__ void take(u32x2 codes, float scale) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if constexpr (kBf16) {
        const u32x2 y = codes_to_bf16(codes[i], scale);
        raw[0][2 * i] = y.x;
        raw[0][2 * i + 1] = y.y;
      } else {
        raw[kBf16 ? 0 : i] = __builtin_bit_cast(u32x4, codes_to_f32(codes[i], scale));
      }
    }
  }
};

// One row's part of a lane to its page; LANES lanes have the row.  Every lane of the wave gets here (the scale is found across lanes).
template <bool kBf16, bool kCodes, int LANES>
__device__ __forceinline__ void store_row(const Eight<kBf16> &x, unsigned char *pages, uint8_t *scales, size_t row, int part, bool on) {
  constexpr int kBytes = kBf16 ? 2 : 4;
  if constexpr (!kCodes) {
    if (on) x.store(pages + (row * LANES + part) * 8 * kBytes);
  } else {
    float v[8], most = 0.f;
    x.values(v);
#pragma unroll
    for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(v[i]) < INFINITY ? fabsf(v[i]) : 0.f);
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) most = fmaxf(most, __shfl_xor(most, o, kWave));
    const int power = scale_power(most);
    const u32x2 codes = codes_of(v, power_of_two(-power));
    if (on) {
      *reinterpret_cast<u32x2 *>(pages + (row * LANES + part) * 8) = codes;
      if (part == 0) scales[row] = (uint8_t)(power + 127);
    }
  }
}

// Workgroups (x, b): the rows of sequence b in turn.  An item is a row of one head; neighbouring items are neighbouring rows of it.
template <bool kBf16, bool kCodes, int D>
__global__ __launch_bounds__(kRowThreads) void paged_write_kernel(WriteParams p) {
  constexpr int LANES = D / 8, kBytes = kBf16 ? 2 : 4, kGroups = kRowThreads / LANES;
  const int b = blockIdx.y;
  const Append n = append_of(p, b);
  const int T = p.n_nodes ? clamped(p.n_nodes[b] - 1, p.S - 1) + 1 : p.S;
  const int part = threadIdx.x % LANES, group = threadIdx.x / LANES, items = n.rows * p.H_kv;
  for (int item0 = blockIdx.x * (kGroups * kRowItems); item0 < items; item0 += gridDim.x * (kGroups * kRowItems)) {  // uniform
    Eight<kBf16> k[kRowItems], v[kRowItems];
    size_t to[kRowItems];
    bool on[kRowItems];
#pragma unroll
    for (int x = 0; x < kRowItems; ++x) {
      const int wanted = item0 + x * kGroups + group, item = wanted < items ? wanted : item0;
      const int h = item / n.rows, j = item - h * n.rows;
      int s = p.index ? p.index[(size_t)b * p.stride + j] : j;
      const int page = page_of(p.pages, b, n.L + j);
      on[x] = wanted < items && s >= 0 && s < T && page >= 0;
      s = s >= 0 && s < T ? s : 0;
      to[x] = row_in_pool(p.pages, page < 0 ? 0 : page, h, p.H_kv, n.L + j);
      const size_t from = ((((size_t)b * p.H_kv + h) * p.S + s) * LANES + part) * 8 * kBytes;
      k[x].load_once(p.k + from);
      v[x].load_once(p.v + from);
    }
#pragma unroll
    for (int x = 0; x < kRowItems; ++x) {
      store_row<kBf16, kCodes, LANES>(k[x], p.pages.k, p.pages.k_scale, to[x], part, on[x]);
      store_row<kBf16, kCodes, LANES>(v[x], p.pages.v, p.pages.v_scale, to[x], part, on[x]);
    }
  }
  if (blockIdx.x != 0) return;
  if (p.seq_lens_out) {
    __syncthreads();  // in place: every thread has read the old length
    if (threadIdx.x == 0) p.seq_lens_out[b] = n.L + n.rows;
  }
  if (p.out_tokens) {
    for (int j = threadIdx.x; j < p.out_stride; j += kRowThreads) {
      int t = -1;
      if (j + 1 < n.a) {
        const int node = p.index[(size_t)b * p.stride + j + 1];
        if (node >= 0 && node < T) t = p.token[(size_t)b * p.S + node];
      } else if (j + 1 == n.a) {
        t = p.next_token[b];
      }
      p.out_tokens[(size_t)b * p.out_stride + j] = t;
    }
  }
}

// The new lengths where they are written over the old ones and several workgroups read those.
__global__ __launch_bounds__(kRowThreads) void paged_lengths_kernel(WriteParams p, int32_t *out) {
  const int b = blockIdx.x * kRowThreads + threadIdx.x;
  if (b >= p.B) return;
  const Append n = append_of(p, b);
  out[b] = n.L + n.rows;
}

struct ReadParams {
  Pages pages;
  const int32_t *seq_lens, *first;
  unsigned char *k, *v;
  int S, H_kv, B;
};

// Workgroups (tile of rows, b * H_kv + h)
template <bool kBf16, bool kCodes, int D>
__global__ __launch_bounds__(kRowThreads) void paged_read_kernel(ReadParams p) {
  constexpr int LANES = D / 8, kBytes = kBf16 ? 2 : 4, kGroups = kRowThreads / LANES;
  const unsigned unit = blockIdx.y;
  const int b = (int)(unit / (unsigned)p.H_kv), h = (int)(unit - (unsigned)b * (unsigned)p.H_kv);
  const int L = clamped(p.seq_lens[b], p.pages.capacity), first = p.first ? clamped(p.first[b], L) : 0;
  const int rows = L - first < p.S ? L - first : p.S;
  const int part = threadIdx.x % LANES, group = threadIdx.x / LANES, s0 = blockIdx.x * (kGroups * kRowItems) + group;
  if ((int)blockIdx.x * (kGroups * kRowItems) >= rows) return;
  u32x2 kc[kRowItems], vc[kRowItems];
  float ks[kRowItems], vs[kRowItems];
  Eight<kBf16> k[kRowItems], v[kRowItems];
  bool there[kRowItems];
#pragma unroll
  for (int x = 0; x < kRowItems; ++x) {
    const int wanted = s0 + x * kGroups, s = wanted < rows ? wanted : rows - 1;
    const int page = page_of(p.pages, b, first + s);
    there[x] = page >= 0;
    const size_t row = row_in_pool(p.pages, page < 0 ? 0 : page, h, p.H_kv, first + s);
    if constexpr (kCodes) {
      kc[x] = *reinterpret_cast<const u32x2 *>(p.pages.k + (row * LANES + part) * 8);
      vc[x] = *reinterpret_cast<const u32x2 *>(p.pages.v + (row * LANES + part) * 8);
      ks[x] = scale_of(p.pages.k_scale[row]);
      vs[x] = scale_of(p.pages.v_scale[row]);
    } else {
      k[x].load(p.pages.k + (row * LANES + part) * 8 * kBytes);
      v[x].load(p.pages.v + (row * LANES + part) * 8 * kBytes);
    }
  }
#pragma unroll
  for (int x = 0; x < kRowItems; ++x) {
    const int s = s0 + x * kGroups;
    if (s >= rows) continue;
    if constexpr (kCodes) {
      k[x].take(kc[x], ks[x]);
      v[x].take(vc[x], vs[x]);
    }
    if (!there[x]) {
#pragma unroll
      for (int i = 0; i < (kBf16 ? 1 : 2); ++i) k[x].raw[i] = v[x].raw[i] = u32x4{0, 0, 0, 0};
    }
    const size_t to = (((size_t)unit * p.S + s) * LANES + part) * 8 * kBytes;
    k[x].store_once(p.k + to);
    v[x].store_once(p.v + to);
  }
}

template <bool kBf16, bool kCodes, int D>
static void launch_write(const WriteParams &p, dim3 grid, hipStream_t st) {
  hipLaunchKernelGGL((paged_write_kernel<kBf16, kCodes, D>), grid, dim3(kRowThreads), 0, st, p);
}

// All rows and, unless several workgroups of a sequence read a length that is to be written over, the lengths.
static propd_status write_rows(WriteParams p, propd_dtype dt, bool codes, int d, int most_rows, int32_t *seq_lens_out, hipStream_t st) {
  const int per_group = kRowThreads / (d / 8) * kRowItems;
  const long long full = ((long long)most_rows * p.H_kv + per_group - 1) / per_group;
  const bool in_place = seq_lens_out == p.seq_lens;
  long long x = full;
  const long long most = 65536 / p.B > 1 ? 65536 / p.B : 1;
  if (x > most) x = most;
  if (x < 1) x = 1;
  const bool together = !in_place || x == 1;
  p.seq_lens_out = together ? seq_lens_out : nullptr;
  const dim3 grid((unsigned)x, (unsigned)p.B);
  const bool bf16 = dt == PROPD_BF16;
  if (d == 128) {
    if (bf16) codes ? launch_write<true, true, 128>(p, grid, st) : launch_write<true, false, 128>(p, grid, st);
    else codes ? launch_write<false, true, 128>(p, grid, st) : launch_write<false, false, 128>(p, grid, st);
  } else {
    if (bf16) codes ? launch_write<true, true, 64>(p, grid, st) : launch_write<true, false, 64>(p, grid, st);
    else codes ? launch_write<false, true, 64>(p, grid, st) : launch_write<false, false, 64>(p, grid, st);
  }
  if (!launch_ok()) return PROPD_ERR_DEVICE;
  if (!together) {
    hipLaunchKernelGGL(paged_lengths_kernel, dim3((unsigned)((p.B + kRowThreads - 1) / kRowThreads)), dim3(kRowThreads), 0, st, p, seq_lens_out);
    if (!launch_ok()) return PROPD_ERR_DEVICE;
  }
  return PROPD_OK;
}

static bool aligned(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// What the calls of this file have in common
static propd_status check_rows(propd_dtype dt, int B, int S, int H_kv, int d, const void *k, const void *v, const propd_paged_cache *cache,
                               const int32_t *seq_lens) {
  if (B < 1 || S < 1 || H_kv < 1 || !k || !v || !seq_lens || !aligned(k) || !aligned(v)) return PROPD_ERR_INVALID_ARG;
  if (dt != PROPD_BF16 && dt != PROPD_F32) return PROPD_ERR_INVALID_ARG;
  const propd_status status = paged_cache_check(cache, dt);
  if (status != PROPD_OK) return status;
  if (d != 64 && d != 128) return PROPD_ERR_UNSUPPORTED;
  // (the number of rows of a sequence, and the batch as a grid's second dimension)
  if ((long long)S * H_kv > (1ll << 30) || B > 65535) return PROPD_ERR_UNSUPPORTED;
  return PROPD_OK;
}

}  // namespace propd

extern "C" propd_status propd_paged_commit(const propd_tree *tree, propd_dtype dt, int32_t H_kv, int32_t d, const int32_t *accept_len,
                                           const int32_t *accept_path, int32_t path_stride, const int32_t *next_token, const void *k_tree,
                                           const void *v_tree, const propd_paged_cache *cache, const int32_t *seq_lens, int32_t *seq_lens_out,
                                           int32_t *out_tokens, int32_t out_stride, void *hip_stream) {
  using namespace propd;
  if (!tree || tree->T_max > PROPD_MAX_TREE || path_stride < 1 || !tree->n_nodes || !accept_len || !accept_path || !seq_lens_out)
    return PROPD_ERR_INVALID_ARG;
  const propd_status status = check_rows(dt, tree->B, tree->T_max, H_kv, d, k_tree, v_tree, cache, seq_lens);
  if (status != PROPD_OK) return status;
  if (out_tokens && (out_stride < 1 || !tree->token || !next_token)) return PROPD_ERR_INVALID_ARG;
  if ((long long)path_stride * H_kv > (1ll << 30)) return PROPD_ERR_UNSUPPORTED;
  WriteParams p = {};
  p.pages = pages_of(cache);
  p.k = reinterpret_cast<const unsigned char *>(k_tree);
  p.v = reinterpret_cast<const unsigned char *>(v_tree);
  p.n_append = accept_len;
  p.index = accept_path;
  p.stride = path_stride;
  p.n_nodes = tree->n_nodes;
  p.seq_lens = seq_lens;
  p.token = tree->token;
  p.next_token = next_token;
  p.out_tokens = out_tokens;
  p.out_stride = out_stride;
  p.B = tree->B;
  p.S = tree->T_max;
  p.H_kv = H_kv;
  return write_rows(p, dt, cache->dt == PROPD_E4M3, d, path_stride < tree->T_max ? path_stride : tree->T_max, seq_lens_out, as_stream(hip_stream));
}

extern "C" propd_status propd_paged_prompt(propd_dtype dt, int32_t B, int32_t S, int32_t H_kv, int32_t d, const int32_t *n_rows,
                                           const void *k, const void *v, const propd_paged_cache *cache, const int32_t *seq_lens,
                                           int32_t *seq_lens_out, void *hip_stream) {
  using namespace propd;
  if (!seq_lens_out) return PROPD_ERR_INVALID_ARG;
  const propd_status status = check_rows(dt, B, S, H_kv, d, k, v, cache, seq_lens);
  if (status != PROPD_OK) return status;
  WriteParams p = {};
  p.pages = pages_of(cache);
  p.k = reinterpret_cast<const unsigned char *>(k);
  p.v = reinterpret_cast<const unsigned char *>(v);
  p.n_append = n_rows;
  p.seq_lens = seq_lens;
  p.B = B;
  p.S = S;
  p.H_kv = H_kv;
  return write_rows(p, dt, cache->dt == PROPD_E4M3, d, S, seq_lens_out, as_stream(hip_stream));
}

extern "C" propd_status propd_paged_read(propd_dtype dt, int32_t B, int32_t S, int32_t H_kv, int32_t d, const propd_paged_cache *cache,
                                         const int32_t *seq_lens, const int32_t *first, void *k_out, void *v_out, void *hip_stream) {
  using namespace propd;
  const propd_status status = check_rows(dt, B, S, H_kv, d, k_out, v_out, cache, seq_lens);
  if (status != PROPD_OK) return status;
  if ((long long)B * H_kv > 65535) return PROPD_ERR_UNSUPPORTED;
  ReadParams p;
  p.pages = pages_of(cache);
  p.seq_lens = seq_lens;
  p.first = first;
  p.k = reinterpret_cast<unsigned char *>(k_out);
  p.v = reinterpret_cast<unsigned char *>(v_out);
  p.S = S;
  p.H_kv = H_kv;
  p.B = B;
  const int per_group = kRowThreads / (d / 8) * kRowItems;
  const dim3 grid((unsigned)((S + per_group - 1) / per_group), (unsigned)(B * H_kv));
  hipStream_t st = as_stream(hip_stream);
  const bool bf16 = dt == PROPD_BF16, codes = cache->dt == PROPD_E4M3;
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kRowThreads), 0, st, p); };
  if (d == 128) {
    if (bf16) codes ? launch(paged_read_kernel<true, true, 128>) : launch(paged_read_kernel<true, false, 128>);
    else codes ? launch(paged_read_kernel<false, true, 128>) : launch(paged_read_kernel<false, false, 128>);
  } else {
    if (bf16) codes ? launch(paged_read_kernel<true, true, 64>) : launch(paged_read_kernel<true, false, 64>);
    else codes ? launch(paged_read_kernel<false, true, 64>) : launch(paged_read_kernel<false, false, 64>);
  }
  return launch_ok() ? PROPD_OK : PROPD_ERR_DEVICE;
}
