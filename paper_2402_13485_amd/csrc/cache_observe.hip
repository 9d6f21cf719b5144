// What the accepted nodes of a step paid to every row of a cache: paid[j] = sum of exp(s_rj - lse_r) over the
// accepted nodes and the query heads that share the K/V head; the rows' weights decay and take it up.
//
// One pass over K (a softmax needs two, but the attention has left lse), bound by its bytes: a wave walks KT tiles of 16 keys at a time,
// the next ones requested in front of the work on these, as the B operand of S = Q . K^T (16x16 products); the accepted queries are
// the A operand, 16 rows to a group, the first kHeld groups of which stay in registers.  A lane then holds four queries' scores of
// one key, adds their weights up, and the four lanes of a key meet at the end.  K rows are read straight from memory in the operand's
// layout, 64 bytes of 16 rows per load.
// 16 x 8 heads x 4096 rows of 128: 50 us (2.9 TB/s), 41 of them without any work on the rows.  The attention reads such rows at
// 5 TB/s: what is lost are the rounds of tiles (257 over 48 places are six where 5.35 are needed), the chain path -> query -> lse at the start,
// and query rows beyond 16 * kHeld, which every batch of tiles fetches again.  57 us with one batch of tiles per wave, each of which then paid for the chain path -> query -> lse.  Rings in LDS
// that direct loads fill, per wave and without barriers, took 55 us with three tiles of 4 KB in flight per wave, 58 to 84 with
// other depths and numbers of waves.
#include <type_traits>

#include "score_rule.h"

namespace propd {

constexpr int kObserveWaves = 4, kObserveThreads = kObserveWaves * kWave;

struct ObserveParams {
  const void *q, *k_cache, *k_tree;
  const float *lse, *slopes, *weight;
  const int32_t *seq_lens, *n_nodes, *dropped, *position, *accept_len, *accept_path;
  int32_t *position_out;
  float *weight_out;
  int H, H_kv, group, T_max, L_max, path_stride;
  int chunks;  // workgroups per unit
  int window;
  float scale, scale_log2e, cap, inv_cap, decay;
};

// Operands of 16 rows: KF fragments of 16 bytes, fragment f of lane l holds row l % 16 and, of every fragment's share of d, part l / 16.
template <class E, int D>
struct Rows;
template <int D>
struct Rows<uint16_t, D> {
  static constexpr int kF = D / 32;
  bf16x8 f[kF];
  __device__ __forceinline__ void load(const uint16_t *row, int part) {
#pragma unroll
    for (int i = 0; i < kF; ++i) f[i] = *reinterpret_cast<const bf16x8 *>(row + 32 * i + 8 * part);
  }
  __device__ __forceinline__ f32x4 times(const Rows &b) const {
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kF; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[i], b.f[i], acc, 0, 0, 0);
    return acc;
  }
};
template <int D>
struct Rows<float, D> {
  static constexpr int kF = D / 16;
  f32x4 f[kF];
  __device__ __forceinline__ void load(const float *row, int part) {
#pragma unroll
    for (int i = 0; i < kF; ++i) f[i] = *reinterpret_cast<const f32x4 *>(row + 16 * i + 4 * part);
  }
  __device__ __forceinline__ f32x4 times(const Rows &b) const {
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kF; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(f[i][j], b.f[i][j], acc, 0, 0, 0);
    return acc;
  }
};

// Every tile meets every accepted query row, also the path's own: device memory that claims a path of millions must not take hours.
constexpr int kMostPath = 1 << 16;

constexpr int kHeld = 2;  // groups of 16 query rows that stay in registers

constexpr int observe_per_cu(size_t element, int d) { return element == 2 ? (d == 64 ? 4 : 3) : d == 64 ? 3 : 2; }  // workgroups, by registers

// What a query row needs: the exponent of a key's weight is products * scale + slope * (place of the key - place on the path) - shift, all in
// the log2 domain, places being positions less the root's; it sees places from `lowest` on.  (The bias is made of the distance itself: with
// slope * place on the path in the shift, two large terms would cancel for the last nodes of a long path, and their
// last bits would not be those of the attention that left lse.)
struct QueryRow {
  float slope, shift, lowest;
  int place;  // on the path; -1: no query
};

// kPlace: positions take part (a window, a bias, or rows at positions of their own).
template <class E, int D, int KT, bool kPlace>
__global__ __launch_bounds__(kObserveThreads, observe_per_cu(sizeof(E), D)) void cache_observe_kernel(ObserveParams p) {
  // of the first 16 * kHeld query rows (row = place on the path * group + head)
  __shared__ __attribute__((aligned(16))) float s_slope[16 * kHeld], s_shift[16 * kHeld], s_lowest[16 * kHeld];
  __shared__ __attribute__((aligned(16))) int s_place[16 * kHeld], s_row[16 * kHeld];  // place on the path (-1: no query), row of q
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c16 = lane & 15, part = lane >> 4;
  const int unit = (int)(blockIdx.x / (unsigned)p.chunks), chunk = (int)(blockIdx.x - (unsigned)unit * (unsigned)p.chunks);
  const int b = unit / p.H_kv, hk = unit - b * p.H_kv;
  const Lengths n = lengths_of(p.seq_lens, p.n_nodes, p.dropped, p.L_max, p.T_max, b);
  int a = p.accept_len[b];
  a = a < 0 ? 0 : (a > p.path_stride ? p.path_stride : a);
  const int32_t *path = p.accept_path + (size_t)b * p.path_stride;
  const int cached = (n.L + 15) / 16, tiles = cached + (a + 15) / 16;
  if (chunk * kObserveWaves * KT >= tiles) return;  // the whole workgroup
  const int step = p.chunks * kObserveWaves * KT;
  int tile0 = (chunk * kObserveWaves + wave) * KT;
  const E *q = reinterpret_cast<const E *>(p.q), *k_cache = reinterpret_cast<const E *>(p.k_cache) + (size_t)unit * p.L_max * D;
  const E *k_tree = reinterpret_cast<const E *>(p.k_tree) + (size_t)unit * p.T_max * D;
  const int rows = a * p.group;

  // ---- a batch of tiles: 16 cached rows each, or 16 places of the path.  Keys past the last take a valid row.
  struct Batch {
    Rows<E, D> keys[KT];
    int at[KT];     // positions
    float old[KT];  // weights so far
  };
  auto load = [&](Batch &x, int t0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < KT; ++i) {
      const int t = t0 + i < tiles ? t0 + i : tiles - 1;  // uniform
      if (t < cached) {
        const int j = 16 * t + c16, row = j < n.L ? j : n.L - 1;
        x.at[i] = p.position ? p.position[(size_t)unit * p.L_max + row] : n.dropped + row;
        x.old[i] = p.weight[(size_t)unit * p.L_max + row];
        x.keys[i].load(k_cache + (size_t)row * D, part);
      } else {
        const int r = 16 * (t - cached) + c16, node = path[r < a ? r : a - 1];
        const bool valid = node >= 0 && node < n.T;
        x.at[i] = valid ? n.P + r : -1;
        x.old[i] = 0.f;
        x.keys[i].load(k_tree + (size_t)(valid ? node : 0) * D, part);
      }
    }
  };
  Batch now, next;
  if (tile0 < tiles) load(now, tile0);

  // ---- the query rows that are held
  const int held = rows < 16 * kHeld ? rows : 16 * kHeld;
  auto line_of = [&](int row, QueryRow &x) __attribute__((always_inline)) -> int {  // its row of q within the sequence
    const bool there = row < rows;
    const int r = there ? row / p.group : 0, head = hk * p.group + (there ? row - r * p.group : 0);
    const int node = there ? path[r] : -1;
    const bool valid = node >= 0 && node < n.T;
    const int line = head * p.T_max + (valid ? node : 0);
    const float lse = p.lse[(size_t)b * p.H * p.T_max + line];
    x.place = valid && lse != -INFINITY ? r : -1;
    x.slope = p.slopes ? p.slopes[head] * kLog2e : 0.f;
    x.shift = lse * kLog2e;
    x.lowest = (float)(sight_of(n.P + r, p.window).lowest - n.P);
    return line;
  };
  if (threadIdx.x < 16 * kHeld) {
    QueryRow x = {0.f, 0.f, 0.f, -1};
    s_row[threadIdx.x] = rows > 0 ? line_of(threadIdx.x, x) : 0;
    s_place[threadIdx.x] = x.place;
    s_slope[threadIdx.x] = x.slope;
    s_shift[threadIdx.x] = x.shift;
    s_lowest[threadIdx.x] = x.lowest;
  }
  __syncthreads();
  const E *q_base = q + (size_t)b * p.H * p.T_max * D;
  Rows<E, D> queries[kHeld];
#pragma unroll
  for (int g = 0; g < kHeld; ++g)
    if (16 * g < held) queries[g].load(q_base + (size_t)s_row[16 * g + c16] * D, part);

  float paid[KT], place[KT];
  // what 16 query rows pay to tile i of the batch
  auto pay = [&](const Rows<E, D> &keys, int i, auto own_keys, const Rows<E, D> &rows16, const f32x4 slope, const f32x4 shift, const f32x4 lowest,
                 const int (&on_path)[4]) __attribute__((always_inline)) {
    constexpr bool own = decltype(own_keys)::value;
    f32x4 x = rows16.times(keys);
    mfma_settle();
    if (p.cap > 0.f) {  // uniform
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = capped(x[j] * p.scale, p.cap, p.inv_cap) * kLog2e;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] *= p.scale_log2e;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (kPlace || own) x[j] = fmaf(slope[j], place[i] - (float)on_path[j], x[j]);
      const float w = __builtin_amdgcn_exp2f(x[j] - shift[j]);
      bool seen = on_path[j] >= 0;
      if constexpr (kPlace || own) seen = seen && place[i] >= lowest[j];
      if constexpr (own) seen = seen && place[i] <= (float)on_path[j];
      paid[i] += seen ? w : 0.f;
    }
  };
  auto pay_batch = [&](const Batch &x, const Rows<E, D> &rows16, const f32x4 slope, const f32x4 shift, const f32x4 lowest,
                       const int (&on_path)[4]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < KT; ++i) {
      if (tile0 + i < cached) pay(x.keys[i], i, std::false_type{}, rows16, slope, shift, lowest, on_path);
      else pay(x.keys[i], i, std::true_type{}, rows16, slope, shift, lowest, on_path);
    }
  };
  for (; tile0 < tiles; tile0 += step) {
    const bool more = tile0 + step < tiles;
    if (more) load(next, tile0 + step);
    // places of the keys; one without a row, or cached and not before the root, lies below everything
#pragma unroll
    for (int i = 0; i < KT; ++i) {
      paid[i] = 0.f;
      const bool own = tile0 + i >= cached;
      place[i] = own ? (now.at[i] >= 0 ? (float)(now.at[i] - n.P) : -0x1p31f) : (unsigned)now.at[i] < (unsigned)n.P ? (float)(now.at[i] - n.P) : -0x1p31f;
    }
#pragma unroll
    for (int g = 0; g < kHeld; ++g)
      if (16 * g < held) {  // uniform
        const int r4 = 16 * g + 4 * part;
        const int on_path[4] = {s_place[r4], s_place[r4 + 1], s_place[r4 + 2], s_place[r4 + 3]};
        pay_batch(now, queries[g], *reinterpret_cast<const f32x4 *>(s_slope + r4), *reinterpret_cast<const f32x4 *>(s_shift + r4),
                  *reinterpret_cast<const f32x4 *>(s_lowest + r4), on_path);
      }
    for (int row0 = 16 * kHeld; row0 < rows; row0 += 16) {  // the rows that are not held
      Rows<E, D> rows16;
      QueryRow x;
      rows16.load(q_base + (size_t)line_of(row0 + c16, x) * D, part);
      f32x4 slope, shift, lowest;
      int on_path[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        line_of(row0 + 4 * part + j, x);
        slope[j] = x.slope, shift[j] = x.shift, lowest[j] = x.lowest, on_path[j] = x.place;
      }
      pay_batch(now, rows16, slope, shift, lowest, on_path);
    }
    // ---- the four lanes of a key; lanes of part i write tile i
#pragma unroll
    for (int i = 0; i < KT; ++i) {
      paid[i] += __shfl_xor(paid[i], 16, kWave);
      paid[i] += __shfl_xor(paid[i], 32, kWave);
    }
#pragma unroll
    for (int i = 0; i < KT; ++i) {
      const int t = tile0 + i;
      const bool own = t >= cached;
      const int key = 16 * (own ? t - cached : t) + c16;
      if (part != i || t >= tiles || key >= (own ? a : n.L) || (own && n.L + key >= p.L_max)) continue;
      const size_t w = (size_t)unit * p.L_max + (own ? n.L + key : key);
      p.weight_out[w] = own ? (now.at[i] < 0 ? 0.f : paid[i]) : fmaf(p.decay, now.old[i], paid[i]);
      if (p.position_out) p.position_out[w] = now.at[i];
    }
    if (more) now = next;
  }
}

template <class E, int D, bool kPlace>
static bool launch_observe(ObserveParams p, long long units, hipStream_t st) {
  const long long tiles = (p.L_max + 15ll) / 16 + (p.path_stride + 15ll) / 16;
  constexpr int KT = sizeof(E) == 2 ? 2 : 1;
  // as many workgroups as run at once (a third more of them: 55 us instead of 51), as long as every wave has a batch
  long long chunks = compute_units() * observe_per_cu(sizeof(E), D) / units;
  const long long most = (tiles + kObserveWaves * KT - 1) / (kObserveWaves * KT);
  chunks = chunks < 1 ? 1 : (chunks > most ? most : chunks);
  p.chunks = (int)chunks;
  hipLaunchKernelGGL((cache_observe_kernel<E, D, KT, kPlace>), dim3((unsigned)(units * chunks)), dim3(kObserveThreads), 0, st, p);
  return launch_ok();
}

template <class E>
static bool launch_observe(const ObserveParams &p, int d, bool place, long long units, hipStream_t st) {
  return d == 64 ? (place ? launch_observe<E, 64, true>(p, units, st) : launch_observe<E, 64, false>(p, units, st))
                 : (place ? launch_observe<E, 128, true>(p, units, st) : launch_observe<E, 128, false>(p, units, st));
}

}  // namespace propd

extern "C" propd_status propd_cache_observe(const propd_tree *tree, propd_dtype dt, int32_t H, int32_t H_kv, int32_t d,
                                            const propd_score_rule *rule, float decay, const int32_t *accept_len,
                                            const int32_t *accept_path, int32_t path_stride, const void *q, const float *lse,
                                            const void *k_cache, const void *k_tree, const int32_t *seq_lens,
                                            const int32_t *dropped, const int32_t *position, const float *weight, int32_t L_max,
                                            int32_t *position_out, float *weight_out, void *hip_stream) {
  using namespace propd;
  if (!tree || tree->B < 1 || tree->T_max < 1 || tree->T_max > PROPD_MAX_TREE || H < 1 || H_kv < 1 || H % H_kv != 0 || L_max < 1 ||
      path_stride < 1 || !score_rule_ok(rule) || !(decay > 0.f) || !(decay <= 1.f) || !tree->n_nodes || !accept_len || !accept_path ||
      !q || !lse || !k_cache || !k_tree || !seq_lens || !weight || !weight_out || !position != !position_out)
    return PROPD_ERR_INVALID_ARG;
  if (dt != PROPD_BF16 && dt != PROPD_F32) return PROPD_ERR_INVALID_ARG;
  if (d != 64 && d != 128) return PROPD_ERR_UNSUPPORTED;
  for (const void *ptr : {q, k_cache, k_tree})
    if (reinterpret_cast<uintptr_t>(ptr) % 16 != 0) return PROPD_ERR_INVALID_ARG;
  const long long units = (long long)tree->B * H_kv;
  if (L_max > (1 << 30) || units > (1ll << 22) || (long long)tree->B * H > (1ll << 24) || (long long)H * tree->T_max > (1ll << 30) || (long long)path_stride * (H / H_kv) > (1ll << 30) || path_stride > kMostPath) return PROPD_ERR_UNSUPPORTED;
  ObserveParams p;
  p.q = q;
  p.k_cache = k_cache;
  p.k_tree = k_tree;
  p.lse = lse;
  p.slopes = rule->slopes;
  p.weight = weight;
  p.seq_lens = seq_lens;
  p.n_nodes = tree->n_nodes;
  p.dropped = dropped;
  p.position = position;
  p.accept_len = accept_len;
  p.accept_path = accept_path;
  p.position_out = position_out;
  p.weight_out = weight_out;
  p.H = H;
  p.H_kv = H_kv;
  p.group = H / H_kv;
  p.T_max = tree->T_max;
  p.L_max = L_max;
  p.path_stride = path_stride;
  p.window = window_of(rule);
  p.scale = rule->scale;
  p.scale_log2e = rule->scale * kLog2e;
  p.cap = rule->cap;
  p.inv_cap = rule->cap > 0.f ? 1.f / rule->cap : 0.f;
  p.decay = decay;
  hipStream_t st = as_stream(hip_stream);
  const bool place = position || rule->window > 0 || rule->slopes;
  const bool ok = dt == PROPD_BF16 ? launch_observe<uint16_t>(p, d, place, units, st) : launch_observe<float>(p, d, place, units, st);
  return ok ? PROPD_OK : PROPD_ERR_DEVICE;
}
