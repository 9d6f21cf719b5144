// What the accepted nodes of a step paid to every row of a cache: paid[j] = sum of exp(s_rj - lse_r) over the
// accepted nodes and the query heads that share the K/V head; the rows' weights decay and take it up.
//
// One pass over K (a softmax needs two, but the attention has left lse), bound by its bytes: a wave owns KT tiles of 16 keys and keeps
// their rows in registers as the B operand of S = Q . K^T (16x16 products), the accepted queries come 16 at a time as the A
// operand, from the L2.  A lane then holds four queries' scores of one key, adds their weights up, and the
// four lanes of a key meet at the end.  Rows are read straight from memory in the operand's layout, 64 bytes of 16 rows per load.
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
  float scale, cap, inv_cap, decay;
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

template <class E, int D, int KT>
__global__ __launch_bounds__(kObserveThreads) void cache_observe_kernel(ObserveParams p) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c16 = lane & 15, part = lane >> 4;
  const int unit = (int)(blockIdx.x / (unsigned)p.chunks), chunk = (int)(blockIdx.x - (unsigned)unit * (unsigned)p.chunks);
  const int b = unit / p.H_kv, hk = unit - b * p.H_kv;
  const Lengths n = lengths_of(p.seq_lens, p.n_nodes, p.dropped, p.L_max, p.T_max, b);
  int a = p.accept_len[b];
  a = a < 0 ? 0 : (a > p.path_stride ? p.path_stride : a);
  const int32_t *path = p.accept_path + (size_t)b * p.path_stride;
  const int cached = (n.L + 15) / 16, tiles = cached + (a + 15) / 16;
  const int tile0 = (chunk * kObserveWaves + wave) * KT;
  if (tile0 >= tiles) return;
  const E *q = reinterpret_cast<const E *>(p.q), *k_cache = reinterpret_cast<const E *>(p.k_cache) + (size_t)unit * p.L_max * D;
  const E *k_tree = reinterpret_cast<const E *>(p.k_tree) + (size_t)unit * p.T_max * D;

  // ---- this lane's keys: tile t is 16 cached rows, or 16 places of the path.  Keys past the last take a valid row.
  Rows<E, D> keys[KT];
  int key[KT], at[KT];  // place in its kind (-1: none), position
#pragma unroll
  for (int x = 0; x < KT; ++x) {
    const int t = tile0 + x < tiles ? tile0 + x : tiles - 1;
    if (t < cached) {
      const int j = 16 * t + c16, row = j < n.L ? j : n.L - 1;
      key[x] = tile0 + x < tiles && j < n.L ? j : -1;
      at[x] = p.position ? p.position[(size_t)unit * p.L_max + row] : n.dropped + row;
      keys[x].load(k_cache + (size_t)row * D, part);
    } else {
      const int r = 16 * (t - cached) + c16, node = path[r < a ? r : a - 1];
      key[x] = tile0 + x < tiles && r < a ? r : -1;
      const bool valid = node >= 0 && node < n.T;
      at[x] = valid ? n.P + r : -1;
      keys[x].load(k_tree + (size_t)(valid ? node : 0) * D, part);
    }
  }
  float paid[KT];
#pragma unroll
  for (int x = 0; x < KT; ++x) paid[x] = 0.f;

  const int rows = a * p.group;  // row = place on the path * group + head
  for (int row0 = 0; row0 < rows; row0 += 16) {
    Rows<E, D> queries;
    {
      const int row = row0 + c16 < rows ? row0 + c16 : rows - 1, r = row / p.group, head = row - r * p.group;
      int node = path[r];
      node = node >= 0 && node < n.T ? node : 0;
      queries.load(q + (((size_t)b * p.H + hk * p.group + head) * p.T_max + node) * D, part);
    }
    // the four queries whose scores this lane gets
    float lse[4], slope[4];
    Sight sight[4];
    int place[4];  // on the path; -1: no query
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = row0 + 4 * part + j, r = row < rows ? row / p.group : 0, head = row < rows ? row - r * p.group : 0;
      const int node = path[r];
      const bool valid = row < rows && node >= 0 && node < n.T;
      place[j] = valid ? r : -1;
      const size_t h = (size_t)hk * p.group + head;
      lse[j] = p.lse[((size_t)b * p.H + h) * p.T_max + (valid ? node : 0)];
      slope[j] = p.slopes ? p.slopes[h] : 0.f;
      sight[j] = sight_of(n.P + r, p.window);
    }
#pragma unroll
    for (int x = 0; x < KT; ++x) {
      const f32x4 raw = queries.times(keys[x]);
      mfma_settle();
      const bool own = tile0 + x >= cached;  // a key of the path
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float s = raw[j] * p.scale;
        if (p.cap > 0.f) s = capped(s, p.cap, p.inv_cap);
        s = fmaf(-slope[j], (float)(sight[j].p_i - at[x]), s);
        const float w = __builtin_amdgcn_exp2f((s - lse[j]) * kLog2e);
        const bool seen = place[j] >= 0 && in_sight(sight[j], at[x]) && (own ? key[x] <= place[j] : at[x] < n.P);
        paid[x] += seen ? w : 0.f;
      }
    }
  }

  // ---- the four lanes of a key; lanes of part x write tile x
#pragma unroll
  for (int x = 0; x < KT; ++x) {
    paid[x] += __shfl_xor(paid[x], 16, kWave);
    paid[x] += __shfl_xor(paid[x], 32, kWave);
  }
#pragma unroll
  for (int x = 0; x < KT; ++x) {
    if (part != x || key[x] < 0) continue;
    const size_t base = (size_t)unit * p.L_max;
    if (tile0 + x < cached) {
      const size_t i = base + key[x];
      p.weight_out[i] = p.decay * p.weight[i] + paid[x];
      if (p.position_out) p.position_out[i] = at[x];
    } else if (n.L + key[x] < p.L_max) {
      const size_t i = base + n.L + key[x];
      p.weight_out[i] = at[x] < 0 ? 0.f : paid[x];
      if (p.position_out) p.position_out[i] = at[x];
    }
  }
}

template <class E, int D>
static bool launch_observe(ObserveParams p, long long units, hipStream_t st) {
  const long long tiles = (p.L_max + 15ll) / 16 + (p.path_stride + 15ll) / 16;
  constexpr int kMany = sizeof(E) == 2 ? 4 : 2;
  // several tiles per wave once the chip is full of waves without
  const bool many = units * tiles > 8192ll;
  const int per = kObserveWaves * (many ? kMany : 1);
  const long long chunks = (tiles + per - 1) / per;
  p.chunks = (int)chunks;
  const dim3 grid((unsigned)(units * chunks));
  if (many) hipLaunchKernelGGL((cache_observe_kernel<E, D, kMany>), grid, dim3(kObserveThreads), 0, st, p);
  else hipLaunchKernelGGL((cache_observe_kernel<E, D, 1>), grid, dim3(kObserveThreads), 0, st, p);
  return launch_ok();
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
  if ((long long)tree->B * H > (1ll << 24) || (long long)path_stride * (H / H_kv) > (1ll << 30)) return PROPD_ERR_UNSUPPORTED;
  // (a workgroup takes 8 tiles at least where there are many)
  if (units * ((L_max + 15ll) / 16 + (path_stride + 15ll) / 16) > (1ll << 26)) return PROPD_ERR_UNSUPPORTED;
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
  p.cap = rule->cap;
  p.inv_cap = rule->cap > 0.f ? 1.f / rule->cap : 0.f;
  p.decay = decay;
  hipStream_t st = as_stream(hip_stream);
  const bool ok = dt == PROPD_BF16 ? (d == 64 ? launch_observe<uint16_t, 64>(p, units, st) : launch_observe<uint16_t, 128>(p, units, st))
                                   : (d == 64 ? launch_observe<float, 64>(p, units, st) : launch_observe<float, 128>(p, units, st));
  return ok ? PROPD_OK : PROPD_ERR_DEVICE;
}
