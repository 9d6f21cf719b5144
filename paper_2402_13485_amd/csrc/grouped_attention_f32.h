// Tree attention with shared K/V heads, fp32 operands, fp32 throughout.  Included by grouped_attention.hip inside
// namespace propd.
//
// As in tree_attention_f32.h the fp32 matrix instructions (157 TFLOP/s on the chip) are what has to be fed: a wave owns 16 * QG
// columns of a unit (the nodes of all query heads that read one K/V head, side by side) and walks 16-row tiles of K and V
// straight from memory, four waves take the tiles of a range in turn, and a unit's keys are split over workgroups
// while the chip is not full.  v_mfma_f32_16x16x4_f32 wants row lane % 16, k = lane / 16 and any order of k: a lane loads 16 bytes
// k = 16 c + 4 (lane / 16) .. + 3 of its row.  S^T = K . Q^T leaves a lane the scores of column lane % 16 and keys
// 4 (lane / 16) + r, which are the B operand of O^T += V^T . P^T; block (h, e), row i of O^T stands for d = 64 h + 4 i + e.
#pragma once

constexpr int kF32Waves = 4, kF32Threads = kF32Waves * kWave;
constexpr int kF32Splits = 16;  // ranges of a unit, at most

struct GroupedParamsF32 : GroupedParams {
  const float *qf, *kc, *vc, *kt, *vt;
  float *outf, *part;  // part: [units][column pairs][splits] records of (O [32][D], max [32], sum [32])
  float scale, cap, inv_cap;
  int splits, pairs;
};

__host__ __device__ constexpr size_t grouped_f32_part_floats(int D) { return (size_t)32 * (D + 2); }

// QG groups of 16 columns of one key range of one unit; s_o, s_ml: the workgroup's LDS.
template <int D, int QG, bool kPlace>
__device__ __forceinline__ void grouped_f32_range(const GroupedParamsF32 &p, int unit, int pair, int split, int b, int q0,
                                                  const Lengths &n, float *s_o, float *s_ml, int *s_node) {
  constexpr int kC = D / 16, kH = D / 64, kRow = D + 4;  // chunks of 16 floats; LDS row, padded
  constexpr int kRows = 16 * QG;
  int *s_at = s_node + 32;
  float *s_slope = reinterpret_cast<float *>(s_node + 64);
  float *s_m = s_ml, *s_l = s_ml + kF32Waves * 32;  // [wave][32]
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int c16 = lane & 15, kq = lane >> 4;
  const int L = n.L, T = n.T, columns = p.group * T;
  const bool in_order = p.position == nullptr;
  const int first = kPlace && in_order && L > p.window ? (L - p.window + 1) / 16 : 0;  // tiles that a window hides
  const int n_cache = (L + 15) / 16 - first, n_tiles = n_cache + (T + 15) / 16;
  const int lo = (int)((long long)n_tiles * split / p.splits), hi = (int)((long long)n_tiles * (split + 1) / p.splits);
  const float *kc = p.kc + (size_t)unit * p.L_max * D, *vc = p.vc + (size_t)unit * p.L_max * D;
  const float *kt = p.kt + (size_t)unit * p.T_max * D, *vt = p.vt + (size_t)unit * p.T_max * D;
  const int32_t *place = in_order ? nullptr : p.position + (size_t)unit * p.L_max;
  const uint64_t *anc = p.anc + (size_t)b * p.T_max * 2;
  auto row0_of = [&](int tile) { return 16 * (tile >= n_cache ? tile - n_cache : tile + first); };

  f32x4 kf[kC], vf[4][kH];
  auto load_k = [&](int tile) {
    const bool tree = tile >= n_cache;
    const int j0 = row0_of(tile), last = (tree ? T : L) - 1;
    const int row = j0 + c16 < last ? j0 + c16 : last;  // rows past the end: the last one, masked
    const float *src = (tree ? kt : kc) + (size_t)row * D + 4 * kq;
#pragma unroll
    for (int c = 0; c < kC; ++c) kf[c] = *reinterpret_cast<const f32x4 *>(src + 16 * c);
  };
  auto load_v = [&](int tile) {
    const bool tree = tile >= n_cache;
    const int j0 = row0_of(tile), last = (tree ? T : L) - 1;
    const float *src = (tree ? vt : vc) + 4 * c16;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = j0 + 4 * kq + r < last ? j0 + 4 * kq + r : last;
#pragma unroll
      for (int h = 0; h < kH; ++h) vf[r][h] = *reinterpret_cast<const f32x4 *>(src + (size_t)row * D + 64 * h);
    }
  };
  int tile = lo + wave;
  if (tile < hi) {
    load_k(tile);
    load_v(tile);
  }
  // columns (lanes past the last take the last: valid memory, never stored)
  f32x4 qf[QG][kC];
#pragma unroll
  for (int g = 0; g < QG; ++g) {
    const int column = q0 + 16 * g + c16 < columns ? q0 + 16 * g + c16 : columns - 1;
    const int h = unit % p.H_kv * p.group + column / T, t = column % T;
    const float *src = p.qf + (((size_t)b * p.H + h) * p.T_max + t) * D + 4 * kq;
#pragma unroll
    for (int c = 0; c < kC; ++c) qf[g][c] = *reinterpret_cast<const f32x4 *>(src + 16 * c);
    // what a column needs in every tile, in LDS, registers being short: all waves write the same, each reads what it wrote
    s_node[16 * g + c16] = t;
    if constexpr (kPlace) {
      s_at[16 * g + c16] = n.P + __popcll(anc[2 * t]) + __popcll(anc[2 * t + 1]) - 1;
      s_slope[16 * g + c16] = p.slopes ? p.slopes[h] : 0.f;
    }
  }
  float m_run[QG], l_run[QG];
  f32x4 o[QG][kH][4];
#pragma unroll
  for (int g = 0; g < QG; ++g) {
    m_run[g] = -INFINITY;
    l_run[g] = 0.f;
#pragma unroll
    for (int h = 0; h < kH; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[g][h][e] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  for (; tile < hi; tile += kF32Waves) {
    f32x4 sc[QG];
#pragma unroll
    for (int g = 0; g < QG; ++g) sc[g] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < kC; ++c)
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int g = 0; g < QG; ++g) sc[g] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[c][j], qf[g][c][j], sc[g], 0, 0, 0);
    mfma_settle();
    if (tile + kF32Waves < hi) load_k(tile + kF32Waves);
    const bool tree = tile >= n_cache;
    const int j0 = row0_of(tile), n_valid = (tree ? T : L) - j0;
    int at[4];  // positions of this lane's four keys
    if constexpr (kPlace) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int j = j0 + 4 * kq + r < (tree ? T : L) ? j0 + 4 * kq + r : (tree ? T : L) - 1;
        if (tree) {
          at[r] = n.P + __popcll(anc[2 * j]) + __popcll(anc[2 * j + 1]) - 1;
        } else {
          at[r] = in_order ? n.dropped + j : place[(unsigned)j];
          at[r] = at[r] < n.P ? at[r] : -1;
        }
      }
    }
    float least = INFINITY;
#pragma unroll
    for (int g = 0; g < QG; ++g) {
      const int p_i = kPlace ? s_at[16 * g + c16] : 0;
      const float slope = kPlace ? s_slope[16 * g + c16] : 0.f;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float x = sc[g][r] * p.scale;
        if (p.cap > 0.f) x = capped(x, p.cap, p.inv_cap);
        if constexpr (kPlace)  // (at and window are at most 2^30: no difference wraps into the window)
          x = at[r] >= 0 && (unsigned)(p_i - at[r]) < (unsigned)p.window ? fmaf(-slope, (float)(p_i - at[r]), x) : -INFINITY;
        sc[g][r] = x;
      }
      if (tree || n_valid < 16) {  // uniform
        // rows of the tile that exist and (tree rows) that the query's root path holds
        uint32_t vis = n_valid >= 16 ? 0xffffu : (1u << n_valid) - 1u;
        if (tree) vis &= (uint32_t)(anc[2 * s_node[16 * g + c16] + (j0 >> 6)] >> (j0 & 63));
        vis >>= 4 * kq;
#pragma unroll
        for (int r = 0; r < 4; ++r) sc[g][r] = ((vis >> r) & 1u) ? sc[g][r] : -INFINITY;
      }
      float m_new = fmaxf(fmaxf(sc[g][0], sc[g][1]), fmaxf(sc[g][2], sc[g][3]));
      m_new = fmaxf(m_new, __shfl_xor(m_new, 16, kWave));
      m_new = fmaxf(m_new, __shfl_xor(m_new, 32, kWave));
      m_new = fmaxf(m_new, m_run[g]);
      const float m_safe = m_new == -INFINITY ? 0.f : m_new;  // nothing visible so far: weights 0
      const float alpha = fast_exp2((m_run[g] - m_safe) * kLog2e);
      m_run[g] = m_new;
      float sum = 0.f;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        sc[g][r] = fast_exp2((sc[g][r] - m_safe) * kLog2e);  // the difference first: it rounds less than the parts would
        sum += sc[g][r];
        least = fminf(least, sc[g][r]);
      }
      l_run[g] = l_run[g] * alpha + sum;
#pragma unroll
      for (int h = 0; h < kH; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int r = 0; r < 4; ++r) o[g][h][e][r] *= alpha;
    }
    if (__ballot(least < 0x1p-126f) != 0) {  // weights of zero: V is looked through, see not_finite_sum
      uint32_t top = 0;
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int h = 0; h < kH; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t twice = __float_as_uint(vf[r][h][e]) << 1;
            top = twice > top ? twice : top;
          }
      if (__ballot(top >= 0xff000000u) != 0) {
#pragma unroll
        for (int h = 0; h < kH; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
#pragma unroll
            for (int g = 0; g < QG; ++g) {
              f32x4 codes = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int r = 0; r < 4; ++r)
                codes = __builtin_amdgcn_mfma_f32_16x16x4f32(not_finite_code(__float_as_uint(vf[r][h][e])),
                                                             sc[g][r] != 0.f ? 1.f : 0.f, codes, 0, 0, 0);
              mfma_settle();
#pragma unroll
              for (int r = 0; r < 4; ++r) o[g][h][e][r] += not_finite_sum(codes[r]);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r)
              vf[r][h][e] = not_finite_code(__float_as_uint(vf[r][h][e])) != 0.f ? 0.f : vf[r][h][e];
          }
      }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int h = 0; h < kH; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int g = 0; g < QG; ++g)
            o[g][h][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[r][h][e], sc[g][r], o[g][h][e], 0, 0, 0);
    mfma_settle();
    if (tile + kF32Waves < hi) load_v(tile + kF32Waves);
  }

  // ---- merge the four waves: O[column][d = 64 h + 16 kq + 4 r + e]
#pragma unroll
  for (int g = 0; g < QG; ++g) {
#pragma unroll
    for (int h = 0; h < kH; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const f32x4 v = {o[g][h][0][r], o[g][h][1][r], o[g][h][2][r], o[g][h][3][r]};
        *reinterpret_cast<f32x4 *>(s_o + (wave * kRows + 16 * g + c16) * kRow + 64 * h + 16 * kq + 4 * r) = v;
      }
    float l = l_run[g];
    l += __shfl_xor(l, 16, kWave);
    l += __shfl_xor(l, 32, kWave);
    if (kq == 0) {
      s_m[wave * 32 + 16 * g + c16] = m_run[g];
      s_l[wave * 32 + 16 * g + c16] = l;
    }
  }
  __syncthreads();
  // thread -> column tid / LPQ, every LPQ-th 16-byte piece of its row
  constexpr int LPQ = kF32Threads / (16 * QG), kPieces = D / 4 / LPQ;
  const int row = threadIdx.x / LPQ, part = threadIdx.x % LPQ, column = q0 + row;
  float M = -INFINITY, total = 0.f, f[kF32Waves];
#pragma unroll
  for (int w = 0; w < kF32Waves; ++w) M = fmaxf(M, s_m[w * 32 + row]);
  const float m_safe = M == -INFINITY ? 0.f : M;
#pragma unroll
  for (int w = 0; w < kF32Waves; ++w) {
    f[w] = fast_exp2((s_m[w * 32 + row] - m_safe) * kLog2e);
    total += s_l[w * 32 + row] * f[w];
  }
  f32x4 acc[kPieces];
#pragma unroll
  for (int x = 0; x < kPieces; ++x) {
    acc[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kF32Waves; ++w) {
      const f32x4 v = *reinterpret_cast<const f32x4 *>(s_o + (w * kRows + row) * kRow + 4 * (part + LPQ * x));
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[x][j] += counted(v[j], f[w]) * f[w];
    }
  }
  if (p.splits == 1) {
    if (column >= columns) return;
    const size_t at_row = column_row(p, b, unit % p.H_kv, column, T);
#pragma unroll
    for (int x = 0; x < kPieces; ++x) {
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[x][j] = total == 0.f ? 0.f : acc[x][j] / total;
      *reinterpret_cast<f32x4 *>(p.outf + at_row * D + 4 * (part + LPQ * x)) = acc[x];
    }
    if (p.lse && part == 0) p.lse[at_row] = M + logf(total);
    return;
  }
  float *rec = p.part + (((size_t)unit * p.pairs + pair) * p.splits + split) * grouped_f32_part_floats(D);
#pragma unroll
  for (int x = 0; x < kPieces; ++x) *reinterpret_cast<f32x4 *>(rec + row * D + 4 * (part + LPQ * x)) = acc[x];
  if (part == 0) {
    rec[32 * D + row] = M;
    rec[32 * D + 32 + row] = total;
  }
}

// One workgroup per (unit, 32 columns, split).  MQ: groups of 16 columns it may find (1 when there are at most 16).
template <int D, int MQ, bool kPlace>
__global__ __launch_bounds__(kF32Threads, 2) void grouped_attn_f32_kernel(GroupedParamsF32 p) {
  __shared__ __attribute__((aligned(16))) float s_o[kF32Waves * 16 * MQ * (D + 4)];
  __shared__ float s_ml[2 * kF32Waves * 32];
  __shared__ int s_node[3 * 32];  // of each column: node, position, slope
  // the column groups of one key range run on one XCD where the counts allow (its L2 holds the rows)
  const unsigned units = (unsigned)p.B * (unsigned)p.H_kv, per_pair = units * (unsigned)p.splits;
  const unsigned long long block = (unsigned long long)blockIdx.y * gridDim.x + blockIdx.x;
  if (block >= (unsigned long long)per_pair * p.pairs) return;  // the last row of the grid need not be full
  const int pair = (int)(block / per_pair);
  const unsigned us = (unsigned)(block - (unsigned long long)pair * per_pair);
  const int unit = (int)(us / (unsigned)p.splits), split = (int)(us - (unsigned)unit * (unsigned)p.splits);
  const int b = unit / p.H_kv, q0 = 32 * pair;
  const Lengths n = lengths_of(p, b);
  if (q0 >= p.group * n.T) return;
  if (MQ == 1 || q0 + 16 >= p.group * n.T) grouped_f32_range<D, 1, kPlace>(p, unit, pair, split, b, q0, n, s_o, s_ml, s_node);
  else grouped_f32_range<D, MQ, kPlace>(p, unit, pair, split, b, q0, n, s_o, s_ml, s_node);
}

// Units split over workgroups: as grouped_attn_merge_kernel, all of a thread's pieces requested before the first is
// used.  One thread per 16 bytes of the result.
template <int D>
__global__ __launch_bounds__(kF32Threads) void grouped_attn_f32_merge_kernel(GroupedParamsF32 p) {
  constexpr int LPQ = D / 4, kRows = kF32Threads / LPQ, kBlocks = 32 / kRows;
  const unsigned up = blockIdx.x / kBlocks;
  const int unit = (int)(up / (unsigned)p.pairs), pair = (int)(up - (unsigned)unit * (unsigned)p.pairs);
  const int b = unit / p.H_kv;
  int T = p.n_nodes[b];
  T = T < 1 ? 1 : (T > p.T_max ? p.T_max : T);
  const int columns = p.group * T;
  const int row = (blockIdx.x % kBlocks) * kRows + threadIdx.x / LPQ, part = threadIdx.x % LPQ, column = 32 * pair + row;
  if (32 * pair + (int)(blockIdx.x % kBlocks) * kRows >= columns) return;  // uniform
  // (columns beyond the last within its group of 16 have partial results too; beyond that nobody wrote any)
  const int safe = column < columns ? row : 0;
  const float *rec = p.part + (size_t)up * p.splits * grouped_f32_part_floats(D);
  f32x4 v[kF32Splits];
  float m[kF32Splits], l[kF32Splits];
#pragma unroll
  for (int s = 0; s < kF32Splits; ++s) {
    const float *q = rec + (s < p.splits ? s : 0) * grouped_f32_part_floats(D);
    v[s] = *reinterpret_cast<const f32x4 *>(q + safe * D + 4 * part);
    m[s] = q[32 * D + safe];
    l[s] = q[32 * D + 32 + safe];
  }
  float M = -INFINITY;
#pragma unroll
  for (int s = 0; s < kF32Splits; ++s) M = fmaxf(M, m[s]);  // past the last split: the first once more
  const float m_safe = M == -INFINITY ? 0.f : M;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  float total = 0.f;
#pragma unroll
  for (int s = 0; s < kF32Splits; ++s) {
    if (s < p.splits) {  // uniform
      const float f = fast_exp2((m[s] - m_safe) * kLog2e);
      total += l[s] * f;
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] += counted(v[s][j], f) * f;
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) acc[j] = total == 0.f ? 0.f : acc[j] / total;
  if (column >= columns) return;
  const size_t at_row = column_row(p, b, unit % p.H_kv, column, T);
  *reinterpret_cast<f32x4 *>(p.outf + at_row * D + 4 * part) = acc;
  if (p.lse && part == 0) p.lse[at_row] = M + logf(total);
}

// Ranges per unit and 32 columns.  The matrix instructions are the bound, a workgroup keeps all four of a compute unit's busy with
// one wave each, and workgroups that share it take turns: the time is the number of workgroups per compute unit times (the
// rounds of tiles of a wave, about 2 us each at d = 128, and two rounds' worth of first loads and merging), and another
// round for the merge kernel (whose grid has room for 2^16 of them).  2 x 4 units of 192 columns x 1024 keys: 8 ranges (384 workgroups) 26 us, 5 (240) 23.5.
static int grouped_f32_splits(long long base, int tiles, int cus, long long room) {
  long long best = 1, least = 1ll << 62;
  for (long long s = 1; s <= kF32Splits && s <= room && s <= tiles && (s == 1 || base < (1 << 16)); ++s) {
    const long long rounds = (tiles + kF32Waves * s - 1) / (kF32Waves * s);
    const long long cost = (base * s + cus - 1) / cus * (rounds + 2) + (s > 1 ? 1 : 0);
    if (cost < least) {
      least = cost;
      best = s;
    }
  }
  return (int)best;
}

template <int D, bool kPlace>
static bool launch_grouped_f32(GroupedParamsF32 p, size_t workspace_bytes, hipStream_t st) {
  const long long units = (long long)p.B * p.H_kv, base = units * p.pairs;
  const int tiles = (int)((p.L_max + 15ll) / 16) + (p.T_max + 15) / 16;
  // (of what propd_workspace_bytes asks for: a caller who gives more gets the same bits)
  const long long room = (long long)(workspace_bytes / (grouped_f32_part_floats(D) * 4)) / base;
  p.splits = grouped_f32_splits(base, tiles, compute_units(), room);
  // a dimension of the grid holds fewer than 2^32 threads
  constexpr long long kGridX = 1ll << 22;
  const long long blocks = base * p.splits;
  const dim3 grid((unsigned)(blocks < kGridX ? blocks : kGridX), (unsigned)((blocks + kGridX - 1) / kGridX));
  if (p.group * p.T_max <= 16)
    hipLaunchKernelGGL((grouped_attn_f32_kernel<D, 1, kPlace>), grid, dim3(kF32Threads), 0, st, p);
  else
    hipLaunchKernelGGL((grouped_attn_f32_kernel<D, 2, kPlace>), grid, dim3(kF32Threads), 0, st, p);
  if (!launch_ok()) return false;
  if (p.splits == 1) return true;
  constexpr unsigned kBlocks = 32 / (kF32Threads / (D / 4));
  hipLaunchKernelGGL(grouped_attn_f32_merge_kernel<D>, dim3((unsigned)base * kBlocks), dim3(kF32Threads), 0, st, p);
  return launch_ok();
}

static bool launch_grouped_f32(const GroupedParams &common, float scale, float cap, int d, bool place, void *workspace,
                               size_t workspace_bytes, hipStream_t st) {
  GroupedParamsF32 p;
  static_cast<GroupedParams &>(p) = common;
  p.qf = reinterpret_cast<const float *>(common.q);
  p.kc = reinterpret_cast<const float *>(common.k_cache);
  p.vc = reinterpret_cast<const float *>(common.v_cache);
  p.kt = reinterpret_cast<const float *>(common.k_tree);
  p.vt = reinterpret_cast<const float *>(common.v_tree);
  p.outf = reinterpret_cast<float *>(common.out);
  p.part = reinterpret_cast<float *>(workspace);
  p.scale = scale;
  p.cap = cap;
  p.inv_cap = cap > 0.f ? 1.f / cap : 0.f;
  p.pairs = (p.group * p.T_max + 31) / 32;
  return d == 64 ? (place ? launch_grouped_f32<64, true>(p, workspace_bytes, st) : launch_grouped_f32<64, false>(p, workspace_bytes, st))
                 : (place ? launch_grouped_f32<128, true>(p, workspace_bytes, st) : launch_grouped_f32<128, false>(p, workspace_bytes, st));
}
