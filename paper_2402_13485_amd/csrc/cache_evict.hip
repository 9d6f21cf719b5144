// Eviction from a cache by accumulated attention weight: every K/V head of a sequence keeps its `budget` best rows, and
// the kept rows that lie beyond move into the places that became free.  Rows need no order (each has its position), so no other
// row moves: K and V bytes are two times the rows that move, nothing in a sequence that is not too long.
//
// cache_select_kernel, one workgroup per (sequence, K/V head).  Rows are ranked by a 32-bit key (rank_key), and the budget-th
// largest key is found in four passes over the keys, which stay in registers: 6.1 us for 1032 rows, 24 us for 8192 (counting by ballots
// instead, two bits at a time, took 2.5 and 4 us longer).  Wave w owns rows w * share .. in order, so that all that
// depends on the order (which of the equal keys stay, the lists of free places and of rows that move) takes a prefix over
// the waves' totals and one within the wave.  No result depends on the order of the additions in LDS.
// cache_move_kernel moves what the lists say, spread over the chip, and writes the new lengths: nobody reads them any more.
#include "score_rule.h"

namespace propd {

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / kWave;
constexpr int kMoveThreads = 256;

struct EvictParams {
  const int32_t *seq_lens, *dropped, *position;
  const float *weight;
  int32_t *seq_lens_out, *dropped_out, *position_out;
  float *weight_out;
  unsigned char *k_cache, *v_cache;
  int32_t *lists;  // [units][2][room]: free places, rows that move
  int32_t *moves;  // [units]: how many
  int32_t *left;   // [B][2]: new length, new dropped
  int B, H_kv, L_max, budget, recent, sinks, room, row_bytes, parts;
};

// The order of rows as a number, larger first: protected rows, weights, everything else (see propd.h).
__device__ __forceinline__ uint32_t rank_key(float weight, int position, int next, int recent, int sinks) {
  if (position < 0) return 0u;
  // (64-bit: next - recent may be far below zero)
  if ((long long)position >= (long long)next - recent || position < sinks) return ~0u;
  const uint32_t bits = __float_as_uint(weight == 0.f ? 0.f : weight);  // -0 counts as 0
  if (!(weight > -INFINITY)) return 0u;                                 // NaN too
  return bits >> 31 ? ~bits : bits | 0x80000000u;
}

// KEYS: keys of a thread that stay in registers; 0: read again for every pass.
template <int KEYS>
__global__ __launch_bounds__(kSelectThreads) void cache_select_kernel(EvictParams p) {
  __shared__ int s_bins[4][256];
  __shared__ int s_total[3][kSelectWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int unit = blockIdx.x, b = unit / p.H_kv;
  const Lengths n = lengths_of(p.seq_lens, nullptr, p.dropped, p.L_max, 1, b);
  const int L = n.L, budget = p.budget;
  const size_t base = (size_t)unit * p.L_max;
  const float *weight = p.weight + base;
  const int32_t *position = p.position + base;
  const bool elsewhere = p.weight_out != p.weight || p.position_out != p.position;
  if (tid == 0 && unit == b * p.H_kv) {
    const int over = L > budget ? L - budget : 0;
    p.left[2 * b] = L - over;
    p.left[2 * b + 1] = n.dropped + over;
  }
  if (L <= budget) {
    if (tid == 0) p.moves[unit] = 0;
    if (elsewhere)
      for (int j = tid; j < L; j += kSelectThreads) {
        p.weight_out[base + j] = weight[j];
        p.position_out[base + j] = position[j];
      }
    return;
  }
  // rows of this wave: start + 64 i + lane, i < rounds
  const int share = (L + kSelectThreads - 1) / kSelectThreads * kWave, start = wave * share;
  const int rounds = share / kWave;  // at most KEYS where that is not 0
  auto key_at = [&](int i) -> uint32_t {
    const int j = start + kWave * i + lane;
    return j < L ? rank_key(weight[j], position[j], n.P, p.recent, p.sinks) : 0u;
  };
  uint32_t keys[KEYS ? KEYS : 1];
  if constexpr (KEYS > 0) {
#pragma unroll
    for (int i = 0; i < KEYS; ++i) keys[i] = i < rounds ? key_at(i) : 0u;
  }
  auto for_keys = [&](auto &&f) __attribute__((always_inline)) {
    if constexpr (KEYS > 0) {
#pragma unroll
      for (int i = 0; i < KEYS; ++i)
        if (i < rounds) f(i, keys[i]);  // uniform
    } else {
      for (int i = 0; i < rounds; ++i) f(i, key_at(i));
    }
  };

  // ---- the budget-th largest key, eight bits at a time: how many of the keys that share the bits found so far have which
  //      next eight.  Lanes that would all add to one bin (weights alike) add once.
  uint32_t threshold = 0u;
  int above = 0;  // keys > threshold
  for (int i = tid; i < 4 * 256; i += kSelectThreads) s_bins[0][i] = 0;
  __syncthreads();
#pragma unroll 1
  for (int turn = 0; turn < 4; ++turn) {
    const int shift = 24 - 8 * turn;
    for_keys([&](int i, uint32_t key) __attribute__((always_inline)) {
      const bool mine = start + kWave * i + lane < L && (turn == 0 || (key ^ threshold) >> (shift + 8) == 0u);
      const uint64_t who = __ballot(mine);
      if (who == 0) return;
      const int bin = (int)(key >> shift & 255u);
      const int one = __builtin_amdgcn_readlane(bin, __builtin_ctzll(who));
      if (__ballot(mine && bin != one) == 0) {
        if (lane == 0) atomicAdd(&s_bins[turn][one], __popcll(who));
      } else if (mine) {
        atomicAdd(&s_bins[turn][bin], 1);
      }
    });
    __syncthreads();
    // Lane l has bins 255 - 4 l and the three below: counts from the top, by every wave for itself.
    const int top = 255 - 4 * lane;
    int c[4], sum = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) sum += c[k] = s_bins[turn][top - k];
    int upto = sum;  // of this lane's bins and those above
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x111, 0xf, 0xf, false);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x112, 0xf, 0xf, false);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x114, 0xf, 0xf, false);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x118, 0xf, 0xf, false);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x142, 0xa, 0xf, false);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x143, 0xc, 0xf, false);
    const int wanted = budget - above;  // the wanted-th of these keys from the top
    const int holder = __builtin_ctzll(__ballot(upto >= wanted));
    int before = upto - sum, bin = top, in_bin = c[0];
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (before + c[k] < wanted && bin == top - k) {
        before += c[k];
        bin = top - k - 1;
        in_bin = c[k + 1];
      }
    above += __builtin_amdgcn_readlane(before, holder);
    threshold |= (uint32_t)__builtin_amdgcn_readlane(bin, holder) << shift;
    if (above + __builtin_amdgcn_readlane(in_bin, holder) == budget) {  // all keys from here on stay, and no others
      threshold -= 1u;  // (not from 0: fewer keys stay than there are)
      above = budget;
      break;
    }
  }

  // ---- which of the keys equal to the threshold stay: the first ones
  auto sum_before = [&](int which) {  // of the waves in front of this one
    int x = s_total[which][lane & 15];
    x = (lane & 15) < wave ? x : 0;
    x += __builtin_amdgcn_update_dpp(0, x, 0x128, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x124, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x122, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x121, 0xf, 0xf, false);
    return __builtin_amdgcn_readfirstlane(x);
  };
  const uint64_t below = (1ull << lane) - 1ull;
  const int wanted = budget - above;
  int equal = 0;
  for_keys([&](int i, uint32_t key) __attribute__((always_inline)) {
    equal += __popcll(__ballot(start + kWave * i + lane < L && key == threshold));
  });
  if (lane == 0) s_total[0][wave] = equal;
  __syncthreads();
  const int equal_before = sum_before(0);
  auto for_rows = [&](auto &&f) __attribute__((always_inline)) {  // f(row, whether it is kept)
    int seen = equal_before;
    for_keys([&](int i, uint32_t key) __attribute__((always_inline)) {
      const int j = start + kWave * i + lane;
      const uint64_t same = __ballot(j < L && key == threshold);
      f(j, j < L && (key > threshold || (key == threshold && seen + __popcll(same & below) < wanted)));
      seen += __popcll(same);
    });
  };
  // ---- free places below the budget and kept rows beyond it, both in rising order
  int holes = 0, late = 0;
  for_rows([&](int j, bool keep) __attribute__((always_inline)) {
    holes += __popcll(__ballot(j < budget && !keep));
    late += __popcll(__ballot(j >= budget && keep));
  });
  if (lane == 0) {
    s_total[1][wave] = holes;
    s_total[2][wave] = late;
  }
  __syncthreads();
  int hole = sum_before(1), row = sum_before(2);
  int32_t *const free_places = p.lists + (size_t)unit * 2 * p.room, *const moving = free_places + p.room;
  for_rows([&](int j, bool keep) __attribute__((always_inline)) {
    const uint64_t h = __ballot(j < budget && !keep), m = __ballot(j >= budget && keep);
    if (j < budget && !keep) free_places[hole + __popcll(h & below)] = j;
    if (j >= budget && keep) moving[row + __popcll(m & below)] = j;
    if (elsewhere && j < budget && keep) {
      p.weight_out[base + j] = weight[j];
      p.position_out[base + j] = position[j];
    }
    hole += __popcll(h);
    row += __popcll(m);
  });
  if (tid == kSelectThreads - 1) p.moves[unit] = row;  // the last wave's end
}

// One workgroup per (unit, part): rows part, part + parts, ... in blocks, 16 bytes per thread, K and V of two rows requested together.
__global__ __launch_bounds__(kMoveThreads) void cache_move_kernel(EvictParams p) {
  const int unit = blockIdx.x / p.parts, part = blockIdx.x - unit * p.parts, b = unit / p.H_kv;
  const int count = p.moves[unit];
  if (threadIdx.x == 0 && part == 0 && unit == b * p.H_kv) {
    p.seq_lens_out[b] = p.left[2 * b];
    p.dropped_out[b] = p.left[2 * b + 1];
  }
  const int32_t *const free_places = p.lists + (size_t)unit * 2 * p.room, *const moving = free_places + p.room;
  const size_t base = (size_t)unit * p.L_max;
  for (int k = part * kMoveThreads + threadIdx.x; k < count; k += p.parts * kMoveThreads) {
    const size_t to = base + free_places[k], from = base + moving[k];
    p.weight_out[to] = p.weight[from];
    p.position_out[to] = p.position[from];
  }
  const uint32_t pieces = (uint32_t)p.row_bytes / 16u, items = (uint32_t)count * pieces, step = (uint32_t)p.parts * kMoveThreads;
  for (uint32_t item = (uint32_t)part * kMoveThreads + threadIdx.x; item < items; item += 2u * step) {
    const bool two = items - item > step;
    const uint32_t other = two ? item + step : item, k0 = item / pieces, k1 = other / pieces;
    const uint32_t c0 = (item - k0 * pieces) * 16u, c1 = (other - k1 * pieces) * 16u;
    const size_t from0 = (base + moving[k0]) * p.row_bytes + c0, to0 = (base + free_places[k0]) * p.row_bytes + c0;
    const size_t from1 = (base + moving[k1]) * p.row_bytes + c1, to1 = (base + free_places[k1]) * p.row_bytes + c1;
    const u32x4 ka = *reinterpret_cast<const u32x4 *>(p.k_cache + from0), va = *reinterpret_cast<const u32x4 *>(p.v_cache + from0);
    const u32x4 kb = *reinterpret_cast<const u32x4 *>(p.k_cache + from1), vb = *reinterpret_cast<const u32x4 *>(p.v_cache + from1);
    *reinterpret_cast<u32x4 *>(p.k_cache + to0) = ka;
    *reinterpret_cast<u32x4 *>(p.v_cache + to0) = va;
    if (two) {
      *reinterpret_cast<u32x4 *>(p.k_cache + to1) = kb;
      *reinterpret_cast<u32x4 *>(p.v_cache + to1) = vb;
    }
  }
}

// A sequence of L rows moves at most min(budget, L - budget) of them per head.
static int evict_room(int L_max) { return L_max / 2 + 1; }

size_t cache_evict_workspace_bytes(int B, int H_kv, int L_max) {
  const size_t units = (size_t)B * H_kv;
  return align_up(units * 2 * evict_room(L_max) * 4, 256) + align_up(units * 4, 256) + align_up((size_t)B * 8, 256);
}

}  // namespace propd

extern "C" propd_status propd_cache_evict(int32_t B, propd_dtype dt, int32_t H_kv, int32_t d, int32_t L_max, int32_t budget,
                                          int32_t recent, int32_t sinks, void *k_cache, void *v_cache,
                                          const propd_cache_rows *rows, const propd_cache_rows *rows_out, void *workspace,
                                          size_t workspace_bytes, void *hip_stream) {
  using namespace propd;
  if (B < 1 || H_kv < 1 || d < 1 || L_max < 1 || budget < 1 || budget > L_max || recent < 0 || sinks < 0 || !k_cache || !v_cache)
    return PROPD_ERR_INVALID_ARG;
  for (const propd_cache_rows *r : {rows, rows_out})
    if (!r || !r->seq_lens || !r->dropped || !r->position || !r->weight) return PROPD_ERR_INVALID_ARG;
  if (dt != PROPD_BF16 && dt != PROPD_F32) return PROPD_ERR_INVALID_ARG;
  const long long row_bytes = (long long)d * (dt == PROPD_BF16 ? 2 : 4);
  if (row_bytes % 16 != 0 || row_bytes > (1 << 20)) return PROPD_ERR_UNSUPPORTED;
  for (const void *ptr : {(const void *)k_cache, (const void *)v_cache, (const void *)workspace})
    if (reinterpret_cast<uintptr_t>(ptr) % 16 != 0) return PROPD_ERR_INVALID_ARG;
  const long long units = (long long)B * H_kv;
  // (2^28 pieces of 16 bytes: indices of rows and pieces stay below 2^31)
  if (units > (1ll << 20) || (L_max / 2 + 1ll) * (row_bytes / 16) > (1ll << 28)) return PROPD_ERR_UNSUPPORTED;
  if (!workspace || workspace_bytes < cache_evict_workspace_bytes(B, H_kv, L_max)) return PROPD_ERR_WORKSPACE;
  hipStream_t st = as_stream(hip_stream);
  EvictParams p;
  p.seq_lens = rows->seq_lens;
  p.dropped = rows->dropped;
  p.position = rows->position;
  p.weight = rows->weight;
  p.seq_lens_out = rows_out->seq_lens;
  p.dropped_out = rows_out->dropped;
  p.position_out = rows_out->position;
  p.weight_out = rows_out->weight;
  p.k_cache = reinterpret_cast<unsigned char *>(k_cache);
  p.v_cache = reinterpret_cast<unsigned char *>(v_cache);
  p.B = B;
  p.H_kv = H_kv;
  p.L_max = L_max;
  p.budget = budget;
  p.recent = recent;
  p.sinks = sinks;
  p.room = evict_room(L_max);
  p.row_bytes = (int)row_bytes;
  char *ws = reinterpret_cast<char *>(workspace);
  p.lists = reinterpret_cast<int32_t *>(ws);
  ws += align_up((size_t)units * 2 * p.room * 4, 256);
  p.moves = reinterpret_cast<int32_t *>(ws);
  ws += align_up((size_t)units * 4, 256);
  p.left = reinterpret_cast<int32_t *>(ws);
  // Keys in registers for as long as the registers last.  Read again for every pass: 1032 rows 7.6 us instead of 6.1, 8192 34 instead of 24.
  const dim3 grid((unsigned)units), threads(kSelectThreads);
  if (L_max <= 4 * kSelectThreads) hipLaunchKernelGGL((cache_select_kernel<4>), grid, threads, 0, st, p);
  else if (L_max <= 16 * kSelectThreads) hipLaunchKernelGGL((cache_select_kernel<16>), grid, threads, 0, st, p);
  else hipLaunchKernelGGL((cache_select_kernel<0>), grid, threads, 0, st, p);
  if (!launch_ok()) return PROPD_ERR_DEVICE;
  // As many workgroups as fill the chip several times (1024 or 16384 in all take as long), no more than the most rows that can
  // move give work.
  const long long most = (long long)(budget < L_max - budget ? budget : L_max - budget) * (row_bytes / 16);
  long long parts = (4096 + units - 1) / units;
  if (parts > (most + kMoveThreads - 1) / kMoveThreads) parts = (most + kMoveThreads - 1) / kMoveThreads;
  p.parts = parts < 1 ? 1 : (int)parts;
  hipLaunchKernelGGL(cache_move_kernel, dim3((unsigned)(units * p.parts)), dim3(kMoveThreads), 0, st, p);
  return launch_ok() ? PROPD_OK : PROPD_ERR_DEVICE;
}
