// Acceptance by sampling: drafted tokens against the target's probabilities, with given random numbers.
//
// Two kernels, and a third in front of the last where candidates were drawn:
//   sampled_stats_kernel  largest value and sum of exponentials of the logits rows of nodes that have children (the target's, and the draft's
//                         if it is given), in slices of 4096 values that stay in registers between the two
//   sampled_walk_kernel   (drawn candidates) one workgroup per sequence: the probabilities of all candidates at once, then the tests along the path.  What a
//                         refused candidate leaves of the target needs no distribution of its own: after k refusals r = (p - s_k q)+ / W_k
//                         with s_0 = 0, W_0 = 1, W_k = sum over the vocabulary of (p - s_k q)+ and s_{k+1} = s_k + W_k, since
//                         ((p - s q)+ / W - q)+ = (p - (s + W) q)+ / W.  Only a candidate that has refused siblings before it needs the sum.
//   sampled_next_kernel   the token after the path: what is left in chunks of 4096 tokens, by all workgroups of a sequence; the one that ends
//                         last finds the chunk, and in it the token.  Candidates that were not drawn need no sums: every workgroup walks by itself.
// 64 bits throughout: a vocabulary has so many borders between tokens that an error of 2^-24 of a sum would move one token in a few hundred.
// What bounds it: latency.  One sequence of 16 nodes takes 18.4 us, of them 4.5 in the first kernel; 16 sequences of 64 nodes 29.1, 13 in the first, whose
// exponentials (19 fp64 instructions each, at the rate of fp32 ones) take as long as its reads; drawn candidates of 4 sequences 50 to 60, 35 and more in the walk by how many
// of them are refused.
#include <math.h>

#include <type_traits>

#include "common.h"

namespace propd {

// Threads by tokens of each, us: one sequence of 16 nodes / 16 of 64 nodes (32000 tokens, three kernels): 256 x 16 22.1 / 37.0, 512 x 8 20.2 / 35.2,
// 1024 x 4 22.2 / 39.0, 256 x 8 20.5 / 41.5.
constexpr int kOf = 8, kSampledThreads = 512, kSliceTokens = kOf * kSampledThreads;
constexpr int kWalkThreads = 1024;  // where the draft's distributions take part
constexpr int kMostVocab = 1 << 20;
constexpr float kMostInverse = 0x1p20f;

struct SliceStat {  // of one slice of one row: the largest logit, and the sum of exp((logit - largest) * inv_temperature)
  float most;
  float pad;
  double sum;
};

struct WalkEnd {  // where a sequence's path ends, and what is left there: p, without refused tokens, or p - much * q
  int32_t node, cut;
  float p_most, q_most;
  double p_scale, q_scale, much;
};

struct SampledParams {
  const int32_t *n_nodes, *parent, *token;
  const void *logits, *draft;
  const float *u, *u_next;
  double inv, draft_inv;
  int B, T_max, V, slices, stride, per_sequence;
  int aligned;            // rows of logits start on 16 bytes
  SliceStat *p_stat, *q_stat;  // [B*T_max][slices]
  SliceStat *left;             // [B][slices]: what is left in a chunk
  WalkEnd *end;                // [B]
  int32_t *arrived;            // [B]
  int32_t *accept_len, *accept_path, *next_token;
};

// 2^t for t up to 0: t = n + f with |f| <= 1/2, the series of 2^f = exp(f log 2) up to f^11 (6e-15 off).  Below 2^-1074 it is 0.
__device__ __forceinline__ double exp2_below(double t) {
  t = fmax(t, -1100.0);
  const double n = rint(t), f = t - n;
  double s = 4.4455382718708116e-10;  // log(2)^k / k! for k = 11, 10, ..., 1
  s = fma(s, f, 7.0549116208011233e-09);
  s = fma(s, f, 1.0178086009239699e-07);
  s = fma(s, f, 1.3215486790144307e-06);
  s = fma(s, f, 1.5252733804059841e-05);
  s = fma(s, f, 1.5403530393381608e-04);
  s = fma(s, f, 1.3333558146428443e-03);
  s = fma(s, f, 9.6181291076284772e-03);
  s = fma(s, f, 5.5504108664821580e-02);
  s = fma(s, f, 2.4022650695910071e-01);
  s = fma(s, f, 6.9314718055994531e-01);
  s = fma(s, f, 1.0);
  return __builtin_amdgcn_ldexp(s, (int)n);
}

// The weights of a row's tokens: exp((x - most) * inv) times a scale of at most 1, as 2^((x - most) * slope + log2(scale)).  The difference comes first: it is
// exactly 0 at the row's largest logit and negative elsewhere, however large the logits are (most * slope alone is off by 1e22 for a row masked with
// fp32's lowest value).  Where `most` is infinite, those that are it have the scale and the others nothing.
struct Weights {
  double most, slope, offset;
  bool infinite;
  __device__ __forceinline__ Weights(float row_most, double inv, double scale = 1.0) {
    infinite = row_most == INFINITY;
    most = row_most == -INFINITY || infinite ? 0.0 : (double)row_most;  // (a row of -inf: every weight is 0)
    slope = inv * 1.4426950408889634;
    offset = scale == 1.0 ? 0.0 : scale > 0.0 ? log2(scale) : -INFINITY;
  }
  __device__ __forceinline__ double operator()(float x) const {
    return exp2_below(infinite ? (x == INFINITY ? offset : -INFINITY) : fma((double)x - most, slope, offset));
  }
};

__device__ __forceinline__ float no_nan(float x) { return x == x ? x : -INFINITY; }

template <bool kBf16>
__device__ __forceinline__ float logit_at(const void *rows, size_t row, int V, int v) {
  const size_t at = row * (size_t)V + v;
  return no_nan(kBf16 ? bf16_bits_to_f32(reinterpret_cast<const uint16_t *>(rows)[at]) : reinterpret_cast<const float *>(rows)[at]);
}

// Neighbouring values of a row; -inf beyond the vocabulary.
template <bool kBf16>
__device__ __forceinline__ void load_tokens(const SampledParams &p, const void *rows, size_t row, int first, float (&x)[kOf]) {
  if (p.aligned && first + kOf <= p.V) {
    if constexpr (kBf16) {
      typedef uint32_t Pairs __attribute__((ext_vector_type(kOf / 2)));
      const Pairs a = *reinterpret_cast<const Pairs *>(reinterpret_cast<const uint16_t *>(rows) + row * (size_t)p.V + first);
#pragma unroll
      for (int i = 0; i < kOf / 2; ++i) {
        x[2 * i] = no_nan(__uint_as_float(a[i] << 16));
        x[2 * i + 1] = no_nan(__uint_as_float(a[i] & 0xffff0000u));
      }
    } else {
      const f32x4 *src = reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(rows) + row * (size_t)p.V + first);
      f32x4 a[kOf / 4];
#pragma unroll
      for (int i = 0; i < kOf / 4; ++i) a[i] = src[i];
#pragma unroll
      for (int i = 0; i < kOf; ++i) x[i] = no_nan(a[i / 4][i % 4]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kOf; ++i) x[i] = first + i < p.V ? logit_at<kBf16>(rows, row, p.V, first + i) : -INFINITY;
  }
}

// Sums and extremes over the lanes up to each, by data-parallel moves between registers (a few cycles a step, a tenth of what one through LDS
// takes); `idle` fills the lanes that a step does not reach.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t moved(uint32_t v, uint32_t idle) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)idle, (int)v, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ float moved(float v, float idle) {
  return __uint_as_float(moved<CTRL, ROWS>(__float_as_uint(v), __float_as_uint(idle)));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ int moved(int v, int idle) {
  return (int)moved<CTRL, ROWS>((uint32_t)v, (uint32_t)idle);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved(double v, double idle) {
  const uint64_t a = __builtin_bit_cast(uint64_t, v), z = __builtin_bit_cast(uint64_t, idle);
  const uint64_t lo = moved<CTRL, ROWS>((uint32_t)a, (uint32_t)z), hi = moved<CTRL, ROWS>((uint32_t)(a >> 32), (uint32_t)(z >> 32));
  return __builtin_bit_cast(double, lo | hi << 32);
}
template <class T, class F>
__device__ __forceinline__ T scan_of_16(T v, T idle, F &&join) {  // within each row of 16 lanes
  v = join(v, moved<0x111, 0xf>(v, idle));  // row_shr:1
  v = join(v, moved<0x112, 0xf>(v, idle));  // row_shr:2
  v = join(v, moved<0x114, 0xf>(v, idle));  // row_shr:4
  return join(v, moved<0x118, 0xf>(v, idle));  // row_shr:8
}
template <class T, class F>
__device__ __forceinline__ T scan_of_wave(T v, T idle, F &&join) {
  v = scan_of_16(v, idle, join);
  v = join(v, moved<0x142, 0xa>(v, idle));  // row_bcast:15 into rows 1 and 3
  return join(v, moved<0x143, 0xc>(v, idle));  // row_bcast:31 into rows 2 and 3
}
__device__ __forceinline__ int of_lane(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
__device__ __forceinline__ float of_lane(float v, int lane) { return __uint_as_float((uint32_t)of_lane((int)__float_as_uint(v), lane)); }
__device__ __forceinline__ double of_lane(double v, int lane) {
  const uint64_t a = __builtin_bit_cast(uint64_t, v);
  const uint64_t lo = (uint32_t)of_lane((int)(uint32_t)a, lane), hi = (uint32_t)of_lane((int)(uint32_t)(a >> 32), lane);
  return __builtin_bit_cast(double, lo | hi << 32);
}

// Over the workgroup (of up to 16 waves), in a fixed order; every thread gets the result.  `room`: one entry per wave, used by one call at a time.
template <class T, class F>
__device__ __forceinline__ T block_reduce(T v, T idle, T *room, F &&join) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x / kWave, waves = blockDim.x / kWave;
  v = scan_of_wave(v, idle, join);
  __syncthreads();  // whoever read the room before is done
  if (lane == 63) room[wave] = v;
  __syncthreads();
  return of_lane(scan_of_16((lane & 15) < waves ? room[lane & 15] : idle, idle, join), 15);
}
__device__ __forceinline__ float block_max(float v, float *room) {
  return block_reduce(v, -INFINITY, room, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ double block_sum(double v, double *room) {
  return block_reduce(v, 0.0, room, [](double a, double b) { return a + b; });
}

// The sum over the threads before this one, and over all, in a fixed order.
__device__ __forceinline__ double block_before(double v, double *room, double &total) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = blockDim.x / kWave;
  auto add = [](double a, double b) { return a + b; };
  const double upto = scan_of_wave(v, 0.0, add);
  __syncthreads();
  if (lane == 63) room[wave] = upto;
  __syncthreads();
  const double waves_upto = scan_of_16((lane & 15) < waves ? room[lane & 15] : 0.0, 0.0, add);
  total = of_lane(waves_upto, 15);
  const double before = wave > 0 ? of_lane(waves_upto, wave - 1) : 0.0;
  return before + moved<0x138, 0xf>(upto, 0.0);  // wave_shr:1
}

__device__ __forceinline__ int tree_size(const SampledParams &p, int b) {
  const int T = p.n_nodes[b];
  return T < 1 ? 1 : (T > p.T_max ? p.T_max : T);
}

// Largest value and sum of a slice, by the workgroup.
template <bool kBf16>
__device__ __forceinline__ SliceStat slice_stat(const SampledParams &p, const void *rows, size_t row, int slice, double inv, float *f_room,
                                                double *d_room) {
  float x[kOf];
  load_tokens<kBf16>(p, rows, row, slice * kSliceTokens + kOf * (int)threadIdx.x, x);
  float most = -INFINITY;
#pragma unroll
  for (int i = 0; i < kOf; ++i) most = fmaxf(most, x[i]);
  most = block_max(most, f_room);
  double sum = 0.0;
  const Weights weight(most, inv);
  if (most > -INFINITY) {
#pragma unroll
    for (int i = 0; i < kOf; ++i) sum += weight(x[i]);
  }
  sum = block_sum(sum, d_room);
  return {most, 0.f, sum};
}

// The nodes of a sequence that have children, counted off to its workgroups slice by slice.
template <bool kBf16>
__global__ __launch_bounds__(kSampledThreads) void sampled_stats_kernel(SampledParams p) {
  __shared__ uint64_t s_inner[2];
  __shared__ float f_room[kSampledThreads / kWave];
  __shared__ double d_room[kSampledThreads / kWave];
  const int b = blockIdx.x / p.per_sequence, at = blockIdx.x - b * p.per_sequence, tid = threadIdx.x;
  const int T = tree_size(p, b);
  if (at == 0 && tid == 0) p.arrived[b] = 0;  // of the last kernel
  if (tid < 2) s_inner[tid] = 0;
  __syncthreads();
  if (tid > 0 && tid < T) {
    const int above = p.parent[(size_t)b * p.T_max + tid];
    if (above >= 0 && above < tid) atomicOr(reinterpret_cast<unsigned long long *>(s_inner + (above >> 6)), 1ull << (above & 63));
  }
  __syncthreads();
  uint64_t lo = s_inner[0], hi = s_inner[1];
  const int items = (__popcll(lo) + __popcll(hi)) * p.slices;
  int passed = 0;  // nodes taken out of the set
  for (int item = at; item < items; item += p.per_sequence) {
    const int rank = item / p.slices, slice = item - rank * p.slices;
    for (; passed < rank; ++passed) {
      if (lo) lo &= lo - 1;
      else hi &= hi - 1;
    }
    const int node = lo ? __ffsll((unsigned long long)lo) - 1 : 63 + __ffsll((unsigned long long)hi);
    const size_t row = (size_t)b * p.T_max + node;
    const SliceStat s = slice_stat<kBf16>(p, p.logits, row, slice, p.inv, f_room, d_room);
    if (tid == 0) p.p_stat[row * p.slices + slice] = s;
    if (p.draft) {
      const SliceStat t = slice_stat<kBf16>(p, p.draft, row, slice, p.draft_inv, f_room, d_room);
      if (tid == 0) p.q_stat[row * p.slices + slice] = t;
    }
  }
}

struct RowStat {
  float most;
  double scale;  // 1 / sum; 0 where the row has no probability
};
// Of all slices of a row; eight of them are requested together.
__device__ __forceinline__ RowStat row_stat(const SliceStat *s, int slices, double inv) {
  float most = -INFINITY;
  double sum = 0.0;
  for (int i0 = 0; i0 < slices; i0 += 8) {
    SliceStat x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = s[i0 + i < slices ? i0 + i : i0];
    float top = most;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, x[i].most);
    if (top == -INFINITY) continue;
    const Weights weight(top, inv);
    sum = most == -INFINITY ? 0.0 : sum * weight(most);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += i0 + i < slices && x[i].most > -INFINITY ? x[i].sum * weight(x[i].most) : 0.0;
    most = top;
  }
  return {most, sum > 0.0 ? 1.0 / sum : 0.0};
}

struct NodeSet {
  uint64_t w[2];
};
__device__ __forceinline__ int take_first(NodeSet &s) {  // the lowest node of a set that has one
  const int i = s.w[0] ? __ffsll((unsigned long long)s.w[0]) - 1 : 63 + __ffsll((unsigned long long)s.w[1]);
  if (s.w[0]) s.w[0] &= s.w[0] - 1;
  else s.w[1] &= s.w[1] - 1;
  return i;
}
__device__ __forceinline__ bool in_set(const NodeSet &s, int i) { return (s.w[i >> 6] >> (i & 63)) & 1; }
__device__ __forceinline__ bool some(const NodeSet &s) { return (s.w[0] | s.w[1]) != 0; }

// What a workgroup knows of its sequence's tree.
struct Walk {
  int token[PROPD_MAX_TREE], path[PROPD_MAX_TREE], next[PROPD_MAX_TREE];
  NodeSet children[PROPD_MAX_TREE];
  RowStat row_p[PROPD_MAX_TREE], row_q[PROPD_MAX_TREE];  // of nodes that have children
  double p[PROPD_MAX_TREE], q[PROPD_MAX_TREE];           // of every candidate's token at its parent
  float u[PROPD_MAX_TREE];
  uint64_t passes[2];
  int full;  // nodes of the path
};

// The probabilities of all candidates at once.  Threads from PROPD_MAX_TREE on only meet the barriers; returns the parent of node threadIdx.x, -1 if
// it is no candidate (kDraft: if its token lies outside the vocabulary).
template <bool kBf16, bool kDraft>
__device__ __forceinline__ int meet_candidates(const SampledParams &p, int b, int T, Walk &s) {
  const int i = threadIdx.x;
  const size_t base = (size_t)b * p.T_max;
  bool child = i > 0 && i < T;
  int above = 0, token = -1;
  float u = 0.f;
  if (child) {
    above = p.parent[base + i];
    token = p.token[base + i];
    u = p.u[base + i];
    child = above >= 0 && above < i;
  }
  const bool inside = child && token >= 0 && token < p.V;
  child = kDraft ? inside : child;
  float x = 0.f, y = 0.f;
  if (inside) {  // (on its way meanwhile)
    x = logit_at<kBf16>(p.logits, base + above, p.V, token);
    if constexpr (kDraft) y = logit_at<kBf16>(p.draft, base + above, p.V, token);
  }
  if (i < PROPD_MAX_TREE) {
    s.token[i] = token;
    s.next[i] = -1;
    s.children[i].w[0] = s.children[i].w[1] = 0;
    s.u[i] = u;
  }
  __syncthreads();
  if (child) atomicOr(reinterpret_cast<unsigned long long *>(&s.children[above].w[i >> 6]), 1ull << (i & 63));
  __syncthreads();
  if (i < T && some(s.children[i])) {
    s.row_p[i] = row_stat(p.p_stat + (base + i) * p.slices, p.slices, p.inv);
    if constexpr (kDraft) s.row_q[i] = row_stat(p.q_stat + (base + i) * p.slices, p.slices, p.draft_inv);
  }
  __syncthreads();
  if (i < PROPD_MAX_TREE) {
    double pc = 0.0, qc = 0.0;
    if (inside) {
      const RowStat r = s.row_p[above];
      pc = r.scale > 0.0 ? Weights(r.most, p.inv)(x) * r.scale : 0.0;
      if constexpr (kDraft) {
        const RowStat r2 = s.row_q[above];
        qc = r2.scale > 0.0 ? Weights(r2.most, p.draft_inv)(y) * r2.scale : 0.0;
      }
    }
    s.p[i] = pc;
    s.q[i] = qc;
  }
  __syncthreads();
  return child ? above : -1;
}

// The path of candidates that were not drawn, into s.path and s.full.
template <bool kBf16>
__device__ __forceinline__ void walk_given(const SampledParams &p, int b, int T, Walk &s) {
  const int i = threadIdx.x, above = meet_candidates<kBf16, false>(p, b, T, s);
  // every candidate's test, as if its siblings before it had been refused: the first that passes is taken
  NodeSet before = {{0, 0}};
  bool again = false;
  if (above >= 0) {
    uint64_t lo, hi;
    mask_below(i, lo, hi);
    before = {{s.children[above].w[0] & lo, s.children[above].w[1] & hi}};
    for (NodeSet m = before; some(m);) again = s.token[take_first(m)] == s.token[i] || again;
  }
  const double mine = above < 0 || again ? 0.0 : s.p[i];
  __syncthreads();
  if (i < PROPD_MAX_TREE) s.p[i] = mine;  // (a token refused before has nothing left)
  __syncthreads();
  double left = 1.0;
  for (NodeSet m = before; some(m);) left -= s.p[take_first(m)];
  const bool passes = above >= 0 && (double)s.u[i] * (left > 0.0 ? left : 0.0) < mine;
  const uint64_t word = __ballot(passes);
  if (i < PROPD_MAX_TREE && (i & 63) == 0) s.passes[i >> 6] = word;
  __syncthreads();
  if (passes && ((before.w[0] & s.passes[0]) | (before.w[1] & s.passes[1])) == 0) s.next[above] = i;
  __syncthreads();
  if (i == 0) {
    int node = 0, n = 0;
    do {
      s.path[n++] = node;
      node = s.next[node];
    } while (node >= 0);
    s.full = n;
  }
  __syncthreads();
}

// Writes the path.  A path buffer shorter than it keeps its first nodes; the next node's token goes on with the same output.
__device__ __forceinline__ bool write_path(const SampledParams &p, int b, const Walk &s, int full) {
  const int len = full < p.stride ? full : p.stride;
  for (int j = threadIdx.x; j < p.stride; j += blockDim.x) p.accept_path[(size_t)b * p.stride + j] = j < len ? s.path[j] : -1;
  if (threadIdx.x == 0) {
    p.accept_len[b] = len;
    if (full > len) p.next_token[b] = s.token[s.path[len]];
  }
  return full > len;
}

// The path of candidates that were drawn.
template <bool kBf16>
__global__ __launch_bounds__(kWalkThreads) void sampled_walk_kernel(SampledParams p) {
  __shared__ Walk s;
  __shared__ double d_room[kWalkThreads / kWave];
  const int b = blockIdx.x, i = threadIdx.x, T = tree_size(p, b);
  const size_t base = (size_t)b * p.T_max;
  double much = 0.0;
  int last = 0, full = 0;
  meet_candidates<kBf16, true>(p, b, T, s);
  // (every thread goes along; child and what it needs are the same for all)
  int node = 0;
  while (true) {
    if (i == 0) s.path[full] = node;
    ++full;
    last = node;
    much = 0.0;
    double mass = 1.0;
    int taken = -1;
    bool known = true;  // mass belongs to much
    const size_t row = base + node;
    for (NodeSet m = s.children[node]; some(m);) {
      const int j = take_first(m);
      if (!known) {
        const RowStat ps = s.row_p[node], qs = s.row_q[node];
        const Weights weight_p(ps.most, p.inv, ps.scale), weight_q(qs.most, p.draft_inv, qs.scale);
        double sum = 0.0;
        for (int first = kOf * i; first < p.V; first += kOf * kWalkThreads) {
          float x[kOf], y[kOf];
          load_tokens<kBf16>(p, p.logits, row, first, x);
          load_tokens<kBf16>(p, p.draft, row, first, y);
#pragma unroll
          for (int e = 0; e < kOf; ++e) sum += fmax(fma(-much, weight_q(y[e]), weight_p(x[e])), 0.0);
        }
        mass = block_sum(sum, d_room);
        known = true;
      }
      const double left = s.p[j] - much * s.q[j];
      if ((double)s.u[j] * mass * s.q[j] < left) {
        taken = j;
        break;
      }
      much += mass;
      known = false;
    }
    if (taken < 0) break;
    node = taken;
  }
  __syncthreads();
  const bool cut = write_path(p, b, s, full);
  if (i == 0) {
    WalkEnd e = {last, cut, 0.f, 0.f, 0.0, 0.0, much};
    if (much > 0.0) {
      e.p_most = s.row_p[last].most;
      e.p_scale = s.row_p[last].scale;
      e.q_most = s.row_q[last].most;
      e.q_scale = s.row_q[last].scale;
    }
    p.end[b] = e;
  }
}

// The likeliest token of a row, the lowest id among equal ones, by the workgroup.
template <bool kBf16>
__device__ __forceinline__ void likeliest_token(const SampledParams &p, size_t row, float *f_room, int *found, int32_t *to) {
  float best = -INFINITY;
  int at = 0x7fffffff;
  for (int v = threadIdx.x; v < p.V; v += blockDim.x) {
    const float y = logit_at<kBf16>(p.logits, row, p.V, v);
    if (y > best || at == 0x7fffffff) {
      best = y;
      at = v;
    }
  }
  const float top = block_max(best, f_room);
  __syncthreads();
  if (threadIdx.x == 0) *found = 0x7fffffff;
  __syncthreads();
  if (best == top) atomicMin(found, at);
  __syncthreads();
  if (threadIdx.x == 0) *to = *found < p.V ? *found : 0;
}

// What is left of a thread's tokens of a chunk.  refused: a bit per token of the chunk.
template <bool kBf16, bool kDraft>
__device__ __forceinline__ void left_of(const SampledParams &p, const WalkEnd &e, const float (&x)[kOf], size_t row, int chunk, float most,
                                        const uint32_t *refused, double (&w)[kOf]) {
  if (kDraft && e.much > 0.0) {
    float y[kOf];
    load_tokens<kBf16>(p, p.draft, row, chunk * kSliceTokens + kOf * (int)threadIdx.x, y);
    const Weights weight_p(e.p_most, p.inv, e.p_scale), weight_q(e.q_most, p.draft_inv, e.q_scale);
#pragma unroll
    for (int i = 0; i < kOf; ++i) w[i] = fmax(fma(-e.much, weight_q(y[i]), weight_p(x[i])), 0.0);
  } else {
    const Weights weight(most, p.inv);
    const uint32_t gone = kDraft ? 0 : refused[threadIdx.x * kOf / 32] >> (threadIdx.x * kOf % 32);
#pragma unroll
    for (int i = 0; i < kOf; ++i) w[i] = x[i] > -INFINITY && !((gone >> i) & 1) ? weight(x[i]) : 0.0;
  }
}

template <bool kBf16, bool kDraft>
__global__ __launch_bounds__(kSampledThreads) void sampled_next_kernel(SampledParams p) {
  __shared__ float f_room[kSampledThreads / kWave];
  __shared__ double d_room[kSampledThreads / kWave];
  __shared__ uint32_t s_refused[kSliceTokens / 32];  // a bit per token
  __shared__ std::conditional_t<kDraft, char, Walk> s_walk;
  __shared__ double s_goal;
  __shared__ int s_last, s_found;
  const int b = blockIdx.x / p.slices, own = blockIdx.x - b * p.slices, tid = threadIdx.x;
  const int T = tree_size(p, b);
  const size_t base = (size_t)b * p.T_max;
  WalkEnd e = {};
  if constexpr (kDraft) {
    e = p.end[b];
    if (e.cut) return;
  } else {  // every workgroup walks by itself: the path is short, and a kernel of its own takes longer
    walk_given<kBf16>(p, b, T, s_walk);
    e.node = s_walk.path[s_walk.full - 1];
    if (own == 0) write_path(p, b, s_walk, s_walk.full);
    if (s_walk.full > p.stride) return;
  }
  const size_t row = base + e.node;
  const bool relative = !(kDraft && e.much > 0.0);  // what is left is p itself, in a chunk relative to its largest logit
  double w[kOf], sum;
  int c = own;
#pragma nounroll
  for (bool all = true;; all = false) {  // all workgroups, a chunk each; then the last of them, the token's chunk
    float x[kOf], most = -INFINITY;
    load_tokens<kBf16>(p, p.logits, row, c * kSliceTokens + kOf * tid, x);
    if constexpr (!kDraft) {
      for (int j = tid; j < kSliceTokens / 32; j += kSampledThreads) s_refused[j] = 0;
      __syncthreads();
      if (tid < T && in_set(s_walk.children[e.node], tid)) {  // all of them were refused
        const int token = s_walk.token[tid], t = token - c * kSliceTokens;
        if (token >= 0 && t >= 0 && t < kSliceTokens) atomicOr(s_refused + (t >> 5), 1u << (t & 31));
      }
    }
#pragma unroll
    for (int i = 0; i < kOf; ++i) most = fmaxf(most, x[i]);
    most = block_max(most, f_room);  // (its barriers stand behind the set)
    left_of<kBf16, kDraft>(p, e, x, row, c, most, s_refused, w);
    sum = 0.0;
#pragma unroll
    for (int i = 0; i < kOf; ++i) sum += w[i];
    if (!all) break;
    const double here = block_sum(sum, d_room);
    if (tid == 0) {
      SliceStat *to = p.left + (size_t)b * p.slices + own;
      __hip_atomic_store(&to->most, relative ? most : 0.f, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(&to->sum, here, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      s_last = __hip_atomic_fetch_add(p.arrived + b, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == p.slices - 1;
      s_found = -1;
    }
    __syncthreads();
    if (!s_last) return;

    // ---- the last workgroup of the sequence: which chunk
    SliceStat mine = {-INFINITY, 0.f, 0.0};
    if (tid < p.slices) {
      const SliceStat *from = p.left + (size_t)b * p.slices + tid;
      mine.most = __hip_atomic_load(&from->most, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      mine.sum = __hip_atomic_load(&from->sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    const float top = block_max(mine.sum > 0.0 ? mine.most : -INFINITY, f_room);
    const double scale = mine.sum > 0.0 ? (relative ? Weights(top, p.inv)(mine.most) : 1.0) : 0.0, share = mine.sum * scale;
    double total;
    const double before = block_before(share, d_room, total);
    const double goal = (double)p.u_next[b] * total;
    // the first chunk whose end lies beyond the goal; where rounding leaves none, the last that has anything
    if (share > 0.0 && before + share > goal) atomicMin(reinterpret_cast<unsigned int *>(&s_found), (unsigned)tid);
    __syncthreads();
    c = s_found;
    if (c < 0) {
      __syncthreads();
      if (share > 0.0) atomicMax(&s_found, tid);
      __syncthreads();
      c = s_found;
    }
    if (c < 0) {  // nothing is left: the likeliest token
      __syncthreads();
      likeliest_token<kBf16>(p, row, f_room, &s_found, p.next_token + b);
      return;
    }
    __syncthreads();
    if (tid == c) {
      s_goal = (goal - before) / scale;  // in the chunk's own measure
      s_found = 0x7fffffff;
    }
    __syncthreads();
    if (c == own) break;  // (its weights are at hand)
  }

  // ---- and which token of it
  double all_of_it;
  double here = block_before(sum, d_room, all_of_it);
  int first = 0x7fffffff, final = -1;
  const int v0 = c * kSliceTokens + kOf * tid;
#pragma unroll
  for (int i = 0; i < kOf; ++i) {
    here += w[i];
    if (w[i] > 0.0) {
      if (here > s_goal && first == 0x7fffffff) first = v0 + i;
      final = v0 + i;
    }
  }
  if (first != 0x7fffffff) atomicMin(&s_found, first);
  const int end = block_reduce(final, -1, reinterpret_cast<int *>(f_room), [](int a, int b) { return a > b ? a : b; });
  if (tid == 0) p.next_token[b] = s_found != 0x7fffffff ? s_found : end;
}

// ------------------------------------------------------------------------------------
// host side
// ------------------------------------------------------------------------------------
static int slices_of(int V) { return (V + kSliceTokens - 1) / kSliceTokens; }

size_t accept_sampled_workspace_bytes(int B, int T_max, int V) {
  const size_t rows = (size_t)B * T_max, slices = (size_t)slices_of(V);
  return 2 * align_up(rows * slices * sizeof(SliceStat), 256) + align_up((size_t)B * slices * sizeof(SliceStat), 256) +
         align_up((size_t)B * sizeof(WalkEnd), 256) + align_up((size_t)B * 4, 256);
}

template <bool kBf16>
static propd_status run_sampled(const SampledParams &p, hipStream_t st) {
  hipLaunchKernelGGL(sampled_stats_kernel<kBf16>, dim3((unsigned)(p.B * p.per_sequence)), dim3(kSampledThreads), 0, st, p);
  if (!launch_ok()) return PROPD_ERR_DEVICE;
  if (p.draft) {
    hipLaunchKernelGGL(sampled_walk_kernel<kBf16>, dim3((unsigned)p.B), dim3(kWalkThreads), 0, st, p);
    if (!launch_ok()) return PROPD_ERR_DEVICE;
  }
  const dim3 grid((unsigned)(p.B * p.slices));
  if (p.draft) hipLaunchKernelGGL((sampled_next_kernel<kBf16, true>), grid, dim3(kSampledThreads), 0, st, p);
  else hipLaunchKernelGGL((sampled_next_kernel<kBf16, false>), grid, dim3(kSampledThreads), 0, st, p);
  return launch_ok() ? PROPD_OK : PROPD_ERR_DEVICE;
}

}  // namespace propd

extern "C" propd_status propd_accept_sampled(const propd_tree *tree, propd_dtype dt, int32_t vocab, const void *logits, float inv_temperature,
                                             const void *draft_logits, float draft_inv_temperature, const float *u, const float *u_next,
                                             int32_t *accept_len, int32_t *accept_path, int32_t path_stride, int32_t *next_token,
                                             void *workspace, size_t workspace_bytes, void *hip_stream) {
  using namespace propd;
  if (!tree || tree->B < 1 || tree->T_max < 1 || tree->T_max > PROPD_MAX_TREE || vocab < 1 || path_stride < 1 || !tree->n_nodes || !tree->parent ||
      !tree->token || !logits || !u || !u_next || !accept_len || !accept_path || !next_token)
    return PROPD_ERR_INVALID_ARG;
  if (dt != PROPD_BF16 && dt != PROPD_F32) return PROPD_ERR_INVALID_ARG;
  if (!(inv_temperature > 0.f && inv_temperature <= kMostInverse)) return PROPD_ERR_INVALID_ARG;
  if (draft_logits && !(draft_inv_temperature > 0.f && draft_inv_temperature <= kMostInverse)) return PROPD_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(workspace) % 16 != 0) return PROPD_ERR_INVALID_ARG;
  if (vocab > kMostVocab || (long long)tree->B * slices_of(vocab) > (1ll << 21)) return PROPD_ERR_UNSUPPORTED;
  const size_t needed = accept_sampled_workspace_bytes(tree->B, tree->T_max, vocab);
  if (!workspace || workspace_bytes < needed) return PROPD_ERR_WORKSPACE;
  SampledParams p;
  p.n_nodes = tree->n_nodes;
  p.parent = tree->parent;
  p.token = tree->token;
  p.logits = logits;
  p.draft = draft_logits;
  p.u = u;
  p.u_next = u_next;
  p.inv = inv_temperature;
  p.draft_inv = draft_inv_temperature;
  p.B = tree->B;
  p.T_max = tree->T_max;
  p.V = vocab;
  p.slices = slices_of(vocab);
  p.stride = path_stride;
  const size_t size = dt == PROPD_BF16 ? 2 : 4;
  p.aligned = (size_t)vocab * size % 16 == 0 && reinterpret_cast<uintptr_t>(logits) % 16 == 0 && reinterpret_cast<uintptr_t>(draft_logits) % 16 == 0;
  char *ws = reinterpret_cast<char *>(workspace);
  const size_t rows = (size_t)p.B * p.T_max;
  p.p_stat = reinterpret_cast<SliceStat *>(ws);
  ws += align_up(rows * p.slices * sizeof(SliceStat), 256);
  p.q_stat = reinterpret_cast<SliceStat *>(ws);
  ws += align_up(rows * p.slices * sizeof(SliceStat), 256);
  p.left = reinterpret_cast<SliceStat *>(ws);
  ws += align_up((size_t)p.B * p.slices * sizeof(SliceStat), 256);
  p.end = reinterpret_cast<WalkEnd *>(ws);
  ws += align_up((size_t)p.B * sizeof(WalkEnd), 256);
  p.arrived = reinterpret_cast<int32_t *>(ws);
  p.accept_len = accept_len;
  p.accept_path = accept_path;
  p.next_token = next_token;
  // workgroups of a sequence: about as many as run at once, no more than there can be slices of nodes with children
  const long long most = (long long)(p.T_max > 1 ? p.T_max - 1 : 1) * p.slices, fair = 2048 / p.B > 1 ? 2048 / p.B : 1;
  p.per_sequence = (int)(most < fair ? most : fair);
  return dt == PROPD_BF16 ? run_sampled<true>(p, as_stream(hip_stream)) : run_sampled<false>(p, as_stream(hip_stream));
}
