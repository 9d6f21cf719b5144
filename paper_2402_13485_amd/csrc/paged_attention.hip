// Tree attention over a paged cache: rows as they are or in 8 bits, K/V heads shared by several query heads, capped and biased scores, a window.
//
// A unit is a (sequence, K/V head, block of query columns): the nodes of all query heads that read the K/V head lie side by side, column r is
// node r % T of head r / T, so that a row is read once for all of them.  Its rows come in stages of 32, the tree's own first, then the cached ones.
//   - A workgroup takes a range of a unit's stages.  Its four waves are kCw blocks of kN query columns by 4 / kCw rows of stages: up to 16 columns
//     (a single token) each wave streams stages of its own and waits for nobody; up to 64 columns, and beyond with 32 a wave, four waves share
//     every stage.
//   - The next stage's rows are on their way to registers while a stage is multiplied; from there they go to LDS, 8-bit rows
//     as the bf16 or fp32 values that they stand for (once per workgroup, not once per wave that multiplies them).
//   - S^T = K . Q^T, so that a lane owns a column: running maximum and sum, position, slope and ancestor set are per-lane scalars, and the weights
//     are the B operand of O^T += V^T . P^T as they are.  bf16: products of 32x32x16 or 16x16x32, V^T by transposing LDS reads, a weight as the sum
//     of two bf16 values (off by 2^-17; one alone would add 40 % to the result's own rounding).  fp32: products of 32x32x2 or 16x16x4.
//   - Ranges of a unit leave partial results, which a second kernel joins in their order.
//   - A range whose sums are not finite, or could leave fp32 when joined, is done once more with care: values of V that are not finite are taken out of the
//     products and counted by sign for the columns that see their rows, and weights are small enough that no sum exceeds its largest value.
// What bounds it: a single token or few, memory (32 x 8 heads of 8192 rows in 8 bits 96 us, 5.6 TB/s); large trees, vector and matrix instructions that hardly
// overlap (16 x 40 heads on 8, 128 nodes, 4096 rows 300 us, matrix unit busy 43 %); small calls, a chain of dependent reads (1 x 32 heads of 1024 rows 13 us).
#include "attention_device.h"
#include "paged_cache.h"
#include "score_rule.h"

namespace propd {

constexpr int kPagedThreads = 256;

struct PagedParams {
  Pages pages;
  const unsigned char *q, *k_tree, *v_tree;
  unsigned char *out;
  float *lse;
  const int32_t *seq_lens, *n_nodes;
  const uint64_t *anc;
  const float *slopes;
  int B, H, H_kv, group, T_max;
  int blocks;   // blocks of kN * kCw columns of a unit's tree of T_max nodes
  int window;   // window_of
  float scale_log2e, cap_in, cap_log2e;  // cap_in: scale / cap
  float *part_o, *part_ml;
  int32_t *records;  // [B * H_kv * blocks][4]: first slot, slots between pieces, pieces
  int resident;      // workgroups that run at once
  int least;         // steps of a range, at least
  int may_split;
};

// What the kernel's types and shapes make.  kN: columns of a wave, 16 or 32; a product has as many rows.
template <bool kBf16, int D, int kN, int kCw>
struct PagedGeo {
  static constexpr int kColumns = kN * kCw;
  static constexpr int kRw = 4 / kCw;                  // stages at work at once
  static constexpr int kRowBytes = D * (kBf16 ? 2 : 4);
  static constexpr int kPart = kStageRows * kRowBytes;  // K part of a stage; the V part follows
  static constexpr int kStage = 2 * kPart;
  static constexpr int kSlots = kCw == 1 ? 1 : 2;      // places for stages; a wave's own needs one
  static constexpr int kChunks = kRowBytes / 16;
  static constexpr int kGroups = 64 / kN;              // lanes that have a column
  static constexpr int kScores = 32 / kGroups;         // scores of a lane per stage; number x is of row 4 * kGroups * (x / 4) + 4 * group + x % 4
  static constexpr int kBlocks = D / kN, kAcc = kN * kN / 64;  // products that make O, and their registers
  static constexpr int kQuads = D / (4 * kGroups);     // O of a lane in fours of neighbouring d; quad x starts at d = 4 * kGroups * x + 4 * group
  static constexpr int kThreads = 64 * kCw;            // that load a stage
  static constexpr int kLds = kRw * kSlots * kStage + 512;
  // Chunk c of row r of a stage lies at chunk position c ^ key(r): a fragment read's rows fall into different banks.  A key picks bits of
  // r, so that key(R + q) = key(R) ^ key(q) where R and q have no bit in common: what a lane reads or writes lies at an address of
  // its own (q, c) with some bits flipped and a number added (R, C), both known at compile time.
  static __device__ __forceinline__ int k_key(int r) { return kBf16 ? Geo<D>::k_key(r) : r & (kChunks - 1); }
  static __device__ __forceinline__ int v_key(int r) {
    return kBf16 ? Geo<D>::v_key(r) : kN == 32 ? ((r >> 2) & 1) << 3 : ((r >> 2) & 3) << 2;
  }
};

template <int kN>
using Acc = std::conditional_t<kN == 32, f32x16, f32x4>;

template <int kN>
__device__ __forceinline__ Acc<kN> product(u32x4 a, u32x4 b, Acc<kN> c) {
  if constexpr (kN == 32) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <int kN>
__device__ __forceinline__ Acc<kN> product(float a, float b, Acc<kN> c) {
  if constexpr (kN == 32) return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}
template <class V>
__device__ __forceinline__ void clear(V &v) {
#pragma unroll
  for (int r = 0; r < (int)(sizeof(V) / 4); ++r) v[r] = 0.f;
}

// A number that the compiler takes for another one every time, so that what is made of it is made again where it is needed and
// takes no registers meanwhile.
__device__ __forceinline__ uint32_t made_anew(uint32_t v) {
  asm volatile("" : "+v"(v));
  return v;
}

// Stages of a unit: the tree's, then cached ones from row 32 * `first` on.
struct PagedStages {
  int tree, first, cached;
};
__device__ __forceinline__ PagedStages paged_stages(int L, int T, int window) {
  PagedStages s;
  s.tree = (T + kStageRows - 1) / kStageRows;
  s.first = (L > window ? L - window + 1 : 0) / kStageRows;  // the first row that the root sees
  s.cached = (L + kStageRows - 1) / kStageRows - s.first;
  s.cached = s.cached < 0 ? 0 : s.cached;
  return s;
}

// How the units are cut, in steps of kRw stages.  Every workgroup works the same plan out from the lengths.
//   As many units as run at once or fewer: ranges that are equally long per unit, of the fewest steps at most whose ranges all run at once (from an equal
//   share on, a sixteenth of it longer at a time).
//   More: as many units as there are rounds of workgroups for come first, whole unless they are longer than an equal share of everything; the units
//   left over are cut as above, so that the last round is as short as the others' rest.
struct PagedPlan {
  int whole;        // units that come first
  int big, small;   // most steps of a range of those, and of the others
  int n1, n2;       // ranges of those, and of the others; their slots for partial results are n2 and more, and from 0 on
};
constexpr float kBack = 0x1p-31f, kForth = 0x1p31f;  // (a sequence has at most 2^30 cached rows and 128 others)
constexpr float kMostPlain = 0x1p96f;  // sums of more are made with care: a call's pieces of less can be added up

struct PagedSequence {
  int L, T, steps, units;  // units 0 beyond the batch
};
template <int kN, int kCw>
__device__ __forceinline__ PagedSequence paged_sequence(const PagedParams &p, int b) {
  PagedSequence q = {0, 0, 0, 0};
  if (b >= p.B) return q;
  q.L = clamped(p.seq_lens[b], p.pages.capacity);
  q.T = clamped(p.n_nodes[b] - 1, p.T_max - 1) + 1;
  const PagedStages s = paged_stages(q.L, q.T, p.window);
  q.steps = (s.tree + s.cached + 4 / kCw - 1) / (4 / kCw);
  q.units = p.H_kv * ((p.group * q.T + kN * kCw - 1) / (kN * kCw));
  return q;
}

// Pieces of a unit.  The second kernel takes 16 of them at a time, which costs as much as half a step: no more than make the two least together.
__device__ __forceinline__ int paged_pieces(int steps, int most) {
  const int enough = (int)ceilf(sqrtf((float)steps * (1.f / 24.f)));
  most = most > enough ? most : enough;
  return most >= steps ? 1 : (int)((unsigned)(steps + most - 1) / (unsigned)most);
}
__device__ __forceinline__ int paged_scan(int v) {
  return wave_scan_i32(v, 0, [](int x, int y) { return x + y; });
}
__device__ __forceinline__ int paged_sum(int v) { return __builtin_amdgcn_readlane(paged_scan(v), 63); }
__device__ __forceinline__ float paged_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v)));  // (what follows from it is the same for all lanes, in scalar registers)
}

// Units of a lane's sequence that come first, and the others; `before`: units of the sequences before those of the lanes.
struct PagedShare {
  int first, rest;
};
__device__ __forceinline__ PagedShare paged_share(int units, int before, int whole) {
  const int start = before + paged_scan(units) - units, first = clamped(whole - start, units);
  return {first, units - first};
}

template <int kN, int kCw>
__device__ __forceinline__ PagedPlan paged_plan(const PagedParams &p, const PagedSequence &lanes) {
  const int lane = threadIdx.x & 63;
  auto over = [&](auto &&each) __attribute__((always_inline)) {  // each(sequence, units before the 64 sequences)
    int before = 0;
    for (int b0 = 0; b0 < p.B; b0 += kWave) {
      const PagedSequence q = b0 == 0 ? lanes : paged_sequence<kN, kCw>(p, b0 + lane);
      each(q, before);
      if (b0 + kWave < p.B) before += paged_sum(q.units);
    }
  };
  int units = 0;
  float total = 0.f;
  over([&](const PagedSequence &q, int) {
    units += paged_sum(q.units);
    total += paged_sum((float)q.units * (float)q.steps);
  });
  PagedPlan plan = {units, 1 << 30, 1 << 30, units, 0};
  if (!p.may_split) return plan;
  plan.whole = units <= p.resident ? 0 : units / p.resident * p.resident;
  float rest = total;
  if (plan.whole > 0) {
    plan.big = (int)ceilf(total * 1.0001f / (float)p.resident);  // (a little more: the bound on their pieces holds however sums are rounded)
    plan.n1 = 0;
    rest = 0.f;
    over([&](const PagedSequence &q, int before) {
      const PagedShare s = paged_share(q.units, before, plan.whole);
      plan.n1 += paged_sum(s.first * paged_pieces(q.steps, plan.big));
      rest += paged_sum((float)s.rest * (float)q.steps);
    });
  } else {
    plan.n1 = 0;
  }
  const float share = fmaxf(rest / (float)p.resident, (float)p.least);
  for (int step = 0; step <= 64; ++step) {
    plan.small = step == 64 ? 1 << 30 : (int)ceilf(share * (1.f + .0625f * (float)step * (float)(step < 16 ? 1 : step - 14)));
    plan.n2 = 0;
    over([&](const PagedSequence &q, int before) { plan.n2 += paged_sum(paged_share(q.units, before, plan.whole).rest * paged_pieces(q.steps, plan.small)); });
    if (plan.n2 <= p.resident) break;  // (as few as the units left over fit in any case)
  }
  return plan;
}

template <class V>
using LdsPtr = __attribute__((address_space(3))) V *;
__device__ __forceinline__ void lds_to(uint32_t at, u32x4 v) { *reinterpret_cast<LdsPtr<u32x4>>((uintptr_t)at) = v; }
template <class V>
__device__ __forceinline__ V lds_from(uint32_t at) {
  return *reinterpret_cast<LdsPtr<const V>>((uintptr_t)at);
}

// Four neighbouring values of a result
template <bool kBf16>
__device__ __forceinline__ void store_quad(unsigned char *out, size_t at, f32x4 v, float inv) {
  if constexpr (kBf16) *reinterpret_cast<u32x2 *>(reinterpret_cast<uint16_t *>(out) + at) = u32x2{cvt_pk_bf16(v[0] * inv, v[1] * inv), cvt_pk_bf16(v[2] * inv, v[3] * inv)};
  else *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(out) + at) = f32x4{v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv};
}

// A part of a result times a factor that may be zero: a row that is seen has a weight above zero, however little it is, so that what an infinity or a NaN
// of V made stays, in whatever order rows and ranges come.
__device__ __forceinline__ float weighed(float o, float f) { return fabsf(o) < INFINITY ? o * f : o; }

__device__ __forceinline__ float inverse(float l) { return l > 0.f ? 1.f / l : l == 0.f ? 0.f : l; }  // NaN stays

// LDS written before is seen by the workgroup; loads from memory stay in flight.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <bool kBf16, bool kCodes, int D, int kN, int kCw>
__global__ __launch_bounds__(kPagedThreads, kBf16 ? 2 : 1) void paged_attn_kernel(PagedParams p) {
  using G = PagedGeo<kBf16, D, kN, kCw>;
  constexpr int kRw = G::kRw, kRowBytes = G::kRowBytes, kGroups = G::kGroups, kScores = G::kScores, kBlocks = G::kBlocks, kAcc = G::kAcc;
  constexpr int kSrcRow = kCodes ? D : kRowBytes, kSrcChunks = kSrcRow / 16;       // of a paged row
  constexpr int kLoads = 2 * kStageRows * kSrcChunks / G::kThreads;                // of a thread per stage, K and V
  constexpr int kTreeLoads = 2 * kStageRows * G::kChunks / G::kThreads;
  constexpr int kQf = kRowBytes / 16 / kGroups;                                     // 16-byte pieces of a lane's part of q
  constexpr int kParts = 2;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  float *const tree_place = reinterpret_cast<float *>(smem + kRw * G::kSlots * G::kStage);  // [128]: depths of the nodes
  __shared__ float s_ml[4][2][kWave];
  __shared__ int s_any;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int cw = wave % kCw, rw = wave / kCw, loader = tid % G::kThreads;
  if (tid == 0) s_any = 0;

  // ---- which range
  int b = 0, hk, block, piece, pieces, slot, steps, L, T;
  {
    const PagedSequence lanes = paged_sequence<kN, kCw>(p, lane);
    const PagedPlan plan = paged_plan<kN, kCw>(p, lanes);
    int at = blockIdx.x;
    if (at >= plan.n1 + plan.n2) return;
    const bool second = at >= plan.n1;
    at -= second ? plan.n1 : 0;
    const int n = second ? plan.n2 : plan.n1, even = n / 8 * 8, most = second ? plan.small : plan.big;
    at = at < even ? at % 8 * (even / 8) + at / 8 : at;  // neighbouring ranges (blocks of one unit's columns among them) on one XCD
    int before = 0, units_before = 0, cut_before = 0, start = 0, cut = 0, first = 0, count = 1;
    for (int b0 = 0; b0 < p.B; b0 += kWave) {
      const PagedSequence q = b0 == 0 ? lanes : paged_sequence<kN, kCw>(p, b0 + lane);
      const PagedShare s = paged_share(q.units, units_before, plan.whole);
      const int here = second ? s.rest : s.first, parts = paged_pieces(q.steps, most), mine = here * parts, incl = paged_scan(mine);
      const int cut_mine = parts > 1 ? mine : 0, cut_incl = paged_scan(cut_mine);
      const uint64_t le = __ballot(mine > 0 && before + incl - mine <= at);
      if (le != 0) {
        const int src = 63 - __builtin_clzll(le);
        b = b0 + src;
        start = __builtin_amdgcn_readlane(before + incl - mine, src);
        cut = __builtin_amdgcn_readlane(cut_before + cut_incl - cut_mine, src);
        first = second ? __builtin_amdgcn_readlane(s.first, src) : 0;
        count = __builtin_amdgcn_readlane(here, src);
      }
      before += __builtin_amdgcn_readlane(incl, 63);
      if (before > at || b0 + kWave >= p.B) break;
      cut_before += __builtin_amdgcn_readlane(cut_incl, 63);
      units_before += paged_sum(q.units);
    }
    // (the lengths of the first 64 sequences are at hand)
    const PagedSequence q = p.B <= kWave ? lanes : paged_sequence<kN, kCw>(p, b);
    const int src = p.B <= kWave ? b : 0;
    steps = __builtin_amdgcn_readlane(q.steps, src);
    L = __builtin_amdgcn_readlane(q.L, src);
    T = __builtin_amdgcn_readlane(q.T, src);
    const int n_blocks = __builtin_amdgcn_readlane(q.units, src) / p.H_kv, rest = at - start;
    pieces = paged_pieces(steps, most);
    // units next to each other, blocks of one K/V head first, then pieces
    piece = rest / count;
    const int u = first + rest - piece * count;
    hk = u / n_blocks;
    block = u - hk * n_blocks;
    const int first_slot = (second ? 0 : plan.n2) + cut + (rest - piece * count);
    slot = first_slot + piece * count;
    if (tid == 0 && piece == 0)
      *reinterpret_cast<u32x4 *>(p.records + 4 * (((size_t)b * p.H_kv + hk) * p.blocks + block)) =
          u32x4{(uint32_t)first_slot, (uint32_t)count, (uint32_t)pieces, 0};
  }
  const PagedStages st = paged_stages(L, T, p.window);
  const int quot = steps / pieces, extra = steps - quot * pieces;
  const int step0 = piece * quot + (piece < extra ? piece : extra), n_steps = quot + (piece < extra ? 1 : 0);
  const int n_stages = st.tree + st.cached;
  const size_t unit = (size_t)b * p.H_kv + hk;

  // ---- this lane's column
  const int columns = p.group * T, column = (block * kCw + cw) * kN + lane % kN;
  const bool there = column < columns, active = (block * kCw + cw) * kN < columns;
  const int col = there ? column : 0;  // lanes past the last column take the first: valid memory, never stored
  const int head = col / T, node = col - head * T;
  const size_t row_out = ((size_t)b * p.H + hk * p.group + head) * p.T_max + node;
  u32x4 qf[kQf];
#pragma unroll
  for (int x = 0; x < kQf; ++x) qf[x] = *reinterpret_cast<const u32x4 *>(p.q + row_out * kRowBytes + (kGroups * x + lane / kN) * 16);
  const u32x4 anc = *reinterpret_cast<const u32x4 *>(p.anc + ((size_t)b * p.T_max + node) * 2);
  const float slope = p.slopes ? p.slopes[hk * p.group + head] * kLog2e : 0.f;
  const float depth = (float)(__popc(anc.x) + __popc(anc.y) + __popc(anc.z) + __popc(anc.w) - 1);
  // places: positions less the root's.  A column sees those from `lowest` on, from all_see on every column of the wave does.
  const float lowest = p.window > kMostWindow ? -INFINITY : depth - (float)p.window + 1.f;
  float all_see = lowest;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) all_see = fmaxf(all_see, __shfl_xor(all_see, o, kWave));
  if (tid < T) {
    const u32x4 a = *reinterpret_cast<const u32x4 *>(p.anc + ((size_t)b * p.T_max + tid) * 2);
    tree_place[tid] = (float)(__popc(a.x) + __popc(a.y) + __popc(a.z) + __popc(a.w) - 1);
  } else if (tid < 128) {
    tree_place[tid] = 0.f;
  }
  lds_barrier();

  // ---- loader
  const uint32_t lds = (uint32_t)(uintptr_t)(lds_void *)smem + rw * (G::kSlots * G::kStage);
  constexpr int kWiden = kRowBytes / kSrcRow;                // chunks that one of a paged row becomes
  constexpr int kAtOnce = G::kThreads / kSrcChunks;          // rows that the threads load together; 64: those of K and of V
  static_assert(kAtOnce <= 64, "");
  const int ld_row = loader / kSrcChunks % kStageRows, ld_chunk = loader % kSrcChunks;
  const bool ld_v = kAtOnce == 64 && loader / kSrcChunks >= kStageRows;
  // (row and key of a thread's first load; of V where the first is V's)
  const uint32_t ld_k_at = ld_row * kRowBytes + (((kWiden * ld_chunk) ^ (ld_v ? G::v_key(ld_row) : G::k_key(ld_row))) << 4) + (ld_v ? G::kPart : 0);
  const uint32_t ld_v_at = ld_row * kRowBytes + (((kWiden * ld_chunk) ^ G::v_key(ld_row)) << 4) + G::kPart;
  const uint32_t ld_from = (ld_row & 15) * kSrcRow + ld_chunk * 16;
  int ids = -1, ids_from = -64;  // pages of the 16-row pieces of 32 steps' stages, a piece per lane
  auto stage_at = [&](int step) { return (step0 + step) * kRw + rw; };
  auto cached_row = [&](int stage) { return (stage - st.tree + st.first) * kStageRows; };
  // this wave's steps: the tree's stages, then cached ones
  const int steps_here = n_stages - rw - step0 * kRw <= 0 ? 0 : (n_stages - rw - step0 * kRw + kRw - 1) / kRw;  // to the unit's end
  const int steps_own = steps_here < n_steps ? steps_here : n_steps;
  const int tree_here = st.tree - rw - step0 * kRw <= 0 ? 0 : (st.tree - rw - step0 * kRw + kRw - 1) / kRw;
  const int steps_tree = tree_here < steps_own ? tree_here : steps_own, steps_cached = steps_own - steps_tree;
  u32x4 data[kLoads];
  uint32_t scale_byte[kLoads];
  uint32_t rows_there = 0;  // of the stage on its way
  // Requests a cached stage.  Without a branch around the loads: they stay on their way until their rows are stored.
  auto issue = [&](int step) __attribute__((always_inline)) {
    rows_there = 0;
    const int stage = stage_at(step);
    if (step >= ids_from + 32) {
      ids_from = step;
      const int at = stage_at(step + (lane >> 1)), row = cached_row(at) + 16 * (lane & 1);
      ids = at >= st.tree && row < L ? page_of(p.pages, b, row) : -1;
    }
    const int row0 = cached_row(stage), in_page = (1 << p.pages.shift) - 1;
    size_t row[2];  // where the two halves of the stage lie in the pool
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int page = __builtin_amdgcn_readlane(ids, 2 * (step - ids_from) + half);
      int n = L - row0 - 16 * half;
      n = n > 16 ? 16 : n;
      if (page >= 0 && n > 0) rows_there |= ((1u << n) - 1u) << (16 * half);
      row[half] = row_in_pool(p.pages, page < 0 ? 0 : page, hk, p.H_kv, (row0 + 16 * half) & in_page);
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int first = i * kAtOnce;  // of the 32 rows of K and then those of V
      const bool v = kAtOnce == 64 ? ld_v : first >= kStageRows;
      const bool second = kAtOnce >= 32 ? (ld_row & 16) != 0 : (first & 16) != 0;
      const size_t at = second ? row[1] : row[0];
      const int in_half = kAtOnce >= 16 ? 0 : first & 15;
      const u32x4 *from = reinterpret_cast<const u32x4 *>((v ? p.pages.v : p.pages.k) + at * kSrcRow + in_half * kSrcRow + ld_from);
      // Up to 64 columns no other workgroup reads these rows, and they need not stay in the caches: 32 x 8 heads of 8192 rows in 8 bits 108 -> 97 us.
      // (Rows that blocks of columns share 327 -> 331.)
      data[i] = kN == 16 ? __builtin_nontemporal_load(from) : *from;
      if constexpr (kCodes) scale_byte[i] = (v ? p.pages.v_scale : p.pages.k_scale)[at + in_half + (ld_row & 15)];
    }
  };
  // What issue() requested to LDS; rows that are not there as zeros, so that weights of zero meet nothing else.
  auto land = [&](uint32_t slot, uint32_t is_there) __attribute__((always_inline)) {
    const uint32_t k_at = made_anew(lds + slot + ld_k_at), v_at = made_anew(lds + slot + ld_v_at);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int first = i * kAtOnce, row = first % kStageRows;
      const bool v = kAtOnce < 64 && first >= kStageRows;
      const uint32_t at = v ? v_at : k_at, key = v ? G::v_key(row) : G::k_key(row);
      u32x4 x = data[i];
      if (is_there != ~0u) {  // uniform
        const bool ok = (is_there >> (ld_row + row)) & 1;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = ok ? x[j] : 0u;
      }
      if constexpr (!kCodes) {
        lds_to((at ^ (key << 4)) + row * kRowBytes, x);
      } else {
        const float scale = scale_of(scale_byte[i]);
        if constexpr (kBf16) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const u32x2 a = codes_to_bf16(x[2 * j], scale), z = codes_to_bf16(x[2 * j + 1], scale);
            lds_to((at ^ ((j ^ key) << 4)) + row * kRowBytes, u32x4{a.x, a.y, z.x, z.y});
          }
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) lds_to((at ^ ((j ^ key) << 4)) + row * kRowBytes, __builtin_bit_cast(u32x4, codes_to_f32(x[j], scale)));
        }
      }
    }
  };
  auto land_tree = [&](uint32_t slot, int stage) __attribute__((always_inline)) {
    const int left = T - stage * kStageRows;
    const size_t row0 = unit * p.T_max + stage * kStageRows;
    const int ln = (int)made_anew((uint32_t)loader) & (G::kThreads - 1);
#pragma unroll
    for (int i = 0; i < kTreeLoads; ++i) {
      const int x = i * G::kThreads + ln, part = x / (kStageRows * G::kChunks), row = x / G::kChunks % kStageRows, c = x % G::kChunks;
      u32x4 v = {0, 0, 0, 0};
      if (row < left) v = *reinterpret_cast<const u32x4 *>((part ? p.v_tree : p.k_tree) + (row0 + row) * kRowBytes + c * 16);
      lds_to(lds + slot + part * G::kPart + row * kRowBytes + ((c ^ (part ? G::v_key(row) : G::k_key(row))) << 4), v);
    }
  };

  float m_run, l_run;
  Acc<kN> o_acc[kBlocks];
  constexpr float kTau = 8.f;

  // ---- a stage: its scores, weights and what they add to O.  `seen`: a bit per row of the stage that exists.
  const int in_n = lane % kN, g = lane / kN;
  const uint32_t k_read = lds + in_n * kRowBytes + ((g ^ G::k_key(in_n)) << 4);
  uint32_t v_read = lds + G::kPart;  // bf16: a transposing read's row and 8 bytes; fp32: a number of row 4 * g
  if constexpr (kBf16) {
    const int q = 4 * g + ((lane & 15) >> 2), c = (kN == 32 ? 2 * ((lane >> 4) & 1) : 0) + ((lane & 3) >> 1);
    v_read += q * kRowBytes + ((c ^ G::v_key(q)) << 4) + 8 * (lane & 1);
  } else {
    v_read += 4 * g * kRowBytes + (((in_n >> 2) ^ G::v_key(4 * g)) << 4) + 4 * (in_n & 3);
  }
  auto take_stage = [&](uint32_t slot, int stage, uint32_t seen, auto with_care) __attribute__((always_inline)) {
    constexpr bool kCareful = decltype(with_care)::value;
    const bool tree = stage < st.tree;
    const uint32_t k_at = made_anew(k_read + slot), v_at = made_anew(v_read + slot);
    float sc[kScores];
#pragma unroll
    for (int tile = 0; tile < 32 / kN; ++tile) {
      Acc<kN> acc;
      clear(acc);
      constexpr int kBatch = kQf < 8 ? kQf : 8;  // pieces that are requested together, so that products wait for LDS once
#pragma unroll
      for (int x0 = 0; x0 < kQf; x0 += kBatch) {
        u32x4 a[kBatch];
#pragma unroll
        for (int x = 0; x < kBatch; ++x)
          a[x] = lds_from<u32x4>((k_at ^ (((kGroups * (x0 + x)) ^ G::k_key(tile * kN)) << 4)) + tile * kN * kRowBytes);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int x = 0; x < kBatch; ++x) {
          if constexpr (kBf16) {
            acc = product<kN>(a[x], qf[x0 + x], acc);
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) acc = product<kN>(__uint_as_float(a[x][j]), __uint_as_float(qf[x0 + x][j]), acc);
          }
        }
      }
#pragma unroll
      for (int r = 0; r < kAcc; ++r) sc[tile * kAcc + r] = acc[r];
    }
    mfma_settle();
    // ---- scores; times `unit_of` they are in the exponent's (log2) domain
    float unit_of = p.scale_log2e;
    if (p.cap_in > 0.f) {
      unit_of = 1.f;
      // cap tanh(x / cap) as in capped(), whose fraction alone does where no score of the wave is beyond 3/4 of the cap
      float most = 0.f;
#pragma unroll
      for (int x = 0; x < kScores; ++x) most = fmaxf(most, fabsf(sc[x]));
      if (__builtin_amdgcn_ballot_w64(!(most * p.cap_in < .75f)) == 0) {
#pragma unroll
        for (int x = 0; x < kScores; ++x) {
          const float y = sc[x] * p.cap_in, y2 = y * y;
          sc[x] = sc[x] * p.scale_log2e * fmaf(y2, y2 + 105.f, 945.f) * __builtin_amdgcn_rcpf(fmaf(y2, fmaf(15.f, y2, 420.f), 945.f));
        }
      } else {
#pragma unroll
        for (int x = 0; x < kScores; ++x) sc[x] = capped(sc[x], p.cap_log2e, p.cap_in);
      }
    }
    const float first = tree ? 0.f : (float)(cached_row(stage) - L);  // place of the stage's first cached row
    if (p.slopes || first < all_see) {
#pragma unroll
      for (int x4 = 0; x4 < kScores / 4; ++x4) {
        const int row = 4 * kGroups * x4 + 4 * g;
        f32x4 place = {first + (float)row, first + (float)(row + 1), first + (float)(row + 2), first + (float)(row + 3)};
        if (tree) place = *reinterpret_cast<const f32x4 *>(tree_place + stage * kStageRows + row);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (p.slopes) sc[4 * x4 + j] = fmaf(slope, place[j] - depth, sc[4 * x4 + j] * unit_of);
          sc[4 * x4 + j] = place[j] >= lowest ? sc[4 * x4 + j] : -INFINITY;
        }
      }
      if (p.slopes) unit_of = 1.f;
    }
    if (tree) seen &= stage == 0 ? anc.x : stage == 1 ? anc.y : stage == 2 ? anc.z : anc.w;
    if (tree || seen != ~0u) {  // uniform
      const uint32_t vis = seen >> (4 * g);
#pragma unroll
      for (int x = 0; x < kScores; ++x) sc[x] = ((vis >> (4 * kGroups * (x >> 2) + (x & 3))) & 1u) ? sc[x] : -INFINITY;
    }
    float m_blk = -INFINITY;
#pragma unroll
    for (int x = 0; x < kScores; ++x) m_blk = fmaxf(m_blk, sc[x]);
    {  // the column's other scores are in the lanes 32 (and 16) away
      uint32_t lo = __float_as_uint(m_blk), hi = lo;
      swap_halves(lo, hi);
      m_blk = fmaxf(__uint_as_float(lo), __uint_as_float(hi));
      if constexpr (kN == 16) m_blk = fmaxf(m_blk, __shfl_xor(m_blk, 16, kWave));
    }
    m_blk *= unit_of;
    // A new reference is adopted only when the maximum exceeds the old one by 2^8: weights then exceed 1, by a factor that fp32 sums and bf16
    // weights hold, and O is hardly ever scaled.  With care they are at most kBack as they meet V: no sum exceeds its largest value.
    if (__builtin_amdgcn_ballot_w64(m_blk > (kCareful ? m_run : m_run + kTau)) != 0) {
      const float m_new = fmaxf(m_run, m_blk), m_safe = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = fast_exp2(m_run - m_safe);
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < kBlocks; ++db)
#pragma unroll
        for (int r = 0; r < kAcc; ++r) o_acc[db][r] = kCareful ? weighed(o_acc[db][r], alpha) : o_acc[db][r] * alpha;
      m_run = m_new;
    }
    const float neg_m = -(m_run == -INFINITY ? 0.f : m_run);
    uint32_t live = 0;  // scores of rows that are seen
    if constexpr (kCareful) {
#pragma unroll
      for (int x = 0; x < kScores; ++x) live |= sc[x] > -INFINITY ? 1u << x : 0u;
    }
    // V^T of the rows of 8 scores, requested ahead of what they are multiplied with
    u32x4 vt[kBf16 ? 2 : 1][kBf16 ? kBlocks : 1];
    auto read_v = [&](int half) __attribute__((always_inline)) {
#pragma unroll
      for (int db = 0; db < kBlocks; ++db)
#pragma unroll
        for (int hi = 0; hi < 2; ++hi) {
          const int row = 4 * kGroups * (2 * half + hi);
          const uint32_t at = (v_at ^ (((db * (kN / 8)) ^ G::v_key(row)) << 4)) + row * kRowBytes;
          const u32x2 t = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<LdsPtr<s16x4>>((uintptr_t)at)));
          vt[half & 1][db][2 * hi] = t.x;
          vt[half & 1][db][2 * hi + 1] = t.y;
        }
      __builtin_amdgcn_sched_barrier(0);
    };
    if constexpr (kBf16) read_v(0);
#pragma unroll
    for (int x = 0; x < kScores; ++x) {
      sc[x] = fast_exp2(fmaf(sc[x], unit_of, neg_m));
      l_run += sc[x];  // of the weights as they are: lse is an fp32 result
      if constexpr (kCareful) sc[x] *= kBack;
    }
    if constexpr (kBf16) {
#pragma unroll
      for (int half = 0; half < kScores / 8; ++half) {  // a product's rows are those of 8 scores
        if (half + 1 < kScores / 8) read_v(half + 1);
        uint32_t pw[kParts][4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          float p0 = sc[8 * half + 2 * x], p1 = sc[8 * half + 2 * x + 1];
#pragma unroll
          for (int part = 0; part < kParts; ++part) {  // rounded to bf16, and what that leaves
            const uint32_t w2 = cvt_pk_bf16(p0, p1);
            pw[part][x] = w2;
            p0 -= __uint_as_float(w2 << 16);
            p1 -= __uint_as_float(w2 & 0xffff0000u);
          }
        }
#pragma unroll
        for (int db = 0; db < kBlocks; ++db) {
          u32x4 &v = vt[half & 1][db];
          if constexpr (kCareful) {
            u32x4 code, one;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              one[x] = (live >> (8 * half + 2 * x) & 1 ? 0x3f80u : 0u) | (live >> (8 * half + 2 * x + 1) & 1 ? 0x3f800000u : 0u);
              uint32_t pair = v[x];
              code[x] = take_not_finite(pair);
              v[x] = pair;
            }
            Acc<kN> codes;
            clear(codes);
            codes = product<kN>(code, one, codes);
            mfma_settle();
#pragma unroll
            for (int r = 0; r < kAcc; ++r) o_acc[db][r] += not_finite_sum(codes[r]);
          }
#pragma unroll
          for (int part = kParts - 1; part >= 0; --part)  // the small part first
            o_acc[db] = product<kN>(v, u32x4{pw[part][0], pw[part][1], pw[part][2], pw[part][3]}, o_acc[db]);
        }
      }
    } else {
#pragma unroll
      for (int db = 0; db < kBlocks; ++db) {
        Acc<kN> codes;
        if constexpr (kCareful) clear(codes);
#pragma unroll
        for (int x = 0; x < kScores; ++x) {  // the product's rows are those of score x of the column's lanes
          const int row = 4 * kGroups * (x >> 2) + (x & 3);
          float v = lds_from<float>((v_at ^ (((db * (kN / 4)) ^ G::v_key(row)) << 4)) + row * kRowBytes);
          if constexpr (kCareful) {
            const float code = not_finite_code(__float_as_uint(v));
            v = code == 0.f ? v : 0.f;
            codes = product<kN>(code, live >> x & 1 ? 1.f : 0.f, codes);
          }
          o_acc[db] = product<kN>(v, sc[x], o_acc[db]);
        }
        if constexpr (kCareful) {
          mfma_settle();
#pragma unroll
          for (int r = 0; r < kAcc; ++r) o_acc[db][r] += not_finite_sum(codes[r]);
        }
      }
    }
  };
  auto walk = [&](auto with_care) __attribute__((always_inline)) {
    m_run = -INFINITY;
    l_run = 0.f;
#pragma unroll
    for (int db = 0; db < kBlocks; ++db) clear(o_acc[db]);
    ids_from = -64;
    if (steps_cached > 0) issue(steps_tree);  // (before the tree's own rows are waited for)
    for (int step = 0; step < steps_tree; ++step) {
      const int stage = stage_at(step), left = T - stage * kStageRows;
      const uint32_t slot = G::kSlots == 2 ? (step & 1) * G::kStage : 0;
      land_tree(slot, stage);
      if constexpr (kCw > 1) lds_barrier();
      if (active) take_stage(slot, stage, left >= 32 ? ~0u : (1u << left) - 1u, with_care);
    }
    for (int step = steps_tree; step < steps_tree + steps_cached; ++step) {
      const uint32_t slot = G::kSlots == 2 ? (step & 1) * G::kStage : 0, seen = rows_there;
      land(slot, seen);
      issue(step + 1 < steps_tree + steps_cached ? step + 1 : step);  // behind the last: that once more, not used
      if constexpr (kCw > 1) lds_barrier();
      if (active && seen != 0) take_stage(slot, stage_at(step), seen, with_care);
    }
    mfma_settle();  // O is read by what follows (within the loop it is read behind the next scores' wait)
  };
  // What was requested so far is here: the loops' waits are for their own requests alone.
  __builtin_amdgcn_s_waitcnt(0);
  walk(std::false_type{});
  bool careful;
  {
    // Zero weights times values of V that are not finite, or sums that leave the range of fp32 (or would, joined): such a range is done once more, with care.
    float sum = 0.f;
#pragma unroll
    for (int db = 0; db < kBlocks; ++db)
#pragma unroll
      for (int r = 0; r < kAcc; ++r) sum += fabsf(o_acc[db][r]);
    if (active && __builtin_amdgcn_ballot_w64(!(sum < kMostPlain)) != 0 && lane == 0) s_any = 1;
    lds_barrier();
    careful = s_any != 0;
    if (careful) {
      lds_barrier();
      walk(std::true_type{});
    }
  }

  // ---- results.  Waves of other rows have parts of the same columns: they meet in LDS, and share the quads of O.
#pragma unroll
  for (int o = kN; o < kWave; o <<= 1) l_run += __shfl_xor(l_run, o, kWave);
  constexpr int kOwn = G::kQuads / kRw;  // quads that a wave stores
  f32x4 mine[kOwn];
  const int first_quad = rw * kOwn;
  auto quad_of = [&](int x) __attribute__((always_inline)) {
    const Acc<kN> &o = o_acc[x / (kAcc / 4)];
    const int r = x % (kAcc / 4) * 4;
    return f32x4{o[r], o[r + 1], o[r + 2], o[r + 3]};
  };
  if constexpr (kRw > 1) {
    s_ml[wave][0][lane] = m_run;
    s_ml[wave][1][lane] = l_run;
    lds_barrier();  // everyone is done with the stages too
    float M = -INFINITY, total = 0.f;
#pragma unroll
    for (int w = 0; w < kRw; ++w) M = fmaxf(M, s_ml[w * kCw + cw][0][lane]);
    const float safe = M == -INFINITY ? 0.f : M;
#pragma unroll
    for (int w = 0; w < kRw; ++w) {
      total += fast_exp2(s_ml[w * kCw + cw][0][lane] - safe) * s_ml[w * kCw + cw][1][lane];  // (sums are finite, or NaN that stays)
    }
    const float f = fast_exp2(m_run - safe);
    f32x4 *const room = reinterpret_cast<f32x4 *>(smem);  // [4 waves][quads][lanes]
#pragma unroll
    for (int x = 0; x < G::kQuads; ++x) {
      const f32x4 v = quad_of(x);
      room[(wave * G::kQuads + x) * kWave + lane] = f32x4{weighed(v[0], f), weighed(v[1], f), weighed(v[2], f), weighed(v[3], f)};
    }
    lds_barrier();
#pragma unroll
    for (int x = 0; x < kOwn; ++x) {
      mine[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kRw; ++w) mine[x] += room[((w * kCw + cw) * G::kQuads + first_quad + x) * kWave + lane];
    }
    m_run = M;
    l_run = total;
  } else {
#pragma unroll
    for (int x = 0; x < kOwn; ++x) mine[x] = quad_of(x);
  }
  if (!there) return;
  if (pieces == 1) {
    const float inv = inverse(l_run) * (careful ? kForth : 1.f);
#pragma unroll
    for (int x = 0; x < kOwn; ++x) store_quad<kBf16>(p.out, row_out * D + 4 * kGroups * (first_quad + x) + 4 * (lane / kN), mine[x], inv);
    if (p.lse && rw == 0 && lane < kN) p.lse[row_out] = (m_run + __builtin_amdgcn_logf(l_run)) * kLn2;
  } else {
    const size_t part = (size_t)slot * kCw + cw;
#pragma unroll
    for (int x = 0; x < kOwn; ++x) *reinterpret_cast<f32x4 *>(p.part_o + ((part * G::kQuads + first_quad + x) * kWave + lane) * 4) = mine[x];
    if (rw == 0) {
      p.part_ml[(part * 2 + 0) * kWave + lane] = m_run;
      p.part_ml[(part * 2 + 1) * kWave + lane] = careful ? -l_run : l_run;  // the sign says so: sums are not negative
    }
  }
}

// out = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s over the pieces s of a unit, always in the same order.  A workgroup has kN columns of a
// unit and four quads of O; its waves take the pieces in turn and meet in LDS.
template <bool kBf16, int D, int kN, int kCw, int kWaves>
__global__ __launch_bounds__(kWaves *kWave) void paged_merge_kernel(PagedParams p) {
  using G = PagedGeo<kBf16, D, kN, kCw>;
  constexpr int kShare = G::kQuads / 4;  // workgroups that share the columns' O
  __shared__ float s_part[kWaves > 1 ? kWaves - 1 : 1][18][kWave];
  const int share = blockIdx.x % kShare, cw = blockIdx.x / kShare % kCw;
  const unsigned item = blockIdx.x / (kCw * kShare);
  const unsigned unit = item / (unsigned)p.blocks, b = unit / (unsigned)p.H_kv;
  const int block = (int)(item - unit * (unsigned)p.blocks), hk = (int)(unit - b * (unsigned)p.H_kv);
  const u32x4 record = *reinterpret_cast<const u32x4 *>(p.records + 4 * (size_t)item);  // (on its way with the number of nodes; not looked at beyond the columns)
  const int T = clamped(p.n_nodes[b] - 1, p.T_max - 1) + 1, columns = p.group * T;
  if ((block * kCw + cw) * kN >= columns) return;
  const int first = (int)record.x, stride = (int)record.y, P = (int)record.z;
  if (P <= 1) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), column = (block * kCw + cw) * kN + lane % kN;
  const bool there = column < columns;
  const int ln = there ? lane : 0;  // lanes past the last column read lane 0's data and store nothing
  float acc[16], M = -INFINITY, total = 0.f;
  bool careful = false;  // acc is kBack of what it stands for, as are pieces made with care
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[r] = 0.f;
  auto join = [&](const float (&o)[16], float m, float signed_l) __attribute__((always_inline)) {
    const bool theirs = signbit(signed_l);
    const float M_new = fmaxf(M, m), safe = M_new == -INFINITY ? 0.f : M_new, l = fabsf(signed_l);
    float a_old = fast_exp2(M - safe), a_new = fast_exp2(m - safe);
    total = total * a_old + l * a_new;  // (finite, or NaN that stays)
    a_old *= theirs && !careful ? kBack : 1.f;
    a_new *= careful && !theirs ? kBack : 1.f;
    careful = careful || theirs;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = weighed(acc[r], a_old) + weighed(o[r], a_new);
    M = M_new;
  };
  constexpr int kTogether = 4;  // pieces of a wave that are requested together
  for (int s0 = wave; s0 < P; s0 += kTogether * kWaves) {
    f32x4 o[kTogether][4];
    float m[kTogether], l[kTogether];
#pragma unroll
    for (int k = 0; k < kTogether; ++k) {
      const int s = s0 + k * kWaves < P ? s0 + k * kWaves : P - 1;  // past the last: that once more, not used
      const size_t part = ((size_t)first + (size_t)s * stride) * kCw + cw;
      m[k] = p.part_ml[(part * 2 + 0) * kWave + ln];
      l[k] = p.part_ml[(part * 2 + 1) * kWave + ln];
#pragma unroll
      for (int x = 0; x < 4; ++x) o[k][x] = *reinterpret_cast<const f32x4 *>(p.part_o + ((part * G::kQuads + 4 * share + x) * kWave + ln) * 4);
    }
    __builtin_amdgcn_sched_barrier(0);  // all of them are requested first
#pragma unroll
    for (int k = 0; k < kTogether; ++k) {
      if (s0 + k * kWaves < P) {  // uniform
        float x[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = o[k][r / 4][r % 4];
        join(x, m[k], l[k]);
      }
    }
  }
  if constexpr (kWaves > 1) {
    if (wave > 0) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s_part[wave - 1][r][lane] = acc[r];
      s_part[wave - 1][16][lane] = M;
      s_part[wave - 1][17][lane] = careful ? -total : total;
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 0; w < kWaves - 1; ++w) {
      float x[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = s_part[w][r][lane];
      join(x, s_part[w][16][lane], s_part[w][17][lane]);
    }
  }
  if (!there) return;
  const int head = column / T, node = column - head * T;
  const size_t row = ((size_t)b * p.H + hk * p.group + head) * p.T_max + node;
  const float inv = inverse(total) * (careful ? kForth : 1.f);
#pragma unroll
  for (int x = 0; x < 4; ++x)
    store_quad<kBf16>(p.out, row * D + 4 * G::kGroups * (4 * share + x) + 4 * (lane / kN), f32x4{acc[4 * x], acc[4 * x + 1], acc[4 * x + 2], acc[4 * x + 3]}, inv);
  if (p.lse && share == 0 && lane < kN) p.lse[row] = (M + __builtin_amdgcn_logf(total)) * kLn2;
}

// ------------------------------------------------------------------------------------
// host side
// ------------------------------------------------------------------------------------
// Partial results of a call, at most: as many ranges as run at once, of units that are left over, and twice as many of units that come first (a unit that
// is cut is longer than an equal share: it has fewer pieces than twice its shares).
constexpr int kPagedResident = 512, kPagedSlots = 3 * kPagedResident;
constexpr long long kPagedUnits = 8 * kPagedResident;  // from so many on none is cut: the last round is an eighth of the call at most

static long long paged_slots(int B, int H, int L_max) {
  const long long stages = (L_max + kStageRows - 1ll) / kStageRows + PROPD_MAX_TREE / kStageRows;
  const long long most = (long long)B * H * 4 * stages;  // blocks of a unit: no more than four per head
  return most < kPagedSlots ? most : kPagedSlots;
}

size_t paged_attention_workspace_bytes(int B, int H, int L_max, int T_max) {
  const size_t slots = (size_t)paged_slots(B, H, L_max), blocks = (size_t)(T_max + 31) / 32;
  return slots * (4 * 16 * kWave * 4 * 4) + slots * (4 * 2 * kWave * 4) + align_up((size_t)B * H * blocks * 16, 256);
}

template <bool kBf16, bool kCodes, int D, int kN, int kCw>
static bool launch_paged(PagedParams p, int L_max, hipStream_t st) {
  using G = PagedGeo<kBf16, D, kN, kCw>;
  static std::atomic<uint64_t> set{0};
  if (!allow_lds(reinterpret_cast<const void *>(&paged_attn_kernel<kBf16, kCodes, D, kN, kCw>), G::kLds, set)) return false;
  p.blocks = (p.group * p.T_max + G::kColumns - 1) / G::kColumns;
  const long long units = (long long)p.B * p.H_kv * p.blocks;
  const int resident = (kBf16 ? 2 : 1) * compute_units();
  p.resident = resident < kPagedResident ? resident : kPagedResident;
  const long long steps = ((L_max + kStageRows - 1ll) / kStageRows + (p.T_max + kStageRows - 1) / kStageRows + G::kRw - 1) / G::kRw;
  // Few steps are not worth a second kernel (8 units of two steps 9.0 us instead of 12.0), nor a short range of 128 columns its partial result of 64 KB: 32
  // units of 20 steps in pieces of at least 6 / 4 / 2 steps 18.6 / 19.0 / 24.2, 80 of 11 23.5 / 26.7 / 27.7; fp32 products take longer: 24 of 34 23.5 / 21.3 / 20.6.
  p.least = G::kRw > 1 ? 1 : kN == 32 && kBf16 ? 6 : 2;
  p.may_split = units < kPagedUnits && steps > (G::kRw == 1 ? p.least : 2) ? 1 : 0;
  // (ranges that come first: units, and the pieces of those that are cut; then the others')
  long long grid = units;
  if (p.may_split) {
    grid += units <= p.resident ? p.resident : 3ll * p.resident;
    if (grid > units * steps) grid = units * steps;
  }
  hipLaunchKernelGGL((paged_attn_kernel<kBf16, kCodes, D, kN, kCw>), dim3((unsigned)grid), dim3(kPagedThreads), G::kLds, st, p);
  if (!launch_ok()) return false;
  if (!p.may_split) return true;
  const dim3 merge((unsigned)(units * kCw * (G::kQuads / 4)));
  if (units * kCw <= 64) hipLaunchKernelGGL((paged_merge_kernel<kBf16, D, kN, kCw, 4>), merge, dim3(4 * kWave), 0, st, p);
  else hipLaunchKernelGGL((paged_merge_kernel<kBf16, D, kN, kCw, 1>), merge, dim3(kWave), 0, st, p);
  return launch_ok();
}

template <bool kBf16, bool kCodes, int D>
static bool launch_paged(const PagedParams &p, int L_max, hipStream_t st) {
  const int columns = p.group * p.T_max;
  if (columns <= 16) return launch_paged<kBf16, kCodes, D, 16, 1>(p, L_max, st);
  // Blocks of 64 columns read every row from LDS twice as often per product as those of 128, and there are more of them: better where all stages of a
  // call hardly fill the chip.  Calls (sequences, query heads on K/V heads, nodes, rows; 8 bits, d = 128), us, 64 / 128 columns:
  //   bf16  1, 32 on 8, 32, 500: 15.3 / 16.4     3, 64 on 8, 113, 12: 19.0 / 29.0     2, 16 on 4, 48, 1024: 26.0 / 23.7    4, 32 on 8, 64, 2048: 42 / 36
  //   fp32                      20.3 / 24.6                          40.4 / 40.4                          29.2 / 32.1                          123 / 101
  const long long blocks = (long long)p.B * p.H_kv * ((columns + 127) / 128);
  const long long stages = (L_max + kStageRows - 1ll) / kStageRows + (p.T_max + kStageRows - 1) / kStageRows;
  // The lengths are on the device: stages are those that the table has room for, here and where a second kernel is chosen.  In tables of 8192 rows (and of
  // 131072) the first of these takes 19.0 (bf16) and 24.6 (fp32), one token over 40 rows 10.0 instead of 7.7, calls of more stages what they take otherwise.
  const bool few = blocks * stages <= 1024 && (!kBf16 || stages <= 20);
  return columns <= 64 || few ? launch_paged<kBf16, kCodes, D, 16, 4>(p, L_max, st) : launch_paged<kBf16, kCodes, D, 32, 4>(p, L_max, st);
}

}  // namespace propd

extern "C" propd_status propd_paged_attention(const propd_tree *tree, propd_dtype dt, int32_t H, int32_t H_kv, int32_t d,
                                              const propd_score_rule *rule, const void *q, const propd_paged_cache *cache, const void *k_tree,
                                              const void *v_tree, const int32_t *seq_lens, void *out, float *lse, void *workspace,
                                              size_t workspace_bytes, void *hip_stream) {
  using namespace propd;
  if (!tree || tree->B < 1 || tree->T_max < 1 || tree->T_max > PROPD_MAX_TREE || H < 1 || H_kv < 1 || H % H_kv != 0 || !score_rule_ok(rule) ||
      !tree->n_nodes || !tree->anc || !q || !k_tree || !v_tree || !seq_lens || !out)
    return PROPD_ERR_INVALID_ARG;
  if (dt != PROPD_BF16 && dt != PROPD_F32) return PROPD_ERR_INVALID_ARG;
  const propd_status status = paged_cache_check(cache, dt);
  if (status != PROPD_OK) return status;
  if (d != 64 && d != 128) return PROPD_ERR_UNSUPPORTED;
  for (const void *ptr : {q, k_tree, v_tree, (const void *)out, (const void *)tree->anc, (const void *)workspace})
    if (reinterpret_cast<uintptr_t>(ptr) % 16 != 0) return PROPD_ERR_INVALID_ARG;
  const long long nodes = (long long)tree->B * H * tree->T_max;
  if (nodes > (1ll << 27) || (long long)tree->B * H > (1ll << 20)) return PROPD_ERR_UNSUPPORTED;
  const int L_max = cache->table_pages * cache->page_rows;
  const size_t needed = paged_attention_workspace_bytes(tree->B, H, L_max, tree->T_max);
  if (!workspace || workspace_bytes < needed) return PROPD_ERR_WORKSPACE;
  PagedParams p;
  p.pages = pages_of(cache);
  p.q = reinterpret_cast<const unsigned char *>(q);
  p.k_tree = reinterpret_cast<const unsigned char *>(k_tree);
  p.v_tree = reinterpret_cast<const unsigned char *>(v_tree);
  p.out = reinterpret_cast<unsigned char *>(out);
  p.lse = lse;
  p.seq_lens = seq_lens;
  p.n_nodes = tree->n_nodes;
  p.anc = tree->anc;
  p.slopes = rule->slopes;
  p.B = tree->B;
  p.H = H;
  p.H_kv = H_kv;
  p.group = H / H_kv;
  p.T_max = tree->T_max;
  p.blocks = 0;
  p.window = window_of(rule);
  p.scale_log2e = rule->scale * kLog2e;
  p.cap_in = rule->cap > 0.f ? rule->scale / rule->cap : 0.f;
  p.cap_log2e = rule->cap * kLog2e;
  const long long slots = paged_slots(p.B, H, L_max);
  char *ws = reinterpret_cast<char *>(workspace);
  p.part_o = reinterpret_cast<float *>(ws);
  ws += (size_t)slots * (4 * 16 * kWave * 4 * 4);
  p.part_ml = reinterpret_cast<float *>(ws);
  ws += (size_t)slots * (4 * 2 * kWave * 4);
  p.records = reinterpret_cast<int32_t *>(ws);
  p.resident = p.least = p.may_split = 0;  // by the shape of the waves
  hipStream_t st = as_stream(hip_stream);
  const bool bf16 = dt == PROPD_BF16, codes = cache->dt == PROPD_E4M3;
  bool ok;
  if (d == 128) {
    ok = bf16 ? (codes ? launch_paged<true, true, 128>(p, L_max, st) : launch_paged<true, false, 128>(p, L_max, st))
              : (codes ? launch_paged<false, true, 128>(p, L_max, st) : launch_paged<false, false, 128>(p, L_max, st));
  } else {
    ok = bf16 ? (codes ? launch_paged<true, true, 64>(p, L_max, st) : launch_paged<true, false, 64>(p, L_max, st))
              : (codes ? launch_paged<false, true, 64>(p, L_max, st) : launch_paged<false, false, 64>(p, L_max, st));
  }
  return ok ? PROPD_OK : PROPD_ERR_DEVICE;
}
