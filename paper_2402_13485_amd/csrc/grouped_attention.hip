// Tree attention whose K/V heads are shared by several query heads, with capped and biased scores, a window and cached
// rows at positions of their own.
//
// bf16 path.  A unit is a (sequence, K/V head, block of 128 query columns): the nodes of all query heads that read
// the K/V head lie side by side, column r is node r % T of head r / T, so that a K or V row is read once for all of them.
//   - A workgroup takes one range of a unit's 32-row stages of K and V (cached rows, then tree rows) and streams it through
//     a ring in LDS by direct loads; its four waves own 32 columns each.
//   - S^T = K . Q^T by the 32x32x16 products, so that a lane owns a column: the softmax statistics, the query's
//     position, slope and ancestor set are per-lane scalars, and the weights, as sums of bf16 values (kParts), are the B
//     operand of O^T += V^T . P^T (V^T by the transposing LDS read).  The scores of stage i + 1 are multiplied in front
//     of the softmax of stage i.
//   - A unit is cut into as many ranges as the chip needs (plan_ranges); partial results are merged by a second kernel, in
//     the order of the ranges.
#include "attention_device.h"
#include "score_rule.h"

namespace propd {

constexpr int kGroupThreads = 256;
// Workgroups that run at once, and partial results of a call (two per share), at most.  The chip has 256 compute units.
constexpr int kMostResident = 512, kGroupSlots = 2 * kMostResident;

struct GroupedParams {
  const uint16_t *q, *k_cache, *v_cache, *k_tree, *v_tree;
  uint16_t *out;
  float *lse;
  const int32_t *seq_lens, *n_nodes, *position, *dropped;
  const uint64_t *anc;
  const float *slopes;
  int B, H, H_kv, group, T_max, L_max;
  int blocks;           // blocks of 128 columns of a unit's tree of T_max nodes
  int window;           // window_of
  float scale_log2e, cap_in, cap_log2e;  // cap_in: scale / cap
  float *part_o;        // [slots][4 waves][16 blocks][64 lanes][4]
  float *part_ml;       // [slots][4 waves][m | l][64 lanes]
  int32_t *records;     // [B * H_kv * blocks][4]: first slot, slots between pieces, pieces (1: no merge), how much earlier the later ones lie
  int slots, resident;  // partial results there is room for; workgroups that run at once
  int may_split;
};

__device__ __forceinline__ Lengths lengths_of(const GroupedParams &p, int b) {
  return lengths_of(p.seq_lens, p.n_nodes, p.dropped, p.L_max, p.T_max, b);
}

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Stages of a unit of a sequence: cached rows from `first_stage` on (a window hides those before it where rows
// lie in the order of their positions), then tree rows.
struct Stages {
  int first, cached, tree;
};
__device__ __forceinline__ Stages stages_of(int L, int T, int window, bool in_order) {
  Stages s;
  const int row = in_order && L > window ? L - window + 1 : 0;  // the first row that the root sees
  s.first = row / kStageRows;
  s.cached = (L + kStageRows - 1) / kStageRows - s.first;
  s.cached = s.cached < 0 ? 0 : s.cached;
  s.tree = (T + kStageRows - 1) / kStageRows;
  return s;
}

// Quotients of whole numbers without the long sequence of a division.  below(n, d): n / d rounded down, exact for n below
// 2^20.  pieces_of(n, d): n / d rounded up for any n >= 1, d >= 1, at least 1 and at most n; off by one at most far
// beyond 2^20 (and the same value wherever it is asked for).
__device__ __forceinline__ int below(int n, int d) { return (int)(((float)n + .5f) * __builtin_amdgcn_rcpf((float)d)); }
__device__ __forceinline__ int quotient(int n, int d) { return n < (1 << 20) ? below(n, d) : n / d; }
__device__ __forceinline__ int pieces_of(int n, int d) {
  const int x = (int)(((float)n + (float)d - .5f) * __builtin_amdgcn_rcpf((float)d));
  return x < 1 ? 1 : (x > n ? n : x);
}

// The lengths of a sequence, of this lane's or of one for all lanes, and what they make: stages of a unit, units of the sequence (0
// beyond the batch).
struct Sequence {
  int L, T, dropped;
  __device__ __forceinline__ Stages stages(const GroupedParams &p) const { return stages_of(L, T, p.window, p.position == nullptr); }
  __device__ __forceinline__ int blocks(const GroupedParams &p) const { return (p.group * T + 127) / 128; }
  __device__ __forceinline__ int count(const GroupedParams &p) const {
    const Stages s = stages(p);
    return T > 0 ? s.cached + s.tree : 0;
  }
  __device__ __forceinline__ int units(const GroupedParams &p) const { return p.H_kv * blocks(p); }
};
__device__ __forceinline__ Sequence lane_sequence(const GroupedParams &p, int b) {
  if (b >= p.B) return {0, 0, 0};
  const Lengths n = lengths_of(p, b);
  return {n.L, n.T, n.dropped};
}

// How the units are cut.  Every workgroup works the same plan out from the lengths, in few steps: they stand in front of its first
// load.
//   kAlike   All sequences alike: as many whole units as there are workgroups that run at once, as often as that goes, then
//            the units left over in `pieces` ranges each, piece by piece.  After whole units these are as many ranges as there are compute
//            units, however long: 128 units of 132 stages left of 640 take 281 us in 256 ranges, 301 in 512.
//   kRanges  A range is at most `most` stages, a unit of s stages has pieces_of(s, most) of them, equally long; the least
//            `most` whose ranges all run at once.
//   kShares  Every workgroup has an equal share of the list of all stages, which may cross units (each crossing: another unit's first
//            loads and a partial result).
// How many workgroups run at once (`slots`): one per compute unit, two where that leaves ranges of more than kLongRange
// stages.  A stage of a workgroup that shares its compute unit takes 1.6 (d = 64) to 1.9 of the time, so two halves of a range save little, and
// each range costs about 5 us of first loads and result and 128 KB of partial result written and read.  Calls, us, 256 / 512
// ranges: 40 units of 49 stages 31 / 33, 128 of 66 54 / 51, 128 of 128 82 / 75, 256 of 130 capped 174 / 163, with positions and d = 64 147 / 118;
// 256 of 34 48 / 54.
// Up to as many units as workgroups take kRanges where its ranges are not much longer than an equal share: up to twice as long, up to a
// quarter longer where that share is more than kLongRange stages, which one more crossing adds little to.  Where one workgroup per
// compute unit leaves no room to cut a unit, two may.  Calls of 8 K/V heads, us, ranges / shares: 24 sequences of up to 1024 rows (17 stages) 54 / 60,
// 16 of 256 and one of 8192 (13 stages) 35.5 / 48, 32 of up to 2048 rows at positions of their own (42 stages, ranges 1.44 times as long) 112 / 102;
// 31 of 256 and one of 8192 in 256 units, not cut / cut for two workgroups 231 / 43, in 512 units, not cut / shares 215 / 54.
// More units take shares, and from twice as many on only those of which one takes longer than two shares: 63 of 256 and one of 8192
// (1024 units), whole / shares 247 / 95.
// `most` and shares are at least kLeastStages stages (where one is cut or crosses units, its parts may be shorter).
enum PlanKind { kAlike, kRanges, kShares };
struct Plan {
  int kind;
  int n_ranges;     // of the call; kShares: workgroups
  int whole, left;  // kAlike: units done whole, first; units left over
  int pieces;       // kAlike
  int most;         // kRanges
  int quot, rest;   // kShares: stages of a share; the first `rest` shares have one more
  __device__ __forceinline__ int share_start(int w) const { return w * quot + (w < rest ? w : rest); }
  __device__ __forceinline__ int share_of(int x) const {
    const int big = rest * (quot + 1);
    return x < big ? (int)((unsigned)x / (unsigned)(quot + 1)) : rest + (int)((unsigned)(x - big) / (unsigned)quot);
  }
};
constexpr int kLeastStages = 3, kLongRange = 32;

__device__ __forceinline__ int wave_sum_i32(int v) {
  return __builtin_amdgcn_readlane(wave_scan_i32(v, 0, [](int x, int y) { return x + y; }), 63);
}

__device__ __forceinline__ int wave_max_i32(int v) {
  return __builtin_amdgcn_readlane(wave_scan_i32(v, 0, [](int x, int y) { return x > y ? x : y; }), 63);
}

__device__ __forceinline__ Plan plan_ranges(const GroupedParams &p, const Sequence &first) {
  const int lane = threadIdx.x & 63;
  int units = 0, total = 0;  // (the total is looked at where it is below 2^30: see propd_grouped_attention)
  const int s_first = uniform(first.count(p)), u_first = uniform(first.units(p));
  bool alike = true;
  for (int b0 = 0; b0 < p.B; b0 += kWave) {
    const Sequence q = b0 == 0 ? first : lane_sequence(p, b0 + lane);
    const int s = q.count(p), u = q.units(p);
    alike = alike && __ballot(b0 + lane < p.B && (s != s_first || u != u_first)) == 0;
    units += wave_sum_i32(u);
    total += wave_sum_i32(s * u);
  }
  Plan plan = {alike ? kAlike : kRanges, units, 0, units, 1, 1 << 30, 0, 0};
  if (!p.may_split) return plan;
  const int half = p.resident / 2;
  const int slots = total > half * kLongRange ? p.resident : half;
  if (alike) {
    plan.whole = units / p.resident * p.resident;
    plan.left = units - plan.whole;
    if (plan.left > 0) {
      const int room = plan.whole > 0 ? half : slots;
      int pieces = below(room, plan.left);
      pieces = pieces < below(s_first, kLeastStages) ? pieces : below(s_first, kLeastStages);
      plan.pieces = pieces < 1 ? 1 : pieces;
      plan.n_ranges = plan.whole + plan.left * plan.pieces;
    }
    return plan;
  }
  if (units <= p.resident) {
    for (int room = slots;; room = p.resident) {
      // from an equal share on, a sixteenth of it longer at a time
      const float equal = (float)total / (float)room;
      const int steps = equal > (float)kLongRange ? 4 : 16;
      for (int step = 0; step <= steps; ++step) {
        const int m = (int)ceilf(equal * (1.f + .0625f * (float)step));
        const int most = m > kLeastStages ? m : kLeastStages;
        int n = 0;
        for (int b0 = 0; b0 < p.B; b0 += kWave) {
          const Sequence q = b0 == 0 ? first : lane_sequence(p, b0 + lane);
          n += wave_sum_i32(q.T > 0 ? q.units(p) * pieces_of(q.count(p), most) : 0);
        }
        if (n <= room || n <= units) {
          plan.most = most;
          plan.n_ranges = n;
          return plan;
        }
      }
      if (room == p.resident) break;
    }
  } else if (units >= 2 * p.resident) {  // two rounds and more
    int longest = 0;
    for (int b0 = 0; b0 < p.B; b0 += kWave) {
      const Sequence q = b0 == 0 ? first : lane_sequence(p, b0 + lane);
      const int x = wave_max_i32(q.count(p));
      longest = x > longest ? x : longest;
    }
    if (longest <= 2 * (total / p.resident)) return plan;
  }
  int shares = total / kLeastStages;
  shares = shares < p.resident ? shares : p.resident;
  shares = shares < p.slots / 2 ? shares : p.slots / 2;
  if (shares < 1) return plan;
  plan.kind = kShares;
  plan.n_ranges = shares;
  plan.quot = total / shares;
  plan.rest = total - plan.quot * shares;
  return plan;
}

// A lane's columns of the result, and where they lie.
__device__ __forceinline__ size_t column_row(const GroupedParams &p, int b, int hk, int column, int T) {
  const int g = quotient(column, T), i = column - g * T;
  return ((size_t)b * p.H + hk * p.group + g) * p.T_max + i;
}

// One direct load of a wave: 64 lanes x 4 bytes, contiguous in LDS.
__device__ __forceinline__ void dma4(const void *src, uint32_t lds_at) {
  __builtin_amdgcn_global_load_lds((global_void *)src, (lds_void *)(uintptr_t)lds_at, 4, 0, 0);
}

// an address with some bits flipped, by an instruction that stays where it is used
template <int BITS>
__device__ __forceinline__ uint32_t flipped(uint32_t at) {
  if constexpr (BITS == 0) return at;
  uint32_t to;
  asm volatile("v_xor_b32 %0, %1, %2" : "=v"(to) : "n"(BITS), "v"(at));
  return to;
}

// Whether any of these is NaN or infinite (or their sum is).
template <int MB>
__device__ __forceinline__ bool not_finite(const f32x16 (&o)[MB]) {
  float sum = 0.f;
#pragma unroll
  for (int mb = 0; mb < MB; ++mb)
#pragma unroll
    for (int r = 0; r < 16; ++r) sum += o[mb][r];
  return !(fabsf(sum) < INFINITY);
}

// kCap: capped scores.  kPlace: positions take part (a window, a bias, or rows at positions of their own).
// A weight is multiplied as a sum of kParts bf16 values, each the rest of the one before rounded.  d = 64: three, all 24 bits of it.
// d = 128: two, off by 2^-17 at most (with three the kernels that keep positions spill).  In one piece a weight is off by 2^-8, as much as the
// result's own rounding: error against 64 bits 2.3e-3 of the result instead of 1.66e-3.  One / two / three parts, us: 16 x 40 heads
// on 8, 128 nodes, 4096 keys 217 / 275 / -, capped 4 x 32 heads 29.4 / 31.5 / -, evicted 32 x 32 heads of 64 74 / 87 / 100.
template <int D, bool kCap, bool kPlace>
__global__ __launch_bounds__(kGroupThreads, 2) void grouped_attn_bf16_kernel(GroupedParams p) {
  using G_ = Geo<D>;
  constexpr int kRowBytes = G_::kRowBytes, kHalfStage = G_::kHalfStage, kStageBytes = G_::kStageBytes;
  constexpr int kMb = G_::kMb, kLoads = G_::kLoads, kQf = D / 16;
  constexpr int NS = D == 128 ? 4 : 6, kAhead = NS - 2;  // two stages are in use by the math, the rest is in flight
  constexpr bool kRaw = !kCap && !kPlace;                // the softmax scale is applied inside the exponent
  constexpr int kParts = D == 64 ? 3 : 2;
  constexpr int kPerStage = 2 * kLoads + (kPlace ? 1 : 0);  // loads of a wave per stage
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const uint32_t ring = (uint32_t)(uintptr_t)(lds_void *)smem;
  u32x4 *const tree_anc = reinterpret_cast<u32x4 *>(smem + NS * kStageBytes);  // [128] ancestor sets
  const uint32_t place_ring = ring + NS * kStageBytes + 2048;                  // [NS][4 waves][64] positions
  // places: positions less that of the root, as numbers that are exact where they matter
  float *const stage_place = reinterpret_cast<float *>(smem + NS * kStageBytes + 2048 + NS * 1024);  // [4 waves][32], of the stage at work
  float *const tree_place = stage_place + 4 * 32;                                             // [128], of the tree's nodes
  __shared__ int s_any[2];

  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int l32 = lane & 31, g = lane >> 5;
  const bool in_order = p.position == nullptr;

  // (registers are short: the lengths of the first 64 sequences lie in LDS; every wave writes the same)
  __shared__ int s_lengths[3][kWave];
  Plan plan;
  {
    const Sequence lanes = lane_sequence(p, lane);
    s_lengths[0][lane] = lanes.L;
    s_lengths[1][lane] = lanes.T;
    s_lengths[2][lane] = lanes.dropped;
    plan = plan_ranges(p, lanes);
  }
  auto sequence_at = [&](int b) -> Sequence {  // of this lane's number, or of one for all lanes
    if (b < kWave) return {s_lengths[0][b], s_lengths[1][b], s_lengths[2][b]};
    return lane_sequence(p, b);
  };

  // ---- where a lane reads in a stage: K as the A operand (row l32, chunk 2 ks + g), V^T by transposing reads
  constexpr bool kFew = D == 128 && kPlace;  // registers are short: addresses are made of two by flipping bits
  uint32_t k_rd[kFew ? 1 : kQf], v_rd[kFew ? 1 : kMb][2];
#pragma unroll
  for (int ks = 0; ks < (kFew ? 1 : kQf); ++ks) k_rd[ks] = ring + l32 * kRowBytes + (((2 * ks + g) ^ G_::k_key(l32)) << 4);
#pragma unroll
  for (int mb = 0; mb < (kFew ? 1 : kMb); ++mb)
#pragma unroll
    for (int hi = 0; hi < 2; ++hi) {
      const int r = 4 * g + 8 * hi + ((lane & 15) >> 2);
      const int chunk = mb * 4 + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
      v_rd[mb][hi] = ring + kHalfStage + r * kRowBytes + ((chunk ^ G_::v_key(r)) << 4) + 8 * (lane & 1);
    }
  const int ld_row = G_::kLdRows * wave + lane / G_::kChunks;
  const uint32_t k_lane = ld_row * kRowBytes + (((lane % G_::kChunks) ^ G_::k_key(ld_row)) << 4);
  const uint32_t v_lane = ld_row * kRowBytes + (((lane % G_::kChunks) ^ G_::v_key(ld_row)) << 4);
  if (tid < 2) s_any[tid] = 0;
  int n_any = 0;

  // ---- ranges.  The blocks of a unit read the same rows: they run next to each other on one XCD (workgroups go to the 8
  //      XCDs in turn), so that the rows come from its L2 but for the first time.  What does not fill a span stays in order.
  const int span = 8 * p.blocks;
  int at = blockIdx.x, x = 0, x_end = 0;  // the next range; kShares: what is left of this workgroup's share
  if (plan.kind == kShares) {
    if (at >= plan.n_ranges) return;
    const int even = plan.n_ranges / 8 * 8;  // an XCD has neighbouring shares
    at = at < even ? at % 8 * (even / 8) + at / 8 : at;
    x = plan.share_start(at);
    x_end = plan.share_start(at + 1);
  }
  bool first_range = true;
  int found_at = 0, found_before = 0;  // where the last search for a sequence ended, a multiple of 64, and the items before that
  while (plan.kind == kShares ? x < x_end : at < plan.n_ranges) {
    int b = 0, block, hk, s0, n_st, slot, first_slot, stride, P, late = 0;  // late: see the merge
    // The sequence that holds item `which` of a list that has of(x) items per sequence, and the items before that sequence.  From where the
    // last search ended: all of them together pass a batch once, also where it has many more sequences than a workgroup has units.
    auto locate = [&](int which, auto &&of) __attribute__((always_inline)) {
      int start = 0;
      if (which < found_before) found_at = found_before = 0;
      for (int b0 = found_at, before = found_before; b0 < p.B; b0 += kWave) {
        const Sequence q = sequence_at(b0 + lane);
        const int mine = of(q), incl = wave_scan_i32(mine, 0, [](int x, int y) { return x + y; });
        const uint64_t le = __ballot(b0 + lane < p.B && before + incl - mine <= which);
        if (le == 0) break;
        found_at = b0;
        found_before = before;
        const int src = __popcll(le) - 1;
        b = b0 + src;
        start = __builtin_amdgcn_readlane(before + incl - mine, src);
        before += __builtin_amdgcn_readlane(incl, 63);
      }
      return start;
    };
    Sequence n;
    int n_stages, n_blocks;
    auto take_lengths = [&]() __attribute__((always_inline)) {
      const Sequence m = sequence_at(b);
      n = {uniform(m.L), uniform(m.T), uniform(m.dropped)};
      n_stages = n.count(p);
      n_blocks = n.blocks(p);
    };
    if (plan.kind == kShares) {
      const int in_sequence = x - locate(x, [&](const Sequence &q) { return q.count(p) * q.units(p); });
      take_lengths();
      const int u = quotient(in_sequence, n_stages);
      hk = quotient(u, n_blocks);
      block = u - hk * n_blocks;
      s0 = in_sequence - u * n_stages;
      n_st = n_stages - s0 < x_end - x ? n_stages - s0 : x_end - x;
      P = s0 == 0 ? plan.share_of(x + n_stages - 1) - at + 1 : 2;  // 2: more than one
      slot = 2 * at + (s0 == 0 ? 1 : 0);
      first_slot = slot;
      stride = 2;
      late = 1;
      x += n_st;
    } else {
      const int part0 = at < plan.whole ? 0 : plan.whole, part_n = at < plan.whole ? plan.whole : plan.n_ranges - plan.whole;
      const int local = at - part0, in_span = local - quotient(local, span) * span;
      const int range = local < quotient(part_n, span) * span ? local - in_span + in_span % 8 * p.blocks + in_span / 8 : local;  // within its part
      int piece = 0;
      if (plan.kind == kAlike) {
        const int per_sequence = uniform(sequence_at(0).units(p));
        int u = part0 + range;
        P = 1;
        first_slot = 0;
        stride = 1;
        if (at >= plan.whole) {
          P = plan.pieces;
          piece = quotient(range, plan.left);
          first_slot = range - piece * plan.left;
          stride = plan.left;
          u = plan.whole + first_slot;
        }
        b = quotient(u, per_sequence);
        take_lengths();
        const int in_sequence = u - b * per_sequence;
        hk = quotient(in_sequence, n_blocks);
        block = in_sequence - hk * n_blocks;
      } else {
        const int most = plan.most;
        const int rest = range - locate(range, [&](const Sequence &q) { return q.T > 0 ? q.units(p) * pieces_of(q.count(p), most) : 0; });
        take_lengths();
        P = pieces_of(n_stages, most);
        const int in_order_of_blocks = quotient(rest, n_blocks);
        block = rest - in_order_of_blocks * n_blocks;
        hk = quotient(in_order_of_blocks, P);
        piece = in_order_of_blocks - hk * P;
        stride = n_blocks;
        first_slot = range - piece * n_blocks;
      }
      slot = first_slot + piece * stride;
      const int quot = quotient(n_stages, P), extra = n_stages - quot * P;
      s0 = piece * quot + (piece < extra ? piece : extra);
      n_st = quot + (piece < extra ? 1 : 0);
      at += gridDim.x;
    }
    const Stages st = n.stages(p);
    const int L = n.L, T = n.T, columns = p.group * T, root = root_position(L, n.dropped);
    const size_t unit = (size_t)b * p.H_kv + hk;

    // ---- this lane's column
    const int column = block * 128 + wave * 32 + l32;
    const bool active = block * 128 + wave * 32 < columns, there = column < columns;
    const int col = there ? column : 0;  // lanes past the last column take the first: valid memory, never stored
    const int head = quotient(col, T), node = col - head * T;
    const size_t row_out = ((size_t)b * p.H + hk * p.group + head) * p.T_max + node;
    u32x4 qf[kQf];
    {
      const uint16_t *src = p.q + row_out * D + g * 8;
#pragma unroll
      for (int ks = 0; ks < kQf; ++ks) qf[ks] = *reinterpret_cast<const u32x4 *>(src + ks * 16);
    }
    u32x4 ancv;
    if constexpr (kPlace) ancv = *reinterpret_cast<const u32x4 *>(p.anc + ((size_t)b * p.T_max + node) * 2);
    const u32x4 anc_row = *reinterpret_cast<const u32x4 *>(p.anc + ((size_t)b * p.T_max + (tid < T ? tid : 0)) * 2);  // of node tid
    float slope = 0.f;
    if constexpr (kPlace) {
      if (p.slopes) slope = p.slopes[hk * p.group + head] * kLog2e;
    }
    if (!first_range) __builtin_amdgcn_s_barrier();  // the range before is done with the ring and the table
    first_range = false;

    // ---- loader.  One direct load moves 64 lanes x 16 bytes into 1 KB of LDS, contiguous in lane order, so that the swizzle is
    //      applied by the lanes' addresses.  It walks the cached rows and then the tree's, a stage at a time; rows past the last
    //      valid one re-read that row: data that the mask discards (K) or that meets a zero weight (V).
    int ld_left;  // rows left in the segment, from the next stage to issue
    const unsigned char *ld_k, *ld_v;
    const int32_t *ld_place;
    bool ld_tree;
    auto segment = [&](bool tree, int row0) {
      const size_t base = unit * (size_t)(tree ? p.T_max : p.L_max) + row0;
      ld_tree = tree;
      ld_left = (tree ? T : L) - row0;
      ld_k = reinterpret_cast<const unsigned char *>(tree ? p.k_tree : p.k_cache) + base * kRowBytes;
      ld_v = reinterpret_cast<const unsigned char *>(tree ? p.v_tree : p.v_cache) + base * kRowBytes;
      if constexpr (kPlace) ld_place = tree || in_order ? nullptr : p.position + base;
    };
    auto issue = [&](int slot) __attribute__((always_inline)) {
      unsigned char *dst = smem + slot * kStageBytes + wave * 1024;
      if (ld_left >= kStageRows) {  // uniform
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          __builtin_amdgcn_global_load_lds((global_void *)(ld_k + i * 4096 + k_lane), (lds_void *)(dst + i * 4096), 16, 0, 2 /* nt */);
          __builtin_amdgcn_global_load_lds((global_void *)(ld_v + i * 4096 + v_lane), (lds_void *)(dst + kHalfStage + i * 4096), 16, 0, 2);
        }
      } else {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          int row = 4 * G_::kLdRows * i + ld_row;
          row = (row < ld_left ? row : ld_left - 1) - ld_row;
          __builtin_amdgcn_global_load_lds((global_void *)(ld_k + (row * kRowBytes + (int)k_lane)), (lds_void *)(dst + i * 4096), 16, 0, 2);
          __builtin_amdgcn_global_load_lds((global_void *)(ld_v + (row * kRowBytes + (int)v_lane)), (lds_void *)(dst + kHalfStage + i * 4096), 16, 0, 2);
        }
      }
      if constexpr (kPlace) {  // tree stages and rows in order need none; the count of loads stays the same
        const int row = l32 < ld_left ? l32 : ld_left - 1;
        dma4(ld_place ? ld_place + row : p.seq_lens + b, place_ring + slot * 1024 + wave * 256);
      }
      if (ld_left > kStageRows) {
        ld_left -= kStageRows;
        ld_k += kHalfStage;
        ld_v += kHalfStage;
        if constexpr (kPlace) ld_place += ld_place ? kStageRows : 0;
      } else if (!ld_tree) {
        segment(true, 0);
      }
    };
    auto slot_of = [](int x) { return (int)((unsigned)x % (unsigned)NS); };
    auto start = [&]() {
      if (s0 < st.cached) segment(false, (s0 + st.first) * kStageRows);
      else segment(true, (s0 - st.cached) * kStageRows);
#pragma unroll
      for (int x = 0; x < kAhead; ++x)
        if (x < n_st) issue(x);
    };
    start();
    // A column sees places from `lowest` on; `all_see`: from here on every column of the wave does.  (The bias is made of the
    // distance itself: slope * place alone would cost the last bits of a deep node's lse.)
    float lowest = 0.f, all_see = 0.f, depth = 0.f;
    if constexpr (kPlace) {
      const int deep = __popc(ancv.x) + __popc(ancv.y) + __popc(ancv.z) + __popc(ancv.w) - 1;
      lowest = (float)(sight_of(root + deep, p.window).lowest - root);
      depth = (float)deep;
      all_see = lowest;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) all_see = fmaxf(all_see, __shfl_xor(all_see, o, kWave));
      all_see = __uint_as_float(uniform(__float_as_uint(all_see)));
      if (tid < 128) tree_place[tid] = (float)(__popc(anc_row.x) + __popc(anc_row.y) + __popc(anc_row.z) + __popc(anc_row.w) - 1);
    }
    if (tid < 128) tree_anc[tid] = anc_row;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // both seen by all behind the first stage's barrier
    // Stage x is there for all waves, and its place kAhead stages on is free: everyone is done with stage x - 2.  A wave's
    // loads complete in order, so that at most the younger stages' loads outstanding means that stage x has landed.
    auto acquire = [&](int x) {
      int younger = n_st - 1 - x;
      younger = younger < kAhead - 1 ? younger : kAhead - 1;
      if constexpr (kAhead > 3) {
        if (younger == 3) wait_vmem<3 * kPerStage>();
      }
      if constexpr (kAhead > 2) {
        if (younger == 2) wait_vmem<2 * kPerStage>();
      }
      if (younger == 1) wait_vmem<kPerStage>();
      if (younger <= 0) wait_vmem<0>();
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      if (x + kAhead < n_st) issue(slot_of(x + kAhead));
    };

    float m_run, l_run;
    f32x16 o_acc[kMb];
    u32x2 vt[2][2 * kMb];
    // (a slot known at compile time goes into the offsets of the LDS reads)
    auto scores = [&](auto slot) __attribute__((always_inline)) -> f32x16 {
      const uint32_t so = (uint32_t)(int)slot * kStageBytes;
      f32x16 acc;
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[r] = 0.f;
      static_for_i<kQf>([&](auto step) __attribute__((always_inline)) {
        constexpr int ks = decltype(step)::value;
        const uint32_t at = kFew ? flipped<32 * ks>(k_rd[0]) : k_rd[kFew ? 0 : ks];
        const bf16x8 a = *reinterpret_cast<const __attribute__((address_space(3))) bf16x8 *>((uintptr_t)(at + so));
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, __builtin_bit_cast(bf16x8, qf[ks]), acc, 0, 0, 0);
      });
      return acc;
    };
    auto read_v = [&](auto slot, auto half) __attribute__((always_inline)) {
      constexpr int kHalf = decltype(half)::value;
      constexpr bool kKnown = !std::is_same_v<decltype(slot), int>;
      constexpr int kAt = 16 * kRowBytes * kHalf + (kKnown ? (int)decltype(std::conditional_t<kKnown, decltype(slot), std::integral_constant<int, 0>>{})::value : 0) * kStageBytes;
      const uint32_t so = kKnown ? 0u : (uint32_t)(int)slot * kStageBytes;
      static_for_i<kMb>([&](auto block) __attribute__((always_inline)) {
        constexpr int mb = decltype(block)::value, kFlip = kFew ? 64 * mb : 0;
        vt[kHalf][2 * mb] = lds_read_tr16<kAt>(flipped<kFlip>(v_rd[kFew ? 0 : mb][0]) + so);
        vt[kHalf][2 * mb + 1] = lds_read_tr16<kAt>(flipped<kFlip>(v_rd[kFew ? 0 : mb][1]) + so);
      });
    };
    // Values of V that are not finite: out of the V registers of 16 rows, and what they add to O to it.
    auto take_out = [&](const uint32_t (&pw)[kParts][4], auto half) __attribute__((always_inline)) {
      constexpr int kHalf = decltype(half)::value;
#pragma unroll
      for (int mb = 0; mb < kMb; ++mb) {
        uint32_t v4[4] = {vt[kHalf][2 * mb].x, vt[kHalf][2 * mb].y, vt[kHalf][2 * mb + 1].x, vt[kHalf][2 * mb + 1].y};
        u32x4 code, seen;  // seen: 1 for a weight
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const uint32_t w2 = pw[0][x];  // (zero only for weights below the least bf16 value)
          seen[x] = (w2 & 0xffffu ? 0x3f80u : 0u) | (w2 >> 16 ? 0x3f800000u : 0u);
          code[x] = take_not_finite(v4[x]);
        }
        vt[kHalf][2 * mb] = u32x2{v4[0], v4[1]};
        vt[kHalf][2 * mb + 1] = u32x2{v4[2], v4[3]};
        f32x16 codes;
#pragma unroll
        for (int r = 0; r < 16; ++r) codes[r] = 0.f;
        codes = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, code), __builtin_bit_cast(bf16x8, seen), codes, 0, 0, 0);
        mfma_settle();  // O too: its last products came before
#pragma unroll
        for (int r = 0; r < 16; ++r) o_acc[mb][r] += not_finite_sum(codes[r]);
      }
    };
    // a new running maximum is adopted only when it exceeds the reference by 2^8 in the exponent: weights then exceed 1, by a
    // factor that fp32 sums and bf16 weights hold, and O is hardly ever scaled.  Products with values of V beyond 2^120 may not hold it: with care
    // weights are at most 1.
    const float tau = kRaw ? fminf(8.f / p.scale_log2e, 1e38f) : 8.f;

    // The weights of stage i from its products, and what they add to O.
    // kInside: a full stage of cached rows.  next: called once the scores are no longer needed as they were.
    auto take_stage = [&](int i, auto slot, const f32x16 &raw, auto inside, auto with_care, auto &&next) __attribute__((always_inline)) {
      constexpr bool kCareful = decltype(with_care)::value, kInside = decltype(inside)::value;
      float sc[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[r] = raw[r];
      const int s = s0 + i;
      const bool tree = !kInside && s >= st.cached;
      const int j0 = (tree ? s - st.cached : s + st.first) * kStageRows;
      int n_valid = (tree ? T : L) - j0;
      n_valid = n_valid > kStageRows ? kStageRows : n_valid;
      // ---- scores in the exponent's (log2) domain.  Register r holds row j0 + 8 * (r / 4) + 4 * g + r % 4.
      if constexpr (kCap) {
        // cap tanh(x / cap) as in capped(), whose fraction alone does where no score of the wave is beyond 3/4 of the cap.
        // (cap - 2 cap / (exp(2 x / cap) + 1) is 27 us instead of 29.5 for 4 x 8 heads of 2048 rows, and off by cap * 2^-23.)
        float most = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) most = fmaxf(most, fabsf(sc[r]));
        if (__builtin_amdgcn_ballot_w64(!(most * p.cap_in < .75f)) == 0) {
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float y = sc[r] * p.cap_in, y2 = y * y;
            sc[r] = sc[r] * p.scale_log2e * fmaf(y2, y2 + 105.f, 945.f) * __builtin_amdgcn_rcpf(fmaf(y2, fmaf(15.f, y2, 420.f), 945.f));
          }
        } else {
#pragma unroll
          for (int r = 0; r < 16; ++r) sc[r] = capped(sc[r], p.cap_log2e, p.cap_in);
        }
      } else if constexpr (kPlace) {
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[r] *= p.scale_log2e;
      }
      if constexpr (kPlace) {
        if (in_order && !tree) {
          const float first = (float)(j0 - L + 4 * g);  // row j of the cache has place j - L
          if (p.slopes) {  // uniform, as the next
#pragma unroll
            for (int r = 0; r < 16; ++r) sc[r] = fmaf(slope, first - depth + (float)(8 * (r >> 2) + (r & 3)), sc[r]);
          }
          if ((float)(j0 - L) < all_see) {
#pragma unroll
            for (int r = 0; r < 16; ++r) sc[r] = first + (float)(8 * (r >> 2) + (r & 3)) >= lowest ? sc[r] : -INFINITY;
          }
        } else {
          const float *from = tree ? tree_place + j0 : stage_place + 32 * wave;
          bool all = true;
          if (tree) {
            all = 0.f >= all_see;
          } else {
            // the 32 positions become places; a row without one, or that is not before the root, lies below everything
            const int at = *reinterpret_cast<const __attribute__((address_space(3))) int *>((uintptr_t)(place_ring + (uint32_t)(int)slot * 1024 + wave * 256 + 4 * l32));
            const float place = (unsigned)at < (unsigned)root ? (float)(at - root) : -0x1p31f;
            stage_place[32 * wave + l32] = place;
            all = __ballot(place < all_see) == 0;
          }
          float place[16];
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            const f32x4 at4 = *reinterpret_cast<const f32x4 *>(from + 8 * q4 + 4 * g);
#pragma unroll
            for (int j = 0; j < 4; ++j) place[4 * q4 + j] = at4[j];
          }
          if (p.slopes) {
#pragma unroll
            for (int r = 0; r < 16; ++r) sc[r] = fmaf(slope, place[r] - depth, sc[r]);
          }
          if (!all) {
#pragma unroll
            for (int r = 0; r < 16; ++r) sc[r] = place[r] >= lowest ? sc[r] : -INFINITY;
          }
        }
      }
      if (!kInside && (tree || n_valid < kStageRows)) {  // uniform
        uint32_t vis = n_valid >= 32 ? ~0u : ((1u << n_valid) - 1u);
        // tree stages start at 0, 32, 64, 96: a word of the node's set each
        if (tree) vis &= reinterpret_cast<const uint32_t *>(tree_anc + node)[j0 >> 5];
        vis >>= 4 * g;
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[r] = ((vis >> (8 * (r >> 2) + (r & 3))) & 1u) ? sc[r] : -INFINITY;
      }
      float m_blk = -INFINITY;
#pragma unroll
      for (int r = 0; r < 16; ++r) m_blk = fmaxf(m_blk, sc[r]);
      {  // the other half of the stage's rows is in the lane 32 away
        uint32_t lo = __float_as_uint(m_blk), hi = lo;
        swap_halves(lo, hi);
        m_blk = fmaxf(__uint_as_float(lo), __uint_as_float(hi));
      }
      if (__builtin_amdgcn_ballot_w64(m_blk > (kCareful ? m_run : m_run + tau)) != 0) {
        const float m_new = fmaxf(m_run, m_blk), m_safe = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = fast_exp2((m_run - m_safe) * (kRaw ? p.scale_log2e : 1.f));
        l_run *= alpha;
        mfma_settle();
#pragma unroll
        for (int mb = 0; mb < kMb; ++mb)
#pragma unroll
          for (int r = 0; r < 16; ++r) o_acc[mb][r] *= alpha;
        m_run = m_new;
      }
      const float neg_m = -(m_run == -INFINITY ? 0.f : m_run) * (kRaw ? p.scale_log2e : 1.f);
      next();  // products of the next stage, in one block with what follows
      read_v(slot, std::integral_constant<int, 0>{});
      // weights of the rows of one half: pw[part][x] has those of registers 8 * half + 2 x and 2 x + 1
      uint32_t pw[2][kParts][4];
      auto weights = [&](auto half) __attribute__((always_inline)) {
        constexpr int kHalf = decltype(half)::value;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int r = 8 * kHalf + 2 * x;
          float p0 = fast_exp2(kRaw ? fmaf(sc[r], p.scale_log2e, neg_m) : sc[r] + neg_m);
          float p1 = fast_exp2(kRaw ? fmaf(sc[r + 1], p.scale_log2e, neg_m) : sc[r + 1] + neg_m);
          l_run += p0 + p1;  // of the weights as they are: lse is an fp32 result
#pragma unroll
          for (int part = 0; part < kParts; ++part) {  // rounded to bf16, and what that leaves
            const uint32_t w2 = cvt_pk_bf16(p0, p1);
            pw[kHalf][part][x] = w2;
            p0 -= __uint_as_float(w2 << 16);
            p1 -= __uint_as_float(w2 & 0xffff0000u);
          }
        }
      };
      weights(std::integral_constant<int, 0>{});
      weights(std::integral_constant<int, 1>{});
      read_v(slot, std::integral_constant<int, 1>{});
      static_for_i<2>([&](auto half) __attribute__((always_inline)) {
        constexpr int kHalf = decltype(half)::value;
        wait_lds<kHalf == 0 ? 2 * kMb : 0>(vt[kHalf]);
        if constexpr (kCareful) take_out(pw[kHalf], half);
#pragma unroll
        for (int part = kParts - 1; part >= 0; --part) {  // the small parts first
          const u32x4 pv = {pw[kHalf][part][0], pw[kHalf][part][1], pw[kHalf][part][2], pw[kHalf][part][3]};
#pragma unroll
          for (int mb = 0; mb < kMb; ++mb) {
            const u32x4 aw = {vt[kHalf][2 * mb].x, vt[kHalf][2 * mb].y, vt[kHalf][2 * mb + 1].x, vt[kHalf][2 * mb + 1].y};
            o_acc[mb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, aw), __builtin_bit_cast(bf16x8, pv), o_acc[mb], 0, 0, 0);
          }
        }
      });
    };
    auto clear = [&]() {
      m_run = -INFINITY;
      l_run = 0.f;
#pragma unroll
      for (int mb = 0; mb < kMb; ++mb)
#pragma unroll
        for (int r = 0; r < 16; ++r) o_acc[mb][r] = 0.f;
    };

    const int n_inside = L / kStageRows - st.first - s0;  // full stages of cached rows, from the first on
    using yes = std::true_type;
    using no = std::false_type;
    clear();
    acquire(0);
    if (active) {
      f32x16 raw = scores(std::integral_constant<int, 0>{});
      int i = 0;
      // whole turns of the ring while there is more to come than is in flight
      for (; i + NS <= n_inside && i + NS + kAhead < n_st; i += NS) {
        static_for_i<NS>([&](auto k) __attribute__((always_inline)) {
          constexpr int kSlot = decltype(k)::value, kNext = (kSlot + 1) % NS, kFree = (kSlot + 1 + kAhead) % NS;
          wait_vmem<(kAhead - 1) * kPerStage>();
          __builtin_amdgcn_s_barrier();
          asm volatile("" ::: "memory");
          issue(kFree);
          mfma_settle();  // raw was written by products of the stage before
          f32x16 raw_next;
          take_stage(i + kSlot, k, raw, yes{}, no{}, [&]() __attribute__((always_inline)) { raw_next = scores(std::integral_constant<int, kNext>{}); });
          raw = raw_next;
        });
      }
      for (; i < n_st; ++i) {
        const bool more = i + 1 < n_st;
        if (more) acquire(i + 1);
        mfma_settle();
        f32x16 raw_next = raw;
        take_stage(i, slot_of(i), raw, no{}, no{}, [&]() __attribute__((always_inline)) {
          if (more) raw_next = scores(slot_of(i + 1));
        });
        raw = raw_next;
      }
      mfma_settle();
    } else {
      for (int i = 1; i < n_st; ++i) acquire(i);  // columns beyond the last: loads and barriers only
    }
    // Zero weights times values of V that are not finite, or products that leave the range of fp32: such a range is done once more,
    // with care.
    ++n_any;
    int *word = s_any + (n_any & 1);
    if (active && __builtin_amdgcn_ballot_w64(not_finite(o_acc)) != 0) *word = n_any;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (uniform(*word) == n_any) {
      start();
      clear();
      for (int i = 0; i < n_st; ++i) {
        acquire(i);
        if (!active) continue;
        const f32x16 raw = scores(slot_of(i));
        mfma_settle();
        take_stage(i, slot_of(i), raw, no{}, yes{}, [] {});
        mfma_settle();
      }
    }

    // ---- results
    l_run += __shfl_xor(l_run, 32, kWave);
    if constexpr (kRaw) m_run *= p.scale_log2e;
    if (tid == 0 && s0 == 0)
      *reinterpret_cast<u32x4 *>(p.records + 4 * (unit * p.blocks + block)) =
          u32x4{(uint32_t)first_slot, (uint32_t)stride, (uint32_t)P, (uint32_t)late};
    if (there && P == 1) {
      const float inv = l_run > 0.f ? 1.f / l_run : l_run == 0.f ? 0.f : l_run;  // NaN stays
#pragma unroll
      for (int mb = 0; mb < kMb; ++mb) store_out_block<false>(p.out + row_out * D, o_acc[mb], inv, g, mb);
      if (p.lse && g == 0) p.lse[row_out] = (m_run + __builtin_amdgcn_logf(l_run)) * kLn2;
    } else if (there) {
#pragma unroll
      for (int mb = 0; mb < kMb; ++mb)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4)
          *reinterpret_cast<f32x4 *>(p.part_o + part_o_index(slot, wave, 4 * mb + q4, lane)) =
              f32x4{o_acc[mb][4 * q4], o_acc[mb][4 * q4 + 1], o_acc[mb][4 * q4 + 2], o_acc[mb][4 * q4 + 3]};
      p.part_ml[part_ml_index(slot, wave, 0, lane)] = m_run;
      p.part_ml[part_ml_index(slot, wave, 1, lane)] = l_run;
    }
  }
}

// A result to be merged with factor f: left out where the factor is zero (an infinity would be NaN).
__device__ __forceinline__ float counted(float o, float f) { return f == 0.f ? 0.f : o; }

// out = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s over the pieces s of a unit, always in the same order.  A workgroup has 32
// columns of a unit and a 32-wide block of d.  W waves take the pieces in turn, up to 8 of them requested together, and meet
// through LDS: what costs is the chain of their loads.
template <int D, int W>
__global__ __launch_bounds__(W *kWave) void grouped_attn_merge_kernel(GroupedParams p) {
  constexpr int kMb = Geo<D>::kMb;
  __shared__ float s_part[W > 1 ? W - 1 : 1][18][kWave];
  const int mb = blockIdx.x % kMb, group = blockIdx.x / kMb % 4;
  const unsigned item = blockIdx.x / (4 * kMb);
  const unsigned unit = item / (unsigned)p.blocks, b = unit / (unsigned)p.H_kv;
  const int block = (int)(item - unit * (unsigned)p.blocks), hk = (int)(unit - b * (unsigned)p.H_kv);
  int T = p.n_nodes[b];
  T = T < 1 ? 1 : (T > p.T_max ? p.T_max : T);
  const int columns = p.group * T;
  if (block * 128 + group * 32 >= columns) return;
  const u32x4 record = *reinterpret_cast<const u32x4 *>(p.records + 4 * (size_t)item);
  const int first = (int)record.x, stride = (int)record.y, P = (int)record.z, late = (int)record.w;
  if (P <= 1) return;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), g = lane >> 5, column = block * 128 + group * 32 + (lane & 31);
  const bool there = column < columns;
  const int ln = there ? lane : 0;  // lanes past the last column read lane 0's data and store nothing
  f32x16 acc;
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[r] = 0.f;
  float M = -INFINITY, total = 0.f;
  auto join = [&](const f32x16 &o, float m, float l) {
    const float M_new = fmaxf(M, m), M_safe = M_new == -INFINITY ? 0.f : M_new;
    const float a_old = fast_exp2(M - M_safe), a_new = fast_exp2(m - M_safe);
    total = total * a_old + l * a_new;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = counted(acc[r], a_old) * a_old + counted(o[r], a_new) * a_new;
    M = M_new;
  };
  auto take = [&](int s0, auto count) __attribute__((always_inline)) {  // pieces s0, s0 + W, ... requested together
    constexpr int N = decltype(count)::value;
    f32x4 o[N][4];
    float m[N], l[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int s = s0 + k * W < P ? s0 + k * W : P - 1;  // past the last: that once more, not used
      const size_t slot = first + (size_t)s * stride - (s > 0 ? late : 0);
      m[k] = p.part_ml[part_ml_index(slot, group, 0, ln)];
      l[k] = p.part_ml[part_ml_index(slot, group, 1, ln)];
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) o[k][q4] = *reinterpret_cast<const f32x4 *>(p.part_o + part_o_index(slot, group, 4 * mb + q4, ln));
    }
    __builtin_amdgcn_sched_barrier(0);  // all of them are requested first
#pragma unroll
    for (int k = 0; k < N; ++k) {
      if (s0 + k * W < P) {  // uniform
        f32x16 x;
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = o[k][r / 4][r % 4];
        join(x, m[k], l[k]);
      }
    }
  };
  for (int s0 = wave; s0 < P;) {
    const int mine = (P - s0 + W - 1) / W;
    if (mine > 4) take(s0, std::integral_constant<int, 8>{}), s0 += 8 * W;
    else if (mine > 2) take(s0, std::integral_constant<int, 4>{}), s0 += 4 * W;
    else take(s0, std::integral_constant<int, 2>{}), s0 += 2 * W;
  }
  if constexpr (W > 1) {
    if (wave > 0) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s_part[wave - 1][r][lane] = acc[r];
      s_part[wave - 1][16][lane] = M;
      s_part[wave - 1][17][lane] = total;
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 0; w < W - 1; ++w) {
      f32x16 x;
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = s_part[w][r][lane];
      join(x, s_part[w][16][lane], s_part[w][17][lane]);
    }
  }
  if (!there) return;
  const size_t row = column_row(p, (int)b, hk, column, T);
  const float inv = total > 0.f ? 1.f / total : total == 0.f ? 0.f : total;
  store_out_block<false>(p.out + row * D, acc, inv, g, mb);
  if (p.lse && mb == 0 && g == 0) p.lse[row] = (M + __builtin_amdgcn_logf(total)) * kLn2;
}

// ------------------------------------------------------------------------------------
// host side
// ------------------------------------------------------------------------------------
// Slots for partial results, a bound that needs no device: no more than stages, than ranges that run at once, or than two per share.
// (Up to a hundred units a `most` of a quarter more than an equal share is always found, so that there are no shares.)
static long long grouped_slots(int B, int H, int T_max, int L_max) {
  const long long stages = (L_max + kStageRows - 1ll) / kStageRows + (T_max + kStageRows - 1) / kStageRows;
  const long long most = (long long)B * H * stages, plan = (long long)B * H <= 100 ? kMostResident : kGroupSlots;
  return most < plan ? most : plan;
}

size_t grouped_attention_workspace_bytes(int B, int H, int L_max, int T_max) {
  const size_t slots = (size_t)grouped_slots(B, H, T_max, L_max);
  return align_up(slots * kPartOFloats * 4, 256) + align_up(slots * kPartMlFloats * 4, 256) + align_up((size_t)B * H * 16, 256);
}

template <int D, bool kCap, bool kPlace>
static bool launch_grouped(const GroupedParams &p, unsigned grid, hipStream_t st) {
  constexpr int NS = D == 128 ? 4 : 6;
  constexpr int lds_bytes = NS * Geo<D>::kStageBytes + 2048 + (kPlace ? NS * 1024 + 1024 : 0);
  static std::atomic<uint64_t> set{0};
  if (!allow_lds(reinterpret_cast<const void *>(&grouped_attn_bf16_kernel<D, kCap, kPlace>), lds_bytes, set)) return false;
  hipLaunchKernelGGL((grouped_attn_bf16_kernel<D, kCap, kPlace>), dim3(grid), dim3(kGroupThreads), lds_bytes, st, p);
  if (!launch_ok()) return false;
  if (!p.may_split) return true;
  const unsigned units = (unsigned)p.B * (unsigned)p.H_kv * (unsigned)p.blocks;
  const dim3 merge(units * 4u * Geo<D>::kMb);
  // Few units have more pieces than a wave requests at once.  Four waves and one, us: 8 units of 11 pieces 3.9 / 4.6, 56 of 4
  // 7.0 / 4.8, 128 of 2 among 640 24 / 9.
  if (units <= 16) hipLaunchKernelGGL((grouped_attn_merge_kernel<D, 4>), merge, dim3(4 * kWave), 0, st, p);
  else hipLaunchKernelGGL((grouped_attn_merge_kernel<D, 1>), merge, dim3(kWave), 0, st, p);
  return launch_ok();
}

template <int D>
static bool launch_grouped(const GroupedParams &p, bool cap, bool place, unsigned grid, hipStream_t st) {
  return cap ? (place ? launch_grouped<D, true, true>(p, grid, st) : launch_grouped<D, true, false>(p, grid, st))
             : (place ? launch_grouped<D, false, true>(p, grid, st) : launch_grouped<D, false, false>(p, grid, st));
}

#include "grouped_attention_f32.h"

}  // namespace propd

extern "C" propd_status propd_grouped_attention(const propd_tree *tree, propd_dtype dt, int32_t H, int32_t H_kv, int32_t d,
                                                const propd_score_rule *rule, const void *q, const void *k_cache,
                                                const void *v_cache, const void *k_tree, const void *v_tree,
                                                const int32_t *seq_lens, const int32_t *position, const int32_t *dropped,
                                                int32_t L_max, void *out, float *lse, void *workspace,
                                                size_t workspace_bytes, void *hip_stream) {
  using namespace propd;
  if (!tree || tree->B < 1 || tree->T_max < 1 || tree->T_max > PROPD_MAX_TREE || H < 1 || H_kv < 1 || H % H_kv != 0 || L_max < 0 ||
      !score_rule_ok(rule) || !tree->n_nodes || !tree->anc || !q || !k_tree || !v_tree || !seq_lens || !out ||
      (L_max > 0 && (!k_cache || !v_cache)))
    return PROPD_ERR_INVALID_ARG;
  if (dt != PROPD_BF16 && dt != PROPD_F32) return PROPD_ERR_INVALID_ARG;
  if (d != 64 && d != 128) return PROPD_ERR_UNSUPPORTED;
  for (const void *ptr : {q, k_cache, v_cache, k_tree, v_tree, (const void *)out, (const void *)tree->anc, (const void *)workspace})
    if (reinterpret_cast<uintptr_t>(ptr) % 16 != 0) return PROPD_ERR_INVALID_ARG;
  const long long nodes = (long long)tree->B * H * tree->T_max;
  if (L_max > (1 << 30) || nodes > (1ll << 30) || (long long)tree->B * H > (1ll << 24)) return PROPD_ERR_UNSUPPORTED;
  const size_t needed = grouped_attention_workspace_bytes(tree->B, H, L_max, tree->T_max);
  if (!workspace || workspace_bytes < needed) return PROPD_ERR_WORKSPACE;
  hipStream_t st = as_stream(hip_stream);
  GroupedParams p;
  p.q = reinterpret_cast<const uint16_t *>(q);
  p.k_cache = reinterpret_cast<const uint16_t *>(k_cache);
  p.v_cache = reinterpret_cast<const uint16_t *>(v_cache);
  p.k_tree = reinterpret_cast<const uint16_t *>(k_tree);
  p.v_tree = reinterpret_cast<const uint16_t *>(v_tree);
  p.out = reinterpret_cast<uint16_t *>(out);
  p.lse = lse;
  p.seq_lens = seq_lens;
  p.n_nodes = tree->n_nodes;
  p.position = L_max > 0 ? position : nullptr;
  p.dropped = dropped;
  p.anc = tree->anc;
  p.slopes = rule->slopes;
  p.B = tree->B;
  p.H = H;
  p.H_kv = H_kv;
  p.group = H / H_kv;
  p.T_max = tree->T_max;
  p.L_max = L_max;
  p.blocks = (p.group * p.T_max + 127) / 128;
  p.window = window_of(rule);
  p.scale_log2e = rule->scale * kLog2e;
  p.cap_in = rule->cap > 0.f ? rule->scale / rule->cap : 0.f;
  p.cap_log2e = rule->cap * kLog2e;
  const bool cap = rule->cap > 0.f, place = p.position || rule->window > 0 || rule->slopes;
  if (dt == PROPD_F32) return launch_grouped_f32(p, rule->scale, rule->cap, d, place, workspace, needed, st) ? PROPD_OK : PROPD_ERR_DEVICE;
  const size_t slots = (size_t)grouped_slots(tree->B, H, tree->T_max, L_max);
  char *ws = reinterpret_cast<char *>(workspace);
  p.part_o = reinterpret_cast<float *>(ws);
  ws += align_up(slots * kPartOFloats * 4, 256);
  p.part_ml = reinterpret_cast<float *>(ws);
  ws += align_up(slots * kPartMlFloats * 4, 256);
  p.records = reinterpret_cast<int32_t *>(ws);
  p.slots = (int)slots;
  p.resident = 2 * compute_units() < kMostResident ? 2 * compute_units() : kMostResident;
  const long long units = (long long)p.B * H_kv * p.blocks;
  const long long stages = (L_max + kStageRows - 1ll) / kStageRows + (p.T_max + kStageRows - 1) / kStageRows;
  p.may_split = (long long)p.B * H_kv < 4ll * p.resident && units < (1ll << 20) && units * stages < (1ll << 30) ? 1 : 0;
  // With so many units that they fill the chip four times over none is cut, and there is no merge: 256 sequences of 512 rows, 8 K/V
  // heads, one token 103 us instead of 113.  (One of 4096 rows among 255 of 64 takes 127 instead of 63.)
  long long grid = p.may_split ? units * stages : units;
  if (grid > p.resident) grid = p.resident;
  return (d == 64 ? launch_grouped<64>(p, cap, place, (unsigned)grid, st) : launch_grouped<128>(p, cap, place, (unsigned)grid, st))
             ? PROPD_OK
             : PROPD_ERR_DEVICE;
}
