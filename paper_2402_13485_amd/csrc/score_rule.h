// What the calls of a bounded cache share: lengths and positions of a sequence, and how scores are made of products.
#pragma once

#include <math.h>

#include "common.h"

namespace propd {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kMaxPosition = 1 << 30;  // positions lie below
// Distances up to this are exact in fp32: positions less the root's are held as such, and a window's edge is one of them.
constexpr int kMostWindow = 1 << 24;

// A cap beyond these is none of scores, nor is a scale beyond this, which would not be finite any more with log2(e) or over the cap.
constexpr float kLeastCap = 0x1p-10f, kMostCap = 1024.f, kMostScale = 0x1p64f;

inline bool score_rule_ok(const propd_score_rule *r) {
  return r && r->scale > 0.f && r->scale <= kMostScale && (r->cap == 0.f || (r->cap >= kLeastCap && r->cap <= kMostCap)) && r->window >= 0 &&
         r->window <= kMostWindow;
}

// positions back that a query sees, its own included
inline int window_of(const propd_score_rule *r) {
  return r->window > 0 ? r->window : kMaxPosition + 1;
}

struct Lengths {
  int L, T;        // cached rows, tree nodes
  int dropped, P;  // positions without a row, the root's position
};

__device__ __forceinline__ int root_position(int L, int dropped) {
  const long long P = (long long)L + dropped;
  return P > kMaxPosition ? kMaxPosition : (int)P;
}

// (what is read from device memory is made safe)
__device__ __forceinline__ Lengths lengths_of(const int32_t *seq_lens, const int32_t *n_nodes, const int32_t *dropped, int L_max,
                                              int T_max, int b) {
  Lengths n;
  n.L = seq_lens[b];
  n.L = n.L < 0 ? 0 : (n.L > L_max ? L_max : n.L);
  n.T = n_nodes ? n_nodes[b] : 1;
  n.T = n.T < 1 ? 1 : (n.T > T_max ? T_max : n.T);
  n.dropped = dropped ? dropped[b] : 0;
  n.dropped = n.dropped < 0 ? 0 : (n.dropped > kMaxPosition ? kMaxPosition : n.dropped);
  n.P = root_position(n.L, n.dropped);
  return n;
}

// The positions that a query at p_i sees are lowest .. lowest + reach: (unsigned)(p_j - lowest) <= reach also leaves negative
// positions out, since reach and lowest are at most 2^30.
struct Sight {
  int p_i, lowest, reach;
};
__device__ __forceinline__ Sight sight_of(int p_i, int window) {
  Sight s;
  s.p_i = p_i;
  s.lowest = p_i - window + 1 > 0 ? p_i - window + 1 : 0;
  s.reach = p_i - s.lowest;
  return s;
}
__device__ __forceinline__ bool in_sight(const Sight &s, int p_j) { return (unsigned)(p_j - s.lowest) <= (unsigned)s.reach; }

// cap tanh(x / cap) to fp32 precision, x finite or not.  With y = |x| / cap: below 3/4 the continued fraction of tanh
// cut behind 9, y (945 + 105 y^2 + y^4) / (945 + 420 y^2 + 15 y^4), 5e-9 off; above it (1 - e) / (1 + e) with e =
// exp(-2 y), whose subtraction loses two bits at most.
__device__ __forceinline__ float capped(float x, float cap, float inv_cap) {
  const float y = fabsf(x) * inv_cap, y2 = y * y;
  const float e = __builtin_amdgcn_exp2f(-2.f * kLog2e * y);
  const bool small = y < .75f;
  const float over = small ? y * fmaf(y2, y2 + 105.f, 945.f) : 1.f - e;
  const float under = small ? fmaf(y2, fmaf(15.f, y2, 420.f), 945.f) : 1.f + e;
  return copysignf(cap * over * __builtin_amdgcn_rcpf(under), x);
}

}  // namespace propd
