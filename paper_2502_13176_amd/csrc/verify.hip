// Verification of drafted tokens against the target's probabilities from given random numbers (baklava_verify_draft).
//
// With p_i = softmax(x_i / T) of node i's row and q_i = softmax(d_i / T), the distribution node i's token t_i was drawn from (without
// draft rows, or at T = 0: all of it on t_i; p_i at T = 0: all of it on the first of the largest logits):
//
//   cur = 0, r = p_0;  for every node i with parent cur, in turn:  u_i q_i(t_i) < r(t_i):  cur = i, r = p_i
//                                                                  else  r = max(r - q_i, 0) / its sum
//
// and the next token is the first v with r(0) + ... + r(v) > u_0 (r(0) + ... + r(V - 1)).  So whatever the drafts are, the tokens
// are distributed as if the target had been sampled one by one.
//
// What decides between tokens next to each other is held in 64 bits: a vocabulary has 1e5 borders, and an error of 1e-7 in the sums
// would hand one draw in a hundred to a neighbour.  So are the sums of nodes with several children, of whose rows little may be left
// when a child's turn comes.  The one probability that a single child is tested against may be off by some 1e-8 (2e-7 at most: a
// quarter of the sum's error, 2^-22 of the exponentials and up to 9 * 2^-24 of rounded differences of fp32 logits): its sum takes the
// hardware's exponential, with what its argument lacks put back.
//
// Launches: the largest logit and the sum of exponentials of parts of the rows that a decision can need (a node without children is
// none; point masses: without the tokens that its children drafted); the walk, and the weights of parts of the last node's row, of which the last workgroup to end takes the token.  With
// draft rows what is left of a distribution is a difference, so the walk is a launch of its own that also sums up the rows it
// ends with in 64 bits.
//
// Latency bounds it: chains of memory reads, and code that is run through once and comes from memory itself (a launch of 16 KB
// of straight-line code takes 8 us, of 32 KB 29), which is why loops are kept as loops.  Chain of 5, 32000 tokens, greedy: 12 us (4.7 and 7.6); 8 trees of up to 32 nodes, 131072
// tokens: 31 us (28 with sums by the hardware's exponential there, too); 16 chains of 6 with draft rows, 100003 tokens in fp32: 51 us (20 for 77
// MB, 12.5, 19).  Siblings with draft rows are the costly ones, by how many fail: 8 trees of 16 nodes, 131072 tokens in bf16, 56 us; of 32
// nodes, paths of 2 to 5, 510.
#include "common.h"

namespace baklava {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kPer = kVerifyPart / kThreads;  // elements of a part that a thread takes
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kMost = 3.402823466e38f;

// Logits as they count: NaN is none, infinity the largest finite one.
__device__ __forceinline__ float logit(float x) { return x == x ? fminf(x, kMost) : kNegInf; }

// Elements v .. v + 7 of a row of V; -inf behind it.  (Rows lie at any multiple of an element.)
template <bool F32>
__device__ __forceinline__ void load8(float (&x)[8], const void* row, int v, int V) {
  if (F32) {
    const float* at = reinterpret_cast<const float*>(row) + v;
    if (v + 8 <= V) {
      __builtin_memcpy(x, at, 32);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = logit(x[e]);
      return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = v + e < V ? logit(at[e]) : kNegInf;
  } else {
    const uint16_t* at = reinterpret_cast<const uint16_t*>(row) + v;
    if (v + 8 <= V) {
      uint32_t w[4];
      __builtin_memcpy(w, at, 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[2 * e] = logit(__uint_as_float(w[e] << 16));
        x[2 * e + 1] = logit(__uint_as_float(w[e] & 0xffff0000u));
      }
      return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = v + e < V ? logit(__uint_as_float((uint32_t)at[e] << 16)) : kNegInf;
  }
}

template <bool F32>
__device__ __forceinline__ float load1(const void* row, int v) {
  return logit(F32 ? reinterpret_cast<const float*>(row)[v] : __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(row)[v] << 16));
}

template <bool F32>
__device__ __forceinline__ const void* row_at(const void* data, int64_t row) {
  return reinterpret_cast<const char*>(data) + row * (F32 ? 4 : 2);
}

// 2^((x - top) c) for x <= top, 0 where x is -inf (top may be, too: y is NaN); c = log2(e) / temperature.  The fraction f of the exponent, at most
// 1/2, goes into the series sum (f ln 2)^k / k!, whose next term is below 2^-47 of it; equal logits give exactly 1.
__device__ __forceinline__ double weight(float x, float top, double c) {
  const double y = ((double)x - (double)top) * c, n = __builtin_rint(y), f = y - n;
  double s = 7.0549116208011233e-9;                  // ln2^10 / 10!
  s = __builtin_fma(s, f, 1.0178086009239699e-7);    // ln2^9 / 9!
  s = __builtin_fma(s, f, 1.3215486790144307e-6);
  s = __builtin_fma(s, f, 1.5252733804059840e-5);
  s = __builtin_fma(s, f, 1.5403530393381608e-4);
  s = __builtin_fma(s, f, 1.3333558146428443e-3);
  s = __builtin_fma(s, f, 9.6181291076284771e-3);
  s = __builtin_fma(s, f, 5.5504108664821579e-2);
  s = __builtin_fma(s, f, 2.4022650695910071e-1);
  s = __builtin_fma(s, f, 6.9314718055994531e-1);
  s = __builtin_fma(s, f, 1.0);
  return y > -1080.0 ? __builtin_amdgcn_ldexp(s, (int)n) : 0.0;  // (far below, f is the product's rounding and s anything)
}

__device__ __forceinline__ int nodes_of(const VerifyParams& p, int b) { return p.n_nodes ? min(max(p.n_nodes[b], 0), p.N) : p.N; }
__device__ __forceinline__ double exponent_scale(const VerifyParams& p, int b) {  // log2(e) / temperature; 0: greedy
  const float t = p.temp ? p.temp[b] : 1.f;
  return t > 0.f ? __builtin_fmax(1.4426950408889634 / (double)t, 1e-300) : 0.0;  // (of an infinite one no more than a sign is left)
}

// x of the lane ROR further on in its row of 16.
template <int ROR>
__device__ __forceinline__ int row_turn(int x) { return __builtin_amdgcn_update_dpp(0, x, 0x120 + ROR, 0xf, 0xf, true); }
template <int ROR>
__device__ __forceinline__ float row_turn(float x) { return __int_as_float(row_turn<ROR>(__float_as_int(x))); }
template <int ROR>
__device__ __forceinline__ double row_turn(double x) {
  return __hiloint2double(row_turn<ROR>(__double2hiint(x)), row_turn<ROR>(__double2loint(x)));
}
__device__ __forceinline__ double of_lane(double x, int lane) {
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(x), lane), __builtin_amdgcn_readlane(__double2loint(x), lane));
}
// Sum over a row of 16 lanes, in each of them.  (Lanes l and l + 8 first: whichever a lane starts from, the same pairs are added.)
__device__ __forceinline__ double sum_row(double x) {
  x += row_turn<8>(x);
  x += row_turn<4>(x);
  x += row_turn<2>(x);
  x += row_turn<1>(x);
  return x;
}
__device__ __forceinline__ double sum_wave(double x) {
  x = sum_row(x);
  return of_lane(x, 0) + of_lane(x, 16) + of_lane(x, 32) + of_lane(x, 48);
}
// Sum over the wavefront's lanes up to and with the calling one.
template <int CTRL, int ROWS>
__device__ __forceinline__ double shifted(double x) {  // 0 where there is no lane to come from
  return __hiloint2double(__builtin_amdgcn_update_dpp(0, __double2hiint(x), CTRL, ROWS, 0xf, false),
                          __builtin_amdgcn_update_dpp(0, __double2loint(x), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ double scan_wave(double x) {
  x += shifted<0x111, 0xf>(x);  // row_shr:1
  x += shifted<0x112, 0xf>(x);
  x += shifted<0x114, 0xf>(x);
  x += shifted<0x118, 0xf>(x);
  x += shifted<0x142, 0xa>(x);  // row_bcast:15 into rows 1 and 3
  x += shifted<0x143, 0xc>(x);  // row_bcast:31 into rows 2 and 3
  return x;
}
// Sums over the workgroup, in an order that does not change.
__device__ __forceinline__ double sum_threads(double x, double* lds) {
  x = sum_wave(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) s += lds[w];
  return s;
}

struct Top {
  float x;
  int first;
};
__device__ __forceinline__ Top higher(Top a, Top b) { return b.x > a.x || (b.x == a.x && b.first < a.first) ? b : a; }
template <int ROR>
__device__ __forceinline__ Top row_turn(Top t) { return Top{row_turn<ROR>(t.x), row_turn<ROR>(t.first)}; }
__device__ __forceinline__ Top top_row(Top t) {
  t = higher(t, row_turn<8>(t));
  t = higher(t, row_turn<4>(t));
  t = higher(t, row_turn<2>(t));
  return higher(t, row_turn<1>(t));
}
__device__ __forceinline__ Top of_lane(Top t, int lane) {
  return Top{__int_as_float(__builtin_amdgcn_readlane(__float_as_int(t.x), lane)), __builtin_amdgcn_readlane(t.first, lane)};
}
__device__ __forceinline__ Top top_of_threads(Top t, Top* lds) {
  t = top_row(t);
  t = higher(higher(of_lane(t, 0), of_lane(t, 16)), higher(of_lane(t, 32), of_lane(t, 48)));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = t;
  __syncthreads();
  t = lds[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) t = higher(t, lds[w]);
  return t;
}

// The same by the hardware's exponential: c = (hi + lo) unit, and what the product with the difference lacks goes in behind it.  unit
// is 1, or, where a difference beyond fp32 may weigh something (c < 2^-100), 2^-64: what the difference loses then at its lower end
// is nothing to the exponent.  Below 2^-150, where the product may be -inf too (or NaN: x is -inf), it is 0.
__device__ __forceinline__ float quick_weight(float x, float top, float unit, float hi, float lo) {
  const float d = fmaf(x, unit, -top * unit), y = d * hi, rest = fmaf(d, lo, fmaf(d, hi, -y));
  const float w = __builtin_amdgcn_exp2f(y);
  return y > -150.f ? fmaf(w, rest * 0.69314718f, w) : 0.f;
}

// One part of one row: workgroups over the parts first, then the nodes, then target and draft rows.
template <bool F32>
__global__ __launch_bounds__(kThreads) void verify_stat_kernel(VerifyParams p) {
  __shared__ double sums[kWaves];
  __shared__ Top tops[kWaves];
  __shared__ int32_t children[kMostNodes];
  __shared__ uint32_t taken[kThreads];        // bits of the part's elements that are a child's token
  static_assert(kVerifyPart == 32 * kThreads, "a word for every thread");
  const int part = (uint32_t)blockIdx.x % (uint32_t)p.parts, r = (uint32_t)blockIdx.x / (uint32_t)p.parts;
  const bool draft = r >= p.n_seq * p.N;
  const int at = draft ? r - p.n_seq * p.N : r, b = (uint32_t)at / (uint32_t)p.N, i = (uint32_t)at % (uint32_t)p.N;
  const int n = nodes_of(p, b), tid = threadIdx.x;
  const double c = exponent_scale(p, b);
  if (!draft && i == 0 && part == 0 && tid == 0) p.ticket[b] = 0;
  if (i >= n) return;
  children[tid] = 0;
  taken[tid] = 0;
  // Drafted tokens that are point masses: what the children of a node leave of its row is added up from what is left, never a
  // difference, so their tokens are no part of its sum.
  const bool apart = !p.draft && c > 0.0;
  int up = -1, mine = -1;
  if (tid < n) {
    up = p.parent[(int64_t)b * p.N + tid];
    if (apart) mine = p.token[(int64_t)b * p.N + tid];
  }
  if (up < 0 || up >= tid) up = -1;
  __syncthreads();
  if (up >= 0) atomicAdd(&children[up], 1);
  if (up == i && mine >= 0 && mine / kVerifyPart == part) atomicOr(&taken[mine % kVerifyPart / 32], 1u << (mine & 31));
  if (draft) {
    if (!__syncthreads_or(tid == i && up >= 0) || c == 0.0) return;
  } else {
    __syncthreads();
    if (children[i] == 0) return;
  }
  // Nodes with several children: what rejected ones leave of a distribution is a part of it, as small as 2^-24 of it each time, and
  // decides what becomes of the next one.  (Draft rows: with any such node of the sequence.)
  const bool precise = c > 0.0 && (p.draft ? __syncthreads_or(children[tid] > 1) : children[i] > 1);
  const void* row = row_at<F32>(draft ? p.draft : p.logits, at * (draft ? p.draft_row : p.row));
  const int v0 = part * kVerifyPart + tid * 8;
  float x[kPer / 8][8];
#pragma unroll
  for (int k = 0; k < kPer / 8; ++k) load8<F32>(x[k], row, v0 + k * kThreads * 8, p.V);
  if (apart) {
#pragma unroll
    for (int k = 0; k < kPer / 8; ++k) {
      const uint32_t bits = reinterpret_cast<const uint8_t*>(taken)[k * kThreads + tid];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[k][e] = bits >> e & 1 ? kNegInf : x[k][e];
    }
  }
  Top t{kNegInf, INT32_MAX};
#pragma unroll
  for (int k = 0; k < kPer / 8; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (x[k][e] > t.x) t = Top{x[k][e], v0 + k * kThreads * 8 + e};
  t = top_of_threads(t, tops);
  double s = 0.0;
  if (precise) {
#pragma unroll
    for (int k = 0; k < kPer / 8; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) s += weight(x[k][e], t.x, c);
    s = sum_threads(s, sums);
  } else if (c > 0.0) {
    const float unit = c < 0x1p-100 ? 0x1p-64f : 1.f;
    const double scale = c / (double)unit;
    const float hi = (float)__builtin_fmin(scale, 1e38), lo = scale > 1e38 ? 0.f : (float)(scale - (double)hi);
#pragma unroll
    for (int k = 0; k < kPer / 8; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) s += (double)quick_weight(x[k][e], t.x, unit, hi, lo);
    s = sum_threads(s, sums);
  }
  if (tid == 0) p.stat[(int64_t)r * p.parts + part] = VerifyStat{s, t.x, t.first};
}

// All of a row from its parts, by 16 neighbouring lanes; the same in each.
__device__ __forceinline__ VerifyStat merged(const VerifyStat* s, int parts, double c) {
  const int l = threadIdx.x & 15;
  Top t{kNegInf, INT32_MAX};
  for (int i = l; i < parts; i += 16) t = higher(t, Top{s[i].top, s[i].first});
  t = top_row(t);
  double sum = 0.0;
  if (c > 0.0) {
    for (int i = l; i < parts; i += 16) sum += s[i].sum * weight(s[i].top, t.x, c);
    sum = sum_row(sum);
  }
  return VerifyStat{sum, t.x, t.first};
}

// Probabilities of elements v .. v + 7 of a node's row (logits x) when what n_tried children have left of it is known: of all but the
// last one divided by its sum.  before: without the last one.  (target, drafts: merged statistics of the node's row and of the draft
// rows.)  Elements behind the row: 0.
template <bool F32>
__device__ __forceinline__ void rest_of(double (&r)[8], double (&before)[8], const VerifyParams& p, int64_t node0, const VerifyStat& target,
                                        const VerifyStat* drafts, const float (&x)[8], int v, const int32_t* tried, const double* left,
                                        int n_tried, double c) {
  const double one = target.sum > 0.0 ? 1.0 / target.sum : 0.0;
#pragma unroll
  for (int e = 0; e < 8; ++e) before[e] = r[e] = weight(x[e], target.top, c) * one;
#pragma unroll 1
  for (int k = 0; k < n_tried; ++k) {
    const int j = tried[k];
    const VerifyStat d = drafts[j];
    const double unit = d.sum > 0.0 ? 1.0 / d.sum : 0.0, open = k + 1 < n_tried ? 1.0 / left[k] : 1.0;
    float y[8];
    load8<F32>(y, row_at<F32>(p.draft, (node0 + j) * p.draft_row), v, p.V);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      before[e] = r[e];
      r[e] = __builtin_fmax(r[e] - weight(y[e], d.top, c) * unit, 0.0) * open;
    }
  }
}
// ... of one element, all divided.
template <bool F32>
__device__ __forceinline__ double rest_of_one(const VerifyParams& p, int64_t node0, const VerifyStat& target, const VerifyStat* drafts, int v,
                                              const void* row, const int32_t* tried, const double* left, int n_tried, double c) {
  double r = target.sum > 0.0 ? weight(load1<F32>(row, v), target.top, c) * (1.0 / target.sum) : 0.0;
#pragma unroll 1
  for (int k = 0; k < n_tried; ++k) {
    const int j = tried[k];
    const VerifyStat d = drafts[j];
    const double q = d.sum > 0.0 ? weight(load1<F32>(row_at<F32>(p.draft, (node0 + j) * p.draft_row), v), d.top, c) * (1.0 / d.sum) : 0.0;
    r = __builtin_fmax(r - q, 0.0) / left[k];
  }
  return r;
}

// What the walk of a sequence leaves.
struct Walk {
  // tried: children of the last node that have had an effect (walk_points: their tokens)
  int32_t parent[kMostNodes], token[kMostNodes], tried[kMostNodes];
  // of node i's token: under its parent's row, under its own draft row.  Point masses: weight of the token in its parent's row, and of all
  // those in it that no child has drafted, relative to the row's largest logit; at T = 0 the probability, and 0.
  double prob[kMostNodes], from[kMostNodes];
  double left[kMostNodes];                    // what is left by tried[k], before it is divided
  VerifyStat target[kMostNodes], drafts[kMostNodes];
  int32_t peak[kMostNodes];                   // point masses: the largest logit that a child has drafted, ordered as whole numbers are
  float u[kMostNodes];
  double sums[kWaves];
  unsigned long long stands[kMostNodes / 64];  // bits of nodes that are accepted if they are tried
  int32_t n_tried;
};

// Logits as whole numbers of the same order, and back.
__device__ __forceinline__ int ordered(int x) { return x ^ (x >> 31 & 0x7fffffff); }

// Nodes of a sequence into LDS, with what the rows of those that have children say (rows: and the draft rows), and the probabilities
// of each node's token.  Returns node threadIdx.x's parent, or -1.
template <bool F32>
__device__ __forceinline__ int load_nodes(const VerifyParams& p, int b, int n, double c, bool rows, Walk& w) {
  static_assert(kMostNodes == kThreads, "a thread for every node");
  const int tid = threadIdx.x;
  const int64_t node0 = (int64_t)b * p.N;
  int up = -1, mine = -1;
  if (tid < n) {
    w.u[tid] = p.u[node0 + tid];
    up = p.parent[node0 + tid];
    mine = p.token[node0 + tid];
  }
  if (tid == 0 || up < 0 || up >= tid) up = -1;
  if (mine < 0 || mine >= p.V) mine = -1;     // (never accepted, and takes nothing off)
  w.parent[tid] = up;
  w.token[tid] = mine;
  w.tried[tid] = 0;                           // (for now: the children of node tid)
  w.peak[tid] = INT32_MIN;
  __syncthreads();
  if (up >= 0) atomicAdd(&w.tried[up], 1);
  float x = 0.f, y = 0.f;                     // logits of the node's token
  if (up >= 0 && mine >= 0) {
    x = load1<F32>(row_at<F32>(p.logits, (node0 + up) * p.row), mine);
    if (rows) y = load1<F32>(row_at<F32>(p.draft, (node0 + tid) * p.draft_row), mine);
    else atomicMax(&w.peak[up], ordered(__float_as_int(x)));
  }
  __syncthreads();
#pragma unroll 1
  for (int k = tid / 16; k < (rows ? 2 * n : n); k += kThreads / 16) {  // target rows, then draft rows
    const bool draft = k >= n;
    const int i = draft ? k - n : k;
    if (!draft ? w.tried[i] == 0 : w.parent[i] < 0) continue;
    const VerifyStat s = merged(p.stat + ((draft ? (int64_t)p.n_seq * p.N : 0) + node0 + i) * p.parts, p.parts, c);
    if (tid % 16 == 0) (draft ? w.drafts : w.target)[i] = s;
  }
  __syncthreads();
  double pr = 0.0, q = 0.0;
  if (up >= 0 && mine >= 0) {
    const VerifyStat s = w.target[up];
    if (c == 0.0) {
      pr = s.top > kNegInf && s.first == mine ? 1.0 : 0.0;
    } else if (rows) {
      if (s.sum > 0.0) pr = weight(x, s.top, c) * (1.0 / s.sum);
      const VerifyStat d = w.drafts[tid];
      q = d.sum > 0.0 ? weight(y, d.top, c) * (1.0 / d.sum) : 0.0;
    } else {
      const float top = fmaxf(s.top, __int_as_float(ordered(w.peak[up])));
      pr = weight(x, top, c);
      q = s.sum * weight(s.top, top, c);
    }
  }
  w.prob[tid] = pr;
  w.from[tid] = q;
  __syncthreads();
  return up;
}

__device__ __forceinline__ void write_path(const VerifyParams& p, int64_t node0, int b, int n_path) {
  const int tid = threadIdx.x;
  if (tid >= n_path && tid < p.N) p.path[node0 + tid] = -1;
  if (tid == 0) p.n_path[b] = n_path;
}

// The walk where drafted tokens are point masses, by a workgroup together; write: its path goes out.  n > 0.  What those tried before
// a node have left follows from its siblings, so whether a node would be accepted is known without the walk:
//   r(token) = its weight / (weights of the tokens that no sibling has drafted + of those of siblings from it on),
// a sum of what is left, whose error stays relative to it however little that is.
template <bool F32>
__device__ __forceinline__ VerifyEnd walk_points(const VerifyParams& p, int b, int n, double c, Walk& w, bool write) {
  const int tid = threadIdx.x, lane = tid & 63;
  const int64_t node0 = (int64_t)b * p.N;
  const int up = load_nodes<F32>(p, b, n, c, false, w);
  const int mine = w.token[tid], wave = tid >> 6;
  if (tid < 4) w.stands[tid] = 0;
  if (tid == 0) w.n_tried = 0;
  // Nodes that have siblings, one after the other against all of a wavefront.
  auto siblings = [&](auto&& against) {
    if (wave * 64 >= n) return;
#pragma unroll 1
    for (int g = 0; g * 64 < n; ++g) {
      const int at = g * 64 + lane, its_up = w.parent[at], its_token = w.token[at];
      const double its_weight = w.prob[at];
      unsigned long long todo = __ballot(its_up >= 0 && w.tried[its_up < 0 ? 0 : its_up] > 1);
#pragma unroll 1
      while (todo) {
        const int j = __builtin_ctzll(todo);
        todo &= todo - 1;
        against(g * 64 + j, __builtin_amdgcn_readlane(its_up, j) == up, __builtin_amdgcn_readlane(its_token, j), of_lane(its_weight, j));
      }
    }
  };
  bool again = false;                         // a sibling before has this token, which is then gone already
  siblings([&](int j, bool mine_too, int its_token, double) { again = again || (mine_too && j < tid && its_token == mine); });
  __syncthreads();
  if (again) w.prob[tid] = 0.0;
  __syncthreads();
  const double own = w.prob[tid];
  double after = w.from[tid];                 // what is left behind this node
  siblings([&](int j, bool mine_too, int, double its_weight) { after += mine_too && j > tid ? its_weight : 0.0; });
  const bool stands = up >= 0 && own > 0.0 && (double)w.u[tid] < own / (after + own);
  const unsigned long long these = __ballot(stands);
  if (lane == 0) w.stands[tid / 64] = these;
  __syncthreads();
  int cur = 0, n_path = 1;
  if (write && tid == 0) p.path[node0] = 0;
#pragma unroll 1
  for (int g = 0; g * 64 < n;) {              // the children of cur among nodes 64 g .. + 63, the same in all wavefronts
    const unsigned long long hit = __ballot(w.parent[g * 64 + lane] == cur) & w.stands[g];
    if (hit == 0) {
      ++g;
      continue;
    }
    cur = g * 64 + __builtin_ctzll(hit);
    if (write && tid == 0) p.path[node0 + n_path] = cur;
    n_path += 1;
  }
  // (a token without weight takes nothing off, and one that has all that is left leaves it as it is)
  if (up == cur && own > 0.0 && after > 0.0) w.tried[atomicAdd(&w.n_tried, 1)] = mine;  // (its token)
  __syncthreads();
  if (write) write_path(p, node0, b, n_path);
  return VerifyEnd{cur, w.n_tried};
}

// The walk where they were drawn from the draft rows, one child after the other.
template <bool F32>
__device__ __forceinline__ VerifyEnd walk_rows(const VerifyParams& p, int b, int n, double c, Walk& w, bool write) {
  const int tid = threadIdx.x, lane = tid & 63;
  const int64_t node0 = (int64_t)b * p.N;
  load_nodes<F32>(p, b, n, c, true, w);
  int cur = 0, n_path = 1, n_tried = 0;
  if (write && tid == 0) p.path[node0] = 0;
#pragma unroll 1
  for (int g = 0; g * 64 < n;) {              // the children of cur among nodes 64 g .. + 63
    unsigned long long todo = __ballot(w.parent[g * 64 + lane] == cur);
    bool moved = false;
#pragma unroll 1
    while (todo) {
      const int i = g * 64 + __builtin_ctzll(todo);
      todo &= todo - 1;
      const int t = w.token[i];
      if (t < 0) continue;
      double r = w.prob[i];
      if (n_tried > 0) {                      // the sum that the child before has left
        const VerifyStat s = w.target[cur];
        const void* row = row_at<F32>(p.logits, (node0 + cur) * p.row);
        double z = 0.0;
#pragma unroll 1
        for (int v = tid * 8; v < p.V; v += kThreads * 8) {
          float x8[8];
          double y8[8], unused[8];
          load8<F32>(x8, row, v, p.V);
          rest_of<F32>(y8, unused, p, node0, s, w.drafts, x8, v, w.tried, w.left, n_tried, c);
#pragma unroll
          for (int e = 0; e < 8; ++e) z += y8[e];
        }
        z = sum_threads(z, w.sums);
        if (z > 0.0) {
          if (tid == 0) w.left[n_tried - 1] = z;
        } else {
          n_tried -= 1;                       // nothing: it stays as it was before
        }
        __syncthreads();
        if (n_tried > 0) r = rest_of_one<F32>(p, node0, s, w.drafts, t, row, w.tried, w.left, n_tried, c);
      }
      if ((double)w.u[i] * w.from[i] < r) {
        cur = i;
        if (write && tid == 0) p.path[node0 + n_path] = i;
        n_path += 1;
        n_tried = 0;
        moved = true;
        break;
      }
      __syncthreads();                        // (tried has been read)
      if (tid == 0) w.tried[n_tried] = i;
      n_tried += 1;
      __syncthreads();
    }
    g = moved ? cur / 64 : g + 1;
  }
  if (write) write_path(p, node0, b, n_path);
  return VerifyEnd{cur, n_tried};
}

// A sequence without nodes.
__device__ __forceinline__ void no_walk(const VerifyParams& p, int b) {
  const int tid = threadIdx.x;
  if (tid < p.N) p.path[(int64_t)b * p.N + tid] = -1;
  if (tid == 0) {
    p.n_path[b] = 0;
    p.next[b] = -1;
  }
}

// With draft rows: the walk, by every workgroup of a sequence, and the sums over a part of the rows it has ended with, in 64 bits.
template <bool F32>
__global__ __launch_bounds__(kThreads) void verify_walk_kernel(VerifyParams p) {
  __shared__ Walk w;
  const int part = (uint32_t)blockIdx.x % (uint32_t)p.parts, b = (uint32_t)blockIdx.x / (uint32_t)p.parts, tid = threadIdx.x;
  const int n = nodes_of(p, b);
  const double c = exponent_scale(p, b);
  if (n == 0) {
    if (part == 0) no_walk(p, b);
    return;
  }
  const VerifyEnd e = c > 0.0 ? walk_rows<F32>(p, b, n, c, w, part == 0) : walk_points<F32>(p, b, n, c, w, part == 0);
  const int64_t node0 = (int64_t)b * p.N;
  if (part == 0) {
    if (tid < e.n_tried) {
      p.tried[node0 + tid] = w.tried[tid];
      p.left[node0 + tid] = w.left[tid];
    }
    if (tid == 0) p.end[b] = e;
  }
  if (c == 0.0) return;
#pragma unroll 1
  for (int k = -1; k < e.n_tried && e.n_tried > 0; ++k) {
    const int i = k < 0 ? e.last : w.tried[k];
    VerifyStat* st = p.exact + ((int64_t)(k < 0 ? 0 : p.n_seq * p.N) + node0 + i) * p.parts + part;
    const VerifyStat was = p.stat[((int64_t)(k < 0 ? 0 : p.n_seq * p.N) + node0 + i) * p.parts + part];
    const void* row = row_at<F32>(k < 0 ? p.logits : p.draft, (node0 + i) * (k < 0 ? p.row : p.draft_row));
    float x[kPer / 8][8];
    const int v0 = part * kVerifyPart + tid * 8;
#pragma unroll
    for (int g = 0; g < kPer / 8; ++g) load8<F32>(x[g], row, v0 + g * kThreads * 8, p.V);
    double s = 0.0;
#pragma unroll
    for (int g = 0; g < kPer / 8; ++g)
#pragma unroll
      for (int e8 = 0; e8 < 8; ++e8) s += weight(x[g][e8], was.top, c);
    s = sum_threads(s, w.sums);
    if (tid == 0) *st = VerifyStat{s, was.top, was.first};
  }
}

// Weights of the last node's row, a part of kPick elements each; the last workgroup of a sequence to end picks the token.  WALK: each
// workgroup takes the walk itself first (there are no draft rows).
constexpr int kPick = kVerifyPick, kHeldParts = 256;
static_assert(kPick == kThreads * 8, "eight elements a thread");
template <bool F32, bool WALK>
__global__ __launch_bounds__(kThreads) void verify_pick_kernel(VerifyParams p) {
  __shared__ Walk w;
  __shared__ Top tops[kWaves];
  __shared__ VerifyMass held[kHeldParts];
  __shared__ int found, is_last;
  const int part = (uint32_t)blockIdx.x % (uint32_t)p.picks, b = (uint32_t)blockIdx.x / (uint32_t)p.picks;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = nodes_of(p, b);
  const double c = exponent_scale(p, b);
  if (n == 0) {
    if (WALK && part == 0) no_walk(p, b);
    return;
  }
  const int64_t node0 = (int64_t)b * p.N;
  VerifyEnd e;
  if (WALK) e = walk_points<F32>(p, b, n, c, w, part == 0);
  else e = p.end[b];
  const bool rows = !WALK && c > 0.0 && e.n_tried > 0;
  if (rows) {
    if (tid < e.n_tried) {
      w.tried[tid] = p.tried[node0 + tid];
      w.left[tid] = p.left[node0 + tid];
    }
    __syncthreads();
    for (int k = tid / 16 - 1; k < e.n_tried; k += kThreads / 16) {
      const int i = k < 0 ? e.last : w.tried[k];
      const VerifyStat s = merged(p.exact + ((int64_t)(k < 0 ? 0 : p.n_seq * p.N) + node0 + i) * p.parts, p.parts, c);
      if (tid % 16 == 0) (k < 0 ? w.target : w.drafts)[i] = s;
    }
    __syncthreads();
  }
  const void* row = row_at<F32>(p.logits, (node0 + e.last) * p.row);
  // Eight elements of a part as they count: point masses that were taken off are gone.
  auto load = [&](float (&x)[8], int v) {
    load8<F32>(x, row, v, p.V);
    if (WALK && c > 0.0)
      for (int j = 0; j < e.n_tried; ++j) {
        const int at = w.tried[j] - v;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = at == i ? kNegInf : x[i];
      }
  };
  // What other workgroups read is written and read past the caches that the chip's parts do not share.
  VerifyMass* const parts = p.mass + (int64_t)b * p.picks;
  int at = part, which = 0;
  double want = 0.0, before = 0.0;
  Top t;
  // First its own part; the last workgroup then goes over the part that holds the token.
#pragma unroll 1
  for (int pass = 0;; ++pass) {
    float x[8];
    const int v = at * kPick + tid * 8;
    load(x, v);
    if (pass == 0) {
      t = Top{kNegInf, INT32_MAX};
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (x[i] > t.x) t = Top{x[i], v + i};
      t = top_of_threads(t, tops);
    }
    double y[8], prev[8], sum = 0.0, sum_prev = 0.0;
    if (rows) {
      rest_of<F32>(y, prev, p, node0, w.target[e.last], w.drafts, x, v, w.tried, w.left, e.n_tried, c);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        sum_prev += prev[i];
        y[i] = which ? prev[i] : y[i];
      }
    } else if (c > 0.0) {  // relative to the part's largest logit at first, so that the whole row's is not needed
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = weight(x[i], t.x, c);
    }
    if (c > 0.0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += y[i];
    }
    if (pass == 1) {
      double end = scan_wave(sum);
      if (lane == 63) w.sums[wave] = end;
      __syncthreads();
      for (int i = 0; i < wave; ++i) end += w.sums[i];
      // The first element whose sum exceeds; where rounding leaves none, the last one that has any weight.
      double s = before + end - sum;
      int last = -1, hit = -1;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        s += y[i];
        if (y[i] > 0.0) last = v + i;
        if (hit < 0 && y[i] > 0.0 && s > want) hit = v + i;
      }
      if (hit >= 0) atomicMin(&found, hit);
      __syncthreads();
      const bool none = found == INT32_MAX;
      __syncthreads();
      if (none) {
        if (tid == 0) found = -1;
        __syncthreads();
        if (last >= 0) atomicMax(&found, last);
        __syncthreads();
      }
      if (tid == 0) p.next[b] = found;
      return;
    }
    if (c > 0.0) sum = sum_threads(sum, w.sums);
    if (rows) sum_prev = sum_threads(sum_prev, w.sums);
    if (tid == 0) {
      __hip_atomic_store(&parts[part].all, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(&parts[part].without, sum_prev, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(&parts[part].top, t.x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(&parts[part].first, t.first, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      // The four have arrived before the ticket is drawn.  (They go past the caches as they are: an ordering of the atomic's own
      // would write back and empty the L2 of a whole part of the chip, for every workgroup.)
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      is_last = __hip_atomic_fetch_add(p.ticket + b, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == p.picks - 1;
      found = INT32_MAX;
    }
    __syncthreads();
    if (!is_last) return;
    // Parts as far as they fit into LDS are fetched once.
    auto fetch = [&](int i) {
      VerifyMass m;
      m.all = __hip_atomic_load(&parts[i].all, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      m.without = __hip_atomic_load(&parts[i].without, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      m.top = __hip_atomic_load(&parts[i].top, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      m.first = __hip_atomic_load(&parts[i].first, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      return m;
    };
    t = Top{kNegInf, INT32_MAX};
    for (int i = tid; i < p.picks; i += kThreads) {
      const VerifyMass m = fetch(i);
      if (i < kHeldParts) held[i] = m;
      t = higher(t, Top{m.top, m.first});
    }
    t = top_of_threads(t, tops);  // (its barriers also stand between the writes and the reads of `held`)
    if (t.x == kNegInf || c == 0.0) {
      if (tid == 0) p.next[b] = t.x == kNegInf ? -1 : t.first;
      return;
    }
    // The part, by every wavefront for itself.
    auto mass_of = [&](int i) {
      if (i >= p.picks) return 0.0;
      const VerifyMass m = i < kHeldParts ? held[i] : fetch(i);
      const double y = which ? m.without : m.all;
      return rows ? y : y * weight(m.top, t.x, c);
    };
    double total = 0.0;
#pragma unroll 1
    for (which = 0;; which = 1) {
      for (int i = lane; i < p.picks; i += 64) total += mass_of(i);
      total = sum_wave(total);
      if (total > 0.0 || !rows || which == 1) break;  // (nothing was left by the last child that was tried: as it was before)
      total = 0.0;
    }
    want = fmin(fmax((double)(WALK ? w.u[0] : p.u[node0]), 0.0), 1.0) * total;
    at = -1;
    double c0 = 0.0;
    for (int i0 = 0; i0 < p.picks; i0 += 64) {
      const double m = mass_of(i0 + lane), s = c0 + scan_wave(m);
      const unsigned long long over = __ballot(m > 0.0 && s > want), some = __ballot(m > 0.0);
      if (over | some) {
        const int l = over ? __builtin_ctzll(over) : 63 - __builtin_clzll(some);  // (without one: the last that has any weight)
        at = i0 + l;
        before = of_lane(s - m, l);
      }
      if (over) break;
      c0 = of_lane(s, 63);
    }
    if (at < 0) {
      if (tid == 0) p.next[b] = -1;
      return;
    }
  }
}

template <bool F32>
hipError_t launch(const VerifyParams& p, hipStream_t s) {
  const int64_t rows = (int64_t)p.n_seq * p.N * (p.draft ? 2 : 1);
  const dim3 b(kThreads), picks((unsigned)(p.n_seq * p.picks));
  verify_stat_kernel<F32><<<dim3((unsigned)(rows * p.parts)), b, 0, s>>>(p);
  if (p.draft) {
    verify_walk_kernel<F32><<<dim3((unsigned)(p.n_seq * p.parts)), b, 0, s>>>(p);
    verify_pick_kernel<F32, false><<<picks, b, 0, s>>>(p);
  } else {
    verify_pick_kernel<F32, true><<<picks, b, 0, s>>>(p);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_verify_draft(const VerifyParams& p, int dtype, hipStream_t s) {
  return dtype == 1 ? launch<true>(p, s) : launch<false>(p, s);
}

}  // namespace baklava
