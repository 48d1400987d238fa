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
// Everything that decides is held in 64 bits: a vocabulary has 1e5 borders between tokens, and an error of 1e-7 in the sums
// would hand one draw in a hundred to a neighbour.  Launches: the largest logit and the sum of exponentials of parts of the rows
// that a decision can need (a node without children is none); the walk, a workgroup for each sequence; the weights of parts of
// the last node's row; the part and the token in it.
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

// 2^((x - top) c) for x <= top, 0 where x is -inf (top may be, too); c = log2(e) / temperature.  The fraction f of the exponent, at most
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
  return x > kNegInf ? __builtin_amdgcn_ldexp(s, (int)__builtin_fmax(n, -2000.0)) : 0.0;
}

__device__ __forceinline__ int nodes_of(const VerifyParams& p, int b) { return p.n_nodes ? min(max(p.n_nodes[b], 0), p.N) : p.N; }
__device__ __forceinline__ double exponent_scale(const VerifyParams& p, int b) {  // log2(e) / temperature; 0: greedy
  const float t = p.temp ? p.temp[b] : 1.f;
  return t > 0.f ? 1.4426950408889634 / (double)t : 0.0;
}

// Sums over the workgroup, in an order that does not change.
__device__ __forceinline__ double sum_threads(double x, double* lds) {
#pragma unroll
  for (int i = 32; i >= 1; i /= 2) x += __shfl_xor(x, i);
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
__device__ __forceinline__ Top top_of_threads(Top t, Top* lds) {
#pragma unroll
  for (int i = 32; i >= 1; i /= 2) t = higher(t, Top{__shfl_xor(t.x, i), __shfl_xor(t.first, i)});
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = t;
  __syncthreads();
  t = lds[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) t = higher(t, lds[w]);
  return t;
}

// One part of one row: workgroups over the parts first, then the nodes, then target and draft rows.
template <bool F32>
__global__ __launch_bounds__(kThreads) void verify_stat_kernel(VerifyParams p) {
  __shared__ double sums[kWaves];
  __shared__ Top tops[kWaves];
  const int part = (uint32_t)blockIdx.x % (uint32_t)p.parts, r = (uint32_t)blockIdx.x / (uint32_t)p.parts;
  const bool draft = r >= p.n_seq * p.N;
  const int at = draft ? r - p.n_seq * p.N : r, b = (uint32_t)at / (uint32_t)p.N, i = (uint32_t)at % (uint32_t)p.N;
  const int n = nodes_of(p, b), tid = threadIdx.x;
  const double inv = exponent_scale(p, b);
  if (i >= n) return;
  if (draft) {
    if (i == 0 || inv == 0.0) return;
    const int up = p.parent[(int64_t)b * p.N + i];
    if (up < 0 || up >= i) return;
  } else {
    bool child = false;
    for (int j = i + 1 + tid; j < n; j += kThreads) child = child || p.parent[(int64_t)b * p.N + j] == i;
    if (!__syncthreads_or(child)) return;
  }
  const void* row = row_at<F32>(draft ? p.draft : p.logits, at * (draft ? p.draft_row : p.row));
  const int v0 = part * kVerifyPart + tid * 8;
  float x[kPer / 8][8];
#pragma unroll
  for (int k = 0; k < kPer / 8; ++k) load8<F32>(x[k], row, v0 + k * kThreads * 8, p.V);
  Top t{kNegInf, INT32_MAX};
#pragma unroll
  for (int k = 0; k < kPer / 8; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (x[k][e] > t.x) t = Top{x[k][e], v0 + k * kThreads * 8 + e};
  t = top_of_threads(t, tops);
  double s = 0.0;
  if (inv > 0.0) {
#pragma unroll
    for (int k = 0; k < kPer / 8; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) s += weight(x[k][e], t.x, inv);
    s = sum_threads(s, sums);
  }
  if (tid == 0) p.stat[(int64_t)r * p.parts + part] = VerifyStat{s, t.x, t.first};
}

// All of a row from its parts, by 16 neighbouring lanes; the same in each.
__device__ __forceinline__ VerifyStat merged(const VerifyStat* s, int parts, double c) {
  const int l = threadIdx.x & 15;
  Top t{kNegInf, INT32_MAX};
  for (int i = l; i < parts; i += 16) t = higher(t, Top{s[i].top, s[i].first});
#pragma unroll
  for (int i = 8; i >= 1; i /= 2) t = higher(t, Top{__shfl_xor(t.x, i), __shfl_xor(t.first, i)});
  double sum = 0.0;
  if (c > 0.0) {
    for (int i = l; i < parts; i += 16) sum += s[i].sum * weight(s[i].top, t.x, c);
#pragma unroll
    for (int i = 8; i >= 1; i /= 2) sum += __shfl_xor(sum, i);
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

template <bool F32>
__global__ __launch_bounds__(kThreads) void verify_walk_kernel(VerifyParams p) {
  __shared__ int32_t parent[kMostNodes], token[kMostNodes], tried[kMostNodes];
  __shared__ double prob[kMostNodes], from[kMostNodes], left[kMostNodes];  // of node i's token: under its parent's row, under its own draft row
  __shared__ VerifyStat target[kMostNodes], drafts[kMostNodes];
  __shared__ float u[kMostNodes];
  __shared__ double sums[kWaves];
  static_assert(kMostNodes == kThreads, "a thread for every node");
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int n = nodes_of(p, b);
  const int64_t node0 = (int64_t)b * p.N;
  if (n == 0) {
    if (tid < p.N) p.path[node0 + tid] = -1;
    if (tid == 0) {
      p.n_path[b] = 0;
      p.end[b] = VerifyEnd{-1, 0};
    }
    return;
  }
  const double inv = exponent_scale(p, b);
  const bool rows = p.draft && inv > 0.0;
  int up = -1, mine = -1;
  if (tid < n && tid > 0) {
    up = p.parent[node0 + tid];
    if (up < 0 || up >= tid) up = -1;
    mine = p.token[node0 + tid];
    if (mine < 0 || mine >= p.V) mine = -1;  // (never accepted, and takes nothing off)
  }
  parent[tid] = up;
  token[tid] = mine;
  u[tid] = tid < n ? p.u[node0 + tid] : 0.f;
  tried[tid] = 0;                    // (until the walk: whether node tid has children)
  __syncthreads();
  if (up >= 0) tried[up] = 1;
  __syncthreads();
  for (int i = tid / 16; i < n; i += kThreads / 16) {
    if (tried[i]) {
      const VerifyStat s = merged(p.stat + (node0 + i) * p.parts, p.parts, inv);
      if (tid % 16 == 0) target[i] = p.all[node0 + i] = s;
    }
    if (rows && parent[i] >= 0) {
      const VerifyStat s = merged(p.stat + ((int64_t)p.n_seq * p.N + node0 + i) * p.parts, p.parts, inv);
      if (tid % 16 == 0) drafts[i] = p.draft_all[node0 + i] = s;
    }
  }
  __syncthreads();
  double pr = 0.0, q = 1.0;
  if (up >= 0 && mine >= 0) {
    const VerifyStat s = target[up];
    if (inv == 0.0) pr = s.top > kNegInf && s.first == mine ? 1.0 : 0.0;
    else if (s.sum > 0.0) pr = weight(load1<F32>(row_at<F32>(p.logits, (node0 + up) * p.row), mine), s.top, inv) * (1.0 / s.sum);
    if (rows) {
      const VerifyStat d = drafts[tid];
      q = d.sum > 0.0 ? weight(load1<F32>(row_at<F32>(p.draft, (node0 + tid) * p.draft_row), mine), d.top, inv) * (1.0 / d.sum) : 0.0;
    }
  }
  prob[tid] = pr;
  from[tid] = q;
  __syncthreads();

  // The walk, the same in all threads.
  int cur = 0, n_path = 1, n_tried = 0;
  double off = 0.0;                  // what the point masses of those tried have taken off
  if (tid == 0) p.path[node0] = 0;
  for (int w = 0; w * 64 < n;) {     // the children of cur among nodes 64 w .. + 63
    const int j = w * 64 + lane;
    unsigned long long todo = __ballot(j > cur && j < n && parent[j < n ? j : 0] == cur);
    bool moved = false;
    while (todo) {
      const int i = w * 64 + __builtin_ctzll(todo);
      todo &= todo - 1;
      const int t = token[i];
      if (t < 0) continue;
      double r = prob[i];
      bool again = false;            // a point mass on this token has been taken off already
      if (rows && n_tried > 0) {     // the sum that the child before has left
        const VerifyStat s = target[cur];
        const void* row = row_at<F32>(p.logits, (node0 + cur) * p.row);
        double z = 0.0;
#pragma unroll 1
        for (int v = tid * 8; v < p.V; v += kThreads * 8) {
          float x[8];
          double y[8], unused[8];
          load8<F32>(x, row, v, p.V);
          rest_of<F32>(y, unused, p, node0, s, drafts, x, v, tried, left, n_tried, inv);
#pragma unroll
          for (int e = 0; e < 8; ++e) z += y[e];
        }
        z = sum_threads(z, sums);
        if (z > 0.0) {
          if (tid == 0) left[n_tried - 1] = z;
        } else {
          n_tried -= 1;              // nothing: it stays as it was before
        }
        __syncthreads();
        if (n_tried > 0) r = rest_of_one<F32>(p, node0, s, drafts, t, row, tried, left, n_tried, inv);
      } else if (!rows) {
        for (int k = 0; k < n_tried; ++k) again = again || token[tried[k]] == t;
        r = again ? 0.0 : r / (1.0 - off);
      }
      if ((double)u[i] * from[i] < r) {
        cur = i;
        if (tid == 0) p.path[node0 + n_path] = i;
        n_path += 1;
        n_tried = 0;
        off = 0.0;
        moved = true;
        break;
      }
      // (a token without weight takes nothing off, and one that has all of it leaves it as it is)
      if (rows || (!again && r > 0.0 && 1.0 - off - prob[i] > 0.0)) {
        off += prob[i];
        __syncthreads();             // (tried has been read)
        if (tid == 0) tried[n_tried] = i;
        n_tried += 1;
        __syncthreads();
      }
    }
    w = moved ? cur / 64 : w + 1;
  }
  if (tid >= n_path && tid < p.N) p.path[node0 + tid] = -1;
  if (tid < n_tried) {
    p.tried[node0 + tid] = tried[tid];
    p.left[node0 + tid] = left[tid];
  }
  if (tid == 0) {
    p.n_path[b] = n_path;
    p.end[b] = VerifyEnd{cur, n_tried};
  }
}

// Tokens whose point masses were taken off have no weight: -inf in their place.  x[k][e]: element v0 + k kThreads 8 + e.
template <int K>
__device__ __forceinline__ void take_off(const VerifyParams& p, int64_t node0, int n_tried, float (&x)[K][8], int v0) {
#pragma unroll 1
  for (int j = 0; j < n_tried; ++j) {
    const int at = p.token[node0 + p.tried[node0 + j]] - v0;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (at == k * kThreads * 8 + e) x[k][e] = kNegInf;
  }
}

// Weights of the last node's row, a part each.
template <bool F32>
__global__ __launch_bounds__(kThreads) void verify_mass_kernel(VerifyParams p) {
  __shared__ double sums[kWaves];
  __shared__ Top tops[kWaves];
  const int part = (uint32_t)blockIdx.x % (uint32_t)p.parts, b = (uint32_t)blockIdx.x / (uint32_t)p.parts, tid = threadIdx.x;
  const VerifyEnd e = p.end[b];
  if (e.last < 0) return;
  const int64_t node0 = (int64_t)b * p.N;
  const double inv = exponent_scale(p, b);
  const void* row = row_at<F32>(p.logits, (node0 + e.last) * p.row);
  const int v0 = part * kVerifyPart + tid * 8;
  float x[kPer / 8][8];
#pragma unroll
  for (int k = 0; k < kPer / 8; ++k) load8<F32>(x[k], row, v0 + k * kThreads * 8, p.V);
  const bool rows = p.draft && inv > 0.0 && e.n_tried > 0;
  if (!rows && inv > 0.0) take_off(p, node0, e.n_tried, x, v0);
  Top t{kNegInf, INT32_MAX};
#pragma unroll
  for (int k = 0; k < kPer / 8; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (x[k][i] > t.x) t = Top{x[k][i], v0 + k * kThreads * 8 + i};
  t = top_of_threads(t, tops);
  double all = 0.0, without = 0.0;
  if (inv > 0.0) {
    if (rows) {
      const VerifyStat s = p.all[node0 + e.last];
#pragma unroll 1
      for (int k = 0; k < kPer / 8; ++k) {
        const int v = v0 + k * kThreads * 8;
        if (v >= p.V) break;
        float y[8];
        double r[8], before[8];
        load8<F32>(y, row, v, p.V);
        rest_of<F32>(r, before, p, node0, s, p.draft_all + node0, y, v, p.tried + node0, p.left + node0, e.n_tried, inv);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          all += r[i];
          without += before[i];
        }
      }
    } else {
      // relative to the part's largest logit, so that the whole row's is not needed
#pragma unroll
      for (int k = 0; k < kPer / 8; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) all += weight(x[k][i], t.x, inv);
      without = all;
    }
    all = sum_threads(all, sums);
    without = sum_threads(without, sums);
  }
  if (tid == 0) {
    p.mass[((int64_t)b * p.parts + part) * 2] = all;
    p.mass[((int64_t)b * p.parts + part) * 2 + 1] = without;
    p.top[(int64_t)b * p.parts + part] = VerifyStat{0.0, t.x, t.first};
  }
}

template <bool F32>
__global__ __launch_bounds__(kThreads) void verify_pick_kernel(VerifyParams p) {
  __shared__ double w[kVerifyPart + kThreads];  // weights of the part's elements: a place is left out behind every kPer
  __shared__ double sums[kWaves];
  __shared__ Top tops[kWaves];
  __shared__ int found;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const VerifyEnd e = p.end[b];
  if (e.last < 0) {
    if (tid == 0) p.next[b] = -1;
    return;
  }
  const int64_t node0 = (int64_t)b * p.N;
  const double inv = exponent_scale(p, b);
  const VerifyStat* tops_of = p.top + (int64_t)b * p.parts;
  Top t{kNegInf, INT32_MAX};
  for (int i = tid; i < p.parts; i += kThreads) t = higher(t, Top{tops_of[i].top, tops_of[i].first});
  t = top_of_threads(t, tops);
  if (t.x == kNegInf || inv == 0.0) {
    if (tid == 0) p.next[b] = t.x == kNegInf ? -1 : t.first;
    return;
  }
  // The part, by every wavefront for itself.
  const bool rows = p.draft && e.n_tried > 0;
  const double* mass = p.mass + (int64_t)b * p.parts * 2;
  auto mass_of = [&](int i, int which) { return i >= p.parts ? 0.0 : rows ? mass[2 * i + which] : mass[2 * i] * weight(tops_of[i].top, t.x, inv); };
  auto total_of = [&](int which) {
    double s = 0.0;
    for (int i = lane; i < p.parts; i += 64) s += mass_of(i, which);
#pragma unroll
    for (int i = 32; i >= 1; i /= 2) s += __shfl_xor(s, i);
    return s;
  };
  auto scan = [&](double x) {
#pragma unroll
    for (int i = 1; i < 64; i *= 2) {
      const double y = __shfl_up(x, i);
      x += lane >= i ? y : 0.0;
    }
    return x;
  };
  double total = total_of(0);
  int which = 0;
  if (rows && !(total > 0.0)) {  // nothing was left by the last child that was tried: as it was before
    which = 1;
    total = total_of(1);
  }
  const double want = fmin(fmax((double)p.u[node0], 0.0), 1.0) * total;
  int part = -1;
  double before = 0.0, c0 = 0.0;
  for (int i0 = 0; i0 < p.parts; i0 += 64) {
    const double m = mass_of(i0 + lane, which), c = c0 + scan(m);
    const unsigned long long over = __ballot(m > 0.0 && c > want), some = __ballot(m > 0.0);
    if (over | some) {
      const int l = over ? __builtin_ctzll(over) : 63 - __builtin_clzll(some);  // (without one: the last that has any weight)
      part = i0 + l;
      before = __shfl(c - m, l);
    }
    if (over) break;
    c0 = __shfl(c, 63);
  }
  if (part < 0) {
    if (tid == 0) p.next[b] = -1;
    return;
  }
  const void* row = row_at<F32>(p.logits, (node0 + e.last) * p.row);
  auto place = [](int i) { return i + i / kPer; };
#pragma unroll 1
  for (int k = 0; k < kPer / 8; ++k) {
    const int at = k * kThreads * 8 + tid * 8, v = part * kVerifyPart + at;
    float x[1][8];
    double y[8];
    load8<F32>(x[0], row, v, p.V);
    if (rows) {
      double prev[8];
      rest_of<F32>(y, prev, p, node0, p.all[node0 + e.last], p.draft_all + node0, x[0], v, p.tried + node0, p.left + node0, e.n_tried, inv);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = which ? prev[i] : y[i];
    } else {
      take_off(p, node0, e.n_tried, x, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = weight(x[0][i], t.x, inv);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) w[place(at + i)] = y[i];
  }
  if (tid == 0) found = INT32_MAX;
  __syncthreads();
  const double* mine = w + tid * (kPer + 1);
  double sum = 0.0;
#pragma unroll 8
  for (int i = 0; i < kPer; ++i) sum += mine[i];
  double end = scan(sum);
  if (lane == 63) sums[wave] = end;
  __syncthreads();
  for (int x = 0; x < wave; ++x) end += sums[x];
  // The first element whose sum exceeds; where rounding leaves none, the last one that has any weight.
  double c = before + end - sum;
  int last = -1, hit = -1;
#pragma unroll 8
  for (int i = 0; i < kPer; ++i) {
    const double y = mine[i];
    c += y;
    if (y > 0.0) last = i;
    if (hit < 0 && y > 0.0 && c > want) hit = i;
  }
  const int v0 = part * kVerifyPart + tid * kPer;
  if (hit >= 0) atomicMin(&found, v0 + hit);
  __syncthreads();
  const bool none = found == INT32_MAX;
  __syncthreads();
  if (none) {
    if (tid == 0) found = -1;
    __syncthreads();
    if (last >= 0) atomicMax(&found, v0 + last);
    __syncthreads();
  }
  if (tid == 0) p.next[b] = found;
}

template <bool F32>
hipError_t launch(const VerifyParams& p, hipStream_t s) {
  const int64_t rows = (int64_t)p.n_seq * p.N * (p.draft ? 2 : 1);
  if (rows * p.parts > INT32_MAX / kThreads) return hipErrorInvalidValue;
  verify_stat_kernel<F32><<<dim3((unsigned)(rows * p.parts)), dim3(kThreads), 0, s>>>(p);
  verify_walk_kernel<F32><<<dim3((unsigned)p.n_seq), dim3(kThreads), 0, s>>>(p);
  verify_mass_kernel<F32><<<dim3((unsigned)(p.n_seq * p.parts)), dim3(kThreads), 0, s>>>(p);
  verify_pick_kernel<F32><<<dim3((unsigned)p.n_seq), dim3(kThreads), 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_verify_draft(const VerifyParams& p, int dtype, hipStream_t s) {
  return dtype == 1 ? launch<true>(p, s) : launch<false>(p, s);
}

}  // namespace baklava
