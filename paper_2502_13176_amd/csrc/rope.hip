// Norm of every query and key row and rotation by its token's position (baklava_qk_norm_rope).
//
//   n = x w / sqrt(mean(x^2) + eps);  (a, b) <- (a cos - b sin, a sin + b cos) for the pairs of the first rot_dim elements
//
// Bound by HBM: every row is read and written once.  A row is spread over D / 16 lanes, eight pairs each, chosen so that a
// lane holds both elements of its pairs: no exchange but the sum of squares.  A workgroup takes `tok` tokens with all their
// heads, so that an angle is formed once: one thread per token and pair takes it, reduced in 64 bits (a position times a
// frequency needs more bits than fp32 has: at 131072 the error would be 0.008), through LDS to the lanes that need it, while
// the first rows are on their way.
//
// 32768 tokens of 40 heads of 128 bf16 elements take 115 to 119 us, 5.6 to 5.8 TB/s read and written (6.2 is what a copy reaches),
// 12000 of 24 heads in fp32 48 us, 6.1 TB/s; 8 tokens 4.7 us on the device, which the 16 us of a call from Python hide.
#include "common.h"

#include <algorithm>
#include <type_traits>

namespace baklava {

namespace {

constexpr int kThreads = 256;
constexpr int kMostWgs = (1 << 24) - 1;  // a grid's first dimension holds fewer than 2^32 threads
// Bytes of a workgroup's rows, about, from 4096 tokens of all sequences on (smaller launches take a token each, to fill the chip);
// a workgroup's tokens are of one sequence.  us, a token each / as here: 64 sequences of 2048 bf16 tokens of 14 heads of 64 230 /
// 76, of 2 heads 289 / 28, 16 of 2048 tokens of 40 heads of 128 142 / 127, 1024 of 17 tokens of 14 heads of 64 34.8 / 16.6.  What
// is on its way together must not lie far apart, and a workgroup must have some to hide its angles behind.  us, 12 / 20 / 32 KiB:
// 32768 bf16 tokens of 40 heads of 128 136 / 119 / 119, 30000 of 24 heads of 64 33.0 / 33.5 / 37.3; fp32, whose rows take half the
// arithmetic for a byte, 12000 of 24 heads of 128 48.4 / 48.2 / 54.2, 20000 of 16 heads of 64 30.3 / 37.9 / 46.0.
constexpr int kWgBytes16 = 20 * 1024, kWgBytes32 = 12 * 1024;

// Sum over four or eight neighbouring lanes, every one of them receiving it.
template <int LANES>
__device__ __forceinline__ float group_sum(float v) {
  auto dpp = [](float x, auto ctrl) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  v += dpp(v, std::integral_constant<int, 0xb1>{});  // quad_perm:[1,0,3,2]
  v += dpp(v, std::integral_constant<int, 0x4e>{});  // quad_perm:[2,3,0,1]
  if (LANES == 8) v += dpp(v, std::integral_constant<int, 0x141>{});  // row_half_mirror
  return v;
}

// RUN elements as they lie in memory, in fp32, and back with one rounding.
template <int RUN>
__device__ __forceinline__ void load_run(const uint16_t* at, float* f) {
  uint32_t w[RUN / 2];
  if constexpr (RUN == 8) {
    const uint4 r = *reinterpret_cast<const uint4*>(at);
    w[0] = r.x; w[1] = r.y; w[2] = r.z; w[3] = r.w;
  } else {
    const uint2 r = *reinterpret_cast<const uint2*>(at);
    w[0] = r.x; w[1] = r.y;
  }
#pragma unroll
  for (int i = 0; i < RUN / 2; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
template <int RUN>
__device__ __forceinline__ void load_run(const float* at, float* f) {
#pragma unroll
  for (int i = 0; i < RUN; i += 4) {
    const float4 r = *reinterpret_cast<const float4*>(at + i);
    f[i] = r.x; f[i + 1] = r.y; f[i + 2] = r.z; f[i + 3] = r.w;
  }
}
template <int RUN>
__device__ __forceinline__ void store_run(uint16_t* at, const float* f) {
  typedef __bf16 bf16x8_t __attribute__((ext_vector_type(RUN)));
  bf16x8_t v;
#pragma unroll
  for (int i = 0; i < RUN; ++i) v[i] = (__bf16)f[i];
  __builtin_nontemporal_store(v, reinterpret_cast<bf16x8_t*>(at));
}
template <int RUN>
__device__ __forceinline__ void store_run(float* at, const float* f) {
  typedef float floatx4_t __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int i = 0; i < RUN; i += 4)
    __builtin_nontemporal_store(floatx4_t{f[i], f[i + 1], f[i + 2], f[i + 3]}, reinterpret_cast<floatx4_t*>(at + i));
}
__device__ __forceinline__ float load_one(const uint16_t* at) { return __uint_as_float((uint32_t)*at << 16); }
__device__ __forceinline__ float load_one(const float* at) { return *at; }
__device__ __forceinline__ void store_one(uint16_t* at, float f) { *at = __builtin_bit_cast(uint16_t, (__bf16)f); }
__device__ __forceinline__ void store_one(float* at, float f) { *at = f; }

// A lane holds eight pairs of a row, x[j] the first element of pair j and x[8 + j] the second (INTER: the elements as they lie).
// RUN: they lie in runs of 8 or 4 elements, and the lanes of a row take neighbouring runs; 1: element by element (halves whose
// length is no multiple of four).  Pairs that are not rotated are of neighbours.
template <typename T, int D, bool INTER, int RUN>
__global__ __launch_bounds__(kThreads) void qk_norm_rope_kernel(RopeParams p) {
  constexpr int kLanes = D / 16, kPairs = D / 2, kRows = kThreads / kLanes;  // rows at a time
  extern __shared__ __attribute__((aligned(16))) float2 turn[];              // [tok][kPairs] (cos, sin)
  const int tid = threadIdx.x;
  const int b = p.seq0 + blockIdx.y, tok0 = p.tok0 + blockIdx.x * p.tok, n_here = min(p.tok, p.T - tok0);
  const int64_t n_tok = (int64_t)p.n_seq * p.T;
  const int32_t* pos = p.pos + (int64_t)b * p.T + tok0;
  const int sub = tid % kLanes;
  const int half = p.rot / 2;
  auto pair_of = [&](int j) {  // pair j's number, j < 8
    if (INTER) return RUN / 2 * (sub + kLanes * (2 * j / RUN)) + j % (RUN / 2);
    return RUN > 1 ? RUN * (sub + kLanes * (j / RUN)) + j % RUN : 8 * sub + j;
  };
  auto place = [&](int j) {  // of x[j] in the row
    if (INTER) return 2 * pair_of(j / 2) + j % 2;
    const int i = pair_of(j % 8), in_run = RUN > 1 ? j % RUN : 0;
    return i - in_run < half ? i + j / 8 * half : 2 * i - in_run + j / 8 * RUN;
  };
  auto load = [&](const T* at, float (&x)[16]) {
    if constexpr (RUN > 1) {
#pragma unroll
      for (int j = 0; j < 16; j += RUN) load_run<RUN>(at + place(j), x + j);
    } else {
#pragma unroll
      for (int j = 0; j < 16; ++j) x[j] = load_one(at + place(j));
    }
  };
  // The rows of queries, then those of keys: row r is head r % H of token r / H.  Addresses of a row from the first token's first.
  struct Side {
    const T* in;
    T* out;
    uint32_t in_tok, out_tok;
    uint64_t in_head, out_head;
    const T* weight;
    int heads;
  };
  auto side = [&](const Rows& in, const Rows& out, const void* w, int heads) {
    return Side{reinterpret_cast<const T*>(in.data) + b * in.seq + tok0 * in.tok,
                reinterpret_cast<T*>(out.data) + b * out.seq + tok0 * out.tok,
                (uint32_t)in.tok, (uint32_t)out.tok, (uint64_t)in.head, (uint64_t)out.head,
                reinterpret_cast<const T*>(w), heads};
  };
  const int row0 = tid / kLanes;
  float next[16];
  const Side first = p.Hq > 0 ? side(p.q, p.q_out, p.q_weight, p.Hq) : side(p.k, p.k_out, p.k_weight, p.Hkv);
  if (row0 < n_here * first.heads)  // on its way while the angles are formed
    load(first.in + row0 % first.heads * first.in_head + (uint32_t)(row0 / first.heads) * first.in_tok, next);
  for (int i = tid; i < n_here * kPairs; i += kThreads) {
    const int pair = i % kPairs;
    float2 cs = make_float2(1.f, 0.f);
    if (pair < half) {
      const double turns = (double)pos[p.axis[pair] * n_tok + i / kPairs] * p.turns[pair];
      const float in_pi = (float)(2.0 * (turns - rint(turns)));
      sincospif(in_pi, &cs.y, &cs.x);
    }
    turn[i] = cs;
  }
  __syncthreads();

  auto rows = [&](const Side& sd, bool requested) {
    const int n_rows = n_here * sd.heads;
    if (row0 >= n_rows) return;
    int t = row0 / sd.heads, h = row0 % sd.heads;
    if (!requested) load(sd.in + h * sd.in_head + (uint32_t)t * sd.in_tok, next);
    float w[16];
    if (sd.weight) load(sd.weight, w);
    for (int r = row0; r < n_rows;) {
      const float2* cs = turn + t * kPairs;
      T* dst = sd.out + h * sd.out_head + (uint32_t)t * sd.out_tok;
      float x[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) x[j] = next[j];
      r += kRows;
      h += kRows;
      while (h >= sd.heads) {
        h -= sd.heads;
        ++t;
      }
      if (r < n_rows) load(sd.in + h * sd.in_head + (uint32_t)t * sd.in_tok, next);
      if (sd.weight) {
        float ss = 0.f;
#pragma unroll
        for (int j = 0; j < 16; ++j) ss = fmaf(x[j], x[j], ss);
        ss = group_sum<kLanes>(ss);
        const float inv = rsqrtf(ss * (1.f / D) + p.eps);
#pragma unroll
        for (int j = 0; j < 16; ++j) x[j] *= inv * w[j];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int a = INTER ? 2 * j : j, c = INTER ? 2 * j + 1 : j + 8;
        const int pair = pair_of(j);
        const float2 m = cs[pair];
        const bool turns = (INTER || RUN == 1 ? pair : pair - j % RUN) < half;  // (a run is rotated as a whole)
        const float xa = x[a], xc = x[c];
        x[a] = turns ? xa * m.x - xc * m.y : xa;
        x[c] = turns ? xa * m.y + xc * m.x : xc;
      }
      if constexpr (RUN > 1) {
#pragma unroll
        for (int j = 0; j < 16; j += RUN) store_run<RUN>(dst + place(j), x + j);
      } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) store_one(dst + place(j), x[j]);
      }
    }
  };
  rows(first, true);
  if (p.Hq > 0 && p.Hkv > 0) rows(side(p.k, p.k_out, p.k_weight, p.Hkv), false);
}

// Runs of 16 bytes where halves are made of them, of four 16-bit elements where their length is a multiple of four, else element by
// element: 12000 bf16 tokens of 24 heads of 128, halves of 64 / 12 / 11 pairs 25.3 / 33.2 / 129 us, fp32 43.7 / 56.1 / 193.
template <typename T, int D>
void launch(const RopeParams& p, bool inter, dim3 grid, hipStream_t s) {
  constexpr int kRun = 16 / sizeof(T);
  const size_t lds = (size_t)p.tok * (D / 2) * sizeof(float2);
  if (inter) qk_norm_rope_kernel<T, D, true, kRun><<<grid, dim3(kThreads), lds, s>>>(p);
  else if (p.rot % (2 * kRun) == 0) qk_norm_rope_kernel<T, D, false, kRun><<<grid, dim3(kThreads), lds, s>>>(p);
  else if (p.rot % 8 == 0) qk_norm_rope_kernel<T, D, false, 4><<<grid, dim3(kThreads), lds, s>>>(p);
  else qk_norm_rope_kernel<T, D, false, 1><<<grid, dim3(kThreads), lds, s>>>(p);
}

}  // namespace

hipError_t launch_qk_norm_rope(const RopeParams& p_in, int dtype, int D, bool interleaved, hipStream_t s) {
  if (p_in.n_seq <= 0 || p_in.T <= 0 || p_in.Hq + p_in.Hkv <= 0) return hipSuccess;
  RopeParams p = p_in;
  const int token_bytes = (p.Hq + p.Hkv) * D * (dtype == 0 ? 2 : 4);
  p.tok = (int64_t)p.n_seq * p.T < 4096 ? 1 : std::max(1, std::min({16, p.T, (dtype == 0 ? kWgBytes16 : kWgBytes32) / token_bytes}));
  const int most_tok = kMostWgs * p.tok;
  for (int64_t seq0 = 0; seq0 < p.n_seq; seq0 += 65535) {  // a grid's second dimension holds no more
    p.seq0 = (int32_t)seq0;
    for (p.tok0 = 0; p.tok0 < p.T; p.tok0 += most_tok) {
      const dim3 grid((std::min(most_tok, p.T - p.tok0) + p.tok - 1) / p.tok, std::min(65535, p.n_seq - p.seq0));
      if (dtype == 0) {
        if (D == 128) launch<uint16_t, 128>(p, interleaved, grid, s);
        else launch<uint16_t, 64>(p, interleaved, grid, s);
      } else {
        if (D == 128) launch<float, 128>(p, interleaved, grid, s);
        else launch<float, 64>(p, interleaved, grid, s);
      }
    }
  }
  return hipGetLastError();
}

}  // namespace baklava
