// Norm of every query and key row and rotation by its token's position (baklava_qk_norm_rope).
//
//   n = x w / sqrt(mean(x^2) + eps);  (a, b) <- (a cos - b sin, a sin + b cos) for the pairs of the first rot_dim elements
//
// Bound by HBM: every row is read and written once.  A row is spread over D / 16 lanes, eight pairs each, chosen so that a
// lane holds both elements of its pairs: no exchange but the sum of squares.  A workgroup takes `tok` tokens with all their
// heads, so that an angle is formed once: one thread per token and pair takes it, reduced in 64 bits (a position times a
// frequency needs more bits than fp32 has: at 131072 the error would be 0.008), through LDS to the lanes that need it.
#include "common.h"

#include <algorithm>

namespace baklava {

namespace {

constexpr int kThreads = 256;

template <typename T> struct Piece;  // eight elements
template <> struct Piece<uint16_t> {
  __device__ static void load(const void* at, float* f) {
    const uint4 r = *reinterpret_cast<const uint4*>(at);
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  __device__ static void store(void* at, const float* f) {
    typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
    bf16x8_t v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (__bf16)f[i];
    *reinterpret_cast<bf16x8_t*>(at) = v;
  }
  __device__ static float one(const uint16_t* at) { return __uint_as_float((uint32_t)*at << 16); }
  __device__ static void put(uint16_t* at, float f) { *at = __builtin_bit_cast(uint16_t, (__bf16)f); }
};
template <> struct Piece<float> {
  __device__ static void load(const void* at, float* f) {
    const float4 a = reinterpret_cast<const float4*>(at)[0], b = reinterpret_cast<const float4*>(at)[1];
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
  __device__ static void store(void* at, const float* f) {
    reinterpret_cast<float4*>(at)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4*>(at)[1] = make_float4(f[4], f[5], f[6], f[7]);
  }
  __device__ static float one(const float* at) { return *at; }
  __device__ static void put(float* at, float f) { *at = f; }
};

// Where the elements of a lane's eight pairs lie: WHOLE: two runs of eight elements (a lane's pairs are neighbours of one run
// with INTER); otherwise (halves whose length is no multiple of eight) element by element.
template <typename T, int D, bool INTER, bool WHOLE>
__global__ __launch_bounds__(kThreads) void qk_norm_rope_kernel(RopeParams p) {
  constexpr int kLanes = D / 16, kPairs = D / 2, kRows = kThreads / kLanes;  // rows at a time
  extern __shared__ __attribute__((aligned(16))) float2 turn[];              // [tok][kPairs] (cos, sin)
  const int tid = threadIdx.x;
  const int b = p.seq0 + blockIdx.y, tok0 = blockIdx.x * p.tok, n_here = min(p.tok, p.T - tok0);
  const int64_t n_tok = (int64_t)p.n_seq * p.T;
  const int32_t* pos = p.pos + (int64_t)b * p.T + tok0;
  for (int i = tid; i < n_here * kPairs; i += kThreads) {
    const int pair = i % kPairs;
    float2 cs = make_float2(1.f, 0.f);
    if (pair < p.rot / 2) {
      const double t = (double)pos[p.axis[pair] * n_tok + i / kPairs] * p.turns[pair];
      const float half = (float)(2.0 * (t - rint(t)));  // in units of pi
      sincospif(half, &cs.y, &cs.x);
    }
    turn[i] = cs;
  }
  __syncthreads();
  const int sub = tid % kLanes, heads = p.Hq + p.Hkv;
  const int half = p.rot / 2;
  // first elements of the two runs
  const int at_a = INTER || 8 * sub >= half ? 16 * sub : 8 * sub, at_b = INTER || 8 * sub >= half ? 16 * sub + 8 : half + 8 * sub;
  const auto index = [&](int j, int second) {  // of pair 8 sub + j, where they do not lie in runs
    const int i = 8 * sub + j;
    return i < half ? i + second * half : 2 * i + second;
  };
  for (int r = tid / kLanes; r < n_here * heads; r += kRows) {
    const int t = r / heads, h = r % heads;
    const bool is_q = h < p.Hq;
    const int64_t tt = tok0 + t;
    const Rows& in = is_q ? p.q : p.k;
    const Rows& out = is_q ? p.q_out : p.k_out;
    const int hh = is_q ? h : h - p.Hq;
    const T* src = reinterpret_cast<const T*>(in.data) + b * in.seq + tt * in.tok + hh * in.head;
    T* dst = reinterpret_cast<T*>(out.data) + b * out.seq + tt * out.tok + hh * out.head;
    const T* w = reinterpret_cast<const T*>(is_q ? p.q_weight : p.k_weight);
    float x[16], wv[16];
    if (WHOLE) {
      Piece<T>::load(src + at_a, x);
      Piece<T>::load(src + at_b, x + 8);
    } else {
#pragma unroll
      for (int j = 0; j < 16; ++j) x[j] = Piece<T>::one(src + index(j % 8, j / 8));
    }
    if (w) {
      if (WHOLE) {
        Piece<T>::load(w + at_a, wv);
        Piece<T>::load(w + at_b, wv + 8);
      } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) wv[j] = Piece<T>::one(w + index(j % 8, j / 8));
      }
      float ss = 0.f;
#pragma unroll
      for (int j = 0; j < 16; ++j) ss = fmaf(x[j], x[j], ss);
#pragma unroll
      for (int o = 1; o < kLanes; o <<= 1) ss += __shfl_xor(ss, o);
      const float inv = 1.f / sqrtf(ss * (1.f / D) + p.eps);
#pragma unroll
      for (int j = 0; j < 16; ++j) x[j] *= inv * wv[j];
    }
    const float2* cs = turn + t * kPairs + 8 * sub;
    float y[16];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int a = INTER ? 2 * j : j, c = INTER ? 2 * j + 1 : j + 8;
      const float2 m = cs[j];
      y[a] = x[a] * m.x - x[c] * m.y;
      y[c] = x[a] * m.y + x[c] * m.x;
    }
    if (WHOLE && !INTER && 8 * sub >= half) {  // (not rotated, and the runs are neighbours: pairs do not matter)
#pragma unroll
      for (int j = 0; j < 16; ++j) y[j] = x[j];
    }
    if (WHOLE) {
      Piece<T>::store(dst + at_a, y);
      Piece<T>::store(dst + at_b, y + 8);
    } else {
#pragma unroll
      for (int j = 0; j < 16; ++j) Piece<T>::put(dst + index(j % 8, j / 8), y[j]);
    }
  }
}

template <typename T, int D>
void launch(const RopeParams& p, bool inter, dim3 grid, hipStream_t s) {
  const size_t lds = (size_t)p.tok * (D / 2) * sizeof(float2);
  if (inter) qk_norm_rope_kernel<T, D, true, true><<<grid, dim3(kThreads), lds, s>>>(p);
  else if (p.rot % 16 == 0) qk_norm_rope_kernel<T, D, false, true><<<grid, dim3(kThreads), lds, s>>>(p);
  else qk_norm_rope_kernel<T, D, false, false><<<grid, dim3(kThreads), lds, s>>>(p);
}

}  // namespace

hipError_t launch_qk_norm_rope(const RopeParams& p_in, int dtype, int D, bool interleaved, hipStream_t s) {
  if (p_in.n_seq <= 0 || p_in.T <= 0 || p_in.Hq + p_in.Hkv <= 0) return hipSuccess;
  RopeParams p = p_in;
  p.tok = p.T >= 4096 ? 4 : 1;
  for (p.seq0 = 0; p.seq0 < p.n_seq; p.seq0 += 65535) {  // a grid's second dimension holds no more
    const dim3 grid((p.T + p.tok - 1) / p.tok, std::min(65535, p.n_seq - p.seq0));
    if (dtype == 0) {
      if (D == 128) launch<uint16_t, 128>(p, interleaved, grid, s);
      else launch<uint16_t, 64>(p, interleaved, grid, s);
    } else {
      if (D == 128) launch<float, 128>(p, interleaved, grid, s);
      else launch<float, 64>(p, interleaved, grid, s);
    }
  }
  return hipGetLastError();
}

}  // namespace baklava
