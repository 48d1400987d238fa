// Decode attention over ragged caches of 4-bit rows (BAKLAVA_MXFP4), up to 16 query heads per KV head.
//
// The two products of 32 rows are those of the bf16 kernel (v_mfma_f32_16x16x32_bf16):
//
//   S^T[row, g]  = K[row, :] . Q[g, :]          O^T[d, g] += V^T[d, rows] . P^T[rows, g]
//
// and so are the pipeline of a wavefront that streams its own slabs, the softmax on the accumulators' layout and the records
// of the calls whose weights are owed to the scores.  What differs is how rows become operands.  A lane loads D / 8 bytes of a
// K row, the D / 4 elements (jg D / 4 ...) of row n16 for lane (n16, jg), and the first product numbers the head dimension the
// same way (chunk c of lane group jg: elements jg D / 4 + 8 c .. + 8), so that codes become the A operand where they lie, two
// per conversion instruction, without a trip through LDS.  Values of codes are exact in bf16.  V has to be transposed: its
// codes are converted in the lane that loaded them, the bf16 rows go to LDS and are read back transposed.  Weights enter the
// second product as three bf16 terms, which is all of their 24 bits.  (The instruction that multiplies 4-bit operands as they lie,
// v_mfma_scale_f32_16x16x128_f8f6f4, adds with an error of 5e-5 relative, measured; logits deserve better.)
//
// Bound by the read rate and by what a launch costs: 136 bytes per row of 128 elements.  Four heads, 64 caches of 9830 rows on
// average, tracked: 20 us of which 12 are the bytes at 7.06 TB/s; calls of different sizes lie on 7 to 10 us + bytes / 6.57 TB/s.
// The merge of the split caches is a kernel of its own (some 3 us); inside this one, by the last workgroup of a cache to
// arrive, it took as long.  Recorded calls cost a pass over K in one call out of `lag_batch`; the flush of eight calls of four
// heads over 2.5 million rows takes 45 us (27 for the bytes).  Nothing in it is saturated (vector ALUs 58% of the cycles in which
// a compute unit is busy, matrix pipe 23%): a slab is a chain of requests, products, exponentials, exchanges through LDS and a
// write to the ring, and a wavefront waits for data half of its time and for its turn to issue 30%.  Two slabs requested ahead
// instead of one make no difference.  The attention kernel is no different: vector ALUs 46% (four heads, one workgroup per compute
// unit) to 58% (seven heads, two), matrix pipe 23 to 28%, LDS 35 to 42%, two fifths of that bank conflicts.
#include "common.h"
#include "decode_tail.h"
#include "mxfp4.h"

namespace baklava {

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float floatx4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

constexpr int kTiles = 2;             // tiles of 16 rows per wavefront iteration
constexpr int kSlab = 16 * kTiles;
constexpr int kWaves = 8;
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLowest = -3.402823466e38f;

template <int D>
struct Shape {
  static constexpr int kBytes = D / 2;             // of a row's codes
  static constexpr int kWords = D / 32;            // words (eight codes) a lane takes of a row, a chunk of the first product each
  static constexpr int kChunks = D / 32;
  static constexpr int kBlocks = D / 16;
  static constexpr int kQRow = D * 2;              // bytes of a query row
  static constexpr int kVStride = D * 2 + 32;      // bytes between staged V rows
};

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ bf16x8_t as_bf16x8(uint4 x) { return __builtin_bit_cast(bf16x8_t, x); }

// D / 8 bytes of codes.
template <int W> struct Codes { uint32_t w[W]; };
__device__ __forceinline__ void load_codes(Codes<4>& c, const void* at) {
  const uint4 r = load_nt16(at);
  c.w[0] = r.x; c.w[1] = r.y; c.w[2] = r.z; c.w[3] = r.w;
}
__device__ __forceinline__ void load_codes(Codes<2>& c, const void* at) {
  typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
  const u32x2_t r = __builtin_nontemporal_load(reinterpret_cast<const u32x2_t*>(at));
  c.w[0] = r.x; c.w[1] = r.y;
}

// The recorded calls of one cache, as in the bf16 kernel but for the numbering of the head dimension.
constexpr int kSets = 2;
template <int D>
struct Record {
  bf16x8_t q[kSets][Shape<D>::kChunks];
  float m[kSets][4], inv[kSets][4];
  int n_slot[kSets];
};

template <int D>
__device__ __forceinline__ void load_record(const DecodeParams& p, int c, int G, int pending, int n16, int jg, Record<D>& r) {
  constexpr int kRow = Shape<D>::kQRow;
  const int gp_mask = (1 << p.lag_gp_log2) - 1;
  const unsigned char* lq = reinterpret_cast<const unsigned char*>(p.lag_q) + (int64_t)c * kLagRows * kRow;
#pragma unroll
  for (int e = 0; e < kSets; ++e) {
    const int R = 16 * e + n16;
#pragma unroll
    for (int ch = 0; ch < Shape<D>::kChunks; ++ch) {
      uint4 raw = make_uint4(0, 0, 0, 0);  // rows beyond the G heads of a call, calls not on record: zero
      if ((R & gp_mask) < G && (R >> p.lag_gp_log2) < pending)
        raw = *reinterpret_cast<const uint4*>(lq + R * kRow + jg * (D / 2) + ch * 16);
      r.q[e][ch] = as_bf16x8(raw);
    }
    const int slot = (16 * e + 4 * jg) >> p.lag_gp_log2;
    r.n_slot[e] = 0;
    if (slot < pending) r.n_slot[e] = p.lag_n[(int64_t)c * kLagCalls + slot];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int m = 16 * e + 4 * jg + i;
      r.m[e][i] = 0.f;
      r.inv[e][i] = 0.f;
      if ((m & gp_mask) < G && slot < pending) {
        r.m[e][i] = p.lag_ml[((int64_t)c * kLagRows + m) * 2];
        r.inv[e][i] = p.lag_ml[((int64_t)c * kLagRows + m) * 2 + 1];
      }
    }
  }
}

// Weights of the recorded calls for the rows of a slab; on return lane l < kSlab holds that of row l.
template <int D>
__device__ __forceinline__ float record_weights(const floatx4_t (&sp)[kSets][kTiles], const Record<D>& r, float cs, int row_first,
                                                int lane) {
  const int n16 = lane & 15;
  float w[kTiles];
#pragma unroll
  for (int T = 0; T < kTiles; ++T) {
    w[T] = 0.f;
#pragma unroll
    for (int e = 0; e < kSets; ++e) {
      float acc = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) acc += fast_exp2(sp[e][T][i] * cs - r.m[e][i]) * r.inv[e][i];
      w[T] += (row_first + T * 16 + n16 < r.n_slot[e]) ? acc : 0.f;
    }
    w[T] += __shfl_xor(w[T], 16);
    w[T] += __shfl_xor(w[T], 32);
  }
  float mine = w[0];
#pragma unroll
  for (int T = 1; T < kTiles; ++T) mine = lane >> 4 == T ? w[T] : mine;
  return mine;
}

// The new row of a fused append, rounded, into slot n_old (see append_new_row).
template <int D>
__device__ __forceinline__ void append_new_row_mx(const DecodeParams& p, const Item& it, int n_old, int64_t off_c, int token_pos) {
  if (!(n_old >= it.start && n_old < it.start + it.count)) return;  // uniform over the workgroup
  const int tid = threadIdx.x, value = tid / (D / 8), piece = tid % (D / 8);
  const int64_t row = off_c + n_old;
  if (value < 2)
    mx_store<D>(reinterpret_cast<const uint4*>(value ? p.v_new : p.k_new)[(int64_t)(it.c - p.cache_begin) * (D / 8) + piece], piece,
                value ? p.v : p.k, p.kv_scale, row, value);
  if (tid == 64 * kWaves - 1) {
    p.score[row] = 0.f;
    p.pos[row] = token_pos;
  }
  __syncthreads();
}

// One slab of a plane: tiles of 16 rows with the scale of each lane's elements.
template <int D>
struct Slab {
  Codes<Shape<D>::kWords> c[kTiles];
  uint32_t s[kTiles];
};

// plane, scale: this lane's place in the first row of the first tile of the work item
template <int D>
__device__ __forceinline__ void load_slab(Slab<D>& b, const unsigned char* plane, const uint8_t* scale, int t0, int row, int cnt) {
  if (t0 + kSlab <= cnt) {
#pragma unroll
    for (int T = 0; T < kTiles; ++T) {
      load_codes(b.c[T], plane + (uint32_t)t0 * Shape<D>::kBytes + T * 16 * Shape<D>::kBytes);
      b.s[T] = scale[(uint32_t)t0 * (D / 16) + T * 16 * (D / 16)];
    }
  } else {  // rows past the last one repeat it: they weigh nothing
#pragma unroll
    for (int T = 0; T < kTiles; ++T) {
      const int r = min(t0 + T * 16, cnt - 1 - row);
      load_codes(b.c[T], plane + r * Shape<D>::kBytes);
      b.s[T] = scale[r * (D / 16)];
    }
  }
}

// The weights of the recorded calls for rows [0, cnt) of a work item whose first row is row `start` of its cache: K alone is
// read, scores are read with it, and the new ones wait in LDS (this wavefront's `slots` slabs at `ring`), so that they are
// written together.
template <int D>
__device__ __forceinline__ void add_recorded(const DecodeParams& p, const Item& it, int cnt, int pending, float* ring, int slots) {
  using S = Shape<D>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n16 = lane & 15, jg = lane >> 4;
  Record<D> rec;
  load_record<D>(p, it.c, p.G, pending, n16, jg, rec);
  const unsigned char* Kb = reinterpret_cast<const unsigned char*>(p.k) + (it.row0 + n16) * S::kBytes + jg * (D / 8);
  const uint8_t* Sb = p.kv_scale + (it.row0 + n16) * (D / 16) + (D == 128 ? jg : jg / 2);
  float* const sc_base = p.score + it.row0;
  const float cs = p.scale_log2e;
  Slab<D> kr;
  float sc_cur = 0.f;
  int ring_n = 0, ring_t0 = 0;
  auto flush_ring = [&]() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    for (int i = lane; i < ring_n * kSlab; i += 64) {
      const int r = ring_t0 + i / kSlab * (kWaves * kSlab) + i % kSlab;
      if (r < cnt) sc_base[r] = ring[i];
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();  // the area may be written again
    ring_n = 0;
  };
  int t0 = wave * kSlab;
  if (t0 < cnt) {
    load_slab<D>(kr, Kb, Sb, t0, n16, cnt);
    if (lane < kSlab) sc_cur = sc_base[min(t0 + lane, cnt - 1)];
  }
  for (; t0 < cnt; t0 += kWaves * kSlab) {
    const int tn = t0 + kWaves * kSlab;
    floatx4_t sp[kSets][kTiles];
#pragma unroll
    for (int T = 0; T < kTiles; ++T) {
#pragma unroll
      for (int e = 0; e < kSets; ++e) sp[e][T] = floatx4_t{0.f, 0.f, 0.f, 0.f};
      const float scale = mx_scale(kr.s[T]);
#pragma unroll
      for (int c = 0; c < S::kChunks; ++c) {
        const bf16x8_t a = as_bf16x8(mx_values(kr.c[T].w[c], scale));
#pragma unroll
        for (int e = 0; e < kSets; ++e) sp[e][T] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(rec.q[e][c], a, sp[e][T], 0, 0, 0);
      }
    }
    const float sc_old = sc_cur;
    if (tn < cnt) {
      load_slab<D>(kr, Kb, Sb, tn, n16, cnt);
      if (lane < kSlab) sc_cur = sc_base[min(tn + lane, cnt - 1)];
    }
    const float wr = record_weights<D>(sp, rec, cs, it.start + t0, lane);
    if (ring_n == 0) ring_t0 = t0;
    if (lane < kSlab) ring[ring_n * kSlab + lane] = sc_old + wr;
    if (++ring_n == slots) flush_ring();
  }
  if (ring_n > 0) flush_ring();
}

template <int D, bool TRACK>
__global__ __launch_bounds__(64 * kWaves, 4) void decode_partial_mxfp4(DecodeParams p) {
  using S = Shape<D>;
  constexpr int kVStride = S::kVStride;
  __shared__ __attribute__((aligned(16))) unsigned char lds[kWaves * kSlab * kVStride];

  const Item it = p.items[blockIdx.x];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n16 = lane & 15, jg = lane >> 4;
  const int G = p.G;
  const int v_row = lane >> 2, v_piece = lane & 3;
  const unsigned char* Kb = reinterpret_cast<const unsigned char*>(p.k) + (it.row0 + n16) * S::kBytes + jg * (D / 8);
  const unsigned char* Vb = reinterpret_cast<const unsigned char*>(p.v) + (it.row0 + v_row) * S::kBytes + v_piece * (D / 8);
  const uint8_t* KSb = p.kv_scale + (it.row0 + n16) * (D / 16) + (D == 128 ? jg : jg / 2);
  const uint8_t* VSb = p.kv_scale + (it.row0 + v_row) * (D / 16) + D / 32 + (D == 128 ? v_piece : v_piece / 2);
  // The first slab is requested before the cache's length is known (its rows lie within the capacity); a slab that turns out
  // not to be made of old rows alone is requested again.
  Slab<D> kr, vr;
  int t0 = wave * kSlab;
  if (t0 + kSlab <= it.count) {
    load_slab<D>(kr, Kb, KSb, t0, n16, it.count);
    load_slab<D>(vr, Vb, VSb, t0, v_row, it.count);
  }
  const int n_old = p.len[it.c];
  const int64_t off_c = it.row0 - it.start;
  const int add = (p.fused_append && n_old < p.cap[it.c]) ? 1 : 0;
  const int n = n_old + add;
  const int token_pos = p.token_pos_dev ? *p.token_pos_dev : p.token_pos;
  const int pending = TRACK ? p.lag_cnt[(int64_t)it.c * G] : 0;
  if (p.fused_append) {
    if (add) append_new_row_mx<D>(p, it, n_old, off_c, token_pos);
    else if (it.start == 0 && threadIdx.x == 0) *p.status = 1;
  }
  int cnt = min(it.start + it.count, n) - it.start;
  if (cnt < 0) cnt = 0;
  unsigned char* myl = lds + wave * (kSlab * kVStride);
  // A full record: its weights are added first, by a pass over the K rows of their own, which the attention then finds in a
  // cache.  (In one pass the record's operands and results are live beside everything else: 216 registers instead of 128.)
  if (TRACK && pending >= p.lag_batch) add_recorded<D>(p, it, cnt, pending, reinterpret_cast<float*>(myl), kVStride / 4);

  const int64_t qrow0 = (int64_t)(it.c - p.cache_begin) * G;
  floatx4_t o[S::kBlocks];
#pragma unroll
  for (int b = 0; b < S::kBlocks; ++b) o[b] = floatx4_t{0.f, 0.f, 0.f, 0.f};
  float m_run = kLowest;  // running max of head n16, log2 units (see the bf16 kernel)
  float l_part = 0.f;
  const float cs = p.scale_log2e;
  if (t0 < cnt && t0 + kSlab > min(it.count, n_old - it.start)) {
    load_slab<D>(kr, Kb, KSb, t0, n16, cnt);
    load_slab<D>(vr, Vb, VSb, t0, v_row, cnt);
  }
  bf16x8_t qb[S::kChunks];  // B operand: lane (g, jg), chunk c holds Q[g][jg D / 4 + 8 c .. + 8]
#pragma unroll
  for (int c = 0; c < S::kChunks; ++c) {
    uint4 raw = make_uint4(0, 0, 0, 0);
    if (n16 < G)
      raw = *reinterpret_cast<const uint4*>(reinterpret_cast<const unsigned char*>(p.q) + (qrow0 + n16) * S::kQRow + jg * (D / 2) + c * 16);
    qb[c] = as_bf16x8(raw);
  }

  for (; t0 < cnt; t0 += kWaves * kSlab) {
    const int tn = t0 + kWaves * kSlab;
    // ---- S^T = K Q^T ---------------------------------------------------------------------------
    floatx4_t s[kTiles];
#pragma unroll
    for (int T = 0; T < kTiles; ++T) {
      s[T] = floatx4_t{0.f, 0.f, 0.f, 0.f};
      const float scale = mx_scale(kr.s[T]);
#pragma unroll
      for (int c = 0; c < S::kChunks; ++c)
        s[T] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(mx_values(kr.c[T].w[c], scale)), qb[c], s[T], 0, 0, 0);
    }
    if (tn < cnt) load_slab<D>(kr, Kb, KSb, tn, n16, cnt);

    // ---- V rows as bf16 in LDS -------------------------------------------------------------------
#pragma unroll
    for (int T = 0; T < kTiles; ++T) {
      const float scale = mx_scale(vr.s[T]);
#pragma unroll
      for (int c = 0; c < S::kWords; ++c)
        *reinterpret_cast<uint4*>(myl + (T * 16 + v_row) * kVStride + v_piece * (D / 2) + c * 16) = mx_values(vr.c[T].w[c], scale);
    }
    if (tn < cnt) load_slab<D>(vr, Vb, VSb, tn, v_row, cnt);

    // ---- online softmax on the accumulator layout ------------------------------------------------
    if (t0 + kSlab > cnt) {
#pragma unroll
      for (int T = 0; T < kTiles; ++T)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (t0 + T * 16 + jg * 4 + i >= cnt) s[T][i] = kNegInf;
    }
    float mx = s[0][0];
#pragma unroll
    for (int T = 0; T < kTiles; ++T)
#pragma unroll
      for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[T][i]);
    mx *= cs;
    if (__any(mx > m_run)) {
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float mn = fmaxf(m_run, mx);
      const float alpha = fast_exp2(m_run - mn);
      m_run = mn;
      l_part *= alpha;
#pragma unroll
      for (int b = 0; b < S::kBlocks; ++b) o[b] *= alpha;
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    // ---- O^T += V^T P^T, 32 rows at a time (transposed reads as in the bf16 kernel) ---------------
#pragma unroll
    for (int u = 0; u < kTiles / 2; ++u) {
      u32x4_t ph, pm;
      bf16x8_t pl;
#pragma unroll
      for (int e = 0; e < 8; e += 2) {  // three terms: 8 bits, the next 8, and the rest
        const float p0 = fast_exp2(fmaf(s[2 * u + e / 4][e % 4], cs, -m_run)), p1 = fast_exp2(fmaf(s[2 * u + e / 4][e % 4 + 1], cs, -m_run));
        l_part += p0 + p1;
        const uint32_t u0 = __float_as_uint(p0), u1 = __float_as_uint(p1);
        ph[e / 2] = (u0 >> 16) | (u1 & 0xffff0000u);
        const float r0 = p0 - __uint_as_float(u0 & 0xffff0000u), r1 = p1 - __uint_as_float(u1 & 0xffff0000u);
        const uint32_t w0 = __float_as_uint(r0), w1 = __float_as_uint(r1);
        pm[e / 2] = (w0 >> 16) | (w1 & 0xffff0000u);
        pl[e] = (__bf16)(r0 - __uint_as_float(w0 & 0xffff0000u));
        pl[e + 1] = (__bf16)(r1 - __uint_as_float(w1 & 0xffff0000u));
      }
      const unsigned char* tr0 = myl + (u * 32 + jg * 4 + (n16 >> 2)) * kVStride + (n16 & 3) * 8;
#pragma unroll
      for (int b = 0; b < S::kBlocks; ++b) {
        typedef __attribute__((address_space(3))) s16x4_t* lds_ptr_t;
        const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr_t)(tr0 + b * 32));
        const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr_t)(tr0 + 16 * kVStride + b * 32));
        const bf16x8_t a = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        o[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8_t, ph), o[b], 0, 0, 0);
        o[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8_t, pm), o[b], 0, 0, 0);
        o[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pl, o[b], 0, 0, 0);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }

  float l_tot = l_part;
  l_tot += __shfl_xor(l_tot, 16);
  l_tot += __shfl_xor(l_tot, 32);
  __syncthreads();
  float* sm_o = reinterpret_cast<float*>(lds);   // [kWaves][16][D]
  float* sm_m = sm_o + kWaves * 16 * D;          // [kWaves][16]
  float* sm_l = sm_m + kWaves * 16;              // [kWaves][16]
  static_assert((kWaves * 16 * D + 2 * kWaves * 16) * 4 <= kWaves * kSlab * kVStride, "LDS reuse");
  if (n16 < G) {
#pragma unroll
    for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) sm_o[(wave * 16 + n16) * D + b * 16 + jg * 4 + i] = o[b][i];
    if (jg == 0) {
      sm_m[wave * 16 + n16] = m_run;
      sm_l[wave * 16 + n16] = l_tot;
    }
  }
  __syncthreads();
  finish_item<D, 16, kWaves>(p, it, G, n, sm_o, sm_m, sm_l);
}

// The recorded calls' weights from the K rows alone (see score_flush_mfma, also for the tickets).
template <int D>
__global__ __launch_bounds__(64 * kWaves) void score_flush_mxfp4(DecodeParams p) {
  const Item it = p.items[blockIdx.x];
  const int G = p.G;
  const int pending = p.lag_cnt[(int64_t)it.c * G];
  if (pending == 0) return;
  auto clear_record = [&]() {
    if (!p.flush_ticket) return;
    __syncthreads();  // every wavefront has read the count
    if (threadIdx.x != 0) return;
    if (it.nsplit > 1) {
      int32_t* const ticket = p.flush_ticket + (int64_t)it.c * kTicketStride;
      if (__hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != it.nsplit - 1) return;
      __hip_atomic_store(ticket, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    for (int g = 0; g < G; ++g) p.lag_cnt[(int64_t)it.c * G + g] = 0;
  };
  int n_seen = 0;
  for (int s = 0; s < kLagCalls; ++s)
    if (s < pending) n_seen = max(n_seen, p.lag_n[(int64_t)it.c * kLagCalls + s]);
  const int cnt = min(it.start + it.count, n_seen) - it.start;
  if (cnt <= 0) {
    clear_record();
    return;
  }
  constexpr int kSlots = 64;
  __shared__ __attribute__((aligned(16))) float ring[kWaves * kSlots * kSlab];
  add_recorded<D>(p, it, cnt, pending, ring + (threadIdx.x >> 6) * (kSlots * kSlab), kSlots);
  clear_record();
}

}  // namespace

hipError_t launch_decode_mxfp4(const DecodeParams& p, int D, int n_items, hipStream_t s) {
  if (n_items <= 0) return hipSuccess;
  if (p.G > 16) return hipErrorInvalidValue;
  const dim3 grid(n_items), block(64 * kWaves);
  if (D == 128) {
    if (p.lag) decode_partial_mxfp4<128, true><<<grid, block, 0, s>>>(p);
    else decode_partial_mxfp4<128, false><<<grid, block, 0, s>>>(p);
  } else {
    if (p.lag) decode_partial_mxfp4<64, true><<<grid, block, 0, s>>>(p);
    else decode_partial_mxfp4<64, false><<<grid, block, 0, s>>>(p);
  }
  return hipGetLastError();
}

hipError_t launch_score_flush_mxfp4(const DecodeParams& p, int D, int n_items, hipStream_t s) {
  if (n_items <= 0) return hipSuccess;
  if (D == 128) score_flush_mxfp4<128><<<dim3(n_items), dim3(64 * kWaves), 0, s>>>(p);
  else score_flush_mxfp4<64><<<dim3(n_items), dim3(64 * kWaves), 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace baklava
