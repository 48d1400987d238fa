// Decode attention over ragged caches of 4-bit rows (BAKLAVA_MXFP4), up to 16 query heads per KV head.
//
// The two products of a slab of 32 rows are those of the bf16 kernel (v_mfma_f32_16x16x32_bf16):
//
//   S^T[row, g]  = K[row, :] . Q[g, :]          O^T[d, g] += V^T[d, rows] . P^T[rows, g]
//
// and so are the pipeline of a wavefront that streams its own slabs, the softmax on the accumulators' layout and the records
// of the calls whose weights are owed to the scores.  What differs is how rows become operands.  A lane loads D / 8 bytes of a
// K row, the D / 4 elements (jg D / 4 ...) of row n16 for lane (n16, jg), and the first product numbers the head dimension the
// same way (chunk c of lane group jg: elements jg D / 4 + 8 c .. + 8), so that codes become the A operand where they lie, two
// per conversion instruction, without a trip through LDS.  Values of codes are exact in bf16.  V has to be transposed: its
// codes are converted in the lane that loaded them, the bf16 rows go to LDS and are read back transposed.  Weights enter the
// second product as three bf16 terms, which is all of their 24 bits.
#include "common.h"
#include "decode_tail.h"
#include "mxfp4.h"

#include <algorithm>
#include <type_traits>

namespace baklava {

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float floatx4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

constexpr int kSlab = 32;   // rows per wavefront iteration, two tiles of 16
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
  static constexpr int kStatic = kWaves * kSlab * kVStride;
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

// Weights of the recorded calls for the 32 rows of a slab; on return lane l < 32 holds that of row l.
template <int D>
__device__ __forceinline__ float record_weights(const floatx4_t (&sp)[kSets][2], const Record<D>& r, float cs, int row_first,
                                                int lane) {
  const int n16 = lane & 15;
  float w[2];
#pragma unroll
  for (int T = 0; T < 2; ++T) {
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
  return (lane & 16) ? w[1] : w[0];
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

// One slab of a plane: two tiles of 16 rows with the scale of each lane's elements.
template <int D>
struct Slab {
  Codes<Shape<D>::kWords> c[2];
  uint32_t s[2];
};

template <int D>
__device__ __forceinline__ void load_slab(Slab<D>& b, const unsigned char* plane, const uint8_t* scale, int t0, int row, int piece,
                                          int last) {
#pragma unroll
  for (int T = 0; T < 2; ++T) {
    const uint32_t r = (uint32_t)min(t0 + T * 16 + row, last);
    load_codes(b.c[T], plane + r * (uint32_t)Shape<D>::kBytes + piece * (D / 8));
    b.s[T] = scale[r * (uint32_t)(D / 16) + (D == 128 ? piece : piece / 2)];
  }
}

template <int D, bool TRACK>
__global__ __launch_bounds__(64 * kWaves, 2) void decode_partial_mxfp4(DecodeParams p) {
  using S = Shape<D>;
  constexpr int kVStride = S::kVStride;
  __shared__ __attribute__((aligned(16))) unsigned char lds[kWaves * kSlab * kVStride];
  extern __shared__ __attribute__((aligned(16))) float lds_ring[];  // new scores that wait ([32] per slab and wavefront)

  const Item it = p.items[blockIdx.x];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n16 = lane & 15, jg = lane >> 4;
  const int G = p.G;
  const int n_old = p.len[it.c];
  const int64_t off_c = it.row0 - it.start;
  const int add = (p.fused_append && n_old < p.cap[it.c]) ? 1 : 0;
  const int n = n_old + add;
  const int token_pos = p.token_pos_dev ? *p.token_pos_dev : p.token_pos;
  const int pending = TRACK ? p.lag_cnt[(int64_t)it.c * G] : 0;
  const bool apply = TRACK && pending >= p.lag_batch;
  Record<D> rec;
  if (TRACK && apply) load_record<D>(p, it.c, G, pending, n16, jg, rec);
  if (p.fused_append) {
    if (add) append_new_row_mx<D>(p, it, n_old, off_c, token_pos);
    else if (it.start == 0 && threadIdx.x == 0) *p.status = 1;
  }
  int cnt = min(it.start + it.count, n) - it.start;
  if (cnt < 0) cnt = 0;
  const int64_t row0 = it.row0;
  const unsigned char* Kb = reinterpret_cast<const unsigned char*>(p.k) + row0 * S::kBytes;
  const unsigned char* Vb = reinterpret_cast<const unsigned char*>(p.v) + row0 * S::kBytes;
  const uint8_t* Sb = p.kv_scale + row0 * (D / 16);
  unsigned char* myl = lds + wave * (kSlab * kVStride);
  const int64_t qrow0 = (int64_t)(it.c - p.cache_begin) * G;

  floatx4_t o[S::kBlocks];
#pragma unroll
  for (int b = 0; b < S::kBlocks; ++b) o[b] = floatx4_t{0.f, 0.f, 0.f, 0.f};
  float m_run = kLowest;  // running max of head n16, log2 units (see the bf16 kernel)
  float l_part = 0.f;
  const float cs = p.scale_log2e;
  const int last = cnt - 1;  // rows past it repeat it and weigh nothing
  const int v_row = lane >> 2, v_piece = lane & 3;
  Slab<D> kr, vr;

  float* const sc_base = p.score + row0;
  float sc_cur = 0.f;
  float* const ring = lds_ring + wave * p.ring_slots * kSlab;
  int ring_n = 0, ring_t0 = 0;
  auto flush_ring = [&]() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    for (int sidx = lane >> 5; sidx < ring_n; sidx += 2) {
      const int r = ring_t0 + sidx * (kWaves * kSlab) + (lane & 31);
      if (r < cnt) sc_base[r] = ring[sidx * kSlab + (lane & 31)];
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    ring_n = 0;
  };

  auto stream_rows = [&](auto apply_tag) {
  constexpr bool APPLY = decltype(apply_tag)::value;
  int t0 = wave * kSlab;
  if (t0 < cnt) {
    load_slab<D>(kr, Kb, Sb, t0, n16, jg, last);
    if (APPLY && lane < kSlab) sc_cur = sc_base[min(t0 + lane, last)];
  }
  bf16x8_t qb[S::kChunks];  // B operand: lane (g, jg), chunk c holds Q[g][jg D / 4 + 8 c .. + 8]
#pragma unroll
  for (int c = 0; c < S::kChunks; ++c) {
    uint4 raw = make_uint4(0, 0, 0, 0);
    if (n16 < G)
      raw = *reinterpret_cast<const uint4*>(reinterpret_cast<const unsigned char*>(p.q) + (qrow0 + n16) * S::kQRow + jg * (D / 2) + c * 16);
    qb[c] = as_bf16x8(raw);
  }
  if (t0 < cnt) load_slab<D>(vr, Vb, Sb + D / 32, t0, v_row, v_piece, last);

  for (; t0 < cnt; t0 += kWaves * kSlab) {
    const int tn = t0 + kWaves * kSlab;
    // ---- S^T = K Q^T ---------------------------------------------------------------------------
    floatx4_t s[2], sp[kSets][2];
#pragma unroll
    for (int T = 0; T < 2; ++T) {
      s[T] = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < kSets; ++e) sp[e][T] = floatx4_t{0.f, 0.f, 0.f, 0.f};
      const float scale = mx_scale(kr.s[T]);
#pragma unroll
      for (int c = 0; c < S::kChunks; ++c) {
        const bf16x8_t a = as_bf16x8(mx_values(kr.c[T].w[c], scale));
        s[T] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qb[c], s[T], 0, 0, 0);
        if (APPLY) {
#pragma unroll
          for (int e = 0; e < kSets; ++e) sp[e][T] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(rec.q[e][c], a, sp[e][T], 0, 0, 0);
        }
      }
    }
    load_slab<D>(kr, Kb, Sb, tn, n16, jg, last);  // past the end every row clamps to the last live row: harmless re-reads
    const float sc_old = sc_cur;
    if (APPLY && lane < kSlab) sc_cur = sc_base[min(tn + lane, last)];

    // ---- V rows as bf16 in LDS -------------------------------------------------------------------
#pragma unroll
    for (int T = 0; T < 2; ++T) {
      const float scale = mx_scale(vr.s[T]);
#pragma unroll
      for (int c = 0; c < S::kWords; ++c)
        *reinterpret_cast<uint4*>(myl + (T * 16 + v_row) * kVStride + v_piece * (D / 2) + c * 16) = mx_values(vr.c[T].w[c], scale);
    }
    load_slab<D>(vr, Vb, Sb + D / 32, tn, v_row, v_piece, last);

    // ---- online softmax on the accumulator layout ------------------------------------------------
    float x[8];
#pragma unroll
    for (int T = 0; T < 2; ++T)
#pragma unroll
      for (int i = 0; i < 4; ++i) x[T * 4 + i] = s[T][i] * cs;
    if (t0 + kSlab > cnt) {
#pragma unroll
      for (int T = 0; T < 2; ++T)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (t0 + T * 16 + jg * 4 + i >= cnt) x[T * 4 + i] = kNegInf;
    }
    if (APPLY) {
      const float wr = record_weights<D>(sp, rec, cs, it.start + t0, lane);
      if (ring_n == 0) ring_t0 = t0;
      if (lane < kSlab) ring[ring_n * kSlab + lane] = sc_old + wr;
      if (++ring_n == p.ring_slots) flush_ring();
    }
    float mx = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) mx = fmaxf(mx, x[e]);
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
    u32x4_t ph, pm;
    bf16x8_t pl;
#pragma unroll
    for (int e = 0; e < 8; e += 2) {  // three terms: 8 bits, the next 8, and the rest
      const float p0 = fast_exp2(x[e] - m_run), p1 = fast_exp2(x[e + 1] - m_run);
      l_part += p0 + p1;
      const uint32_t u0 = __float_as_uint(p0), u1 = __float_as_uint(p1);
      ph[e / 2] = (u0 >> 16) | (u1 & 0xffff0000u);
      const float r0 = p0 - __uint_as_float(u0 & 0xffff0000u), r1 = p1 - __uint_as_float(u1 & 0xffff0000u);
      const uint32_t w0 = __float_as_uint(r0), w1 = __float_as_uint(r1);
      pm[e / 2] = (w0 >> 16) | (w1 & 0xffff0000u);
      pl[e] = (__bf16)(r0 - __uint_as_float(w0 & 0xffff0000u));
      pl[e + 1] = (__bf16)(r1 - __uint_as_float(w1 & 0xffff0000u));
    }

    // ---- O^T += V^T P^T (transposed reads as in the bf16 kernel) ---------------------------------
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    const unsigned char* tr0 = myl + (jg * 4 + (n16 >> 2)) * kVStride + (n16 & 3) * 8;
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
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  if (APPLY && ring_n > 0) flush_ring();
  };  // stream_rows
  if (TRACK && apply) stream_rows(std::integral_constant<bool, TRACK>{});
  else stream_rows(std::false_type{});

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
  using S = Shape<D>;
  extern __shared__ __attribute__((aligned(16))) float lds_ring[];
  const Item it = p.items[blockIdx.x];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n16 = lane & 15, jg = lane >> 4;
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
  Record<D> rec;
  load_record<D>(p, it.c, G, pending, n16, jg, rec);
  const int last = cnt - 1;
  const unsigned char* Kb = reinterpret_cast<const unsigned char*>(p.k) + it.row0 * S::kBytes;
  const uint8_t* Sb = p.kv_scale + it.row0 * (D / 16);
  float* const sc_base = p.score + it.row0;
  float* const ring = lds_ring + wave * p.ring_slots * kSlab;
  const float cs = p.scale_log2e;
  Slab<D> kr;
  float sc_cur = 0.f;
  int ring_n = 0, ring_t0 = 0;
  auto flush_ring = [&]() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    for (int sidx = lane >> 5; sidx < ring_n; sidx += 2) {
      const int r = ring_t0 + sidx * (kWaves * kSlab) + (lane & 31);
      if (r < cnt) sc_base[r] = ring[sidx * kSlab + (lane & 31)];
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    ring_n = 0;
  };
  int t0 = wave * kSlab;
  if (t0 < cnt) {
    load_slab<D>(kr, Kb, Sb, t0, n16, jg, last);
    if (lane < kSlab) sc_cur = sc_base[min(t0 + lane, last)];
  }
  for (; t0 < cnt; t0 += kWaves * kSlab) {
    const int tn = t0 + kWaves * kSlab;
    floatx4_t sp[kSets][2];
#pragma unroll
    for (int T = 0; T < 2; ++T) {
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
    load_slab<D>(kr, Kb, Sb, tn, n16, jg, last);
    if (lane < kSlab) sc_cur = sc_base[min(tn + lane, last)];
    const float wr = record_weights<D>(sp, rec, cs, it.start + t0, lane);
    if (ring_n == 0) ring_t0 = t0;
    if (lane < kSlab) ring[ring_n * kSlab + lane] = sc_old + wr;
    if (++ring_n == p.ring_slots) flush_ring();
  }
  if (ring_n > 0) flush_ring();
  clear_record();
}

constexpr int kLdsTotal = 160 * 1024;
template <int D> constexpr int dyn_alone() { return kLdsTotal - Shape<D>::kStatic - 512; }           // beside no other workgroup
template <int D> constexpr int dyn_shared() { return (kLdsTotal - 2 * Shape<D>::kStatic - 1024) / 2; }
constexpr int kFlushDyn = 48 * 1024;
static_assert(dyn_shared<128>() >= kWaves * kSlab * 4, "room for one slab of scores per wavefront");

int ring_slots(int bytes, int max_count) {
  const int need = ((max_count + kSlab - 1) / kSlab + kWaves - 1) / kWaves;
  return std::max(1, std::min(bytes / (kWaves * kSlab * 4), need));
}

template <int D>
hipError_t launch_d(DecodeParams p, int n_items, int max_count, bool one_wave, hipStream_t s) {
  const dim3 grid(n_items), block(64 * kWaves);
  p.ring_slots = 0;
  if (!p.lag) {
    decode_partial_mxfp4<D, false><<<grid, block, 0, s>>>(p);
    return hipGetLastError();
  }
  p.ring_slots = ring_slots(one_wave ? dyn_alone<D>() : dyn_shared<D>(), max_count);
  decode_partial_mxfp4<D, true><<<grid, block, (size_t)p.ring_slots * kWaves * kSlab * 4, s>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t prepare_decode_mxfp4() {
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(decode_partial_mxfp4<128, true>),
                                     hipFuncAttributeMaxDynamicSharedMemorySize, dyn_alone<128>());
  if (e != hipSuccess) return e;
  e = hipFuncSetAttribute(reinterpret_cast<const void*>(decode_partial_mxfp4<64, true>),
                          hipFuncAttributeMaxDynamicSharedMemorySize, dyn_alone<64>());
  if (e != hipSuccess) return e;
  e = hipFuncSetAttribute(reinterpret_cast<const void*>(score_flush_mxfp4<128>), hipFuncAttributeMaxDynamicSharedMemorySize, kFlushDyn);
  if (e != hipSuccess) return e;
  return hipFuncSetAttribute(reinterpret_cast<const void*>(score_flush_mxfp4<64>), hipFuncAttributeMaxDynamicSharedMemorySize, kFlushDyn);
}

hipError_t launch_decode_mxfp4(const DecodeParams& p, int D, int n_items, int max_count, bool one_wave, hipStream_t s) {
  if (n_items <= 0) return hipSuccess;
  if (p.G > 16) return hipErrorInvalidValue;
  return D == 128 ? launch_d<128>(p, n_items, max_count, one_wave, s) : launch_d<64>(p, n_items, max_count, one_wave, s);
}

hipError_t launch_score_flush_mxfp4(const DecodeParams& p_in, int D, int n_items, int max_count, hipStream_t s) {
  if (n_items <= 0) return hipSuccess;
  DecodeParams p = p_in;
  p.ring_slots = ring_slots(kFlushDyn, max_count);
  const size_t dyn = (size_t)p.ring_slots * kWaves * kSlab * 4;
  if (D == 128) score_flush_mxfp4<128><<<dim3(n_items), dim3(64 * kWaves), dyn, s>>>(p);
  else score_flush_mxfp4<64><<<dim3(n_items), dim3(64 * kWaves), dyn, s>>>(p);
  return hipGetLastError();
}

}  // namespace baklava
