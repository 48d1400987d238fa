// Causal attention over whole prompts of different lengths with grouped heads (baklava_prompt_attn).
//
// A dense contraction (4 D flops per query head and visible pair), on the matrix cores as v_mfma_f32_32x32x16_bf16:
//
//   S^T[key, token]  = K[key, :] . Q[token, :]          A = K rows from LDS, B = Q (registers)
//   O^T[d, token]   += V^T[d, keys] . P^T[keys, token]   A = V^T (LDS, transposed read), B = P^T
//
// The accumulator of S^T (lane (token, h), register i: key 8 (i / 4) + 4 h + i % 4) is already a valid B operand of the second
// product once the 16 keys of an instruction are numbered the way the lane holds them, so the softmax weights never leave
// their lane; V^T is read from LDS with the same numbering.  One pass over the keys with the running maximum and sum of
// every token in fp32.  The weights enter the second product as one bf16 term, rounded to the nearest: that is as much as
// the rounding of the output to bf16 loses (a second term would be exact to 2^-17, at half as many products again).
//
// A workgroup of 4 wavefronts owns 128 consecutive tokens of one head, 32 per wavefront.  Keys and values go from memory to
// LDS without a stop in registers, in tiles of 64 rows, double-buffered.  The tiles that all of its tokens see form a software
// pipeline: the first product of tile n + 1 runs beside the exponentials of tile n.  The others follow, masked.
#include "common.h"

namespace baklava {

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float floatx16_t __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;
constexpr int kKeyTile = 64;        // rows per LDS stage, two slabs of 32
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLowest = -3.402823466e38f;
constexpr float kMaxSlack = 8.f;    // a logit may exceed its token's reference maximum by this much

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ bf16x8_t as_bf16x8(u32x4_t x) { return __builtin_bit_cast(bf16x8_t, x); }

// N: groups of 32 tokens per wavefront.
template <int D, int N>
__global__ __launch_bounds__(64 * kWaves, N == 1 ? 2 : 1) void prompt_attn_kernel(PromptParams p) {
  constexpr int kTokPerWave = 32 * N, kTokPerWg = kWaves * kTokPerWave;
  constexpr int kRow = D * 2;             // bytes of a row
  constexpr int kPieces = D / 8;          // 16-byte pieces of a row
  constexpr int kChunks = D / 16;         // head-dim steps of the first product
  constexpr int kBlocks = D / 32;         // 32-element blocks of the second product's result
  constexpr int kCopyRows = 64 / kPieces; // rows per copy instruction
  constexpr int kCopies = kKeyTile / kWaves / kCopyRows;
  __shared__ __attribute__((aligned(16))) unsigned char lds_k[2][kKeyTile * kRow];
  __shared__ __attribute__((aligned(16))) unsigned char lds_v[2][kKeyTile * kRow];

  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n32 = lane & 31, jh = lane >> 5;
  // Query heads that share a KV head meet on the same XCDs (consecutive workgroups go round them) while the number of KV
  // heads allows it.
  const int G = p.Hq / p.Hkv;
  const int kv_head = blockIdx.x % p.Hkv, rest = blockIdx.x / p.Hkv;
  const int head = kv_head * G + rest % G, rank = rest / G;
  int at = 0;  // the sequence of this tile: as many end in front of it
  for (int i0 = 0; i0 < p.n_seq; i0 += 64)
    at += __popcll(__ballot(i0 + lane < p.n_seq && p.seq[i0 + lane < p.n_seq ? i0 + lane : 0].tile_end <= rank));
  at = __builtin_amdgcn_readfirstlane(at);
  const PromptParams::Seq sq = p.seq[at];
  const int n_q = sq.q_len, n_k = sq.k_len;
  const int tile = sq.tile_end - 1 - rank;  // the last tokens, which see most keys, first

  const unsigned char* Qb = reinterpret_cast<const unsigned char*>(p.q.data) + p.q.begin(sq.b, sq.q_first) + head * p.q.head;
  const unsigned char* Kb = reinterpret_cast<const unsigned char*>(p.k.data) + p.k.begin(sq.b, sq.k_first) + kv_head * p.k.head;
  const unsigned char* Vb = reinterpret_cast<const unsigned char*>(p.v.data) + p.v.begin(sq.b, sq.k_first) + kv_head * p.v.head;
  const int64_t out0 = p.out.begin(sq.b, sq.q_first) + head * p.out.head;
  const int64_t lse0 = p.lse.begin(sq.b, sq.q_first) + head * p.lse.head;

  const int q0 = tile * kTokPerWg;          // first token of the workgroup
  const int qw0 = q0 + wave * kTokPerWave;  // first token of this wavefront
  const int before = n_k - n_q;             // keys in front of the first token's own (less than 0: tokens that see none)
  const int last_key = before + min(q0 + kTokPerWg, n_q) - 1;
  const int n_key_tiles = last_key < 0 ? 0 : last_key / kKeyTile + 1;
  // tiles without a masked pair, an even number; at least one follows
  const int n_full = min(max(0, before + q0 + 1) / kKeyTile, max(0, n_key_tiles - 1)) & ~1;

  // Staging: a wavefront copies 16 rows of each plane per tile, 1 KiB of LDS, in lane order, per instruction.  The 16-byte
  // pieces of a row are permuted on the way, so that the operand reads spread over the banks.  Rows past the last key
  // repeat it; they are masked.
  uint32_t k_off[kCopies], v_off[kCopies], k_row[kCopies];
#pragma unroll
  for (int i = 0; i < kCopies; ++i) {
    const int row = wave * (kKeyTile / kWaves) + i * kCopyRows + lane / kPieces, slot = lane % kPieces;
    k_row[i] = row;
    k_off[i] = (D == 128 ? slot ^ (row & 15) : slot ^ (row >> 1 & 7)) * 16;
    v_off[i] = (D == 128 ? slot ^ 4 * (row & 3) : slot ^ 4 * (row >> 1 & 1)) * 16;
  }
  const uint32_t lds_k0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds_k + wave * (kKeyTile / kWaves) * kRow;
  const uint32_t lds_v0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds_v + wave * (kKeyTile / kWaves) * kRow;
  auto copy_rows = [&](uint32_t dst, const unsigned char* plane, int64_t stride, int kt, const uint32_t (&off)[kCopies]) {
    const unsigned char* src = plane + kt * (kKeyTile * stride);
    const uint32_t most = n_k - 1 - kt * kKeyTile;
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const uint32_t o = min(k_row[i], most) * (uint32_t)stride + off[i];
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                   :: "s"(dst + i * 1024), "v"(o), "s"(src) : "memory", "m0");
    }
  };
  auto stage_k = [&](int kt) { copy_rows(lds_k0 + (kt & 1) * (kKeyTile * kRow), Kb, p.k.tok, kt, k_off); };
  auto stage_v = [&](int kt) { copy_rows(lds_v0 + (kt & 1) * (kKeyTile * kRow), Vb, p.v.tok, kt, v_off); };
  auto publish = [&]() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  };

  // B operand of the first product: lane (token, h), chunk c holds Q[token][16c + 8h .. +8).
  int tok[N];
  bf16x8_t qb[N][kChunks];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    tok[n] = qw0 + 32 * n + n32;
    const int row = min(tok[n], n_q - 1);  // tokens past the sequence repeat the last one and are never written
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
      qb[n][c] = as_bf16x8(*reinterpret_cast<const u32x4_t*>(Qb + row * p.q.tok + c * 32 + jh * 16));
  }

  // Second product for a slab that some tokens do not see in part, value by value: a weight of zero times an infinite or NaN
  // value is left out.
  auto outputs_seen = [&](floatx16_t (&o)[kBlocks], int kt, int sl, const bf16x8_t (&pb)[2], int most) {
    for (int j = 0; j < 32; ++j) {
      float w = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (8 * (i / 4) + i % 4 == (j & ~4)) w = (float)pb[i / 8][i % 8];
      w = __shfl(w, n32 + 8 * (j & 4));  // from the half that holds key j
      if (kt * kKeyTile + sl * 32 + j > most) continue;
      const int row = sl * 32 + j;
      const unsigned char* src = lds_v[kt & 1] + row * kRow;
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int piece = 4 * b + q;
          const uint2 raw = *reinterpret_cast<const uint2*>(src + (D == 128 ? piece ^ 4 * (row & 3) : piece ^ 4 * (row >> 1 & 1)) * 16 + jh * 8);
          o[b][4 * q] = fmaf(w, __uint_as_float(raw.x << 16), o[b][4 * q]);
          o[b][4 * q + 1] = fmaf(w, __uint_as_float(raw.x & 0xffff0000u), o[b][4 * q + 1]);
          o[b][4 * q + 2] = fmaf(w, __uint_as_float(raw.y << 16), o[b][4 * q + 2]);
          o[b][4 * q + 3] = fmaf(w, __uint_as_float(raw.y & 0xffff0000u), o[b][4 * q + 3]);
        }
    }
  };

  floatx16_t o[N][kBlocks];  // lane (token, h), register i of block b: O[token][32 b + 8 (i / 4) + 4 h + i % 4]
  // Reference maximum of the exponent, log2 units.  It starts at the lowest finite value, so that a masked logit weighs
  // 2^-inf = 0 and not 2^(-inf + inf), also where nothing has been visible yet.
  float m_ref[N];
  float l_part[N];           // this lane's share of the running sum
  const float cs = p.scale_log2e;

  auto logits = [&](floatx16_t (&s)[N][2], int kt) {
    const unsigned char* base = lds_k[kt & 1] + n32 * kRow;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      const int piece = 2 * c + jh, slot = (D == 128 ? piece ^ (n32 & 15) : piece ^ (n32 >> 1 & 7)) * 16;
#pragma unroll
      for (int sl = 0; sl < 2; ++sl) {
        const u32x4_t a = *reinterpret_cast<const u32x4_t*>(base + sl * 32 * kRow + slot);
        const floatx16_t zero = {};
#pragma unroll
        for (int n = 0; n < N; ++n)
          s[n][sl] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(a), qb[n][c], c == 0 ? zero : s[n][sl], 0, 0, 0);
      }
    }
  };
  auto max_of = [&](const floatx16_t (&s)[2]) {
    float mx = s[0][0];
#pragma unroll
    for (int sl = 0; sl < 2; ++sl)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[sl][i]);
    return mx * cs;
  };
  // Lazy running maximum: a token's reference only moves when a logit exceeds it by more than kMaxSlack (log2 units), so
  // weights stay below 2^kMaxSlack and the rescale of the accumulators is rare after the first tile.
  auto follow_max = [&](int n, float mx) {
    if (__any(mx > m_ref[n] + kMaxSlack)) {
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float mn = fmaxf(m_ref[n], mx);
      const float alpha = fast_exp2(m_ref[n] - mn);
      m_ref[n] = mn;
      l_part[n] *= alpha;
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) o[n][b] *= alpha;
    }
  };
  // Weights of a slab of 32 keys as B operands, 16 keys each.
  auto weights = [&](int n, const floatx16_t& s, bf16x8_t (&pb)[2]) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float w = fast_exp2(fmaf(s[8 * u + e], cs, -m_ref[n]));
        l_part[n] += w;
        pb[u][e] = (__bf16)w;
      }
  };
  // Second product for a slab.  A transposed read hands lane m of a 16-lane group element m of the 16 d values the group points
  // at, for 4 consecutive keys: the group (h, d half) reads keys 4 h .. + 3 of each 8, two reads per 16 keys.
  auto outputs = [&](int kt, int sl, const bf16x8_t (&pb)[N][2]) {
    const int n16 = lane & 15, half = (lane >> 4) & 1, k4 = n16 >> 2;
    const unsigned char* row = lds_v[kt & 1] + (sl * 32 + 4 * jh + k4) * kRow + half * 32 + (n16 & 3) * 8;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        typedef __attribute__((address_space(3))) s16x4_t* lds_ptr_t;
        const unsigned char* at = row + u * 16 * kRow + (D == 128 ? b ^ k4 : b ^ (k4 >> 1)) * 64;
        const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr_t)at);
        const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr_t)(at + 8 * kRow));
        const bf16x8_t a = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int n = 0; n < N; ++n) o[n][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pb[n][u], o[n][b], 0, 0, 0);
      }
  };

  auto clear = [&]() {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      m_ref[n] = kLowest;
      l_part[n] = 0.f;
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[n][b][i] = 0.f;
    }
  };
  auto mask = [&](floatx16_t (&s)[2], int n, int kt) {
#pragma unroll
    for (int sl = 0; sl < 2; ++sl)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (kt * kKeyTile + sl * 32 + 8 * (i / 4) + 4 * jh + i % 4 > before + tok[n]) s[sl][i] = kNegInf;
  };

  clear();
  if (n_key_tiles > 0) {
    stage_k(0);
    stage_v(0);
    if (n_key_tiles > 1) stage_k(1);
    publish();
    floatx16_t s[N][2];
    float mx[N];
    logits(s, 0);
#pragma unroll
    for (int n = 0; n < N; ++n) mx[n] = max_of(s[n]);
    __syncthreads();  // tile 0's K rows are overwritten by tile 2's in the first step
    bf16x8_t pb[2][N][2];
    // One pipeline step: tile kt from its logits in `s`, the next tile's logits into `sn`.
    auto step = [&](const floatx16_t (&s)[N][2], floatx16_t (&sn)[N][2], int kt) {
      if (kt + 2 < n_key_tiles) stage_k(kt + 2);
      stage_v(kt + 1);
#pragma unroll
      for (int n = 0; n < N; ++n) follow_max(n, mx[n]);
      logits(sn, kt + 1);
#pragma unroll
      for (int sl = 0; sl < 2; ++sl) {
#pragma unroll
        for (int n = 0; n < N; ++n) weights(n, s[n][sl], pb[sl][n]);
        outputs(kt, sl, pb[sl]);
      }
#pragma unroll
      for (int n = 0; n < N; ++n) mx[n] = max_of(sn[n]);
      publish();
    };
    int kt = 0;
    for (; kt < n_full; kt += 2) {
      floatx16_t sn[N][2];
      step(s, sn, kt);
      step(sn, s, kt + 1);
    }
    for (; kt < n_key_tiles; ++kt) {
      const int kt0 = kt * kKeyTile;
      // (K of tile kt + 1 was staged by the step before, or in front of the loop; that of kt + 2 is not on its way yet)
      if (kt + 1 < n_key_tiles) stage_v(kt + 1);
      if (kt + 2 < n_key_tiles) stage_k(kt + 2);
      if (kt0 <= before + qw0 + kTokPerWave - 1) {  // else wholly behind what this wavefront's tokens see
#pragma unroll
        for (int n = 0; n < N; ++n) {
          mask(s[n], n, kt);
          follow_max(n, max_of(s[n]));
        }
#pragma unroll
        for (int sl = 0; sl < 2; ++sl) {
#pragma unroll
          for (int n = 0; n < N; ++n) weights(n, s[n][sl], pb[sl][n]);
          outputs(kt, sl, pb[sl]);
        }
        if (kt + 1 < n_key_tiles) logits(s, kt + 1);
      }
      publish();
    }
  }
  float sum = 0.f;  // not finite where one of them is not
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) sum = fmaf(o[n][b][i], 0.f, sum);
  if (__syncthreads_or(sum != 0.f)) {
    // An infinite or NaN value that some of a tile's tokens do not see may have reached them, through the product of a zero
    // weight with it: all again, step by step, with the tiles that are masked in part value by value.
    clear();
    for (int kt = 0; kt < n_key_tiles; ++kt) {
      stage_k(kt);
      stage_v(kt);
      publish();
      floatx16_t s[N][2];
      logits(s, kt);
#pragma unroll
      for (int n = 0; n < N; ++n) {
        mask(s[n], n, kt);
        follow_max(n, max_of(s[n]));
      }
#pragma unroll
      for (int sl = 0; sl < 2; ++sl) {
        bf16x8_t pb[N][2];
#pragma unroll
        for (int n = 0; n < N; ++n) weights(n, s[n][sl], pb[n]);
        if ((kt + 1) * kKeyTile <= before + q0 + 1) {
          outputs(kt, sl, pb);
        } else {
#pragma unroll
          for (int n = 0; n < N; ++n) outputs_seen(o[n], kt, sl, pb[n], before + tok[n]);
        }
      }
      __syncthreads();
    }
  }

#pragma unroll
  for (int n = 0; n < N; ++n) {
    const float l_tot = l_part[n] + __shfl_xor(l_part[n], 32);
    const bool none = before + tok[n] < 0;  // sees no key
    const float inv = none ? 0.f : 1.f / l_tot;
    if (tok[n] >= n_q) continue;
    unsigned char* dst = reinterpret_cast<unsigned char*>(p.out.data) + out0 + tok[n] * p.out.tok;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
        bf16x4_t r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = (__bf16)(o[n][b][4 * q + i] * inv);
        *reinterpret_cast<bf16x4_t*>(dst + (b * 32 + q * 8 + jh * 4) * 2) = r;
      }
    if (p.lse.data && jh == 0)
      *reinterpret_cast<float*>(reinterpret_cast<unsigned char*>(p.lse.data) + lse0 + tok[n] * p.lse.tok) =
          none ? kNegInf : m_ref[n] + __builtin_log2f(l_tot);
  }
}

}  // namespace

constexpr int kN = 1;
int prompt_tile_tokens() { return 32 * kN * kWaves; }

hipError_t launch_prompt_attn(const PromptParams& p, int D, int n_tiles, hipStream_t s) {
  const int64_t grid = (int64_t)n_tiles * p.Hq;
  if (grid <= 0) return hipSuccess;
  if (grid > INT32_MAX / (64 * kWaves)) return hipErrorInvalidValue;
  if (D == 128) prompt_attn_kernel<128, kN><<<dim3((unsigned)grid), dim3(64 * kWaves), 0, s>>>(p);
  else prompt_attn_kernel<64, kN><<<dim3((unsigned)grid), dim3(64 * kWaves), 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace baklava
