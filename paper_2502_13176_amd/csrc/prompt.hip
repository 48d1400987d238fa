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
// pipeline: the first product of tile n + 1 runs beside the exponentials of tile n.  The others follow, masked.  Small launches
// take workgroups of 64 tokens, two wavefronts to 32 tokens, each with one half of every tile of keys; their sums are added at
// the end (rule and figures at prompt_tile_tokens).  Outputs that are not finite are computed a second time, by a loop of its own
// at the end: in the main loop the test alone cost registers that went to scratch memory (8 prompts of 4096, 28 heads, 1229 / 1005
// us).
//
// One prompt of 16384, 32 heads of 128: 1.97 to 2.05 ms by the box, 1.07 to 1.12 PFLOP/s, where a product of two matrices of
// 16384^2 reaches 1.28 to 1.30.  The power of the products bounds it: the matrix cores are busy 63% of the time at some 1.6 GHz,
// and orders of instructions or waves' priorities make no difference.  (64 tokens per wavefront, one wavefront per SIMD, whose
// operands from LDS serve twice as many products: 728 TFLOP/s, nothing runs beside a wavefront's exponentials.)  Heads of 64: 0.94
// to 0.97 PFLOP/s (1.14 to 1.17 ms), bound by the vector ALUs, whose exponentials stand beside half the products.  8 prompts of 128
// to 8192 tokens, 28 heads, 2.35 ms.
#include "common.h"

namespace baklava {

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float floatx16_t __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x8_t __attribute__((ext_vector_type(8)));

constexpr int kWaves = 4;
constexpr int kKeyTile = 64;        // rows per LDS stage, two slabs of 32
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLowest = -3.402823466e38f;
constexpr float kMaxSlack = 8.f;    // a logit may exceed its token's reference maximum by this much

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ bf16x8_t as_bf16x8(u32x4_t x) { return __builtin_bit_cast(bf16x8_t, x); }

// KS: wavefronts that share 32 tokens.  1: each takes both slabs of a tile of keys; 2: each takes one of them, and the two add up
// what they have at the end.
template <int D, int KS>
__global__ __launch_bounds__(64 * kWaves, 2) void prompt_attn_kernel(PromptParams p) {
  constexpr int kTokPerWg = 32 * kWaves / KS, kSlabs = 2 / KS;
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
  int idx = blockIdx.x;
  if (idx >= p.reversed_from) idx = p.reversed_from + (int)gridDim.x - 1 - idx;
  const int kv_head = idx % p.Hkv, rest = idx / p.Hkv;
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
  const int qw0 = q0 + wave / KS * 32;      // first token of this wavefront
  const int sl0 = KS == 1 ? 0 : wave & 1;   // its first slab of a tile
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
  const int tok = qw0 + n32;
  const int tok_row = min(tok, n_q - 1);  // tokens past the sequence repeat the last one and are never written
  bf16x8_t qb[kChunks];
#pragma unroll
  for (int c = 0; c < kChunks; ++c)
    qb[c] = as_bf16x8(*reinterpret_cast<const u32x4_t*>(Qb + tok_row * p.q.tok + c * 32 + jh * 16));

  // What a slab that some tokens do not see in part leaves out of the second product, its infinite and NaN values, for the
  // tokens that see them.
  auto add_seen = [&](floatx16_t (&o)[kBlocks], int kt, int sl, const bf16x8_t (&pb)[2], int most) {
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
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float x = __uint_as_float(((e & 2 ? raw.y : raw.x) << (e & 1 ? 0 : 16)) & 0xffff0000u);
            if ((__float_as_uint(x) & 0x7f800000u) == 0x7f800000u) o[b][4 * q + e] = fmaf(w, x, o[b][4 * q + e]);
          }
        }
    }
  };

  floatx16_t o[kBlocks];  // lane (token, h), register i of block b: O[token][32 b + 8 (i / 4) + 4 h + i % 4]
  // Reference maximum of the exponent, log2 units.  It starts at the lowest finite value, so that a masked logit weighs
  // 2^-inf = 0 and not 2^(-inf + inf), also where nothing has been visible yet.
  float m_ref;
  float l_part;           // this lane's share of the running sum
  const float cs = p.scale_log2e;

  auto logits = [&](floatx16_t (&s)[kSlabs], int kt) {
    const unsigned char* base = lds_k[kt & 1] + (sl0 * 32 + n32) * kRow;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      const int piece = 2 * c + jh, slot = (D == 128 ? piece ^ (n32 & 15) : piece ^ (n32 >> 1 & 7)) * 16;
#pragma unroll
      for (int sl = 0; sl < kSlabs; ++sl) {
        const u32x4_t a = *reinterpret_cast<const u32x4_t*>(base + sl * 32 * kRow + slot);
        const floatx16_t zero = {};
        s[sl] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(a), qb[c], c == 0 ? zero : s[sl], 0, 0, 0);
      }
    }
  };
  auto max_of = [&](const floatx16_t (&s)[kSlabs]) {
    float mx = s[0][0];
#pragma unroll
    for (int sl = 0; sl < kSlabs; ++sl)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[sl][i]);
    return mx * cs;
  };
  // Lazy running maximum: a token's reference only moves when a logit exceeds it by more than kMaxSlack (log2 units), so
  // weights stay below 2^kMaxSlack and the rescale of the accumulators is rare after the first tile.
  auto follow_max = [&](float mx) {
    if (__any(mx > m_ref + kMaxSlack)) {
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float mn = fmaxf(m_ref, mx);
      const float alpha = fast_exp2(m_ref - mn);
      m_ref = mn;
      l_part *= alpha;
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) o[b] *= alpha;
    }
  };
  // Weights of a slab of 32 keys as B operands, 16 keys each.
  auto weights = [&](const floatx16_t& s, bf16x8_t (&pb)[2]) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float w = fast_exp2(fmaf(s[8 * u + e], cs, -m_ref));
        l_part += w;
        pb[u][e] = (__bf16)w;
      }
  };
  // Second product for a slab.  A transposed read hands lane m of a 16-lane group element m of the 16 d values the group points
  // at, for 4 consecutive keys: the group (h, d half) reads keys 4 h .. + 3 of each 8, two reads per 16 keys.  finite: infinite
  // and NaN values count as zero.
  auto outputs = [&](int kt, int sl, const bf16x8_t (&pb)[2], bool finite = false) {
    const int n16 = lane & 15, half = (lane >> 4) & 1, k4 = n16 >> 2;
    const unsigned char* row = lds_v[kt & 1] + ((sl0 + sl) * 32 + 4 * jh + k4) * kRow + half * 32 + (n16 & 3) * 8;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        typedef __attribute__((address_space(3))) s16x4_t* lds_ptr_t;
        const unsigned char* at = row + u * 16 * kRow + (D == 128 ? b ^ k4 : b ^ (k4 >> 1)) * 64;
        const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr_t)at);
        const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr_t)(at + 8 * kRow));
        s16x8_t v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        if (finite) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if ((v[e] & 0x7f80) == 0x7f80) v[e] = 0;
        }
        const bf16x8_t a = __builtin_bit_cast(bf16x8_t, v);
        o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pb[u], o[b], 0, 0, 0);
      }
  };

  auto clear = [&]() {
    m_ref = kLowest;
    l_part = 0.f;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[b][i] = 0.f;
  };
  auto mask = [&](floatx16_t (&s)[kSlabs], int kt) {
#pragma unroll
    for (int sl = 0; sl < kSlabs; ++sl)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (kt * kKeyTile + (sl0 + sl) * 32 + 8 * (i / 4) + 4 * jh + i % 4 > before + tok) s[sl][i] = kNegInf;
  };

  clear();
  if (n_key_tiles > 0) {
    stage_k(0);
    stage_v(0);
    if (n_key_tiles > 1) stage_k(1);
    publish();
    floatx16_t s[kSlabs];
    logits(s, 0);
    float mx = max_of(s);
    __syncthreads();  // tile 0's K rows are overwritten by tile 2's in the first step
    bf16x8_t pb[kSlabs][2];
    // One pipeline step: tile kt from its logits in `s`, the next tile's logits into `sn`.
    auto step = [&](const floatx16_t (&s)[kSlabs], floatx16_t (&sn)[kSlabs], int kt) {
      if (kt + 2 < n_key_tiles) stage_k(kt + 2);
      stage_v(kt + 1);
      follow_max(mx);
      logits(sn, kt + 1);
#pragma unroll
      for (int sl = 0; sl < kSlabs; ++sl) {
        weights(s[sl], pb[sl]);
        outputs(kt, sl, pb[sl]);
      }
      mx = max_of(sn);
      publish();
    };
    int kt = 0;
    for (; kt < n_full; kt += 2) {
      floatx16_t sn[kSlabs];
      step(s, sn, kt);
      step(sn, s, kt + 1);
    }
    for (; kt < n_key_tiles; ++kt) {
      // (K of tile kt + 1 was staged by the step before, or in front of the loop; that of kt + 2 is not on its way yet)
      if (kt + 1 < n_key_tiles) stage_v(kt + 1);
      if (kt + 2 < n_key_tiles) stage_k(kt + 2);
      if (kt * kKeyTile + sl0 * 32 <= before + qw0 + 31) {  // else wholly behind what this wavefront's tokens see
        mask(s, kt);
        follow_max(max_of(s));
#pragma unroll
        for (int sl = 0; sl < kSlabs; ++sl) {
          weights(s[sl], pb[sl]);
          outputs(kt, sl, pb[sl]);
        }
        if (kt + 1 < n_key_tiles) logits(s, kt + 1);
      }
      publish();
    }
  }
  float sum = 0.f;  // not finite where one of them is not
#pragma unroll
  for (int b = 0; b < kBlocks; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) sum = fmaf(o[b][i], 0.f, sum);
  if (__syncthreads_or(sum != 0.f)) {
    // An infinite or NaN value that some of a tile's tokens do not see may have reached them, through the product of a zero
    // weight with it: all again, step by step, and the tiles that are masked in part without such values, which follow one by
    // one.  The other tokens get the same bits as in front of such a value.
    clear();
    for (int kt = 0; kt < n_key_tiles; ++kt) {
      stage_k(kt);
      stage_v(kt);
      publish();
      floatx16_t s[kSlabs];
      logits(s, kt);
      mask(s, kt);
      follow_max(max_of(s));
#pragma unroll
      for (int sl = 0; sl < kSlabs; ++sl) {
        bf16x8_t pb[2];
        weights(s[sl], pb);
        const bool in_part = (kt + 1) * kKeyTile > before + q0 + 1;
        outputs(kt, sl, pb, in_part);
        if (in_part) add_seen(o, kt, sl0 + sl, pb, before + tok);
      }
      __syncthreads();
    }
  }

  float l_tot = l_part + __shfl_xor(l_part, 32);
  if (KS == 2) {  // the second wavefront of a pair hands over what it has (the staged tiles have been read)
    float* const o_sum = reinterpret_cast<float*>(&lds_k[0][0]) + (wave >> 1) * (kBlocks * 16 * 64);  // [register][lane]
    float2* const ml = reinterpret_cast<float2*>(&lds_v[0][0] + (wave | 1) * (32 * kRow));  // (where no rows will lie: the second one returns)
    static_assert(sizeof(lds_k) >= kWaves / 2 * kBlocks * 16 * 64 * 4, "outputs of half the wavefronts");
    if (wave & 1) {
      ml[lane] = make_float2(m_ref, l_tot);
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o_sum[(b * 16 + i) * 64 + lane] = o[b][i];
    }
    __syncthreads();
    if (wave & 1) return;
    const float2 other = ml[lane];
    const float m = fmaxf(m_ref, other.x), mine = fast_exp2(m_ref - m), theirs = fast_exp2(other.x - m);
    m_ref = m;
    l_tot = l_tot * mine + other.y * theirs;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[b][i] = o[b][i] * mine + o_sum[(b * 16 + i) * 64 + lane] * theirs;
  }
  const bool none = before + tok < 0;  // sees no key
  const float inv = none ? 0.f : 1.f / l_tot;
  if (p.lse.data && jh == 0 && tok < n_q)
    *reinterpret_cast<float*>(reinterpret_cast<unsigned char*>(p.lse.data) + lse0 + tok * p.lse.tok) =
        none ? kNegInf : m_ref + __builtin_log2f(l_tot);
  // Rows of bf16 through LDS (this wavefront's part of where V was), so that whole rows are stored.
  unsigned char* const rows = &lds_v[0][0] + wave * (32 * kRow);
  static_assert(sizeof(lds_v) >= kWaves * 32 * kRow, "a wavefront's rows");
#pragma unroll
  for (int b = 0; b < kBlocks; ++b)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
      bf16x4_t r;
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] = (__bf16)(o[b][4 * q + i] * inv);
      const int piece = 4 * b + q;
      *reinterpret_cast<bf16x4_t*>(rows + n32 * kRow + (D == 128 ? piece ^ (n32 & 15) : piece ^ (n32 >> 1 & 7)) * 16 + jh * 8) = r;
    }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
  for (int i = 0; i < 32 / kCopyRows; ++i) {
    const int r = i * kCopyRows + lane / kPieces, piece = lane % kPieces;
    const u32x4_t x = *reinterpret_cast<const u32x4_t*>(rows + r * kRow + (D == 128 ? piece ^ (r & 15) : piece ^ (r >> 1 & 7)) * 16);
    if (qw0 + r < n_q)
      *reinterpret_cast<u32x4_t*>(reinterpret_cast<unsigned char*>(p.out.data) + out0 + (qw0 + r) * p.out.tok + piece * 16) = x;
  }
}

template <int D>
void launch(const PromptParams& p, int tile_tokens, unsigned grid, hipStream_t s) {
  if (tile_tokens == 32 * kWaves) prompt_attn_kernel<D, 1><<<dim3(grid), dim3(64 * kWaves), 0, s>>>(p);
  else prompt_attn_kernel<D, 2><<<dim3(grid), dim3(64 * kWaves), 0, s>>>(p);
}

}  // namespace

// A call that would leave compute units idle, or give each no more than one workgroup of 128 tokens, whose chain of tiles it then
// waits for, takes workgroups of 64 tokens that share their keys.  us, 128 / 64 tokens, 32 heads of 128: one prompt of 512
// tokens 15.9 / 12.4, of 1024 (one workgroup for each) 24.4 / 20.7, 4 of 500 (two) 23.7 / 28.9, one of 2048 47.4 / 52.1; 8 heads,
// one of 4096 75.6 / 57.6, of 8192 156 / 161.  Keys are not split over workgroups: few tokens behind many keys take as long as their
// chain of key tiles, 1 to 128 tokens of 32 heads behind 32768 keys 345 to 370 us, where the keys and values are read in 19.
int prompt_tile_tokens(int64_t n_tiles128, int n_cus) { return n_tiles128 <= n_cus ? 16 * kWaves : 32 * kWaves; }

hipError_t launch_prompt_attn(const PromptParams& p_in, int D, int tile_tokens, int n_tiles, int n_cus, hipStream_t s) {
  const int64_t grid = (int64_t)n_tiles * p_in.Hq;
  if (grid <= 0) return hipSuccess;
  if (grid > INT32_MAX / (64 * kWaves)) return hipErrorInvalidValue;
  // Longest first, which evens out many rounds of workgroups.  Where all run at once, two to a compute unit, those that join
  // the first ones there come in the opposite order: the shortest beside the longest.
  PromptParams p = p_in;
  p.reversed_from = grid <= 2 * n_cus ? n_cus : INT32_MAX;
  if (D == 128) launch<128>(p, tile_tokens, (unsigned)grid, s);
  else launch<64>(p, tile_tokens, (unsigned)grid, s);
  return hipGetLastError();
}

}  // namespace baklava
