// Attention of a tree of drafted tokens over ragged caches (baklava_tree_attn).
//
// A query row is a node of a sequence's tree and one of the G heads of a KV head (row r: node r / G, head r % G).  It sees every
// live row of the cache, and of the drafted rows those of its ancestors and its own.  Both products run on the matrix cores, in
// blocks of 32 query rows and slabs of 32 keys, with the keys on the M side:
//
//   S^T[key, row]  = K[key, :] . Q[row, :]          A = K from LDS, B = Q (registers)
//   O^T[d, row]   += V^T[d, keys] . P^T[keys, row]   A = V from LDS, B = P^T
//
// The accumulator of S^T (lane (row, h), register i: key 8 (i / 4) + 4 h + i % 4) is a B operand of the second product once that
// product's keys are numbered the way the lane holds them, so the softmax weights never leave their lane.  bf16 rows, and 4-bit
// rows, whose values are bf16 numbers: v_mfma_f32_32x32x16_bf16, weights rounded to bf16 (as much as the rounding of the output
// loses).  fp32 rows: v_mfma_f32_32x32x2_f32 throughout.
//
// One pass over the keys with the running maximum and sum of every row in fp32.  The keys of all caches of a launch are cut into
// work items of equal length, as the lengths on the device are (so a replayed launch is balanced too); each workgroup finds its
// item by a scan over the lengths.  Caches of several items are merged by a kernel of their own.
//
// A workgroup of four wavefronts, two of them to a compute unit, owns 128 query rows (64 where pairs share their rows) and shares
// tiles of 64 keys in LDS.  16 caches of 39321 bf16 rows, 448 query rows: 188 us of which 110 are the products at the rate of a library
// product (1306 TFLOP/s); the matrix cores are busy 47% of the cycles, at 1.7 GHz: start and end take some 15 us, one wavefront in eight
// has no rows of the last workgroup, and a step of 2.2 us ends with a wait for the tiles asked for at its start.  64 caches of 8200 rows,
// 64 query rows on average: 53 us (271 MB, 39 at 7 TB/s), and 12 for the merge of their partials.  128 caches of 9830 4-bit rows, 52
// query rows: 66 us (155 MB, 22): conversions, exponentials and LDS, none of them saturated.
#include "common.h"
#include "mxfp4.h"
#include "tree.h"

namespace baklava {

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef float floatx4_t __attribute__((ext_vector_type(4)));
typedef float floatx16_t __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x8_t __attribute__((ext_vector_type(8)));

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLowest = -3.402823466e38f;
constexpr float kMaxSlack = 8.f;  // a logit may exceed its row's reference maximum by this much (log2 units)

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

constexpr int kKeyTile = 64;  // keys per LDS stage
// Workgroups that fit a compute unit.
constexpr int tree_resident(int type, int D) { return 4 * kKeyTile * D * (type == 1 ? 4 : 2) > 72 * 1024 ? 1 : 2; }

// What follows from the rows' type (BAKLAVA_BF16, F32, MXFP4), the head dimension and KS, the wavefronts that share 32 query rows.
template <int TYPE, int D, int KS>
struct Shape {
  static constexpr bool kF32 = TYPE == 1, kMx = TYPE == 2;
  static constexpr int kRows = 32 * kWaves / KS;             // query rows of a workgroup
  static constexpr int kTile = kKeyTile;
  static constexpr int kSlabs = kTile / 32 / KS;             // slabs of 32 keys that a wavefront takes of it
  static constexpr int kRow = D * (kF32 ? 4 : 2);            // bytes of a row in LDS
  static constexpr int kPieces = kRow / 16;
  static constexpr int kChunks = kPieces / 2;                // pieces of a row that a lane takes in the first product
  static constexpr int kBlocks = D / 32;
  static constexpr int kStage = kTile * kRow;                // bytes of a plane's stage
  // direct copies into LDS: rows per instruction, instructions per wavefront and plane
  static constexpr int kCopyRows = 64 / kPieces, kCopies = kTile / kWaves / kCopyRows;
  // 4-bit rows: 16-byte pieces (32 codes) of a row, and per thread of a plane's tile
  static constexpr int kMxPieces = D / 32, kMxPer = (kTile * kMxPieces + kThreads - 1) / kThreads;
  // Where piece `x` of a row lies in LDS: permuted so that the operand reads spread over the banks.
  static __device__ __forceinline__ int k_slot(int row, int x) {
    return kF32 || D == 128 ? x ^ (row & 15) : x ^ (row >> 1 & 7);
  }
  static __device__ __forceinline__ int v_slot(int row, int x) {
    if (kF32) return x ^ 8 * (row >> 2 & 1);
    // (values of 4-bit rows are written 16 bytes at a time, by lanes of few pieces of several rows: these spread, too)
    return D == 128 ? x ^ 4 * (row & 3) ^ (kMx ? (row ^ row >> 2) & 3 : 0) : x ^ 4 * (row >> 1 & 1);
  }
};

// ONCE: a work item's rows are read by one workgroup, past the caches (577 MB are read in 88 us so, in 101 with the ordinary hint).
template <int TYPE, int D, int KS, bool ONCE>
__global__ __launch_bounds__(kThreads, 2) void tree_attn_kernel(TreeParams p) {
  using S = Shape<TYPE, D, KS>;
  constexpr int kSlabs = S::kSlabs, kBlocks = S::kBlocks, kRow = S::kRow, kTile = S::kTile;
  __shared__ __attribute__((aligned(16))) unsigned char lds_k[2][S::kStage];
  __shared__ __attribute__((aligned(16))) unsigned char lds_v[2][S::kStage];
  __shared__ unsigned long long above[kMostNodes / 64][kMostNodes];  // [word][node]: the nodes that a node sees
  __shared__ int32_t scan[kWaves + 3];

  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n32 = lane & 31, jh = lane >> 5;
  // The workgroups of an item's query rows follow each other on one XCD (consecutive workgroups go round them).
  const int group = (uint32_t)blockIdx.x / (uint32_t)(8 * p.row_tiles), in_group = (uint32_t)blockIdx.x % (uint32_t)(8 * p.row_tiles);
  const int item = group * 8 + (in_group & 7), row_tile = in_group >> 3;
  // Tiles of live rows, then those of drafted rows.
  auto tiles = [&](int c) {
    const int n = tree_nodes(p, (uint32_t)c / (uint32_t)p.Hkv % (uint32_t)p.batch);
    return n > 0 ? (p.len[p.cache0 + c] + kTile - 1) / kTile + (n + kTile - 1) / kTile : 0;
  };
  Span sp;
  if (!find_span<kThreads>(p.n_caches, p.target, 1, item, tiles, scan, sp)) return;
  const int h = sp.c_rel % p.Hkv, s_rel = sp.c_rel / p.Hkv, b = s_rel % p.batch;
  const int n_nodes = __builtin_amdgcn_readfirstlane(tree_nodes(p, b)), n_rows = n_nodes * p.G;
  const int n_live = __builtin_amdgcn_readfirstlane(p.len[p.cache0 + sp.c_rel]), live_tiles = (n_live + kTile - 1) / kTile;
  const int r0 = row_tile * S::kRows;  // first query row of the workgroup
  if (row_tile == 0 && sp.part == 0 && tid == 0) p.table[sp.c_rel] = make_int2(sp.slot, sp.n_parts);
  if (r0 >= n_rows) return;
  const int64_t row0 = uniform(p.off[p.cache0 + sp.c_rel]);

  // ---- query rows ------------------------------------------------------------------------------
  const int rw0 = r0 + wave / KS * 32;      // first row of this wavefront
  const int sl0 = wave % KS * kSlabs;       // its first slab of a tile
  const bool idle = rw0 >= n_rows;          // (such a wavefront helps with the copies)
  const int row = min(rw0 + n32, n_rows - 1);  // rows past the last repeat it and are not written
  const int node = row / p.G, head = h * p.G + row % p.G;
  const unsigned char* Qr = reinterpret_cast<const unsigned char*>(p.q.data) + s_rel * p.q.seq + node * p.q.tok + head * p.q.head;
  u32x4_t qb[S::kChunks];  // chunk c: piece 2 c + h of the row
#pragma unroll
  for (int c = 0; c < S::kChunks; ++c) qb[c] = *reinterpret_cast<const u32x4_t*>(Qr + c * 32 + jh * 16);

  floatx16_t o[kBlocks];  // lane (row, h), register i of block b: O[row][32 b + 8 (i / 4) + 4 h + i % 4]
#pragma unroll
  for (int x = 0; x < kBlocks; ++x)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[x][i] = 0.f;
  // Reference maximum of the exponent, log2 units.  It starts at the lowest finite value, so that a masked logit weighs 2^-inf = 0.
  float m_ref = kLowest, l_part = 0.f;
  const float cs = p.scale_log2e;

  // ---- one tile from LDS -----------------------------------------------------------------------
  auto logits = [&](floatx16_t (&s)[kSlabs], int buf) {
    const unsigned char* base = lds_k[buf] + (sl0 * 32 + n32) * kRow;
#pragma unroll
    for (int c = 0; c < S::kChunks; ++c) {
      const int slot = S::k_slot(n32, 2 * c + jh) * 16;  // (32 rows further the permutation is the same)
#pragma unroll
      for (int sl = 0; sl < kSlabs; ++sl) {
        const u32x4_t a = *reinterpret_cast<const u32x4_t*>(base + sl * 32 * kRow + slot);
        const floatx16_t zero = {};
        if constexpr (S::kF32) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            s[sl] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[e]), __uint_as_float(qb[c][e]), c == 0 && e == 0 ? zero : s[sl], 0, 0, 0);
        } else {
          s[sl] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, qb[c]), c == 0 ? zero : s[sl], 0, 0, 0);
        }
      }
    }
  };
  // Lazy running maximum: a row's reference only moves when a logit exceeds it by more than kMaxSlack, so weights stay below
  // 2^kMaxSlack and the rescale of the accumulators is rare after the first tile.
  auto max_of = [&](const floatx16_t (&s)[kSlabs]) {
    float mx = s[0][0];
#pragma unroll
    for (int sl = 0; sl < kSlabs; ++sl)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[sl][i]);
    return mx * cs;
  };
  auto follow_max = [&](float mx) {
    if (__any(mx > m_ref + kMaxSlack)) {
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float mn = mx > m_ref + kMaxSlack ? mx : m_ref;  // (a row's bits do not depend on the others)
      const float alpha = fast_exp2(m_ref - mn);
      m_ref = mn;
      l_part *= alpha;
#pragma unroll
      for (int x = 0; x < kBlocks; ++x) o[x] *= alpha;
    }
  };
  // Weights of a slab and what they add to the outputs.  finite: infinite and NaN values count as zero (see add_seen).
  auto outputs = [&](const floatx16_t& s, int buf, int sl, bool finite) {
    const unsigned char* base = lds_v[buf] + (sl0 + sl) * 32 * kRow;
    if constexpr (S::kF32) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float w = fast_exp2(fmaf(s[i], cs, -m_ref));
        l_part += w;
        const int key = 8 * (i / 4) + 4 * jh + i % 4;
#pragma unroll
        for (int x = 0; x < kBlocks; ++x) {
          float v = *reinterpret_cast<const float*>(base + key * kRow + S::v_slot(key, 8 * x) * 16 + n32 * 4);
          if (finite && (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u) v = 0.f;
          o[x] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, w, o[x], 0, 0, 0);
        }
      }
    } else {
      // A transposed read hands lane m of a 16-lane group element m of the 16 d values the group points at, for 4 consecutive
      // keys: the group (h, d half) reads keys 4 h .. + 3 of each 8, two reads per 16 keys.
      const int n16 = lane & 15, half = (lane >> 4) & 1, k4 = n16 >> 2;
      const unsigned char* at0 = base + (4 * jh + k4) * kRow + (n16 & 1) * 8;
      const int piece = 2 * half + (n16 >> 1 & 1);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        bf16x8_t pb;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float w = fast_exp2(fmaf(s[8 * u + e], cs, -m_ref));
          l_part += w;
          pb[e] = (__bf16)w;
        }
#pragma unroll
        for (int x = 0; x < kBlocks; ++x) {
          typedef __attribute__((address_space(3))) s16x4_t* lds_ptr_t;
          const unsigned char* at = at0 + u * 16 * kRow;  // (keys 16 u + 4 h + k4 and 8 further)
          const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr_t)(at + S::v_slot(4 * jh + k4, 4 * x + piece) * 16));
          const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr_t)(at + 8 * kRow + S::v_slot(8 + 4 * jh + k4, 4 * x + piece) * 16));
          s16x8_t v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
          if (finite) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if ((v[e] & 0x7f80) == 0x7f80) v[e] = 0;
          }
          o[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, v), pb, o[x], 0, 0, 0);
        }
      }
    }
  };

  // ---- live rows into LDS ----------------------------------------------------------------------
  const unsigned char* Kp = reinterpret_cast<const unsigned char*>(p.k_plane);
  const unsigned char* Vp = reinterpret_cast<const unsigned char*>(p.v_plane);
  constexpr int kStored = S::kMx ? D / 2 : kRow;  // bytes of a row in the arena
  uint32_t k_off[S::kCopies], v_off[S::kCopies], c_row[S::kCopies];
  if constexpr (!S::kMx) {
#pragma unroll
    for (int i = 0; i < S::kCopies; ++i) {
      const int r = wave * (kTile / kWaves) + i * S::kCopyRows + lane / S::kPieces, slot = lane % S::kPieces;
      c_row[i] = r;
      k_off[i] = S::k_slot(r, slot) * 16;
      v_off[i] = S::v_slot(r, slot) * 16;
    }
  }
  // bf16 and fp32 rows go straight to LDS, 1 KiB in lane order per instruction (the permutation of a row's pieces is in the
  // addresses); 4-bit rows go through registers, and `put` puts their values into LDS.  Rows past the last live one repeat it;
  // they are masked.
  struct Codes {
    u32x4_t c[S::kMx ? S::kMxPer : 1];
    uint32_t byte[S::kMx ? S::kMxPer : 1];
  };
  auto request = [&](Codes& codes, int value, int kt) {
    const uint32_t most = n_live - 1 - kt * kTile;
    const int64_t first = row0 + (int64_t)kt * kTile;
    const unsigned char* src = (value ? Vp : Kp) + first * kStored;
    if constexpr (S::kMx) {
      const uint8_t* scale = p.kv_scale + first * (D / 16) + value * (D / 32);
#pragma unroll
      for (int i = 0; i < S::kMxPer; ++i) {
        const uint32_t x = i * kThreads + tid, r = min(x / S::kMxPieces, most), piece = x % S::kMxPieces;
        codes.c[i] = *reinterpret_cast<const u32x4_t*>(src + (r * kStored + piece * 16));
        codes.byte[i] = scale[r * (D / 16) + piece];
      }
    } else {
      const uint32_t dst = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)(value ? lds_v[kt & 1] : lds_k[kt & 1]) +
                           wave * (kTile / kWaves) * kRow;
#pragma unroll
      for (int i = 0; i < S::kCopies; ++i) {
        const uint32_t at = min(c_row[i], most) * (uint32_t)kStored + (value ? v_off[i] : k_off[i]);
        if constexpr (ONCE)
          asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" :: "s"(dst + i * 1024), "v"(at), "s"(src) : "memory", "m0");
        else
          asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(dst + i * 1024), "v"(at), "s"(src) : "memory", "m0");
      }
    }
  };
  auto put_mx = [&](int buf, int value, int r, int piece, u32x4_t codes, uint32_t byte) {
    unsigned char* dst = (value ? lds_v[buf] : lds_k[buf]) + r * kRow;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      *reinterpret_cast<uint4*>(dst + (value ? S::v_slot(r, 4 * piece + e) : S::k_slot(r, 4 * piece + e)) * 16) = mx_values(codes[e], mx_scale(byte));
  };
  auto put = [&](const Codes& codes, int value, int kt) {
    if constexpr (S::kMx) {
#pragma unroll
      for (int i = 0; i < S::kMxPer; ++i) {
        const int x = i * kThreads + tid;
        if (x < kTile * S::kMxPieces) put_mx(kt & 1, value, x / S::kMxPieces, x % S::kMxPieces, codes.c[i], codes.byte[i]);
      }
    }
  };
  auto arrive = [&]() {
    if constexpr (!S::kMx) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  };

  // ---- live rows: a software pipeline, the first product of tile kt + 1 beside the exponentials of tile kt -------------------
  // In a step the K rows of tile kt + 2 and the V rows of kt + 1 come in.  Copies to LDS are asked for at its start; codes, which
  // wait in registers until their values can go to LDS, a step earlier.
  const int live_end = min(sp.last, live_tiles);
  if (sp.first < live_end) {
    int kt = sp.first;
    Codes ck, cv, nk, nv;
    request(ck, 0, kt);
    request(cv, 1, kt);
    put(ck, 0, kt);
    put(cv, 1, kt);
    if (kt + 1 < live_end) {
      request(ck, 0, kt + 1);
      put(ck, 0, kt + 1);
    }
    auto ask = [&](Codes& k, Codes& v, int kt) {
      if (kt + 2 < live_end) request(k, 0, kt + 2);
      if (kt + 1 < live_end) request(v, 1, kt + 1);
    };
    if constexpr (S::kMx) ask(ck, cv, kt);
    arrive();
    floatx16_t s[kSlabs];
    float mx = kLowest;
    if (!idle) {
      logits(s, kt & 1);
      mx = max_of(s);
    }
    __syncthreads();  // (the first tile's K rows are overwritten in the first step)
    auto step = [&](const floatx16_t (&s)[kSlabs], floatx16_t (&sn)[kSlabs], int kt, Codes& ck, Codes& cv, Codes& nk, Codes& nv) {
      if constexpr (S::kMx) {
        request(nk, 0, kt + 3);
        request(nv, 1, kt + 2);
      } else {
        request(ck, 0, kt + 2);
        request(cv, 1, kt + 1);
      }
      if (!idle) {
        follow_max(mx);
        logits(sn, kt + 1 & 1);
#pragma unroll
        for (int sl = 0; sl < kSlabs; ++sl) outputs(s[sl], kt & 1, sl, false);
        mx = max_of(sn);
      }
      put(ck, 0, kt + 2);
      put(cv, 1, kt + 1);
      arrive();
    };
    for (; kt + 4 < live_end; kt += 2) {
      floatx16_t sn[kSlabs];
      step(s, sn, kt, ck, cv, nk, nv);
      step(sn, s, kt + 1, nk, nv, ck, cv);
    }
    for (; kt < live_end; ++kt) {
      if constexpr (!S::kMx) ask(ck, cv, kt);
      if ((kt + 1) * kTile > n_live) {  // (a weight of zero times an infinity of the row that was repeated would be NaN)
        for (int x = (n_live - kt * kTile) * S::kPieces + tid; x < kTile * S::kPieces; x += kThreads)
          *reinterpret_cast<u32x4_t*>(lds_v[kt & 1] + x * 16) = u32x4_t{};
        __syncthreads();
      }
      if (!idle) {
        if ((kt + 1) * kTile > n_live) {
#pragma unroll
          for (int sl = 0; sl < kSlabs; ++sl)
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (kt * kTile + (sl0 + sl) * 32 + 8 * (i / 4) + 4 * jh + i % 4 >= n_live) s[sl][i] = kNegInf;
        }
        follow_max(max_of(s));
#pragma unroll
        for (int sl = 0; sl < kSlabs; ++sl) outputs(s[sl], kt & 1, sl, false);
        if (kt + 1 < live_end) logits(s, kt + 1 & 1);
      }
      if (kt + 2 < live_end) put(ck, 0, kt + 2);
      if (kt + 1 < live_end) put(cv, 1, kt + 1);
      if constexpr (S::kMx) ask(ck, cv, kt + 1);
      arrive();
    }
  }

  // ---- drafted rows ----------------------------------------------------------------------------
  if (sp.last > live_tiles) {
    static_assert(kMostNodes == kThreads, "a thread for every node");
    int up = -1;  // (a parent that is no earlier node is none)
    if (tid < n_nodes) up = p.parent[(int64_t)b * p.N + tid];
    if (up < 0 || up >= tid) up = -1;
    __syncthreads();  // (the last tile has been read)
    find_ancestors(up, n_nodes, above, reinterpret_cast<int32_t*>(lds_k[0]));
    const int first_dt = max(sp.first - live_tiles, 0), last_dt = sp.last - live_tiles;
    const unsigned char* Kd = reinterpret_cast<const unsigned char*>(p.k.data) + s_rel * p.k.seq + h * p.k.head;
    const unsigned char* Vd = reinterpret_cast<const unsigned char*>(p.v.data) + s_rel * p.v.seq + h * p.v.head;
    for (int dt = first_dt; dt < last_dt; ++dt) {
      // Rows past the last node repeat it; nobody sees them.
      bool wild = false;  // an infinite or NaN value
      auto is_wild = [](uint32_t w) {
        return S::kF32 ? (w & 0x7f800000u) == 0x7f800000u : (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
      };
      constexpr int kGroup = S::kMx ? 4 : 1;  // pieces of a row that a thread takes together: those of a scale
      for (int x = tid; x < 2 * kTile * S::kPieces / kGroup; x += kThreads) {
        const int value = x / (kTile * S::kPieces / kGroup), y = x % (kTile * S::kPieces / kGroup);
        const int r = y / (S::kPieces / kGroup), piece = y % (S::kPieces / kGroup);
        const int j = min(dt * kTile + r, n_nodes - 1);
        const unsigned char* src = (value ? Vd + j * p.v.tok : Kd + j * p.k.tok) + piece * kGroup * 16;
        u32x4_t w[kGroup];
#pragma unroll
        for (int e = 0; e < kGroup; ++e) w[e] = *reinterpret_cast<const u32x4_t*>(src + e * 16);
        if (value) {
#pragma unroll
          for (int e = 0; e < kGroup; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) wild = wild || is_wild(w[e][i]);
        }
        if constexpr (S::kMx) {  // rounded to 4 bits, as they will be in a cache
          uint32_t top = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) top = max(top, max(w[e][i] & 0x7fffu, w[e][i] >> 16 & 0x7fffu));
          const uint32_t byte = mx_scale_byte(top);
          u32x4_t codes;
#pragma unroll
          for (int e = 0; e < 4; ++e) codes[e] = mx_codes(make_uint4(w[e][0], w[e][1], w[e][2], w[e][3]), byte);
          put_mx(0, value, r, piece, codes, byte);
        } else {
          *reinterpret_cast<u32x4_t*>((value ? lds_v[0] : lds_k[0]) + r * kRow + (value ? S::v_slot(r, piece) : S::k_slot(r, piece)) * 16) = w[0];
        }
      }
      wild = __syncthreads_or(wild);
      if (!idle) {
        floatx16_t s[kSlabs];
        logits(s, 0);
        uint32_t seen[kSlabs];
#pragma unroll
        for (int sl = 0; sl < kSlabs; ++sl) {
          const int key0 = dt * kTile + (sl0 + sl) * 32;
          seen[sl] = key0 < n_nodes ? (uint32_t)(above[key0 / 64][node] >> (key0 & 32)) : 0u;
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (!(seen[sl] >> (8 * (i / 4) + 4 * jh + i % 4) & 1)) s[sl][i] = kNegInf;
        }
        follow_max(max_of(s));
#pragma unroll
        for (int sl = 0; sl < kSlabs; ++sl) {
          outputs(s[sl], 0, sl, wild);
          // An infinite or NaN value counts for the rows that see it, one by one: the product of a zero weight with it would reach
          // all the others.
          if (wild) {
            for (int j = 0; j < 32; ++j) {
              float w = 0.f;
#pragma unroll
              for (int i = 0; i < 16; ++i)
                if (8 * (i / 4) + i % 4 == (j & ~4)) w = fast_exp2(fmaf(s[sl][i], cs, -m_ref));
              w = __shfl(w, n32 + 8 * (j & 4));  // from the half that holds key j
              if (!(seen[sl] >> j & 1)) continue;
              const int r = (sl0 + sl) * 32 + j;
#pragma unroll
              for (int x = 0; x < kBlocks; ++x)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                  const int d = 32 * x + 8 * (i / 4) + 4 * jh + i % 4;
                  const unsigned char* src = lds_v[0] + r * kRow + S::v_slot(r, d * (S::kF32 ? 4 : 2) / 16) * 16;
                  const float v = S::kF32 ? *reinterpret_cast<const float*>(src + d % 4 * 4)
                                          : __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(src + d % 8 * 2) << 16);
                  if ((__float_as_uint(v) & 0x7f800000u) == 0x7f800000u) o[x][i] = fmaf(w, v, o[x][i]);
                }
            }
          }
        }
      }
      __syncthreads();
    }
  }

  // ---- the end of a work item ------------------------------------------------------------------
  float l_tot = l_part + __shfl_xor(l_part, 32);
  if constexpr (KS > 1) {  // the other wavefronts of the same rows hand over what they have
    constexpr int kPart = kBlocks * 16 * 64;  // floats, [register][lane]
    static_assert(sizeof(lds_v) >= kWaves * 64 * sizeof(float2), "maxima and sums");
    static_assert(sizeof(lds_k) >= (kWaves / KS) * kPart * 4, "outputs of one wavefront of each block");
    float* const o_sum = reinterpret_cast<float*>(&lds_k[0][0]) + wave / KS * kPart;
    float2* const ml = reinterpret_cast<float2*>(&lds_v[0][0]) + wave * 64;
#pragma unroll
    for (int other = 1; other < KS; ++other) {
      __syncthreads();
      if (wave % KS == other) {
        ml[lane] = make_float2(m_ref, l_tot);
#pragma unroll
        for (int x = 0; x < kBlocks; ++x)
#pragma unroll
          for (int i = 0; i < 16; ++i) o_sum[(x * 16 + i) * 64 + lane] = o[x][i];
      }
      __syncthreads();
      if (wave % KS == 0) {
        const float2 got = ml[other * 64 + lane];
        const float m = fmaxf(m_ref, got.x), mine = fast_exp2(m_ref - m), theirs = fast_exp2(got.x - m);
        m_ref = m;
        l_tot = l_tot * mine + got.y * theirs;
#pragma unroll
        for (int x = 0; x < kBlocks; ++x)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[x][i] = o[x][i] * mine + o_sum[(x * 16 + i) * 64 + lane] * theirs;
      }
    }
    if (wave % KS) return;
  }
  if (rw0 + n32 >= n_rows) return;
  if (sp.n_parts == 1) {
    const float inv = 1.f / l_tot;
    if (p.lse.data && jh == 0)
      *reinterpret_cast<float*>(reinterpret_cast<unsigned char*>(p.lse.data) + s_rel * p.lse.seq + node * p.lse.tok + head * p.lse.head) =
          m_ref + __builtin_log2f(l_tot);
    unsigned char* dst = reinterpret_cast<unsigned char*>(p.out.data) + s_rel * p.out.seq + node * p.out.tok + head * p.out.head;
#pragma unroll
    for (int x = 0; x < kBlocks; ++x)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int d = 32 * x + 8 * q + 4 * jh;
        if constexpr (S::kF32) {
          floatx4_t r;
#pragma unroll
          for (int i = 0; i < 4; ++i) r[i] = o[x][4 * q + i] * inv;
          *reinterpret_cast<floatx4_t*>(dst + d * 4) = r;
        } else {
          bf16x4_t r;
#pragma unroll
          for (int i = 0; i < 4; ++i) r[i] = (__bf16)(o[x][4 * q + i] * inv);
          *reinterpret_cast<bf16x4_t*>(dst + d * 2) = r;
        }
      }
  } else {
    const int64_t at = (int64_t)(sp.slot + sp.part) * p.rows + row;
    if (jh == 0) p.part_ml[at] = make_float2(m_ref, l_tot);
#pragma unroll
    for (int x = 0; x < kBlocks; ++x)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        floatx4_t r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = o[x][4 * q + i];
        *reinterpret_cast<floatx4_t*>(p.part_o + at * D + 32 * x + 8 * q + 4 * jh) = r;
      }
  }
}

// Partials of caches that have several work items.  D / 4 lanes take a query row's elements, kGroups of them its work items in
// turn: with a workgroup to kMergeRows rows a small launch still has a few hundred wavefronts, each with four loads on the way.
constexpr int kMergeRows = 2;
template <int D, bool F32>
__global__ __launch_bounds__(kThreads) void tree_merge_kernel(TreeParams p) {
  constexpr int kLanes = D / 4, kPer = kThreads / kMergeRows, kGroups = kPer / kLanes;
  __shared__ float weight[kMergeRows][kMostTreeItems];
  __shared__ float2 sums[kMergeRows][kPer / 64];
  __shared__ floatx4_t part_sum[kMergeRows][kGroups][kLanes];
  const int c_rel = blockIdx.x, s_rel = c_rel / p.Hkv, h = c_rel % p.Hkv, b = s_rel % p.batch;
  const int n_rows = tree_nodes(p, b) * p.G;
  const int r0 = blockIdx.y * kMergeRows;
  if (r0 >= n_rows) return;
  const int2 t = p.table[c_rel];  // (written for every sequence that has nodes)
  const int n_parts = t.y;
  if (n_parts <= 1) return;
  const int tid = threadIdx.x, at = tid / kPer, in = tid % kPer;
  const int row = min(r0 + at, n_rows - 1);  // (a row past the last repeats it)
  const float2* ml = p.part_ml + (int64_t)t.x * p.rows + row;
  // weights of the items: 2^(m_i - m)
  float m = kLowest;
  for (int i = in; i < n_parts; i += kPer) {
    const float x = ml[(int64_t)i * p.rows].x;
    weight[at][i] = x;
    m = fmaxf(m, x);
  }
#pragma unroll
  for (int i = 32; i >= 1; i /= 2) m = fmaxf(m, __shfl_xor(m, i));
  if (tid % 64 == 0) sums[at][in / 64].x = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kPer / 64; ++w) m = fmaxf(m, sums[at][w].x);
  float l = 0.f;
  for (int i = in; i < n_parts; i += kPer) {
    const float a = fast_exp2(weight[at][i] - m);
    weight[at][i] = a;
    l += ml[(int64_t)i * p.rows].y * a;
  }
#pragma unroll
  for (int i = 32; i >= 1; i /= 2) l += __shfl_xor(l, i);
  if (tid % 64 == 0) sums[at][in / 64].y = l;
  __syncthreads();
  l = 0.f;
#pragma unroll
  for (int w = 0; w < kPer / 64; ++w) l += sums[at][w].y;
  const int d = in % kLanes, group = in / kLanes;
  const floatx4_t* part = reinterpret_cast<const floatx4_t*>(p.part_o + ((int64_t)t.x * p.rows + row) * D) + d;
  const int64_t step = (int64_t)p.rows * (D / 4);
  floatx4_t o = {0.f, 0.f, 0.f, 0.f};
  int i = group;
  for (; i + 3 * kGroups < n_parts; i += 4 * kGroups) {
    floatx4_t x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = part[(i + e * kGroups) * step];
#pragma unroll
    for (int e = 0; e < 4; ++e) o += x[e] * weight[at][i + e * kGroups];
  }
  for (; i < n_parts; i += kGroups) o += part[i * step] * weight[at][i];
  part_sum[at][group][d] = o;
  __syncthreads();
  if (group != 0 || r0 + at >= n_rows) return;
#pragma unroll
  for (int g = 1; g < kGroups; ++g) o += part_sum[at][g][d];
  const int node = row / p.G, head = h * p.G + row % p.G;
  if (p.lse.data && d == 0)
    *reinterpret_cast<float*>(reinterpret_cast<unsigned char*>(p.lse.data) + s_rel * p.lse.seq + node * p.lse.tok + head * p.lse.head) =
        m + __builtin_log2f(l);
  unsigned char* dst = reinterpret_cast<unsigned char*>(p.out.data) + s_rel * p.out.seq + node * p.out.tok + head * p.out.head;
  const float inv = 1.f / l;
  if (F32) {
    reinterpret_cast<floatx4_t*>(dst)[d] = o * inv;
  } else {
    bf16x4_t r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = (__bf16)(o[e] * inv);
    reinterpret_cast<bf16x4_t*>(dst)[d] = r;
  }
}

template <int TYPE, int D>
hipError_t launch(const TreeParams& p, int ks, unsigned grid, hipStream_t s) {
  if constexpr (TYPE != 0) {  // (bf16 launches of as few rows are the streaming kernel's: rule at tree_launch)
    if (ks == 2) {
      tree_attn_kernel<TYPE, D, 2, true><<<dim3(grid), dim3(kThreads), 0, s>>>(p);
      return hipGetLastError();
    }
  }
  if (p.row_tiles == 1) tree_attn_kernel<TYPE, D, 1, true><<<dim3(grid), dim3(kThreads), 0, s>>>(p);
  else tree_attn_kernel<TYPE, D, 1, false><<<dim3(grid), dim3(kThreads), 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace

// The streaming kernel takes up to 64 query rows over bf16 caches, up to 32 over the others, where two blocks of them cost it too many
// registers.  us a call, it / this one with pairs of wavefronts, 64 caches of 10240 rows: bf16, D = 128, 64 rows 61.8 / 65.9, D = 64
// 36.4 / 40.7, 1 row 59.0 / 69.2; 4-bit rows, 32 rows 29.7 / 41.9, D = 64 22.0 / 34.3, 52 rows (128 caches of 9830) 130 / 73; fp32, 32
// caches of 4096 rows, D = 64, 64 rows 43.0 / 42.1, D = 128 78.4 / 65.5, 32 rows 47.2 / 59.9.  Here up to 64 rows are taken by pairs of
// wavefronts, each with half of a tile's keys: the 52 rows of 4 bits 73, without pairs 92.
TreeLaunch tree_launch(int type, int D, int rows, int n_cus) {
  TreeLaunch t;
  if (rows <= (type == 0 ? kStreamRows : kStreamRows / 2)) {
    t.ks = 0;
    t.row_tiles = 1;
    t.target = n_cus < kMostTreeItems ? n_cus : kMostTreeItems;
    return t;
  }
  t.ks = rows <= 64 ? 2 : 1;
  const int per = 32 * kWaves / t.ks;
  t.row_tiles = (rows + per - 1) / per;
  const int resident = tree_resident(type, D);
  const int all = resident * n_cus < kMostTreeItems ? resident * n_cus : kMostTreeItems;
  t.target = all / t.row_tiles > 1 ? all / t.row_tiles : 1;
  return t;
}

hipError_t launch_tree_attn(const TreeParams& p, const TreeLaunch& t, int type, int D, int n_caches, hipStream_t s) {
  const int64_t grid = ((int64_t)t.target + n_caches + 7) / 8 * 8 * t.row_tiles;  // (of 512 threads at most)
  const int merge_rows = (p.rows + kMergeRows - 1) / kMergeRows;
  if (grid > INT32_MAX / 512 || merge_rows > 65535) return hipErrorInvalidValue;
  hipError_t e = t.ks == 0   ? launch_tree_stream(p, type, D, t.target + n_caches, s)
                 : type == 1 ? D == 128 ? launch<1, 128>(p, t.ks, (unsigned)grid, s) : launch<1, 64>(p, t.ks, (unsigned)grid, s)
                 : type == 2 ? D == 128 ? launch<2, 128>(p, t.ks, (unsigned)grid, s) : launch<2, 64>(p, t.ks, (unsigned)grid, s)
                             : D == 128 ? launch<0, 128>(p, t.ks, (unsigned)grid, s) : launch<0, 64>(p, t.ks, (unsigned)grid, s);
  if (e != hipSuccess) return e;
  const dim3 mg((unsigned)n_caches, (unsigned)merge_rows);
  if (type == 1) {
    if (D == 128) tree_merge_kernel<128, true><<<mg, dim3(kThreads), 0, s>>>(p);
    else tree_merge_kernel<64, true><<<mg, dim3(kThreads), 0, s>>>(p);
  } else {
    if (D == 128) tree_merge_kernel<128, false><<<mg, dim3(kThreads), 0, s>>>(p);
    else tree_merge_kernel<64, false><<<mg, dim3(kThreads), 0, s>>>(p);
  }
  return hipGetLastError();
}

}  // namespace baklava
