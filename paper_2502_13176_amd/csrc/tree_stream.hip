// Attention of a tree of drafted tokens over ragged caches, few query rows (nodes times query heads of a KV head): up to 64, or 32
// (rule at tree_launch).
//
// Products, layouts and work items are those of tree.hip.  Here every wavefront takes all query rows, in one or (bf16) two blocks of 32, and
// streams slabs of 32 keys of its own, without a barrier: the K rows of its next slab are requested as soon as the first product
// has read the last ones, the V rows as soon as the second one has, so that its requests follow each other at any time and the
// wavefronts' do not come and go together.  bf16 and fp32 rows are copied straight to LDS.  Of 4-bit rows a lane takes half a row's
// codes, which are an operand of the first product once the head dimension is numbered that way; V's values pass through LDS to
// be transposed.  At the end the wavefronts' outputs are added up in LDS and leave as whole rows.
//
// HBM bounds it from some 100 MB on: 64 caches of 10240 bf16 rows, one query row, 59 us with the merge (335 MB, 47 at 7.1 TB/s).  Small
// calls are bound by their start: 8 caches of 4096 rows, 16 query rows, 11 us, of 64 rows 9: lengths, scan, first rows, drafted rows
// and the way out are a chain of memory latencies, and the code itself (some 10 KB, run through once) comes from memory too.
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

constexpr int kSlab = 32;
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLowest = -3.402823466e38f;
constexpr float kMaxSlack = 8.f;  // a logit may exceed its row's reference maximum by this much (log2 units)

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

constexpr int stream_waves(int type, int D) { return type == 1 && D == 128 ? 4 : 8; }

template <int TYPE, int D, int RB>
struct Shape {
  static constexpr bool kF32 = TYPE == 1, kMx = TYPE == 2;
  static constexpr int kRow = D * (kF32 ? 4 : 2);             // bytes of a row as the products take it
  static constexpr int kStored = kMx ? D / 2 : kRow;          // ... and in the arena
  static constexpr int kPieces = kRow / 16, kChunks = kPieces / 2, kBlocks = D / 32;
  static constexpr int kWaves = stream_waves(TYPE, D), kThreads = 64 * kWaves;
  static constexpr int kSlabBytes = kSlab * kRow;
  static constexpr int kArea = (kMx ? 1 : 2) * kSlabBytes;    // LDS of a wavefront: a slab of K, one of V
  static constexpr int kOut = kSlab * D * 4;                  // outputs of 32 query rows
  static constexpr int kLds = kWaves * (kArea > kOut ? kArea : kOut);
  static constexpr int kCopyRows = 64 / kPieces, kCopies = kSlab / kCopyRows;
  static constexpr int kWords = D / 16;                       // 4-bit rows: words of codes in half a row
  static constexpr int kAhead = kMx ? 2 : 1;                  // slabs on the way
  static constexpr bool kQueriesInLds = RB == 2;              // (registers run out)
  // piece of a row that lane half h takes as chunk c of the first product
  static __device__ __forceinline__ int piece(int c, int h) { return kMx ? h * kChunks + c : 2 * c + h; }
  // where piece x of row r lies in LDS
  static __device__ __forceinline__ int k_slot(int r, int x) { return kF32 || D == 128 ? x ^ (r & 15) : x ^ (r >> 1 & 7); }
  static __device__ __forceinline__ int v_slot(int r, int x) {
    if (kF32) return x ^ 8 * (r >> 2 & 1);
    // (values of 4-bit rows are written 16 bytes at a time, by lanes of few pieces of several rows: these spread, too)
    return D == 128 ? x ^ 4 * (r & 3) ^ (kMx ? (r ^ r >> 2) & 3 : 0) : x ^ 4 * (r >> 1 & 1);
  }
};

template <int TYPE, int D, int RB>
__global__ __launch_bounds__(64 * stream_waves(TYPE, D), stream_waves(TYPE, D) / 4) void tree_stream_kernel(TreeParams p) {
  using S = Shape<TYPE, D, RB>;
  constexpr int kBlocks = S::kBlocks, kRow = S::kRow, kWaves = S::kWaves, kChunks = S::kChunks;
  __shared__ __attribute__((aligned(16))) unsigned char lds[S::kLds];
  __shared__ __attribute__((aligned(16))) unsigned char lds_q[S::kQueriesInLds ? RB * 32 * kRow : 16];
  __shared__ unsigned long long above[kMostNodes / 64][kMostNodes];
  __shared__ float2 sums[kWaves][RB * 32];
  __shared__ int32_t scan[kWaves + 3];

  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n32 = lane & 31, jh = lane >> 5;
  // Slabs of live rows, then those of drafted rows.
  auto tiles = [&](int c) {
    const int n = tree_nodes(p, (uint32_t)c / (uint32_t)p.Hkv % (uint32_t)p.batch);
    return n > 0 ? (p.len[p.cache0 + c] + kSlab - 1) / kSlab + (n + kSlab - 1) / kSlab : 0;
  };
  Span sp;
  if (!find_span<S::kThreads>(p.n_caches, p.target, kWaves, blockIdx.x, tiles, scan, sp)) return;
  const int h = sp.c_rel % p.Hkv, s_rel = sp.c_rel / p.Hkv, b = s_rel % p.batch;
  const int n_nodes = __builtin_amdgcn_readfirstlane(tree_nodes(p, b)), n_rows = n_nodes * p.G;
  const int n_live = __builtin_amdgcn_readfirstlane(p.len[p.cache0 + sp.c_rel]), live_slabs = (n_live + kSlab - 1) / kSlab;
  const int64_t row0 = uniform(p.off[p.cache0 + sp.c_rel]);
  if (sp.part == 0 && tid == 0) p.table[sp.c_rel] = make_int2(sp.slot, sp.n_parts);
  const bool drafted = sp.last > live_slabs;
  int up = -1;  // (a parent that is no earlier node is none)
  if (drafted && tid < n_nodes) {
    up = p.parent[(int64_t)b * p.N + tid];
    if (up < 0 || up >= tid) up = -1;
  }

  // ---- query rows: lane (row, h), chunk c: piece(c, h) of row 32 rb + n32 --------------------------------------------
  int node[RB];
  u32x4_t qb[S::kQueriesInLds ? 1 : RB][kChunks];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = min(rb * 32 + n32, n_rows - 1);  // rows past the last repeat it and are not written
    node[rb] = row / p.G;
    if constexpr (!S::kQueriesInLds) {
      const unsigned char* src = row_of(p.q, s_rel, node[rb], h * p.G + row % p.G);
#pragma unroll
      for (int c = 0; c < kChunks; ++c) qb[rb][c] = *reinterpret_cast<const u32x4_t*>(src + S::piece(c, jh) * 16);
    }
  }
  if constexpr (S::kQueriesInLds) {
    for (int x = tid; x < RB * 32 * S::kPieces; x += S::kThreads) {
      const int r = x / S::kPieces, row = min(r, n_rows - 1), piece = x % S::kPieces;
      *reinterpret_cast<u32x4_t*>(lds_q + r * kRow + S::k_slot(r, piece) * 16) =
          *reinterpret_cast<const u32x4_t*>(row_of(p.q, s_rel, row / p.G, h * p.G + row % p.G) + piece * 16);
    }
  }

  // ---- requests ----------------------------------------------------------------------------------
  unsigned char* const my_v = lds + wave * S::kArea;
  unsigned char* const my_k = my_v + S::kSlabBytes;  // (not of 4-bit rows)
  const unsigned char* Kp = reinterpret_cast<const unsigned char*>(p.k_plane);
  const unsigned char* Vp = reinterpret_cast<const unsigned char*>(p.v_plane);
  uint32_t c_row[S::kCopies], k_off[S::kCopies], v_off[S::kCopies];
#pragma unroll
  for (int i = 0; i < S::kCopies; ++i) {
    c_row[i] = i * S::kCopyRows + lane / S::kPieces;
    k_off[i] = S::k_slot(c_row[i], lane % S::kPieces) * 16;
    v_off[i] = S::v_slot(c_row[i], lane % S::kPieces) * 16;
  }
  struct Codes {  // of half a row, with its scales
    u32x4_t c[S::kMx ? S::kWords / 4 : 1];
    uint32_t bytes;
  };
  // Rows past the last live one repeat it; they are masked.
  auto request = [&](Codes& codes, int value, int slab) {
    const uint32_t most = n_live - 1 - slab * kSlab;
    const int64_t first = row0 + (int64_t)slab * kSlab;
    const unsigned char* src = (value ? Vp : Kp) + first * S::kStored;
    if constexpr (S::kMx) {
      const uint32_t r = min((uint32_t)n32, most);
      const uint8_t* scale = p.kv_scale + first * (D / 16) + value * (D / 32);
#pragma unroll
      for (int i = 0; i < S::kWords / 4; ++i) codes.c[i] = *reinterpret_cast<const u32x4_t*>(src + (r * S::kStored + jh * (D / 4) + i * 16));
      codes.bytes = D == 128 ? *reinterpret_cast<const uint16_t*>(scale + (r * (D / 16) + jh * 2)) : scale[r * (D / 16) + jh];
    } else {
      const uint32_t dst = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)(value ? my_v : my_k);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (what lay there has been read)
#pragma unroll
      for (int i = 0; i < S::kCopies; ++i)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt"
                     :: "s"(dst + i * 1024), "v"(min(c_row[i], most) * (uint32_t)S::kStored + (value ? v_off[i] : k_off[i])), "s"(src) : "memory", "m0");
    }
  };
  // Waits for a request, behind which `later` others have been made.
  auto wait = [&](bool later) {
    if constexpr (!S::kMx) {
      if (later) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(S::kCopies) : "memory");
      else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
  };
  auto values = [&](const Codes& codes, int c) {  // chunk c of half a row
    const uint4 x = mx_values(codes.c[c / 4][c % 4], mx_scale(codes.bytes >> (8 * (c / 4)) & 255));
    return u32x4_t{x.x, x.y, x.z, x.w};
  };
  auto put_v = [&](const Codes& codes) {
    if constexpr (S::kMx) {
#pragma unroll
      for (int c = 0; c < kChunks; ++c)
        *reinterpret_cast<u32x4_t*>(my_v + n32 * kRow + S::v_slot(n32, jh * kChunks + c) * 16) = values(codes, c);
    }
  };

  // What lanes of the wavefront have written to LDS, or read there, before others read it or write there.  (LDS serves a wavefront in
  // order: this only keeps the compiler from moving accesses of different lanes past each other.)
  auto exchange = [&]() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };

  // ---- one slab ----------------------------------------------------------------------------------
  floatx16_t o[RB][kBlocks];  // lane (row, h), register i of block x: O[row][32 x + 8 (i / 4) + 4 h + i % 4]
  // Reference maximum of the exponent, log2 units.  It starts at the lowest finite value, so that a masked logit weighs 2^-inf = 0.
  float m_ref[RB], l_part[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    m_ref[rb] = kLowest;
    l_part[rb] = 0.f;
#pragma unroll
    for (int x = 0; x < kBlocks; ++x)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[rb][x][i] = 0.f;
  }
  const float cs = p.scale_log2e;
  auto query = [&](int rb, int c) {
    if constexpr (S::kQueriesInLds) return *reinterpret_cast<const u32x4_t*>(lds_q + (rb * 32 + n32) * kRow + S::k_slot(n32, S::piece(c, jh)) * 16);
    else return qb[rb][c];
  };
  auto logits = [&](floatx16_t (&s)[RB], const Codes& codes) {
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      u32x4_t a;
      if constexpr (S::kMx) a = values(codes, c);
      else a = *reinterpret_cast<const u32x4_t*>(my_k + n32 * kRow + S::k_slot(n32, 2 * c + jh) * 16);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const u32x4_t q = query(rb, c);
        const floatx16_t zero = {};
        if constexpr (S::kF32) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            s[rb] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[e]), __uint_as_float(q[e]), c == 0 && e == 0 ? zero : s[rb], 0, 0, 0);
        } else {
          s[rb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, q), c == 0 ? zero : s[rb], 0, 0, 0);
        }
      }
    }
  };
  // Lazy running maximum: a row's reference only moves when a logit exceeds it by more than kMaxSlack, so weights stay below
  // 2^kMaxSlack and the rescale of the accumulators is rare after the first slab.
  auto follow_max = [&](const floatx16_t (&s)[RB]) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      float mx = s[rb][0];
#pragma unroll
      for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[rb][i]);
      mx *= cs;
      if (__any(mx > m_ref[rb] + kMaxSlack)) {
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float mn = mx > m_ref[rb] + kMaxSlack ? mx : m_ref[rb];  // (a row's bits do not depend on the others)
        const float alpha = fast_exp2(m_ref[rb] - mn);
        m_ref[rb] = mn;
        l_part[rb] *= alpha;
#pragma unroll
        for (int x = 0; x < kBlocks; ++x) o[rb][x] *= alpha;
      }
    }
  };
  // Logits into weights, in place.
  auto weigh = [&](floatx16_t (&s)[RB]) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[rb][i] = fast_exp2(fmaf(s[rb][i], cs, -m_ref[rb]));
        l_part[rb] += s[rb][i];
      }
  };
  // finite: infinite and NaN values count as zero (see below).
  auto outputs = [&](const floatx16_t (&s)[RB], bool finite) {
    if constexpr (S::kF32) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = 8 * (i / 4) + 4 * jh + i % 4;
#pragma unroll
        for (int x = 0; x < kBlocks; ++x) {
          float v = *reinterpret_cast<const float*>(my_v + key * kRow + S::v_slot(key, 8 * x) * 16 + n32 * 4);
          if (finite && (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u) v = 0.f;
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) o[rb][x] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[rb][i], o[rb][x], 0, 0, 0);
        }
      }
    } else {
      const int n16 = lane & 15, half = (lane >> 4) & 1, k4 = n16 >> 2;
      const unsigned char* at0 = my_v + (4 * jh + k4) * kRow + (n16 & 1) * 8;
      const int piece = 2 * half + (n16 >> 1 & 1);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        bf16x8_t pb[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
          for (int e = 0; e < 8; ++e) pb[rb][e] = (__bf16)s[rb][8 * u + e];
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
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) o[rb][x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, v), pb[rb], o[rb][x], 0, 0, 0);
        }
      }
    }
  };

  // ---- live rows ---------------------------------------------------------------------------------
  const int live_end = min(sp.last, live_slabs);
  int slab = sp.first + wave;
  Codes ck[S::kAhead], cv[S::kAhead];
#pragma unroll
  for (int a = 0; a < S::kAhead; ++a)
    if (slab + a * kWaves < live_end) {
      request(ck[a], 0, slab + a * kWaves);
      request(cv[a], 1, slab + a * kWaves);
    }
  if (drafted) find_ancestors(up, n_nodes, above, reinterpret_cast<int32_t*>(sums));
  else if (S::kQueriesInLds) __syncthreads();
  static_assert(sizeof(sums) >= kMostNodes * 4, "a word for every node");
  auto one = [&](Codes& ck, Codes& cv) {
    const int ahead = slab + S::kAhead * kWaves;
    const bool more = ahead < live_end;
    floatx16_t s[RB];
    wait(true);
    logits(s, ck);
    if (more) request(ck, 0, ahead);
    if ((slab + 1) * kSlab > n_live) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (slab * kSlab + 8 * (i / 4) + 4 * jh + i % 4 >= n_live) s[rb][i] = kNegInf;
    }
    follow_max(s);
    weigh(s);
    put_v(cv);
    wait(more);
    if constexpr (S::kMx) exchange();
    if ((slab + 1) * kSlab > n_live) {  // (a weight of zero times an infinity of the row that was repeated would be NaN)
      if (slab * kSlab + n32 >= n_live) {
#pragma unroll
        for (int c = 0; c < kChunks; ++c) *reinterpret_cast<u32x4_t*>(my_v + n32 * kRow + (jh * kChunks + c) * 16) = u32x4_t{};
      }
      exchange();
    }
    outputs(s, false);
    if constexpr (S::kMx) exchange();  // (the next slab's values go there)
    if (more) request(cv, 1, ahead);
    slab += kWaves;
  };
  while (slab < live_end) {
    one(ck[0], cv[0]);
    if (S::kAhead > 1 && slab < live_end) one(ck[S::kAhead - 1], cv[S::kAhead - 1]);
  }

  // ---- drafted rows: a lane takes half a row ---------------------------------------------------------
  if (drafted) {
    int ds = max(sp.first - live_slabs, 0) + wave;
    for (; ds < sp.last - live_slabs; ds += kWaves) {
      const int j = min(ds * kSlab + n32, n_nodes - 1);  // rows past the last node repeat it; nobody sees them
      bool wild = false;  // an infinite or NaN value
      Codes codes[2] = {};
#pragma unroll
      for (int value = 0; value < 2; ++value) {
        const unsigned char* src = row_of(value ? p.v : p.k, s_rel, j, h) + jh * (kRow / 2);
        u32x4_t w[kChunks];
#pragma unroll
        for (int c = 0; c < kChunks; ++c) w[c] = *reinterpret_cast<const u32x4_t*>(src + c * 16);
        if (value) {
#pragma unroll
          for (int c = 0; c < kChunks; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              wild = wild || (w[c][i] & 0x7f800000u) == 0x7f800000u || (!S::kF32 && (w[c][i] & 0x7f80u) == 0x7f80u);
          wild = __any(wild);
        }
        if constexpr (S::kMx) {  // rounded to 4 bits, as they will be in a cache
#pragma unroll
          for (int sc = 0; sc < kChunks / 4; ++sc) {
            uint32_t top = 0;
#pragma unroll
            for (int c = 4 * sc; c < 4 * sc + 4; ++c)
#pragma unroll
              for (int i = 0; i < 4; ++i) top = max(top, max(w[c][i] & 0x7fffu, w[c][i] >> 16 & 0x7fffu));
            const uint32_t byte = mx_scale_byte(top);
            codes[value].bytes |= byte << (8 * sc);
#pragma unroll
            for (int c = 4 * sc; c < 4 * sc + 4; ++c) codes[value].c[c / 4][c % 4] = mx_codes(make_uint4(w[c][0], w[c][1], w[c][2], w[c][3]), byte);
          }
          if (value) put_v(codes[1]);
        } else {
#pragma unroll
          for (int c = 0; c < kChunks; ++c) {
            const int piece = jh * kChunks + c;
            if (value) *reinterpret_cast<u32x4_t*>(my_v + n32 * kRow + S::v_slot(n32, piece) * 16) = w[c];
            else *reinterpret_cast<u32x4_t*>(my_k + n32 * kRow + S::k_slot(n32, piece) * 16) = w[c];
          }
        }
      }
      exchange();
      floatx16_t s[RB];
      logits(s, codes[0]);
      uint32_t seen[RB];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        seen[rb] = (uint32_t)(above[ds / 2][node[rb]] >> (ds % 2 * 32));
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (!(seen[rb] >> (8 * (i / 4) + 4 * jh + i % 4) & 1)) s[rb][i] = kNegInf;
      }
      follow_max(s);
      weigh(s);
      outputs(s, wild);
      // An infinite or NaN value counts for the rows that see it, one by one: the product of a zero weight with it would reach all the
      // others.
      if (wild) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
          for (int jj = 0; jj < 32; ++jj) {
            float wt = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (8 * (i / 4) + i % 4 == (jj & ~4)) wt = s[rb][i];
            wt = __shfl(wt, n32 + 8 * (jj & 4));  // from the half that holds key jj
            if (!(seen[rb] >> jj & 1)) continue;
#pragma unroll
            for (int x = 0; x < kBlocks; ++x)
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const int d = 32 * x + 8 * (i / 4) + 4 * jh + i % 4;
                const unsigned char* src = my_v + jj * kRow + S::v_slot(jj, d * (S::kF32 ? 4 : 2) / 16) * 16;
                const float v = S::kF32 ? *reinterpret_cast<const float*>(src + d % 4 * 4)
                                        : __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(src + d % 8 * 2) << 16);
                if ((__float_as_uint(v) & 0x7f800000u) == 0x7f800000u) o[rb][x][i] = fmaf(wt, v, o[rb][x][i]);
              }
          }
      }
      exchange();  // (the area may be written again)
    }
  }

  // ---- the end of a work item: the wavefronts' sums, whole rows out --------------------------------
  __syncthreads();  // (jump words and slabs have been read)
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const float l = l_part[rb] + __shfl_xor(l_part[rb], 32);
    if (jh == 0) sums[wave][rb * 32 + n32] = make_float2(m_ref[rb], l);
  }
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    if (rb * 32 >= n_rows) break;
    if (rb > 0) __syncthreads();
    float* const mine = reinterpret_cast<float*>(lds + wave * S::kOut) + n32 * D;
#pragma unroll
    for (int x = 0; x < kBlocks; ++x)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        floatx4_t r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = o[rb][x][4 * q + i];
        const int piece = 8 * x + 2 * q + jh;
        *reinterpret_cast<floatx4_t*>(mine + (piece ^ (n32 & 15)) * 4) = r;
      }
    __syncthreads();
    const int rows = min(32, n_rows - rb * 32);
    for (int y = tid; y < rows * (D / 4); y += S::kThreads) {
      const int r = y / (D / 4), piece = y % (D / 4), row = rb * 32 + r;
      float m = kLowest;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) m = fmaxf(m, sums[w][row].x);
      float l = 0.f;
      floatx4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float2 ml = sums[w][row];
        const float a = fast_exp2(ml.x - m);
        l += ml.y * a;
        sum += *reinterpret_cast<const floatx4_t*>(reinterpret_cast<const float*>(lds + w * S::kOut) + r * D + (piece ^ (r & 15)) * 4) * a;
      }
      if (sp.n_parts > 1) {
        const int64_t at = (int64_t)(sp.slot + sp.part) * p.rows + row;
        if (piece == 0) p.part_ml[at] = make_float2(m, l);
        *reinterpret_cast<floatx4_t*>(p.part_o + at * D + piece * 4) = sum;
      } else {
        const int nd = row / p.G, head = h * p.G + row % p.G;
        if (p.lse.data && piece == 0) *reinterpret_cast<float*>(row_of(p.lse, s_rel, nd, head)) = m + __builtin_log2f(l);
        const float inv = 1.f / l;
        unsigned char* dst = row_of(p.out, s_rel, nd, head);
        if constexpr (S::kF32) {
          reinterpret_cast<floatx4_t*>(dst)[piece] = sum * inv;
        } else {
          bf16x4_t x;
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = (__bf16)(sum[i] * inv);
          reinterpret_cast<bf16x4_t*>(dst)[piece] = x;
        }
      }
    }
  }
}

template <int TYPE, int D>
hipError_t launch(const TreeParams& p, unsigned grid, hipStream_t s) {
  constexpr bool kOne = TYPE != 0;  // (rule at tree_launch)
  if (kOne || p.rows <= 32) tree_stream_kernel<TYPE, D, 1><<<dim3(grid), dim3(Shape<TYPE, D, 1>::kThreads), 0, s>>>(p);
  else if constexpr (!kOne) tree_stream_kernel<TYPE, D, 2><<<dim3(grid), dim3(Shape<TYPE, D, 2>::kThreads), 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_tree_stream(const TreeParams& p, int type, int D, int n_items, hipStream_t s) {
  const unsigned grid = (unsigned)n_items;
  return type == 1   ? D == 128 ? launch<1, 128>(p, grid, s) : launch<1, 64>(p, grid, s)
         : type == 2 ? D == 128 ? launch<2, 128>(p, grid, s) : launch<2, 64>(p, grid, s)
                     : D == 128 ? launch<0, 128>(p, grid, s) : launch<0, 64>(p, grid, s);
}

}  // namespace baklava
