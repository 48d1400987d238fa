// The accepted path of a tree of drafted tokens into the caches (baklava_append_accepted): its rows behind the live ones, and with
// score tracking the weights of its attention on every row.
//
// A cache's part: rows k[path[t]], v[path[t]] become rows n + t, and
//   score[j] += sum over path nodes t that see row j, and over the G heads, of 2^(q_t . k_j log2(e) / sqrt(D) - lse_t)
// One launch copies the rows and advances the lengths; with tracking a second one reads K, the new rows among it, once:
//
//   S[row, key] = Q[row, :] . K[key, :]     A = Q (row t * G + g of the path), B = K, blocks of 32 x 32
//
// so that a lane holds 16 rows' logits of one key, and a key's sum is 16 additions and one exchange between the lane halves.  Each
// wavefront streams slabs of 32 keys of its own, without a barrier; nothing is merged, so every workgroup takes as many tiles as any
// other, whichever caches they belong to.  HBM bounds it, K and the scores: 256 caches of 8200 bf16 rows, 20 query rows, 99 us (577 MB,
// 88 by a plain read; with a work item for each part of a cache, whose start takes some 10 us, 119).  4-bit rows 42 us (167 MB, 24): the
// chain of a slab (conversions, products one behind the other, exponentials) with four wavefronts to a SIMD.  fp32 rows, where 20 rows cost
// the products of 32: 128 caches of 8640, 124 us (578 MB, 82; the products 61 at the rate of a library product).
#include "common.h"

#include "mxfp4.h"
#include "tree.h"

namespace baklava {

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float floatx4_t __attribute__((ext_vector_type(4)));
typedef float floatx16_t __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kSlab = 32;

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Nodes on the accepted path of sequence b: as many as are given, up to the first that is no node.
__device__ __forceinline__ int path_nodes(const AcceptParams& p, int b) {
  const int most = min(max(p.n_path[b], 0), p.N), lane = threadIdx.x & 63;
  for (int t0 = 0; t0 < most; t0 += 64) {
    const int t = t0 + lane;
    const int node = t < most ? p.path[(int64_t)b * p.N + t] : 0;
    const unsigned long long bad = __ballot(node < 0 || node >= p.N);
    if (bad) return t0 + __builtin_ctzll(bad);
  }
  return most;
}

// PIECES: 16-byte pieces of a row as the caller holds it.  A workgroup for each cache.
template <int PIECES, bool MX>
__global__ __launch_bounds__(kThreads) void accept_rows_kernel(AcceptParams p) {
  const int c_rel = blockIdx.x, c = p.cache0 + c_rel, h = c_rel % p.Hkv, s_rel = c_rel / p.Hkv, b = s_rel % p.batch;
  const int tid = threadIdx.x;
  int n = path_nodes(p, b);
  const int n_old = p.len[c];
  if (n > p.cap[c] - n_old) {  // no room: the cache stays as it is
    if (tid == 0) *p.status = 1;
    n = 0;
  }
  if (p.table && tid == 0) p.table[c_rel] = make_int2(n_old, n);
  if (n == 0) return;
  const int64_t row0 = p.off[c] + n_old;
  for (int x = tid; x < n * PIECES; x += kThreads) {
    const int t = x / PIECES, piece = x % PIECES;
    const int node = p.path[(int64_t)b * p.N + t];
    const uint4 k = reinterpret_cast<const uint4*>(p.k.data)[s_rel * p.k.seq + node * p.k.tok + h * p.k.head + piece];
    const uint4 v = reinterpret_cast<const uint4*>(p.v.data)[s_rel * p.v.seq + node * p.v.tok + h * p.v.head + piece];
    if constexpr (MX) {  // (whole rows: all lanes of a quad take part)
      mx_store<PIECES * 8>(k, piece, p.k_plane, p.kv_scale, row0 + t, 0);
      mx_store<PIECES * 8>(v, piece, p.v_plane, p.kv_scale, row0 + t, 1);
    } else {
      reinterpret_cast<uint4*>(p.k_plane)[(row0 + t) * PIECES + piece] = k;
      reinterpret_cast<uint4*>(p.v_plane)[(row0 + t) * PIECES + piece] = v;
    }
  }
  for (int t = tid; t < n; t += kThreads) {
    p.score[row0 + t] = 0.f;
    p.pos[row0 + t] = p.pos0[b] + t;
  }
  __syncthreads();  // (every wavefront has read the length)
  if (tid == 0) p.len[c] = n_old + n;
}

// TYPE: BAKLAVA_BF16, F32, MXFP4.
constexpr int score_waves(int type, int D) { return type == 1 && D == 128 ? 4 : 8; }
template <int TYPE, int D>
struct Shape {
  static constexpr bool kF32 = TYPE == 1, kMx = TYPE == 2;
  static constexpr int kWaves = score_waves(TYPE, D), kThreads = 64 * kWaves;
  static constexpr int kRow = D * (kF32 ? 4 : 2);       // bytes of a query row, and of a key row unless it has 4-bit elements
  static constexpr int kPieces = kRow / 16, kChunks = kPieces / 2;
  static constexpr int kAhead = 2;                      // slabs of a wavefront on the way
  // 4-bit rows are little to wait for and much to compute: query rows in LDS leave room for twice as many wavefronts.
  static constexpr bool kQueriesInLds = kMx;
  static constexpr int kResident = kMx ? 2 : 1;         // workgroups of a compute unit
  static constexpr int kStored = kMx ? D / 2 : kRow;    // bytes of a row in the arena
  static constexpr int kStage = kSlab * kStored;        // bytes of a staged slab
  static constexpr int kRing = 8;                       // slabs of a wavefront whose new scores wait in LDS
  static constexpr int kCopyPieces = kStored / 16, kCopyRows = 64 / kCopyPieces, kCopies = kSlab / kCopyRows;
  static constexpr int kRequests = kCopies + (kMx ? 2 : 1);  // load instructions of a slab: rows, scores, scales
  // 4-bit rows: a lane takes one half of a row's codes, elements h D / 2 .. of it: chunk c is word c.
  static constexpr int kWords = D / 16;
  // piece of a row that lane half h takes as chunk c
  static __device__ __forceinline__ int piece(int c, int h) { return kMx ? h * kChunks + c : 2 * c + h; }
  // where piece x of a stored row lies in LDS
  static __device__ __forceinline__ int slot(int row, int x) {
    if (kMx) return D == 128 ? x ^ (row >> 2 & 3) : x ^ (row >> 3 & 1);
    return q_slot(row, x);
  }
  static __device__ __forceinline__ int q_slot(int row, int x) { return kF32 || D == 128 ? x ^ (row & 15) : x ^ (row >> 1 & 7); }
};

template <int TYPE, int D>
__global__ __launch_bounds__(64 * score_waves(TYPE, D), score_waves(TYPE, D) / 4 * (TYPE == 2 ? 2 : 1)) void accept_scores_kernel(AcceptParams p) {
  using S = Shape<TYPE, D>;
  constexpr int kWaves = S::kWaves, kTile = kWaves * kSlab;
  __shared__ __attribute__((aligned(16))) unsigned char lds[kWaves * S::kAhead * S::kStage];
  __shared__ float lds_score[kWaves * S::kAhead * 64];
  __shared__ uint32_t lds_scale[S::kMx ? kWaves * S::kAhead * 64 : 1];
  __shared__ float ring[kWaves * S::kRing * kSlab];
  __shared__ __attribute__((aligned(16))) float lse[64];  // of the query rows in registers (or LDS)
  __shared__ __attribute__((aligned(16))) unsigned char lds_q[S::kQueriesInLds ? 64 * S::kRow : 16];
  __shared__ int32_t scan[kWaves + 3];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n32 = lane & 31, jh = lane >> 5;
  auto tiles = [&](int c) {
    const int2 t = p.table[c];
    return t.y > 0 ? (t.x + t.y + kTile - 1) / kTile : 0;
  };
  int c_rel, tile, total, left = 0;
  auto first_tile = [&](int total) {  // every workgroup takes as many tiles
    left = __builtin_amdgcn_readfirstlane(ceil_div(total, gridDim.x));
    return (int)blockIdx.x * left;
  };
  if (!find_tile<S::kThreads>(p.n_caches, tiles, first_tile, scan, c_rel, tile, total)) return;
  left = min(left, total - (int)blockIdx.x * left);
  const float cs = p.scale_log2e;
  const unsigned char* Kp = reinterpret_cast<const unsigned char*>(p.k_plane);
  uint32_t off[S::kCopies], c_row[S::kCopies];
#pragma unroll
  for (int i = 0; i < S::kCopies; ++i) {
    c_row[i] = i * S::kCopyRows + lane / S::kCopyPieces;
    off[i] = S::slot(c_row[i], lane % S::kCopyPieces) * 16;
  }
  float* const mine = ring + wave * S::kRing * kSlab;

  for (;; ++c_rel, tile = 0) {  // the caches it has a part of
    const int2 t = p.table[c_rel];
    const int n_old = __builtin_amdgcn_readfirstlane(t.x), n_path = __builtin_amdgcn_readfirstlane(t.y);
    if (n_path == 0) continue;  // (tiles are left, so there is another cache)
    const int64_t row0 = uniform(p.off[p.cache0 + c_rel]);
    const int n = n_old + n_path, n_rows = n_path * p.G, n_blocks = (n_rows + 31) / 32;
    const int tile_end = min(tile + left, (n + kTile - 1) / kTile);
    left -= tile_end - tile;
    const int slab_end = min(tile_end * kWaves, (n + kSlab - 1) / kSlab);
    // Rows, scores and scales of a slab, straight to LDS.  (Codes are read with the ordinary hint: a cache line of theirs is asked for
    // by two instructions, and is fetched twice without a stay in the cache, 53 / 58 us.)
    auto request = [&](int buf, int slab) {
      const uint32_t most = n - 1 - slab * kSlab;  // rows past the last repeat it
      const int64_t first = row0 + (int64_t)slab * kSlab;
      const uint32_t at = wave * S::kAhead + buf;
      const uint32_t dst = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds + at * S::kStage;
      const uint32_t dst_score = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) float*)lds_score + at * 256;
      const unsigned char* src = Kp + first * S::kStored;
      const float* src_score = p.score + first;
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (what lay there has been read)
#pragma unroll
      for (int i = 0; i < S::kCopies; ++i) {
        const uint32_t from = min(c_row[i], most) * (uint32_t)S::kStored + off[i];
        if constexpr (S::kMx)
          asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(dst + i * 1024), "v"(from), "s"(src) : "memory", "m0");
        else
          asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" :: "s"(dst + i * 1024), "v"(from), "s"(src) : "memory", "m0");
      }
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
                   :: "s"(dst_score), "v"(min((uint32_t)n32, most) * 4), "s"(src_score) : "memory", "m0");
      if constexpr (S::kMx) {  // a row's D / 16 scale bytes: two words or one
        const uint8_t* src_scale = p.kv_scale + first * (D / 16);
        const uint32_t dst_scale = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint32_t*)lds_scale + at * 256;
        const uint32_t r = D == 128 ? lane / 2 : n32, from = min(r, most) * (D / 16) + (D == 128 ? lane % 2 * 4 : 0);
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" :: "s"(dst_scale), "v"(from), "s"(src_scale) : "memory", "m0");
      }
    };
    int slab = tile * kWaves + wave;
#pragma unroll
    for (int a = 0; a < S::kAhead; ++a)
      if (slab + a * kWaves < slab_end) request(a, slab + a * kWaves);

    // Query row r of the path; rows past the last repeat it and weigh nothing.
    const int h = (uint32_t)c_rel % (uint32_t)p.Hkv, s_rel = (uint32_t)c_rel / (uint32_t)p.Hkv, b = (uint32_t)s_rel % (uint32_t)p.batch;
    const int32_t* const path = p.path + (int64_t)b * p.N;
    auto load_q = [&](u32x4_t (&qa)[S::kChunks], int r0) {
      const uint32_t at = min(r0 + n32, n_rows - 1);
      const unsigned char* src = row_of(p.q, s_rel, path[at / (uint32_t)p.G], h * p.G + at % (uint32_t)p.G);
#pragma unroll
      for (int c = 0; c < S::kChunks; ++c) qa[c] = *reinterpret_cast<const u32x4_t*>(src + S::piece(c, jh) * 16);
    };
    auto lse_of = [&](int r) {
      return r < n_rows ? *reinterpret_cast<const float*>(row_of(p.lse, s_rel, path[(uint32_t)r / (uint32_t)p.G], h * p.G + (uint32_t)r % (uint32_t)p.G))
                        : __builtin_huge_valf();
    };
    u32x4_t qa[S::kQueriesInLds ? 1 : 2][S::kChunks];
    if constexpr (!S::kQueriesInLds) {
      load_q(qa[0], 0);
      if (n_blocks > 1) load_q(qa[1], 32);
    }
    __syncthreads();  // (what the cache before needed has been read)
    if (tid < 64) lse[tid] = lse_of(tid);
    if constexpr (S::kQueriesInLds) {
      for (int x = tid; x < min(n_blocks, 2) * 32 * S::kPieces; x += S::kThreads) {  // (rows past the last repeat it)
        const uint32_t r = x / S::kPieces, piece = x % S::kPieces, at = min(r, (uint32_t)n_rows - 1);
        *reinterpret_cast<u32x4_t*>(lds_q + r * S::kRow + S::q_slot(r, piece) * 16) =
            *reinterpret_cast<const u32x4_t*>(row_of(p.q, s_rel, path[at / (uint32_t)p.G], h * p.G + at % (uint32_t)p.G) + piece * 16);
      }
    }
    __syncthreads();
    // register i of a block's logits: row 32 blk + 8 (i / 4) + 4 h + i % 4; a path's row j is seen by its nodes from j on
    auto product = [&](floatx16_t& s, const u32x4_t& q, const u32x4_t& k, bool first) {
      const floatx16_t zero = {};
      if constexpr (S::kF32) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(q[e]), __uint_as_float(k[e]), first && e == 0 ? zero : s, 0, 0, 0);
      } else {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, q), __builtin_bit_cast(bf16x8_t, k), first ? zero : s, 0, 0, 0);
      }
    };
    auto weights = [&](const floatx16_t& s, int blk, int slab, float& sum) {
      const float* z = lse + blk * 32 + 4 * jh;
      const bool fresh = (slab + 1) * kSlab > n_old;  // new rows among them
      const int first_row = fresh ? (slab * kSlab + n32 - n_old) * p.G - blk * 32 - 4 * jh : INT32_MIN;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (blk * 32 + 8 * q >= n_rows) break;
        const floatx4_t y = *reinterpret_cast<const floatx4_t*>(z + 8 * q);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float w = fast_exp2(fmaf(s[4 * q + i], cs, -y[i]));
          sum += 8 * q + i >= first_row ? w : 0.f;
        }
      }
    };
    // Blocks beyond those two, of long paths: their rows and normalisers come from memory, again for every slab.
    auto weights_of_far_rows = [&](const floatx16_t& s, int blk, int slab, float& sum) {
      const int first_row = max(slab * kSlab + n32 - n_old, 0) * p.G - blk * 32 - 4 * jh;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int r = 8 * (i / 4) + i % 4;
        const float w = fast_exp2(fmaf(s[i], cs, -lse_of(blk * 32 + 4 * jh + r)));
        sum += r >= first_row ? w : 0.f;
      }
    };
    // New scores are stored several slabs at a time: whoever waits for a load also waits for the stores in front of it.
    int waiting = 0;
    auto store = [&](int first) {
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      for (int i = lane; i < waiting * kSlab; i += 64) {
        const int row = (first + i / kSlab * kWaves) * kSlab + i % kSlab;
        if (row < n) p.score[row0 + row] = mine[i];
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();  // (the ring may be written again)
      waiting = 0;
    };
    for (int buf = 0; slab < slab_end; slab += kWaves) {
      // (loads come back in order: with as many outstanding as have been asked for behind them, stores among them or not, this slab's
      // are there)
      if (slab + (S::kAhead - 1) * kWaves < slab_end) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(S::kRequests * (S::kAhead - 1)) : "memory");
      else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      const int at = wave * S::kAhead + buf;
      const unsigned char* src = lds + at * S::kStage + n32 * S::kStored;
      u32x4_t codes[S::kMx ? S::kWords / 4 : 1];  // half a row's
      uint32_t bytes = 0;
      if constexpr (S::kMx) {
#pragma unroll
        for (int i = 0; i < S::kWords / 4; ++i) codes[i] = *reinterpret_cast<const u32x4_t*>(src + S::slot(n32, jh * (S::kWords / 4) + i) * 16);
        bytes = D == 128 ? lds_scale[at * 64 + n32 * 2] >> (16 * jh) : lds_scale[at * 64 + n32] >> (8 * jh);
      }
      auto key = [&](int c) {  // chunk c of row n32 of the slab
        if constexpr (S::kMx) {
          const uint4 x = mx_values(codes[c / 4][c % 4], mx_scale(bytes >> (8 * (c / 4)) & 255));
          return u32x4_t{x.x, x.y, x.z, x.w};
        } else {
          return *reinterpret_cast<const u32x4_t*>(src + S::slot(n32, 2 * c + jh) * 16);
        }
      };
      const float before = lds_score[at * 64 + n32];
      float sum = 0.f;
      floatx16_t s0;
      auto far_rows = [&]() {
#pragma unroll 1
        for (int blk = 2; blk < n_blocks; ++blk) {
          u32x4_t q[S::kChunks];
          load_q(q, blk * 32);
#pragma unroll
          for (int c = 0; c < S::kChunks; ++c) product(s0, q[c], key(c), c == 0);
          weights_of_far_rows(s0, blk, slab, sum);
        }
      };
      const int ahead = slab + S::kAhead * kWaves;
      if constexpr (S::kQueriesInLds) {  // (the codes are in registers)
        if (ahead < slab_end) request(buf, ahead);
#pragma unroll 1
        for (int blk = 0; blk < min(n_blocks, 2); ++blk) {
#pragma unroll
          for (int c = 0; c < S::kChunks; ++c)
            product(s0, *reinterpret_cast<const u32x4_t*>(lds_q + (blk * 32 + n32) * S::kRow + S::q_slot(n32, S::piece(c, jh)) * 16), key(c), c == 0);
          weights(s0, blk, slab, sum);
        }
        far_rows();
      } else {
        floatx16_t s1;
        if (n_blocks == 1) {
#pragma unroll
          for (int c = 0; c < S::kChunks; ++c) product(s0, qa[0][c], key(c), c == 0);
        } else {
#pragma unroll
          for (int c = 0; c < S::kChunks; ++c) {
            const u32x4_t k = key(c);
            product(s0, qa[0][c], k, c == 0);
            product(s1, qa[1][c], k, c == 0);
          }
        }
        if (n_blocks <= 2 && ahead < slab_end) request(buf, ahead);
        weights(s0, 0, slab, sum);
        if (n_blocks > 1) weights(s1, 1, slab, sum);
        if (n_blocks > 2) {
          far_rows();
          if (ahead < slab_end) request(buf, ahead);
        }
      }
      buf = buf + 1 == S::kAhead ? 0 : buf + 1;
      sum += __shfl_xor(sum, 32);
      if (jh == 0) mine[waiting * kSlab + n32] = before + sum;
      if (++waiting == S::kRing) store(slab - (S::kRing - 1) * kWaves);
    }
    if (waiting > 0) store(slab - waiting * kWaves);
    if (left == 0) break;
  }
}

template <int TYPE, int D>
hipError_t launch_scores(const AcceptParams& p, unsigned grid, hipStream_t s) {
  static_assert(Shape<TYPE, D>::kResident == (TYPE == 2 ? 2 : 1), "");
  accept_scores_kernel<TYPE, D><<<dim3(grid), dim3(Shape<TYPE, D>::kThreads), 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_append_accepted(const AcceptParams& p, int type, int D, int n_cus, hipStream_t s) {
  const dim3 g((unsigned)p.n_caches), b(kThreads);
  if (type == 2) {
    if (D == 128) accept_rows_kernel<16, true><<<g, b, 0, s>>>(p);
    else accept_rows_kernel<8, true><<<g, b, 0, s>>>(p);
  } else {
    const int pieces = D * (type == 1 ? 4 : 2) / 16;
    if (pieces == 32) accept_rows_kernel<32, false><<<g, b, 0, s>>>(p);
    else if (pieces == 16) accept_rows_kernel<16, false><<<g, b, 0, s>>>(p);
    else accept_rows_kernel<8, false><<<g, b, 0, s>>>(p);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !p.table) return e;
  const unsigned grid = (unsigned)n_cus * (type == 2 ? 2 : 1);  // one round
  return type == 1   ? D == 128 ? launch_scores<1, 128>(p, grid, s) : launch_scores<1, 64>(p, grid, s)
         : type == 2 ? D == 128 ? launch_scores<2, 128>(p, grid, s) : launch_scores<2, 64>(p, grid, s)
                     : D == 128 ? launch_scores<0, 128>(p, grid, s) : launch_scores<0, 64>(p, grid, s);
}

}  // namespace baklava
