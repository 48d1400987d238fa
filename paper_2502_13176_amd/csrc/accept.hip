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
// wavefront streams slabs of 32 keys of its own, without a barrier.  HBM bounds it: K and the scores.
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
  static constexpr int kAhead = kMx ? 3 : 2;            // slabs of a wavefront on the way
  static constexpr int kStage = kMx ? 0 : kSlab * kRow; // bytes of a staged slab
  static constexpr int kRing = kMx ? 32 : 8;            // slabs of a wavefront whose new scores wait in LDS
  static constexpr int kCopyRows = 64 / kPieces, kCopies = kSlab / kCopyRows;
  // 4-bit rows: a lane takes one half of a row's codes, elements h D / 2 .. of it: chunk c is word c.
  static constexpr int kWords = D / 16;
  // piece of a row that lane half h takes as chunk c
  static __device__ __forceinline__ int piece(int c, int h) { return kMx ? h * kChunks + c : 2 * c + h; }
  static __device__ __forceinline__ int slot(int row, int x) { return kF32 || D == 128 ? x ^ (row & 15) : x ^ (row >> 1 & 7); }
};

template <int TYPE, int D>
__global__ __launch_bounds__(64 * score_waves(TYPE, D), score_waves(TYPE, D) / 4) void accept_scores_kernel(AcceptParams p) {
  using S = Shape<TYPE, D>;
  constexpr int kWaves = S::kWaves, kTile = kWaves * kSlab;
  __shared__ __attribute__((aligned(16))) unsigned char lds[S::kMx ? 16 : kWaves * S::kAhead * S::kStage];
  __shared__ float lds_score[S::kMx ? 1 : kWaves * S::kAhead * 64];
  __shared__ float ring[kWaves * S::kRing * kSlab];
  __shared__ __attribute__((aligned(16))) float lse[kAcceptRows];
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
    c_row[i] = i * S::kCopyRows + lane / S::kPieces;
    off[i] = S::slot(c_row[i], lane % S::kPieces) * 16;
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
  struct Request {  // 4-bit rows: a lane's codes with their scales, and the score of row n32; others are on their way to LDS
    u32x4_t codes[S::kMx ? S::kWords / 4 : 1];
    uint32_t bytes;
    float score;
  } rq[S::kAhead];
  auto request = [&](Request& r, int buf, int slab) {
    const uint32_t most = n - 1 - slab * kSlab;  // rows past the last repeat it
    const int64_t first = row0 + (int64_t)slab * kSlab;
    const uint32_t at = min((uint32_t)n32, most);
    if constexpr (S::kMx) {
      const unsigned char* src = Kp + first * (D / 2);
      const uint8_t* scale = p.kv_scale + first * (D / 16);
#pragma unroll
      for (int i = 0; i < S::kWords / 4; ++i) r.codes[i] = *reinterpret_cast<const u32x4_t*>(src + (at * (D / 2) + jh * (D / 4) + i * 16));
      r.bytes = D == 128 ? *reinterpret_cast<const uint16_t*>(scale + (at * (D / 16) + jh * 2)) : scale[at * (D / 16) + jh];
      r.score = p.score[first + at];
    } else {
      const uint32_t dst = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds + (wave * S::kAhead + buf) * S::kStage;
      const uint32_t dst_score = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) float*)lds_score + (wave * S::kAhead + buf) * 256;
      const unsigned char* src = Kp + first * S::kRow;
      const float* src_score = p.score + first;
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (what lay there has been read)
#pragma unroll
      for (int i = 0; i < S::kCopies; ++i)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                     :: "s"(dst + i * 1024), "v"(min(c_row[i], most) * (uint32_t)S::kRow + off[i]), "s"(src) : "memory", "m0");
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" :: "s"(dst_score), "v"(at * 4), "s"(src_score) : "memory", "m0");
    }
  };
  int slab = tile * kWaves + wave;
#pragma unroll
  for (int a = 0; a < S::kAhead; ++a)
    if (slab + a * kWaves < slab_end) request(rq[a], a, slab + a * kWaves);

  // Query row r of the path; rows past the last repeat it and weigh nothing.
  const int h = (uint32_t)c_rel % (uint32_t)p.Hkv, s_rel = (uint32_t)c_rel / (uint32_t)p.Hkv, b = (uint32_t)s_rel % (uint32_t)p.batch;
  const int32_t* const path = p.path + (int64_t)b * p.N;
  auto load_q = [&](u32x4_t (&qa)[S::kChunks], int r0) {
    const uint32_t at = min(r0 + n32, n_rows - 1);
    const unsigned char* src = row_of(p.q, s_rel, path[at / (uint32_t)p.G], h * p.G + at % (uint32_t)p.G);
#pragma unroll
    for (int c = 0; c < S::kChunks; ++c) qa[c] = *reinterpret_cast<const u32x4_t*>(src + S::piece(c, jh) * 16);
  };
  u32x4_t qa[2][S::kChunks];
  load_q(qa[0], 0);
  if (n_blocks > 1) load_q(qa[1], 32);
  __syncthreads();  // (the normalisers of the cache before have been read)
  for (int r = tid; r < n_blocks * 32; r += S::kThreads)
    lse[r] = r < n_rows ? *reinterpret_cast<const float*>(row_of(p.lse, s_rel, path[(uint32_t)r / (uint32_t)p.G], h * p.G + (uint32_t)r % (uint32_t)p.G))
                        : __builtin_huge_valf();
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
    if ((slab + 1) * kSlab > n_old) {
      const int first_row = (slab * kSlab + n32 - n_old) * p.G - blk * 32 - 4 * jh;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float w = fast_exp2(fmaf(s[i], cs, -z[8 * (i / 4) + i % 4]));
        sum += 8 * (i / 4) + i % 4 >= first_row ? w : 0.f;
      }
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const floatx4_t y = *reinterpret_cast<const floatx4_t*>(z + 8 * q);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += fast_exp2(fmaf(s[4 * q + i], cs, -y[i]));
      }
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
    if constexpr (!S::kMx) {
      // (loads come back in order: with that many outstanding, stores among them or not, this slab's are there)
      if (slab + (S::kAhead - 1) * kWaves < slab_end) asm volatile("s_waitcnt vmcnt(%0)" :: "n"((S::kCopies + 1) * (S::kAhead - 1)) : "memory");
      else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    const unsigned char* src = lds + (wave * S::kAhead + buf) * S::kStage + n32 * S::kRow;
    auto key = [&](int c) {  // chunk c of row n32 of the slab
      if constexpr (S::kMx) {
        const uint4 x = mx_values(rq[0].codes[c / 4][c % 4], mx_scale(rq[0].bytes >> (8 * (c / 4)) & 255));
        return u32x4_t{x.x, x.y, x.z, x.w};
      } else {
        return *reinterpret_cast<const u32x4_t*>(src + S::slot(n32, 2 * c + jh) * 16);
      }
    };
    const float before = S::kMx ? rq[0].score : lds_score[(wave * S::kAhead + buf) * 64 + n32];
    float sum = 0.f;
    floatx16_t s0, s1;
    if (n_blocks == 1) {
#pragma unroll
      for (int c = 0; c < S::kChunks; ++c) product(s0, qa[0][c], key(c), c == 0);
    } else if (n_blocks == 2) {
#pragma unroll
      for (int c = 0; c < S::kChunks; ++c) {
        const u32x4_t k = key(c);
        product(s0, qa[0][c], k, c == 0);
        product(s1, qa[1][c], k, c == 0);
      }
    } else {  // query rows beyond those in registers: from memory, again for every slab
#pragma unroll 1
      for (int blk = 0; blk < n_blocks; ++blk) {
        load_q(qa[0], blk * 32);
#pragma unroll
        for (int c = 0; c < S::kChunks; ++c) product(s0, qa[0][c], key(c), c == 0);
        weights(s0, blk, slab, sum);
      }
    }
    const int ahead = slab + S::kAhead * kWaves;
    if constexpr (S::kMx) {
#pragma unroll
      for (int a = 0; a + 1 < S::kAhead; ++a) rq[a] = rq[a + 1];
      if (ahead < slab_end) request(rq[S::kAhead - 1], 0, ahead);
    } else {
      if (ahead < slab_end) request(rq[0], buf, ahead);
      buf = buf + 1 == S::kAhead ? 0 : buf + 1;
    }
    if (n_blocks <= 2) weights(s0, 0, slab, sum);
    if (n_blocks == 2) weights(s1, 1, slab, sum);
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
  const unsigned grid = (unsigned)n_cus;
  return type == 1   ? D == 128 ? launch_scores<1, 128>(p, grid, s) : launch_scores<1, 64>(p, grid, s)
         : type == 2 ? D == 128 ? launch_scores<2, 128>(p, grid, s) : launch_scores<2, 64>(p, grid, s)
                     : D == 128 ? launch_scores<0, 128>(p, grid, s) : launch_scores<0, 64>(p, grid, s);
}

}  // namespace baklava
