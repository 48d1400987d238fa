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

constexpr int kWaves = 4, kThreads = 64 * kWaves, kSlab = 32, kTile = kWaves * kSlab;

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
template <int TYPE, int D>
struct Shape {
  static constexpr bool kF32 = TYPE == 1, kMx = TYPE == 2;
  static constexpr int kRow = D * (kF32 ? 4 : 2);       // bytes of a query row, and of a key row unless it has 4-bit elements
  static constexpr int kPieces = kRow / 16, kChunks = kPieces / 2;
  static constexpr int kStage = kMx ? 0 : kSlab * kRow; // bytes of a staged slab
  static constexpr int kCopyRows = 64 / kPieces, kCopies = kSlab / kCopyRows;
  // 4-bit rows: a lane takes one half of a row's codes, elements h D / 2 .. of it: chunk c is word c.
  static constexpr int kWords = D / 16;
  // piece of a row that lane half h takes as chunk c
  static __device__ __forceinline__ int piece(int c, int h) { return kMx ? h * kChunks + c : 2 * c + h; }
  static __device__ __forceinline__ int slot(int row, int x) { return kF32 || D == 128 ? x ^ (row & 15) : x ^ (row >> 1 & 7); }
};

template <int TYPE, int D>
__global__ __launch_bounds__(kThreads, 2) void accept_scores_kernel(AcceptParams p) {
  using S = Shape<TYPE, D>;
  __shared__ __attribute__((aligned(16))) unsigned char lds[S::kMx ? 16 : kWaves * 2 * S::kStage];
  __shared__ __attribute__((aligned(16))) float lse[kAcceptRows];
  __shared__ int32_t scan[kWaves + 3];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n32 = lane & 31, jh = lane >> 5;
  auto tiles = [&](int c) {
    const int2 t = p.table[c];
    return t.y > 0 ? (t.x + t.y + kTile - 1) / kTile : 0;
  };
  Span sp;
  if (!find_span<kThreads>(p.n_caches, p.target, 1, blockIdx.x, tiles, scan, sp)) return;
  const int h = sp.c_rel % p.Hkv, s_rel = sp.c_rel / p.Hkv, b = s_rel % p.batch;
  const int2 t = p.table[sp.c_rel];
  const int n_old = __builtin_amdgcn_readfirstlane(t.x), n_path = __builtin_amdgcn_readfirstlane(t.y);
  const int n = n_old + n_path, n_rows = n_path * p.G;
  const int64_t row0 = uniform(p.off[p.cache0 + sp.c_rel]);
  const int32_t* const path = p.path + (int64_t)b * p.N;
  const float cs = p.scale_log2e;

  // Where query row r of the path lies; rows past the last repeat it and weigh nothing.
  auto query = [&](int r) {
    const int at = min(r, n_rows - 1), tt = at / p.G;
    return reinterpret_cast<const unsigned char*>(p.q.data) + s_rel * p.q.seq + path[tt] * p.q.tok + (h * p.G + at % p.G) * p.q.head;
  };
  auto load_q = [&](u32x4_t (&qa)[S::kChunks], int r0) {
    const unsigned char* src = query(r0 + n32);
#pragma unroll
    for (int c = 0; c < S::kChunks; ++c) qa[c] = *reinterpret_cast<const u32x4_t*>(src + S::piece(c, jh) * 16);
  };

  const int slab_end = min(sp.last * kWaves, (n + kSlab - 1) / kSlab);
  const unsigned char* Kp = reinterpret_cast<const unsigned char*>(p.k_plane);
  u32x4_t codes[S::kMx ? S::kWords / 4 : 1];
  uint32_t bytes = 0;  // scales of this lane's half row
  float old = 0.f;     // score of row n32 of the requested slab
  uint32_t off[S::kCopies], c_row[S::kCopies];
#pragma unroll
  for (int i = 0; i < S::kCopies; ++i) {
    c_row[i] = i * S::kCopyRows + lane / S::kPieces;
    off[i] = S::slot(c_row[i], lane % S::kPieces) * 16;
  }
  auto request = [&](int slab) {
    const uint32_t most = n - 1 - slab * kSlab;  // rows past the last repeat it
    const int64_t first = row0 + (int64_t)slab * kSlab;
    old = p.score[first + min((uint32_t)n32, most)];
    if constexpr (S::kMx) {
      const int64_t r = first + min((uint32_t)n32, most);
#pragma unroll
      for (int i = 0; i < S::kWords / 4; ++i) codes[i] = *reinterpret_cast<const u32x4_t*>(Kp + r * (D / 2) + jh * (D / 4) + i * 16);
      if (D == 128) bytes = *reinterpret_cast<const uint16_t*>(p.kv_scale + r * (D / 16) + jh * 2);
      else bytes = p.kv_scale[r * (D / 16) + jh];
    } else {
      const uint32_t dst = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds +
                           (wave * 2 + (slab / kWaves & 1)) * S::kStage;
      const unsigned char* src = Kp + first * S::kRow;
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (what lay there has been read)
#pragma unroll
      for (int i = 0; i < S::kCopies; ++i)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                     :: "s"(dst + i * 1024), "v"(min(c_row[i], most) * (uint32_t)S::kRow + off[i]), "s"(src) : "memory", "m0");
    }
  };

  int slab = sp.first * kWaves + wave;
  if (slab < slab_end) request(slab);
  for (int r = tid; r < (n_rows + 31) / 32 * 32; r += kThreads) {
    float x = __builtin_huge_valf();
    if (r < n_rows) {
      const int tt = r / p.G;
      x = *reinterpret_cast<const float*>(reinterpret_cast<const unsigned char*>(p.lse.data) + s_rel * p.lse.seq + path[tt] * p.lse.tok +
                                          (h * p.G + r % p.G) * p.lse.head);
    }
    lse[r] = x;
  }
  const int n_blocks = (n_rows + 31) / 32;
  u32x4_t qa[S::kChunks];
  load_q(qa, 0);
  __syncthreads();

  for (; slab < slab_end; slab += kWaves) {
    const int key = slab * kSlab + n32;
    float sum = 0.f;
    u32x4_t kb[S::kChunks];
    if constexpr (S::kMx) {
#pragma unroll
      for (int c = 0; c < S::kChunks; ++c) {
        const uint4 x = mx_values(codes[c / 4][c % 4], mx_scale(bytes >> (8 * (c / 4)) & 255));
        kb[c] = u32x4_t{x.x, x.y, x.z, x.w};
      }
    } else {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      const unsigned char* src = lds + (wave * 2 + (slab / kWaves & 1)) * S::kStage + n32 * S::kRow;
#pragma unroll
      for (int c = 0; c < S::kChunks; ++c) kb[c] = *reinterpret_cast<const u32x4_t*>(src + S::slot(n32, 2 * c + jh) * 16);
    }
    const float before = old;
    if (slab + kWaves < slab_end) request(slab + kWaves);
    for (int blk = 0; blk < n_blocks; ++blk) {
      if (blk > 0) load_q(qa, blk * 32);
      floatx16_t s = {};
#pragma unroll
      for (int c = 0; c < S::kChunks; ++c) {
        if constexpr (S::kF32) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(qa[c][e]), __uint_as_float(kb[c][e]), s, 0, 0, 0);
        } else {
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, qa[c]), __builtin_bit_cast(bf16x8_t, kb[c]), s, 0, 0, 0);
        }
      }
      // register i: row blk * 32 + 8 (i / 4) + 4 h + i % 4; a path's row j is seen by its nodes from j on
      const int first_row = (key - n_old) * p.G;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int r = blk * 32 + 8 * q + 4 * jh;
        const floatx4_t z = *reinterpret_cast<const floatx4_t*>(lse + r);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float w = fast_exp2(fmaf(s[4 * q + i], cs, -z[i]));
          sum += r + i >= first_row ? w : 0.f;
        }
      }
    }
    if (n_blocks > 1) load_q(qa, 0);
    sum += __shfl_xor(sum, 32);
    if (jh == 0 && key < n) p.score[row0 + key] = before + sum;
  }
}

template <int TYPE, int D>
hipError_t launch_scores(const AcceptParams& p, unsigned grid, hipStream_t s) {
  accept_scores_kernel<TYPE, D><<<dim3(grid), dim3(kThreads), 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_append_accepted(const AcceptParams& p_in, int type, int D, int n_cus, hipStream_t s) {
  AcceptParams p = p_in;
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
  p.target = 2 * n_cus;
  const unsigned grid = (unsigned)p.target + (unsigned)p.n_caches;
  if (grid > INT32_MAX / kThreads) return hipErrorInvalidValue;
  return type == 1   ? D == 128 ? launch_scores<1, 128>(p, grid, s) : launch_scores<1, 64>(p, grid, s)
         : type == 2 ? D == 128 ? launch_scores<2, 128>(p, grid, s) : launch_scores<2, 64>(p, grid, s)
                     : D == 128 ? launch_scores<0, 128>(p, grid, s) : launch_scores<0, 64>(p, grid, s);
}

}  // namespace baklava
