// Prompts into the caches and cache rows back out (baklava_append_prompt, baklava_read_rows).
//
// Both move rows, so HBM bounds them: a workgroup takes kTile rows of one cache, requests all of them, whole rows at a time, and
// stores them (rounded to 4 bits on the way, see mxfp4.h).  Read and written together, behind a projection's output that the
// last-level cache may hold in part, us a call: 8 x 32768 bf16 rows of 128 elements into 4 bits 25 (2 of them the launch for
// the lengths), 6.8 TB/s, of 16 bits 39, 6.9; back out of 4 bits 25, 6.7 TB/s.  (A loop that requested rows four at a
// time, tiles in front of heads, took 35 us.)
#include "common.h"
#include "mxfp4.h"

namespace baklava {

namespace {

constexpr int kThreads = 256, kTile = 64;

// MX: 4-bit rows.  PIECES: 16-byte pieces of a row as the caller holds it.  Workgroups go over the heads of a tile of tokens
// first: a token's heads lie next to each other in what a projection writes.
template <int PIECES, bool MX>
__global__ __launch_bounds__(kThreads) void append_prompt_kernel(PromptRowsParams p) {
  constexpr int kRows = kThreads / PIECES, kPer = kTile / kRows, D = PIECES * 8;  // (D: bf16 rows, where it matters)
  const int i = blockIdx.y, h_rel = (uint32_t)blockIdx.x % (uint32_t)p.n_heads, h = p.head0 + h_rel;
  const PromptRowsParams::Seq q = p.seq[i];
  const int r0 = (p.tile0 + (uint32_t)blockIdx.x / (uint32_t)p.n_heads) * kTile;
  if (r0 >= q.n) return;
  const int c = p.cache0 + i * p.Hkv + h;
  const int tid = threadIdx.x, piece = tid % PIECES, row = r0 + tid / PIECES;
  const int e = min(r0 + kTile, q.n);
  const uint4* src_k = reinterpret_cast<const uint4*>(p.k.data) + p.k.begin(p.seq0 + i, q.first) + h * p.k.head + piece;
  const uint4* src_v = reinterpret_cast<const uint4*>(p.v.data) + p.v.begin(p.seq0 + i, q.first) + h * p.v.head + piece;
  uint4 k[kPer], v[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j) {  // rows past the last one repeat it and are not written
    const int64_t r = min(row + j * kRows, e - 1);
    k[j] = src_k[r * p.k.tok];
    v[j] = src_v[r * p.v.tok];
  }
  // Rows go behind the live ones as the device counts them: replays of captured steps move that count without the host's
  // knowledge.  The tile that is the last of its cache to have read it advances it.
  int start;
  if (p.from_len) {
    __shared__ int live;
    if (tid == 0) live = p.len[c];
    __syncthreads();
    start = live;
    if (tid == 0 && p.ticket) {
      const int tiles = (q.n + kTile - 1) / kTile;
      int32_t* const ticket = p.ticket + (int64_t)c * kTicketStride;
      if (tiles == 1 || __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == tiles - 1) {
        if (tiles > 1) __hip_atomic_store(ticket, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (start <= p.cap[c] - q.n) p.len[c] = start + q.n;
        else *p.status = 1;
      }
    }
    if (start > p.cap[c] - q.n) return;  // all or nothing of a prompt
  } else {
    start = p.start[i * p.n_heads + h_rel];
    if (r0 == 0 && tid == 0) p.len[c] = start + q.n;
  }
  const int64_t row0 = p.off[c] + start;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int r = row + j * kRows;
    if (MX) {
      const uint32_t bk = mx_scale_byte(mx_top(k[j])), bv = mx_scale_byte(mx_top(v[j]));
      const uint32_t ck = mx_codes(k[j], bk), cv = mx_codes(v[j], bv);
      const uint2 scales = mx_row_scales<D>(bk, bv, piece);
      if (r < e) {
        reinterpret_cast<uint32_t*>(p.k_plane)[(row0 + r) * (D / 8) + piece] = ck;
        reinterpret_cast<uint32_t*>(p.v_plane)[(row0 + r) * (D / 8) + piece] = cv;
        if (piece == 0) {
          if (D == 128) reinterpret_cast<uint2*>(p.kv_scale)[row0 + r] = scales;
          else reinterpret_cast<uint32_t*>(p.kv_scale)[row0 + r] = scales.x | scales.y << 16;
        }
      }
    } else if (r < e) {
      store_nt16(reinterpret_cast<uint4*>(p.k_plane) + (row0 + r) * PIECES + piece, k[j]);
      store_nt16(reinterpret_cast<uint4*>(p.v_plane) + (row0 + r) * PIECES + piece, v[j]);
    }
  }
  if (tid < e - r0) {
    const int r = r0 + tid;
    p.score[row0 + r] = p.scores.data ? reinterpret_cast<const float*>(p.scores.data)[p.scores.begin(p.seq0 + i, q.first) +
                                                                                      r * p.scores.tok + h * p.scores.head]
                                      : 0.f;
    p.pos[row0 + r] = q.pos0 + r;
  }
}

// Lengths behind rows whose tiles drew no tickets.
__global__ __launch_bounds__(kThreads) void advance_lengths_kernel(PromptRowsParams p, int n_caches) {
  for (int i = threadIdx.x; i < n_caches; i += kThreads) {
    const int n = p.seq[i / p.n_heads].n, c = p.cache0 + i / p.n_heads * p.Hkv + p.head0 + i % p.n_heads;
    if (n == 0) continue;
    if (p.len[c] <= p.cap[c] - n) p.len[c] += n;
    else *p.status = 1;
  }
}

template <int PIECES, bool MX>
__global__ __launch_bounds__(kThreads) void read_rows_kernel(ReadRowsParams p) {
  constexpr int kRows = kThreads / PIECES, kPer = kTile / kRows, D = PIECES * 8;
  const int c = p.cache0 + blockIdx.y;
  const int r0 = blockIdx.x * kTile, e = min(r0 + kTile, p.n);
  const int skip = p.n - p.len[c];  // places in front of the cache's first row (or rows in front of the first one asked for)
  const int64_t row0 = p.off[c] - skip, out0 = (int64_t)blockIdx.y * p.n;
  const int tid = threadIdx.x, piece = tid % PIECES, row = r0 + tid / PIECES;
  uint4 k[kPer], v[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int r = min(row + j * kRows, e - 1);
    k[j] = v[j] = make_uint4(0, 0, 0, 0);
    if (r >= skip) {
      if (MX) {
        k[j] = mx_load<D>(piece, p.k_plane, p.kv_scale, row0 + r, 0);
        v[j] = mx_load<D>(piece, p.v_plane, p.kv_scale, row0 + r, 1);
      } else {
        k[j] = reinterpret_cast<const uint4*>(p.k_plane)[(row0 + r) * PIECES + piece];
        v[j] = reinterpret_cast<const uint4*>(p.v_plane)[(row0 + r) * PIECES + piece];
      }
    }
  }
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int r = row + j * kRows;
    if (r < e) {
      store_nt16(reinterpret_cast<uint4*>(p.k_out) + (out0 + r) * PIECES + piece, k[j]);
      store_nt16(reinterpret_cast<uint4*>(p.v_out) + (out0 + r) * PIECES + piece, v[j]);
    }
  }
}

// The new row of a decode step, rounded (baklava_append over 4-bit rows).
template <int D>
__global__ __launch_bounds__(64) void append_mx_kernel(AppendParams p) {
  const int c = p.cache_begin + blockIdx.x;
  const int n = p.len[c];
  if (n >= p.cap[c]) return;  // the host has already refused this case
  const int64_t row = p.off[c] + n;
  const int lane = threadIdx.x, value = lane / (D / 8), piece = lane % (D / 8);
  if (value < 2)
    mx_store<D>(reinterpret_cast<const uint4*>(value ? p.v_new : p.k_new)[(int64_t)blockIdx.x * (D / 8) + piece], piece,
                value ? p.v : p.k, p.kv_scale, row, value);
  if (lane == 63) {
    p.score[row] = 0.f;
    p.pos[row] = p.token_pos;
  }
  __syncthreads();
  if (lane == 0) p.len[c] = n + 1;
}

}  // namespace

hipError_t launch_append_prompt(const PromptRowsParams& p_in, int pieces, bool mx, int n_seq, int most, hipStream_t s) {
  if (p_in.n_heads <= 0 || n_seq <= 0 || most <= 0) return hipSuccess;
  PromptRowsParams p = p_in;
  const int tiles = (most + kTile - 1) / kTile, per_launch = (1 << 23) / p.n_heads;  // a grid dimension holds fewer than 2^32 threads
  // Tickets of one cache follow each other, some 15 ns apart.  us with tickets / with a launch more: 8 caches of 512 rows (8
  // tickets each) 7.5 / 10.7, 32 of 3001 (47) 13.2 / 14.8, 8 of 32768 (512) 25.6 / 25.5, one of 65536 (1024) 15.6 / 10.3.
  if (tiles > kMostTickets) p.ticket = nullptr;
  for (p.tile0 = 0; p.tile0 < tiles; p.tile0 += per_launch) {
    const dim3 grid((tiles - p.tile0 < per_launch ? tiles - p.tile0 : per_launch) * p.n_heads, n_seq), block(kThreads);
    if (mx && pieces == 16) append_prompt_kernel<16, true><<<grid, block, 0, s>>>(p);
    else if (mx && pieces == 8) append_prompt_kernel<8, true><<<grid, block, 0, s>>>(p);
    else if (pieces == 32) append_prompt_kernel<32, false><<<grid, block, 0, s>>>(p);
    else if (pieces == 16) append_prompt_kernel<16, false><<<grid, block, 0, s>>>(p);
    else if (pieces == 8) append_prompt_kernel<8, false><<<grid, block, 0, s>>>(p);
    else return hipErrorInvalidValue;
  }
  if (p.from_len && !p.ticket) advance_lengths_kernel<<<dim3(1), dim3(kThreads), 0, s>>>(p, n_seq * p.n_heads);
  return hipGetLastError();
}

hipError_t launch_read_rows(const ReadRowsParams& p_in, int pieces, bool mx, int n_caches, hipStream_t s) {
  ReadRowsParams p = p_in;
  const dim3 block(kThreads);
  for (int at = 0; at < n_caches; at += 65535) {  // a grid's second dimension holds no more
    const dim3 grid((p.n + kTile - 1) / kTile, n_caches - at < 65535 ? n_caches - at : 65535);
    if (mx && pieces == 16) read_rows_kernel<16, true><<<grid, block, 0, s>>>(p);
    else if (mx && pieces == 8) read_rows_kernel<8, true><<<grid, block, 0, s>>>(p);
    else if (pieces == 32) read_rows_kernel<32, false><<<grid, block, 0, s>>>(p);
    else if (pieces == 16) read_rows_kernel<16, false><<<grid, block, 0, s>>>(p);
    else if (pieces == 8) read_rows_kernel<8, false><<<grid, block, 0, s>>>(p);
    else return hipErrorInvalidValue;
    p.cache0 += 65535;
    p.k_out = reinterpret_cast<uint4*>(p.k_out) + (int64_t)65535 * p.n * pieces;
    p.v_out = reinterpret_cast<uint4*>(p.v_out) + (int64_t)65535 * p.n * pieces;
  }
  return hipGetLastError();
}

hipError_t launch_append_mx(const AppendParams& p, int D, int n_caches, hipStream_t s) {
  if (n_caches <= 0) return hipSuccess;
  if (D == 128) append_mx_kernel<128><<<dim3(n_caches), dim3(64), 0, s>>>(p);
  else append_mx_kernel<64><<<dim3(n_caches), dim3(64), 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace baklava
