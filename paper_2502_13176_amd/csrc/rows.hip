// Prompts into the caches and cache rows back out (baklava_append_prompt, baklava_read_rows).  Both move rows and are bound by
// HBM; a workgroup takes kTile rows of one cache, whole rows at a time.
#include "common.h"
#include "mxfp4.h"

namespace baklava {

namespace {

constexpr int kThreads = 256, kTile = 64;

// MX: 4-bit rows.  PIECES: 16-byte pieces of a row as the caller holds it.
template <int PIECES, bool MX>
__global__ __launch_bounds__(kThreads) void append_prompt_kernel(PromptRowsParams p) {
  constexpr int kRows = kThreads / PIECES, D = PIECES * 8;  // (D: bf16 rows, where it matters)
  const int i = blockIdx.z, h = p.head0 + blockIdx.y;
  const PromptRowsParams::Seq q = p.seq[i];
  const int r0 = blockIdx.x * kTile;
  if (r0 >= q.n) return;
  const int c = p.cache0 + i * p.Hkv + h, start = p.start[i * gridDim.y + blockIdx.y];
  const int64_t row0 = p.off[c] + start;
  const int tid = threadIdx.x, piece = tid % PIECES;
  const int e = min(r0 + kTile, q.n);
  const uint4* src_k = reinterpret_cast<const uint4*>(p.k.data) + p.k.begin(p.seq0 + i, q.first) + h * p.k.head + piece;
  const uint4* src_v = reinterpret_cast<const uint4*>(p.v.data) + p.v.begin(p.seq0 + i, q.first) + h * p.v.head + piece;
#pragma unroll 4
  for (int r = r0 + tid / PIECES; r < e; r += kRows) {
    const uint4 k = src_k[r * p.k.tok], v = src_v[r * p.v.tok];
    if (MX) {
      mx_store<D>(k, piece, p.k_plane, p.kv_scale, row0 + r, 0);
      mx_store<D>(v, piece, p.v_plane, p.kv_scale, row0 + r, 1);
    } else {
      reinterpret_cast<uint4*>(p.k_plane)[(row0 + r) * PIECES + piece] = k;
      reinterpret_cast<uint4*>(p.v_plane)[(row0 + r) * PIECES + piece] = v;
    }
  }
  if (tid < e - r0) {
    const int r = r0 + tid;
    p.score[row0 + r] = 0.f;
    if (p.scores.data)
      p.score[row0 + r] = reinterpret_cast<const float*>(p.scores.data)[p.scores.begin(p.seq0 + i, q.first) + r * p.scores.tok + h * p.scores.head];
    p.pos[row0 + r] = q.pos0 + r;
  }
  if (r0 == 0 && tid == 0) p.len[c] = start + q.n;
}

template <int PIECES, bool MX>
__global__ __launch_bounds__(kThreads) void read_rows_kernel(ReadRowsParams p) {
  constexpr int kRows = kThreads / PIECES, D = PIECES * 8;
  const int c = p.cache0 + blockIdx.y;
  const int r0 = blockIdx.x * kTile, e = min(r0 + kTile, p.n);
  const int skip = p.n - p.len[c];  // places in front of the cache's first row (or rows in front of the first one asked for)
  const int64_t row0 = p.off[c] - skip;
  const int tid = threadIdx.x, piece = tid % PIECES;
#pragma unroll 4
  for (int r = r0 + tid / PIECES; r < e; r += kRows) {
    uint4 k = make_uint4(0, 0, 0, 0), v = k;
    if (r >= skip) {
      if (MX) {
        k = mx_load<D>(piece, p.k_plane, p.kv_scale, row0 + r, 0);
        v = mx_load<D>(piece, p.v_plane, p.kv_scale, row0 + r, 1);
      } else {
        k = reinterpret_cast<const uint4*>(p.k_plane)[(row0 + r) * PIECES + piece];
        v = reinterpret_cast<const uint4*>(p.v_plane)[(row0 + r) * PIECES + piece];
      }
    }
    const int64_t at = ((int64_t)blockIdx.y * p.n + r) * PIECES + piece;
    reinterpret_cast<uint4*>(p.k_out)[at] = k;
    reinterpret_cast<uint4*>(p.v_out)[at] = v;
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

hipError_t launch_append_prompt(const PromptRowsParams& p, int pieces, bool mx, int n_heads, int n_seq, int most, hipStream_t s) {
  if (n_heads <= 0 || n_seq <= 0 || most <= 0) return hipSuccess;
  const dim3 grid((most + kTile - 1) / kTile, n_heads, n_seq), block(kThreads);
  if (mx && pieces == 16) append_prompt_kernel<16, true><<<grid, block, 0, s>>>(p);
  else if (mx && pieces == 8) append_prompt_kernel<8, true><<<grid, block, 0, s>>>(p);
  else if (pieces == 32) append_prompt_kernel<32, false><<<grid, block, 0, s>>>(p);
  else if (pieces == 16) append_prompt_kernel<16, false><<<grid, block, 0, s>>>(p);
  else if (pieces == 8) append_prompt_kernel<8, false><<<grid, block, 0, s>>>(p);
  else return hipErrorInvalidValue;
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
