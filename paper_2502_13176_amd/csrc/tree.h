// Work items of launches over the ragged caches that are cut by the lengths on the device: the tiles of all caches of a launch,
// in items of equal length.  Each workgroup finds its own by a scan over the caches.
#ifndef BAKLAVA_TREE_H
#define BAKLAVA_TREE_H

#include "common.h"

namespace baklava {

#ifdef __HIPCC__
// A value that is the same in all lanes, in scalar registers.
__device__ __forceinline__ int64_t uniform(int64_t x) {
  return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 |
                   (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
}

// Tiles [first, last) of cache c_rel of the launch: number `part` of its n_parts items.  slot: the cache's first partial slot.
struct Span {
  int c_rel, first, last, part, n_parts, slot;
};

// Sum of x over the wavefront's lanes up to and with the calling one.
__device__ __forceinline__ int scan_wave(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);  // row_shr:2
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);  // row_shr:4
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);  // row_shr:8
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15 into rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast:31 into rows 2 and 3
  return x;
}
// x / y rounded up, 0 <= x < 2^31, y > 0, both in unsigned 32 bits.
__device__ __forceinline__ int ceil_div(int x, int y) { return (int)(((uint32_t)x + (uint32_t)y - 1) / (uint32_t)y); }
// Sum of x over the workgroup's threads up to and with the calling one, and over all of them.
template <int THREADS>
__device__ __forceinline__ int scan_threads(int x, int32_t* lds, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  x = scan_wave(x);
  __syncthreads();  // (lds may still be read)
  if (lane == 63) lds[wave] = x;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    const int y = lds[w];
    before += w < wave ? y : 0;
    total += y;
  }
  return x + before;
}

// The item number `item` of n_caches caches of tiles(c) tiles each; false: there is none.  Items have at most `run` tiles: a
// multiple of `unit`, and all tiles / target at least, so that there are at most target + n_caches.  Where there are few caches run
// grows until there are at most target: a launch of one round of workgroups would otherwise take a second one for a few of them.
// The items of a cache are of equal length but for one tile.  Partial slots go to the caches of several items alone, which have
// fewer than 2 target of them (ceil(x) < 2 x for x > 1).  lds: THREADS / 64 + 3 words, free for other use behind the next barrier.
template <int THREADS, class Tiles>
__device__ __forceinline__ bool find_span(int n_caches, int target, int unit, int item, const Tiles& tiles, int32_t* lds, Span& sp) {
  constexpr int kAt = THREADS / 64;
  // (any growth will do; float arithmetic is the same in every workgroup)
  auto next_run = [&](int run, int count) { return run + unit * max(1, (int)((float)run * (float)(count - target) / (float)(target * unit))); };
  int run, t;
  if (n_caches <= 64) {  // every wavefront for itself
    const int lane = threadIdx.x & 63;
    const int mine = lane < n_caches ? tiles(lane) : 0;
    run = max(ceil_div(__builtin_amdgcn_readlane(scan_wave(mine), 63), target * unit), 1) * unit;
    int parts = ceil_div(mine, run), end = scan_wave(parts);
    if (2 * n_caches <= target) {
#pragma unroll 1
      for (int i = 0; i < 4; ++i) {
        const int count = __builtin_amdgcn_readlane(end, 63);
        if (count <= target) break;
        run = next_run(run, count);
        parts = ceil_div(mine, run);
        end = scan_wave(parts);
      }
    }
    const int slots = parts > 1 ? parts : 0, slot_end = scan_wave(slots);
    const unsigned long long hit = __ballot(item < end && item >= end - parts);
    if (!hit) return false;
    const int c = __builtin_ctzll(hit);
    sp.c_rel = c;
    sp.slot = __builtin_amdgcn_readlane(slot_end - slots, c);
    sp.part = item - __builtin_amdgcn_readlane(end - parts, c);
    t = __builtin_amdgcn_readlane(mine, c);
  } else {
    const int tid = threadIdx.x;
    const int mine = tid < n_caches ? tiles(tid) : 0;  // (of the first caches, often all of them)
    int all = mine;
    for (int c = tid + THREADS; c < n_caches; c += THREADS) all += tiles(c);
    int total;
    scan_threads<THREADS>(all, lds, total);
    run = max(ceil_div(total, target * unit), 1) * unit;
    if (2 * n_caches <= target && n_caches <= THREADS) {
#pragma unroll 1
      for (int i = 0; i < 4; ++i) {
        int count;
        scan_threads<THREADS>(ceil_div(mine, run), lds, count);
        if (count <= target) break;
        run = next_run(run, count);
      }
    }
    if (tid == 0) lds[kAt] = -1;
    int items0 = 0, slots0 = 0;
    for (int c0 = 0; c0 < n_caches; c0 += THREADS) {
      const int c = c0 + tid;
      const int x = c0 == 0 ? mine : c < n_caches ? tiles(c) : 0;
      const int parts = ceil_div(x, run);
      int n_items, n_slots;
      const int end = items0 + scan_threads<THREADS>(parts, lds, n_items);
      const int slot_end = slots0 + scan_threads<THREADS>(parts > 1 ? parts : 0, lds, n_slots);
      if (item < end && item >= end - parts) {
        lds[kAt] = c;
        lds[kAt + 1] = slot_end - (parts > 1 ? parts : 0);
        lds[kAt + 2] = item - (end - parts);
      }
      items0 += n_items;
      slots0 += n_slots;
      if (item < items0) break;
    }
    __syncthreads();
    const int c = __builtin_amdgcn_readfirstlane(lds[kAt]);
    if (c < 0) return false;
    sp.c_rel = c;
    sp.slot = __builtin_amdgcn_readfirstlane(lds[kAt + 1]);
    sp.part = __builtin_amdgcn_readfirstlane(lds[kAt + 2]);
    t = __builtin_amdgcn_readfirstlane(tiles(c));
  }
  run = __builtin_amdgcn_readfirstlane(run);
  sp.n_parts = __builtin_amdgcn_readfirstlane(ceil_div(t, run));
  const int per = __builtin_amdgcn_readfirstlane((int)((uint32_t)t / (uint32_t)sp.n_parts)), more = t - per * sp.n_parts;  // the first `more` items have one tile more
  sp.first = sp.part * per + min(sp.part, more);
  sp.last = sp.first + per + (sp.part < more ? 1 : 0);
  return true;
}

// For launches whose work items need not be merged: tile number `at` of all, counted cache by cache, as cache and tile of it; false:
// there are not as many.  total: all tiles (known before `at` has to be: at = f(total)).
template <int THREADS, class Tiles, class At>
__device__ __forceinline__ bool find_tile(int n_caches, const Tiles& tiles, const At& at_of, int32_t* lds, int& c_rel, int& tile, int& total) {
  constexpr int kAt = THREADS / 64;
  const int tid = threadIdx.x;
  if (n_caches <= 64) {  // every wavefront for itself
    const int lane = tid & 63, mine = lane < n_caches ? tiles(lane) : 0, end = scan_wave(mine);
    total = __builtin_amdgcn_readlane(end, 63);
    const int at = at_of(total);
    if (at >= total) return false;
    c_rel = __builtin_ctzll(__ballot(at < end));
    tile = at - __builtin_amdgcn_readlane(end - mine, c_rel);
    return true;
  }
  const int first = tid < n_caches ? tiles(tid) : 0;
  int all = first;
  for (int c = tid + THREADS; c < n_caches; c += THREADS) all += tiles(c);
  scan_threads<THREADS>(all, lds, total);
  total = __builtin_amdgcn_readfirstlane(total);
  const int at = at_of(total);
  if (at >= total) return false;
  int before = 0;
  for (int c0 = 0;; c0 += THREADS) {
    const int mine = c0 == 0 ? first : c0 + tid < n_caches ? tiles(c0 + tid) : 0;
    int sum;
    const int end = before + scan_threads<THREADS>(mine, lds, sum);
    if (at < end && at >= end - mine) {
      lds[kAt] = c0 + tid;
      lds[kAt + 1] = at - (end - mine);
    }
    before += sum;
    if (at < before) break;
  }
  __syncthreads();
  c_rel = __builtin_amdgcn_readfirstlane(lds[kAt]);
  tile = __builtin_amdgcn_readfirstlane(lds[kAt + 1]);
  return true;
}

__device__ __forceinline__ int tree_nodes(const TreeParams& p, int b) {
  return p.n_nodes ? min(max(p.n_nodes[b], 0), p.N) : p.N;
}

// Who sees whom, as bits above[word][node]: a node's ancestors by doubling, all nodes at once.  up: parent of node threadIdx.x, or -1.
// jump: kMostNodes words.  Threads beyond the nodes take part in the barriers.
__device__ __forceinline__ void find_ancestors(int up, int n_nodes, unsigned long long (*above)[kMostNodes], int32_t* jump) {
  constexpr int kWords = kMostNodes / 64;
  const int tid = threadIdx.x;
  const int words = (n_nodes + 63) / 64;
  const bool node = tid < kMostNodes;
  if (node) {
    jump[tid] = up;
    for (int w = 0; w < words; ++w) above[w][tid] = tid / 64 == w ? 1ull << (tid & 63) : 0ull;
  }
  __syncthreads();
  for (int reach = 1; reach < n_nodes; reach *= 2) {
    unsigned long long more[kWords];
    const int to = node ? jump[tid] : -1;
    int next = -1;
    if (to >= 0) {
      next = jump[to];
#pragma unroll
      for (int w = 0; w < kWords; ++w) more[w] = w < words ? above[w][to] : 0;
    }
    if (!__syncthreads_or(to >= 0)) break;
    if (to >= 0) {
      jump[tid] = next;
#pragma unroll
      for (int w = 0; w < kWords; ++w)
        if (w < words) above[w][tid] |= more[w];
    }
    __syncthreads();
  }
}

// Row (s_rel, node, head) of rows by byte strides.
__device__ __forceinline__ unsigned char* row_of(const Rows& r, int s_rel, int node, int head) {
  return reinterpret_cast<unsigned char*>(r.data) + s_rel * r.seq + node * r.tok + head * r.head;
}
#endif

}  // namespace baklava
#endif
