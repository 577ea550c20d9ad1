// The shares of the attention of several new tokens per request: every CTA works out, from lengths that are known on the device only, which items and
// which of their tiles are its own.
//
// Items lie in a line: request, key head, place.  As long as there are two for every CTA, CTA c takes items c, c + G, .. as a whole: CTAs that run side by side
// then read the same keys and values at about the same time.  The last G to 2 G items even out what the CTAs have: CTA c takes the beginning
// of the c-th of them, as many tiles as it may still have, and what is left of them all is a line of tiles that the CTAs with room share.  A CTA that shares a
// head with others so begins at its first rows, as they do.  The join puts together what was cut.
#pragma once
#include "chunk.cuh"
#include "chunk_tiles.h"

namespace pact {

struct ChunkRequest : ChunkLengths {
  bool bad;
  long long row0;                          // its first row of Q and out
};
__device__ __forceinline__ ChunkRequest chunk_request(const ChunkArgs &a, int b) {
  ChunkRequest q;
  const long long room = (long long)a.width * a.page;
  const int len = a.length[b], want = a.n_new[b * a.n_new_stride];
  q.len = len < 0 ? 0 : len > room ? (int)room : len;
  q.want = max(0, want);
  long long have = a.row_stride;
  q.row0 = b * (long long)a.row_stride;
  if (!a.row_stride) {
    q.row0 = a.row_start[b];
    have = q.row0 < 0 || q.row0 > a.n_rows ? 0 : a.n_rows - q.row0;
  }
  q.n = (int)min((long long)q.want, have);
  q.bad = q.len != len || q.n != q.want || q.want > q.len;
  return q;
}

// Tiles [j0, j1) of an item of k tiles.
struct ChunkSegment : ChunkRequest {
  int b, kv, rows, first;                  // rows of the item, its first row among the request's (token row / group, head row % group)
  int k, j0, j1;
  int slot;                                // of its part, -1: the whole item
  int place;                               // the slot that it may use meanwhile, its own in any case
  __device__ __forceinline__ int limit(int token, bool causal) const { return chunk_seen(*this, token, causal); }   // rows that a token sees
};

constexpr int kChunkPreInSmem = 33;        // entries of `pre` that are kept in shared memory
constexpr int kChunkKept = 16;             // requests that are

struct ChunkLine {
  const int *pre, *head;
  const ChunkRequest *kept;                // the requests where there are no more than kChunkKept
  int rounds, last, r;                     // rounds of whole items, the first item after them, how many there are
  int q, off, tail;                        // where this CTA's part of the rests begins, and its tiles
  // walking through the segments
  int done, stage;
  template <int ROWS, int TILE> __device__ __forceinline__ void item(const ChunkArgs &a, int x, ChunkSegment &s) const {
    int lo = 0, hi = a.B;
    const int H = a.n_kvh;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (pre[mid] * H <= x) lo = mid;
      else hi = mid;
    }
    static_cast<ChunkRequest &>(s) = a.B <= kChunkKept ? kept[lo] : chunk_request(a, lo);
    const int n = pre[lo + 1] - pre[lo], at = x - pre[lo] * H;
    s.b = lo;
    s.kv = at / n;
    const int i = at - s.kv * n;
    s.first = i * ROWS;
    s.rows = min(ROWS, s.n * a.group - s.first);
    s.k = chunk_tiles(s, i, a.group, ROWS, TILE, a.causal);
  }
  template <int ROWS, int TILE> __device__ __forceinline__ bool next(const ChunkArgs &a, ChunkSegment &s) {
    const int G = gridDim.x, me = blockIdx.x;
    if (done < rounds) {
      item<ROWS, TILE>(a, me + done++ * G, s);
      s.j0 = 0;
      s.j1 = s.k;
      s.slot = -1;
      s.place = me;                        // (the CTA's beginning of an item comes later)
      return true;
    }
    if (stage == 0) {
      stage = 1;
      if (me < r && head[me] > 0) {
        item<ROWS, TILE>(a, last + me, s);
        s.j0 = 0;
        s.j1 = head[me];
        s.slot = s.j1 == s.k ? -1 : me;
        s.place = me;
        return true;
      }
    }
    while (tail > 0) {
      item<ROWS, TILE>(a, last + q, s);
      s.j0 = (q < G ? head[q] : 0) + off;
      s.j1 = min(s.k, s.j0 + tail);
      s.place = G + q + me;
      s.slot = s.j0 == 0 && s.j1 == s.k ? -1 : s.place;
      ++q;
      off = 0;
      if (s.j1 <= s.j0) continue;
      tail -= s.j1 - s.j0;
      return true;
    }
    return false;
  }
};

// Shared memory of the set-up: kept (`pre`, where the rests begin) and passing (for the set-up alone).
struct ChunkLineKept {
  ChunkRequest request[kChunkKept];
  int pre[kChunkPreInSmem];
  int q, off;
};
struct ChunkLineSetup {
  unsigned long long tiles, rows;
  int warp[32];
  int dp[kChunkMaxSms];                    // tiles of the whole items of each CTA
  int lp[2 * kChunkMaxSms + 1];            // rests before each item of the last round
  int tp[kChunkMaxSms + 1];                // tiles that the CTAs before have room for
};

// Exclusive sums of a value per thread; ends with a barrier.
template <int THREADS> __device__ __forceinline__ int chunk_scan(int v, int *warp_sums, int *total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  int before = 0, all = 0;
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w < warp) before += warp_sums[w];
    all += warp_sums[w];
  }
  *total = all;
  return before + x - v;
}

// What the join has to know about items `me` and `me + G` of the last round; written by one warp while the others go on, from what all warps took before the set-up's
// shared memory was given to the copies.
struct ChunkCuts {
  static constexpr int kWords = (kChunkMaxSms + 31) / 32;
  int tp[kWords];                          // set.tp[32 i + lane], INT32_MAX past the last
  int from[2], to[2];                      // set.lp of the two items and of the ones after them
  __device__ __forceinline__ void take(const ChunkLine &line, const ChunkLineSetup &set, int G, int me) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      const int c = i * 32 + (threadIdx.x & 31);
      tp[i] = c < G ? set.tp[c] : INT32_MAX;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int q = me + k * G;
      from[k] = q < line.r ? set.lp[q] : 0;
      to[k] = q < line.r ? set.lp[q + 1] : 0;
    }
  }
  __device__ __forceinline__ int owner(int t) const {                // the CTA that has tile t of the rests: the last one that begins at or before it
    int n = 0;
#pragma unroll
    for (int i = 0; i < kWords; ++i) n += __popc(__ballot_sync(0xffffffffu, tp[i] <= t));
    return n - 1;
  }
  template <int ROWS, int TILE> __device__ __forceinline__ void write(const ChunkArgs &a, const ChunkLine &line) const {   // a whole warp
    const int G = gridDim.x, me = blockIdx.x;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int q = me + k * G;
      ChunkCut cut = {0, q < G && q < line.r && line.head[q] > 0, 0, -1, 0, 0, 0, 0, 0};
      if (to[k] > from[k]) {
        cut.first = owner(from[k]);
        cut.last = owner(to[k] - 1);
        cut.cut = cut.head || cut.first != cut.last;
        ChunkSegment s;
        line.item<ROWS, TILE>(a, line.last + q, s);
        cut.kv = s.kv;
        cut.rows = s.rows;
        cut.first_row = s.first;
        cut.row0 = s.row0;
      }
      if ((threadIdx.x & 31) == 0) a.cut[q] = cut;
    }
  }
};

// Called by all threads of the CTA, at least as many as the grid has CTAs.
template <int THREADS, int ROWS, int TILE> __device__ __forceinline__ ChunkLine chunk_line(const ChunkArgs &a, ChunkLineKept &kept, ChunkLineSetup &set, ChunkCuts &cuts) {
  static_assert(THREADS >= kChunkMaxSms, "");
  constexpr int PER = (2 * kChunkMaxSms + THREADS - 1) / THREADS;    // items of the last round that a thread looks at
  const int tid = threadIdx.x, G = gridDim.x, me = blockIdx.x;
  int *pre = a.B < kChunkPreInSmem ? kept.pre : a.pre + (long long)me * (a.B + 1), *head = a.head + me * G;
  ChunkLine line;
  line.pre = pre;
  line.head = head;
  line.kept = kept.request;
  line.done = line.stage = 0;
  if (tid == 0) {
    set.tiles = set.rows = 0;
    kept.q = kept.off = 0;
  }
  __syncthreads();
  {
    const int per = (a.B + THREADS - 1) / THREADS, b0 = min(a.B, tid * per), b1 = min(a.B, b0 + per);
    int mine = 0, total;
    unsigned long long tiles = 0, rows = 0;
    for (int b = b0; b < b1; ++b) {
      const ChunkRequest q = chunk_request(a, b);
      if (a.B <= kChunkKept) kept.request[b] = q;
      if (q.bad && me == 0 && a.status) atomicMin(a.status, (int)PACT_ERR_INVALID_ARG);
      pre[b] = mine;
      mine += chunk_items(q, a.group, ROWS);
      rows += q.n;
      tiles += chunk_tiles_of_head(q, a.group, ROWS, TILE, a.causal);
    }
    if (tiles) {
      atomicAdd(&set.tiles, tiles);
      atomicAdd(&set.rows, rows);
    }
    const int before = chunk_scan<THREADS>(mine, set.warp, &total);
    for (int b = b0; b < b1; ++b) pre[b] += before;
    if (tid == 0) pre[a.B] = total;
  }
  __syncthreads();
  const bool fits = chunk_rows_fit(set.rows, a.n_rows);
  if (!fits && me == 0 && tid == 0 && a.status) atomicMin(a.status, (int)PACT_ERR_INVALID_ARG);
  const int items = fits ? pre[a.B] * a.n_kvh : 0;                   // (of nothing else is there more than was checked)
  const long long T = fits ? (long long)set.tiles * a.n_kvh : 0;
  line.rounds = items >= 2 * G ? items / G - 1 : 0;
  line.last = line.rounds * G;
  line.r = items - line.last;
  ChunkSegment s;
  if (tid < G) set.dp[tid] = 0;
  __syncthreads();
  for (int x = tid; x < line.last; x += THREADS) {
    line.item<ROWS, TILE>(a, x, s);
    atomicAdd(&set.dp[x % G], s.k);
  }
  __syncthreads();
  // tiles that a CTA may have: those with more already are left out of the mean
  int most = (int)((T + G - 1) / G);
  if (line.rounds > 0)
    for (int round = 0; round < 4; ++round) {
      const int mine = tid < G && set.dp[tid] > most ? set.dp[tid] : 0;
      int over, n;
      (void)chunk_scan<THREADS>(mine, set.warp, &over);
      n = __syncthreads_count(mine > 0);
      if (n == 0 || n == G) break;
      most = (int)((T - over + G - n - 1) / (G - n));
    }
  int begins[PER], rest[PER], room[PER], sum_rest = 0, sum_room = 0, all, rests;
  for (int k = 0; k < PER; ++k) {
    const int q = tid * PER + k;
    begins[k] = rest[k] = room[k] = 0;
    if (q < G) room[k] = max(0, most - set.dp[q]);
    if (q < line.r) {
      line.item<ROWS, TILE>(a, line.last + q, s);
      begins[k] = min(s.k, room[k]);
      rest[k] = s.k - begins[k];
    }
    if (q < G) head[q] = begins[k];
    room[k] -= begins[k];
    sum_rest += rest[k];
    sum_room += room[k];
  }
  int lp = chunk_scan<THREADS>(sum_rest, set.warp, &rests), tp = chunk_scan<THREADS>(sum_room, set.warp, &all);
  for (int k = 0; k < PER; ++k) {
    const int q = tid * PER + k;
    if (q < line.r) set.lp[q] = lp;
    if (q < G) set.tp[q] = min(tp, rests);
    lp += rest[k];
    tp += room[k];
  }
  if (tid == 0) {
    set.lp[line.r] = rests;
    set.tp[G] = rests;                     // (the last CTA has whatever is left)
  }
  __syncthreads();
  const int t0 = set.tp[me];
  line.tail = set.tp[me + 1] - t0;
  if (me == 0 && tid < G) a.tail[tid] = set.tp[tid + 1] - set.tp[tid];
  for (int k = 0; k < PER; ++k) {
    const int q = tid * PER + k;
    if (q < line.r && set.lp[q] <= t0 && t0 < set.lp[q] + rest[k]) {
      kept.q = q;
      kept.off = t0 - set.lp[q];
    }
  }
  cuts.take(line, set, G, me);
  __syncwarp();
  __syncthreads();
  line.q = kept.q;
  line.off = kept.off;
  return line;
}

}  // namespace pact
