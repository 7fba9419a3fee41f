// What the chunk attention's host side and kernels share: its arguments and the split of its work over the thread blocks.
#pragma once

#include "common.cuh"

namespace mixkvq {

constexpr int kChunkMaxSeqs = 128;     // sequences of one launch (a larger batch goes in several)
constexpr int kChunkMaxCtas = 148;     // thread blocks of one launch: one per SM (sizes the scratch memory)
constexpr int kChunkRows = 256;        // query rows of an item
constexpr int kChunkTile = 128;        // keys of a tile
constexpr int kChunkParts = 3;         // results of a thread block: of its first item, of its last one, of a later piece of an item

struct ChunkItem;
struct ChunkSeq {
  int units;                           // packed 32-token units
  int tail;                            // residual and sink rows: r | n_sink << 16
  int n;                               // new tokens
};

// An item: up to 256 query rows of a stream (its g heads of neighbouring new tokens side by side) against all keys that the last of them sees.
// Its key tiles: those of the packed blocks, then those of the unquantized rows (residual window, sink, new tokens), 128 rows each.  The items of all
// streams lie one behind another on a line, an item of more than 128 rows two positions long per key tile, any other one; thread block c has
// the positions [total c / ctas, total (c + 1) / ctas).
struct ChunkArgs {
  struct ChunkItem* at;                // per thread block: the item that its first position lies in (behind parts; the merge reads it)
  const uint16_t *k, *v, *q;           // [B, Hkv, stride, 128], [B, Hq, stride, 128] bf16
  void* out;                           // [B, Hq, stride, 128]
  float* parts;                        // kChunkParts results of rows_cap rows per thread block: [rows_cap][128] sums, [rows_cap] (maximum, denominator)
  int out_bf16, stride, ctas, rows_cap;
  float scale_log2e;
  uint32_t max_polls, test_silent;     // test_silent: the first key tile is never announced (test hook)
  long long total;
  ChunkSeq seq[kChunkMaxSeqs];
  long long prefix[kChunkMaxSeqs + 1]; // positions of the sequences before this one
};

struct ChunkItem {
  int b, hk, rt;                       // sequence, KV head, row tile
  int n_rt, rows;                      // row tiles of the stream, rows of the item
  int packed_tiles, kt;                // key tiles of the packed blocks, of the item
  int weight;                          // positions per key tile
  long long x0;                        // its first position
};

__host__ __device__ inline int chunk_tail_rows(const ChunkSeq& s) { return (s.tail & 0xFFFF) + (s.tail >> 16); }
__host__ __device__ inline long long chunk_begin(long long total, int ctas, int c) { return total * c / ctas; }

// Fills in what follows from (b, hk, rt).
__host__ __device__ inline void chunk_item_of(const ChunkSeq& s, int g, ChunkItem& it) {
  const int rows = s.n * g, end = rows < kChunkRows * (it.rt + 1) ? rows : kChunkRows * (it.rt + 1);
  it.n_rt = (rows + kChunkRows - 1) / kChunkRows;
  it.rows = end - kChunkRows * it.rt;
  it.packed_tiles = (s.units + 3) / 4;
  it.kt = it.packed_tiles + (chunk_tail_rows(s) + (end - 1) / g + kChunkTile) / kChunkTile;
  it.weight = it.rows > kChunkTile ? 2 : 1;
}

// The item at position x (0 <= x < total), found by a whole warp: row tiles 32 at a time.
__device__ inline ChunkItem chunk_locate(const ChunkArgs& a, int B, int Hkv, int g, long long x, int lane) {
  ChunkItem it;
  int lo = 0, hi = B;                  // prefix[lo] <= x < prefix[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.prefix[mid] <= x) lo = mid; else hi = mid;
  }
  it.b = lo;
  const long long per = (a.prefix[lo + 1] - a.prefix[lo]) / Hkv;
  it.hk = (int)((x - a.prefix[lo]) / per);
  it.x0 = a.prefix[lo] + per * it.hk;
  const ChunkSeq s = a.seq[lo];
  const int n_rt = (s.n * g + kChunkRows - 1) / kChunkRows;
  for (int first = 0;; first += 32) {
    it.rt = first + lane < n_rt ? first + lane : n_rt - 1;
    chunk_item_of(s, g, it);
    long long end = first + lane < n_rt ? (long long)it.weight * it.kt : 0;            // positions up to the end of the lane's row tile
    for (int d = 1; d < 32; d <<= 1) {
      const long long other = __shfl_up_sync(0xffffffffu, end, d);
      if (lane >= d) end += other;
    }
    const uint32_t behind = __ballot_sync(0xffffffffu, it.x0 + end > x);
    if (behind != 0u || first + 32 >= n_rt) {
      const int hit = behind != 0u ? __ffs(behind) - 1 : n_rt - 1 - first;
      const long long before = __shfl_sync(0xffffffffu, end, hit > 0 ? hit - 1 : 0);
      it.x0 += hit > 0 ? before : 0;
      it.rt = first + hit;
      chunk_item_of(s, g, it);
      return it;
    }
    it.x0 += __shfl_sync(0xffffffffu, end, 31);
  }
}

// The item behind it; its position is known to be below the total.
__device__ inline void chunk_next(const ChunkArgs& a, int Hkv, int g, ChunkItem& it) {
  it.x0 += (long long)it.weight * it.kt;
  if (++it.rt == it.n_rt) {
    it.rt = 0;
    if (++it.hk == Hkv) {
      it.hk = 0;
      do ++it.b; while (a.prefix[it.b + 1] == a.prefix[it.b]);
    }
  }
  chunk_item_of(a.seq[it.b], g, it);
}

// Key tiles [j0, j1) of the item that a thread block with the positions [begin, end) has.
__host__ __device__ inline void chunk_tiles(const ChunkItem& it, long long begin, long long end, int& j0, int& j1) {
  const long long len = (long long)it.weight * it.kt;
  const long long lo = begin > it.x0 ? begin - it.x0 : 0, hi = end < it.x0 + len ? end - it.x0 : len;
  j0 = (int)(lo >> (it.weight - 1));
  j1 = (int)(hi >> (it.weight - 1));
}

size_t chunk_scratch_bytes(int g, int n_tokens);
cudaError_t chunk_attention_setup();
// Splits the work, enqueues the attention and, where items are shared, the merge; fills in what of the arguments follows from the sequences.
cudaError_t launch_chunk_attention(const LayerView& lv, ChunkArgs& a, int n_sms, cudaStream_t stream, int* launches);

}  // namespace mixkvq
