// The paged 4-bit cache: where a token's codes and scales lie, what its kernels take, and the rotation of a part of the head that its append and
// rope_partial share.
//
// Pool: [layer][page][KV head] pieces of page_tokens tokens, a piece is page_tokens / 16 tiles of 16 tokens:
//   [K codes 1024 B][V codes 1024 B][K scales 16 x 512/G B][V scales 16 x 512/G B]
// A token has 64 bytes of codes in each of the two (Eq. 2 with 16 levels per group of G channels) and 128 / G words {z bf16, s bf16}: the scale above, so that words compare like scales.  Keys: channel
// c = 32 j + 8 t + i at byte 16 t + 4 j + i / 2, nibble i % 2, so that lane t of a quad finds eight channels of every group of 32 in one 16-byte load, in
// the order of a matrix operand.  Values: channel c = 32 j + 4 r + x at byte 8 r + 2 j + x / 2, nibble x % 2, the two halves of the 64 bytes swapped in
// tokens with bit 2 set: the eight bytes that lane group r takes of four tokens lie on different banks.
#pragma once

#include "common.cuh"

namespace mixkvq {

constexpr int kPagedTile = 16;                   // tokens

__host__ __device__ inline uint32_t paged_meta_bytes(int G) { return 512u / (uint32_t)G; }                  // of a token's keys (or values)
__host__ __device__ inline uint32_t paged_tile_bytes(int G) { return 2048u + 32u * paged_meta_bytes(G); }
__host__ __device__ inline uint32_t paged_k_meta(int row, int G) { return 2048u + (uint32_t)row * paged_meta_bytes(G); }
__host__ __device__ inline uint32_t paged_v_meta(int row, int G) { return 2048u + (uint32_t)(16 + row) * paged_meta_bytes(G); }

// One layer of a pool and a call's sequences.
struct PagedView {
  char* pool;                 // the layer's pages
  uint32_t* status;
  const int32_t* pages;       // [B][max_pages], rows pages_stride apart
  const int32_t* lens;        // [B] tokens held
  const int32_t* counts;      // [B] tokens of the call, null: n each
  uint64_t page_bytes;
  uint32_t piece_bytes, tile_bytes;
  int B, n, Hq, Hkv, g, G;
  int n_pages, lg_page, max_pages, pages_stride;
  int add_counts;             // attention: the tokens of the call come on top of lens (they have just been appended)

  // tokens of the call in sequence b
  __device__ int count(int b) const {
    if (counts == nullptr) return n;
    const int c = counts[b], ok = min(max(c, 0), n);
    if (ok != c) atomicOr(status, (uint32_t)MIXKVQ_DEV_BAD_LENGTH);
    return ok;
  }
  // tokens of sequence b in its pages
  __device__ int length(int b, int more) const {
    const long long l = (long long)lens[b] + more, most = (long long)max_pages << lg_page;
    const int ok = (int)(l < 0 ? 0 : l > most ? most : l);
    if (ok != l) atomicOr(status, (uint32_t)MIXKVQ_DEV_BAD_LENGTH);
    return ok;
  }
  // where token i behind the lens[b] of sequence b goes, -1: nowhere
  __device__ int place(int b, int i) const {
    const long long t = (long long)lens[b] + i;
    if (t >= 0 && t < (long long)max_pages << lg_page) return (int)t;
    atomicOr(status, (uint32_t)MIXKVQ_DEV_BAD_LENGTH);
    return -1;
  }
  // the piece of KV head h that token t (0 <= t < max_pages << lg_page) of sequence b is on, null where its page is none of the pool's
  __device__ char* piece(int b, int h, int t) const {
    const int p = pages[(size_t)b * pages_stride + (t >> lg_page)];
    if (p < 0 || p >= n_pages) {
      atomicOr(status, (uint32_t)MIXKVQ_DEV_BAD_PAGE);
      return nullptr;
    }
    return pool + (uint64_t)p * page_bytes + (uint64_t)h * piece_bytes;
  }
  __device__ uint32_t tile_of(int t) const { return (uint32_t)((t & ((1 << lg_page) - 1)) >> 4) * tile_bytes; }
};

struct RopeTurn {
  const float *cos_t, *sin_t;              // [n_positions][rotary / 2]; null: no rotation
  const int32_t* positions;                // [B][n]; null: the token's place in its sequence
  int n_positions, rotary, interleaved;
};

struct PagedAppend {
  PagedView view;
  RopeTurn turn;
  const void *k, *v, *q;                   // q null: keys and values alone
  void* q_out;                             // [B][Hq][n][128]
  RopeTensor tk, tv, tq;
};
struct PagedRead {
  PagedView view;
  void *k, *v;                             // [B][Hkv][n][128] bf16
};
struct PagedAttention {
  PagedView view;
  const void* q;                           // [B][Hq][n][128] bf16
  void* out;                               // [B][Hq][n][128]
  int out_bf16;
  float scale_log2e;
  float* parts;                            // workspace
  uint32_t max_polls, test_extra;
};
struct RopePartial {
  RopeTurn turn;
  const void *q, *k, *v;
  void *q_out, *k_out, *v_out;
  RopeTensor tq, tk, tv;
  uint32_t* status;
  int B, Hq, Hkv, n;
};
struct RopeTables {
  double turns[64];                        // the frequency of every pair, in half turns per position
  double factor;                           // of every entry
  float *cos_t, *sin_t;
  long long start;
  int n, half;
};

cudaError_t launch_paged_append(const PagedAppend& a, int n_sms, cudaStream_t stream);
cudaError_t launch_paged_read(const PagedRead& a, int n_sms, cudaStream_t stream);
cudaError_t launch_paged_attention(const PagedAttention& a, int n_sms, cudaStream_t stream, int* launches);
size_t paged_workspace_bytes(int Hkv, int g, int batch, int n, long long capacity);
// many query rows (tcgen05); capacity: tokens that the pages of a sequence hold at most
bool paged_chunk_fits(long long capacity);
size_t paged_chunk_workspace_bytes(int Hkv, int batch, long long capacity);
cudaError_t paged_chunk_setup();
cudaError_t launch_paged_chunk(const PagedAttention& a, int n_sms, cudaStream_t stream, int* launches);
cudaError_t paged_attention_setup();
cudaError_t launch_rope_partial(const RopePartial& a, int n_sms, cudaStream_t stream);
cudaError_t launch_rope_tables(const RopeTables& a, int n_sms, cudaStream_t stream);

namespace {

// What a thread turns its 8 channels (chunk c of a row of 16) by.  Sixteen neighbouring lanes have a row.
struct TurnChunk {
  float c[8], s[8];
  int other;                               // pairs in halves: the lane of the row that has the other channel of every pair
  int mode;                                // 0: left as they are, 1: first halves, 2: second halves, 3: pairs of neighbours
};
__device__ __forceinline__ TurnChunk turn_chunk_load(const RopeTurn& t, int pos, int c) {
  TurnChunk x;
  const int half = t.rotary >> 4;          // chunks of half a rotated part
  x.other = c;
  x.mode = t.cos_t == nullptr || c >= 2 * half ? 0 : t.interleaved ? 3 : c < half ? 1 : 2;
  if (x.mode == 1) x.other = c + half;
  if (x.mode == 2) x.other = c - half;
#pragma unroll
  for (int i = 0; i < 8; ++i) x.c[i] = 1.f, x.s[i] = 0.f;
  if (x.mode == 0) return x;
  const size_t at = (size_t)pos * (t.rotary >> 1) + (x.mode == 3 ? 4 * c : 8 * (x.mode == 1 ? c : c - half));
  const float4 c0 = *reinterpret_cast<const float4*>(t.cos_t + at), s0 = *reinterpret_cast<const float4*>(t.sin_t + at);
  x.c[0] = c0.x; x.c[1] = c0.y; x.c[2] = c0.z; x.c[3] = c0.w;
  x.s[0] = s0.x; x.s[1] = s0.y; x.s[2] = s0.z; x.s[3] = s0.w;
  if (x.mode != 3) {
    const float4 c1 = *reinterpret_cast<const float4*>(t.cos_t + at + 4), s1 = *reinterpret_cast<const float4*>(t.sin_t + at + 4);
    x.c[4] = c1.x; x.c[5] = c1.y; x.c[6] = c1.z; x.c[7] = c1.w;
    x.s[4] = s1.x; x.s[5] = s1.y; x.s[6] = s1.z; x.s[7] = s1.w;
  }
  return x;
}
__device__ __forceinline__ float bf16_half(uint32_t w, int e) { return e ? __uint_as_float(w & 0xFFFF0000u) : __uint_as_float(w << 16); }
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// The thread's 8 channels turned (every lane of the warp calls this): the arithmetic of rotate_one, that is single fp32 operations without contraction and
// one rounding to bf16.
__device__ __forceinline__ uint4 turn_chunk(uint4 own, const TurnChunk& t) {
  const uint32_t a[4] = {own.x, own.y, own.z, own.w};
  uint32_t b[4], y[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) b[j] = __shfl_sync(0xffffffffu, a[j], t.other, 16);
  if (t.mode == 0) return own;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (t.mode == 3) {
      const float x0 = bf16_half(a[j], 0), x1 = bf16_half(a[j], 1);
      y[j] = bf16_pair(rotate_one(x0, x1, t.c[j], t.s[j], true), rotate_one(x1, x0, t.c[j], t.s[j], false));
    } else {
      y[j] = bf16_pair(rotate_one(bf16_half(a[j], 0), bf16_half(b[j], 0), t.c[2 * j], t.s[2 * j], t.mode == 1),
                       rotate_one(bf16_half(a[j], 1), bf16_half(b[j], 1), t.c[2 * j + 1], t.s[2 * j + 1], t.mode == 1));
    }
  }
  return make_uint4(y[0], y[1], y[2], y[3]);
}

}  // namespace

}  // namespace mixkvq
