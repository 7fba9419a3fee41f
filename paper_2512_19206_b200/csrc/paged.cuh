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
  // both, their loads under way together
  __device__ void sequence(int b, int& c, int& l) const {
    const int given = counts == nullptr ? n : counts[b];
    const long long held = lens[b], most = (long long)max_pages << lg_page;
    c = min(max(given, 0), n);
    const long long all = held + (add_counts ? c : 0);
    l = (int)(all < 0 ? 0 : all > most ? most : all);
    if (c != given || l != all) atomicOr(status, (uint32_t)MIXKVQ_DEV_BAD_LENGTH);
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
  uint64_t minus_zero = 0x8000000080000000ull;      // two of them (see f2_mul)
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
cudaError_t launch_paged_attention(const PagedAttention& a, int n_sms, cudaStream_t stream, int* launches, int* form);      // form: MIXKVQ_PAGED_*
// capacity: tokens that the pages of a sequence hold at most.  _need: what a launch of these sizes uses; _bytes: that or more, never less for a larger batch, n or capacity
size_t paged_workspace_need(int Hkv, int g, int batch, int n, long long capacity);
size_t paged_workspace_bytes(int Hkv, int g, int batch, int n, long long capacity);
// many query rows (tcgen05)
long long paged_chunk_capacity();                // the largest that it takes
size_t paged_chunk_workspace_need(int Hkv, int batch, long long capacity);
size_t paged_chunk_workspace_bytes(int Hkv, int batch, long long capacity);
cudaError_t paged_chunk_setup();
cudaError_t launch_paged_chunk(const PagedAttention& a, int n_sms, cudaStream_t stream, int* launches);
cudaError_t paged_attention_setup();
cudaError_t launch_rope_partial(const RopePartial& a, int n_sms, cudaStream_t stream);
cudaError_t launch_rope_tables(const RopeTables& a, int n_sms, cudaStream_t stream);

namespace {

__device__ __forceinline__ float bf16_half(uint32_t w, int e) { return e ? __uint_as_float(w & 0xFFFF0000u) : __uint_as_float(w << 16); }
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// ---- Rotation, two channels per instruction of the FMA pipe.  The arithmetic is that of rotate_one: every product and every sum a single fp32 operation rounded to
// nearest (no contraction: the products and sums below are instructions of their own), the result rounded to bf16.
struct F2 {
  uint64_t v;
};
__device__ __forceinline__ F2 f2(float a, float b) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
  return r;
}
// (As a multiply-add of -0, which is the product with its sign: a product instruction of this form is contracted with the sum behind it, its .rn notwithstanding, and 1 bf16 result
// in 60000 differed.  The -0 is a parameter of the launch: one that the assembler sees leads to the same.)
__device__ __forceinline__ F2 f2_mul(F2 a, F2 b, F2 minus_zero) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(minus_zero.v));
  return r;
}
__device__ __forceinline__ F2 f2_add(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 f2_sub(F2 a, F2 b) {
  F2 r;
  asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ void f2_get(F2 x, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x.v)); }

// 8 cosines and sines of a token: pairs at .. at + 7 of the table row, two per register pair.
struct Angles {
  F2 c[4], s[4];
};
__device__ __forceinline__ void load_angles(const float* cos_t, const float* sin_t, size_t at, int n, Angles& x) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (4 * k >= n) break;
    const float4 c = *reinterpret_cast<const float4*>(cos_t + at + 4 * k), s = *reinterpret_cast<const float4*>(sin_t + at + 4 * k);
    x.c[2 * k] = f2(c.x, c.y);
    x.c[2 * k + 1] = f2(c.z, c.w);
    x.s[2 * k] = f2(s.x, s.y);
    x.s[2 * k + 1] = f2(s.z, s.w);
  }
}
// Two pairs whose first channels are a and whose second channels are b.
__device__ __forceinline__ void turn2(F2& a, F2& b, F2 c, F2 s, F2 mz) {
  const F2 y = f2_sub(f2_mul(a, c, mz), f2_mul(b, s, mz));
  b = f2_add(f2_mul(b, c, mz), f2_mul(a, s, mz));
  a = y;
}
// Pairs of neighbours in two words.
__device__ __forceinline__ void turn_neighbours(uint32_t& w0, uint32_t& w1, F2 c, F2 s, F2 mz) {
  F2 a = f2(bf16_half(w0, 0), bf16_half(w1, 0)), b = f2(bf16_half(w0, 1), bf16_half(w1, 1));
  turn2(a, b, c, s, mz);
  float a0, a1, b0, b1;
  f2_get(a, a0, a1);
  f2_get(b, b0, b1);
  w0 = bf16_pair(a0, b0);
  w1 = bf16_pair(a1, b1);
}

// Rows that are turned and nothing else: eight lanes have a row, a lane two chunks of 8 channels: in halves the two chunks of 8 pairs, otherwise neighbours; lanes behind the
// rotated part have two neighbouring chunks.
struct PairLane {
  int first, second;                       // chunks
  int mode;                                // 0: left as they are, 1: halves, 2: neighbours
  Angles x;
};
__device__ __forceinline__ PairLane pair_lane(const RopeTurn& t, int pos, int l, bool turns) {
  PairLane p;
  const int half = t.rotary >> 4;          // lanes with rotated channels
  p.mode = !turns || l >= half ? 0 : t.interleaved ? 2 : 1;
  p.first = turns && !t.interleaved ? (l < half ? l : 2 * l) : 2 * l;       // (l >= half: 2 half + 2 (l - half))
  p.second = p.mode == 1 ? l + half : p.first + 1;
  if (p.mode != 0) load_angles(t.cos_t, t.sin_t, (size_t)pos * (t.rotary >> 1) + 8 * l, 8, p.x);
  return p;
}
__device__ __forceinline__ void turn_pair(uint4& wa, uint4& wb, const PairLane& p, F2 mz) {
  if (p.mode == 0) return;
  uint32_t a[4] = {wa.x, wa.y, wa.z, wa.w}, b[4] = {wb.x, wb.y, wb.z, wb.w};
  if (p.mode == 1) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      F2 u = f2(bf16_half(a[j], 0), bf16_half(a[j], 1)), w = f2(bf16_half(b[j], 0), bf16_half(b[j], 1));
      turn2(u, w, p.x.c[j], p.x.s[j], mz);
      float lo, hi;
      f2_get(u, lo, hi);
      a[j] = bf16_pair(lo, hi);
      f2_get(w, lo, hi);
      b[j] = bf16_pair(lo, hi);
    }
  } else {
    turn_neighbours(a[0], a[1], p.x.c[0], p.x.s[0], mz);
    turn_neighbours(a[2], a[3], p.x.c[1], p.x.s[1], mz);
    turn_neighbours(b[0], b[1], p.x.c[2], p.x.s[2], mz);
    turn_neighbours(b[2], b[3], p.x.c[3], p.x.s[3], mz);
  }
  wa = make_uint4(a[0], a[1], a[2], a[3]);
  wb = make_uint4(b[0], b[1], b[2], b[3]);
}

}  // namespace

}  // namespace mixkvq
