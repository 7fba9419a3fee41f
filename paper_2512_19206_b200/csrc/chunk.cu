// Attention of a chunk of new tokens over the mixed-precision cache and, causally, over itself, on the tcgen05 tensor cores.
//
//   o_j = sum_t softmax_t(scale q_j . k_t) v_t,   t over the sink, the packed blocks (dequantized, Eq. 3), the residual window and the
//   new tokens up to j.
//
// One thread block of 896 threads per SM, persistent over its share of the (item, key tile) line (chunk.cuh).  Per key tile of 128 keys:
//   warps 8-15, 16-23   make the tiles: four warps the keys of even tiles, four those of odd ones, eight the values.  Packed codes become fp16 in registers
//                       (c s + z, one rounding) and go to shared memory in the tensor core's canonical layout; an unquantized row is copied
//                       with bf16 -> fp16.  The packed bytes are read once per 256 query rows and never written back dequantized.
//   warp 24             issues every tcgen05.mma: S = Q K^T (operands in shared memory), O += P V (P in tensor memory).
//   warp 25, warp 26    the thread block's segments (its part of an item), two ahead; requests of later tiles' bytes into the L2 cache.
//   warps 0-3, 4-7      two softmax groups ("slots"), thread = query row = lane of tensor memory.  An item of more than 128 rows has its first 128 rows
//                       in slot 0 and the others in slot 1; in a smaller one both slots have the same rows, slot 0 the even key tiles and slot 1
//                       the odd ones, and their results meet at the end: the tensor core works for one slot while the other is in its softmax.
// Codes lie in the cache as mma.sync A fragments: the lane with row r and pair t of an 8 x 8 piece holds its two neighbouring channels (keys) or
// tokens (values).  With keys and values both stored K-major in shared memory that pair is 4 bytes at 16 r + 4 t = 4 lane of a core matrix, so a
// warp's store is 128 contiguous bytes (the keys': four of them).
// The running maximum is raised (and O rescaled, in tensor memory) only when a row's logits exceed it by more than 2^10, so that the rescaling is rare.  P is
// fp16 (11 significant bits), 2^5 times the probability relative to that maximum: below 2^15, inside fp16, and numbers down to 2^-19 of the maximum are rounded
// by 2^-11 of themselves, smaller ones by 2^-30 of the maximum.  The denominator sums P as it was rounded.  Sums, maxima, O are fp32.
// (Without the factor weights below 2^-25 were zero in P: 16384 keys 17.4 nats below one with values of zero gave nothing.)
//
// What bounds it (B200).  Few rows, long caches: the making of the tiles.  A key tile of 128 x 128 takes about 6850 warp instructions, three fifths of them logic,
// fp16 operations and stores of codes; 57 % of the issue slots are taken, a tile every 2500 cycles (2900 with start and end).  Eight sequences of 32768 tokens,
// 7b shape, 5 new tokens each: 104 us (the first version 225), 1.05 TB/s of the packed bytes.  Many rows: a slot's chain of
// product, softmax (3400 cycles of 128 logits a thread beside the tiles' making) and product, 5100 cycles per tile of 256 rows: 2048 tokens behind 32768, 7b
// shape, 1211 us = 0.82 PFLOP/s (2328 at first), the tensor pipe a third of the time.
#include <algorithm>

#include "chunk.cuh"
#include "tc_ops.cuh"

namespace mixkvq {

namespace {

constexpr int kTile = kChunkTile;
constexpr int kTileBytes = kTile * kD * 2;
constexpr int kThreads = 896;                             // 72 registers a thread at launch, shared out anew among the roles
constexpr int kSoftmaxThreads = 256;
constexpr int kIssueWarp = 24;
constexpr int kScratchOff = 6 * kTileBytes;               // per producer warp 640 bytes: scales and zero-points as fp16 pairs
constexpr int kMlOff = kScratchOff + 16 * 640;            // slot 1's maxima and denominators (128 x 8 bytes)
constexpr int kBarOff = kMlOff + 1024;
constexpr int kBars = 21;
constexpr int kReaders = 26;                              // of a segment: 8 softmax, 16 producer warps, the issuing one, the L2 requests
constexpr int kSegOff = kBarOff + 8 * kBars + 16;         // (the tensor-memory address and the producers' progress behind the barriers)
constexpr int kPoisonOff = kSegOff + 2 * 64;            // two segments' Poison
constexpr int kSmem = kPoisonOff + 2 * (4 + 3 * kD * 4);
enum Bar { kQFull = 0, kKFull = 1, kVFull = 3, kKEmpty = 5, kVEmpty = 7, kSFull = 9, kPReady = 11, kODone = 13, kDone = 15, kSegFull = 17, kSegEmpty = 19 };
constexpr uint32_t kPolls = 1u << 19;                    // of 4 us each: two seconds
constexpr float kRaise = 10.f;
constexpr float kShift = 5.f;
constexpr int kAhead = 8;
// Tiles whose values the tensor core sums.  It truncates: 3.5e-7 of the sum per tile, all in one direction, and addends below 2^-24 of it vanish.  Behind 512
// tiles (1.8e-4) a sum is set aside and joined with the next one in fp32.  524288 keys of equal weight: 1.4e-3 below the mean in one sum.  (A joint costs
// about 15 us of a segment's 1.4 ms; that there can be one, 1165 -> 1185 us for 2048 new tokens behind 32768, under 1 % elsewhere.)
constexpr int kMaxTiles = 512;

__device__ __forceinline__ void sts32(uint32_t a, uint32_t x) { asm volatile("st.shared.u32 [%0], %1;" ::"r"(a), "r"(x) : "memory"); }
__device__ __forceinline__ void sts16(uint32_t a, uint32_t x) { asm volatile("st.shared.u16 [%0], %1;" ::"r"(a), "h"((uint16_t)x) : "memory"); }
__device__ __forceinline__ void sts128(uint32_t a, uint4 x) {
  asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
}
// Four 8 x 8 pieces of 16-bit elements, a lane holding two neighbouring ones of row lane / 4 of each; lane 8 m + i gives the address of row i of piece m.
__device__ __forceinline__ void store_pieces(uint32_t a, uint32_t x0, uint32_t x1, uint32_t x2, uint32_t x3) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(x0), "r"(x1), "r"(x2), "r"(x3) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ uint32_t lds16(uint32_t a) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(a));
  return v;
}
__device__ __forceinline__ uint32_t hfma2_u(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
__device__ __forceinline__ bool phase_over(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(ok)
               : "r"(bar), "r"(parity)
               : "memory");
  return ok != 0;
}
// Polls a phase of a barrier up to max_polls times; false if it never completed.  A poll that finds nothing suspends the warp and returns after 7840 cycles (4.0
// us at 1.96 GHz), the same with other warps arriving on this barrier or completing phases of others beside it; a phase that completes ends it at once.
// Sleeping between polls gained nothing (20 to 500 ns: within 0.6 % in all of eight cases, either way).
__device__ __forceinline__ bool wait_phase(uint32_t bar, uint32_t parity, uint32_t max_polls) {
#pragma unroll 1
  for (uint32_t n = 0; !phase_over(bar, parity); ++n)
    if (n >= max_polls) return false;
  return true;
}
__device__ __forceinline__ uint4 rows_to_half(uint4 x) {
  return make_uint4(bf16x2_to_f16x2(x.x), bf16x2_to_f16x2(x.y), bf16x2_to_f16x2(x.z), bf16x2_to_f16x2(x.w));
}

__device__ __forceinline__ uint32_t hadd2_u(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("add.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t hmul2_u(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t hsub2_u(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// 1 where a half of a is above that of b, else 0
__device__ __forceinline__ uint32_t above2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("set.gt.f16x2.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
constexpr uint32_t kQuarter2 = 0x34003400u;               // the fp16 pair (0.25, 0.25)

// c s + z of field f (2 bits at bit 2 f of each half word), one rounding.  The number with the field's bits in its mantissa is 1024 + c (f even) or
// 1024 + 4 c (f odd), less 1024 it is exact, and for odd fields `s` is a quarter of the scale (it has 8 significant bits: exact too from 2^-15 on, below that
// off by up to 2^-25, 4 c times which goes into the value; fewer than two shifts and one constant per pair of fields, where a scale factor per field would cost a
// register or a move each).
__device__ __forceinline__ uint32_t and_or(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
// Products whose operands' descriptors (canonical layout, 128 bytes and 2048 bytes between core matrices) are given by their low words, address / 16 with the
// first distance: neighbouring steps differ by one 32-bit addition.
constexpr uint32_t kDescHi = (2048 >> 4) | (1u << 14);
__device__ __forceinline__ uint32_t desc_lo(uint32_t saddr) { return ((saddr >> 4) & 0x3FFFu) | ((128u >> 4) << 16); }
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 a, {%1, %5};\n\tmov.b64 b, {%2, %5};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t}" ::"r"(d),
      "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "n"(kDescHi)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a_tmem, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 b, {%2, %5};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n\t}" ::"r"(d),
      "r"(a_tmem), "r"(b_lo), "r"(idesc), "r"(accumulate), "n"(kDescHi)
      : "memory");
}

struct Magic {                           // the fp16 pairs 1024 and -1024, kept in registers (as literals each use cost a move)
  uint32_t plus, minus;
  __device__ __forceinline__ Magic() {
    asm volatile("mov.u32 %0, 0x64006400;" : "=r"(plus));
    asm volatile("mov.u32 %0, 0xE400E400;" : "=r"(minus));
  }
};
__device__ __forceinline__ uint32_t dequant2(const Magic& m, uint32_t w, int f, uint32_t s, uint32_t z) {
  const uint32_t x = and_or(w >> (4 * (f >> 1)), 0x00030003u << (2 * (f & 1)), m.plus);
  return hfma2_u(hadd2_u(x, m.minus), s, z);
}
// The same for 4-bit codes whose low and high pairs of bits are in two planes.
__device__ __forceinline__ uint32_t dequant4(const Magic& m, uint32_t lo, uint32_t hi, int f, uint32_t s, uint32_t z) {
  const int sh = 4 * (f >> 1), p = 2 * (f & 1);
  const uint32_t low = 0x00030003u << p, l = lo >> sh, h = sh == 0 ? hi << 2 : hi >> (sh - 2);
  const uint32_t c = (l & low) | (h & ~low), x = and_or(c, 0x000F000Fu << p, m.plus);
  return hfma2_u(hadd2_u(x, m.minus), s, z);
}

__device__ __forceinline__ void prefetch_bulk(const void* p, uint32_t bytes) {
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p), "r"(bytes) : "memory");
}

struct Rows {                            // a stream's unquantized rows: residual window, sink, new tokens
  const uint16_t *res, *sink, *fresh;
  int r, c0, total;                      // rows of the window; of the window and the sink; all
  __device__ __forceinline__ const uint4* row(int i) const {
    return reinterpret_cast<const uint4*>(i < r ? res + (size_t)i * kD : i < c0 ? sink + (size_t)(i - r) * kD : fresh + (size_t)(i - c0) * kD);
  }
};

// A warp's unit: every fourth (the keys' warps: every eighth) one of the stream, from tile to tile.  (Blocks and units are counted on; a division and
// two long multiplications per tile and warp were a fifth of the instructions.)
struct Cursor {
  const char* blk;                       // its block
  const uint2* entry;                    // the block's table entry
  int unit, u;                           // its number in the stream and in the block
  uint32_t shift;                        // units of a key group: 2^shift
  __device__ __forceinline__ Cursor(const LayerView& lv, int stream, int first) {
    const int bi = first / lv.U;
    blk = lv.base + (size_t)stream * lv.base_stride + (size_t)bi * lv.base_bytes;
    entry = reinterpret_cast<const uint2*>(lv.table + (size_t)stream * lv.table_stride) + bi;
    unit = first;
    u = first - bi * lv.U;
    shift = lv.VG == 4 ? 0u : lv.VG == 2 ? 1u : 2u;
  }
  // n units on: n / U blocks and n % U units
  __device__ __forceinline__ void next(const LayerView& lv, int n, int blocks, int units) {
    unit += n;
    u += units;
    if (u >= lv.U) {
      u -= lv.U;
      blocks += 1;
    }
    blk += (uint32_t)blocks * lv.base_bytes;
    entry += blocks;
  }
  __device__ __forceinline__ const char* codes(const LayerView& lv) const { return blk + ((uint32_t)u * lv.unit_bytes + 512u * (((uint32_t)u >> shift) + 1)); }
  __device__ __forceinline__ const char* meta(const LayerView& lv) const {
    const uint32_t group = (uint32_t)u >> shift;
    return blk + ((group << shift) * lv.unit_bytes + 512u * group);
  }
};

// Half a unit's packed values (a unit's keys) on their way to shared memory: requested one tile ahead.
struct Packed {
  uint4 c, h;
  uint2 meta;
};
struct PackedKeys {
  uint4 c0, c1, h0, h1, meta;
};

// ---- keys: warp w of four makes rows 32 w .. 32 w + 31 of the tile at shared address `tile`; two such groups of warps take the tiles in turn, so that two
// are on their way at any time (a tile is mostly latency: loads, barriers, chains of a few dependent instructions)
// A block's promoted channels: `id` is the lane's entry of the list of BF16 channels, raw their first two pairs (the lane's token), `pair4` the lane's
// entry of the list of UINT4 channel pairs, high the first four pairs' high plane, ex the block's extras, exu this unit's.
struct Promoted {
  int n16, n4;
  uint32_t id, raw[2], pair4, high[4];
  const char *ex, *exu;
};
// Word of the UINT4 high plane that holds the lane's token, of pair 0, and the place of its two bits there (the pair's second channel: 16 further on)
__device__ __forceinline__ const uint32_t* high_plane(const Promoted& p, int lane) {
  return reinterpret_cast<const uint32_t*>(p.exu + 128 * ((p.n16 + 1) >> 1)) + (lane & 3);
}
__device__ __forceinline__ int high_bit(int lane) { return 8 * ((lane >> 2) & 1) + 2 * (2 * (lane >> 4) + ((lane >> 3) & 1)); }
template <int kU4>
__device__ __forceinline__ Promoted request_promoted(const char* extras, uint2 entry, int u, int lane) {
  Promoted p;
  p.n16 = entry.y & 0xFF;
  p.n4 = (entry.y >> 8) & 0xFF;
  p.id = kD;
  p.raw[0] = p.raw[1] = 0u;
  p.ex = extras + (size_t)entry.x * 16;
  p.exu = p.ex + extras_header_bytes(p.n16, p.n4) + (uint32_t)u * extras_unit_bytes(p.n16, p.n4, kU4 == 2);
  if (lane < p.n16) p.id = reinterpret_cast<const uint8_t*>(p.ex)[lane];
  if (p.n16 > 0) p.raw[0] = reinterpret_cast<const uint32_t*>(p.exu)[lane];
  if (p.n16 > 2) p.raw[1] = reinterpret_cast<const uint32_t*>(p.exu)[32 + lane];
  if (kU4 == 1 && p.n4 > 0) {
    const int pairs = (p.n4 + 1) >> 1;
    p.pair4 = 0xFFFFu;
    if (lane < pairs) p.pair4 = reinterpret_cast<const uint16_t*>(p.ex + ((p.n16 + 1) & ~1))[lane];
    const uint32_t* high = high_plane(p, lane);
#pragma unroll
    for (int i = 0; i < 4; ++i) p.high[i] = i < pairs ? high[4 * i] : 0u;
  }
  return p;
}
template <int kU4>
__device__ __forceinline__ PackedKeys request_keys(const LayerView& lv, const Cursor& at, const Promoted& more, int lane) {
  PackedKeys p{};
  const uint4* codes = reinterpret_cast<const uint4*>(at.codes(lv)) + lane;
  p.c0 = codes[0];
  p.c1 = codes[32];
  p.meta = reinterpret_cast<const uint4*>(at.meta(lv))[lane];
  if (kU4 == 2 && more.n4 != 0) {
    const uint4* hi = reinterpret_cast<const uint4*>(more.exu + 128 * ((more.n16 + 1) >> 1)) + lane;
    p.h0 = hi[0];
    p.h1 = hi[32];
  }
  return p;
}

// The unit's two-bit (kU4 = 2: four-bit) codes.
template <int kU4>
__device__ __forceinline__ void make_keys(const PackedKeys& p, uint32_t tile, uint32_t scratch, int w, int lane, const Magic& magic) {
  // Scales and zero-points of channel pairs (16 kt + 8 ch + 2 t, + 1) as fp16 pairs: word 36 ch + 8 t + kt, zero-points 72 words on (odd kt: a quarter of the
  // scale).  The lane has the pairs 2 lane and 2 lane + 1: kt = lane / 4, ch = lane / 2 % 2, t = 2 (lane % 2) and the next.
  {
    const uint32_t at = scratch + 4 * (36 * ((lane >> 1) & 1) + 16 * (lane & 1) + (lane >> 2));
    const uint32_t s0 = bf16x2_to_f16x2(__byte_perm(p.meta.x, p.meta.y, 0x5410)), s1 = bf16x2_to_f16x2(__byte_perm(p.meta.z, p.meta.w, 0x5410));
    sts32(at, lane & 4 ? hmul2_u(s0, kQuarter2) : s0);
    sts32(at + 32, lane & 4 ? hmul2_u(s1, kQuarter2) : s1);
    sts32(at + 288, bf16x2_to_f16x2(__byte_perm(p.meta.x, p.meta.y, 0x7632)));
    sts32(at + 320, bf16x2_to_f16x2(__byte_perm(p.meta.z, p.meta.w, 0x7632)));
  }
  __syncwarp();
  // (a rolled loop: every role's straight-line code together runs out of the instruction cache.  Without UINT4 channels two rounds of it are shorter, 8 x 32768
  // tokens of the 7b shape with drafts 104.7 us and 106.0; with them longer, 124.7 and 119.7 over ragged lengths.  Four pieces a store: against a store of 4 bytes per piece
  // and lane, draft-sized chunk over 8 sequences of the 7b shape 108 us and 111; the values' warps, which have fewer registers, gained nothing by it.)
  const uint32_t out = tile + 4 * w * 2048 + 256 * (lane >> 3) + 16 * (lane & 7), in = scratch + 32 * (lane & 3);
#pragma unroll (kU4 == 0 ? 2 : 1)
  for (int i = 0; i < 4; ++i) {          // of every 16 channels the upper or lower 8 (ch), channels 64 kh ..
    const int ch = i >> 1, kh = i & 1;
    const uint32_t at = in + 144 * ch + 16 * kh, to = out + 128 * ch + 1024 * kh;
    const uint4 s4 = lds128(at), z4 = lds128(at + 288);
    const uint32_t s[4] = {s4.x, s4.y, s4.z, s4.w}, z[4] = {z4.x, z4.y, z4.z, z4.w};
    const uint32_t c[4] = {(ch ? p.c0.z : p.c0.x) >> (8 * kh), (ch ? p.c0.w : p.c0.y) >> (8 * kh), (ch ? p.c1.z : p.c1.x) >> (8 * kh),
                           (ch ? p.c1.w : p.c1.y) >> (8 * kh)};
    const uint32_t h[4] = {(ch ? p.h0.z : p.h0.x) >> (8 * kh), (ch ? p.h0.w : p.h0.y) >> (8 * kh), (ch ? p.h1.z : p.h1.x) >> (8 * kh),
                           (ch ? p.h1.w : p.h1.y) >> (8 * kh)};
#pragma unroll
    for (int r = 0; r < 4; ++r)          // rows 8 r ..
    {
      uint32_t x[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = kU4 == 2 ? dequant4(magic, c[r], h[r], k, s[k], z[k]) : dequant2(magic, c[r], k, s[k], z[k]);
      store_pieces(to + r * 2048, x[0], x[1], x[2], x[3]);
    }
  }
}

// The promoted channels replace their codes' values.
template <int kU4>
__device__ __forceinline__ void put_promoted(Promoted& p, uint32_t tile, uint32_t scratch, int w, int lane) {
  if ((p.n16 | (kU4 == 1 ? p.n4 : 0)) == 0) return;
  __syncwarp();                          // the base codes are stored
  const uint32_t row = tile + (4 * w + (lane >> 3)) * 2048 + (lane & 7) * 16;           // the lane's token
  auto offset = [](uint32_t d) { return (d >> 3) * 128 + (d & 7) * 2; };
  uint32_t mine = offset(p.id);          // of the lane's list entry
#pragma unroll 1
  for (int i = 0; 2 * i < p.n16; ++i) {
    const uint32_t o0 = __shfl_sync(0xffffffffu, mine, (2 * i) & 31), o1 = __shfl_sync(0xffffffffu, mine, (2 * i + 1) & 31), both = bf16x2_to_f16x2(p.raw[0]);
    sts16(row + o0, both & 0xFFFFu);
    if (2 * i + 1 < p.n16) sts16(row + o1, both >> 16);
    p.raw[0] = p.raw[1];
    if (2 * i + 4 < p.n16) p.raw[1] = reinterpret_cast<const uint32_t*>(p.exu)[(i + 2) * 32 + lane];
    if (((2 * i + 2) & 31) == 0 && 2 * i + 2 + lane < p.n16) mine = offset(reinterpret_cast<const uint8_t*>(p.ex)[2 * i + 2 + lane]);
  }
  if (kU4 == 1 && p.n4 > 0) {
    // UINT4 channels: (c_lo + 4 c_hi) s + z, one rounding.  The low code is found again from what the base store left, c_lo s + z rounded: less z it lies
    // nearest to its own multiple of s (where s is below the rounding, that of another multiple may be as near: the value is then off by at most
    // three halves of a step instead of a half).  Both channels of a pair in fp16 pairs: 121 us for a draft-sized chunk of eight sequences, 7b shape, three
    // tiers; one after the other in fp32 138; with the high code's 4 c_hi s added to the rounded c_lo s + z, a second rounding, 127.  (The low codes
    // read again cost a round trip to the L2 cache every four channels.)
    const int pairs = (p.n4 + 1) >> 1, bit = high_bit(lane);
    const uint32_t* high = high_plane(p, lane);
#pragma unroll 1
    for (int i0 = 0; i0 < pairs; i0 += 4) {
      if (i0 == 32) p.pair4 = 32 + lane < pairs ? reinterpret_cast<const uint16_t*>(p.ex + ((p.n16 + 1) & ~1))[32 + lane] : 0xFFFFu;
      uint32_t hw[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        hw[k] = p.high[k];
        if (i0 + 4 + k < pairs) p.high[k] = high[4 * (i0 + 4 + k)];
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t two = i0 + k < pairs ? __shfl_sync(0xffffffffu, p.pair4, (i0 + k) & 31) : 0xFFFFu;
        const uint32_t d0 = two & 0xFFu, d1 = two >> 8;
        if (d0 < kD) {                   // (the whole warp's decision, and whether the pair has a second channel)
          const uint32_t e1 = d1 < kD ? d1 : d0, at0 = row + offset(d0), at1 = row + offset(e1);
          auto meta = [&](uint32_t d) { return scratch + 4 * (36 * ((d >> 3) & 1) + 8 * ((d & 7) >> 1) + (d >> 4)) + 2 * (d & 1); };
          auto both = [](uint32_t a0, uint32_t a1) { return __byte_perm(lds16(a0), lds16(a1), 0x5410); };
          const uint32_t m0 = meta(d0), m1 = meta(e1);
          // (odd 16-channel pieces have a quarter of the scale in store)
          const uint32_t s = hmul2_u(both(m0, m1), (d0 & 16 ? 0x4400u : 0x3C00u) | (e1 & 16 ? 0x44000000u : 0x3C000000u)), z = both(m0 + 288, m1 + 288);
          const uint32_t low = hsub2_u(both(at0, at1), z), twice = hadd2_u(low, low);
          uint32_t c = hadd2_u(((hw[k] >> bit << 2) & 0x000C000Cu) | 0x64006400u, 0xE400E400u);      // 4 c_hi
          c = hadd2_u(c, above2(twice, s));
          c = hadd2_u(c, above2(twice, hmul2_u(s, 0x42004200u)));            // 3 s
          c = hadd2_u(c, above2(twice, hmul2_u(s, 0x45004500u)));            // 5 s
          const uint32_t y = hfma2_u(c, s, z);
          sts16(at0, y & 0xFFFFu);
          if (d1 < kD) sts16(at1, y >> 16);
        }
      }
    }
  }
}

// ---- values: warp (w, half) makes keys 32 w .. 32 w + 31 of channels 64 half .. + 63, stored channel by channel (K-major for O = P V)
// meta0, meta1: where the lane's token has the scales of the half's two groups of 32 channels (the same one twice where a group is wider)
template <bool kV4>
__device__ __forceinline__ Packed request_values(const LayerView& lv, const Cursor& at, int half, int lane, uint32_t meta0, uint32_t meta1) {
  Packed p{};
  const char* unit = at.codes(lv);
  p.c = reinterpret_cast<const uint4*>(unit + 1024)[32 * half + lane];
  p.meta = make_uint2(*reinterpret_cast<const uint32_t*>(unit + meta0), *reinterpret_cast<const uint32_t*>(unit + meta1));
  if (kV4) p.h = reinterpret_cast<const uint4*>(unit + 2048 + 128 * lv.VG)[32 * half + lane];
  return p;
}

template <bool kV4>
__device__ __forceinline__ void make_values(const Packed& p, uint32_t tile, uint32_t scratch, int w, int half, int lane, const Magic& magic) {
  // scales of tokens (8 o + 2 t, + 1) as fp16 pairs: word 16 i + 4 t + o for 32 channels i, zero-points 32 words on; the lane has token
  // 8 o + 2 t + e = lane
  {
    const uint32_t at = scratch + 4 * (4 * ((lane >> 1) & 3) + (lane >> 3)) + 2 * (lane & 1);
    const uint32_t a = bf16x2_to_f16x2(p.meta.x), b = bf16x2_to_f16x2(p.meta.y);
    sts16(at, (lane & 8 ? hmul2_u(a, kQuarter2) : a) & 0xFFFFu);       // (odd o: a quarter of the scale)
    sts16(at + 128, a >> 16);
    sts16(at + 64, (lane & 8 ? hmul2_u(b, kQuarter2) : b) & 0xFFFFu);
    sts16(at + 192, b >> 16);
  }
  __syncwarp();
  uint32_t c0 = p.c.x, c1 = p.c.y, h0 = p.h.x, h1 = p.h.y;
  uint32_t to = tile + half * 8 * 2048 + 4 * w * 128 + 4 * lane, at = scratch + 16 * (lane & 3);
#pragma unroll 1
  for (int i = 0; i < 2; ++i) {          // 32 channels
    const uint4 s4 = lds128(at), z4 = lds128(at + 128);
    const uint32_t s[4] = {s4.x, s4.y, s4.z, s4.w}, z[4] = {z4.x, z4.y, z4.z, z4.w};
#pragma unroll
    for (int f = 0; f < 8; ++f)
      sts32(to + (f >> 2) * 2048 + (f & 3) * 128, kV4 ? dequant4(magic, c0, h0, f, s[f & 3], z[f & 3]) : dequant2(magic, c0, f, s[f & 3], z[f & 3]));
#pragma unroll
    for (int f = 0; f < 8; ++f)
      sts32(to + (2 + (f >> 2)) * 2048 + (f & 3) * 128, kV4 ? dequant4(magic, c1, h1, f, s[f & 3], z[f & 3]) : dequant2(magic, c1, f, s[f & 3], z[f & 3]));
    c0 = p.c.z;
    c1 = p.c.w;
    h0 = p.h.z;
    h1 = p.h.w;
    to += 4 * 2048;
    at += 64;
  }
}

// Unquantized rows 32 w .. + 31 of tail tile t, rows past the last as zeros.  Keys K-major (warp w), values as they lie (MN-major; warp (w, half): channels
// 64 half .. + 63).
__device__ __forceinline__ void copy_key_rows(const Rows& x, int t, uint32_t tile, int w, int lane) {
#pragma unroll
  for (int c = 0; c < 16; c += 4) {      // (all at once took more registers than the warps have)
    uint4 y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = kTile * t + 32 * w + 8 * i + (lane & 7);
      y[i] = make_uint4(0u, 0u, 0u, 0u);
      if (row < x.total) y[i] = x.row(row)[c + (lane >> 3)];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) sts128(tile + (4 * w + i) * 2048 + (c + (lane >> 3)) * 128 + (lane & 7) * 16, rows_to_half(y[i]));
  }
}
// Values that are no numbers (in fp16: beyond 65504 too).  The tensor core multiplies a masked value with a probability of 0, and 0 times NaN or infinity
// is NaN: one such element among the new tokens would reach the rows before its own.  They go to the product as zeros, and what they do to the rows that see
// them is kept per channel: the first new token (-1: a row of the window or the sink) with a NaN, with infinity, with minus infinity.  `any`: there is one.
struct Poison {
  int any, first[3][kD];
};
constexpr int kNever = 0x7FFFFFFF;
__device__ __forceinline__ float poison_of(const Poison& p, int channel, int tok) {     // what a row of token tok has to add
  const bool nan = p.first[0][channel] <= tok, plus = p.first[1][channel] <= tok, minus = p.first[2][channel] <= tok;
  return nan || (plus && minus) ? __int_as_float(0x7FFFFFFF) : plus ? INFINITY : minus ? -INFINITY : 0.f;
}
__device__ __forceinline__ uint32_t not_finite(uint32_t h) { return ((h & 0x7C007C00u) + 0x04000400u) & 0x80008000u; }   // (either half of an fp16 pair)

__device__ __forceinline__ void copy_value_rows(const Rows& x, int t, uint32_t tile, int w, int half, int lane, Poison* poison) {
  const int row = kTile * t + 32 * w + lane;
  const uint4* src = row < x.total ? x.row(row) + 8 * half : nullptr;
  const uint32_t to = tile + 8 * half * 2048 + (4 * w + (lane >> 3)) * 128 + (lane & 7) * 16;
  uint32_t bad = 0u;
#pragma unroll
  for (int c = 0; c < 8; c += 4) {
    uint4 y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = src != nullptr ? src[c + i] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y[i] = rows_to_half(y[i]);
      bad |= not_finite(y[i].x) | not_finite(y[i].y) | not_finite(y[i].z) | not_finite(y[i].w);
      sts128(to + (c + i) * 2048, y[i]);
    }
  }
  if (bad != 0u) {                       // (the lane's own pieces; a call here took the kernel's registers apart)
#pragma unroll 1
    for (int e = 0; e < kD / 2; ++e) {
      const uint32_t at = to + (e >> 3) * 2048 + 2 * (e & 7), h = lds16(at);
      if ((h & 0x7C00u) != 0x7C00u) continue;
      atomicMin(&poison->first[(h & 0x3FFu) ? 0 : (h & 0x8000u) ? 2 : 1][64 * half + e], row < x.c0 ? -1 : row - x.c0);
      sts16(at, 0u);
    }
    *reinterpret_cast<volatile int*>(&poison->any) = 1;
  }
}

__device__ __forceinline__ void tmem_ld32_issue(uint32_t taddr, uint32_t (&u)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,"
      "%27,%28,%29,%30,%31}, [%32];"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]), "=r"(u[10]),
        "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]), "=r"(u[17]), "=r"(u[18]), "=r"(u[19]), "=r"(u[20]),
        "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]), "=r"(u[25]), "=r"(u[26]), "=r"(u[27]), "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_wait_ld32(uint32_t (&u)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(u[0]), "+r"(u[1]), "+r"(u[2]), "+r"(u[3]), "+r"(u[4]), "+r"(u[5]), "+r"(u[6]), "+r"(u[7]), "+r"(u[8]), "+r"(u[9]),
                 "+r"(u[10]), "+r"(u[11]), "+r"(u[12]), "+r"(u[13]), "+r"(u[14]), "+r"(u[15]), "+r"(u[16]), "+r"(u[17]), "+r"(u[18]), "+r"(u[19]),
                 "+r"(u[20]), "+r"(u[21]), "+r"(u[22]), "+r"(u[23]), "+r"(u[24]), "+r"(u[25]), "+r"(u[26]), "+r"(u[27]), "+r"(u[28]), "+r"(u[29]),
                 "+r"(u[30]), "+r"(u[31])
               :
               : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&u)[32]) {
  tmem_ld32_issue(taddr, u);
  tmem_wait_ld32(u);
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&u)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7])
               : "r"(taddr)
               : "memory");
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(u[0]), "+r"(u[1]), "+r"(u[2]), "+r"(u[3]), "+r"(u[4]), "+r"(u[5]), "+r"(u[6]), "+r"(u[7])
               :
               : "memory");
}
// The state of a row's softmax: its reference (in the log2 domain) and the sum of its probabilities, two halves.
struct RowState {
  float m, l0, l1;
  __device__ __forceinline__ float sum() const { return l0 + l1; }
};

// Raises the reference to mx if that is above it: what lies in tensor memory on the old one is rescaled, the sums at o_addr (unless they are the first tile's,
// which are not there yet) and the row's `written` pieces of P at s_addr.  At mx itself the largest probability is a power of two, which fp16 holds: the
// error of a decode-sized call over 8000 tokens is 2.7e-5 of the output's norm (6.4e-5 with references a whole number higher).  Only where the row has
// pieces of P already and rises because another row of the warp does, by 2^kRaise at most, it rises by a whole number: another factor would
// round those pieces again, and weights of more than 2^-10.  (Such rows not raised: 0.9 % longer for 2048 new tokens behind 32768.)  The
// products before this tile are complete: S is behind them in the tensor core's order.
__device__ __forceinline__ void raise(uint32_t s_addr, uint32_t o_addr, int written, bool first, float mx, RowState& row) {
  float by = fmaxf(mx - row.m, 0.f);
  if (written > 0 && by <= kRaise) by = floorf(by);
  const float m_new = row.m == -INFINITY ? mx : row.m + by, alpha = row.m == -INFINITY ? 1.f : ex2(-by);
  row.l0 *= alpha;
  row.l1 *= alpha;
  row.m = m_new;
  if (!first) {
#pragma unroll 1
    for (int d = 0; d < kD; d += 8) {
      uint32_t u[8];
      tmem_ld8(o_addr + d, u);
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = __float_as_uint(__uint_as_float(u[i]) * alpha);
      tmem_st8(o_addr + d, u);
    }
  }
  // (in fp32: a factor of 2^-20 has four bits in fp16.  2048 new tokens behind 32768 1204 us with that, 1211.)
#pragma unroll 1
  for (int h = 0; h < 4 * written; ++h) {
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
    uint32_t u[8];
    tmem_ld8(s_addr + 8 * h, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
      u[i] = pack_half2(p.x * alpha, p.y * alpha);
    }
    tmem_st8(s_addr + 8 * h, u);
  }
}

// l0 and l1 plus the halves of an fp16 pair.  (The denominator sums the probabilities as the product takes them: what rounding does to a dominating one is
// then in both.  With the ones before the rounding the error of the outputs was up to twice as large; 1185 us and 1204 for 2048 new tokens behind 32768,
// under 2 % elsewhere.  Converted first and added in pairs: 1271.  A piece is summed by itself: the same 65000 probabilities one after the other made the
// denominator wrong by up to 4.9e-4, and 32 of them are exact.)
__device__ __forceinline__ void add_half2(float& l0, float& l1, uint32_t pair) {
  asm("{\n\t.reg .f16 a, b;\n\tmov.b32 {a, b}, %2;\n\tadd.rn.f32.f16 %0, a, %0;\n\tadd.rn.f32.f16 %1, b, %1;\n\t}" : "+f"(l0), "+f"(l1) : "r"(pair));
}

// One tile of one slot's softmax, in one pass: the thread's row of S (128 fp32 at s_addr) becomes P (fp16 pairs over the first 64 of those columns), 32
// columns at a time.  Piece h of P lies inside the columns of S's pieces <= h.  The reference is raised only when a piece's largest logit exceeds it by
// more than 2^kRaise: P stays below 2^(kRaise + kShift), inside fp16, and that is rare behind the first tile.  The row's own pieces are h0 .. h1 - 1 (another lane has
// the same row's others); P is zero in the others.  kMask: the row sees the columns <= last only.
template <bool kMask>
__device__ __forceinline__ void softmax_tile(uint32_t s_addr, uint32_t o_addr, int h0, int h1, int last, bool first, float scale_log2e, RowState& row) {
  const uint64_t scale2 = pack2(scale_log2e, scale_log2e);
#pragma unroll 1
  for (int h = 0; h < 2; ++h) {
    if (2 * h >= h0 && 2 * h < h1) {
      uint32_t u[64];
      uint32_t(&ua)[32] = *reinterpret_cast<uint32_t(*)[32]>(&u[0]);
      uint32_t(&ub)[32] = *reinterpret_cast<uint32_t(*)[32]>(&u[32]);
      tmem_ld32_issue(s_addr + 64 * h, ua);
      tmem_ld32_issue(s_addr + 64 * h + 32, ub);
      tmem_wait_ld32(ua);
      tmem_wait_ld32(ub);
      const int lim = last - 64 * h;
      float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int i = 0; i < 64; i += 2) {
        if (kMask) {
          u[i] = i > lim ? 0xFF800000u : u[i];
          u[i + 1] = i + 1 > lim ? 0xFF800000u : u[i + 1];
        }
        mx4[(i >> 1) & 3] = fmaxf(fmaxf(mx4[(i >> 1) & 3], __uint_as_float(u[i])), __uint_as_float(u[i + 1]));
      }
      const float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * scale_log2e;
      if (__any_sync(0xffffffffu, mx > row.m + kRaise)) raise(s_addr, o_addr, 2 * h > h0 ? h : 0, first, mx, row);
      const float ref = row.m == -INFINITY ? 0.f : row.m - kShift;      // a row that has seen no key yet: all its logits are -inf, its P is 0
      const uint64_t ref2 = pack2(-ref, -ref);
      float l0 = 0.f, l1 = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint32_t wd[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float x0, x1;
          unpack2(fma2(pack2u(u[16 * k + 2 * i], u[16 * k + 2 * i + 1]), scale2, ref2), x0, x1);
          const float p0 = ex2(x0), p1 = ex2(x1);
          wd[i] = pack_half2(p0, p1);
          add_half2(l0, l1, wd[i]);
        }
        tmem_st8(s_addr + 32 * h + 8 * k, wd);
      }
      row.l0 += l0;
      row.l1 += l1;
    } else {
      const uint32_t zero[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
      tmem_st8(s_addr + 32 * h, zero);
      tmem_st8(s_addr + 32 * h + 8, zero);
      tmem_st8(s_addr + 32 * h + 16, zero);
      tmem_st8(s_addr + 32 * h + 24, zero);
    }
  }
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

// 32 channels of an output row
__device__ __forceinline__ void store_row(const ChunkArgs& a, size_t row, int d, const float (&y)[32]) {
  if (a.out_bf16) {
    uint4* dst = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.out) + row * kD + d);
#pragma unroll
    for (int i = 0; i < 32; i += 8) {
      uint32_t w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(y[i + 2 * k], y[i + 2 * k + 1]);
        w[k] = *reinterpret_cast<const uint32_t*>(&h);
      }
      dst[i / 8] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  } else {
    float4* dst = reinterpret_cast<float4*>(static_cast<float*>(a.out) + row * kD + d);
#pragma unroll
    for (int i = 0; i < 32; i += 4) dst[i / 4] = make_float4(y[i], y[i + 1], y[i + 2], y[i + 3]);
  }
}

// warps that arrive on a barrier
__device__ constexpr int arrivals(int i) {
  if (i == kQFull || i == kVFull || i == kVFull + 1) return 8;
  if (i == kKFull || i == kKFull + 1 || i == kPReady || i == kPReady + 1) return 4;
  return i == kSegEmpty || i == kSegEmpty + 1 ? kReaders : 1;
}

// What the roles need to know of a segment (a thread block's key tiles of one item, or up to kMaxTiles of them); stream < 0: there is none left.
struct Segment {
  int stream, j0, j1, packed_tiles;
  int units, r, c0, total;               // packed units; residual rows; residual and sink rows; unquantized rows that the item's rows may see
  int row0, rows_all, dual, whole;       // first row; rows of the stream; more than 128 rows; all of the item's key tiles end here: the result is its output
  int part, behind, pad[2];              // which of the thread block's two results; it holds that of the item's tiles before these
};

template <int n>
struct Literal {
  __host__ __device__ constexpr operator int() const { return n; }
};

// the first lane's value, the whole warp's
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }
__device__ __forceinline__ bool elect_one() {
  uint32_t e;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
  return e != 0;
}

// Weight of a partial result (maximum m, denominator l) in a sum that refers to `top`.  A NaN among the logits makes l NaN, whatever m is, and the row too,
// even where its weight would round to zero.
__device__ __forceinline__ float weight_of(float m, float l, float top) { return l != l ? l : m == -INFINITY ? 0.f : ex2(m - top); }
// sum + w y
__device__ __forceinline__ void add_scaled(float w, float4 y, float4& sum) {
  sum.x = fmaf(w, y.x, sum.x); sum.y = fmaf(w, y.y, sum.y); sum.z = fmaf(w, y.z, sum.z); sum.w = fmaf(w, y.w, sum.w);
}
// Infinities and NaNs of y.  A weight that has rounded to zero is positive all the same: they stay what they are.
__device__ __forceinline__ void add_not_finite(float4 y, float4& sum) {
  sum.x += isfinite(y.x) ? 0.f : y.x; sum.y += isfinite(y.y) ? 0.f : y.y; sum.z += isfinite(y.z) ? 0.f : y.z; sum.w += isfinite(y.w) ? 0.f : y.w;
}

__device__ __forceinline__ void softmax_sync() { asm volatile("barrier.cta.sync 1, 256;" ::: "memory"); }

// 4 channels of an output row
__device__ __forceinline__ void store4(const ChunkArgs& a, size_t at, float4 y) {
  if (a.out_bf16) {
    const __nv_bfloat162 p0 = __floats2bfloat162_rn(y.x, y.y), p1 = __floats2bfloat162_rn(y.z, y.w);
    *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + at) =
        make_uint2(*reinterpret_cast<const uint32_t*>(&p0), *reinterpret_cast<const uint32_t*>(&p1));
  } else {
    *reinterpret_cast<float4*>(static_cast<float*>(a.out) + at) = y;
  }
}

// Registers per thread of the roles: together no more than the block is launched with.  (Eight more for the keys' warps at the softmax warps' cost, 112 and
// 72: one sequence of 120000 tokens, 8b shape, one new token, 94 us and 91; 7b shape, a chunk of 2048 tokens behind 32768, 1162 and 1173.)
constexpr int kLaunchRegs = 72, kIssueRegs = 40;
struct Registers {
  int softmax, keys, values;
};
__host__ __device__ constexpr Registers registers_of(bool v4) { return v4 ? Registers{96, 80, 56} : Registers{104, 80, 48}; }
__host__ __device__ constexpr bool registers_fit(Registers r) { return 256 * (r.softmax + r.keys + r.values) + 128 * kIssueRegs <= kThreads * kLaunchRegs; }
static_assert(registers_fit(registers_of(false)) && registers_fit(registers_of(true)), "the shares are taken from what the thread block was launched with");
template <bool kMore, int kRegs>
__device__ __forceinline__ void set_registers() {
  if constexpr (kMore)
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegs) : "memory");
  else
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegs) : "memory");
}

// kU4: how the configuration can use the UINT4 tier: 0 never (no threshold or budget puts a channel there), 1 some channels (high plane per channel pair),
// 2 the 4-bit base (dense high plane)
template <int kU4, bool kV4>
__global__ void __launch_bounds__(kThreads, 1) chunk_attention_kernel(const __grid_constant__ LayerView lv, const __grid_constant__ ChunkArgs a) {
  constexpr Registers kRegs = registers_of(kV4);
  extern __shared__ __align__(128) unsigned char smem[];
  const uint32_t sbase = smem_u32(smem), qs = sbase, ks = sbase + 2 * kTileBytes, vs = sbase + 4 * kTileBytes;
  auto bar = [&](int i) { return sbase + (uint32_t)kBarOff + 8u * (uint32_t)i; };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + kBarOff + 8 * kBars);
  volatile int* progress = reinterpret_cast<volatile int*>(tmem_slot + 1);     // the tile that the producers are at
  Segment* segments = reinterpret_cast<Segment*>(smem + kSegOff);              // two places
  Poison* poison = reinterpret_cast<Poison*>(smem + kPoisonOff);               // of the segments in them
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (warp == kIssueWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (tid == 0) {
    for (int i = 0; i < kBars; ++i) mbar_init(bar(i), arrivals(i));
    *progress = 0;
    poison[0].any = poison[1].any = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (tid < 2 * 3 * kD) poison[tid / (3 * kD)].first[tid / kD % 3][tid % kD] = kNever;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tbase = *tmem_slot;
  dependency_wait();
  // tensor-memory columns: S / P of slot 0 at 0, of slot 1 at 128, O of slot 0 at 256, of slot 1 at 384
  bool dead = false;
  auto wait = [&](int i, uint32_t parity) {
    if (!dead && !wait_phase(bar(i), parity, a.max_polls)) {
      dead = true;
      atomicOr(lv.status, (uint32_t)MIXKVQ_DEV_COPY_TIMEOUT);
    }
    return !dead;
  };
  // The same for a whole warp.  (The first poll apart from the loop of `wait`: 2048 new tokens behind 32768, 7b shape, 1163 us and 1265.)
  auto there = [&](int i, uint32_t parity) {
    if (__all_sync(0xffffffffu, phase_over(bar(i), parity))) return true;
    return __all_sync(0xffffffffu, wait(i, parity)) != 0;
  };
  // The same for a group of `threads` threads: one warp polls, the others wait for it in the named barrier `id`.  The polling warp comes to the barrier in any
  // case, and all learn what it saw.
  auto group_wait = [&](int id, int threads, bool polls, int i, uint32_t parity) {
    uint32_t ok = 1;
    if (polls && i >= 0) ok = wait(i, parity);
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %0, 0;\n\tbarrier.cta.red.and.pred q, %1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "+r"(ok)
                 : "r"(id), "r"(threads)
                 : "memory");
    return ok != 0;
  };
  // the n-th segment is there; (a reader's warp has taken what it needs)
  auto segment_there = [&](int n) { return wait(kSegFull + (n & 1), (uint32_t)(n >> 1) & 1u); };
  auto segment_taken = [&](int n) {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar(kSegEmpty + (n & 1)));
  };

  if (warp >= kIssueWarp) {
    set_registers<false, kIssueRegs>();
    if (warp == kIssueWarp) {
      // ---------------------------------------------------------------- tensor-core issue
      // The whole warp goes through the loops and one lane issues; slots and stages are literals, and tensor memory starts at 0 (all of it was allocated), so
      // that descriptors and addresses are constants in uniform registers: moved there word by word, they took longer than the products.
      constexpr uint32_t kIdesc = make_idesc(128, 128, 0, 0), kIdescRows = make_idesc(128, 128, 0, 1);
      constexpr uint32_t kStep = kTileBytes >> 4;        // a tile further, in a descriptor
      const uint32_t qd = desc_lo(qs), kd = desc_lo(ks), vd = desc_lo(vs);
      const bool leader = elect_one();
      uint32_t used = 0, cnt = 0;                        // bit st: parity of the tiles that stage st has had; bit slot: parity of the slot's steps
      // S of `slot` from Q tile `qt` and key stage st; kLast: the stage's last use
      auto issue_s = [&](auto slot_, auto st_, auto qt_, auto last_) {
        constexpr int slot = slot_, st = st_, qt = qt_;
        tc_fence_after();
        if (leader) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            mma_ss(128 * slot, qd + qt * kStep + 16 * i, kd + st * kStep + 16 * i, kIdesc, i > 0);
          tc_commit(bar(kSFull + slot));
          if (last_) tc_commit(bar(kKEmpty + st));
        }
      };
      auto issue_o = [&](auto slot_, auto st_, auto last_, uint32_t idesc, bool first, bool end) {
        constexpr int slot = slot_, st = st_;
        if (!there(kPReady + slot, (cnt >> slot) & 1u)) return false;
        cnt ^= 1u << slot;
        tc_fence_after();
        if (leader) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            mma_ts(256 + 128 * slot, 128 * slot + 8 * i, vd + st * kStep + 16 * i, idesc, i > 0 || !first);
          if (last_) tc_commit(bar(kVEmpty + st));
          if (end) tc_commit(bar(kODone + slot));
        }
        return true;
      };
      constexpr Literal<0> k0{};
      constexpr Literal<1> k1{};
      for (int n = 0; there(kSegFull + (n & 1), (uint32_t)(n >> 1) & 1u); ++n) {
        const Segment& sg = segments[n & 1];
        const int stream = uniform(sg.stream), nt = uniform(sg.j1 - sg.j0), packed = uniform(sg.packed_tiles - sg.j0), dual = uniform(sg.dual);
        segment_taken(n);
        if (stream < 0 || !there(kQFull, n & 1)) break;
        auto keys_there = [&](int st) { return there(kKFull + st, (used >> st) & 1u); };
        auto idesc_of = [&](int j) { return j < packed ? kIdesc : kIdescRows; };
        bool ok;
        if (dual) {
          // tile j in stage j % 2, both slots: S(slot, j + 1) goes in behind O(slot, j)
          auto tile = [&](auto st, auto next, int j) {
            const uint32_t idesc = idesc_of(j);
            const bool more = j + 1 < nt;
            if (!there(kVFull + st, (used >> st) & 1u)) return false;
            used ^= 1u << st;
            if (!issue_o(k0, st, k0, idesc, j == 0, !more)) return false;
            if (more) {
              if (!keys_there(next)) return false;
              issue_s(k0, next, k0, k0);
            }
            if (!issue_o(k1, st, k1, idesc, j == 0, !more)) return false;
            if (more) issue_s(k1, next, k1, k1);
            return true;
          };
          ok = keys_there(0);
          if (ok) {
            issue_s(k0, k0, k0, k0);
            issue_s(k1, k0, k1, k1);
          }
          for (int j = 0; ok && j < nt; j += 2) {
            ok = tile(k0, k1, j);
            if (ok && j + 1 < nt) ok = tile(k1, k0, j + 1);
          }
        } else {
          // tile j in stage and slot j % 2: S(j + 2) goes in behind O(j)
          auto tile = [&](auto st, int j) {
            if (!there(kVFull + st, (used >> st) & 1u)) return false;
            used ^= 1u << st;
            if (!issue_o(st, st, k1, idesc_of(j), j < 2, j + 2 >= nt)) return false;
            if (j + 2 < nt) {
              if (!keys_there(st)) return false;
              issue_s(st, st, k0, k1);
            }
            return true;
          };
          ok = keys_there(0);
          if (ok) issue_s(k0, k0, k0, k1);
          if (ok && nt > 1) {
            ok = keys_there(1);
            if (ok) issue_s(k1, k1, k0, k1);
          }
          for (int j = 0; ok && j < nt; j += 2) {
            ok = tile(k0, j);
            if (ok && j + 1 < nt) ok = tile(k1, j + 1);
          }
        }
        if (!ok) break;
      }
      if (leader) tc_commit(bar(kDone));                 // every product issued above has finished when this one fires
      dead = false;
      there(kDone, 0);
    } else if (warp == kIssueWarp + 1) {
      // ---------------------------------------------------------------- the thread block's segments
      const int g = lv.g;
      const long long begin = chunk_begin(a.total, a.ctas, blockIdx.x), end = chunk_begin(a.total, a.ctas, blockIdx.x + 1);
      ChunkItem it = chunk_locate(a, lv.B, lv.Hkv, g, begin, lane);
      if (lane == 0) {
        a.at[blockIdx.x] = it;
        int n = 0;
        // the place of the n-th segment, once the one before in it is over
        auto place = [&]() -> Segment* {
          if (n >= 2 && !wait_phase(bar(kSegEmpty + (n & 1)), (uint32_t)((n >> 1) - 1) & 1u, a.max_polls)) {
            atomicOr(lv.status, (uint32_t)MIXKVQ_DEV_COPY_TIMEOUT);
            return nullptr;
          }
          if (n >= 2 && poison[n & 1].any != 0) {
#pragma unroll 1
            for (int i = 0; i < 3 * kD; ++i) poison[n & 1].first[0][i] = kNever;
            poison[n & 1].any = 0;
          }
          return &segments[n & 1];
        };
        auto announce = [&]() {
          mbar_arrive(bar(kSegFull + (n & 1)));
          n += 1;
        };
        Segment* sg = nullptr;
        for (;;) {
          int j, j1;
          chunk_tiles(it, begin, end, j, j1);
          const bool whole = j == 0 && j1 == it.kt;
          int behind = 0;
#pragma unroll 1
          while (j < j1) {
            sg = place();
            if (sg == nullptr) break;
            const ChunkSeq sq = a.seq[it.b];
            const int left = j1 - j, next = left <= kMaxTiles ? j1 : j + (left >= 2 * kMaxTiles ? kMaxTiles : left / 2);
            sg->stream = it.b * lv.Hkv + it.hk;
            sg->j0 = j;
            sg->j1 = next;
            sg->packed_tiles = it.packed_tiles;
            sg->units = sq.units;
            sg->r = sq.tail & 0xFFFF;
            sg->c0 = chunk_tail_rows(sq);
            sg->total = sg->c0 + sq.n;
            sg->row0 = kChunkRows * it.rt;
            sg->rows_all = sq.n * g;
            sg->dual = it.weight - 1;
            sg->whole = whole && next == j1;
            // (a whole item's pieces meet in the second result, which only the block's last item leaves to the merge)
            sg->part = it.x0 <= begin && !whole ? 0 : 1;
            sg->behind = behind;
            announce();
            behind = 1;
            j = next;
          }
          if (j < j1 || it.x0 + (long long)it.weight * it.kt >= end) break;
          chunk_next(a, lv.Hkv, g, it);
        }
        if (sg != nullptr || n == 0) {
          sg = place();
          if (sg != nullptr) {
            sg->stream = -1;
            announce();
          }
        }
      }
    } else if (warp == kIssueWarp + 2) {
      // ---------------------------------------------------------------- requests into L2
      // The producers load one tile ahead, which is less than a round trip to memory: what they will load goes to L2 kAhead tiles before.  Lanes 0 .. 3
      // the units of a tile, lanes 4 .. 7 their blocks' promoted channels.
      const int step_blocks = 4 / lv.U, step_units = 4 - step_blocks * lv.U;
      int kc = 0;
      for (int n = 0; segment_there(n); ++n) {
        const Segment& sg = segments[n & 1];
        const int stream = sg.stream, j0 = sg.j0, j1 = min(sg.j1, sg.packed_tiles), nt = sg.j1 - j0, units = sg.units;
        segment_taken(n);
        if (stream < 0) break;
        Cursor at(lv, stream, 4 * j0 + (lane & 3));
        const char* extras = lv.extras + (size_t)stream * lv.extras_stride;
        for (int j = j0; j < j1; ++j) {
          // (a bounded wait, and nothing depends on it)
          for (int i = 0; i < 100 && *progress + kAhead < kc + j - j0; ++i) __nanosleep(200);
          if (lane < 8 && at.unit < units) {
            if (lane < 4) {
              prefetch_bulk(at.codes(lv) - 512, lv.unit_bytes + 512);
            } else {
              const uint2 e = *at.entry;
              const int n16 = e.y & 0xFF, n4 = (e.y >> 8) & 0xFF;
              const uint32_t bytes = extras_unit_bytes(n16, n4, kU4 == 2);               // (a multiple of 16)
              if (n16 + n4 > 0) prefetch_bulk(extras + (size_t)e.x * 16 + extras_header_bytes(n16, n4) + (uint32_t)at.u * bytes, bytes);
            }
          }
          at.next(lv, 4, step_blocks, step_units);
        }
        kc += nt;
      }
    }
  } else if (warp >= 16) {
    set_registers<false, kRegs.values>();
    // ------------------------------------------------------------------ value tiles
    const int w = (warp >> 1) & 3, half = warp & 1;
    const uint32_t scratch = sbase + kScratchOff + (warp - 8) * 640;
    const int step_blocks = 4 / lv.U, step_units = 4 - step_blocks * lv.U;
    const uint32_t meta0 = 2048 + 4 * (lane * lv.VG + (lv.VG == 4 ? 2 * half : lv.VG == 2 ? half : 0)), meta1 = meta0 + (lv.VG == 4 ? 4 : 0);
    const Magic magic;
    uint32_t st = 0, had[2] = {0, 0};                    // the tile's stage (a segment starts in stage 0); tiles that each stage has had
    bool ok = true;
    auto stage = [&]() { return vs + st * kTileBytes; };
    auto free_stage = [&]() {
      const uint32_t h = st ? had[1] : had[0];
      return group_wait(6, 256, warp == 16, h == 0 ? -1 : (int)(kVEmpty + st), (h - 1) & 1u);
    };
    auto made = [&]() {
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(kVFull + st));
      if (st) ++had[1]; else ++had[0];
      st ^= 1;
    };
    for (int n = 0; group_wait(6, 256, warp == 16, kSegFull + (n & 1), (uint32_t)(n >> 1) & 1u); ++n) {
      const Segment& sg = segments[n & 1];
      const int stream = sg.stream, j1 = sg.j1, packed_tiles = sg.packed_tiles, units = sg.units, r = sg.r, c0 = sg.c0, total = sg.total;
      int j = sg.j0;
      segment_taken(n);
      if (stream < 0) break;
      st = 0;
      const int end = min(j1, packed_tiles);
      if (j < end) {
        Cursor at(lv, stream, 4 * j + w);
        Packed p{};
        if (at.unit < units) p = request_values<kV4>(lv, at, half, lane, meta0, meta1);
        for (; j < end; ++j) {
          if (!(ok = free_stage())) break;
          if (at.unit < units) {
            make_values<kV4>(p, stage(), scratch, w, half, lane, magic);
          } else {
            // past the last block: the probabilities are zeros, and so must the values be (a NaN from earlier contents would survive the product)
            for (int i = lane; i < 8 * 32; i += 32)
              sts128(stage() + (8 * half + (i >> 5)) * 2048 + (4 * w) * 128 + (i & 31) * 16, make_uint4(0u, 0u, 0u, 0u));
          }
          at.next(lv, 4, step_blocks, step_units);
          if (at.unit < units) p = request_values<kV4>(lv, at, half, lane, meta0, meta1);
          made();
        }
      }
      for (; j < j1 && ok; ++j) {
        const Rows x{reinterpret_cast<const uint16_t*>(lv.resv + (size_t)stream * lv.resv_stride),
                     reinterpret_cast<const uint16_t*>(lv.sink + (size_t)stream * lv.sink_stride) + (size_t)lv.sink_len * kD,
                     a.v + (size_t)stream * a.stride * kD, r, c0, total};
        if (!(ok = free_stage())) break;
        copy_value_rows(x, j - packed_tiles, stage(), w, half, lane, poison + (n & 1));
        made();
      }
      if (!ok) break;
    }
  } else if (warp >= 8) {
    set_registers<(kRegs.keys > kLaunchRegs), kRegs.keys>();
    // ------------------------------------------------------------------ key tiles
    // (the group's tiles are the even or the odd ones of every segment: it has one stage to itself)
    const int w = warp & 3, group = (warp >> 2) & 1, first_warp = 8 + 4 * group;
    const uint32_t scratch = sbase + kScratchOff + (warp - 8) * 640, stage = ks + group * kTileBytes;
    const int step_blocks = 8 / lv.U, step_units = 8 - step_blocks * lv.U;
    const Magic magic;
    int kc = 0, made_tiles = 0;                          // tiles of the thread block before the segment; tiles that this group has made
    bool ok = true;
    auto free_stage = [&]() { return group_wait(2 + group, 128, warp == first_warp, made_tiles == 0 ? -1 : kKEmpty + group, (uint32_t)(made_tiles - 1) & 1u); };
    auto made = [&]() {
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0 && !(a.test_silent && group == 0 && made_tiles == 0)) mbar_arrive(bar(kKFull + group));
      ++made_tiles;
    };
    for (int n = 0; group_wait(2 + group, 128, warp == first_warp, kSegFull + (n & 1), (uint32_t)(n >> 1) & 1u); ++n) {
      const Segment& sg = segments[n & 1];
      const int stream = sg.stream, j1 = sg.j1, packed_tiles = sg.packed_tiles, units = sg.units, r = sg.r, c0 = sg.c0, total = sg.total;
      const int j0 = sg.j0;
      segment_taken(n);
      if (stream < 0) break;
      int j = j0 + group;
      const int end = min(j1, packed_tiles);
      if (j < end) {
        // the unit that is worked on, its promoted channels and codes; the next one's block's table entry
        const char* extras = lv.extras + (size_t)stream * lv.extras_stride;
        Cursor at(lv, stream, 4 * j + w);
        Promoted more{};
        PackedKeys p{};
        if (at.unit < units) {
          more = request_promoted<kU4>(extras, *at.entry, at.u, lane);
          p = request_keys<kU4>(lv, at, more, lane);
        }
        for (; j < end; j += 2) {
          Cursor next = at;
          next.next(lv, 8, step_blocks, step_units);
          uint2 entry = make_uint2(0u, 0u);
          if (next.unit < units) entry = *next.entry;
          if (!(ok = free_stage())) break;
          if (w == 0 && lane == 0) *progress = kc + j - j0;
          // (past the last block the logits are masked, whatever the keys are)
          if (at.unit < units) {
            make_keys<kU4>(p, stage, scratch, w, lane, magic);
            put_promoted<kU4>(more, stage, scratch, w, lane);
          }
          at = next;
          if (at.unit < units) {
            more = request_promoted<kU4>(extras, entry, at.u, lane);
            p = request_keys<kU4>(lv, at, more, lane);
          }
          made();
        }
      }
      for (; j < j1 && ok; j += 2) {
        const Rows x{reinterpret_cast<const uint16_t*>(lv.resk + (size_t)stream * lv.resk_stride),
                     reinterpret_cast<const uint16_t*>(lv.sink + (size_t)stream * lv.sink_stride), a.k + (size_t)stream * a.stride * kD, r, c0, total};
        if (!(ok = free_stage())) break;
        if (w == 0 && lane == 0) *progress = kc + j - j0;
        copy_key_rows(x, j - packed_tiles, stage, w, lane);
        made();
      }
      if (!ok) break;
      kc += j1 - j0;
    }
  } else {
    set_registers<true, kRegs.softmax>();
    // ------------------------------------------------------------------ softmax and output rows
    const int slot = warp >> 2, row_in = tid & 127, g = lv.g;
    const uint32_t lane_base = tbase + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t s_addr = lane_base + 128 * slot, o_addr = lane_base + 256 + 128 * slot;
    int cnt = 0, ended[2] = {0, 0};                      // steps of this slot, segments in which a slot had steps
    // (what follows a wait is the whole warp's: tensor-memory loads and stores)
    auto all_wait = [&](int i, uint32_t parity) { return __all_sync(0xffffffffu, wait(i, parity)) != 0; };
    for (int n = 0;; ++n) {
      // (both slots are behind the segment before: the queries may go, and what slot 1 left there for slot 0)
      if (!group_wait(1, kSoftmaxThreads, warp == 0, kSegFull + (n & 1), (uint32_t)(n >> 1) & 1u)) break;
      // (read again where it is needed: the tiles' loop has no registers to keep it in)
      const volatile Segment& sg = segments[n & 1];
      if (sg.stream < 0) break;
      // Rows of a tile: with more than 128 rows slot 0 has the first 128 of them and slot 1 the others.  Otherwise both have the same ones, and with at most
      // 64 every row twice, 64 lanes apart, each copy for half of the tile's keys: a warp's softmax is that much shorter, and the copies' results
      // meet at the end like the slots'.  (The logarithm of the copies.  One copy / two, us: 120000 tokens, 8b shape, 4, 32 and 64 rows 99.8 / 93.9, 118.7 /
      // 107.2, 135.5 / 125.1; 8 x 32768, 7b shape, 7, 35 and 63 rows 106.2 / 102.6, 114.3 / 105.4, 116.5 / 107.0; 1024 tokens, 4 rows 18.1 / 18.5.)
      auto copies_of = [&]() { return sg.rows_all - sg.row0 > 64 ? 0 : 1; };
      {
        const int row0 = sg.row0, rows_all = sg.rows_all, dual = sg.dual, per = kTile >> copies_of();
        // 16-byte piece p of the image: lane 8 (p / 128) + p % 8, channels 8 (p / 8 % 16) ..  A thread's pieces are 16 lanes apart; eight of them are
        // under way at once, and their rows divided by the heads by one multiplication (one after the other, each behind a division, they took 18 thousand
        // cycles of a 256-row item).
        const uint16_t* qb = a.q + (size_t)sg.stream * g * a.stride * kD + 8 * ((tid >> 3) & 15);
        const uint32_t inv_g = g == 1 ? 0u : 0xFFFFFFFFu / (uint32_t)g + 1u;         // exact for rows below 2^29
#pragma unroll 1
        for (int i0 = 0; i0 < 8 << dual; i0 += 8) {
          uint4 y[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int at = 16 * (i0 + i) + 8 * (tid >> 7) + (tid & 7), row = row0 + (dual ? at : at & (per - 1));
            y[i] = make_uint4(0u, 0u, 0u, 0u);
            if (row < rows_all) {
              const int tok = inv_g == 0u ? row : (int)__umulhi((uint32_t)row, inv_g);
              y[i] = *reinterpret_cast<const uint4*>(qb + ((size_t)(row - tok * g) * a.stride + tok) * kD);
            }
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) sts128(qs + 16 * (tid + 256 * (i0 + i)), rows_to_half(y[i]));
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(kQFull));
      RowState state{-INFINITY, 0.f, 0.f};
      bool ok = true;
      {
        const int dual = sg.dual, lg_copies = copies_of(), step = 2 - dual, j1 = sg.j1, packed_tiles = sg.packed_tiles, units = sg.units;
        const int row = sg.row0 + (dual ? slot * kTile + row_in : row_in & ((kTile >> lg_copies) - 1));
        const bool idle = (row & ~31) >= sg.rows_all;    // no row of the warp exists
        const int sees = sg.c0 + min(row, sg.rows_all - 1) / g + kTile * packed_tiles;          // the last unquantized row that the row sees
        const int h0 = (row_in >> (7 - lg_copies)) << (2 - lg_copies), h1 = h0 + (4 >> lg_copies);
        bool first = true;
        for (int j = sg.j0 + (dual ? 0 : slot); j < j1; j += step, ++cnt) {
          ok = there(kSFull + slot, (uint32_t)cnt & 1u);
          if (!ok) break;
          tc_fence_after();
          if (!idle) {
            const int last = (j < packed_tiles ? 32 * units - 1 : sees) - kTile * j;
            if (__all_sync(0xffffffffu, last >= kTile - 1))
              softmax_tile<false>(s_addr, o_addr, h0, h1, 0, first, a.scale_log2e, state);
            else
              softmax_tile<true>(s_addr, o_addr, h0, h1, last, first, a.scale_log2e, state);
            first = false;
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(kPReady + slot));
        }
      }
      // ---- the segment's result
      const int stream = sg.stream, dual = sg.dual, row0 = sg.row0, rows_all = sg.rows_all, behind = sg.behind, whole = sg.whole && !behind;
      const int rows = min(rows_all - row0, kChunkRows), lg_copies = copies_of(), per = kTile >> lg_copies;
      const int row = row0 + (dual ? slot * kTile + row_in : row_in & (per - 1));
      const bool idle = (row & ~31) >= rows_all;
      const bool both = dual || sg.j1 - sg.j0 > 1;       // slot 1 had steps (slot 0 has in every segment)
      bool mine = ok && (slot == 0 || both) && all_wait(kODone + slot, (uint32_t)ended[slot] & 1u);
      if (!dual && both) mine = all_wait(kODone + 1 - slot, (uint32_t)ended[1 - slot] & 1u) && mine;      // (the sums go where the queries were)
      tc_fence_after();
      ended[0] += 1;
      ended[1] += both;
      const size_t part_floats = (size_t)a.rows_cap * (kD + 2);
      float* part = a.parts + ((size_t)blockIdx.x * kChunkParts + (behind ? kChunkParts - 1 : sg.part)) * part_floats;
      const float l_run = mine ? state.sum() : 0.f, m_run = mine ? state.m : -INFINITY;
      if (dual) {
        if (!idle) {
          const bool exists = row < rows_all;
          // (every row sees a key: a sum of 0 means that all its logits are -inf, and gives NaN)
          const float inv = whole ? 1.f / l_run : l_run == 0.f ? 0.f : 1.f;
          const int tok = min(row, rows_all - 1) / g;
          const size_t orow = ((size_t)stream * g + (row - tok * g)) * a.stride + tok;
#pragma unroll 1
          for (int d = 0; d < kD; d += 32) {
            uint32_t u[32];
            float y[32];
            tmem_ld32(o_addr + d, u);
            if (!exists) continue;
#pragma unroll
            for (int i = 0; i < 32; ++i) y[i] = inv == 0.f ? 0.f : __uint_as_float(u[i]) * inv;
            if (whole) {
              store_row(a, orow, d, y);
            } else {
              float4* dst = reinterpret_cast<float4*>(part + (size_t)(row - row0) * kD + d);
#pragma unroll
              for (int i = 0; i < 32; i += 4) dst[i / 4] = make_float4(y[i], y[i + 1], y[i + 2], y[i + 3]);
            }
          }
          if (!whole && exists) reinterpret_cast<float2*>(part + (size_t)a.rows_cap * kD)[row - row0] = make_float2(m_run, l_run);
        }
      } else {
        // Both slots' and all copies' results of a row: slot 1 leaves its lanes' sums in shared memory (16-byte piece c of lane r at piece
        // c ^ (r % 32)), slot 0 adds its own, then all 256 threads finish rows, 2 << lg_copies threads each.
        float2* ml = reinterpret_cast<float2*>(smem + kMlOff);
        const uint32_t at = qs + row_in * 512;
        auto piece_at = [&](int c) { return at + ((c ^ (row_in & 31)) << 4); };
        if (slot == 1) {
          ml[row_in] = make_float2(m_run, l_run);
          if (!idle && both) {
#pragma unroll 1
            for (int d = 0; d < kD; d += 32) {
              uint32_t u[32];
              tmem_ld32(o_addr + d, u);
#pragma unroll
              for (int i = 0; i < 32; i += 4) sts128(piece_at((d + i) / 4), make_uint4(u[i], u[i + 1], u[i + 2], u[i + 3]));
            }
          }
        }
        softmax_sync();
        if (slot == 0 && !idle) {
          const float2 other = ml[row_in];
          const float top = fmaxf(m_run, other.x), f0 = l_run == 0.f ? 0.f : weight_of(m_run, l_run, top), f1 = weight_of(other.x, other.y, top);
          ml[row_in] = make_float2(top, l_run * f0 + other.y * f1);
#pragma unroll 1
          for (int d = 0; d < kD; d += 32) {
            uint32_t u[32];
            tmem_ld32(o_addr + d, u);
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
              float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
              if (f0 != 0.f)
                y = make_float4(__uint_as_float(u[i]) * f0, __uint_as_float(u[i + 1]) * f0, __uint_as_float(u[i + 2]) * f0, __uint_as_float(u[i + 3]) * f0);
              const uint32_t p = piece_at((d + i) / 4);
              if (f1 != 0.f) {
                const uint4 o = lds128(p);
                y.x = fmaf(__uint_as_float(o.x), f1, y.x);
                y.y = fmaf(__uint_as_float(o.y), f1, y.y);
                y.z = fmaf(__uint_as_float(o.z), f1, y.z);
                y.w = fmaf(__uint_as_float(o.w), f1, y.w);
              }
              sts128(p, make_uint4(__float_as_uint(y.x), __float_as_uint(y.y), __float_as_uint(y.z), __float_as_uint(y.w)));
            }
          }
        }
        softmax_sync();
        const int lg_threads = 1 + lg_copies, r = tid >> lg_threads;             // row r of the item, pieces of 4 channels from c on
        if (r < rows) {
          const float2 x0 = ml[r], x1 = lg_copies ? ml[r + per] : make_float2(-INFINITY, 0.f);
          const float top = fmaxf(x0.x, x1.x), f0 = weight_of(x0.x, x0.y, top), f1 = weight_of(x1.x, x1.y, top), l = x0.y * f0 + x1.y * f1;
          const float inv = whole ? 1.f / l : 1.f;
          const int t = (row0 + r) / g;
          const size_t orow = ((size_t)stream * g + (row0 + r - t * g)) * a.stride + t;
#pragma unroll 1
          for (int c = tid & ((1 << lg_threads) - 1); c < 32; c += 1 << lg_threads) {
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
            auto add = [&](int v, float f) {             // lane v's sums
              if (f == 0.f) return;
              const uint4 o = lds128(qs + v * 512 + ((c ^ (v & 31)) << 4));
              y.x = fmaf(__uint_as_float(o.x), f, y.x);
              y.y = fmaf(__uint_as_float(o.y), f, y.y);
              y.z = fmaf(__uint_as_float(o.z), f, y.z);
              y.w = fmaf(__uint_as_float(o.w), f, y.w);
            };
            add(r, f0);
            if (lg_copies) add(r + per, f1);
            y.x *= inv; y.y *= inv; y.z *= inv; y.w *= inv;
            if (whole)
              store4(a, orow * kD + 4 * c, y);
            else
              reinterpret_cast<float4*>(part + (size_t)r * kD)[c] = y;
          }
          if (!whole && (tid & ((1 << lg_threads) - 1)) == 0) reinterpret_cast<float2*>(part + (size_t)a.rows_cap * kD)[r] = make_float2(top, l);
        }
      }
      if (behind) {
        // a later piece of the block's part of the item: its result joins that of the pieces before it (the same threads left both)
        const int lg_threads = dual ? 0 : 1 + lg_copies, r = tid >> lg_threads, t = (row0 + r) / g;
        const size_t orow = ((size_t)stream * g + (row0 + r - t * g)) * a.stride + t;
        float* before = a.parts + ((size_t)blockIdx.x * kChunkParts + sg.part) * part_floats;
        float2* before_ml = reinterpret_cast<float2*>(before + (size_t)a.rows_cap * kD) + r;
        softmax_sync();
        float2 x = make_float2(-INFINITY, 0.f), y = x;
        if (r < rows) {
          x = *before_ml;
          y = reinterpret_cast<const float2*>(part + (size_t)a.rows_cap * kD)[r];
        }
        const float top = fmaxf(x.x, y.x), fx = weight_of(x.x, x.y, top), fy = weight_of(y.x, y.y, top), l = x.y * fx + y.y * fy, inv = sg.whole ? 1.f / l : 1.f;
        softmax_sync();
#pragma unroll 1
        for (int c = tid & ((1 << lg_threads) - 1); c < 32 && r < rows; c += 1 << lg_threads) {
          float4* dst = reinterpret_cast<float4*>(before + (size_t)r * kD) + c;
          float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
          const float4 fresh = reinterpret_cast<const float4*>(part + (size_t)r * kD)[c];
          if (fx != 0.f) add_scaled(fx, *dst, sum);
          else add_not_finite(*dst, sum);
          if (fy != 0.f) add_scaled(fy, fresh, sum);
          else add_not_finite(fresh, sum);
          if (sg.whole)
            store4(a, orow * kD + 4 * c, make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv));
          else
            *dst = sum;
        }
        if (!sg.whole && r < rows && (tid & ((1 << lg_threads) - 1)) == 0) *before_ml = make_float2(top, l);
        part = before;
      }
      if (*reinterpret_cast<volatile int*>(&poison[n & 1].any) != 0) {     // (the segment's products are over, and the thread's own outputs stored)
        const int lg_threads = dual ? 0 : 1 + lg_copies, r = tid >> lg_threads, t = (row0 + r) / g;
        const size_t orow = ((size_t)stream * g + (row0 + r - t * g)) * a.stride + t;
#pragma unroll 1
        for (int d = 0; d < kD && r < rows; ++d) {
          const float x = poison_of(poison[n & 1], d, t);
          if (x == 0.f || (((d >> 2) ^ tid) & ((1 << lg_threads) - 1)) != 0) continue;
          if (!sg.whole)
            part[(size_t)r * kD + d] += x;
          else if (a.out_bf16)
            static_cast<__nv_bfloat16*>(a.out)[orow * kD + d] += __float2bfloat16_rn(x);
          else
            static_cast<float*>(a.out)[orow * kD + d] += x;
        }
      }
      segment_taken(n);
      tc_fence_before();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kIssueWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tbase), "r"(512) : "memory");
}

// The items that several thread blocks share: block x has the one around the boundary x + 1, if no earlier boundary lies inside it.  kRows rows at a time of
// 8 / kRows warps each; a warp takes every (8 / kRows)-th result of its row, kFlight of them in flight.
template <int kRows>
__global__ void __launch_bounds__(256, 3) chunk_merge_kernel(const __grid_constant__ LayerView lv, const __grid_constant__ ChunkArgs a, int rows_per_block) {
  constexpr int kWarps = 8 / kRows, kFlight = 8;
  __shared__ float2 mlS[8];
  __shared__ __align__(16) float oS[8][kD];
  __shared__ int partS[kChunkMaxCtas];                     // the results that there are, by thread block: which of its two, or -1
  __shared__ int wholeS;
  const int g = lv.g, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c1 = blockIdx.x + 1;
  const long long x = chunk_begin(a.total, a.ctas, c1), x_before = chunk_begin(a.total, a.ctas, c1 - 1);
  if (threadIdx.x == 0) wholeS = 0;
  dependency_wait();
  const ChunkItem it = a.at[c1];
  const int row_first = blockIdx.y * rows_per_block, row_end = min(it.rows, row_first + rows_per_block);
  if (it.x0 == x || (c1 > 1 && x_before > it.x0) || row_first >= row_end) return;
  const long long x1 = it.x0 + (long long)it.weight * it.kt;
  const int c0 = c1 - 1, count = (int)((x1 * a.ctas + a.total - 1) / a.total) - c0;
  __syncthreads();
  if ((int)threadIdx.x < count) {
    const long long begin = chunk_begin(a.total, a.ctas, c0 + threadIdx.x), end = chunk_begin(a.total, a.ctas, c0 + threadIdx.x + 1);
    int j0, j1;
    chunk_tiles(it, begin, end, j0, j1);
    partS[threadIdx.x] = j0 < j1 ? (it.x0 <= begin ? 0 : 1) : -1;
    // (positions come two to a tile: an item across a boundary may still be one block's, which then wrote the output)
    if (j0 == 0 && j1 == it.kt) wholeS = 1;
  }
  __syncthreads();
  if (wholeS) return;
  const size_t part_floats = (size_t)a.rows_cap * (kD + 2);
  const int sub = warp % kWarps;
  for (int row0 = row_first; row0 < row_end; row0 += kRows) {
    const int prow = row0 + warp / kWarps;
    const bool exists = prow < row_end;
    float M = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    bool lost = false;                                     // a result's weight has rounded to zero
    auto part_of = [&](int i) { return a.parts + ((size_t)(c0 + i) * kChunkParts + partS[i]) * part_floats; };
    for (int i0 = sub; exists && i0 < count; i0 += kWarps * kFlight) {
      float2 ml[kFlight];
      float4 y[kFlight];
#pragma unroll
      for (int k = 0; k < kFlight; ++k) {
        const int i = i0 + k * kWarps;
        ml[k] = make_float2(-INFINITY, 0.f);
        y[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i < count && partS[i] >= 0) {
          const float* part = part_of(i);
          ml[k] = reinterpret_cast<const float2*>(part + (size_t)a.rows_cap * kD)[prow];
          y[k] = reinterpret_cast<const float4*>(part + (size_t)prow * kD)[lane];
        }
      }
      float top = M;
#pragma unroll
      for (int k = 0; k < kFlight; ++k) top = fmaxf(top, ml[k].x);
      const float f = weight_of(M, l, top);
      lost = lost || (f == 0.f && l != 0.f);
      l *= f;
      o = f == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(o.x * f, o.y * f, o.z * f, o.w * f);
#pragma unroll
      for (int k = 0; k < kFlight; ++k) {
        const float w = weight_of(ml[k].x, ml[k].y, top);
        if (w != 0.f) {
          l = fmaf(w, ml[k].y, l);
          add_scaled(w, y[k], o);
        }
        lost = lost || (w == 0.f && ml[k].y != 0.f);
      }
      M = top;
    }
    if (lost)
#pragma unroll 1
      for (int i = sub; i < count; i += kWarps)
        if (partS[i] >= 0) add_not_finite(reinterpret_cast<const float4*>(part_of(i) + (size_t)prow * kD)[lane], o);
    if constexpr (kWarps > 1) {
      if (lane == 0) mlS[warp] = make_float2(M, l);
      reinterpret_cast<float4*>(oS[warp])[lane] = o;
      __syncthreads();
      if (sub == 0) {
        // lane w: the weight of warp w's result
        const float2 ml = lane < kWarps ? mlS[warp + lane] : make_float2(-INFINITY, 0.f);
        float top = ml.x;
#pragma unroll
        for (int d = 1; d < kWarps; d *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        const float w = weight_of(ml.x, ml.y, top);
        float sum = w * ml.y;
#pragma unroll
        for (int d = 1; d < kWarps; d *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        l = __shfl_sync(0xffffffffu, sum, 0);
        o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int i = 0; i < kWarps; ++i) {
          const float wi = __shfl_sync(0xffffffffu, w, i);
          if (wi != 0.f) add_scaled(wi, reinterpret_cast<const float4*>(oS[warp + i])[lane], o);
        }
        if (__any_sync(0xffffffffu, w == 0.f && ml.y != 0.f))
#pragma unroll 1
          for (int i = 0; i < kWarps; ++i) add_not_finite(reinterpret_cast<const float4*>(oS[warp + i])[lane], o);
      }
    }
    if (exists && sub == 0) {
      const float inv = 1.f / l;
      const int row = kChunkRows * it.rt + prow, tok = row / g;
      const size_t at = ((((size_t)it.b * lv.Hq + it.hk * g + (row - tok * g)) * a.stride + tok) * kD) + 4 * lane;
      store4(a, at, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
    }
    if constexpr (kWarps > 1) __syncthreads();
  }
}

template <int kU4, bool kV4>
cudaError_t launch_one(const LayerView& lv, const ChunkArgs& a, cudaStream_t stream) {
  return launch_dependent(chunk_attention_kernel<kU4, kV4>, dim3((unsigned)a.ctas), kThreads, kSmem, stream, lv, a);
}

}  // namespace

cudaError_t chunk_attention_setup() {
  for (auto kernel : {chunk_attention_kernel<0, false>, chunk_attention_kernel<0, true>, chunk_attention_kernel<1, false>, chunk_attention_kernel<1, true>,
                      chunk_attention_kernel<2, false>, chunk_attention_kernel<2, true>}) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

// Rows that a thread block's result can have: an item's, and an even number, so that every result starts on 16 bytes.
static int rows_cap(int g, int n_tokens) { return (int)std::min<long long>(kChunkRows, ((long long)n_tokens * g + 1) & ~1ll); }

static size_t parts_bytes(int g, int n_tokens) { return (size_t)kChunkMaxCtas * kChunkParts * rows_cap(g, n_tokens) * (kD + 2) * sizeof(float); }

size_t chunk_scratch_bytes(int g, int n_tokens) { return parts_bytes(g, n_tokens) + kChunkMaxCtas * sizeof(ChunkItem); }

cudaError_t launch_chunk_attention(const LayerView& lv, ChunkArgs& a, int n_sms, cudaStream_t stream, int* launches) {
  *launches = 0;
  a.prefix[0] = 0;
  long long items = 0;
  for (int b = 0; b < lv.B; ++b) {
    long long per = 0;
    ChunkItem it{};
    if (a.seq[b].n > 0) {
      do {
        chunk_item_of(a.seq[b], lv.g, it);
        per += (long long)it.weight * it.kt;
        items += lv.Hkv;
      } while (++it.rt < it.n_rt);
    }
    a.prefix[b + 1] = a.prefix[b] + per * lv.Hkv;
  }
  a.total = a.prefix[lv.B];
  if (a.total == 0) return cudaSuccess;
  a.rows_cap = rows_cap(lv.g, a.stride);
  a.ctas = (int)std::min<long long>(std::min(n_sms, kChunkMaxCtas), (a.total + 1) / 2);
  a.at = reinterpret_cast<ChunkItem*>(reinterpret_cast<char*>(a.parts) + parts_bytes(lv.g, a.stride));
  a.max_polls = a.max_polls ? a.max_polls : kPolls;
  const bool some = lv.budget_bf16 + lv.budget_u4 > 0 ? lv.budget_u4 > 0 : lv.tau_u4 < lv.tau_bf16;
  cudaError_t e = lv.dense_hi ? (lv.v_bits == 4 ? launch_one<2, true>(lv, a, stream) : launch_one<2, false>(lv, a, stream))
                  : some      ? (lv.v_bits == 4 ? launch_one<1, true>(lv, a, stream) : launch_one<1, false>(lv, a, stream))
                              : (lv.v_bits == 4 ? launch_one<0, true>(lv, a, stream) : launch_one<0, false>(lv, a, stream));
  if (e != cudaSuccess) return e;
  *launches = 1;
  if (a.ctas == 1) return cudaSuccess;
  // A warp per row, 16 rows per block; or, for items of more results than a warp has in flight, the eight warps of a block share a row's results, a row per
  // block: where the rows are no more than the results, or the blocks no more than run at a time.  The whole call, us, a warp / a block per row, results an
  // item x rows: 148 x 1 46.4 / 27.3, 74 x 5 36.0 / 26.9, 37 x 7 55.5 / 51.7, 18 x 4 95.7 / 92.6, 37 x 35 64.8 / 60.7, 12 x 16 (one item) 19.1 / 15.6;
  // 12 x 7 (eight items) 17.6 / 18.0, 18 x 35 63.2 / 65.4, 9 x 35 63.1 / 69.7, 18 x 256 95.7 / 143.6.
  const bool few_rows = a.rows_cap * items <= a.ctas || (a.ctas - 1) * a.rows_cap <= 3 * n_sms;
  if (a.ctas > 8 * items && few_rows)
    e = launch_dependent(chunk_merge_kernel<1>, dim3((unsigned)(a.ctas - 1), (unsigned)a.rows_cap), 256, 0, stream, lv, a, 1);
  else
    e = launch_dependent(chunk_merge_kernel<8>, dim3((unsigned)(a.ctas - 1), (unsigned)((a.rows_cap + 15) / 16)), 256, 0, stream, lv, a, 16);
  if (e != cudaSuccess) return e;
  *launches = 2;
  return cudaSuccess;
}

}  // namespace mixkvq
