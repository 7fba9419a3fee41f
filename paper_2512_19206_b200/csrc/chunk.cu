// Attention of a chunk of new tokens over the mixed-precision cache and, causally, over itself, on the tcgen05 tensor cores.
//
//   o_j = sum_t softmax_t(scale q_j . k_t) v_t,   t over the sink, the packed blocks (dequantized, Eq. 3), the residual window and the
//   new tokens up to j.
//
// One thread block of 640 threads per SM, persistent over its share of the (item, key tile) line (chunk.cuh).  Per key tile of 128 keys:
//   warps 8-11, 12-15   make the tile: four warps the keys, four the values, one 32-token unit each.  Packed codes become fp16 in registers
//                       (c s + z, one rounding) and go to shared memory in the tensor core's canonical layout; an unquantized row is copied
//                       with bf16 -> fp16.  The packed bytes are read once per 256 query rows and never written back dequantized.
//   warp 16             one thread issues every tcgen05.mma: S = Q K^T (operands in shared memory), O += P V (P in tensor memory).
//   warps 0-3, 4-7      two softmax groups ("slots"), thread = query row = lane of tensor memory.  An item of more than 128 rows has its first 128 rows
//                       in slot 0 and the others in slot 1; in a smaller one both slots have the same rows, slot 0 the even key tiles and slot 1
//                       the odd ones, and their results meet at the end: the tensor core works for one slot while the other is in its softmax.
// Codes lie in the cache as mma.sync A fragments: the lane with row r and pair t of an 8 x 8 piece holds its two neighbouring channels (keys) or
// tokens (values).  With keys and values both stored K-major in shared memory that pair is 4 bytes at 16 r + 4 t = 4 lane of a core matrix, so a
// warp's store is 128 contiguous bytes.
// The running maximum is raised (and O rescaled, in tensor memory) only when a row's logits exceed it by more than 2^8: P stays below 256, far
// inside fp16, and the rescaling is rare.  P is fp16 (11 significant bits); sums, maxima, O are fp32.
#include <algorithm>

#include "chunk.cuh"
#include "tc_ops.cuh"

namespace mixkvq {

namespace {

constexpr int kTile = kChunkTile;
constexpr int kTileBytes = kTile * kD * 2;
constexpr int kThreads = 640;                             // 96 registers a thread at launch: 61440, shared out below as 2 x 128 x 112, 2 x 128 x 112, 128 x 32
constexpr int kSoftmaxThreads = 256;
constexpr int kScratchOff = 6 * kTileBytes;               // per producer warp 1 KB: scales and zero-points as fp16 pairs
constexpr int kMlOff = kScratchOff + 8 * 1024;            // slot 1's maxima and denominators (128 x 8 bytes)
constexpr int kBarOff = kMlOff + 1024;
constexpr int kBars = 17;
constexpr int kSmem = kBarOff + 8 * kBars + 8;
enum Bar { kQFull = 0, kKFull = 1, kVFull = 3, kKEmpty = 5, kVEmpty = 7, kSFull = 9, kPReady = 11, kODone = 13, kDone = 15 };
constexpr uint32_t kPolls = 1u << 21;
constexpr float kRaise = 8.f;

__device__ __forceinline__ void sts32(uint32_t a, uint32_t x) { asm volatile("st.shared.u32 [%0], %1;" ::"r"(a), "r"(x) : "memory"); }
__device__ __forceinline__ void sts16(uint32_t a, uint32_t x) { asm volatile("st.shared.u16 [%0], %1;" ::"r"(a), "h"((uint16_t)x) : "memory"); }
__device__ __forceinline__ void sts128(uint32_t a, uint4 x) {
  asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ uint32_t hfma2_u(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
__device__ __forceinline__ uint4 rows_to_half(uint4 x) {
  return make_uint4(bf16x2_to_f16x2(x.x), bf16x2_to_f16x2(x.y), bf16x2_to_f16x2(x.z), bf16x2_to_f16x2(x.w));
}
__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// fp16 pair of 4^-f and of -1024 4^-f, f = 0 .. 4
__device__ __forceinline__ constexpr uint32_t inv_pow4(int f) { return (uint32_t)((15 - 2 * f) << 10) * 0x00010001u; }
__device__ __forceinline__ constexpr uint32_t neg_1024_pow4(int f) { return (0x8000u | (uint32_t)((25 - 2 * f) << 10)) * 0x00010001u; }

// The codes of field f (2 bits at bit 2 f of each half word) as an fp16 pair: 1024 + c 4^f is the number with the field's bits in its
// mantissa, and (1024 + c 4^f) 4^-f - 1024 4^-f is exact.  f is at most 4 after the shift (the mantissa has 10 bits).
__device__ __forceinline__ uint32_t codes2(uint32_t w, int f) {
  const int sh = f > 4 ? 10 : 0, ff = f > 4 ? f - 5 : f;
  return hfma2_u(((w >> sh) & (0x00030003u << (2 * ff))) | 0x64006400u, inv_pow4(ff), neg_1024_pow4(ff));
}
// The same for 4-bit codes whose low and high pairs of bits are in two planes: hi4 = high plane << 2.  The top field's high bits are taken after the
// shift, where hi4's lost ones are still there (`hi` itself).
__device__ __forceinline__ uint32_t codes4(uint32_t lo, uint32_t hi, int f) {
  const int sh = f > 3 ? 8 : 0, ff = f > 3 ? f - 4 : f;
  const uint32_t l = lo >> sh, h = sh ? hi >> (sh - 2) : hi << 2;
  return hfma2_u((l & (0x00030003u << (2 * ff))) | (h & (0x000C000Cu << (2 * ff))) | 0x64006400u, inv_pow4(ff), neg_1024_pow4(ff));
}

struct Stream {                          // where an item's keys and values are
  const char *base, *extras;
  const uint32_t* table;
  const uint16_t *resk, *resv, *sinkk, *sinkv, *newk, *newv;
  int units, r, c0, total;               // packed units; residual rows; residual and sink rows; all unquantized rows that the item may see
};
__device__ inline Stream stream_of(const LayerView& lv, const ChunkArgs& a, const ChunkItem& it) {
  Stream x;
  const int s = it.b * lv.Hkv + it.hk;
  const ChunkSeq sq = a.seq[it.b];
  x.base = lv.base + (size_t)s * lv.base_stride;
  x.extras = lv.extras + (size_t)s * lv.extras_stride;
  x.table = reinterpret_cast<const uint32_t*>(lv.table + (size_t)s * lv.table_stride);
  x.resk = reinterpret_cast<const uint16_t*>(lv.resk + (size_t)s * lv.resk_stride);
  x.resv = reinterpret_cast<const uint16_t*>(lv.resv + (size_t)s * lv.resv_stride);
  x.sinkk = reinterpret_cast<const uint16_t*>(lv.sink + (size_t)s * lv.sink_stride);
  x.sinkv = x.sinkk + (size_t)lv.sink_len * kD;
  x.newk = a.k + (size_t)s * a.stride * kD;
  x.newv = a.v + (size_t)s * a.stride * kD;
  x.units = sq.units;
  x.r = sq.tail & 0xFFFF;
  x.c0 = chunk_tail_rows(sq);
  x.total = x.c0 + sq.n;
  return x;
}
__device__ __forceinline__ const uint16_t* tail_row(const uint16_t* res, const uint16_t* sink, const uint16_t* fresh, const Stream& x, int i) {
  return i < x.r ? res + (size_t)i * kD : i < x.c0 ? sink + (size_t)(i - x.r) * kD : fresh + (size_t)(i - x.c0) * kD;
}

// One unit's packed keys or values on their way to shared memory: requested one tile ahead.
struct Packed {
  uint4 c0, c1, h0, h1, meta;
};

// ---- keys: warp w makes rows 32 w .. 32 w + 31 of the tile at shared address `tile`
template <bool kDense>
__device__ __forceinline__ Packed request_keys(const LayerView& lv, const Stream& x, int unit, uint2 entry, int lane) {
  Packed p;
  const int bi = unit / lv.U, u = unit - bi * lv.U;
  const char* blk = x.base + (size_t)bi * lv.base_bytes;
  const uint4* codes = reinterpret_cast<const uint4*>(blk + frag_unit_off(u, lv.G, lv.unit_bytes));
  p.c0 = codes[lane];
  p.c1 = codes[32 + lane];
  p.meta = reinterpret_cast<const uint4*>(blk + frag_meta_off((u * 32) / lv.G, lv.G, lv.unit_bytes))[lane];
  if (kDense) {
    const int n16 = entry.y & 0xFF, n4 = (entry.y >> 8) & 0xFF;
    if (n4 != 0) {
      const uint4* hi = reinterpret_cast<const uint4*>(x.extras + (size_t)entry.x * 16 + extras_header_bytes(n16, n4) +
                                                       (size_t)u * extras_unit_bytes(n16, n4, true) + 128 * ((n16 + 1) >> 1));
      p.h0 = hi[lane];
      p.h1 = hi[32 + lane];
    } else {
      p.h0 = p.h1 = make_uint4(0u, 0u, 0u, 0u);
    }
  }
  return p;
}

template <bool kDense>
__device__ __forceinline__ void make_keys(const LayerView& lv, const Stream& x, const Packed& p, int unit, uint2 entry, uint32_t tile, uint32_t scratch,
                                          int w, int lane) {
  const int bi = unit / lv.U, u = unit - bi * lv.U;
  const int n16 = entry.y & 0xFF, n4 = (entry.y >> 8) & 0xFF, n16p = (n16 + 1) >> 1;
  const char* ex = x.extras + (size_t)entry.x * 16;
  const char* exu = ex + extras_header_bytes(n16, n4) + (size_t)u * extras_unit_bytes(n16, n4, kDense);
  // the promoted channels' first four pairs and their numbers are under way while the codes are worked on
  uint4 head = make_uint4(~0u, ~0u, ~0u, ~0u);
  uint32_t raw[4] = {0u, 0u, 0u, 0u};
  if (n16 > 0) {
    head = *reinterpret_cast<const uint4*>(ex);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n16p) raw[i] = reinterpret_cast<const uint32_t*>(exu)[i * 32 + lane];
  }
  // scales and zero-points of channel pairs (16 kt + 8 ch + 2 t, + 1) as fp16 pairs: word 16 t + 8 ch + kt, zero-points 64 words on.  The lane has the
  // pairs 2 lane and 2 lane + 1: kt = lane / 4, ch = lane / 2 % 2, t = 2 (lane % 2) and the next.
  {
    const uint32_t at = scratch + 4 * (16 * 2 * (lane & 1) + 8 * ((lane >> 1) & 1) + (lane >> 2));
    sts32(at, bf16x2_to_f16x2(__byte_perm(p.meta.x, p.meta.y, 0x5410)));
    sts32(at + 256, bf16x2_to_f16x2(__byte_perm(p.meta.x, p.meta.y, 0x7632)));
    sts32(at + 64, bf16x2_to_f16x2(__byte_perm(p.meta.z, p.meta.w, 0x5410)));
    sts32(at + 64 + 256, bf16x2_to_f16x2(__byte_perm(p.meta.z, p.meta.w, 0x7632)));
  }
  __syncwarp();
  const uint32_t c[2][4] = {{p.c0.x, p.c0.y, p.c0.z, p.c0.w}, {p.c1.x, p.c1.y, p.c1.z, p.c1.w}};
  const uint32_t h[2][4] = {{p.h0.x, p.h0.y, p.h0.z, p.h0.w}, {p.h1.x, p.h1.y, p.h1.z, p.h1.w}};
  const uint32_t out = tile + 4 * w * 2048 + 4 * lane;
#pragma unroll
  for (int ch = 0; ch < 2; ++ch) {
    const uint32_t at = scratch + 4 * (16 * (lane & 3) + 8 * ch);
    const uint4 sa = lds128(at), sb = lds128(at + 16), za = lds128(at + 256), zb = lds128(at + 272);
    const uint32_t s[8] = {sa.x, sa.y, sa.z, sa.w, sb.x, sb.y, sb.z, sb.w}, z[8] = {za.x, za.y, za.z, za.w, zb.x, zb.y, zb.z, zb.w};
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int rh = 0; rh < 2; ++rh) {
        const uint32_t wd = c[mt][2 * ch + rh], hd = h[mt][2 * ch + rh];
#pragma unroll
        for (int kt = 0; kt < 8; ++kt)
          sts32(out + (2 * mt + rh) * 2048 + (2 * kt + ch) * 128, hfma2_u(kDense ? codes4(wd, hd, kt) : codes2(wd, kt), s[kt], z[kt]));
      }
  }
  if ((n16 | (kDense ? 0 : n4)) == 0) return;
  __syncwarp();                          // the base codes are stored: promoted channels replace theirs.  The lane's token: 32 w + lane
  const uint32_t row = tile + (4 * w + (lane >> 3)) * 2048 + (lane & 7) * 16;
  auto put = [&](uint32_t d, float value) { sts16(row + (d >> 3) * 128 + (d & 7) * 2, (uint32_t)__half_as_ushort(__float2half_rn(value))); };
#pragma unroll 1
  for (int i0 = 0; i0 < n16p; i0 += 4) {
    uint32_t ids[2] = {head.x, head.y};
    if (i0 > 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i0 + i < n16p) raw[i] = reinterpret_cast<const uint32_t*>(exu)[(i0 + i) * 32 + lane];
      const uint2 more = *reinterpret_cast<const uint2*>(ex + 2 * i0);
      ids[0] = more.x;
      ids[1] = more.y;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i0 + i < n16p) {
        const uint32_t id = ids[i >> 1] >> (16 * (i & 1)), d0 = id & 0xFF, d1 = (id >> 8) & 0xFF;
        if (d0 < kD) put(d0, bf_lo(raw[i]));
        if (d1 < kD) put(d1, bf_hi(raw[i]));
      }
  }
  if (!kDense && n4 > 0) {               // UINT4 channels: c = c_lo + 4 c_hi, with s and z from the block's scales
    const char* blk = x.base + (size_t)bi * lv.base_bytes;
    const uint32_t* low = reinterpret_cast<const uint32_t*>(blk + frag_unit_off(u, lv.G, lv.unit_bytes));
    const uint32_t* meta = reinterpret_cast<const uint32_t*>(blk + frag_meta_off((u * 32) / lv.G, lv.G, lv.unit_bytes));
    const uint32_t* high = reinterpret_cast<const uint32_t*>(exu + 128 * n16p);
    const int mt = lane >> 4, rh = (lane >> 3) & 1, r = lane & 7;
    const int lane_word = mt * 128 + 16 * r + rh, hi_bit = 8 * (r >> 2) + 2 * (2 * mt + rh);
#pragma unroll 2
    for (int i = 0; i < (n4 + 1) >> 1; ++i) {
      const uint32_t id = *reinterpret_cast<const uint16_t*>(ex + 2 * n16p + 2 * i), hw = high[4 * i + (r & 3)] >> hi_bit;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t d = (id >> (8 * e)) & 0xFF;
        if (d < kD) {
          const uint32_t lw = low[lane_word + 4 * ((d & 7) >> 1) + 2 * ((d >> 3) & 1)], mz = meta[d];
          const uint32_t code = ((lw >> (16 * (d & 1) + 2 * (d >> 4))) & 3u) | (((hw >> (16 * e)) & 3u) << 2);
          put(d, fmaf((float)code, bf_lo(mz), bf_hi(mz)));
        }
      }
    }
  }
}

// ---- values: warp w makes keys 32 w .. 32 w + 31 of the tile, stored channel by channel (K-major for O = P V)
template <bool kV4>
__device__ __forceinline__ Packed request_values(const LayerView& lv, const Stream& x, int unit, int lane) {
  Packed p;
  const int bi = unit / lv.U, u = unit - bi * lv.U;
  const char* at = x.base + (size_t)bi * lv.base_bytes + frag_unit_off(u, lv.G, lv.unit_bytes);
  p.c0 = reinterpret_cast<const uint4*>(at + 1024)[lane];
  p.c1 = reinterpret_cast<const uint4*>(at + 1024)[32 + lane];
  const char* meta = at + 2048 + lane * 4 * lv.VG;
  p.meta = make_uint4(0u, 0u, 0u, 0u);
  if (lv.VG == 4) {
    p.meta = *reinterpret_cast<const uint4*>(meta);
  } else if (lv.VG == 2) {
    const uint2 m = *reinterpret_cast<const uint2*>(meta);
    p.meta.x = m.x;
    p.meta.y = m.y;
  } else {
    p.meta.x = *reinterpret_cast<const uint32_t*>(meta);
  }
  if (kV4) {
    const uint4* hi = reinterpret_cast<const uint4*>(at + 2048 + 128 * lv.VG);
    p.h0 = hi[lane];
    p.h1 = hi[32 + lane];
  }
  return p;
}

template <bool kV4>
__device__ __forceinline__ void make_values(const LayerView& lv, const Packed& p, uint32_t tile, uint32_t scratch, int w, int lane) {
  // scales of tokens (8 o + 2 t, + 1) as fp16 pairs: word 16 vg + 4 t + o, zero-points 64 words on; the lane has token 8 o + 2 t + e = lane
  {
    const uint32_t m[4] = {p.meta.x, p.meta.y, p.meta.z, p.meta.w};
    const uint32_t at = scratch + 4 * (4 * ((lane >> 1) & 3) + (lane >> 3)) + 2 * (lane & 1);
#pragma unroll
    for (int vg = 0; vg < 4; ++vg)
      if (vg < lv.VG) {
        const uint32_t h = bf16x2_to_f16x2(m[vg]);
        sts16(at + 64 * vg, h & 0xFFFFu);
        sts16(at + 64 * vg + 256, h >> 16);
      }
  }
  __syncwarp();
  const uint32_t c[8] = {p.c0.x, p.c0.y, p.c0.z, p.c0.w, p.c1.x, p.c1.y, p.c1.z, p.c1.w};
  const uint32_t h[8] = {p.h0.x, p.h0.y, p.h0.z, p.h0.w, p.h1.x, p.h1.y, p.h1.z, p.h1.w};
  const uint32_t out = tile + 4 * w * 128 + 4 * lane;
  const int lg = lv.VG == 4 ? 1 : lv.VG == 2 ? 2 : 3;        // a value group has 2^lg pieces of 16 channels
  uint4 s4 = make_uint4(0u, 0u, 0u, 0u), z4 = s4;
#pragma unroll
  for (int ct = 0; ct < 8; ++ct) {
    if ((ct & ((1 << lg) - 1)) == 0) {
      const uint32_t at = scratch + 64 * (ct >> lg) + 16 * (lane & 3);
      s4 = lds128(at);
      z4 = lds128(at + 256);
    }
    const uint32_t s[4] = {s4.x, s4.y, s4.z, s4.w}, z[4] = {z4.x, z4.y, z4.z, z4.w};
#pragma unroll
    for (int rh = 0; rh < 2; ++rh)
#pragma unroll
      for (int o = 0; o < 4; ++o)
        sts32(out + (2 * ct + rh) * 2048 + o * 128, hfma2_u(kV4 ? codes4(c[ct], h[ct], 4 * rh + o) : codes2(c[ct], 4 * rh + o), s[o], z[o]));
  }
}

// Unquantized rows 128 t + 32 w .. + 31: keys K-major, values as they lie (MN-major); rows past the last are zeros.
__device__ __forceinline__ void copy_key_rows(const Stream& x, int t, uint32_t tile, int w, int lane) {
  uint4 y[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int row = kTile * t + 32 * w + 8 * (i & 3) + (lane & 7);
    y[i] = make_uint4(0u, 0u, 0u, 0u);
    if (row < x.total) y[i] = reinterpret_cast<const uint4*>(tail_row(x.resk, x.sinkk, x.newk, x, row))[4 * (i >> 2) + (lane >> 3)];
  }
#pragma unroll
  for (int i = 0; i < 16; ++i)
    sts128(tile + (4 * w + (i & 3)) * 2048 + (4 * (i >> 2) + (lane >> 3)) * 128 + (lane & 7) * 16, rows_to_half(y[i]));
}
__device__ __forceinline__ void copy_value_rows(const Stream& x, int t, uint32_t tile, int w, int lane) {
  const int row = kTile * t + 32 * w + lane;
  const uint4* src = row < x.total ? reinterpret_cast<const uint4*>(tail_row(x.resv, x.sinkv, x.newv, x, row)) : nullptr;
  uint4 y[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) y[i] = src != nullptr ? src[i] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
  for (int i = 0; i < 16; ++i) sts128(tile + i * 2048 + (4 * w + (lane >> 3)) * 128 + (lane & 7) * 16, rows_to_half(y[i]));
}

__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&u)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,"
      "%27,%28,%29,%30,%31}, [%32];"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]), "=r"(u[10]),
        "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]), "=r"(u[17]), "=r"(u[18]), "=r"(u[19]), "=r"(u[20]),
        "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]), "=r"(u[25]), "=r"(u[26]), "=r"(u[27]), "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
      : "r"(taddr)
      : "memory");
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(u[0]), "+r"(u[1]), "+r"(u[2]), "+r"(u[3]), "+r"(u[4]), "+r"(u[5]), "+r"(u[6]), "+r"(u[7]), "+r"(u[8]), "+r"(u[9]),
                 "+r"(u[10]), "+r"(u[11]), "+r"(u[12]), "+r"(u[13]), "+r"(u[14]), "+r"(u[15]), "+r"(u[16]), "+r"(u[17]), "+r"(u[18]), "+r"(u[19]),
                 "+r"(u[20]), "+r"(u[21]), "+r"(u[22]), "+r"(u[23]), "+r"(u[24]), "+r"(u[25]), "+r"(u[26]), "+r"(u[27]), "+r"(u[28]), "+r"(u[29]),
                 "+r"(u[30]), "+r"(u[31])
               :
               : "memory");
}

// One tile of one slot's softmax: the thread's row of S (128 fp32 at s_addr) becomes P (fp16 pairs over the first 64 of those columns).  kMask: the row
// sees the columns <= last only.
template <bool kMask>
__device__ __forceinline__ void softmax_tile(uint32_t s_addr, uint32_t o_addr, int last, bool first, float scale_log2e, float& m_ref, float& l_run) {
  float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
  for_pieces<true>(s_addr, 8, [&](int h, const uint32_t (&u)[16]) {
    const int lim = last - 16 * h;
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const float x0 = kMask && i > lim ? -INFINITY : __uint_as_float(u[i]);
      const float x1 = kMask && i + 1 > lim ? -INFINITY : __uint_as_float(u[i + 1]);
      mx4[(i >> 1) & 3] = fmaxf(fmaxf(mx4[(i >> 1) & 3], x0), x1);
    }
  });
  const float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * scale_log2e;
  if (first) {
    m_ref = mx;
  } else if (__any_sync(0xffffffffu, mx > m_ref + kRaise)) {
    // (the products before this tile are complete: S is behind them in the tensor core's order)
    const float m_new = fmaxf(m_ref, mx), alpha = m_new == -INFINITY ? 1.f : ex2(m_ref - m_new);
#pragma unroll
    for (int d = 0; d < kD; d += 16) {
      uint32_t u[16];
      tmem_ld16_issue(o_addr + d, u);
      tmem_wait_ld16(u);
      uint32_t a[8], b[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        a[i] = __float_as_uint(__uint_as_float(u[i]) * alpha);
        b[i] = __float_as_uint(__uint_as_float(u[8 + i]) * alpha);
      }
      tmem_st8(o_addr + d, a);
      tmem_st8(o_addr + d + 8, b);
    }
    l_run *= alpha;
    m_ref = m_new;
  }
  const float ref = m_ref == -INFINITY ? 0.f : m_ref;          // a row that has seen no key yet: all its logits are -inf, its P is 0
  const uint64_t scale2 = pack2(scale_log2e, scale_log2e), ref2 = pack2(-ref, -ref);
  uint64_t sum[2] = {0ull, 0ull};
  for_pieces<true>(s_addr, 8, [&](int h, const uint32_t (&u)[16]) {
    uint32_t wd[8];
    const int lim = last - 16 * h;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float x0, x1;
      unpack2(fma2(pack2u(u[2 * i], u[2 * i + 1]), scale2, ref2), x0, x1);
      float p0 = ex2(x0), p1 = ex2(x1);
      if constexpr (kMask) {
        p0 = 2 * i <= lim ? p0 : 0.f;
        p1 = 2 * i + 1 <= lim ? p1 : 0.f;
      }
      sum[i & 1] = add2(sum[i & 1], pack2(p0, p1));
      wd[i] = pack_half2(p0, p1);
    }
    tmem_st8(s_addr + 8 * h, wd);
  });
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
  float s0, s1;
  unpack2(add2(sum[0], sum[1]), s0, s1);
  l_run += s0 + s1;
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

template <bool kDense, bool kV4>
__global__ void __launch_bounds__(kThreads, 1) chunk_attention_kernel(const __grid_constant__ LayerView lv, const __grid_constant__ ChunkArgs a) {
  extern __shared__ __align__(128) unsigned char smem[];
  const uint32_t sbase = smem_u32(smem), qs = sbase, ks = sbase + 2 * kTileBytes, vs = sbase + 4 * kTileBytes;
  auto bar = [&](int i) { return sbase + (uint32_t)kBarOff + 8u * (uint32_t)i; };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + kBarOff + 8 * kBars);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lv.g;
  const long long begin = chunk_begin(a.total, a.ctas, blockIdx.x), end = chunk_begin(a.total, a.ctas, blockIdx.x + 1);

  if (warp == 16) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (tid == 0) {
    for (int i = 0; i < kBars; ++i)
      mbar_init(bar(i), i == kQFull ? kSoftmaxThreads : (i >= kKFull && i < kKEmpty) ? 4 : (i >= kPReady && i < kODone) ? kTile : 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tbase = *tmem_slot;
  dependency_wait();
  // tensor-memory columns: S / P of slot 0 at 0, of slot 1 at 128, O of slot 0 at 256, of slot 1 at 384
  bool dead = false;
  auto wait = [&](int i, uint32_t parity) {
    if (!dead && !mbar_wait_polls(bar(i), parity, a.max_polls)) {
      dead = true;
      atomicOr(lv.status, (uint32_t)MIXKVQ_DEV_COPY_TIMEOUT);
    }
    return !dead;
  };
  // walks the thread block's segments: f(item, first key tile, key tiles behind the last)
  auto for_segments = [&](auto f) {
    if (begin >= end) return;
    ChunkItem it = chunk_locate(a, lv.B, lv.Hkv, g, begin);
    for (;;) {
      int j0, j1;
      chunk_tiles(it, begin, end, j0, j1);
      if (j0 < j1) f(it, j0, j1);
      if (it.x0 + (long long)it.weight * it.kt >= end) break;
      chunk_next(a, lv.Hkv, g, it);
    }
  };

  if (warp >= 16) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 32;" ::: "memory");
    if (warp == 16 && lane == 0) {
      // ---------------------------------------------------------------- tensor-core issue
      const uint32_t idesc_s = make_idesc(128, 128, 0, 0), idesc_packed = make_idesc(128, 128, 0, 0), idesc_rows = make_idesc(128, 128, 0, 1);
      int tile0 = 0, seg = 0, cnt[2] = {0, 0};           // key tiles and segments before this one; steps per slot
      for_segments([&](const ChunkItem& it, int j0, int j1) {
        if (dead) return;
        const bool dual = it.weight == 2;
        const int nt = j1 - j0, steps = dual ? 2 * nt : nt;
        if (!wait(kQFull, seg & 1)) return;
        tc_fence_after();
        auto issue_s = [&](int u) {
          const int slot = u & 1, kc = tile0 + (dual ? u >> 1 : u), st = kc & 1;
          if (!wait(kKFull + st, (kc >> 1) & 1)) return false;
          tc_fence_after();
          const uint64_t qd = make_desc(qs + (dual ? slot : 0) * kTileBytes, 128, 2048), kd = make_desc(ks + st * kTileBytes, 128, 2048);
#pragma unroll
          for (int i = 0; i < 8; ++i) tc_mma_ss(tbase + 128 * slot, qd + (uint64_t)(16 * i), kd + (uint64_t)(16 * i), idesc_s, i > 0);
          tc_commit(bar(kSFull + slot));
          if (!dual || slot == 1) tc_commit(bar(kKEmpty + st));
          return true;
        };
        auto issue_o = [&](int u) {
          const int slot = u & 1, j = dual ? u >> 1 : u, kc = tile0 + j, st = kc & 1;
          if (!wait(kVFull + st, (kc >> 1) & 1) || !wait(kPReady + slot, cnt[slot] & 1)) return false;
          cnt[slot] += 1;
          tc_fence_after();
          const uint64_t vd = make_desc(vs + st * kTileBytes, 128, 2048);
          const uint32_t idesc = j0 + j < it.packed_tiles ? idesc_packed : idesc_rows, o = tbase + 256 + 128 * slot, p = tbase + 128 * slot;
#pragma unroll
          for (int i = 0; i < 8; ++i) tc_mma_ts(o, p + 8 * i, vd + (uint64_t)(16 * i), idesc, u > 1 || i > 0);
          if (!dual || slot == 1) tc_commit(bar(kVEmpty + st));
          if (u + 2 >= steps) tc_commit(bar(kODone + slot));
          return true;
        };
        bool ok = issue_s(0);
        if (ok && steps > 1) ok = issue_s(1);
        for (int u = 0; ok && u < steps; ++u) {
          ok = issue_o(u);
          if (ok && u + 2 < steps) ok = issue_s(u + 2);
        }
        tile0 += nt;
        seg += 1;
      });
      tc_commit(bar(kDone));                             // every product issued above has finished when this one fires
      dead = false;
      wait(kDone, 0);
    }
  } else if (warp >= 8) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 112;" ::: "memory");
    // ------------------------------------------------------------------ key and value tiles
    const bool keys = warp < 12;
    const int w = warp & 3;
    const uint32_t scratch = sbase + kScratchOff + (warp - 8) * 1024, tiles = keys ? ks : vs;
    const int full = keys ? kKFull : kVFull, empty = keys ? kKEmpty : kVEmpty;
    int kc = 0;
    for_segments([&](const ChunkItem& it, int j0, int j1) {
      if (dead) return;
      const Stream x = stream_of(lv, a, it);
      auto entry_of = [&](int j) {
        const int unit = 4 * j + w;
        return j < it.packed_tiles && unit < x.units ? *reinterpret_cast<const uint2*>(x.table + 2 * (unit / lv.U)) : make_uint2(0u, 0u);
      };
      auto request = [&](int j, uint2 entry) {
        const int unit = 4 * j + w;
        Packed p{};
        if (j < it.packed_tiles && unit < x.units) p = keys ? request_keys<kDense>(lv, x, unit, entry, lane) : request_values<kV4>(lv, x, unit, lane);
        return p;
      };
      uint2 entry = make_uint2(0u, 0u), entry_next = entry;
      if (keys) {
        entry = entry_of(j0);
        entry_next = j0 + 1 < j1 ? entry_of(j0 + 1) : entry;
      }
      Packed next = request(j0, entry);
      for (int j = j0; j < j1; ++j, ++kc) {
        const Packed cur = next;
        const uint2 entry_cur = entry;
        entry = entry_next;
        if (j + 1 < j1) next = request(j + 1, entry);
        if (keys && j + 2 < j1) entry_next = entry_of(j + 2);
        const int st = kc & 1;
        const uint32_t tile = tiles + st * kTileBytes;
        if (kc >= 2 && !wait(empty + st, ((kc >> 1) - 1) & 1)) return;
        if (j >= it.packed_tiles) {
          if (keys)
            copy_key_rows(x, j - it.packed_tiles, tile, w, lane);
          else
            copy_value_rows(x, j - it.packed_tiles, tile, w, lane);
        } else if (4 * j + w < x.units) {
          if (keys)
            make_keys<kDense>(lv, x, cur, 4 * j + w, entry_cur, tile, scratch, w, lane);
          else
            make_values<kV4>(lv, cur, tile, scratch, w, lane);
        } else if (!keys) {
          // past the last block: the probabilities are zeros, and so must the values be (a NaN from earlier contents would survive the product)
          for (int i = lane; i < 16 * 32; i += 32) sts128(tile + (i >> 5) * 2048 + (4 * w) * 128 + (i & 31) * 16, make_uint4(0u, 0u, 0u, 0u));
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0 && !(a.test_silent && keys && kc == 0)) mbar_arrive(bar(full + st));
      }
    });
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 112;" ::: "memory");
    // ------------------------------------------------------------------ softmax and output rows
    const int slot = warp >> 2, row_in = tid & 127;
    const uint32_t lane_base = tbase + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t s_addr = lane_base + 128 * slot, o_addr = lane_base + 256 + 128 * slot;
    int cnt = 0, ended[2] = {0, 0};                      // steps of this slot, segments in which a slot had steps
    // (what follows a wait is the whole warp's: tensor-memory loads and stores)
    auto all_wait = [&](int i, uint32_t parity) { return __all_sync(0xffffffffu, wait(i, parity)) != 0; };
    for_segments([&](const ChunkItem& it, int j0, int j1) {
      const bool dual = it.weight == 2;
      const ChunkSeq sq = a.seq[it.b];
      const int nt = j1 - j0, rows_all = sq.n * g, c0 = chunk_tail_rows(sq);
      // both slots are behind the segment before: the queries may go, and what slot 1 left there for slot 0
      asm volatile("bar.sync 1, 256;" ::: "memory");
      {
        // 16-byte piece p of the image: row 8 (p / 128) + p % 8, channels 8 (p / 8 % 16) ..
        const int pieces = dual ? 4096 : 2048;
        const uint16_t* qb = a.q + ((size_t)it.b * lv.Hq + it.hk * g) * a.stride * kD;
#pragma unroll 8
        for (int p = tid; p < pieces; p += kSoftmaxThreads) {
          const int row = kChunkRows * it.rt + 8 * (p >> 7) + (p & 7), c = (p >> 3) & 15;
          uint4 y = make_uint4(0u, 0u, 0u, 0u);
          if (row < rows_all) {
            const int tok = row / g;
            y = reinterpret_cast<const uint4*>(qb + ((size_t)(row - tok * g) * a.stride + tok) * kD)[c];
          }
          sts128(qs + 16 * p, rows_to_half(y));
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      tc_fence_before();
      mbar_arrive(bar(kQFull));
      const int row = kChunkRows * it.rt + (dual ? slot * kTile : 0) + row_in;
      const int tok = min(row, rows_all - 1) / g;
      const bool idle = (row & ~31) >= rows_all;         // no row of the warp exists
      float m_ref = -INFINITY, l_run = 0.f;
      const int stride = dual ? 1 : 2;
      bool ok = true;
      for (int j = j0 + (dual ? 0 : slot); j < j1; j += stride, ++cnt) {
        ok = all_wait(kSFull + slot, cnt & 1);
        if (!ok) break;
        tc_fence_after();
        if (!idle) {
          const int last = j < it.packed_tiles ? 32 * (sq.units - 4 * j) - 1 : c0 + tok - kTile * (j - it.packed_tiles);
          const bool first = j < j0 + stride;
          if (__all_sync(0xffffffffu, last >= kTile - 1))
            softmax_tile<false>(s_addr, o_addr, 0, first, a.scale_log2e, m_ref, l_run);
          else
            softmax_tile<true>(s_addr, o_addr, last, first, a.scale_log2e, m_ref, l_run);
        }
        tc_fence_before();
        mbar_arrive(bar(kPReady + slot));
      }
      // ---- the segment's result
      const bool had[2] = {true, dual || nt > 1};
      const bool whole = j0 == 0 && j1 == it.kt;
      auto o_ready = [&](int s) { return had[s] && all_wait(kODone + s, ended[s] & 1); };
      bool mine = o_ready(slot) && ok;
      const bool apart = dual || !had[1];                // this slot's rows are no other's
      if (!apart) {
        mine = o_ready(1 - slot) && mine;                // slot 1's sums go where the queries were: no product may still read them
        tc_fence_after();
        // slot 1's row to shared memory: 16-byte piece c of row r at piece c ^ (r % 32)
        if (slot == 1) {
          const uint32_t at = qs + row_in * 512;
#pragma unroll
          for (int d = 0; d < kD; d += 32) {
            uint32_t u[32];
            tmem_ld32(o_addr + d, u);
#pragma unroll
            for (int i = 0; i < 32; i += 4) sts128(at + (((d + i) / 4) ^ (row_in & 31)) * 16, make_uint4(u[i], u[i + 1], u[i + 2], u[i + 3]));
          }
          reinterpret_cast<float2*>(smem + kMlOff)[row_in] = make_float2(mine ? m_ref : -INFINITY, mine ? l_run : 0.f);
        }
        asm volatile("bar.sync 1, 256;" ::: "memory");
      }
      if (had[0]) ended[0] += 1;
      if (had[1]) ended[1] += 1;
      if ((dual || slot == 0) && !idle) {
        const bool exists = row < rows_all;
        tc_fence_after();
        float m = mine ? m_ref : -INFINITY, l = mine ? l_run : 0.f, f0 = 1.f, f1 = 0.f;
        if (!apart) {
          const float2 other = reinterpret_cast<const float2*>(smem + kMlOff)[row_in];
          const float top = fmaxf(m, other.x);
          f0 = m == -INFINITY ? 0.f : ex2(m - top);
          f1 = other.x == -INFINITY ? 0.f : ex2(other.x - top);
          l = l * f0 + other.y * f1;
          m = top;
        }
        if (l_run == 0.f || !mine) f0 = 0.f;
        const int first_seg = it.x0 <= begin ? 0 : 1;
        float* part = a.parts + ((size_t)blockIdx.x * 2 + first_seg) * a.rows_cap * (kD + 2);
        const int prow = (dual ? slot * kTile : 0) + row_in;
        const float inv = whole ? (l > 0.f ? 1.f / l : 0.f) : 1.f;
        const size_t orow = ((size_t)it.b * lv.Hq + it.hk * g + (row - tok * g)) * a.stride + tok;
#pragma unroll 1
        for (int d = 0; d < kD; d += 32) {
          uint32_t u[32];
          float y[32];
          tmem_ld32(o_addr + d, u);
#pragma unroll
          for (int i = 0; i < 32; ++i) y[i] = f0 == 0.f ? 0.f : __uint_as_float(u[i]) * f0;
          if (f1 != 0.f) {
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
              const uint4 o = lds128(qs + row_in * 512 + (((d + i) / 4) ^ (row_in & 31)) * 16);
              y[i] = fmaf(__uint_as_float(o.x), f1, y[i]);
              y[i + 1] = fmaf(__uint_as_float(o.y), f1, y[i + 1]);
              y[i + 2] = fmaf(__uint_as_float(o.z), f1, y[i + 2]);
              y[i + 3] = fmaf(__uint_as_float(o.w), f1, y[i + 3]);
            }
          }
          if (!exists) continue;
          if (whole) {
#pragma unroll
            for (int i = 0; i < 32; ++i) y[i] *= inv;
            store_row(a, orow, d, y);
          } else {
            float4* dst = reinterpret_cast<float4*>(part + (size_t)prow * kD + d);
#pragma unroll
            for (int i = 0; i < 32; i += 4) dst[i / 4] = make_float4(y[i], y[i + 1], y[i + 2], y[i + 3]);
          }
        }
        if (!whole && exists) reinterpret_cast<float2*>(part + (size_t)a.rows_cap * kD)[prow] = make_float2(m, l);
      }
      tc_fence_before();
    });
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 16) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tbase), "r"(512) : "memory");
}

// The items that several thread blocks share: block x has the one around the boundary x + 1, if no earlier boundary lies inside it.  kRows rows of
// 8 / kRows warps each; a warp takes every (8 / kRows)-th result, kFlight of them in flight.
template <int kRows>
__global__ void __launch_bounds__(256) chunk_merge_kernel(const __grid_constant__ LayerView lv, const __grid_constant__ ChunkArgs a) {
  constexpr int kWarps = 8 / kRows, kFlight = 8;
  __shared__ float2 mlS[8];
  __shared__ __align__(16) float oS[8][kD];
  const int g = lv.g, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c1 = blockIdx.x + 1;
  const long long x = chunk_begin(a.total, a.ctas, c1);
  const ChunkItem it = chunk_locate(a, lv.B, lv.Hkv, g, x);
  dependency_wait();
  const int prow = blockIdx.y * kRows + warp / kWarps, sub = warp % kWarps;
  if (it.x0 == x || (c1 > 1 && chunk_begin(a.total, a.ctas, c1 - 1) > it.x0) || (int)blockIdx.y * kRows >= it.rows) return;
  const long long x1 = it.x0 + (long long)it.weight * it.kt;
  const int c0 = c1 - 1, count = (int)((x1 * a.ctas + a.total - 1) / a.total) - c0;
  auto share = [&](int i, int& j0, int& j1) {
    chunk_tiles(it, chunk_begin(a.total, a.ctas, c0 + i), chunk_begin(a.total, a.ctas, c0 + i + 1), j0, j1);
  };
  // (positions come two to a tile: an item across a boundary may still be one block's, which then wrote the output)
  for (int i = 0; i < min(count, 2); ++i) {
    int j0, j1;
    share(i, j0, j1);
    if (j0 == 0 && j1 == it.kt) return;
  }
  const bool exists = prow < it.rows;
  const size_t part_floats = (size_t)a.rows_cap * (kD + 2);
  float M = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i0 = sub; exists && i0 < count; i0 += kWarps * kFlight) {
    float2 ml[kFlight];
    float4 y[kFlight];
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {
      const int i = i0 + k * kWarps;
      ml[k] = make_float2(-INFINITY, 0.f);
      y[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (i < count) {
        int j0, j1;
        share(i, j0, j1);
        if (j0 < j1) {
          const float* part = a.parts + ((size_t)(c0 + i) * 2 + (it.x0 <= chunk_begin(a.total, a.ctas, c0 + i) ? 0 : 1)) * part_floats;
          ml[k] = reinterpret_cast<const float2*>(part + (size_t)a.rows_cap * kD)[prow];
          y[k] = reinterpret_cast<const float4*>(part + (size_t)prow * kD)[lane];
        }
      }
    }
    float top = M;
#pragma unroll
    for (int k = 0; k < kFlight; ++k) top = fmaxf(top, ml[k].x);
    const float f = M == -INFINITY ? 0.f : exp2f(M - top);
    l *= f;
    o.x *= f; o.y *= f; o.z *= f; o.w *= f;
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {
      // (NaN sums of a row whose logits hold a NaN: their maximum may be -inf, and they count all the same)
      const float w = ml[k].x == -INFINITY ? (ml[k].y == 0.f ? 0.f : 1.f) : exp2f(ml[k].x - top);
      if (w != 0.f) {
        l = fmaf(w, ml[k].y, l);
        o.x = fmaf(w, y[k].x, o.x); o.y = fmaf(w, y[k].y, o.y); o.z = fmaf(w, y[k].z, o.z); o.w = fmaf(w, y[k].w, o.w);
      }
    }
    M = top;
  }
  if constexpr (kWarps > 1) {
    if (lane == 0) mlS[warp] = make_float2(M, l);
    reinterpret_cast<float4*>(oS[warp])[lane] = o;
    __syncthreads();
    if (sub != 0) return;
    float top = M;
    for (int w = 1; w < kWarps; ++w) top = fmaxf(top, mlS[warp + w].x);
    const float f = M == -INFINITY ? (l == 0.f ? 0.f : 1.f) : exp2f(M - top);
    l *= f;
    o.x *= f; o.y *= f; o.z *= f; o.w *= f;
    for (int w = 1; w < kWarps; ++w) {
      const float2 ml = mlS[warp + w];
      const float fw = ml.x == -INFINITY ? (ml.y == 0.f ? 0.f : 1.f) : exp2f(ml.x - top);
      if (fw != 0.f) {
        const float4 y = reinterpret_cast<const float4*>(oS[warp + w])[lane];
        l = fmaf(fw, ml.y, l);
        o.x = fmaf(fw, y.x, o.x); o.y = fmaf(fw, y.y, o.y); o.z = fmaf(fw, y.z, o.z); o.w = fmaf(fw, y.w, o.w);
      }
    }
  }
  if (!exists) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int row = kChunkRows * it.rt + prow, tok = row / g;
  const size_t at = ((((size_t)it.b * lv.Hq + it.hk * g + (row - tok * g)) * a.stride + tok) * kD) + 4 * lane;
  o.x *= inv; o.y *= inv; o.z *= inv; o.w *= inv;
  if (a.out_bf16) {
    const __nv_bfloat162 p0 = __floats2bfloat162_rn(o.x, o.y), p1 = __floats2bfloat162_rn(o.z, o.w);
    *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + at) =
        make_uint2(*reinterpret_cast<const uint32_t*>(&p0), *reinterpret_cast<const uint32_t*>(&p1));
  } else {
    *reinterpret_cast<float4*>(static_cast<float*>(a.out) + at) = o;
  }
}

template <bool kDense, bool kV4>
cudaError_t launch_one(const LayerView& lv, const ChunkArgs& a, cudaStream_t stream) {
  return launch_dependent(chunk_attention_kernel<kDense, kV4>, dim3((unsigned)a.ctas), kThreads, kSmem, stream, lv, a);
}

}  // namespace

cudaError_t chunk_attention_setup() {
  for (auto kernel : {chunk_attention_kernel<false, false>, chunk_attention_kernel<false, true>, chunk_attention_kernel<true, false>,
                      chunk_attention_kernel<true, true>}) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

// Rows that a thread block's result can have: an item's, and an even number, so that every result starts on 16 bytes.
static int rows_cap(int g, int n_tokens) { return (int)std::min<long long>(kChunkRows, ((long long)n_tokens * g + 1) & ~1ll); }

size_t chunk_scratch_bytes(int g, int n_tokens) { return (size_t)kChunkMaxCtas * 2 * rows_cap(g, n_tokens) * (kD + 2) * sizeof(float); }

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
  a.max_polls = a.max_polls ? a.max_polls : kPolls;
  cudaError_t e = lv.dense_hi ? (lv.v_bits == 4 ? launch_one<true, true>(lv, a, stream) : launch_one<true, false>(lv, a, stream))
                              : (lv.v_bits == 4 ? launch_one<false, true>(lv, a, stream) : launch_one<false, false>(lv, a, stream));
  if (e != cudaSuccess) return e;
  *launches = 1;
  if (a.ctas == 1) return cudaSuccess;
  if (a.ctas > 8 * items)
    e = launch_dependent(chunk_merge_kernel<1>, dim3((unsigned)(a.ctas - 1), (unsigned)a.rows_cap), 256, 0, stream, lv, a);
  else
    e = launch_dependent(chunk_merge_kernel<8>, dim3((unsigned)(a.ctas - 1), (unsigned)((a.rows_cap + 7) / 8)), 256, 0, stream, lv, a);
  if (e != cudaSuccess) return e;
  *launches = 2;
  return cudaSuccess;
}

}  // namespace mixkvq
