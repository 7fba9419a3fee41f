// Tokens into the pages of the 4-bit cache, and the values that they hold back out of them.
//
// append_kernel: new tokens' keys and queries turn by their positions (rotary positions of part of the head, either pairing), keys and values are quantized
// (Eq. 2 with 16 levels, a group of G channels of one token) and go to the page and slot of the token.  Memory-bound by its bytes, by instruction issue in its first form
// (16384 prompt tokens of 8 KV heads and 32 query heads, 356 MB: 176 us; now 74, 0.74 of the rate of a copy: half of the issue slots and half of the DRAM throughput, as the warps wait for their rows first).  Thread blocks for keys and values: sixteen lanes have a row, a lane 8 channels, so that a lane's eight
// codes are one word and the extrema of a group two to four exchanges; thread blocks for queries: eight lanes have a row (turn_pair).  A thread has one token and goes
// through a range of heads.
#include <algorithm>
#include <type_traits>

#include "paged.cuh"

namespace mixkvq {

namespace {

constexpr int kTokens = 16;                // of a thread block for keys and values, twice as many of one for queries
constexpr int kBatch = 4;                  // rows in flight per thread

// What a lane of sixteen turns its 8 channels by.
struct ChunkLane {
  Angles x;                                // sines negative where the channels are the first of their pairs
  int other;                               // the lane of the row with the other channels
  int mode;                                // 0: left as they are, 1: halves, 2: neighbours
};
__device__ __forceinline__ ChunkLane chunk_lane(const RopeTurn& t, int pos, int c, bool turns) {
  ChunkLane l;
  const int half = t.rotary >> 4;
  l.mode = !turns || c >= 2 * half ? 0 : t.interleaved ? 2 : 1;
  l.other = l.mode != 1 ? c : c < half ? c + half : c - half;
#pragma unroll
  for (int i = 0; i < 4; ++i) l.x.c[i] = l.x.s[i] = f2(0.f, 0.f);
  if (l.mode == 0) return l;
  const size_t row = (size_t)pos * (t.rotary >> 1);
  if (l.mode == 2) {
    load_angles(t.cos_t, t.sin_t, row + 4 * c, 4, l.x);
  } else {
    load_angles(t.cos_t, t.sin_t, row + 8 * (c < half ? c : c - half), 8, l.x);
    if (c < half) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float lo, hi;
        f2_get(l.x.s[i], lo, hi);
        l.x.s[i] = f2(-lo, -hi);           // x c - y s is x c + y (-s), the product rounds alike
      }
    }
  }
  return l;
}
// Every lane of the warp calls this.
__device__ __forceinline__ uint4 turn_chunk(uint4 own, const ChunkLane& l, F2 mz) {
  const uint32_t a[4] = {own.x, own.y, own.z, own.w};
  uint32_t y[4] = {own.x, own.y, own.z, own.w}, b[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) b[j] = __shfl_sync(0xffffffffu, a[j], l.other, 16);
  if (l.mode == 1) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float lo, hi;
      f2_get(f2_add(f2_mul(f2(bf16_half(a[j], 0), bf16_half(a[j], 1)), l.x.c[j], mz), f2_mul(f2(bf16_half(b[j], 0), bf16_half(b[j], 1)), l.x.s[j], mz)), lo, hi);
      y[j] = bf16_pair(lo, hi);
    }
  } else if (l.mode == 2) {
    turn_neighbours(y[0], y[1], l.x.c[0], l.x.s[0], mz);
    turn_neighbours(y[2], y[3], l.x.c[1], l.x.s[1], mz);
  }
  return make_uint4(y[0], y[1], y[2], y[3]);
}

// Scale, zero-point and codes of a row's groups.  Every lane of the warp calls this; kLanes = G / 8 neighbouring lanes share a group.
//
// The code of an element is the rounded single-precision quotient (x - z) / s.  With r = 1 / s within 2^-23 of itself (the approximation's bound), (x - z) r is off that
// quotient's exact value by 2^-23 + 2^-24 of itself at most and the quotient by 2^-24: 3.6e-6 together, as no quotient is above 15.  So unless the product lies within 5e-6 of a
// half-integer both round to the same whole number; the few that do (exact ties of bf16 numbers among them) are divided, and so is what has no product: NaN, infinities,
// groups without a scale.  The product and its rounding may be contracted: that moves the result by less than the rest of the margin.
// The scale likewise: range times 1 / 15 is within two units of the last place of the quotient, whose low 16 bits are then rounded up; where they are that near to nothing the
// range is divided.
struct Quantized {
  uint32_t codes;                          // channel i at bits 4 i
  uint32_t meta;                           // z | s << 16, bf16 bits
};
__device__ __forceinline__ uint32_t bf16_min2(uint32_t a, uint32_t b) {      // (passes over NaNs)
  uint32_t y;
  asm("min.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
  return y;
}
__device__ __forceinline__ float scale_of(float hi, float lo) {
  const float range = __fsub_rn(hi, lo), near = __fmul_rn(range, 0.06666667f);
  const uint32_t u = __float_as_uint(near);
  // (u + 2) mod 2^16 below 5: the quotient may be a bf16 number, or the product on the other side of one; tiny and infinite ranges have no such product
  if (((u + 2u) & 0xFFFFu) < 5u || !(near > 1e-37f && near < 3e38f)) return stored_scale(hi, lo, 15.f);
  return __uint_as_float((u + 0x10000u) & 0xFFFF0000u);
}
template <int kLanes>
__device__ __forceinline__ Quantized quantize_chunk(uint4 w) {
  // the least of the values and of their negatives, two at a time
  uint32_t lo2 = bf16_min2(bf16_min2(w.x, w.y), bf16_min2(w.z, w.w));
  uint32_t hi2 = bf16_min2(bf16_min2(w.x ^ 0x80008000u, w.y ^ 0x80008000u), bf16_min2(w.z ^ 0x80008000u, w.w ^ 0x80008000u));
  uint32_t both = bf16_min2(__byte_perm(lo2, hi2, 0x5410), __byte_perm(lo2, hi2, 0x7632));      // least value | least negative << 16
#pragma unroll
  for (int d = 1; d < kLanes; d <<= 1) both = bf16_min2(both, __shfl_xor_sync(0xffffffffu, both, d));
  const float lo = bf16_half(both, 0), s = scale_of(-bf16_half(both, 1), lo);
  float inv;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
  constexpr float kMagic = 12582912.f, kMargin = 0.5f - 5e-6f;      // 1.5 2^23: adding it rounds to a whole number, the low bits of the sum
  const F2 lo_2 = f2(lo, lo), inv_2 = f2(inv, inv), magic_2 = f2(kMagic, kMagic), zero_2 = f2(0.f, 0.f);
  const uint32_t a[4] = {w.x, w.y, w.z, w.w};
  uint32_t codes = 0;
  bool near = false;
#pragma unroll
  for (int i = 3; i >= 0; --i) {
    const F2 y = f2_mul(f2_sub(f2(bf16_half(a[i], 0), bf16_half(a[i], 1)), lo_2), inv_2, zero_2), f = f2_add(y, magic_2), d = f2_sub(y, f2_sub(f, magic_2));
    float f0, f1, d0, d1;
    f2_get(f, f0, f1);
    f2_get(d, d0, d1);
    near = near || !(fabsf(d0) <= kMargin) || !(fabsf(d1) <= kMargin);
    codes = codes * 256u + (__float_as_uint(f1) * 16u + __float_as_uint(f0));      // (what is above the codes is taken off at the end)
  }
  codes -= (uint32_t)(0x4B400000ull * 0x11111111ull);
  if (near) {                              // some element (one as a rule) is divided
    uint32_t which = 0;
    codes = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float y = __fmul_rn(__fsub_rn(bf16_half(a[i >> 1], i & 1), lo), inv), f = __fadd_rn(y, kMagic);
      which |= fabsf(__fsub_rn(y, __fsub_rn(f, kMagic))) <= kMargin ? 0u : 1u << i;
      codes |= (__float_as_uint(f) & 15u) << (4 * i);
    }
#pragma unroll 1
    for (; which != 0; which &= which - 1) {
      const int i = __ffs(which) - 1;
      const uint32_t w2 = i < 4 ? (i < 2 ? w.x : w.y) : (i < 6 ? w.z : w.w);
      codes = (codes & ~(15u << (4 * i))) | (uint32_t)quant_code(__uint_as_float(i & 1 ? w2 & 0xFFFF0000u : w2 << 16), lo, s, 15) << (4 * i);
    }
  }
  Quantized y;
  y.codes = codes;
  y.meta = (both & 0xFFFFu) | (__float_as_uint(s) & 0xFFFF0000u);
  return y;
}

// Token i of sequence b of an append: where it goes and what it turns by; false: nowhere.
__device__ __forceinline__ bool token_place(const PagedAppend& a, int tok, int& b, int& i, int& place, int& pos) {
  const PagedView& v = a.view;
  b = i = place = pos = 0;
  if (tok >= v.B * v.n) return false;      // (the host takes no call of 2^27 tokens or more)
  b = tok / v.n;
  i = tok - b * v.n;
  if (i >= v.count(b)) return false;
  place = v.place(b, i);
  if (place < 0) return false;
  if (a.turn.cos_t != nullptr) {
    pos = a.turn.positions != nullptr ? a.turn.positions[tok] : place;
    if (pos >= a.turn.n_positions) atomicOr(v.status, (uint32_t)MIXKVQ_DEV_BAD_POSITION);
    if (pos < 0 || pos >= a.turn.n_positions) return false;
  }
  return true;
}

template <int kLanes>
__global__ void __launch_bounds__(256, 3)
append_kernel(const __grid_constant__ PagedAppend a, int kv_blocks, int kv_each, int kv_splits, int q_each, int q_splits) {
  dependency_wait();
  const PagedView& v = a.view;
  int b, i, place, pos;
  if ((int)blockIdx.x >= kv_blocks) {
    // ---- queries
    const int block = blockIdx.x - kv_blocks, tokens = block / q_splits, split = block - tokens * q_splits;
    const int tok = tokens * (2 * kTokens) + (threadIdx.x >> 3);
    // (a token on a page that is none is not stored, and its queries are left alone like its keys)
    if (!token_place(a, tok, b, i, place, pos) || v.piece(b, 0, place) == nullptr) return;
    const PairLane p = pair_lane(a.turn, pos, threadIdx.x & 7, a.turn.cos_t != nullptr);
    const int h0 = split * q_each, h1 = min(h0 + q_each, v.Hq);
    const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(a.q) + b * a.tq.batch + h0 * a.tq.head + i * a.tq.token;
    __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(a.q_out) + (((size_t)b * v.Hq + h0) * v.n + i) * kD;
    const size_t out_head = (size_t)v.n * kD;
    for (int h = h0; h < h1; h += kBatch) {
      uint4 w[kBatch][2];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const uint4* from = reinterpret_cast<const uint4*>(src);
        w[k][0] = from[p.first];
        w[k][1] = from[p.second];
        if (h + k + 1 < h1) src += a.tq.head;    // (the last row again beyond it)
      }
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        if (h + k >= h1) break;
        turn_pair(w[k][0], w[k][1], p, F2{a.turn.minus_zero});
        uint4* to = reinterpret_cast<uint4*>(dst);
        to[p.first] = w[k][0];
        to[p.second] = w[k][1];
        dst += out_head;
      }
    }
    return;
  }
  // ---- keys, then values
  const int tokens = blockIdx.x / kv_splits, split = blockIdx.x - tokens * kv_splits, c = threadIdx.x & 15;
  const bool found = token_place(a, tokens * kTokens + (threadIdx.x >> 4), b, i, place, pos);
  char* piece = found ? v.piece(b, 0, place) : nullptr;
  const bool live = piece != nullptr;
  if (live) piece += v.tile_of(place);
  const ChunkLane lane = chunk_lane(a.turn, pos, c, live && a.turn.cos_t != nullptr);
  constexpr int G = 8 * kLanes;
  const int row = place & 15;
  const int v_at = (16 * (c & 3) + 2 * (c >> 2)) ^ ((row & 4) << 3);
  const bool first = c % kLanes == 0;
  const int h0 = split * kv_each, h1 = min(h0 + kv_each, 2 * v.Hkv);
  // heads h0 .. h1 - 1 of keys, then values
  auto rows = [&](auto keys_, const void* in, const RopeTensor& t, int from, int to) {
    constexpr bool keys = decltype(keys_)::value;
    const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(in) + b * t.batch + from * t.head + i * t.token + 8 * c;
    char* at = piece + (uint64_t)from * v.piece_bytes;
    char* codes_to = at + (keys ? row * 64 + 16 * (c & 3) + 4 * (c >> 2) : 1024 + row * 64 + v_at);
    char* meta_to = at + (keys ? paged_k_meta(row, G) : paged_v_meta(row, G)) + 4 * (c / kLanes);
    for (int h = from; h < to; h += kBatch) {
      uint4 w[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        w[k] = make_uint4(0u, 0u, 0u, 0u);
        if (live) w[k] = *reinterpret_cast<const uint4*>(src);
        if (h + k + 1 < to) src += t.head;       // (the last row again beyond it)
      }
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        if (h + k >= to) break;
        const Quantized z = quantize_chunk<kLanes>(keys ? turn_chunk(w[k], lane, F2{a.turn.minus_zero}) : w[k]);
        if (live) {
          if (keys) {
            *reinterpret_cast<uint32_t*>(codes_to) = z.codes;
          } else {
            *reinterpret_cast<uint16_t*>(codes_to) = (uint16_t)z.codes;
            *reinterpret_cast<uint16_t*>(codes_to + 8) = (uint16_t)(z.codes >> 16);
          }
          if (first) *reinterpret_cast<uint32_t*>(meta_to) = z.meta;
        }
        codes_to += v.piece_bytes;
        meta_to += v.piece_bytes;
      }
    }
  };
  if (h0 < v.Hkv) rows(std::true_type{}, a.k, a.tk, h0, min(h1, v.Hkv));
  if (h1 > v.Hkv) rows(std::false_type{}, a.v, a.tv, max(h0, v.Hkv) - v.Hkv, h1 - v.Hkv);
}

// A thread has 8 channels of one token and goes through the heads, some rows' loads under way together.  Memory-bound: the 16384 tokens back take 20 us for 88 MB, most of them written.
__global__ void __launch_bounds__(256)
read_kernel(const __grid_constant__ PagedRead a, int heads_per_block) {
  dependency_wait();
  const PagedView& v = a.view;
  const int c = threadIdx.x & 15, tok = blockIdx.x * kTokens + (threadIdx.x >> 4);
  if (tok >= v.B * v.n) return;
  const int b = tok / v.n, i = tok - b * v.n;
  if (i >= v.count(b)) return;
  const int place = v.place(b, i);
  if (place < 0) return;
  const char* piece = v.piece(b, 0, place);
  if (piece == nullptr) return;
  piece += v.tile_of(place);
  const int row = place & 15, G = v.G, grp = c / (G / 8);
  const int v_at = (16 * (c & 3) + 2 * (c >> 2)) ^ ((row & 4) << 3);
  const int h0 = blockIdx.y * heads_per_block, h1 = min(h0 + heads_per_block, 2 * v.Hkv);
  // heads h0 .. h1 - 1 of keys, then values
  auto rows = [&](auto keys_, void* out, int from, int to) {
    constexpr bool keys = decltype(keys_)::value;
    const char* at = piece + (uint64_t)from * v.piece_bytes;
    const char* codes_at = at + (keys ? row * 64 + 16 * (c & 3) + 4 * (c >> 2) : 1024 + row * 64 + v_at);
    const char* meta_at = at + (keys ? paged_k_meta(row, G) : paged_v_meta(row, G)) + 4 * grp;
    __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(out) + (((size_t)b * v.Hkv + from) * v.n + i) * kD + 8 * c;
    const size_t out_head = (size_t)v.n * kD;
    for (int h = from; h < to; h += kBatch) {
      uint32_t codes[kBatch], meta[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        if (keys)
          codes[k] = *reinterpret_cast<const uint32_t*>(codes_at);
        else
          codes[k] = *reinterpret_cast<const uint16_t*>(codes_at) | (uint32_t)*reinterpret_cast<const uint16_t*>(codes_at + 8) << 16;
        meta[k] = *reinterpret_cast<const uint32_t*>(meta_at);
        if (h + k + 1 < to) {                    // (the last row again beyond it)
          codes_at += v.piece_bytes;
          meta_at += v.piece_bytes;
        }
      }
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        if (h + k >= to) break;
        const float s = bf16_half(meta[k], 1), z = bf16_half(meta[k], 0);
        uint32_t y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)         // (code times scale is exact: 4 bits by 8)
          y[j] = bf16_pair(fmaf((float)(codes[k] >> (8 * j) & 15u), s, z), fmaf((float)(codes[k] >> (8 * j + 4) & 15u), s, z));
        *reinterpret_cast<uint4*>(dst) = make_uint4(y[0], y[1], y[2], y[3]);
        dst += out_head;
      }
    }
  };
  if (h0 < v.Hkv) rows(std::true_type{}, a.k, h0, min(h1, v.Hkv));
  if (h1 > v.Hkv) rows(std::false_type{}, a.v, max(h0, v.Hkv) - v.Hkv, h1 - v.Hkv);
}

// Heads per thread block: all of a token's, halved until there are four thread blocks per SM (but what a thread has in flight).  Append and read of 16384 tokens, and of 1246 tokens:
// 93.7 and 18.8 us; until there is one per SM 95 and 21; until there are eight 99 and 18.8, as the tables and the token's place are read once for each range.
int split_heads(long long blocks, int heads, int n_sms) {
  int each = heads;
  while (each > kBatch && blocks * ((heads + each - 1) / each) < 4 * n_sms) each = (each + 1) / 2;
  return each;
}

}  // namespace

cudaError_t launch_paged_append(const PagedAppend& a, int n_sms, cudaStream_t stream) {
  const long long tokens = (long long)a.view.B * a.view.n, kv = (tokens + kTokens - 1) / kTokens, q = a.q != nullptr ? (tokens + 2 * kTokens - 1) / (2 * kTokens) : 0;
  const int kv_each = split_heads(kv, 2 * a.view.Hkv, n_sms), q_each = split_heads(std::max(q, 1ll), a.view.Hq, n_sms);
  const int kv_splits = (2 * a.view.Hkv + kv_each - 1) / kv_each, q_splits = (a.view.Hq + q_each - 1) / q_each;
  const auto kernel = a.view.G == 32 ? append_kernel<4> : a.view.G == 64 ? append_kernel<8> : append_kernel<16>;
  return launch_dependent(kernel, dim3((unsigned)(kv * kv_splits + q * q_splits)), 256, 0, stream, a, (int)(kv * kv_splits), kv_each, kv_splits, q_each, q_splits);
}

cudaError_t launch_paged_read(const PagedRead& a, int n_sms, cudaStream_t stream) {
  const long long blocks = ((long long)a.view.B * a.view.n + kTokens - 1) / kTokens;
  const int heads = 2 * a.view.Hkv, each = split_heads(blocks, heads, n_sms);
  return launch_dependent(read_kernel, dim3((unsigned)blocks, (unsigned)((heads + each - 1) / each)), 256, 0, stream, a, each);
}

}  // namespace mixkvq
