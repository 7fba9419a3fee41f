// Tokens into the pages of the 4-bit cache, and the values that they hold back out of them.
//
// append_kernel: new tokens' keys and queries turn by their positions (rotary positions of part of the head, either pairing), keys and values are quantized
// (Eq. 2 with 16 levels, a group of G channels of one token) and go to the page and slot of the token.  Memory-bound; a thread has 8 channels of one token and goes
// through a range of heads, sixteen lanes have a row: the extrema of a group are two to four exchanges between them, a lane's eight codes are one word.
#include <algorithm>

#include "paged.cuh"

namespace mixkvq {

namespace {

constexpr int kTokens = 16;
constexpr int kBatch = 4;

// Scale, zero-point and codes of a row's groups.  Every lane of the warp calls this; group_lanes = G / 8 neighbouring lanes share a group.
struct Quantized {
  uint32_t codes;                          // channel i at bits 4 i
  uint32_t meta;                           // z | s << 16, bf16 bits
};
__device__ __forceinline__ Quantized quantize_chunk(uint4 w, int group_lanes) {
  const uint32_t a[4] = {w.x, w.y, w.z, w.w};
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = bf16_half(a[i >> 1], i & 1);
  float lo = x[0], hi = x[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    lo = fminf(lo, x[i]);
    hi = fmaxf(hi, x[i]);
  }
  for (int d = 1; d < group_lanes; d <<= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, d));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, d));
  }
  const float s = stored_scale(hi, lo, 15.f);
  Quantized y;
  y.codes = 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i) y.codes |= (uint32_t)quant_code(x[i], lo, s, 15) << (4 * i);
  y.meta = (__float_as_uint(lo) >> 16) | (__float_as_uint(s) & 0xFFFF0000u);
  return y;
}

__global__ void __launch_bounds__(256)
append_kernel(const __grid_constant__ PagedAppend a, int heads_per_block) {
  dependency_wait();
  const PagedView& v = a.view;
  const int c = threadIdx.x & 15;
  const long long tok = (long long)blockIdx.x * kTokens + (threadIdx.x >> 4);
  const bool there = tok < (long long)v.B * v.n;
  const int b = there ? (int)(tok / v.n) : 0, i = there ? (int)(tok - (long long)b * v.n) : 0;
  bool live = there && i < v.count(b);
  int place = 0, pos = 0;
  if (live) {
    place = v.place(b, i);
    live = place >= 0;
  }
  if (live && a.turn.cos_t != nullptr) {
    pos = a.turn.positions != nullptr ? a.turn.positions[tok] : place;
    if (pos >= a.turn.n_positions) atomicOr(v.status, (uint32_t)MIXKVQ_DEV_BAD_POSITION);
    live = pos >= 0 && pos < a.turn.n_positions;
  }
  char* piece = live ? v.piece(b, 0, place) : nullptr;
  live = piece != nullptr;
  if (live) piece += v.tile_of(place);
  RopeTurn turn = a.turn;
  if (!live) turn.cos_t = nullptr;
  const TurnChunk x = turn_chunk_load(turn, pos, c);
  const int row = place & 15, G = v.G;
  // heads: keys, values, queries
  const int heads = 2 * v.Hkv + (a.q != nullptr ? v.Hq : 0);
  const int h0 = blockIdx.y * heads_per_block, h1 = min(h0 + heads_per_block, heads);
  for (int h = h0; h < h1; h += kBatch) {
    uint4 w[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      w[k] = make_uint4(0u, 0u, 0u, 0u);
      const int hh = h + k;
      if (hh >= h1 || !live) continue;
      const int which = hh < v.Hkv ? 1 : hh < 2 * v.Hkv ? 2 : 0, head = which == 1 ? hh : which == 2 ? hh - v.Hkv : hh - 2 * v.Hkv;
      const RopeTensor& s = which == 0 ? a.tq : which == 1 ? a.tk : a.tv;
      w[k] = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(which == 0 ? a.q : which == 1 ? a.k : a.v) + b * s.batch + head * s.head + i * s.token +
                                             8 * c);
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int hh = h + k;
      if (hh >= h1) break;
      const int which = hh < v.Hkv ? 1 : hh < 2 * v.Hkv ? 2 : 0, head = which == 1 ? hh : which == 2 ? hh - v.Hkv : hh - 2 * v.Hkv;
      const uint4 y = which == 2 ? w[k] : turn_chunk(w[k], x);
      Quantized z{0u, 0u};
      if (which != 0) z = quantize_chunk(y, G / 8);
      if (live && which == 0) {
        *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.q_out) + (((size_t)b * v.Hq + head) * v.n + i) * kD + 8 * c) = y;
      } else if (live) {
        char* tile = piece + (uint64_t)head * v.piece_bytes;
        if (which == 1) {
          *reinterpret_cast<uint32_t*>(tile + row * 64 + 16 * (c & 3) + 4 * (c >> 2)) = z.codes;
        } else {
          const int at = (16 * (c & 3) + 2 * (c >> 2)) ^ ((row & 4) << 3);
          *reinterpret_cast<uint16_t*>(tile + 1024 + row * 64 + at) = (uint16_t)z.codes;
          *reinterpret_cast<uint16_t*>(tile + 1024 + row * 64 + at + 8) = (uint16_t)(z.codes >> 16);
        }
        if (c % (G / 8) == 0)
          *reinterpret_cast<uint32_t*>(tile + (which == 1 ? paged_k_meta(row, G) : paged_v_meta(row, G)) + 4 * (c / (G / 8))) = z.meta;
      }
    }
  }
}

// A thread has 8 channels of one token and goes through the heads.
__global__ void __launch_bounds__(256)
read_kernel(const __grid_constant__ PagedRead a, int heads_per_block) {
  dependency_wait();
  const PagedView& v = a.view;
  const int c = threadIdx.x & 15;
  const long long tok = (long long)blockIdx.x * kTokens + (threadIdx.x >> 4);
  if (tok >= (long long)v.B * v.n) return;
  const int b = (int)(tok / v.n), i = (int)(tok - (long long)b * v.n);
  if (i >= v.count(b)) return;
  const int place = v.place(b, i);
  if (place < 0) return;
  const char* piece = v.piece(b, 0, place);
  if (piece == nullptr) return;
  piece += v.tile_of(place);
  const int row = place & 15, G = v.G, grp = c / (G / 8);
  const int h0 = blockIdx.y * heads_per_block, h1 = min(h0 + heads_per_block, 2 * v.Hkv);
  for (int h = h0; h < h1; ++h) {
    const bool keys = h < v.Hkv;
    const int head = keys ? h : h - v.Hkv;
    const char* tile = piece + (uint64_t)head * v.piece_bytes;
    uint32_t codes, meta;
    if (keys) {
      codes = *reinterpret_cast<const uint32_t*>(tile + row * 64 + 16 * (c & 3) + 4 * (c >> 2));
      meta = *reinterpret_cast<const uint32_t*>(tile + paged_k_meta(row, G) + 4 * grp);
    } else {
      const int at = (16 * (c & 3) + 2 * (c >> 2)) ^ ((row & 4) << 3);
      codes = *reinterpret_cast<const uint16_t*>(tile + 1024 + row * 64 + at) | (uint32_t)*reinterpret_cast<const uint16_t*>(tile + 1024 + row * 64 + at + 8) << 16;
      meta = *reinterpret_cast<const uint32_t*>(tile + paged_v_meta(row, G) + 4 * grp);
    }
    const float s = bf16_half(meta, 1), z = bf16_half(meta, 0);
    uint32_t y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)             // (code times scale is exact: 4 bits by 8)
      y[j] = bf16_pair(fmaf((float)(codes >> (8 * j) & 15u), s, z), fmaf((float)(codes >> (8 * j + 4) & 15u), s, z));
    *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(keys ? a.k : a.v) + (((size_t)b * v.Hkv + head) * v.n + i) * kD + 8 * c) = make_uint4(y[0], y[1], y[2], y[3]);
  }
}

// Heads per thread block: all of a token's, fewer as long as the SMs have room.
int split_heads(long long blocks, int heads, int n_sms) {
  int each = heads;
  while (each > 1 && blocks * ((heads + each - 1) / each) < 4 * n_sms) each = (each + 1) / 2;
  return each;
}

}  // namespace

cudaError_t launch_paged_append(const PagedAppend& a, int n_sms, cudaStream_t stream) {
  const long long blocks = ((long long)a.view.B * a.view.n + kTokens - 1) / kTokens;
  const int heads = 2 * a.view.Hkv + (a.q != nullptr ? a.view.Hq : 0), each = split_heads(blocks, heads, n_sms);
  return launch_dependent(append_kernel, dim3((unsigned)blocks, (unsigned)((heads + each - 1) / each)), 256, 0, stream, a, each);
}

cudaError_t launch_paged_read(const PagedRead& a, int n_sms, cudaStream_t stream) {
  const long long blocks = ((long long)a.view.B * a.view.n + kTokens - 1) / kTokens;
  const int heads = 2 * a.view.Hkv, each = split_heads(blocks, heads, n_sms);
  return launch_dependent(read_kernel, dim3((unsigned)blocks, (unsigned)((heads + each - 1) / each)), 256, 0, stream, a, each);
}

}  // namespace mixkvq
