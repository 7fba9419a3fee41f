// Attention of many query rows over the pages of the 4-bit cache, on the tcgen05 tensor cores.
//
// The codes of a token are used by thousands of query rows, so they are unpacked once: unpack_kernel writes tiles of 128 tokens of a KV head as fp16 images in the tensor
// core's shared-memory layout, so that a tile arrives as one 32 KB bulk copy.  c s + z is rounded to fp16 once (2^-11 of itself); every tile is scaled by a power of two of
// its own to a largest element of 2^14 to 2^15, and every query row likewise, so that operands of any magnitude stay inside fp16's range (a value tile's power is 2^96 at most: values
// below 2^-110 lose bits).  The scales of a key tile and a query row go into the factor of the logits, that of a value tile into the sum of the products.
//
// attend_kernel: one thread block per SM of 384 threads:
//   warps 0-3, 4-7   two softmax groups of 128 query rows (thread = row = lane of tensor memory); a row is head x % g of token x / g;
//   warp 8           one thread issues every tcgen05.mma;
//   warp 9           one thread issues the bulk copies of the key and value tiles into two-stage rings.
// Per key tile and group: S = Q K^T; the thread takes its row of S into registers, writes its row of P = 2^(S - reference + 4) as fp16 over S; O += P V in tensor memory.
// A reference is raised, and the row of O rescaled, only when a logit comes 2^8 above it, so that almost no tile touches O outside the tensor core.  The scale of a value tile goes into
// the exponents of P as its ratio to the scale that O has.  The tensor core truncates its sums, about 3.5e-7 of O per tile
// in one direction: after 512 tiles O is added to a sum in memory and begins again.
//
// Split: a row tile of 256 rows of a KV head is an item with as many positions as its last row sees key tiles; all items' positions in one line are cut evenly over the
// thread blocks, on the device.  A thread block that has a part of an item leaves sums, which join_kernel puts together.
//
// What bounds it: a group's chain of product, softmax, product and the hand-overs between them, about 4000 cycles for a key tile of both groups whose products take 2048 of the tensor core.
// 2048 tokens over 32768 more, 7b shape (9.9e11 operations): 1055 us, 940 TFLOP/s, with the images and the join; tensor pipe 46 %, exponentials 46 % of their unit, 1000 W when calls
// follow each other.  The exponentials are not it: with half of them left out the kernel takes as long.  Measured against it: sums of every tile added up in registers, which left
// none for the row of S (read twice), 1078; weights from the reference before the tile 1242; steps of 64 keys with two S under way 1267.
#include <algorithm>

#include "paged.cuh"
#include "tc_ops.cuh"

namespace mixkvq {

namespace {

constexpr int kTile = 128;                       // tokens of a tile, query rows of a group
constexpr int kTileBytes = kTile * kD * 2;
constexpr int kRows = 2 * kTile;                 // of an item
constexpr int kThreads = 384;
constexpr int kPartFloats = kD + 4;              // sums of a row: o[128], reference, denominator, lost channels, (pad)
constexpr int kAhead = 2;                        // positions that the beginning of an item counts as
constexpr uint32_t kPolls = 1u << 19;            // (a poll that finds nothing returns after about 4 us)
constexpr size_t kImageBytes = (size_t)512 << 20;      // of images at a time: sequences (or heads) beyond are a pass of their own
constexpr int kShift = 4;                        // the weight of a logit equal to the reference is 2^kShift
constexpr float kRise = 8.f;                     // a logit this much above the reference raises it: weights are 2^12 at most
constexpr int kSlack = 3;                        // powers of two that a value tile's scale may be above that of O: 2^15 at most
constexpr int kFlush = 512;                      // tiles summed up in tensor memory
constexpr float kLeast = 0x1p-120f;              // the factor of the logits is no less: sums of products are below 2^38, so smaller ones give the same weights, and -infinity stays what it is
constexpr int kDown = 30;                        // and sums of values 2^-kDown as large: they keep off fp32's end

struct __align__(16) TileHead {
  float k_scale, v_scale;                        // what the images' elements are to be multiplied with (values: times 2^-kDown)
  uint32_t flags;                                // bits 0 .. 7: which 16 tokens are there, bit 8: some element is not finite
  uint32_t pad;
  uint8_t lost[kTile];                           // per token: bits 0 .. 3: quarters of the value that are not finite, bit 4: the key is not
};
struct __align__(16) Broken {                    // an item that begins in a thread block's range and ends in another's
  int b, h, r, last;                             // last: the thread block that has its end; 0 or less: none
};

struct ChunkPlan {
  unsigned char *k_images, *v_images;            // [streams][max_tiles][32 KB]
  TileHead* heads;                               // [streams][max_tiles]
  float* parts;                                  // [2 * thread blocks][256][kPartFloats]
  Broken* broken;                                // [thread blocks]
  int b0, nb, h0, nh;                            // sequences and KV heads of this pass
  int max_tiles;
};

__device__ __forceinline__ float pow2i(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }
__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t u = __float_as_uint(x) & 0x7FFFFFFFu;
  return u < 0x7F800000u ? u : 0u;
}
// e of the 2^e that brings a largest magnitude (its bits) to 2^14 .. 2^15
__device__ __forceinline__ int scale_exponent(uint32_t bits) { return min(max(14 + 127 - (int)(bits >> 23), -113), 126); }

// ---------------------------------------------------------------------------------------------------------------- unpacking
// A thread block per (tile, KV head, sequence); a thread has half of a token's channels, quarters 2 half and 2 half + 1.
__global__ void __launch_bounds__(256)
unpack_kernel(const __grid_constant__ PagedAttention a, const __grid_constant__ ChunkPlan plan) {
  dependency_wait();
  const PagedView& v = a.view;
  const int tile = blockIdx.x, h = plan.h0 + blockIdx.y, b = plan.b0 + blockIdx.z, tid = threadIdx.x, G = v.G;
  const int count = v.count(b), len = v.length(b, v.add_counts ? count : 0);
  if (count == 0 || (tile > 0 && tile * kTile >= len)) return;
  const size_t at = (size_t)(blockIdx.z * plan.nh + blockIdx.y) * plan.max_tiles + tile;
  const int row = tid >> 1, half = tid & 1, tok = tile * kTile + row, r = tok & 15, groups = kD / G, meta = 4 * groups;
  const char* from = tok < len ? v.piece(b, h, tok) : nullptr;
  if (from != nullptr) from += v.tile_of(tok);
  uint2 kw[4];                                   // words 2 half, 2 half + 1 of the four 16-byte pieces
  uint32_t vw[8], km[2], vm[2], lost = 0, mk = 0, mv = 0;
  if (from != nullptr) {
#pragma unroll
    for (int t = 0; t < 4; ++t) kw[t] = *reinterpret_cast<const uint2*>(from + r * 64 + 16 * t + 8 * half);
#pragma unroll
    for (int t = 0; t < 8; ++t) vw[t] = *reinterpret_cast<const uint32_t*>(from + 1024 + r * 64 + ((8 * t) ^ ((r & 4) << 3)) + 4 * half);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int g = (2 * half + q) * groups / 4;
      km[q] = *reinterpret_cast<const uint32_t*>(from + 2048 + r * meta + 4 * g);
      vm[q] = *reinterpret_cast<const uint32_t*>(from + 2048 + (16 + r) * meta + 4 * g);
    }
  } else {
#pragma unroll
    for (int t = 0; t < 4; ++t) kw[t] = make_uint2(0u, 0u);
#pragma unroll
    for (int t = 0; t < 8; ++t) vw[t] = 0u;
    km[0] = km[1] = vm[0] = vm[1] = 0u;
  }
  // The largest magnitudes, from the scales alone: a group lies between z and z + 15 s.  A group that does not end below infinity is taken out of the images and noted.
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const float kz = bf16_half(km[q], 0), kt = fmaf(15.f, bf16_half(km[q], 1), kz), vz = bf16_half(vm[q], 0), vt = fmaf(15.f, bf16_half(vm[q], 1), vz);
    if (isfinite(kz) && isfinite(kt)) {
      mk = max(mk, max(finite_bits(kz), finite_bits(kt)));
    } else {
      lost |= 16u;
      km[q] = 0u;
    }
    if (isfinite(vz) && isfinite(vt)) {
      mv = max(mv, max(finite_bits(vz), finite_bits(vt)));
    } else {
      lost |= 1u << (2 * half + q);
      vm[q] = 0u;
    }
  }
  __shared__ uint32_t top_k[8], top_v[8], any_lost[8], missing[8];
  const uint32_t wk = __reduce_max_sync(0xffffffffu, mk), wv = __reduce_max_sync(0xffffffffu, mv), wl = __reduce_or_sync(0xffffffffu, lost);
  const uint32_t wm = __reduce_or_sync(0xffffffffu, tok < len && from == nullptr ? 1u : 0u);      // (a warp has 16 tokens: one page)
  if ((tid & 31) == 0) {
    top_k[tid >> 5] = wk;
    top_v[tid >> 5] = wv;
    any_lost[tid >> 5] = wl;
    missing[tid >> 5] = wm;
  }
  __syncthreads();
  uint32_t tk = 0, tv = 0, tl = 0, flags = 0xFFu;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    tk = max(tk, top_k[i]);
    tv = max(tv, top_v[i]);
    tl |= any_lost[i];
    flags &= ~((missing[i] & 1u) << i);
  }
  const int ek = scale_exponent(tk), ev = min(scale_exponent(tv), 126 - kDown);
  TileHead* head = plan.heads + at;
  if (tid == 0) {
    head->k_scale = pow2i(-ek);
    head->v_scale = pow2i(max(-ev - kDown, -126));
    head->flags = flags | (tl != 0 ? 256u : 0u);
  }
  lost |= __shfl_xor_sync(0xffffffffu, lost, 1);
  if (half == 0) head->lost[row] = (uint8_t)lost;
  const float fk = pow2i(ek), fv = pow2i(ev);
  unsigned char* kd = plan.k_images + at * kTileBytes + (row >> 3) * 2048 + (row & 7) * 16;
  unsigned char* vd = plan.v_images + at * kTileBytes + row * 16;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const float ks = bf16_half(km[q], 1) * fk, kz = bf16_half(km[q], 0) * fk, vs = bf16_half(vm[q], 1) * fv, vz = bf16_half(vm[q], 0) * fv;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int c = 4 * (2 * half + q) + t;      // 8 channels 8 c ..
      const uint32_t kc = q ? kw[t].y : kw[t].x, vc = __byte_perm(vw[2 * t], vw[2 * t + 1], q ? 0x7632 : 0x5410);
      uint32_t y[4], z[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        y[i] = pack_half2(fmaf((float)(kc >> (8 * i) & 15u), ks, kz), fmaf((float)(kc >> (8 * i + 4) & 15u), ks, kz));
        z[i] = pack_half2(fmaf((float)(vc >> (8 * i) & 15u), vs, vz), fmaf((float)(vc >> (8 * i + 4) & 15u), vs, vz));
      }
      *reinterpret_cast<uint4*>(kd + c * 128) = make_uint4(y[0], y[1], y[2], y[3]);
      *reinterpret_cast<uint4*>(vd + c * 2048) = make_uint4(z[0], z[1], z[2], z[3]);
    }
  }
}

// ---------------------------------------------------------------------------------------------------------------- attention
// Polls a phase of a barrier up to max_polls times; false if it never completed.  Without a suspend hint: a phase that completes ends the poll at once.
__device__ __forceinline__ bool wait_phase(uint32_t bar, uint32_t parity, uint32_t max_polls) {
  uint32_t ok;
#pragma unroll 1
  for (uint32_t n = 0;; ++n) {
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    if (ok != 0) return true;
    if (n >= max_polls) return false;
  }
}
enum Bar { kKFull = 0, kVFull = 2, kKEmpty = 4, kVEmpty = 6, kSFull = 8, kPHalf = 10, kPReady = 12, kDone = 14, kQReady = 16, kAllDone = 18, kBars = 19 };
constexpr int kBehind = 6 * kTileBytes;          // bytes of shared memory before the barriers
constexpr int kSmem = kBehind + 256;             // and before the sequences' positions

// The items of a sequence, and where a thread block is in the line of positions.
struct Walk {
  int i, h, r;                                   // sequence and KV head of the pass, row tile
  int count, len, rows;                          // of the sequence
  long long pos, end;
  int off;                                       // position in the item: kAhead, then its tiles
};
__device__ __forceinline__ int tiles_of(int len, int count, int rows, int g, int r) {
  const int last = min((r + 1) * kRows, rows) - 1, sees = min(len, max(0, len - count + last / g + 1));
  return max(1, (sees + kTile - 1) / kTile);
}
__device__ __forceinline__ void enter_sequence(const PagedView& v, const ChunkPlan& plan, Walk& w) {
  w.count = v.count(plan.b0 + w.i);
  w.len = v.length(plan.b0 + w.i, v.add_counts ? w.count : 0);
  w.rows = w.count * v.g;
}
struct Segment {
  int j0, j1, tiles;                             // key tiles of this thread block, and of the item
};
// The tiles of the present item that are this thread block's (j0 == j1: none); w moves behind them, but not to the next item.
__device__ __forceinline__ Segment take(const PagedView& v, Walk& w) {
  Segment s;
  s.tiles = tiles_of(w.len, w.count, w.rows, v.g, w.r);
  const long long first = w.pos - w.off + kAhead;
  s.j0 = max(0, w.off - kAhead);
  s.j1 = (int)min((long long)s.tiles, w.end - first);
  if (s.j1 < s.j0) s.j1 = s.j0;
  w.pos = min(w.end, first + s.tiles);
  return s;
}
__device__ __forceinline__ void next_item(const PagedView& v, const ChunkPlan& plan, Walk& w) {
  w.off = 0;
  if ((++w.r) * kRows < w.rows) return;
  w.r = 0;
  if (++w.h < plan.nh) return;
  w.h = 0;
  do {
    ++w.i;
    if (w.i >= plan.nb) return;                  // (the line ends here)
    enter_sequence(v, plan, w);
  } while (w.rows == 0);
}

// The thread block whose range has position u: the last one that begins at or before it.
__device__ __forceinline__ int owner_of(long long u, long long total, int parts) {
  int c = (int)min((long long)parts - 1, (long long)((double)u * parts / (double)total));
  while (c > 0 && split_begin(total, parts, c) > u) --c;
  while (c + 1 < parts && split_begin(total, parts, c + 1) <= u) ++c;
  return c;
}

// 32 columns of the thread's tensor-memory row; valid after the wait, which names them.
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t* u) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]),
        "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]), "=r"(u[17]), "=r"(u[18]), "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]), "=r"(u[25]),
        "=r"(u[26]), "=r"(u[27]), "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_wait32(uint32_t* u) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(u[0]), "+r"(u[1]), "+r"(u[2]), "+r"(u[3]), "+r"(u[4]), "+r"(u[5]), "+r"(u[6]), "+r"(u[7]), "+r"(u[8]), "+r"(u[9]), "+r"(u[10]), "+r"(u[11]), "+r"(u[12]),
                 "+r"(u[13]), "+r"(u[14]), "+r"(u[15]), "+r"(u[16]), "+r"(u[17]), "+r"(u[18]), "+r"(u[19]), "+r"(u[20]), "+r"(u[21]), "+r"(u[22]), "+r"(u[23]), "+r"(u[24]), "+r"(u[25]),
                 "+r"(u[26]), "+r"(u[27]), "+r"(u[28]), "+r"(u[29]), "+r"(u[30]), "+r"(u[31])
               :
               : "memory");
}
__device__ __forceinline__ float fmax_of(const uint32_t* u, float m) {      // of 32 values and m, four chains
  float a[4] = {m, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
  for (int i = 0; i < 32; i += 2) a[i >> 1 & 3] = fmaxf(fmaxf(a[i >> 1 & 3], __uint_as_float(u[i])), __uint_as_float(u[i + 1]));
  return fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3]));
}

// What a thread keeps of its row over the tiles of a segment.
struct Row {
  float ref, denom;                        // in powers of two; sum of the weights
  float v_scale;                           // what O is to be multiplied with
  bool flushed;                            // the row of `parts` has the sums of earlier tiles, at the reference that it says
};

// Adds the row of O to its sums in memory (kPartFloats floats at `to`), relative to the present reference, which is left there.
__device__ __forceinline__ void flush_row(uint32_t o_addr, float* to, Row& row) {
  const float old = row.flushed ? ex2(to[kD] - row.ref) : 0.f;
#pragma unroll 1
  for (int h = 0; h < 8; ++h) {
    uint32_t x[16];
    tmem_ld16_issue(o_addr + 16 * h, x);
    tmem_wait_ld16(x);
#pragma unroll
    for (int k = 0; k < 16; k += 4) {
      float4 y = row.flushed ? *reinterpret_cast<const float4*>(to + 16 * h + k) : make_float4(0.f, 0.f, 0.f, 0.f);
      y.x = fmaf(__uint_as_float(x[k]), row.v_scale, row.flushed ? y.x * old : 0.f);
      y.y = fmaf(__uint_as_float(x[k + 1]), row.v_scale, row.flushed ? y.y * old : 0.f);
      y.z = fmaf(__uint_as_float(x[k + 2]), row.v_scale, row.flushed ? y.z * old : 0.f);
      y.w = fmaf(__uint_as_float(x[k + 3]), row.v_scale, row.flushed ? y.w * old : 0.f);
      *reinterpret_cast<float4*>(to + 16 * h + k) = y;
    }
  }
  to[kD] = row.ref;
  row.flushed = true;
}

// One key tile of a row's softmax; S is at s_addr, O at o_addr.  masked: the row sees the columns <= last of those 16 that `there` has.  fresh: O has nothing yet.
__device__ __forceinline__ void softmax_tile(uint32_t s_addr, uint32_t o_addr, bool masked, int last, uint32_t there, bool fresh, float factor, float v_scale, Row& row,
                                             uint32_t half_bar) {
  uint32_t u[128];
  float mx = -INFINITY;
  tmem_ld32(s_addr, u);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    tmem_wait32(u + 32 * q);
    if (q < 3) tmem_ld32(s_addr + 32 * (q + 1), u + 32 * (q + 1));
    if (masked) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int lim = there >> (2 * q + h) & 1u ? last - 32 * q - 16 * h : -1;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (i > lim) u[32 * q + 16 * h + i] = 0xFF800000u;      // weight 0
      }
    }
    mx = fmax_of(u + 32 * q, mx);
  }
  mx *= factor;
  // ---- the reference of the row and the scale of O
  if (fresh) {
    if (mx > row.ref + kRise || row.ref == -1e30f) {               // (what memory has of the row is brought to the new reference when it is added to)
      const float up = mx > -INFINITY ? mx : row.ref;
      row.denom *= ex2(row.ref - up);
      row.ref = up;
    }
    row.v_scale = v_scale;
  }
  const bool rises = !fresh && mx > row.ref + kRise;
  int v_shift = (int)(__float_as_uint(v_scale) >> 23) - (int)(__float_as_uint(row.v_scale) >> 23);      // (powers of two)
  const bool outgrown = v_shift > kSlack;
  if (__any_sync(0xffffffffu, rises || outgrown)) {
    float f = 1.f;
    if (rises) {
      f = ex2(row.ref - mx);
      row.denom *= f;
      row.ref = mx;
    }
    if (outgrown) {
      f *= pow2i(max(-v_shift, -126));
      row.v_scale = v_scale;
      v_shift = 0;
    }
#pragma unroll 1
    for (int h = 0; h < 8; ++h) {
      uint32_t x[16];
      tmem_ld16_issue(o_addr + 16 * h, x);
      tmem_wait_ld16(x);
#pragma unroll
      for (int k = 0; k < 16; ++k) x[k] = __float_as_uint(__uint_as_float(x[k]) * f);
      tmem_st8(o_addr + 16 * h, reinterpret_cast<uint32_t(&)[8]>(x[0]));
      tmem_st8(o_addr + 16 * h + 8, reinterpret_cast<uint32_t(&)[8]>(x[8]));
    }
  }
  // ---- weights
  v_shift = max(v_shift, -100);
  const float offset = (float)(kShift + v_shift) - row.ref;
  const uint64_t factor2 = pack2(factor, factor), offset2 = pack2(offset, offset);
  uint64_t sum[2] = {0ull, 0ull};
#pragma unroll
  for (int h = 0; h < 8; ++h) {
    uint32_t wd[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float x0, x1;
      unpack2(fma2(pack2u(u[16 * h + 2 * i], u[16 * h + 2 * i + 1]), factor2, offset2), x0, x1);
      const float p0 = ex2(x0), p1 = ex2(x1);
      sum[i & 1] = add2(sum[i & 1], pack2(p0, p1));
      wd[i] = pack_half2(p0, p1);
    }
    tmem_st8(s_addr + 8 * h, wd);
    if (h == 3) {
      asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
      tc_fence_before();
      mbar_arrive(half_bar);
    }
  }
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
  float s0, s1;
  unpack2(add2(sum[0], sum[1]), s0, s1);
  row.denom = fmaf(s0 + s1, pow2i(-v_shift), row.denom);
}

// A row of results; lost: quarters (bits 0 .. 3) that are not finite, bit 4: all of them.
__device__ __forceinline__ void store32(void* to, const uint32_t (&y)[8], bool wide) {
  if (wide) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3]), "r"(y[4]), "r"(y[5]), "r"(y[6]), "r"(y[7])
                 : "memory");
  } else {
    reinterpret_cast<uint4*>(to)[0] = make_uint4(y[0], y[1], y[2], y[3]);
    reinterpret_cast<uint4*>(to)[1] = make_uint4(y[4], y[5], y[6], y[7]);
  }
}

__global__ void __launch_bounds__(kThreads, 1)
attend_kernel(const __grid_constant__ PagedAttention a, const __grid_constant__ ChunkPlan plan) {
  extern __shared__ __align__(128) unsigned char smem[];
  unsigned char* Qs = smem;                              // two tiles
  unsigned char* Ks = smem + 2 * kTileBytes;             // two stages
  unsigned char* Vs = smem + 4 * kTileBytes;             // two stages
  const uint32_t bars = smem_u32(smem + kBehind);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + kBehind + 8 * kBars);
  int* start = reinterpret_cast<int*>(smem + kBehind + 8 * kBars + 8);       // i, h, r, off
  long long* line = reinterpret_cast<long long*>(smem + kSmem);              // [nb + 1] positions before each sequence
  auto bar = [&](int i) { return bars + 8u * (uint32_t)i; };
  const PagedView& v = a.view;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (tid == 9 * 32) {
    for (int i = 0; i < kBars; ++i) mbar_init(bar(i), (i >= kPHalf && i < kDone) || (i >= kQReady && i < kAllDone) ? kTile : 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  dependency_wait();
  // ---- the line: positions of every sequence, then where this thread block begins
  for (int i = warp; i < plan.nb; i += kThreads / 32) {
    const int count = v.count(plan.b0 + i), len = v.length(plan.b0 + i, v.add_counts ? count : 0), rows = count * v.g;
    long long sum = 0;
    for (int r = lane; r * kRows < rows; r += 32) sum += kAhead + tiles_of(len, count, rows, v.g, r);
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if (lane == 0) line[i + 1] = sum * plan.nh;
  }
  if (tid == 0) line[0] = 0;
  __syncthreads();
  if (warp == 0) {
    long long sum = 0;
    for (int i0 = 0; i0 < plan.nb; i0 += 32) {
      long long x = i0 + lane < plan.nb ? line[i0 + lane + 1] : 0;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += y;
      }
      if (i0 + lane < plan.nb) line[i0 + lane + 1] = sum + x;
      sum += __shfl_sync(0xffffffffu, x, 31);
    }
  }
  __syncthreads();
  const long long total = line[plan.nb];
  const int parts = (int)min((long long)gridDim.x, max(1ll, total / (kAhead + 2)));
  Walk walk{};
  const bool any = (int)blockIdx.x < parts && total > 0;
  walk.pos = any ? split_begin(total, parts, blockIdx.x) : 0;
  walk.end = any ? split_begin(total, parts, blockIdx.x + 1) : 0;
  if (warp == 0 && any) {
    int lo = 0, hi = plan.nb;                    // the last sequence that begins at or before the position
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (line[mid] <= walk.pos) lo = mid; else hi = mid;
    }
    while (line[lo + 1] <= walk.pos) ++lo;
    walk.i = lo;
    enter_sequence(v, plan, walk);
    const long long per_head = (line[lo + 1] - line[lo]) / plan.nh;
    long long off = walk.pos - line[lo];
    const int h = (int)(off / per_head);
    off -= h * per_head;
    int r = 0;
    for (;; r += 32) {                           // items before the position, 32 at a time
      long long x = (r + lane) * kRows < walk.rows ? kAhead + tiles_of(walk.len, walk.count, walk.rows, v.g, r + lane) : 0;
      const long long own = x;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += y;
      }
      const uint32_t behind = __ballot_sync(0xffffffffu, x > off);
      if (behind != 0) {
        const int k = __ffs(behind) - 1;
        off -= __shfl_sync(0xffffffffu, x - own, k);
        r += k;
        break;
      }
      off -= __shfl_sync(0xffffffffu, x, 31);
      if ((r + 32) * kRows >= walk.rows) break;  // (not reached)
    }
    if (lane == 0) {
      start[0] = lo;
      start[1] = h;
      start[2] = r;
      start[3] = (int)off;
    }
  }
  if (tid == 0) plan.broken[blockIdx.x] = Broken{0, 0, 0, -1};
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tbase = *tmem_slot;
  if (any) {
    walk.i = start[0];
    walk.h = start[1];
    walk.r = start[2];
    walk.off = start[3];
    enter_sequence(v, plan, walk);
  }
  // tensor-memory columns: S_A / P_A at 0, S_B / P_B at 128, O_A at 256, O_B at 384
  const uint32_t max_polls = a.max_polls ? a.max_polls : kPolls;
  bool dead = false;
  auto wait = [&](int i, uint32_t parity) {
    if (!dead && !wait_phase(bar(i), parity, max_polls)) {
      dead = true;
      atomicOr(v.status, (uint32_t)MIXKVQ_DEV_COPY_TIMEOUT);
    }
    return !dead;
  };
  // The same for a whole warp: all of its lanes go on or none, as the instructions on tensor memory and the votes behind a wait are the warp's.
  auto wait_warp = [&](int i, uint32_t parity) {
    dead = __all_sync(0xffffffffu, wait(i, parity)) == 0;
    return !dead;
  };
  auto two_groups = [&](const Walk& w) { return w.r * kRows + kTile < w.rows; };

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 104;" ::: "memory");
    if (warp == 8 && lane == 0) {
      // ---------------------------------------------------------------- tensor-core issue
      const uint32_t idesc_qk = make_idesc(128, 128, 0, 0), idesc_pv = make_idesc(128, 128, 0, 1);
      uint32_t t = 0, tiles_b = 0, segs = 0, segs_b = 0;                     // key tiles so far (group A has all of them), group B's, segments, those with a group B
      auto issue_s = [&](int g, uint32_t tile) {
        const uint64_t qd = make_desc(smem_u32(Qs + g * kTileBytes), 128, 2048), kd = make_desc(smem_u32(Ks + (tile & 1) * kTileBytes), 128, 2048);
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) tc_mma_ss(tbase + 128 * g, qd + (uint64_t)(ks * 16), kd + (uint64_t)(ks * 16), idesc_qk, ks > 0);
        tc_commit(bar(kSFull + g));
      };
      auto issue_o = [&](int g, uint32_t tile, uint32_t parity, bool more) {
        const uint64_t vd = make_desc(smem_u32(Vs + (tile & 1) * kTileBytes), 128, 2048);
        const uint32_t o = tbase + 256 + 128 * g, p = tbase + 128 * g;
        if (!wait(kPHalf + g, parity)) return false;
        tc_fence_after();
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) tc_mma_ts(o, p + 8 * ks, vd + (uint64_t)(ks * 16), idesc_pv, ks > 0 || more);
        if (!wait(kPReady + g, parity)) return false;
        tc_fence_after();
#pragma unroll
        for (int ks = 4; ks < 8; ++ks) tc_mma_ts(o, p + 8 * ks, vd + (uint64_t)(ks * 16), idesc_pv, 1);
        return true;
      };
      while (walk.pos < walk.end && !dead) {
        const Segment s = take(v, walk);
        const bool both = two_groups(walk);
        if (s.j1 > s.j0) {
          if (!wait(kQReady, segs & 1) || (both && !wait(kQReady + 1, segs_b & 1))) break;
          ++segs;
          if (both) ++segs_b;
          if (!wait(kKFull + (t & 1), t >> 1 & 1)) break;
          tc_fence_after();
          issue_s(0, t);
          if (both) issue_s(1, t);
          tc_commit(bar(kKEmpty + (t & 1)));
          bool ok = true;
          for (int j = s.j0; j < s.j1; ++j, ++t) {
            const bool more = j + 1 < s.j1;
            if (!(ok = wait(kVFull + (t & 1), t >> 1 & 1))) break;
            tc_fence_after();
            if (!(ok = issue_o(0, t, t & 1, (j - s.j0) % kFlush != 0))) break;
            if (!both) tc_commit(bar(kVEmpty + (t & 1)));
            if (!more) tc_commit(bar(kDone));
            if (more) {
              if (!(ok = wait(kKFull + ((t + 1) & 1), (t + 1) >> 1 & 1))) break;
              tc_fence_after();
              issue_s(0, t + 1);
              if (!both) tc_commit(bar(kKEmpty + ((t + 1) & 1)));
            }
            if (both) {
              if (!(ok = issue_o(1, t, tiles_b & 1, (j - s.j0) % kFlush != 0))) break;
              ++tiles_b;
              tc_commit(bar(kVEmpty + (t & 1)));
              if (!more) tc_commit(bar(kDone + 1));
              if (more) {
                issue_s(1, t + 1);
                tc_commit(bar(kKEmpty + ((t + 1) & 1)));
              }
            }
          }
          if (!ok) break;
        }
        if (walk.pos < walk.end) next_item(v, plan, walk);
      }
      tc_commit(bar(kAllDone));                          // every product issued above has finished when this one fires
      dead = false;
      wait(kAllDone, 0);
    } else if (warp == 9 && lane == 0) {
      // ---------------------------------------------------------------- bulk copies of the key and value tiles
      uint32_t t = 0;                                    // tiles asked for
      while (walk.pos < walk.end && !dead) {
        const Segment s = take(v, walk);
        const size_t tiles = (size_t)(walk.i * plan.nh + walk.h) * plan.max_tiles;
        for (int j = s.j0; j < s.j1; ++j, ++t) {
          const int st = t & 1;
          const uint32_t before = ((t >> 1) - 1) & 1;
          if (t >= 2 && !wait(kKEmpty + st, before)) break;
          mbar_expect_tx(bar(kKFull + st), kTileBytes + (t == 0 ? a.test_extra : 0u));
          bulk_copy(smem_u32(Ks + st * kTileBytes), plan.k_images + (tiles + j) * kTileBytes, kTileBytes, bar(kKFull + st));
          if (t >= 2 && !wait(kVEmpty + st, before)) {   // the key copy above is awaited below like the others
            mbar_expect_tx(bar(kVFull + st), 0);
            ++t;
            break;
          }
          mbar_expect_tx(bar(kVFull + st), kTileBytes);
          bulk_copy(smem_u32(Vs + st * kTileBytes), plan.v_images + (tiles + j) * kTileBytes, kTileBytes, bar(kVFull + st));
        }
        if (walk.pos < walk.end) next_item(v, plan, walk);
      }
      // no copy may be in flight when the thread block ends: the last copy into each stage has landed once its barrier's phase is over
      for (uint32_t k = t < 2 ? 0 : t - 2; k < t; ++k) {
        dead = false;                                    // every one of these waits is made, whatever the others did
        wait(kKFull + (k & 1), k >> 1 & 1);
        dead = false;
        wait(kVFull + (k & 1), k >> 1 & 1);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 200;" ::: "memory");
    // ------------------------------------------------------------------ softmax and output rows
    const int g = warp >> 2;
    const uint32_t lane_base = tbase + ((uint32_t)((warp & 3) * 32) << 16), s_addr = lane_base + 128 * g, o_addr = lane_base + 256 + 128 * g;
    const bool wide = (reinterpret_cast<uintptr_t>(a.out) & 31u) == 0;
    uint32_t t = 0, segs = 0;                            // of this group
    while (walk.pos < walk.end) {                        // (a warp whose wait has run out has nothing to add, and says so in every place that is read later)
      const Segment s = take(v, walk);
      if (s.j1 > s.j0 && (g == 0 || two_groups(walk))) {
        const int x = walk.r * kRows + g * kTile + (tid & 127);
        const bool mine = x < walk.rows;
        // (a row behind the last sees what that one sees, with a query of zeros)
        const int xi = min(x, walk.rows - 1) / v.g, head = x - xi * v.g;
        const int sees = min(walk.len, max(0, walk.len - walk.count + xi + 1));
        const size_t row = ((size_t)(plan.b0 + walk.i) * v.Hq + (size_t)(plan.h0 + walk.h) * v.g + (mine ? head : 0)) * v.n + xi;
        float factor = 0.f;
        if (!dead) {
          uint4 w[16];
          const uint4* src = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + row * kD);
#pragma unroll
          for (int c = 0; c < 16; ++c) w[c] = mine ? src[c] : make_uint4(0u, 0u, 0u, 0u);
          uint32_t top = 0;
#pragma unroll
          for (int c = 0; c < 16; ++c) {
            const uint32_t y[4] = {w[c].x, w[c].y, w[c].z, w[c].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) top = max(top, max(y[k] << 16 & 0x7FFFFFFFu, y[k] & 0x7FFF0000u));
          }
          const int e = scale_exponent(top);
          const float up = pow2i(e);
          factor = a.scale_log2e * pow2i(-e);
          unsigned char* to = Qs + g * kTileBytes + ((tid & 127) >> 3) * 2048 + (tid & 7) * 16;
#pragma unroll
          for (int c = 0; c < 16; ++c) {
            const uint32_t y[4] = {w[c].x, w[c].y, w[c].z, w[c].w};
            uint32_t z[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) z[k] = pack_half2(__uint_as_float(y[k] << 16) * up, __uint_as_float(y[k] & 0xFFFF0000u) * up);
            *reinterpret_cast<uint4*>(to + c * 128) = make_uint4(z[0], z[1], z[2], z[3]);
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          mbar_arrive(bar(kQReady + g));
        }
        const int warp_sees = __reduce_min_sync(0xffffffffu, sees);
        const TileHead* heads = plan.heads + (size_t)(walk.i * plan.nh + walk.h) * plan.max_tiles;
        Row sums{-1e30f, 0.f, 0.f, false};
        uint32_t lost = 0;
        const bool whole = s.j0 == 0 && s.j1 == s.tiles;
        // the thread block's first part of an item and its last have a place each; a whole item's sums in between take the second one
        float* to = plan.parts + ((size_t)(2 * blockIdx.x + (s.j0 == 0 ? 1 : 0)) * kRows + g * kTile + (tid & 127)) * kPartFloats;
#pragma unroll 1
        for (int j = s.j0; j < s.j1 && !dead; ++j) {
          const float4 head_of = *reinterpret_cast<const float4*>(heads + j);       // (under way while the thread waits)
          const uint32_t flags = __float_as_uint(head_of.z);
          const bool masked = (j + 1) * kTile > warp_sees || flags != 0xFFu, fresh = (j - s.j0) % kFlush == 0;
          if (!wait_warp(kSFull + g, t & 1)) break;
          tc_fence_after();
          if (fresh && j > s.j0) flush_row(o_addr, to, sums);
          softmax_tile(s_addr, o_addr, masked, sees - 1 - j * kTile, flags, fresh, fmaxf(factor * head_of.x, kLeast), head_of.y, sums, bar(kPHalf + g));
          if (flags >> 8 & 1u)
            for (int k = 0; k < kTile && j * kTile + k < sees; ++k) lost |= heads[j].lost[k];
          tc_fence_before();
          mbar_arrive(bar(kPReady + g));
          ++t;
        }
        const bool done = !dead && wait_warp(kDone + g, segs & 1);
        if (done) {
          tc_fence_after();
          if (sums.flushed) flush_row(o_addr, to, sums);
        } else {
          sums = Row{-1e30f, 0.f, 0.f, false};
          lost = 0;
        }
        const float inv = whole ? (sums.denom == 0.f ? 0.f : pow2i(kDown) / sums.denom) : 1.f;
#pragma unroll 1
        for (int q = 0; q < 4; ++q) {                  // 32 channels
          float y[32];
          {
            uint32_t x[32];
            if (done) {
              tmem_ld32(o_addr + 32 * q, x);
              tmem_wait32(x);
            } else {
#pragma unroll
              for (int d = 0; d < 32; ++d) x[d] = 0u;
            }
            const float f = lost >> q & 1u || lost & 16u ? NAN : inv;
#pragma unroll
            for (int d = 0; d < 32; ++d) y[d] = (sums.flushed ? to[32 * q + d] : __uint_as_float(x[d]) * sums.v_scale) * (whole ? f : 1.f);
          }
          if (!whole) {
            if (!sums.flushed) {
#pragma unroll
              for (int d = 0; d < 32; d += 4) *reinterpret_cast<float4*>(to + 32 * q + d) = make_float4(y[d], y[d + 1], y[d + 2], y[d + 3]);
            }
          } else if (mine && a.out_bf16) {
            char* out = static_cast<char*>(a.out) + row * (2 * kD) + 64 * q;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              uint32_t z[8];
#pragma unroll
              for (int d = 0; d < 8; ++d) z[d] = bf16_pair(y[16 * k + 2 * d], y[16 * k + 2 * d + 1]);
              store32(out + 32 * k, z, wide);
            }
          } else if (mine) {
            char* out = static_cast<char*>(a.out) + row * (4 * kD) + 128 * q;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              uint32_t z[8];
#pragma unroll
              for (int d = 0; d < 8; ++d) z[d] = __float_as_uint(y[8 * k + d]);
              store32(out + 32 * k, z, wide);
            }
          }
        }
        if (!whole) {
          *reinterpret_cast<float4*>(to + kD) = make_float4(sums.ref, sums.denom, __uint_as_float(lost), 0.f);
          if (tid == 0 && s.j0 == 0)
            plan.broken[blockIdx.x] = Broken{walk.i, walk.h, walk.r, owner_of(split_begin(total, parts, blockIdx.x + 1) + (s.tiles - s.j1) - 1, total, parts)};
        }
        ++segs;
      }
      if (walk.pos < walk.end) next_item(v, plan, walk);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 8) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tbase), "r"(512));
}

// Joins the parts of the item that begins in thread block blockIdx.x of attend_kernel and ends in another: a warp has a row, a lane four channels, eight parts' loads are
// under way together.
constexpr int kJoinBlocks = 16;                  // thread blocks of an item
__global__ void __launch_bounds__(256)
join_kernel(const __grid_constant__ PagedAttention a, const __grid_constant__ ChunkPlan plan) {
  dependency_wait();
  const PagedView& v = a.view;
  const Broken it = plan.broken[blockIdx.x];
  if (it.last <= (int)blockIdx.x) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rows = v.count(plan.b0 + it.b) * v.g, c0 = blockIdx.x;
  for (int k = blockIdx.y * 8 + warp; k < kRows; k += 8 * kJoinBlocks) {
    const int x = it.r * kRows + k;
    if (x >= rows) return;
    float ref = -1e30f, denom = 0.f, y[4] = {0.f, 0.f, 0.f, 0.f};
    uint32_t lost = 0;
    for (int c = c0; c <= it.last; c += 8) {
      float4 o[8], m[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int part = min(c + i, it.last);
        const float* from = plan.parts + ((size_t)(2 * part + (part == c0 ? 1 : 0)) * kRows + k) * kPartFloats;
        o[i] = *reinterpret_cast<const float4*>(from + 4 * lane);
        m[i] = *reinterpret_cast<const float4*>(from + kD);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (c + i > it.last) break;
        const float up = fmaxf(ref, m[i].x), f0 = ex2(ref - up), f1 = ex2(m[i].x - up);
        ref = up;
        denom = denom * f0 + m[i].y * f1;
        lost |= __float_as_uint(m[i].z);
        y[0] = y[0] * f0 + o[i].x * f1;
        y[1] = y[1] * f0 + o[i].y * f1;
        y[2] = y[2] * f0 + o[i].z * f1;
        y[3] = y[3] * f0 + o[i].w * f1;
      }
    }
    float inv = denom == 0.f ? 0.f : pow2i(kDown) / denom;
    if (lost >> (lane >> 3) & 1u || lost & 16u) inv = NAN;
    const int i = x / v.g, head = x - i * v.g;
    const size_t at = (((size_t)(plan.b0 + it.b) * v.Hq + (size_t)(plan.h0 + it.h) * v.g + head) * v.n + i) * kD + 4 * lane;
    if (a.out_bf16)
      *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + at) = make_uint2(bf16_pair(y[0] * inv, y[1] * inv), bf16_pair(y[2] * inv, y[3] * inv));
    else
      *reinterpret_cast<float4*>(static_cast<float*>(a.out) + at) = make_float4(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
  }
}

constexpr int kMostBlocks = 148;

// What a pass takes: whole sequences while their images fit, or some heads of one.
void pass_of(int B, int Hkv, long long tiles, int* nb, int* nh) {
  const long long streams = std::max(1ll, (long long)(kImageBytes / (2 * (size_t)kTileBytes)) / tiles);
  *nh = (int)std::min((long long)Hkv, streams);
  *nb = *nh < Hkv ? 1 : (int)std::min((long long)B, streams / Hkv);
}
size_t rounded(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

long long paged_chunk_capacity() { return (long long)(kImageBytes / (2 * (size_t)kTileBytes)) * kTile; }

static size_t bytes_of(size_t images) {
  return images * 2 * kTileBytes + rounded(images * sizeof(TileHead)) + rounded((size_t)2 * kMostBlocks * kRows * kPartFloats * 4) + rounded(kMostBlocks * sizeof(Broken)) + 256;
}
size_t paged_chunk_workspace_need(int Hkv, int batch, long long capacity) {
  const long long tiles = (capacity + kTile - 1) / kTile;
  int nb, nh;
  pass_of(batch, Hkv, tiles, &nb, &nh);
  return bytes_of((size_t)nb * nh * tiles);
}
// No less than what any smaller batch or capacity needs: a pass holds whole streams, so that what it needs falls where one fewer fits.
size_t paged_chunk_workspace_bytes(int Hkv, int batch, long long capacity) {
  const long long tiles = (capacity + kTile - 1) / kTile;
  return bytes_of((size_t)std::min((long long)batch * Hkv * tiles, (long long)(kImageBytes / (2 * (size_t)kTileBytes))));
}

cudaError_t paged_chunk_setup() { return cudaFuncSetAttribute(attend_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem + 8 * (MIXKVQ_PAGED_MAX_BATCH + 1)); }

cudaError_t launch_paged_chunk(const PagedAttention& a, int n_sms, cudaStream_t stream, int* launches) {
  const PagedView& v = a.view;
  ChunkPlan plan{};
  plan.max_tiles = (int)((((long long)v.max_pages << v.lg_page) + kTile - 1) / kTile);
  int nb, nh;
  pass_of(v.B, v.Hkv, plan.max_tiles, &nb, &nh);
  const size_t images = (size_t)nb * nh * plan.max_tiles;
  unsigned char* at = reinterpret_cast<unsigned char*>(rounded(reinterpret_cast<size_t>(a.parts)));
  plan.k_images = at;
  plan.v_images = at + images * kTileBytes;
  at += images * 2 * kTileBytes;
  plan.heads = reinterpret_cast<TileHead*>(at);
  at += rounded(images * sizeof(TileHead));
  plan.parts = reinterpret_cast<float*>(at);
  at += rounded((size_t)2 * kMostBlocks * kRows * kPartFloats * 4);
  plan.broken = reinterpret_cast<Broken*>(at);
  const unsigned blocks = (unsigned)std::min(kMostBlocks, n_sms);
  for (int b0 = 0; b0 < v.B; b0 += nb)
    for (int h0 = 0; h0 < v.Hkv; h0 += nh) {
      plan.b0 = b0;
      plan.nb = std::min(nb, v.B - b0);
      plan.h0 = h0;
      plan.nh = std::min(nh, v.Hkv - h0);
      cudaError_t e = launch_dependent(unpack_kernel, dim3((unsigned)plan.max_tiles, (unsigned)plan.nh, (unsigned)plan.nb), 256, 0, stream, a, plan);
      if (e != cudaSuccess) return e;
      e = launch_dependent(attend_kernel, dim3(blocks), kThreads, kSmem + 8 * (size_t)(plan.nb + 1), stream, a, plan);
      if (e != cudaSuccess) return e;
      e = launch_dependent(join_kernel, dim3(blocks, kJoinBlocks), 256, 0, stream, a, plan);
      if (e != cudaSuccess) return e;
      *launches += 3;
    }
  return cudaSuccess;
}

}  // namespace mixkvq
