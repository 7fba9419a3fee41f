// Attention of the newest tokens of every sequence over the pages of the 4-bit cache.
//
// Mathematics.  A key is k_c = s_g c_c + z_g in group g of G channels, so a logit is sum_g s_g (sum_{c in g} q_c c_c) + z_g (sum_{c in g} q_c): the codes enter the
// tensor core as they are (a nibble masked out of a word is an fp16 subnormal, 2^-24 or 2^-20 times the code; the factor 16 is taken out of the query), the sums of a group
// are scaled behind it in fp32.  A value is s_g c + z_g with a scale per token, so the weight p s_g of (token, group) is the other operand of the second product, in fp16,
// and sum p z_g is added up in fp32.  One pass over the tokens with a running reference of the logits.
//
// Operands stay inside fp16's range whatever the inputs' magnitudes (a value far smaller than the largest of its group so far keeps fewer bits): a query row is scaled by a power of two (exactly) to a largest entry of 2^14 to 2^15, and p s_g by a power of
// two per group, lowered as larger scales come.  References are raised, and sums rescaled, only when a logit comes 8 (in powers of two) above the largest so far.
//
// Split: work is units of 32 tokens of one (sequence, KV head, block of query rows), all of them in one line, cut evenly over the thread blocks on the device (the
// lengths are known there alone).  A thread block goes through the pieces of streams in its range, its warps through the units of a piece, each with a ring of
// bulk copies of its own, so that no warp waits for another before the end of a piece.  A piece that is no whole stream leaves sums, which merge_kernel joins.
//
// What bounds it: each warp's chain of instructions with three warps per scheduler to cover it, not the bytes.  7b shape, 8 x 32768 tokens, one new each (168 MB, G = 32): 46 us, 0.56 of
// the rate of a copy; 360 warp instructions per 16 tokens, 54 % of the issue slots; thread blocks that share an SM end unevenly (27 to 35 us); about 10 us are the beginning (lengths, page, first copies, one behind the other) and the end with the
// merge.  Measured against it: four warps per scheduler (128 registers) 48.8 us; 16 query rows' operands in shared memory (drafts) 58.4 against 58.1.
// Rows in blocks of 16 cost 1.44 times blocks of 8, so that 9 to 72 rows are taken in several passes over the pages, which the L2 cache holds.
#include <algorithm>

#include "paged.cuh"
#include "warp_ops.cuh"

namespace mixkvq {

namespace {

constexpr int kWarps = 4;                        // of a thread block with pieces of streams, 16 of one with a whole short stream
constexpr int kUnit = 32;                        // tokens
constexpr int kStages = 2;                       // units in a warp's ring, per tile of 8 query rows
constexpr int kQueryBytes = 2048;                // operands of 8 query rows
constexpr int kPartFloats = kD + 4;              // of a row's sums: o[128], reference, denominator, (pad)
constexpr uint32_t kPolls = 1u << 21;
constexpr int kBelow = 16;                       // a reference is brought this much (in powers of two) above its row's largest logit: sums of large values keep off fp32's end
constexpr int kRise = 8;                         // and raised when a logit comes this much nearer
constexpr int kScaleTo = 5 + kBelow;             // the largest value scale of a group times its factor is brought to 2^21 .. 2^22, and lowered when it comes to 2^23
constexpr int kAhead = 12;                       // units that the beginning of a piece counts as

struct __align__(16) Broken {                    // a stream that begins in a thread block's range and ends in another's
  int last, row0, rows, pad;                     // last: the thread block that has its end, -1: none; its query rows
  long long out;                                 // where its KV head's first query row is in the output: (sequence * query heads + head) * n
  long long pad2;
};
struct Plan {
  int rows;                                      // of a block of query rows
  int direct;                                    // a thread block per stream, nothing to merge
  uint32_t g_inv;                                // x / g is the upper half of x * g_inv (x below 2^28; 0: g is 1)
  float* parts;                                  // [2 * thread blocks][rows][kPartFloats]
  Broken* broken;                                // [thread blocks]
};

__device__ __forceinline__ float pow2i(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }

__device__ __forceinline__ int row_blocks(int count, int g, int rows) { return (count * g + rows - 1) / rows; }
__device__ __forceinline__ int over_heads(const Plan& plan, int x) { return plan.g_inv == 0u ? x : (int)__umulhi((uint32_t)x, plan.g_inv); }
// total * i / parts, in 32 bits where that is enough
__device__ __forceinline__ long long cut(long long total, int parts, int i) {
  const unsigned long long x = (unsigned long long)total * (unsigned)i;
  return x >> 32 ? (long long)(x / (unsigned)parts) : (long long)((unsigned)x / (unsigned)parts);
}

// A stream: a block of query rows of a KV head of a sequence.
struct Stream {
  int b, h, row0;                                // first row of the block: token * g + head
  int len, count, units;
};

// The state of one warp over its units of a piece.
template <int kNG, int kNT>
struct WarpState {
  float acc[8][4 * kNT];                         // tile 2 j + e: channels 32 j + 4 r + e (and + 2), per row tile; times 2^-24 (e = 0), 2^-20 (e = 1) and the group's factor
  float zsum[kNG][2 * kNT];                      // sum p z of the lane's tokens
  float ref[2 * kNT], l[2 * kNT];
  float factor[kNG];
  uint32_t limit[kNG];                           // a word of a larger scale than this lowers the factor
};
// the largest word of a scale whose product with 2^e stays below 2^23
__device__ __forceinline__ uint32_t limit_of(int e) { return ((uint32_t)min(127 + kScaleTo + 2 - e, 254) << 23) - 1u; }

// The words {z, s} of a token's groups.
template <int kNG>
__device__ __forceinline__ void load_meta(uint32_t a, uint32_t (&w)[kNG]) {
  if constexpr (kNG == 4) {
    const uint4 x = lds128(a);
    w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
  } else if constexpr (kNG == 2) {
    const uint2 x = lds64(a);
    w[0] = x.x; w[1] = x.y;
  } else {
    w[0] = lds32(a);
  }
}

template <int kG, int kNT, int kW>
__global__ void __launch_bounds__(kW * 32, kW > kWarps ? 1 : kNT == 1 ? 3 : 2)
pages_kernel(const __grid_constant__ PagedAttention a, const __grid_constant__ Plan plan) {
  constexpr int kNG = kD / kG, kMeta = 512 / kG, kTileBytes = 2048 + 32 * kMeta, kRows = 8 * kNT, kUnitBytes = 2 * kTileBytes, stages = kStages * kNT;
  extern __shared__ __align__(128) unsigned char smem[];
  const PagedView& v = a.view;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, r = lane >> 2, t = lane & 3;
  const uint32_t ring = smem_u32(smem) + (uint32_t)(warp * stages * kUnitBytes);
  unsigned char* behind = smem + kW * stages * kUnitBytes;
  // The queries' operands: in registers for 16 rows; for 8 rows, where they would cost the SM four warps, in shared memory (a copy per warp: no barrier)
  constexpr bool kQueriesInRegisters = kNT > 1;
  const uint32_t q_at = smem_u32(behind) + (uint32_t)(warp * kQueryBytes) + 16u * (uint32_t)lane;
  if constexpr (!kQueriesInRegisters) behind += kW * kQueryBytes;
  const uint32_t bars = smem_u32(behind) + 8u * (uint32_t)(warp * stages);
  long long* prefix = reinterpret_cast<long long*>(behind + 8 * kW * stages);
  if (lane == 0) {
    for (int i = 0; i < stages; ++i) mbar_init(bars + 8u * i, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  dependency_wait();
  auto units_of = [&](int len) { return max(1, (len + kUnit - 1) / kUnit); };
  auto over_g = [&](int x) { return over_heads(plan, x); };
  auto positions = [&](int count, int len) { return (long long)row_blocks(count, v.g, kRows) * v.Hkv * (kAhead + units_of(len)); };
  // ---- the line: the positions of all sequences, in a lane each where there are 32 at most (no shared memory, no barrier), and the thread block's range of them
  const bool few = v.B <= 32;
  int seq_count = 0, seq_len = 0;
  long long pos, end, total = 0, upto = 0;       // upto: positions of the sequences up to the lane's
  int parts = gridDim.x;
  if (plan.direct) {
    pos = 0;
    end = 1;
  } else {
    if (few) {
      if (lane < v.B) {
        v.sequence(lane, seq_count, seq_len);
        upto = positions(seq_count, seq_len);
      }
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += y;
      }
      total = __shfl_sync(0xffffffffu, upto, 31);
    } else {
      for (int b = tid; b < v.B; b += kW * 32) {
        int count, len;
        v.sequence(b, count, len);
        prefix[b + 1] = positions(count, len);
      }
      if (tid == 0) prefix[0] = 0;
      __syncthreads();
      if (warp == 0) {
        long long sum = 0;
        for (int b0 = 0; b0 < v.B; b0 += 32) {
          long long x = b0 + lane < v.B ? prefix[b0 + lane + 1] : 0;
#pragma unroll
          for (int d = 1; d < 32; d <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, x, d);
            if (lane >= d) x += y;
          }
          if (b0 + lane < v.B) prefix[b0 + lane + 1] = sum + x;
          sum += __shfl_sync(0xffffffffu, x, 31);
        }
      }
      __syncthreads();
      total = prefix[v.B];
    }
    // at least a unit for every warp
    parts = (int)min((long long)gridDim.x, (total + kW - 1) / kW);
    if (tid == 0) plan.broken[blockIdx.x].last = -1;
    if ((int)blockIdx.x >= parts) return;
    pos = cut(total, parts, blockIdx.x);
    end = cut(total, parts, blockIdx.x + 1);
  }
  const int pi = r ^ (r >> 1 & 1);               // token of a tile that the lane's rows of its products are (and 8 more)
  uint32_t phase = 0;                            // of the warp's barriers, a bit each
  bool dead = false;
  auto wait = [&](uint32_t bar, uint32_t parity) {
    if (!__all_sync(0xffffffffu, mbar_wait_polls(bar, parity, a.max_polls ? a.max_polls : kPolls))) {
      dead = true;
      if (lane == 0) atomicOr(v.status, (uint32_t)MIXKVQ_DEV_COPY_TIMEOUT);
    }
  };

  while (pos < end) {
    // ---- the piece: units u0 .. u1 - 1 of a stream
    Stream st;
    int u0, u1;
    long long first;
    if (plan.direct) {
      const int blocks = row_blocks(v.n, v.g, kRows), stream = blockIdx.x;
      st.b = stream / (blocks * v.Hkv);
      v.sequence(st.b, st.count, st.len);
      const int s = stream - st.b * blocks * v.Hkv;
      st.h = s / blocks;
      st.row0 = (s - st.h * blocks) * kRows;
      st.units = units_of(st.len);
      u0 = 0;
      u1 = st.units;
      pos = 1;
      first = 0;
      if (st.row0 >= st.count * v.g) return;
    } else {
      long long off;
      if (few) {
        st.b = __ffs(__ballot_sync(0xffffffffu, upto > pos)) - 1;
        st.count = __shfl_sync(0xffffffffu, seq_count, st.b);
        st.len = __shfl_sync(0xffffffffu, seq_len, st.b);
        const long long before = __shfl_sync(0xffffffffu, upto, max(st.b - 1, 0));
        off = pos - (st.b > 0 ? before : 0);
      } else {
        int lo = 0, hi = v.B;                    // the last sequence that begins at or before the position, and has any
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (prefix[mid] <= pos) lo = mid; else hi = mid;
        }
        while (prefix[lo + 1] <= pos) ++lo;
        st.b = lo;
        v.sequence(st.b, st.count, st.len);
        off = pos - prefix[st.b];
      }
      st.units = units_of(st.len);
      const int blocks = row_blocks(st.count, v.g, kRows), each = kAhead + st.units;
      const int s = off >> 32 ? (int)(off / each) : (int)((uint32_t)off / (uint32_t)each);
      st.h = s / blocks;
      st.row0 = (s - st.h * blocks) * kRows;
      first = pos - (off - (long long)s * each) + kAhead;     // where the stream's first unit is in the line
      u0 = (int)max(0ll, pos - first);
      u1 = (int)min((long long)st.units, end - first);
      pos = min(end, first + st.units);
      if (u1 <= u0) continue;                    // nothing but the beginning
    }
    const bool begins = u0 == 0, whole = begins && u1 == st.units;
    // tokens that the last row of the block sees: units behind them are left out
    const int last_row = min(st.row0 + kRows, st.count * v.g) - 1;
    const int most = min(st.len, max(0, st.len - st.count + over_g(last_row) + 1));
    const int u_last = min(u1, (most + kUnit - 1) / kUnit);
    const int mine = !dead && u_last > u0 + warp ? (u_last - u0 - warp + kW - 1) / kW : 0;      // units of the warp: u0 + warp + kW i

    // ---- the queries' loads, under way before the page numbers are waited for
    uint4 qw[kNT][4];
#pragma unroll
    for (int nt = 0; nt < kNT; ++nt) {
      const int row = st.row0 + 8 * nt + r;
      const bool there = row < st.count * v.g;
      const int i = over_g(row), head = row - i * v.g;
      const uint16_t* src = static_cast<const uint16_t*>(a.q) + (((size_t)st.b * v.Hq + st.h * v.g + head) * v.n + i) * kD + 8 * t;
#pragma unroll
      for (int j = 0; j < 4; ++j) qw[nt][j] = there ? *reinterpret_cast<const uint4*>(src + 32 * j) : make_uint4(0u, 0u, 0u, 0u);
    }

    // ---- copies: a lane has one of 32 of the warp's units: where it lies (and the page of its second half where a page is half a unit)
    const char* src0 = nullptr;
    int p1 = 0;
    bool gaps = false;                           // some page so far was none
    const int32_t* page_row = v.pages + (size_t)st.b * v.pages_stride;
    auto issue = [&](int i) {
      if ((i & 31) == 0) {
        const int tok = (u0 + warp + kW * (i + lane)) * kUnit;
        const bool need0 = i + lane < mine, need1 = need0 && tok + 16 < most;
        const int p0 = need0 && tok < most ? page_row[tok >> v.lg_page] : 0;
        p1 = v.lg_page == 4 ? (need1 ? page_row[(tok + 16) >> 4] : 0) : p0;
        const bool bad = p0 < 0 || p0 >= v.n_pages || p1 < 0 || p1 >= v.n_pages;
        if (bad) atomicOr(v.status, (uint32_t)MIXKVQ_DEV_BAD_PAGE);
        gaps = gaps || __any_sync(0xffffffffu, bad);
        src0 = p0 < 0 || p0 >= v.n_pages || tok >= most ? nullptr : v.pool + (uint64_t)(uint32_t)p0 * v.page_bytes + (uint64_t)st.h * v.piece_bytes + v.tile_of(tok);
        if (p1 >= v.n_pages || !need1) p1 = -1;
      }
      if (lane == (i & 31)) {
        const uint32_t at = (uint32_t)(i % stages), bar = bars + 8u * at, dst = ring + at * kUnitBytes;
        const bool ok0 = src0 != nullptr, ok1 = p1 >= 0, one = ok0 && ok1 && v.lg_page > 4;
        const uint32_t bytes = one ? 2 * kTileBytes : kTileBytes;
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar),
                     "r"(((ok0 ? 1u : 0u) + (ok1 ? 1u : 0u)) * kTileBytes + (i == 0 ? a.test_extra : 0u))
                     : "memory");
        if (ok0)
          asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src0), "r"(bytes), "r"(bar) : "memory");
        if (ok1 && !one) {
          const char* src1 = v.pool + (uint64_t)(uint32_t)p1 * v.page_bytes + (uint64_t)st.h * v.piece_bytes;
          asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst + kTileBytes), "l"(src1), "r"(kTileBytes),
                       "r"(bar)
                       : "memory");
        }
      }
    };
    int asked = min(stages, mine);               // units asked for
    for (int i = 0; i < asked; ++i) issue(i);

    // ---- queries: lane (r, t) has channels 32 j + 8 t .. + 7 of row r of every row tile as operands
    uint32_t qb[kQueriesInRegisters ? kNT : 1][4][4];                      // word j: {0,4} {2,6} {1,5}/16 {3,7}/16
    uint32_t qz[kNT][3];                         // sums of the row's groups as three bf16 terms each: {sum of group t, 0}
    float qscale[kNT][2];
    int sees[kNT][2], fewest = st.len;
#pragma unroll
    for (int nt = 0; nt < kNT; ++nt) {
      const uint4(&w)[4] = qw[nt];
      uint32_t top = 0;                          // the largest magnitude's bits (finite or not)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t x[4] = {w[j].x, w[j].y, w[j].z, w[j].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) top = max(top, max(x[k] & 0x7FFFu, x[k] >> 16 & 0x7FFFu));
      }
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      // 2^e: the largest entry to 2^14 .. 2^15 (or as near as a factor of 2^126 brings it)
      const int e = min(max(14 + 127 - (int)(top >> 7), -114), 126);
      const float up = pow2i(e);
      float part[kNG];
#pragma unroll
      for (int k = 0; k < kNG; ++k) part[k] = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t x[4] = {w[j].x, w[j].y, w[j].z, w[j].w};
        float f[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          f[2 * k] = bf_lo(x[k]);
          f[2 * k + 1] = bf_hi(x[k]);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) part[j * kNG / 4] += f[k];
        qb[nt][j][0] = pack_half2(f[0] * up, f[4] * up);
        qb[nt][j][1] = pack_half2(f[2] * up, f[6] * up);
        qb[nt][j][2] = pack_half2(f[1] * (up * 0.0625f), f[5] * (up * 0.0625f));
        qb[nt][j][3] = pack_half2(f[3] * (up * 0.0625f), f[7] * (up * 0.0625f));
        if constexpr (!kQueriesInRegisters) sts128(q_at + 512 * j, qb[nt][j][0], qb[nt][j][1], qb[nt][j][2], qb[nt][j][3]);      // (the lane's own words: no other reads them)
      }
#pragma unroll
      for (int k = 0; k < kNG; ++k) {
        part[k] += __shfl_xor_sync(0xffffffffu, part[k], 1);
        part[k] += __shfl_xor_sync(0xffffffffu, part[k], 2);
      }
      float rest = 0.f;
#pragma unroll
      for (int k = 0; k < kNG; ++k) rest = t == k ? part[k] * a.scale_log2e : rest;
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        qz[nt][k] = pack_bf162(rest, 0.f);
        rest -= bf_lo(qz[nt][k]);
      }
      // the columns of the lane's products: rows 2 t and 2 t + 1
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int from = 4 * (2 * t + c);
        // what a sum is multiplied with.  Where fp32 has no room for the 2^24 of the codes (queries from 2^117 on or so) it is left out and the sign says so: such sums
        // are brought up first, in masked units, which all units of the piece then are.  (e is -114 for rows that are not finite; their results are not either.)
        const int e_row = __shfl_sync(0xffffffffu, e, from);
        const float back = a.scale_log2e * pow2i(-e_row);
        qscale[nt][c] = back >= 0x1p103f && e_row > -114 ? -back : back * 16777216.f;
        const int x = st.row0 + 8 * nt + 2 * t + c;
        // (rows that are none are computed like the others and written nowhere)
        sees[nt][c] = x < st.count * v.g ? max(0, st.len - st.count + over_g(x) + 1) : st.len;
        if (qscale[nt][c] < 0.f) fewest = 0;
      }
    }
#pragma unroll
    for (int nt = 0; nt < kNT; ++nt) fewest = min(fewest, min(sees[nt][0], sees[nt][1]));
    fewest = __reduce_min_sync(0xffffffffu, fewest);

    WarpState<kNG, kNT> w;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int k = 0; k < 4 * kNT; ++k) w.acc[i][k] = 0.f;
#pragma unroll
    for (int i = 0; i < kNG; ++i) {
      w.factor[i] = pow2i(126);
      w.limit[i] = limit_of(126);
#pragma unroll
      for (int k = 0; k < 2 * kNT; ++k) w.zsum[i][k] = 0.f;
    }
#pragma unroll
    for (int k = 0; k < 2 * kNT; ++k) {
      w.ref[k] = 0.f;
      w.l[k] = 0.f;
    }
    bool fresh = true;                           // no reference yet: the first tile's largest logits, whatever they are

    // ---- one unit: tokens tok .. tok + 31.  there: which of its tiles of 16 tokens are
    auto unit_step = [&](uint32_t base, int tok, uint32_t there, auto masked) {
      constexpr bool kMask = decltype(masked)::value;
      // logits above the references; row r: columns 2 t, 2 t + 1, then row r + 8
      float x[2][kNT][4];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const uint32_t tile = base + m * kTileBytes;
        const uint4 k0 = lds128(tile + pi * 64 + t * 16), k1 = lds128(tile + (pi + 8) * 64 + t * 16);
        uint32_t m0[kNG], m1[kNG];
        load_meta<kNG>(tile + 2048 + pi * kMeta, m0);
        load_meta<kNG>(tile + 2048 + (pi + 8) * kMeta, m1);
        // {z, s} of the lane's group as an operand: the scales meet zeros
        const uint32_t zt = tile + 2048 + pi * kMeta + 4 * (t % kNG), z0 = lds32(zt), z1 = lds32(zt + 8 * kMeta);
        const uint32_t w0[4] = {k0.x, k0.y, k0.z, k0.w}, w1[4] = {k1.x, k1.y, k1.z, k1.w};
        float sum[kNT][4], zs[kNT][4];
#pragma unroll
        for (int nt = 0; nt < kNT; ++nt) {
          mma_bf16_k8_to(zs[nt], z0, z1, qz[nt][0], -w.ref[2 * nt], -w.ref[2 * nt + 1], -w.ref[2 * nt], -w.ref[2 * nt + 1]);
          mma_bf16_k8(zs[nt], z0, z1, qz[nt][1]);
          mma_bf16_k8(zs[nt], z0, z1, qz[nt][2]);
        }
#pragma unroll
        for (int g = 0; g < kNG; ++g) {
          float c[kNT][4];
#pragma unroll
          for (int j = g * 4 / kNG; j < (g + 1) * 4 / kNG; ++j) {
            const uint32_t h0 = w0[j] >> 8, h1 = w1[j] >> 8;
            const uint32_t e0 = w0[j] & 0x000F000Fu, e1 = w1[j] & 0x000F000Fu, e2 = h0 & 0x000F000Fu, e3 = h1 & 0x000F000Fu;
            const uint32_t o0 = w0[j] & 0x00F000F0u, o1 = w1[j] & 0x00F000F0u, o2 = h0 & 0x00F000F0u, o3 = h1 & 0x00F000F0u;
#pragma unroll
            for (int nt = 0; nt < kNT; ++nt) {
              uint4 q;
              if constexpr (kQueriesInRegisters)
                q = make_uint4(qb[nt][j][0], qb[nt][j][1], qb[nt][j][2], qb[nt][j][3]);
              else
                q = lds128(q_at + 512 * j);
              if (j == g * 4 / kNG)
                mma_f16_to(c[nt], e0, e1, e2, e3, q.x, q.y, 0.f, 0.f, 0.f, 0.f);
              else
                mma_f16(c[nt], e0, e1, e2, e3, q.x, q.y);
              mma_f16(c[nt], o0, o1, o2, o3, q.z, q.w);
            }
          }
          const float s0 = bf_hi(m0[g]), s1 = bf_hi(m1[g]);
#pragma unroll
          for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
            for (int k = 0; k < 4; ++k) sum[nt][k] = g == 0 ? (k < 2 ? s0 : s1) * c[nt][k] : fmaf(k < 2 ? s0 : s1, c[nt][k], sum[nt][k]);
        }
#pragma unroll
        for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float by = qscale[nt][k & 1];
            if constexpr (!kMask) {
              x[m][nt][k] = fmaf(sum[nt][k], by, zs[nt][k]);
            } else {
              x[m][nt][k] = fmaf(by < 0.f ? sum[nt][k] * 16777216.f : sum[nt][k], fabsf(by), zs[nt][k]);
              if (tok + 16 * m + pi + (k < 2 ? 0 : 8) >= sees[nt][k & 1] || !(there >> m & 1)) x[m][nt][k] = -INFINITY;
            }
          }
      }
      // ---- whether a reference or a factor has to move (scales are not negative: words compare like them)
      auto value_meta = [&](int m, uint32_t (&vm)[2][kNG]) {
        const uint32_t at = base + m * kTileBytes + 2048 + 16 * kMeta + pi * kMeta;
        load_meta<kNG>(at, vm[0]);
        load_meta<kNG>(at + 8 * kMeta, vm[1]);
        if constexpr (kMask) {                   // what lies behind the last token may be anything
#pragma unroll
          for (int g = 0; g < kNG; ++g) {
            if (tok + 16 * m + pi >= most || !(there >> m & 1)) vm[0][g] = 0u;
            if (tok + 16 * m + pi + 8 >= most || !(there >> m & 1)) vm[1][g] = 0u;
          }
        }
      };
      uint32_t largest[kNG];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        uint32_t vm[2][kNG];
        value_meta(m, vm);
#pragma unroll
        for (int g = 0; g < kNG; ++g) largest[g] = m == 0 ? max(vm[0][g], vm[1][g]) : max(largest[g], max(vm[0][g], vm[1][g]));
      }
      bool move = false;
#pragma unroll
      for (int g = 0; g < kNG; ++g) move = move || largest[g] > w.limit[g];
      float above = -INFINITY;
#pragma unroll
      for (int i = 0; i < 2 * kNT; ++i) {
        const float* y = x[i & 1][i >> 1];
        above = fmaxf(fmaxf(above, fmaxf(y[0], y[1])), fmaxf(y[2], y[3]));
      }
      if (__any_sync(0xffffffffu, move || fresh || above > kRise - kBelow)) {
#pragma unroll
        for (int c = 0; c < 2 * kNT; ++c) {
          const int nt = c >> 1, k = c & 1;
          float up = fmaxf(fmaxf(x[0][nt][k], x[0][nt][k + 2]), fmaxf(x[1][nt][k], x[1][nt][k + 2]));
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) up = fmaxf(up, __shfl_xor_sync(0xffffffffu, up, d));
          // (a row moves by its own logits alone: its result does not depend on the rows beside it)
          up = up > kRise - kBelow || (fresh && up > -INFINITY) ? up + kBelow : 0.f;
          const float f = ex2_approx(-up);
          w.ref[c] += up;
#pragma unroll
          for (int m = 0; m < 2; ++m) {
            x[m][nt][k] -= up;
            x[m][nt][k + 2] -= up;
          }
          w.l[c] *= f;
#pragma unroll
          for (int g = 0; g < kNG; ++g) w.zsum[g][c] *= f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            w.acc[i][4 * nt + k] *= f;
            w.acc[i][4 * nt + k + 2] *= f;
          }
        }
#pragma unroll
        for (int g = 0; g < kNG; ++g) {
          // the largest scale of the group; one that is not finite moves nothing (its products are not finite whatever the factor), and hides none of the lane's others
          uint32_t s = largest[g] & 0xFFFF0000u;
          if (s >= 0x7F800000u) {
            s = 0u;
#pragma unroll
            for (int m = 0; m < 2; ++m) {
              uint32_t vm[2][kNG];
              value_meta(m, vm);
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const uint32_t one = vm[i][g] & 0xFFFF0000u;
                s = max(s, one < 0x7F800000u ? one : 0u);
              }
            }
          }
          s = __reduce_max_sync(0xffffffffu, s);
          if (s > w.limit[g]) {
            const int e = min(max(kScaleTo + 127 - (int)(s >> 23), -122), 126);
            const float down = pow2i(e), f = down / w.factor[g];
            w.factor[g] = down;
            w.limit[g] = limit_of(e);
#pragma unroll
            for (int i = g * 8 / kNG; i < (g + 1) * 8 / kNG; ++i)
#pragma unroll
              for (int k = 0; k < 4 * kNT; ++k) w.acc[i][k] *= f;
          }
        }
        fresh = fresh && there == 0;
      }
      // ---- weights and the second product
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const uint32_t tile = base + m * kTileBytes;
        uint32_t vm[2][kNG];
        value_meta(m, vm);
        uint2 vw[4];                               // tokens of the operand's columns 2 t, 2 t + 1, 2 t + 8, 2 t + 9
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = 2 * t + (i & 1), token = (row ^ (row >> 1 & 1)) + 8 * (i >> 1);
          vw[i] = lds64(tile + 1024 + token * 64 + ((8 * r) ^ ((token & 4) << 3)));
        }
        float p[kNT][4];
#pragma unroll
        for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            p[nt][k] = ex2_approx(x[m][nt][k]);
            w.l[2 * nt + (k & 1)] += p[nt][k];
          }
#pragma unroll
        for (int g = 0; g < kNG; ++g) {
          uint32_t ub[kNT][2];
          const float sk[2] = {bf_hi(vm[0][g]) * w.factor[g], bf_hi(vm[1][g]) * w.factor[g]}, zv[2] = {bf_lo(vm[0][g]), bf_lo(vm[1][g])};
#pragma unroll
          for (int nt = 0; nt < kNT; ++nt) {
            float u[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              float pz = p[nt][k] * zv[k >> 1];
              u[k] = p[nt][k] * sk[k >> 1];
              if constexpr (kMask) {               // a row that does not see a token takes nothing of it, an infinity neither
                if (x[m][nt][k] == -INFINITY) u[k] = pz = 0.f;
              }
              w.zsum[g][2 * nt + (k & 1)] += pz;
            }
            ub[nt][0] = movmatrix_trans(pack_half2(u[0], u[1]));
            ub[nt][1] = movmatrix_trans(pack_half2(u[2], u[3]));
          }
#pragma unroll
          for (int j = g * 4 / kNG; j < (g + 1) * 4 / kNG; ++j) {
            const uint32_t sel = j & 1 ? 0x7632u : 0x5410u;
            const uint32_t ab = __byte_perm(j < 2 ? vw[0].x : vw[0].y, j < 2 ? vw[1].x : vw[1].y, sel);
            const uint32_t cd = __byte_perm(j < 2 ? vw[2].x : vw[2].y, j < 2 ? vw[3].x : vw[3].y, sel);
            const uint32_t ab8 = ab >> 8, cd8 = cd >> 8;
#pragma unroll
            for (int nt = 0; nt < kNT; ++nt) {
              mma_f16(reinterpret_cast<float(&)[4]>(w.acc[2 * j][4 * nt]), ab & 0x000F000Fu, ab8 & 0x000F000Fu, cd & 0x000F000Fu, cd8 & 0x000F000Fu, ub[nt][0], ub[nt][1]);
              mma_f16(reinterpret_cast<float(&)[4]>(w.acc[2 * j + 1][4 * nt]), ab & 0x00F000F0u, ab8 & 0x00F000F0u, cd & 0x00F000F0u, cd8 & 0x00F000F0u, ub[nt][0], ub[nt][1]);
            }
          }
        }
      }
    };
    int done = 0;                                // units waited for
    for (; done < mine; ++done) {
      const int stage = done % stages, tok = (u0 + warp + kW * done) * kUnit;
      uint32_t there = tok + 16 < most ? 3u : 1u;
      if (gaps) {
        const int q0 = page_row[tok >> v.lg_page], q1 = there == 3u ? page_row[(tok + 16) >> v.lg_page] : -1;
        there = (q0 >= 0 && q0 < v.n_pages ? 1u : 0u) | (q1 >= 0 && q1 < v.n_pages ? 2u : 0u);
      }
      wait(bars + 8u * stage, phase >> stage & 1u);
      if (dead) break;
      phase ^= 1u << stage;
      const uint32_t base = ring + (uint32_t)(stage * kUnitBytes);
      if (tok + kUnit > fewest || there != 3u) {
        unit_step(base, tok, there, std::true_type{});
      } else {
        unit_step(base, tok, 3u, std::false_type{});
      }
      __syncwarp();
      if (asked < mine) issue(asked++);
    }
    if (dead) {
      // what is under way is waited for, and the piece is left without this warp's part
      for (int i = done; i < asked; ++i) {
        const int stage = i % stages;
        wait(bars + 8u * stage, phase >> stage & 1u);
      }
#pragma unroll
      for (int k = 0; k < 2 * kNT; ++k) {
        w.l[k] = 0.f;
#pragma unroll
        for (int g = 0; g < kNG; ++g) w.zsum[g][k] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) w.acc[i][4 * (k >> 1) + (k & 1)] = w.acc[i][4 * (k >> 1) + (k & 1) + 2] = 0.f;
      }
    }

    // ---- the warp's sums into its ring: [rows][132] floats: o[128], reference, denominator
#pragma unroll
    for (int k = 0; k < 2 * kNT; ++k) {
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) {
        w.l[k] += __shfl_xor_sync(0xffffffffu, w.l[k], d);
#pragma unroll
        for (int g = 0; g < kNG; ++g) w.zsum[g][k] += __shfl_xor_sync(0xffffffffu, w.zsum[g][k], d);
      }
      if (w.l[k] == 0.f) w.ref[k] = -1e30f;      // nothing seen
    }
    constexpr int kStride = kD + 4;
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 2 * kNT; ++c) {
      const int nt = c >> 1, k = c & 1, row = 8 * nt + 2 * t + k;
      const uint32_t at = ring + (uint32_t)row * (kStride * 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int g = j * kNG / 4;
        const float back = pow2i(127 - (int)(__float_as_uint(w.factor[g]) >> 23)), z = w.zsum[g][c];
        const float y0 = fmaf(w.acc[2 * j][4 * nt + k] * 16777216.f, back, z), y2 = fmaf(w.acc[2 * j][4 * nt + k + 2] * 16777216.f, back, z);
        const float y1 = fmaf(w.acc[2 * j + 1][4 * nt + k] * 1048576.f, back, z), y3 = fmaf(w.acc[2 * j + 1][4 * nt + k + 2] * 1048576.f, back, z);
        sts128(at + (32 * j + 4 * r) * 4, __float_as_uint(y0), __float_as_uint(y1), __float_as_uint(y2), __float_as_uint(y3));
      }
      if (r == 0) sts64(at + kD * 4, __float_as_uint(w.ref[c]), __float_as_uint(w.l[c]));
    }
    __syncthreads();
    // ---- the warps' sums together: a warp per row, a lane four channels
    const uint32_t base0 = smem_u32(smem);
    for (int row = warp; row < kRows; row += kW) {
      const int x = st.row0 + row;
      if (x >= st.count * v.g) break;
      float m[kW], l[kW], top = -1e30f;
#pragma unroll
      for (int i = 0; i < kW; ++i) {
        const uint2 ml = lds64(base0 + (uint32_t)(i * stages * kUnitBytes + (row * kStride + kD) * 4));
        m[i] = __uint_as_float(ml.x);
        l[i] = __uint_as_float(ml.y);
        top = fmaxf(top, m[i]);
      }
      float y[4] = {0.f, 0.f, 0.f, 0.f}, sum = 0.f;
#pragma unroll
      for (int i = 0; i < kW; ++i) {
        const float f = ex2_approx(m[i] - top);
        const uint4 o = lds128(base0 + (uint32_t)(i * stages * kUnitBytes + (row * kStride + 4 * lane) * 4));
        sum = fmaf(l[i], f, sum);
        y[0] = fmaf(__uint_as_float(o.x), f, y[0]);
        y[1] = fmaf(__uint_as_float(o.y), f, y[1]);
        y[2] = fmaf(__uint_as_float(o.z), f, y[2]);
        y[3] = fmaf(__uint_as_float(o.w), f, y[3]);
      }
      if (whole) {
        const int i = over_g(x), head = x - i * v.g;
        const size_t at = (((size_t)st.b * v.Hq + st.h * v.g + head) * v.n + i) * kD + 4 * lane;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        if (a.out_bf16)
          *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + at) = make_uint2(pack_bf162(y[0] * inv, y[1] * inv), pack_bf162(y[2] * inv, y[3] * inv));
        else
          *reinterpret_cast<float4*>(static_cast<float*>(a.out) + at) = make_float4(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
      } else {
        float* to = plan.parts + ((size_t)(2 * blockIdx.x + (begins ? 1 : 0)) * kRows + row) * kPartFloats;
        *reinterpret_cast<float4*>(to + 4 * lane) = make_float4(y[0], y[1], y[2], y[3]);
        if (lane == 0) *reinterpret_cast<float2*>(to + kD) = make_float2(top, sum);
      }
    }
    if (begins && !whole && tid == 0) {
      // the thread block whose range has the stream's last unit: the last one that begins at or before it
      const long long u = first + st.units - 1;
      int c = min(parts - 1, (int)((double)u * parts / (double)total));
      while (c > 0 && cut(total, parts, c) > u) --c;
      while (c + 1 < parts && cut(total, parts, c + 1) <= u) ++c;
      plan.broken[blockIdx.x] = Broken{c, st.row0, min(kRows, st.count * v.g - st.row0), 0, ((long long)st.b * v.Hq + st.h * v.g) * v.n, 0};
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // the rings take copies again
    __syncthreads();
  }
}

// Joins the pieces of the stream that begins in thread block blockIdx.x of pages_kernel and ends in another.  Eight warps share the rows, or where there are few the rows and
// their pieces; a lane has four channels, and the weight of one of 32 pieces at a time.
__global__ void __launch_bounds__(256)
merge_kernel(const __grid_constant__ PagedAttention a, const __grid_constant__ Plan plan) {
  dependency_wait();
  const Broken it = plan.broken[blockIdx.x];
  const int c0 = blockIdx.x, c1 = it.last;
  if (c1 <= c0) return;
  const PagedView& v = a.view;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int share = it.rows <= 1 ? 8 : it.rows <= 2 ? 4 : it.rows <= 4 ? 2 : 1;          // warps of a row
  const int mine = warp % share;
  const size_t stride = (size_t)2 * plan.rows * kPartFloats;                 // from a thread block's first piece to the next one's
  __shared__ float join[8][kD + 4];
  for (int row = warp / share; row < it.rows; row += 8 / share) {            // (one round where a row has several warps)
    const float* from = plan.parts + (size_t)row * kPartFloats;
    float m = -1e30f, l = 0.f, y[4] = {0.f, 0.f, 0.f, 0.f};
    for (int c = c0 + 32 * mine; c <= c1; c += 32 * share) {
      const int n = min(32, c1 - c + 1);
      // a thread block's second piece is the one that begins its stream
      auto piece = [&](int k) { return from + (c + k) * stride + (c + k == c0 ? stride / 2 : 0); };
      float4 o[12];
#pragma unroll
      for (int i = 0; i < 12; ++i) o[i] = *reinterpret_cast<const float4*>(piece(min(i, n - 1)) + 4 * lane);
      float2 ml = *reinterpret_cast<const float2*>(piece(min(lane, n - 1)) + kD);
      if (lane >= n) ml = make_float2(-1e30f, 0.f);
      float top = ml.x;
#pragma unroll
      for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
      top = fmaxf(top, m);
      const float old = ex2_approx(m - top), w = ex2_approx(ml.x - top);
      float sum = ml.y * w;
#pragma unroll
      for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      m = top;
      l = fmaf(l, old, sum);
#pragma unroll
      for (int k = 0; k < 4; ++k) y[k] *= old;
      for (int i0 = 0; i0 < n; i0 += 12) {
#pragma unroll
        for (int i = 0; i < 12; ++i) {
          const float f = __shfl_sync(0xffffffffu, w, i0 + i);
          if (i0 + i < n) {
            y[0] = fmaf(o[i].x, f, y[0]);
            y[1] = fmaf(o[i].y, f, y[1]);
            y[2] = fmaf(o[i].z, f, y[2]);
            y[3] = fmaf(o[i].w, f, y[3]);
          }
        }
        if (i0 + 12 < n) {
#pragma unroll
          for (int i = 0; i < 12; ++i) o[i] = *reinterpret_cast<const float4*>(piece(min(i0 + 12 + i, n - 1)) + 4 * lane);
        }
      }
    }
    if (share > 1) {
      *reinterpret_cast<float4*>(&join[warp][4 * lane]) = make_float4(y[0], y[1], y[2], y[3]);
      if (lane == 0) *reinterpret_cast<float2*>(&join[warp][kD]) = make_float2(m, l);
      asm volatile("bar.sync %0, %1;" ::"r"(1 + warp / share), "r"(32 * share) : "memory");      // the row's warps
      if (mine != 0) return;
      for (int i = 1; i < share; ++i) {
        const float m1 = join[warp + i][kD], l1 = join[warp + i][kD + 1], top = fmaxf(m, m1), f0 = ex2_approx(m - top), f1 = ex2_approx(m1 - top);
        m = top;
        l = l * f0 + l1 * f1;
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] = y[k] * f0 + join[warp + i][4 * lane + k] * f1;
      }
    }
    const int x = it.row0 + row, i = over_heads(plan, x), head = x - i * v.g;
    const size_t at = ((size_t)it.out + (size_t)head * v.n + i) * kD + 4 * lane;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (a.out_bf16)
      *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + at) = make_uint2(pack_bf162(y[0] * inv, y[1] * inv), pack_bf162(y[2] * inv, y[3] * inv));
    else
      *reinterpret_cast<float4*>(static_cast<float*>(a.out) + at) = make_float4(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
  }
}

// Capacity up to which a thread block has a stream to itself.  7b shape, us direct / in pieces: 1 x 100 tokens 6.1 / 7.4, 8 x 500 7.8 / 9.7, 64 x 500 15.3 / 18.7; at a capacity of 1024
// 1 x 1000 10.1 / 8.6, 64 x 1000 20.0 / 23.2 (and the longest sequence decides).
constexpr int kDirectTokens = 512;
// Query rows of a KV head above which unpacking the pages pays: kUnpackRows, and more where there is little to unpack (kUnpackWork / tokens of all KV heads), as its three
// launches take longer than two.  By what the pages could hold, the lengths being unknown here (and by the largest count): measured with page tables as wide as the sequences are long,
// so under a much wider one short sequences are unpacked from fewer rows on than pays.  7b shape, us with the pages as they are / unpacked: 8 x 32768 tokens 63 rows 214 / 248,
// 98 rows 355 / 250; 8 x 8192 63 rows 69 / 84, 98 rows 107 / 85; 1 x 32768 98 rows 59 / 61, 126 rows 65 / 61; 1 x 8192 189 rows 35 / 45, 448 rows 62 / 49; 8 x 1024 63 rows 25 / 29,
// 252 rows 58 / 42; 1 x 1024 448 rows 23 / 34, 896 rows 34 / 36.
constexpr int kUnpackRows = 72;
constexpr double kUnpackWork = 5e6;
constexpr int kMostBlocks = 148 * 4;             // thread blocks of the split kernel: sizes the workspace

using Kernel = void (*)(PagedAttention, Plan);
template <int kNT, int kW>
Kernel kernel_for(int G) {
  return G == 32 ? pages_kernel<32, kNT, kW> : G == 64 ? pages_kernel<64, kNT, kW> : pages_kernel<128, kNT, kW>;
}
// Short streams of 8 query rows: sixteen warps, a unit or two each.  (16 rows need the registers of four warps.)
constexpr int kDirectWarps = 16;
Kernel kernel_of(int G, int tiles, bool direct) { return tiles == 1 ? (direct ? kernel_for<1, kDirectWarps>(G) : kernel_for<1, kWarps>(G)) : kernel_for<2, kWarps>(G); }
int warps_of(int tiles, bool direct) { return tiles == 1 && direct ? kDirectWarps : kWarps; }
int tiles_of(int g, int n) { return g * n <= 8 ? 1 : 2; }
size_t smem_bytes(int G, int tiles, int B, bool direct) {
  const int warps = warps_of(tiles, direct);
  return (size_t)warps * (kStages * tiles * 2 * paged_tile_bytes(G) + (tiles == 1 ? kQueryBytes : 0)) + 8 * warps * kStages * tiles + (direct || B <= 32 ? 0 : 8 * (size_t)(B + 1));
}

}  // namespace

// Whether a call goes to the kernel that unpacks the pages once for all query rows.
static bool unpacks(int Hkv, int g, int batch, int n, long long capacity) {
  return (double)g * n > kUnpackRows + kUnpackWork / ((double)batch * Hkv * capacity) && capacity <= paged_chunk_capacity();
}

static size_t pieces_bytes(int g, int n) { return (size_t)2 * kMostBlocks * 8 * tiles_of(g, n) * kPartFloats * 4 + kMostBlocks * sizeof(Broken); }
size_t paged_workspace_need(int Hkv, int g, int batch, int n, long long capacity) {
  return unpacks(Hkv, g, batch, n, capacity) ? paged_chunk_workspace_need(Hkv, batch, capacity) : pieces_bytes(g, n);
}
// (a capacity beyond what is unpacked counts as the largest that is: a narrower page table may need that)
size_t paged_workspace_bytes(int Hkv, int g, int batch, int n, long long capacity) {
  const long long most = std::min(capacity, paged_chunk_capacity());
  return unpacks(Hkv, g, batch, n, most) ? std::max(paged_chunk_workspace_bytes(Hkv, batch, most), pieces_bytes(g, n)) : pieces_bytes(g, n);
}

cudaError_t paged_attention_setup() {
  for (int G = 32; G <= 128; G *= 2)
    for (int k = 0; k < 3; ++k) {
      const int tiles = k == 2 ? 2 : 1;
      const bool direct = k == 1;
      const cudaError_t e = cudaFuncSetAttribute(kernel_of(G, tiles, direct), cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                 (int)smem_bytes(G, tiles, MIXKVQ_PAGED_MAX_BATCH, direct));
      if (e != cudaSuccess) return e;
    }
  return paged_chunk_setup();
}

cudaError_t launch_paged_attention(const PagedAttention& a, int n_sms, cudaStream_t stream, int* launches, int* form) {
  const PagedView& v = a.view;
  *launches = 0;
  if (unpacks(v.Hkv, v.g, v.B, v.n, (long long)v.max_pages << v.lg_page)) {
    *form = MIXKVQ_PAGED_UNPACKED;
    return launch_paged_chunk(a, n_sms, stream, launches);
  }
  const int tiles = tiles_of(v.g, v.n);
  Plan plan{};
  plan.rows = 8 * tiles;
  plan.parts = a.parts;
  const int most = std::min(kMostBlocks, n_sms * (tiles == 1 ? 3 : 2));
  plan.broken = reinterpret_cast<Broken*>(a.parts + (size_t)2 * kMostBlocks * plan.rows * kPartFloats);
  plan.g_inv = v.g == 1 ? 0u : (uint32_t)(((1ull << 32) + v.g - 1) / v.g);
  // Sequences whose pages hold few tokens at most: a thread block each, no merge.
  const long long streams = (long long)v.B * v.Hkv * ((v.n * (long long)v.g + plan.rows - 1) / plan.rows);
  plan.direct = ((long long)v.max_pages << v.lg_page) <= kDirectTokens;
  const int warps = warps_of(tiles, plan.direct);
  cudaError_t e = launch_dependent(kernel_of(v.G, tiles, plan.direct), dim3((unsigned)(plan.direct ? streams : most)), warps * 32, smem_bytes(v.G, tiles, v.B, plan.direct), stream,
                                   a, plan);
  *form = plan.direct ? MIXKVQ_PAGED_DIRECT : MIXKVQ_PAGED_PIECES;
  *launches = 1;
  if (e != cudaSuccess || plan.direct) return e;
  *launches = 2;
  return launch_dependent(merge_kernel, dim3((unsigned)most), 256, 0, stream, a, plan);
}

}  // namespace mixkvq
