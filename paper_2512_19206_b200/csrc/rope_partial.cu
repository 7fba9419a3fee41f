// Rotary positions of a part of the head in either pairing, and the tables of scaled frequencies that they turn by.
//
// rope_partial_kernel: channels 0 .. d-1 of a row turn by the row of the token's position, the others are copied; pairs (i, i + d/2) or (2 i, 2 i + 1).
// Memory-bound: every row is read and written once.  Eight lanes have a token's rows, a lane 8 pairs; it keeps their cosines and sines in registers while it goes through a
// range of heads, so that the tables are read once per token and range instead of once per row, and no lane needs another's channels.  Ranges are halved until there are sixteen thread
// blocks per SM: 16004 tokens of 56 rows take 74.8 us (0.95 of the rate of a copy), with four per SM 77.4, with one 87, as the last wave is then a large part of the whole.
//
// rope_tables_kernel: cos and sin of p f_i.  Angles of far positions need more than 32 bits (p f of 10^5 rad leaves 2^-7 of a turn in fp32), so they are 64-bit, in
// half turns, which are reduced exactly.  A 64-bit sine and cosine per entry would cost more than writing them; a thread has one pair and some neighbouring
// positions, computes the first and turns it from one to the next by a complex product: 4 operations, and an error of 2^-52 a step where the entry has 24 bits.
// Neighbours: as many as leave an SM 1024 threads, 32 at most.  131072 positions of 64 pairs take 13.8 us (floor 10.4, the bytes written), 72 with one position a thread.
#include <algorithm>

#include "paged.cuh"

namespace mixkvq {

namespace {

constexpr int kTokens = 32;                                // of a thread block
constexpr int kBatch = 4;                                  // rows in flight per thread

__global__ void __launch_bounds__(256)
rope_partial_kernel(const __grid_constant__ RopePartial a, int heads_per_block) {
  dependency_wait();
  const long long tok = (long long)blockIdx.x * kTokens + (threadIdx.x >> 3);
  if (tok >= (long long)a.B * a.n) return;
  const int pos = a.turn.positions[tok];
  if (pos >= a.turn.n_positions) atomicOr(a.status, (uint32_t)MIXKVQ_DEV_BAD_POSITION);
  if (pos < 0 || pos >= a.turn.n_positions) return;
  const int b = (int)(tok / a.n), t = (int)(tok - (long long)b * a.n);
  const PairLane p = pair_lane(a.turn, pos, threadIdx.x & 7, true);
  const int heads = a.Hq + a.Hkv + (a.v != nullptr ? a.Hkv : 0);
  const int h0 = blockIdx.y * heads_per_block, h1 = min(h0 + heads_per_block, heads);
  for (int h = h0; h < h1; h += kBatch) {
    uint4 w[kBatch][2];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int hh = min(h + i, h1 - 1);
      const int which = hh < a.Hq ? 0 : hh < a.Hq + a.Hkv ? 1 : 2, head = which == 0 ? hh : which == 1 ? hh - a.Hq : hh - a.Hq - a.Hkv;
      const RopeTensor& s = which == 0 ? a.tq : which == 1 ? a.tk : a.tv;
      const uint4* src = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(which == 0 ? a.q : which == 1 ? a.k : a.v) + b * s.batch + head * s.head + t * s.token);
      w[i][0] = src[p.first];
      w[i][1] = src[p.second];
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int hh = h + i;
      if (hh >= h1) break;
      const int which = hh < a.Hq ? 0 : hh < a.Hq + a.Hkv ? 1 : 2, head = which == 0 ? hh : which == 1 ? hh - a.Hq : hh - a.Hq - a.Hkv;
      if (which != 2) turn_pair(w[i][0], w[i][1], p, F2{a.turn.minus_zero});
      uint4* dst = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(which == 0 ? a.q_out : which == 1 ? a.k_out : a.v_out) +
                                            (((size_t)b * (which == 0 ? a.Hq : a.Hkv) + head) * a.n + t) * kD);
      dst[p.first] = w[i][0];
      dst[p.second] = w[i][1];
    }
  }
}

__global__ void __launch_bounds__(256)
rope_tables_kernel(const __grid_constant__ RopeTables a, int run) {
  dependency_wait();
  const long long idx = (long long)blockIdx.x * 256 + threadIdx.x;
  const long long first = idx / a.half * run;
  const int pair = (int)(idx % a.half);
  if (first >= a.n) return;
  const int last = (int)min((long long)a.n, first + run);
  const double f = a.turns[pair];
  double s, c, ds, dc;
  sincospi((double)(a.start + first) * f, &s, &c);
  sincospi(f, &ds, &dc);
  for (int p = (int)first; p < last; ++p) {
    a.cos_t[(size_t)p * a.half + pair] = (float)(c * a.factor);
    a.sin_t[(size_t)p * a.half + pair] = (float)(s * a.factor);
    const double next = fma(c, dc, -s * ds);
    s = fma(s, dc, c * ds);
    c = next;
  }
}

}  // namespace

cudaError_t launch_rope_partial(const RopePartial& a, int n_sms, cudaStream_t stream) {
  const long long blocks = ((long long)a.B * a.n + kTokens - 1) / kTokens;
  const int heads = a.Hq + a.Hkv + (a.v != nullptr ? a.Hkv : 0);
  int each = heads;
  while (each > 1 && blocks * ((heads + each - 1) / each) < 16 * n_sms) each = (each + 1) / 2;
  return launch_dependent(rope_partial_kernel, dim3((unsigned)blocks, (unsigned)((heads + each - 1) / each)), 256, 0, stream, a, each);
}

cudaError_t launch_rope_tables(const RopeTables& a, int n_sms, cudaStream_t stream) {
  const long long entries = (long long)a.n * a.half;
  const int run = (int)std::max(1ll, std::min(32ll, entries / (n_sms * 1024ll)));
  const long long threads = (a.n + run - 1) / run * a.half;
  return launch_dependent(rope_tables_kernel, dim3((unsigned)((threads + 255) / 256)), 256, 0, stream, a, run);
}

}  // namespace mixkvq
