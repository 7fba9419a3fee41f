// Rotary position embedding of the keys and queries of an append, in place (Appendix D: importance scores and keys
// are taken after the rotation, so every caller rotates right before it appends).
//
// (The arithmetic is rotate_chunk in common.cuh; a fused decode step rotates in the split kernel instead.)
//
// rope_axes_kernel rotates with several coordinates per token (time, height, width): channel pair i of a row takes its angle from the table row of the
// coordinate that the pair belongs to.  Memory-bound: every row is read and written once.  What could cost more is the table: with interleaved axes the
// 64 pairs of a token come from up to four rows, one scalar at a time, so a thread block takes up to 16 neighbouring tokens of a sequence, gathers their 64
// cosines and sines into shared memory once and turns all query and key heads with them; the values are copied beside.  Consecutive rows of a block are
// consecutive tokens of one head: the stores are one contiguous piece per head whatever the layout of the input.
#include "common.cuh"

namespace mixkvq {

namespace {

// rows: the B * Hkv * n key rows, then the B * Hq * n query rows; token index of a row = row % n.
// One thread rotates eight pairs of one row: channels 8c .. 8c+7 and 64 + 8c .. 64 + 8c+7.
__global__ void __launch_bounds__(256)
rope_kernel(__nv_bfloat16* __restrict__ k, __nv_bfloat16* __restrict__ q, const float* __restrict__ cos_t,
            const float* __restrict__ sin_t, long long k_rows, long long rows, int n_tokens, int pos0) {
  dependency_wait();
  const long long idx = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  const long long row = idx >> 3;
  const int c = (int)(idx & 7);
  if (row >= rows) return;
  __nv_bfloat16* x = (row < k_rows ? k + row * kD : q + (row - k_rows) * kD) + 8 * c;
  const int pos = pos0 + (int)(row % n_tokens);
  const float *cos_row = cos_t + (size_t)pos * 64, *sin_row = sin_t + (size_t)pos * 64;
  const uint4 lo = *reinterpret_cast<const uint4*>(x), hi = *reinterpret_cast<const uint4*>(x + 64);
  *reinterpret_cast<uint4*>(x) = rotate_chunk(lo, hi, cos_row, sin_row, c);
  *reinterpret_cast<uint4*>(x + 64) = rotate_chunk(hi, lo, cos_row, sin_row, c + 8);
}

__global__ void __launch_bounds__(256)
rope_axes_kernel(const __grid_constant__ RopeAxes a, int lg_tokens, int blocks_per_seq) {
  extern __shared__ __align__(16) float table[];                       // [tokens][64] cosines, then sines, then [tokens] whether the token is turned
  dependency_wait();
  const int T = 1 << lg_tokens, tid = threadIdx.x;
  const int b = blockIdx.x / blocks_per_seq, t0 = (blockIdx.x - b * blocks_per_seq) << lg_tokens, nt = min(T, a.n - t0);
  float *cosS = table, *sinS = table + T * 64;
  int* turnS = reinterpret_cast<int*>(table + T * 128);
  const int32_t* pos = a.positions + (size_t)b * a.n + t0;
  const size_t axis_stride = (size_t)a.B * a.n;
  if (tid < nt) {
    int turn = 1;
    for (int x = 0; x < a.n_axes; ++x)
      if (a.used >> x & 1) {
        const int p = pos[x * axis_stride + tid];
        if (p < 0) turn = 0;                                           // no token
        if (p >= a.n_positions) {
          turn = 0;
          atomicOr(a.status, (uint32_t)MIXKVQ_DEV_BAD_POSITION);
        }
      }
    turnS[tid] = turn;
  }
  for (int i = tid; i < nt * 64; i += 256) {
    const int t = i >> 6, pair = i & 63, p = pos[a.axis_of_pair[pair] * axis_stride + t];
    const bool in = p >= 0 && p < a.n_positions;
    cosS[i] = in ? a.cos_t[(size_t)p * 64 + pair] : 0.f;
    sinS[i] = in ? a.sin_t[(size_t)p * 64 + pair] : 0.f;
  }
  __syncthreads();
  // item: 8 channel pairs (channels 8 c .. and 64 + 8 c ..) of a row, for the values 8 channels twice
  const int rows = (a.Hq + 2 * a.Hkv) << lg_tokens, last = (a.v != nullptr ? rows : (a.Hq + a.Hkv) << lg_tokens) * 8;
#pragma unroll 2
  for (int i = tid; i < last; i += 256) {
    const int row = i >> 3, c = i & 7, t = row & (T - 1), head = row >> lg_tokens;
    if (t >= nt || !turnS[t]) continue;
    const int which = head < a.Hq ? 0 : head < a.Hq + a.Hkv ? 1 : 2, h = which == 0 ? head : which == 1 ? head - a.Hq : head - a.Hq - a.Hkv;
    const RopeTensor& x = which == 0 ? a.tq : which == 1 ? a.tk : a.tv;
    const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(which == 0 ? a.q : which == 1 ? a.k : a.v) + b * x.batch + h * x.head + (t0 + t) * x.token + 8 * c;
    __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(which == 0 ? a.q_out : which == 1 ? a.k_out : a.v_out) +
                         (((size_t)b * (which == 0 ? a.Hq : a.Hkv) + h) * a.n + t0 + t) * kD + 8 * c;
    uint4 lo = *reinterpret_cast<const uint4*>(src), hi = *reinterpret_cast<const uint4*>(src + 64);
    if (which < 2) {
      const uint4 y = rotate_chunk(lo, hi, cosS + t * 64, sinS + t * 64, c);
      hi = rotate_chunk(hi, lo, cosS + t * 64, sinS + t * 64, c + 8);
      lo = y;
    }
    *reinterpret_cast<uint4*>(dst) = lo;
    *reinterpret_cast<uint4*>(dst + 64) = hi;
  }
}

}  // namespace

cudaError_t launch_rope_axes(const RopeAxes& a, int n_sms, cudaStream_t stream) {
  // 16 tokens per thread block, fewer as long as an SM has room for more of them than it gets: eight at a time.  (With two per SM as the aim: one prompt of
  // 4000 tokens, 7b shape, 19.0 us and 16.9; 4 of 777, 8b shape, 16.8 and 16.0.  Loads of two or four pieces together gained at some sizes and lost at others.)
  int lg = 4;
  while (lg > 0 && (long long)a.B * ((a.n + (1 << lg) - 1) >> lg) < 8 * n_sms) --lg;
  const int blocks = (a.n + (1 << lg) - 1) >> lg;
  return launch_dependent(rope_axes_kernel, dim3((unsigned)(a.B * blocks)), 256, ((size_t)129 * 4) << lg, stream, a, lg, blocks);
}

cudaError_t launch_rope(void* k, void* q, const float* cos_t, const float* sin_t, int B, int Hkv, int Hq, int n_tokens,
                        int pos0, cudaStream_t stream) {
  const long long k_rows = (long long)B * Hkv * n_tokens, rows = k_rows + (long long)B * Hq * n_tokens;
  const long long threads = rows * 8;
  return launch_dependent(rope_kernel, dim3((unsigned)((threads + 255) / 256)), 256, 0, stream, static_cast<__nv_bfloat16*>(k),
                          static_cast<__nv_bfloat16*>(q), cos_t, sin_t, k_rows, rows, n_tokens, pos0);
}

}  // namespace mixkvq
