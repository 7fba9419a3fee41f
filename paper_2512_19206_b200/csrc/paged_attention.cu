// Attention of the newest tokens of every sequence over the pages of the 4-bit cache.
//
// The plain form: a thread block per query row, a warp goes through every fourth token, a lane has four channels.
#include <algorithm>

#include "paged.cuh"

namespace mixkvq {

namespace {

__global__ void __launch_bounds__(128)
row_kernel(const __grid_constant__ PagedAttention a) {
  dependency_wait();
  const PagedView& v = a.view;
  const int i = blockIdx.x % v.n, hq = blockIdx.x / v.n % v.Hq, b = blockIdx.x / v.n / v.Hq;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, h = hq / v.g, G = v.G;
  const int count = v.count(b), len = v.length(b, v.add_counts ? count : 0);
  if (i >= count) return;
  const int sees = min(len, len - count + i + 1);
  const size_t at = (((size_t)b * v.Hq + hq) * v.n + i) * kD + 4 * lane;
  const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(a.q) + at);
  const float q[4] = {bf16_half(w.x, 0), bf16_half(w.x, 1), bf16_half(w.y, 0), bf16_half(w.y, 1)};
  float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  const int c = 4 * lane;                                   // the lane's channels
  for (int t = warp; t < sees; t += 4) {
    const char* tile = v.piece(b, h, t);
    if (tile == nullptr) continue;
    tile += v.tile_of(t);
    const int row = t & 15;
    const uint32_t kc = *reinterpret_cast<const uint16_t*>(tile + row * 64 + 16 * ((c >> 3) & 3) + 4 * (c >> 5) + ((c & 7) >> 1));
    const uint32_t vc = *reinterpret_cast<const uint16_t*>(tile + 1024 + row * 64 + ((8 * ((c & 31) >> 2) + 2 * (c >> 5)) ^ ((row & 4) << 3)));
    const uint32_t km = *reinterpret_cast<const uint32_t*>(tile + paged_k_meta(row, G) + 4 * (c / G)), vm = *reinterpret_cast<const uint32_t*>(tile + paged_v_meta(row, G) + 4 * (c / G));
    float x = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) x = fmaf(q[k], fmaf((float)(kc >> (4 * k) & 15u), bf16_half(km, 0), bf16_half(km, 1)), x);
#pragma unroll
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    x *= a.scale_log2e;
    const float top = fmaxf(m, x), f = m == -INFINITY ? 0.f : exp2f(m - top), p = exp2f(x - top);
    l = l * f + p;
#pragma unroll
    for (int k = 0; k < 4; ++k) o[k] = o[k] * f + p * fmaf((float)(vc >> (4 * k) & 15u), bf16_half(vm, 0), bf16_half(vm, 1));
    m = top;
  }
  __shared__ float part[4][kD + 2];
  if (lane == 0) {
    part[warp][kD] = m;
    part[warp][kD + 1] = l;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) part[warp][c + k] = o[k];
  __syncthreads();
  if (warp == 0) {
    float top = -INFINITY, sum = 0.f, y[4] = {0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < 4; ++k) top = fmaxf(top, part[k][kD]);
    for (int k = 0; k < 4; ++k) {
      const float f = part[k][kD + 1] == 0.f ? 0.f : exp2f(part[k][kD] - top);
      sum += f * part[k][kD + 1];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] += f * part[k][c + e];
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    if (a.out_bf16)
      *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + at) = make_uint2(bf16_pair(y[0] * inv, y[1] * inv), bf16_pair(y[2] * inv, y[3] * inv));
    else
      *reinterpret_cast<float4*>(static_cast<float*>(a.out) + at) = make_float4(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
  }
}

}  // namespace

size_t paged_workspace_bytes(int, int, int, int) { return 256; }
cudaError_t paged_attention_setup() { return cudaSuccess; }

cudaError_t launch_paged_attention(const PagedAttention& a, int, cudaStream_t stream, int* launches) {
  *launches = 1;
  return launch_dependent(row_kernel, dim3((unsigned)((long long)a.view.B * a.view.Hq * a.view.n)), 128, 0, stream, a);
}

}  // namespace mixkvq
