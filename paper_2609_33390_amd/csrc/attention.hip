// Attention of a block over a shared prefix and a paged cache (Section 2.1:
// one model evaluation verifies and proposes all positions of a block).
//
//   s_j = scale <q, k_j>,  m = max_j s_j,  l = sum_j exp(s_j - m)
//   out = sum_j exp(s_j - m) v_j / l,  lse = m + log l
#include "kernels.h"
#include "kv_common.h"

namespace brisk {

namespace {

// One workgroup a row: each wavefront takes every fourth key, a lane two
// elements of it, and the four running maxima and sums are joined at the end.
template <bool F16>
__global__ __launch_bounds__(256) void attention_kernel(AttentionArgs a) {
  __shared__ float s_m[4], s_l[4], s_o[4][128];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row = blockIdx.x;
  const int h = static_cast<int>(row % a.H), bi = static_cast<int>(row / a.H), b = bi / a.L;
  const int hk = h / (a.H / a.Hkv), n = kv_len(a.kv, b, a.max_seq_len), base = n - a.L;
  const uint64_t mask = a.mask ? a.mask[bi] : ~0ull;
  const uint16_t* q = a.q + bi * a.q_row_stride + h * a.q_head_stride;
  const int e0 = lane * 2;
  const bool on = e0 < a.D;
  const float q0 = on ? half_to_f32<F16>(q[e0]) : 0.f, q1 = on ? half_to_f32<F16>(q[e0 + 1]) : 0.f;
  float m = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f;
  for (int64_t j = wave; j < static_cast<int64_t>(a.prefix_len) + n; j += 4) {
    const uint16_t *k, *v;
    if (j < a.prefix_len) {
      const int64_t at = j * a.pre_slot_stride + hk * a.pre_head_stride;
      k = a.pre_k + at;
      v = a.pre_v + at;
    } else {
      const int s = static_cast<int>(j - a.prefix_len);
      if (s >= base && !block_sees(mask, s - base)) continue;
      const int64_t at = kv_slot(a.kv, b, s) + hk * a.kv.head_stride;
      k = a.kv.k + at;
      v = a.kv.v + at;
    }
    const float s = a.scale * wave_sum(on ? q0 * half_to_f32<F16>(k[e0]) + q1 * half_to_f32<F16>(k[e0 + 1]) : 0.f);
    const float M = fmaxf(m, s);
    if (M == -INFINITY) continue;
    const float keep = __expf(m - M), p = __expf(s - M);
    l = l * keep + p;
    o0 = o0 * keep + (on ? p * half_to_f32<F16>(v[e0]) : 0.f);
    o1 = o1 * keep + (on ? p * half_to_f32<F16>(v[e0 + 1]) : 0.f);
    m = M;
  }
  if (lane == 0) {
    s_m[wave] = m;
    s_l[wave] = l;
  }
  s_o[wave][e0] = o0;
  s_o[wave][e0 + 1] = o1;
  __syncthreads();
  if (wave != 0) return;
  const float M = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
  float L = 0.f, a0 = 0.f, a1 = 0.f;
  for (int w = 0; w < 4 && M > -INFINITY; ++w) {
    const float f = __expf(s_m[w] - M);
    L += f * s_l[w];
    a0 += f * s_o[w][e0];
    a1 += f * s_o[w][e0 + 1];
  }
  if (on) {
    uint16_t* out = a.out + row * a.D;
    out[e0] = f32_to_half<F16>(M > -INFINITY ? a0 / L : 0.f);
    out[e0 + 1] = f32_to_half<F16>(M > -INFINITY ? a1 / L : 0.f);
  }
  if (lane == 0 && a.lse) a.lse[row] = M > -INFINITY ? M + __logf(L) : -INFINITY;
}

}  // namespace

size_t attention_workspace_bytes(int B, int L, int H, int Hkv, int D, int prefix_len, int max_seq_len) { return 0; }

void launch_attention(const AttentionArgs& a, bool f16, void* ws, hipStream_t s) {
  const dim3 grid(a.B * a.L * a.H);
  if (f16)
    hipLaunchKernelGGL(attention_kernel<true>, grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(attention_kernel<false>, grid, dim3(256), 0, s, a);
}

}  // namespace brisk
