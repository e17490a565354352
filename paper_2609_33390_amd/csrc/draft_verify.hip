// Verification of drafted tokens against given probabilities (Section 3.3:
// accept with probability min{1, p / pi}; after a rejection draw from the
// positive part of p - pi).
//
// With Exp(1) variates e_v, argmax_v w_v / e_v follows the law w / sum w, so
// one pass over the row draws without normalising or ordering it.
#include "kernels.h"
#include "kv_common.h"

namespace brisk {

namespace {

// One workgroup a block.
__global__ __launch_bounds__(256) void draft_verify_kernel(DraftArgs a) {
  __shared__ int s_a;
  __shared__ uint64_t s_key[2][4];
  __shared__ int s_any[4];
  const int b = blockIdx.x, tid = threadIdx.x;
  const int n = a.draft_len ? min(max(a.draft_len[b], 0), a.L) : a.L;
  if (tid == 0) s_a = n;
  __syncthreads();
  for (int i = tid; i < n; i += 256) {
    const int64_t r = static_cast<int64_t>(b) * a.L + i;
    const int x = clamp_id(a.tok[r], a.V);
    const float q = a.draft[r * a.draft_stride + x];
    const float p = a.target[(static_cast<int64_t>(b) * (a.L + 1) + i) * a.target_stride + x];
    if (!(a.u[r] * q < p)) atomicMin(&s_a, i);
  }
  __syncthreads();
  const int acc = s_a;
  const float* p = a.target + (static_cast<int64_t>(b) * (a.L + 1) + acc) * a.target_stride;
  const float* q = acc < n ? a.draft + (static_cast<int64_t>(b) * a.L + acc) * a.draft_stride : nullptr;
  const float* e = a.noise + b * a.noise_stride;
  uint64_t best = 0, all = 0;  // 0: nothing drawn
  bool any = false;            // whether the difference is positive somewhere
  for (int v = tid; v < a.V; v += 256) {
    const float pv = p[v], w = q ? pv - q[v] : pv;
    any |= w > 0.f;
    if (w > 0.f && w / e[v] > 0.f) best = max(best, make_key(w / e[v], v));
    if (pv > 0.f && pv / e[v] > 0.f) all = max(all, make_key(pv / e[v], v));
  }
  any = __ballot(any) != 0;
  best = wave_max_u64(best);
  all = wave_max_u64(all);
  if ((tid & 63) == 0) {
    s_key[0][tid >> 6] = best;
    s_key[1][tid >> 6] = all;
    s_any[tid >> 6] = any;
  }
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < 4; ++w) {
      best = max(best, s_key[0][w]);
      all = max(all, s_key[1][w]);
      any |= s_any[w] != 0;
    }
    if (!any) best = all;
    a.accept_len[b] = acc;
    a.token[b] = best ? key_id(best) : -1;
  }
}

}  // namespace

size_t draft_verify_workspace_bytes(int B, int V) { return 0; }

void launch_draft_verify(const DraftArgs& a, void* ws, hipStream_t s) {
  hipLaunchKernelGGL(draft_verify_kernel, dim3(a.B), dim3(256), 0, s, a);
}

}  // namespace brisk
