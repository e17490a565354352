// Verification of drafted tokens against given probabilities (Section 3.3:
// accept with probability min{1, p / pi}; after a rejection draw from the
// positive part of p - pi).
//
// With Exp(1) variates e_v, argmax_v w_v / e_v follows the law w / sum w, so
// one pass over the row draws without normalising or ordering it.  The ratios
// are compared as candidate keys (ratio descending, id ascending), whose
// maximum does not depend on how the row is split.
//
// Bound by the read of three fp32 rows a block (12 V bytes); a lone block by
// latency: the gathers of the accept test, then the rows, then the merge.
#include "kernels.h"
#include "kv_common.h"

namespace brisk {

namespace {

constexpr int kThreads = 256;
constexpr uint64_t kNothing = 0;      // no positive weight seen
constexpr uint64_t kUndrawable = 1;   // a positive weight, but no positive ratio; below every ratio's key

struct Law {
  const float *p, *q, *e;  // q null: w = p
};

__device__ __forceinline__ void consider(uint64_t& best, float& floor, float p, float q, float e, int v) {
  const float w = p - q;
  // A division only where the ratio can reach the lane's best (2^-20 covers the rounding of the product).
  if (!(w > 0.f) || w < floor * e) return;
  const float r = w / e;
  const uint64_t key = r > 0.f ? make_key(r, v) : kUndrawable;
  if (key > best) {
    best = key;
    floor = r > 0.f ? r * (1.f - 0x1p-20f) : 0.f;
  }
}

// This thread's best of tokens [v0, v1).  Rows may start anywhere, so the
// 16-byte loads are only 4-byte aligned.
__device__ __forceinline__ uint64_t best_of(const Law& law, int v0, int v1) {
  typedef float float4u __attribute__((ext_vector_type(4), aligned(4)));
  uint64_t best = kNothing;
  float floor = 0.f;
  const int whole = v0 + (v1 - v0) / (4 * kThreads) * (4 * kThreads);
  int v = v0 + threadIdx.x * 4;
#pragma unroll 2
  for (; v < whole; v += 4 * kThreads) {
    const float4u p = *reinterpret_cast<const float4u*>(law.p + v), e = *reinterpret_cast<const float4u*>(law.e + v);
    const float4u q = law.q ? *reinterpret_cast<const float4u*>(law.q + v) : float4u{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) consider(best, floor, p[i], q[i], e[i], v + i);
  }
  for (v = whole + threadIdx.x; v < v1; v += kThreads)
    consider(best, floor, law.p[v], law.q ? law.q[v] : 0.f, law.e[v], v);
  return best;
}

__device__ __forceinline__ uint64_t workgroup_max(uint64_t x, uint64_t* s_key) {
  x = wave_max_u64(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s_key[threadIdx.x >> 6] = x;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / kWave; ++w) x = s_key[w] > x ? s_key[w] : x;
  return x;
}

// Positions accepted by block b, in every thread.
__device__ __forceinline__ int accepted(const DraftArgs& a, int b, int n, int* s_first) {
  if (threadIdx.x == 0) *s_first = n;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const int64_t r = static_cast<int64_t>(b) * a.L + i;
    const int x = clamp_id(a.tok[r], a.V);
    const float q = a.draft[r * a.draft_stride + x];
    const float p = a.target[(static_cast<int64_t>(b) * (a.L + 1) + i) * a.target_stride + x];
    if (!(a.u[r] * q < p)) atomicMin(s_first, i);
  }
  __syncthreads();
  return *s_first;
}

__device__ __forceinline__ Law law_of(const DraftArgs& a, int b, int acc, int n) {
  return {a.target + (static_cast<int64_t>(b) * (a.L + 1) + acc) * a.target_stride,
          acc < n ? a.draft + (static_cast<int64_t>(b) * a.L + acc) * a.draft_stride : nullptr,
          a.noise + static_cast<int64_t>(b) * a.noise_stride};
}

__device__ __forceinline__ void finish(const DraftArgs& a, int b, int acc, uint64_t best, Law law, uint64_t* s_key) {
  if (best == kNothing && law.q) {  // the difference is positive nowhere: draw from the target itself
    law.q = nullptr;
    best = workgroup_max(best_of(law, 0, a.V), s_key);
  }
  if (threadIdx.x == 0) {
    a.accept_len[b] = acc;
    a.token[b] = best > kUndrawable ? key_id(best) : -1;
  }
}

// One workgroup a share of a block's row (the accept test is repeated by each
// of them: at most 16 bytes a position); a block of one share ends here.
__global__ __launch_bounds__(kThreads) void draft_share_kernel(DraftArgs a, int shares, int share, uint64_t* keys) {
  __shared__ int s_first;
  __shared__ uint64_t s_key[kThreads / kWave];
  const int b = blockIdx.x / shares, s = blockIdx.x % shares;
  const int n = a.draft_len ? min(max(a.draft_len[b], 0), a.L) : a.L;
  const int acc = accepted(a, b, n, &s_first);
  const Law law = law_of(a, b, acc, n);
  const uint64_t best = workgroup_max(best_of(law, s * share, min(a.V, (s + 1) * share)), s_key);
  if (shares == 1)
    finish(a, b, acc, best, law, s_key);
  else if (threadIdx.x == 0)
    keys[blockIdx.x] = best;
}

__global__ __launch_bounds__(kThreads) void draft_merge_kernel(DraftArgs a, int shares, const uint64_t* keys) {
  __shared__ int s_first;
  __shared__ uint64_t s_key[kThreads / kWave];
  const int b = blockIdx.x;
  uint64_t best = kNothing;
  for (int s = threadIdx.x; s < shares; s += kThreads) {
    const uint64_t k = keys[static_cast<int64_t>(b) * shares + s];
    best = k > best ? k : best;
  }
  const int n = a.draft_len ? min(max(a.draft_len[b], 0), a.L) : a.L;
  const int acc = accepted(a, b, n, &s_first);
  best = workgroup_max(best, s_key);
  finish(a, b, acc, best, law_of(a, b, acc, n), s_key);
}

// Shares of a row: enough workgroups for the whole GPU (about eight a CU),
// none below 1024 tokens.
struct Shares { int count, tokens; };
Shares shares_of(int B, int V) {
  const int want = B >= 2048 ? 1 : (2048 + B - 1) / B, most = (V + 1023) / 1024;
  const int count = want < most ? want : most;
  const int tokens = ((V + count - 1) / count + 1023) / 1024 * 1024;
  return {(V + tokens - 1) / tokens, tokens};
}

}  // namespace

size_t draft_verify_workspace_bytes(int B, int V) {
  const Shares s = shares_of(B, V);
  return s.count > 1 ? static_cast<size_t>(B) * s.count * sizeof(uint64_t) : 0;
}

void launch_draft_verify(const DraftArgs& a, void* ws, hipStream_t s) {
  const Shares sh = shares_of(a.B, a.V);
  uint64_t* keys = static_cast<uint64_t*>(ws);
  hipLaunchKernelGGL(draft_share_kernel, dim3(a.B * sh.count), dim3(kThreads), 0, s, a, sh.count, sh.tokens, keys);
  if (sh.count > 1) hipLaunchKernelGGL(draft_merge_kernel, dim3(a.B), dim3(kThreads), 0, s, a, sh.count, keys);
}

}  // namespace brisk
