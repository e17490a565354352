// What keeps a paged cache short: the attention weight each key received, and
// the eviction of the keys that received least.
#include "kernels.h"
#include "kv_common.h"

namespace brisk {

namespace {

// One wavefront a slot: the products with every row of the group, one row at
// a time, in a fixed order.
template <bool F16>
__global__ __launch_bounds__(256) void score_kernel(ScoreArgs a) {
  const int lane = threadIdx.x & 63, j = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int b = blockIdx.y / a.Hkv, hk = blockIdx.y % a.Hkv, G = a.H / a.Hkv;
  if (j >= a.cap) return;
  const int64_t at = static_cast<int64_t>(blockIdx.y) * a.cap + j;
  const int n = kv_len(a.kv, b, min(a.cap, a.kv.max_pages << a.kv.page_shift)), t = j - (n - a.L);
  if (j >= n) {
    if (lane == 0) a.score_out[at] = 0.f;
    return;
  }
  const uint16_t* k = a.kv.k + kv_slot(a.kv, b, j) + hk * a.kv.head_stride;
  const int e0 = lane * 2;
  const bool on = e0 < a.D;
  const float k0 = on ? half_to_f32<F16>(k[e0]) : 0.f, k1 = on ? half_to_f32<F16>(k[e0 + 1]) : 0.f;
  float sum = 0.f;
  for (int i = 0; i < a.L; ++i) {
    const int64_t bi = static_cast<int64_t>(b) * a.L + i;
    if (t >= 0 && a.mask && !block_sees(a.mask[bi], t)) continue;
    for (int g = 0; g < G; ++g) {
      const int h = hk * G + g;
      const uint16_t* q = a.q + bi * a.q_row_stride + h * a.q_head_stride;
      const float lse = a.lse[bi * a.H + h];
      const float s = a.scale * wave_sum(on ? k0 * half_to_f32<F16>(q[e0]) + k1 * half_to_f32<F16>(q[e0 + 1]) : 0.f);
      if (lse != -INFINITY) sum += __expf(s - lse);
    }
  }
  if (lane == 0) a.score_out[at] = a.decay * a.score_in[at] + sum;
}

// Slots in the order of eviction's choice as unsigned integers: the latest
// tokens first, then larger scores; NaN lowest, -0 as +0.
__device__ __forceinline__ uint32_t keep_key(float score, bool late) {
  if (late) return 0xFFFFFFFFu;
  if (score != score) return 0u;
  const uint32_t u = __float_as_uint(score + 0.0f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// One workgroup a (sequence, head): every slot counts the slots chosen before it.
__global__ __launch_bounds__(256) void evict_select_kernel(EvictArgs a) {
  __shared__ int s_src, s_dst;
  const int b = blockIdx.x / a.Hkv, n = kv_len(a.kv, b, min(a.cap, a.kv.max_pages << a.kv.page_shift));
  const int64_t at = static_cast<int64_t>(blockIdx.x) * a.cap;
  const int m = min(n, a.budget);
  if (threadIdx.x == 0 && blockIdx.x % a.Hkv == 0) a.new_len[b] = m;
  for (int j = threadIdx.x; j < a.cap; j += 256) {
    a.score_out[at + j] = j < m ? a.score_in[at + j] : 0.f;
    a.pos_out[at + j] = j < m ? a.pos_in[at + j] : -1;
  }
  if (threadIdx.x == 0) s_src = s_dst = 0;
  __syncthreads();
  if (n <= m) {
    if (threadIdx.x == 0) a.count[blockIdx.x] = 0;
    return;
  }
  const int from = a.next_pos[b] - a.recent;
  const int64_t list = static_cast<int64_t>(blockIdx.x) * a.list_len;
  for (int j0 = 0; j0 < n; j0 += 256) {
    const int j = j0 + threadIdx.x;
    int before = 0;
    if (j < n) {
      const uint32_t key = keep_key(a.score_in[at + j], a.pos_in[at + j] >= from);
      for (int o = 0; o < n; ++o) {
        const uint32_t other = keep_key(a.score_in[at + o], a.pos_in[at + o] >= from);
        before += other > key || (other == key && o < j);
      }
    }
    for (int t = 0; t < 256; ++t) {  // in the slots' order
      if (t == static_cast<int>(threadIdx.x) && j < n) {
        const bool kept = before < m;
        if (kept && j >= m) a.src[list + s_src++] = j;
        if (!kept && j < m) a.dst[list + s_dst++] = j;
      }
      __syncthreads();
    }
  }
  if (threadIdx.x == 0) a.count[blockIdx.x] = s_src;
}

__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a) {
  const int b = blockIdx.y / a.Hkv, hk = blockIdx.y % a.Hkv;
  const int64_t at = static_cast<int64_t>(blockIdx.y) * a.cap, list = static_cast<int64_t>(blockIdx.y) * a.list_len;
  const int lane = threadIdx.x & 15;
  for (int r = blockIdx.x * 16 + (threadIdx.x >> 4); r < a.count[blockIdx.y]; r += gridDim.x * 16) {
    const int src = a.src[list + r], dst = a.dst[list + r];
    const int64_t from = kv_slot(a.kv, b, src) + hk * a.kv.head_stride, to = kv_slot(a.kv, b, dst) + hk * a.kv.head_stride;
    if (lane * 8 < a.D) {
      *reinterpret_cast<uint4*>(a.k + to + lane * 8) = *reinterpret_cast<const uint4*>(a.k + from + lane * 8);
      *reinterpret_cast<uint4*>(a.v + to + lane * 8) = *reinterpret_cast<const uint4*>(a.v + from + lane * 8);
    }
    if (lane == 0) {
      a.score_out[at + dst] = a.score_in[at + src];
      a.pos_out[at + dst] = a.pos_in[at + src];
    }
  }
}

}  // namespace

void launch_cache_score(const ScoreArgs& a, bool f16, hipStream_t s) {
  const dim3 grid((a.cap + 3) / 4, a.B * a.Hkv);
  if (f16)
    hipLaunchKernelGGL(score_kernel<true>, grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(score_kernel<false>, grid, dim3(256), 0, s, a);
}

// Workspace: a count for each (sequence, head), then the lists of sources and
// targets, at most min(budget, cap - budget) entries each.
size_t evict_workspace_bytes(int B, int Hkv, int cap, int budget) {
  const size_t heads = static_cast<size_t>(B) * Hkv, len = evict_list_len(cap, budget);
  return ((heads + 3) / 4 * 4 + 2 * heads * len) * sizeof(int32_t);
}

int evict_list_len(int cap, int budget) { return max(0, min(budget, cap - budget)); }

void launch_cache_evict(EvictArgs a, void* ws, hipStream_t s) {
  const size_t heads = static_cast<size_t>(a.B) * a.Hkv;
  a.list_len = evict_list_len(a.cap, a.budget);
  a.count = static_cast<int32_t*>(ws);
  a.src = a.count + (heads + 3) / 4 * 4;
  a.dst = a.src + heads * a.list_len;
  hipLaunchKernelGGL(evict_select_kernel, dim3(heads), dim3(256), 0, s, a);
  if (a.list_len > 0) hipLaunchKernelGGL(evict_move_kernel, dim3((a.list_len + 63) / 64, heads), dim3(256), 0, s, a);
}

}  // namespace brisk
