// What keeps a paged cache short: the attention weight each key received, and
// the eviction of the keys that received least.
#include "half_mfma.h"
#include "kernels.h"

namespace brisk {

namespace {

// ---------------------------------------------------------------------------
// score'_j = decay score_j + sum_rows exp(scale <q, k_j> - lse_row)
//
// S = Q K^T with a key a lane: the sum over rows is a sum over a lane's
// registers and its partner in the other half, in a fixed order.  A wavefront
// keeps KT tiles of 32 keys in registers and passes over the rows of the
// sequence's group (L x heads of the group), which the workgroup stages 64 at
// a time in LDS, so each key is read from memory once.
// ---------------------------------------------------------------------------
constexpr int kScoreWaves = 4, kScoreRows = 64, kKeyTiles = 2;
constexpr int kScoreKeys = kScoreWaves * kKeyTiles * 32;  // of a workgroup

template <bool F16, int ND>
__global__ __launch_bounds__(64 * kScoreWaves) void score_kernel(ScoreArgs a, int runs) {
  constexpr int RB = ND > 2 ? 256 : 128, NC = 2 * ND, CH = RB / 16;
  __shared__ __attribute__((aligned(16))) uint8_t s_q[kScoreRows * RB];
  __shared__ __attribute__((aligned(16))) float s_lse[kScoreRows];  // times log2 e; +inf: the row adds nothing
  __shared__ uint64_t s_word[kScoreRows];
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int bh = blockIdx.x / runs, b = bh / a.Hkv, hk = bh % a.Hkv, G = a.H / a.Hkv;
  const int first = blockIdx.x % runs * kScoreKeys + wave * (kKeyTiles * 32);
  const int n = kv_len(a.kv, b, min(a.cap, a.kv.max_pages << a.kv.page_shift));
  const int64_t at = static_cast<int64_t>(bh) * a.cap;
  if (blockIdx.x % runs * kScoreKeys >= n) {  // the whole workgroup is past the sequence
    for (int j = first + lane; j < min(a.cap, first + kKeyTiles * 32); j += 64) a.score_out[at + j] = 0.f;
    return;
  }
  const int base = n - a.L;
  const float c = a.scale * kLog2e;

  uint4 k[kKeyTiles][NC];
#pragma unroll
  for (int t = 0; t < kKeyTiles; ++t) {
    const int j = first + t * 32 + col;
    const uint16_t* src = a.kv.k + kv_slot(a.kv, b, min(j, n - 1)) + hk * a.kv.head_stride;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int e = 16 * i + 8 * half;
      k[t][i] = j < n && e < a.D ? *reinterpret_cast<const uint4*>(src + e) : make_uint4(0, 0, 0, 0);
    }
  }
  float sum[kKeyTiles] = {};
  const int rows = a.L * G;
  for (int r0 = 0; r0 < rows; r0 += kScoreRows) {
    __syncthreads();
    for (int x = tid; x < kScoreRows * CH; x += 64 * kScoreWaves) {
      const int r = x / CH, e = x % CH * 8, row = r0 + r;
      const int64_t bi = static_cast<int64_t>(b) * a.L + row / G;
      const bool on = row < rows && e < a.D;
      *reinterpret_cast<uint4*>(s_q + r * RB + (((e / 8) ^ row_swizzle<RB>(r)) << 4)) =
          on ? *reinterpret_cast<const uint4*>(a.q + bi * a.q_row_stride + (hk * G + row % G) * a.q_head_stride + e)
             : make_uint4(0, 0, 0, 0);
    }
    if (tid < kScoreRows) {
      const int row = r0 + tid;
      const int64_t bi = static_cast<int64_t>(b) * a.L + row / G;
      const float z = row < rows ? a.lse[bi * a.H + hk * G + row % G] : -INFINITY;
      s_lse[tid] = z == -INFINITY ? INFINITY : z * kLog2e;
      s_word[tid] = row < rows && a.mask ? a.mask[bi] : ~0ull;
    }
    __syncthreads();
#pragma unroll
    for (int q0 = 0; q0 < kScoreRows; q0 += 32) {
      if (r0 + q0 >= rows) break;
      floatx16 s[kKeyTiles];
#pragma unroll
      for (int t = 0; t < kKeyTiles; ++t) s[t] = floatx16{};
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const int r = q0 + col;
        const uint4 q = *reinterpret_cast<const uint4*>(s_q + r * RB + (((2 * i + half) ^ row_swizzle<RB>(r)) << 4));
#pragma unroll
        for (int t = 0; t < kKeyTiles; ++t) s[t] = mfma32<F16>(q, k[t][i], s[t]);
      }
      const bool block = a.mask && first + kKeyTiles * 32 > base;
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const int row = q0 + 8 * (r / 4) + 4 * half;
        const float4 z4 = *reinterpret_cast<const float4*>(s_lse + row);
        const float z[4] = {z4.x, z4.y, z4.z, z4.w};
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int t = 0; t < kKeyTiles; ++t) {
            float p = __builtin_amdgcn_exp2f(fmaf(s[t][r + x], c, -z[x]));
            bool off = z[x] == INFINITY;
            if (block) {
              const int place = first + t * 32 + col - base;
              off |= place >= 0 && !block_sees(s_word[row + x], place);
            }
            sum[t] += off ? 0.f : p;
          }
      }
    }
  }
#pragma unroll
  for (int t = 0; t < kKeyTiles; ++t) {
    const float x = swap32_sum(sum[t]);
    const int j = first + t * 32 + col;
    if (half == 0 && j < a.cap) a.score_out[at + j] = j < n ? a.decay * a.score_in[at + j] + x : 0.f;
  }
}

// ---------------------------------------------------------------------------
// Eviction.  One workgroup a (sequence, head) finds the budget-th largest key
// by three histogram passes (11 + 11 + 10 bits), then lists the kept slots at
// or above the budget and the evicted ones below it, both ascending; a second
// launch moves the rows.
// ---------------------------------------------------------------------------
// Slots in the order of eviction's choice as unsigned integers: the latest
// tokens first, then larger scores; NaN lowest, -0 as +0.
__device__ __forceinline__ uint32_t keep_key(float score, bool late) {
  if (late) return 0xFFFFFFFFu;
  if (score != score) return 0u;
  const uint32_t u = __float_as_uint(score + 0.0f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / kWave, kBins = 2048;
constexpr int kLdsSlots = 32768;  // keys of a workgroup that fit in LDS beside the histogram

// IN_LDS: the keys of a sequence are computed once and held in LDS; longer
// sequences compute them anew from scores and positions in each pass.
template <bool IN_LDS>
__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(EvictArgs a) {
  extern __shared__ uint32_t s_keys[];
  __shared__ uint32_t s_hist[kBins];
  __shared__ uint32_t s_wave[2][kSelectWaves];
  __shared__ uint32_t s_digit, s_left;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int b = blockIdx.x / a.Hkv, n = kv_len(a.kv, b, min(a.cap, a.kv.max_pages << a.kv.page_shift));
  const int m = min(n, a.budget);
  const int64_t at = static_cast<int64_t>(blockIdx.x) * a.cap;
  const float* const score = a.score_in + at;
  const int32_t* const pos = a.pos_in + at;
  const int from = a.next_pos[b] - a.recent;
  if (tid == 0 && blockIdx.x % a.Hkv == 0) a.new_len[b] = m;
  auto compute = [&](int j) { return keep_key(score[j], pos[j] >= from); };
  for (int j = tid; j < a.cap; j += kSelectThreads) {
    const float s = j < n ? score[j] : 0.f;
    const int x = j < n ? pos[j] : -1;
    if constexpr (IN_LDS)
      if (j < n) s_keys[j] = keep_key(s, x >= from);
    a.score_out[at + j] = j < m ? s : 0.f;
    a.pos_out[at + j] = j < m ? x : -1;
  }
  if (n <= m) {
    if (tid == 0) a.count[blockIdx.x] = 0;
    return;
  }
  auto key_of = [&](int j) {
    if constexpr (IN_LDS)
      return s_keys[j];
    else
      return compute(j);
  };
  // ---- the m-th largest key: `found` holds its leading bits, `left` how many of the
  // keys that share them are still to be taken
  uint32_t found = 0, left = m;
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
    for (int i = tid; i < kBins; i += kSelectThreads) s_hist[i] = 0;
    __syncthreads();
    for (int j0 = 0; j0 < n; j0 += kSelectThreads * 4) {
      uint32_t key[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int j = j0 + u * kSelectThreads + tid;
        key[u] = j < n ? key_of(j) : 0;
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int j = j0 + u * kSelectThreads + tid;
        const bool in = j < n && (pass == 0 || (key[u] >> (shift + bits)) == found);
        const uint32_t digit = (key[u] >> shift) & ((1u << bits) - 1);
        // equal digits of a whole wavefront (scores that are all alike) are added at once
        const uint64_t active = __ballot(in);
        if (!active) continue;
        const uint32_t one = __builtin_amdgcn_readlane(digit, __builtin_ctzll(active));
        if (__ballot(in && digit == one) == active) {
          if (lane == 0) atomicAdd(&s_hist[one], static_cast<uint32_t>(__popcll(active)));
        } else if (in) {
          atomicAdd(&s_hist[digit], 1u);
        }
      }
    }
    __syncthreads();
    // the bin where the count from above reaches `left`: each thread sums two bins
    // (descending), wavefronts scan, then the one bin that crosses writes
    const int hi = kBins - 1 - 2 * tid;
    const uint32_t c0 = s_hist[hi], c1 = s_hist[hi - 1];
    uint32_t run = c0 + c1;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const uint32_t o = __shfl_up(run, off, kWave);
      if (lane >= off) run += o;
    }
    if (lane == 63) s_wave[0][wave] = run;
    __syncthreads();
    uint32_t before = run - c0 - c1;
    for (int w = 0; w < wave; ++w) before += s_wave[0][w];
    if (before < left && before + c0 >= left) {
      s_digit = hi;
      s_left = left - before;
    } else if (before + c0 < left && before + c0 + c1 >= left) {
      s_digit = hi - 1;
      s_left = left - before - c0;
    }
    __syncthreads();
    found = (found << bits) | s_digit;
    left = s_left;
    __syncthreads();
  }
  // ---- the first half of the wavefronts take [0, m), the others [m, n), each a run of slots
  constexpr int kHalf = kSelectWaves / 2;
  const int w = wave % kHalf, lo = wave < kHalf ? 0 : m, len = wave < kHalf ? m : n - m;
  const int per = (len + kHalf * kWave - 1) / (kHalf * kWave) * kWave;
  const int j0 = min(lo + w * per, lo + len), j1 = min(j0 + per, lo + len);
  uint32_t above = 0, ties = 0;
  for (int j = j0; j < j1; j += kWave * 4) {
    uint32_t key[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) key[u] = j + u * kWave + lane < j1 ? key_of(j + u * kWave + lane) : 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const bool in = j + u * kWave + lane < j1;
      above += __popcll(__ballot(in && key[u] > found));
      ties += __popcll(__ballot(in && key[u] == found));
    }
  }
  if (lane == 0) {
    s_wave[0][wave] = above;
    s_wave[1][wave] = ties;
  }
  __syncthreads();
  uint32_t tie = 0, rank = 0;  // ties, and listed slots of this half, in the runs before
  for (int x = 0; x < wave; ++x) {
    const uint32_t taken = min(s_wave[1][x], left > tie ? left - tie : 0u);
    if (x / kHalf == wave / kHalf) {
      const int l0 = x < kHalf ? 0 : m, ln = x < kHalf ? m : n - m;
      const int a0 = min(l0 + x % kHalf * per, l0 + ln), a1 = min(a0 + per, l0 + ln);
      const uint32_t kept = s_wave[0][x] + taken;
      rank += x < kHalf ? (a1 - a0) - kept : kept;
    }
    tie += s_wave[1][x];
  }
  int32_t* const list = (wave < kHalf ? a.dst : a.src) + static_cast<int64_t>(blockIdx.x) * a.list_len;
  const uint64_t below = (1ull << lane) - 1;
  for (int j = j0; j < j1; j += kWave * 4) {
    uint32_t key[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) key[u] = j + u * kWave + lane < j1 ? key_of(j + u * kWave + lane) : 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int x = j + u * kWave + lane;
      const bool in = x < j1;
      const uint64_t same = __ballot(in && key[u] == found);
      const bool kept = key[u] > found || (key[u] == found && tie + __popcll(same & below) < left);
      const uint64_t listed = __ballot(in && kept == (wave >= kHalf));
      if (in && kept == (wave >= kHalf)) list[rank + __popcll(listed & below)] = x;
      tie += __popcll(same);
      rank += __popcll(listed);
    }
  }
  if (wave == kSelectWaves - 1 && lane == 0) a.count[blockIdx.x] = rank;
}

// Moves listed rows, 16 lanes a row and kRowsInFlight rows at once.
constexpr int kRowsInFlight = 4, kMoveRows = 16 * kRowsInFlight;
__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a, int runs) {
  const int bh = blockIdx.x / runs, r0 = blockIdx.x % runs * kMoveRows;
  const int count = a.count[bh];
  if (r0 >= count) return;
  const int b = bh / a.Hkv, hk = bh % a.Hkv;
  const int64_t at = static_cast<int64_t>(bh) * a.cap, list = static_cast<int64_t>(bh) * a.list_len;
  const int lane = threadIdx.x & 15, e = min(lane * 8, a.D - 8);  // narrow heads: the last lanes repeat a chunk
  int src[kRowsInFlight], dst[kRowsInFlight];
#pragma unroll
  for (int u = 0; u < kRowsInFlight; ++u) {
    const int r = min(r0 + u * 16 + static_cast<int>(threadIdx.x >> 4), count - 1);  // past the end: the last row again
    src[u] = a.src[list + r];
    dst[u] = a.dst[list + r];
  }
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  u32x4 k[kRowsInFlight], v[kRowsInFlight];
  int64_t to[kRowsInFlight];
#pragma unroll
  for (int u = 0; u < kRowsInFlight; ++u) {
    const int64_t from = kv_slot(a.kv, b, src[u]) + hk * a.kv.head_stride + e;
    to[u] = kv_slot(a.kv, b, dst[u]) + hk * a.kv.head_stride + e;
    k[u] = *reinterpret_cast<const u32x4*>(a.k + from);
    v[u] = *reinterpret_cast<const u32x4*>(a.v + from);
  }
#pragma unroll
  for (int u = 0; u < kRowsInFlight; ++u) {
    *reinterpret_cast<u32x4*>(a.k + to[u]) = k[u];
    *reinterpret_cast<u32x4*>(a.v + to[u]) = v[u];
    if (lane == 0) {
      a.score_out[at + dst[u]] = a.score_in[at + src[u]];
      a.pos_out[at + dst[u]] = a.pos_in[at + src[u]];
    }
  }
}

template <bool F16>
void launch_score(const ScoreArgs& a, hipStream_t s) {
  const int runs = (a.cap + kScoreKeys - 1) / kScoreKeys;
  const dim3 grid(static_cast<uint32_t>(a.B) * a.Hkv * runs), threads(64 * kScoreWaves);
  if (a.D <= 64)
    hipLaunchKernelGGL((score_kernel<F16, 2>), grid, threads, 0, s, a, runs);
  else if (a.D <= 96)
    hipLaunchKernelGGL((score_kernel<F16, 3>), grid, threads, 0, s, a, runs);
  else
    hipLaunchKernelGGL((score_kernel<F16, 4>), grid, threads, 0, s, a, runs);
}

}  // namespace

void launch_cache_score(const ScoreArgs& a, bool f16, hipStream_t s) {
  if (f16)
    launch_score<true>(a, s);
  else
    launch_score<false>(a, s);
}

int evict_list_len(int cap, int budget) { return cap > budget ? (budget < cap - budget ? budget : cap - budget) : 0; }

// Workspace: a count for each (sequence, head), then the lists of sources and
// targets, at most min(budget, cap - budget) entries each.
size_t evict_workspace_bytes(int B, int Hkv, int cap, int budget) {
  const size_t heads = static_cast<size_t>(B) * Hkv, len = evict_list_len(cap, budget);
  return ((heads + 3) / 4 * 4 + 2 * heads * len) * sizeof(int32_t);
}

void launch_cache_evict(EvictArgs a, void* ws, hipStream_t s) {
  const size_t heads = static_cast<size_t>(a.B) * a.Hkv;
  a.list_len = evict_list_len(a.cap, a.budget);
  a.count = static_cast<int32_t*>(ws);
  a.src = a.count + (heads + 3) / 4 * 4;
  a.dst = a.src + heads * a.list_len;
  if (a.cap <= kLdsSlots)
    hipLaunchKernelGGL(evict_select_kernel<true>, dim3(heads), dim3(kSelectThreads), a.cap * sizeof(uint32_t), s, a);
  else
    hipLaunchKernelGGL(evict_select_kernel<false>, dim3(heads), dim3(kSelectThreads), 0, s, a);
  if (a.list_len > 0) {
    const int runs = (a.list_len + kMoveRows - 1) / kMoveRows;
    hipLaunchKernelGGL(evict_move_kernel, dim3(heads * runs), dim3(256), 0, s, a, runs);
  }
}

}  // namespace brisk
