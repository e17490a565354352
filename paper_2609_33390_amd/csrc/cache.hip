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
// holds 64 rows of the sequence's group (L x heads of the group) in registers
// and passes over its run of 32-key tiles, copied to LDS one tile ahead; groups
// of more than 64 rows pass over the run again, whose keys then come from the
// L2, and add to what the passes before left.  No wavefront waits for another.
// ---------------------------------------------------------------------------
constexpr int kScoreWaves = 4, kMaxTiles = 8;

// QT: 32-row tiles of queries in registers.
template <bool F16, int ND, int QT>
__global__ __launch_bounds__(64 * kScoreWaves) void score_kernel(ScoreArgs a, int tiles) {
  constexpr int RB = ND > 2 ? 256 : 128, NC = 2 * ND, kTile = 32 * RB, NI = kTile / 1024, RPI = 1024 / RB;
  constexpr int kScoreRows = 32 * QT;
  __shared__ __attribute__((aligned(1024))) uint8_t s_keys[kScoreWaves][2][kTile];
  __shared__ __attribute__((aligned(16))) float s_lse[kScoreWaves][kScoreRows];  // times log2 e; +inf: adds nothing
  __shared__ uint64_t s_word[kScoreWaves][kScoreRows];
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // first runs of all sequences, then second ones, ...: the runs past the shorter
  // sequences then spread over the XCDs
  const int heads = a.B * a.Hkv, bh = blockIdx.x % heads, b = bh / a.Hkv, hk = bh % a.Hkv, G = a.H / a.Hkv;
  const int first = (blockIdx.x / heads * kScoreWaves + wave) * tiles * 32;
  if (first >= a.cap) return;
  const int n = kv_len(a.kv, b, min(a.cap, a.kv.max_pages << a.kv.page_shift)), base = n - a.L;
  const int64_t at = static_cast<int64_t>(bh) * a.cap;
  const int held_tiles = min(tiles, (n - first + 31) / 32);  // tiles that hold keys
  const float c = a.scale * kLog2e;
  const int rows = a.L * G;
  const uint8_t* const k_src = reinterpret_cast<const uint8_t*>(a.kv.k + hk * a.kv.head_stride);

  // the slot this lane holds the place of; slots past the sequence repeat its last key
  int page = 0;
  auto held_slot = [&](int t) { return max(min(first + t * 32 + held_key<RB>(lane) % 32, n - 1), 0); };
  auto look_up = [&](int t) {
    page = a.kv.table[static_cast<int64_t>(b) * a.kv.max_pages + (held_slot(t) >> a.kv.page_shift)];
  };
  auto stage = [&](int t, int buf) {
    const int j = held_slot(t);
    const int64_t at_held = 2 * (clamp_id(page, a.kv.n_pages) * a.kv.page_stride +
                                 (j & ((1 << a.kv.page_shift) - 1)) * a.kv.slot_stride);
    each_index<NI>([&](auto index) {
      constexpr int i = index;
      const int key = i * RPI + lane / (RB / 16), chunk = lane % (RB / 16) ^ row_swizzle<RB>(key);
      const void* src = k_src + held_offset<RB, i>(at_held) + chunk * 16;
      const void* zeros = g_zeros;
      copy_to_lds(chunk * 8 < a.D ? src : zeros, s_keys[wave][buf] + i * 1024);
    });
  };

  int buf = 0;
  if (held_tiles > 0) {
    look_up(0);
    stage(0, 0);
    look_up(held_tiles > 1 ? 1 : 0);
  }
  // What a tile's scores start from is loaded, and its result stored, a tile
  // away from its products: loads and stores count with the copies, so a wait
  // for either here would be a wait for the next tile's keys.
  auto start_of = [&](int t, int r0) {
    const int j = min(first + t * 32 + col, n - 1);
    return (r0 == 0 ? a.score_in : a.score_out)[at + j];
  };
  float old = held_tiles > 0 ? start_of(0, 0) : 0.f, done = 0.f;
  int done_tile = -1;
  auto flush = [&] {
    const int j = first + done_tile * 32 + col;
    if (done_tile >= 0 && half == 0 && j < n) a.score_out[at + j] = done;
    done_tile = -1;
  };
  for (int r0 = 0; r0 < rows && held_tiles > 0; r0 += kScoreRows) {
    // ---- a tile of queries, their log-sum-exps and mask words; the rows past the last
    // repeat it and add nothing
    uint4 q[QT][NC];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const int row = min(r0 + t * 32 + col, rows - 1);
      const int64_t bi = static_cast<int64_t>(b) * a.L + row / G;
      const uint16_t* src = a.q + bi * a.q_row_stride + (hk * G + row % G) * a.q_head_stride;
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const int e = 16 * i + 8 * half;
        q[t][i] = e < a.D ? *reinterpret_cast<const uint4*>(src + e) : make_uint4(0, 0, 0, 0);
      }
    }
    const int row_in = r0 + lane % kScoreRows;
    const int64_t bi_in = static_cast<int64_t>(b) * a.L + min(row_in, rows - 1) / G;
    const float z_in = row_in < rows ? a.lse[bi_in * a.H + hk * G + row_in % G] : -INFINITY;
    s_lse[wave][lane % kScoreRows] = z_in == -INFINITY ? INFINITY : z_in * kLog2e;
    s_word[wave][lane % kScoreRows] = a.mask ? a.mask[bi_in] : ~0ull;
    const bool holes = __any(z_in == -INFINITY);   // rows that add nothing
    __builtin_amdgcn_wave_barrier();
    for (int t = 0; t < held_tiles; ++t) {
      copies_landed();
      __builtin_amdgcn_wave_barrier();
      const uint8_t* kt = s_keys[wave][buf];
      buf ^= 1;
      const int next = t + 1 < held_tiles ? t + 1 : 0;  // and round again for the next rows
      const float begin = r0 == 0 ? a.decay * old : old;
      flush();
      if (next > 0 || r0 + kScoreRows < rows) {
        stage(next, buf);
        look_up(next + 1 < held_tiles ? next + 1 : 0);
        // the next rows' start at a run of one tile is this tile's own result
        if (held_tiles > 1) old = start_of(next, next > 0 ? r0 : r0 + kScoreRows);
      }
      floatx16 s[QT];
#pragma unroll
      for (int u = 0; u < QT; ++u) s[u] = floatx16{};
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const uint4 k = *reinterpret_cast<const uint4*>(kt + col * RB + (((2 * i + half) ^ row_swizzle<RB>(col)) << 4));
#pragma unroll
        for (int u = 0; u < QT; ++u) s[u] = mfma32<F16>(q[u][i], k, s[u]);
      }
      const int j = first + t * 32 + col, place = j - base;
      float sum = 0.f;
      // What a lane adds; `plain`: every row adds its weight, whichever the key
      auto add_up = [&](auto plain) {
#pragma unroll
        for (int u = 0; u < QT; ++u)
#pragma unroll
          for (int r = 0; r < 16; r += 4) {
            const int row = u * 32 + 8 * (r / 4) + 4 * half;
            const float4 z4 = *reinterpret_cast<const float4*>(s_lse[wave] + row);
            const float z[4] = {z4.x, z4.y, z4.z, z4.w};
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const float p = __builtin_amdgcn_exp2f(fmaf(s[u][r + x], c, -z[x]));
              if constexpr (decltype(plain)::value) {
                sum += p;
              } else {
                const bool off = (z[x] == INFINITY) | (place >= 0 && !block_sees(s_word[wave][row + x], place));
                sum += off ? 0.f : p;
              }
            }
          }
      };
      if (holes || (a.mask && first + t * 32 + 32 > base))
        add_up(std::false_type{});
      else
        add_up(std::true_type{});
      done = begin + swap32_sum(sum);
      done_tile = t;
      if (held_tiles == 1) old = done;
    }
    __builtin_amdgcn_wave_barrier();
  }
  flush();
  for (int j = max(first, n) + lane; j < min(a.cap, first + tiles * 32); j += kWave) a.score_out[at + j] = 0.f;
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

// The keys of sequences too long for LDS, and the outputs as they are before
// any slot moves: many workgroups, where the selection below has one a head.
__global__ __launch_bounds__(256) void evict_keys_kernel(EvictArgs a) {
  const int heads = a.B * a.Hkv, bh = blockIdx.x % heads, b = bh / a.Hkv;
  const int n = kv_len(a.kv, b, min(a.cap, a.kv.max_pages << a.kv.page_shift)), m = min(n, a.budget);
  const int64_t at = static_cast<int64_t>(bh) * a.cap;
  const int from = a.next_pos[b] - a.recent;
  const int j0 = blockIdx.x / heads * 1024 + threadIdx.x;
  float s[4];
  int x[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int j = min(j0 + u * 256, a.cap - 1);
    s[u] = a.score_in[at + j];
    x[u] = a.pos_in[at + j];
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int j = j0 + u * 256;
    if (j >= a.cap) break;
    a.keys[at + j] = keep_key(s[u], x[u] >= from);
    a.score_out[at + j] = j < m ? s[u] : 0.f;
    a.pos_out[at + j] = j < m ? x[u] : -1;
  }
}

// IN_LDS: the keys of a sequence are computed here and held in LDS; otherwise
// evict_keys_kernel left them in memory, and each pass keeps more of them in flight.
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
  constexpr int kFlight = IN_LDS ? 4 : 16;
  if (tid == 0 && blockIdx.x % a.Hkv == 0) a.new_len[b] = m;
  if constexpr (IN_LDS) {
    const int from = a.next_pos[b] - a.recent;
    for (int j0 = tid; j0 < a.cap; j0 += kSelectThreads * 4) {
      float s[4];
      int x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int j = min(j0 + u * kSelectThreads, a.cap - 1);
        s[u] = score[j];
        x[u] = pos[j];
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int j = j0 + u * kSelectThreads;
        if (j >= a.cap) break;
        s_keys[j] = keep_key(s[u], x[u] >= from);
        a.score_out[at + j] = j < m ? s[u] : 0.f;
        a.pos_out[at + j] = j < m ? x[u] : -1;
      }
    }
  }
  if (n <= m) {
    if (tid == 0) a.count[blockIdx.x] = 0;
    return;
  }
  auto key_of = [&](int j) {
    if constexpr (IN_LDS)
      return s_keys[j];
    else
      return a.keys[at + j];
  };
  // ---- the m-th largest key: `found` holds its leading bits, `left` how many of the
  // keys that share them are still to be taken
  uint32_t found = 0, left = m;
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
    for (int i = tid; i < kBins; i += kSelectThreads) s_hist[i] = 0;
    __syncthreads();
    for (int j0 = 0; j0 < n; j0 += kSelectThreads * kFlight) {
      uint32_t key[kFlight];
#pragma unroll
      for (int u = 0; u < kFlight; ++u) {
        const int j = j0 + u * kSelectThreads + tid;
        key[u] = j < n ? key_of(j) : 0;
      }
#pragma unroll
      for (int u = 0; u < kFlight; ++u) {
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
  for (int j = j0; j < j1; j += kWave * kFlight) {
    uint32_t key[kFlight];
#pragma unroll
    for (int u = 0; u < kFlight; ++u) key[u] = j + u * kWave + lane < j1 ? key_of(j + u * kWave + lane) : 0;
#pragma unroll
    for (int u = 0; u < kFlight; ++u) {
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
  for (int j = j0; j < j1; j += kWave * kFlight) {
    uint32_t key[kFlight];
#pragma unroll
    for (int u = 0; u < kFlight; ++u) key[u] = j + u * kWave + lane < j1 ? key_of(j + u * kWave + lane) : 0;
#pragma unroll
    for (int u = 0; u < kFlight; ++u) {
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
__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a) {
  const int heads = a.B * a.Hkv, bh = blockIdx.x % heads, r0 = blockIdx.x / heads * kMoveRows;
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

// Tiles of a wavefront: eight, so that its start and its queries are paid once
// for 256 keys, unless that leaves CUs without a workgroup.
template <bool F16>
void launch_score(const ScoreArgs& a, hipStream_t s) {
  const int64_t whole = static_cast<int64_t>(a.B) * a.Hkv;
  int tiles = kMaxTiles;
  auto runs_of = [&](int t) { return (a.cap + kScoreWaves * t * 32 - 1) / (kScoreWaves * t * 32); };
  while (tiles > 1 && whole * runs_of(tiles) < 512) tiles /= 2;
  const int runs = runs_of(tiles);
  const dim3 grid(static_cast<uint32_t>(whole * runs)), threads(64 * kScoreWaves);
  const bool two = a.L * (a.H / a.Hkv) > 32;
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, threads, 0, s, a, tiles); };
  if (a.D <= 64)
    two ? go(score_kernel<F16, 2, 2>) : go(score_kernel<F16, 2, 1>);
  else if (a.D <= 96)
    two ? go(score_kernel<F16, 3, 2>) : go(score_kernel<F16, 3, 1>);
  else
    two ? go(score_kernel<F16, 4, 2>) : go(score_kernel<F16, 4, 1>);
}

}  // namespace

void launch_cache_score(const ScoreArgs& a, bool f16, hipStream_t s) {
  if (f16)
    launch_score<true>(a, s);
  else
    launch_score<false>(a, s);
}

int evict_list_len(int cap, int budget) { return cap > budget ? (budget < cap - budget ? budget : cap - budget) : 0; }

// Workspace: a count for each (sequence, head), the lists of sources and
// targets, at most min(budget, cap - budget) entries each, and the keys where
// they do not fit LDS.
size_t evict_workspace_bytes(int B, int Hkv, int cap, int budget) {
  const size_t heads = static_cast<size_t>(B) * Hkv, len = evict_list_len(cap, budget);
  return ((heads + 3) / 4 * 4 + 2 * heads * len + (cap > kLdsSlots ? heads * cap : 0)) * sizeof(int32_t);
}

void launch_cache_evict(EvictArgs a, void* ws, hipStream_t s) {
  const size_t heads = static_cast<size_t>(a.B) * a.Hkv;
  a.list_len = evict_list_len(a.cap, a.budget);
  a.count = static_cast<int32_t*>(ws);
  a.src = a.count + (heads + 3) / 4 * 4;
  a.dst = a.src + heads * a.list_len;
  a.keys = reinterpret_cast<uint32_t*>(a.dst + heads * a.list_len);
  if (a.cap <= kLdsSlots) {
    hipLaunchKernelGGL(evict_select_kernel<true>, dim3(heads), dim3(kSelectThreads), a.cap * sizeof(uint32_t), s, a);
  } else {
    hipLaunchKernelGGL(evict_keys_kernel, dim3(heads * ((a.cap + 1023) / 1024)), dim3(256), 0, s, a);
    hipLaunchKernelGGL(evict_select_kernel<false>, dim3(heads), dim3(kSelectThreads), 0, s, a);
  }
  if (a.list_len > 0) {
    const int runs = (a.list_len + kMoveRows - 1) / kMoveRows;
    hipLaunchKernelGGL(evict_move_kernel, dim3(heads * runs), dim3(256), 0, s, a);
  }
}

}  // namespace brisk
