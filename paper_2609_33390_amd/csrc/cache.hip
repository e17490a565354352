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
  constexpr int RB = lds_row_bytes(ND), NC = 2 * ND, kTile = 32 * RB, NI = kTile / 1024, RPI = 1024 / RB;
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
// Eviction.  The budget-th largest key is found by three histogram passes (11 +
// 11 + 10 bits); then the evicted slots below the budget and the kept ones at
// or above it are listed, and a last launch moves the rows.  A slot's place in
// a list follows from the number of kept slots before it: the hole at slot j is
// number j - kept(j), and a mover at slot j has budget - kept(j) kept slots
// from it on, itself included (the list of movers runs backwards).
//
// Caches of up to 32768 slots are selected by one workgroup each, with the keys
// in LDS (one launch; 64 x 8 heads of 4100 slots: 20 us).  One workgroup is bound
// by its own instructions beyond that (120000 slots: 130 us), so longer caches are
// cut into chunks, each with a workgroup and a histogram of its own; every
// workgroup adds the histograms up for itself, which also tells it how many keys
// lie above and at the wanted one in the chunks before its own.
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
constexpr int kPasses = 3;
constexpr int kShift[kPasses] = {21, 10, 0}, kBits[kPasses] = {11, 11, 10};

struct SelectShared {
  uint32_t hist[kBins];
  uint32_t wave[2][kSelectWaves];
  uint32_t digit, left;
};

// Adds a wavefront's keys to the histogram.  The keys that share the first
// one's digit are added at once: scores are often all alike.
__device__ __forceinline__ void count_digit(uint32_t* hist, uint32_t digit, bool in) {
  const uint64_t active = __ballot(in);
  if (!active) return;
  const int leader = __builtin_ctzll(active);
  const uint32_t one = __builtin_amdgcn_readlane(digit, leader);
  const uint64_t same = __ballot(in && digit == one);
  if (static_cast<int>(threadIdx.x & 63) == leader) atomicAdd(&hist[one], static_cast<uint32_t>(__popcll(same)));
  if (in && digit != one) atomicAdd(&hist[digit], 1u);
}

__device__ __forceinline__ bool shares_prefix(uint32_t key, int pass, uint32_t found) {
  return pass == 0 || (key >> (kShift[pass] + kBits[pass])) == found;
}
__device__ __forceinline__ uint32_t digit_of(uint32_t key, int pass) {
  return (key >> kShift[pass]) & ((1u << kBits[pass]) - 1);
}

// The bin in which the count from the top reaches `left`, and what is left to
// be taken in it, into sh.digit and sh.left.  Thread t brings the counts of
// bins kBins - 1 - 2 t (c0) and the one below it (c1).
__device__ __forceinline__ void find_digit(SelectShared& sh, uint32_t c0, uint32_t c1, uint32_t left) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, hi = kBins - 1 - 2 * tid;
  uint32_t run = c0 + c1;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const uint32_t o = __shfl_up(run, off, kWave);
    if (lane >= off) run += o;
  }
  if (lane == 63) sh.wave[0][wave] = run;
  __syncthreads();
  uint32_t before = run - c0 - c1;
  for (int w = 0; w < wave; ++w) before += sh.wave[0][w];
  if (before < left && before + c0 >= left) {
    sh.digit = hi;
    sh.left = left - before;
  } else if (before + c0 < left && before + c0 + c1 >= left) {
    sh.digit = hi - 1;
    sh.left = left - before - c0;
  }
  __syncthreads();
}

// Lists the slots [j0, j1) of one wavefront, in order: `above` and `ties` are
// the keys above and at `found` before j0, `left` the ties to be kept.
template <int kFlight, class KeyOf>
__device__ __forceinline__ void list_slots(const EvictArgs& a, int head, int m, int j0, int j1, uint32_t found,
                                           uint32_t left, uint32_t above, uint32_t ties, KeyOf key_of) {
  const int lane = threadIdx.x & 63;
  int32_t* const src = a.src + static_cast<int64_t>(head) * a.list_len;
  int32_t* const dst = a.dst + static_cast<int64_t>(head) * a.list_len;
  const uint64_t below = (1ull << lane) - 1;
  for (int j = j0; j < j1; j += kWave * kFlight) {
    uint32_t key[kFlight];
#pragma unroll
    for (int u = 0; u < kFlight; ++u) key[u] = j + u * kWave + lane < j1 ? key_of(j + u * kWave + lane) : 0;
#pragma unroll
    for (int u = 0; u < kFlight; ++u) {
      const int x = j + u * kWave + lane;
      const bool in = x < j1;
      const uint64_t more = __ballot(in && key[u] > found), same = __ballot(in && key[u] == found);
      const uint32_t tie = ties + __popcll(same & below);
      const int kept = above + __popcll(more & below) + min(tie, left);  // slots kept before this one
      const bool keep = key[u] > found || (key[u] == found && tie < left);
      if (in && x < m && !keep) dst[x - kept] = x;
      if (in && x >= m && keep) src[m - kept - 1] = x;
      if (in && x == m) a.count[head] = m - kept;
      above += __popcll(more);
      ties += __popcll(same);
    }
  }
}

// How many keys of [j0, j1) lie above and at `found`, for the whole wavefront.
template <int kFlight, class KeyOf>
__device__ __forceinline__ uint2 count_slots(int j0, int j1, uint32_t found, KeyOf key_of) {
  const int lane = threadIdx.x & 63;
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
  return make_uint2(above, ties);
}

// The outputs as they are before any slot moves, and the keys: loads of four slots
// a thread in flight.
template <class Store>
__device__ __forceinline__ void start_outputs(const EvictArgs& a, int64_t at, int n, int m, int from, int j0, int end,
                                              int stride, Store store_key) {
  for (int j = j0; j < end; j += stride * 4) {
    float s[4];
    int x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = min(j + u * stride, a.cap - 1);
      s[u] = a.score_in[at + i];
      x[u] = a.pos_in[at + i];
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = j + u * stride;
      if (i >= end) break;
      if (i < n) store_key(i, keep_key(s[u], x[u] >= from));
      a.score_out[at + i] = i < m ? s[u] : 0.f;
      a.pos_out[at + i] = i < m ? x[u] : -1;
    }
  }
}

// One workgroup a (sequence, head), keys in LDS.
__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(EvictArgs a) {
  extern __shared__ uint32_t s_keys[];
  __shared__ SelectShared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = blockIdx.x, b = head / a.Hkv, n = kv_len(a.kv, b, min(a.cap, a.kv.max_pages << a.kv.page_shift));
  const int m = min(n, a.budget);
  if (tid == 0 && head % a.Hkv == 0) a.new_len[b] = m;
  start_outputs(a, static_cast<int64_t>(head) * a.cap, n, m, a.next_pos[b] - a.recent, tid, a.cap, kSelectThreads,
                [&](int j, uint32_t key) { s_keys[j] = key; });
  if (n <= m) {
    if (tid == 0) a.count[head] = 0;
    return;
  }
  uint32_t found = 0, left = m;
#pragma unroll
  for (int pass = 0; pass < kPasses; ++pass) {
    for (int i = tid; i < kBins; i += kSelectThreads) sh.hist[i] = 0;
    __syncthreads();
    for (int j0 = 0; j0 < n; j0 += kSelectThreads) {
      const int j = j0 + tid;
      const uint32_t key = j < n ? s_keys[j] : 0;
      count_digit(sh.hist, digit_of(key, pass), j < n && shares_prefix(key, pass, found));
    }
    __syncthreads();
    find_digit(sh, sh.hist[kBins - 1 - 2 * tid], sh.hist[kBins - 2 - 2 * tid], left);
    found = (found << kBits[pass]) | sh.digit;
    left = sh.left;
    __syncthreads();
  }
  // a run of slots for each wavefront
  const int per = (n + kSelectThreads - 1) / kSelectThreads * kWave, j0 = min(wave * per, n), j1 = min(j0 + per, n);
  auto key_of = [&](int j) { return s_keys[j]; };
  const uint2 mine = count_slots<4>(j0, j1, found, key_of);
  if (lane == 0) {
    sh.wave[0][wave] = mine.x;
    sh.wave[1][wave] = mine.y;
  }
  __syncthreads();
  uint32_t above = 0, ties = 0;
  for (int w = 0; w < wave; ++w) {
    above += sh.wave[0][w];
    ties += sh.wave[1][w];
  }
  list_slots<4>(a, head, m, j0, j1, found, left, above, ties, key_of);
}

// Chunks of a long cache: at most 64, so that adding up their histograms stays
// short, and of at least 4096 slots.
int evict_chunk(int cap) { return max(4096, ((cap + 63) / 64 + 4095) / 4096 * 4096); }
int evict_chunks(int cap) { return (cap + evict_chunk(cap) - 1) / evict_chunk(cap); }

// What the passes over a long cache know of it so far.
struct ChunkState { uint32_t found, left, above; };  // above: keys above `found`'s digits in the chunks before

// Pass 0 starts the outputs, writes the keys and counts their first digit; pass
// 1 and 2 count the next ones; pass 3 lists.
template <int PASS>
__global__ __launch_bounds__(kSelectThreads) void evict_chunk_kernel(EvictArgs a, int chunk, int chunks, uint32_t* keys,
                                                                     uint32_t* hists, ChunkState* states) {
  __shared__ SelectShared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int heads = a.B * a.Hkv, head = blockIdx.x % heads, mine = blockIdx.x / heads, b = head / a.Hkv;
  const int n = kv_len(a.kv, b, min(a.cap, a.kv.max_pages << a.kv.page_shift)), m = min(n, a.budget);
  const int begin = mine * chunk, end = min(begin + chunk, a.cap);
  uint32_t* const key = keys + static_cast<int64_t>(head) * a.cap;
  auto hist_of = [&](int pass) { return hists + (static_cast<int64_t>(pass) * heads + head) * chunks * kBins; };
  if constexpr (PASS == 0) {
    if (tid == 0 && mine == 0) {
      if (head % a.Hkv == 0) a.new_len[b] = m;
      if (n <= m) a.count[head] = 0;
    }
    for (int i = tid; i < kBins; i += kSelectThreads) sh.hist[i] = 0;
    __syncthreads();
    start_outputs(a, static_cast<int64_t>(head) * a.cap, n, m, a.next_pos[b] - a.recent, begin + tid, end, kSelectThreads,
                  [&](int j, uint32_t k) {
                    key[j] = k;
                    count_digit(sh.hist, digit_of(k, 0), true);
                  });
    if (n <= m) return;
  } else {
    if (n <= m) return;
    ChunkState st = {0, static_cast<uint32_t>(m), 0};
    if constexpr (PASS > 1) st = states[(static_cast<int64_t>(PASS - 2) * heads + head) * chunks + mine];
    // the histograms of the pass before, all of them and those of the chunks before this one
    const uint2* h = reinterpret_cast<const uint2*>(hist_of(PASS - 1)) + (kBins / 2 - 1 - tid);
    uint32_t c0 = 0, c1 = 0, p0 = 0, p1 = 0;
    for (int c = 0; c < chunks; c += 16) {         // 16 loads in flight
      uint2 x[16];
#pragma unroll
      for (int u = 0; u < 16; ++u) x[u] = h[min(c + u, chunks - 1) * (kBins / 2)];
#pragma unroll
      for (int u = 0; u < 16; ++u) {
        const bool in = c + u < chunks, before = c + u < mine;
        c0 += in ? x[u].y : 0;
        c1 += in ? x[u].x : 0;
        p0 += before ? x[u].y : 0;
        p1 += before ? x[u].x : 0;
      }
    }
    find_digit(sh, c0, c1, st.left);
    const uint32_t digit = sh.digit, hi = kBins - 1 - 2 * tid;
    st.found = (st.found << kBits[PASS - 1]) | digit;
    st.left = sh.left;
    uint32_t up = (hi > digit ? p0 : 0) + (hi - 1 > digit ? p1 : 0), tie = hi == digit ? p0 : hi - 1 == digit ? p1 : 0;
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
      up += __shfl_xor(up, off, kWave);
      tie += __shfl_xor(tie, off, kWave);
    }
    if (lane == 0) {
      sh.wave[0][wave] = up;
      sh.wave[1][wave] = tie;
    }
    if constexpr (PASS < kPasses)
      for (int i = tid; i < kBins; i += kSelectThreads) sh.hist[i] = 0;
    __syncthreads();
    uint32_t ties = 0;
    for (int w = 0; w < kSelectWaves; ++w) {
      st.above += sh.wave[0][w];
      ties += sh.wave[1][w];
    }
    const int last = min(end, n);
    if constexpr (PASS < kPasses) {
      if (tid == 0) states[(static_cast<int64_t>(PASS - 1) * heads + head) * chunks + mine] = st;
      for (int j0 = begin; j0 < last; j0 += kSelectThreads * 4) {
        uint32_t k[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) k[u] = key[min(j0 + u * kSelectThreads + tid, last - 1)];
#pragma unroll
        for (int u = 0; u < 4; ++u)
          count_digit(sh.hist, digit_of(k[u], PASS),
                      j0 + u * kSelectThreads + tid < last && shares_prefix(k[u], PASS, st.found));
      }
    } else {
      const int per = (max(last - begin, 0) + kSelectThreads - 1) / kSelectThreads * kWave;
      const int j0 = min(begin + wave * per, last), j1 = min(j0 + per, last);
      auto key_of = [&](int j) { return key[j]; };
      __syncthreads();
      const uint2 c = count_slots<4>(j0, j1, st.found, key_of);
      if (lane == 0) {
        sh.wave[0][wave] = c.x;
        sh.wave[1][wave] = c.y;
      }
      __syncthreads();
      for (int w = 0; w < wave; ++w) {
        st.above += sh.wave[0][w];
        ties += sh.wave[1][w];
      }
      list_slots<4>(a, head, m, j0, j1, st.found, st.left, st.above, ties, key_of);
    }
  }
  if constexpr (PASS < kPasses) {
    __syncthreads();
    uint32_t* const out = hist_of(PASS) + static_cast<int64_t>(mine) * kBins;
    for (int i = tid; i < kBins; i += kSelectThreads) out[i] = sh.hist[i];
  }
}

// Moves listed rows, 16 lanes a row and kRowsInFlight rows at once.
constexpr int kMoveThreads = 256, kRowsInFlight = 4, kMoveRows = kMoveThreads / 16 * kRowsInFlight;
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(EvictArgs a) {
  const int heads = a.B * a.Hkv, bh = blockIdx.x % heads, r0 = blockIdx.x / heads * kMoveRows;
  const int count = a.count[bh];
  if (r0 >= count) return;
  const int b = bh / a.Hkv, hk = bh % a.Hkv;
  const int64_t at = static_cast<int64_t>(bh) * a.cap, list = static_cast<int64_t>(bh) * a.list_len;
  const int lane = threadIdx.x & 15, e = min(lane * 8, a.D - 8);  // narrow heads: the last lanes repeat a chunk
  int src[kRowsInFlight], dst[kRowsInFlight];  // the movers' list runs backwards
#pragma unroll
  for (int u = 0; u < kRowsInFlight; ++u) {
    const int r = min(r0 + u * 16 + static_cast<int>(threadIdx.x >> 4), count - 1);  // past the end: the last row again
    src[u] = a.src[list + count - 1 - r];
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

// A launch has fewer than 2^32 threads.
bool launchable(int64_t workgroups, int threads) { return workgroups * threads < int64_t{1} << 32; }

// Tiles of a wavefront: eight, so that its start and its queries are paid once
// for 256 keys, unless that leaves CUs without a workgroup.
struct ScoreRuns { int tiles, runs; };
ScoreRuns score_runs(int64_t whole, int cap) {
  auto runs_of = [&](int t) { return (cap + kScoreWaves * t * 32 - 1) / (kScoreWaves * t * 32); };
  int tiles = kMaxTiles;
  while (tiles > 1 && whole * runs_of(tiles) < 512) tiles /= 2;
  return {tiles, runs_of(tiles)};
}

template <bool F16>
void launch_score(const ScoreArgs& a, hipStream_t s) {
  const int64_t whole = static_cast<int64_t>(a.B) * a.Hkv;
  const auto [tiles, runs] = score_runs(whole, a.cap);
  const dim3 grid(static_cast<uint32_t>(whole * runs)), threads(64 * kScoreWaves);
  const bool two = a.L * (a.H / a.Hkv) > 32;
  const int per = tiles;
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, threads, 0, s, a, per); };
  switch (head_slices(a.D)) {
    case 2: two ? go(score_kernel<F16, 2, 2>) : go(score_kernel<F16, 2, 1>); break;
    case 3: two ? go(score_kernel<F16, 3, 2>) : go(score_kernel<F16, 3, 1>); break;
    default: two ? go(score_kernel<F16, 4, 2>) : go(score_kernel<F16, 4, 1>); break;
  }
}

}  // namespace

bool score_launchable(int B, int Hkv, int cap) {
  const int64_t whole = static_cast<int64_t>(B) * Hkv;
  return launchable(whole * score_runs(whole, cap).runs, 64 * kScoreWaves);
}

void launch_cache_score(const ScoreArgs& a, bool f16, hipStream_t s) {
  if (f16)
    launch_score<true>(a, s);
  else
    launch_score<false>(a, s);
}

int evict_list_len(int cap, int budget) { return cap > budget ? (budget < cap - budget ? budget : cap - budget) : 0; }

// Workspace: a count for each (sequence, head), the lists of sources and
// targets, at most min(budget, cap - budget) entries each; for long caches the
// keys, and a histogram of each pass and a state of each chunk.
namespace {
struct EvictSpace {
  size_t count, lists, keys, hists, states, words;
  EvictSpace(int B, int Hkv, int cap, int budget) {
    const size_t heads = static_cast<size_t>(B) * Hkv, chunks = cap > kLdsSlots ? evict_chunks(cap) : 0;
    auto even = [](size_t x) { return (x + 3) / 4 * 4; };
    count = 0;
    lists = even(heads);
    keys = lists + even(2 * heads * evict_list_len(cap, budget));
    hists = keys + (chunks ? even(heads * cap) : 0);
    states = hists + kPasses * heads * chunks * kBins;
    words = states + 2 * heads * chunks * (sizeof(ChunkState) / sizeof(uint32_t));
  }
};
}  // namespace

bool evict_launchable(int B, int Hkv, int cap, int budget) {
  const int64_t heads = static_cast<int64_t>(B) * Hkv;
  const int moves = (evict_list_len(cap, budget) + kMoveRows - 1) / kMoveRows;
  return launchable(heads * (cap > kLdsSlots ? evict_chunks(cap) : 1), kSelectThreads) && launchable(heads * moves, kMoveThreads);
}

size_t evict_workspace_bytes(int B, int Hkv, int cap, int budget) {
  return EvictSpace(B, Hkv, cap, budget).words * sizeof(uint32_t);
}

void launch_cache_evict(EvictArgs a, void* ws, hipStream_t s) {
  const uint32_t heads = static_cast<uint32_t>(a.B) * a.Hkv;
  const EvictSpace at(a.B, a.Hkv, a.cap, a.budget);
  a.list_len = evict_list_len(a.cap, a.budget);
  a.count = static_cast<int32_t*>(ws) + at.count;
  a.src = static_cast<int32_t*>(ws) + at.lists;
  a.dst = a.src + static_cast<size_t>(heads) * a.list_len;
  if (a.cap <= kLdsSlots) {
    hipLaunchKernelGGL(evict_select_kernel, dim3(heads), dim3(kSelectThreads), a.cap * sizeof(uint32_t), s, a);
  } else {
    uint32_t* const words = static_cast<uint32_t*>(ws);
    const int chunks = evict_chunks(a.cap);
    auto go = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3(heads * chunks), dim3(kSelectThreads), 0, s, a, evict_chunk(a.cap), chunks,
                         words + at.keys, words + at.hists, reinterpret_cast<ChunkState*>(words + at.states));
    };
    go(evict_chunk_kernel<0>);
    go(evict_chunk_kernel<1>);
    go(evict_chunk_kernel<2>);
    go(evict_chunk_kernel<3>);
  }
  if (a.list_len > 0) {
    const uint32_t runs = (a.list_len + kMoveRows - 1) / kMoveRows;
    hipLaunchKernelGGL(evict_move_kernel, dim3(heads * runs), dim3(kMoveThreads), 0, s, a);
  }
}

}  // namespace brisk
