// Attention of a block over a shared prefix and a paged cache (Section 2.1:
// one model evaluation verifies and proposes all positions of a block).
//
//   s_j = scale <q, k_j>,  m = max_j s_j,  l = sum_j exp(s_j - m)
//   out = sum_j exp(s_j - m) v_j / l,  lse = m + log l
//
// All rows that read the same keys share one pass over them: the prefix is
// read by tiles of rows of the whole batch (rows of every sequence and of
// every query head of a group), a sequence's own cache by the rows of its
// block.  A workgroup takes a tile of rows and a run of keys; runs of the same
// rows are joined afterwards from their normalised sums and log-sum-exps:
//   out = sum_r exp(lse_r - lse) out_r,  lse = log sum_r exp(lse_r)
//
// Inside a wavefront the logits are computed transposed, S^T = K Q^T, so that
// a lane holds one row's logits: the softmax statistics need one exchange
// between the wavefront's halves, and the probabilities are already the
// operand of out^T = V^T P^T, with the keys in an order that the transposed
// LDS reads of V follow.
//
// Keys and values come to LDS by asynchronous copies, a tile ahead.  Few rows
// are bound by the read of the cache: 64 sequences x 8 heads x 2048 keys of 128
// elements, 32 rows each, run at 5.1 TB/s (a large copy: 4.9), 64 rows at 5.0.
// Many rows are bound by the matrix cores and by what feeds them from LDS: 32768
// rows (4096 a key head) over 16384 shared keys, 275 GFLOP, take 0.32 ms, 0.85
// PFLOP/s where a library product of 8192^3 reaches 1.19; with the LDS reads left
// out 0.28, with the softmax left out too 0.24.  Small calls are bound by latency:
// lengths, page ids, keys, join.
#include "attention_plan.h"
#include "half_mfma.h"
#include "kernels.h"

namespace brisk {

namespace {

typedef short shortx4 __attribute__((ext_vector_type(4)));

// In base 2: the subtracted logit may be kLag behind the maximum, and the probabilities are held
// kLift higher than that, which l and the log-sum-exp share.  f16 has no steps below 2^-24, so its
// probabilities use its range from the top: at most 2^15, and a key's weight is off by at most
// 2^-37 of the largest one's, besides its rounding to 11 bits (unlifted, 65536 keys of 2^-25 of the
// largest weight, 0.2% of it together, count as nothing).  bf16 has the range of fp32.
template <bool F16> constexpr float kLag = F16 ? 3.f : 8.f;
template <bool F16> constexpr float kLift = F16 ? 12.f : 0.f;
constexpr float kFine = 0x1p20f;   // up to here a float holds a subtracted logit to 2^-5

// What one launch works on: prefix items, then own items.
struct AttnPlan {
  float* part;           // [rows][splits][D] normalised sums, null when every row has one run
  float* part_lse;       // [rows][splits]
  int pre_groups, pre_tiles, pre_splits, pre_run;  // (head, split) pairs, row tiles, runs of pre_run keys
  int own_groups, own_tiles, own_splits, own_run;  // (sequence, head, split) triples, ...
  int splits;            // pre_splits + own_splits of all launches of the call
  int own_first;         // index of the first own split
};

// Which of 32 keys a row sees: bit x is set when x < left and the key's place
// in the block, at + x, is negative (before the block) or set in `word`.
__device__ __forceinline__ uint32_t seen32(uint64_t word, int at, int left) {
  uint64_t bits = at >= 64 ? 0 : at >= 0 ? word >> at : at > -32 ? (word << -at) | ((1ull << -at) - 1) : ~0ull;
  bits = left >= 32 ? bits : left <= 0 ? 0 : bits & ((1ull << left) - 1);
  return static_cast<uint32_t>(bits);
}

// Values take another permutation than keys, for the transposed b64 reads of
// four chunks of 4 keys.
template <int RB>
__device__ __forceinline__ int v_swizzle(int key) { return RB == 256 ? (key & 3) << 2 : ((key >> 1) & 1) << 2; }

// ND: 32-wide slices of the head.  A wavefront has 32 rows; RW wavefronts of
// different rows share each tile of 32 * NT keys, KW groups of them take
// alternate tiles, one in LDS and the next one on its way.  (Wavefronts of 64
// rows read each key and value from LDS once for two products, but leave no
// registers for a second wavefront on the SIMD: 64 caches of 16 to 2048 keys, 64
// rows each, took 93 us that way and 82 us as two wavefronts of 32 rows.)
template <bool F16, int ND, int RW, int KW, int NT>
__global__ __launch_bounds__(64 * RW * KW, RW >= 2 ? 2 : 1) void attend_kernel(AttentionArgs a, AttnPlan p) {
  constexpr int RB = lds_row_bytes(ND), T = 32 * NT, NC = 2 * ND;
  constexpr int RPI = 1024 / RB;                 // rows of a wavefront's copy
  constexpr int NI = T / RPI / RW;               // copies of K (and of V) a wavefront
  constexpr int kTile = T * RB;                  // bytes of K (or V) of a tile
  constexpr int kStage = 2 * kTile;
  constexpr int kRows = RW * 32;
  constexpr int kOutRow = ND * 32 + 4;           // floats of a row of the join
  constexpr int kJoin = KW > 1 ? KW * kRows * (kOutRow + 2) * 4 : RW * 8192;
  constexpr int kLds = 2 * kStage * KW > kJoin ? 2 * kStage * KW : kJoin;
  static_assert(T % (RPI * RW) == 0 && kLds <= 163840);
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kLds];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), rw = wave % RW, kw = wave / RW;
  const int half = lane >> 5, col = lane & 31;
  const int G = a.H / a.Hkv;

  // ---- which rows and keys
  int bid = blockIdx.x;
  const int pre_grid = tile_grid(p.pre_groups, p.pre_tiles);
  const bool own = bid >= pre_grid;
  if (own) bid -= pre_grid;
  const int groups = own ? p.own_groups : p.pre_groups;
  const auto [group, tile] = group_tile(bid, groups, own ? p.own_tiles : p.pre_tiles);
  if (group >= groups) return;
  int b = 0, hk, split, key0, key1, row0, rows;
  const int held = rw * NI * RPI + held_key<RB>(lane);  // the key of a tile whose place this lane works out
  int page = 0;                                  // page id of the held key, a tile ahead
  if (own) {
    // first runs of all sequences, then second ones, ...: later runs are fewer where lengths differ
    hk = group % a.Hkv;
    b = group / a.Hkv % a.B;
    split = group / a.Hkv / a.B;
    // The first tile's pages are on their way while the length is (entries past it are not used).
    if (a.max_seq_len > 0)
      page = a.kv.table[static_cast<int64_t>(b) * a.kv.max_pages +
                        (min(split * p.own_run + kw * T + held, a.max_seq_len - 1) >> a.kv.page_shift)];
    const int n = kv_len(a.kv, b, a.max_seq_len);
    key0 = split * p.own_run;
    key1 = min(n, key0 + p.own_run);
    row0 = b * a.L * G;
    rows = a.L * G;
    split += p.own_first;
    if (key0 >= n && p.part) {                   // a run past the sequence: the join reads that it is empty
      for (int r = tile * kRows + tid; r < min(rows, (tile + 1) * kRows); r += 64 * RW * KW) {
        const int row = row0 + r;
        p.part_lse[(static_cast<int64_t>(row / G) * a.H + hk * G + row % G) * p.splits + split] = -INFINITY;
      }
      return;
    }
  } else {
    split = group % p.pre_splits;
    hk = group / p.pre_splits;
    key0 = split * p.pre_run;
    key1 = min(a.prefix_len, key0 + p.pre_run);
    row0 = 0;
    rows = a.B * a.L * G;
  }
  row0 += tile * kRows;
  rows = min(kRows, rows - tile * kRows);
  const int base = own ? kv_len(a.kv, b, a.max_seq_len) - a.L : 0;  // first slot of the block itself
  const bool masked = own && a.mask;
  const float c = a.scale * kLog2e;

  // ---- this wavefront's queries, as the second operand of K Q^T
  uint4 q[NC];
  uint64_t word;                                 // what its row sees of the block
  {
    const int row = row0 + min(rw * 32 + col, rows - 1), bi = row / G;
    const uint16_t* src = a.q + bi * a.q_row_stride + (hk * G + row % G) * a.q_head_stride;
    word = masked ? a.mask[bi] : ~0ull;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int e = 16 * i + 8 * half;
      q[i] = e < a.D ? *reinterpret_cast<const uint4*>(src + e) : make_uint4(0, 0, 0, 0);
    }
  }

  // ---- copies of keys and values to LDS
  // A copy is 1 KiB: RPI keys, RB / 16 lanes a key.  The place of a key in
  // memory is worked out once, by the lane that holds it for this wavefront's
  // copies, and handed to the key's lanes by broadcasts inside 16-lane rows.
  const uint8_t* const k_src = reinterpret_cast<const uint8_t*>(
      own ? a.kv.k + hk * a.kv.head_stride : a.pre_k + hk * a.pre_head_stride);
  const uint8_t* const v_src = reinterpret_cast<const uint8_t*>(
      own ? a.kv.v + hk * a.kv.head_stride : a.pre_v + hk * a.pre_head_stride);
  uint8_t* const lds = smem + kw * (2 * kStage);
  const int pc = lane % (RB / 16), key_in = lane / (RB / 16);  // this lane's chunk, and its key in a copy
  const bool whole = head_fills_row(a.D, ND);
  auto look_up = [&](int j0) {
    const int j = max(min(j0 + held, key1 - 1), 0);
    if (own) page = a.kv.table[static_cast<int64_t>(b) * a.kv.max_pages + (j >> a.kv.page_shift)];
  };
  // Copies the tile at j0; slots from v_end on get no value (key1, or where the block begins).
  auto stage = [&](int j0, int buf, int v_end) {
    const int j = max(min(j0 + held, key1 - 1), 0);
    const int64_t at = 2 * (own ? clamp_id(page, a.kv.n_pages) * a.kv.page_stride +
                                      (j & ((1 << a.kv.page_shift) - 1)) * a.kv.slot_stride
                                : j * a.pre_slot_stride);
    const bool plain = whole && j0 + T <= v_end;
    uint8_t* dst = lds + buf * kStage + rw * NI * 1024;
    each_index<NI>([&](auto index) {
      constexpr int i = index;
      const int64_t off = held_offset<RB, i>(at);
      const int key = (rw * NI + i) * RPI + key_in;
      const int ck = pc ^ row_swizzle<RB>(key), cv = pc ^ v_swizzle<RB>(key);
      const void *sk = k_src + off + ck * 16, *sv = v_src + off + cv * 16;
      if (!plain) {
        const void* zeros = g_zeros;
        sk = j0 + key < key1 && ck * 8 < a.D ? sk : zeros;
        sv = j0 + key < v_end && cv * 8 < a.D ? sv : zeros;
      }
      copy_to_lds(sk, dst + i * 1024);
      copy_to_lds(sv, dst + i * 1024 + kTile);
    });
  };

  floatx16 o[ND];
  // m: the subtracted logit (unscaled); mc = c * m - kLift; l: this lane's part of the sum, zero while
  // the row has seen no key (NaN logits pass the maximum by, but not the sum)
  float m, mc, l;
  bool wide;                                     // a row's mc is past kFine (the same in all lanes)
  const int steps = (key1 - key0 + T * KW - 1) / (T * KW);

  // The second time round only where values that some rows must not see are
  // not finite: the block's own values then join by vector arithmetic, row by row.
  for (int careful = 0;; ++careful) {
    m = -INFINITY;
    mc = l = 0.f;
    wide = false;
#pragma unroll
    for (int d = 0; d < ND; ++d) o[d] = floatx16{};
    const int v_end = careful ? min(key1, max(base, 0)) : key1;
    int j0 = key0 + kw * T;
    if (steps > 0) {
      if (careful) look_up(j0);
      stage(j0, 0, v_end);
      look_up(j0 + T * KW);
    }
    for (int step = 0; step < steps; ++step, j0 += T * KW) {
      const int buf = step & 1;
      copies_landed();
      if constexpr (RW > 1)
        __syncthreads();
      else
        __builtin_amdgcn_wave_barrier();         // no other wavefront writes or reads this one's tiles
      if (j0 >= key1) continue;  // uniform in the wavefront; this tile and all later ones are past the run
      const uint8_t* kt = lds + buf * kStage;
      const uint8_t* vt = kt + kTile;

      // ---- S^T = K Q^T: register r of a lane is key 8 (r / 4) + 4 half + r % 4 of each 32
      // All reads first (the fences keep the compiler from putting each one in front of
      // the product that needs it), so that the products follow each other.
      floatx16 s[NT];
      {
        uint4 kf[NT][NC];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < NC; ++i) {
            const int key = n * 32 + col;
            kf[n][i] = *reinterpret_cast<const uint4*>(kt + key * RB + (((2 * i + half) ^ row_swizzle<RB>(key)) << 4));
          }
        __builtin_amdgcn_sched_barrier(0);
        if (step + 1 < steps) {
          stage(j0 + T * KW, buf ^ 1, v_end);
          look_up(j0 + 2 * T * KW);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          s[n] = floatx16{};
#pragma unroll
          for (int i = 0; i < NC; ++i) s[n] = mfma32<F16>(kf[n][i], q[i], s[n]);
        }
      }
      // The values of 16 keys, as the first operand: 8 keys of a lane's column in the
      // order in which the lane holds their probabilities.
      auto values = [&](int g, uint4 (&vf)[ND]) {
        const int key = g * 16 + 4 * half + (lane & 15) / 4;  // and 8 further
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          const int chunk = 4 * d + 2 * ((lane >> 4) & 1) + (lane & 3) / 2, in = (lane & 1) * 8;
          const uint8_t* v0 = vt + key * RB + ((chunk ^ v_swizzle<RB>(key)) << 4) + in;
          const uint8_t* v1 = v0 + 8 * RB;                      // of the same permutation
          const shortx4 x0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4*)(v0));
          const shortx4 x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4*)(v1));
          const uint2 y0 = __builtin_bit_cast(uint2, x0), y1 = __builtin_bit_cast(uint2, x1);
          vf[d] = make_uint4(y0.x, y0.y, y1.x, y1.y);
        }
      };
      uint4 vf[2][ND];
      values(0, vf[0]);
      __builtin_amdgcn_sched_barrier(0);
      if (j0 + T > key1 || (masked && j0 + T > base)) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const int first = j0 + n * 32 + 4 * half;  // the key of this lane's first register
          const uint32_t seen = seen32(masked ? word : ~0ull, masked ? first - base : 0, key1 - first);
#pragma unroll
          for (int r = 0; r < 16; ++r) s[n][r] = (seen >> (8 * (r / 4) + r % 4)) & 1 ? s[n][r] : -INFINITY;
        }
      }
      // ---- softmax statistics and P^T
      float top = s[0][0];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, s[n][r]);
      top = swap32_max(top);
      // The subtracted logit follows the maximum only once that is kLag ahead.
      if (__any((top - m) * c > kLag<F16>)) {
        const float up = fmaxf(m, top);
        const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - up) * c);
        l *= f;
#pragma unroll
        for (int d = 0; d < ND; ++d) o[d] *= f;
        m = up;
        mc = up == -INFINITY ? 0.f : up * c - kLift<F16>;
        wide = __any(fabsf(mc) > kFine);
      }
      // s c - mc is off by the rounding of mc, by the same for all of a row, which cancels in the
      // quotient; but past kFine that may be more than the exponent range.
      float sub = mc;
      if (wide) {
        const float from = m == -INFINITY ? 0.f : m;
        sub = -kLift<F16>;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[n][r] -= from;
      }
      // Probabilities are rounded to the cache's type here, as the products take them (their
      // sum is of the unrounded ones): relative to sum p |v|, as large an error as that of rounding
      // the output, and in f16 that of kLift.
      uint4 pf[2 * NT];
      float sum = 0.f;  // a tile's, so that many small ones beside a large one reach l together
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        uint32_t w[8];
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
          const float p0 = __builtin_amdgcn_exp2f(fmaf(s[n][r], c, -sub));
          const float p1 = __builtin_amdgcn_exp2f(fmaf(s[n][r + 1], c, -sub));
          sum += p0 + p1;
          w[r / 2] = pack2<F16>(p0, p1);
        }
        pf[2 * n] = make_uint4(w[0], w[1], w[2], w[3]);
        pf[2 * n + 1] = make_uint4(w[4], w[5], w[6], w[7]);
      }
      l += sum;
      // ---- out^T += V^T P^T, 16 keys at a time, the next ones' values on the way
#pragma unroll
      for (int g = 0; g < 2 * NT; ++g) {
        if (g + 1 < 2 * NT) values(g + 1, vf[(g + 1) & 1]);
#pragma unroll
        for (int d = 0; d < ND; ++d) o[d] = mfma32<F16>(vf[g & 1][d], pf[g], o[d]);
      }
      if (careful && j0 + T > base) {
#pragma unroll 1
        for (int j = max(j0, base); j < min(j0 + T, key1); ++j) {
          const int key = j - j0;
          const uint16_t* v = reinterpret_cast<const uint16_t*>(v_src) + kv_slot(a.kv, b, j);
          float dot = 0.f;
#pragma unroll
          for (int i = 0; i < NC; ++i) {
            const uint4 kf = *reinterpret_cast<const uint4*>(kt + key * RB + (((2 * i + half) ^ row_swizzle<RB>(key)) << 4));
            const uint32_t kw4[4] = {kf.x, kf.y, kf.z, kf.w};
            uint32_t qw4[4] = {q[i].x, q[i].y, q[i].z, q[i].w};
            // converted here, not ahead of the loop: this path is rare and the registers are not
            asm volatile("" : "+v"(qw4[0]), "+v"(qw4[1]), "+v"(qw4[2]), "+v"(qw4[3]));
#pragma unroll
            for (int w = 0; w < 4; ++w)
              dot += half_to_f32<F16>(kw4[w] & 0xFFFF) * half_to_f32<F16>(qw4[w] & 0xFFFF) +
                     half_to_f32<F16>(kw4[w] >> 16) * half_to_f32<F16>(qw4[w] >> 16);
          }
          const float w = __builtin_amdgcn_exp2f(fmaf(swap32_sum(dot) - (wide && m != -INFINITY ? m : 0.f), c, -sub));
          const bool see = block_sees(word, j - base);
#pragma unroll
          for (int d = 0; d < ND; ++d) {
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
              const int e = 32 * d + 8 * (r / 4);
              if (e >= a.D) continue;
              const uint2 x = *reinterpret_cast<const uint2*>(v + e + 4 * half);
              const float x4[4] = {half_to_f32<F16>(x.x & 0xFFFF), half_to_f32<F16>(x.x >> 16),
                                   half_to_f32<F16>(x.y & 0xFFFF), half_to_f32<F16>(x.y >> 16)};
#pragma unroll
              for (int u = 0; u < 4; ++u) o[d][r + u] = see ? fmaf(w, x4[u], o[d][r + u]) : o[d][r + u];
            }
            asm volatile("" ::: "memory");  // a few loads in flight
          }
        }
      }
    }
    if (!masked || careful) break;
    bool odd = false;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) odd |= !(fabsf(o[d][r]) < INFINITY);
    if (!__syncthreads_or(odd)) break;
  }
  l = swap32_sum(l);

  // ---- join the key groups and write
  auto out_row = [&](int row) { return row / G * a.H + hk * G + row % G; };
  auto put = [&](int64_t out, int e, float4 x) {  // elements e..e+3 of a row's normalised sum
    if (p.part) {
      *reinterpret_cast<float4*>(p.part + (out * p.splits + split) * a.D + e) = x;
    } else {
      *reinterpret_cast<uint2*>(a.out + out * a.D + e) = make_uint2(pack2<F16>(x.x, x.y), pack2<F16>(x.z, x.w));
    }
  };
  auto put_lse = [&](int64_t out, float x) {
    if (p.part)
      p.part_lse[out * p.splits + split] = x;
    else if (a.lse)
      a.lse[out] = x;
  };
  if constexpr (KW == 1) {
    // Through LDS, 64 elements of a wavefront's rows at a time, so that stores cover whole lines:
    // from the registers a store would reach 32 rows with 32 bytes each (prefix of 16384 keys, 32768
    // rows: 336 us that way).  A row's 16-byte chunks are permuted by its number.
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int left = rows - rw * 32, out = out_row(row0 + min(rw * 32 + col, rows - 1));
    if (half == 0 && col < left) put_lse(out, l == 0.f ? -INFINITY : (mc + __builtin_amdgcn_logf(l)) * kLn2);
    float4* const turn = reinterpret_cast<float4*>(smem + rw * 8192);  // [32][16]
    __syncthreads();                               // the tiles have been read
#pragma unroll
    for (int e0 = 0; e0 < 32 * ND; e0 += 64) {
#pragma unroll
      for (int d = e0 / 32; d < ND && d < e0 / 32 + 2; ++d)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          const int chunk = 8 * (d % 2) + 2 * (r / 4) + half;
          turn[col * 16 + (chunk ^ (col & 15))] =
              make_float4(o[d][r] * inv, o[d][r + 1] * inv, o[d][r + 2] * inv, o[d][r + 3] * inv);
        }
      asm volatile("" ::: "memory");               // LDS works in order for a wavefront; so must the compiler
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int r = 4 * u + lane / 16, chunk = lane & 15, e = e0 + 4 * chunk;
        const float4 x = turn[r * 16 + (chunk ^ (r & 15))];
        const int to = __shfl(out, r, kWave);
        if (r < left && e < a.D) put(to, e, x);
      }
      asm volatile("" ::: "memory");
      __builtin_amdgcn_wave_barrier();
    }
  } else {
    float* const acc = reinterpret_cast<float*>(smem);                   // [KW][kRows][kOutRow]
    float* const stat = acc + KW * kRows * kOutRow;                      // [KW][kRows][2]
    __syncthreads();
    const int r0 = kw * kRows + rw * 32 + col;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        *reinterpret_cast<float4*>(acc + r0 * kOutRow + 32 * d + 8 * (r / 4) + 4 * half) =
            make_float4(o[d][r], o[d][r + 1], o[d][r + 2], o[d][r + 3]);
    if (half == 0) {
      stat[r0 * 2] = l == 0.f ? -INFINITY : mc;
      stat[r0 * 2 + 1] = l;
    }
    __syncthreads();
    for (int x = tid; x < rows * (ND * 8); x += 64 * RW * KW) {
      const int r = x / (ND * 8), e = x % (ND * 8) * 4;
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int w = 0; w < KW; ++w) M = fmaxf(M, stat[(w * kRows + r) * 2]);
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        const float mw = stat[(w * kRows + r) * 2];
        if (mw == -INFINITY) continue;             // no key seen
        const float f = __builtin_amdgcn_exp2f(mw - M);
        L += f * stat[(w * kRows + r) * 2 + 1];
        const float4 y = *reinterpret_cast<const float4*>(acc + (w * kRows + r) * kOutRow + e);
        sum.x += f * y.x;
        sum.y += f * y.y;
        sum.z += f * y.z;
        sum.w += f * y.w;
      }
      const float inv = L == 0.f ? 0.f : 1.f / L;
      if (e < a.D) put(out_row(row0 + r), e, make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv));
      if (e == 0) put_lse(out_row(row0 + r), L == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * kLn2);
    }
  }
}

// Joins the runs of a row, prefix and own.  One wavefront a row; a half takes
// every second run with four elements a lane, and four runs of a half are in
// flight.  What an empty run (log-sum-exp -inf) left in its sums is not used.
template <bool F16>
__global__ __launch_bounds__(256) void join_kernel(AttentionArgs a, AttnPlan p) {
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (row >= static_cast<int64_t>(a.B) * a.L * a.H) return;
  const float* part = p.part + row * p.splits * a.D;
  const float* lse = p.part_lse + row * p.splits;
  const int runs = p.splits;  // at most 128
  const float z0 = lane < runs ? lse[lane] : -INFINITY, z1 = lane + 64 < runs ? lse[lane + 64] : -INFINITY;
  const float M = wave_allmax(fmaxf(z0, z1)), sub = M == -INFINITY ? 0.f : M;
  // fmaxf passes over a NaN, the exponentials and their sum do not
  const float f0 = __builtin_amdgcn_exp2f((z0 - sub) * kLog2e), f1 = __builtin_amdgcn_exp2f((z1 - sub) * kLog2e);
  const float L = wave_allsum(f0 + f1);
  const int e = (lane & 31) * 4, at = min(e, a.D - 4);
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s = 0; s < runs; s += 8) {
    float4 x[4];
    float f[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int r = s + 2 * u + half;
      x[u] = *reinterpret_cast<const float4*>(part + static_cast<int64_t>(min(r, runs - 1)) * a.D + at);
      f[u] = __shfl(s < 64 ? f0 : f1, r & 63, kWave);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (f[u] == 0.f || s + 2 * u + half >= runs) continue;  // an empty run adds nothing
      o.x += f[u] * x[u].x;
      o.y += f[u] * x[u].y;
      o.z += f[u] * x[u].z;
      o.w += f[u] * x[u].w;
    }
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  o = make_float4(swap32_sum(o.x) * inv, swap32_sum(o.y) * inv, swap32_sum(o.z) * inv, swap32_sum(o.w) * inv);
  if (half == 0 && e < a.D)
    *reinterpret_cast<uint2*>(a.out + row * a.D + e) = make_uint2(pack2<F16>(o.x, o.y), pack2<F16>(o.z, o.w));
  if (lane == 0 && a.lse) a.lse[row] = L == 0.f ? -INFINITY : sub + __builtin_amdgcn_logf(L) * kLn2;
}

// The tile of a launch: rows, keys of a step of the whole workgroup, and the
// workgroups that the GPU holds at once (two a CU, but one of the 256-row tile).
// The smallest tile that holds the rows wastes the fewest of the matrix cores'
// rows; from 129 rows on the 256-row tile reads each key once where 128-row
// tiles read it twice (1365 rows over 1003 keys: 16 us against 25).
struct TileShape { int rows, keys, slots; };
constexpr TileShape kShapes[] = {{32, 64, 2 * kCUs}, {64, 64, 2 * kCUs}, {128, 64, 2 * kCUs}, {256, 64, kCUs}};
int shape_for(int64_t rows) { return rows <= 32 ? 0 : rows <= 64 ? 1 : rows <= 128 ? 2 : 3; }

struct CallPlan {
  AttnPlan p;
  int pre_shape, own_shape;  // -1: nothing to do
};

CallPlan make_plan(int B, int L, int H, int Hkv, int D, int prefix_len, int max_seq_len) {
  CallPlan c{};
  const int G = H / Hkv;
  c.pre_shape = c.own_shape = -1;
  if (prefix_len > 0) {
    const int64_t rows = static_cast<int64_t>(B) * L * G;
    c.pre_shape = shape_for(rows);
    const TileShape t = kShapes[c.pre_shape];
    c.p.pre_tiles = ceil_div(rows, t.rows);
    const Runs r = runs_of(prefix_len, static_cast<int64_t>(c.p.pre_tiles) * Hkv, t.keys, t.slots);
    c.p.pre_run = r.keys;
    c.p.pre_splits = r.count;
    c.p.pre_groups = Hkv * r.count;
  }
  if (max_seq_len > 0 || prefix_len == 0) {
    const int rows = L * G;
    c.own_shape = shape_for(rows);
    const TileShape t = kShapes[c.own_shape];
    c.p.own_tiles = ceil_div(rows, t.rows);
    const Runs r = runs_of(max_seq_len > 0 ? max_seq_len : 1, static_cast<int64_t>(B) * Hkv * c.p.own_tiles, t.keys,
                           t.slots);
    c.p.own_run = r.keys;
    c.p.own_splits = r.count;
    c.p.own_groups = B * Hkv * c.p.own_splits;
  }
  c.p.own_first = c.p.pre_splits;
  c.p.splits = c.p.pre_splits + c.p.own_splits;
  return c;
}

template <bool F16, int ND>
void launch_shape(int shape, const AttentionArgs& a, const AttnPlan& p, hipStream_t s) {
  const dim3 grid(tile_grid(p.pre_groups, p.pre_tiles) + tile_grid(p.own_groups, p.own_tiles));
  switch (shape) {
    case 0: hipLaunchKernelGGL((attend_kernel<F16, ND, 1, 2, 1>), grid, dim3(128), 0, s, a, p); break;
    case 1: hipLaunchKernelGGL((attend_kernel<F16, ND, 2, 2, 1>), grid, dim3(256), 0, s, a, p); break;
    case 2: hipLaunchKernelGGL((attend_kernel<F16, ND, 4, 1, 2>), grid, dim3(256), 0, s, a, p); break;
    default: hipLaunchKernelGGL((attend_kernel<F16, ND, 8, 1, 2>), grid, dim3(512), 0, s, a, p); break;
  }
}

template <bool F16>
void launch_join(const AttentionArgs& a, const AttnPlan& p, hipStream_t s) {
  const int64_t rows = static_cast<int64_t>(a.B) * a.L * a.H;
  hipLaunchKernelGGL(join_kernel<F16>, dim3(ceil_div(rows, 4)), dim3(256), 0, s, a, p);
}

template <bool F16>
void launch_all(const AttentionArgs& a, const CallPlan& c, hipStream_t s) {
  auto go = [&](int shape, const AttnPlan& p) {
    switch (head_slices(a.D)) {
      case 2: launch_shape<F16, 2>(shape, a, p, s); break;
      case 3: launch_shape<F16, 3>(shape, a, p, s); break;
      default: launch_shape<F16, 4>(shape, a, p, s); break;
    }
  };
  if (c.pre_shape == c.own_shape) {
    go(c.pre_shape, c.p);
  } else {
    AttnPlan pre = c.p, own = c.p;
    pre.own_groups = own.pre_groups = 0;
    if (c.pre_shape >= 0) go(c.pre_shape, pre);
    if (c.own_shape >= 0) go(c.own_shape, own);
  }
  if (c.p.part) launch_join<F16>(a, c.p, s);
}

}  // namespace

// Workspace: where rows have several runs, a log-sum-exp and D sums of each.
size_t attention_workspace_bytes(int B, int L, int H, int Hkv, int D, int prefix_len, int max_seq_len) {
  const CallPlan c = make_plan(B, L, H, Hkv, D, prefix_len, max_seq_len);
  if (c.p.splits <= 1) return 0;
  const size_t runs = static_cast<size_t>(B) * L * H * c.p.splits;
  return (runs + 3) / 4 * 16 + runs * D * sizeof(float);
}

void launch_attention(const AttentionArgs& a, bool f16, void* ws, hipStream_t s) {
  CallPlan c = make_plan(a.B, a.L, a.H, a.Hkv, a.D, a.prefix_len, a.max_seq_len);
  if (c.p.splits > 1) {
    const size_t runs = static_cast<size_t>(a.B) * a.L * a.H * c.p.splits;
    c.p.part_lse = static_cast<float*>(ws);
    c.p.part = c.p.part_lse + (runs + 3) / 4 * 4;
  }
  if (f16)
    launch_all<true>(a, c, s);
  else
    launch_all<false>(a, c, s);
}

// The prefix's part of a call whose own keys are another kernel's: runs 0 .. prefix_splits - 1 of `splits`.
int attention_prefix_splits(int B, int L, int H, int Hkv, int prefix_len) {
  return make_plan(B, L, H, Hkv, 0, prefix_len, 0).p.pre_splits;
}

void launch_attention_prefix(const AttentionArgs& a, bool f16, float* part, float* part_lse, int splits, hipStream_t s) {
  CallPlan c = make_plan(a.B, a.L, a.H, a.Hkv, a.D, a.prefix_len, 0);
  c.p.part = part;
  c.p.part_lse = part_lse;
  c.p.splits = splits;
  auto go = [&](auto type) {
    constexpr bool kF16 = type;
    switch (head_slices(a.D)) {
      case 2: launch_shape<kF16, 2>(c.pre_shape, a, c.p, s); break;
      case 3: launch_shape<kF16, 3>(c.pre_shape, a, c.p, s); break;
      default: launch_shape<kF16, 4>(c.pre_shape, a, c.p, s); break;
    }
  };
  f16 ? go(std::true_type{}) : go(std::false_type{});
}

void launch_attention_join(const AttentionArgs& a, bool f16, float* part, float* part_lse, int splits, hipStream_t s) {
  AttnPlan p{};
  p.part = part;
  p.part_lse = part_lse;
  p.splits = splits;
  f16 ? launch_join<true>(a, p, s) : launch_join<false>(a, p, s);
}

}  // namespace brisk
