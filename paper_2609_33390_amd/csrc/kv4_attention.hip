// Attention of a block over a shared prefix and a cache held in 4 bits.
//
// With key j held as z_j + s_j c_j and value j as y_j + r_j d_j, per head:
//   a_j = scale (s_j <q, c_j> + z_j sum_d q_d),   p_j = exp(a_j - m)
//   out = (sum_j (p_j r_j) (d_j - 8) + sum_j p_j (y_j + 8 r_j)) / sum_j p_j
// The matrix instructions work on the codes alone, whole numbers that their types
// hold exactly; steps and lowest values meet the logits and the probabilities in
// fp32.  A bf16 code is made with one instruction for two of them, by putting its
// bits under an exponent (16 + c, 128 + d), and the 16 and 128 are taken out again:
// from the logits through the lowest value, from the sums (with the 8) through the sum
// of the rounded weights.  An f16 code is its own bits, a subnormal number (8 c and d or
// 16 d times 2^-24), whose power of two the scale and the last step take out.
//
// Codes come from memory to registers in operand order, 32 slots of a head a step
// of a wavefront, the next ones' on the way; the wavefronts of a workgroup take
// steps in turn and join through LDS.
#include <algorithm>
#include <cmath>

#include "attention_plan.h"
#include "kernels.h"
#include "kv4_common.h"

namespace brisk {

namespace {

constexpr int kCUs = 256;
// As in the attention over 2-byte caches: the subtracted logit may be kLag behind the maximum (in base
// 2).  Weights are further divided by 2^unit, the same for all rows of a wavefront, which the
// sum of the probabilities shares: in f16 the largest step seen, so that f16's range is used from
// the top (times 2^12, so at most 2^15); in bf16 only what keeps steps past 2^60 from
// overflowing sums.
template <bool F16> constexpr float kLag = F16 ? 3.f : 8.f;
template <bool F16> constexpr int kTop = F16 ? 12 : 0;
template <bool F16> constexpr int kLeastUnit = F16 ? -24 : 0;
constexpr float kFine = 0x1p20f;

struct Kv4Plan {
  float* part;           // [rows][splits][D], null when every row has one run
  float* part_lse;       // [rows][splits]
  int groups, tiles, run;  // (sequence, head, split) triples, row tiles, slots of a run
  int splits, own_first;
  int by_length;         // whether long sequences go first
};

// What the sum of the rounded weights is times, in `add`: weights are of codes about 8, so that their
// rounding counts by how far a value lies from the middle of its head's range, not from the lowest one
// (64 caches of 500 to 8000 keys: outputs off by 0.0046 from that, by 0.0022 from this); bf16
// codes stand on 128 besides.
template <bool F16> constexpr float kMiddle = F16 ? 8.f : 136.f;

// acc - kMiddle times the sum of a pair.
template <bool F16>
__device__ __forceinline__ float less_middle(uint32_t pair, float acc) {
  if constexpr (F16) {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(h2, pair), h2{-8, -8}, acc, false);
  } else {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(b2, pair), __builtin_bit_cast(b2, 0xC308C308u), acc, false);
  }
}

// c + A B for A [16, 32] and B [32, 16]: lane l holds elements 8 (l / 16) .. + 7 of row (column)
// l % 16; register r of c is row 4 (l / 16) + r, column l % 16.
template <bool F16>
__device__ __forceinline__ floatx4 mfma16(uint4 a, uint4 b, floatx4 c) {
  if constexpr (F16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// The masks of the codes in vector registers and what they stand on in scalar ones: an and-or takes
// no literals, and one scalar operand.
struct CodeBits {
  uint32_t key = 0x00780078, value = 0x000F000F, key_base = 0x41804180, value_base = 0x43004300;
  __device__ __forceinline__ CodeBits() {
    asm("" : "+v"(key));
    asm("" : "+v"(value));
    asm("" : "+s"(key_base));
    asm("" : "+s"(value_base));
  }
};

// Eight codes of a key: 16 + c in bf16, 8 c 2^-24 in f16.
template <bool F16>
__device__ __forceinline__ uint4 key_codes(uint32_t w, const CodeBits& k) {
  const uint32_t w1 = w >> 4, w2 = w >> 8, w3 = __builtin_amdgcn_alignbit(w, w, 12);
  if constexpr (F16) return make_uint4(w & k.key, w1 & k.key, w2 & k.key, w3 & k.key);
  return make_uint4((w & k.key) | k.key_base, (w1 & k.key) | k.key_base, (w2 & k.key) | k.key_base, (w3 & k.key) | k.key_base);
}

// Nibble j of both halves of a word of values: 128 + d in bf16, d 2^-24 or (odd j) 16 d 2^-24 in f16.
template <bool F16, int J>
__device__ __forceinline__ uint32_t value_codes(uint32_t w, const CodeBits& k) {
  if constexpr (F16) return (w >> (J / 2 * 8)) & (J % 2 ? k.value << 4 : k.value);
  return ((w >> (4 * J)) & k.value) | k.value_base;
}

// Which of four slots a row sees, the first one `at` slots past the block's begin and `left` before the end.
__device__ __forceinline__ uint32_t seen4(uint64_t word, int at, int left) {
  const uint64_t bits = at >= 64 ? 0 : at >= 0 ? word >> at : at > -4 ? (word << -at) | ((1ull << -at) - 1) : ~0ull;
  return static_cast<uint32_t>(bits) & (left >= 4 ? 15u : left <= 0 ? 0u : (1u << left) - 1);
}

__device__ __forceinline__ uint32_t part_of(uint4 v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// RT tiles of 16 rows a workgroup, KW wavefronts.
template <bool F16, int W, int RT, int KW>
__global__ __launch_bounds__(64 * KW, RT == 1 ? 4 : 2) void kv4_attend_kernel(Kv4AttentionArgs a, Kv4Plan p) {
  constexpr int M = 16 * RT, NF = W / 32, NO = W / 16, kStep = 32;
  constexpr int kAhead = 1;                        // steps on their way
  constexpr int kLooked = 31;                      // steps whose pages are looked up at once, besides those ahead
  constexpr int kOutRow = W + 4;
  __shared__ __attribute__((aligned(16))) float acc[KW * M * kOutRow];
  __shared__ float stat[KW * M * 2];
  __shared__ __attribute__((aligned(16))) float2 marks[KW * 64];     // (step, lowest) of a step's keys and values

  const int tid = threadIdx.x, lane = tid & 63, t = lane >> 4, x = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = a.H / a.Hkv;
  const int bid = blockIdx.x, group = bid / 8 / p.tiles * 8 + bid % 8, tile = bid / 8 % p.tiles;
  if (group >= p.groups) return;
  // first runs of all sequences, then second ones, ...: later runs are fewer where lengths differ
  const int hk = group % a.Hkv;
  int b = group / a.Hkv % a.B, split = group / a.Hkv / a.B;
  if (p.by_length) {                               // the b-th longest sequence, of at most 64
    const int len = lane < a.B ? kv4_len(a.kv, lane, a.max_seq_len) : -1;
    int before = 0;
    for (int i = 0; i < a.B; ++i) {
      const int other = __builtin_amdgcn_readlane(len, i);
      before += other > len || (other == len && i < lane);
    }
    b = __builtin_ctzll(__ballot(before == b));
  }
  const int n = kv4_len(a.kv, b, a.max_seq_len);
  const int key0 = split * p.run, key1 = min(n, key0 + p.run), base = n - a.L;
  const int row0 = b * a.L * G + tile * M, rows = min(M, a.L * G - tile * M);
  split += p.own_first;
  if (key0 >= n && p.part) {                       // a run past the sequence: the join reads that it is empty
    for (int r = tid; r < rows; r += 64 * KW) {
      const int row = row0 + r;
      p.part_lse[(static_cast<int64_t>(row / G) * a.H + hk * G + row % G) * p.splits + split] = -INFINITY;
    }
    return;
  }
  const bool masked = a.mask != nullptr;

  // ---- queries, as the second operand of K Q^T: row x of each tile, elements t W / 4 + ...
  uint4 q[RT][NF];
  // f16 logits are held 2^-21 of what they are
  const float c = a.scale * kLog2e * (F16 ? 0x1p21f : 1.f);
  float qz[RT];                                    // sum of q, as the logits are held
  // what a row sees of the block; one tile, short of registers, reads it where it is used
  uint64_t word[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int row = row0 + min(16 * r + x, rows - 1), bi = row / G;
    const uint16_t* src = a.q + bi * a.q_row_stride + (hk * G + row % G) * a.q_head_stride;
    word[r] = RT > 1 && masked ? a.mask[bi] : ~0ull;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NF; ++i) {
      const int e = t * (W / 4) + 8 * i;
      q[r][i] = e < a.D ? *reinterpret_cast<const uint4*>(src + e) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int w = 0; w < 4; ++w)
        sum += half_to_f32<F16>(part_of(q[r][i], w) & 0xFFFF) + half_to_f32<F16>(part_of(q[r][i], w) >> 16);
    }
    sum = swap32_sum(swap16_sum(sum));
    qz[r] = F16 ? sum * 0x1p-21f : sum;
  }

  // ---- loads.  Step i of this wavefront begins at slot key0 + 32 (KW i + wave).  Pages are looked up for kLooked
  // steps and those ahead of them at once, block k of the i-th by lane 2 i + k, while the steps before are worked on.
  const int last = max(key1 - 1, 0) & ~(kKv4Block - 1);
  const int64_t table = static_cast<int64_t>(b) * a.kv.max_pages;
  const int my0 = key0 + kStep * wave;
  auto pages_of = [&](int step) {
    return a.kv.table[table + (min(my0 + kStep * KW * (step + lane / 2) + kKv4Block * (lane & 1), last) >> a.kv.page_shift)];
  };
  const uint8_t* const head = a.kv.pages + hk * a.kv.head_stride;
  auto block = [&](int held, int nth, int step, int k) {
    const int page = clamp_id(__builtin_amdgcn_readlane(held, 2 * nth + k), a.kv.n_pages);
    const int j = min(my0 + kStep * KW * step + kKv4Block * k, last);
    return head + page * a.kv.page_stride + (j & ((1 << a.kv.page_shift) - 1)) / kKv4Block * kv4_block_bytes(W);
  };
  typedef uint32_t Codes __attribute__((ext_vector_type(W / 32)));
  // chunk `lane` of a block's keys or values: a wavefront reads them in one piece
  auto codes = [&](const uint8_t* blk) { return *reinterpret_cast<const Codes*>(blk + lane * static_cast<uint32_t>(sizeof(Codes))); };
  // the pair of key lane % 32 in the lower lanes, of value lane % 32 in the upper ones
  auto mark_of = [&](const uint8_t* b0, const uint8_t* b1) {
    return *reinterpret_cast<const uint32_t*>((lane & 16 ? b1 : b0) + static_cast<uint32_t>(16 * W + (lane & 32 ? 64 : 0) + 4 * x));
  };

  floatx4 o[RT][NO];
  // m: the subtracted logit (unscaled); mc = c m - lift, lift = kTop - unit; l: this lane's part of the
  // sum of the weights; add: its part of what joins every element of the output
  float m[RT], mc[RT], l[RT], add[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    m[r] = -INFINITY;
    mc[r] = l[r] = add[r] = 0.f;
#pragma unroll
    for (int d = 0; d < NO; ++d) o[r][d] = floatx4{};
  }
  int unit = kLeastUnit<F16>;
  float limit = lane & 32 ? __builtin_ldexpf(1.f, F16 ? unit : unit + 60) : INFINITY;  // of a value's size within that unit
  bool wide = false;                               // a row's mc is past kFine (the same in all lanes)
  float2* const my_marks = marks + 64 * wave;
  // what joins a slot's lowest value, in steps: of a value the middle of its codes, of a key less what bf16 codes
  // stand on
  const float middle = lane & 32 ? 8.f : F16 ? 0.f : -16.f;
  const CodeBits bits;

  const int steps = key1 > my0 ? (key1 - my0 + kStep * KW - 1) / (kStep * KW) : 0;
  if (steps > 0) {
    int held = pages_of(0);
    const uint8_t *blk[kAhead][2];
    Codes k[kAhead][2], v[kAhead][2];
    uint32_t mark[kAhead];
    each_index<kAhead>([&](auto index) {
      constexpr int s = index;
      blk[s][0] = block(held, s, s, 0);
      blk[s][1] = block(held, s, s, 1);
      k[s][0] = codes(blk[s][0]);
      k[s][1] = codes(blk[s][1]);
      mark[s] = mark_of(blk[s][0], blk[s][1]);
      __builtin_amdgcn_sched_barrier(0);           // in the order in which the loop has them on their way
      v[s][0] = codes(blk[s][0] + 8 * W);
      v[s][1] = codes(blk[s][1] + 8 * W);
      __builtin_amdgcn_sched_barrier(0);
    });
    // One step, from register set s, which then gets the step kAhead later.
    auto attend = [&](auto set, int step, int nth) {
      constexpr int s = set;
      const int j0 = my0 + kStep * KW * step;
      // ---- S^T = K Q^T over the codes: register u of block i is slot 16 i + 4 t + u
      floatx4 z[RT][2];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int f = 0; f < NF; ++f) {
          const uint4 kf = key_codes<F16>(k[s][i][f], bits);
#pragma unroll
          for (int r = 0; r < RT; ++r) z[r][i] = mfma16<F16>(kf, q[r][f], f == 0 ? floatx4{} : z[r][i]);
        }
      // ---- steps and lowest values: one slot a lane, handed round through LDS
      {
        float st = kv4_step<F16>(mark[s]), y = kv4_low<F16>(mark[s]);
        if (j0 + kStep > key1 && j0 + (lane & 31) >= key1) st = y = 0.f;   // what lies past the run may be anything
        const float size = fmaxf(st, fabsf(y) * 0.0625f);
        my_marks[lane] = make_float2(st, fmaf(middle, st, y));
        if (__any(size > limit)) {
          const float finite = lane & 32 && size < INFINITY ? size : 0.f;
          const int grown = max(unit, __builtin_amdgcn_frexp_expf(wave_allmax(finite)) - (F16 ? 0 : 60));
          const float f = __builtin_ldexpf(1.f, unit - grown);
#pragma unroll
          for (int r = 0; r < RT; ++r) {
            l[r] *= f;
            add[r] *= f;
#pragma unroll
            for (int d = 0; d < NO; ++d) o[r][d] *= f;
            mc[r] = m[r] == -INFINITY ? 0.f : m[r] * c - static_cast<float>(kTop<F16> - grown);
          }
          unit = grown;
          limit = lane & 32 ? __builtin_ldexpf(1.f, F16 ? unit : unit + 60) : INFINITY;
        }
      }
      asm volatile("" ::: "memory");               // LDS works in order for a wavefront; so must the compiler
      __builtin_amdgcn_wave_barrier();
      // ---- the keys of a later step
      blk[s][0] = block(held, nth + kAhead, step + kAhead, 0);
      blk[s][1] = block(held, nth + kAhead, step + kAhead, 1);
      k[s][0] = codes(blk[s][0]);
      k[s][1] = codes(blk[s][1]);
      mark[s] = mark_of(blk[s][0], blk[s][1]);
      __builtin_amdgcn_sched_barrier(0);

      // slots 16 i + 4 t + 2 u and the next one; a block's at a time, for want of registers
      auto pairs = [&](int of, int i, int u) { return *reinterpret_cast<const float4*>(my_marks + of + 16 * i + 4 * t + 2 * u); };
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const float4 p = pairs(0, i, u);
#pragma unroll
          for (int r = 0; r < RT; ++r) {
            z[r][i][2 * u] = fmaf(p.x, z[r][i][2 * u], p.y * qz[r]);
            z[r][i][2 * u + 1] = fmaf(p.z, z[r][i][2 * u + 1], p.w * qz[r]);
          }
        }
        if (RT == 1) __builtin_amdgcn_sched_barrier(0);
      }
      const bool cut = j0 + kStep > key1 || (masked && j0 + kStep > base);
      uint32_t seen[RT];                           // bit 4 i + u: slot 16 i + 4 t + u
      if (cut) {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          seen[r] = 0;
          if (RT == 1 && masked) word[0] = a.mask[(row0 + min(x, rows - 1)) / G];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int first = j0 + 16 * i + 4 * t;
            seen[r] |= seen4(word[r], masked ? first - base : 0, key1 - first) << (4 * i);
#pragma unroll
            for (int u = 0; u < 4; ++u) z[r][i][u] = (seen[r] >> (4 * i + u)) & 1 ? z[r][i][u] : -INFINITY;
          }
        }
      }
      // ---- softmax statistics.  The subtracted logit follows the maximum only once that is kLag ahead.
      float top[RT];
      bool behind = false;
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        top[r] = z[r][0][0];
#pragma unroll
        for (int i = 1; i < 8; ++i) top[r] = fmaxf(top[r], z[r][i / 4][i % 4]);
        behind |= (top[r] - m[r]) * c > kLag<F16>;
      }
      if (__any(behind)) {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          const float up = fmaxf(m[r], swap32_max(swap16_max(top[r])));
          const float f = m[r] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m[r] - up) * c);
          l[r] *= f;
          add[r] *= f;
#pragma unroll
          for (int d = 0; d < NO; ++d) o[r][d] *= f;
          m[r] = up;
          mc[r] = up == -INFINITY ? 0.f : up * c - static_cast<float>(kTop<F16> - unit);
        }
        bool far = false;
#pragma unroll
        for (int r = 0; r < RT; ++r) far |= fabsf(mc[r]) > kFine;
        wide = __any(far);
      }
      float sub[RT];
#pragma unroll
      for (int r = 0; r < RT; ++r) sub[r] = mc[r];
      if (wide) {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          const float from = m[r] == -INFINITY ? 0.f : m[r];
          sub[r] = static_cast<float>(unit - kTop<F16>);
#pragma unroll
          for (int i = 0; i < 8; ++i) z[r][i / 4][i % 4] -= from;
        }
      }
      // ---- weights.  p s is rounded to the cache's type, as the products take it; the sums of p and
      // p y are of unrounded numbers.
      uint32_t w[RT][4];
      float sum[RT], lows[RT];
#pragma unroll
      for (int r = 0; r < RT; ++r) sum[r] = lows[r] = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 both = pairs(32, i / 2, i % 2);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          float4 y = both;
          if (cut) {                               // what a row does not see may hold anything
            const bool see0 = (seen[r] >> (2 * i)) & 1, see1 = (seen[r] >> (2 * i + 1)) & 1;
            y = make_float4(see0 ? y.x : 0.f, see0 ? y.y : 0.f, see1 ? y.z : 0.f, see1 ? y.w : 0.f);
          }
          const float p0 = __builtin_amdgcn_exp2f(fmaf(z[r][i / 2][2 * (i % 2)], c, -sub[r]));
          const float p1 = __builtin_amdgcn_exp2f(fmaf(z[r][i / 2][2 * (i % 2) + 1], c, -sub[r]));
          sum[r] += p0 + p1;
          lows[r] = fmaf(p0, y.y, fmaf(p1, y.w, lows[r]));
          w[r][i] = pack2<F16>(p0 * y.x, p1 * y.z);
          lows[r] = less_middle<F16>(w[r][i], lows[r]);
        }
        if (RT == 1 && i == 1) __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        l[r] += sum[r];
        add[r] += lows[r];
      }
      asm volatile("" ::: "memory");
      __builtin_amdgcn_wave_barrier();
      // ---- out^T += D^T W^T over the codes
      each_index<NO>([&](auto index) {
        constexpr int d = index, y = 2 * (d / 4), j = d % 4;
        const uint4 f = make_uint4(value_codes<F16, j>(v[s][0][y], bits), value_codes<F16, j>(v[s][0][y + 1], bits),
                                   value_codes<F16, j>(v[s][1][y], bits), value_codes<F16, j>(v[s][1][y + 1], bits));
#pragma unroll
        for (int r = 0; r < RT; ++r) o[r][d] = mfma16<F16>(f, make_uint4(w[r][0], w[r][1], w[r][2], w[r][3]), o[r][d]);
      });
      v[s][0] = codes(blk[s][0] + 8 * W);
      v[s][1] = codes(blk[s][1] + 8 * W);
      __builtin_amdgcn_sched_barrier(0);
    };
    for (int step0 = 0; step0 < steps; step0 += kLooked) {
      const int held_next = pages_of(step0 + kLooked), end = min(steps - step0, kLooked);
      for (int nth = 0; nth < end; ++nth) {
        attend(std::integral_constant<int, 0>{}, step0 + nth, nth);
        if constexpr (kAhead == 2) {
          if (++nth >= end) break;
          attend(std::integral_constant<int, 1>{}, step0 + nth, nth);
        }
      }
      held = held_next;
    }
  }

  // ---- join the wavefronts and write
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int at = wave * M + 16 * r + x;
    const float total = swap32_sum(swap16_sum(l[r])), all = swap32_sum(swap16_sum(add[r]));
    each_index<NO>([&](auto index) {
      constexpr int d = index;
      constexpr float f = !F16 ? 1.f : d % 2 ? 0x1p20f : 0x1p24f;
      *reinterpret_cast<float4*>(acc + at * kOutRow + 16 * d + 4 * t) =
          make_float4(fmaf(o[r][d][0], f, all), fmaf(o[r][d][1], f, all), fmaf(o[r][d][2], f, all), fmaf(o[r][d][3], f, all));
    });
    if (t == 0) {
      stat[at * 2] = total == 0.f ? -INFINITY : mc[r];
      stat[at * 2 + 1] = total;
    }
  }
  __syncthreads();
  for (int i = tid; i < rows * (W / 4); i += 64 * KW) {
    const int r = i / (W / 4), e = i % (W / 4) * 4;
    float top = -INFINITY, total = 0.f;
#pragma unroll
    for (int w = 0; w < KW; ++w) top = fmaxf(top, stat[(w * M + r) * 2]);
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      const float mw = stat[(w * M + r) * 2];
      if (mw == -INFINITY) continue;               // no key seen
      const float f = __builtin_amdgcn_exp2f(mw - top);
      total += f * stat[(w * M + r) * 2 + 1];
      const float4 y = *reinterpret_cast<const float4*>(acc + (w * M + r) * kOutRow + e);
      sum.x += f * y.x;
      sum.y += f * y.y;
      sum.z += f * y.z;
      sum.w += f * y.w;
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
    const int row = row0 + r;
    const int64_t out = static_cast<int64_t>(row / G) * a.H + hk * G + row % G;
    if (e < a.D) {
      if (p.part)
        *reinterpret_cast<float4*>(p.part + (out * p.splits + split) * a.D + e) =
            make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv);
      else
        *reinterpret_cast<uint2*>(a.out + out * a.D + e) =
            make_uint2(pack2<F16>(sum.x * inv, sum.y * inv), pack2<F16>(sum.z * inv, sum.w * inv));
    }
    if (e == 0) {
      const float lse = total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * kLn2;
      if (p.part)
        p.part_lse[out * p.splits + split] = lse;
      else if (a.lse)
        a.lse[out] = lse;
    }
  }
}

// A launch's rows a tile, and the workgroups that the GPU holds at once.
struct Shape { int rows, waves, slots; };
Shape shape_for(int64_t rows) { return rows <= 16 ? Shape{16, 4, 4 * kCUs} : Shape{32, 4, 2 * kCUs}; }

// Runs of the own keys.  A workgroup's start, its join and the partial sums of its rows, written and read
// again, count as `start` keys.  One sequence's runs are of one length, and take rounds of workgroups.
// Sequences differ in lengths that are not known here: the last workgroup to end then has at most a run
// more than its share of all.
Runs kv4_runs(int keys, int B, int64_t whole, Shape shape, int rows) {
  const int step = 32 * shape.waves;
  const double start = 500. + 24. * rows;
  Runs best{};
  double least = 1e300;
  for (int s = 1; s <= 64; ++s) {
    const int run = ceil_div(ceil_div(keys, s), step) * step, count = ceil_div(keys, run);
    if (s > 1 && whole * count > kMostRuns) break;
    const double rounds = static_cast<double>(whole * count) / shape.slots;
    const double cost = (count > 1 ? 128. : 0.) + (B == 1 ? std::ceil(rounds) * (run + start) : run + start * std::max(1., rounds));
    if (cost < least) {
      least = cost;
      best = {count, run};
    }
  }
  return best;
}

struct CallPlan {
  Kv4Plan p;
  int pre_splits;
};

CallPlan make_plan(int B, int L, int H, int Hkv, int prefix_len, int max_seq_len) {
  CallPlan c{};
  c.pre_splits = prefix_len > 0 ? attention_prefix_splits(B, L, H, Hkv, prefix_len) : 0;
  if (max_seq_len > 0 || prefix_len == 0) {
    const int rows = L * (H / Hkv);
    const Shape s = shape_for(rows);
    c.p.tiles = ceil_div(rows, s.rows);
    const Runs r = kv4_runs(max_seq_len > 0 ? max_seq_len : 1, B, static_cast<int64_t>(B) * Hkv * c.p.tiles, s, std::min(rows, s.rows));
    c.p.run = r.keys;
    c.p.groups = B * Hkv * r.count;
    c.p.splits = r.count;
    c.p.by_length = r.count == 1 && B > 1 && B <= 64 && B * Hkv * c.p.tiles > s.slots;
  }
  c.p.own_first = c.pre_splits;
  c.p.splits += c.pre_splits;
  return c;
}

template <bool F16, int W>
void launch_own(const Kv4AttentionArgs& a, const Kv4Plan& p, hipStream_t s) {
  const dim3 grid((p.groups + 7) / 8 * 8 * p.tiles);
  switch (shape_for(static_cast<int64_t>(a.L) * (a.H / a.Hkv)).rows) {
    case 16: hipLaunchKernelGGL((kv4_attend_kernel<F16, W, 1, 4>), grid, dim3(256), 0, s, a, p); break;
    default: hipLaunchKernelGGL((kv4_attend_kernel<F16, W, 2, 4>), grid, dim3(256), 0, s, a, p); break;
  }
}

}  // namespace

// Workspace: where rows have several runs, a log-sum-exp and D sums of each.
size_t kv4_attention_workspace_bytes(int B, int L, int H, int Hkv, int D, int prefix_len, int max_seq_len) {
  const CallPlan c = make_plan(B, L, H, Hkv, prefix_len, max_seq_len);
  if (c.p.splits <= 1) return 0;
  const size_t runs = static_cast<size_t>(B) * L * H * c.p.splits;
  return (runs + 3) / 4 * 16 + runs * D * sizeof(float);
}

void launch_kv4_attention(const Kv4AttentionArgs& a, const AttentionArgs& pre, bool f16, void* ws, hipStream_t s) {
  CallPlan c = make_plan(a.B, a.L, a.H, a.Hkv, pre.prefix_len, a.max_seq_len);
  if (c.p.splits > 1) {
    const size_t runs = static_cast<size_t>(a.B) * a.L * a.H * c.p.splits;
    c.p.part_lse = static_cast<float*>(ws);
    c.p.part = c.p.part_lse + (runs + 3) / 4 * 4;
  }
  if (c.pre_splits) launch_attention_prefix(pre, f16, c.p.part, c.p.part_lse, c.p.splits, s);
  if (c.p.groups) {
    const bool wide = kv4_width(a.D) == 128;
    if (f16)
      wide ? launch_own<true, 128>(a, c.p, s) : launch_own<true, 64>(a, c.p, s);
    else
      wide ? launch_own<false, 128>(a, c.p, s) : launch_own<false, 64>(a, c.p, s);
  }
  if (c.p.part) launch_attention_join(pre, f16, c.p.part, c.p.part_lse, c.p.splits, s);
}

}  // namespace brisk
