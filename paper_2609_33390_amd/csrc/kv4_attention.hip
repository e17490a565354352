// Attention of a block over a shared prefix and a cache held in 4 bits.
//
// With key j held as z_j + s_j c_j and value j as y_j + r_j d_j, per head:
//   a_j = scale (s_j <q, c_j> + z_j sum_d q_d),   p_j = exp(a_j - m)
//   out = (sum_j (p_j r_j) (d_j - 8) + sum_j p_j (y_j + 8 r_j)) / sum_j p_j
// The matrix instructions work on the codes alone, whole numbers that their types
// hold exactly; steps and lowest values meet the logits and the probabilities in
// fp32.  Two codes are made with one instruction, by putting their bits under an exponent
// (bf16 16 + c and 128 + d, f16 64 + d), and the 16, 128 and 64 are taken out again:
// from the logits through the lowest value, from the sums (with the 8) through the sum
// of the rounded weights.  An f16 key's code is its own bits, a subnormal number (8 c times
// 2^-24), whose power of two the scale takes out.  Sums over such numbers are truncated
// early, at about 2^-17 of the largest factor: logits have room for that, but outputs over long
// caches had not (45000 slots of which 50 count: 4.9e-4 off, all to one side, where 2.6e-4 is
// what the roundings of weights and outputs cost).
//
// Codes come from memory to registers in operand order, 32 slots of a head a step
// of a wavefront, the next ones' on the way; the wavefronts of a workgroup take
// steps in turn and join through LDS.
//
// What bounds it.  Single tokens of a batch: the read of the cache (64 caches of 500 to 8000 slots of 8 heads, 296 MB in
// 51 us, 5.8 TB/s).  32 rows: vector instructions, 290 a step (56 make the keys' codes, 56 the values', 32 take steps and lowest
// values to the logits, 104 make the weights and their sums) beside its 32 products.  Of the cycles in which a CU has
// wavefronts its SIMDs spend 68% on them and 25% on products, a third of those beside vector instructions; 17% on neither (64
// blocks of 16 over 16 to 4096 slots: 62 us, 0.55 PFLOP/s).  64 rows a wavefront make the codes once for twice as many: 63% and
// 30% (one block of 32 over 65568 slots: 50 us, 0.69 PFLOP/s; with the join 55, with tiles of 32 rows 60).
// A wavefront's 800 instructions before and after its steps count as two or three of them.
#include <algorithm>
#include <cmath>
#include <iterator>
#include <type_traits>

#include "attention_plan.h"
#include "kernels.h"
#include "kv4_common.h"

namespace brisk {

namespace {

// As in the attention over 2-byte caches: the subtracted logit may be kLag behind the maximum (in base
// 2).  A row's weights are further divided by 2^unit, which the sum of the probabilities shares: in f16 the
// largest step of the values that it sees, so that f16's range is used from the top (times 2^12, so at most 2^15,
// and a weight times a step is off by at most 2^-36 of the largest step besides its rounding); in bf16 only what
// keeps steps past 2^60 from overflowing sums.
template <bool F16> constexpr float kLag = F16 ? 3.f : 8.f;
template <bool F16> constexpr int kTop = F16 ? 12 : 0;
template <bool F16> constexpr int kLeastUnit = F16 ? -24 : 0;
constexpr float kFine = 0x1p20f;

struct Kv4Plan {
  float* part;           // [rows][splits][D], null when every row has one run
  float* part_lse;       // [rows][splits]
  int groups, tiles, run;  // (sequence, head, split) triples, row tiles, slots of a run
  int splits, own_first;
  int by_length;         // whether long runs go first
};

// What the sum of the rounded weights is times, in `add`: weights are of codes about 8, so that their
// rounding counts by how far a value lies from the middle of its head's range, not from the lowest one
// (64 caches of 500 to 8000 keys: outputs off by 0.0046 from that, by 0.0022 from this); bf16
// codes stand on 128 besides, f16 ones on 64.
template <bool F16> constexpr float kMiddle = F16 ? 72.f : 136.f;

// acc + f times the sum of a pair; f is a number of the type.
template <bool F16>
__device__ __forceinline__ float plus_pair(uint32_t pair, float f, float acc) {
  if constexpr (F16) {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    const auto g = static_cast<_Float16>(f);
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(h2, pair), h2{g, g}, acc, false);
  } else {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    const auto g = static_cast<__bf16>(f);
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(b2, pair), b2{g, g}, acc, false);
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
template <bool F16>
struct CodeBits {
  uint32_t key = 0x00780078, value = F16 ? 0x00F000F0 : 0x000F000F;
  uint32_t key_base = 0x41804180, value_base = F16 ? 0x54005400 : 0x43004300;
  __device__ __forceinline__ CodeBits() {
    asm("" : "+v"(key));
    asm("" : "+v"(value));
    asm("" : "+s"(key_base));
    asm("" : "+s"(value_base));
  }
};

// Eight codes of a key: 16 + c in bf16, 8 c 2^-24 in f16.
template <bool F16>
__device__ __forceinline__ uint4 key_codes(uint32_t w, const CodeBits<F16>& k) {
  const uint32_t w1 = w >> 4, w2 = w >> 8, w3 = __builtin_amdgcn_alignbit(w, w, 12);
  if constexpr (F16) return make_uint4(w & k.key, w1 & k.key, w2 & k.key, w3 & k.key);
  return make_uint4((w & k.key) | k.key_base, (w1 & k.key) | k.key_base, (w2 & k.key) | k.key_base, (w3 & k.key) | k.key_base);
}

// Nibble j of both halves of a word of values: 128 + d in bf16, 64 + d in f16.
template <bool F16, int J>
__device__ __forceinline__ uint32_t value_codes(uint32_t w, const CodeBits<F16>& k) {
  constexpr int right = 4 * (F16 ? J - 1 : J);
  return ((right < 0 ? w << 4 : w >> (right < 0 ? 0 : right)) & k.value) | k.value_base;
}

__device__ __forceinline__ float uniform(float v) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v))); }

// Which of four slots a row sees, the first one `at` slots past the block's begin and `left` before the end.
__device__ __forceinline__ uint32_t seen4(uint64_t word, int at, int left) {
  const uint64_t bits = at >= 64 ? 0 : at >= 0 ? word >> at : at > -4 ? (word << -at) | ((1ull << -at) - 1) : ~0ull;
  return static_cast<uint32_t>(bits) & (left >= 4 ? 15u : left <= 0 ? 0u : (1u << left) - 1);
}

__device__ __forceinline__ uint32_t part_of(uint4 v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// v where the banks (four lanes each of a row of 16) of `BANKS` have it, old elsewhere.
template <int BANKS>
__device__ __forceinline__ float in_banks(float old, float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, old), __builtin_bit_cast(int, v), 0xE4, 0xF, BANKS, false));
}
// v of the lane N further in the row of 16 (SHIFT 0x100: the last ones get 0; 0x120: round the row).
template <int SHIFT, int N>
__device__ __forceinline__ uint32_t along_row(uint32_t v) {
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), SHIFT + N, 0xF, 0xF, true));
}
template <int N> __device__ __forceinline__ float round_row(float v) { return __uint_as_float(along_row<0x120, N>(__float_as_uint(v))); }

// v, and what is made of it made where it is used: four tiles' registers are not enough to hold it over the loop, and a
// reload of what spilled waits for the codes on their way.
template <bool SHORT>
__device__ __forceinline__ int anew(int v) {
  if constexpr (SHORT) asm volatile("" : "+v"(v));
  return v;
}

// Over the lanes that share a row: the four quarters and, of a row on SP lanes of each, those.
template <int SP>
__device__ __forceinline__ float row_sum(float v) {
  v = swap32_sum(swap16_sum(v));
  if constexpr (SP > 1) v += round_row<8>(v);
  if constexpr (SP > 2) v += round_row<4>(v);
  return v;
}
template <int SP>
__device__ __forceinline__ float row_max(float v) {
  v = swap32_max(swap16_max(v));
  if constexpr (SP > 1) v = fmaxf(v, round_row<8>(v));
  if constexpr (SP > 2) v = fmaxf(v, round_row<4>(v));
  return v;
}

// Sum of v over the lanes before this one.
__device__ __forceinline__ int sum_before(int v, int lane) {
  int sum = v;
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    const int other = __shfl_up(sum, d, kWave);
    sum += lane >= d ? other : 0;
  }
  return sum - v;
}

// Which rows and slots a workgroup has.
struct Place {
  int hk, b, split, tile;
};
__device__ __forceinline__ bool place_of(const Kv4AttentionArgs& a, const Kv4Plan& p, int lane, Place& w) {
  const auto [group, tile] = group_tile(blockIdx.x, p.groups, p.tiles);
  if (group >= p.groups) return false;
  // first runs of all sequences go first, then second ones, ...: later runs are fewer where lengths differ
  w = {group % a.Hkv, group / a.Hkv % a.B, group / a.Hkv / a.B, tile};
  if (p.by_length) {
    // Long runs first (single tokens of 64 caches of 500 to 8000 slots: 64 us in the order above, 53 so; blocks of 16 over
    // 16 to 4096: 76, 67; for more caches than that the search costs what the order gains): the whole ones,
    // then the last ones of all sequences (at most 64, one a lane) by length, then what lies past them.
    const int runs = p.splits - p.own_first, nth = group / a.Hkv;
    const int len = lane < a.B ? kv4_len(a.kv, lane, a.max_seq_len) : 0;
    const int whole = lane < a.B ? min(len / p.run, runs - 1) : 0, rest = len - whole * p.run;
    const int first = sum_before(whole, lane), wholes = __builtin_amdgcn_readlane(first + whole, 63);
    if (nth < wholes) {
      w.b = __builtin_ctzll(__ballot(nth >= first && nth < first + whole));
      w.split = nth - __builtin_amdgcn_readlane(first, w.b);
    } else if (nth < wholes + a.B) {
      // the sequence that so many come before, from the highest bit of the lengths down
      uint64_t those = __ballot(lane < a.B);
      int before = nth - wholes;
      for (int bit = 31 - __builtin_clz(p.run); bit >= 0; --bit) {
        const uint64_t ones = those & __ballot((rest >> bit) & 1);
        const int n = __builtin_popcountll(ones);
        those = before < n ? ones : those & ~ones;
        before -= before < n ? 0 : n;
      }
      for (; before > 0; --before) those &= those - 1;
      w.b = __builtin_ctzll(those);
      w.split = __builtin_amdgcn_readlane(whole, w.b);
    } else {
      const int left = lane < a.B ? runs - 1 - whole : 0, from = wholes + a.B + sum_before(left, lane);
      w.b = __builtin_ctzll(__ballot(nth >= from && nth < from + left));
      w.split = __builtin_amdgcn_readlane(whole, w.b) + 1 + nth - __builtin_amdgcn_readlane(from, w.b);
    }
  }
  return true;
}

// A run past the sequence: the join reads that it is empty.
__device__ __forceinline__ void leave_empty(const Kv4AttentionArgs& a, const Kv4Plan& p, const Place& w, int row0, int rows) {
  const int G = a.H / a.Hkv;
  for (int r = threadIdx.x; r < rows; r += blockDim.x) {
    const int row = row0 + r;
    p.part_lse[(static_cast<int64_t>(row / G) * a.H + w.hk * G + row % G) * p.splits + p.own_first + w.split] = -INFINITY;
  }
}

// A wavefront's 16 RT rows: row x = lane % 16 of each tile, of which quarter t = lane / 16 has the logits
// and the elements 4 t .. 4 t + 3 of every 16.
// Up to 16 / SP rows stand SP times among the 16, and each of a row's lanes takes the weights of some of its logits only
// (of 8 a lane 8 / SP): a cache of 1500 slots 10.4 us with SP = 4, 11.1 with 1.
// `LEAN`: for wavefronts whose registers are few, values are read where they are used.
template <bool F16, int W, int RT, bool LEAN, int SP>
struct Rows {
  static constexpr int NF = W / 32, NO = W / 16, NZ = 8 / SP, kRows = 16 / SP;
  static_assert(SP == 1 || RT == 1);
  static constexpr bool kHeld = RT < 4;            // queries in registers; else each wavefront brings a tile to LDS
  uint4 q[kHeld ? RT : 1][NF];                     // elements t W / 4 + ..., the second operand of K Q^T
  uint4* far;                                      // [RT][NF][64] in LDS
  float qz[RT];                                    // sum of q, as the logits are held
  uint64_t word[LEAN ? 1 : RT];                    // what a row sees of the block
  floatx4 o[RT][NO];
  // m: the subtracted logit (unscaled); mc = c m - lift, lift = kTop - unit; l: this lane's part of the
  // sum of the weights; add: its part of what joins every element of the output
  float m[RT], mc[RT], l[RT], add[RT];
  float* units;                                    // [RT][kRows] in LDS: they are wanted where sizes or maxima grow
  float limit;                                     // of a value's size within all rows' units (the same in all lanes)
  bool wide;                                       // a row's mc is past kFine (the same in all lanes)
  float c;                                         // f16 logits are held 2^-21 of what they are
  int key1, base, row0, rows;                      // end of the run, begin of the block, the wavefront's rows
  const uint64_t* mask;
  int slot0;                                       // first of a step's slots whose weights this lane takes

  __device__ __forceinline__ uint64_t sees(int r, int x, int G) const {
    if (!LEAN) return word[r];
    if (!mask) return ~0ull;
    return mask[(row0 + min(16 * r + anew<true>(x) % kRows, rows - 1)) / G];
  }

  // The queries, which wait for nothing that the kernel reads first.
  __device__ __forceinline__ void load(const Kv4AttentionArgs& a, int hk, int first_row, int n_rows, int lane, int wave, uint4* lds) {
    const int t = lane >> 4, x = lane & 15, G = a.H / a.Hkv;
    row0 = first_row;
    rows = n_rows;
    mask = a.mask;
    far = lds;
#pragma unroll
    for (int r = 0; r < (LEAN ? 0 : RT); ++r) word[r] = mask ? mask[(row0 + min(16 * r + x % kRows, rows - 1)) / G] : ~0ull;
#pragma unroll
    for (int r = 0; r < (kHeld ? RT : 1); ++r) {
      const int row = row0 + min(16 * (kHeld ? r : wave) + x % kRows, rows - 1), bi = row / G;
      const uint16_t* src = a.q + bi * a.q_row_stride + (hk * G + row % G) * a.q_head_stride;
#pragma unroll
      for (int i = 0; i < NF; ++i) q[r][i] = *reinterpret_cast<const uint4*>(src + min(t * (W / 4) + 8 * i, a.D - 8));
    }
  }

  // (the same in all wavefronts of a workgroup where queries are in LDS)
  __device__ __forceinline__ void begin(const Kv4AttentionArgs& a, int n, int end, int lane, int wave, float* unit_lds) {
    const int t = lane >> 4, skip = (lane & 15) / kRows * NZ;
    slot0 = 16 * (skip / 4) + 4 * t + skip % 4;
    key1 = end;
    base = n - a.L;
    c = uniform(a.scale * kLog2e * (F16 ? 0x1p21f : 1.f));
    float sums[kHeld ? RT : 1];
#pragma unroll
    for (int r = 0; r < (kHeld ? RT : 1); ++r) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < NF; ++i) {
        if (t * (W / 4) + 8 * i >= a.D) q[r][i] = make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int w = 0; w < 4; ++w) sum = plus_pair<F16>(part_of(q[r][i], w), 1.f, sum);
      }
      sum = swap32_sum(swap16_sum(sum));
      sums[r] = F16 ? sum * 0x1p-21f : sum;
    }
    if constexpr (!kHeld) {
      float* const all = reinterpret_cast<float*>(far + RT * NF * 64);
#pragma unroll
      for (int i = 0; i < NF; ++i) far[(wave * NF + i) * 64 + lane] = q[0][i];
      if (t == 0) all[16 * wave + lane] = sums[0];
      __syncthreads();
#pragma unroll
      for (int r = 0; r < RT; ++r) qz[r] = all[16 * r + (lane & 15)];
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      if constexpr (kHeld) qz[r] = sums[r];
      m[r] = -INFINITY;
      mc[r] = l[r] = add[r] = 0.f;
#pragma unroll
      for (int d = 0; d < NO; ++d) o[r][d] = floatx4{};
    }
    wide = false;
    units = unit_lds;
#pragma unroll
    for (int r = 0; r < RT; ++r) unit_of(r, lane & 15) = kLeastUnit<F16>;
    limit = __builtin_ldexpf(1.f, kLeastUnit<F16> + kRoom);
  }

  // Sizes up to 2^(unit + kRoom) fit a unit.
  static constexpr int kRoom = F16 ? 0 : 60;
  // (every lane of a row writes the row's, and reads what it wrote)
  __device__ __forceinline__ float& unit_of(int r, int x) const {
    return units[kRows * r + anew<LEAN>(x) % kRows];
  }
  // Of a value: its step, and in bf16 the middle of its range.
  static __device__ __forceinline__ float size_of(float step, float middle) {
    return F16 ? step : fmaxf(step, fabsf(middle) * 0.0625f);
  }

  // Which of this lane's slots a row of that word sees, of those from slot `at` of the step on (one of its fours).
  __device__ __forceinline__ uint32_t seen_from(uint64_t row, int at, int j0) const {
    return seen4(row, mask ? j0 + at - base : 0, key1 - j0 - at) & ((1 << min(NZ, 4)) - 1);
  }

  // Grows the rows' units to what the values that they see need, the upper lanes' `own` where all rows see all of them.
  // Slots that a row does not see leave its unit as it is: they have no effect on it.
  __device__ __forceinline__ void fit(float own, const float2* values, int j0, int lane, int G) {
    const int x = lane & 15;
    float size = lane & 32 && own < INFINITY ? own : 0.f, least = INFINITY;
    const bool some = cut(j0);
    if (!some) size = wave_allmax(size);
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      if (some) {
        const uint64_t row = sees(r, x, G);
        size = 0.f;
#pragma unroll
        for (int i = 0; i < NZ; i += 4) {
          const int at = slot0 + i / 4 * 16;
          const uint32_t seen = seen_from(row, at, j0);
#pragma unroll
          for (int u = 0; u < min(NZ, 4); ++u) {
            const float2 y = values[at + u];
            const float of = size_of(y.x, y.y);
            if ((seen >> u) & 1 && of < INFINITY) size = fmaxf(size, of);
          }
        }
        size = row_max<SP>(size);
      }
      const float unit = unit_of(r, x);
      const float need = size > 0.f ? fmaxf(unit, static_cast<float>(__builtin_amdgcn_frexp_expf(size) - kRoom)) : unit;
      if (need > unit) {
        const float f = __builtin_ldexpf(1.f, static_cast<int>(unit - need));
        l[r] *= f;
        add[r] *= f;
#pragma unroll
        for (int d = 0; d < NO; ++d) o[r][d] *= f;
        unit_of(r, x) = need;
        mc[r] = m[r] == -INFINITY ? 0.f : m[r] * c - (kTop<F16> - need);
      }
      least = fminf(least, need);
    }
    limit = __builtin_ldexpf(1.f, static_cast<int>(-wave_allmax(-least)) + kRoom);
  }

  // Whether some row does not see some of the slots j0 .. j0 + 31 (the same in all lanes).
  __device__ __forceinline__ bool cut(int j0) const { return j0 + 32 > key1 || (mask && j0 + 32 > base); }

  // From products with the codes of the keys at slots j0 .. j0 + 31 (register u of block i is slot 16 i + 4 t + u)
  // to weights, times the values' steps, as the second operand of D^T W^T.  `keys` and `values`: the slots'
  // steps and lowest values, in LDS.  Where cut(j0), those of values that are not finite are 0 there, since a
  // weight of 0 does not take them out, and `odd` says which: they count for the rows that see them.
  __device__ __forceinline__ void weigh(const floatx4 (&dots)[RT][2], const float2* keys, const float2* values, uint32_t odd, int j0, int lane,
                                        int G, uint32_t (&w)[RT][4]) {
    const int x = lane & 15;
    // a lane's logit i is of slot slot0 + i, or on from 16 after four
    auto pairs = [&](const float2* of, int i) { return *reinterpret_cast<const float4*>(of + slot0 + i / 4 * 16 + i % 4); };
    float z[RT][NZ];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int i = 0; i < NZ; ++i) {
        z[r][i] = dots[r][i / 4][i % 4];
        if constexpr (SP == 2) z[r][i] = in_banks<0xC>(z[r][i], dots[r][1][i]);
        if constexpr (SP == 4) {
          z[r][i] = in_banks<2>(z[r][i], dots[r][0][2 + i]);
          z[r][i] = in_banks<4>(z[r][i], dots[r][1][i]);
          z[r][i] = in_banks<8>(z[r][i], dots[r][1][2 + i]);
        }
      }
#pragma unroll
    for (int i = 0; i < NZ; i += 2) {
      const float4 p = pairs(keys, i);
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        z[r][i] = fmaf(p.x, z[r][i], p.y * qz[r]);
        z[r][i + 1] = fmaf(p.z, z[r][i + 1], p.w * qz[r]);
      }
    }
    if (cut(j0)) {
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const uint64_t row = sees(r, x, G);
#pragma unroll
        for (int i = 0; i < NZ; i += 4) {
          const int at = slot0 + i / 4 * 16;
          const uint32_t seen = seen_from(row, at, j0);
#pragma unroll
          for (int u = 0; u < min(NZ, 4); ++u) z[r][i + u] = (seen >> u) & 1 ? z[r][i + u] : -INFINITY;
          if (seen & odd >> at) add[r] = NAN;
        }
      }
    }
    // The subtracted logit follows a row's maximum only once that is kLag ahead, and no other row's: what that row sees
    // and this one does not has no effect on it.
    float top[RT];
    bool behind = false;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      top[r] = z[r][0];
#pragma unroll
      for (int i = 1; i < NZ; ++i) top[r] = fmaxf(top[r], z[r][i]);
      behind |= (top[r] - m[r]) * c > kLag<F16>;
    }
    if (__any(behind)) {
      bool far = false;
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const float best = row_max<SP>(top[r]);
        const bool moves = (best - m[r]) * c > kLag<F16>;
        if (__any(moves)) {                        // most often a tile of few, or of none
          if (__any(moves && m[r] != -INFINITY)) { // (nothing to scale in a row's first step)
            const float f = !moves ? 1.f : m[r] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m[r] - best) * c);
            l[r] *= f;
            add[r] *= f;
#pragma unroll
            for (int d = 0; d < NO; ++d) o[r][d] *= f;
          }
          if (moves) {
            m[r] = best;
            mc[r] = best * c - (kTop<F16> - unit_of(r, x));
          }
        }
        far |= fabsf(mc[r]) > kFine;
      }
      wide = __any(far);
    }
    float sub[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) sub[r] = mc[r];
    // c z - mc is off by the rounding of mc, by the same for all of a row, which cancels in the quotient;
    // but past kFine that may be more than the exponent range.
    if (wide) {
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const bool far = fabsf(mc[r]) > kFine;
        const float from = far ? m[r] : 0.f;
        sub[r] = far ? unit_of(r, x) - kTop<F16> : mc[r];
#pragma unroll
        for (int i = 0; i < NZ; ++i) z[r][i] -= from;
      }
    }
    // p s is rounded to the cache's type, as the products take it: relative to sum p s |d - 8|, as large an
    // error as that of rounding the output.  The sums of p and p y are of unrounded numbers.
    float sum[RT], lows[RT];                       // a step's, so that many small ones beside a large one count together
    uint32_t own[RT][NZ / 2];
#pragma unroll
    for (int i = 0; i < NZ / 2; ++i) {
      const float4 y = pairs(values, 2 * i);
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(z[r][2 * i], c, -sub[r]));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(z[r][2 * i + 1], c, -sub[r]));
        sum[r] = i == 0 ? p0 + p1 : sum[r] + (p0 + p1);
        lows[r] = fmaf(p0, y.y, i == 0 ? p1 * y.w : fmaf(p1, y.w, lows[r]));
        own[r][i] = pack2<F16>(p0 * y.x, p1 * y.z);
        lows[r] = plus_pair<F16>(own[r][i], -kMiddle<F16>, lows[r]);
      }
    }
    // the products take a row's weights from its first lane
#pragma unroll
    for (int r = 0; r < RT; ++r) {
#pragma unroll
      for (int i = 0; i < NZ / 2; ++i) w[r][i] = own[r][i];
      if constexpr (SP == 2) {
        w[r][2] = along_row<0x100, 8>(own[r][0]);
        w[r][3] = along_row<0x100, 8>(own[r][1]);
      }
      if constexpr (SP == 4) {
        w[r][1] = along_row<0x100, 4>(own[r][0]);
        w[r][2] = along_row<0x100, 8>(own[r][0]);
        w[r][3] = along_row<0x100, 12>(own[r][0]);
      }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      l[r] += sum[r];
      add[r] += lows[r];
    }
  }

  // Brings what joins every element into the sums, which are then of values about the middle of their heads' ranges.
  // Sums of codes on 64 or 128 grow with the length, sums about the middle with its root, and so do their roundings
  // (131072 slots a run: f16 outputs off by 6.5e-4 without this, by 3.1e-4 to 3.5e-4 with it once in 31 steps).
  __device__ __forceinline__ void center() {
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const float all = row_sum<SP>(add[r]);
#pragma unroll
      for (int d = 0; d < NO; ++d) o[r][d] += all;
      add[r] = 0.f;
    }
  }

  // Sums of the rows over the wavefront; then elements 16 d + 4 t .. + 3 of the (unnormalised) output are elements<d>(r).
  __device__ __forceinline__ void finish() {
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      l[r] = row_sum<SP>(l[r]);
      add[r] = row_sum<SP>(add[r]);
    }
  }
  template <int d>
  __device__ __forceinline__ float4 elements(int r) const {
    return make_float4(o[r][d][0] + add[r], o[r][d][1] + add[r], o[r][d][2] + add[r], o[r][d][3] + add[r]);
  }
};

// RT tiles of 16 rows a workgroup, KW wavefronts that take steps of 32 slots in turn, each from
// registers that its loads filled in operand order.
template <bool F16, int W, int RT, int KW, int SP>
__global__ __launch_bounds__(64 * KW, RT == 1 && KW < 8 ? 3 : 2) void kv4_attend_kernel(Kv4AttentionArgs a, Kv4Plan p) {
  using R = Rows<F16, W, RT, RT != 2, SP>;
  constexpr int M = RT * R::kRows, NF = R::NF, NO = R::NO, kStep = 32;
  constexpr int kLooked = 31;                      // steps whose pages are looked up at once, besides the one ahead
  constexpr int kPart = RT < 4 ? W : W / 4, kOutRow = kPart + 4;     // elements joined at once
  // Few rows: as much LDS as leaves a CU 1, 3 or 6 workgroups of 8, 4 or 2 wavefronts.  More of them at once only let short
  // caches slow down long ones (64 caches of 16 to 8000 slots 51.4 us without this, 48.6 so; 128 of up to 4000 68.5, 63.6;
  // 256 of up to 2000 56.8, 54.0), fewer of 2 leave gaps (256 of 512: 4 34.3, 6 29.5).
  constexpr int kLeast = RT > 1 ? 0 : (KW == 8 ? 82 : KW == 4 ? 42 : 25) * 256, kSums = KW * M * kOutRow;
  __shared__ __attribute__((aligned(16))) float acc[kSums > kLeast ? kSums : kLeast];
  __shared__ __attribute__((aligned(16))) uint4 queries[R::kHeld ? 1 : RT * NF * 64 + RT * 4];
  __shared__ float stat[KW * M * 2], factor[KW * M];
  __shared__ int place[M];
  __shared__ __attribute__((aligned(16))) float2 marks[KW * 64];     // (step, lowest) of a step's keys, then values

  const int tid = threadIdx.x, lane = tid & 63, t = lane >> 4, x = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = a.H / a.Hkv;
  Place w;
  if (!place_of(a, p, lane, w)) return;
  // ---- pages.  Step i of this wavefront begins at slot key0 + 32 (KW i + wave).  Pages are looked up for kLooked
  // steps and the one ahead at once, block k of the i-th by lane 2 i + k, the first ones while the length is
  // (entries past it are not used).
  const int key0 = w.split * p.run, my0 = key0 + kStep * wave, most = max(a.max_seq_len - 1, 0);
  const int64_t table = static_cast<int64_t>(w.b) * a.kv.max_pages;
  auto pages_of = [&](int step) {
    return a.kv.table[table + (min(my0 + kStep * KW * (step + lane / 2) + kKv4Block * (lane & 1), most) >> a.kv.page_shift)];
  };
  int held = pages_of(0);
  const int row0 = w.b * a.L * G + w.tile * M, rows = min(M, a.L * G - w.tile * M);
  R rs;
  rs.load(a, w.hk, row0, rows, lane, wave, queries);
  const int n = kv4_len(a.kv, w.b, a.max_seq_len), key1 = min(n, key0 + p.run);
  if (key0 >= n && p.part) return leave_empty(a, p, w, row0, rows);

  const int last = max(key1 - 1, 0) & ~(kKv4Block - 1);
  const uint8_t* const head = a.kv.pages + w.hk * a.kv.head_stride;
  auto block = [&](int nth, int step, int k) {
    const int page = clamp_id(__builtin_amdgcn_readlane(held, 2 * nth + k), a.kv.n_pages);
    const int j = min(my0 + kStep * KW * step + kKv4Block * k, last);
    return head + page * a.kv.page_stride + (j & ((1 << a.kv.page_shift) - 1)) / kKv4Block * kv4_block_bytes(W);
  };
  typedef uint32_t Codes __attribute__((ext_vector_type(W / 32)));
  // Chunk `lane` of a block's keys or values: a wavefront reads them in one piece, and one tile's rows are the only
  // ones to read them (64 caches of 500 to 8000 keys: 58 us as ordinary loads, 53 so; 32 of 40 to 4000 with 32 heads: 56, 51).
  auto codes = [&](const uint8_t* blk) {
    const auto* at = reinterpret_cast<const Codes*>(blk + anew<(RT > 2)>(lane) * static_cast<uint32_t>(sizeof(Codes)));
    if constexpr (RT == 1) return __builtin_nontemporal_load(at);
    return *at;
  };
  // the pair of key lane % 32 in the lower lanes, of value lane % 32 in the upper ones
  auto mark_of = [&](const uint8_t* b0, const uint8_t* b1) {
    return *reinterpret_cast<const uint32_t*>((lane & 16 ? b1 : b0) + static_cast<uint32_t>(16 * W + (lane & 32 ? 64 : 0) + 4 * x));
  };
  float2* const my_marks = marks + 64 * wave;
  const CodeBits<F16> bits;

  const int steps = key1 > my0 ? (key1 - my0 + kStep * KW - 1) / (kStep * KW) : 0;
  // (of a wavefront without steps: of slots that are there to be read, and not used)
  const uint8_t *b0 = block(0, 0, 0), *b1 = block(0, 0, 1);
  Codes k[2], v[2];
  k[0] = codes(b0);
  k[1] = codes(b1);
  uint32_t mark = mark_of(b0, b1);
  __builtin_amdgcn_sched_barrier(0);             // in the order in which the loop has them on their way
  v[0] = codes(b0 + 8 * W);
  v[1] = codes(b1 + 8 * W);
  __builtin_amdgcn_sched_barrier(0);
  rs.begin(a, n, key1, lane, wave, stat + 2 * M * wave);   // (which the join takes when they are done with)
  for (int step0 = 0; step0 < steps; step0 += kLooked) {
    const int end = min(steps - step0, kLooked);
    for (int nth = 0; nth < end; ++nth) {
      const int step = step0 + nth, j0 = my0 + kStep * KW * step;
      // ---- steps and lowest values: one slot a lane, handed round through LDS
      const int slot = anew<(RT > 2)>(lane);
      float st = kv4_step<F16>(mark), y = kv4_low<F16>(mark);
      uint32_t odd = 0;
      if (rs.cut(j0)) {
        const bool past = j0 + (slot & 31) >= key1;                     // what lies past the run may be anything
        const bool finite = fabsf(st) < INFINITY && fabsf(y) < INFINITY;
        odd = static_cast<uint32_t>(__ballot(!past && !finite) >> 32);
        if (past || (slot & 32 && !finite)) st = y = 0.f;
      }
      // what joins the lowest value, in steps: of a value the middle of its codes, of a key less what bf16 codes stand on
      const float mid = fmaf(slot & 32 ? 8.f : F16 ? 0.f : -16.f, st, y);
      my_marks[slot] = make_float2(st, mid);
      const float size = R::size_of(st, mid);
      const bool large = __ballot(size > rs.limit) >> 32;                // of the values, which upper lanes have
      asm volatile("" ::: "memory");             // LDS works in order for a wavefront; so must the compiler
      __builtin_amdgcn_wave_barrier();
      // ---- S^T = K Q^T over the codes
      floatx4 z[RT][2];
      if constexpr (R::kHeld) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int f = 0; f < NF; ++f) {
            const uint4 kf = key_codes<F16>(k[i][f], bits);
#pragma unroll
            for (int r = 0; r < RT; ++r) z[r][i] = mfma16<F16>(kf, rs.q[r][f], f == 0 ? floatx4{} : z[r][i]);
          }
      } else {
#pragma unroll
        for (int f = 0; f < NF; ++f) {
          asm volatile("" ::: "memory");         // queries from LDS no sooner than they are needed
          uint4 qf[RT];
#pragma unroll
          for (int r = 0; r < RT; ++r) qf[r] = queries[(r * NF + f) * 64 + lane];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint4 kf = key_codes<F16>(k[i][f], bits);
#pragma unroll
            for (int r = 0; r < RT; ++r) z[r][i] = mfma16<F16>(kf, qf[r], f == 0 ? floatx4{} : z[r][i]);
          }
        }
      }
      if (large) rs.fit(size, my_marks + 32, j0, lane, G);
      // ---- the next step's keys
      b0 = block(nth + 1, step + 1, 0);
      b1 = block(nth + 1, step + 1, 1);
      k[0] = codes(b0);
      k[1] = codes(b1);
      mark = mark_of(b0, b1);
      __builtin_amdgcn_sched_barrier(0);
      uint32_t wt[RT][4];
      rs.weigh(z, my_marks, my_marks + 32, odd, j0, lane, G, wt);
      asm volatile("" ::: "memory");
      __builtin_amdgcn_wave_barrier();
      // ---- out^T += D^T W^T over the codes
      each_index<NO>([&](auto index) {
        constexpr int d = index, u = 2 * (d / 4), j = d % 4;
        const uint4 f = make_uint4(value_codes<F16, j>(v[0][u], bits), value_codes<F16, j>(v[0][u + 1], bits),
                                   value_codes<F16, j>(v[1][u], bits), value_codes<F16, j>(v[1][u + 1], bits));
#pragma unroll
        for (int r = 0; r < RT; ++r) rs.o[r][d] = mfma16<F16>(f, make_uint4(wt[r][0], wt[r][1], wt[r][2], wt[r][3]), rs.o[r][d]);
      });
      v[0] = codes(b0 + 8 * W);
      v[1] = codes(b1 + 8 * W);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (step0 + kLooked < steps) {
      held = pages_of(step0 + kLooked);
      rs.center();
      asm volatile("" : "+v"(held));             // waited for here: in the loop each step's codes would be waited for with it
    }
  }

  // ---- join the wavefronts and write
  if constexpr (!R::kHeld) {                       // or what is joined would be made in the loop, and kept
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int d = 0; d < NO; ++d) asm volatile("" : "+v"(rs.o[r][d]));
  }
  rs.finish();
  auto put = [&](auto from) {                      // elements from .. + kPart
#pragma unroll
    for (int r = 0; r < RT; ++r)
      if (x < R::kRows)
        each_index<kPart / 16>([&](auto index) {
          constexpr int d = from / 16 + index;
          *reinterpret_cast<float4*>(acc + (wave * M + 16 * r + x) * kOutRow + 16 * index + 4 * t) = rs.template elements<d>(r);
        });
  };
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int at = wave * M + 16 * r + x;
    if (x < R::kRows && t == 0) {
      stat[at * 2] = rs.l[r] == 0.f ? -INFINITY : rs.mc[r];
      stat[at * 2 + 1] = rs.l[r];
    }
  }
  put(std::integral_constant<int, 0>{});
  __syncthreads();
  if (tid < rows) {                                // what the wavefronts' sums of a row are times
    float top = -INFINITY, total = 0.f, f[KW];
#pragma unroll
    for (int v = 0; v < KW; ++v) top = fmaxf(top, stat[(v * M + tid) * 2]);
#pragma unroll
    for (int v = 0; v < KW; ++v) {
      const float mw = stat[(v * M + tid) * 2];
      f[v] = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw - top);   // no key seen
      total += f[v] * stat[(v * M + tid) * 2 + 1];
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
    for (int v = 0; v < KW; ++v) factor[tid * KW + v] = f[v] * inv;
    const int row = row0 + tid;
    const int out = row / G * a.H + w.hk * G + row % G, at = out * p.splits + p.own_first + w.split;   // below 2^22, 2^29
    place[tid] = p.part ? at : out;
    const float lse = total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * kLn2;
    if (p.part)
      p.part_lse[at] = lse;
    else if (a.lse)
      a.lse[out] = lse;
  }
  __syncthreads();
  auto join = [&](int e0) {
    for (int i = tid; i < rows * (kPart / 4); i += 64 * KW) {
      const int r = i / (kPart / 4), e = i % (kPart / 4) * 4;
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
  #pragma unroll
      for (int v = 0; v < KW; ++v) {
        const float f = factor[r * KW + v];
        const float4 y = *reinterpret_cast<const float4*>(acc + (v * M + r) * kOutRow + e);
        sum.x += f * y.x;
        sum.y += f * y.y;
        sum.z += f * y.z;
        sum.w += f * y.w;
      }
      if (e0 + e < a.D) {
        const int64_t to = static_cast<int64_t>(place[r]) * a.D + e0 + e;
        if (p.part)
          *reinterpret_cast<float4*>(p.part + to) = sum;
        else
          *reinterpret_cast<uint2*>(a.out + to) = make_uint2(pack2<F16>(sum.x, sum.y), pack2<F16>(sum.z, sum.w));
      }
    }
  };
  join(0);
  if constexpr (kPart < W)
    each_index<W / kPart - 1>([&](auto index) {
      __syncthreads();
      put(std::integral_constant<int, (index + 1) * kPart>{});
      __syncthreads();
      join((index + 1) * kPart);
    });
}

// A launch's workgroups: rows of a tile, wavefronts, and the runs of the own keys.
struct Shape {
  int rows, waves;
  Runs runs;
};
constexpr int kHeld = 2 * 4 * kCUs;                // wavefronts that the GPU works on without a wait for a place

// Whether a launch's workgroups go by length: those of more than a round, and lengths that a wavefront has at hand.
bool by_length(int B, double rounds) { return B > 1 && B <= 64 && rounds > 1; }

constexpr int kSplits[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64};

// More than 16 rows: tiles of 32 or 64, by what a plan would take in us.  A round of workgroups takes `start` and `step` for
// each of its steps of 128 slots; a batch's lengths may be all the same or anything up to the bound, and the second
// counts twice: a plan for it loses less where they are the same than the other way round.  Tiles of 64 make the codes half as
// often, but take longer to start and join, and leave fewer workgroups to even out lengths with.  In us with 64 and with 32 rows:
// one block of 32 with 4 heads a key head over 65568 slots 55 and 60; one of 64 with 8 heads over 32768 91 and 107; 8 of 32 over
// 8192 53 and 63, over 32 to 8192 52 and 43; 64 of 16 over 4096 98 and 114, over 16 to 4096 74 and 63; 13 of 21 with 5 over 5 to
// 1777 44 and 38.  (A bound far past the lengths is planned for as if they reached it.)
Shape many_rows(int keys, int B, int64_t whole, int rows, int64_t all_rows, bool prefix) {
  constexpr double kTwo = 4., kRow = 2e-4;
  Shape best{32, 4, {}};
  double least = 1e300;
  for (int tile : {32, 64}) {
    if (tile > 32 && rows <= 32) break;
    const double step = tile > 32 ? 2.45 : 1.6, start = tile > 32 ? 11. : 6.;
    const int64_t groups = whole * ceil_div(rows, tile);
    for (int s : kSplits) {
      const int run = (keys + s * 128 - 1) / (s * 128) * 128, count = (keys + run - 1) / run;
      if (s > 1 && groups * count > kMostRuns) break;
      const double steps = run / 128 * step, rounds = static_cast<double>(groups * count) * 4 / kHeld;
      const double same = std::max(1., B > 1 && rounds > 2 ? rounds : std::ceil(rounds)) * (steps + start);
      const double total = rounds * (steps / 2 + start), longest = steps + start;
      const double other = by_length(B, rounds) || rounds <= 1 ? std::max(longest, total) : total + steps / 2;
      const double cost = (B > 1 ? (same + 2 * other) / 3 : same) + (count > 1 || prefix ? kTwo + kRow * all_rows * count : 0.);
      if (cost < least) {
        least = cost;
        best.rows = tile;
        best.runs = {count, run};
      }
      if (run == 128) break;                       // no shorter ones
    }
  }
  return best;
}

// Up to 16 rows: 2, 4 or 8 wavefronts a workgroup, by what a plan would take in us.  A round of wavefronts takes
// kStart and kStep for each of its steps; lengths may be all the same or anything up to the bound, and the
// plan is for the mean of both: weighed as for more rows, 8 caches of 16384 slots would be split in 8 (32 us; 28 in 4; of 100 to
// 16384 slots 25 and 23).  Runs cost a second launch, the scratch (together at least kTwo a call,
// where one launch takes kOne) and the partial sums.  So a batch is split when it does not fill the GPU, and otherwise takes the
// wavefronts that make two rounds, the long caches first: 64 caches of 500 to 8000 slots 52 us with 8 (64 with 4 and 112 with 2,
// in one round; 55 with 4 and 2 runs), 32 of 40 to 4000 with 32 heads 48 with 4 (58 with 8, 65 with 2), 128 of 600 17 with 2 (20
// with 4, 25 with 8), 16 of 6000 22 in 2 runs with 8 (28 whole), one of 1500 9.9 whole with 8 (12.6 in runs), 4 of 32768 27 in 8
// runs with 8 (32 in 16, 40 in 4).  At the edge of two plans the mean is for the one and loses by the other: 128 caches of
// 4000 slots take 84 with 2 (93 with 8, 97 with 4), but of 16 to 4000 65 (59, 58).
Shape few_rows(int keys, int B, int64_t whole, int64_t rows, bool prefix) {
  constexpr double kStart = 4.3, kStep = 1.1, kOne = 9., kTwo = 12.5, kRow = 2 * 512 / 5e6;
  Shape best{16, 8, {}};
  double least = 1e300;
  for (int waves : {2, 4, 8}) {
    const int step = 32 * waves;
    for (int s : kSplits) {
      const int run = (keys + s * step - 1) / (s * step) * step, count = (keys + run - 1) / run;
      if (s > 1 && whole * count > kMostRuns) break;
      const double steps = run / step * kStep, rounds = static_cast<double>(whole * count) * waves / kHeld;
      // with 2 and 4 wavefronts the GPU holds half as many again, which then take as much longer; a last round that
      // does not fill it shows where nothing is ordered
      const double thirds = B > 64 && waves < 8 && rounds > 1 ? std::ceil(rounds / 1.5) * 1.5 : rounds;
      const double same = std::max(1., B > 1 && rounds > 2 ? thirds : std::ceil(thirds)) * (steps + kStart);
      const double total = rounds * (steps / 2 + kStart), longest = steps + kStart;
      const double other = by_length(B, rounds) || rounds <= 1 ? std::max(longest, total) : total + steps / 2;
      const bool two = count > 1 || prefix;
      const double cost = std::max((B > 1 ? (same + other) / 2 : same) + (two ? 4.5 + kRow * rows * count : 0.), two ? kTwo : kOne);
      if (cost < least) {
        least = cost;
        best.waves = waves;
        best.runs = {count, run};
      }
      if (run == step) break;                      // no shorter ones
    }
  }
  return best;
}

struct CallPlan {
  Kv4Plan p;
  int pre_splits, rows, waves;
};

CallPlan make_plan(int B, int L, int H, int Hkv, int prefix_len, int max_seq_len) {
  CallPlan c{};
  c.pre_splits = prefix_len > 0 ? attention_prefix_splits(B, L, H, Hkv, prefix_len) : 0;
  if (max_seq_len > 0 || prefix_len == 0) {
    const int rows = L * (H / Hkv), keys = std::max(max_seq_len, 1);
    const int64_t whole = static_cast<int64_t>(B) * Hkv;
    const int64_t all_rows = static_cast<int64_t>(B) * L * H;
    const Shape s = rows > 16 ? many_rows(keys, B, whole, rows, all_rows, prefix_len > 0) : few_rows(keys, B, whole, all_rows, prefix_len > 0);
    c.p.tiles = ceil_div(rows, s.rows);
    c.rows = s.rows;
    c.waves = s.waves;
    c.p.run = s.runs.keys;
    c.p.groups = B * Hkv * s.runs.count;
    c.p.splits = s.runs.count;
    c.p.by_length = by_length(B, static_cast<double>(c.p.groups) * c.p.tiles * s.waves / kHeld);
  }
  c.p.own_first = c.pre_splits;
  c.p.splits += c.pre_splits;
  return c;
}

size_t bytes_of(const CallPlan& c, int64_t rows, int D) {
  if (c.p.splits <= 1) return 0;
  const size_t runs = static_cast<size_t>(rows) * c.p.splits;
  return (runs + 3) / 4 * 16 + runs * D * sizeof(float);
}

// Lanes of each quarter that share a row, of up to 16.
int lanes_of(int rows) { return rows <= 4 ? 4 : rows <= 8 ? 2 : 1; }

template <bool F16, int W>
void launch_own(const Kv4AttentionArgs& a, const CallPlan& c, hipStream_t s) {
  const dim3 grid(tile_grid(c.p.groups, c.p.tiles)), threads(64 * c.waves);
  const int rows = a.L * (a.H / a.Hkv);
  auto few = [&](auto waves) {
    constexpr int KW = waves;
    switch (lanes_of(rows)) {
      case 4: hipLaunchKernelGGL((kv4_attend_kernel<F16, W, 1, KW, 4>), grid, threads, 0, s, a, c.p); break;
      case 2: hipLaunchKernelGGL((kv4_attend_kernel<F16, W, 1, KW, 2>), grid, threads, 0, s, a, c.p); break;
      default: hipLaunchKernelGGL((kv4_attend_kernel<F16, W, 1, KW, 1>), grid, threads, 0, s, a, c.p);
    }
  };
  if (c.rows > 32)
    hipLaunchKernelGGL((kv4_attend_kernel<F16, W, 4, 4, 1>), grid, threads, 0, s, a, c.p);
  else if (c.rows > 16)
    hipLaunchKernelGGL((kv4_attend_kernel<F16, W, 2, 4, 1>), grid, threads, 0, s, a, c.p);
  else if (c.waves == 8)
    few(std::integral_constant<int, 8>{});
  else if (c.waves == 4)
    few(std::integral_constant<int, 4>{});
  else
    few(std::integral_constant<int, 2>{});
}

}  // namespace

// Workspace: where rows have several runs, a log-sum-exp and D sums of each.
size_t kv4_attention_workspace_bytes(int B, int L, int H, int Hkv, int D, int prefix_len, int max_seq_len) {
  return bytes_of(make_plan(B, L, H, Hkv, prefix_len, max_seq_len), static_cast<int64_t>(B) * L * H, D);
}

// What the own keys of a call run on: the kernel's width, rows of a tile, wavefronts and lanes a row, then its row tiles,
// runs, slots of a run, and whether long runs go first.  False where there is no such launch.
bool kv4_attention_plan_info(int B, int L, int H, int Hkv, int D, int prefix_len, int max_seq_len, int* out) {
  const CallPlan c = make_plan(B, L, H, Hkv, prefix_len, max_seq_len);
  if (!c.p.groups) return false;
  const int info[] = {kv4_width(D), c.rows, c.waves, c.rows > 16 ? 1 : lanes_of(L * (H / Hkv)), c.p.tiles,
                      c.p.splits - c.p.own_first, c.p.run, c.p.by_length};
  std::copy(std::begin(info), std::end(info), out);
  return true;
}

bool launch_kv4_attention(const Kv4AttentionArgs& a, const AttentionArgs& pre, bool f16, void* ws, size_t ws_bytes, hipStream_t s) {
  CallPlan c = make_plan(a.B, a.L, a.H, a.Hkv, pre.prefix_len, a.max_seq_len);
  const int64_t rows = static_cast<int64_t>(a.B) * a.L * a.H;
  const size_t need = bytes_of(c, rows, a.D);
  if (ws_bytes < need || (need > 0 && !ws)) return false;
  if (need > 0) {
    c.p.part_lse = static_cast<float*>(ws);
    c.p.part = c.p.part_lse + (static_cast<size_t>(rows) * c.p.splits + 3) / 4 * 4;
  }
  if (c.pre_splits) launch_attention_prefix(pre, f16, c.p.part, c.p.part_lse, c.p.splits, s);
  if (c.p.groups) {
    const bool wide = kv4_width(a.D) == 128;
    if (f16)
      wide ? launch_own<true, 128>(a, c, s) : launch_own<true, 64>(a, c, s);
    else
      wide ? launch_own<false, 128>(a, c, s) : launch_own<false, 64>(a, c, s);
  }
  if (c.p.part) launch_attention_join(pre, f16, c.p.part, c.p.part_lse, c.p.splits, s);
  return true;
}

}  // namespace brisk
