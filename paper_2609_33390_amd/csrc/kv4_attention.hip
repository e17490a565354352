// Attention of a block over a shared prefix and a cache held in 4 bits.
//
// With key j held as z_j + s_j c_j and value j as y_j + r_j d_j, per head:
//   a_j = scale (s_j <q, c_j> + z_j sum_d q_d),   p_j = exp(a_j - m)
//   out = (sum_j (p_j r_j) (d_j - 8) + sum_j p_j (y_j + 8 r_j)) / sum_j p_j
// The matrix instructions work on the codes alone, whole numbers that their types
// hold exactly; steps and lowest values meet the logits and the probabilities in
// fp32.  A bf16 code is made with one instruction for two of them, by putting its
// bits under an exponent (16 + c, 128 + d), and the 16 and 128 are taken out again:
// from the logits through what the products begin from, from the sums (with the 8)
// through the sum of the rounded weights.  An f16 code is its own bits, a subnormal number (8 c and d or
// 16 d times 2^-24), whose power of two the scale and the last step take out.
//
// Codes come from memory to registers in operand order, 32 slots of a head a step
// of a wavefront, the next ones' on the way; the wavefronts of a workgroup take
// steps in turn and join through LDS.
#include <type_traits>

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

// Eight codes of a key: 16 + c in bf16, 8 c 2^-24 in f16.
template <bool F16>
__device__ __forceinline__ uint4 key_codes(uint32_t w) {
  constexpr uint32_t kMask = 0x00780078, kBase = F16 ? 0 : 0x41804180;
  return make_uint4((w & kMask) | kBase, ((w >> 4) & kMask) | kBase, ((w >> 8) & kMask) | kBase,
                    (__builtin_amdgcn_alignbit(w, w, 12) & kMask) | kBase);
}

// Nibble j of both halves of a word of values: 128 + d in bf16, d 2^-24 or (odd j) 16 d 2^-24 in f16.
template <bool F16, int J>
__device__ __forceinline__ uint32_t value_codes(uint32_t w) {
  if constexpr (F16) return (w >> (J / 2 * 8)) & (J % 2 ? 0x00F000F0u : 0x000F000Fu);
  return ((w >> (4 * J)) & 0x000F000Fu) | 0x43004300u;
}

// Which of four slots a row sees, the first one `at` slots past the block's begin and `left` before the end.
__device__ __forceinline__ uint32_t seen4(uint64_t word, int at, int left) {
  const uint64_t bits = at >= 64 ? 0 : at >= 0 ? word >> at : at > -4 ? (word << -at) | ((1ull << -at) - 1) : ~0ull;
  return static_cast<uint32_t>(bits) & (left >= 4 ? 15u : left <= 0 ? 0u : (1u << left) - 1);
}

__device__ __forceinline__ float swap16_max(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ uint32_t part_of(uint4 v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// What a wavefront loads of 32 slots: two blocks.  M = 16 rows: a lane has chunk `lane` of
// each block.  M = 32: it has two chunks of the keys of its own slot, and of each block its half
// of two chunks of values.
template <int W, int M>
struct Slots {
  static constexpr int NQ = M == 16 ? 2 : 4;       // groups of four slots, of which this lane has the logits
  static constexpr int NV = M == 16 ? W / 32 : 4;
  uint32_t k[2][W / 32], v[2][NV];
  uint4 kp[NQ], vp[NQ];
  uint32_t mark;                                   // the pair of value `lane % 32`
};

// M rows a workgroup, KW wavefronts.
template <bool F16, int W, int M, int KW>
__global__ __launch_bounds__(64 * KW, M == 16 ? 4 : 2) void kv4_attend_kernel(Kv4AttentionArgs a, Kv4Plan p) {
  constexpr int NQ = Slots<W, M>::NQ, NS = 4 * NQ, NO = M == 16 ? W / 16 : W / 32, NF = W / 32;
  constexpr int R = M == 16 ? 4 : 16;              // registers of an accumulator
  constexpr int kStep = 32;                        // slots of a wavefront's step
  constexpr int kOutRow = W + 4;
  using Acc = std::conditional_t<M == 16, floatx4, floatx16>;
  __shared__ __attribute__((aligned(16))) float acc[KW * M * kOutRow];
  __shared__ float stat[KW * M * 2];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = a.H / a.Hkv;
  const int bid = blockIdx.x, group = bid / 8 / p.tiles * 8 + bid % 8, tile = bid / 8 % p.tiles;
  if (group >= p.groups) return;
  // first runs of all sequences, then second ones, ...: later runs are fewer where lengths differ
  const int hk = group % a.Hkv, b = group / a.Hkv % a.B;
  int split = group / a.Hkv / a.B;
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

  // M = 16: quarter t, row or slot or element x.  M = 32: half t, x = col % 16.
  const int col = M == 16 ? lane & 15 : lane & 31, t = M == 16 ? lane >> 4 : lane >> 5, x = lane & 15;

  // ---- queries, as the second operand of K Q^T, and their sums
  constexpr int NQF = M == 16 ? NF : 2 * NF;
  uint4 q[NQF];
  uint64_t word;
  float qsum = 0.f;
  {
    const int row = row0 + min(col, rows - 1), bi = row / G;
    const uint16_t* src = a.q + bi * a.q_row_stride + (hk * G + row % G) * a.q_head_stride;
    word = masked ? a.mask[bi] : ~0ull;
#pragma unroll
    for (int i = 0; i < NQF; ++i) {
      const int e = t * (M == 16 ? W / 4 : W / 2) + 8 * i;
      q[i] = e < a.D ? *reinterpret_cast<const uint4*>(src + e) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int w = 0; w < 4; ++w)
        qsum += half_to_f32<F16>(part_of(q[i], w) & 0xFFFF) + half_to_f32<F16>(part_of(q[i], w) >> 16);
    }
    if constexpr (M == 16) qsum = swap16_sum(qsum);
    qsum = swap32_sum(qsum);
  }
  Acc start;                                       // what the products begin from
#pragma unroll
  for (int r = 0; r < R; ++r) start[r] = F16 ? 0.f : -16.f * qsum;
  // f16 logits are held 2^-21 of what they are
  const float c = a.scale * kLog2e * (F16 ? 0x1p21f : 1.f), qz = F16 ? qsum * 0x1p-21f : qsum;

  // ---- loads
  using Raw = Slots<W, M>;
  const int last = max(key1 - 1, 0) & ~(kKv4Block - 1);
  auto load = [&](int j0, Raw& s) {
    const uint8_t* blk[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) blk[i] = kv4_block<W>(a.kv, b, hk, min(j0 + 16 * i, last));
    if constexpr (M == 16) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if constexpr (W == 128) {
          const uint4 kw = *reinterpret_cast<const uint4*>(blk[i] + lane * 16);
          const uint4 vw = *reinterpret_cast<const uint4*>(blk[i] + 8 * W + lane * 16);
#pragma unroll
          for (int w = 0; w < 4; ++w) s.k[i][w] = part_of(kw, w), s.v[i][w] = part_of(vw, w);
        } else {
          const uint2 kw = *reinterpret_cast<const uint2*>(blk[i] + lane * 8);
          const uint2 vw = *reinterpret_cast<const uint2*>(blk[i] + 8 * W + lane * 8);
          s.k[i][0] = kw.x, s.k[i][1] = kw.y, s.v[i][0] = vw.x, s.v[i][1] = vw.y;
        }
        s.kp[i] = *reinterpret_cast<const uint4*>(blk[i] + 16 * W + 16 * t);
        s.vp[i] = *reinterpret_cast<const uint4*>(blk[i] + 16 * W + 64 + 16 * t);
      }
    } else {
      const uint8_t* own = col < 16 ? blk[0] : blk[1];
#pragma unroll
      for (int i = 0; i < 2; ++i) {                // chunks 2 t + i of the lane's slot; chunks t + 2 u of both blocks' values
        const uint8_t* kc = own + (16 * (2 * t + i) + x) * (W / 8);
        if constexpr (W == 128) {
          const uint4 kw = *reinterpret_cast<const uint4*>(kc);
#pragma unroll
          for (int w = 0; w < 4; ++w) s.k[i][w] = part_of(kw, w);
        } else {
          const uint2 kw = *reinterpret_cast<const uint2*>(kc);
          s.k[i][0] = kw.x, s.k[i][1] = kw.y;
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {              // W = 128: elements x + 64 (col / 16) + 16 d; W = 64: x + 32 (col / 16) + 16 d
          const uint2 vw = *reinterpret_cast<const uint2*>(blk[i] + 8 * W + (16 * (t + 2 * u) + x) * (W / 8) + (W == 128 ? 8 * (col / 16) : 0));
          const int down = W == 128 ? 0 : 8 * (col / 16);
          s.v[i][2 * u] = vw.x >> down, s.v[i][2 * u + 1] = vw.y >> down;
        }
      }
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        s.kp[i] = *reinterpret_cast<const uint4*>(blk[i / 2] + 16 * W + 16 * (2 * (i % 2) + t));
        s.vp[i] = *reinterpret_cast<const uint4*>(blk[i / 2] + 16 * W + 64 + 16 * (2 * (i % 2) + t));
      }
    }
    s.mark = *reinterpret_cast<const uint32_t*>((lane & 16 ? blk[1] : blk[0]) + 16 * W + 64 + 4 * x);
  };

  Acc o[NO];
#pragma unroll
  for (int d = 0; d < NO; ++d) o[d] = Acc{};
  // m: the subtracted logit (unscaled); mc = c m - lift, lift = kTop - unit; l: this lane's part of the
  // sum of the weights; add: its part of what joins every element of the output
  float m = -INFINITY, mc = 0.f, l = 0.f, add = 0.f;
  int unit = kLeastUnit<F16>;
  bool wide = false;                               // a row's mc is past kFine (the same in all lanes)

  auto attend = [&](const Raw& s, int j0) {
    // ---- S^T = K Q^T over the codes
    float z[NS];
    if constexpr (M == 16) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        floatx4 r = start;
#pragma unroll
        for (int f = 0; f < NF; ++f) r = mfma16<F16>(key_codes<F16>(s.k[i][f]), q[f], r);
#pragma unroll
        for (int u = 0; u < 4; ++u) z[4 * i + u] = r[u];
      }
    } else {
      floatx16 r = start;
#pragma unroll
      for (int f = 0; f < 2 * NF; ++f) r = mfma32<F16>(key_codes<F16>(s.k[f / NF][f % NF]), q[f], r);
#pragma unroll
      for (int u = 0; u < NS; ++u) z[u] = r[u];
    }
    float step[NS], low[NS];                       // of the values
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const uint32_t kp = part_of(s.kp[i / 4], i % 4), vp = part_of(s.vp[i / 4], i % 4);
      z[i] = fmaf(kv4_step<F16>(kp), z[i], kv4_low<F16>(kp) * qz);
      step[i] = kv4_step<F16>(vp);
      low[i] = fmaf(8.f, step[i], kv4_low<F16>(vp));
    }
    const bool cut = j0 + kStep > key1 || (masked && j0 + kStep > base);
    if (cut) {
#pragma unroll
      for (int i = 0; i < NS; i += 4) {
        const int first = j0 + (M == 16 ? 4 * i : 2 * i) + 4 * t;
        const uint32_t seen = seen4(masked ? word : ~0ull, masked ? first - base : 0, key1 - first);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const bool see = (seen >> u) & 1;
          z[i + u] = see ? z[i + u] : -INFINITY;
          step[i + u] = see ? step[i + u] : 0.f;   // what is not seen may hold anything
          low[i + u] = see ? low[i + u] : 0.f;
        }
      }
    }
    // ---- softmax statistics
    float top = z[0];
#pragma unroll
    for (int i = 1; i < NS; ++i) top = fmaxf(top, z[i]);
    if constexpr (M == 16) top = swap16_max(top);
    top = swap32_max(top);
    float size = fmaxf(kv4_step<F16>(s.mark), fabsf(kv4_low<F16>(s.mark)) * 0.0625f);
    size = j0 + (lane & 31) < key1 && size < INFINITY ? size : 0.f;
    // The subtracted logit follows the maximum only once that is kLag ahead.
    if (__any((top - m) * c > kLag<F16> || size > __builtin_ldexpf(1.f, F16 ? unit : unit + 60))) {
      const float largest = wave_allmax(size);
      const int need = largest > 0.f ? __builtin_amdgcn_frexp_expf(largest) - (F16 ? 0 : 60) : kLeastUnit<F16>;
      const int grown = max(unit, need);
      const float up = fmaxf(m, top);
      const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(fmaf(m - up, c, static_cast<float>(unit - grown)));
      l *= f;
      add *= f;
#pragma unroll
      for (int d = 0; d < NO; ++d) o[d] *= f;
      m = up;
      unit = grown;
      mc = up == -INFINITY ? 0.f : up * c - static_cast<float>(kTop<F16> - unit);
      wide = __any(fabsf(mc) > kFine);
    }
    float sub = mc;
    if (wide) {
      const float from = m == -INFINITY ? 0.f : m;
      sub = static_cast<float>(unit - kTop<F16>);
#pragma unroll
      for (int i = 0; i < NS; ++i) z[i] -= from;
    }
    // ---- weights.  p s is rounded to the cache's type, as the products take it; the sums of p and
    // p y are of unrounded numbers.
    uint32_t w[NS / 2];
    float sum = 0.f, lows = 0.f;
#pragma unroll
    for (int i = 0; i < NS; i += 2) {
      const float p0 = __builtin_amdgcn_exp2f(fmaf(z[i], c, -sub)), p1 = __builtin_amdgcn_exp2f(fmaf(z[i + 1], c, -sub));
      sum += p0 + p1;
      lows = fmaf(p0, low[i], fmaf(p1, low[i + 1], lows));
      w[i / 2] = pack2<F16>(p0 * step[i], p1 * step[i + 1]);
      lows = less_middle<F16>(w[i / 2], lows);
    }
    l += sum;
    add += lows;
    // ---- out^T += D^T W^T over the codes
    each_index<NO>([&](auto index) {
      constexpr int d = index, j = M == 16 ? d % 4 : d;
      if constexpr (M == 16) {
        constexpr int y = 2 * (d / 4);
        const uint4 f = make_uint4(value_codes<F16, j>(s.v[0][y]), value_codes<F16, j>(s.v[0][y + 1]),
                                   value_codes<F16, j>(s.v[1][y]), value_codes<F16, j>(s.v[1][y + 1]));
        o[d] = mfma16<F16>(f, make_uint4(w[0], w[1], w[2], w[3]), o[d]);
      } else {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          const uint4 f = make_uint4(value_codes<F16, j>(s.v[g][0]), value_codes<F16, j>(s.v[g][1]),
                                     value_codes<F16, j>(s.v[g][2]), value_codes<F16, j>(s.v[g][3]));
          o[d] = mfma32<F16>(f, make_uint4(w[4 * g], w[4 * g + 1], w[4 * g + 2], w[4 * g + 3]), o[d]);
        }
      }
    });
  };

  int j0 = key0 + wave * kStep;
  if (j0 < key1) {
    Raw cur;
    load(j0, cur);
    for (; j0 < key1; j0 += kStep * KW) {
      Raw next;
      load(j0 + kStep * KW, next);
      attend(cur, j0);
      cur = next;
    }
  }
  if constexpr (M == 16) {
    l = swap16_sum(l);
    add = swap16_sum(add);
  }
  l = swap32_sum(l);
  add = swap32_sum(add);

  // ---- join the wavefronts and write
  {
    float* const to = acc + (wave * M + col) * kOutRow;
    each_index<NO>([&](auto index) {
      constexpr int d = index, j = M == 16 ? d % 4 : d;
      constexpr float f = !F16 ? 1.f : j % 2 ? 0x1p20f : 0x1p24f;
#pragma unroll
      for (int r = 0; r < R; r += 4) {
        const int e = M == 16 ? 16 * d + 4 * t : 8 * (r / 4 % 2) + 4 * t + 16 * (W / 32 * (r / 8) + d);
        *reinterpret_cast<float4*>(to + e) = make_float4(fmaf(o[d][r], f, add), fmaf(o[d][r + 1], f, add),
                                                         fmaf(o[d][r + 2], f, add), fmaf(o[d][r + 3], f, add));
      }
    });
    if (t == 0) {
      stat[(wave * M + col) * 2] = l == 0.f ? -INFINITY : mc;
      stat[(wave * M + col) * 2 + 1] = l;
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
    const Runs r = runs_of(max_seq_len > 0 ? max_seq_len : 1, static_cast<int64_t>(B) * Hkv * c.p.tiles, 32 * s.waves, s.slots);
    c.p.run = r.keys;
    c.p.groups = B * Hkv * r.count;
    c.p.splits = r.count;
  }
  c.p.own_first = c.pre_splits;
  c.p.splits += c.pre_splits;
  return c;
}

template <bool F16, int W>
void launch_own(const Kv4AttentionArgs& a, const Kv4Plan& p, hipStream_t s) {
  const dim3 grid((p.groups + 7) / 8 * 8 * p.tiles);
  if (shape_for(static_cast<int64_t>(a.L) * (a.H / a.Hkv)).rows == 16)
    hipLaunchKernelGGL((kv4_attend_kernel<F16, W, 16, 4>), grid, dim3(256), 0, s, a, p);
  else
    hipLaunchKernelGGL((kv4_attend_kernel<F16, W, 32, 4>), grid, dim3(256), 0, s, a, p);
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
