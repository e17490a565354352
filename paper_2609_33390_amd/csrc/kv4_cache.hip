// Writing tokens to the 4-bit cache, and reading them back.
//
//   z = min_d x_d,  s = type((max_d x_d - z) / 15),  c_d = min(rne((x_d - z) / s), 15)
//
// A wavefront takes 16 slots of a head, aligned to the cache's blocks.  Lane
// (q, key) = (lane / 16, lane % 16) holds a quarter of the key and a quarter of the
// value, in the pieces that the block's layout keeps together, so that codes leave it as
// whole words and a block is written by one wavefront alone: tokens next to each other, which
// a decoding step and a prompt give alike, share no bytes across wavefronts.
//
// Both passes are bound by memory.  Writing 8 x 4096 tokens of 8 heads of 128 (134 MB in, 36 MB out) takes
// 20 us (the last-level cache helps: more than a copy's rate); reading 16 x 8190 slots back (97 MB in, 537 MB out)
// takes 90 us on one cache over and over, 7.0 TB/s, and 103 on several in turn.  64 single tokens take 5.1 us to
// write and 4.7 to read, of which the launch is 3.
#include "kernels.h"
#include "kv4_common.h"

namespace brisk {

namespace {

constexpr int kWaves = 4;

// x of lane ^ 1 and lane ^ 2.
__device__ __forceinline__ uint32_t quad_xor1(uint32_t v) { return __builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0xB1, 0xF, 0xF, false); }
__device__ __forceinline__ uint32_t quad_xor2(uint32_t v) { return __builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x4E, 0xF, 0xF, false); }

// Lane u of each four gets what lane v had in w[u], as w[v].
__device__ __forceinline__ void quad_transpose(uint32_t (&w)[4], int lane) {
  const bool odd = lane & 1, high = lane & 2;
#pragma unroll
  for (int i = 0; i < 4; i += 2) {
    const uint32_t get = quad_xor1(odd ? w[i] : w[i + 1]);
    w[i] = odd ? get : w[i];
    w[i + 1] = odd ? w[i + 1] : get;
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t get = quad_xor2(high ? w[i] : w[i + 2]);
    w[i] = high ? get : w[i];
    w[i + 2] = high ? w[i + 2] : get;
  }
}

// Over the four lanes that share a slot.
__device__ __forceinline__ float quarters_max(float v) { return swap32_max(swap16_max(v)); }

// acc, or NaN where a number of the pair is not finite.
template <bool F16>
__device__ __forceinline__ float poisoned(uint32_t pair, float acc) {
  if constexpr (F16) {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(h2, pair), h2{0, 0}, acc, false);
  } else {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(b2, pair), __builtin_bit_cast(b2, 0u), acc, false);
  }
}

// How a head is held.  The quotient t / s is taken as t (1 / s) with the reciprocal in two parts,
// good to 2^-46: rounded to 32 bits that is a tie between two codes only where the quotient
// is one, since t has 24 bits and s at most 11 (a quotient that is none is at least 2^-24 of
// itself away from one, and 2^-35 of itself past the middle of its rounding).  Past s = 2^103, which
// bf16 has, the second part would be a subnormal number and short of bits: beyond 2^64 both t and s are taken 2^-64 times,
// which changes neither t's rounding nor the quotient.
struct Scheme {
  float low, unit, inv, inv_rest;                  // low: -z, times the unit
  uint32_t pair;
};

template <bool F16>
__device__ __forceinline__ Scheme scheme_of(float lowest, float highest, float poison) {
  Scheme h;
  const float range = highest - lowest;
  uint32_t step = f32_to_half<F16>(range / 15.f);
  // not a number where an element is not finite, or their range
  const bool bad = !(range + poison < INFINITY);
  if (!F16 && step < 0x0080) step = 0;             // steps below the normal numbers: the head is its lowest value
  const uint32_t low = bad ? (F16 ? 0x7E00u : 0x7FC0u) : f32_to_half<F16>(lowest);
  if (bad) step = 0;
  h.pair = step | low << 16;
  float s = half_to_f32<F16>(step);
  h.unit = !F16 && s > 0x1p64f ? 0x1p-64f : 1.f;
  s *= h.unit;
  h.low = -lowest * h.unit;
  h.inv = step ? 1.f / s : 0.f;
  h.inv_rest = fmaf(-s, h.inv, step ? 1.f : 0.f) * h.inv;
  return h;
}

// The code as a float (what a head without a step gives is not used).  A normal step is within 2^-8 of
// a fifteenth of the range, so only a subnormal one, which f16 may have, can give more than 15.
template <bool F16>
__device__ __forceinline__ float code_of(float x, const Scheme& h) {
  const float t = F16 ? x + h.low : fmaf(x, h.unit, h.low), y = fmaf(t, h.inv, t * h.inv_rest);
  return __builtin_rintf(F16 ? fminf(y, 15.f) : y);
}

template <bool F16>
__device__ __forceinline__ void widen(uint32_t w, float& lo, float& hi) {
  lo = half_to_f32<F16>(w & 0xFFFF);
  hi = F16 ? half_to_f32<F16>(w >> 16) : __uint_as_float(w & 0xFFFF0000u);
}

// First slot of the block that slot j lies in, also below 0.
__device__ __forceinline__ int64_t block_begin(int64_t j) { return j & ~static_cast<int64_t>(kKv4Block - 1); }

// Place in a block of the word of a key's elements e .. e + 7.
template <int W>
__device__ __forceinline__ int key_word(int key, int e) {
  return (16 * (e / (W / 4)) + key) * (W / 8) + e % (W / 4) / 8 * 4;
}

template <bool F16, int W>
__global__ __launch_bounds__(64 * kWaves) void kv4_write_kernel(Kv4WriteArgs a, int blocks, int items) {
  constexpr int NK = W / 32, NV = W / 16;
  const int lane = threadIdx.x & 63, q = lane >> 4, key = lane & 15;
  const int item = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (item >= items) return;
  const int h = item % a.Hkv, b = item / a.Hkv / blocks, nth = item / a.Hkv % blocks;
  const int64_t first = a.first[b], count = a.count ? min(max(a.count[b], 0), a.T) : a.T;
  const int64_t cap = static_cast<int64_t>(a.kv.max_pages) << a.kv.page_shift;
  const int64_t j0 = block_begin(first) + 16 * static_cast<int64_t>(nth);
  if (count < 1 || j0 < 0 || j0 >= cap || j0 >= first + count || j0 + 16 <= first) return;
  // A lane whose slot gets no token, and one that holds no elements (D < W), works on others' and stores nothing.
  const int64_t tok = j0 + key - first;
  const bool valid = tok >= 0 && tok < count;
  const int64_t src = b * a.seq_stride + min(max(tok, int64_t{0}), count - 1) * a.row_stride + h * a.head_stride;

  uint4 kw[NK], vw[NV / 2];                        // elements 32 i + 8 q + 0 .. 7
#pragma unroll
  for (int i = 0; i < NK; ++i) kw[i] = *reinterpret_cast<const uint4*>(a.k + src + min(32 * i + 8 * q, a.D - 8));
  // Of the values lanes of even q load 8 elements of an even 16, lanes of odd q of the next 16: each
  // will give its neighbour half.
#pragma unroll
  for (int i = 0; i < NV; i += 2)
    vw[i / 2] = *reinterpret_cast<const uint4*>(a.v + src + min(16 * (i + (q & 1)) + 8 * (q >> 1), a.D - 8));
  uint8_t* const blk = kv4_block<W>(a.kv, b, h, static_cast<int>(j0));

  auto scheme = [&](auto& words) {
    float lo = INFINITY, hi = -INFINITY, poison = 0.f;
    for (const uint4& v : words) {
      const uint32_t w4[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float x0, x1;
        widen<F16>(w4[i], x0, x1);
        lo = fminf(fminf(x0, x1), lo);
        hi = fmaxf(fmaxf(x0, x1), hi);
        poison = poisoned<F16>(w4[i], poison);
      }
    }
    return scheme_of<F16>(-quarters_max(-lo), quarters_max(hi), swap32_sum(swap16_sum(poison)));
  };

  {  // ---- the key
    const Scheme s = scheme(kw);
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      const uint32_t w4[4] = {kw[i].x, kw[i].y, kw[i].z, kw[i].w};
      // element e is nibble e / 2 of half e % 2
      float half[2] = {0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        float x0, x1;
        widen<F16>(w4[e / 2], x0, x1);
        half[0] = fmaf(code_of<F16>(x0, s), static_cast<float>(1 << (2 * e)), half[0]);
        half[1] = fmaf(code_of<F16>(x1, s), static_cast<float>(1 << (2 * e)), half[1]);
      }
      uint32_t w = static_cast<uint32_t>(half[0]) | static_cast<uint32_t>(half[1]) << 16;
      if (32 * i + 8 * q >= a.D || (s.pair & 0xFFFF) == 0) w = 0;
      if (valid) *reinterpret_cast<uint32_t*>(blk + key_word<W>(key, 32 * i + 8 * q)) = w << 3 | w >> 29;
    }
    if (valid && q == 0) *reinterpret_cast<uint32_t*>(blk + 16 * W + 4 * key) = s.pair;
  }

  {  // ---- the value: elements x + 16 (4 y + j) for x = 4 q + 0 .. 3
    const Scheme s = scheme(vw);
    float half[4][2] = {};                         // for each x the codes of y = 0 and of y = 1
#pragma unroll
    for (int i = 0; i < NV; i += 2) {
      const uint4 v = vw[i / 2];
      const auto lo = __builtin_amdgcn_permlane16_swap(v.x, v.z, false, false);
      const auto hi = __builtin_amdgcn_permlane16_swap(v.y, v.w, false, false);
#pragma unroll
      for (int n = 0; n < 2; ++n) {                // elements 16 (i + n) + 4 q + 0 .. 3
        float x[4];
        widen<F16>(lo[n], x[0], x[1]);
        widen<F16>(hi[n], x[2], x[3]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          half[e][i / 4] = fmaf(code_of<F16>(x[e], s), static_cast<float>(1 << (4 * ((i + n) % 4))), half[e][i / 4]);
      }
    }
    // the 16 bits of y = 0 and, above them, of y = 1; elements past D are code 0
    const int own = min(max((a.D - 4 * q + 15) / 16, 0), 8);
    const uint32_t keep = (s.pair & 0xFFFF) == 0 ? 0u : own == 8 ? ~0u : (1u << (4 * own)) - 1;
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = (static_cast<uint32_t>(half[e][0]) | static_cast<uint32_t>(half[e][1]) << 16) & keep;
    uint8_t* const val = blk + 8 * W;
    const int t = key >> 2, u = key & 3;
    if (__all(valid)) {
      quad_transpose(w, lane);                     // now of x = 4 q + u, slots 4 t + 0 .. 3
      uint8_t* const to = val + (16 * t + 4 * q + u) * (W / 8);
      const uint2 y0 = make_uint2((w[0] & 0xFFFF) | w[1] << 16, (w[2] & 0xFFFF) | w[3] << 16);
      if constexpr (W == 128)
        *reinterpret_cast<uint4*>(to) = make_uint4(y0.x, y0.y, w[0] >> 16 | (w[1] & 0xFFFF0000u), w[2] >> 16 | (w[3] & 0xFFFF0000u));
      else
        *reinterpret_cast<uint2*>(to) = y0;
    } else if (valid) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int y = 0; y < W / 64; ++y)
          *reinterpret_cast<uint16_t*>(val + (16 * t + 4 * q + e) * (W / 8) + 8 * y + 2 * u) = static_cast<uint16_t>(w[e] >> (16 * y));
    }
    if (valid && q == 1) *reinterpret_cast<uint32_t*>(blk + 16 * W + 64 + 4 * key) = s.pair;
  }
}

// z + s c, rounded to the cache's type.
template <bool F16>
__device__ __forceinline__ uint32_t value_of(uint32_t code, float step, float low) {
  return f32_to_half<F16>(fmaf(step, static_cast<float>(code), low));
}

__device__ __forceinline__ void stream_out(uint16_t* p, uint4 v) {
  typedef uint32_t u4 __attribute__((ext_vector_type(4)));
  __builtin_nontemporal_store(__builtin_bit_cast(u4, v), reinterpret_cast<u4*>(p));
}

template <bool F16, int W>
__global__ __launch_bounds__(64 * kWaves) void kv4_read_kernel(Kv4ReadArgs a, int blocks, int items) {
  constexpr int NK = W / 32, NV = W / 16;
  const int lane = threadIdx.x & 63, q = lane >> 4, key = lane & 15;
  const int item = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (item >= items) return;
  const int h = item % a.Hkv, b = item / a.Hkv / blocks, nth = item / a.Hkv % blocks;
  const int64_t first = a.first ? a.first[b] : 0;
  const int n = kv4_len(a.kv, b, static_cast<int>(static_cast<int64_t>(a.kv.max_pages) << a.kv.page_shift));
  const int64_t j0 = block_begin(first) + 16 * static_cast<int64_t>(nth);
  const int64_t tok = j0 + key - first;
  if (!__any(tok >= 0 && tok < a.T)) return;
  const bool held = j0 + key >= 0 && j0 + key < n;
  // slots that nobody holds read the place of one that the table addresses, and are not used
  const uint8_t* const blk = kv4_block<W>(a.kv, b, h, static_cast<int>(min(max(j0, int64_t{0}), (static_cast<int64_t>(a.kv.max_pages) << a.kv.page_shift) - 16)));

  uint32_t kc[NK];
#pragma unroll
  for (int i = 0; i < NK; ++i) kc[i] = *reinterpret_cast<const uint32_t*>(blk + key_word<W>(key, 32 * i + 8 * q));
  const int t = key >> 2, u = key & 3;
  const uint8_t* const from = blk + 8 * W + (16 * t + 4 * q + u) * (W / 8);
  uint4 vc = make_uint4(0, 0, 0, 0);
  if constexpr (W == 128) {
    vc = *reinterpret_cast<const uint4*>(from);
  } else {
    const uint2 x = *reinterpret_cast<const uint2*>(from);
    vc = make_uint4(x.x, x.y, 0, 0);
  }
  const uint32_t kp = *reinterpret_cast<const uint32_t*>(blk + 16 * W + 4 * key);
  const uint32_t vp = *reinterpret_cast<const uint32_t*>(blk + 16 * W + 64 + 4 * key);

  // Heads go out through LDS, row after row, so that a store instruction covers whole lines, and past the
  // caches, which the outputs do not fit (16 x 8190 slots: 206 us from the registers, 148 through LDS, 90 so); a
  // row's 16-byte pieces are permuted by its number.
  constexpr int kPieces = W / 8, kRowsOut = 64 / kPieces;
  __shared__ uint4 rows[kWaves][16 * kPieces];
  uint4* const mine = rows[threadIdx.x >> 6];
  auto put = [&](int e, uint4 v) { mine[key * kPieces + ((e / 8) ^ (key % kPieces))] = v; };
  auto out = [&](uint16_t* to) {
    asm volatile("" ::: "memory");                 // LDS works in order for a wavefront; so must the compiler
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int g = 0; g < 16 / kRowsOut; ++g) {
      const int row = g * kRowsOut + lane / kPieces, piece = lane % kPieces;
      const int64_t at = j0 + row - first;
      const uint4 v = mine[row * kPieces + (piece ^ (row % kPieces))];
      if (at >= 0 && at < a.T && 8 * piece < a.D)
        stream_out(to + ((b * static_cast<int64_t>(a.T) + at) * a.Hkv + h) * a.D + 8 * piece, v);
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
  };
  {
    const float s = kv4_step<F16>(kp), z = kv4_low<F16>(kp);
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      const uint32_t w = kc[i] >> 3 | kc[i] << 29;
      uint32_t o[4];
#pragma unroll
      for (int p = 0; p < 4; ++p)
        o[p] = held ? value_of<F16>((w >> (4 * p)) & 15, s, z) | value_of<F16>((w >> (4 * p + 16)) & 15, s, z) << 16 : 0;
      put(32 * i + 8 * q, make_uint4(o[0], o[1], o[2], o[3]));
    }
    out(a.k);
  }
  {
    // of x = 4 q + u, slots 4 t + 0 .. 3: to this lane's slot, x = 4 q + 0 .. 3
    uint32_t w[4] = {(vc.x & 0xFFFF) | vc.z << 16, vc.x >> 16 | (vc.z & 0xFFFF0000u),
                     (vc.y & 0xFFFF) | vc.w << 16, vc.y >> 16 | (vc.w & 0xFFFF0000u)};
    quad_transpose(w, lane);
    const float s = kv4_step<F16>(vp), z = kv4_low<F16>(vp);
    // Elements 16 i + 4 q + 0 .. 3 of two i at a time: lanes of even q take the first i's of their own and
    // of the next quarter's, lanes of odd q the second i's, so that a piece is of 16 bytes.
#pragma unroll
    for (int i = 0; i < NV; i += 2) {
      uint32_t o[2][2];
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int p = 0; p < 2; ++p)
          o[n][p] = held ? value_of<F16>((w[2 * p] >> (4 * (i + n))) & 15, s, z) | value_of<F16>((w[2 * p + 1] >> (4 * (i + n))) & 15, s, z) << 16 : 0;
      const auto x = __builtin_amdgcn_permlane16_swap(o[0][0], o[1][0], false, false);
      const auto y = __builtin_amdgcn_permlane16_swap(o[0][1], o[1][1], false, false);
      put(16 * (i + (q & 1)) + 8 * (q >> 1), make_uint4(x[0], y[0], x[1], y[1]));
    }
    out(a.v);
  }
}

// Blocks of 16 slots that T tokens can touch, wherever they begin.
int blocks_of(int T) { return (T + 2 * kKv4Block - 2) / kKv4Block; }

}  // namespace

// (A step at a time: the three sizes together may pass 64 bits.)
bool kv4_launchable(int B, int Hkv, int T) {
  constexpr int64_t kMost = 1 << 25;
  const int64_t heads = static_cast<int64_t>(B) * Hkv;
  return heads < kMost && heads * blocks_of(T) < kMost;
}

template <class Args, class Fn>
static void launch_blocks(const Args& a, Fn kernel, hipStream_t s) {
  const int blocks = blocks_of(a.T);
  const int items = a.B * a.Hkv * blocks;          // kv4_launchable: below 2^25
  hipLaunchKernelGGL(kernel, dim3((items + kWaves - 1) / kWaves), dim3(64 * kWaves), 0, s, a, blocks, items);
}

void launch_kv4_write(const Kv4WriteArgs& a, bool f16, hipStream_t s) {
  const bool wide = kv4_width(a.D) == 128;
  if (f16)
    launch_blocks(a, wide ? kv4_write_kernel<true, 128> : kv4_write_kernel<true, 64>, s);
  else
    launch_blocks(a, wide ? kv4_write_kernel<false, 128> : kv4_write_kernel<false, 64>, s);
}

void launch_kv4_read(const Kv4ReadArgs& a, bool f16, hipStream_t s) {
  const bool wide = kv4_width(a.D) == 128;
  if (f16)
    launch_blocks(a, wide ? kv4_read_kernel<true, 128> : kv4_read_kernel<true, 64>, s);
  else
    launch_blocks(a, wide ? kv4_read_kernel<false, 128> : kv4_read_kernel<false, 64>, s);
}

}  // namespace brisk
