// Decode attention of a batch whose sequences share long prefixes, each prefix held once in a quantized cache
// (tkv_quant_attn_decode_shared): Eq. 3 over the prefix's tokens and the sequence's own, one softmax.
//
// The query heads of all sequences that share a prefix are rows of one matrix per KV head (up to 64 sequences x 8
// heads), so a block of 32 tokens' codes is read and unpacked once for 16 NQ of them, and both products are plain fp16 ones with
// float32 sums:
//   * q.K-hat = sum_c q[c] (s[c] code'[t][c]) + sum_c q[c] (z[c] + c0 s[c]), code' = code - c0.  The first factor's product is
//     exact in fp16: code' is 0, 1 (1 bit) or -1 .. 2; at 4 bits, -8 .. 7, the scaler goes in two parts of 8 and 3 bits, each exact
//     times code', by two matrix instructions.  The second sum does not depend on the token: sixteen (4 bits: eight) groups at once
//     are one operand's rows, and the results wait in an LDS table to be added to the logits of a group's blocks as one number.
//     (K-hat rounded to fp16 would be off by up to 2.7e-3 in outputs where outlier channels are ten times the others.)
//   * p.V-hat likewise: sum_t p[t] (s[t] code'[t]), exact products, and sum_t p[t] z[t], sum_t p[t] s[t] of every channel group and the
//     weights' own sum as the rows of one more operand.  (V-hat rounded to fp16 takes the outputs' error against float64 from 2.9e-4 of
//     their norm to 3.5e-4, 2.1e-4 of which is their own rounding; one product instead of two at 4 bits, scaler times code rounded, to
//     3.4e-4, for 127 us instead of 147 where 64 sequences share 32770 tokens.)  The weights are rounded to fp16, off by at most 2^-11
//     of each, and divided by the sum of the rounded ones (those of tokens still in the ring added up as they are made).
// A wave takes 32-token blocks on its own: the codes lie in the order of the 16x16x32 matrix operands, S^T = K Q^T
// leaves a query's logits in the lanes where O^T = V^T P^T wants its weights, and nothing is exchanged
// between lanes but a rare rise of the running maximum.
//
// Latency bounds it: with 64 rows the vector units work half of the time or more (unpacking, exponentials) and the matrix cores a quarter
// (2 bits) to two fifths (4 bits); a wave goes from logits over their maximum and weights to the values' products one block at a time, and
// there are two waves on a SIMD to fill each other's gaps.  131072 tokens under 16 sequences of 32/8 heads, 2 bits: 61 us (568
// TFLOP/s; the codes alone would take 24 us), 32770 under 64 of 64/8, 4 bits: 146 us, two prefixes of 48413, 1 bit: 23 us, 2000 under 4: 12.7 us.
//
// Prefix and own tokens are split over workgroups in proportion to their cost; partial (reference, sum, weighted V) results
// go through the workspace to a second launch that joins them.
#include <algorithm>

#include "tkv_common.h"

namespace {

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));
typedef uint32_t uintx2 __attribute__((ext_vector_type(2)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;
typedef lds_char* lds_at;  // (pointers, not numbers: so that constant offsets go into the instructions)

constexpr int kWaves = 8;
constexpr int kSlots = 3;            // blocks of a wave on their way or in use
constexpr float kNone = -1e30f;      // reference of a row without a token so far
// Weights are 2^(logit - reference + kShift), the reference follows the maximum when that is kLazy above it: at most 2^15 in
// fp16, and fp16's subnormal numbers begin 2^-21 below the reference's weight.
constexpr float kLazy = 8.f, kShift = 7.f;
constexpr int kRowFloats = TKV_D + 2;

struct SharedCache {
  const char* k_codes;
  const char* k_scale;
  const char* k_zero;
  const char* v_codes;
  const char* v_scale;
  const char* v_zero;
  const char* k_resid;
  const char* v_resid;
  int32_t residual, capacity;
};

struct SharedParams {
  SharedCache cache[2];  // the batch's own, the prefixes'
  const __half* q;
  __half* out;
  float* parts;          // [row slot][128]
  float* ml;             // [row slot][2]
  float scale2;
  int32_t hq, hkv, group, batch, n_prefix;
  int32_t prefix_items;  // items of the prefixes come first
  // own sequences
  int32_t len[TKV_MAX_BATCH], first[TKV_MAX_BATCH], chunks[TKV_MAX_BATCH], slot[TKV_MAX_BATCH];
  // prefixes: tokens, first item, chunks, first row slot; their sequences are order[begin .. begin + count)
  int32_t p_len[TKV_MAX_BATCH], p_first[TKV_MAX_BATCH], p_chunks[TKV_MAX_BATCH], p_slot[TKV_MAX_BATCH];
  uint8_t p_begin[TKV_MAX_BATCH], p_count[TKV_MAX_BATCH], order[TKV_MAX_BATCH];
  uint8_t prefix_of[TKV_MAX_BATCH], rank[TKV_MAX_BATCH];  // of every sequence; 255: no prefix
};

__device__ inline floatx4 mfma(uintx4 a, uintx4 b, floatx4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
}
// (words by value: a bit cast applied directly to a vector's element reads element 0 with this compiler)
__device__ inline half2_t as_half2(uint32_t w) { return __builtin_bit_cast(half2_t, w); }
__device__ inline uint32_t as_word(half2_t h) { return __builtin_bit_cast(uint32_t, h); }

// Operand X (0 .. 7) of a block's codes, less C0: K: 4 tau + (c / 32), V: c / 16.  `w`: the lane's words of the block (2 bit: word
// X / 2; 4 bit: word X; 1 bit: word X / 4).  Register j holds two codes, p bits up in fp16's mantissa once 1024 is or-ed in:
// 1024 + code 2^p, which one multiply-add turns into the code exactly.  (`or_in`: 0x64006400 in a vector register, so that mask and
// or are one instruction, which takes one scalar.)
template <int BITS, int X, int C0>
__device__ inline void codes(const uint32_t* w, uint32_t or_in, half2_t (&c)[4]) {
  const uint32_t word = BITS == 4 ? w[X] : BITS == 2 ? w[X / 2] : w[X / 4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int bit = BITS == 4 ? 4 * j : BITS == 2 ? 2 * j + 8 * (X % 2) : j + 4 * (X % 4);
    const int p = bit % 8;  // (the upper eight bits of a half are brought down first)
    const uint32_t mask = (uint32_t)((1 << BITS) - 1) * 0x00010001u << p;
    const uint32_t x = ((bit >= 8 ? word >> 8 : word) & mask) | or_in;
    const _Float16 down = (_Float16)(1.f / (1 << p)), off = (_Float16)(-1024.f / (1 << p) - C0);
    c[j] = __builtin_elementwise_fma(as_half2(x), (half2_t){down, down}, (half2_t){off, off});
  }
}

__device__ inline uintx4 lds_read16(lds_at at) { return *(__attribute__((address_space(3))) uintx4*)at; }
__device__ inline void lds_write16(lds_at at, uintx4 v) { *(__attribute__((address_space(3))) uintx4*)at = v; }
__device__ inline uint32_t lds_word(lds_at at) { return *(__attribute__((address_space(3))) uint32_t*)at; }
__device__ inline uintx2 lds_read_tr(lds_at at) {
  return __builtin_bit_cast(uintx2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4*)at));
}
// 16 bytes per lane straight to LDS, in lane order from `to` (uniform) on; the caller waits (vmcnt).  By hand, so that the compiler
// makes no LDS read wait for loads of other slots.  (m0 is used by nothing else here: the compiler, which
// cannot be told of it, since it is reserved, never does; tests/test_lds_loads.py looks.)
__device__ inline void to_lds(const char* base, uint32_t lane_offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(lane_offset), "s"(base) : "memory");
}
__device__ inline void to_lds(const char* from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "memory");
}

template <int BITS>
constexpr int code_bytes() { return BITS == 4 ? 2048 : 1024; }  // LDS room of a block's K or V codes (1 bit: half of it used)
template <int BITS>
constexpr int slot_bytes() { return 2 * code_bytes<BITS>() + 1024; }
template <int BITS>
constexpr int code_zero() { return BITS == 1 ? 0 : BITS == 2 ? 1 : 8; }  // c0
template <int BITS>
constexpr int span_groups() { return BITS == 4 ? 8 : 16; }  // groups whose token-independent terms are worked out at once
// Two scalers in the parts whose products with codes are exact: at 4 bits the upper eight bits of the significand, then the lower three.
template <int BITS>
__device__ inline uint32_t scaler_part(uint32_t w, int part) {
  if (BITS < 4) return w;
  const uint32_t high = w & 0xFFF8FFF8u;
  return part == 0 ? high : as_word(as_half2(w) - as_half2(high));
}
template <int BITS, int NQ>
constexpr int lds_bytes() {
  constexpr int ring = kWaves * kSlots * slot_bytes<BITS>(), q = NQ * 4096, join = (NQ > 1 ? 2 : 1) * kWaves * 8192;
  constexpr int terms = kWaves * span_groups<BITS>() * NQ * 64;
  return (ring + q + terms > join ? ring + q + terms : join) + kWaves * 16 * NQ * 8 + 16;
}

// One segment's rows (16 NQ of them) over one chunk of its tokens.
template <int BITS, int GS, int NQ, int MAXQ>
__device__ __attribute__((always_inline)) inline void attend(const SharedParams& p, const SharedCache& c, int seq, int n, int h, int chunk, int chunks,
                              const uint8_t* order, int row0, int rows, int64_t slot0) {
  constexpr int G = 32 * GS, CB = code_bytes<BITS>(), SB = slot_bytes<BITS>();
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const lds_at lds0 = (lds_at)lds;
  const int lane = threadIdx.x % 64, kb = lane / 16, col = lane % 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  constexpr int kRing = kWaves * kSlots * SB;
  constexpr int kStats = lds_bytes<BITS, MAXQ>() - 16 - kWaves * 16 * MAXQ * 8, kOnes = lds_bytes<BITS, MAXQ>() - 16;
  constexpr int SPAN = span_groups<BITS>(), C0 = code_zero<BITS>(), kScalerParts = BITS == 4 ? 2 : 1;
  const lds_at ring = lds0 + wave * kSlots * SB, q_at = lds0 + kRing, stats = lds0 + kStats;
  const lds_at terms = q_at + MAXQ * 4096 + wave * SPAN * NQ * 64;  // [group][tile][16 columns] float32

  // blocks of the segment: quantized ones, then the ring's rows in pieces of 32; this wave's share of the chunk's
  const int nq = tkv::n_quantized(n, c.residual, G), coded = nq / 32, blocks = coded + (n - nq + 31) / 32;
  // (Waves of the upper half, which go first below, take three blocks where the others take two, once there are enough to divide so;
  // with even shares the lower half ran a third of the time alone: 62.0 -> 61.2 us for 131072 tokens under 16 sequences, 24.4 -> 23.6
  // for two prefixes of 48413 at 1 bit.)
  constexpr int kHalf = kWaves / 2;
  const bool many = blocks >= 4 * kWaves * chunks;
  const int low = many ? 2 : 1, high = many ? 3 : 1;
  const int part = chunk * kHalf * (low + high) + low * min(wave, kHalf) + high * max(wave - kHalf, 0), of = chunks * kHalf * (low + high);
  const int b0 = (int)((int64_t)blocks * part / of), b1 = (int)((int64_t)blocks * (part + (wave < kHalf ? low : high)) / of);
  const int64_t head = (int64_t)seq * p.hkv + h;
  const char* kc = c.k_codes + head * c.capacity * (16 * BITS);
  const char* vc = c.v_codes + head * c.capacity * (16 * BITS);
  // The block that is sent for next: its keys' and values' codes, and a lane's sixteen bytes of its scalers and zero-points: k_scale,
  // k_zero, v_scale, v_zero, 256 bytes each (values in groups of 64: 128, read twice).
  const char* next_k = kc + (int64_t)b0 * (512 * BITS);
  const char* next_v = vc + (int64_t)b0 * (512 * BITS);
  const char* next_meta;
  uint32_t step_even, step_odd;  // from an even block to the next, from an odd one (keys in groups of 64: every other time)
  {
    const int64_t per_head = (int64_t)c.capacity * (256 / G);  // bytes: tokens / G groups of 128 fp16; as many for values
    if (kb < 2) {
      next_meta = (kb ? c.k_zero : c.k_scale) + head * per_head + 16 * col + (int64_t)(b0 / GS) * 256;
      step_even = GS == 2 ? 0u : 256u;
      step_odd = 256u;
    } else {
      next_meta = (kb == 3 ? c.v_zero : c.v_scale) + head * per_head + 16 * (GS == 2 ? col % 8 : col) + (int64_t)b0 * (256 / GS);
      step_even = step_odd = 256u / GS;
    }
  }
  const uint32_t lane_at = BITS == 1 ? 16u * (uint32_t)(lane % 32) : 16u * (uint32_t)lane;
  auto stage = [&](int slot) {
    const uint32_t to = (uint32_t)(uintptr_t)(ring + slot * SB);
#pragma unroll
    for (int y = 0; y < CB / 1024; ++y) to_lds(next_k + 1024 * y, lane_at, to + 1024 * y);
#pragma unroll
    for (int y = 0; y < CB / 1024; ++y) to_lds(next_v + 1024 * y, lane_at, to + CB + 1024 * y);
    to_lds(next_meta, to + 2 * CB);
  };
  auto advance = [&](int j, int end) {  // from block j, where there is one behind it (otherwise it is sent for again)
    const uint32_t on = j + 1 < end ? 1u : 0u;
    next_k += on * (512 * BITS);
    next_v += on * (512 * BITS);
    next_meta += on * (GS == 2 && j % 2 == 0 ? step_even : step_odd);
  };
  constexpr int kLoads = 2 * (CB / 1024) + 1;
  const int c1 = min(b1, coded);  // quantized blocks [b0, c1), then pieces of the ring [max(b0, coded), b1)
  if (b0 < c1) {
    stage(0);
    advance(b0, c1);
    stage(1);
  }

  // the rows' queries in operand order, shared by all waves: wave w lays out tiles w, w + 8, ...
  for (int y = wave; y < 4 * NQ; y += kWaves) {
    const int row = 16 * (y / 4) + col, at = row0 + row;
    uintx4 v = {0u, 0u, 0u, 0u};
    if (row < rows) {
      const int b = order ? order[at / p.group] : seq, g = order ? at % p.group : at;
      const uint32_t* from = (const uint32_t*)(p.q + ((int64_t)b * p.hq + h * p.group + g) * TKV_D + 32 * (y % 4) + 8 * kb);
      v = (uintx4){from[0], from[1], from[2], from[3]};
    }
    lds_write16(q_at + y * 1024 + 16 * lane, v);
  }
  if (threadIdx.x == 0) lds_write16(lds0 + kOnes, (uintx4){0x3C003C00u, 0x3C003C00u, 0x3C003C00u, 0x3C003C00u});
  __syncthreads();

  // (Two waves of a SIMD in step wait for the matrix cores and for the vector unit at the same time; with one of them always first they
  // fall out of step: 65.9 -> 64.6 us (then) for 131072 tokens under 16 sequences, 138 -> 134 for 32770 under 64 at 4 bits.)
  if (wave >= kHalf) __builtin_amdgcn_s_setprio(2);
  floatx4 o[NQ][8], oz[NQ];  // oz: row u: weights with zero-points of channel group u, row 4 + u: with its scalers, row 8: the weights' sum
  float ref[NQ], sum[NQ];
#pragma unroll
  for (int t = 0; t < NQ; ++t) {
    ref[t] = kNone;
    sum[t] = 0.f;
    oz[t] = (floatx4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < 8; ++x) o[t][x] = (floatx4){0.f, 0.f, 0.f, 0.f};
  }
  // logits s, to which base[t] is to be added, to weights; Sum: the rounded weights are added up here, not by the operand's row of ones
  auto soften = [&](floatx4 (&s)[2][NQ], const float (&base)[NQ], uintx4 (&w)[NQ], auto Sum) {
    // (Whether a weight is too large, its exponent itself says, rounded once as it will be: with logits of 2^23 and more float32's steps
    // are 1 to 8, and a maximum rounded by itself can be below what the exponents come to.)
    float largest = -INFINITY;
    float top[NQ], less[NQ];
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
      top[t] = s[0][t][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) top[t] = fmaxf(top[t], s[i / 4][t][i % 4]);
      less[t] = base[t] + kShift - ref[t];
      largest = fmaxf(largest, __builtin_fmaf(top[t], p.scale2, less[t]));
    }
    if (__builtin_amdgcn_ballot_w64(largest > kLazy + kShift) != 0) {
#pragma unroll
      for (int t = 0; t < NQ; ++t) {
        const float next = fmaxf(ref[t], tkv::over_rows(__builtin_fmaf(top[t], p.scale2, base[t]), tkv::MaxOf{}));
        const float shrink = __builtin_amdgcn_exp2f(ref[t] - next);
        ref[t] = next;
        less[t] = base[t] + kShift - next;
        sum[t] *= shrink;
#pragma unroll
        for (int x = 0; x < 8; ++x) o[t][x] *= shrink;
        oz[t] *= shrink;
      }
    }
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
      half8 v;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i / 4][t][i % 4], p.scale2, less[t]));
        v[i] = (_Float16)e;
        if constexpr (decltype(Sum)::value) sum[t] += (float)v[i];
      }
      w[t] = __builtin_bit_cast(uintx4, v);
    }
  };

  // row col of the operand of zero-points and scalers: zero-points of u = col, scalers of u = col - 4 (rows of no u: whatever is there), ones
  const int zs_at = 2 * CB + (col % 8 < 4 ? 768 : 512) + 64 * (col % 4) + 16 * kb;
  uint32_t or_in = 0x64006400u;
  asm("" : "+v"(or_in));
  // The terms of SPAN groups from block j's on: sum_c q[c] (z[c] + c0 s[c]), in units of the exponent.
  auto work_out_terms = [&](int j) {
    const int g0 = j / GS, g_end = (c1 - 1) / GS;
    const int64_t row = (head * (c.capacity / G) + min(g0 + col % SPAN, g_end)) * 256 + 16 * kb;
    uintx4 z[4], sc[4];
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      z[m] = *(const uintx4*)(c.k_zero + row + 64 * m);
      if constexpr (C0 > 0) sc[m] = *(const uintx4*)(c.k_scale + row + 64 * m);
    }
    if constexpr (C0 > 1) {
#pragma unroll
      for (int m = 0; m < 4; ++m) sc[m] = __builtin_bit_cast(uintx4, __builtin_bit_cast(half8, sc[m]) * (_Float16)C0);  // (a power of two)
    }
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
      floatx4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const uintx4 q = lds_read16(q_at + 16 * lane + (4 * t + m) * 1024);
        v = mfma(z[m], q, v);
        if constexpr (C0 > 0) v = mfma(sc[m], q, v);
      }
      if (4 * kb < SPAN) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *(__attribute__((address_space(3))) float*)(terms + ((4 * kb + i) * NQ + t) * 64 + 4 * col) = v[i] * p.scale2;
      }
    }
  };

  auto words = [&](lds_at from, uint32_t* w) {
    if constexpr (BITS == 1) {
      w[0] = lds_word(from + 4 * lane);
      w[1] = lds_word(from + 4 * lane + 256);
    } else {
      const uintx4 a = lds_read16(from + 16 * lane);
      w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
      if constexpr (BITS == 4) {
        const uintx4 b = lds_read16(from + 16 * lane + 1024);
        w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
      }
    }
  };
  // A block's LDS reads go out a stage ahead of their use: the keys' codes and the first channels' scalers and queries during the
  // products of the block before, those of the next 32 channels during each quarter of the logits, the values' before the weights.
  uint32_t kw[8];
  uintx4 ks[2], q[2][NQ];
  auto read_channels = [&](int m, lds_at at) {  // 32 m on
    ks[m % 2] = lds_read16(at + 16 * kb + (2 * CB + 64 * m));
#pragma unroll
    for (int t = 0; t < NQ; ++t) q[m % 2][t] = lds_read16(q_at + 16 * lane + (4 * t + m) * 1024);
  };
  if (b0 < c1) {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");
    words(ring, kw);
    read_channels(0, ring);
  }
  int slot = 0, span_end = b0;
  lds_at term_at = terms;
  for (int j = b0; j < c1; ++j) {
    if (j >= span_end) {
      work_out_terms(j);
      span_end = (j / GS + SPAN) * GS;
      term_at = terms;
    }
    // (the next block but one goes where the previous block was, whose reads are done)
    advance(j + 1, c1);
    stage(slot == 0 ? 2 : slot - 1);
    const lds_at at = ring + slot * SB;
    slot = slot == kSlots - 1 ? 0 : slot + 1;
    floatx4 s[2][NQ];
#pragma unroll
    for (int t = 0; t < NQ; ++t) s[0][t] = s[1][t] = (floatx4){0.f, 0.f, 0.f, 0.f};
    auto keys = [&](auto M) {  // channels 32 m on
      constexpr int m = decltype(M)::value;
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (m < 3) read_channels(m + 1, at);
      half2_t code0[4], code1[4];
      codes<BITS, m, C0>(kw, or_in, code0);
      codes<BITS, 4 + m, C0>(kw, or_in, code1);
#pragma unroll
      for (int part = 0; part < kScalerParts; ++part) {
        uintx4 k0, k1;
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const uint32_t sw = scaler_part<BITS>(ks[m % 2][y], part);
          k0[y] = as_word(code0[y] * as_half2(sw));
          k1[y] = as_word(code1[y] * as_half2(sw));
        }
#pragma unroll
        for (int t = 0; t < NQ; ++t) {
          s[0][t] = mfma(k0, q[m % 2][t], s[0][t]);
          s[1][t] = mfma(k1, q[m % 2][t], s[1][t]);
        }
      }
    };
    keys(std::integral_constant<int, 0>{});
    keys(std::integral_constant<int, 1>{});
    keys(std::integral_constant<int, 2>{});
    float base[NQ];
#pragma unroll
    for (int t = 0; t < NQ; ++t) base[t] = __uint_as_float(lds_word(term_at + 4 * col + 64 * t));
    if (GS == 1 || j % 2 == 1) term_at += NQ * 64;
    keys(std::integral_constant<int, 3>{});
    constexpr int U = 128 / G;
    uint32_t vw[8];
    uintx4 vs[U], vz;
    words(at + CB, vw);
#pragma unroll
    for (int u = 0; u < U; ++u) vs[u] = lds_read16(at + 16 * kb + (2 * CB + 512 + 64 * u));
    vz = lds_read16(col == 8 ? lds0 + kOnes : at + zs_at);
    __builtin_amdgcn_sched_barrier(0);
    uintx4 w[NQ];
    soften(s, base, w, std::false_type{});
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");  // block j + 1 is there
    words(ring + slot * SB, kw);
    read_channels(0, ring + slot * SB);
    __builtin_amdgcn_sched_barrier(0);
    auto values = [&](auto X) {  // channels 16 x on
      constexpr int x = decltype(X)::value, u = x * 16 / G;
      half2_t cv[4];
      codes<BITS, x, C0>(vw, or_in, cv);
#pragma unroll
      for (int part = 0; part < kScalerParts; ++part) {
        uintx4 v;
#pragma unroll
        for (int y = 0; y < 4; ++y) v[y] = as_word(cv[y] * as_half2(scaler_part<BITS>(vs[u][y], part)));
#pragma unroll
        for (int t = 0; t < NQ; ++t) o[t][x] = mfma(v, w[t], o[t][x]);
      }
    };
#pragma unroll
    for (int t = 0; t < NQ; ++t) oz[t] = mfma(vz, w[t], oz[t]);
    values(std::integral_constant<int, 0>{});
    values(std::integral_constant<int, 1>{});
    values(std::integral_constant<int, 2>{});
    values(std::integral_constant<int, 3>{});
    values(std::integral_constant<int, 4>{});
    values(std::integral_constant<int, 5>{});
    values(std::integral_constant<int, 6>{});
    values(std::integral_constant<int, 7>{});
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (long there: this block's last reads, before its slot is given away)
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // no load may land after the ring is used otherwise

  for (int j = max(b0, coded); j < b1; ++j) {
    // 32 rows of the ring side by side (the ring's length and the first row are multiples of 32); those behind the last token are
    // not read: masked keys, values of zero
    const int t0 = nq + 32 * (j - coded), ring_len = c.residual + G, left = min(32, n - t0);
    const int64_t row = head * ring_len + t0 % ring_len;
    const auto vr = __builtin_amdgcn_make_buffer_rsrc((void*)(c.v_resid + row * 256), 0, left * 256, 0x00020000);
    const auto kr = __builtin_amdgcn_make_buffer_rsrc((void*)(c.k_resid + row * 256), 0, left * 256, 0x00020000);
    uintx4 vv[8];
#pragma unroll
    for (int y = 0; y < 8; ++y) vv[y] = __builtin_amdgcn_raw_buffer_load_b128(vr, 1024 * y + 16 * lane, 0, 0);
    uintx4 kk[8];
    const int token = 8 * (col / 4) + col % 4;
#pragma unroll
    for (int x = 0; x < 8; ++x) kk[x] = __builtin_amdgcn_raw_buffer_load_b128(kr, (token + 4 * (x / 4)) * 256 + 64 * (x % 4) + 16 * kb, 0, 0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int y = 0; y < 8; ++y) lds_write16(ring + 16 * lane + 1024 * y, vv[y]);
    floatx4 s[2][NQ];
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
      s[0][t] = s[1][t] = (floatx4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const uintx4 q = lds_read16(q_at + 16 * lane + (4 * t + m) * 1024);
        s[0][t] = mfma(kk[m], q, s[0][t]);
        s[1][t] = mfma(kk[4 + m], q, s[1][t]);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (8 * kb + i >= left) s[i / 4][t][i % 4] = -INFINITY;
    }
    uintx4 w[NQ];
    float base[NQ];
#pragma unroll
    for (int t = 0; t < NQ; ++t) base[t] = 0.f;
    soften(s, base, w, std::true_type{});
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      // tokens 8 kb to 8 kb + 7 of channel 16 x + col: two blocks of four rows, transposed
      const lds_at from = ring + ((8 * kb + col / 4) * 256 + 8 * (col % 4)) + 32 * x;
      const uintx2 lo = lds_read_tr(from), hi = lds_read_tr(from + 1024);
      const uintx4 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3);
#pragma unroll
      for (int t = 0; t < NQ; ++t) o[t][x] = mfma(v, w[t], o[t][x]);
    }
  }

#pragma unroll
  for (int t = 0; t < NQ; ++t)
#pragma unroll
    for (int u = 0; u < 128 / G; ++u) {
      const float zero = __shfl(oz[t][u], col, 64), scale = __shfl(oz[t][u], 16 + col, 64);
#pragma unroll
      for (int x = u * G / 16; x < (u + 1) * G / 16; ++x) o[t][x] += zero + C0 * scale;
    }

  // ---- the waves' results joined: references and sums first, then a tile of rows at a time, wave w channels 16 w on
  __syncthreads();
#pragma unroll
  for (int t = 0; t < NQ; ++t) {
    const float total = tkv::over_rows(sum[t], tkv::SumOf{}) + __shfl(oz[t][0], 32 + col, 64);
    if (kb == 0) {
      auto* st = (__attribute__((address_space(3))) float*)(stats + ((t * kWaves + wave) * 16 + col) * 8);
      st[0] = ref[t];
      st[1] = total;
    }
  }
  __syncthreads();
#pragma unroll
  for (int t = 0; t < NQ; ++t) {
    float m[kWaves], l = 0.f, top = kNone;
    const auto* st = (const __attribute__((address_space(3))) float*)(stats + (t * kWaves * 16 + col) * 8);
#pragma unroll
    for (int y = 0; y < kWaves; ++y) {
      m[y] = st[32 * y];
      top = fmaxf(top, m[y]);
    }
#pragma unroll
    for (int y = 0; y < kWaves; ++y) l = __builtin_fmaf(st[32 * y + 1], __builtin_amdgcn_exp2f(m[y] - top), l);
    const float mine = __builtin_amdgcn_exp2f(ref[t] - top);
    const lds_at area = lds0 + (t & 1) * kWaves * 8192;
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      floatx4 v = o[t][x] * mine;
      lds_write16(area + wave * 1024 + 16 * lane + x * kWaves * 1024, __builtin_bit_cast(uintx4, v));
    }
    __syncthreads();
    const int row = 16 * t + col;
#pragma unroll
    for (int z = 0; z < 8 / kWaves; ++z) {
      const int x = wave * (8 / kWaves) + z;
      floatx4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int y = 0; y < kWaves; ++y) v += __builtin_bit_cast(floatx4, lds_read16(area + x * kWaves * 1024 + 16 * lane + y * 1024));
      if (row < rows) *(floatx4*)(p.parts + (slot0 + row) * TKV_D + 16 * x + 4 * kb) = v;
    }
    if (row < rows && wave == 0 && kb == 0) *(float2*)(p.ml + (slot0 + row) * 2) = make_float2(top, l);
  }
}

template <int BITS, int GS, int NQ>
__global__ __launch_bounds__(64 * kWaves, NQ == 1 ? 4 : 2) void shared_attn_kernel(SharedParams p) {
  const int lane = threadIdx.x % 64;
  const int h = blockIdx.x % p.hkv, it = blockIdx.x / p.hkv;
  const bool own = it >= p.prefix_items;
  const int count = own ? p.batch : p.n_prefix;
  // the last segment that begins at or before the item (segments without items share their successor's beginning)
  const int at = min(lane, count - 1);
  const bool before = lane < count && (own ? p.first[at] : p.p_first[at]) <= it;
  const int x = __builtin_amdgcn_readfirstlane(__builtin_popcountll(__builtin_amdgcn_ballot_w64(before)) - 1);
  if (own) {
    const int chunk = it - p.first[x], chunks = p.chunks[x];
    attend<BITS, GS, 1, NQ>(p, p.cache[0], x, p.len[x], h, chunk, chunks, nullptr, 0, p.group,
                            p.slot[x] + (int64_t)(h * chunks + chunk) * p.group);
  } else {
    const int rows = p.p_count[x] * p.group, groups = (rows + 16 * NQ - 1) / (16 * NQ), r = it - p.p_first[x];
    const int chunk = r / groups, chunks = p.p_chunks[x], row0 = 16 * NQ * (r % groups);
    attend<BITS, GS, NQ, NQ>(p, p.cache[1], x, p.p_len[x], h, chunk, chunks, p.order + p.p_begin[x], row0, min(16 * NQ, rows - row0),
                             p.p_slot[x] + (int64_t)(h * chunks + chunk) * rows + row0);
  }
}

// Joins a query head's partial results, those of its prefix's chunks and of its own, a lane two channels.  ONE: a wave per head;
// otherwise a workgroup, every wave a quarter of the parts.  (64 sequences of 64 heads, about 10 parts each: 4.9 us with a wave,
// 11.0 with a workgroup; whole calls of 16 sequences of 32 heads, 29 parts: 67.7, 65.9; 8 of 32, about 40 parts: 27.5, 24.9.)
template <bool ONE>
__global__ __launch_bounds__(256) void shared_merge_kernel(SharedParams p) {
  __shared__ float acc_s[4][TKV_D], l_s[4], m_s[4];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int row = ONE ? 4 * blockIdx.x + wave : blockIdx.x, first = ONE ? 0 : wave;
  constexpr int kStep = ONE ? 1 : 4;
  if (row >= p.batch * p.hq) return;
  const int b = row / p.hq, head = row % p.hq, h = head / p.group, g = head % p.group;
  const int pf = p.prefix_of[b], at_p = min(pf, TKV_MAX_BATCH - 1);
  const bool none = pf == 255;
  const int rows = none ? 0 : p.p_count[at_p] * p.group, n_p = none ? 0 : p.p_chunks[at_p], n = n_p + p.chunks[b];
  const int64_t base_p = p.p_slot[at_p] + (int64_t)h * n_p * rows + p.rank[b] * p.group + g;
  const int64_t base_o = p.slot[b] + (int64_t)h * p.chunks[b] * p.group + g;
  float m = kNone, l = 0.f;
  float2 acc = make_float2(0.f, 0.f);
  // (requests of eight parts at a time, absent ones those of the first with a weight of zero)
  for (int i0 = first; i0 < n; i0 += 8 * kStep) {
    float2 st[8], v[8];
#pragma unroll
    for (int y = 0; y < 8; ++y) {
      const int i = i0 + kStep * y < n ? i0 + kStep * y : i0;
      const int64_t s = i < n_p ? base_p + (int64_t)i * rows : base_o + (int64_t)(i - n_p) * p.group;
      st[y] = *(const float2*)(p.ml + s * 2);
      v[y] = *(const float2*)(p.parts + s * TKV_D + 2 * lane);
    }
    float top = m;
#pragma unroll
    for (int y = 0; y < 8; ++y) top = fmaxf(top, st[y].x);
    const float shrink = __builtin_amdgcn_exp2f(m - top);
    m = top;
    l *= shrink;
    acc.x *= shrink;
    acc.y *= shrink;
#pragma unroll
    for (int y = 0; y < 8; ++y) {
      const float w = i0 + kStep * y < n ? __builtin_amdgcn_exp2f(st[y].x - m) : 0.f;
      l = __builtin_fmaf(st[y].y, w, l);
      acc.x = __builtin_fmaf(v[y].x, w, acc.x);
      acc.y = __builtin_fmaf(v[y].y, w, acc.y);
    }
  }
  if constexpr (ONE) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    *(__half2*)(p.out + (int64_t)row * TKV_D + 2 * lane) = __floats2half2_rn(acc.x * inv, acc.y * inv);
    return;
  }
  *(float2*)(acc_s[wave] + 2 * lane) = acc;
  if (lane == 0) l_s[wave] = l, m_s[wave] = m;
  __syncthreads();
  if (threadIdx.x >= TKV_D) return;
  const int c = threadIdx.x;
  const float top = fmaxf(fmaxf(m_s[0], m_s[1]), fmaxf(m_s[2], m_s[3]));
  float total = 0.f, v = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float f = __builtin_amdgcn_exp2f(m_s[w] - top);
    total = __builtin_fmaf(l_s[w], f, total);
    v = __builtin_fmaf(acc_s[w][c], f, v);
  }
  p.out[(int64_t)row * TKV_D + c] = __float2half_rn(total == 0.f ? 0.f : v / total);
}

// What a workgroup takes, in units of 0.8 ns: a block of 32 tokens for a row group of 16 NQ, and its fixed part (a first round
// trip, the join of its waves); measured at 2 bits and used for all (at 4 bits a block of 64 rows takes half as much again, which changes all
// prefixes' parts alike).
constexpr double block_cost(int nq) { return nq == 1 ? 200 : nq == 2 ? 300 : 464; }
constexpr double fixed_cost(int nq) { return nq == 1 ? 6000 : nq == 2 ? 8000 : 10000; }
constexpr int kWorkgroups = 256;  // workgroups at a time, at most: one per compute unit (it takes most of the LDS)

int tiles_of(int rows) { return rows <= 16 ? 1 : rows <= 32 ? 2 : 4; }

int64_t blocks_of(const tkv_quant_desc* d, int n) {
  const int nq = tkv::n_quantized(n, d->residual, d->group_size);
  return nq / 32 + (n - nq + 31) / 32;
}

// Row slots that any call may need: each segment's rows once per KV head, and those of the chunks beyond the first, of
// which there are at most kWorkgroups of 64 rows or of one sequence's.
int64_t max_slots(const tkv_quant_desc* d) { return 2 * (int64_t)d->batch * d->n_q_heads + kWorkgroups * (64 + 8); }

int32_t check_pair(const tkv_quant_desc* pd, const tkv_quant_desc* d) {
  int32_t st = tkv::check_quant_desc(pd);
  if (st == TKV_OK) st = tkv::check_quant_desc(d);
  if (st != TKV_OK) return st;
  if (pd->n_q_heads != d->n_q_heads || pd->n_kv_heads != d->n_kv_heads || pd->bits != d->bits || pd->group_size != d->group_size)
    return TKV_E_INVAL;
  return TKV_OK;
}

bool cache_ok(const tkv_quant_cache* c) {
  if (!c || !c->seq_len_host) return false;
  for (const void* x : {c->k_codes, c->k_scale, c->k_zero, c->v_codes, c->v_scale, c->v_zero, c->k_resid, c->v_resid})
    if (!x || ((uintptr_t)x & 15) != 0) return false;
  return true;
}

SharedCache cache_of(const tkv_quant_desc* d, const tkv_quant_cache* c) {
  return {(const char*)c->k_codes, (const char*)c->k_scale, (const char*)c->k_zero, (const char*)c->v_codes, (const char*)c->v_scale,
          (const char*)c->v_zero, (const char*)c->k_resid, (const char*)c->v_resid, d->residual, d->capacity};
}

template <int BITS, int GS, int NQ>
int32_t launch_shared(const SharedParams& p, int64_t items, hipStream_t s) {
  constexpr int lds = lds_bytes<BITS, NQ>();
  static_assert(lds <= 160 * 1024, "LDS of one compute unit");
  static const bool lds_ok = hipFuncSetAttribute(reinterpret_cast<const void*>(&shared_attn_kernel<BITS, GS, NQ>),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, lds) == hipSuccess;
  if (!lds_ok) return TKV_E_HIP;
  TKV_LAUNCH((shared_attn_kernel<BITS, GS, NQ>), dim3((uint32_t)(items * p.hkv)), 64 * kWaves, lds, s, p);
  return TKV_OK;
}
template <int BITS, int GS>
int32_t launch_tiles(const SharedParams& p, int tiles, int64_t items, hipStream_t s) {
  return tiles == 1 ? launch_shared<BITS, GS, 1>(p, items, s) : tiles == 2 ? launch_shared<BITS, GS, 2>(p, items, s) : launch_shared<BITS, GS, 4>(p, items, s);
}

}  // namespace

extern "C" int32_t tkv_quant_attn_decode_shared_sizes(const tkv_quant_desc* pd, const tkv_quant_desc* d, size_t* workspace_bytes) {
  const int32_t st = check_pair(pd, d);
  if (st != TKV_OK) return st;
  if (!workspace_bytes) return TKV_E_INVAL;
  *workspace_bytes = (size_t)max_slots(d) * kRowFloats * sizeof(float);
  return TKV_OK;
}

extern "C" int32_t tkv_quant_attn_decode_shared(const tkv_quant_desc* pd, const tkv_quant_cache* prefix, const tkv_quant_desc* d,
                                                const tkv_quant_cache* cache, const int32_t* prefix_of_host, const void* q, void* out,
                                                float sm_scale, void* workspace, size_t workspace_bytes, void* stream) {
  const int32_t st = check_pair(pd, d);
  if (st != TKV_OK) return st;
  if (!cache_ok(prefix) || !cache_ok(cache) || !q || !out || !workspace) return TKV_E_INVAL;
  if (((uintptr_t)q & 3) != 0 || ((uintptr_t)out & 3) != 0 || ((uintptr_t)workspace & 15) != 0) return TKV_E_INVAL;
  const float scale2 = sm_scale * 1.4426950408889634f;
  if (!(sm_scale > 0.f) || !(scale2 <= 3.402823466e38f)) return TKV_E_INVAL;
  for (int i = 0; i < pd->batch; ++i)
    if (prefix->seq_len_host[i] < 0 || prefix->seq_len_host[i] > pd->capacity) return TKV_E_INVAL;
  for (int b = 0; b < d->batch; ++b) {
    if (cache->seq_len_host[b] < 0 || cache->seq_len_host[b] > d->capacity) return TKV_E_INVAL;
    if (prefix_of_host && (prefix_of_host[b] < -1 || prefix_of_host[b] >= pd->batch)) return TKV_E_INVAL;
  }
  const int64_t slots_max = max_slots(d);
  if (workspace_bytes < (size_t)slots_max * kRowFloats * sizeof(float)) return TKV_E_WORKSPACE;

  SharedParams p;
  p.cache[0] = cache_of(d, cache);
  p.cache[1] = cache_of(pd, prefix);
  p.q = (const __half*)q;
  p.out = (__half*)out;
  p.parts = (float*)workspace;
  p.ml = (float*)workspace + slots_max * TKV_D;
  p.scale2 = scale2;
  p.hq = d->n_q_heads; p.hkv = d->n_kv_heads; p.group = d->n_q_heads / d->n_kv_heads;
  p.batch = d->batch; p.n_prefix = pd->batch;

  // sequences in the order of their prefixes
  int most = 0, at = 0;
  for (int i = 0; i < pd->batch; ++i) {
    p.p_len[i] = prefix->seq_len_host[i];
    p.p_begin[i] = (uint8_t)at;
    for (int b = 0; b < d->batch; ++b) {
      if ((prefix_of_host ? prefix_of_host[b] : 0) != i) continue;
      p.prefix_of[b] = (uint8_t)i;
      p.rank[b] = (uint8_t)(at - p.p_begin[i]);
      p.order[at++] = (uint8_t)b;
    }
    p.p_count[i] = (uint8_t)(at - p.p_begin[i]);
    if (p.p_count[i] > most) most = p.p_count[i];
  }
  int64_t own_blocks[TKV_MAX_BATCH], prefix_blocks[TKV_MAX_BATCH], longest = 0;
  const int tiles = tiles_of(most * p.group);
  auto groups_of = [&](int i) { return (p.p_count[i] * p.group + 16 * tiles - 1) / (16 * tiles); };
  double all = 0;
  for (int b = 0; b < d->batch; ++b) {
    if (prefix_of_host && prefix_of_host[b] < 0) p.prefix_of[b] = 255, p.rank[b] = 0;
    p.len[b] = cache->seq_len_host[b];
    own_blocks[b] = blocks_of(d, p.len[b]);
    all += (double)own_blocks[b] * block_cost(1);
    if (own_blocks[b] > longest) longest = own_blocks[b];
  }
  for (int i = 0; i < pd->batch; ++i) {
    prefix_blocks[i] = p.p_count[i] ? blocks_of(pd, p.p_len[i]) : 0;
    all += (double)prefix_blocks[i] * groups_of(i) * block_cost(tiles);
    if (prefix_blocks[i] > longest) longest = prefix_blocks[i];
  }
  all *= p.hkv;

  // Chunks of at most `per` each, no smaller than a block per wave.  Of a dozen sizes from an even share of everything on, the one with the
  // shortest time: rounds of the prefixes' workgroups, which come first, or everything shared out evenly, the last own
  // ones behind it.
  auto chunks_of = [](int64_t blocks, double cost, double per) {
    const double whole = (double)blocks * cost;
    int64_t n = (int64_t)(whole / per);
    if ((double)n * per < whole) ++n;
    const int64_t fill = (blocks + kWaves - 1) / kWaves;
    return (int32_t)(n < fill ? n : fill);
  };
  const auto s = (hipStream_t)stream;
  const int units = std::min(kWorkgroups, tkv::stream_compute_units(s));
  const double even = all / units > 1 ? all / units : 1;
  double best = even, least = 0;
  for (double per = even; per < 4 * even && per < 1.2 * (double)longest * block_cost(tiles) + 1; per *= 1.12) {
    double n_prefix = 0, n_own = 0, long_prefix = 0, long_own = 0, sum = 0;
    for (int i = 0; i < pd->batch; ++i) {
      const int n = chunks_of(prefix_blocks[i], block_cost(tiles), per), copies = groups_of(i) * p.hkv;
      if (n == 0) continue;
      const double each = (double)prefix_blocks[i] * block_cost(tiles) / n + fixed_cost(tiles);
      n_prefix += (double)n * copies;
      sum += each * n * copies;
      if (each > long_prefix) long_prefix = each;
    }
    for (int b = 0; b < d->batch; ++b) {
      const int n = chunks_of(own_blocks[b], block_cost(1), per);
      if (n == 0) continue;
      const double each = (double)own_blocks[b] * block_cost(1) / n + fixed_cost(1);
      n_own += (double)n * p.hkv;
      sum += each * n * p.hkv;
      if (each > long_own) long_own = each;
    }
    double time = (double)(int64_t)((n_prefix + units - 1) / units) * long_prefix;
    const double shared_out = sum / units + (n_prefix + n_own > units ? long_own / 2 : 0);
    if (shared_out > time) time = shared_out;
    if (long_own > time) time = long_own;
    if (least == 0 || time < least) least = time, best = per;
  }
  int64_t items = 0, slots = 0;
  for (int i = 0; i < pd->batch; ++i) {
    p.p_chunks[i] = chunks_of(prefix_blocks[i], block_cost(tiles), best);
    p.p_first[i] = (int32_t)items;
    p.p_slot[i] = (int32_t)slots;
    items += (int64_t)p.p_chunks[i] * groups_of(i);
    slots += (int64_t)p.p_chunks[i] * p.p_count[i] * p.group * p.hkv;
  }
  p.prefix_items = (int32_t)items;
  for (int b = 0; b < d->batch; ++b) {
    p.chunks[b] = chunks_of(own_blocks[b], block_cost(1), best);
    p.first[b] = (int32_t)items;
    p.slot[b] = (int32_t)slots;
    items += p.chunks[b];
    slots += (int64_t)p.chunks[b] * p.group * p.hkv;
  }
  int most_parts = 0;
  for (int b = 0; b < d->batch; ++b) {
    const int n = p.chunks[b] + (p.prefix_of[b] == 255 ? 0 : p.p_chunks[p.prefix_of[b]]);
    if (n > most_parts) most_parts = n;
  }
  if (slots > slots_max) return TKV_E_WORKSPACE;  // (cannot be)

  int32_t r = TKV_OK;
  if (items) {
    const int key = 10 * d->bits + d->group_size / 32;
    switch (key) {
      case 11: r = launch_tiles<1, 1>(p, tiles, items, s); break;
      case 12: r = launch_tiles<1, 2>(p, tiles, items, s); break;
      case 21: r = launch_tiles<2, 1>(p, tiles, items, s); break;
      case 22: r = launch_tiles<2, 2>(p, tiles, items, s); break;
      case 41: r = launch_tiles<4, 1>(p, tiles, items, s); break;
      default: r = launch_tiles<4, 2>(p, tiles, items, s); break;
    }
    if (r != TKV_OK) return r;
  }
  const uint32_t heads = (uint32_t)(p.batch * p.hq);
  if (most_parts <= 16) TKV_LAUNCH(shared_merge_kernel<true>, dim3((heads + 3) / 4), 256, 0, s, p);
  else TKV_LAUNCH(shared_merge_kernel<false>, dim3(heads), 256, 0, s, p);
  return TKV_OK;
}
