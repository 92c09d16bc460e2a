// Attention over whole prompts (tkv_prompt_attn): softmax(sm q K^T) V, causal or not, grouped heads, sequences of
// different lengths, chunks of a prompt over earlier keys, single tokens.
//
// The query heads of a KV head are rows of one matrix (row = token * G + head), so that a tile of keys and values
// serves all of them whatever their number, and a tile of rows spans few tokens: little of a causal tile is masked.
//
// Both products are transposed: S^T = K Q^T has a query per lane column, so a row's softmax statistics are
// one number per lane (two lanes share a row), and its weights already lie where O^T = V^T P^T wants them: the sixteen
// keys that a lane's weights belong to are read in that order on the V side (a sum over keys does not mind their order), by
// LDS reads that transpose 4 x 16 elements on the way.  One pass over the keys: running maximum and
// sum in float32, weights rounded to the inputs' type for the second product (off by at most 2^-11 or 2^-8 of each, beside the
// output's own rounding of as much: against float64 2.6e-4 of the outputs' norm in fp16, 2.1e-4 of them the latter).  They are divided
// by the sum of the unrounded ones: over keys that differ the errors differ and mostly cancel, over equal keys all weights are off
// alike, and so is the output, by as much again as its own rounding at most.  (Divided by the sum of the rounded ones, a mixed product
// per two of them, equal values came out exactly: 16384 tokens in fp16 2150 -> 2210 us, packed prompts in bfloat16 885 -> 920, with no
// change of the error over keys that differ.  Not kept: the logarithm of the sum would need the other sum beside it.)
//
// Long prompts fill no unit: the matrix cores are busy for 52 % of the time, the vector units for 44 % or more, and LDS for about 37 %
// (a workgroup reads 128 KiB of keys, at up to 221 bytes a clock and compute unit as measured, and 128 KiB of values, transposing,
// 150 bytes a clock, in a tile's 3950 clocks).  A turn (below) lasts 1975 clocks for 1024 of products: what bounds it is the wait of
// products for the reads just before them and of the halves for each other, and the clock, which falls to 1.6-1.8 GHz.  32 query
// heads over 8, causal: 4096 tokens 147-152 us (905-935 TFLOP/s), 16384 2090-2180 us (1010-1050; the same products alone 1553 us,
// without the LDS reads 1770).  A workgroup's beginning and end, about 9 us with one of them on a unit, are hidden by nothing: a tenth
// of 4096 tokens.  64 rows a wave would halve the reads; as the compiler placed them, 69 registers spilled.
#include <algorithm>

#include "tkv_common.h"

namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx8 __attribute__((ext_vector_type(8)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));
typedef uint32_t uintx2 __attribute__((ext_vector_type(2)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 bhalf8 __attribute__((ext_vector_type(8)));

constexpr int kKeys = 64;       // keys of a tile
constexpr int kWaves = 8;
constexpr int kRows = 32 * kWaves;  // rows of a workgroup
constexpr int kMaxParts = 256;      // partial results that the workspace has room for: one per compute unit
constexpr int kPartFloats = kRows * (TKV_D + 2);
// Weights are 2^(logit - reference + kShift): the reference follows the running maximum only when a weight is above 2^15, inside
// fp16's range, and fp16's subnormal numbers begin 2^-21 below the reference's weight, not 2^-14.
constexpr float kShift = 7.f;
template <typename T>
constexpr uint32_t too_large() { return __is_same(T, _Float16) ? 0x7800u : 0x4700u; }  // 2^15's bits
constexpr float kNone = -3.402823466e38f;  // reference of a row without a key so far (finite: kNone - kNone is 0)

struct PromptSeq {
  int32_t q_start, q_len, k_start, k_len;
};

struct PromptParams {
  const void* q;
  const void* k;
  const void* v;
  void* out;
  float* lse;    // NULL: not wanted
  float* parts;  // [part][rows of a tile][128] weighted sums
  float* ml;     // [part][rows of a tile][2] (reference, sum)
  int64_t q_st, q_sh, k_st, k_sh, v_st, v_sh, o_st, o_sh;
  int32_t hq, hkv, group, batch, causal;
  float scale2;  // sm_scale * log2(e)
  PromptSeq seq[TKV_MAX_BATCH];
  int32_t first_item[TKV_MAX_BATCH];  // in (row tile, piece) pairs
  int32_t first_part[TKV_MAX_BATCH];  // -1: the sequence's rows are not split
  int32_t pieces[TKV_MAX_BATCH];
  int32_t first_row[TKV_MAX_BATCH];   // of the split sequences' rows (of one KV head), for the joining launch
  int32_t tile_rows;                  // rows of a tile: kRows, or kFew
  int32_t split_rows, most_pieces;
};

template <typename T>
__device__ inline floatx16 mfma32(uintx4 a, uintx4 b, floatx16 c) {
  if constexpr (__is_same(T, _Float16))
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bhalf8, a), __builtin_bit_cast(bhalf8, b), c, 0, 0, 0);
}

template <typename T>
__device__ inline uintx4 pack8(floatx8 x) {
  typedef T T8 __attribute__((ext_vector_type(8)));
  return __builtin_bit_cast(uintx4, __builtin_convertvector(x, T8));
}

typedef __attribute__((address_space(3))) char lds_char;

__device__ inline uintx4 lds_read16(lds_char* at) {
  return *(__attribute__((address_space(3))) uintx4*)at;
}
// 4 x 16 elements transposed over sixteen lanes: lane 4 r + c of the sixteen names row r's columns 4 c to 4 c + 3,
// lane c receives column c of the four rows.
__device__ inline uintx2 lds_read_tr(lds_char* at) {
  return __builtin_bit_cast(uintx2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4*)at));
}

// 16 bytes per lane from a descriptor's array straight to LDS, in lane order from `to` (uniform) on.  By hand, because the
// compiler lets every transposing LDS read wait for all such loads, those of the next tile's buffer too; nothing lands in
// registers, and the caller waits itself (vmcnt) before anyone reads the buffer.  (m0 is used by nothing else here.)
__device__ inline void to_lds(__amdgpu_buffer_rsrc_t from, uint32_t to, uint32_t lane_offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(lane_offset), "s"(from) : "memory");
}

__device__ inline float other_half(float v, int half) {
  const auto s = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  const uint32_t a = s[0], b = s[1];
  return __builtin_bit_cast(float, half ? a : b);
}

// What a workgroup works on: sequence, row tile, piece of the tile's keys.
struct Item {
  int b, tile, piece;
};
__device__ inline Item find_item(const PromptParams& p, int it) {
  // the last sequence that begins at or before the item; sequences without rows share their successor's beginning
  const int lane = threadIdx.x % 64;
  const bool before = lane < p.batch && p.first_item[min(lane, p.batch - 1)] <= it;
  Item x;
  x.b = __builtin_popcountll(__builtin_amdgcn_ballot_w64(before)) - 1;
  x.b = __builtin_amdgcn_readfirstlane(x.b);
  const int r = it - p.first_item[x.b], pieces = p.pieces[x.b];
  const int tiles = (p.seq[x.b].q_len * p.group + kRows - 1) / kRows;
  x.tile = tiles - 1 - r / pieces;  // the tiles with the most keys first
  x.piece = r % pieces;
  return x;
}

// A wave's work on a tile of 64 keys is two products on the matrix cores, 1024 cycles, and the softmax between them on the vector
// units, about 900.  Two waves of a SIMD left to themselves fall into step and wait for the same unit, so the workgroup's two halves
// (waves 0 to 3 and 4 to 7: one of each on every SIMD) take turns (16384 tokens: 2267 -> 2110 us): while one multiplies (the weights of its last tile with the
// values, the queries with the next keys), the other works out weights, and a barrier changes the parts.
template <typename T>
__global__ __launch_bounds__(64 * kWaves, 2) void prompt_attn_kernel(PromptParams p) {
  __shared__ __attribute__((aligned(1024))) char lds[2 * 2 * kKeys * TKV_D * 2];  // two K tiles, two V tiles
  constexpr int kTile = kKeys * TKV_D * 2;
  const int lane = threadIdx.x % 64, half = lane / 32, col = lane % 32;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int late = wave / (kWaves / 2);
  const int h = blockIdx.x % p.hkv;
  const Item it = find_item(p, blockIdx.x / p.hkv);
  const PromptSeq sq = p.seq[it.b];
  const int rows = sq.q_len * p.group, ahead = sq.k_len - sq.q_len;

  // keys that the workgroup's last row sees, then this piece of them
  const int last_row = min(rows, (it.tile + 1) * kRows) - 1;
  const int seen = p.causal ? max(0, last_row / p.group + ahead + 1) : sq.k_len;  // (<= k_len: the last token's is k_len)
  const int all_tiles = (seen + kKeys - 1) / kKeys, pieces = p.pieces[it.b];
  const int t0 = (int)((int64_t)all_tiles * it.piece / pieces), t1 = (int)((int64_t)all_tiles * (it.piece + 1) / pieces);

  // this lane's row, and the last key it sees
  const int row = it.tile * kRows + 32 * wave + col;
  const int row_ok = min(row, rows - 1), token = row_ok / p.group, head = row_ok - token * p.group;
  const int limit = p.causal ? token + ahead : sq.k_len - 1;
  // ... and those of the wave's first and last row
  const int w_first = min(it.tile * kRows + 32 * wave, rows - 1), w_last = min(it.tile * kRows + 32 * wave + 31, rows - 1);
  const int limit_low = p.causal ? w_first / p.group + ahead : sq.k_len - 1;
  const int limit_high = p.causal ? w_last / p.group + ahead : sq.k_len - 1;
  const bool wave_on = it.tile * kRows + 32 * wave < rows;
  const int my_end = wave_on ? min(t1, limit_high / kKeys + (limit_high >= 0 ? 1 : 0)) : t0;  // the wave has work in [t0, my_end)

  uintx4 qf[8];
  {
    const T* q = (const T*)p.q + ((int64_t)(sq.q_start + token) * p.q_st + (int64_t)(h * p.group + head) * p.q_sh + 8 * half);
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) qf[kk] = *(const uintx4*)(q + 16 * kk);
  }

  // staging: an instruction of a wave brings four rows; LDS keeps a row's sixteen 16-byte places in an order that depends on the
  // row, so that the reads below (a column of keys, a block of four keys) meet all banks
  constexpr int kLoads = 16 / kWaves;  // per wave and tile of keys or values
  uint32_t k_off[kLoads], v_off[kLoads];
#pragma unroll
  for (int j = 0; j < kLoads; ++j) {
    const int r = 4 * (kLoads * wave + j) + lane / 16, place = lane % 16;
    k_off[j] = (uint32_t)(r * p.k_st * 2) + 16u * (uint32_t)(place ^ (r & 15));
    v_off[j] = (uint32_t)(r * p.v_st * 2) + 16u * (uint32_t)(place ^ (((r & 3) << 2) | ((r >> 2) & 3)));
  }
  const char* k_base = (const char*)p.k + ((int64_t)sq.k_start * p.k_st + (int64_t)h * p.k_sh) * 2;
  const char* v_base = (const char*)p.v + ((int64_t)sq.k_start * p.v_st + (int64_t)h * p.v_sh) * 2;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)lds;
  auto stage = [&](const char* base, int64_t st, const uint32_t (&off)[kLoads], int t, uint32_t to) {
    const int left = min(kKeys, sq.k_len - t * kKeys);  // rows behind the sequence's last read as zeros
    const auto r = __builtin_amdgcn_make_buffer_rsrc((void*)(base + (int64_t)t * kKeys * st * 2), 0, (int)((left - 1) * st * 2 + TKV_D * 2), 0x00020000);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) to_lds(r, to + 1024 * (kLoads * wave + j), off[j]);
  };
  // K tile t goes to buffer t - t0 mod 2, V tile t to the two behind; everyone has left a buffer two turns before it is filled again
  auto stage_k = [&](int t) { if (t < t1) stage(k_base, p.k_st, k_off, t, lds0 + ((t - t0) & 1) * kTile); };
  auto stage_v = [&](int t) { if (t < t1) stage(v_base, p.v_st, v_off, t, lds0 + (2 + ((t - t0) & 1)) * kTile); };

  // LDS places of the operands, without buffer, key step and tile
  lds_char* ka[8];
  lds_char* va[8];
#pragma unroll
  for (int kk = 0; kk < 8; ++kk) ka[kk] = (lds_char*)lds + (col * 256 + 16 * ((2 * kk + half) ^ (col & 15)));
  {
    const int l16 = lane % 16, right = (lane / 16) % 2;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int key = 8 * s + 4 * half + l16 / 4;
        const int place = (4 * dt + 2 * right + (l16 % 4) / 2) ^ (((key & 3) << 2) | ((key >> 2) & 3));
        va[2 * dt + s] = (lds_char*)lds + (2 * kTile + key * 256 + 16 * place + 8 * (l16 % 2));
      }
  }

  floatx16 o[4], s[2];
  uintx4 pf[4];
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
  float ref = kNone, sum = 0.f;

  auto logits = [&](int t) {  // of tile t, into s
    const int at = ((t - t0) & 1) * kTile;
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[y][i] = 0.f;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk)
#pragma unroll
      for (int y = 0; y < 2; ++y) s[y] = mfma32<T>(lds_read16(ka[kk] + at + 8192 * y), qf[kk], s[y]);
  };
  auto products = [&](int t) {  // the weights of tile t with its values
    const int at = ((t - t0) & 1) * kTile;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) {
        const uintx2 lo = lds_read_tr(va[2 * dt] + at + 4096 * ks), hi = lds_read_tr(va[2 * dt + 1] + at + 4096 * ks);
        const uintx4 vf = __builtin_shufflevector(lo, hi, 0, 1, 2, 3);
        o[dt] = mfma32<T>(vf, pf[ks], o[dt]);
      }
  };
  auto weights = [&](int t) {
    const int key0 = t * kKeys;
    if (key0 + kKeys - 1 > limit_low || key0 + kKeys > sq.k_len) {
#pragma unroll
      for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          s[y][i] = key0 + 32 * y + 8 * (i / 4) + 4 * half + i % 4 <= limit ? s[y][i] : -INFINITY;
    }
    // The weights at once: they are positive, so their bits compare as numbers, two at a time, and the logits' maximum is worked out
    // only where one is too large.
    typedef uint16_t ushort2_t __attribute__((ext_vector_type(2)));
    float part;
    auto weigh = [&] {
      const float less = kShift - ref;
      part = 0.f;
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        floatx8 e;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[y / 2][8 * (y % 2) + i], p.scale2, less));
          part += e[i];
        }
        pf[y] = pack8<T>(e);
      }
    };
    weigh();
    ushort2_t large = {0, 0};
#pragma unroll
    for (int y = 0; y < 4; ++y)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t x = pf[y][i];
        large = __builtin_elementwise_max(large, __builtin_bit_cast(ushort2_t, x));
      }
    if (__builtin_amdgcn_ballot_w64(max((uint32_t)large.x, (uint32_t)large.y) > too_large<T>()) != 0) {
      float top = fmaxf(s[0][0], s[1][0]);
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, fmaxf(s[0][i], s[1][i]));
      top = fmaxf(top, other_half(top, half)) * p.scale2;
      const float next = fmaxf(ref, top), shrink = __builtin_amdgcn_exp2f(ref - next);
      ref = next;
      sum *= shrink;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) o[dt] *= shrink;
      weigh();
    }
    sum += part;
  };

  // (The query rows are waited for here: the compiler, which does not know of the loads to LDS, would wait for them and those
  // inside the loop.)
#pragma unroll
  for (int kk = 0; kk < 8; ++kk) asm volatile("" : "+v"(qf[kk]));
  stage_k(t0);
  asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
  // Turn 2 i: the early half multiplies (tile i), the late half works out weights (of i - 1); turn 2 i + 1: the other way round.  K tile
  // i + 1 and V tile i are sent for at the beginning of turn 2 i and waited for at the end of turn 2 i + 1.
  if (late) {
    stage_k(t0 + 1);
    stage_v(t0);
    asm volatile("s_barrier" ::: "memory");
  }
  for (int t = t0; t < t1; ++t) {
    if (!late) {
      stage_k(t + 1);
      stage_v(t);
    }
    __builtin_amdgcn_s_setprio(1);
    if (t > t0 && t - 1 < my_end) products(t - 1);
    if (t < my_end) logits(t);
    __builtin_amdgcn_s_setprio(0);
    if (late) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    if (late) {
      stage_k(t + 2);
      stage_v(t + 1);
    }
    if (t < my_end) weights(t);
    if (!late) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  }
  if (t1 > t0 && t1 - 1 < my_end) products(t1 - 1);
  if (!late) asm volatile("s_barrier" ::: "memory");  // (as many as the late half)

  sum += other_half(sum, half);
  if (!wave_on || row >= rows) return;
  if (p.first_part[it.b] >= 0) {
    const size_t part = (size_t)p.first_part[it.b] + ((size_t)it.tile * pieces + it.piece) * p.hkv + h;
    const int r = 32 * wave + col;
    if (half == 0) *(float2*)(p.ml + (part * kRows + r) * 2) = make_float2(ref, sum);
    float* to = p.parts + (part * kRows + r) * TKV_D;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int y = 0; y < 4; ++y)
        *(floatx4*)(to + 32 * dt + 8 * y + 4 * half) = (floatx4){o[dt][4 * y], o[dt][4 * y + 1], o[dt][4 * y + 2], o[dt][4 * y + 3]};
    return;
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;  // (no key: zeros)
  T* to = (T*)p.out + ((int64_t)(sq.q_start + token) * p.o_st + (int64_t)(h * p.group + head) * p.o_sh);
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      typedef T T4 __attribute__((ext_vector_type(4)));
      const floatx4 x = (floatx4){o[dt][4 * y], o[dt][4 * y + 1], o[dt][4 * y + 2], o[dt][4 * y + 3]} * inv;
      *(T4*)(to + 32 * dt + 8 * y + 4 * half) = __builtin_convertvector(x, T4);
    }
  if (p.lse && half == 0)
    p.lse[(int64_t)(sq.q_start + token) * p.hq + h * p.group + head] =
        sum == 0.f ? -INFINITY : (ref - kShift + __builtin_amdgcn_logf(sum)) * 0.69314718055994531f;
}

// Few rows (single tokens, a few tokens of few heads: up to 32 of a sequence and KV head).  The keys' bytes bound this:
// every wave takes 32-key tiles of its own through a ring of two of its own, with no barrier until the waves join.
// (Single tokens of four sequences, 201 MB of keys and values: 34 us, 5.9 TB/s, and 4 us for the join.  With this kernel / with the one
// above, 32 query heads over 8: a token over 500 keys 8.5 / 11.5 us, 8 over 32768 of four sequences 101 / 111, 4 over 2000 of 64 95 / 103;
// a token over 32768 28.4 / 27.8.)
constexpr int kFew = 32, kFewWaves = 4, kFewKeys = 32;

template <typename T>
__global__ __launch_bounds__(64 * kFewWaves, 1) void prompt_few_kernel(PromptParams p) {
  constexpr int kTile = kFewKeys * TKV_D * 2;
  extern __shared__ __attribute__((aligned(1024))) char few_lds[];  // [wave][2][K, V tile]
  const int lane = threadIdx.x % 64, half = lane / 32, col = lane % 32;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int h = blockIdx.x % p.hkv;
  const Item it = find_item(p, blockIdx.x / p.hkv);
  const PromptSeq sq = p.seq[it.b];
  const int rows = sq.q_len * p.group, ahead = sq.k_len - sq.q_len, pieces = p.pieces[it.b];
  const int all_tiles = (sq.k_len + kFewKeys - 1) / kFewKeys;
  const int share = it.piece * kFewWaves + wave, shares = pieces * kFewWaves;
  const int t0 = (int)((int64_t)all_tiles * share / shares), t1 = (int)((int64_t)all_tiles * (share + 1) / shares);
  const int row_ok = min(col, rows - 1), token = row_ok / p.group, head = row_ok - token * p.group;
  const int limit = p.causal ? token + ahead : sq.k_len - 1;
  const int limit_low = p.causal ? ahead : sq.k_len - 1;

  uint32_t k_off[8], v_off[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int r = 4 * j + lane / 16, place = lane % 16;
    k_off[j] = (uint32_t)(r * p.k_st * 2) + 16u * (uint32_t)(place ^ (r & 15));
    v_off[j] = (uint32_t)(r * p.v_st * 2) + 16u * (uint32_t)(place ^ (((r & 3) << 2) | ((r >> 2) & 3)));
  }
  const char* k_base = (const char*)p.k + ((int64_t)sq.k_start * p.k_st + (int64_t)h * p.k_sh) * 2;
  const char* v_base = (const char*)p.v + ((int64_t)sq.k_start * p.v_st + (int64_t)h * p.v_sh) * 2;
  lds_char* const ring = (lds_char*)few_lds + wave * 4 * kTile;
  const uint32_t ring0 = (uint32_t)(uintptr_t)ring;
  auto stage = [&](int t) {
    t = min(t, t1 - 1);  // (as many loads in every step)
    const int left = min(kFewKeys, sq.k_len - t * kFewKeys);  // rows behind the sequence's last read as zeros
    const auto kr = __builtin_amdgcn_make_buffer_rsrc((void*)(k_base + (int64_t)t * kFewKeys * p.k_st * 2), 0, (int)((left - 1) * p.k_st * 2 + TKV_D * 2), 0x00020000);
    const auto vr = __builtin_amdgcn_make_buffer_rsrc((void*)(v_base + (int64_t)t * kFewKeys * p.v_st * 2), 0, (int)((left - 1) * p.v_st * 2 + TKV_D * 2), 0x00020000);
    return [=](int buf) {
      const uint32_t to = ring0 + (uint32_t)(buf * 2 * kTile);
#pragma unroll
      for (int j = 0; j < 8; ++j) to_lds(kr, to + 1024 * j, k_off[j]);
#pragma unroll
      for (int j = 0; j < 8; ++j) to_lds(vr, to + kTile + 1024 * j, v_off[j]);
    };
  };
  if (t0 < t1) stage(t0)(0);
  uintx4 qf[8];
  {
    const T* q = (const T*)p.q + ((int64_t)(sq.q_start + token) * p.q_st + (int64_t)(h * p.group + head) * p.q_sh + 8 * half);
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) qf[kk] = *(const uintx4*)(q + 16 * kk);
  }
  lds_char* ka[8];
  lds_char* va[8];
#pragma unroll
  for (int kk = 0; kk < 8; ++kk) ka[kk] = ring + (col * 256 + 16 * ((2 * kk + half) ^ (col & 15)));
  {
    const int l16 = lane % 16, right = (lane / 16) % 2;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int key = 8 * s + 4 * half + l16 / 4;
        const int place = (4 * dt + 2 * right + (l16 % 4) / 2) ^ (((key & 3) << 2) | ((key >> 2) & 3));
        va[2 * dt + s] = ring + (kTile + key * 256 + 16 * place + 8 * (l16 % 2));
      }
  }
  floatx16 o[4];
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
  float ref = kNone, sum = 0.f;
#pragma unroll
  for (int kk = 0; kk < 8; ++kk) asm volatile("" : "+v"(qf[kk]));  // (waited for here, not in the loop)

  for (int t = t0; t < t1; ++t) {
    const int at = ((t - t0) & 1) * 2 * kTile, key0 = t * kFewKeys;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the other buffer's reads are done)
    stage(t + 1)((t + 1 - t0) & 1);
    asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
    floatx16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) s = mfma32<T>(lds_read16(ka[kk] + at), qf[kk], s);
    if (key0 + kFewKeys - 1 > limit_low || key0 + kFewKeys > sq.k_len) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = key0 + 8 * (i / 4) + 4 * half + i % 4 <= limit ? s[i] : -INFINITY;
    }
    float top = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
    top = fmaxf(top, other_half(top, half)) * p.scale2;
    if (__builtin_amdgcn_ballot_w64(top > ref + 8.f) != 0) {
      const float next = fmaxf(ref, top), shrink = __builtin_amdgcn_exp2f(ref - next);
      ref = next;
      sum *= shrink;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) o[dt] *= shrink;
    }
    const float less = kShift - ref;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], p.scale2, less));
      sum += s[i];
    }
    uintx4 pf[2];
    pf[0] = pack8<T>(__builtin_shufflevector(s, s, 0, 1, 2, 3, 4, 5, 6, 7));
    pf[1] = pack8<T>(__builtin_shufflevector(s, s, 8, 9, 10, 11, 12, 13, 14, 15));
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) {
        const uintx2 lo = lds_read_tr(va[2 * dt] + at + 4096 * ks), hi = lds_read_tr(va[2 * dt + 1] + at + 4096 * ks);
        o[dt] = mfma32<T>(__builtin_shufflevector(lo, hi, 0, 1, 2, 3), pf[ks], o[dt]);
      }
  }
  sum += other_half(sum, half);
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // no load may land after the ring is used otherwise
  __syncthreads();

  // the waves joined: everyone's sums and references into LDS, then wave w works out channels 32 w to 32 w + 31
  float* const ml_s = (float*)few_lds;                              // [wave][32][2]
  float* const o_s = (float*)few_lds + kFewWaves * kFew * 2;        // [wave][32 rows][132]
  constexpr int kRowStride = TKV_D + 4;
  if (half == 0) {
    ml_s[(wave * kFew + col) * 2] = ref;
    ml_s[(wave * kFew + col) * 2 + 1] = sum;
  }
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int y = 0; y < 4; ++y)
      *(floatx4*)(o_s + (wave * kFew + col) * kRowStride + 32 * dt + 8 * y + 4 * half) = (floatx4){o[dt][4 * y], o[dt][4 * y + 1], o[dt][4 * y + 2], o[dt][4 * y + 3]};
  __syncthreads();
  if (col >= rows) return;
  float m[kFewWaves], top = kNone, total = 0.f;
#pragma unroll
  for (int w = 0; w < kFewWaves; ++w) top = fmaxf(top, m[w] = ml_s[(w * kFew + col) * 2]);
#pragma unroll
  for (int w = 0; w < kFewWaves; ++w) {
    m[w] = __builtin_amdgcn_exp2f(m[w] - top);
    total = __builtin_fmaf(ml_s[(w * kFew + col) * 2 + 1], m[w], total);
  }
  floatx4 x[4];  // row col, channels 32 wave + 16 half + 0 .. 15
  const int c0 = 32 * wave + 16 * half;
#pragma unroll
  for (int y = 0; y < 4; ++y) {
    x[y] = (floatx4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) x[y] += *(const floatx4*)(o_s + (w * kFew + col) * kRowStride + c0 + 4 * y) * m[w];
  }
  if (p.first_part[it.b] >= 0) {
    const size_t part = (size_t)p.first_part[it.b] + (size_t)it.piece * p.hkv + h;
    if (wave == 0 && half == 0) *(float2*)(p.ml + (part * kFew + col) * 2) = make_float2(top, total);
    float* to = p.parts + (part * kFew + col) * TKV_D + c0;
#pragma unroll
    for (int y = 0; y < 4; ++y) *(floatx4*)(to + 4 * y) = x[y];
    return;
  }
  const float inv = total == 0.f ? 0.f : 1.f / total;  // (no key: zeros)
  T* to = (T*)p.out + ((int64_t)(sq.q_start + token) * p.o_st + (int64_t)(h * p.group + head) * p.o_sh) + c0;
#pragma unroll
  for (int y = 0; y < 2; ++y)
    *(uintx4*)(to + 8 * y) = pack8<T>(__builtin_shufflevector(x[2 * y] * inv, x[2 * y + 1] * inv, 0, 1, 2, 3, 4, 5, 6, 7));
  if (p.lse && wave == 0 && half == 0)
    p.lse[(int64_t)(sq.q_start + token) * p.hq + h * p.group + head] =
        total == 0.f ? -INFINITY : (top - kShift + __builtin_amdgcn_logf(total)) * 0.69314718055994531f;
}

// Joins the pieces of the split rows, a lane two channels.  ONE: a wave per row; otherwise a workgroup, every wave a quarter of the pieces.
// (Whole calls, again and again on the same inputs, with a workgroup / a wave per row: 1024 tokens of 32 heads over 2048 keys in 2 pieces
// 98 / 64 us, 512 over 4096 in 4 85 / 55, 333 over 65869 in 5 398 / 386; one token over 32768, in 32 pieces, 27.8 with a workgroup.)
template <typename T, bool ONE>
__global__ __launch_bounds__(256) void prompt_merge_kernel(PromptParams p) {
  __shared__ float acc_s[4][TKV_D], l_s[4], m_s[4];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int item = ONE ? 4 * blockIdx.x + wave : blockIdx.x, first = ONE ? 0 : wave;
  constexpr int kStep = ONE ? 1 : 4;
  if (item >= p.split_rows * p.hkv) return;
  const int h = item % p.hkv, at = item / p.hkv;
  // the last sequence that begins at or before the row (those that are not split share their successor's beginning)
  const bool before = lane < p.batch && p.first_row[min(lane, p.batch - 1)] <= at;
  const int b = __builtin_amdgcn_readfirstlane(__builtin_popcountll(__builtin_amdgcn_ballot_w64(before)) - 1);
  const int row = at - p.first_row[b], tile = row / p.tile_rows, r = row - tile * p.tile_rows;
  const int token = row / p.group, head = row - token * p.group, pieces = p.pieces[b];
  const size_t slot0 = ((size_t)p.first_part[b] + (size_t)tile * pieces * p.hkv + h) * p.tile_rows + r;
  const size_t step = (size_t)p.hkv * p.tile_rows;
  float m = kNone, l = 0.f;
  float2 acc = make_float2(0.f, 0.f);
  // (requests of eight pieces at a time, absent ones those of the first with a weight of zero)
  for (int i0 = first; i0 < pieces; i0 += 8 * kStep) {
    float2 st[8], v[8];
#pragma unroll
    for (int y = 0; y < 8; ++y) {
      const size_t s = slot0 + (i0 + kStep * y < pieces ? i0 + kStep * y : 0) * step;
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
      const float w = i0 + kStep * y < pieces ? __builtin_amdgcn_exp2f(st[y].x - m) : 0.f;
      l = __builtin_fmaf(st[y].y, w, l);
      acc.x = __builtin_fmaf(v[y].x, w, acc.x);
      acc.y = __builtin_fmaf(v[y].y, w, acc.y);
    }
  }
  T* to = (T*)p.out + ((int64_t)(p.seq[b].q_start + token) * p.o_st + (int64_t)(h * p.group + head) * p.o_sh);
  float* lse = p.lse ? p.lse + ((int64_t)(p.seq[b].q_start + token) * p.hq + h * p.group + head) : nullptr;
  if constexpr (ONE) {
    typedef T T2 __attribute__((ext_vector_type(2)));
    const float inv = l == 0.f ? 0.f : 1.f / l;
    *(T2*)(to + 2 * lane) = (T2){(T)(acc.x * inv), (T)(acc.y * inv)};
    if (lse && lane == 0) *lse = l == 0.f ? -INFINITY : (m - kShift + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
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
  to[c] = (T)(total == 0.f ? 0.f : v / total);
  if (lse && c == 0) *lse = total == 0.f ? -INFINITY : (top - kShift + __builtin_amdgcn_logf(total)) * 0.69314718055994531f;
}

// What the plan goes by, in us: a workgroup's beginning and end and a tile of its keys (64; few rows: 32 for each wave, longer the more
// workgroups share the memory), and the joining launch with the partial results' way out and back.  Measured with one
// sequence, 32 query heads, 8 KV heads, whole / in pieces: 512 tokens 22 / 34, 1024 over 1024 35 / 51, 512 over 4096 107 / 55, 333 over 65869
// 1592 / 386, one over 500 8.5 / 8.8, one over 4000 29.9 / 9.3.  (With all units at work for long a tile takes about 2 us, as the clock falls:
// the constants are for calls short enough that the choice matters.)
constexpr double kFixed = 9.5, kTileTime = 1.55, kFewFixed = 5.3, kFewTile = 0.8, kFewLoad = 0.0092;
constexpr double kJoin = 3, kJoinRow = 3e-4, kJoinPart = 1.7e-4;

template <typename T>
int32_t launch_prompt(const PromptParams& p, bool few, int32_t items, hipStream_t s) {
  const dim3 grid((uint32_t)items * (uint32_t)p.hkv);
  if (few) {
    constexpr int lds = kFewWaves * 4 * kFewKeys * TKV_D * 2;
    static_assert(lds <= 160 * 1024 && kFewWaves * kFew * (TKV_D + 4 + 2) * 4 <= lds, "LDS of one compute unit");
    static const bool lds_ok = hipFuncSetAttribute(reinterpret_cast<const void*>(&prompt_few_kernel<T>),
                                                   hipFuncAttributeMaxDynamicSharedMemorySize, lds) == hipSuccess;
    if (!lds_ok) return TKV_E_HIP;
    TKV_LAUNCH(prompt_few_kernel<T>, grid, 64 * kFewWaves, lds, s, p);
  } else {
    TKV_LAUNCH(prompt_attn_kernel<T>, grid, 64 * kWaves, 0, s, p);
  }
  const uint32_t joins = (uint32_t)p.split_rows * (uint32_t)p.hkv;
  if (joins && p.most_pieces <= 16) TKV_LAUNCH((prompt_merge_kernel<T, true>), dim3((joins + 3) / 4), 256, 0, s, p);
  else if (joins) TKV_LAUNCH((prompt_merge_kernel<T, false>), dim3(joins), 256, 0, s, p);
  return TKV_OK;
}

int32_t check_prompt_desc(const tkv_prompt_desc* d) {
  if (!d || d->struct_size != sizeof(tkv_prompt_desc)) return TKV_E_INVAL;
  if (d->n_q_heads <= 0 || d->n_kv_heads <= 0 || d->head_dim <= 0 || d->batch <= 0) return TKV_E_INVAL;
  if (d->n_q_heads % d->n_kv_heads != 0) return TKV_E_INVAL;
  if (d->dtype != TKV_F16 && d->dtype != TKV_BF16) return TKV_E_INVAL;
  if ((d->causal != 0 && d->causal != 1) || d->reserved != 0) return TKV_E_INVAL;
  if (d->head_dim != TKV_D || d->batch > TKV_MAX_BATCH || d->n_q_heads > 1024) return TKV_E_UNSUPPORTED;
  return TKV_OK;
}

bool good_strides(const int64_t* s) {
  // (a tile's rows are addressed with 32 bits)
  return s[0] >= 0 && s[1] >= 0 && s[0] % 8 == 0 && s[1] % 8 == 0 && s[0] <= (1 << 22) && s[1] <= ((int64_t)1 << 40);
}

// Whether no two rows of 128 elements overlap, one at every t s[0] + h s[1].
bool rows_apart(const int64_t* s, int64_t tokens, int64_t heads) {
  if (tokens == 0) return true;
  if ((tokens > 1 && s[0] < TKV_D) || (heads > 1 && s[1] < TKV_D)) return false;
  // heads within a token, or tokens within a head: all but strides made by hand
  if (tokens == 1 || heads == 1 || s[0] >= (heads - 1) * s[1] + TKV_D || s[1] >= (tokens - 1) * s[0] + TKV_D) return true;
  for (int64_t h = 1; h < heads; ++h) {  // the two tokens whose rows lie next to those h heads on
    const int64_t t = h * s[1] / s[0], r = h * s[1] % s[0];
    if ((t < tokens && r < TKV_D) || (t + 1 < tokens && s[0] - r < TKV_D)) return false;
  }
  return true;
}

}  // namespace

extern "C" int32_t tkv_prompt_attn_sizes(const tkv_prompt_desc* d, size_t* workspace_bytes) {
  const int32_t st = check_prompt_desc(d);
  if (st != TKV_OK) return st;
  if (!workspace_bytes) return TKV_E_INVAL;
  *workspace_bytes = (size_t)kMaxParts * kPartFloats * sizeof(float);
  return TKV_OK;
}

extern "C" int32_t tkv_prompt_attn(const tkv_prompt_desc* d, const void* q, const void* k, const void* v, void* out, float* lse,
                                   const int32_t* q_start_host, const int32_t* q_len_host, const int32_t* k_start_host,
                                   const int32_t* k_len_host, float sm_scale, void* workspace, size_t workspace_bytes,
                                   void* stream) {
  const int32_t st = check_prompt_desc(d);
  if (st != TKV_OK) return st;
  if (!q_start_host || !q_len_host || !k_start_host || !k_len_host || !workspace) return TKV_E_INVAL;
  const float scale2 = sm_scale * 1.4426950408889634f;
  if (!(sm_scale > 0.f) || !(scale2 <= 3.402823466e38f)) return TKV_E_INVAL;
  if (!good_strides(d->q_stride) || !good_strides(d->k_stride) || !good_strides(d->v_stride) || !good_strides(d->o_stride)) return TKV_E_INVAL;
  PromptParams p;
  p.group = d->n_q_heads / d->n_kv_heads;
  int64_t tiles = 0, any_keys = 0, q_first = 0, q_last = 0;  // (rows of out: from q_first on, q_last not among them)
  for (int b = 0; b < d->batch; ++b) {
    if (q_start_host[b] < 0 || q_len_host[b] < 0 || k_start_host[b] < 0 || k_len_host[b] < 0) return TKV_E_INVAL;
    if ((int64_t)q_len_host[b] * p.group > (1 << 30) || k_len_host[b] > (1 << 30)) return TKV_E_UNSUPPORTED;
    if ((int64_t)q_start_host[b] + q_len_host[b] > 0x7FFFFFFF || (int64_t)k_start_host[b] + k_len_host[b] > 0x7FFFFFFF) return TKV_E_INVAL;
    tiles += ((int64_t)q_len_host[b] * p.group + kRows - 1) / kRows;
    any_keys |= k_len_host[b];
    if (q_len_host[b] == 0) continue;
    if (q_last == 0 || q_start_host[b] < q_first) q_first = q_start_host[b];
    q_last = std::max<int64_t>(q_last, q_start_host[b] + q_len_host[b]);
  }
  // No row of two sequences.  (In order, as nearly always, one look at each says so.)
  auto q_end = [&](int b) { return q_start_host[b] + q_len_host[b]; };
  bool in_order = true;
  for (int b = 0, end = 0; b < d->batch; ++b) {
    if (q_len_host[b] == 0) continue;
    in_order = in_order && q_start_host[b] >= end;
    end = q_end(b);
  }
  for (int b = 1; b < d->batch && !in_order; ++b)
    for (int a = 0; a < b; ++a)
      if (q_len_host[a] && q_len_host[b] && q_start_host[a] < q_end(b) && q_start_host[b] < q_end(a)) return TKV_E_INVAL;
  if (tiles * d->n_kv_heads >= 1 << 23) return TKV_E_UNSUPPORTED;  // (a launch has fewer than 2^32 threads)
  if (!rows_apart(d->o_stride, q_last - q_first, d->n_q_heads)) return TKV_E_INVAL;
  if (workspace_bytes < (size_t)kMaxParts * kPartFloats * sizeof(float)) return TKV_E_WORKSPACE;
  for (const void* x : {q, k, v, (const void*)out, (const void*)workspace})
    if (((uintptr_t)x & 15) != 0) return TKV_E_INVAL;
  if (((uintptr_t)lse & 3) != 0) return TKV_E_INVAL;
  if (tiles == 0) return TKV_OK;
  if (!q || !out || (any_keys && (!k || !v))) return TKV_E_INVAL;
  p.q = q; p.k = k; p.v = v; p.out = out; p.lse = lse;
  p.q_st = d->q_stride[0]; p.q_sh = d->q_stride[1];
  p.k_st = d->k_stride[0]; p.k_sh = d->k_stride[1];
  p.v_st = d->v_stride[0]; p.v_sh = d->v_stride[1];
  p.o_st = d->o_stride[0]; p.o_sh = d->o_stride[1];
  p.hq = d->n_q_heads; p.hkv = d->n_kv_heads; p.batch = d->batch; p.causal = d->causal;
  p.scale2 = scale2;

  bool few = true;
  for (int b = 0; b < d->batch; ++b) few = few && (int64_t)q_len_host[b] * p.group <= kFew;
  p.tile_rows = few ? kFew : kRows;
  const int keys = few ? kFewKeys * kFewWaves : kKeys;
  auto key_tiles = [&](int b) { return (k_len_host[b] + keys - 1) / keys; };
  auto row_tiles = [&](int b) { return (q_len_host[b] * p.group + p.tile_rows - 1) / p.tile_rows; };
  int64_t work = 0, whole = 0;
  int most_tiles = 0;
  for (int b = 0; b < d->batch; ++b) {
    work += (int64_t)row_tiles(b) * key_tiles(b) * d->n_kv_heads;
    whole += (int64_t)row_tiles(b) * d->n_kv_heads;
    if (row_tiles(b) && key_tiles(b) > most_tiles) most_tiles = key_tiles(b);
  }
  // A row tile whose keys are more than a compute unit's even share (a workgroup of either kernel takes most of its unit's registers
  // or LDS): keys are split into pieces of at most `per` tiles, by the size of least estimated time.  Fewer row tiles than units
  // stay one round of workgroups.  (One token of each of 33 sequences, 65536 keys and 32 times 100: 560 us whole, 55 in pieces; 41 prompts of
  // 40 x 64 and 200 tokens, the latter over 40000 keys: 980, 176.)
  auto pieces_of = [&](int b, double per) {
    const int n = key_tiles(b), pieces = (int)(n / per);
    return pieces * per < n ? pieces + 1 : pieces > 1 ? pieces : 1;
  };
  const auto s = (hipStream_t)stream;
  const int units = most_tiles > 1 ? std::min(kMaxParts, tkv::stream_compute_units(s)) : 1;
  const int64_t max_parts = kMaxParts * (kRows / p.tile_rows);
  double best = 1e18;
  const double share = work > units ? (double)work / units : 1;
  if (most_tiles > share) {
    double least = 0;
    bool split = true;
    for (double per = share; split; per *= 1.15) {  // (at last one piece each)
      int64_t workgroups = 0, joins = 0, join_parts = 0, parts = 0;
      int longest = 0;
      split = false;
      for (int b = 0; b < d->batch; ++b) {
        if (!row_tiles(b)) continue;
        const int n = pieces_of(b, per), most = (key_tiles(b) + n - 1) / n;
        workgroups += (int64_t)row_tiles(b) * n * d->n_kv_heads;
        if (most > longest) longest = most;
        if (n == 1) continue;
        split = true;
        parts += (int64_t)row_tiles(b) * n * d->n_kv_heads;
        joins += (int64_t)q_len_host[b] * d->n_q_heads;
        join_parts += (int64_t)q_len_host[b] * d->n_q_heads * n;
      }
      if (parts > max_parts || (whole <= units && workgroups > units)) continue;
      const double tiles_each = longest > share ? longest : share, rounds = (double)((workgroups + units - 1) / units);
      const double tile_time = few ? kFewTile + kFewLoad * (workgroups < units ? workgroups : units) : kTileTime;
      double time = (few ? kFewFixed : kFixed) * rounds + tile_time * tiles_each;
      if (split) time += kJoin + kJoinRow * joins + kJoinPart * join_parts;
      if (least == 0 || time < least) least = time, best = per;
    }
  }
  int32_t items = 0, parts = 0;
  p.split_rows = p.most_pieces = 0;
  for (int b = 0; b < d->batch; ++b) {
    p.seq[b] = {q_start_host[b], q_len_host[b], k_start_host[b], k_len_host[b]};
    p.pieces[b] = pieces_of(b, best);
    p.first_item[b] = items;
    p.first_part[b] = -1;
    p.first_row[b] = p.split_rows;
    items += row_tiles(b) * p.pieces[b];
    if (p.pieces[b] > 1 && row_tiles(b) > 0) {
      p.first_part[b] = parts;
      parts += row_tiles(b) * p.pieces[b] * d->n_kv_heads;
      p.split_rows += q_len_host[b] * p.group;
      if (p.pieces[b] > p.most_pieces) p.most_pieces = p.pieces[b];
    }
  }
  p.parts = (float*)workspace;
  p.ml = p.parts + (size_t)kMaxParts * kRows * TKV_D;
  return d->dtype == TKV_F16 ? launch_prompt<_Float16>(p, few, items, s) : launch_prompt<__bf16>(p, few, items, s);
}
