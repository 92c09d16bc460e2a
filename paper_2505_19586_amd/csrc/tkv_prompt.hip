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
// sum in float32, weights rounded to the inputs' type for the second product (a relative error of 2^-12 or 2^-9 each, random,
// beside the output's own rounding of as much).
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
constexpr int kRows = 128;      // rows of a workgroup: four waves of 32
constexpr int kMaxParts = 1024; // partial results that the workspace has room for
constexpr int kPartFloats = kRows * (TKV_D + 2);
// Weights are 2^(logit - reference + kShift): the reference follows the running maximum only when that
// is kLazy above it, so the largest weight is 2^(kLazy + kShift) = 2^15, inside fp16's range, and fp16's subnormal numbers begin 2^-21 below
// the reference's weight, not 2^-14.
constexpr float kLazy = 8.f, kShift = 7.f;
constexpr float kNone = -1e30f;  // reference of a row without a key so far

struct PromptSeq {
  int32_t q_start, q_len, k_start, k_len;
};

struct PromptParams {
  const void* q;
  const void* k;
  const void* v;
  void* out;
  float* lse;    // NULL: not wanted
  float* parts;  // [part][kRows][128] weighted sums, then [part][kRows][2] (reference, sum)
  int64_t q_st, q_sh, k_st, k_sh, v_st, v_sh, o_st, o_sh;
  int32_t hq, hkv, group, batch, causal;
  float scale2;  // sm_scale * log2(e)
  PromptSeq seq[TKV_MAX_BATCH];
  int32_t first_item[TKV_MAX_BATCH];  // in (row tile, piece) pairs
  int32_t first_part[TKV_MAX_BATCH];  // -1: the sequence's rows are not split
  int32_t pieces[TKV_MAX_BATCH];
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

__device__ inline uintx4 lds_read16(uint32_t at) {
  return *(__attribute__((address_space(3))) uintx4*)(lds_char*)(uintptr_t)at;
}
// 4 x 16 elements transposed over sixteen lanes: lane 4 r + c of the sixteen names row r's columns 4 c to 4 c + 3,
// lane c receives column c of the four rows.
__device__ inline uintx2 lds_read_tr(uint32_t at) {
  return __builtin_bit_cast(uintx2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4*)(lds_char*)(uintptr_t)at));
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

template <typename T>
__global__ __launch_bounds__(256, 2) void prompt_attn_kernel(PromptParams p) {
  __shared__ __attribute__((aligned(1024))) char lds[2 * 2 * kKeys * TKV_D * 2];  // two buffers of a K and a V tile
  constexpr int kTile = kKeys * TKV_D * 2;
  const int lane = threadIdx.x % 64, half = lane / 32, col = lane % 32;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
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

  uintx4 qf[8];
  {
    const T* q = (const T*)p.q + ((int64_t)(sq.q_start + token) * p.q_st + (int64_t)(h * p.group + head) * p.q_sh + 8 * half);
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) qf[kk] = *(const uintx4*)(q + 16 * kk);
  }

  // staging: an instruction of a wave brings four rows; LDS keeps a row's sixteen 16-byte places in an order that depends on the
  // row, so that the reads below (a column of keys, a block of four keys) meet all banks
  uint32_t k_off[4], v_off[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int r = 16 * wave + 4 * j + lane / 16, place = lane % 16;
    k_off[j] = (uint32_t)(r * p.k_st * 2) + 16u * (uint32_t)(place ^ (r & 15));
    v_off[j] = (uint32_t)(r * p.v_st * 2) + 16u * (uint32_t)(place ^ (((r & 3) << 2) | ((r >> 2) & 3)));
  }
  const char* k_base = (const char*)p.k + ((int64_t)sq.k_start * p.k_st + (int64_t)h * p.k_sh) * 2;
  const char* v_base = (const char*)p.v + ((int64_t)sq.k_start * p.v_st + (int64_t)h * p.v_sh) * 2;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)lds;
  auto stage = [&](int t, int buf) {
    const int left = min(kKeys, sq.k_len - t * kKeys);  // rows behind the sequence's last read as zeros
    const auto kr = __builtin_amdgcn_make_buffer_rsrc((void*)(k_base + (int64_t)t * kKeys * p.k_st * 2), 0, (int)((left - 1) * p.k_st * 2 + TKV_D * 2), 0x00020000);
    const auto vr = __builtin_amdgcn_make_buffer_rsrc((void*)(v_base + (int64_t)t * kKeys * p.v_st * 2), 0, (int)((left - 1) * p.v_st * 2 + TKV_D * 2), 0x00020000);
    const uint32_t to = lds0 + (uint32_t)(buf * 2 * kTile + wave * 4096);
#pragma unroll
    for (int j = 0; j < 4; ++j) to_lds(kr, to + 1024 * j, k_off[j]);
#pragma unroll
    for (int j = 0; j < 4; ++j) to_lds(vr, to + kTile + 1024 * j, v_off[j]);
  };

  // LDS addresses of the operands, without buffer, key step and tile
  uint32_t ka[8], va[8];
#pragma unroll
  for (int kk = 0; kk < 8; ++kk) ka[kk] = lds0 + (uint32_t)(col * 256 + 16 * ((2 * kk + half) ^ (col & 15)));
  {
    const int l16 = lane % 16, right = (lane / 16) % 2;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int key = 8 * s + 4 * half + l16 / 4;
        const int place = (4 * dt + 2 * right + (l16 % 4) / 2) ^ (((key & 3) << 2) | ((key >> 2) & 3));
        va[2 * dt + s] = lds0 + (uint32_t)(kTile + key * 256 + 16 * place + 8 * (l16 % 2));
      }
  }

  floatx16 o[4];
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
  float ref = kNone, sum = 0.f;

  // (The query rows are waited for here: the compiler, which does not know of the loads to LDS, would wait for them and those
  // inside the loop.)
#pragma unroll
  for (int kk = 0; kk < 8; ++kk) asm volatile("" : "+v"(qf[kk]));
  if (t0 < t1) stage(t0, 0);
  for (int t = t0; t < t1; ++t) {
    const int buf = (t - t0) & 1;
    asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");  // the tile is there, everyone is done with the other buffer
    if (t + 1 < t1) stage(t + 1, buf ^ 1);
    const int key0 = t * kKeys;
    if (!wave_on || key0 > limit_high) continue;
    const uint32_t at = (uint32_t)(buf * 2 * kTile);
    floatx16 s[2];
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[y][i] = 0.f;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk)
#pragma unroll
      for (int y = 0; y < 2; ++y) s[y] = mfma32<T>(lds_read16(ka[kk] + at + 8192 * y), qf[kk], s[y]);
    if (key0 + kKeys - 1 > limit_low || key0 + kKeys > sq.k_len) {
#pragma unroll
      for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          s[y][i] = key0 + 32 * y + 8 * (i / 4) + 4 * half + i % 4 <= limit ? s[y][i] : -INFINITY;
    }
    float top = fmaxf(s[0][0], s[1][0]);
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, fmaxf(s[0][i], s[1][i]));
    top = fmaxf(top, other_half(top, half)) * p.scale2;
    if (__builtin_amdgcn_ballot_w64(top > ref + kLazy) != 0) {
      const float next = fmaxf(ref, top), shrink = __builtin_amdgcn_exp2f(ref - next);
      ref = next;
      sum *= shrink;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) o[dt] *= shrink;
    }
    const float less = kShift - ref;
    uintx4 pf[4];
#pragma unroll
    for (int y = 0; y < 2; ++y) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[y][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[y][i], p.scale2, less));
        sum += s[y][i];
      }
      pf[2 * y] = pack8<T>(__builtin_shufflevector(s[y], s[y], 0, 1, 2, 3, 4, 5, 6, 7));
      pf[2 * y + 1] = pack8<T>(__builtin_shufflevector(s[y], s[y], 8, 9, 10, 11, 12, 13, 14, 15));
    }
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) {
        const uintx2 lo = lds_read_tr(va[2 * dt] + at + 4096 * ks), hi = lds_read_tr(va[2 * dt + 1] + at + 4096 * ks);
        const uintx4 vf = __builtin_shufflevector(lo, hi, 0, 1, 2, 3);
        o[dt] = mfma32<T>(vf, pf[ks], o[dt]);
      }
  }

  sum += other_half(sum, half);
  if (!wave_on || row >= rows) return;
  if (p.first_part[it.b] >= 0) {
    const size_t part = (size_t)p.first_part[it.b] + ((size_t)it.tile * pieces + it.piece) * p.hkv + h;
    const int r = 32 * wave + col;
    float* ml = p.parts + (size_t)kMaxParts * kRows * TKV_D + (part * kRows + r) * 2;
    if (half == 0) *(float2*)ml = make_float2(ref, sum);
    if (sum == 0.f) return;  // (its weighted sum is not read)
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

// Joins the pieces of the split rows: a wave per row, blockIdx.y the row tile's quads of rows.
template <typename T>
__global__ __launch_bounds__(256) void prompt_merge_kernel(PromptParams p) {
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int h = blockIdx.x % p.hkv;
  // (the grid runs over tiles: the items of pieces 0)
  int tile = blockIdx.x / p.hkv, b = 0;
  for (; b < p.batch; ++b) {
    if (p.first_part[b] < 0) continue;
    const int tiles = (p.seq[b].q_len * p.group + kRows - 1) / kRows;
    if (tile < tiles) break;
    tile -= tiles;
  }
  if (b >= p.batch) return;
  const int r = 4 * blockIdx.y + wave, row = tile * kRows + r;
  if (row >= p.seq[b].q_len * p.group) return;
  const int token = row / p.group, head = row - token * p.group, pieces = p.pieces[b];
  const size_t part0 = (size_t)p.first_part[b] + (size_t)tile * pieces * p.hkv + h;
  const float* ml = p.parts + (size_t)kMaxParts * kRows * TKV_D;
  float m = kNone, l = 0.f;
  if (lane < pieces) {
    const float2 x = *(const float2*)(ml + ((part0 + (size_t)lane * p.hkv) * kRows + r) * 2);
    m = x.x, l = x.y;
  }
  const float top = tkv::over_wave(m, tkv::MaxOf{});
  const float w = __builtin_amdgcn_exp2f(m - top);
  const float total = tkv::over_wave(l * w, tkv::SumOf{});
  float2 acc = make_float2(0.f, 0.f);
  for (int i = 0; i < pieces; ++i) {
    const float li = __shfl(l, i, 64), wi = __shfl(w, i, 64);
    if (li == 0.f) continue;
    const float2 x = *(const float2*)(p.parts + ((part0 + (size_t)i * p.hkv) * kRows + r) * TKV_D + 2 * lane);
    acc.x = __builtin_fmaf(x.x, wi, acc.x);
    acc.y = __builtin_fmaf(x.y, wi, acc.y);
  }
  const float inv = total == 0.f ? 0.f : 1.f / total;
  T* to = (T*)p.out + ((int64_t)(p.seq[b].q_start + token) * p.o_st + (int64_t)(h * p.group + head) * p.o_sh);
  typedef T T2 __attribute__((ext_vector_type(2)));
  typedef float floatx2 __attribute__((ext_vector_type(2)));
  *(T2*)(to + 2 * lane) = __builtin_convertvector((floatx2){acc.x * inv, acc.y * inv}, T2);
  if (p.lse && lane == 0)
    p.lse[(int64_t)(p.seq[b].q_start + token) * p.hq + h * p.group + head] =
        total == 0.f ? -INFINITY : (top - kShift + __builtin_amdgcn_logf(total)) * 0.69314718055994531f;
}

int32_t check_prompt_desc(const tkv_prompt_desc* d) {
  if (!d || d->struct_size != sizeof(tkv_prompt_desc)) return TKV_E_INVAL;
  if (d->n_q_heads <= 0 || d->n_kv_heads <= 0 || d->head_dim <= 0 || d->batch <= 0) return TKV_E_INVAL;
  if (d->n_q_heads % d->n_kv_heads != 0) return TKV_E_INVAL;
  if (d->dtype != TKV_F16 && d->dtype != TKV_BF16) return TKV_E_INVAL;
  if (d->causal != 0 && d->causal != 1) return TKV_E_INVAL;
  if (d->head_dim != TKV_D || d->batch > TKV_MAX_BATCH || d->n_q_heads > 1024) return TKV_E_UNSUPPORTED;
  return TKV_OK;
}

bool good_strides(const int64_t* s) {
  // (a tile's rows are addressed with 32 bits)
  return s[0] >= 0 && s[1] >= 0 && s[0] % 8 == 0 && s[1] % 8 == 0 && s[0] <= (1 << 22) && s[1] <= ((int64_t)1 << 40);
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
  if (!(sm_scale > 0.f) || !(sm_scale <= 3.402823466e38f)) return TKV_E_INVAL;
  if (!good_strides(d->q_stride) || !good_strides(d->k_stride) || !good_strides(d->v_stride) || !good_strides(d->o_stride)) return TKV_E_INVAL;
  if (workspace_bytes < (size_t)kMaxParts * kPartFloats * sizeof(float)) return TKV_E_WORKSPACE;
  for (const void* x : {q, k, v, (const void*)out, (const void*)workspace})
    if (((uintptr_t)x & 15) != 0) return TKV_E_INVAL;
  if (((uintptr_t)lse & 3) != 0) return TKV_E_INVAL;
  PromptParams p;
  p.group = d->n_q_heads / d->n_kv_heads;
  int64_t tiles = 0, any_keys = 0;
  for (int b = 0; b < d->batch; ++b) {
    if (q_start_host[b] < 0 || q_len_host[b] < 0 || k_start_host[b] < 0 || k_len_host[b] < 0) return TKV_E_INVAL;
    if ((int64_t)q_len_host[b] * p.group > (1 << 30) || k_len_host[b] > (1 << 30)) return TKV_E_UNSUPPORTED;
    if ((int64_t)q_start_host[b] + q_len_host[b] > 0x7FFFFFFF || (int64_t)k_start_host[b] + k_len_host[b] > 0x7FFFFFFF) return TKV_E_INVAL;
    tiles += ((int64_t)q_len_host[b] * p.group + kRows - 1) / kRows;
    any_keys |= k_len_host[b];
  }
  if (tiles == 0) return TKV_OK;
  if (!q || !out || (any_keys && (!k || !v))) return TKV_E_INVAL;
  if (tiles * 64 * d->n_kv_heads > 0x7FFFFFFF) return TKV_E_UNSUPPORTED;
  p.q = q; p.k = k; p.v = v; p.out = out; p.lse = lse; p.parts = (float*)workspace;
  p.q_st = d->q_stride[0]; p.q_sh = d->q_stride[1];
  p.k_st = d->k_stride[0]; p.k_sh = d->k_stride[1];
  p.v_st = d->v_stride[0]; p.v_sh = d->v_stride[1];
  p.o_st = d->o_stride[0]; p.o_sh = d->o_stride[1];
  p.hq = d->n_q_heads; p.hkv = d->n_kv_heads; p.batch = d->batch; p.causal = d->causal;
  p.scale2 = sm_scale * 1.4426950408889634f;

  // Few row tiles: their keys are split into pieces so that about two workgroups per compute unit have work.
  auto key_tiles = [&](int b) { return (k_len_host[b] + kKeys - 1) / kKeys; };
  auto row_tiles = [&](int b) { return (q_len_host[b] * p.group + kRows - 1) / kRows; };
  int64_t per_piece = 0;
  if (tiles * d->n_kv_heads < 384) {
    int64_t work = 0;
    for (int b = 0; b < d->batch; ++b) work += (int64_t)row_tiles(b) * key_tiles(b) * d->n_kv_heads;
    per_piece = work / 512 < 4 ? 4 : work / 512;
  }
  int32_t items = 0, parts = 0, split_tiles = 0;
  for (;; per_piece *= 2) {
    items = parts = split_tiles = 0;
    for (int b = 0; b < d->batch; ++b) {
      p.seq[b] = {q_start_host[b], q_len_host[b], k_start_host[b], k_len_host[b]};
      int64_t pieces = per_piece ? (key_tiles(b) + per_piece - 1) / per_piece : 1;
      pieces = pieces < 1 ? 1 : pieces > 64 ? 64 : pieces;
      p.pieces[b] = (int32_t)pieces;
      p.first_item[b] = items;
      p.first_part[b] = -1;
      items += row_tiles(b) * p.pieces[b];
      if (pieces > 1 && row_tiles(b) > 0) {
        p.first_part[b] = parts;
        parts += row_tiles(b) * p.pieces[b] * d->n_kv_heads;
        split_tiles += row_tiles(b);
      }
    }
    if (parts <= kMaxParts) break;
  }
  const auto s = (hipStream_t)stream;
  const dim3 grid((uint32_t)items * (uint32_t)d->n_kv_heads), merge((uint32_t)split_tiles * (uint32_t)d->n_kv_heads, kRows / 4);
  if (d->dtype == TKV_F16) {
    TKV_LAUNCH(prompt_attn_kernel<_Float16>, grid, 256, 0, s, p);
    if (split_tiles) TKV_LAUNCH(prompt_merge_kernel<_Float16>, merge, 256, 0, s, p);
  } else {
    TKV_LAUNCH(prompt_attn_kernel<__bf16>, grid, 256, 0, s, p);
    if (split_tiles) TKV_LAUNCH(prompt_merge_kernel<__bf16>, merge, 256, 0, s, p);
  }
  return TKV_OK;
}
