// Paged caches: rows read back from their pages (tkv_paged_gather) and attention over them (tkv_paged_attn).
#include <algorithm>

#include "tkv_paged.h"

namespace {

typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx8 __attribute__((ext_vector_type(8)));
typedef uint32_t uintx2 __attribute__((ext_vector_type(2)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 bhalf8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char lds_char;


struct GatherParams {
  tkv::Pages pages;
  const int32_t* slots;
  void* k_out;
  void* v_out;
  int32_t n_tokens;
  int32_t waves;
};

// Rows from pages, contiguous.  A wave takes sixteen tokens of one head's keys or values, sixteen lanes a row: neighbours in a page
// are read side by side (64 bytes a row in 4 bits), and rows are written whole.  Bound by the memory's rate.
template <typename T, int BITS>
__global__ __launch_bounds__(256) void paged_gather_kernel(GatherParams p) {
  const int lane = threadIdx.x % 64, sub = lane / 16, place = lane % 16;
  const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + threadIdx.x / 64);
  if (wave >= p.waves) return;
  const int heads = 2 * p.pages.hkv, tile = wave / heads, hv = wave - tile * heads;
  const bool is_v = hv >= p.pages.hkv;
  const int h = is_v ? hv - p.pages.hkv : hv;
  const int64_t sp = is_v ? p.pages.v_sp : p.pages.k_sp, st = is_v ? p.pages.v_st : p.pages.k_st;
  const char* const base = (const char*)(is_v ? p.pages.v : p.pages.k) + (int64_t)h * (is_v ? p.pages.v_sh : p.pages.k_sh) * (BITS == 16 ? 2 : 1);
  T* const out = (T*)(is_v ? p.v_out : p.k_out);
  int32_t slot[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int t = 16 * tile + 4 * j + sub;
    slot[j] = t < p.n_tokens ? p.slots[t] : -1;
    if (slot[j] >> p.pages.shift >= p.pages.n_pages) slot[j] = -1;
  }
  uintx4 x[4];
  uint32_t codes[4], scale[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t page = slot[j] >> p.pages.shift, at = slot[j] & ((1 << p.pages.shift) - 1);
    x[j] = (uintx4){0u, 0u, 0u, 0u};
    codes[j] = scale[j] = 0u;
    if (slot[j] < 0) continue;
    if constexpr (BITS == 16) {
      x[j] = *(const uintx4*)(base + (page * sp + at * st) * 2 + 16 * place);
    } else {
      const char* const block = base + page * sp;
      codes[j] = *(const uint32_t*)(block + at * tkv::kRow4 + 4 * place);
      scale[j] = *(const uint8_t*)(block + ((int64_t)tkv::kRow4 << p.pages.shift) + at * tkv::kScales4 + place / 4);
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int t = 16 * tile + 4 * j + sub;
    if (t >= p.n_tokens) continue;
    if constexpr (BITS == 4) x[j] = __builtin_bit_cast(uintx4, tkv::values_of<T>(codes[j], tkv::scale_of(scale[j])));
    *(uintx4*)(out + ((int64_t)t * p.pages.hkv + h) * TKV_D + 8 * place) = x[j];
  }
}

constexpr int kWaves = 4;        // of a workgroup
constexpr int kRowFloats = TKV_D + 4;  // of a row of partial sums in LDS (the four keep the banks apart)
// Weights are 2^(logit - reference + kShift), and the reference follows a row's maximum only when that is 8 above it: at most 2^15, inside
// fp16's range.
constexpr float kShift = 7.f;
constexpr float kNone = -3.402823466e38f;  // reference of a row without a key so far (finite: kNone - kNone is 0)

struct PagedParams {
  tkv::Pages pages;
  const void* q;
  void* out;
  float* lse;  // NULL: not wanted
  const int32_t* table;
  const int32_t* k_lens;
  const int32_t* q_starts;  // NULL: a token of each sequence
  float* parts;             // [2 per workgroup][rows of a tile][128] weighted sums
  float* ml;                // [2 per workgroup][rows of a tile][2] (reference, sum)
  int32_t n_tokens, batch, hq, group, pages_each;
  int32_t workgroups;
  float scale2;  // sm_scale * log2(e)
};

// How the work is shared out.  Every (sequence, KV head, tile of rows) is an item, its keys so many tiles of TK; all items' tiles in
// a row are cut into as many equal ranges as there are workgroups.  Lengths lie on the device, so every workgroup works that out for
// itself: 64 sequences at a time, one a lane.
struct Sequence {
  int32_t index, k_len, q_start, q_len, key_tiles, row_tiles;
  uint32_t first;  // of its tiles, among all
};

template <int TK, int ROWS>
struct Walk {
  const PagedParams& p;
  int32_t chunk;       // first sequence of those at hand
  int32_t k_len, q_start, q_len;  // per lane
  uint32_t first, count;          // per lane: tiles before its sequence, and of it
  uint32_t all;                   // tiles up to the chunk's end

  __device__ explicit Walk(const PagedParams& params) : p(params), chunk(0) { load(0, 0); }

  __device__ int32_t key_tiles(int32_t n) const { return max(1, (n + TK - 1) / TK); }
  __device__ int32_t row_tiles(int32_t n) const { return (n * p.group + ROWS - 1) / ROWS; }

  __device__ void load(int32_t at, uint32_t before) {
    const int lane = threadIdx.x % 64, b = min(at + lane, p.batch - 1);
    chunk = at;
    k_len = (int32_t)max((int64_t)0, min((int64_t)p.k_lens[b], (int64_t)p.pages_each << p.pages.shift));
    q_start = b;
    q_len = 1;
    if (p.q_starts) {
      q_start = min(max(p.q_starts[b], 0), p.n_tokens);
      q_len = max(0, min(p.q_starts[b + 1], p.n_tokens) - q_start);
    }
    count = at + lane < p.batch ? (uint32_t)(key_tiles(k_len) * row_tiles(q_len)) * (uint32_t)p.pages.hkv : 0u;
    uint32_t sum = count;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const uint32_t x = __shfl_up(sum, d, 64);
      if (lane >= d) sum += x;
    }
    first = before + sum - count;
    all = before + (uint32_t)__builtin_amdgcn_readlane((int)sum, 63);
  }
  __device__ uint32_t total() {
    while (chunk + 64 < p.batch) load(chunk + 64, all);
    const uint32_t t = all;
    if (chunk != 0) load(0, 0);
    return t;
  }
  // The sequence of tile number `at` (below total(), not before the chunk at hand); index -1 where there is none.
  __device__ Sequence find(uint32_t at) {
    while (at >= all && chunk + 64 < p.batch) load(chunk + 64, all);
    // the last of those that begin at or before it (one without tiles shares its successor's beginning)
    const int lane = threadIdx.x % 64;
    const uint64_t before = __builtin_amdgcn_ballot_w64(count != 0u && first <= at && at < first + count);
    Sequence s;
    s.index = -1;
    if (before == 0) return s;
    const int l = 63 - __builtin_clzll(before);
    (void)lane;
    s.index = chunk + l;
    s.k_len = __builtin_amdgcn_readlane(k_len, l);
    s.q_start = __builtin_amdgcn_readlane(q_start, l);
    s.q_len = __builtin_amdgcn_readlane(q_len, l);
    s.first = (uint32_t)__builtin_amdgcn_readlane((int)first, l);
    s.key_tiles = key_tiles(s.k_len);
    s.row_tiles = row_tiles(s.q_len);
    return s;
  }
};

// Tiles of a workgroup's range: as even as can be, and one for each wave at least.
__device__ inline uint32_t range_of(uint32_t total, int workgroups) {
  return max((uint32_t)kWaves, (total + (uint32_t)workgroups - 1) / (uint32_t)workgroups);
}

template <typename T>
__device__ inline floatx4 mfma16(uintx4 a, uintx4 b, floatx4 c) {
  if constexpr (__is_same(T, _Float16))
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bhalf8, a), __builtin_bit_cast(bhalf8, b), c, 0, 0, 0);
}

template <typename T>
__device__ inline uintx4 pack8(floatx8 x) {
  typedef T T8 __attribute__((ext_vector_type(8)));
  return __builtin_bit_cast(uintx4, __builtin_convertvector(x, T8));
}

__device__ inline uintx4 lds_read16(lds_char* at) { return *(__attribute__((address_space(3))) uintx4*)at; }
__device__ inline void lds_write16(lds_char* at, uintx4 x) { *(__attribute__((address_space(3))) uintx4*)at = x; }
// 4 x 16 elements transposed over sixteen lanes: lane 4 r + c of the sixteen names row r's columns 4 c to 4 c + 3,
// lane c receives column c of the four rows.
__device__ inline uintx2 lds_read_tr(lds_char* at) {
  return __builtin_bit_cast(uintx2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4*)at));
}
// 16 bytes per lane from a descriptor's array straight to LDS, in lane order from `to` (uniform) on.  By hand, because the compiler
// lets every transposing LDS read wait for all such loads, those of the next tile too; nothing lands in registers, and the caller
// waits itself (vmcnt) before anyone reads the buffer.  (m0 is used by nothing else here.)
__device__ inline void to_lds(__amdgpu_buffer_rsrc_t from, uint32_t to, uint32_t lane_offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(lane_offset), "s"(from) : "memory");
}

// What a wave carries over a segment (some of an item's tiles): weighted sums, transposed (lane: row lane % 16 of each sixteen, channels
// 16 ct + 4 (lane / 16) + i), reference and its share of the sum of weights.
template <int NT>
struct Rows {
  floatx4 o[NT][8];
  float ref[NT], sum[NT];
  int32_t limit[NT];  // last key that the lane's row sees
  int32_t limit_low;  // ... and the item's first row
};

// Weights of 16 Y keys from key0 on, from their logits s (lane: row, keys key0 + 16 y + 4 (lane / 16) + i) for the next product:
// element 4 (y % 2) + i of operand y / 2.
template <typename T, int NT, int Y>
__device__ inline void weigh(Rows<NT>& r, floatx4 (&s)[NT][Y], uintx4 (&w)[NT][Y / 2], int key0, float scale2, int quarter) {
  const bool mask = key0 + 16 * Y - 1 > r.limit_low;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    if (mask) {
#pragma unroll
      for (int y = 0; y < Y; ++y)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[n][y][i] = key0 + 16 * y + 4 * quarter + i <= r.limit[n] ? s[n][y][i] : -INFINITY;
    }
    float top = s[n][0][0];
#pragma unroll
    for (int y = 0; y < Y; ++y)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, s[n][y][i]);
    top *= scale2;
    if (__builtin_amdgcn_ballot_w64(top > r.ref[n] + 8.f) != 0) {
      top = tkv::over_rows(top, [](float a, float b) { return fmaxf(a, b); });
      const float next = fmaxf(r.ref[n], top), shrink = __builtin_amdgcn_exp2f(r.ref[n] - next);
      r.ref[n] = next;
      r.sum[n] *= shrink;
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) r.o[n][ct] *= shrink;
    }
    const float less = kShift - r.ref[n];
#pragma unroll
    for (int y = 0; y < Y; ++y)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[n][y][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][y][i], scale2, less));
        r.sum[n] += s[n][y][i];
      }
#pragma unroll
    for (int y = 0; y < Y / 2; ++y) w[n][y] = pack8<T>(__builtin_shufflevector(s[n][2 * y], s[n][2 * y + 1], 0, 1, 2, 3, 4, 5, 6, 7));
  }
}

// The pages of a wave's next 64 sixteens of keys, one a lane: those of its tiles t0, t0 + kWaves, ... of PER sixteens each.
template <int PER>
__device__ inline int32_t some_pages(const PagedParams& p, const Sequence& sq, int t0) {
  const int lane = threadIdx.x % 64;
  const int64_t key = 16 * ((int64_t)(t0 + kWaves * (lane / PER)) * PER + lane % PER);
  const int64_t at = key >> p.pages.shift;
  const int32_t id = key < sq.k_len ? p.table[(int64_t)sq.index * p.pages_each + at] : -1;
  return id < p.pages.n_pages ? id : -1;
}

// A place of 16 bytes in a row of LDS: rows of 256 bytes keep their sixteen places in an order that depends on the row, so that the reads
// (a column of keys; a 4 x 16 block of values) and writes meet all banks.
__device__ inline int k_place(int row, int place) { return place ^ (row & 15); }
__device__ inline int v_place(int row, int place) { return place ^ (((row & 7) << 1) | ((row >> 3) & 1)); }

// 16 bits: the bytes bound this.  Every wave takes tiles of 32 keys of its own through a ring of two in LDS, filled by loads that
// do not pass through registers; no barrier until the waves join.
template <typename T, int NT>
__device__ inline void segment16(const PagedParams& p, const Sequence& sq, int h, int t0, int t1, const uintx4 (&qf)[NT][4], Rows<NT>& r,
                                 lds_char* ring) {
  constexpr int kTile = 32 * TKV_D * 2;
  const int lane = threadIdx.x % 64, col = lane % 16, quarter = lane / 16;
  if (t0 >= t1) return;
  uint32_t k_off[4], v_off[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int row = 4 * j + quarter;
    k_off[j] = (uint32_t)(row * p.pages.k_st * 2) + 16u * (uint32_t)k_place(row, col);
    v_off[j] = (uint32_t)(row * p.pages.v_st * 2) + 16u * (uint32_t)v_place(row, col);
  }
  const char* const k_head = (const char*)p.pages.k + (int64_t)h * p.pages.k_sh * 2;
  const char* const v_head = (const char*)p.pages.v + (int64_t)h * p.pages.v_sh * 2;
  const uint32_t ring0 = (uint32_t)(uintptr_t)ring;
  int32_t pages = some_pages<2>(p, sq, t0);
  int last = 0;  // the tile that `pages` begins with, in the wave's own count
  const int mine = (t1 - t0 + kWaves - 1) / kWaves;
  auto stage = [&](int n) {
    const int t = t0 + kWaves * n;
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int key = 32 * t + 16 * y, at = key & ((1 << p.pages.shift) - 1);
      const int32_t id = __builtin_amdgcn_readlane(pages, 2 * (n - last) + y);
      const int valid = id < 0 ? 0 : min(16, sq.k_len - key);  // rows behind the sequence's last, and pages outside, read as zeros
      const int64_t page = max(id, 0);
      const char* const kb = k_head + (page * p.pages.k_sp + at * p.pages.k_st) * 2;
      const char* const vb = v_head + (page * p.pages.v_sp + at * p.pages.v_st) * 2;
      const auto kr = __builtin_amdgcn_make_buffer_rsrc((void*)kb, 0, valid <= 0 ? 0 : (int)((valid - 1) * p.pages.k_st * 2 + TKV_D * 2), 0x00020000);
      const auto vr = __builtin_amdgcn_make_buffer_rsrc((void*)vb, 0, valid <= 0 ? 0 : (int)((valid - 1) * p.pages.v_st * 2 + TKV_D * 2), 0x00020000);
      const uint32_t to = ring0 + (uint32_t)((n & 1) * 2 * kTile + 4096 * y);
#pragma unroll
      for (int j = 0; j < 4; ++j) to_lds(kr, to + 1024 * j, k_off[j]);
#pragma unroll
      for (int j = 0; j < 4; ++j) to_lds(vr, to + kTile + 1024 * j, v_off[j]);
    }
  };
  lds_char* ka[4];
  lds_char* va[8];
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) ka[kk] = ring + (col * 256 + 16 * k_place(col, 4 * kk + quarter));
  {
    const int row = 4 * quarter + col / 4;
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) va[ct] = ring + (kTile + row * 256 + 16 * v_place(row, 2 * ct + (col % 4) / 2) + 8 * (col % 2));
  }
  stage(0);
  for (int n = 0; n < mine; ++n) {
    const int at = (n & 1) * 2 * kTile, key0 = 32 * (t0 + kWaves * n);
    if (n + 1 - last == 32) {
      last = n + 1;
      pages = some_pages<2>(p, sq, t0 + kWaves * last);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the other buffer's reads are done)
    if (n + 1 < mine) {
      stage(n + 1);
      asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
    } else {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    floatx4 s[NT][2];
#pragma unroll
    for (int m = 0; m < NT; ++m)
#pragma unroll
      for (int y = 0; y < 2; ++y) s[m][y] = (floatx4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const uintx4 a = lds_read16(ka[kk] + at + 4096 * y);
#pragma unroll
        for (int m = 0; m < NT; ++m) s[m][y] = mfma16<T>(a, qf[m][kk], s[m][y]);
      }
    uintx4 w[NT][1];
    weigh<T, NT, 2>(r, s, w, key0, p.scale2, quarter);
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) {
      const uintx2 lo = lds_read_tr(va[ct] + at), hi = lds_read_tr(va[ct] + at + 4096);
      const uintx4 a = __builtin_shufflevector(lo, hi, 0, 1, 2, 3);
#pragma unroll
      for (int m = 0; m < NT; ++m) r.o[m][ct] = mfma16<T>(a, w[m][0], r.o[m][ct]);
    }
  }
}

// 4 bits: tiles of 64 keys; codes go to registers (a lane has 32 channels of a key: one block, and eight channels for each of four
// products, which do not mind the order of the channels), keys from there to the matrix cores, values, as numbers of the type, through LDS,
// whose reads transpose them.
template <typename T, int NT>
__device__ inline void segment4(const PagedParams& p, const Sequence& sq, int h, int t0, int t1, const uintx4 (&qf)[NT][4], Rows<NT>& r,
                                lds_char* area) {
  const int lane = threadIdx.x % 64, col = lane % 16, quarter = lane / 16;
  if (t0 >= t1) return;
  const int64_t block = (int64_t)(tkv::kRow4 + tkv::kScales4) << p.pages.shift;
  const int scales = tkv::kRow4 << p.pages.shift;
  int32_t pages = some_pages<4>(p, sq, t0);
  int last = 0;
  const int mine = (t1 - t0 + kWaves - 1) / kWaves;
  struct Tile {
    uintx4 k[4], v[4];
    uint32_t ks[4], vs[4];
  };
  auto fetch = [&](int n, Tile& x) {
    const int t = t0 + kWaves * n;
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const int key = 64 * t + 16 * y, at = key & ((1 << p.pages.shift) - 1);
      const int32_t id = __builtin_amdgcn_readlane(pages, 4 * (n - last) + y);
      const int valid = id < 0 ? 0 : max(0, min(16, sq.k_len - key));
      const int64_t off = ((int64_t)max(id, 0) * p.pages.hkv + h) * block;
      // (rows behind the sequence's last have scales of 0, whatever their codes)
      auto codes = [&](const void* base) { return __builtin_amdgcn_make_buffer_rsrc((char*)base + off + at * tkv::kRow4, 0, valid * tkv::kRow4, 0x00020000); };
      auto scale = [&](const void* base) { return __builtin_amdgcn_make_buffer_rsrc((char*)base + off + scales + at * tkv::kScales4, 0, valid * tkv::kScales4, 0x00020000); };
      x.k[y] = __builtin_amdgcn_raw_buffer_load_b128(codes(p.pages.k), col * 64 + quarter * 16, 0, 0);
      x.ks[y] = __builtin_amdgcn_raw_buffer_load_b8(scale(p.pages.k), col * 4 + quarter, 0, 0);
      x.v[y] = __builtin_amdgcn_raw_buffer_load_b128(codes(p.pages.v), col * 64 + quarter * 16, 0, 0);
      x.vs[y] = __builtin_amdgcn_raw_buffer_load_b8(scale(p.pages.v), col * 4 + quarter, 0, 0);
    }
  };
  lds_char* const row_at = area + col * 256;
  int to[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) to[i] = 16 * v_place(col, 4 * quarter + i);
  lds_char* va[8];
  {
    const int row = 4 * quarter + col / 4;
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) va[ct] = area + (row * 256 + 16 * v_place(row, 2 * ct + (col % 4) / 2) + 8 * (col % 2));
  }
  Tile x;
  fetch(0, x);
  for (int n = 0; n < mine; ++n) {
    const int key0 = 64 * (t0 + kWaves * n);
    if (n + 1 - last == 16) {
      last = n + 1;
      pages = some_pages<4>(p, sq, t0 + kWaves * last);
    }
    Tile now = x;
    if (n + 1 < mine) fetch(n + 1, x);
    floatx4 s[NT][4];
#pragma unroll
    for (int y = 0; y < 4; ++y) {
#pragma unroll
      for (int m = 0; m < NT; ++m) s[m][y] = (floatx4){0.f, 0.f, 0.f, 0.f};
      const float scale = tkv::scale_of(now.ks[y]);
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        const uintx4 a = __builtin_bit_cast(uintx4, tkv::values_of<T>(now.k[y][kk], scale));
#pragma unroll
        for (int m = 0; m < NT; ++m) s[m][y] = mfma16<T>(a, qf[m][kk], s[m][y]);
      }
    }
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const float scale = tkv::scale_of(now.vs[y]);
#pragma unroll
      for (int i = 0; i < 4; ++i) lds_write16(row_at + 4096 * y + to[i], __builtin_bit_cast(uintx4, tkv::values_of<T>(now.v[y][i], scale)));
    }
    uintx4 w[NT][2];
    weigh<T, NT, 4>(r, s, w, key0, p.scale2, quarter);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
#pragma unroll
    for (int z = 0; z < 2; ++z)
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) {
        const uintx2 lo = lds_read_tr(va[ct] + 8192 * z), hi = lds_read_tr(va[ct] + 8192 * z + 4096);
        const uintx4 a = __builtin_shufflevector(lo, hi, 0, 1, 2, 3);
#pragma unroll
        for (int m = 0; m < NT; ++m) r.o[m][ct] = mfma16<T>(a, w[m][z], r.o[m][ct]);
      }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  }
}

template <typename T>
__device__ inline void store8(T* to, floatx8 x) { *(uintx4*)to = pack8<T>(x); }

// Keys of a tile, and bytes of LDS: the waves' rings or areas, and the waves' results where they join.
template <int BITS>
constexpr int tile_keys() { return BITS == 16 ? 32 : 64; }
template <int BITS, int NT>
constexpr int lds_bytes() {
  return std::max(kWaves * (BITS == 16 ? 4 * 32 * TKV_D * 2 : 64 * TKV_D * 2), kWaves * 16 * NT * (kRowFloats + 2) * 4);
}

template <typename T, int BITS, int NT>
__global__ __launch_bounds__(64 * kWaves, BITS == 4 && NT < 4 ? 2 : 1) void paged_attn_kernel(PagedParams p) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  constexpr int kRows = 16 * NT, TK = tile_keys<BITS>();
  const int lane = threadIdx.x % 64, col = lane % 16, quarter = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  Walk<TK, kRows> walk(p);
  const uint32_t total = walk.total(), per = range_of(total, p.workgroups);
  const uint64_t begin64 = (uint64_t)blockIdx.x * per;
  if (begin64 >= total) return;
  const uint32_t begin = (uint32_t)begin64, end = (uint32_t)min((uint64_t)total, begin64 + per);
  for (uint32_t at = begin; at < end;) {
    const Sequence sq = walk.find(at);
    if (sq.index < 0) return;
    const uint32_t in = at - sq.first, item = in / (uint32_t)sq.key_tiles;
    const int a = (int)(in - item * (uint32_t)sq.key_tiles);
    const int b = (int)min((uint32_t)sq.key_tiles, (uint32_t)a + (end - at));
    const int h = (int)(item / (uint32_t)sq.row_tiles), tile = (int)(item - (uint32_t)h * (uint32_t)sq.row_tiles);
    const int rows = sq.q_len * p.group, ahead = sq.k_len - sq.q_len;

    Rows<NT> r;
    uintx4 qf[NT][4];
    r.limit_low = tile * kRows / p.group + ahead;
#pragma unroll
    for (int m = 0; m < NT; ++m) {
      const int row = min(tile * kRows + 16 * m + col, rows - 1), token = row / p.group, head = row - token * p.group;
      r.limit[m] = token + ahead;
      r.ref[m] = kNone;
      r.sum[m] = 0.f;
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) r.o[m][ct] = (floatx4){0.f, 0.f, 0.f, 0.f};
      const T* const q = (const T*)p.q + ((int64_t)(sq.q_start + token) * p.hq + h * p.group + head) * TKV_D;
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) qf[m][kk] = *(const uintx4*)(q + (BITS == 16 ? 32 * kk + 8 * quarter : 32 * quarter + 8 * kk));
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) asm volatile("" : "+v"(qf[m][kk]));  // (waited for here, not in the loop)
    }
    if constexpr (BITS == 16) segment16<T, NT>(p, sq, h, a + wave, b, qf, r, (lds_char*)lds + wave * (4 * 32 * TKV_D * 2));
    else segment4<T, NT>(p, sq, h, a + wave, b, qf, r, (lds_char*)lds + wave * (64 * TKV_D * 2));

    // the waves join: everyone's results into LDS, then sixteen threads a row
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // no load may land after the ring is used otherwise
    __syncthreads();
    float* const o_s = (float*)lds;                              // [wave][row][kRowFloats]
    float* const ml_s = o_s + kWaves * kRows * kRowFloats;       // [wave][row][2]
#pragma unroll
    for (int m = 0; m < NT; ++m) {
      const float sum = tkv::over_rows(r.sum[m], [](float x, float y) { return x + y; });
      const int at_row = wave * kRows + 16 * m + col;
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) *(floatx4*)(o_s + at_row * kRowFloats + 16 * ct + 4 * quarter) = r.o[m][ct];
      if (quarter == 0) *(float2*)(ml_s + 2 * at_row) = make_float2(r.ref[m], sum);
    }
    __syncthreads();
    const bool whole = a == 0 && b == sq.key_tiles;
    const int slot = 2 * (int)blockIdx.x + (at == begin ? 0 : 1);
#pragma unroll
    for (int m = 0; m < NT; ++m) {
      const int in_tile = 16 * m + threadIdx.x / 16, row = tile * kRows + in_tile, c = 8 * (threadIdx.x % 16);
      if (row >= rows) continue;
      float f[kWaves], top = kNone, sum = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, f[w] = ml_s[2 * (w * kRows + in_tile)]);
      floatx8 x = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        f[w] = __builtin_amdgcn_exp2f(f[w] - top);
        sum = __builtin_fmaf(ml_s[2 * (w * kRows + in_tile) + 1], f[w], sum);
        const float* const from = o_s + (w * kRows + in_tile) * kRowFloats + c;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __builtin_fmaf(from[i], f[w], x[i]);
      }
      if (!whole) {
        float* const to = p.parts + ((size_t)slot * kRows + in_tile) * TKV_D + c;
        *(floatx4*)to = __builtin_shufflevector(x, x, 0, 1, 2, 3);
        *(floatx4*)(to + 4) = __builtin_shufflevector(x, x, 4, 5, 6, 7);
        if (c == 0) *(float2*)(p.ml + ((size_t)slot * kRows + in_tile) * 2) = make_float2(top, sum);
        continue;
      }
      const int token = row / p.group, head = row - token * p.group;
      const int64_t to = (int64_t)(sq.q_start + token) * p.hq + h * p.group + head;
      store8<T>((T*)p.out + to * TKV_D + c, x * (sum == 0.f ? 0.f : 1.f / sum));  // (no key: zeros)
      if (p.lse && c == 0) p.lse[to] = sum == 0.f ? -INFINITY : (top - kShift + __builtin_amdgcn_logf(sum)) * 0.69314718055994531f;
    }
    __syncthreads();
    at += (uint32_t)(b - a);
  }
}

// Joins the parts of items that were cut: workgroup w looks after the item, if there is one, whose first cut lies behind range w, a wave a
// row, a lane two channels.
template <typename T, int BITS, int NT>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedParams p) {
  constexpr int kRows = 16 * NT;
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  Walk<tile_keys<BITS>(), kRows> walk(p);
  const uint32_t total = walk.total(), per = range_of(total, p.workgroups);
  const uint64_t cut = (uint64_t)(blockIdx.x + 1) * per;
  if (cut >= total) return;
  const Sequence sq = walk.find((uint32_t)cut);
  if (sq.index < 0) return;
  const uint32_t in = (uint32_t)cut - sq.first, item = in / (uint32_t)sq.key_tiles;
  const uint32_t start = sq.first + item * (uint32_t)sq.key_tiles;
  if (start >= cut || start < cut - per) return;
  const int h = (int)(item / (uint32_t)sq.row_tiles), tile = (int)(item - (uint32_t)h * (uint32_t)sq.row_tiles);
  const int in_tile = 4 * blockIdx.y + wave, row = tile * kRows + in_tile;
  if (row >= sq.q_len * p.group) return;
  const int parts = (int)((start + (uint32_t)sq.key_tiles - 1) / per - blockIdx.x) + 1;
  const int first_slot = 2 * (int)blockIdx.x + (start == cut - per ? 0 : 1);
  float m = kNone, l = 0.f;
  float2 acc = make_float2(0.f, 0.f);
  // (requests of eight parts at a time, absent ones those of the first with a weight of zero)
  for (int i0 = 0; i0 < parts; i0 += 8) {
    float2 st[8], v[8];
#pragma unroll
    for (int y = 0; y < 8; ++y) {
      const int i = i0 + y < parts ? i0 + y : 0;
      const size_t at = (size_t)(i == 0 ? first_slot : 2 * ((int)blockIdx.x + i)) * kRows + in_tile;
      st[y] = *(const float2*)(p.ml + at * 2);
      v[y] = *(const float2*)(p.parts + at * TKV_D + 2 * lane);
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
      const float w = i0 + y < parts ? __builtin_amdgcn_exp2f(st[y].x - m) : 0.f;
      l = __builtin_fmaf(st[y].y, w, l);
      acc.x = __builtin_fmaf(v[y].x, w, acc.x);
      acc.y = __builtin_fmaf(v[y].y, w, acc.y);
    }
  }
  const int token = row / p.group, head = row - token * p.group;
  const int64_t to = (int64_t)(sq.q_start + token) * p.hq + h * p.group + head;
  typedef T T2 __attribute__((ext_vector_type(2)));
  const float inv = l == 0.f ? 0.f : 1.f / l;
  *(T2*)((T*)p.out + to * TKV_D + 2 * lane) = (T2){(T)(acc.x * inv), (T)(acc.y * inv)};
  if (p.lse && lane == 0) p.lse[to] = l == 0.f ? -INFINITY : (m - kShift + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
}

constexpr int kMaxWorkgroups = 512;
constexpr size_t kWorkspace = (size_t)2 * kMaxWorkgroups * 64 * (TKV_D + 2) * sizeof(float);

template <typename T, int BITS, int NT>
int32_t launch_attn(PagedParams& p, int units, hipStream_t s) {
  constexpr int lds = lds_bytes<BITS, NT>(), each = lds <= 80 * 1024 && BITS == 4 && NT < 4 ? 2 : 1;
  static_assert(lds <= 160 * 1024, "LDS of one compute unit");
  static const bool lds_ok = hipFuncSetAttribute(reinterpret_cast<const void*>(&paged_attn_kernel<T, BITS, NT>),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, lds) == hipSuccess;
  if (!lds_ok) return TKV_E_HIP;
  p.workgroups = std::min(kMaxWorkgroups, units * each);
  p.ml = p.parts + (size_t)2 * kMaxWorkgroups * 64 * TKV_D;
  TKV_LAUNCH((paged_attn_kernel<T, BITS, NT>), dim3((uint32_t)p.workgroups), 64 * kWaves, lds, s, p);
  if (p.workgroups > 1)
    TKV_LAUNCH((paged_merge_kernel<T, BITS, NT>), dim3((uint32_t)p.workgroups - 1, 4 * NT), 256, 0, s, p);
  return TKV_OK;
}

template <typename T, int BITS>
int32_t launch_rows(PagedParams& p, int64_t rows, int units, hipStream_t s) {
  if (rows <= 16) return launch_attn<T, BITS, 1>(p, units, s);
  if (rows <= 32) return launch_attn<T, BITS, 2>(p, units, s);
  return launch_attn<T, BITS, 4>(p, units, s);
}

// Whether rows of 128 elements at p s[0] + h s[1] + t s[2] do not overlap, each axis beyond all that smaller strides span.
bool rows_apart(const int64_t* s, const int64_t (&count)[3]) {
  int order[3] = {0, 1, 2};
  std::sort(order, order + 3, [&](int a, int b) { return s[a] < s[b]; });
  int64_t span = TKV_D;
  for (int i : order) {
    if (count[i] > 1 && s[i] < span) return false;
    if (count[i] > 1) span += s[i] * (count[i] - 1);
  }
  return true;
}

bool good_strides(const int64_t* s) {
  for (int i = 0; i < 3; ++i)
    if (s[i] < 0 || s[i] % 8 != 0 || s[i] > ((int64_t)1 << 36)) return false;
  return s[2] <= (1 << 22);  // (a tile's rows are addressed with 32 bits)
}

}  // namespace

int32_t tkv::check_paged_desc(const tkv_paged_desc* d) {
  if (!d || d->struct_size != sizeof(tkv_paged_desc)) return TKV_E_INVAL;
  if (d->n_q_heads <= 0 || d->n_kv_heads <= 0 || d->head_dim <= 0 || d->n_pages <= 0 || d->page_size <= 0) return TKV_E_INVAL;
  if (d->n_q_heads % d->n_kv_heads != 0) return TKV_E_INVAL;
  if (d->dtype != TKV_F16 && d->dtype != TKV_BF16) return TKV_E_INVAL;
  if (d->head_dim != TKV_D || d->n_q_heads > 1024 || (d->bits != 16 && d->bits != 4)) return TKV_E_UNSUPPORTED;
  if (d->page_size < 16 || d->page_size > 1024 || (d->page_size & (d->page_size - 1)) != 0) return TKV_E_UNSUPPORTED;
  if ((int64_t)d->n_pages * d->page_size > 0x7FFFFFFF) return TKV_E_UNSUPPORTED;  // (slots are 32 bits)
  if (d->bits == 16) {
    const int64_t count[3] = {d->n_pages, d->n_kv_heads, d->page_size};
    if (!good_strides(d->k_stride) || !good_strides(d->v_stride)) return TKV_E_INVAL;
    if (!rows_apart(d->k_stride, count) || !rows_apart(d->v_stride, count)) return TKV_E_INVAL;
  }
  return TKV_OK;
}

int32_t tkv::paged_view(const tkv_paged_desc* d, void* k_pages, void* v_pages, Pages* out) {
  if (!k_pages || !v_pages || ((uintptr_t)k_pages & 15) != 0 || ((uintptr_t)v_pages & 15) != 0) return TKV_E_INVAL;
  Pages& p = *out;
  p.k = k_pages;
  p.v = v_pages;
  p.hkv = d->n_kv_heads;
  p.n_pages = d->n_pages;
  p.shift = __builtin_ctz((unsigned)d->page_size);
  if (d->bits == 16) {
    p.k_sp = d->k_stride[0]; p.k_sh = d->k_stride[1]; p.k_st = d->k_stride[2];
    p.v_sp = d->v_stride[0]; p.v_sh = d->v_stride[1]; p.v_st = d->v_stride[2];
  } else {
    p.k_st = p.v_st = kRow4;
    p.k_sh = p.v_sh = (int64_t)(kRow4 + kScales4) * d->page_size;
    p.k_sp = p.v_sp = p.k_sh * d->n_kv_heads;
  }
  return TKV_OK;
}

extern "C" int32_t tkv_paged_cache_sizes(const tkv_paged_desc* d, size_t* bytes_each) {
  const int32_t st = tkv::check_paged_desc(d);
  if (st != TKV_OK) return st;
  if (!bytes_each) return TKV_E_INVAL;
  *bytes_each = (size_t)d->n_pages * d->n_kv_heads * d->page_size * (d->bits == 16 ? 2 * TKV_D : tkv::kRow4 + tkv::kScales4);
  return TKV_OK;
}

extern "C" int32_t tkv_paged_gather(const tkv_paged_desc* d, const void* k_pages, const void* v_pages, int32_t n_tokens,
                                    const int32_t* slots, void* k_out, void* v_out, void* stream) {
  int32_t st = tkv::check_paged_desc(d);
  if (st != TKV_OK) return st;
  if (n_tokens < 0) return TKV_E_INVAL;
  if (n_tokens == 0) return TKV_OK;
  if (!slots || !k_out || !v_out || (((uintptr_t)k_out | (uintptr_t)v_out) & 15) != 0 || ((uintptr_t)slots & 3) != 0) return TKV_E_INVAL;
  GatherParams p;
  st = tkv::paged_view(d, const_cast<void*>(k_pages), const_cast<void*>(v_pages), &p.pages);
  if (st != TKV_OK) return st;
  const int64_t waves = ((int64_t)n_tokens + 15) / 16 * 2 * d->n_kv_heads;
  if (waves > 4 * ((1 << 24) - 1)) return TKV_E_UNSUPPORTED;  // (a launch has fewer than 2^32 threads)
  p.slots = slots;
  p.k_out = k_out;
  p.v_out = v_out;
  p.n_tokens = n_tokens;
  p.waves = (int32_t)waves;
  const dim3 grid((uint32_t)((waves + 3) / 4));
  const auto s = (hipStream_t)stream;
  if (d->bits == 16) TKV_LAUNCH((paged_gather_kernel<_Float16, 16>), grid, 256, 0, s, p);
  else if (d->dtype == TKV_F16) TKV_LAUNCH((paged_gather_kernel<_Float16, 4>), grid, 256, 0, s, p);
  else TKV_LAUNCH((paged_gather_kernel<__bf16, 4>), grid, 256, 0, s, p);
  return TKV_OK;
}

extern "C" int32_t tkv_paged_attn_sizes(const tkv_paged_desc* d, size_t* workspace_bytes) {
  const int32_t st = tkv::check_paged_desc(d);
  if (st != TKV_OK) return st;
  if (!workspace_bytes) return TKV_E_INVAL;
  *workspace_bytes = kWorkspace;
  return TKV_OK;
}

extern "C" int32_t tkv_paged_attn(const tkv_paged_desc* d, const void* k_pages, const void* v_pages, int32_t batch, int32_t n_tokens,
                                  int32_t max_q_len, const void* q, void* out, float* lse, const int32_t* page_table,
                                  int32_t pages_each, const int32_t* k_lens, const int32_t* q_starts, float sm_scale, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  int32_t st = tkv::check_paged_desc(d);
  if (st != TKV_OK) return st;
  if (batch < 0 || n_tokens < 0 || max_q_len <= 0 || pages_each < 0 || !workspace) return TKV_E_INVAL;
  const float scale2 = sm_scale * 1.4426950408889634f;
  if (!(sm_scale > 0.f) || !(scale2 <= 3.402823466e38f)) return TKV_E_INVAL;
  if (!q_starts && (n_tokens != batch || max_q_len != 1)) return TKV_E_INVAL;
  if ((int64_t)pages_each * d->page_size > 0x7FFFFFFF) return TKV_E_UNSUPPORTED;
  if (workspace_bytes < kWorkspace) return TKV_E_WORKSPACE;
  if (n_tokens == 0 || batch == 0) return TKV_OK;
  if (!q || !out || !k_lens || (pages_each && !page_table)) return TKV_E_INVAL;
  for (const void* x : {q, (const void*)out, (const void*)workspace})
    if (((uintptr_t)x & 15) != 0) return TKV_E_INVAL;
  for (const void* x : {(const void*)lse, (const void*)page_table, (const void*)k_lens, (const void*)q_starts})
    if (((uintptr_t)x & 3) != 0) return TKV_E_INVAL;
  PagedParams p;
  st = tkv::paged_view(d, const_cast<void*>(k_pages), const_cast<void*>(v_pages), &p.pages);
  if (st != TKV_OK) return st;
  p.q = q; p.out = out; p.lse = lse;
  p.table = page_table; p.k_lens = k_lens; p.q_starts = q_starts;
  p.n_tokens = n_tokens; p.batch = batch; p.pages_each = pages_each;
  p.hq = d->n_q_heads;
  p.group = d->n_q_heads / d->n_kv_heads;
  p.scale2 = scale2;
  p.parts = (float*)workspace;
  // (numbers of tiles are 32 bits: tiles of 16 rows and 32 keys, the smallest)
  const int64_t row_tiles = (int64_t)n_tokens * p.group / 16 + batch, key_tiles = (((int64_t)pages_each * d->page_size) >> 5) + 1;
  if (row_tiles * d->n_kv_heads >= ((int64_t)1 << 31) || row_tiles * d->n_kv_heads * key_tiles >= ((int64_t)1 << 31)) return TKV_E_UNSUPPORTED;
  if ((int64_t)n_tokens * p.group > (1 << 30)) return TKV_E_UNSUPPORTED;
  const int64_t rows = (int64_t)max_q_len * p.group;
  const auto s = (hipStream_t)stream;
  const int units = tkv::stream_compute_units(s);
  if (d->dtype == TKV_F16) return d->bits == 16 ? launch_rows<_Float16, 16>(p, rows, units, s) : launch_rows<_Float16, 4>(p, rows, units, s);
  return d->bits == 16 ? launch_rows<__bf16, 16>(p, rows, units, s) : launch_rows<__bf16, 4>(p, rows, units, s);
}
