// Paged caches: rows read back from their pages (tkv_paged_gather) and attention over them (tkv_paged_attn): softmax(sm q K^T) V over
// keys and values that lie in pages, in 16 bits or as microscaled 4-bit numbers, for single tokens, drafts and short chunks.
//
// The bytes of the cache bound the attention: 16 sequences of 16000 tokens, 8 KV heads, 16 bits (1.05 GB) 182 us, 5.8 TB/s; 4 of
// 131072 in 4 bits (0.57 GB) 106 us, 5.4 TB/s (a read of 2 GiB alone reaches 5.4); short calls are a chain of round trips: one token over
// 128 keys 5.6 us, over 512 8.0, 64 sequences of up to 300 17.
//
// The query heads of a KV head, of all the call's tokens of a sequence, are rows of one matrix, sixteen to an operand, so that keys and values
// are read once for up to 48 of them (4 bits: 32); of more rows every 48 (32) read them again.  Both products are transposed (S^T = K Q^T, O^T = V^T P^T): a lane's column is a row of queries, its
// softmax statistics one number a lane, and its weights lie where the second product wants them: the keys of a lane's eight weights are 16 y
// + 4 (lane / 16) + i, and the values' LDS reads, which transpose 4 x 16 elements on the way, take them in that order (a sum over keys does
// not mind it).  One pass over the keys: running reference and sum in float32, weights rounded to the type for the second product (off by
// half a step of it each, beside the output's own rounding; divided by the sum of the unrounded ones: against float64 2.9e-4 of the outputs'
// norm in fp16, 2.1e-4 of them the output's).
//
// Lengths, tables and starts lie on the device, and nothing on the host depends on them: a captured step replays over a cache that
// grows.  Every wave works its share out by itself (Walk, Plan); the shares are equal whatever the lengths, so that no sequence is too long
// and none too short (one of 20011 tokens among 19 of a few).
#include <algorithm>
#include <type_traits>

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

// Rows from pages, contiguous.  A wave takes 4 J tokens of one head's keys or values, sixteen lanes a row: neighbours in a page are read
// side by side (64 bytes a row in 4 bits), and rows are written whole, past the caches' usual order (nontemporal: 20000 tokens of 16 bits
// 30.6 -> 27.4 us, 100003 of 4 bits 118 -> 111; with 32 instead of 16 tokens a wave 111 -> 101.5, 16 bits 27.6 -> 39).  Bound by the
// memory's rate: 5.9 and 5.1 TB/s.
template <typename T, int BITS, int J>
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
  const int64_t t0 = (int64_t)4 * J * tile + sub;
  int32_t slot[J];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int64_t t = t0 + 4 * j;
    slot[j] = t < p.n_tokens ? p.slots[t] : -1;
    if (slot[j] >> p.pages.shift >= p.pages.n_pages) slot[j] = -1;
  }
  uintx4 x[J];
  uint32_t codes[J], scale[J];
#pragma unroll
  for (int j = 0; j < J; ++j) {
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
  for (int j = 0; j < J; ++j) {
    const int64_t t = t0 + 4 * j;
    if (t >= p.n_tokens) continue;
    if constexpr (BITS == 4) x[j] = __builtin_bit_cast(uintx4, tkv::values_of<T>(codes[j], tkv::scale_of(scale[j])));
    __builtin_nontemporal_store(x[j], (uintx4*)(out + (t * p.pages.hkv + h) * TKV_D + 8 * place));
  }
}

constexpr int kWaves = 4;              // of a workgroup
constexpr int kRowFloats = TKV_D + 4;  // of a row of partial sums in LDS (the four keep the banks apart)
// Weights are 2^(logit - reference + kShift), at most 2^kLargest, inside fp16's range: the reference follows a row's maximum only where a weight
// is larger.  Whether one is, its exponent itself says, worked out as the weights are (one rounding): at logits of 2^26, in float32's steps
// of 8, a maximum that is rounded by itself can be half a step too low.  kShift is 8 for the same reason: a whole number of
// steps up to 2^27 in units of log 2 (logits of 2^26), so that all references are less by the same (7 is one up to 2^24 only, and weights
// under different references were up to 4 times too large beyond); next to a power of two the difference may be rounded by half a step.
constexpr float kShift = 8.f, kLargest = 15.f;
constexpr float kNone = -3.402823466e38f;  // reference of a row without a key so far (finite: kNone - kNone is 0)
constexpr int kMaxUnits = 256;             // compute units that the workspace has room for
constexpr int kMostParts = 64;             // of an item (in workgroups), so that joining them stays short

struct PagedParams {
  tkv::Pages pages;
  const void* q;
  void* out;
  float* lse;  // NULL: not wanted
  const int32_t* table;
  const int32_t* k_lens;
  const int32_t* q_starts;  // NULL: a token of each sequence
  float* parts;             // [2 per wave][rows of a tile][128] weighted sums
  float* ml;                // [2 per wave][rows of a tile][2] (reference, sum)
  uint32_t* arrivals;       // [wave] parts, of the item whose first cut lies behind its range, that have come in
  int32_t n_tokens, batch, max_q_len, hq, group, pages_each;
  uint32_t per_group;  // 2^32 / group, rounded up: rows / group without a division
  int32_t workgroups;
  int32_t clear_rest;  // rows of no sequence get zeros
  float scale2;        // sm_scale * log2(e)
};

// The kernel's arguments, read where they are used: kept in registers from the start on, they and the loop over the tiles have more than
// there are.
typedef const __attribute__((address_space(4))) PagedParams* Args;
__device__ inline Args arguments() {
  Args a = (Args)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(a));
  return a;
}

// How the work is shared out.  Every (sequence, KV head, tile of rows) is an item, its keys so many tiles of TK; all items' tiles in
// a row are cut into as many equal ranges as there are waves.  Lengths lie on the device, so every wave works that out for
// itself: 64 sequences at a time, one a lane.
struct Sequence {
  int32_t index, k_len, q_start, q_len, key_tiles, row_tiles;
  uint32_t first;  // of its tiles, among all
};

// One of an item's tiles, and the item.
struct Place {
  Sequence sq;
  uint32_t start;     // of the item's tiles, among all
  int32_t h, tile, t; // KV head, tile of rows, tile of keys
};

// Every lane: f over the lanes up to it (0 where there is none).  By data-parallel primitives: rows of sixteen, then their last lanes'
// values into the rows behind.
template <typename F>
__device__ inline uint32_t scan(uint32_t x, F f) {
  x = f(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xF, 0xF, true));  // row_shr: 1, 2, 4, 8
  x = f(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xF, 0xF, true));
  x = f(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xF, 0xF, true));
  x = f(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xF, 0xF, true));
  x = f(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xA, 0xF, false));  // row_bcast: 15 into rows 1 and 3, 31 into 2 and 3
  x = f(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xC, 0xF, false));
  return x;
}

template <int TK, int ROWS>
struct Walk {
  int32_t group, batch;
  int32_t chunk;                  // first sequence of those at hand
  int32_t k_len, q_start, q_len;  // per lane
  uint32_t first, count;          // per lane: tiles before its sequence, and of it
  uint32_t all;                   // tiles up to the chunk's end
  int32_t longest;                // tiles of keys of the longest sequence so far

  __device__ Walk() : group(arguments()->group), batch(arguments()->batch), longest(1) { load(0, 0); }

  __device__ int32_t key_tiles(int32_t n) const { return max(1, (n + TK - 1) / TK); }
  __device__ int32_t row_tiles(int32_t n) const { return (n * group + ROWS - 1) / ROWS; }

  __device__ void load(int32_t at, uint32_t before) {
    const Args p = arguments();
    const int lane = threadIdx.x % 64, b = at + lane;
    chunk = at;
    k_len = q_start = q_len = 0;
    if (b < batch) {
      const int32_t* const starts = p->q_starts;
      k_len = (int32_t)max((int64_t)0, min((int64_t)p->k_lens[b], (int64_t)p->pages_each << p->pages.shift));
      q_start = b;
      q_len = 1;
      if (starts) {
        q_start = min(max(starts[b], 0), p->n_tokens);
        q_len = max(0, min(min(max(starts[b + 1], 0), p->n_tokens) - q_start, p->max_q_len));
      }
    }
    count = (uint32_t)(key_tiles(k_len) * row_tiles(q_len)) * (uint32_t)p->pages.hkv;  // (no rows: 0)
    const uint32_t sum = scan(count, [](uint32_t a, uint32_t b) { return a + b; });
    first = before + sum - count;
    all = before + (uint32_t)__builtin_amdgcn_readlane((int)sum, 63);
    const uint32_t most = scan(count ? (uint32_t)key_tiles(k_len) : 0u, [](uint32_t a, uint32_t b) { return max(a, b); });
    longest = max(longest, __builtin_amdgcn_readlane((int)most, 63));
  }
  __device__ uint32_t total() {
    while (chunk + 64 < batch) load(chunk + 64, all);
    const uint32_t t = all;
    if (chunk != 0) load(0, 0);
    return t;
  }
  // The place of tile number `at`, below total() and not before the chunk at hand.
  __device__ Place find(uint32_t at) {
    while (at >= all && chunk + 64 < batch) load(chunk + 64, all);
    const uint64_t here = __builtin_amdgcn_ballot_w64(first <= at && at < first + count);
    const int l = here ? __builtin_ctzll(here) : 0;
    Place x;
    x.sq.index = chunk + l;
    x.sq.k_len = __builtin_amdgcn_readlane(k_len, l);
    x.sq.q_start = __builtin_amdgcn_readlane(q_start, l);
    x.sq.q_len = __builtin_amdgcn_readlane(q_len, l);
    x.sq.first = (uint32_t)__builtin_amdgcn_readlane((int)first, l);
    x.sq.key_tiles = key_tiles(x.sq.k_len);
    x.sq.row_tiles = row_tiles(x.sq.q_len);
    const uint32_t in = at - x.sq.first, item = in / (uint32_t)x.sq.key_tiles;
    x.start = x.sq.first + item * (uint32_t)x.sq.key_tiles;
    x.t = (int32_t)(at - x.start);
    x.h = (int32_t)(item / (uint32_t)x.sq.row_tiles);
    x.tile = (int32_t)(item - (uint32_t)x.h * (uint32_t)x.sq.row_tiles);
    return x;
  }
};

// Tiles of a wave's range: as even as can be, but an item goes to about kMostParts workgroups at most.  (64 parts of one row join in about
// 4 us; one sequence and one KV head would have 256.)
__device__ inline uint32_t range_of(uint32_t total, int32_t longest, int workgroups) {
  const uint32_t waves = (uint32_t)(kWaves * workgroups);
  return max((total + waves - 1) / waves, (uint32_t)(longest + kWaves * kMostParts - 1) / (uint32_t)(kWaves * kMostParts));
}

// Where a wave's next sixteens of keys lie, one a lane: those of tiles begin, begin + (1 << log_step), ..., PER a tile, whatever items they are of.
template <int PER>
struct Plan {
  uint32_t begin, stop;  // of the tiles at hand
  int32_t log_step;      // the next tile is 1 << log_step on
  // per lane
  int64_t k_at, v_at;    // bytes from the pages' beginning: of the first row (16 bits; in 4 bits of the page's and head's block, v_at is k_at)
  uint32_t place, rows;  // first place in the page, rows that are there

  template <typename W>
  __device__ void make(W& walk, uint32_t from, uint32_t end) {
    const Args p = arguments();
    while (from >= walk.all && walk.chunk + 64 < walk.batch) walk.load(walk.chunk + 64, walk.all);
    begin = from;
    stop = min(min(from + ((uint32_t)(64 / PER) << log_step), end), walk.all);
    const int lane = threadIdx.x % 64;
    const uint32_t g = min(from + ((uint32_t)(lane / PER) << log_step), stop - 1u);
    // its sequence: nearly always the first one's, otherwise the last that begins at or before it (one without tiles shares its
    // successor's beginning)
    const uint64_t here = __builtin_amdgcn_ballot_w64(walk.first <= from && from < walk.first + walk.count);
    int l = here ? __builtin_ctzll(here) : 0;
    int32_t k_len = __builtin_amdgcn_readlane(walk.k_len, l), q_len = __builtin_amdgcn_readlane(walk.q_len, l);
    uint32_t first = (uint32_t)__builtin_amdgcn_readlane((int)walk.first, l);
    if (stop > first + (uint32_t)__builtin_amdgcn_readlane((int)walk.count, l)) {
      l = 0;
#pragma unroll
      for (int d = 32; d > 0; d /= 2) {
        const uint32_t f = (uint32_t)__shfl((int)walk.first, l + d, 64);
        if (f <= g) l += d;
      }
      k_len = __shfl(walk.k_len, l, 64);
      q_len = __shfl(walk.q_len, l, 64);
      first = (uint32_t)__shfl((int)walk.first, l, 64);
    }
    const uint32_t key_tiles = (uint32_t)walk.key_tiles(k_len), row_tiles = (uint32_t)max(1, walk.row_tiles(q_len));
    const uint32_t in = g - first, item = in / key_tiles, h = min(item / row_tiles, (uint32_t)p->pages.hkv - 1u);
    const int32_t key = 16 * ((int32_t)(in - item * key_tiles) * PER + lane % PER);
    const int32_t there = max(0, min(16, k_len - key));
    int32_t page = -1;
    if (there > 0 && walk.chunk + l < walk.batch) page = p->table[(int64_t)(walk.chunk + l) * p->pages_each + (key >> p->pages.shift)];
    const bool none = page < 0 || page >= p->pages.n_pages;
    rows = none ? 0u : (uint32_t)there;
    place = (uint32_t)(key & ((1 << p->pages.shift) - 1));
    const int64_t id = none ? 0 : page, by = PER == 2 ? 2 : 1, first_row = PER == 2 ? place : 0;
    k_at = (id * p->pages.k_sp + (int64_t)h * p->pages.k_sh + first_row * p->pages.k_st) * by;
    if (PER == 2) v_at = (id * p->pages.v_sp + (int64_t)h * p->pages.v_sh + first_row * p->pages.v_st) * by;
  }
  __device__ bool has(uint32_t tile) const { return tile < stop; }
  __device__ int lane_of(uint32_t tile) const { return (int)((tile - begin) >> log_step) * PER; }
};

// A lane's 64 bits, for all.
__device__ inline int64_t of_lane(int64_t x, int l) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, l), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)x >> 32), l);
  return (int64_t)((uint64_t)hi << 32 | lo);
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
// Four times 16 bytes per lane from a descriptor's array straight to LDS, 1 KiB each, in lane order from `to` (uniform) on.  By hand,
// because the compiler lets every transposing LDS read wait for all such loads, those of the next tile too; nothing lands in registers, and
// the caller waits itself (vmcnt) before anyone reads the buffer.  (m0 is used by nothing else here: the compiler, which
// cannot be told of it, since it is reserved, never does; and it does not know that a descriptor that the vector unit has just
// written, by readfirstlane, is there for a load five wait states later: the first two instructions.  tests/test_lds_loads.py looks for both.)
__device__ inline void to_lds(__amdgpu_buffer_rsrc_t from, uint32_t to, const uint32_t (&lane_offset)[4]) {
  asm volatile(
      "s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %2, %1, 0 offen lds\n\t"
      "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 %3, %1, 0 offen lds\n\t"
      "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 %4, %1, 0 offen lds\n\t"
      "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 %5, %1, 0 offen lds" ::"s"(to), "s"(from), "v"(lane_offset[0]),
      "v"(lane_offset[1]), "v"(lane_offset[2]), "v"(lane_offset[3])
      : "memory", "scc");
}

// A descriptor of `bytes` bytes from an address that is the same for all lanes, as the assembly above wants it: in scalar registers.
__device__ inline __amdgpu_buffer_rsrc_t uniform_array(const char* at, int32_t bytes) {
  const uint64_t a = (uint64_t)at;
  const uint64_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)a), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32));
  return __builtin_amdgcn_make_buffer_rsrc((void*)(hi << 32 | lo), 0, __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}

// What a wave carries over an item's tiles: weighted sums, transposed (lane: row lane % 16 of each sixteen, channels
// 16 ct + 4 (lane / 16) + i), reference and its share of the sum of weights.
template <int NT>
struct Rows {
  floatx4 o[NT][8];
  float ref[NT], sum[NT];
  int32_t limit[NT];  // last key that the lane's row sees
  int32_t limit_low;  // ... and the item's first row
  float scale2;
};

// Weights of 16 Y keys from key0 on, from their logits s (lane: row, keys key0 + 16 y + 4 (lane / 16) + i) for the next product:
// element 4 (y % 2) + i of operand y / 2.
template <typename T, int NT, int Y>
__device__ inline void weigh(Rows<NT>& r, floatx4 (&s)[NT][Y], uintx4 (&w)[NT][Y / 2], int key0) {
  const float scale2 = r.scale2;
  const bool mask = key0 + 16 * Y - 1 > r.limit_low;
  const int quarter = threadIdx.x % 64 / 16;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    if (__builtin_expect(mask, 0)) {
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
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(__builtin_fmaf(top, scale2, kShift - r.ref[n]) > kLargest) != 0, 0)) {
      top = tkv::over_rows(top * scale2, [](float a, float b) { return fmaxf(a, b); });
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

// A place of 16 bytes in a row of LDS: rows of 256 bytes keep their sixteen places in an order that depends on the row, so that the reads
// (a column of keys; a 4 x 16 block of values) and writes meet all banks (no conflicts counted).  For values eight rows differ in a place's
// upper three bits, for the reads of 32 bytes of a row, and in its lower three, for writes of 16.
__device__ inline int k_place(int row, int place) { return place ^ (row & 15); }
__device__ inline int v_place(int row, int place) { return place ^ (((row & 7) << 1) | (((row >> 2) ^ (row >> 3)) & 1)); }
// Where a lane's transposing read of the first sixteen channels of sixteen values begins (channels 16 ct on: 32 ct in its bits 5 to 7, exclusive or).
__device__ inline int v_read_at() {
  const int lane = threadIdx.x % 64, col = lane % 16, row = 4 * (lane / 16) + col / 4;
  return row * 256 + 16 * v_place(row, (col % 4) / 2) + 8 * (col % 2);
}
// Worked out anew where it is used, by one operation, rather than held in a register for each place.
__device__ inline int anew(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// 16 bits.  Every wave takes tiles of 32 keys of its own through a ring of two in LDS, filled by loads that do not pass through registers:
// 64 KiB on their way in a unit while the matrix cores work for a tenth of the time.
template <typename T, int NT>
struct Tiles16 {
  static constexpr int kKeys = 32, kPer = 2, kTile = kKeys * TKV_D * 2, kBytes = 4 * kTile;
  lds_char* ring;
  const char *k, *v;
  int32_t k_st, v_st;  // bytes
  uint32_t k_off[4], v_off[4];
  int turn;  // the half of the ring that the tile at hand is in
  int ka, va;  // (of kk = 0 and ct = 0; the others differ in some bits: + 64 kk, + 32 ct without a carry)

  __device__ Tiles16(lds_char* lds) : ring(lds), turn(0) {
    const Args p = arguments();
    k = (const char*)p->pages.k;
    v = (const char*)p->pages.v;
    k_st = (int32_t)(2 * p->pages.k_st);
    v_st = (int32_t)(2 * p->pages.v_st);
    const int lane = threadIdx.x % 64, col = lane % 16, quarter = lane / 16;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = 4 * j + quarter;
      k_off[j] = (uint32_t)(row * k_st) + 16u * (uint32_t)k_place(row, col);
      v_off[j] = (uint32_t)(row * v_st) + 16u * (uint32_t)v_place(row, col);
    }
    ka = col * 256 + 16 * k_place(col, quarter);
    va = v_read_at();
  }
  static __device__ int q_channel(int kk) { return 32 * kk + 8 * (int)(threadIdx.x % 64 / 16); }

  __device__ void stage(const Plan<kPer>& plan, uint32_t tile, int half) {
    const uint32_t to0 = (uint32_t)(uintptr_t)ring + (uint32_t)(half * 2 * kTile);
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int l = plan.lane_of(tile) + y, rows = __builtin_amdgcn_readlane((int)plan.rows, l);
      // rows behind the sequence's last, and pages outside, read as zeros
      const auto kr = uniform_array(k + of_lane(plan.k_at, l), rows == 0 ? 0 : (rows - 1) * k_st + TKV_D * 2);
      const auto vr = uniform_array(v + of_lane(plan.v_at, l), rows == 0 ? 0 : (rows - 1) * v_st + TKV_D * 2);
      const uint32_t to = to0 + 4096u * (uint32_t)y;
      to_lds(kr, to, k_off);
      to_lds(vr, to + kTile, v_off);
    }
  }
  __device__ void begin(const Plan<kPer>& plan, uint32_t tile) { stage(plan, tile, 0); }
  // The tile that was sent for last, keys from key0 on; number `tile`, if there are more, is sent for with the plan that next() makes sure of.
  template <typename Next>
  __device__ void work(Plan<kPer>& plan, uint32_t tile, bool more, Next next, int key0, const uintx4 (&qf)[NT][4], Rows<NT>& r) {
    lds_char* const at = ring + turn * 2 * kTile;
    if (more) next();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the other buffer's reads are done)
    if (more) {
      stage(plan, tile, turn ^ 1);
      asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
    } else {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    const int k0 = anew(ka), v0 = anew(va);
    turn ^= 1;
    floatx4 s[NT][2];
#pragma unroll
    for (int m = 0; m < NT; ++m)
#pragma unroll
      for (int y = 0; y < 2; ++y) s[m][y] = (floatx4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const uintx4 a = lds_read16(at + (k0 ^ 64 * kk) + 4096 * y);
#pragma unroll
        for (int m = 0; m < NT; ++m) s[m][y] = mfma16<T>(a, qf[m][kk], s[m][y]);
      }
    uintx4 w[NT][1];
    weigh<T, NT, 2>(r, s, w, key0);
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) {
      const uintx2 lo = lds_read_tr(at + (v0 ^ 32 * ct) + kTile), hi = lds_read_tr(at + (v0 ^ 32 * ct) + kTile + 4096);
      const uintx4 a = __builtin_shufflevector(lo, hi, 0, 1, 2, 3);
#pragma unroll
      for (int m = 0; m < NT; ++m) r.o[m][ct] = mfma16<T>(a, w[m][0], r.o[m][ct]);
    }
  }
};

// 4 bits: tiles of 64 keys; codes go to registers (a lane has 32 channels of a key: one block, and eight channels for each of four
// products, which do not mind the order of the channels), keys from there to the matrix cores, values, as numbers of the type, 32 keys at a
// time through LDS, whose reads transpose them.  The next tile's codes are sent for as soon as this one's have left their registers: eight
// waves a unit with 8.5 KiB each on its way.  (Twelve, as registers would allow with 16 rows: 16 sequences of 100 to 2000 tokens 16.4 -> 14.8
// us, but 4 of 131072 111 -> 117.  Two tiles ahead, in a second set of registers: 111 -> 126.)
template <typename T, int NT>
struct Tiles4 {
  static constexpr int kKeys = 64, kPer = 4, kBytes = 32 * TKV_D * 2;
  lds_char* area;
  const char *k_pages, *v_pages;
  int32_t scales_at, block;  // bytes: where a block's scales begin, all of it
  int to, va;  // (of i = 0 and ct = 0)
  uintx4 k[4], v[4];
  uint32_t ks[4], vs[4];

  __device__ Tiles4(lds_char* lds) : area(lds) {
    const Args p = arguments();
    k_pages = (const char*)p->pages.k;
    v_pages = (const char*)p->pages.v;
    scales_at = tkv::kRow4 << p->pages.shift;
    block = (tkv::kRow4 + tkv::kScales4) << p->pages.shift;
    const int lane = threadIdx.x % 64, col = lane % 16, quarter = lane / 16;
    to = col * 256 + 16 * v_place(col, 4 * quarter);
    va = v_read_at();
  }
  static __device__ int q_channel(int kk) { return 32 * (int)(threadIdx.x % 64 / 16) + 8 * kk; }

  __device__ void fetch(const char* pages, const Plan<kPer>& plan, uint32_t tile, uintx4 (&codes)[4], uint32_t (&scales)[4]) {
    const int lane = threadIdx.x % 64, col = lane % 16, quarter = lane / 16;
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const int l = plan.lane_of(tile) + y, rows = __builtin_amdgcn_readlane((int)plan.rows, l), place = __builtin_amdgcn_readlane((int)plan.place, l);
      const auto from = uniform_array(pages + of_lane(plan.k_at, l), rows == 0 ? 0 : block);  // pages outside read as zeros
      codes[y] = __builtin_amdgcn_raw_buffer_load_b128(from, col * tkv::kRow4 + quarter * 16, place * tkv::kRow4, 0);
      // rows behind the sequence's last have scales of 0, whatever their codes
      const int at = col < rows ? col * tkv::kScales4 + quarter : block;
      scales[y] = __builtin_amdgcn_raw_buffer_load_b8(from, at, scales_at + place * tkv::kScales4, 0);
    }
  }
  // The next tile's codes go out before the other wave of the SIMD works on, and of the two that of the later workgroup, which otherwise
  // comes second every time, comes first (16 sequences of 16000 tokens 62.7 -> 59.3 us, 4 of 131072 110 -> 106.4; without the latter 62, 109).
  __device__ void ahead(const char* pages, const Plan<kPer>& plan, uint32_t tile, uintx4 (&codes)[4], uint32_t (&scales)[4]) {
    __builtin_amdgcn_s_setprio(2);
    fetch(pages, plan, tile, codes, scales);
    if (2 * blockIdx.x >= gridDim.x) __builtin_amdgcn_s_setprio(1);
    else __builtin_amdgcn_s_setprio(0);
  }
  __device__ void begin(const Plan<kPer>& plan, uint32_t tile) {
    fetch(k_pages, plan, tile, k, ks);
    fetch(v_pages, plan, tile, v, vs);
  }
  template <typename Next>
  __device__ void work(Plan<kPer>& plan, uint32_t tile, bool more, Next next, int key0, const uintx4 (&qf)[NT][4], Rows<NT>& r) {
    const int to0 = anew(to), v0 = anew(va);
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      floatx4 s[NT][2];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
#pragma unroll
        for (int m = 0; m < NT; ++m) s[m][y] = (floatx4){0.f, 0.f, 0.f, 0.f};
        const float scale = tkv::scale_of(ks[2 * z + y]);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          const uintx4 a = __builtin_bit_cast(uintx4, tkv::values_of<T>(k[2 * z + y][kk], scale));
#pragma unroll
          for (int m = 0; m < NT; ++m) s[m][y] = mfma16<T>(a, qf[m][kk], s[m][y]);
        }
      }
      if (z == 1 && more) {
        next();
        ahead(k_pages, plan, tile, k, ks);
      }
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const float scale = tkv::scale_of(vs[2 * z + y]);
#pragma unroll
        for (int i = 0; i < 4; ++i) lds_write16(area + (to0 ^ 16 * i) + 4096 * y, __builtin_bit_cast(uintx4, tkv::values_of<T>(v[2 * z + y][i], scale)));
      }
      uintx4 w[NT][1];
      weigh<T, NT, 2>(r, s, w, key0 + 32 * z);
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) {
        const uintx2 lo = lds_read_tr(area + (v0 ^ 32 * ct)), hi = lds_read_tr(area + (v0 ^ 32 * ct) + 4096);
        const uintx4 a = __builtin_shufflevector(lo, hi, 0, 1, 2, 3);
#pragma unroll
        for (int m = 0; m < NT; ++m) r.o[m][ct] = mfma16<T>(a, w[m][0], r.o[m][ct]);
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    }
    if (more) ahead(v_pages, plan, tile, v, vs);
  }
};

template <typename T, int BITS, int NT>
using Tiles = std::conditional_t<BITS == 16, Tiles16<T, NT>, Tiles4<T, NT>>;

// What is left to join by a workgroup whose waves work alone: of each wave, the items at its range's two ends, if it came last.
struct Won {
  int32_t count;
  Place at[2];
};

// Workgroups of a compute unit: 16 bits: what LDS has room for (rings of 128 KiB); 4 bits: registers.  LDS: the waves' rings or areas, the
// waves' results where they join, and what is left to join.
template <int BITS, int NT>
constexpr int workgroups_each() { return BITS == 16 ? 1 : 2; }
template <typename T, int BITS, int NT>
constexpr int lds_bytes() {
  return std::max(kWaves * Tiles<T, BITS, NT>::kBytes, kWaves * 16 * (kRowFloats + 2) * 4 + 16) + (int)sizeof(Won) * kWaves;
}

// Zeros, and -inf, for rows of no sequence: in front of the first, behind the last, and beyond the most that one may have.
template <typename T>
__device__ inline void clear_rows_of_no_sequence() {
  const Args p = arguments();
  const int front = min(max(p->q_starts[0], 0), p->n_tokens), back = min(max(p->q_starts[p->batch], front), p->n_tokens);
  const int none = front + p->n_tokens - back, row_places = p->hq * TKV_D / 8;
  auto clear = [&](int64_t token) {
    for (int c = threadIdx.x; c < row_places; c += 64 * kWaves) ((uintx4*)p->out)[token * row_places + c] = (uintx4){0u, 0u, 0u, 0u};
    for (int c = threadIdx.x; p->lse && c < p->hq; c += 64 * kWaves) p->lse[token * p->hq + c] = -INFINITY;
  };
  for (int i = blockIdx.x; i < none; i += gridDim.x) clear(i < front ? i : back + (i - front));
  for (int b = blockIdx.x; b < p->batch; b += gridDim.x) {
    const int start = min(max(p->q_starts[b], 0), p->n_tokens), end = min(max(p->q_starts[b + 1], 0), p->n_tokens);
    if (__builtin_expect(end - start > p->max_q_len, 0))
      for (int token = start + p->max_q_len; token < end; ++token) clear(token);
  }
}

// An item's parts: where a range's cut lies in it, its tiles are several waves', and their results (sum, reference, weighted sums) have to
// be joined.  They are left in the workspace, a counter says who comes last, and that workgroup joins them: no second launch (3.4 us and
// its way there: one token over 2048 keys 13.7 -> 9 us in all).  Nobody waits for anybody.  A workgroup whose whole range lies in one item
// joins its waves' results itself and has one part (slot 8 g); elsewhere every wave has its own: slot 2 w
// for one that begins with the wave's range, 2 w + 1 otherwise.
struct Parts {
  uint32_t start, pw;           // the item's first tile, tiles of a wave's range
  int32_t w0, g0, g1;           // first wave, first and last workgroup
  bool one0, one1;              // these have one part each
  int32_t head, middle, count;  // parts of the first workgroup, of those between, all

  __device__ Parts(const Place& x, uint32_t range, uint32_t total) : start(x.start), pw(range) {
    const uint32_t end = x.start + (uint32_t)x.sq.key_tiles;
    const int32_t w1 = (int32_t)((end - 1) / pw);
    w0 = (int32_t)(start / pw);
    g0 = w0 / kWaves;
    g1 = w1 / kWaves;
    one0 = within(g0, end, total);
    one1 = within(g1, end, total);
    head = one0 ? 1 : min(w1, kWaves * g0 + kWaves - 1) - w0 + 1;
    middle = max(0, g1 - g0 - 1);
    count = head + middle + (g1 == g0 ? 0 : one1 ? 1 : w1 - kWaves * g1 + 1);
  }
  __device__ bool within(int32_t g, uint32_t end, uint32_t total) const {  // the workgroup's range in the item
    const uint64_t a = (uint64_t)g * kWaves * pw;
    return start <= a && end >= min((uint64_t)total, a + (uint64_t)kWaves * pw);
  }
  __device__ int32_t slot(int32_t i) const {
    if (i < head) {
      const int32_t w = w0 + i;
      return one0 ? 2 * kWaves * g0 : 2 * w + (i == 0 && start > (uint32_t)w * pw ? 1 : 0);
    }
    if (i < head + middle) return 2 * kWaves * (g0 + 1 + i - head);
    return 2 * (kWaves * g1 + (one1 ? 0 : i - head - middle));
  }
};

// Parts cross workgroups through stores and loads that pass by the caches that are not coherent between them ("sc1").
template <int ROWS>
struct PartStore {
  __amdgpu_buffer_rsrc_t o, ml;
  __device__ explicit PartStore(Args p)
      : o(__builtin_amdgcn_make_buffer_rsrc(p->parts, 0, (int)((uint32_t)(2 * kWaves * p->workgroups) * (ROWS * TKV_D * 4u)), 0x00020000)),
        ml(__builtin_amdgcn_make_buffer_rsrc(p->ml, 0, (int)((uint32_t)(2 * kWaves * p->workgroups) * (ROWS * 8u)), 0x00020000)) {}
  __device__ void put(int slot, int row, int c, floatx4 x) const {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(uintx4, x), o, (uint32_t)((slot * ROWS + row) * TKV_D + c) * 4u, 0, 16);
  }
  __device__ void put(int slot, int row, float ref, float sum) const {
    const float2 x = make_float2(ref, sum);
    __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(uintx2, x), ml, (uint32_t)(slot * ROWS + row) * 8u, 0, 16);
  }
};

// The token of a row.  (Exact below 2^32 / group rows; 2^32 / 1 does not fit, and is given as 0.)
__device__ inline int32_t row_token(Args p, int32_t row) {
  const uint32_t m = p->per_group;
  return m == 0u ? row : (int32_t)__umulhi((uint32_t)row, m);
}
// Where a finished row of an item goes, and the logarithm of its sum.
__device__ inline int64_t row_out(Args p, const Place& x, int row) {
  const int group = p->group, token = row_token(p, row), head = row - token * group;
  return (int64_t)(x.sq.q_start + token) * p->hq + x.h * group + head;
}
__device__ inline float log_sum(float ref, float sum) {
  return ref == kNone ? -INFINITY : (ref - kShift + __builtin_amdgcn_logf(sum)) * 0.69314718055994531f;
}

// A wave joins an item's parts for some of its rows, a lane eight channels: row0, row0 + step, ..., each row's parts shared out over the
// wave's four sixteens of lanes (SHARES 4), or from each of these on four rows, a sixteen each (SHARES 1).  What is added up in which order
// depends on SHARES and the number of parts alone: the same bits, whoever comes last.
template <typename T, int ROWS, int SHARES>
__device__ inline void join_rows(Args p, const Place& x, const Parts& parts, int row0, int step) {
  constexpr int kAtOnce = SHARES == 4 ? 4 : 8;  // loads on their way, in rounds of SHARES parts
  const int lane = threadIdx.x % 64, share = SHARES == 4 ? lane / 16 : 0, sub = SHARES == 4 ? 0 : lane / 16, c = 8 * (lane % 16);
  const int rows = min(ROWS, x.sq.q_len * p->group - ROWS * x.tile), rounds = (parts.count + SHARES - 1) / SHARES;
  const tkv::AgentBuf ob(p->parts, (uint32_t)(2 * kWaves * p->workgroups) * (ROWS * TKV_D * 4u));
  const tkv::AgentBuf mb(p->ml, (uint32_t)(2 * kWaves * p->workgroups) * (ROWS * 8u));
  float m = kNone, l = 0.f;
  floatx8 acc = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  int row = row0, round = 0;
#pragma nounroll
  while (row < rows) {
    tkv::tkv_u32x2 st[kAtOnce];
    tkv::tkv_u32x4 lo[kAtOnce], hi[kAtOnce];
    int r = row, n = round;
#pragma unroll
    for (int y = 0; y < kAtOnce; ++y) {
      const int i = SHARES * n + share;
      const uint32_t at = (uint32_t)(parts.slot(min(i, parts.count - 1)) * ROWS + r + sub);
      const bool there = i < parts.count && r + sub < rows;  // (absent ones are zeros)
      st[y] = mb.x2(there ? at * 8u : tkv::AgentBuf::kNone);
      lo[y] = ob.x4(there ? (at * TKV_D + c) * 4u : tkv::AgentBuf::kNone);
      hi[y] = ob.x4(there ? (at * TKV_D + c) * 4u + 16u : tkv::AgentBuf::kNone);
      if (++n == rounds) n = 0, r += step;
    }
#pragma unroll
    for (int y = 0; y < kAtOnce; ++y) {
      if (row >= rows) break;
      const uint32_t ref_bits = st[y].x, sum_bits = st[y].y;
      const float ref = SHARES * round + share < parts.count ? __builtin_bit_cast(float, ref_bits) : kNone;
      const float top = fmaxf(m, ref), shrink = __builtin_amdgcn_exp2f(m - top), w = __builtin_amdgcn_exp2f(ref - top);
      m = top;
      l = __builtin_fmaf(__builtin_bit_cast(float, sum_bits), w, l * shrink);
      const floatx4 a = __builtin_bit_cast(floatx4, lo[y]), b = __builtin_bit_cast(floatx4, hi[y]);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        acc[k] = __builtin_fmaf(a[k], w, acc[k] * shrink);
        acc[4 + k] = __builtin_fmaf(b[k], w, acc[4 + k] * shrink);
      }
      if (++round < rounds) continue;
      // the row's last
      if constexpr (SHARES == 4) {
        auto add = [](float u, float v) { return u + v; };
        const float all = tkv::over_rows(m, [](float u, float v) { return fmaxf(u, v); }), mine = __builtin_amdgcn_exp2f(m - all);
        m = all;
        l = tkv::over_rows(l * mine, add);
#pragma unroll
        for (int k = 0; k < 8; ++k) acc[k] = tkv::over_rows(acc[k] * mine, add);
      }
      if (share == 0 && row + sub < rows) {
        const int64_t to = row_out(p, x, ROWS * x.tile + row + sub);
        *(uintx4*)((T*)p->out + to * TKV_D + c) = pack8<T>(acc * (1.f / l));
        if (p->lse && c == 0) p->lse[to] = log_sum(m, l);
      }
      m = kNone;
      l = 0.f;
      acc = (floatx8){0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      round = 0;
      row += step;
    }
  }
}

template <typename T, int BITS, int NT>
__global__ __launch_bounds__(64 * kWaves, 2) void paged_attn_kernel(PagedParams) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  typedef Tiles<T, BITS, NT> Tile;
  constexpr int kRows = 16 * NT;
  const int lane = threadIdx.x % 64, col = lane % 16, quarter = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  tkv::fetch_arguments<sizeof(PagedParams)>();
  Walk<Tile::kKeys, kRows> walk;
  const uint32_t total = walk.total(), pw = range_of(total, walk.longest, arguments()->workgroups);
  if (arguments()->clear_rest) clear_rows_of_no_sequence<T>();
  const uint64_t group_begin = (uint64_t)blockIdx.x * kWaves * pw;
  if (group_begin >= total) return;
  const uint64_t begin64 = group_begin + (uint64_t)wave * pw;
  uint32_t begin = (uint32_t)min((uint64_t)total, begin64), end = (uint32_t)min((uint64_t)total, begin64 + pw);

  Place x = walk.find(begin < end ? begin : (uint32_t)group_begin);
  // Whether the workgroup's whole range lies in one item (all its waves find the same): then they take its tiles in turn, and join before
  // they hand on.
  const bool together = x.start <= (uint32_t)group_begin &&
                        (uint64_t)x.start + (uint32_t)x.sq.key_tiles >= min((uint64_t)total, group_begin + (uint64_t)kWaves * pw);

  Rows<NT> r;
  uintx4 qf[NT][4];
  auto open = [&](const Place& at) {  // an item's rows, and where their keys end
    const Args p = arguments();
    const int rows = at.sq.q_len * walk.group;
#pragma unroll
    for (int m = 0; m < NT; ++m) {
      const T* const q = (const T*)p->q + row_out(p, at, min(at.tile * kRows + 16 * m + col, rows - 1)) * TKV_D;
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) qf[m][kk] = *(const uintx4*)(q + Tile::q_channel(kk));
    }
  };
  auto reset = [&](const Place& at) {
    const int rows = at.sq.q_len * walk.group, ahead = at.sq.k_len - at.sq.q_len;
    r.scale2 = arguments()->scale2;
    const Args p = arguments();
    r.limit_low = row_token(p, at.tile * kRows) + ahead;
#pragma unroll
    for (int m = 0; m < NT; ++m) {
      const int row = min(at.tile * kRows + 16 * m + col, rows - 1);
      r.limit[m] = row_token(p, row) + ahead;
      r.ref[m] = kNone;
      r.sum[m] = r.limit[m] < 0 ? 1.f : 0.f;  // (no key: 0 / 1, zeros; logits of -inf alone: 0 / 0)
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) r.o[m][ct] = (floatx4){0.f, 0.f, 0.f, 0.f};
    }
    // (The rows are waited for here: the compiler, which does not know of the loads to LDS, would wait for them and those inside
    // the loop.)
#pragma unroll
    for (int m = 0; m < NT; ++m)
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) asm volatile("" : "+v"(qf[m][kk]));
  };
  if (together) {
    begin = (uint32_t)min((uint64_t)total, group_begin + (uint64_t)wave);
    end = (uint32_t)min((uint64_t)total, group_begin + (uint64_t)kWaves * pw);
  }
  Won* const won = (Won*)(lds + lds_bytes<T, BITS, NT>()) - kWaves;
  int wins = 0;
  Tile tiles((lds_char*)lds + wave * Tile::kBytes);
  Plan<Tile::kPer> plan;
  plan.log_step = together ? 2 : 0;
  static_assert(kWaves == 4, "log_step");
  const uint32_t step = 1u << plan.log_step;
  if (begin < end || together) open(x);
  if (begin < end) {
    plan.make(walk, begin, end);
    tiles.begin(plan, begin);
  }
  if (begin < end || together) reset(x);
  for (uint32_t at = begin; begin < end || together;) {
    const uint32_t stop = min(end, x.start + (uint32_t)x.sq.key_tiles);
    const bool begins = at == begin;
    for (; at < stop; at += step)
      tiles.work(plan, at + step, at + step < end, [&] { if (__builtin_expect(!plan.has(at + step), 0)) plan.make(walk, at + step, end); },
                 Tile::kKeys * (int)(at - x.start), qf, r);
    const Place done = x;
    const bool last = together || at >= end;
    if (!last) {  // the next item's rows are on their way while this one's results leave
      x = walk.find(at);
      open(x);
    }
    const Args p = arguments();
    const Parts parts(done, pw, total);
    const PartStore<kRows> store(p);
    const int rows = done.sq.q_len * walk.group;
    if (!together) {
      const int slot = 2 * (kWaves * (int)blockIdx.x + wave) + (begins ? 0 : 1);
#pragma unroll
      for (int m = 0; m < NT; ++m) {
        const float sum = tkv::over_rows(r.sum[m], [](float a, float b) { return a + b; });
        const int row = done.tile * kRows + 16 * m + col;
        if (row >= rows) continue;
        if (parts.count == 1) {
          typedef T T4 __attribute__((ext_vector_type(4)));
          const int64_t to = row_out(p, done, row);
          const float inv = 1.f / sum;
#pragma unroll
          for (int ct = 0; ct < 8; ++ct) *(T4*)((T*)p->out + to * TKV_D + 16 * ct + 4 * quarter) = __builtin_convertvector(r.o[m][ct] * inv, T4);
          if (p->lse && quarter == 0) p->lse[to] = log_sum(r.ref[m], sum);
        } else {
#pragma unroll
          for (int ct = 0; ct < 8; ++ct) store.put(slot, 16 * m + col, 16 * ct + 4 * quarter, r.o[m][ct]);
          if (quarter == 0) store.put(slot, 16 * m + col, r.ref[m], sum);
        }
      }
      if (parts.count > 1) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the part is in memory before the count goes up
        uint32_t before = 0;
        if (lane == 0) before = atomicAdd(p->arrivals + parts.w0, 1u);
        if ((uint32_t)__builtin_amdgcn_readfirstlane((int)before) == (uint32_t)parts.count - 1u) {
          if (lane == 0) won[wave].at[wins] = done;
          ++wins;
        }
      }
    } else {
      // the waves join, sixteen rows at a time: everyone's results into LDS, then sixteen threads a row
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // no load may land after the ring is used otherwise
      float* const o_s = (float*)lds;                      // [wave][row][kRowFloats]
      float* const ml_s = o_s + kWaves * 16 * kRowFloats;  // [wave][row][2]
#pragma unroll
      for (int m = 0; m < NT; ++m) {
        const float part = tkv::over_rows(r.sum[m], [](float a, float b) { return a + b; });
        __syncthreads();
#pragma unroll
        for (int ct = 0; ct < 8; ++ct) *(floatx4*)(o_s + (16 * wave + col) * kRowFloats + 16 * ct + 4 * quarter) = r.o[m][ct];
        if (quarter == 0) *(float2*)(ml_s + 2 * (16 * wave + col)) = make_float2(r.ref[m], part);
        __syncthreads();
        const int at_row = threadIdx.x / 16, in_tile = 16 * m + at_row, row = done.tile * kRows + in_tile, c = 8 * (threadIdx.x % 16);
        if (row >= rows) continue;
        float f[kWaves], top = kNone, sum = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, f[w] = ml_s[2 * (16 * w + at_row)]);
        floatx8 acc = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          f[w] = __builtin_amdgcn_exp2f(f[w] - top);
          sum = __builtin_fmaf(ml_s[2 * (16 * w + at_row) + 1], f[w], sum);
          const float* const from = o_s + (16 * w + at_row) * kRowFloats + c;
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[i] = __builtin_fmaf(from[i], f[w], acc[i]);
        }
        if (parts.count > 1) {
          const int slot = 2 * kWaves * (int)blockIdx.x;
          store.put(slot, in_tile, c, __builtin_shufflevector(acc, acc, 0, 1, 2, 3));
          store.put(slot, in_tile, c + 4, __builtin_shufflevector(acc, acc, 4, 5, 6, 7));
          if (c == 0) store.put(slot, in_tile, top, sum);
          continue;
        }
        const int64_t to = row_out(p, done, row);
        *(uintx4*)((T*)p->out + to * TKV_D + c) = pack8<T>(acc * (1.f / sum));
        if (p->lse && c == 0) p->lse[to] = log_sum(top, sum);
      }
      if (parts.count > 1) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the part is in memory before the count goes up
        __syncthreads();
        uint32_t* const flag = (uint32_t*)(ml_s + 2 * kWaves * 16);
        if (threadIdx.x == 0) *flag = atomicAdd(p->arrivals + parts.w0, 1u);
        __syncthreads();
        wins = *flag == (uint32_t)parts.count - 1u ? 1 : 0;
      }
    }
    if (last) break;
    reset(x);
  }
  uint32_t left = (uint32_t)__builtin_amdgcn_readfirstlane(wins);
  if (!together) {  // all waves take part in what any of them has won: bit 2 w + i
    if (lane == 0) won[wave].count = wins;
    __syncthreads();
    left = (uint32_t)__builtin_amdgcn_ballot_w64(lane < 2 * kWaves && lane % 2 < won[lane / 2 % kWaves].count);
  }
  // Several items go to waves of their own, as many as each has work for (64 sequences of up to 300 tokens 19.1 -> 17.0 us).
  for (int next = 0; left != 0; left &= left - 1) {
    Place at = x;
    static_assert(sizeof(Place) % 4 == 0, "words");
    const int i = __builtin_ctz(left);
    if (!together) {
#pragma unroll
      for (int k = 0; k < (int)sizeof(Place) / 4; ++k) ((int32_t*)&at)[k] = __builtin_amdgcn_readfirstlane(((const int32_t*)&won[i / 2].at[i % 2])[k]);
    }
    const Args p = arguments();
    const Parts parts(at, pw, total);
    if (threadIdx.x == 0) __hip_atomic_store(p->arrivals + parts.w0, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const int rows = at.sq.q_len * walk.group - kRows * at.tile;
    const bool shared = rows <= 4 || (rows <= 8 && parts.count > 8);
    const int team = shared ? (together || rows > 4 || parts.count > 8 ? kWaves : parts.count > 4 ? 2 : 1) : rows <= 8 ? 2 : kWaves;
    const int first = team == 1 ? next % kWaves : team == 2 ? (next + 1) & 2 : 0;
    next = first + team;
    const int mine = wave - first;
    if (mine < 0 || mine >= team) continue;
    if (shared) join_rows<T, kRows, 4>(p, at, parts, mine, team);
    else join_rows<T, kRows, 1>(p, at, parts, 4 * mine, 4 * team);
  }
}

// Room for the parts: two of every wave.
constexpr size_t kPartRows = (size_t)2 * kWaves * kMaxUnits * 64;
static_assert(48 * workgroups_each<16, 3>() <= 64 && 32 * workgroups_each<4, 2>() <= 64 && 16 * workgroups_each<4, 1>() <= 64, "workspace");
static_assert(4 * kWaves * kMaxUnits * workgroups_each<4, 1>() <= TKV_PAGED_COUNTERS, "workspace");
constexpr size_t kWorkspace = kPartRows * (TKV_D + 2) * sizeof(float) + TKV_PAGED_COUNTERS;

template <typename T, int BITS, int NT>
int32_t launch_attn(PagedParams& p, int units, hipStream_t s) {
  constexpr int lds = lds_bytes<T, BITS, NT>();
  static_assert(lds * workgroups_each<BITS, NT>() <= 160 * 1024, "LDS of one compute unit");
  static const bool lds_ok = hipFuncSetAttribute(reinterpret_cast<const void*>(&paged_attn_kernel<T, BITS, NT>),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, lds) == hipSuccess;
  if (!lds_ok) return TKV_E_HIP;
  p.workgroups = std::min(kMaxUnits, units) * workgroups_each<BITS, NT>();
  TKV_LAUNCH((paged_attn_kernel<T, BITS, NT>), dim3((uint32_t)p.workgroups), 64 * kWaves, lds, s, p);
  return TKV_OK;
}

template <typename T, int BITS>
int32_t launch_rows(PagedParams& p, int64_t rows, int units, hipStream_t s) {
  // Tiles of 16, 32 or (16 bits) 48 rows: what a wave's registers have room for, as few tiles as go, as small as go.
  constexpr int kMost = BITS == 16 ? 3 : 2;
  const int64_t sixteens = (rows + 15) / 16, tiles = (sixteens + kMost - 1) / kMost, each = (sixteens + tiles - 1) / tiles;
  if (each == 1) return launch_attn<T, BITS, 1>(p, units, s);
  if constexpr (BITS == 16)
    if (each == 3) return launch_attn<T, BITS, 3>(p, units, s);
  return launch_attn<T, BITS, 2>(p, units, s);
}

// Whether rows of 128 elements at p s[0] + h s[1] + t s[2] do not overlap, each axis beyond all that smaller strides span, and end below
// 2^62.
bool rows_apart(const int64_t* s, const int64_t (&count)[3]) {
  int order[3] = {0, 1, 2};
  std::sort(order, order + 3, [&](int a, int b) { return s[a] < s[b]; });
  int64_t span = TKV_D;
  for (int i : order) {
    if (count[i] > 1 && (s[i] < span || s[i] > ((int64_t)1 << 60) / count[i])) return false;
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
  const int each = d->bits == 16 ? 16 : 32;  // tokens of a wave
  const int64_t waves = ((int64_t)n_tokens + each - 1) / each * 2 * d->n_kv_heads;
  if (waves > 4 * ((1 << 24) - 1)) return TKV_E_UNSUPPORTED;  // (a launch has fewer than 2^32 threads)
  p.slots = slots;
  p.k_out = k_out;
  p.v_out = v_out;
  p.n_tokens = n_tokens;
  p.waves = (int32_t)waves;
  const dim3 grid((uint32_t)((waves + 3) / 4));
  const auto s = (hipStream_t)stream;
  if (d->bits == 16) TKV_LAUNCH((paged_gather_kernel<_Float16, 16, 4>), grid, 256, 0, s, p);
  else if (d->dtype == TKV_F16) TKV_LAUNCH((paged_gather_kernel<_Float16, 4, 8>), grid, 256, 0, s, p);
  else TKV_LAUNCH((paged_gather_kernel<__bf16, 4, 8>), grid, 256, 0, s, p);
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
                                  int32_t pages_each, const int32_t* k_lens, const int32_t* q_starts, int32_t clear_rest, float sm_scale,
                                  void* workspace, size_t workspace_bytes, void* stream) {
  int32_t st = tkv::check_paged_desc(d);
  if (st != TKV_OK) return st;
  if (batch < 0 || n_tokens < 0 || max_q_len <= 0 || pages_each < 0 || !workspace) return TKV_E_INVAL;
  if (clear_rest != 0 && clear_rest != 1) return TKV_E_INVAL;
  const float scale2 = sm_scale * 1.4426950408889634f;
  if (!(sm_scale > 0.f) || !(scale2 <= 3.402823466e38f)) return TKV_E_INVAL;
  if (!q_starts && (n_tokens != batch || max_q_len != 1)) return TKV_E_INVAL;
  if ((int64_t)pages_each * d->page_size > (1 << 30)) return TKV_E_UNSUPPORTED;
  // Numbers of tiles are 32 bits, whatever the device's arrays hold: tiles of 16 rows and 32 keys, the smallest.
  const int64_t group = d->n_q_heads / d->n_kv_heads;
  max_q_len = std::min(max_q_len, std::max(n_tokens, 1));
  if (max_q_len * group > (1 << 24) || max_q_len * group * group >= ((int64_t)1 << 32)) return TKV_E_UNSUPPORTED;
  const int64_t row_tiles = batch * ((max_q_len * group + 15) / 16) * d->n_kv_heads, key_tiles = (((int64_t)pages_each * d->page_size) >> 5) + 1;
  if (row_tiles >= ((int64_t)1 << 31) || row_tiles * key_tiles >= ((int64_t)1 << 31)) return TKV_E_UNSUPPORTED;
  if (workspace_bytes < kWorkspace) return TKV_E_WORKSPACE;
  if (n_tokens == 0 || (batch == 0 && !(q_starts && clear_rest))) return TKV_OK;
  if (!q || !out || (batch && !k_lens) || (batch && pages_each && !page_table)) return TKV_E_INVAL;
  for (const void* x : {q, (const void*)out, (const void*)workspace})
    if (((uintptr_t)x & 15) != 0) return TKV_E_INVAL;
  for (const void* x : {(const void*)lse, (const void*)page_table, (const void*)k_lens, (const void*)q_starts})
    if (((uintptr_t)x & 3) != 0) return TKV_E_INVAL;
  PagedParams p;
  st = tkv::paged_view(d, const_cast<void*>(k_pages), const_cast<void*>(v_pages), &p.pages);
  if (st != TKV_OK) return st;
  p.q = q; p.out = out; p.lse = lse;
  p.table = page_table; p.k_lens = k_lens; p.q_starts = q_starts;
  p.n_tokens = n_tokens; p.batch = batch; p.max_q_len = max_q_len; p.pages_each = pages_each;
  p.hq = d->n_q_heads;
  p.group = (int32_t)group;
  p.per_group = group == 1 ? 0u : (uint32_t)((((uint64_t)1 << 32) + group - 1) / group);
  p.scale2 = scale2;
  p.parts = (float*)workspace;
  p.ml = p.parts + kPartRows * TKV_D;
  p.arrivals = (uint32_t*)(p.ml + kPartRows * 2);
  p.clear_rest = q_starts && clear_rest;
  const int64_t rows = (int64_t)max_q_len * p.group;
  const auto s = (hipStream_t)stream;
  const int units = tkv::stream_compute_units(s);
  if (d->dtype == TKV_F16) return d->bits == 16 ? launch_rows<_Float16, 16>(p, rows, units, s) : launch_rows<_Float16, 4>(p, rows, units, s);
  return d->bits == 16 ? launch_rows<__bf16, 16>(p, rows, units, s) : launch_rows<__bf16, 4>(p, rows, units, s);
}
