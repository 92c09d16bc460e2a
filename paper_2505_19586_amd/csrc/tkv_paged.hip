// Paged caches: rows read back from their pages (tkv_paged_gather) and attention over them (tkv_paged_attn).
#include <algorithm>

#include "tkv_paged.h"

namespace {

typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));

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

struct PagedParams {
  tkv::Pages pages;
  const void* q;
  void* out;
  float* lse;  // NULL: not wanted
  const int32_t* table;
  const int32_t* k_lens;
  const int32_t* q_starts;  // NULL: a token of each sequence
  int32_t n_tokens, batch, hq, group, pages_each;
  float scale2;  // sm_scale * log2(e)
};

// One wave per row of q, a lane two channels, one key after the other.
template <typename T, int BITS>
__global__ __launch_bounds__(256) void paged_attn_plain_kernel(PagedParams p) {
  const int lane = threadIdx.x % 64;
  const int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  if (item >= (int64_t)p.n_tokens * p.hq) return;
  const int token = (int)(item / p.hq), head = (int)(item % p.hq), h = head / p.group;
  int b = token, i = 0, n_q = 1;
  if (p.q_starts) {
    for (b = 0; b < p.batch && !(p.q_starts[b] <= token && token < p.q_starts[b + 1]); ++b) {}
    if (b == p.batch) return;
    i = token - p.q_starts[b];
    n_q = p.q_starts[b + 1] - p.q_starts[b];
  }
  const int page_tokens = 1 << p.pages.shift;
  const int k_len = (int)max((int64_t)0, min((int64_t)p.k_lens[b], (int64_t)p.pages_each * page_tokens));
  const int seen = max(0, k_len - n_q + i + 1);
  const T* const q = (const T*)p.q + item * TKV_D + 2 * lane;
  const float q0 = (float)q[0], q1 = (float)q[1];
  float top = -INFINITY, sum = 0.f, o0 = 0.f, o1 = 0.f;
  for (int key = 0; key < seen; ++key) {
    const int64_t page = p.table[(int64_t)b * p.pages_each + (key >> p.pages.shift)], at = key & (page_tokens - 1);
    float x[4] = {0.f, 0.f, 0.f, 0.f};
    if (page >= 0 && page < p.pages.n_pages) {
      for (int w = 0; w < 2; ++w) {
        const int64_t sp = w ? p.pages.v_sp : p.pages.k_sp, sh = w ? p.pages.v_sh : p.pages.k_sh, st = w ? p.pages.v_st : p.pages.k_st;
        const char* const base = (const char*)(w ? p.pages.v : p.pages.k);
        if constexpr (BITS == 16) {
          const T* const row = (const T*)base + (page * sp + h * sh + at * st) + 2 * lane;
          x[2 * w] = (float)row[0];
          x[2 * w + 1] = (float)row[1];
        } else {
          const char* const block = base + page * sp + h * sh;
          const uint32_t code = *(const uint8_t*)(block + at * tkv::kRow4 + lane);
          const uint32_t scale = *(const uint8_t*)(block + ((int64_t)tkv::kRow4 << p.pages.shift) + at * tkv::kScales4 + lane / 16);
          const floatx2 y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, tkv::scale_of(scale), 0);
          x[2 * w] = y[0];
          x[2 * w + 1] = y[1];
        }
      }
    }
    const float s = tkv::over_wave(q0 * x[0] + q1 * x[1], [](float a, float c) { return a + c; }) * p.scale2;
    const float next = fmaxf(top, s), shrink = __builtin_amdgcn_exp2f(top - next), w = __builtin_amdgcn_exp2f(s - next);
    sum = sum * shrink + w;
    o0 = o0 * shrink + w * x[2];
    o1 = o1 * shrink + w * x[3];
    top = next;
  }
  const float inv = seen == 0 ? 0.f : 1.f / sum;
  T* const to = (T*)p.out + item * TKV_D + 2 * lane;
  to[0] = (T)(o0 * inv);
  to[1] = (T)(o1 * inv);
  if (p.lse && lane == 0) p.lse[item] = seen == 0 ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.69314718055994531f;
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
  *workspace_bytes = 16;
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
  if (workspace_bytes < 16) return TKV_E_WORKSPACE;
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
  const int64_t waves = (int64_t)n_tokens * d->n_q_heads;
  if (waves > 4 * ((1 << 24) - 1)) return TKV_E_UNSUPPORTED;
  const dim3 grid((uint32_t)((waves + 3) / 4));
  const auto s = (hipStream_t)stream;
  if (d->dtype == TKV_F16 && d->bits == 16) TKV_LAUNCH((paged_attn_plain_kernel<_Float16, 16>), grid, 256, 0, s, p);
  else if (d->dtype == TKV_F16) TKV_LAUNCH((paged_attn_plain_kernel<_Float16, 4>), grid, 256, 0, s, p);
  else if (d->bits == 16) TKV_LAUNCH((paged_attn_plain_kernel<__bf16, 16>), grid, 256, 0, s, p);
  else TKV_LAUNCH((paged_attn_plain_kernel<__bf16, 4>), grid, 256, 0, s, p);
  return TKV_OK;
}
