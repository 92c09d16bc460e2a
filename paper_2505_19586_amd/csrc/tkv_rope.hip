// Norm of queries and keys per head with the position rotation in the same pass, values laid out
// beside them (tkv_qk_norm_rope, with positions of several axes tkv_qk_norm_rope_axes) or keys and values put into the pages
// of a cache (tkv_paged_append).
//
//   y_c = x_c w_c / sqrt(mean_c x_c^2 + eps);  pairs (a, b) of the first R channels turn by pos f_i:
//   a cos - b sin, b cos + a sin.
//
// Every element is read once and written once: the memory's rate bounds long prompts (32768 tokens of 48 heads: 136 us, 5.9 TB/s, half
// of the input still in the last-level cache; a large copy reaches 5.1), the latency of one round trip a few tokens (16: 3.3 us).  Eight
// lanes take a row (a head of a token), sixteen channels each, chosen so
// that both channels of every pair lie in one lane: nothing is exchanged but the row's sum of squares.  A token's
// angles are worked out once per wave, one frequency per lane, and handed round.
//
// Several axes cost nothing: the axis of a lane's frequency is two bits of two masks (24640 tokens, three axes: 103 us, 5.9 TB/s).  Into pages
// a row goes straight from its registers (12289 tokens, 16 bits: 54 us, 5.5 TB/s; 32 tokens: 3.9 us), in 4 bits by way of its blocks' largest
// magnitudes, three exchanges over the row's eight lanes each (8191 tokens: 35 us, 5.1 TB/s).
#include <type_traits>

#include "tkv_common.h"
#include "tkv_paged.h"

namespace {

typedef float floatx8 __attribute__((ext_vector_type(8)));

struct RopeParams {
  const void* q;
  const void* k;
  const void* v;  // NULL: none
  void* q_out;
  void* k_out;
  void* v_out;
  const int32_t* positions;
  const float* inv_freq;
  const void* q_weight;  // NULL: ones
  const void* k_weight;
  int64_t q_st, q_sh, k_st, k_sh, v_st, v_sh;  // strides of tokens and heads in elements
  int32_t hq, hkv, n_tokens;
  int32_t rows;      // rows of a token: hq + hkv (+ hkv)
  int32_t per_wave;  // octets of rows that a wave takes
  int32_t parts;     // waves per token
  int32_t pairs8;    // R / 16
  int32_t interleaved, norm;
  float eps;
  uint64_t axis[2];  // bit i of the two: the axis of frequency i, 0 to 3
  // appending only
  const int32_t* slots;
  tkv::Pages pages;
  int32_t lowest;  // smallest exponent of a 4-bit block
};

// Where a row of keys or values goes.
enum RopeDest { kToRows, kToPages16, kToPages4 };

// A row's eight lanes, sixteen numbers each, as 4-bit blocks: block u's exponent is that of its largest magnitude less 2 (so that
// the largest code, 6, is in its reach) and `lowest` at least; codes are rounded to nearest, ties to even, 6 at most.  A block that holds
// an infinity or NaN stands for NaN.
template <typename Out, typename OutV>
__device__ inline void store_blocks(OutV a, OutV b, int ca, int cb, int place, int lowest, char* codes, char* scales) {
  auto top = [](OutV v) {  // as integers infinities and NaN are the largest
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __builtin_bit_cast(uint32_t, (float)v[i]) & 0x7FFFFFFFu);
    return m;
  };
  auto other = [](uint32_t v, auto ctrl) { return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, 0xF, 0xF, true)); };
  const uint32_t ta = top(a), tb = top(b);
  uint32_t word = 0;  // the row's four scales
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    uint32_t m = max(ca / 32 == u ? ta : 0u, cb / 32 == u ? tb : 0u);
    m = other(m, std::integral_constant<int, 0xB1>{});
    m = other(m, std::integral_constant<int, 0x4E>{});
    m = other(m, std::integral_constant<int, 0x141>{});
    word |= (m >= 0x7F800000u ? 255u : (uint32_t)(max((int)(m >> 23) - 129, lowest) + 127)) << (8 * u);
  }
  auto store = [&](OutV v, int c) {
    const uint32_t byte = (word >> (8 * (c / 32))) & 255u;
    const float scale = __builtin_bit_cast(float, byte << 23);
    uint32_t w = 0;
    if constexpr (__is_same(Out, _Float16)) {
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_shufflevector(v, v, 0, 1), scale, 0);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_shufflevector(v, v, 2, 3), scale, 1);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_shufflevector(v, v, 4, 5), scale, 2);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_shufflevector(v, v, 6, 7), scale, 3);
    } else {
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_shufflevector(v, v, 0, 1), scale, 0);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_shufflevector(v, v, 2, 3), scale, 1);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_shufflevector(v, v, 4, 5), scale, 2);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_shufflevector(v, v, 6, 7), scale, 3);
    }
    *(uint32_t*)(codes + c / 2) = byte == 255u ? 0u : w;
  };
  store(a, ca);
  store(b, cb);
  if (place == 0) *(uint32_t*)scales = word;
}

template <typename T>
struct Vec8 {
  typedef T type __attribute__((ext_vector_type(8)));
};

template <typename In, typename Out, RopeDest DEST>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(RopeParams p) {
  typedef typename Vec8<In>::type InV;
  typedef typename Vec8<Out>::type OutV;
  const int lane = threadIdx.x % 64;
  const uint32_t item = (uint32_t)__builtin_amdgcn_readfirstlane(blockIdx.x * 4 + threadIdx.x / 64);
  const int32_t token = (int32_t)(item / (uint32_t)p.parts), part = (int32_t)(item % (uint32_t)p.parts);
  if (token >= p.n_tokens) return;
  const int place = lane % 8, sub = lane / 8;
  // the lane's two runs of eight channels: both channels of eight pairs, or 16 channels that do not turn
  const bool turns = place < p.pairs8;
  const bool halves = !p.interleaved && turns;
  const int ca = 8 * (halves ? place : 2 * place), cb = 8 * (halves ? p.pairs8 + place : 2 * place + 1);

  auto row_of = [&](int row, const In*& src, Out*& dst) {
    if (row < p.hq) {
      src = (const In*)p.q + (token * p.q_st + row * p.q_sh);
      dst = (Out*)p.q_out + ((int64_t)token * p.hq + row) * TKV_D;
    } else if (row < p.hq + p.hkv) {
      const int h = row - p.hq;
      src = (const In*)p.k + (token * p.k_st + h * p.k_sh);
      dst = DEST == kToRows || p.k_out ? (Out*)p.k_out + ((int64_t)token * p.hkv + h) * TKV_D : nullptr;
    } else {
      const int h = row - p.hq - p.hkv;
      src = (const In*)p.v + (token * p.v_st + h * p.v_sh);
      dst = DEST == kToRows ? (Out*)p.v_out + ((int64_t)token * p.hkv + h) * TKV_D : nullptr;
    }
  };
  // (a slot outside the pages is none)
  int32_t slot = -1;
  if constexpr (DEST != kToRows) {
    slot = __builtin_amdgcn_readfirstlane(p.slots[token]);
    if (slot >> p.pages.shift >= p.pages.n_pages) slot = -1;
  }
  const int g0 = part * p.per_wave, g1 = min((p.rows + 7) / 8, g0 + p.per_wave);
  const In* src;
  Out* dst;
  InV a, b;
  int row = 8 * g0 + sub;
  if (row < p.rows) {
    row_of(row, src, dst);
    a = *(const InV*)(src + ca);
    b = *(const InV*)(src + cb);
  }
  InV qwa, qwb, kwa, kwb;
#pragma unroll
  for (int i = 0; i < 8; ++i) qwa[i] = qwb[i] = kwa[i] = kwb[i] = (In)1.f;
  if (p.q_weight) {
    qwa = *(const InV*)((const In*)p.q_weight + ca);
    qwb = *(const InV*)((const In*)p.q_weight + cb);
  }
  if (p.k_weight) {
    kwa = *(const InV*)((const In*)p.k_weight + ca);
    kwb = *(const InV*)((const In*)p.k_weight + cb);
  }
  floatx8 cs, sn;
  {
    // The angle in turns, in 64 bits: rounded to 32, position 131071 would be off by 4e-3 rad.
    float s = 0.f, c = 1.f;
    if (lane < 8 * p.pairs8) {
      const int axis = (int)(p.axis[0] >> lane & 1) + 2 * (int)(p.axis[1] >> lane & 1);
      const double t = (double)p.positions[(int64_t)axis * p.n_tokens + token] * (double)p.inv_freq[lane] * 0.15915494309189533577;
      sincospif((float)(2.0 * (t - __builtin_rint(t))), &s, &c);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      cs[i] = __shfl(c, 8 * place + i, 64);
      sn[i] = __shfl(s, 8 * place + i, 64);
    }
  }
  for (int g = g0; g < g1; ++g) {
    const InV ra = a, rb = b;
    Out* const to = dst;
    const int mine = row;
    row += 8;
    if (g + 1 < g1 && row < p.rows) {  // the next rows are on their way while these are worked on
      row_of(row, src, dst);
      a = *(const InV*)(src + ca);
      b = *(const InV*)(src + cb);
    }
    if (mine >= p.rows) continue;
    floatx8 x = __builtin_convertvector(ra, floatx8), y = __builtin_convertvector(rb, floatx8);
    if (mine < p.hq + p.hkv) {
      if (p.norm) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(x[i], x[i], __builtin_fmaf(y[i], y[i], ss));
        ss += tkv::dpp<0xB1>(ss);   // the other seven lanes of the row
        ss += tkv::dpp<0x4E>(ss);
        ss += tkv::dpp<0x141>(ss);
        const float r = 1.0f / __builtin_sqrtf(ss * (1.0f / TKV_D) + p.eps);
        const bool is_q = mine < p.hq;
        x *= r * __builtin_convertvector(is_q ? qwa : kwa, floatx8);
        y *= r * __builtin_convertvector(is_q ? qwb : kwb, floatx8);
      }
      if (turns) {
        // (which of the two products is rounded is written out, so that every variant of the kernel gives the same bits)
        auto turn = [](float& u, float& w, float c, float s) {
          const float u0 = u, w0 = w;
          u = __builtin_fmaf(u0, c, -(w0 * s));
          w = __builtin_fmaf(u0, s, w0 * c);
        };
        if (p.interleaved) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float x0 = x[2 * i], x1 = x[2 * i + 1], y0 = y[2 * i], y1 = y[2 * i + 1];
            turn(x0, x1, cs[i], sn[i]);
            turn(y0, y1, cs[4 + i], sn[4 + i]);
            x[2 * i] = x0, x[2 * i + 1] = x1, y[2 * i] = y0, y[2 * i + 1] = y1;
          }
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            float u = x[i], w = y[i];
            turn(u, w, cs[i], sn[i]);
            x[i] = u, y[i] = w;
          }
        }
      }
    }
    const OutV oa = __builtin_convertvector(x, OutV), ob = __builtin_convertvector(y, OutV);
    if (DEST == kToRows || to) {
      *(OutV*)(to + ca) = oa;
      *(OutV*)(to + cb) = ob;
    }
    if constexpr (DEST != kToRows) {
      if (mine >= p.hq && slot >= 0) {
        const bool is_v = mine >= p.hq + p.hkv;
        const int64_t h = mine - p.hq - (is_v ? p.hkv : 0);
        const int64_t page = slot >> p.pages.shift, at = slot & ((1 << p.pages.shift) - 1);
        const int64_t sp = is_v ? p.pages.v_sp : p.pages.k_sp, sh = is_v ? p.pages.v_sh : p.pages.k_sh, st = is_v ? p.pages.v_st : p.pages.k_st;
        char* const base = (char*)(is_v ? p.pages.v : p.pages.k);
        if constexpr (DEST == kToPages16) {
          Out* const row16 = (Out*)base + (page * sp + h * sh + at * st);
          *(OutV*)(row16 + ca) = oa;
          *(OutV*)(row16 + cb) = ob;
        } else {
          char* const block = base + (page * sp + h * sh);
          store_blocks<Out>(oa, ob, ca, cb, place, p.lowest, block + at * tkv::kRow4,
                            block + ((int64_t)tkv::kRow4 << p.pages.shift) + at * tkv::kScales4);
        }
      }
    }
  }
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
bool dense_rows(const int64_t* s) { return s[0] >= 0 && s[1] >= 0 && s[0] % 8 == 0 && s[1] % 8 == 0; }

template <typename In, typename Out>
int32_t launch_rope(const RopeParams& p, int bits, hipStream_t s) {
  const int64_t items = (int64_t)p.n_tokens * p.parts;
  const dim3 grid((uint32_t)((items + 3) / 4));
  if (bits == 0) TKV_LAUNCH((qk_norm_rope_kernel<In, Out, kToRows>), grid, 256, 0, s, p);
  else if (bits == 16) TKV_LAUNCH((qk_norm_rope_kernel<In, Out, kToPages16>), grid, 256, 0, s, p);
  else TKV_LAUNCH((qk_norm_rope_kernel<In, Out, kToPages4>), grid, 256, 0, s, p);
  return TKV_OK;
}

int32_t check_rope_desc(const tkv_rope_desc* d, int32_t n_tokens, const uint8_t* axis_of, int32_t n_axes, const void* q_weight,
                        const void* k_weight) {
  if (!d || d->struct_size != sizeof(tkv_rope_desc)) return TKV_E_INVAL;
  if (d->n_q_heads <= 0 || d->n_kv_heads <= 0 || d->head_dim <= 0 || n_tokens < 0) return TKV_E_INVAL;
  if (d->head_dim != TKV_D || d->n_q_heads > 1024 || d->n_kv_heads > 1024) return TKV_E_UNSUPPORTED;
  if ((d->in_dtype != TKV_F16 && d->in_dtype != TKV_BF16) || (d->out_dtype != TKV_F16 && d->out_dtype != TKV_BF16)) return TKV_E_INVAL;
  if ((d->norm != 0 && d->norm != 1) || (d->interleaved != 0 && d->interleaved != 1)) return TKV_E_INVAL;
  if (d->norm && !(d->eps >= 0.f)) return TKV_E_INVAL;
  if (!d->norm && (q_weight || k_weight)) return TKV_E_INVAL;
  if (d->rotary_dim < 0 || d->rotary_dim > TKV_D || d->rotary_dim % 2 != 0) return TKV_E_INVAL;
  if (d->rotary_dim % 16 != 0) return TKV_E_UNSUPPORTED;
  if (axis_of) {
    if (n_axes <= 0) return TKV_E_INVAL;
    if (n_axes > 4) return TKV_E_UNSUPPORTED;
    for (int i = 0; i < d->rotary_dim / 2; ++i)
      if (axis_of[i] >= n_axes) return TKV_E_INVAL;
  }
  return TKV_OK;
}

// What the three entry points have in common once their own arguments are looked at.  The pointers to be aligned are among them; v, if
// not NULL, makes rows of its own.
int32_t enqueue_rope(const tkv_rope_desc* d, int32_t n_tokens, const uint8_t* axis_of, int bits, RopeParams& p, hipStream_t s) {
  for (const void* x : {p.q, p.k, p.v, (const void*)p.q_out, (const void*)p.k_out, (const void*)p.v_out, p.q_weight, p.k_weight})
    if (!aligned16(x)) return TKV_E_INVAL;
  if ((p.q && !dense_rows(d->q_stride)) || !dense_rows(d->k_stride) || (p.v && !dense_rows(d->v_stride))) return TKV_E_INVAL;
  p.q_st = d->q_stride[0]; p.q_sh = d->q_stride[1];
  p.k_st = d->k_stride[0]; p.k_sh = d->k_stride[1];
  p.v_st = d->v_stride[0]; p.v_sh = d->v_stride[1];
  p.hq = p.q ? d->n_q_heads : 0; p.hkv = d->n_kv_heads; p.n_tokens = n_tokens;
  p.rows = p.hq + p.hkv + (p.v ? p.hkv : 0);
  const int octets = (p.rows + 7) / 8;
  // Waves of two octets, the second on its way while the first is worked on, where those fill the machine; otherwise of one.
  // (48 rows a token, in us with one / two / a wave per token: 64 tokens 3.3 / 3.9 / 6.3, 768 5.5 / 5.9, 1024 6.9 / 6.5 / 7.7,
  // 4096 17.9 / 17.4 / 16.8, 32768 140 / 136 / 149.)
  p.per_wave = (int64_t)n_tokens * octets >= 6000 ? 2 : 1;
  p.parts = (octets + p.per_wave - 1) / p.per_wave;
  if ((int64_t)n_tokens * p.parts > 4 * ((1 << 24) - 1)) return TKV_E_UNSUPPORTED;  // (a launch has fewer than 2^32 threads)
  p.pairs8 = d->rotary_dim / 16;
  p.interleaved = d->interleaved; p.norm = d->norm; p.eps = d->eps;
  p.axis[0] = p.axis[1] = 0;
  for (int i = 0; axis_of && i < d->rotary_dim / 2; ++i)
    for (int b = 0; b < 2; ++b) p.axis[b] |= (uint64_t)(axis_of[i] >> b & 1) << i;
  if (d->in_dtype == TKV_F16)
    return d->out_dtype == TKV_F16 ? launch_rope<_Float16, _Float16>(p, bits, s) : launch_rope<_Float16, __bf16>(p, bits, s);
  return d->out_dtype == TKV_F16 ? launch_rope<__bf16, _Float16>(p, bits, s) : launch_rope<__bf16, __bf16>(p, bits, s);
}

int32_t norm_rope(const tkv_rope_desc* d, int32_t n_tokens, const void* q, const void* k, const void* v, const int32_t* positions,
                  const float* inv_freq, const uint8_t* axis_of, int32_t n_axes, const void* q_weight, const void* k_weight, void* q_out,
                  void* k_out, void* v_out, void* stream) {
  const int32_t st = check_rope_desc(d, n_tokens, axis_of, n_axes, q_weight, k_weight);
  if (st != TKV_OK) return st;
  if (n_tokens == 0) return TKV_OK;  // (an empty tensor's address may be NULL)
  if (!q || !k || !q_out || !k_out || (v == nullptr) != (v_out == nullptr)) return TKV_E_INVAL;
  if (d->rotary_dim && (!positions || !inv_freq)) return TKV_E_INVAL;
  RopeParams p = {};
  p.q = q; p.k = k; p.v = v;
  p.q_out = q_out; p.k_out = k_out; p.v_out = v_out;
  p.positions = positions; p.inv_freq = inv_freq;
  p.q_weight = q_weight; p.k_weight = k_weight;
  return enqueue_rope(d, n_tokens, axis_of, 0, p, (hipStream_t)stream);
}

}  // namespace

extern "C" int32_t tkv_qk_norm_rope(const tkv_rope_desc* d, int32_t n_tokens, const void* q, const void* k, const void* v,
                                    const int32_t* positions, const float* inv_freq, const void* q_weight,
                                    const void* k_weight, void* q_out, void* k_out, void* v_out, void* stream) {
  return norm_rope(d, n_tokens, q, k, v, positions, inv_freq, nullptr, 1, q_weight, k_weight, q_out, k_out, v_out, stream);
}

extern "C" int32_t tkv_qk_norm_rope_axes(const tkv_rope_desc* d, int32_t n_tokens, const void* q, const void* k, const void* v,
                                         const int32_t* positions, const float* inv_freq, const uint8_t* axis_of_host, int32_t n_axes,
                                         const void* q_weight, const void* k_weight, void* q_out, void* k_out, void* v_out,
                                         void* stream) {
  if (!axis_of_host) return TKV_E_INVAL;
  return norm_rope(d, n_tokens, q, k, v, positions, inv_freq, axis_of_host, n_axes, q_weight, k_weight, q_out, k_out, v_out, stream);
}

extern "C" int32_t tkv_paged_append(const tkv_paged_desc* desc, const tkv_rope_desc* d, int32_t n_tokens, const void* q, const void* k,
                                    const void* v, const int32_t* positions, const float* inv_freq, const uint8_t* axis_of_host,
                                    int32_t n_axes, const void* q_weight, const void* k_weight, const int32_t* slots, void* q_out,
                                    void* k_out, void* k_pages, void* v_pages, void* stream) {
  int32_t st = tkv::check_paged_desc(desc);
  if (st != TKV_OK) return st;
  st = check_rope_desc(d, n_tokens, axis_of_host, n_axes, q_weight, k_weight);
  if (st != TKV_OK) return st;
  if (d->n_q_heads != desc->n_q_heads || d->n_kv_heads != desc->n_kv_heads || d->out_dtype != desc->dtype) return TKV_E_INVAL;
  if (n_tokens == 0) return TKV_OK;
  if (!k || !v || !slots || ((uintptr_t)slots & 3) != 0 || (q == nullptr) != (q_out == nullptr) || (!q && q_weight)) return TKV_E_INVAL;
  if (d->rotary_dim && (!positions || !inv_freq)) return TKV_E_INVAL;
  RopeParams p = {};
  st = tkv::paged_view(desc, k_pages, v_pages, &p.pages);
  if (st != TKV_OK) return st;
  p.q = q; p.k = k; p.v = v;
  p.q_out = q_out; p.k_out = k_out;
  p.positions = positions; p.inv_freq = inv_freq;
  p.q_weight = q_weight; p.k_weight = k_weight;
  p.slots = slots;
  p.lowest = tkv::lowest_exponent(desc->dtype);
  return enqueue_rope(d, n_tokens, axis_of_host, desc->bits, p, (hipStream_t)stream);
}
