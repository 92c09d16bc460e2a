// Norm of queries and keys per head with the position rotation in the same pass, values laid out
// beside them (tkv_qk_norm_rope).
//
//   y_c = x_c w_c / sqrt(mean_c x_c^2 + eps);  pairs (a, b) of the first R channels turn by pos f_i:
//   a cos - b sin, b cos + a sin.
//
// Every element is read once and written once: the memory's rate bounds long prompts (32768 tokens of 48 heads: 136 us, 5.9 TB/s, half
// of the input still in the last-level cache; a large copy reaches 5.1), the latency of one round trip a few tokens (16: 3.3 us).  Eight lanes take a row (a head of a token), sixteen channels each, chosen so
// that both channels of every pair lie in one lane: nothing is exchanged but the row's sum of squares.  A token's
// angles are worked out once per wave, one frequency per lane, and handed round.
#include "tkv_common.h"

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
};

template <typename T>
struct Vec8 {
  typedef T type __attribute__((ext_vector_type(8)));
};

template <typename In, typename Out>
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
      dst = (Out*)p.k_out + ((int64_t)token * p.hkv + h) * TKV_D;
    } else {
      const int h = row - p.hq - p.hkv;
      src = (const In*)p.v + (token * p.v_st + h * p.v_sh);
      dst = (Out*)p.v_out + ((int64_t)token * p.hkv + h) * TKV_D;
    }
  };
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
      const double t = (double)p.positions[token] * (double)p.inv_freq[lane] * 0.15915494309189533577;
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
        if (p.interleaved) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float x0 = x[2 * i], x1 = x[2 * i + 1], y0 = y[2 * i], y1 = y[2 * i + 1];
            x[2 * i] = x0 * cs[i] - x1 * sn[i];
            x[2 * i + 1] = x1 * cs[i] + x0 * sn[i];
            y[2 * i] = y0 * cs[4 + i] - y1 * sn[4 + i];
            y[2 * i + 1] = y1 * cs[4 + i] + y0 * sn[4 + i];
          }
        } else {
          const floatx8 x0 = x;
          x = x0 * cs - y * sn;
          y = y * cs + x0 * sn;
        }
      }
    }
    *(OutV*)(to + ca) = __builtin_convertvector(x, OutV);
    *(OutV*)(to + cb) = __builtin_convertvector(y, OutV);
  }
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
bool dense_rows(const int64_t* s) { return s[0] >= 0 && s[1] >= 0 && s[0] % 8 == 0 && s[1] % 8 == 0; }

template <typename In, typename Out>
int32_t launch_rope(const RopeParams& p, hipStream_t s) {
  const int64_t items = (int64_t)p.n_tokens * p.parts;
  TKV_LAUNCH((qk_norm_rope_kernel<In, Out>), dim3((uint32_t)((items + 3) / 4)), 256, 0, s, p);
  return TKV_OK;
}

}  // namespace

extern "C" int32_t tkv_qk_norm_rope(const tkv_rope_desc* d, int32_t n_tokens, const void* q, const void* k, const void* v,
                                    const int32_t* positions, const float* inv_freq, const void* q_weight,
                                    const void* k_weight, void* q_out, void* k_out, void* v_out, void* stream) {
  if (!d || d->struct_size != sizeof(tkv_rope_desc)) return TKV_E_INVAL;
  if (d->n_q_heads <= 0 || d->n_kv_heads <= 0 || d->head_dim <= 0 || n_tokens < 0) return TKV_E_INVAL;
  if (d->head_dim != TKV_D || d->n_q_heads > 1024 || d->n_kv_heads > 1024) return TKV_E_UNSUPPORTED;
  if ((d->in_dtype != TKV_F16 && d->in_dtype != TKV_BF16) || (d->out_dtype != TKV_F16 && d->out_dtype != TKV_BF16)) return TKV_E_INVAL;
  if ((d->norm != 0 && d->norm != 1) || (d->interleaved != 0 && d->interleaved != 1)) return TKV_E_INVAL;
  if (d->norm && !(d->eps >= 0.f)) return TKV_E_INVAL;
  if (!d->norm && (q_weight || k_weight)) return TKV_E_INVAL;
  if (d->rotary_dim < 0 || d->rotary_dim > TKV_D || d->rotary_dim % 2 != 0) return TKV_E_INVAL;
  if (d->rotary_dim % 16 != 0) return TKV_E_UNSUPPORTED;
  if (n_tokens == 0) return TKV_OK;  // (an empty tensor's address may be NULL)
  if (!q || !k || !q_out || !k_out || (v == nullptr) != (v_out == nullptr)) return TKV_E_INVAL;
  if (d->rotary_dim && (!positions || !inv_freq)) return TKV_E_INVAL;
  for (const void* x : {q, k, v, (const void*)q_out, (const void*)k_out, (const void*)v_out, q_weight, k_weight})
    if (!aligned16(x)) return TKV_E_INVAL;
  if (!dense_rows(d->q_stride) || !dense_rows(d->k_stride) || (v && !dense_rows(d->v_stride))) return TKV_E_INVAL;
  RopeParams p;
  p.q = q; p.k = k; p.v = v;
  p.q_out = q_out; p.k_out = k_out; p.v_out = v_out;
  p.positions = positions; p.inv_freq = inv_freq;
  p.q_weight = q_weight; p.k_weight = k_weight;
  p.q_st = d->q_stride[0]; p.q_sh = d->q_stride[1];
  p.k_st = d->k_stride[0]; p.k_sh = d->k_stride[1];
  p.v_st = d->v_stride[0]; p.v_sh = d->v_stride[1];
  p.hq = d->n_q_heads; p.hkv = d->n_kv_heads; p.n_tokens = n_tokens;
  p.rows = p.hq + p.hkv + (v ? p.hkv : 0);
  const int octets = (p.rows + 7) / 8;
  // Waves of two octets, the second on its way while the first is worked on, where those fill the machine; otherwise of one.
  // (48 rows a token, in us with one / two / a wave per token: 64 tokens 3.3 / 3.9 / 6.3, 768 5.5 / 5.9, 1024 6.9 / 6.5 / 7.7,
  // 4096 17.9 / 17.4 / 16.8, 32768 140 / 136 / 149.)
  p.per_wave = (int64_t)n_tokens * octets >= 6000 ? 2 : 1;
  p.parts = (octets + p.per_wave - 1) / p.per_wave;
  if ((int64_t)n_tokens * p.parts > 4 * ((1 << 24) - 1)) return TKV_E_UNSUPPORTED;  // (a launch has fewer than 2^32 threads)
  p.pairs8 = d->rotary_dim / 16;
  p.interleaved = d->interleaved; p.norm = d->norm; p.eps = d->eps;
  const auto s = (hipStream_t)stream;
  if (d->in_dtype == TKV_F16)
    return d->out_dtype == TKV_F16 ? launch_rope<_Float16, _Float16>(p, s) : launch_rope<_Float16, __bf16>(p, s);
  return d->out_dtype == TKV_F16 ? launch_rope<__bf16, _Float16>(p, s) : launch_rope<__bf16, __bf16>(p, s);
}
