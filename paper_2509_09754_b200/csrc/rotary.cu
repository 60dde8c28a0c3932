// Rotary positions: pair i of a vector's leading elements turns by positions[token] * freqs[i], in q and k of a
// prompt, or in those of new tokens on their way into the paged cache.
//
// A unit is two 16-byte vectors that hold whole pairs: elements i ... and rotary_dim/2 + i ... where a pair is
// (i, i + rotary_dim/2), two neighbouring vectors where it is (2i, 2i+1) and behind rotary_dim.  A thread has one unit
// of one token, makes its cosines and sines once and takes head after head.
//
// The angle in turns, positions * freqs / (2 pi), is reduced to [-1/2, 1/2] in 64 bits (a position of a million
// times a frequency of one loses 2^-33 of a turn there, in fp32 1/16 of one) and goes to sincospif in fp32.  What it loses
// to fp32 there, up to 9.4e-8 rad, is put back to first order where vectors are fp32: a cosine or sine is off by its own
// rounding then, 1.5 * 2^-24.  Not with bf16, whose outputs are rounded by 2^-9 to 2^-8 (1024 tokens 5.2 us, with it 5.6).
//
// Bound by reading and writing the vectors once: 108 to 110 us at 32K tokens, 6.1 to 6.2 TB/s where a copy has 6.6 (1K
// tokens stay in L2: 5.2 us).
#include <algorithm>

#include <math.h>

#include "lava_internal.cuh"

namespace lava {
namespace {

// Threads of a block; heads that a thread has on their way; blocks per SM that the heads are split for at most.  32K tokens
// of 32 + 8 heads (bf16, 128) and 2049 of them in fp32, us: 128 / 2 / 24 108 / 16.4; one head 120 / 17.3, four 130 / 19.8
// (256 threads, 16 blocks), two heads with 256 threads 114 / 16.6; 12 blocks 112 / 16.9.
constexpr int kThreads = 128;
constexpr int kAhead = 2;
constexpr int kBlocks = 24;

// One array of vectors [tokens][heads][d]; a place in the pool instead of an own array where slots are given.
struct Vectors {
  const char* from;
  char* to;
  long long from_tok, from_head, to_tok, to_head;  // strides in bytes
  int heads;
};

struct RotaryParams {
  const double* freqs;
  const int* positions;
  long long n_tokens;
  int rotary_dim, interleaved;
  float scale, sign;
  Vectors x[3];            // queries, keys, values (which do not turn)
  int n_arrays, n_heads;   // heads of all arrays
  const int* slots;        // [n_tokens, H_kv], or NULL; keys and values go to rows of the pool then
  int pool_rows;
  int tokens_per_block;    // a power of two
};

template <bool BF16>
struct Elems {
  static constexpr int kPer = BF16 ? 8 : 4;
  static __device__ __forceinline__ void unpack(const uint4& raw, float (&x)[kPer]) {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
    if constexpr (BF16) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[2 * j] = __uint_as_float(w[j] << 16);
        x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = __uint_as_float(w[j]);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[kPer]) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (BF16) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * j], x[2 * j + 1]);
        w[j] = *reinterpret_cast<const uint32_t*>(&v);
      } else {
        w[j] = __float_as_uint(x[j]);
      }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

template <int D, bool BF16>
__global__ void __launch_bounds__(kThreads)
rotary_kernel(const __grid_constant__ RotaryParams p) {
  in_stream_order();
  using E = Elems<BF16>;
  constexpr int kPer = E::kPer, kUnits = D / (2 * kPer);
  const int u = threadIdx.x % kUnits, rest = threadIdx.x / kUnits;
  const long long token = (long long)blockIdx.x * p.tokens_per_block + rest % p.tokens_per_block;
  const int head0 = blockIdx.y * (kThreads / kUnits / p.tokens_per_block) + rest / p.tokens_per_block;
  const int step = gridDim.y * (kThreads / kUnits / p.tokens_per_block);
  if (token >= p.n_tokens) return;
  const int half = p.rotary_dim / 2;
  const bool turns = u * kPer < half;
  // first elements of the unit's two vectors
  const bool apart = turns && !p.interleaved;
  const int at0 = apart ? u * kPer : 2 * u * kPer, at1 = apart ? half + u * kPer : at0 + kPer;
  float cs[kPer], sn[kPer];
  if (turns) {
    const double pos = (double)p.positions[token] * 0.15915494309189535;  // 1 / (2 pi)
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const double t = pos * p.freqs[u * kPer + j];
      const double r = t - rint(t);
      const float near = (float)r;
      sincospif(2.0f * near, &sn[j], &cs[j]);
      if constexpr (!BF16) {
        const float rest = (float)(r - near) * 6.2831853f, s = sn[j];  // what fp32 loses of r, in rad: up to 9.4e-8
        sn[j] = fmaf(rest, cs[j], s);
        cs[j] = fmaf(-rest, s, cs[j]);
      }
      sn[j] *= p.sign * p.scale;
      cs[j] *= p.scale;
    }
  }
  const int o0 = at0 * (16 / kPer), o1 = at1 * (16 / kPer);
  for (int h0 = head0; h0 < p.n_heads; h0 += kAhead * step) {
    uint4 r0[kAhead], r1[kAhead];
    char* to[kAhead];
    bool turn[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int h = h0 + j * step;
      to[j] = nullptr;
      if (h >= p.n_heads) continue;
      const int a = h < p.x[0].heads ? 0 : h < p.x[0].heads + p.x[1].heads ? 1 : 2;  // array, head in it
      const int i = h - (a > 0 ? p.x[0].heads : 0) - (a > 1 ? p.x[1].heads : 0);
      const Vectors& x = p.x[a];
      if (p.slots && a > 0) {
        const int slot = p.slots[token * x.heads + i];
        if ((unsigned)slot >= (unsigned)p.pool_rows) continue;
        to[j] = x.to + (long long)slot * (D / kPer * 16);
      } else {
        to[j] = x.to + token * x.to_tok + i * x.to_head;
      }
      turn[j] = turns && a < 2;
      const char* from = x.from + token * x.from_tok + i * x.from_head;
      r0[j] = *reinterpret_cast<const uint4*>(from + o0);
      r1[j] = *reinterpret_cast<const uint4*>(from + o1);
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (!to[j]) continue;
      if (turn[j]) {
        float v0[kPer], v1[kPer];
        E::unpack(r0[j], v0);
        E::unpack(r1[j], v1);
        if (p.interleaved) {
#pragma unroll
          for (int e = 0; e < kPer; e += 2) {
            const float a0 = v0[e], a1 = v1[e];
            v0[e] = a0 * cs[e / 2] - v0[e + 1] * sn[e / 2];
            v0[e + 1] = v0[e + 1] * cs[e / 2] + a0 * sn[e / 2];
            v1[e] = a1 * cs[(kPer + e) / 2] - v1[e + 1] * sn[(kPer + e) / 2];
            v1[e + 1] = v1[e + 1] * cs[(kPer + e) / 2] + a1 * sn[(kPer + e) / 2];
          }
        } else {
#pragma unroll
          for (int e = 0; e < kPer; ++e) {
            const float a0 = v0[e];
            v0[e] = a0 * cs[e] - v1[e] * sn[e];
            v1[e] = v1[e] * cs[e] + a0 * sn[e];
          }
        }
        r0[j] = E::pack(v0);
        r1[j] = E::pack(v1);
      }
      *reinterpret_cast<uint4*>(to[j] + o0) = r0[j];
      *reinterpret_cast<uint4*>(to[j] + o1) = r1[j];
    }
  }
}

lava_status launch_rotary(const lava_rotary_desc& d, RotaryParams p, cudaStream_t stream) {
  p.n_heads = 0;
  for (int a = 0; a < p.n_arrays; ++a) p.n_heads += p.x[a].heads;
  if (p.n_tokens == 0 || p.n_heads == 0) return LAVA_OK;
  const bool bf16 = d.dtype == LAVA_BF16;
  const int units = d.head_dim / (bf16 ? 16 : 8), places = kThreads / units;
  p.tokens_per_block = 1;
  while (p.tokens_per_block < places && p.tokens_per_block < p.n_tokens) p.tokens_per_block *= 2;
  const long long blocks = (p.n_tokens + p.tokens_per_block - 1) / p.tokens_per_block;
  const int rows = places / p.tokens_per_block;
  // Few tokens: heads over more blocks, each of which makes the cosines and sines anew; so a thread has two or four heads as
  // soon as there are blocks enough.  Tokens of 32 + 8 heads, us with one / two / four: 16 2.0 / 2.2 / 2.8; 256 3.5 / 3.1 /
  // 3.4; 1024 8.0 / 5.9 / 5.2; 4096 18.3 / 18.3 / 17.5.
  const int sms = std::max(1, sm_count());
  const long long most = blocks * ((p.n_heads + rows - 1) / rows);
  const int per = most <= 2 * sms ? 1 : most <= 8 * sms ? 2 : 4;
  const long long want = (long long)kBlocks * sms, of_heads = (p.n_heads + rows * per - 1) / (rows * per);
  const int split = (int)std::max(1ll, std::min(of_heads, (want + blocks - 1) / blocks));
  if (blocks > 0x7fffffff) return fail(LAVA_ERR_UNSUPPORTED, "too many tokens");
  const auto kernel = bf16 ? (d.head_dim == 64 ? rotary_kernel<64, true> : rotary_kernel<128, true>)
                           : (d.head_dim == 64 ? rotary_kernel<64, false> : rotary_kernel<128, false>);
  const cudaError_t e = launch_in_order(kernel, dim3((unsigned)blocks, split), kThreads, 0, stream, p);
  count_launches(1);
  return check_cuda(e, "rotary launch");
}

lava_status check_rotary(const lava_rotary_desc* d, const double* freqs, const int32_t* positions, int64_t n_tokens,
                         RotaryParams* p) {
  if (!d) return fail(LAVA_ERR_INVALID_ARG, "rotary is NULL");
  if (d->head_dim != 64 && d->head_dim != 128)
    return fail(LAVA_ERR_UNSUPPORTED, "head_dim must be 64 or 128 (got %d)", d->head_dim);
  if (d->rotary_dim < 0 || d->rotary_dim > d->head_dim)
    return fail(LAVA_ERR_INVALID_ARG, "rotary_dim must be in 0..head_dim (got %d)", d->rotary_dim);
  if (d->rotary_dim % 16 != 0)
    return fail(LAVA_ERR_UNSUPPORTED, "rotary_dim must be a multiple of 16 (got %d)", d->rotary_dim);
  if (d->dtype != LAVA_F32 && d->dtype != LAVA_BF16) return fail(LAVA_ERR_INVALID_ARG, "unknown dtype %d", d->dtype);
  if ((d->interleaved | 1) != 1 || (d->backward | 1) != 1)
    return fail(LAVA_ERR_INVALID_ARG, "interleaved and backward are 0 or 1");
  if (!(d->scale >= 0.f) || isinf(d->scale)) return fail(LAVA_ERR_INVALID_ARG, "scale must be finite and >= 0");
  if (n_tokens < 0) return fail(LAVA_ERR_INVALID_ARG, "n_tokens must be >= 0");
  if ((!positions && n_tokens > 0) || (!freqs && d->rotary_dim > 0))
    return fail(LAVA_ERR_INVALID_ARG, "NULL argument");
  *p = RotaryParams{};
  p->freqs = freqs;
  p->positions = positions;
  p->n_tokens = n_tokens;
  p->rotary_dim = d->rotary_dim;
  p->interleaved = d->interleaved;
  p->scale = d->scale > 0.f ? d->scale : 1.f;
  p->sign = d->backward ? -1.f : 1.f;
  return LAVA_OK;
}

// Bytes from the first to behind the last of an array with these strides (in bytes).
long long span(const lava_rotary_desc& d, long long tokens, int heads, long long st, long long sh) {
  return (tokens - 1) * st + (heads - 1) * sh + d.head_dim * (d.dtype == LAVA_BF16 ? 2 : 4);
}

// Whether the output lies apart from its input or is the input itself.
bool apart_or_same(const lava_rotary_desc& d, long long tokens, const Vectors& x) {
  const bool same = x.from == x.to && (tokens == 1 || x.from_tok == x.to_tok) &&
                    (x.heads == 1 || x.from_head == x.to_head);
  return same || x.from >= x.to + span(d, tokens, x.heads, x.to_tok, x.to_head) ||
         x.to >= x.from + span(d, tokens, x.heads, x.from_tok, x.from_head);
}

lava_status check_vectors(const lava_rotary_desc& d, const char* what, long long tokens, const void* from, int heads,
                          int64_t st, int64_t sh, const void* to, int64_t to_st, int64_t to_sh, Vectors* out) {
  const int es = d.dtype == LAVA_BF16 ? 2 : 4;
  if (heads < 1 || heads > 65535) return fail(LAVA_ERR_INVALID_ARG, "heads of %s must be in 1..65535", what);
  if (!from || !to) return fail(LAVA_ERR_INVALID_ARG, "%s: one of input and output is NULL", what);
  if (!aligned16(from) || !aligned16(to)) return fail(LAVA_ERR_INVALID_ARG, "%s must be 16-byte aligned", what);
  for (const int64_t s : {st, sh, to_st, to_sh})
    if (s < 0 || s % 8 != 0 || s > (1ll << 40))
      return fail(LAVA_ERR_INVALID_ARG, "strides of %s must be non-negative multiples of 8 elements", what);
  // no two output vectors share an element
  const bool tok_inner = (tokens > 1 && to_st < to_sh) || heads == 1;
  const int64_t inner = tok_inner ? to_st : to_sh, outer = tok_inner ? to_sh : to_st;
  const int64_t n_inner = tok_inner ? tokens : heads, n_outer = tok_inner ? heads : tokens;
  if ((n_inner > 1 && inner < d.head_dim) || (n_outer > 1 && outer < (n_inner - 1) * inner + d.head_dim))
    return fail(LAVA_ERR_INVALID_ARG, "output vectors of %s overlap", what);
  *out = {(const char*)from, (char*)to, st * es, sh * es, to_st * es, to_sh * es, heads};
  return LAVA_OK;
}

}  // namespace
}  // namespace lava

using namespace lava;

extern "C" {

lava_status lava_rotary_freqs(int32_t kind, int32_t rotary_dim, double base, double factor, double original_length,
                              double low, double high, double* freqs, float* scale) {
  const double two_pi = 6.283185307179586;
  if (kind < LAVA_ROTARY_PLAIN || kind > LAVA_ROTARY_RAMP)
    return fail(LAVA_ERR_INVALID_ARG, "unknown rotary kind %d", kind);
  if (rotary_dim < 16 || rotary_dim > 128 || rotary_dim % 16 != 0)
    return fail(LAVA_ERR_UNSUPPORTED, "rotary_dim must be a multiple of 16 in 16..128 (got %d)", rotary_dim);
  if (!freqs) return fail(LAVA_ERR_INVALID_ARG, "NULL argument");
  if (!(base > 1.0) || isinf(base)) return fail(LAVA_ERR_INVALID_ARG, "base must be finite and above 1");
  if (kind != LAVA_ROTARY_PLAIN && (!(factor >= 1.0) || isinf(factor)))
    return fail(LAVA_ERR_INVALID_ARG, "factor must be finite and at least 1");
  const bool ranged = kind == LAVA_ROTARY_BANDS || kind == LAVA_ROTARY_RAMP;
  if (ranged && (!(original_length > 0.0) || isinf(original_length) || !(low > 0.0) || !(high > low) || isinf(high)))
    return fail(LAVA_ERR_INVALID_ARG, "original_length > 0 and 0 < low < high are needed");
  const int n = rotary_dim / 2;
  const double r = rotary_dim;
  if (kind == LAVA_ROTARY_BASE) base *= pow(factor, r / (r - 2.0));
  double first = 0.0, last = 0.0;  // RAMP: pairs up to `first` are kept, from `last` on divided
  if (kind == LAVA_ROTARY_RAMP) {
    first = fmax(0.0, floor(r * log(original_length / (high * two_pi)) / (2.0 * log(base))));
    last = fmin(r - 1.0, ceil(r * log(original_length / (low * two_pi)) / (2.0 * log(base))));
  }
  for (int i = 0; i < n; ++i) {
    double f = pow(base, -2.0 * i / r);
    double kept = 1.0;  // share of the frequency that is not divided
    if (kind == LAVA_ROTARY_LINEAR) kept = 0.0;
    if (kind == LAVA_ROTARY_BANDS) kept = fmin(1.0, fmax(0.0, (original_length * f / two_pi - low) / (high - low)));
    if (kind == LAVA_ROTARY_RAMP) kept = 1.0 - fmin(1.0, fmax(0.0, (i - first) / fmax(last - first, 0.001)));
    if (kind != LAVA_ROTARY_PLAIN && kind != LAVA_ROTARY_BASE) f = kept * f + (1.0 - kept) * f / factor;
    freqs[i] = f;
  }
  if (scale) *scale = kind == LAVA_ROTARY_RAMP ? (float)(0.1 * log(factor) + 1.0) : 1.0f;
  return LAVA_OK;
}

lava_status lava_rotary(const lava_rotary_desc* rotary, const double* freqs, int64_t n_tokens,
                        const int32_t* positions, const void* q, int32_t n_q_heads, int64_t q_stride_tok,
                        int64_t q_stride_head, void* q_out, int64_t q_out_stride_tok, int64_t q_out_stride_head,
                        const void* k, int32_t n_kv_heads, int64_t k_stride_tok, int64_t k_stride_head, void* k_out,
                        int64_t k_out_stride_tok, int64_t k_out_stride_head, void* stream) {
  RotaryParams p;
  lava_status rc = check_rotary(rotary, freqs, positions, n_tokens, &p);
  if (rc != LAVA_OK) return rc;
  if (n_tokens == 0) return LAVA_OK;
  if (!q && !q_out && !k && !k_out) return fail(LAVA_ERR_INVALID_ARG, "neither queries nor keys are given");
  if (q || q_out) {
    rc = check_vectors(*rotary, "q", n_tokens, q, n_q_heads, q_stride_tok, q_stride_head, q_out, q_out_stride_tok,
                       q_out_stride_head, &p.x[p.n_arrays++]);
    if (rc != LAVA_OK) return rc;
  }
  if (k || k_out) {
    rc = check_vectors(*rotary, "k", n_tokens, k, n_kv_heads, k_stride_tok, k_stride_head, k_out, k_out_stride_tok,
                       k_out_stride_head, &p.x[p.n_arrays++]);
    if (rc != LAVA_OK) return rc;
  }
  for (int a = 0; a < p.n_arrays; ++a)
    if (!apart_or_same(*rotary, n_tokens, p.x[a]))
      return fail(LAVA_ERR_INVALID_ARG, "an output overlaps its input and is not the input itself");
  return launch_rotary(*rotary, p, (cudaStream_t)stream);
}

lava_status lava_rotary_append(const lava_rotary_desc* rotary, const double* freqs, const lava_cache_desc* cache,
                               int64_t n_tokens, const int32_t* positions, const void* q, int64_t q_stride_tok,
                               int64_t q_stride_head, void* q_out, const void* k, int64_t k_stride_tok,
                               int64_t k_stride_head, const void* v, int64_t v_stride_tok, int64_t v_stride_head,
                               const int32_t* slots, void* k_pages, void* v_pages, void* stream) {
  RotaryParams p;
  Cache c;
  lava_status rc = make_cache(cache, &c);
  if (rc == LAVA_OK) rc = check_rotary(rotary, freqs, positions, n_tokens, &p);
  if (rc != LAVA_OK) return rc;
  if (rotary->head_dim != c.head_dim || rotary->dtype != c.dtype)
    return fail(LAVA_ERR_INVALID_ARG, "rotary and cache differ in head_dim or dtype");
  if (n_tokens == 0) return LAVA_OK;
  if (!slots) return fail(LAVA_ERR_INVALID_ARG, "NULL argument");
  const int d = c.head_dim;
  const struct { const char* name; const void* from; int heads; int64_t st, sh; void* to; } in[3] = {
      {"q", q, c.n_q_heads, q_stride_tok, q_stride_head, q_out},
      {"k", k, c.n_kv_heads, k_stride_tok, k_stride_head, k_pages},
      {"v", v, c.n_kv_heads, v_stride_tok, v_stride_head, v_pages}};
  for (int a = 0; a < 3; ++a) {
    rc = check_vectors(*rotary, in[a].name, n_tokens, in[a].from, in[a].heads, in[a].st, in[a].sh, in[a].to,
                       (int64_t)in[a].heads * d, d, &p.x[a]);
    if (rc != LAVA_OK) return rc;
  }
  if (!apart_or_same(*rotary, n_tokens, p.x[0]))
    return fail(LAVA_ERR_INVALID_ARG, "q_out overlaps q and is not q itself");
  p.n_arrays = 3;
  p.slots = slots;
  p.pool_rows = c.n_pages << c.page_shift;
  return launch_rotary(*rotary, p, (cudaStream_t)stream);
}

}  // extern "C"
