// Device and host helpers of the 8-bit cache (nsn_q8_*): format, addressing, conversions.
#pragma once

#include <type_traits>

#include "nsn_host.h"

namespace nsn {
namespace q8 {

constexpr int kBlock = 64;  // tokens that share a scale

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half4v __attribute__((ext_vector_type(4)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef unsigned uint2v __attribute__((ext_vector_type(2)));
typedef unsigned uint4v __attribute__((ext_vector_type(4)));

struct Geometry {
  int hq, hkv, ratio;
  int max_len, n_pages, page_size;  // page_size 0: contiguous
  int pages_per_seq;
  int unit_tokens;                  // tokens per unit: page_size, or max_len
  nsn::Geometry::Div page_div;      // division by page_size
};

struct View {
  uint8_t* codes;
  float* scales;
  const int32_t* block_table;
};

struct Rows {
  const uint16_t* data;
  int64_t sb, sh, st;
};

// A value that no kernel of the call writes, at an address that is the same for the whole wave: comes through the scalar cache, and
// waiting for it does not wait for the vector loads that were asked for before it
template <typename T>
__device__ __forceinline__ T load_uniform(const T* p) {
  return *(const __attribute__((address_space(4))) T*)(uintptr_t)p;
}

// Place of 64-token block `blk` of sequence b: index of the block among all units' blocks of head 0 .. (times D * 64 bytes: its
// codes), or -1 where its page does not exist.  Pages are multiples of 64 tokens, so a block lies in one page.
// UNIFORM: the same block for the whole wave.
template <bool UNIFORM = false>
__device__ __forceinline__ int64_t block_place(const Geometry& g, const int32_t* table, int b, int h, int blk) {
  int64_t unit = b;
  int in = blk;
  if (g.page_size > 0) {
    const int page = tokens_div(blk * kBlock, g.page_div);
    const int32_t* entry = table + (int64_t)b * g.pages_per_seq + page;
    const int p = UNIFORM ? load_uniform(entry) : *entry;
    if ((unsigned)p >= (unsigned)g.n_pages) return -1;
    unit = p;
    in = blk - page * (g.page_size / kBlock);
  }
  return (unit * g.hkv + h) * (int64_t)(g.unit_tokens / kBlock) + in;
}

// ---- codes -> fp16, exactly ---------------------------------------------------------------------------
// Four codes of one dword.  int8: the bytes with their sign bit flipped are c + 128; under the exponent byte 0x64 they
// are the fp16 numbers 1024 + 128 + c, so one byte permutation and one packed subtraction convert two.  e4m3: one instruction
// converts two.
template <int CODE>
__device__ __forceinline__ void to_half4(unsigned w, half2v& lo, half2v& hi) {
  if constexpr (CODE == NSN_Q8_INT8) {
    const unsigned u = w ^ 0x80808080u, m = 0x64646464u;
    const half2v bias = {(_Float16)1152.0f, (_Float16)1152.0f};
    lo = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(m, u, 0x07010700u)) - bias;
    hi = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(m, u, 0x07030702u)) - bias;
  } else {
    lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false);
    hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true);
  }
}

template <int CODE>
__device__ __forceinline__ void to_float4(unsigned w, float* f) {
  if constexpr (CODE == NSN_Q8_INT8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = (float)(int8_t)(w >> (8 * i));
  } else {
    const float2v a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    f[0] = a[0], f[1] = a[1], f[2] = b[0], f[3] = b[1];
  }
}

// four values (already divided by the scale) -> four codes, to nearest even; a NaN gives 0
template <int CODE>
__device__ __forceinline__ unsigned to_codes(const float* f) {
  if constexpr (CODE == NSN_Q8_INT8) {
    unsigned w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float y = f[i] == f[i] ? fminf(fmaxf(rintf(f[i]), -127.f), 127.f) : 0.f;
      w |= ((unsigned)(int)y & 255u) << (8 * i);
    }
    return w;
  } else {
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = f[i] == f[i] ? fminf(fmaxf(f[i], -448.f), 448.f) : 0.f;
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
    return (unsigned)w;
  }
}

// the scale that a block of largest magnitude amax asks for
template <int CODE>
__device__ __forceinline__ float level_of(float amax) {
  if (!(amax >= 0x1p-117f)) return 0.f;
  if constexpr (CODE == NSN_Q8_INT8) {
    return amax / 127.0f;
  } else {
    // amax = 1.f * 2^x:  448 = 1.75 * 2^8
    const unsigned u = __float_as_uint(amax);
    const int x = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);
    return __uint_as_float((unsigned)(x + 127) << 23);
  }
}
__device__ __forceinline__ float inverse(float level) { return level > 0.f ? 1.0f / level : 0.f; }

template <bool BF>
__device__ __forceinline__ float to_float(uint16_t u) {
  if constexpr (BF)
    return __uint_as_float((unsigned)u << 16);
  else
    return (float)__builtin_bit_cast(_Float16, u);
}
template <bool BF>
__device__ __forceinline__ uint16_t from_float(float f) {  // to nearest even
  if constexpr (BF)
    return __builtin_bit_cast(uint16_t, (__bf16)f);
  else
    return __builtin_bit_cast(uint16_t, (_Float16)f);
}

__device__ __forceinline__ int wave_scan(int v) {  // inclusive prefix sum over the 64 lanes
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // row_shr 1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // row 0's and 2's last lane to the rows behind them
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // the lower half's last lane to the upper half
  return v;
}

inline Geometry make_geometry(const nsn_q8_shape& s) {
  Geometry g;
  g.hq = s.n_q_heads, g.hkv = s.n_kv_heads, g.ratio = s.n_q_heads / s.n_kv_heads;
  g.max_len = s.max_len, g.n_pages = s.n_pages, g.page_size = s.page_size;
  g.pages_per_seq = s.page_size > 0 ? s.max_len / s.page_size : 1;
  g.unit_tokens = s.page_size > 0 ? s.page_size : s.max_len;
  g.page_div = tokens_divisor(g.unit_tokens);
  return g;
}
inline View make_view(const nsn_q8_cache& c) { return {c.codes, c.scales, c.block_table}; }
inline Rows make_rows(const nsn_rows& r) { return {static_cast<const uint16_t*>(r.data), r.batch_stride, r.head_stride, r.token_stride}; }

// byte offset of channel c of token t inside a unit
inline int64_t v_offset(int D, int64_t t, int c) {
  const int n = 256 / D, m = D / 16;
  return t / n * 256 + c / m * 16 + t % n * m + c % m;
}

int append_launch(const nsn_q8_shape& s, const nsn_rows& k, const nsn_rows& v, int max_new, const int32_t* seq_start,
                  const int32_t* n_new, int batch, const nsn_q8_cache& kc, const nsn_q8_cache& vc, hipStream_t stream);

struct AttentionCall {
  nsn_q8_shape shape;
  nsn_rows q;
  int n_q;
  const int32_t* q_lens;
  nsn_q8_cache kc, vc;
  const int32_t* seq_lens;
  int batch, max_seq_len;
  float scale;
  int causal;
  const float* weights_in;
  float* weights_out;
  int n_splits;
  void* out;
  float* lse;
  void* workspace;
  hipStream_t stream;
};
size_t attention_workspace_bytes(const nsn_q8_shape& s, int batch, int n_q, int max_seq_len, int n_splits);
int attention_launch(const AttentionCall& c);

struct EvictCall {
  nsn_q8_shape shape;
  const float* weights;
  const int32_t* seq_lens;
  int batch, max_seq_len, keep, first, recent;
  nsn_q8_cache kc, vc, ko, vo;
  int32_t *kept, *new_lens;
  float* weights_out;
  hipStream_t stream;
};
int evict_launch(const EvictCall& c);

// calls f with integral constants (head_dim, code type, BF16 rows)
template <typename F>
int with_types(const nsn_q8_shape& s, F f) {
  auto with_io = [&](auto d, auto code) {
    return s.io_type == NSN_BF16 ? f(d, code, std::true_type{}) : f(d, code, std::false_type{});
  };
  auto with_code = [&](auto d) {
    return s.code_type == NSN_Q8_INT8 ? with_io(d, std::integral_constant<int, NSN_Q8_INT8>{})
                                      : with_io(d, std::integral_constant<int, NSN_Q8_E4M3>{});
  };
  return s.head_dim == 64 ? with_code(std::integral_constant<int, 64>{}) : with_code(std::integral_constant<int, 128>{});
}

}  // namespace q8
}  // namespace nsn
