// The 8-bit cache's bookkeeping: append of new keys and values, eviction by accumulated attention weight.
#include <algorithm>
#include <type_traits>

#include "nsn_host.h"
#include "nsn_q8.h"

namespace nsn {
namespace q8 {

// ---- append ---------------------------------------------------------------------------------------------
// One workgroup per (64-token block, head, K or V): it reads the block's new rows once into registers, takes the largest
// magnitude across the workgroup, and writes the codes as the 16-byte cells of the format; a thread owns whole cells (K: 16
// channels of a token, V: D / 16 channels of 256 / D tokens), so K and V take the same path and every full cell is one store.
// Bound by memory: 2 bytes read and 1 written per value.
constexpr int kAppendThreads = 256;

template <int D, int CODE, bool BF>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(Geometry g, Rows k_rows, Rows v_rows, int max_new,
                                                                const int32_t* seq_start, const int32_t* n_new, View kc, View vc) {
  constexpr int kCells = 4 * D, kPer = kCells / kAppendThreads;
  constexpr int kTok = 256 / D, kCh = D / 16;  // V cells: tokens, channels of each
  const int b = blockIdx.z, h = blockIdx.y >> 1, tid = threadIdx.x;
  const bool value = blockIdx.y & 1;
  const int start = seq_start[b];
  const int n = min(n_new[b], max_new);
  if (start < 0 || n <= 0 || start >= g.max_len) return;
  const int end = (int)min((int64_t)start + n, (int64_t)g.max_len);
  const int blk = start / kBlock + blockIdx.x;
  if ((int64_t)blk * kBlock >= end) return;
  const int t0 = blk * kBlock, lo = max(start - t0, 0), hi = min(end - t0, kBlock);  // new tokens of the block: [lo, hi)
  const View& cv = value ? vc : kc;
  const Rows& in = value ? v_rows : k_rows;
  const int64_t place = block_place(g, cv.block_table, b, h, blk);
  if (place < 0) return;
  const uint16_t* src = in.data + b * in.sb + h * in.sh + (int64_t)(t0 - start) * in.st;
  uint8_t* dst = cv.codes + place * (int64_t)(kBlock * D);

  alignas(16) uint16_t x[kPer][16];
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int cell = tid + i * kAppendThreads;
    if (!value) {
      const int t = cell / kCh, c = cell % kCh * 16;  // (D / 16 cells per token)
      if (t >= lo && t < hi) {
        const uint4v* p = reinterpret_cast<const uint4v*>(src + (int64_t)t * in.st + c);
        reinterpret_cast<uint4v*>(x[i])[0] = p[0], reinterpret_cast<uint4v*>(x[i])[1] = p[1];
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) x[i][e] = 0;
      }
    } else {
      const int t = cell / 16 * kTok, c = cell % 16 * kCh;
#pragma unroll
      for (int j = 0; j < kTok; ++j) {
        using piece = std::conditional_t<D == 128, uint4v, uint2v>;
        piece v = {};
        if (t + j >= lo && t + j < hi) v = *reinterpret_cast<const piece*>(src + (int64_t)(t + j) * in.st + c);
        *reinterpret_cast<piece*>(&x[i][j * kCh]) = v;
      }
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float a = fabsf(to_float<BF>(x[i][e]));
      if (a < INFINITY) amax = fmaxf(amax, a);
    }
  }
  amax = wave_max(amax);
  __shared__ float wmax[kAppendThreads / 64];
  if ((tid & 63) == 0) wmax[tid >> 6] = amax;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kAppendThreads / 64; ++w) amax = fmaxf(amax, wmax[w]);
  float* scale = cv.scales + place;
  const float before = lo > 0 ? *scale : 0.f;
  const float asked = level_of<CODE>(amax);
  const bool grew = asked > before;
  const float level = grew ? asked : before;
  const float inv = inverse(level), ratio = grew ? before / level : 1.f;

#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int cell = tid + i * kAppendThreads;
    unsigned w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = to_float<BF>(x[i][4 * q + e]) * inv;
      w[q] = to_codes<CODE>(y);
    }
    auto again = [&](unsigned old) {  // a code of a token before, under the larger scale
      float y[4];
      to_float4<CODE>(old, y);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] *= ratio;
      return to_codes<CODE>(y);
    };
    unsigned* at = reinterpret_cast<unsigned*>(dst + cell * 16);
    const int per = value ? kTok : 1, t = value ? cell / 16 * kTok : cell / kCh;
    if (t >= lo && t + per <= hi) {
      *reinterpret_cast<uint4v*>(at) = uint4v{w[0], w[1], w[2], w[3]};
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int tq = value ? t + q * 4 / kCh : t;
        if (tq >= lo && tq < hi)
          at[q] = w[q];
        else if (tq < lo && grew)
          at[q] = again(at[q]);
      }
    }
  }
  __syncthreads();  // (the stored scale has been read by every thread)
  if (tid == 0) *scale = level;
}

int append_launch(const nsn_q8_shape& s, const nsn_rows& k, const nsn_rows& v, int max_new, const int32_t* seq_start,
                  const int32_t* n_new, int batch, const nsn_q8_cache& kc, const nsn_q8_cache& vc, hipStream_t stream) {
  // a sequence's new tokens touch one block more than they fill where they start inside one; none lies beyond the cache
  const int64_t blocks = std::min<int64_t>(((int64_t)max_new + kBlock - 2) / kBlock + 1, s.max_len / kBlock);
  with_types(s, [&](auto d, auto code, auto bf) {
    append_kernel<d.value, code.value, bf.value><<<dim3((unsigned)blocks, 2 * s.n_kv_heads, batch), kAppendThreads, 0, stream>>>(
        make_geometry(s), make_rows(k), make_rows(v), max_new, seq_start, n_new, make_view(kc), make_view(vc));
    return 0;
  });
  return hipGetLastError() == hipSuccess ? NSN_OK : NSN_ERR_HIP;
}

// ---- eviction: which tokens stay ------------------------------------------------------------------------
// One workgroup per (sequence, head).  The weights, ordered as unsigned keys (NaN the least, tokens that stay whatever the others are
// above all), stay in registers where a sequence fits, K consecutive tokens to a thread (a longer one is read again for every
// pass).  The need-th largest key of the middle tokens is found by digits of 11, 11 and 10 bits with a histogram of each in LDS,
// until a bin holds no more than a wave's worth, whose keys are then compared with each other; a first digit of 11 bits spreads weights
// over four bins per power of two.  Then the tokens above the key and the first of those that equal it are counted off in order.
// Integer sums only: the same tokens for any order of the threads.  Bound by latency (a compute unit per head, some ten trips through
// LDS and barriers): 64 heads of 16384 tokens 19 us, 8 of 1088 8 us.
constexpr int kBins = 2048, kFew = 64;
constexpr unsigned kSure = 0xffffffffu;  // (no weight's key: that of infinity is 0xff800000)

__device__ __forceinline__ unsigned weight_key(float w) {
  if (w != w) return 0u;
  const unsigned u = __float_as_uint(w + 0.0f);  // (-0 and 0 are equal)
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// inclusive prefix sums over the workgroup of two values per thread, and their totals; sums: T / 64 pairs of LDS
template <int T>
__device__ __forceinline__ void scan_pair(int& x, int& y, int& all_x, int& all_y, int (&sums)[2][T / 64]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  x = wave_scan(x), y = wave_scan(y);
  if (lane == 63) sums[0][wave] = x, sums[1][wave] = y;
  __syncthreads();
  all_x = all_y = 0;
#pragma unroll
  for (int i = 0; i < T / 64; ++i) {
    const int sx = sums[0][i], sy = sums[1][i];
    if (i < wave) x += sx, y += sy;
    all_x += sx, all_y += sy;
  }
}

template <int T, int K, bool RESIDENT>
__global__ __launch_bounds__(T) void select_kernel(int hkv, int max_len, const float* weights, const int32_t* seq_lens, int max_seq_len,
                                                   int keep, int first, int recent, int32_t* kept, int32_t* new_lens,
                                                   float* weights_out) {
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
  const int len = min(max(seq_lens[b], 0), max_seq_len);
  const int n_keep = min(len, keep);
  const int64_t unit = (int64_t)b * hkv + h;
  const float* w = weights + unit * max_len;
  int32_t* kp = kept + unit * keep;
  float* wo = weights_out ? weights_out + unit * max_len : nullptr;

  __shared__ __attribute__((aligned(16))) int hist[kBins];
  __shared__ int found[3];
  __shared__ unsigned few[kFew];
  __shared__ int sums[2][T / 64];
  const int mid0 = first, mid1 = len - recent;  // the tokens to choose from, where len > keep
  int need = keep - first - recent;
  const bool choose = len > keep && need > 0;
  unsigned key[K];  // of token base + tid * K + i
  auto load_weights = [&](int base, float (&v)[K]) {
    const int live = len - base - tid * K;  // weights of this thread
    const float* p = w + base + tid * K;
#pragma unroll
    for (int i = 0; i < K; i += 4) {
      // (rows are multiples of 64 long: a piece of four that begins inside the sequence lies inside the row)
      const float4v x = i < live ? *reinterpret_cast<const float4v*>(p + i) : float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 4; ++e) v[i + e] = x[e];
    }
  };
  auto load = [&](int base) {
    const int t0 = base + tid * K, m0 = len <= keep ? K : mid0 - t0, m1 = mid1 - t0;
    float v[K];
    load_weights(base, v);
#pragma unroll
    for (int i = 0; i < K; ++i) key[i] = i < m0 || i >= m1 ? kSure : weight_key(v[i]);
  };
  if (RESIDENT) load(0);
  // (what does not hang on the choice, while the weights are on their way)
  if (h == 0 && tid == 0) new_lens[b] = n_keep;
  for (int j = n_keep + tid; j < keep; j += T) kp[j] = -1;
  if (wo)
    for (int j = n_keep + tid; j < max_seq_len; j += T) wo[j] = 0.f;

  unsigned prefix = kSure - 1, mask = 0;  // (where there is nothing to choose: those above it)
  if (choose) {
    prefix = 0;
#pragma unroll 1
    for (int digit = 0; digit < 3; ++digit) {
      const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bits = digit == 2 ? 10 : 11;
      constexpr int kOwn = kBins / T;  // bins of a thread
      static_assert(kOwn >= 2, "two bins to a thread at least");
#pragma unroll
      for (int i = 0; i < kOwn; i += 2) *reinterpret_cast<uint2v*>(&hist[tid * kOwn + i]) = uint2v{0, 0};
      __syncthreads();
      for (int base = 0; base < len; base += T * K) {
        if (!RESIDENT) load(base);
#pragma unroll
        for (int i = 0; i < K; ++i)
          if (digit == 0 ? key[i] != kSure : (key[i] & mask) == prefix) atomicAdd(&hist[(key[i] >> shift) & ((1 << bits) - 1)], 1);
      }
      __syncthreads();
      int c[kOwn], x = 0, y = 0, all = 0, none;
#pragma unroll
      for (int i = 0; i < kOwn; ++i) c[i] = hist[tid * kOwn + i], x += c[i];
      scan_pair<T>(x, y, all, none, sums);
      int above = all - x;  // in the bins of the threads behind
#pragma unroll
      for (int i = kOwn - 1; i >= 0; --i) {
        if (above < need && above + c[i] >= need) found[0] = tid * kOwn + i, found[1] = need - above, found[2] = c[i];
        above += c[i];
      }
      __syncthreads();
      prefix |= (unsigned)found[0] << shift;
      mask |= ((1u << bits) - 1) << shift;
      need = found[1];
      const int left = found[2];
      if (left <= kFew && digit < 2) {
        // the bin's keys, in their order; the one that fewer than need exceed and need or more reach
        int before = 0;
        for (int base = 0; base < len; base += T * K) {
          if (!RESIDENT) load(base);
          int own = 0, zero = 0, all_few, none2;
#pragma unroll
          for (int i = 0; i < K; ++i) own += (key[i] & mask) == prefix;
          int at = own;
          scan_pair<T>(at, zero, all_few, none2, sums);
          at += before - own;
          if (own) {
#pragma unroll
            for (int i = 0; i < K; ++i)
              if ((key[i] & mask) == prefix) few[at++] = key[i];
          }
          before += all_few;
          __syncthreads();  // (the sums are written again)
        }
        if (tid < 64) {
          const unsigned own = tid < left ? few[tid] : 0u;
          int more = 0, same = 0;
          for (int i = 0; i < left; ++i) {
            const unsigned k = (unsigned)__builtin_amdgcn_readlane((int)own, i);
            more += k > own, same += k == own;
          }
          if (tid < left && more < need && more + same >= need) found[0] = (int)own, found[1] = need - more;  // (equal keys write the same)
        }
        __syncthreads();
        prefix = (unsigned)found[0], need = found[1];
        break;
      }
    }
  }
  // In order: the tokens above `prefix`, and the first `need` of those that equal it.
  int base_sure = 0, base_eq = 0;
  for (int base = 0; base < len; base += T * K) {
    if (!RESIDENT) load(base);
    const int t0 = base + tid * K, live = len - t0;
    int own_sure = 0, own_eq = 0, all_sure, all_eq;
    float v[K];
    load_weights(base, v);
#pragma unroll
    for (int i = 0; i < K; ++i) {
      own_sure += i < live && key[i] > prefix;
      own_eq += i < live && key[i] == prefix;
    }
    int sure = own_sure, eq = own_eq;
    __syncthreads();  // (sums are read by the scan before)
    scan_pair<T>(sure, eq, all_sure, all_eq, sums);
    sure += base_sure - own_sure, eq += base_eq - own_eq;  // of the tokens before this thread's
#pragma unroll
    for (int i = 0; i < K; ++i) {
      const bool is_sure = i < live && key[i] > prefix, is_eq = i < live && key[i] == prefix;
      if (is_sure || (is_eq && eq < need)) {
        const int at = sure + min(eq, need);
        kp[at] = t0 + i;
        if (wo) wo[at] = v[i];
      }
      sure += is_sure, eq += is_eq;
    }
    base_sure += all_sure, base_eq += all_eq;
  }
}

// ---- eviction: the kept tokens move -----------------------------------------------------------------------
// One workgroup per 64-token block of the destination and head, K and V together: the block's 64 former indices and scales, one
// per lane, give the new scale and each token's ratio; then the rows' cells are all asked for, rounded again where the
// ratio is not 1, and written.  Bound by memory: each kept byte is read and written once, and of values, whose tokens share 16-byte
// cells, the neighbours of a kept token come along (64 heads of 4096 of up to 16384 tokens: 37 us, 142 MB, 178 with the
// neighbours; four blocks to a workgroup measured the same).
constexpr int kMoveThreads = 256;

// four codes of a live token under a scale that is 1 / r times theirs, r <= 1
template <int CODE>
__device__ __forceinline__ unsigned rescale(unsigned w, float r) {
  if constexpr (CODE == NSN_Q8_INT8) {
    const unsigned u = w ^ 0x80808080u;  // c + 128
    unsigned y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float c = (float)(u >> (8 * i) & 255u) - 128.f;
      const float x = c * r;
      y[i] = __float_as_uint(x + 12582912.f);  // 3 * 2^22: the sum's last bits are the nearest integer (|x| <= 127)
    }
    const unsigned lo = __builtin_amdgcn_perm(y[1], y[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(y[3], y[2], 0x0c0c0400u);
    return lo | hi << 16;
  } else {
    float f[4];
    to_float4<CODE>(w, f);
    int x = __builtin_amdgcn_cvt_pk_fp8_f32(f[0] * r, f[1] * r, 0, false);
    x = __builtin_amdgcn_cvt_pk_fp8_f32(f[2] * r, f[3] * r, x, true);
    return (unsigned)x;
  }
}

template <int D, int CODE>
__global__ __launch_bounds__(kMoveThreads) void move_kernel(Geometry g, const int32_t* seq_lens, int max_seq_len, int keep,
                                                            const int32_t* kept, View kc, View vc, View ko, View vo) {
  constexpr int kPer = 4 * D / kMoveThreads;  // cells of a thread in a block
  constexpr int kTok = 256 / D, kCh = D / 16;
  using piece = std::conditional_t<D == 128, uint2v, unsigned>;  // a token's channels in a cell of values
  const int b = blockIdx.z, h = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int len = min(max(seq_lens[b], 0), max_seq_len);
  const int n_keep = min(len, keep), blk = blockIdx.x, t0 = blk * kBlock;
  if (t0 >= n_keep) return;
  const int live = min(n_keep - t0, kBlock);
  __shared__ int64_t s_row[2][kBlock];  // 64 * block + token inside: the former place; -1: there is none
  __shared__ float s_ratio[2][kBlock];
  __shared__ int64_t s_to[2];            // the blocks written; -1: there is none
  if (wave < 2) {  // a wave: K or V
    const View& from = wave ? vc : kc;
    const View& to = wave ? vo : ko;
    int64_t row = -1;
    float was = 0.f;
    if (lane < live) {
      const int t = kept[((int64_t)b * g.hkv + h) * keep + t0 + lane];
      const int64_t p = block_place(g, from.block_table, b, h, t / kBlock);
      if (p >= 0) {
        row = p * kBlock + t % kBlock;
        was = from.scales[p];
      }
    }
    const int64_t place = block_place(g, to.block_table, b, h, blk);
    const float level = wave_max(was);
    s_row[wave][lane] = row, s_ratio[wave][lane] = level > 0.f ? was / level : 0.f;
    if (lane == 0) {
      s_to[wave] = place;
      if (place >= 0) to.scales[place] = level;
    }
  }
  __syncthreads();
  uint4v x[kPer];
  piece y[kPer][kTok];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int cell = tid + i * kMoveThreads;
    const int64_t r = s_row[0][cell / kCh];
    x[i] = uint4v{0, 0, 0, 0};
    if (r >= 0) x[i] = *reinterpret_cast<const uint4v*>(kc.codes + r * D + cell % kCh * 16);
#pragma unroll
    for (int k = 0; k < kTok; ++k) {
      const int64_t rv = s_row[1][cell / 16 * kTok + k];
      y[i][k] = piece{};
      if (rv >= 0) y[i][k] = *reinterpret_cast<const piece*>(vc.codes + rv / kTok * 256 + cell % 16 * 16 + (int)(rv % kTok) * kCh);
    }
  }
  if (s_to[0] >= 0) {
    uint8_t* dst = ko.codes + s_to[0] * (int64_t)(kBlock * D);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int cell = tid + i * kMoveThreads, t = cell / kCh;
      const float r = s_ratio[0][t];
      if (r != 1.f) {
#pragma unroll
        for (int q = 0; q < 4; ++q) x[i][q] = rescale<CODE>(x[i][q], r);
      }
      if (t < live) *reinterpret_cast<uint4v*>(dst + cell * 16) = x[i];
    }
  }
  if (s_to[1] >= 0) {
    uint8_t* dst = vo.codes + s_to[1] * (int64_t)(kBlock * D);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int cell = tid + i * kMoveThreads, t = cell / 16 * kTok;
      uint4v u;
#pragma unroll
      for (int k = 0; k < kTok; ++k) {
        const float r = s_ratio[1][t + k];
#pragma unroll
        for (int q = 0; q < 4 / kTok; ++q) {
          unsigned c;
          if constexpr (D == 128)
            c = y[i][k][q];
          else
            c = y[i][k];
          u[k * (4 / kTok) + q] = r != 1.f ? rescale<CODE>(c, r) : c;
        }
      }
      if (t + kTok <= live) {
        *reinterpret_cast<uint4v*>(dst + cell * 16) = u;
      } else {  // (places behind the last token stay as they were)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (t + q * 4 / kCh < live) reinterpret_cast<unsigned*>(dst + cell * 16)[q] = u[q];
      }
    }
  }
}

int evict_launch(const EvictCall& c) {
  const nsn_q8_shape& s = c.shape;
  auto select = [&](auto kernel, int threads) {
    kernel<<<dim3(s.n_kv_heads, c.batch), threads, 0, c.stream>>>(s.n_kv_heads, s.max_len, c.weights, c.seq_lens, c.max_seq_len, c.keep,
                                                                  c.first, c.recent, c.kept, c.new_lens, c.weights_out);
  };
  if (c.max_seq_len <= 256 * 8)
    select(select_kernel<256, 8, true>, 256);
  else if (c.max_seq_len <= 1024 * 16)
    select(select_kernel<1024, 16, true>, 1024);
  else
    select(select_kernel<1024, 16, false>, 1024);
  if (hipGetLastError() != hipSuccess) return NSN_ERR_HIP;
  const int blocks = (std::min(c.keep, c.max_seq_len) + kBlock - 1) / kBlock;
  if (blocks == 0) return NSN_OK;
  with_types(s, [&](auto d, auto code, auto) {
    move_kernel<d.value, code.value><<<dim3(blocks, s.n_kv_heads, c.batch), kMoveThreads, 0, c.stream>>>(
        make_geometry(s), c.seq_lens, c.max_seq_len, c.keep, c.kept, make_view(c.kc), make_view(c.vc), make_view(c.ko), make_view(c.vo));
    return 0;
  });
  return hipGetLastError() == hipSuccess ? NSN_OK : NSN_ERR_HIP;
}

}  // namespace q8
}  // namespace nsn
