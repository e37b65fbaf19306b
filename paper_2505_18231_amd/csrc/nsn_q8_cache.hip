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
// One workgroup per (sequence, head).  The weights are ordered as unsigned keys (NaN the least); the need-th largest key of
// the middle tokens is found eight bits at a time with a histogram per pass, then one pass over the tokens in order writes
// those above it and the first of those that equal it.  Integer sums only: the same tokens for any order of the threads.
constexpr int kSelThreads = 1024;

__device__ __forceinline__ unsigned weight_key(float w) {
  if (w != w) return 0u;
  const unsigned u = __float_as_uint(w + 0.0f);  // (-0 and 0 are equal)
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(kSelThreads) void select_kernel(int hkv, int max_len, const float* weights, const int32_t* seq_lens,
                                                             int max_seq_len, int keep, int first, int recent, int32_t* kept,
                                                             int32_t* new_lens, float* weights_out) {
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int len = min(max(seq_lens[b], 0), max_seq_len);
  const int n_keep = min(len, keep);
  const int64_t unit = (int64_t)b * hkv + h;
  const float* w = weights + unit * max_len;
  int32_t* kp = kept + unit * keep;
  float* wo = weights_out ? weights_out + unit * max_len : nullptr;
  if (h == 0 && tid == 0) new_lens[b] = n_keep;

  __shared__ unsigned hist[256];
  __shared__ int found[2];
  __shared__ int wsum[2][kSelThreads / 64];
  const int mid0 = first, mid1 = len - recent;  // the tokens to choose from, where len > keep
  unsigned prefix = 0, mask = 0;
  int need = keep - first - recent;
  const bool choose = len > keep && need > 0;
  if (choose) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int t = mid0 + tid; t < mid1; t += kSelThreads) {
        const unsigned k = weight_key(w[t]);
        if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & 255u], 1u);
      }
      __syncthreads();
      if (wave == 0) {  // lane l owns bins 4 l .. 4 l + 3; counts of the bins above
        unsigned c[4], own_sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = hist[4 * lane + i], own_sum += c[i];
        unsigned above = own_sum;
        for (int m = 1; m < 64; m <<= 1) {
          const unsigned o = __shfl_down(above, m, 64);
          if (lane + m < 64) above += o;
        }
        above -= own_sum;
#pragma unroll
        for (int i = 3; i >= 0; --i) {
          if (above < (unsigned)need && above + c[i] >= (unsigned)need) found[0] = 4 * lane + i, found[1] = need - (int)above;
          above += c[i];
        }
      }
      __syncthreads();
      prefix |= (unsigned)found[0] << shift;
      mask |= 255u << shift;
      need = found[1];
    }
  }
  // in order: need = how many of the tokens whose key equals `prefix` stay (the first ones)
  int base = 0, base_eq = 0;
  for (int t0 = 0; t0 < len; t0 += kSelThreads) {
    const int t = t0 + tid;
    bool sure = false, eq = false;
    float wt = 0.f;
    if (t < len) {
      wt = w[t];
      if (len <= keep || t < first || t >= mid1) {
        sure = true;
      } else if (choose) {
        const unsigned k = weight_key(wt);
        sure = k > prefix, eq = k == prefix;
      }
    }
    const unsigned long long m_eq = __ballot(eq), below = (1ull << lane) - 1;
    if (lane == 0) wsum[0][wave] = __popcll(m_eq);
    __syncthreads();
    int rank_eq = base_eq + __popcll(m_eq & below), all_eq = 0;
    for (int i = 0; i < kSelThreads / 64; ++i) {
      if (i < wave) rank_eq += wsum[0][i];
      all_eq += wsum[0][i];
    }
    const bool stay = sure || (eq && rank_eq < need);
    const unsigned long long m_stay = __ballot(stay);
    if (lane == 0) wsum[1][wave] = __popcll(m_stay);
    __syncthreads();
    int at = base + __popcll(m_stay & below), all = 0;
    for (int i = 0; i < kSelThreads / 64; ++i) {
      if (i < wave) at += wsum[1][i];
      all += wsum[1][i];
    }
    if (stay) {
      kp[at] = t;
      if (wo) wo[at] = wt;
    }
    base += all, base_eq += all_eq;
    // (wsum[0] is written again only after every thread has passed the second barrier, wsum[1] after the next first one)
  }
  for (int j = n_keep + tid; j < keep; j += kSelThreads) kp[j] = -1;
  if (wo)
    for (int j = n_keep + tid; j < max_seq_len; j += kSelThreads) wo[j] = 0.f;
}

// ---- eviction: the kept tokens move -----------------------------------------------------------------------
// One workgroup per (64-token block of the destination, head, K or V): the block's 64 former indices and scales, one per
// lane, give the new scale and each token's ratio; then the rows' cells are gathered, rounded again where the ratio is
// not 1, and written.  Bound by memory: each kept byte is read and written once.
constexpr int kMoveThreads = 256;

template <int D, int CODE>
__global__ __launch_bounds__(kMoveThreads) void move_kernel(Geometry g, const int32_t* seq_lens, int max_seq_len, int keep,
                                                            const int32_t* kept, View kc, View vc, View ko, View vo) {
  constexpr int kCells = 4 * D, kPer = kCells / kMoveThreads;
  constexpr int kTok = 256 / D, kCh = D / 16;
  const int b = blockIdx.z, h = blockIdx.y >> 1, tid = threadIdx.x, lane = tid & 63;
  const bool value = blockIdx.y & 1;
  const int len = min(max(seq_lens[b], 0), max_seq_len);
  const int n_keep = min(len, keep), t0 = blockIdx.x * kBlock;
  if (t0 >= n_keep) return;
  const int live = min(n_keep - t0, kBlock);
  const View& from = value ? vc : kc;
  const View& to = value ? vo : ko;
  const int64_t place = block_place(g, to.block_table, b, h, blockIdx.x);
  if (place < 0) return;
  // every wave by itself: lane = token of the block
  int64_t row = -1;  // 64 * block + token inside: the former place
  float was = 0.f;
  if (lane < live) {
    const int t = kept[((int64_t)b * g.hkv + h) * keep + t0 + lane];
    const int64_t p = block_place(g, from.block_table, b, h, t / kBlock);
    if (p >= 0) {
      row = p * kBlock + t % kBlock;
      was = from.scales[p];
    }
  }
  const float level = wave_max(was);
  const float ratio = level > 0.f ? was / level : 0.f;
  __shared__ int64_t s_row[kBlock];
  __shared__ float s_ratio[kBlock];
  if (tid < kBlock) s_row[lane] = row, s_ratio[lane] = ratio;
  if (tid == 0) to.scales[place] = level;
  __syncthreads();
  uint8_t* dst = to.codes + place * (int64_t)(kBlock * D);
  auto again = [](unsigned old, float r) {
    float y[4];
    to_float4<CODE>(old, y);
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] *= r;
    return to_codes<CODE>(y);
  };
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int cell = tid + i * kMoveThreads;
    unsigned w[4] = {0, 0, 0, 0};
    if (!value) {
      const int t = cell / kCh;
      if (t >= live) continue;
      const int64_t r = s_row[t];
      if (r >= 0) {
        const uint4v v = *reinterpret_cast<const uint4v*>(from.codes + r * D + cell % kCh * 16);
        w[0] = v[0], w[1] = v[1], w[2] = v[2], w[3] = v[3];
        if (s_ratio[t] != 1.f) {
#pragma unroll
          for (int q = 0; q < 4; ++q) w[q] = again(w[q], s_ratio[t]);
        }
      }
      *reinterpret_cast<uint4v*>(dst + cell * 16) = uint4v{w[0], w[1], w[2], w[3]};
    } else {
      const int t = cell / 16 * kTok, n = cell % 16;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int tq = t + q * 4 / kCh;
        if (tq >= live) continue;
        const int64_t r = s_row[tq];
        if (r >= 0) {
          w[q] = *reinterpret_cast<const unsigned*>(from.codes + (r / kTok) * 256 + n * 16 + (int)(r % kTok) * kCh + q * 4 % kCh);
          if (s_ratio[tq] != 1.f) w[q] = again(w[q], s_ratio[tq]);
        }
      }
      if (t + kTok <= live) {
        *reinterpret_cast<uint4v*>(dst + cell * 16) = uint4v{w[0], w[1], w[2], w[3]};
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (t + q * 4 / kCh < live) reinterpret_cast<unsigned*>(dst + cell * 16)[q] = w[q];
      }
    }
  }
}

size_t evict_workspace_bytes(const nsn_q8_shape&, int, int, int) { return 0; }

int evict_launch(const EvictCall& c) {
  const nsn_q8_shape& s = c.shape;
  select_kernel<<<dim3(s.n_kv_heads, c.batch), kSelThreads, 0, c.stream>>>(s.n_kv_heads, s.max_len, c.weights, c.seq_lens, c.max_seq_len,
                                                                          c.keep, c.first, c.recent, c.kept, c.new_lens, c.weights_out);
  if (hipGetLastError() != hipSuccess) return NSN_ERR_HIP;
  const int blocks = (std::min(c.keep, c.max_seq_len) + kBlock - 1) / kBlock;
  if (blocks == 0) return NSN_OK;
  with_types(s, [&](auto d, auto code, auto) {
    move_kernel<d.value, code.value><<<dim3(blocks, 2 * s.n_kv_heads, c.batch), kMoveThreads, 0, c.stream>>>(
        make_geometry(s), c.seq_lens, c.max_seq_len, c.keep, c.kept, make_view(c.kc), make_view(c.vc), make_view(c.ko), make_view(c.vo));
    return 0;
  });
  return hipGetLastError() == hipSuccess ? NSN_OK : NSN_ERR_HIP;
}

}  // namespace q8
}  // namespace nsn
