// Attention over the 8-bit cache (nsn_q8_attention): single tokens and chunks, and the weights that each cached token receives.
//
// Rows.  The queries of a (sequence, kv head) are taken as rows r = i * ratio + g (token i, query head g of the kv head): all of
// them read the same keys and values, so a row is the unit of work and grouped heads cost no second reading of the cache.
//
// Per 64-token block, with codes k, v and scales sk, sv:
//   s = (q . k) * (softmax_scale log2 e sk),  m' = max(m, max s),  p = 2^(s - m'),  l = l 2^(m - m') + sum p,
//   o = o 2^(m - m') + sv (p . v)
// Codes become fp16 without loss (int8 and e4m3 both fit), so q . k is exact up to fp32 accumulation; p is rounded to fp16 (half a
// step 2^-11, below the rounding of the 16-bit output) for the second product.  bf16 queries are multiplied by a power of two
// per row that brings their largest magnitude to 2^14 .. 2^15, and are then fp16 numbers (values 2^-38 below the largest and
// smaller lose their last bits, which fp32 sums would not keep either).
#include <algorithm>
#include <type_traits>

#include "nsn_host.h"
#include "nsn_q8.h"

namespace nsn {
namespace q8 {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

struct Args {
  Geometry g;
  Rows q;
  int n_q, rows;  // rows = n_q * ratio of a (sequence, kv head)
  const int32_t* q_lens;
  View kc, vc;
  const int32_t* seq_lens;
  int max_seq_len;
  float scale_log2;  // softmax_scale * log2 e
  int causal;
  int n_splits, per;  // per: blocks of a split
  uint16_t* out;
  float* lse;
  float* lse2;     // [batch][hkv][rows], in powers of two (workspace)
  float* partial;  // [batch][hkv][rows][split][D + 2] (workspace)
  const float* weights_in;
  float* weights_out;
};

// what a (sequence, kv head) is asked
struct Problem {
  int len, nq, vis0;  // vis0: tokens that query 0 sees (causal), possibly negative
};
__device__ __forceinline__ Problem problem_of(const Args& a, int b) {
  Problem p;
  p.len = min(max(a.seq_lens[b], 0), a.max_seq_len);
  p.nq = a.q_lens ? min(max(a.q_lens[b], 0), a.n_q) : a.n_q;
  p.vis0 = a.causal ? p.len - p.nq + 1 : p.len;
  return p;
}
// tokens that query i sees
__device__ __forceinline__ int visible(const Args& a, const Problem& p, int i) {
  return a.causal ? min(max(p.vis0 + i, 0), p.len) : p.len;
}

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// The 16 rows r0 .. r0 + 15 as the second operand of the 16x16x32 products: lane 16 kg + n holds row n, and of every 64
// channels the 16 from 16 kg on, which is how a lane reads a row of key codes in 16-byte pieces (the order of the channels in
// a product is free as long as both operands share it).  Returns the factor that takes q . k to a power of two.
template <int D, bool BF>
__device__ __forceinline__ float load_queries(const Args& a, int b, int h, int r, int nq, half8v (&q)[D / 32]) {
  const int kg = (threadIdx.x & 63) >> 4;
  const bool there = r < nq * a.g.ratio;
  const int i = there ? r / a.g.ratio : 0, hq = there ? h * a.g.ratio + r % a.g.ratio : 0;
  const uint16_t* p = a.q.data + b * a.q.sb + hq * a.q.sh + i * a.q.st + 16 * kg;
  uint4v w[D / 32];
#pragma unroll
  for (int s = 0; s < D / 32; ++s) w[s] = there ? *reinterpret_cast<const uint4v*>(p + (s >> 1) * 64 + (s & 1) * 8) : uint4v{0, 0, 0, 0};
  if constexpr (!BF) {
#pragma unroll
    for (int s = 0; s < D / 32; ++s) q[s] = __builtin_bit_cast(half8v, w[s]);
    return a.scale_log2;
  } else {
    float amax = 0.f;
#pragma unroll
    for (int s = 0; s < D / 32; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(__uint_as_float(e & 1 ? w[s][e / 2] & 0xffff0000u : w[s][e / 2] << 16)));
    amax = fmaxf(amax, __shfl_xor(amax, 16, 64));
    amax = fmaxf(amax, __shfl_xor(amax, 32, 64));
    const int e2 = amax > 0.f ? 15 - __builtin_amdgcn_frexp_expf(amax) : 0;  // (an infinity or NaN: frexp gives 0)
#pragma unroll
    for (int s = 0; s < D / 32; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        q[s][e] = (_Float16)ldexpf(__uint_as_float(e & 1 ? w[s][e / 2] & 0xffff0000u : w[s][e / 2] << 16), e2);
    return ldexpf(a.scale_log2, -e2);
  }
}

// key codes of a block as the first operand: tile j = tokens 16 j .. 16 j + 15, lane 16 kg + n: token 16 j + n
template <int D>
struct KeyCodes {
  uint4v w[4][D / 64];
  __device__ __forceinline__ void load(const uint8_t* p) {
    const int lane = threadIdx.x & 63, kg = lane >> 4, n = lane & 15;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int s = 0; s < D / 64; ++s) w[j][s] = *reinterpret_cast<const uint4v*>(p + (16 * j + n) * D + s * 64 + kg * 16);
  }
  template <int CODE>
  __device__ __forceinline__ half8v operand(int j, int ks) const {
    half2v a, b, c, d;
    to_half4<CODE>(w[j][ks >> 1][2 * (ks & 1)], a, b);
    to_half4<CODE>(w[j][ks >> 1][2 * (ks & 1) + 1], c, d);
    return half8v{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
  }
};

// Value codes of a block: lane 16 kg + n holds the cells n of the tokens 32 s + 16 half + 4 kg + 0 .. 3, the order in which the
// score product leaves the weights of those tokens in lane group kg.  Channel m n + i of them (m = D / 16) is one operand.
template <int D>
struct ValueCodes {
  static constexpr int kTok = 256 / D, kCellsOf4 = 4 / kTok;  // cells of four tokens
  uint4v w[2][2][kCellsOf4];
  __device__ __forceinline__ void load(const uint8_t* p) {
    const int lane = threadIdx.x & 63, kg = lane >> 4, n = lane & 15;
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int c = 0; c < kCellsOf4; ++c)
          w[s][f][c] = *reinterpret_cast<const uint4v*>(p + ((32 * s + 16 * f + 4 * kg) / kTok + c) * 256 + n * 16);
  }
  // places behind the last token may hold anything, a NaN among it, and 0 * NaN is one: zeros there
  __device__ __forceinline__ void clear_from(int live) {
    const int kg = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int t = 0; t < 4; ++t)
          if (32 * s + 16 * f + 4 * kg + t >= live) {
#pragma unroll
            for (int e = 0; e < 4 / kTok; ++e) w[s][f][t / kTok][t % kTok * (4 / kTok) + e] = 0;
          }
  }
  // operands of channels 2 c2, 2 c2 + 1 of the cells for tokens 32 s .. 32 s + 31
  template <int CODE>
  __device__ __forceinline__ void operands(int s, int c2, half8v& x, half8v& y) const {
    half2v a[4], b[4];
#pragma unroll
    for (int f = 0; f < 2; ++f)
#pragma unroll
      for (int pair = 0; pair < 2; ++pair) {
        const int t = 2 * pair;
        const unsigned u = w[s][f][t / kTok][t % kTok * (4 / kTok) + c2 / 2];
        const unsigned v = w[s][f][(t + 1) / kTok][(t + 1) % kTok * (4 / kTok) + c2 / 2];
        to_half4<CODE>(__builtin_amdgcn_perm(v, u, c2 & 1 ? 0x07030602u : 0x05010400u), a[2 * f + pair], b[2 * f + pair]);
      }
    x = half8v{a[0][0], a[0][1], a[1][0], a[1][1], a[2][0], a[2][1], a[3][0], a[3][1]};
    y = half8v{b[0][0], b[0][1], b[1][0], b[1][1], b[2][0], b[2][1], b[3][0], b[3][1]};
  }
};

// ---- few rows: the token axis is split -------------------------------------------------------------------
// One workgroup of four waves per (16 rows, split); the waves take the split's blocks in turn and are joined through LDS.
constexpr int kWaves = 4;

template <int D, int CODE, bool BF>
__global__ __launch_bounds__(kWaves * 64) void rows_kernel(Args a) {
  constexpr int kCh = D / 16;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, kg = lane >> 4, n = lane & 15;
  const int split = blockIdx.x % a.n_splits, unit = blockIdx.x / a.n_splits;
  const int h = unit % a.g.hkv, tile = unit / a.g.hkv, b = blockIdx.y;
  const Problem pr = problem_of(a, b);
  const int r0 = tile * 16, n_rows = pr.nq * a.g.ratio;
  if (r0 >= n_rows) return;
  const int r = r0 + n, last = min(r0 + 15, n_rows - 1);
  const int vis = r < n_rows ? visible(a, pr, r / a.g.ratio) : pr.len;
  const int vis_min = visible(a, pr, r0 / a.g.ratio), vis_max = visible(a, pr, last / a.g.ratio);
  const int blk0 = split * a.per, blk1 = min(blk0 + a.per, (vis_max + kBlock - 1) / kBlock);

  half8v q[D / 32];
  const float factor = load_queries<D, BF>(a, b, h, r, pr.nq, q);
  float m = -INFINITY, l = 0.f;
  float4v o[kCh];
#pragma unroll
  for (int i = 0; i < kCh; ++i) o[i] = float4v{0.f, 0.f, 0.f, 0.f};

  for (int blk = blk0 + wave; blk < blk1; blk += kWaves) {
    const int64_t pk = block_place(a.g, a.kc.block_table, b, h, blk), pv = block_place(a.g, a.vc.block_table, b, h, blk);
    if (pk < 0 || pv < 0) continue;
    KeyCodes<D> kw;
    ValueCodes<D> vw;
    kw.load(a.kc.codes + pk * (int64_t)(kBlock * D));
    vw.load(a.vc.codes + pv * (int64_t)(kBlock * D));
    const float f = factor * a.kc.scales[pk], sv = a.vc.scales[pv];
    const int t0 = blk * kBlock;
    if (CODE == NSN_Q8_E4M3 && t0 + kBlock > pr.len) vw.clear_from(pr.len - t0);

    float4v s[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      s[j] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < D / 32; ++ks)
        s[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kw.template operand<CODE>(j, ks), q[ks], s[j], 0, 0, 0);
    }
    float top = -INFINITY;
    const bool masked = t0 + kBlock > vis_min;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[j][e] *= f;
        if (masked && t0 + 16 * j + 4 * kg + e >= vis) s[j][e] = -INFINITY;
        top = fmaxf(top, s[j][e]);
      }
    top = fmaxf(top, __shfl_xor(top, 16, 64));
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    const float m_new = fmaxf(m, top), base = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = fast_exp2(m - base);
    m = m_new;
    l *= alpha;
    half8v p[2];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = fast_exp2(s[j][e] - base);
        l += x;
        p[j >> 1][4 * (j & 1) + e] = (_Float16)x;
      }
#pragma unroll
    for (int c2 = 0; c2 < kCh / 2; ++c2) {
      float4v u = {0.f, 0.f, 0.f, 0.f}, v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        half8v x, y;
        vw.template operands<CODE>(st, c2, x, y);
        u = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, p[st], u, 0, 0, 0);
        v = __builtin_amdgcn_mfma_f32_16x16x32_f16(y, p[st], v, 0, 0, 0);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        o[2 * c2][e] = fmaf(sv, u[e], o[2 * c2][e] * alpha);
        o[2 * c2 + 1][e] = fmaf(sv, v[e], o[2 * c2 + 1][e] * alpha);
      }
    }
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);

  // join the four waves: row n of wave w, channels kCh * (4 kg + e) + i
  constexpr int kStride = D + 4;  // (16-byte rows, the 16 rows of a wave on different banks)
  __shared__ float sm_o[kWaves][16][kStride];
  __shared__ float sm_m[kWaves][16], sm_l[kWaves][16];
  if (kg == 0) sm_m[wave][n] = m, sm_l[wave][n] = l;
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int i = 0; i < kCh; ++i) sm_o[wave][n][kCh * (4 * kg + e) + i] = o[i][e];
  __syncthreads();
  // 16 threads per row, D / 16 channels each
  const int row = tid >> 4, c0 = (tid & 15) * kCh;
  if (r0 + row >= n_rows) return;
  float M = -INFINITY, L = 0.f, acc[kCh];
#pragma unroll
  for (int i = 0; i < kCh; ++i) acc[i] = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) M = fmaxf(M, sm_m[w][row]);
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const float e = sm_m[w][row] == -INFINITY && M == -INFINITY ? 0.f : fast_exp2(sm_m[w][row] - M);
    L = fmaf(e, sm_l[w][row], L);
#pragma unroll
    for (int i = 0; i < kCh; ++i) acc[i] = fmaf(e, sm_o[w][row][c0 + i], acc[i]);
  }
  const int64_t line = ((int64_t)b * a.g.hkv + h) * a.rows + r0 + row;
  if (a.n_splits > 1) {
    float* P = a.partial + (line * a.n_splits + split) * (D + 2);
#pragma unroll
    for (int i = 0; i < kCh; ++i) P[c0 + i] = acc[i];
    if (c0 == 0) P[D] = M, P[D + 1] = L;
    return;
  }
  const int i_q = (r0 + row) / a.g.ratio, hq = h * a.g.ratio + (r0 + row) % a.g.ratio;
  const int64_t place = ((int64_t)b * a.n_q + i_q) * a.g.hq + hq;
  const float inv = L > 0.f ? 1.0f / L : (L == 0.f ? 0.f : L);
#pragma unroll
  for (int i = 0; i < kCh; ++i) a.out[place * D + c0 + i] = from_float<BF>(acc[i] * inv);
  if (c0 == 0) {
    const float z = L == 0.f ? -INFINITY : M + __log2f(L);
    if (a.lse) a.lse[place] = z * kLn2;
    if (a.lse2) a.lse2[line] = z;
  }
}

// the splits of a row are joined: one workgroup of D threads per row
template <int D, bool BF>
__global__ __launch_bounds__(D) void merge_kernel(Args a) {
  const int r = blockIdx.x / a.g.hkv, h = blockIdx.x % a.g.hkv, b = blockIdx.y, c = threadIdx.x;
  const Problem pr = problem_of(a, b);
  if (r >= pr.nq * a.g.ratio) return;
  const int64_t line = ((int64_t)b * a.g.hkv + h) * a.rows + r;
  const float* P = a.partial + line * a.n_splits * (D + 2);
  float M = -INFINITY, L = 0.f, acc = 0.f;
  for (int s = 0; s < a.n_splits; ++s) M = fmaxf(M, P[s * (D + 2) + D]);
  for (int s = 0; s < a.n_splits; ++s) {
    const float ms = P[s * (D + 2) + D];
    const float e = ms == -INFINITY && M == -INFINITY ? 0.f : fast_exp2(ms - M);
    L = fmaf(e, P[s * (D + 2) + D + 1], L);
    acc = fmaf(e, P[s * (D + 2) + c], acc);
  }
  const int64_t place = ((int64_t)b * a.n_q + r / a.g.ratio) * a.g.hq + h * a.g.ratio + r % a.g.ratio;
  const float inv = L > 0.f ? 1.0f / L : (L == 0.f ? 0.f : L);
  a.out[place * D + c] = from_float<BF>(acc * inv);
  if (c == 0) {
    const float z = L == 0.f ? -INFINITY : M + __log2f(L);
    if (a.lse) a.lse[place] = z * kLn2;
    if (a.lse2) a.lse2[line] = z;
  }
}

// ---- the weights that each cached token receives ----------------------------------------------------------
// One workgroup per 64-token block and kv head: the block's keys stay in registers, its waves go through the rows 16 at a
// time, add 2^(s - lse) up per token, and are joined in a fixed order.
template <int D, int CODE, bool BF>
__global__ __launch_bounds__(kWaves * 64) void weights_kernel(Args a) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, kg = lane >> 4, n = lane & 15;
  const int blk = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const Problem pr = problem_of(a, b);
  const int t0 = blk * kBlock, n_rows = pr.nq * a.g.ratio;
  if (t0 >= pr.len) return;
  const int64_t pk = block_place(a.g, a.kc.block_table, b, h, blk), pv = block_place(a.g, a.vc.block_table, b, h, blk);
  float4v sum[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) sum[j] = float4v{0.f, 0.f, 0.f, 0.f};
  if (pk >= 0 && pv >= 0) {
    KeyCodes<D> kw;
    kw.load(a.kc.codes + pk * (int64_t)(kBlock * D));
    const float sk = a.kc.scales[pk];
    for (int r0 = wave * 16; r0 < n_rows; r0 += kWaves * 16) {
      if (visible(a, pr, min(r0 + 15, n_rows - 1) / a.g.ratio) <= t0) continue;
      const int r = r0 + n;
      half8v q[D / 32];
      const float f = load_queries<D, BF>(a, b, h, r, pr.nq, q) * sk;
      const float z = r < n_rows ? a.lse2[((int64_t)b * a.g.hkv + h) * a.rows + r] : INFINITY;
      const int vis = r < n_rows ? visible(a, pr, r / a.g.ratio) : 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float4v s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks) s = __builtin_amdgcn_mfma_f32_16x16x32_f16(kw.template operand<CODE>(j, ks), q[ks], s, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[j][e] += t0 + 16 * j + 4 * kg + e < vis ? fast_exp2(fmaf(s[e], f, -z)) : 0.f;
      }
    }
  }
  // over the 16 rows of a tile, then over the waves
  __shared__ float sm[kWaves][kBlock];
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x = xor_sum_w<16>(sum[j][e]);
      if (n == 0) sm[wave][16 * j + 4 * kg + e] = x;
    }
  __syncthreads();
  if (tid < kBlock && t0 + tid < pr.len) {
    const int64_t at = ((int64_t)b * a.g.hkv + h) * a.g.max_len + t0 + tid;
    const float x = (sm[0][tid] + sm[1][tid]) + (sm[2][tid] + sm[3][tid]);
    a.weights_out[at] = a.weights_in ? a.weights_in[at] + x : x;
  }
}

// ---- host side --------------------------------------------------------------------------------------------
static int split_count(const nsn_q8_shape& s, int batch, int n_q, int max_seq_len, int requested) {
  const int blocks = std::max(1, (max_seq_len + kBlock - 1) / kBlock);
  if (requested > 0) return std::min(requested, blocks);
  const int64_t rows = (int64_t)n_q * (s.n_q_heads / s.n_kv_heads), groups = (rows + 15) / 16 * s.n_kv_heads * batch;
  const int64_t most = (blocks + kWaves - 1) / kWaves;
  return (int)std::max<int64_t>(1, std::min<int64_t>(most, 1024 / groups));
}

static int64_t lines(const nsn_q8_shape& s, int batch, int n_q) { return (int64_t)batch * n_q * s.n_q_heads; }
static size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }

size_t attention_workspace_bytes(const nsn_q8_shape& s, int batch, int n_q, int max_seq_len, int n_splits) {
  const int splits = split_count(s, batch, n_q, max_seq_len, n_splits);
  const size_t rows = (size_t)lines(s, batch, n_q);
  return up16(rows * sizeof(float)) + (splits > 1 ? rows * splits * (s.head_dim + 2) * sizeof(float) : 0);
}

int attention_launch(const AttentionCall& c) {
  const nsn_q8_shape& s = c.shape;
  Args a;
  a.g = make_geometry(s);
  a.q = make_rows(c.q);
  a.n_q = c.n_q, a.rows = c.n_q * a.g.ratio, a.q_lens = c.q_lens;
  a.kc = make_view(c.kc), a.vc = make_view(c.vc);
  a.seq_lens = c.seq_lens, a.max_seq_len = c.max_seq_len;
  a.scale_log2 = c.scale * kLog2e, a.causal = c.causal;
  a.n_splits = split_count(s, c.batch, c.n_q, c.max_seq_len, c.n_splits);
  const int blocks = std::max(1, (c.max_seq_len + kBlock - 1) / kBlock);
  a.per = (blocks + a.n_splits - 1) / a.n_splits;
  a.out = static_cast<uint16_t*>(c.out), a.lse = c.lse;
  a.lse2 = static_cast<float*>(c.workspace);
  a.partial = reinterpret_cast<float*>(static_cast<unsigned char*>(c.workspace) + up16(lines(s, c.batch, c.n_q) * sizeof(float)));
  a.weights_in = c.weights_in, a.weights_out = c.weights_out;
  return with_types(s, [&](auto d, auto code, auto bf) -> int {
    constexpr int D = decltype(d)::value, CODE = decltype(code)::value;
    constexpr bool BF = decltype(bf)::value;
    const int tiles = (a.rows + 15) / 16;
    if ((int64_t)tiles * a.g.hkv * a.n_splits > 0x7fffffff || (int64_t)a.rows * a.g.hkv > 0x7fffffff) {
      set_error("q8_attention: n_q * n_q_heads * n_splits is too large for one launch");
      return NSN_ERR_UNSUPPORTED;
    }
    rows_kernel<D, CODE, BF><<<dim3(tiles * a.g.hkv * a.n_splits, c.batch), kWaves * 64, 0, c.stream>>>(a);
    if (hipGetLastError() != hipSuccess) return NSN_ERR_HIP;
    if (a.n_splits > 1) {
      merge_kernel<D, BF><<<dim3(a.rows * a.g.hkv, c.batch), D, 0, c.stream>>>(a);
      if (hipGetLastError() != hipSuccess) return NSN_ERR_HIP;
    }
    if (a.weights_out && c.max_seq_len > 0) {
      weights_kernel<D, CODE, BF><<<dim3(blocks, a.g.hkv, c.batch), kWaves * 64, 0, c.stream>>>(a);
      if (hipGetLastError() != hipSuccess) return NSN_ERR_HIP;
    }
    return NSN_OK;
  });
}

}  // namespace q8
}  // namespace nsn
