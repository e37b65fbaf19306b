// Attention over the 8-bit cache (nsn_q8_attention): single tokens and chunks, and the weights that each cached token receives.
//
// Rows.  The queries of a (sequence, kv head) are taken as rows r = i * ratio + g (token i, query head g of the kv head): all of
// them read the same keys and values, so a row is the unit of work and grouped heads cost no second reading of the cache.
//
// Per 64-token block, with codes k, v and scales sk, sv:
//   s = (q . k) * (softmax_scale log2 e sk),  m' = max(m, max s),  p = 2^(s - m'),  l = l 2^(m - m') + sum p,
//   o = o 2^(m - m') + sv (p . v)
// Codes become fp16 without loss (int8 and e4m3 both fit), so q . k is exact up to fp32 accumulation; p is rounded to fp16 (half a
// step 2^-11, as much as the output where that is fp16) for the second product.  bf16 queries are multiplied by a power of two
// per row that brings their largest magnitude to 2^14 .. 2^15, and are then fp16 numbers (values 2^-38 below the largest and
// smaller lose their last bits, which fp32 sums would not keep either).
#include <algorithm>
#include <type_traits>

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
  int batch;
  int n_runs, per;  // runs, and the fewest blocks of one
  int direct;       // instead: a unit to each workgroup
  uint16_t* out;
  float* lse;
  float* lse2;     // [batch][hkv][rows], in powers of two (workspace)
  float* partial;  // [run][2][a tile's sums] (workspace)
  int* counters;   // of the unit that goes on behind a run, one per 64 bytes: runs that have arrived (workspace)
  int row_tiles;
  float* scores;   // [batch][hkv][rows][score_stride] in powers of two, -infinity where nothing is seen (workspace), or NULL
  int64_t score_stride;
  int weight_parts;  // of the rows, in the pass that adds weights up
  const float* weights_in;
  float* weights_out;
};

constexpr int kWaves = 4;
constexpr int kCounterInts = 16, kMaxCounters = 2048;  // (the workspace starts with them, in every call's layout)

constexpr float kMasked = -1e30f;  // the score of a token that is not seen (finite: a factor of it may be 0)

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

// the wave's number in a scalar register, so that what follows from it is worked out once per wave
__device__ __forceinline__ int wave_index() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Rows of queries as fp16 operands: w holds this lane's pieces of one row, whose other pieces lie in the lanes LANES apart.  Returns the
// factor (not negative: a negative softmax scale turns the row's signs) that takes q . k to a power of two.
template <bool BF, int N, int LANES>
__device__ __forceinline__ float query_operands(float scale, uint4v (&w)[N], half8v (&q)[N]) {
  if (scale < 0.f) {
#pragma unroll
    for (int s = 0; s < N; ++s) w[s] ^= 0x80008000u;
    scale = -scale;
  }
  if constexpr (!BF) {
#pragma unroll
    for (int s = 0; s < N; ++s) q[s] = __builtin_bit_cast(half8v, w[s]);
    return scale;
  } else {
    float amax = 0.f;
#pragma unroll
    for (int s = 0; s < N; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(__uint_as_float(e & 1 ? w[s][e / 2] & 0xffff0000u : w[s][e / 2] << 16)));
#pragma unroll
    for (int d = LANES; d < 64; d *= 2) amax = fmaxf(amax, __shfl_xor(amax, d, 64));
    const int e2 = amax > 0.f ? 15 - __builtin_amdgcn_frexp_expf(amax) : 0;  // (an infinity or NaN: frexp gives 0)
#pragma unroll
    for (int s = 0; s < N; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        q[s][e] = (_Float16)ldexpf(__uint_as_float(e & 1 ? w[s][e / 2] & 0xffff0000u : w[s][e / 2] << 16), e2);
    return ldexpf(scale, -e2);
  }
}

// The 16 rows r0 .. r0 + 15 as the second operand of the 16x16x32 products: lane 16 kg + n holds row n, and of every 64
// channels the 16 from 16 kg on, which is how a lane reads a row of key codes in 16-byte pieces (the order of the channels in
// a product is free as long as both operands share it).
template <int D, bool BF>
__device__ __forceinline__ float load_queries(const Args& a, int b, int h, int r, int nq, half8v (&q)[D / 32]) {
  const int kg = (threadIdx.x & 63) >> 4;
  const bool there = r < nq * a.g.ratio;
  const int i = there ? r / a.g.ratio : 0, hq = there ? h * a.g.ratio + r % a.g.ratio : 0;
  const uint16_t* p = a.q.data + b * a.q.sb + hq * a.q.sh + i * a.q.st + 16 * kg;
  uint4v w[D / 32];
#pragma unroll
  for (int s = 0; s < D / 32; ++s) w[s] = there ? *reinterpret_cast<const uint4v*>(p + (s >> 1) * 64 + (s & 1) * 8) : uint4v{0, 0, 0, 0};
  return query_operands<BF, D / 32, 16>(a.scale_log2, w, q);
}

// The same for the 32x32x16 products: row r in lanes n and 32 + n, channels 16 s + 8 (lane / 32) + 0 .. 7 in operand s.
template <int D, bool BF>
__device__ __forceinline__ float load_query_rows(const Args& a, int b, int h, int r, int nq, half8v (&q)[D / 16]) {
  const bool there = r < nq * a.g.ratio;
  const int i = there ? r / a.g.ratio : 0, hq = there ? h * a.g.ratio + r % a.g.ratio : 0;
  const uint16_t* p = a.q.data + b * a.q.sb + hq * a.q.sh + i * a.q.st + 8 * ((threadIdx.x & 63) >> 5);
  uint4v w[D / 16];
#pragma unroll
  for (int s = 0; s < D / 16; ++s) w[s] = there ? *reinterpret_cast<const uint4v*>(p + 16 * s) : uint4v{0, 0, 0, 0};
  return query_operands<BF, D / 16, 32>(a.scale_log2, w, q);
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

// ---- few rows -------------------------------------------------------------------
// Units of 16 rows.  The four waves of a workgroup take a segment's blocks in turn, each with the next block's codes on their way
// to registers while it works on one, and are joined through LDS.  Bound by memory: every code is read once, and the
// conversions and products of a block fill a third of the time that its bytes take (32 query over 8 kv heads: 8 sequences of 8192
// tokens 32.5 us, 4.1 TB/s; 32 of 512 to 16384, paged, e4m3 102 us, 4.7 TB/s, where a large copy reaches 5.2).

template <int D>
struct Fetched {
  KeyCodes<D> k;
  ValueCodes<D> v;
  float sk, sv;
  bool there;
};

// ---- the running maximum and the values' scale ------------------------------------------------------------
// The output accumulates in the matrix registers from block to block without a pass over it:
//   - a row's running maximum m is moved (and its sums rescaled) only when its scores pass it by 2^kLazy (few rows), or where
//     their weights under it add up to kMost in a lane (many rows: no maximum is taken of most tiles);
//   - a block's value scale sv enters the exponent, p' = 2^(s - m + kLift + log2(sv / sref)), against a power of two sref that
//     follows sv when it is off by more than 2^kSpan.  p' stays below 2^(kLift + kLazy + kSpan + 1) <= 2^15, or kMost, where fp16 ends
//     at 65504; weights down to 2^-20 of the one at m are normal fp16 numbers.
// Then sum p v = sref / 2^kLift * (what o holds), sum p = l / 2^kLift with l += (sum p') * (sref / sv).  The output is divided by the sum
// of the weights as they were rounded (lr), so that a token that holds nearly all of the weight comes out exact; lse goes by l.
constexpr int kLazy = 4, kSpan = 4, kLift = 6;
constexpr float kMost = 60000.f;

// moves a row's maximum to m_new
template <int N, typename V>
__device__ __forceinline__ void move_maximum(float m_new, float& m, float& l, float& lr, V (&o)[N]) {
  const float alpha = m == m_new ? 1.f : fast_exp2(m - m_new);
  m = m_new;
  l *= alpha, lr *= alpha;
#pragma unroll
  for (int i = 0; i < N; ++i) o[i] *= alpha;
}
// ratio = sref / sv, lift = kLift + log2(sv / sref) for a block
template <int N, typename V>
__device__ __forceinline__ void follow_scale(float sv, float& sref, V (&o)[N], float& ratio, float& lift) {
  ratio = 1.f, lift = kLift;
  if (sv > 0.f) {
    // (a jump of more than 2^60 downwards would take the sums out of range: weights that small count as they underflow)
    if (!(sv <= sref * (1 << kSpan) && sv * (1 << kSpan) >= sref) && !(sv < sref * 0x1p-60f)) {
      const float now = ldexpf(0.5f, __builtin_amdgcn_frexp_expf(sv));
      const float turn = sref > 0.f ? sref / now : 0.f;
      sref = now;
#pragma unroll
      for (int i = 0; i < N; ++i) o[i] *= turn;
    }
    // (sref is a power of two, and sv / sref a normal number: the instructions themselves will do, half a dozen of them for two dozen)
    const float inv_sv = __builtin_amdgcn_rcpf(sv);
    ratio = sref * inv_sv;
    lift = kLift - __builtin_amdgcn_logf(ratio);
  }
}

// adds a block's weights up: exact and as rounded
__device__ __forceinline__ float add_rounded(half2v p, float sum) { return __builtin_amdgcn_fdot2(p, half2v{(_Float16)1.f, (_Float16)1.f}, sum, false); }
__device__ __forceinline__ void add_weights(float sum, float rounded, float ratio, float& l, float& lr) {
  l = fmaf(sum, ratio, l);
  lr = fmaf(ratio > 0x1p59f ? sum : rounded, ratio, lr);  // (values so far below the others that the weights underflow: they count all the same)
}

// ---- the list of the work --------------------------------------------------------------------------------
// A unit is a tile of TILE rows of a (sequence, kv head); the list holds the 64-token blocks of all units in the order (sequence,
// head, tile).  It is cut into equal runs, one workgroup each, whatever the sequences' lengths: all workgroups end at about
// the same time, where a grid over units and splits leaves a last round that few take part in.  A run is a few segments, each of one
// unit.  A unit that reaches into other runs leaves partial sums, which the last workgroup to arrive joins.
template <int TILE>
struct Cursor {
  int b, h, tile, cost;  // the unit, and its blocks in the list
  Problem pr;
  int run, per, at, pos, end;  // at: where the unit begins; pos, end: what is left of the run

  // a unit's blocks, and one where its rows see nothing (they are written too); no rows: nothing
  static __device__ __forceinline__ int cost_of(const Args& a, const Problem& p, int tile) {
    const int n_rows = p.nq * a.g.ratio;
    if (tile * TILE >= n_rows) return 0;
    return max(1, (visible(a, p, min(tile * TILE + TILE - 1, n_rows - 1) / a.g.ratio) + kBlock - 1) / kBlock);
  }
  // 64 / K sequences from b0 on, K lanes to each: what a lane's tiles of one head come to
  static __device__ __forceinline__ int lane_cost(const Args& a, int b, int j, int K) {
    if (b >= a.batch) return 0;
    const Problem p = problem_of(a, b);
    if (!a.causal) return j == 0 ? (p.nq * a.g.ratio + TILE - 1) / TILE * cost_of(a, p, 0) : 0;
    int c = 0;
    for (int t = j; t < a.row_tiles; t += K) c += cost_of(a, p, t);
    return c;
  }

  // the run of this workgroup; false: there is none
  __device__ __forceinline__ bool begin(const Args& a, int index) {
    const int lane = threadIdx.x & 63;
    run = index;
    if (a.direct) {  // more units than runs could be useful: one to each workgroup, the last tiles (the longest) first
      h = index % a.g.hkv;
      const int item = index / a.g.hkv;
      b = item % a.batch, tile = a.row_tiles - 1 - item / a.batch;
      pr = problem_of(a, b);
      cost = cost_of(a, pr, tile);
      at = pos = 0, per = end = max(cost, 1), run = 0;
      return cost > 0;
    }
    int shift = 0;  // K = 1 << shift lanes to a sequence
    while ((a.batch << (shift + 1)) <= 64) ++shift;
    const int K = 1 << shift, step = 64 >> shift;
    int scan = 0, total = 0;
    for (int b0 = 0; b0 < a.batch; b0 += step) {
      scan = wave_scan(lane_cost(a, b0 + (lane >> shift), lane & (K - 1), K));
      total += __builtin_amdgcn_readlane(scan, 63);
    }
    total *= a.g.hkv;
    per = max(a.per, (total + a.n_runs - 1) / a.n_runs);
    pos = run * per;
    if (pos >= total) return false;  // (also where no sequence has a query)
    end = min(pos + per, total);
    int before = 0;  // one head's blocks of the sequences before
    for (int b0 = 0;; b0 += step) {
      if (a.batch > step) scan = wave_scan(lane_cost(a, b0 + (lane >> shift), lane & (K - 1), K));
      const unsigned long long found = __ballot((lane & (K - 1)) == K - 1 && (before + scan) * a.g.hkv > pos);
      if (found) {
        const int k = __ffsll(found) - 1;  // the last lane of the sequence
        b = b0 + (k >> shift);
        const int upto = __builtin_amdgcn_readlane(scan, k), from = k >= K ? __builtin_amdgcn_readlane(scan, k - K) : 0;
        at = (before + from) * a.g.hkv;
        h = (pos - at) / (upto - from);
        at += h * (upto - from);
        break;
      }
      before += __builtin_amdgcn_readlane(scan, 63);
    }
    pr = problem_of(a, b);
    for (int t0 = 0;; t0 += 64) {
      const int c = cost_of(a, pr, t0 + lane), upto = wave_scan(c);
      const unsigned long long found = __ballot(at + upto > pos);
      if (found) {
        const int k = __ffsll(found) - 1;
        tile = t0 + k, cost = __builtin_amdgcn_readlane(c, k);
        at += __builtin_amdgcn_readlane(upto, k) - cost;
        break;
      }
      at += __builtin_amdgcn_readlane(upto, 63);
    }
    return true;
  }
  // blocks of the unit that belong to this run: [first, last)
  __device__ __forceinline__ int first() const { return pos - at; }
  __device__ __forceinline__ int last() const { return min(cost, end - at); }
  // the runs that the unit reaches into
  __device__ __forceinline__ int first_run() const { return at / per; }
  __device__ __forceinline__ int runs() const { return (at + cost - 1) / per - at / per + 1; }
  // the next unit of the run; false: the run is done
  __device__ __forceinline__ bool next(const Args& a) {
    pos = at + last();
    if (pos >= end) return false;
    at = pos;
    cost = cost_of(a, pr, ++tile);
    if (cost == 0) {
      tile = 0;
      if (++h == a.g.hkv) h = 0, pr = problem_of(a, ++b);
      while ((cost = cost_of(a, pr, 0)) == 0) pr = problem_of(a, ++b);  // (pos < total: a unit follows)
    }
    return true;
  }
};

__device__ __forceinline__ void store_agent(float* p, float x, float y) {  // 8-byte device-scope store (p is 8-byte aligned)
  __hip_atomic_store(reinterpret_cast<unsigned long long*>(p), ((unsigned long long)__float_as_uint(y) << 32) | __float_as_uint(x),
                     __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2v load_agent(const float* p) {
  const unsigned long long u = __hip_atomic_load(reinterpret_cast<const unsigned long long*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return float2v{__uint_as_float((unsigned)u), __uint_as_float((unsigned)(u >> 32))};
}
// Counts the workgroup in at a counter that `of` workgroups come to; whether it is the last of them.  The partials are device-scope
// stores, which no cache holds back; each wave waits until its own are acknowledged, then one thread counts, and the workgroup that
// counts last reads all partials with device-scope loads.  Nobody waits for anybody else.
// A run is the first of one unit that goes on behind it at most, and a later one of one other, so run numbers name the counters:
// kind 0 and 1 by a unit's first run, kind 2 by a later one.
__device__ __forceinline__ bool arrives_last(const Args& a, int kind, int run, int of, int& arrived) {
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  if (threadIdx.x == 0) {
    int* cnt = a.counters + (kind * kMaxCounters + run) * kCounterInts;
    arrived = __hip_atomic_fetch_add(cnt, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (arrived == of - 1) __hip_atomic_store(cnt, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // ready for the next call
  }
  __syncthreads();
  return arrived == of - 1;
}
// factor of a part whose maximum is m in a sum under the maximum M
__device__ __forceinline__ float part_factor(float m, float M) { return m == -INFINITY ? 0.f : fast_exp2(m - M); }

// one row's result: thread n of 16 holds channels 32 i + 2 n, 32 i + 2 n + 1 (acc: sums under the total L, R as rounded)
template <int D, bool BF>
__device__ __forceinline__ void write_row(const Args& a, int b, int h, int r, int n, float M, float L, float R, const float2v (&acc)[D / 32]) {
  const int64_t place = ((int64_t)b * a.n_q + r / a.g.ratio) * a.g.hq + h * a.g.ratio + r % a.g.ratio;
  const float inv = R > 0.f ? 1.0f / R : (R == 0.f ? 0.f : R);
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
    *reinterpret_cast<unsigned*>(a.out + place * D + 32 * i + 2 * n) =
        (unsigned)from_float<BF>(acc[i][0] * inv) | (unsigned)from_float<BF>(acc[i][1] * inv) << 16;
  if (n == 0) {
    const float z = L == 0.f ? -INFINITY : M + __log2f(L);
    if (a.lse) a.lse[place] = z * kLn2;
    a.lse2[((int64_t)b * a.g.hkv + h) * a.rows + r] = z;
  }
}

template <int D, int CODE, bool BF>
__global__ __launch_bounds__(kWaves * 64, 2) void rows_kernel(Args a) {
  constexpr int kCh = D / 16;
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_index(), kg = lane >> 4, n = lane & 15;
  Cursor<16> cur;
  if (!cur.begin(a, blockIdx.x)) return;
  constexpr int kStride = D + 4, kPairs = D / 32;
  __shared__ __attribute__((aligned(16))) float sm_o[kWaves][16][kStride];
  __shared__ float sm_m[kWaves][16], sm_l[kWaves][16], sm_r[kWaves][16];
  __shared__ int arrived;
  do {  // segments
  const int b = cur.b, h = cur.h;
  const Problem pr = cur.pr;
  const int n_rows = pr.nq * a.g.ratio, r0 = cur.tile * 16, r = r0 + n;
  const int vis_min = visible(a, pr, r0 / a.g.ratio), blocks = (visible(a, pr, min(r0 + 15, n_rows - 1) / a.g.ratio) + kBlock - 1) / kBlock;
  const int vis = r < n_rows ? visible(a, pr, r / a.g.ratio) : pr.len;
  const int blk0 = cur.first(), blk1 = min(blocks, cur.last()), first_run = cur.first_run(), live = cur.runs();
  const int64_t line0 = ((int64_t)b * a.g.hkv + h) * a.rows + r0;

  int64_t next_k = 0, next_v = 0;
  auto look_up = [&](int blk) {  // (a block ahead of its loads, so that these do not wait for the page tables)
    next_k = block_place<true>(a.g, a.kc.block_table, b, h, blk), next_v = block_place<true>(a.g, a.vc.block_table, b, h, blk);
  };
  auto fetch = [&](Fetched<D>& x) {  // (always loads: block 0 of the cache in the place of one that is not there)
    int64_t pk = next_k, pv = next_v;
    x.there = pk >= 0 && pv >= 0;
    if (!x.there) pk = pv = 0;
    x.k.load(a.kc.codes + pk * (int64_t)(kBlock * D));
    x.v.load(a.vc.codes + pv * (int64_t)(kBlock * D));
    x.sk = load_uniform(a.kc.scales + pk), x.sv = load_uniform(a.vc.scales + pv);
  };
  half8v q[D / 32];
  float factor = 0.f, m = -INFINITY, l = 0.f, lr = 0.f, sref = 0.f;
  float4v o[kCh];
#pragma unroll
  for (int i = 0; i < kCh; ++i) o[i] = float4v{0.f, 0.f, 0.f, 0.f};

  auto work = [&](Fetched<D>& x, int blk) {
    const int t0 = blk * kBlock;
    float* sc = a.scores ? a.scores + (line0 + n) * a.score_stride + t0 + 4 * kg : nullptr;
    if (!x.there) {
      if (sc && r < n_rows) {
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<float4v*>(sc + 16 * j) = float4v{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
      }
      return;
    }
    if (CODE == NSN_Q8_E4M3 && t0 + kBlock > pr.len) x.v.clear_from(pr.len - t0);
    const float f = factor * x.sk;
    float4v s[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      s[j] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < D / 32; ++ks)
        s[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x.k.template operand<CODE>(j, ks), q[ks], s[j], 0, 0, 0);
    }
    const bool masked = t0 + kBlock > vis_min;
    if (masked) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (t0 + 16 * j + 4 * kg + e >= vis) s[j][e] = kMasked;
    }
    if (sc && r < n_rows) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float4v y = s[j] * f;
        if (masked) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (t0 + 16 * j + 4 * kg + e >= vis) y[e] = -INFINITY;
        }
        *reinterpret_cast<float4v*>(sc + 16 * j) = y;
      }
    }
    float top = s[0][0];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) top = fmaxf(top, s[j][e]);
    top = fmaxf(top, xor_lane<16>(top));
    top = fmaxf(top, xor_lane<32>(top)) * f;
    if (__any(top > m + kLazy)) move_maximum<kCh>(top > m + kLazy ? top : m, m, l, lr, o);  // (each row by its own scores)
    float ratio, lift;
    follow_scale<kCh>(x.sv, sref, o, ratio, lift);
    const float base = m - lift;
    float sum = 0.f, rounded = 0.f;
    half8v p[2];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[j][e] = fast_exp2(fmaf(s[j][e], f, -base));
    if (masked) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (t0 + 16 * j + 4 * kg + e >= vis) s[j][e] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      sum += (s[j][0] + s[j][1]) + (s[j][2] + s[j][3]);
      const half4v u = __builtin_convertvector(s[j], half4v);
      rounded = add_rounded(half2v{u[2], u[3]}, add_rounded(half2v{u[0], u[1]}, rounded));
#pragma unroll
      for (int e = 0; e < 4; ++e) p[j >> 1][4 * (j & 1) + e] = u[e];
    }
    add_weights(sum, rounded, ratio, l, lr);
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int c2 = 0; c2 < kCh / 2; ++c2) {
        half8v y, z;
        x.v.template operands<CODE>(st, c2, y, z);
        o[2 * c2] = __builtin_amdgcn_mfma_f32_16x16x32_f16(y, p[st], o[2 * c2], 0, 0, 0);
        o[2 * c2 + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(z, p[st], o[2 * c2 + 1], 0, 0, 0);
      }
  };
  int blk = blk0 + wave;
  if (blk < blk1) {
    Fetched<D> x, y;
    look_up(blk);
    fetch(x);
    look_up(min(blk + kWaves, blk1 - 1));
    factor = load_queries<D, BF>(a, b, h, r, pr.nq, q);
    while (true) {
      fetch(y);
      look_up(min(blk + 2 * kWaves, blk1 - 1));
      work(x, blk);
      blk += kWaves;
      if (blk >= blk1) break;
      fetch(x);
      look_up(min(blk + 2 * kWaves, blk1 - 1));
      work(y, blk);
      blk += kWaves;
      if (blk >= blk1) break;
    }
  }
  l += xor_lane<16>(l), lr += xor_lane<16>(lr);
  l += xor_lane<32>(l), lr += xor_lane<32>(lr);

  // join the four waves: row n of wave w, channels kCh * (4 kg + e) + i; sums under 2^(m - kLift)
  if (kg == 0) sm_m[wave][n] = l == 0.f ? -INFINITY : m - kLift, sm_l[wave][n] = l, sm_r[wave][n] = lr;
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int i = 0; i < kCh; i += 4)
      *reinterpret_cast<float4v*>(&sm_o[wave][n][kCh * (4 * kg + e) + i]) = float4v{o[i][e], o[i + 1][e], o[i + 2][e], o[i + 3][e]} * sref;
  __syncthreads();
  const int rows_here = min(16, n_rows - r0);
  // the partial of the unit's k-th run: a run has room for two, one of a unit that began before it and one of a unit that
  // begins in it and goes on behind it
  auto partial_of = [&](int k) { return a.partial + ((int64_t)(first_run + k) * 2 + (k == 0)) * 16 * (D + 4); };
  [&] {
  {
    // 16 threads per row
    const int row = tid >> 4, n16 = tid & 15;
    float M = -INFINITY, L = 0.f, R = 0.f;
    float2v acc[kPairs];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) acc[i] = float2v{0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) M = fmaxf(M, sm_m[w][row]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float e = part_factor(sm_m[w][row], M);
      L = fmaf(e, sm_l[w][row], L), R = fmaf(e, sm_r[w][row], R);
#pragma unroll
      for (int i = 0; i < kPairs; ++i) acc[i] += e * *reinterpret_cast<const float2v*>(&sm_o[w][row][32 * i + 2 * n16]);
    }
    if (live == 1) {
      if (row < rows_here) write_row<D, BF>(a, b, h, r0 + row, n16, M, L, R, acc);
      return;
    }
    if (row < rows_here) {
      float* P = partial_of(cur.run - first_run) + row * (D + 4);
#pragma unroll
      for (int i = 0; i < kPairs; ++i) store_agent(P + 32 * i + 2 * n16, acc[i][0], acc[i][1]);
      if (n16 < 2) store_agent(P + D + 2 * n16, n16 ? R : M, n16 ? 0.f : L);
    }
  }
  // Partials first, first + step, .. of the unit: all of them where they are few; of a unit that reaches into more than 64 runs,
  // sixteen at a time, whose sum takes the place of the first, and then those (one head of 71776 tokens: 27.8 us by
  // one workgroup that reads 225 partials, 17.0 us so).
  constexpr int kGroup = 16;
  const bool two = live > 4 * kGroup;
  const int part = (cur.run - first_run) / kGroup;
  int from = two ? part * kGroup : 0, n_parts = two ? min(kGroup, live - from) : live, step = 1;
  if (!arrives_last(a, two ? (part == 0 ? 1 : 2) : 0, first_run + from, n_parts, arrived)) return;
  // groups of 16 threads take (row, every G-th partial); few rows leave more groups per row, which are joined through LDS
  int shift = 0;
  while ((1 << shift) < rows_here) ++shift;
  const int group = tid >> 4, row = group & ((1 << shift) - 1), g0 = group >> shift, G = 16 >> shift, n16 = tid & 15;
  while (true) {
    float M = -INFINITY, L = 0.f, R = 0.f;
    float2v acc[kPairs];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) acc[i] = float2v{0.f, 0.f};
    auto gather = [&](auto ahead) {
      constexpr int kAhead = decltype(ahead)::value;
      for (int s0 = g0; s0 < n_parts; s0 += kAhead * G) {
        float2v ml[kAhead], lr[kAhead], x[kAhead][kPairs];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const float* ps = partial_of(from + min(s0 + k * G, n_parts - 1) * step) + row * (D + 4);
          ml[k] = load_agent(ps + D), lr[k] = load_agent(ps + D + 2);
#pragma unroll
          for (int i = 0; i < kPairs; ++i) x[k][i] = load_agent(ps + 32 * i + 2 * n16);
        }
        float m2 = M;
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
          if (s0 + k * G < n_parts) m2 = fmaxf(m2, ml[k][0]);
        const float turn = part_factor(M, m2);
        M = m2;
        L *= turn, R *= turn;
#pragma unroll
        for (int i = 0; i < kPairs; ++i) acc[i] *= turn;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const float e = s0 + k * G < n_parts ? part_factor(ml[k][0], M) : 0.f;
          L = fmaf(e, ml[k][1], L), R = fmaf(e, lr[k][0], R);
#pragma unroll
          for (int i = 0; i < kPairs; ++i) acc[i] += e * x[k][i];
        }
      }
    };
    // (a trip to memory takes 2 us, whatever is asked for)
    if (row < rows_here) n_parts > 2 * G ? gather(std::integral_constant<int, 8>{}) : gather(std::integral_constant<int, 2>{});
    float* flat = &sm_o[0][0][0];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) *reinterpret_cast<float2v*>(flat + group * kStride + 32 * i + 2 * n16) = acc[i];
    float *ms = &sm_m[0][0], *ls = &sm_l[0][0], *rs = &sm_r[0][0];
    if (n16 == 0) ms[group] = M, ls[group] = L, rs[group] = R;
    __syncthreads();
    const bool mine = g0 == 0 && row < rows_here;
    if (mine) {
      M = -INFINITY, L = R = 0.f;
      for (int k = 0; k < G; ++k) M = fmaxf(M, ms[(k << shift) + row]);
#pragma unroll
      for (int i = 0; i < kPairs; ++i) acc[i] = float2v{0.f, 0.f};
      for (int k = 0; k < G; ++k) {
        const int at = (k << shift) + row;
        const float e = part_factor(ms[at], M);
        L = fmaf(e, ls[at], L), R = fmaf(e, rs[at], R);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) acc[i] += e * *reinterpret_cast<const float2v*>(flat + at * kStride + 32 * i + 2 * n16);
      }
    }
    if (!two || step > 1) {
      if (mine) write_row<D, BF>(a, b, h, r0 + row, n16, M, L, R, acc);
      return;
    }
    if (mine) {
      float* P = partial_of(from) + row * (D + 4);
#pragma unroll
      for (int i = 0; i < kPairs; ++i) store_agent(P + 32 * i + 2 * n16, acc[i][0], acc[i][1]);
      if (n16 < 2) store_agent(P + D + 2 * n16, n16 ? R : M, n16 ? 0.f : L);
    }
    from = 0, n_parts = (live + kGroup - 1) / kGroup, step = kGroup;
    if (!arrives_last(a, 0, first_run, n_parts, arrived)) return;
  }
  }();
  __syncthreads();  // the joining has left LDS
  } while (cur.next(a));
}

// ---- many rows: tiles in LDS ------------------------------------------------------------------------------
// Units of 128 rows, a wave holding 32 of them.  Each 64-token tile of keys and values is
// converted once per workgroup and staged in LDS as fp16: keys token by token, values transposed, in the order in which the score
// product leaves the weights in a lane, so that both products read their first operand as 16-byte rows and the weights never
// leave their lane.  The next tile's codes are on their way to registers while a tile is worked on; two tiles in LDS, one barrier a tile.
// Bound by the issue of a wave's 32 products of 32x32x16 and some 270 vector instructions per tile, 32 exponentials among them: the matrix
// unit is busy for 39 % of the time, the vector unit for 51 %, and little of the one hides behind the other.  2048 tokens of 32 heads
// over 10240 tokens of 8: 340 us, 910 TFLOP/s.  Tiles of 256 rows by eight waves took 424 us where these took 359.

template <int D>
struct ChunkTile {
  static constexpr int kKeyRow = D + 8, kValRow = kBlock + 8;  // halves per row: 16 bytes more, so that rows start on other banks
  _Float16 k[kBlock][kKeyRow];
  _Float16 v[D][kValRow];  // row 16 i + n: channel (D / 16) n + i; place 16 st + 8 hh + j: token 16 st + 8 (j / 4) + 4 hh + j % 4
};

// operands of a tile that are asked for ahead of their products: LDS answers in about three products' time
constexpr int kAhead = 6;
// products and reads of LDS stay in the order written (left to itself the compiler puts each read before its product, to wait for it)
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0x002 | 0x004 | 0x200); }

// FEW: few tiles, which may reach into many runs each; apart, as that code costs the other calls 4 % (chunk of 2048 over 10240 tokens)
template <int D, int CODE, bool BF, bool FEW>
__global__ __launch_bounds__(kWaves * 64, 2) void chunk_kernel(Args a) {
  constexpr int kCh = D / 16, kTok = 256 / D, kCellsOf4 = 4 / kTok, kKeyCells = D / 64;
  __shared__ ChunkTile<D> sm[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_index(), hh = lane >> 5, n = lane & 31;
  __shared__ int arrived;
  // the workgroups of a compute die (every eighth) take runs that follow each other, so that they read the same keys
  Cursor<32 * kWaves> cur;
  const int dies = gridDim.x % 8 == 0 && !a.direct ? 8 : 1;
  if (!cur.begin(a, blockIdx.x % dies * (gridDim.x / dies) + blockIdx.x / dies)) return;
  do {  // segments
  const int b = cur.b, h = cur.h;
  const Problem pr = cur.pr;
  const int n_rows = pr.nq * a.g.ratio, r0 = cur.tile * 32 * kWaves;
  const int rw = r0 + wave * 32, r = rw + n;
  const int vis = r < n_rows ? visible(a, pr, r / a.g.ratio) : pr.len;
  // what the wave's and the workgroup's rows see at least and at most
  const int last = min(rw + 31, n_rows - 1);
  const int vis_min = rw < n_rows ? visible(a, pr, rw / a.g.ratio) : 0, vis_max = rw < n_rows ? visible(a, pr, last / a.g.ratio) : 0;
  const int vis_all = visible(a, pr, min(r0 + 32 * kWaves - 1, n_rows - 1) / a.g.ratio);
  const int blk0 = cur.first(), blk1 = min((vis_all + kBlock - 1) / kBlock, cur.last());

  half8v q[D / 16];
  const float factor = load_query_rows<D, BF>(a, b, h, r, pr.nq, q);
  float m = -INFINITY, l = 0.f, lr = 0.f, sref = 0.f;
  float16v o[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.f;

  // this thread's part of a tile: 16-byte pieces of key codes, and four tokens of a column of value cells
  const int vn = tid & 15, vhalf = (tid >> 4) & 1, vh = (tid >> 5) & 1, vst = tid >> 6, vt = 16 * vst + 8 * vhalf + 4 * vh;
  uint4v kw[kKeyCells], vw[kCellsOf4];
  float next_sk = 0.f, next_sv = 0.f;
  bool next_there = false;
  auto fetch = [&](int blk) {
    const int64_t pk = block_place<true>(a.g, a.kc.block_table, b, h, blk), pv = block_place<true>(a.g, a.vc.block_table, b, h, blk);
    next_there = pk >= 0 && pv >= 0;
    if (!next_there) return;
    const uint8_t* kp = a.kc.codes + pk * (int64_t)(kBlock * D);
    const uint8_t* vp = a.vc.codes + pv * (int64_t)(kBlock * D);
#pragma unroll
    for (int i = 0; i < kKeyCells; ++i) kw[i] = *reinterpret_cast<const uint4v*>(kp + (tid + i * kWaves * 64) * 16);
#pragma unroll
    for (int c = 0; c < kCellsOf4; ++c) vw[c] = *reinterpret_cast<const uint4v*>(vp + (vt / kTok + c) * 256 + vn * 16);
    next_sk = load_uniform(a.kc.scales + pk), next_sv = load_uniform(a.vc.scales + pv);
    if (CODE == NSN_Q8_E4M3 && (blk + 1) * kBlock > pr.len) {  // places behind the last token may hold NaN: 0 * NaN is one
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if (blk * kBlock + vt + t >= pr.len) {
#pragma unroll
          for (int e = 0; e < 4 / kTok; ++e) vw[t / kTok][t % kTok * (4 / kTok) + e] = 0;
        }
    }
  };
  auto stage = [&](ChunkTile<D>& to) {
#pragma unroll
    for (int i = 0; i < kKeyCells; ++i) {
      const int cell = tid + i * kWaves * 64;
      _Float16* p = &to.k[cell / kCh][cell % kCh * 16];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        half2v u0, u1, u2, u3;
        to_half4<CODE>(kw[i][2 * x], u0, u1);
        to_half4<CODE>(kw[i][2 * x + 1], u2, u3);
        *reinterpret_cast<half8v*>(p + 8 * x) = half8v{u0[0], u0[1], u1[0], u1[1], u2[0], u2[1], u3[0], u3[1]};
      }
    }
#pragma unroll
    for (int c2 = 0; c2 < kCh / 2; ++c2) {
      half2v x[2], y[2];
#pragma unroll
      for (int pair = 0; pair < 2; ++pair) {
        const int t = 2 * pair;
        const unsigned u = vw[t / kTok][t % kTok * (4 / kTok) + c2 / 2], w = vw[(t + 1) / kTok][(t + 1) % kTok * (4 / kTok) + c2 / 2];
        to_half4<CODE>(__builtin_amdgcn_perm(w, u, c2 & 1 ? 0x07030602u : 0x05010400u), x[pair], y[pair]);
      }
      const int at = 16 * vst + 8 * vh + 4 * vhalf;
      *reinterpret_cast<half4v*>(&to.v[16 * (2 * c2) + vn][at]) = half4v{x[0][0], x[0][1], x[1][0], x[1][1]};
      *reinterpret_cast<half4v*>(&to.v[16 * (2 * c2 + 1) + vn][at]) = half4v{y[0][0], y[0][1], y[1][0], y[1][1]};
    }
  };

  if (blk0 < blk1) {
    fetch(blk0);
    if (next_there) stage(sm[0]);
  }
  for (int blk = blk0, buf = 0; blk < blk1; ++blk, buf ^= 1) {
    const bool there = next_there;
    const float sk = next_sk, sv = next_sv;
    const int t0 = blk * kBlock;
    __syncthreads();  // the tile is complete, and everybody has left the one before it
    if (blk + 1 < blk1) fetch(blk + 1);
    if (there && t0 < vis_max) {
      const ChunkTile<D>& tl = sm[buf];
      float16v s[2];
      const float f = factor * sk;
      const bool masked = t0 + kBlock > vis_min;
      auto scores = [&] {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 16; ++e) s[j][e] = 0.f;
        half8v x[kAhead];
        auto read = [&](int i) { x[i % kAhead] = *reinterpret_cast<const half8v*>(&tl.k[32 * (i & 1) + n][16 * (i / 2) + 8 * hh]); };
#pragma unroll
        for (int i = 0; i < kAhead; ++i) read(i);
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
          in_order();
          s[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[i % kAhead], q[i / 2], s[i & 1], 0, 0, 0);
          if (i + kAhead < D / 8) read(i + kAhead);
        }
      };
      auto hide = [&](float with) {  // the tokens that a row does not see, a bit each (compares would take the scalar registers)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int left = vis - t0 - 4 * hh - 32 * j;  // of these 32
          const int seen = left >= 32 ? -1 : (1 << max(left, 0)) - 1;
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int own = __builtin_amdgcn_sbfe(seen, 8 * (e / 4) + e % 4, 1);  // all ones, or 0
            s[j][e] = __uint_as_float((__float_as_uint(s[j][e]) & own) | (__float_as_uint(with) & ~own));
          }
        }
      };
      float sum[2];
      auto weights = [&](float base) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 16; ++e) s[j][e] = fast_exp2(fmaf(s[j][e], f, -base));
        if (masked) hide(0.f);
        sum[0] = sum[1] = 0.f;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 16; e += 2) sum[0] += s[j][e], sum[1] += s[j][e + 1];
      };
      scores();
      float ratio, lift;
      follow_scale<D / 32>(sv, sref, o, ratio, lift);
      weights(m - lift);
      // The weights under the maximum as it was will do unless they come near the end of fp16; only then (the first tile, a
      // rise of more than 2^5) are the scores formed again for their maximum.
      // (what counts for l is their sum times the ratio: more than the weights themselves where the values' scale has dropped)
      const float own = (sum[0] + sum[1]) * fmaxf(ratio, 1.f), most = fmaxf(own, xor_lane<32>(own));
      if (__any(!(most < kMost))) {
        scores();
        if (masked) hide(kMasked);
        float top = s[0][0];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 16; ++e) top = fmaxf(top, s[j][e]);
        top = fmaxf(top, xor_lane<32>(top)) * f;
        move_maximum<D / 32>(most < kMost ? m : fmaxf(m, top), m, l, lr, o);  // (each row by its own weights: its result does not hang on its neighbours)
        weights(m - lift);
      }
      float rounded[2] = {0.f, 0.f};
      half8v p[4];
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          const half2v u = __builtin_convertvector((float2v{s[j][e], s[j][e + 1]}), half2v);
          rounded[j] = add_rounded(u, rounded[j]);
          p[2 * j + e / 8][e % 8] = u[0], p[2 * j + e / 8][e % 8 + 1] = u[1];
        }
      add_weights(sum[0] + sum[1], rounded[0] + rounded[1], ratio, l, lr);
      half8v x[kAhead];
      auto read = [&](int i) { x[i % kAhead] = *reinterpret_cast<const half8v*>(&tl.v[i % (D / 32) * 32 + n][16 * (i / (D / 32)) + 8 * hh]); };
#pragma unroll
      for (int i = 0; i < kAhead; ++i) read(i);
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        in_order();
        o[i % (D / 32)] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[i % kAhead], p[i / (D / 32)], o[i % (D / 32)], 0, 0, 0);
        if (i + kAhead < D / 8) read(i + kAhead);
      }
    }
    if (blk + 1 < blk1 && next_there) stage(sm[buf ^ 1]);
  }
  l += xor_lane<32>(l), lr += xor_lane<32>(lr);
  const int first_run = cur.first_run(), live = cur.runs();  // (here: scalar registers are short in the loop)
  // o[i][e]: row 32 i + 8 (e / 4) + 4 hh + e % 4 of the transposed values; the channels of cell c are its rows 16 x + c
  float M = l == 0.f ? -INFINITY : m - kLift, unit_of_o = sref;
  [&] {
  if (live > 1) {
    // the sums as they lie in the threads, two to a store; joined in the order of the runs
    constexpr int kPairs = D / 4, kThreads = kWaves * 64;
    auto partial_of = [&](int k) { return a.partial + (((int64_t)(first_run + k) * 2 + (k == 0)) * (kPairs + 2) * kThreads + tid) * 2; };
#pragma unroll
    for (int i = 0; i < D / 32; ++i) o[i] *= sref;
    unit_of_o = 1.f;
    // all of them where they are few; of more than 16, eight at a time, and then those sums (two tiles of eight heads over 30000 tokens:
    // 100 us in one go, 70 us so)
    constexpr int kGroup = 8;
    const bool two = FEW && live > 2 * kGroup;
    int mine = cur.run - first_run, from = two ? mine / kGroup * kGroup : 0, n_parts = two ? min(kGroup, live - from) : live, step = 1;
    int kind = two ? (from == 0 ? 1 : 2) : 0;
    while (true) {
      float* P = partial_of(mine);
      if (r < n_rows) {
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
          for (int e = 0; e < 16; e += 2) store_agent(P + (8 * i + e / 2) * kThreads * 2, o[i][e], o[i][e + 1]);
        store_agent(P + kPairs * kThreads * 2, M, l);
        store_agent(P + (kPairs + 1) * kThreads * 2, lr, 0.f);
      }
      if (!arrives_last(a, kind, first_run + from, n_parts, arrived)) return;
      // in the order of the runs, whoever joins them; its own sums it still holds
      float16v total[D / 32];
      float m_all = -INFINITY, l_all = 0.f, lr_all = 0.f;
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) total[i][e] = 0.f;
      if (r < n_rows)
        for (int k = from; k < from + n_parts * step; k += step) {
          float2v ml = {M, l}, rd = {lr, 0.f}, x[kPairs];
          if (k == mine) {
#pragma unroll
            for (int i = 0; i < kPairs; ++i) x[i] = float2v{o[i / 8][i % 8 * 2], o[i / 8][i % 8 * 2 + 1]};
          } else {
            const float* ps = partial_of(k);
            ml = load_agent(ps + kPairs * kThreads * 2), rd = load_agent(ps + (kPairs + 1) * kThreads * 2);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) x[i] = load_agent(ps + i * kThreads * 2);
          }
          const float m2 = fmaxf(m_all, ml[0]), turn = part_factor(m_all, m2), f = part_factor(ml[0], m2);
          m_all = m2;
          l_all = fmaf(f, ml[1], l_all * turn), lr_all = fmaf(f, rd[0], lr_all * turn);
#pragma unroll
          for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) total[i][e] = fmaf(f, x[8 * i + e / 2][e & 1], total[i][e] * turn);
        }
      M = m_all, l = l_all, lr = lr_all;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) o[i] = total[i];
      if (!two || step > 1) break;
      mine = from, from = 0, n_parts = (live + kGroup - 1) / kGroup, step = kGroup, kind = 0;
    }
  }
  if (r >= n_rows) return;
  const int64_t place = ((int64_t)b * a.n_q + r / a.g.ratio) * a.g.hq + h * a.g.ratio + r % a.g.ratio;
  const float inv = lr > 0.f ? unit_of_o / lr : (lr == 0.f ? 0.f : lr);
#pragma unroll
  for (int c4 = 0; c4 < 2; ++c4)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      alignas(16) uint16_t u[kCh];
#pragma unroll
      for (int i = 0; i < kCh; ++i) u[i] = from_float<BF>(o[i / 2][8 * (i & 1) + 4 * c4 + e] * inv);
      uint16_t* to = a.out + place * D + kCh * (8 * c4 + 4 * hh + e);
      if constexpr (kCh == 8)
        *reinterpret_cast<uint4v*>(to) = *reinterpret_cast<const uint4v*>(u);
      else
        *reinterpret_cast<uint2v*>(to) = *reinterpret_cast<const uint2v*>(u);
    }
  if (hh == 0) {
    const float z = l == 0.f ? -INFINITY : M + __log2f(l);
    if (a.lse) a.lse[place] = z * kLn2;
    a.lse2[((int64_t)b * a.g.hkv + h) * a.rows + r] = z;
  }
  }();
  __syncthreads();  // everybody has left the tiles in LDS
  } while (cur.next(a));
}

// ---- the weights that each cached token receives ----------------------------------------------------------
// One workgroup per 256 tokens of a kv head and part of the rows: each wave holds 64 tokens' keys as operands in registers (in the
// queries' own type, which codes fit without loss), the rows come by in LDS tiles of 32 that all four waves read, and a wave adds
// 2^(s - lse) up per token.  Parts are joined in their order by the last workgroup to arrive.  Bound by the exponentials: one
// per row and token, a quarter of the vector rate, with the products beside them.
constexpr int kWeightTokens = 64 * kWaves, kWeightRows = 32;

template <int CODE, bool BF>
__device__ __forceinline__ uint4v to_operand8(unsigned w0, unsigned w1) {
  if constexpr (!BF) {
    half2v a, b, c, d;
    to_half4<CODE>(w0, a, b);
    to_half4<CODE>(w1, c, d);
    return __builtin_bit_cast(uint4v, (half8v{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]}));
  } else {  // (codes have 8 significant bits at most: the upper half of the fp32 number is the bf16 one)
    float f[8];
    to_float4<CODE>(w0, f);
    to_float4<CODE>(w1, f + 4);
    uint4v u;
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = __builtin_amdgcn_perm(__float_as_uint(f[2 * i + 1]), __float_as_uint(f[2 * i]), 0x07060302u);
    return u;
  }
}
typedef __bf16 bfloat8v __attribute__((ext_vector_type(8)));
template <bool BF>
__device__ __forceinline__ float16v product32(uint4v x, uint4v y, float16v c) {
  if constexpr (BF)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bfloat8v, x), __builtin_bit_cast(bfloat8v, y), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8v, x), __builtin_bit_cast(half8v, y), c, 0, 0, 0);
}

template <int D, int CODE, bool BF>
__global__ __launch_bounds__(kWaves * 64, 2) void weights_kernel(Args a) {
  constexpr int kPieces = kWeightRows * D / 8 / (kWaves * 64);  // 16-byte pieces of a tile of rows that a thread brings
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_index(), hh = lane >> 5, n = lane & 31;
  const int part = blockIdx.x % a.weight_parts, group = blockIdx.x / a.weight_parts, h = blockIdx.y, b = blockIdx.z;
  const Problem pr = problem_of(a, b);
  const int g0 = group * kWeightTokens, t0 = g0 + wave * kBlock, n_rows = pr.nq * a.g.ratio;
  if (g0 >= pr.len) return;
  __shared__ __attribute__((aligned(16))) uint16_t sm_q[2][kWeightRows][D + 8];
  __shared__ float sm_z[2][kWeightRows];
  __shared__ int arrived;
  // the rows that see the first token of the group, cut into the parts
  const int first = a.causal ? min(max(g0 - pr.vis0 + 1, 0), pr.nq) * a.g.ratio / kWeightRows : 0;
  const int tiles = (n_rows + kWeightRows - 1) / kWeightRows - first, per = (tiles + a.weight_parts - 1) / a.weight_parts;
  const int tile0 = first + min(part * per, tiles), tile1 = first + min((part + 1) * per, tiles);

  uint4v k[2][D / 16];
  float f = 0.f;
  float16v sum[2];
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int e = 0; e < 16; ++e) sum[j][e] = 0.f;
  bool there = t0 < pr.len;
  if (there) {
    const int64_t pk = block_place<true>(a.g, a.kc.block_table, b, h, t0 / kBlock), pv = block_place<true>(a.g, a.vc.block_table, b, h, t0 / kBlock);
    there = pk >= 0 && pv >= 0;
    if (there) {
      const uint8_t* p = a.kc.codes + pk * (int64_t)(kBlock * D) + 8 * hh;
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          const uint2v w = *reinterpret_cast<const uint2v*>(p + (32 * j + n) * D + 16 * ks);
          k[j][ks] = to_operand8<CODE, BF>(w[0], w[1]);
        }
      f = a.scale_log2 * load_uniform(a.kc.scales + pk);
    }
  }
  uint4v piece[kPieces];
  float z = 0.f;
  auto fetch = [&](int tile) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int x = tid + i * kWaves * 64, r = tile * kWeightRows + x / (D / 8);
      piece[i] = uint4v{0, 0, 0, 0};
      if (r < n_rows)
        piece[i] = *reinterpret_cast<const uint4v*>(a.q.data + b * a.q.sb + (h * a.g.ratio + r % a.g.ratio) * a.q.sh + r / a.g.ratio * a.q.st + x % (D / 8) * 8);
    }
    if (tid < kWeightRows) {
      const int r = tile * kWeightRows + tid;
      z = r < n_rows ? a.lse2[((int64_t)b * a.g.hkv + h) * a.rows + r] : INFINITY;
      if (z == -INFINITY) z = INFINITY;  // (a row that sees nothing gives nothing)
    }
  };
  auto stage = [&](int buf) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int x = tid + i * kWaves * 64;
      *reinterpret_cast<uint4v*>(&sm_q[buf][x / (D / 8)][x % (D / 8) * 8]) = piece[i];
    }
    if (tid < kWeightRows) sm_z[buf][tid] = z;
  };
  if (tile0 < tile1) {
    fetch(tile0);
    stage(0);
  }
  for (int tile = tile0, buf = 0; tile < tile1; ++tile, buf ^= 1) {
    __syncthreads();
    if (tile + 1 < tile1) fetch(tile + 1);
    const int r0 = tile * kWeightRows, r = r0 + n;
    if (there && visible(a, pr, min(r0 + kWeightRows - 1, n_rows - 1) / a.g.ratio) > t0) {
      float16v s[2];
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[j][e] = 0.f;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        const uint4v q = *reinterpret_cast<const uint4v*>(&sm_q[buf][n][16 * ks + 8 * hh]);
#pragma unroll
        for (int j = 0; j < 2; ++j) s[j] = product32<BF>(k[j][ks], q, s[j]);
      }
      const float zr = sm_z[buf][n];
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[j][e] = fast_exp2(fmaf(s[j][e], f, -zr));
      if (visible(a, pr, r0 / a.g.ratio) < t0 + kBlock) {
        const int vis = r < n_rows ? visible(a, pr, r / a.g.ratio) : 0;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (t0 + 32 * j + 8 * (e / 4) + 4 * hh + e % 4 >= vis) s[j][e] = 0.f;
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) sum[j] += s[j];
    }
    if (tile + 1 < tile1) stage(buf ^ 1);
  }
  // over the 32 rows of a tile: one value per token, token 32 j + 8 (e / 4) + 4 hh + e % 4 of the wave in lane 0 of its half
  __shared__ float sm[kWeightTokens];
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float x = xor_sum_w<32>(sum[j][e]);
      if (n == 0) sm[wave * kBlock + 32 * j + 8 * (e / 4) + 4 * hh + e % 4] = x;
    }
  __syncthreads();
  float x = sm[tid];
  if (a.weight_parts > 1) {
    const int64_t place = ((int64_t)(b * gridDim.y + h) * (gridDim.x / a.weight_parts) + group) * a.weight_parts;
    float* P = a.partial + place * kWeightTokens + tid;
    __hip_atomic_store(P + part * kWeightTokens, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (!arrives_last(a, 0, (int)(place / a.weight_parts), a.weight_parts, arrived)) return;
    x = 0.f;
    for (int i = 0; i < a.weight_parts; ++i) x += __hip_atomic_load(P + i * kWeightTokens, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  if (g0 + tid < pr.len) {
    const int64_t at = ((int64_t)b * a.g.hkv + h) * a.g.max_len + g0 + tid;
    a.weights_out[at] = a.weights_in ? a.weights_in[at] + x : x;
  }
}

// The same from the scores that a call of few rows has left behind: a thread takes four tokens and goes through the rows.
constexpr int kScoreThreads = 256;
__global__ __launch_bounds__(kScoreThreads) void weights_of_scores_kernel(Args a) {
  const int h = blockIdx.y, b = blockIdx.z;
  const Problem pr = problem_of(a, b);
  const int t = (blockIdx.x * kScoreThreads + threadIdx.x) * 4, n_rows = pr.nq * a.g.ratio;
  if (t >= pr.len) return;
  const int64_t line0 = ((int64_t)b * a.g.hkv + h) * a.rows;
  float4v x = {0.f, 0.f, 0.f, 0.f};
  for (int r = 0; r < n_rows; ++r) {
    // (a row's scores end with the block of the last token that its tile of rows sees)
    if (t >= (visible(a, pr, min(r | 15, n_rows - 1) / a.g.ratio) + kBlock - 1) / kBlock * kBlock) continue;
    const float4v s = *reinterpret_cast<const float4v*>(a.scores + (line0 + r) * a.score_stride + t);
    const float z = a.lse2[line0 + r];
    if (z == -INFINITY) continue;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] += fast_exp2(s[e] - z);
  }
  const int64_t at = ((int64_t)b * a.g.hkv + h) * a.g.max_len + t;
  for (int e = 0; e < min(4, pr.len - t); ++e) a.weights_out[at + e] = a.weights_in ? a.weights_in[at + e] + x[e] : x[e];
}

// ---- host side --------------------------------------------------------------------------------------------
// Whether rows are taken 128 at a time through tiles in LDS, or 16 at a time.  A tile of 128 rows costs per block three times
// what one of 16 does, and its joining thirty, so it pays for more than two tiles of 16 where there are enough units to
// leave most of them whole (128 units of 32 blocks: 32 rows 30.6 us with 128-row tiles and 29.7 without, 48 rows 34 and 40, 128 rows 45
// and 80; 384 of 5: 48 rows 24.5 and 31), and else from so much work on that the joining does not count (8 units of 128 blocks: 128
// rows 43 and 23, 512 rows 57 and 58, 1024 rows 69 and 100).
static bool use_chunk(int64_t rows, int64_t heads, int blocks) {
  return rows > 32 && ((rows + 32 * kWaves - 1) / (32 * kWaves) * heads >= 128 || (rows + 15) / 16 * heads * blocks >= 28000);
}

static size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }

// How a call is cut, and where its workspace's parts lie
struct Plan {
  bool chunk, direct;
  int64_t tiles;  // of rows
  int runs, per;
  bool scores;
  int64_t weight_groups;  // of 256 tokens
  int weight_parts;
  size_t lse2_at, partial_at, scores_at, bytes;
  int64_t score_stride;
};
// floats of a run's partial sums
static size_t run_floats(bool chunk, int head_dim) { return 2 * (size_t)(chunk ? (head_dim / 2 + 4) * kWaves * 64 : 16 * (head_dim + 4)); }

// ragged: sequences may have fewer queries than n_q
static Plan plan_of(const nsn_q8_shape& s, int batch, int n_q, int max_seq_len, int requested, bool weights, bool ragged) {
  Plan p;
  const int64_t rows = (int64_t)n_q * (s.n_q_heads / s.n_kv_heads), lines = rows * s.n_kv_heads * batch;
  const int blocks = std::max(1, (max_seq_len + kBlock - 1) / kBlock);
  p.chunk = use_chunk(rows, (int64_t)s.n_kv_heads * batch, blocks);
  const int tile_rows = p.chunk ? 32 * kWaves : 16;
  p.tiles = (rows + tile_rows - 1) / tile_rows;
  const int64_t units = p.tiles * s.n_kv_heads * batch;
  // runs: two workgroups to each of the 256 compute units (few rows: or one per unit where there are more).  Where few units reach into
  // many runs each, one workgroup to a compute unit: it keeps memory nearly as busy and leaves half the partials to be joined (8
  // units of 2048 blocks 54.6 us and 62.5 us with two, 64 of 32 14.1 and 15.9; 256 of 8 to 256 blocks 116 and 102, 512 of 16 33.2 and
  // 29.1).  Four blocks at least (few rows: a wave each; chunks of few units eight), as a run's start and joining take as long as some
  // blocks, but no more than a unit has: units one after the other cost their trips to memory one after the other
  const int64_t most = p.chunk ? 512 : kMaxCounters;
  // chunks of many units go one to a workgroup, as joining a cut tile's 128 rows costs about ten of its blocks: with 512 units of 128 to
  // 160 blocks 355 us so and 372 us in equal runs (now 342 so); with ragged chunks of up to 512 units of very different lengths 114 us and 62 us.
  // So do units of few blocks, where joining is most of the time, unless so few of them that compute units are left idle
  // (head_dim 128: 256 units of 5 blocks 20.0 us and 30.6, of 8 26 and 29; 384 of up to 15 blocks, equal 45 and 48, ragged 36 and 35;
  // 128 of 8 23 and 18; ragged, up to 768 units of up to 16 blocks 40 and 43, of 32 77 and 67)
  p.direct = requested <= 0 && (p.chunk ? (blocks <= 16 && blocks * (512 - units) <= 2048) || units >= (ragged ? 1024 : 512) : units > most);
  p.per = requested > 0 ? 1 : std::min(p.chunk && units < 128 ? 8 : 4, blocks);
  const int64_t runs = requested > 0 ? requested * units : p.chunk ? 512 : units <= 64 ? 256 : std::max<int64_t>(512, units);
  p.runs = p.direct ? (int)std::min<int64_t>(units, 0x7fffffff)
                    : (int)std::min<int64_t>(std::min<int64_t>(runs, most), (units * blocks + p.per - 1) / p.per);
  // the pass that adds weights up: up to eight workgroups to a compute unit, as sequences may be shorter than max_seq_len and causal
  // parts unequal, each with four tiles of rows at least; its partial sums come after the attention's and take their place
  p.weight_groups = (blocks + kWaves - 1) / kWaves * (int64_t)s.n_kv_heads * batch;
  p.weight_parts = (int)std::max<int64_t>(1, std::min<int64_t>(kMaxCounters / p.weight_groups, rows / (4 * kWeightRows)));
  size_t partials = p.direct ? 0 : p.runs * run_floats(p.chunk, s.head_dim);
  p.scores = weights && rows <= 16;
  if (weights && p.weight_parts > 1) partials = std::max(partials, (size_t)p.weight_groups * p.weight_parts * kWeightTokens);
  p.score_stride = (int64_t)blocks * kBlock;
  p.lse2_at = (size_t)3 * kMaxCounters * kCounterInts * sizeof(int);
  p.partial_at = p.lse2_at + up16(lines * sizeof(float));
  p.scores_at = p.partial_at + up16(partials * sizeof(float));
  p.bytes = p.scores_at + (p.scores ? (size_t)lines * p.score_stride * sizeof(float) : 0);
  return p;
}

// For calls of up to these sizes, with or without weights: as many runs of either kind as any plan of them has
size_t attention_workspace_bytes(const nsn_q8_shape& s, int batch, int n_q, int max_seq_len, int n_splits) {
  const Plan p = plan_of(s, batch, n_q, max_seq_len, n_splits, true, false);
  const int64_t rows = (int64_t)n_q * (s.n_q_heads / s.n_kv_heads), heads = (int64_t)s.n_kv_heads * batch, blocks = p.score_stride / kBlock;
  auto most = [&](bool chunk, int64_t limit) {
    const int64_t units = (rows + (chunk ? 32 * kWaves : 16) - 1) / (chunk ? 32 * kWaves : 16) * heads;
    return (size_t)std::min(limit, units * blocks) * run_floats(chunk, s.head_dim);
  };
  size_t partials = std::max(most(false, kMaxCounters), p.chunk ? most(true, 512) : 0);
  if (rows >= 8 * kWeightRows) partials = std::max(partials, (size_t)kMaxCounters * kWeightTokens);
  return p.partial_at + up16(partials * sizeof(float)) + (p.bytes - p.scores_at);
}

int attention_launch(const AttentionCall& c) {
  const nsn_q8_shape& s = c.shape;
  const Plan plan = plan_of(s, c.batch, c.n_q, c.max_seq_len, c.n_splits, c.weights_out != nullptr, c.q_lens != nullptr);
  unsigned char* ws = static_cast<unsigned char*>(c.workspace);
  Args a;
  a.g = make_geometry(s);
  a.q = make_rows(c.q);
  a.n_q = c.n_q, a.rows = c.n_q * a.g.ratio, a.q_lens = c.q_lens;
  a.kc = make_view(c.kc), a.vc = make_view(c.vc);
  a.seq_lens = c.seq_lens, a.max_seq_len = c.max_seq_len;
  a.scale_log2 = c.scale * kLog2e, a.causal = c.causal;
  a.batch = c.batch, a.n_runs = plan.runs, a.per = plan.per, a.direct = plan.direct;
  a.out = static_cast<uint16_t*>(c.out), a.lse = c.lse;
  a.counters = reinterpret_cast<int*>(ws);
  a.row_tiles = (int)plan.tiles;
  a.lse2 = reinterpret_cast<float*>(ws + plan.lse2_at);
  a.partial = reinterpret_cast<float*>(ws + plan.partial_at);
  a.scores = plan.scores ? reinterpret_cast<float*>(ws + plan.scores_at) : nullptr;
  a.score_stride = plan.score_stride;
  a.weight_parts = plan.weight_parts;
  a.weights_in = c.weights_in, a.weights_out = c.weights_out;
  return with_types(s, [&](auto d, auto code, auto bf) -> int {
    constexpr int D = decltype(d)::value, CODE = decltype(code)::value;
    constexpr bool BF = decltype(bf)::value;
    const int64_t units = plan.tiles * a.g.hkv * c.batch;
    if (plan.direct ? units > 0x7fffffff : units * (a.score_stride / kBlock) > 0x3fffffff) {
      set_error("q8_attention: batch * n_q * n_q_heads * max_seq_len is too large for one launch");
      return NSN_ERR_UNSUPPORTED;
    }
    if (plan.chunk && units <= 32)
      chunk_kernel<D, CODE, BF, true><<<plan.runs, kWaves * 64, 0, c.stream>>>(a);
    else if (plan.chunk)
      chunk_kernel<D, CODE, BF, false><<<plan.runs, kWaves * 64, 0, c.stream>>>(a);
    else
      rows_kernel<D, CODE, BF><<<plan.runs, kWaves * 64, 0, c.stream>>>(a);
    if (hipGetLastError() != hipSuccess) return NSN_ERR_HIP;
    if (a.weights_out && c.max_seq_len > 0) {
      if (plan.scores)
        weights_of_scores_kernel<<<dim3((c.max_seq_len + 4 * kScoreThreads - 1) / (4 * kScoreThreads), a.g.hkv, c.batch), kScoreThreads, 0, c.stream>>>(a);
      else
        weights_kernel<D, CODE, BF><<<dim3((c.max_seq_len + kWeightTokens - 1) / kWeightTokens * plan.weight_parts, a.g.hkv, c.batch), kWaves * 64, 0, c.stream>>>(a);
      if (hipGetLastError() != hipSuccess) return NSN_ERR_HIP;
    }
    return NSN_OK;
  });
}

}  // namespace q8
}  // namespace nsn
