// Which blocks the queries of a token select by their bounds: the device code of fc_sparse.hip and of
// the attention that selects for itself (fc_attention.hip).
#pragma once

#include <algorithm>

#include "fc_chunk_plan.h"
#include "fc_device.h"

namespace fc {

// ---------------------------------------------------------------------------
// selection.  A score is a sum rounded once, to 64 bits (score_exactly): a product of two fp16 numbers is exact in
// fp32, and which of two blocks is read should follow from the inputs, not from the order in which a sum was made.  All
// scores are made by the matrix cores in fp32 first,
//     S [query heads x blocks] = min(Q, 0) . LO^T + max(Q, 0) . HI^T,
// which is the same sum, off by at most E = 2 D 2^-23 (largest sum of |q|) (largest |bound|): each of 2 D
// additions by 2^-23 of what was added up so far, twice what a rounding loses.  With T the k-th largest of
// them, scores over T + 2 E are among the k best and those below T - 2 E are not; the few between are made
// anew in 64 bits.  (What is infinite or not a number makes E so, and all blocks are "between".)
// In 64 bits throughout, five vector instructions for each product, 48 caches of 1280-7040 tokens, 8 heads of
// 4, took 22 us for the scores alone, and 10 tokens over 28 000-30 000 27; with the matrix cores a workgroup of the former
// spends 3.3 us on its first loads, 3.6 on scores and 4.4 on the selection (medians; latency and barriers), and the
// latter are scored in 7.5 and selected from in 7.9.
// ---------------------------------------------------------------------------

// The order of scores as that of unsigned numbers: larger ones are larger, not a number is the
// largest, both zeros are one; 0 is none of them.
__device__ __forceinline__ uint64_t score_order(double s) {
  const uint64_t bits = __builtin_bit_cast(uint64_t, s + 0.0);
  if (s != s) return ~0ull;
  return bits >> 63 ? ~bits : bits | (1ull << 63);
}

template <int CTRL>
__device__ __forceinline__ double from_lane_f64(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = from_lane_u32<CTRL>((uint32_t)b), hi = from_lane_u32<CTRL>((uint32_t)(b >> 32));
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

__device__ __forceinline__ const _Float16* query_of(const SelectParams& p, int row, int q_head) {
  return p.q.data + (int64_t)row * p.q.token_stride + (int64_t)q_head * p.q.head_stride;
}

// The first product's operands: of up to kRows rows (token * group + query head of the group, zeros behind the last
// one, in tiles of 16) the parts below and above zero, 2 D numbers each, in LDS in the order of the lanes, 32 at a time.
// Requested when this is made, before the bounds: loads are answered in order.
template <int D, int kRows, int kThreadsHere>
struct ScoredQueries {
  static constexpr int KK = 2 * D / 32, PPR = D / 8, kEach = (kRows * PPR + kThreadsHere - 1) / kThreadsHere;
  half8 x[kEach];
  int rows;
  __device__ __forceinline__ ScoredQueries(const SelectParams& p, int first_row, int n_tokens, int head) : rows(n_tokens * p.group) {
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int i = k * kThreadsHere + (int)threadIdx.x, r = i / PPR, c = i % PPR;
      x[k] = half8{};
      if (r < rows) {
        const int t = r / p.group;
        x[k] = load_half8(query_of(p, first_row + t, head * p.group + r - t * p.group) + c * 8);
      }
    }
    requests_first();
  }
  // sm_q: NULL, or for the rows themselves
  __device__ __forceinline__ void put(half8* sm_a, _Float16* sm_q) const {
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int i = k * kThreadsHere + (int)threadIdx.x, r = i / PPR, c = i % PPR;
      if (r >= ((rows + 15) & ~15)) continue;
      if (sm_q && r < rows) store_half8(sm_q + r * D + c * 8, x[k]);
      half8 below, above;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        below[e] = x[k][e] < (_Float16)0.f ? x[k][e] : (_Float16)0.f;
        above[e] = x[k][e] > (_Float16)0.f ? x[k][e] : (_Float16)0.f;
      }
      half8* to = sm_a + (size_t)(r >> 4) * KK * 64 + (r & 15);
      to[(c / 4) * 64 + (c % 4) * 16] = below;
      to[((c + PPR) / 4) * 64 + ((c + PPR) % 4) * 16] = above;
    }
    __syncthreads();
  }
};

// Scores of blocks [b0, b1) for some tokens.  A wavefront has 16 blocks at a time, a block a column.  The first ones
// are requested when this is made: a block's number and its bounds are two latencies, one after the other.
template <int D, int W>
struct BlockScores {  // W: wavefronts of the workgroup
  static constexpr int KK = 2 * D / 32;
  struct Bounds {
    half8 x[KK];
  };
  const SelectParams& p;
  const int32_t* table;
  int head, b0, b1, n, id;  // n: of the wavefront's sixteens; id: of the lane's block in the next one
  Bounds a, b;
  __device__ __forceinline__ BlockScores(const SelectParams& p_, const int32_t* table_, int head_, int b0_, int b1_)
      : p(p_), table(table_), head(head_), b0(b0_), b1(b1_) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    n = max(own_tiles((b1 - b0 + 15) / 16, wave, W), 0);
    id = table[block(0)];
    const int second = table[block(1)];
    request(a);
    id = second;
  }
  __device__ __forceinline__ int first(int i) const { return b0 + ((int)(threadIdx.x >> 6) + W * i) * 16; }
  __device__ __forceinline__ int block(int i) const { return min(first(i) + (int)(threadIdx.x & 15), b1 - 1); }
  __device__ __forceinline__ void request(Bounds& t) const {
    const _Float16* from = p.bounds + ((size_t)clamp_block(id, p.n_blocks) * p.n_heads + head) * 2 * D + ((threadIdx.x & 63) >> 4) * 8;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) t.x[kk] = load_half8(from + kk * 32);
    requests_first();
  }
  // out(token, block, score); room: 16 numbers for every row, the wavefront's own.  Returns the largest
  // magnitude of the bounds that the thread has seen, as fp16 bits.
  template <typename Out>
  __device__ __forceinline__ uint32_t run(int n_tokens, const half8* sm_a, float* room, Out out) {
    const int lane = threadIdx.x & 63, col = lane & 15, part = lane >> 4;
    const int tiles = (n_tokens * p.group + 15) >> 4;
    uint32_t most = 0;
    auto use = [&](int i, const Bounds& t) {
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        const uint4v w = __builtin_bit_cast(uint4v, t.x[kk]);
#pragma unroll
        for (int j = 0; j < 4; ++j) most = max(most, max(w[j] & 0x7fffu, (w[j] >> 16) & 0x7fffu));
      }
      for (int tile = 0; tile < tiles; ++tile) {
        floatx4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
          s = __builtin_amdgcn_mfma_f32_16x16x32_f16(sm_a[(tile * KK + kk) * 64 + lane], t.x[kk], s, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r) room[(tile * 16 + part * 4 + r) * 16 + col] = s[r];
      }
      wave_lds_barrier();
      // (a score that is not a number: E is none, too)
      if (first(i) + col < b1)
        for (int token = part; token < n_tokens; token += 4) {
          float best = -INFINITY;
          for (int h = 0; h < p.group; ++h) best = fmaxf(best, room[(token * p.group + h) * 16 + col]);
          out(token, first(i) + col, best);
        }
      wave_lds_barrier();
    };
    // (behind the last sixteen: the last block again, of which nothing is made)
    for (int i = 0; i < n; i += 2) {
      int ahead = table[block(i + 2)];
      request(b);
      id = ahead;
      use(i, a);
      if (i + 1 == n) break;
      ahead = table[block(i + 3)];
      request(a);
      id = ahead;
      use(i + 1, b);
    }
    return most;
  }
};

// The order of the scores in 64 bits of the n blocks listed, into keys[].  D / 8 neighbouring lanes a block;
// sm_q: the queries [query head of the group][D].
// A score is the sum rounded once, whatever the order: a product is a multiple of 2^-48 below 2^32, more than the 53
// bits of a number can add up (2^30 + 2^-24 - 2^30), so its multiple of 2^-10 and what is left of it are added up apart,
// up to 128 of each in 49 and 44 bits.  (One sum in 64 bits, whose order decides between such blocks: a step of
// single tokens of 48 caches of 1280-7040, 8 heads of 4, 55.5 us, so 55.9; of 10 tokens over 28 000-30 000 32.2, 32.7)
template <int D, int W>
__device__ __forceinline__ void score_exactly(const SelectParams& p, const _Float16* sm_q, int head, const int32_t* blocks, int n,
                                              uint64_t* keys) {
  constexpr int PPR = D / 8;
  const int piece = threadIdx.x % PPR;
  for (int i = threadIdx.x / PPR; i < n; i += 64 * W / PPR) {
    const _Float16* from = p.bounds + ((size_t)clamp_block(blocks[i], p.n_blocks) * p.n_heads + head) * 2 * D + piece * 8;
    const half8 lo = load_half8(from), hi = load_half8(from + D);
    uint64_t best = 0;
    for (int h = 0; h < p.group; ++h) {
      const half8 q = load_half8(sm_q + h * D + piece * 8);
      double upper = 0x1.8p42, lower = 0.0;  // (a last place of 2^-10 for all that is added up)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double x = (double)fmaxf((float)q[e] * (float)lo[e], (float)q[e] * (float)hi[e]);
        const double next = upper + x;
        lower += x - (next - upper);
        upper = next;
      }
      upper -= 0x1.8p42;
      auto join = [](double& x) {
        x += from_lane_f64<0xB1>(x);
        x += from_lane_f64<0x4E>(x);
        x += from_lane_f64<0x141>(x);
        if constexpr (PPR == 16) x += from_lane_f64<0x140>(x);
      };
      join(upper);
      join(lower);
      // (of what is infinite nothing is left that is a number)
      const uint64_t key = score_order(fabs(upper) < INFINITY ? upper + lower : upper);
      best = key > best ? key : best;
    }
    if (piece == 0) keys[i] = best;
  }
}

constexpr int kMaxKeys = kPlanMaxSeqLen / kPlanBlockSize;
template <int W>
constexpr int kPerThread = kMaxKeys / (64 * W);  // blocks of a thread

// set bits of the lanes below this one
__device__ __forceinline__ uint32_t below_lane(uint64_t set) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(set >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)set, 0));
}

// For every element i = j * 64 * W + thread (j < mine): how many before it have the first flag and how many the second,
// in the low and high half of before[j]; returns how many there are of each.  counts: kPerThread<W> * W numbers in
// LDS, free when all threads are here.
template <int W, typename One, typename Two>
__device__ __forceinline__ uint32_t places_of(int mine, One one, Two two, uint32_t* counts, uint32_t* before) {
  static_assert(kPerThread<W> * W <= 64 && kMaxKeys < 1 << 16, "a count a lane, two in a word");
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
  for (int j = 0; j < kPerThread<W>; ++j) {
    const uint64_t a = j < mine ? __ballot(one(j)) : 0, b = j < mine ? __ballot(two(j)) : 0;
    before[j] = below_lane(a) | below_lane(b) << 16;
    if (j < mine && lane == 0) counts[j * W + wave] = __popcll(a) | __popcll(b) << 16;
  }
  __syncthreads();
  const uint32_t own = lane < mine * W ? counts[lane] : 0;
  const uint32_t sum = (uint32_t)wave_scan_add((int)own);
#pragma unroll
  for (int j = 0; j < kPerThread<W>; ++j) before[j] += (uint32_t)__builtin_amdgcn_readlane((int)(sum - own), j * W + wave);
  return (uint32_t)__builtin_amdgcn_readlane((int)sum, 63);
}

// The k-th largest of n > k > 0 keys, key[j] of thread t being that of element j * 64 * W + t (0: none, no key is 0):
// a threshold that exactly k keys reach, or the k-th one itself where more do.  Two bits at a time from the first one
// in which keys differ, with three counts of all keys a step.
template <int W>
__device__ __forceinline__ uint64_t kth_largest(const uint64_t (&key)[kPerThread<W>], int n, int k) {
  typedef int int4v __attribute__((ext_vector_type(4)));
  __shared__ int4v sm_count[2][W];
  __shared__ uint64_t sm_most[W], sm_least[W];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int mine = (n + 64 * W - 1) / (64 * W);  // uniform
  uint64_t most = 0, least = ~0ull;
#pragma unroll
  for (int j = 0; j < kPerThread<W>; ++j) {
    most = key[j] > most ? key[j] : most;
    least = key[j] != 0 && key[j] < least ? key[j] : least;
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const uint64_t a = __shfl_xor((unsigned long long)most, d), b = __shfl_xor((unsigned long long)least, d);
    most = a > most ? a : most;
    least = b < least ? b : least;
  }
  if (lane == 0) {
    sm_most[wave] = most;
    sm_least[wave] = least;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < W; ++w) {
    most = sm_most[w] > most ? sm_most[w] : most;
    least = sm_least[w] < least ? sm_least[w] : least;
  }
  // all keys have the bits above the pair of the first one in which the largest and the smallest differ
  int shift = (63 - __builtin_clzll((most ^ least) | 1)) & ~1;
  uint64_t threshold = shift == 62 ? 0 : most >> (shift + 2) << (shift + 2);
  int reached = n;  // by so many keys
  for (int step = 0; shift >= 0 && reached != k; shift -= 2, ++step) {
    int count[4] = {};
#pragma unroll
    for (int d = 1; d < 4; ++d) {
      const uint64_t candidate = threshold | (uint64_t)d << shift;
#pragma unroll
      for (int j = 0; j < kPerThread<W>; ++j)
        if (j < mine) count[d] += __popcll(__ballot(key[j] >= candidate));
    }
    if (lane == 0) sm_count[step & 1][wave] = int4v{0, count[1], count[2], count[3]};
    __syncthreads();
    int4v sum = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < W; ++w) sum += sm_count[step & 1][w];
    const int d = sum[3] >= k ? 3 : sum[2] >= k ? 2 : sum[1] >= k ? 1 : 0;
    threshold |= (uint64_t)d << shift;
    if (d > 0) reached = d == 3 ? sum[3] : d == 2 ? sum[2] : sum[1];
  }
  return threshold;
}

// What a selection needs of LDS: blocks between, their keys, whether they are kept.
struct Between {
  int32_t* blocks;
  uint64_t* keys;
};
constexpr size_t between_bytes(int n) { return (size_t)((n + 1) / 2 * 2) * (sizeof(int32_t) + sizeof(uint64_t)); }

// What a thread knows of blocks j * 64 * W + thread of a table (-infinity, 0 behind the last one).
template <int W>
struct Scored {
  float score[kPerThread<W>];
  int32_t id[kPerThread<W>];
  int32_t last_id;  // of the token's own block, which is not scored
};

constexpr int kBuckets = 1024;  // of scores, as wide as each other

// The k best of n > k > 0 blocks by their scores, out(place, j) in ascending order.  sm_q as above, made by threads
// that need not have met since; most: the largest magnitude of a bound.
// The k-th largest score T is looked for only as far as the bucket that holds it: what is in its reach, 2 E and the
// bucket, is scored anew.  (With T itself, found bit by bit with a count of all keys and a barrier for each, 5.1 us for
// 1809 blocks and 2.7 for 92; so 1.4.)
template <int D, int W, typename Out>
__device__ __forceinline__ void select_best(const SelectParams& p, const _Float16* sm_q, int head, const Scored<W>& b, int n, int k, float most,
                                            Between between, Out out) {
  static_assert(kBuckets % (64 * W) == 0, "whole");
  constexpr int kOwn = kBuckets / (64 * W);
  __shared__ uint32_t sm_place[kPerThread<W> * W];
  __shared__ uint32_t sm_bucket[kBuckets];
  __shared__ float sm_sum[W], sm_top[W], sm_low[W];
  __shared__ int sm_above[W], sm_found;
  __shared__ uint64_t sm_kept;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int mine = (n + 64 * W - 1) / (64 * W);
  float top = -INFINITY, low = INFINITY;
#pragma unroll
  for (int j = 0; j < kPerThread<W>; ++j) {
    if (j * 64 * W + (int)threadIdx.x >= n) continue;
    top = fmaxf(top, b.score[j]);
    low = fminf(low, b.score[j]);
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    top = fmaxf(top, __shfl_xor(top, d));
    low = fminf(low, __shfl_xor(low, d));
  }
  for (int i = 0; i < kOwn; ++i) sm_bucket[i * 64 * W + threadIdx.x] = 0;
  if (lane == 0) {
    sm_top[wave] = top;
    sm_low[wave] = low;
  }
  __syncthreads();
  // the largest sum of |q|
  float sum = 0.f;
  for (int h = wave; h < p.group; h += W) {
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) s += fabsf((float)sm_q[h * D + lane * (D / 64) + c]);
    s = wave_sum(s);
    sum = s > sum || s != s ? s : sum;
  }
  if (lane == 0) sm_sum[wave] = sum;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    top = fmaxf(top, sm_top[w]);
    low = fminf(low, sm_low[w]);
  }
  // bucket 0: the best.  (Monotone in the score, whatever the rounding; all in one where the range is nothing, or none)
  const float per = kBuckets / (top - low), scale = per < 3e38f ? per : 0.f;
  auto bucket_of = [&](float s) { return min((int)fmaxf((top - s) * scale, 0.f), kBuckets - 1); };
#pragma unroll
  for (int j = 0; j < kPerThread<W>; ++j)
    if (j * 64 * W + (int)threadIdx.x < n) atomicAdd(&sm_bucket[bucket_of(b.score[j])], 1u);
  __syncthreads();
  int own[kOwn], mine_sum = 0;
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    own[i] = (int)sm_bucket[threadIdx.x * kOwn + i];
    mine_sum += own[i];
  }
  const int scan = wave_scan_add(mine_sum);
  if (lane == 63) sm_above[wave] = scan;
  __syncthreads();
  int above = scan - mine_sum;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    above += w < wave ? sm_above[w] : 0;
    sum = sm_sum[w] > sum || sm_sum[w] != sm_sum[w] ? sm_sum[w] : sum;
  }
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    if (above < k && above + own[i] >= k) sm_found = (int)threadIdx.x * kOwn + i;
    above += own[i];
  }
  __syncthreads();
  const int found = sm_found;
  // Sure: over every score of that bucket by more than 2 E; out of reach: as far below.  (The bucket's ends, and a
  // little more than 2 E: this arithmetic is rounded, by less than a thousandth of a bucket and 2^-22 of a score,
  // of which 2 E is 2^-14 at least)
  const float margin = 2.1f * (2 * D) * 0x1p-23f * sum * most;
  const float width = scale > 0.f ? (top - low) * (1.f / kBuckets) : top - low;
  const float sure_from = top - (found - 0.01f) * width + margin, least = top - (found + 1.01f) * width - margin;
  const bool all = !(margin < INFINITY) || !(width < INFINITY);
  auto within = [&](int j) { return j * 64 * W + (int)threadIdx.x < n; };
  auto is_sure = [&](int j) { return within(j) && !all && b.score[j] > sure_from; };
  auto is_between = [&](int j) { return within(j) && (all || (b.score[j] >= least && b.score[j] <= sure_from)); };
  uint32_t before[kPerThread<W>];
  const uint32_t n_both = places_of<W>(mine, is_sure, is_between, sm_place, before);
  const int n_between = (int)(n_both >> 16), wanted = k - (int)(n_both & 0xffff);  // of those between
  if (n_between == wanted) {
#pragma unroll
    for (int j = 0; j < kPerThread<W>; ++j)
      if (is_sure(j) || is_between(j)) out((before[j] & 0xffff) + (before[j] >> 16), j);
    return;
  }
#pragma unroll
  for (int j = 0; j < kPerThread<W>; ++j)
    if (is_between(j)) between.blocks[before[j] >> 16] = b.id[j];
  __syncthreads();
  score_exactly<D, W>(p, sm_q, head, between.blocks, n_between, between.keys);
  __syncthreads();
  if (n_between <= 64) {
    // (ties: the lower blocks, which come first)
    if (wave == 0) {
      const uint64_t own_key = lane < n_between ? between.keys[lane] : 0;
      int rank = 0;
      for (int i = 0; i < n_between; ++i) {
        const uint64_t other = between.keys[i];
        rank += other > own_key || (other == own_key && i < lane) ? 1 : 0;
      }
      const uint64_t kept = __ballot(lane < n_between && rank < wanted);
      if (lane == 0) sm_kept = kept;
    }
    __syncthreads();
    const uint64_t kept = sm_kept;
#pragma unroll
    for (int j = 0; j < kPerThread<W>; ++j) {
      const int i = (int)(before[j] >> 16);
      const bool keep = is_between(j) && (kept >> i & 1);
      if (keep || is_sure(j)) out((before[j] & 0xffff) + (i < 64 ? __popcll(kept & ((1ull << i) - 1)) : __popcll(kept)), j);
    }
    return;
  }
  uint64_t exact[kPerThread<W>];
  const int parts = (n_between + 64 * W - 1) / (64 * W);
#pragma unroll
  for (int j = 0; j < kPerThread<W>; ++j) {
    const int i = j * 64 * W + (int)threadIdx.x;
    exact[j] = i < n_between ? between.keys[i] : 0;
  }
  const uint64_t threshold = kth_largest<W>(exact, n_between, wanted);
  // of the keys that are equal to the threshold the first ones stay
  uint32_t place[kPerThread<W>];
  const uint32_t n_above = places_of<W>(parts, [&](int j) { return exact[j] > threshold; }, [&](int j) { return exact[j] == threshold; },
                                     sm_place, place) & 0xffff;
#pragma unroll
  for (int j = 0; j < kPerThread<W>; ++j) {
    const int i = j * 64 * W + (int)threadIdx.x;
    if (i < n_between) between.blocks[i] = exact[j] > threshold || (exact[j] == threshold && (place[j] >> 16) < (uint32_t)wanted - n_above);
  }
  __syncthreads();
  uint64_t keep = 0;
#pragma unroll
  for (int j = 0; j < kPerThread<W>; ++j)
    if (is_sure(j) || (is_between(j) && between.blocks[before[j] >> 16])) keep |= 1ull << j;
  places_of<W>(mine, [&](int j) { return (keep >> j & 1) != 0; }, [](int) { return false; }, sm_place, place);
#pragma unroll
  for (int j = 0; j < kPerThread<W>; ++j)
    if (keep >> j & 1) out(place[j] & 0xffff, j);
}

// Keys that a token reads which sees so many: whole blocks, but for its own, the last one.
__device__ __forceinline__ int selected_keys(int seen, int n_select) {
  return (min((seen + 15) >> 4, n_select) - 1) * 16 + ((seen - 1) & 15) + 1;
}

// What a token's head reads: the blocks selected, then the token's own one (all, if there are no more).
struct Selection {
  int32_t *ids, *selected;  // blocks of the pool; nullable: entries of the table, -1 behind the last one
  __device__ __forceinline__ Selection(const SelectParams& p, int32_t* ids_, int64_t at)
      : ids(ids_), selected(p.selected ? p.selected + at * p.n_select : nullptr) {}
  __device__ __forceinline__ void put(int place, int block, int32_t id) const {
    ids[place] = id;
    if (selected) selected[place] = block;
  }
  // true if there was nothing to choose
  template <int W>
  __device__ __forceinline__ bool put_all(const SelectParams& p, const int32_t* table, int nb) const {
    if (nb > p.n_select && p.n_select > 1) return false;
    if (nb > p.n_select) {
      if (threadIdx.x == 0) put(0, nb - 1, table[nb - 1]);
      return true;
    }
    for (int b = threadIdx.x; b < p.n_select; b += 64 * W) {
      if (b < nb)
        put(b, b, table[b]);
      else if (selected)
        selected[b] = -1;
    }
    return true;
  }
};
template <int D, int W>
__device__ __forceinline__ void write_selection(const SelectParams& p, const _Float16* sm_q, int nb, int head, const Selection& to,
                                                const Scored<W>& b, float most, Between between) {
  select_best<D, W>(p, sm_q, head, b, nb - 1, p.n_select - 1, most, between,
                    [&](int place, int j) { to.put(place, j * 64 * W + (int)threadIdx.x, b.id[j]); });
  if (threadIdx.x == 0) to.put(p.n_select - 1, nb - 1, b.last_id);
}

// Where the thread's blocks lie; the queries to LDS.
template <int W>
__device__ __forceinline__ void request_blocks(const int32_t* table, int n, Scored<W>& b) {
#pragma unroll
  for (int j = 0; j < kPerThread<W>; ++j) {
    const int i = j * 64 * W + (int)threadIdx.x;
    b.id[j] = i < n ? table[i] : 0;
  }
  b.last_id = table[n];
}
template <int D, int W>
__device__ __forceinline__ void request_queries(const SelectParams& p, int row, int head, _Float16* sm_q) {
  for (int i = threadIdx.x; i < p.group * (D / 8); i += 64 * W) {
    const int h = i / (D / 8), c = i % (D / 8);
    store_half8(sm_q + h * D + c * 8, load_half8(query_of(p, row, head * p.group + h) + c * 8));
  }
}

// The largest of fp16 magnitudes as a number: not one, where one isn't.
__device__ __forceinline__ float magnitude(uint32_t bits) { return (float)__builtin_bit_cast(_Float16, (uint16_t)bits); }


// LDS for the operands of so many rows and the wavefronts' rooms, ...
inline size_t operand_bytes(const SelectParams& p, int rows, int waves) {
  return (size_t)((rows + 15) & ~15) * (2 * p.head_dim * 2 + waves * 16 * sizeof(float));
}
// ... for select_for_token: queries, scores, then the operands and rooms, and in their place what is between.
inline size_t select_bytes(const SelectParams& p, int waves) {
  return (size_t)p.group * p.head_dim * sizeof(_Float16) + ((p.lds_keys * sizeof(float) + 15) & ~(size_t)15) +
         std::max(between_bytes(p.lds_keys), operand_bytes(p, p.group, waves));
}

// Scores and selection by one workgroup of W wavefronts, of the one new token of a request (group up to kScoreRows / 2).
template <int D, int W>
__device__ __forceinline__ void select_for_token(const SelectParams& p, const ChunkReq& rq, int head, const Selection& to, char* sm) {
  __shared__ uint32_t sm_most[W];
  const int nb = (rq.seq_len + 15) >> 4;
  const int32_t* table = p.block_tables + (size_t)rq.table_row * p.max_blocks;
  if (to.put_all<W>(p, table, nb)) return;
  _Float16* sm_q = reinterpret_cast<_Float16*>(sm);
  float* scores = reinterpret_cast<float*>(sm_q + p.group * D);
  char* rest = reinterpret_cast<char*>(scores) + ((p.lds_keys * sizeof(float) + 15) & ~(size_t)15);
  const int rows = (p.group + 15) & ~15;
  half8* sm_a = reinterpret_cast<half8*>(rest);
  float* room = reinterpret_cast<float*>(rest + rows * 2 * D * 2) + (threadIdx.x >> 6) * rows * 16;
  const ScoredQueries<D, kScoreRows / 2, 64 * W> queries(p, rq.row_off, 1, head);
  BlockScores<D, W> blocks(p, table, head, 0, nb - 1);
  Scored<W> b;
  request_blocks<W>(table, nb - 1, b);
  queries.put(sm_a, sm_q);
  uint32_t most = blocks.run(1, sm_a, room, [&](int, int i, float s) { scores[i] = s; });
  most = wave_max(most);
  if ((threadIdx.x & 63) == 0) sm_most[threadIdx.x >> 6] = most;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < W; ++w) most = max(most, sm_most[w]);
#pragma unroll
  for (int j = 0; j < kPerThread<W>; ++j) {
    const int i = j * 64 * W + (int)threadIdx.x;
    b.score[j] = i < nb - 1 ? scores[i] : -INFINITY;
  }
  uint64_t* keys = reinterpret_cast<uint64_t*>(rest);
  write_selection<D, W>(p, sm_q, nb, head, to, b, magnitude(most), Between{reinterpret_cast<int32_t*>(keys + p.lds_keys), keys});
}

}  // namespace fc
