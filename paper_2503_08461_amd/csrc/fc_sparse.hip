// Attention over selected blocks: the bounds of blocks, and which blocks a query selects by them.
// (What is selected is attended to by the kernels of fc_attention.hip, through block tables of
// its own for every token and head.)
//
// bounds: lo_c = min k_c, hi_c = max k_c over the tokens of a block, one head.
// score of a block for query heads q_1 .. q_g of a head of K:
//     max over h of sum over c of max(q_hc lo_c, q_hc hi_c)  >=  q_h . k  for every k of the block.

#include "fc_e2m1.h"

namespace fc {

namespace {

template <typename F>
void with_reqs_of(const ChunkReq* on_device, const ChunkReqs& inline_reqs, F f) {
  if (on_device)
    f(ChunkReqList{on_device});
  else
    f(inline_reqs);
}

// ---------------------------------------------------------------------------
// bounds: workgroup = block of a request; D / 8 neighbouring lanes a head, eight channels each, walk
// the block's rows.  Memory bounds it: K is read once.
// ---------------------------------------------------------------------------
template <int D, int kFormat>
__device__ __forceinline__ half8 key_channels(const void* layer, int blk, int n_heads, int head, int slot, int piece) {
  const size_t row = (size_t)head * 16 + slot;
  if constexpr (kFormat == ROWS_E4M3) {
    const uint8_t* block = static_cast<const uint8_t*>(layer) + (size_t)blk * e4m3_block_bytes(n_heads, D);
    const uint2v c = *reinterpret_cast<const uint2v*>(block + row * D + piece * 8);
    return e4m3_values(c[0], c[1], e4m3_scale(block[(size_t)2 * n_heads * 16 * D + row]));
  } else if constexpr (kFormat == ROWS_E2M1) {
    const uint8_t* block = static_cast<const uint8_t*>(layer) + (size_t)blk * e2m1_block_bytes(n_heads, D);
    const uint32_t c = *reinterpret_cast<const uint32_t*>(block + row * (D / 2) + piece * 4);
    return e2m1_values(c, e4m3_scale(block[e2m1_code_bytes(n_heads, D) + row * (D / 32) + piece / 4]));
  } else {
    return load_half8(static_cast<const _Float16*>(layer) + (size_t)blk * 2 * n_heads * 16 * D + row * D + piece * 8);
  }
}

template <int D, int kFormat, typename Reqs>
__global__ __launch_bounds__(256) void bounds_kernel(BoundsParams p, Reqs reqs) {
  constexpr int PPR = D / 8;
  const ChunkReq rq = reqs.req[request_of(0, p.n_req, blockIdx.x, [&](int i) { return reqs.req[i].unit_start; })];
  const int b = rq.row_off + (int)blockIdx.x - rq.unit_start;
  const int blk = clamp_block(p.block_tables[(size_t)rq.table_row * p.max_blocks + b], p.n_blocks);
  const int tokens = min(16, rq.seq_len - b * 16);
  const int piece = threadIdx.x % PPR;
  for (int head = threadIdx.x / PPR; head < p.n_heads; head += 256 / PPR) {
    half8 x[16];
#pragma unroll
    for (int s = 0; s < 16; ++s)  // (behind the last token: the last one)
      x[s] = key_channels<D, kFormat>(p.kv, blk, p.n_heads, head, min(s, tokens - 1), piece);
    half8 lo = x[0], hi = x[0];
#pragma unroll
    for (int s = 1; s < 16; ++s) {
      // (not a number, where one is)
      lo = __builtin_elementwise_minimum(lo, x[s]);
      hi = __builtin_elementwise_maximum(hi, x[s]);
    }
    _Float16* to = p.bounds + ((size_t)blk * p.n_heads + head) * 2 * D + piece * 8;
    store_half8(to, lo);
    store_half8(to + D, hi);
  }
}

// ---------------------------------------------------------------------------
// selection.  Scores are sums of 64 bits: a product of two fp16 numbers is exact in fp32, and which of
// two blocks is read should follow from the inputs, not from the order in which a sum was made.
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

// The queries of a token's heads that share a head of K, as fp32 numbers in LDS: [query head][D].
template <int D>
__device__ __forceinline__ void queries_to_lds(const SelectParams& p, int row, int head, float* sm_q) {
  for (int i = threadIdx.x; i < p.group * (D / 8); i += kThreads) {
    const int h = i / (D / 8), piece = i % (D / 8);
    const half8 x = load_half8(p.q.data + (int64_t)row * p.q.token_stride + (int64_t)(head * p.group + h) * p.q.head_stride + piece * 8);
#pragma unroll
    for (int e = 0; e < 8; ++e) sm_q[h * D + piece * 8 + e] = (float)x[e];
  }
  __syncthreads();
}

// The order of blocks [b0, b1)'s scores into keys[b].  D / 8 neighbouring lanes a block.
template <int D>
__device__ __forceinline__ void score_blocks(const SelectParams& p, const int32_t* table, int head, const float* sm_q, int b0, int b1,
                                             uint64_t* keys) {
  constexpr int PPR = D / 8, kBlocks = 64 / PPR;  // of a wavefront at a time
  const int lane = threadIdx.x & 63, piece = lane % PPR;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  struct Bounds {
    half8 lo, hi;
  };
  auto block_of = [&](int i) { return b0 + (wave + kWaves * i) * kBlocks + lane / PPR; };
  stream_tiles<Bounds>(
      own_tiles((b1 - b0 + kBlocks - 1) / kBlocks, wave, kWaves),
      [&](int i, Bounds& x) {
        const int blk = clamp_block(table[min(block_of(i), b1 - 1)], p.n_blocks);
        const _Float16* from = p.bounds + ((size_t)blk * p.n_heads + head) * 2 * D + piece * 8;
        x.lo = load_half8(from);
        x.hi = load_half8(from + D);
      },
      [&](int i, const Bounds& x) {
        uint64_t best = 0;
        for (int h = 0; h < p.group; ++h) {
          const float* q = sm_q + h * D + piece * 8;
          double s = 0.0;
#pragma unroll
          for (int e = 0; e < 8; ++e) s += (double)fmaxf(q[e] * (float)x.lo[e], q[e] * (float)x.hi[e]);
          s += from_lane_f64<0xB1>(s);
          s += from_lane_f64<0x4E>(s);
          s += from_lane_f64<0x141>(s);
          if constexpr (PPR == 16) s += from_lane_f64<0x140>(s);
          const uint64_t key = score_order(s);
          best = key > best ? key : best;
        }
        if (piece == 0 && block_of(i) < b1) keys[block_of(i)] = best;
      });
}

// The k largest of n > k > 0 keys (ties: the lower indices) in ascending order of their indices, by one
// workgroup: out(place, index).  A threshold is found bit by bit from the first one in which keys
// differ, until as many keys as wanted reach it, with one count of all keys a bit.
constexpr int kMaxKeys = kPlanMaxSeqLen / kPlanBlockSize, kPerThread = kMaxKeys / kThreads;
template <typename Out>
__device__ __forceinline__ void select_largest(const uint64_t* keys, int n, int k, Out out) {
  __shared__ int sm_count[2][kWaves];
  __shared__ int sm_place[kPerThread * kWaves];
  __shared__ uint64_t sm_most[kWaves], sm_least[kWaves];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int mine = (n + kThreads - 1) / kThreads;  // uniform
  uint64_t key[kPerThread];
  uint64_t most = 0, least = ~0ull;
#pragma unroll
  for (int j = 0; j < kPerThread; ++j) {
    const int i = j * kThreads + (int)threadIdx.x;
    key[j] = 0;
    if (i < n) {
      key[j] = keys[i];
      most = key[j] > most ? key[j] : most;
      least = key[j] < least ? key[j] : least;
    }
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
  for (int w = 0; w < kWaves; ++w) {
    most = sm_most[w] > most ? sm_most[w] : most;
    least = sm_least[w] < least ? sm_least[w] : least;
  }
  // all keys have the bits above the first one in which the largest and the smallest differ
  int bit = 63 - __builtin_clzll((most ^ least) | 1);
  uint64_t threshold = bit == 63 ? 0 : most >> (bit + 1) << (bit + 1);
  int reached = n;
  for (int step = 0; bit >= 0 && reached != k; --bit, ++step) {
    const uint64_t candidate = threshold | 1ull << bit;
    int count = 0;
#pragma unroll
    for (int j = 0; j < kPerThread; ++j)
      if (j < mine) count += __popcll(__ballot(key[j] >= candidate));
    if (lane == 0) sm_count[step & 1][wave] = count;
    __syncthreads();
    count = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) count += sm_count[step & 1][w];
    if (count >= k) {
      threshold = candidate;
      reached = count;
    }
  }
  // `reached` keys are not below the threshold; of those that are equal to it the last ones go
  // places of a wavefront's flags among all of one kind: [j][wave] counts, summed before each
  auto places = [&](auto flag, int* before) {
    uint64_t set[kPerThread];
#pragma unroll
    for (int j = 0; j < kPerThread; ++j) {
      set[j] = j < mine ? __ballot(flag(j)) : 0;
      if (j < mine && lane == 0) sm_place[j * kWaves + wave] = __popcll(set[j]);
    }
    __syncthreads();
    const int own = lane < mine * kWaves ? sm_place[lane] : 0;
    const int sum = wave_scan_add(own) - own;
#pragma unroll
    for (int j = 0; j < kPerThread; ++j)
      before[j] = __builtin_amdgcn_readlane(sum, j * kWaves + wave) + __popcll(set[j] & ((1ull << lane) - 1));
    __syncthreads();
  };
  static_assert(kPerThread * kWaves <= 64, "a count a lane");
  int at[kPerThread];
  int spare = 0;  // of the keys equal to the threshold, how many are kept
  if (reached != k) {
    int above = 0;
#pragma unroll
    for (int j = 0; j < kPerThread; ++j)
      if (j < mine) above += __popcll(__ballot(key[j] > threshold));
    __syncthreads();  // (the last count has been read)
    if (lane == 0) sm_count[0][wave] = above;
    __syncthreads();
    above = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) above += sm_count[0][w];
    spare = k - above;
    places([&](int j) { return key[j] == threshold; }, at);
#pragma unroll
    for (int j = 0; j < kPerThread; ++j)
      if (key[j] == threshold && at[j] >= spare) key[j] = 0;  // (dropped)
  }
  places([&](int j) { return key[j] >= threshold && key[j] != 0; }, at);
#pragma unroll
  for (int j = 0; j < kPerThread; ++j)
    if (j < mine && key[j] >= threshold && key[j] != 0) out(at[j], j * kThreads + (int)threadIdx.x);
}

// What a token's head reads: the blocks selected, then the token's own one (all, if there are no more).
__device__ __forceinline__ void write_selection(const SelectParams& p, const int32_t* table, int nb, int64_t at, const uint64_t* keys) {
  int32_t* ids = p.ids + at * p.n_select;
  int32_t* selected = p.selected ? p.selected + at * p.n_select : nullptr;
  auto put = [&](int place, int b) {
    ids[place] = table[b];
    if (selected) selected[place] = b;
  };
  if (nb <= p.n_select) {
    for (int b = threadIdx.x; b < p.n_select; b += kThreads) {
      if (b < nb)
        put(b, b);
      else if (selected)
        selected[b] = -1;
    }
    return;
  }
  if (p.n_select > 1) select_largest(keys, nb - 1, p.n_select - 1, put);
  if (threadIdx.x == 0) put(p.n_select - 1, nb - 1);
}

// kPart: 0, a workgroup for a token's head, scores and selection; 1, a part of its blocks' scores; 2, the selection.
template <int D, int kPart, typename Reqs>
__global__ __launch_bounds__(kThreads) void select_blocks_kernel(SelectParams p, Reqs reqs) {
  extern __shared__ __align__(16) float sm_q[];  // [group][D], then (0) the keys
  const int at = blockIdx.x / p.n_heads;
  const int head = blockIdx.x - at * p.n_heads;
  int token = at;
  if constexpr (kPart == 1) token = request_of(0, p.n_tokens, at, [&](int i) { return reqs.req[i].unit_start; });
  const ChunkReq rq = reqs.req[token];
  const int nb = (rq.seq_len + 15) >> 4;
  const int32_t* table = p.block_tables + (size_t)rq.table_row * p.max_blocks;
  const int64_t unit = (int64_t)token * p.n_heads + head;
  if constexpr (kPart == 0) {
    uint64_t* keys = reinterpret_cast<uint64_t*>(sm_q + p.group * D);
    if (nb > p.n_select) {
      queries_to_lds<D>(p, rq.row_off, head, sm_q);
      score_blocks<D>(p, table, head, sm_q, 0, nb - 1, keys);
      __syncthreads();
    }
    write_selection(p, table, nb, unit, keys);
  } else if constexpr (kPart == 1) {
    queries_to_lds<D>(p, rq.row_off, head, sm_q);
    const int b0 = (at - rq.unit_start) * p.part_blocks;
    score_blocks<D>(p, table, head, sm_q, b0, min(b0 + p.part_blocks, nb - 1), p.keys + unit * p.key_stride);
  } else {
    write_selection(p, table, nb, unit, p.keys + unit * p.key_stride);
  }
}

}  // namespace

hipError_t launch_bounds(const BoundsParams& p, const ChunkReqs& inline_reqs, hipStream_t s) {
  if (p.n_units == 0) return hipSuccess;
  if (p.head_dim != 64 && p.head_dim != 128) return hipErrorInvalidValue;
  with_reqs_of(p.reqs, inline_reqs, [&](const auto& reqs) {
    using Reqs = std::decay_t<decltype(reqs)>;
    with_row_format(p.head_dim, p.format, [&](auto dim, auto format) {
      bounds_kernel<decltype(dim)::value, decltype(format)::value, Reqs><<<p.n_units, 256, 0, s>>>(p, reqs);
    });
  });
  return hipGetLastError();
}

hipError_t launch_select_blocks(const SelectParams& p, const ChunkReqs& inline_reqs, hipStream_t s) {
  if (p.n_tokens == 0) return hipSuccess;
  if ((p.head_dim != 64 && p.head_dim != 128) || p.n_select < 1 || p.lds_keys > kMaxKeys || (p.part_blocks && p.key_stride > kMaxKeys))
    return hipErrorInvalidValue;
  const unsigned heads = (unsigned)p.n_tokens * p.n_heads;
  const size_t queries = (size_t)p.group * p.head_dim * sizeof(float);
  with_reqs_of(p.reqs, inline_reqs, [&](const auto& reqs) {
    using Reqs = std::decay_t<decltype(reqs)>;
    auto launch = [&](auto dim) {
      constexpr int D = decltype(dim)::value;
      if (p.part_blocks == 0) {
        select_blocks_kernel<D, 0, Reqs><<<heads, kThreads, queries + p.lds_keys * sizeof(uint64_t), s>>>(p, reqs);
        return;
      }
      if (p.n_units > 0) select_blocks_kernel<D, 1, Reqs><<<(unsigned)p.n_units * p.n_heads, kThreads, queries, s>>>(p, reqs);
      select_blocks_kernel<D, 2, Reqs><<<heads, kThreads, 0, s>>>(p, reqs);
    };
    if (p.head_dim == 128)
      launch(std::integral_constant<int, 128>());
    else
      launch(std::integral_constant<int, 64>());
  });
  return hipGetLastError();
}

}  // namespace fc
