// Attention over selected blocks: the bounds of blocks, and, where the scores take a launch of their own, which
// blocks a query selects by them (fc_select_blocks.h).  What is selected is attended to by the kernels of
// fc_attention.hip, through block tables of its own for every token and head.
//
// bounds: lo_c = min k_c, hi_c = max k_c over the tokens of a block, one head.
// score of a block for query heads q_1 .. q_g of a head of K:
//     max over h of sum over c of max(q_hc lo_c, q_hc hi_c)  >=  q_h . k  for every k of the block.

#include <algorithm>
#include <type_traits>

#include "fc_e2m1.h"
#include "fc_select_blocks.h"

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
// bounds: workgroup = block of a request; a lane has 16 bytes of a head's rows, 8, 16 or 32 channels, and walks the
// block's 16 rows, all of them requested before any is used.  Memory bounds it: K is read once (64 caches of 1280-7040
// tokens, 32 heads of 128 channels, 8 bits: 264 us = 5.1 TB/s of 1.08 GB read and 0.27 written).
// The 80 blocks of 640 tokens take 4.4 us, a third of the CUs and one chain of latencies.
// ---------------------------------------------------------------------------
template <int D, int kFormat, typename Reqs>
__global__ __launch_bounds__(256) void bounds_kernel(BoundsParams p, Reqs reqs) {
  constexpr int C = kFormat == ROWS_F16 ? 8 : kFormat == ROWS_E4M3 ? 16 : 32;  // channels of a lane
  constexpr int LPR = D / C;
  const ChunkReq rq = reqs.req[request_of(0, p.n_req, blockIdx.x, [&](int i) { return reqs.req[i].unit_start; })];
  const int b = rq.row_off + (int)blockIdx.x - rq.unit_start;
  const int blk = clamp_block(p.block_tables[(size_t)rq.table_row * p.max_blocks + b], p.n_blocks);
  const int tokens = min(16, rq.seq_len - b * 16);
  const int piece = threadIdx.x % LPR;
  const size_t bytes = kFormat == ROWS_E4M3   ? e4m3_block_bytes(p.n_heads, D)
                       : kFormat == ROWS_E2M1 ? e2m1_block_bytes(p.n_heads, D)
                                              : (size_t)2 * p.n_heads * 16 * D * sizeof(_Float16);
  const uint8_t* block = static_cast<const uint8_t*>(p.kv) + (size_t)blk * bytes;
  for (int head = threadIdx.x / LPR; head < p.n_heads; head += 256 / LPR) {
    const uint8_t* rows = block + (size_t)head * 16 * LPR * 16 + piece * 16;
    uint4v x[16];
    uint32_t e[16];
#pragma unroll
    for (int s = 0; s < 16; ++s) {  // (behind the last token: the last one)
      const int row = min(s, tokens - 1);
      x[s] = __builtin_nontemporal_load(reinterpret_cast<const uint4v*>(rows + row * LPR * 16));
      if constexpr (kFormat == ROWS_E4M3) e[s] = block[(size_t)2 * p.n_heads * 16 * D + head * 16 + row];
      if constexpr (kFormat == ROWS_E2M1) e[s] = block[e2m1_code_bytes(p.n_heads, D) + (head * 16 + row) * LPR + piece];
    }
    half8 lo[C / 8], hi[C / 8];
#pragma unroll
    for (int s = 0; s < 16; ++s)
#pragma unroll
      for (int i = 0; i < C / 8; ++i) {
        half8 y;
        if constexpr (kFormat == ROWS_E4M3)
          y = e4m3_values(x[s][2 * i], x[s][2 * i + 1], e4m3_scale(e[s]));
        else if constexpr (kFormat == ROWS_E2M1)
          y = e2m1_values(x[s][i], e4m3_scale(e[s]));
        else
          y = __builtin_bit_cast(half8, x[s]);
        // (not a number, where one is)
        lo[i] = s == 0 ? y : __builtin_elementwise_minimum(lo[i], y);
        hi[i] = s == 0 ? y : __builtin_elementwise_maximum(hi[i], y);
      }
    _Float16* to = p.bounds + ((size_t)blk * p.n_heads + head) * 2 * D + piece * C;
#pragma unroll
    for (int i = 0; i < C / 8; ++i) {
      store_half8(to + 8 * i, lo[i]);
      store_half8(to + D + 8 * i, hi[i]);
    }
  }
}

// Workgroups of the kernels that select have this many wavefronts (with four, the scores of 1809 blocks, eight a thread,
// took 8.5 us to select from, where 1.6 are for what is read first).
constexpr int kSelectWaves = 8, kSelectThreads = 64 * kSelectWaves;

// Scores: workgroup = (part of the blocks, some tokens of a request, head).  The requests: n_new tokens,
// state_off blocks that the last one scores, in parts of p.part_blocks.
template <int D, typename Reqs>
__global__ __launch_bounds__(kThreads) void block_scores_kernel(SelectParams p, Reqs reqs) {
  extern __shared__ __align__(16) char sm[];
  __shared__ uint32_t sm_most[kWaves];
  const int unit = blockIdx.x / p.n_heads;
  const int head = blockIdx.x - unit * p.n_heads;
  const ChunkReq rq = reqs.req[request_of(0, p.n_req, unit, [&](int i) { return reqs.req[i].unit_start; })];
  const int32_t* table = p.block_tables + (size_t)rq.table_row * p.max_blocks;
  const int parts = (rq.state_off + p.part_blocks - 1) / p.part_blocks;
  const int tile = (unit - rq.unit_start) / parts, part = (unit - rq.unit_start) - tile * parts;
  const int first = tile * p.tile_tokens, n_tokens = min(p.tile_tokens, rq.n_new - first);
  const int rows = (n_tokens * p.group + 15) & ~15;
  half8* sm_a = reinterpret_cast<half8*>(sm);
  float* room = reinterpret_cast<float*>(sm + rows * 2 * D * 2) + (threadIdx.x >> 6) * rows * 16;
  const ScoredQueries<D, kScoreRows, kThreads> queries(p, rq.row_off + first, n_tokens, head);
  BlockScores<D, kWaves> blocks(p, table, head, part * p.part_blocks, min((part + 1) * p.part_blocks, rq.state_off));
  queries.put(sm_a, nullptr);
  float* scores = p.scores + ((int64_t)(rq.row_off + first) * p.n_heads + head) * p.score_stride;
  uint32_t most = blocks.run(n_tokens, sm_a, room,
                             [&](int token, int b, float s) { scores[(int64_t)token * p.n_heads * p.score_stride + b] = s; });
  most = wave_max(most);
  if ((threadIdx.x & 63) == 0) sm_most[threadIdx.x >> 6] = most;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 0; w < kWaves; ++w) most = max(most, sm_most[w]);
    p.most[(int64_t)unit * p.n_heads + head] = most;
  }
}

// The selection: workgroup = (token, head).  The tokens: unit_start the first part's unit, n_new their number.
template <int D, typename Reqs>
__global__ __launch_bounds__(kSelectThreads) void select_scored_kernel(SelectParams p, Reqs reqs) {
  extern __shared__ __align__(16) char sm[];
  const int token = blockIdx.x / p.n_heads;
  const int head = blockIdx.x - token * p.n_heads;
  const ChunkReq rq = reqs.req[token];
  const int nb = (rq.seq_len + 15) >> 4;
  const int32_t* table = p.block_tables + (size_t)rq.table_row * p.max_blocks;
  const int64_t at = (int64_t)token * p.n_heads + head;
  const Selection to(p, p.ids + at * p.n_select, at);
  if (to.put_all<kSelectWaves>(p, table, nb)) return;
  _Float16* sm_q = reinterpret_cast<_Float16*>(sm);
  uint64_t* keys = reinterpret_cast<uint64_t*>(sm_q + p.group * D);
  // (all of it requested before any of it is waited for)
  Scored<kSelectWaves> b;
#pragma unroll
  for (int j = 0; j < kPerThread<kSelectWaves>; ++j) b.score[j] = p.scores[at * p.score_stride + min(j * kSelectThreads + (int)threadIdx.x, nb - 2)];
  request_blocks<kSelectWaves>(table, nb - 1, b);
  uint32_t most = 0;
  for (int i = threadIdx.x & 63; i < rq.n_new; i += 64) most = max(most, p.most[(int64_t)(rq.unit_start + i) * p.n_heads + head]);
  request_queries<D, kSelectWaves>(p, rq.row_off, head, sm_q);
  most = wave_max(most);
  write_selection<D, kSelectWaves>(p, sm_q, nb, head, to, b, magnitude(most), Between{reinterpret_cast<int32_t*>(keys + p.lds_keys), keys});
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

hipError_t launch_select_blocks(const SelectParams& p, const ChunkReqs& inline_tokens, const ChunkReqs& inline_reqs, hipStream_t s) {
  if (p.n_tokens == 0) return hipSuccess;
  if ((p.head_dim != 64 && p.head_dim != 128) || p.group > kScoreRows || p.tile_tokens * p.group > kScoreRows || p.tile_tokens < 1 ||
      p.n_select < 1 || p.part_blocks < 1 || p.lds_keys < 1 || p.lds_keys > kMaxKeys || p.score_stride > kMaxKeys)
    return hipErrorInvalidValue;
  const unsigned heads = (unsigned)p.n_tokens * p.n_heads;
  const size_t between = between_bytes(p.lds_keys), queries = (size_t)p.group * p.head_dim * sizeof(_Float16);
  auto launch = [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    if (p.n_units > 0)
      with_reqs_of(p.reqs, inline_reqs, [&](const auto& reqs) {
        using Reqs = std::decay_t<decltype(reqs)>;
        block_scores_kernel<D, Reqs><<<(unsigned)p.n_units * p.n_heads, kThreads, operand_bytes(p, p.tile_tokens * p.group, kWaves), s>>>(p, reqs);
      });
    with_reqs_of(p.tokens, inline_tokens, [&](const auto& reqs) {
      using Reqs = std::decay_t<decltype(reqs)>;
      select_scored_kernel<D, Reqs><<<heads, kSelectThreads, queries + between, s>>>(p, reqs);
    });
  };
  if (p.head_dim == 128)
    launch(std::integral_constant<int, 128>());
  else
    launch(std::integral_constant<int, 64>());
  return hipGetLastError();
}

}  // namespace fc
