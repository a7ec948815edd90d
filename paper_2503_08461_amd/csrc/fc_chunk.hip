// Chunks of new tokens on their way into the pool: the blocks they need, their K and V rows,
// and the copy of a cache from an fp16 pool into an 8-bit one.  All of it is memory traffic.

#include <type_traits>

#include "fc_e4m3.h"

namespace fc {

// ---------------------------------------------------------------------------
// extend: workgroup = request that gets blocks; pops in batch order.  A few words a request: the
// launch is what it costs.
// ---------------------------------------------------------------------------
template <typename Reqs>
__global__ __launch_bounds__(64) void extend_kernel(ExtendParams p, Reqs reqs) {
  const ExtendReq rq = reqs.req[blockIdx.x];
  int32_t* row = p.block_tables + (size_t)rq.table_row * p.max_blocks + rq.first;
  for (int i = threadIdx.x; i < rq.n_pop; i += 64) {
    const int id = p.stack[p.top_before - 1 - rq.pop_index - i];
    row[i] = clamp_block(id, p.n_blocks);
    // ownership checks (debug mode): a popped block must have been free
    if (p.owner && ((unsigned)id >= (unsigned)p.n_blocks || atomicExch(&p.owner[id], 1) != 0))
      atomicOr(p.error_flag, 4 << 8);
  }
}

hipError_t launch_extend(const ExtendParams& p, const ExtendReqs& inline_reqs, hipStream_t s) {
  if (p.n_req == 0) return hipSuccess;
  if (p.reqs)
    extend_kernel<ExtendReqList><<<p.n_req, 64, 0, s>>>(p, ExtendReqList{p.reqs});
  else
    extend_kernel<ExtendReqs><<<p.n_req, 64, 0, s>>>(p, inline_reqs);
  return hipGetLastError();
}

// the request that unit u belongs to (units ascend with the requests)
template <typename Reqs>
__device__ __forceinline__ int request_of_unit(const Reqs& reqs, int n_req, int u) {
  return request_of(0, n_req, u, [&](int i) { return reqs.req[i].unit_start; });
}

template <typename F>
static void with_chunk_reqs(const ChunkReq* on_device, const ChunkReqs& inline_reqs, F f) {
  if (on_device)
    f(ChunkReqList{on_device});
  else
    f(inline_reqs);
}

// ---------------------------------------------------------------------------
// store: workgroup = new token; its 2 * n_heads rows of one layer go to its slot.  D / 8
// neighbouring lanes have a row, 16 bytes each; for the 8-bit pool they find the row's
// maximum among themselves.  Memory bounds it: 3-5 us for 48 tokens of 8 heads (latency), 17-19 us
// for 2293 tokens of 32 heads (75 MB read and written, 4.3 TB/s), 48 us for 8377 (275 MB, 5.7); 8-bit
// 16-18 us (56 MB, 3.3 TB/s) and 45-47 us (206 MB, 4.5).
// ---------------------------------------------------------------------------
template <int D, bool kE4M3, typename Reqs>
__global__ __launch_bounds__(256) void store_chunk_kernel(StoreParams p, Reqs reqs) {
  constexpr int PPR = D / 8;
  const ChunkReq rq = reqs.req[request_of_unit(reqs, p.n_req, blockIdx.x)];
  const int tok = rq.seq_len - rq.n_new + ((int)blockIdx.x - rq.row_off);
  const int blk = clamp_block(p.block_tables[(size_t)rq.table_row * p.max_blocks + (tok >> 4)], p.n_blocks);
  const int slot = tok & 15;
  const int n_rows = 2 * p.n_heads;
  // (whole rows: n_rows * PPR is a multiple of PPR and so is the step, the lanes of a row leave together)
  for (int i = threadIdx.x; i < n_rows * PPR; i += 256) {
    const int rh = i / PPR, piece = i % PPR;  // rh = kv * n_heads + head
    const RowsView& from = rh < p.n_heads ? p.k : p.v;
    const int head = rh < p.n_heads ? rh : rh - p.n_heads;
    const half8 x = load_half8(from.data + (int64_t)blockIdx.x * from.token_stride + head * from.head_stride + piece * 8);
    if constexpr (kE4M3) {
      uint8_t* block = static_cast<uint8_t*>(p.kv) + (size_t)blk * e4m3_block_bytes(p.n_heads, D);
      const int e = e4m3_exponent(row_max_u32<PPR>(finite_max(x)));
      *reinterpret_cast<uint2v*>(block + ((size_t)rh * 16 + slot) * D + piece * 8) = e4m3_codes(x, e);
      if (piece == 0) block[(size_t)n_rows * 16 * D + rh * 16 + slot] = (uint8_t)e;
    } else {
      _Float16* block = static_cast<_Float16*>(p.kv) + (size_t)blk * n_rows * 16 * D;
      store_half8(block + ((size_t)rh * 16 + slot) * D + piece * 8, x);
    }
  }
}

hipError_t launch_store_chunk(const StoreParams& p, const ChunkReqs& inline_reqs, hipStream_t s) {
  if (p.n_rows == 0) return hipSuccess;
  if (p.head_dim != 64 && p.head_dim != 128) return hipErrorInvalidValue;
  with_chunk_reqs(p.reqs, inline_reqs, [&](const auto& reqs) {
    using Reqs = std::decay_t<decltype(reqs)>;
    if (p.head_dim == 128 && p.e4m3)
      store_chunk_kernel<128, true, Reqs><<<p.n_rows, 256, 0, s>>>(p, reqs);
    else if (p.head_dim == 128)
      store_chunk_kernel<128, false, Reqs><<<p.n_rows, 256, 0, s>>>(p, reqs);
    else if (p.e4m3)
      store_chunk_kernel<64, true, Reqs><<<p.n_rows, 256, 0, s>>>(p, reqs);
    else
      store_chunk_kernel<64, false, Reqs><<<p.n_rows, 256, 0, s>>>(p, reqs);
  });
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// quantise: workgroup = block of a request in one layer: 32 * n_heads rows, read once, and as many
// rows of half the bytes written, in whole lines but for the exponents (32 * n_heads bytes, a few of
// a line at a time, which the L2 joins).  Memory bounds it: 64 caches of 256-1408 tokens, 32 heads
// of 128 channels, 4 layers, 1060 us = 4.85 TB/s read and written, what a large copy reaches here.
// ---------------------------------------------------------------------------
template <int D, typename Reqs>
__global__ __launch_bounds__(256) void quantise_kernel(QuantiseParams p, Reqs reqs) {
  constexpr int PPR = D / 8;
  const int layer = blockIdx.x / p.n_units;
  const int unit = blockIdx.x - layer * p.n_units;
  const ChunkReq rq = reqs.req[request_of_unit(reqs, p.n_req, unit)];
  const int b = unit - rq.unit_start;
  const int from = clamp_block(p.src_tables[(size_t)rq.table_row * p.src_max_blocks + b], p.src_blocks);
  const int to = clamp_block(p.dst_tables[(size_t)rq.table_row * p.dst_max_blocks + b], p.dst_blocks);
  const int slots = min(16, rq.seq_len - b * 16);
  const int n_rows = 2 * p.n_heads;
  const _Float16* src = p.src + ((size_t)layer * p.src_blocks + from) * n_rows * 16 * D;
  uint8_t* dst = p.dst + ((size_t)layer * p.dst_blocks + to) * e4m3_block_bytes(p.n_heads, D);
  for (int i = threadIdx.x; i < n_rows * 16 * PPR; i += 256) {
    const int row = i / PPR, piece = i % PPR;  // row = (kv * n_heads + head) * 16 + slot
    if ((row & 15) >= slots) continue;         // (all lanes of the row)
    const half8 x = load_half8_nt(src + (size_t)row * D + piece * 8);
    const int e = e4m3_exponent(row_max_u32<PPR>(finite_max(x)));
    *reinterpret_cast<uint2v*>(dst + (size_t)row * D + piece * 8) = e4m3_codes(x, e);
    if (piece == 0) dst[(size_t)n_rows * 16 * D + row] = (uint8_t)e;
  }
}

hipError_t launch_quantise(const QuantiseParams& p, const ChunkReqs& inline_reqs, hipStream_t s) {
  if (p.n_units == 0) return hipSuccess;
  if (p.head_dim != 64 && p.head_dim != 128) return hipErrorInvalidValue;
  const unsigned grid = (unsigned)p.n_units * p.n_layers;
  with_chunk_reqs(p.reqs, inline_reqs, [&](const auto& reqs) {
    using Reqs = std::decay_t<decltype(reqs)>;
    if (p.head_dim == 128)
      quantise_kernel<128, Reqs><<<grid, 256, 0, s>>>(p, reqs);
    else
      quantise_kernel<64, Reqs><<<grid, 256, 0, s>>>(p, reqs);
  });
  return hipGetLastError();
}

}  // namespace fc
