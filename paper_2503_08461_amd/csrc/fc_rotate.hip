// New tokens' q and k rotated by their positions, k and v on their way into the pool.
//
// A pair (a, b) of channels of a row at position p becomes (a cos - b sin, b cos + a sin) with the
// table's cosine and sine of p and of the pair.  Sums are made in 64 bits: the products of 16- and 32-bit
// numbers are exact there, so that the fp16 row is the one that the inputs determine, however it is
// computed (rounded to 32 and then to 16 bits), and with it the codes of a pool of fewer bits, whose
// largest channel may lie on either side of a border.
//
// Workgroup = new token.  D / 8 neighbouring lanes have a row, 16 bytes each, and load those of their
// partners beside their own; a thread's channels are the same in all of its rows, so the table's
// numbers are read once.  The next row is requested before this one is turned: a row is some forty
// instructions in 64 bits a lane.  Memory bounds it: 32 prompts of 600-1200 tokens, 32 heads of 128 channels, 283 us =
// 4.8 TB/s read and written, where a copy of 4 GiB reaches 4.7 (one row at a time 372 us); one token of four
// heads 2.2 us, a chain of three loads.

#include "fc_e2m1.h"

namespace fc {

namespace {

// Rounded to 32 bits, then to 16.  (Left to itself the compiler makes one rounding of the two, some
// thirty integer instructions for each number, in some of the kernels.)
__device__ __forceinline__ _Float16 rounded(double x) {
  float f = (float)x;
  asm volatile("" : "+v"(f));
  return (_Float16)f;
}

struct Angles {
  double cos[8], sin[8];  // of a lane's channels, the sine with the sign of the partner's part
};

template <int D, int kFormat, bool kInterleaved, typename Reqs>
__global__ __launch_bounds__(256) void rotate_store_kernel(RotateParams p, Reqs reqs) {
  constexpr int PPR = D / 8;
  const StoreParams& st = p.store;
  const int row = blockIdx.x;
  const ChunkReq rq = reqs.req[request_of(0, st.n_req, row, [&](int i) { return reqs.req[i].unit_start; })];
  const int at = row - rq.row_off;
  const int tok = rq.seq_len - rq.n_new + at;
  const int blk = clamp_block(st.block_tables[(size_t)rq.table_row * st.max_blocks + (tok >> 4)], st.n_blocks);
  const int slot = tok & 15;
  const int piece = threadIdx.x % PPR;  // (the step over rows is whole rows)
  const bool turned = piece * 8 < p.rotary;
  const int half = p.rotary / 2;
  // channels c and c + half are a pair, or 2 c and 2 c + 1: the partners' offset from the lane's channels
  const bool second = !kInterleaved && piece * 8 >= half;
  const int partner = kInterleaved ? 0 : second ? -half : half;
  Angles w;
  if (turned) {
    const float* cosines = p.table + (size_t)(rq.state_off + at) * p.rotary + (kInterleaved ? piece * 4 : piece * 8 - (second ? half : 0));
    float c[8], s[8];
    if constexpr (kInterleaved) {
      *reinterpret_cast<floatx4*>(c) = *reinterpret_cast<const floatx4*>(cosines);
      *reinterpret_cast<floatx4*>(s) = *reinterpret_cast<const floatx4*>(cosines + half);
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        *reinterpret_cast<floatx4*>(c + 4 * i) = *reinterpret_cast<const floatx4*>(cosines + 4 * i);
        *reinterpret_cast<floatx4*>(s + 4 * i) = *reinterpret_cast<const floatx4*>(cosines + half + 4 * i);
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      w.cos[i] = kInterleaved ? c[i / 2] : c[i];
      w.sin[i] = kInterleaved ? (i % 2 ? s[i / 2] : -s[i / 2]) : second ? s[i] : -s[i];
    }
  }
  const int n_kv = 2 * st.n_heads, n_rows = n_kv + p.n_q_heads;
  // rows: K's, V's, then the queries'; the next one is requested before this one is worked on
  struct Row {
    half8 x, y;
  };
  auto request = [&](int i, Row& r) {
    const bool q = i >= n_kv, v = !q && i >= st.n_heads;
    const RowsView& from = q ? p.q : v ? st.v : st.k;
    const int head = q ? i - n_kv : v ? i - st.n_heads : i;
    const _Float16* at_row = from.data + (int64_t)row * from.token_stride + (int64_t)head * from.head_stride + piece * 8;
    r.x = load_half8(at_row);
    if constexpr (!kInterleaved) r.y = load_half8(at_row + (turned && !v ? partner : 0));
    requests_first();
  };
  auto work = [&](int i, const Row& r) {
    const bool q = i >= n_kv, v = !q && i >= st.n_heads;
    half8 x = r.x;
    if (turned && !v) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double own = (double)(float)r.x[e], other = (double)(float)(kInterleaved ? r.x[e ^ 1] : r.y[e]);
        x[e] = rounded(__builtin_fma(own, w.cos[e], other * w.sin[e]));
      }
    }
    if (q)
      // (q itself, perhaps: the wavefront that has the row has read all of it)
      store_half8(p.q_out.data + (int64_t)row * p.q_out.token_stride + (int64_t)(i - n_kv) * p.q_out.head_stride + piece * 8, x);
    else
      write_piece<D, kFormat>(st.kv, blk, st.n_heads, i, slot, piece, x);
  };
  constexpr int kStep = 256 / PPR;
  int i = threadIdx.x / PPR;
  if (i >= n_rows) return;
  Row a, b;
  request(i, a);
  while (true) {  // (behind the last row: the last one again, and nothing is made of it)
    request(min(i + kStep, n_rows - 1), b);
    work(i, a);
    if ((i += kStep) >= n_rows) break;
    request(min(i + kStep, n_rows - 1), a);
    work(i, b);
    if ((i += kStep) >= n_rows) break;
  }
}

}  // namespace

hipError_t launch_rotate_store(const RotateParams& p, const ChunkReqs& inline_reqs, hipStream_t s) {
  if (p.store.n_rows == 0) return hipSuccess;
  const int d = p.store.head_dim;
  if ((d != 64 && d != 128) || p.rotary < 16 || p.rotary % 16 || p.rotary > d) return hipErrorInvalidValue;
  auto with = [&](const auto& reqs) {
    using Reqs = std::decay_t<decltype(reqs)>;
    with_row_format(d, p.store.e4m3, [&](auto dim, auto format) {
      constexpr int D = decltype(dim)::value, kFormat = decltype(format)::value;
      if (p.interleaved)
        rotate_store_kernel<D, kFormat, true, Reqs><<<p.store.n_rows, 256, 0, s>>>(p, reqs);
      else
        rotate_store_kernel<D, kFormat, false, Reqs><<<p.store.n_rows, 256, 0, s>>>(p, reqs);
    });
  };
  if (p.store.reqs)
    with(ChunkReqList{p.store.reqs});
  else
    with(inline_reqs);
  return hipGetLastError();
}

}  // namespace fc
