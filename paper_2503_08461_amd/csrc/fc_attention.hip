// Attention of many query rows: whole prompts (K and V as packed rows) and chunks of new
// tokens over the paged cache (fp16 or 8-bit), causal, with grouped heads.
//
// A row is one (new token, query head); the rows that read the same head of K and V lie one
// after the other, row = token * group + head of the group, and are worked on together: a
// wavefront has 32 of them, and every key that it brings in serves all 32.  Both products
// run on v_mfma_f32_32x32x16_f16 in transposed form,
//     S^T [keys x rows] = K . Q^T          O^T [channels x rows] += V^T . P^T
// with rows on the lane axis throughout: a lane has one row's logits, so its running
// maximum and sum are plain registers (the two halves of a wavefront have different keys
// of the same rows and meet by one lane swap a tile), the factor of a rescale is the lane's
// own, and the numerators leave the first product in registers in the order in which the
// second one takes them as its B operand, but for the order of the keys, which V's operand
// follows: the 4x16 transposing LDS read is given the addresses of those keys' rows.
//
// Soft-max: p = exp2(s * scale * log2 e - m), m the running maximum in those units; sums and
// products in fp32, p rounded to fp16 for the matrix cores (a relative 2^-11 each, where the
// result itself is rounded to as much).
//
// Shapes of a workgroup: four wavefronts of 32 rows each over the same keys (kRowWaves 4:
// prompts and long chunks, bound by the matrix cores), or four wavefronts over the same 32
// rows, each with a quarter of every tile's keys (kRowWaves 1: single tokens and short
// chunks, bound by memory), whose states are joined through LDS.

#include <type_traits>

#include "fc_chunk_plan.h"
#include "fc_e4m3.h"

namespace fc {

namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef __fp16 fp16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) fp16x4* LdsQuad;

constexpr int kWaveRows = 32;
constexpr float kLn2 = 0.69314718055994530942f;

template <int D, int WM, int WK, int SRC>
struct AttnShape {
  static constexpr int kThreads = 64 * WM * WK;
  static constexpr int kRows = kWaveRows * WM;
  static constexpr int kSub = WK == 1 ? 2 : 1;    // 32-key subtiles of a wavefront's share of a tile
  static constexpr int kKeys = 32 * kSub * WK;    // keys of a tile
  static constexpr int kElems = SRC == ATTN_E4M3 ? 16 : 8;  // channels of 16 bytes
  static constexpr int kLanesPerRow = D / kElems;
  static constexpr int kRowsPerPiece = kThreads / kLanesPerRow;
  static constexpr int kPieces = kKeys / kRowsPerPiece;  // 16-byte pieces a thread brings in, of K and of V
  static constexpr int kLdsBytes = 2 * kKeys * D * 2;
  static_assert(kPieces * kRowsPerPiece == kKeys, "whole tiles");
};

// Where 16-byte chunk c of key row r lies in a tile: rows of D / 8 chunks, permuted within
// the row so that the lanes of one read hit all banks.  K is read as 32 rows at one chunk,
// V by the transposing read as four (or eight) rows at four (or two) chunks.
template <int D>
__device__ __forceinline__ int k_chunk(int r, int c) {
  return r * (D / 8) + (D == 128 ? c ^ (r & 15) : c ^ ((r >> 1) & 7));
}
template <int D>
__device__ __forceinline__ int v_chunk(int r, int c) {
  const int swap = D == 128 ? ((r & 3) << 2) | (((r >> 2) & 1) << 1) : (((r >> 1) & 1) << 2) | (((r >> 2) & 1) << 1);
  return r * (D / 8) + (c ^ swap);
}

__device__ __forceinline__ float other_half_max(float v) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float other_half_sum(float v) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

template <typename Reqs>
__device__ __forceinline__ int request_of(const Reqs& reqs, int n_req, int u) {
  int lo = 0, hi = n_req - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (reqs.req[mid].unit_start <= u)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

// Nonzero where one of the eight numbers is infinite or not a number (exponent bits all set).
__device__ __forceinline__ uint32_t nonfinite(half8 x) {
  const uint4v w = __builtin_bit_cast(uint4v, x);
  uint32_t t = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) t |= (w[i] & 0x7c007c00u) + 0x04000400u;
  return t & 0x80008000u;
}
__device__ __forceinline__ half8 finite_only(half8 x) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (abs_bits(x[i]) >= 0x7c00u) x[i] = (_Float16)0.f;
  return x;
}

template <int D, int WM, int WK, int SRC, bool kSplit, typename Reqs>
__global__ __launch_bounds__(64 * WM * WK) void attention_kernel(AttnParams p, Reqs reqs) {
  using Shape = AttnShape<D, WM, WK, SRC>;
  constexpr int kKeys = Shape::kKeys, kSub = Shape::kSub, kPieces = Shape::kPieces;
  constexpr int DT = D / 32;  // 32-channel tiles of the result
  constexpr int KK = D / 16;  // slabs of the first product
  extern __shared__ __align__(16) half8 sm[];
  half8* sm_k = sm;
  half8* sm_v = sm + kKeys * D / 8;

  const int unit = blockIdx.x / p.n_heads;
  const int head = blockIdx.x - unit * p.n_heads;
  const ChunkReq rq = reqs.req[request_of(reqs, p.n_req, unit)];
  const int n_rows = rq.n_new * p.group;
  const int n_tiles = (n_rows + Shape::kRows - 1) / Shape::kRows;
  const int nb = (rq.seq_len + 15) >> 4;
  const int n_seg = kSplit ? decode_segments(nb, p.seg_blocks) : 1;
  const int at = unit - rq.unit_start;
  const int seg = kSplit ? at % n_seg : 0;
  const int tile = n_tiles - 1 - (kSplit ? at / n_seg : at);  // (the last rows see most keys: first)

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = WM == 1 ? 0 : wave % WM, wk = WK == 1 ? 0 : wave / WM;
  const int half = lane >> 5;
  const int first_key = rq.seq_len - rq.n_new;  // what token 0 sees last
  const int row0 = tile * Shape::kRows + wm * kWaveRows;
  const int row = row0 + (lane & 31);
  const bool real = row < n_rows;
  const int token = min(row, n_rows - 1) / p.group;
  const int q_head = head * p.group + min(row, n_rows - 1) - token * p.group;
  const int last_key = first_key + token;  // what this lane's row sees
  // of the workgroup, of the wavefront
  const int tile_last = first_key + (min((tile + 1) * Shape::kRows, n_rows) - 1) / p.group;
  const int wave_first = first_key + min(row0, n_rows - 1) / p.group;
  const int wave_last = first_key + min(row0 + kWaveRows - 1, n_rows - 1) / p.group;
  int key_begin = 0, key_end = tile_last + 1;
  if (kSplit) {
    key_begin = 16 * decode_segment_begin(nb, n_seg, seg);
    key_end = min(key_end, 16 * decode_segment_begin(nb, n_seg, seg + 1));
  }
  const int lane_last = min(last_key, key_end - 1);  // (a segment may end inside a tile)
  const int n_key_tiles = key_end > key_begin ? (key_end - key_begin + kKeys - 1) / kKeys : 0;

  // ---- queries: the B operand (lane: row, eight channels of a slab by half) --------------
  half8 q[KK];
  {
    const _Float16* from = p.q.data + (int64_t)(rq.row_off + token) * p.q.token_stride +
                           (int64_t)q_head * p.q.head_stride + half * 8;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) q[kk] = load_half8(from + kk * 16);
  }

  // ---- bringing in keys: a thread has one 16-byte piece of every kRowsPerPiece-th row ----
  const int in_row = threadIdx.x / Shape::kLanesPerRow;
  const int in_piece = threadIdx.x % Shape::kLanesPerRow;
  const int32_t* table = p.block_tables + (SRC == ATTN_ROWS ? 0 : (size_t)rq.table_row * p.max_blocks);
  const size_t v_off = (size_t)p.n_heads * 16 * D;
  uint4v kr[kPieces], vr[kPieces];
  uint32_t ke[SRC == ATTN_E4M3 ? kPieces : 1], ve[SRC == ATTN_E4M3 ? kPieces : 1];
  auto request = [&](int base) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int r = base + i * Shape::kRowsPerPiece + in_row;
      if constexpr (SRC == ATTN_ROWS) {
        const int64_t t = rq.row_off + min(r, rq.seq_len - 1);
        kr[i] = *reinterpret_cast<const uint4v*>(p.k.data + t * p.k.token_stride + head * p.k.head_stride + in_piece * 8);
        vr[i] = *reinterpret_cast<const uint4v*>(p.v.data + t * p.v.token_stride + head * p.v.head_stride + in_piece * 8);
      } else {
        // (behind the last block: its rows again, which no row of this call sees there)
        const int blk = clamp_block(table[min(r >> 4, nb - 1)], p.n_blocks);
        const size_t at_row = (size_t)head * 16 + (r & 15);
        if constexpr (SRC == ATTN_F16) {
          const _Float16* from = static_cast<const _Float16*>(p.kv) + (size_t)blk * 2 * v_off + at_row * D + in_piece * 8;
          kr[i] = *reinterpret_cast<const uint4v*>(from);
          vr[i] = *reinterpret_cast<const uint4v*>(from + v_off);
        } else {
          const uint8_t* block = static_cast<const uint8_t*>(p.kv) + (size_t)blk * e4m3_block_bytes(p.n_heads, D);
          const uint8_t* from = block + at_row * D + in_piece * 16;
          kr[i] = *reinterpret_cast<const uint4v*>(from);
          vr[i] = *reinterpret_cast<const uint4v*>(from + v_off);
          ke[i] = block[2 * v_off + at_row];
          ve[i] = block[2 * v_off + (size_t)p.n_heads * 16 + at_row];
        }
      }
    }
  };
  auto put = [&] {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int r = i * Shape::kRowsPerPiece + in_row;
      if constexpr (SRC == ATTN_E4M3) {
        const float ks = e4m3_scale(ke[i]), vs = e4m3_scale(ve[i]);
        sm_k[k_chunk<D>(r, 2 * in_piece)] = e4m3_values(kr[i][0], kr[i][1], ks);
        sm_k[k_chunk<D>(r, 2 * in_piece + 1)] = e4m3_values(kr[i][2], kr[i][3], ks);
        sm_v[v_chunk<D>(r, 2 * in_piece)] = e4m3_values(vr[i][0], vr[i][1], vs);
        sm_v[v_chunk<D>(r, 2 * in_piece + 1)] = e4m3_values(vr[i][2], vr[i][3], vs);
      } else {
        sm_k[k_chunk<D>(r, in_piece)] = __builtin_bit_cast(half8, kr[i]);
        sm_v[v_chunk<D>(r, in_piece)] = __builtin_bit_cast(half8, vr[i]);
      }
    }
  };

  floatx16 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
  float m = -INFINITY, z = 0.f;  // z: this lane's keys

  // ---- one tile: this wavefront's keys start at key0 -------------------------------------
  auto attend = [&](int key0, auto masked_) {
    constexpr bool kMasked = decltype(masked_)::value;
    const int sub0 = wk * kSub * 32;
    floatx16 s[kSub];
#pragma unroll
    for (int u = 0; u < kSub; ++u) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[u][r] = 0.f;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
        s[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(sm_k[k_chunk<D>(sub0 + u * 32 + (lane & 31), 2 * kk + half)], q[kk],
                                                      s[u], 0, 0, 0);
    }
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < kSub; ++u)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if constexpr (kMasked) {
          const int key = key0 + u * 32 + (r >> 2) * 8 + half * 4 + (r & 3);
          if (key > lane_last) s[u][r] = -INFINITY;
        }
        top = fmaxf(top, s[u][r]);
      }
    const float mn = fmaxf(m, other_half_max(top) * p.scale_log2e);
    if (__any(mn > m)) {
      // (nothing seen so far: nothing to rescale, but what was not a number, or infinite, stays)
      const float a = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      z *= a;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] *= a;
      m = mn;
    }
    const float base = m == -INFINITY ? 0.f : m;
    // Where some row does not see some key, 0 * inf and 0 * NaN must not reach it: channels of V
    // that are no finite numbers are added where their key is seen, and are zeros in the product.
    bool dirty = false;
    if constexpr (kMasked) {
      uint32_t found = 0;
#pragma unroll
      for (int i = 0; i < kSub * 32 * D / 8 / 64; ++i) found |= nonfinite(sm_v[sub0 * (D / 8) + i * 64 + lane]);
      dirty = __any(found != 0);
      if (dirty) {
#pragma unroll 1
        for (int key = 0; key < kSub * 32; ++key) {
          const bool seen = key0 + key <= lane_last;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int c = dt * 32 + j * 8 + half * 4;
              const half4 x = *reinterpret_cast<const half4*>(
                  reinterpret_cast<const _Float16*>(sm_v + v_chunk<D>(sub0 + key, c / 8)) + half * 4);
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (seen && abs_bits(x[e]) >= 0x7c00u) o[dt][4 * j + e] += (float)x[e];
            }
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kSub; ++u) {
      half8 pb[2];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float w = __builtin_amdgcn_exp2f(fmaf(s[u][r], p.scale_log2e, -base));
        z += w;
        pb[r >> 3][r & 7] = (_Float16)w;
      }
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        // keys 16 kk + 4 half + 0..3 and 8 more: rows (lane % 16) / 4 of the transposing reads
        const int r = sub0 + u * 32 + kk * 16 + half * 4 + ((lane & 15) >> 2);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          const int c = dt * 4 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
          const _Float16* a0 = reinterpret_cast<const _Float16*>(sm_v + v_chunk<D>(r, c)) + (lane & 1) * 4;
          const _Float16* a1 = reinterpret_cast<const _Float16*>(sm_v + v_chunk<D>(r + 8, c)) + (lane & 1) * 4;
          const fp16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4f16((LdsQuad)a0);
          const fp16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4f16((LdsQuad)a1);
          half8 v = {(_Float16)lo[0], (_Float16)lo[1], (_Float16)lo[2], (_Float16)lo[3],
                     (_Float16)hi[0], (_Float16)hi[1], (_Float16)hi[2], (_Float16)hi[3]};
          if constexpr (kMasked) {
            if (dirty) v = finite_only(v);
          }
          o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, pb[kk], o[dt], 0, 0, 0);
        }
      }
    }
  };

  if (n_key_tiles > 0) request(key_begin);
  for (int t = 0; t < n_key_tiles; ++t) {
    const int base = key_begin + t * kKeys;
    __syncthreads();  // the tile before has been read
    put();
    __syncthreads();
    if (t + 1 < n_key_tiles) request(base + kKeys);
    const int key0 = base + wk * kSub * 32;
    if (key0 > min(wave_last, key_end - 1)) continue;  // uniform over the wavefront: none of its rows sees these
    // a segment that ends inside the tile hides the keys behind it, as does the causal mask
    if (key0 + kSub * 32 - 1 <= min(wave_first, key_end - 1))
      attend(key0, std::false_type());
    else
      attend(key0, std::true_type());
  }
  z = other_half_sum(z);

  // ---- joining the wavefronts that shared the rows ----------------------------------------
  // (from here on: o normalised, m the log2 of the sum of the row's numerators, -inf: no key)
  _Float16* out = p.out.data + (int64_t)(rq.row_off + token) * p.out.token_stride + (int64_t)q_head * p.out.head_stride;
  constexpr int kWords = DecodeParams::state_words(D);
  float* state = nullptr;
  if (kSplit && n_seg > 1)
    state = p.states + (((int64_t)(rq.state_off + token) * p.n_heads * p.group + q_head) * p.n_seg + seg) * kWords;
  auto write_lse = [&](float log2_sum) {
    if (!p.lse) return;
    const int i = p.window - rq.n_new + token;
    if (i >= 0) p.lse[(int64_t)rq.table_row * p.lse_stride + (int64_t)q_head * p.window + i] = log2_sum * kLn2;
  };
  if constexpr (WK == 1) {
    const float inv = z == 0.f ? 0.f : 1.f / z;
    const float log2_sum = z == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(z);
    if (!real) return;
    if (kSplit && n_seg > 1) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          floatx4 x;
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = o[dt][4 * j + e] * inv;
          *reinterpret_cast<floatx4*>(state + dt * 32 + j * 8 + half * 4) = x;
        }
      if (half == 0) state[D] = log2_sum;
      return;
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        half4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = (_Float16)(o[dt][4 * j + e] * inv);
        *reinterpret_cast<half4*>(out + dt * 32 + j * 8 + half * 4) = x;
      }
    if (half == 0) write_lse(log2_sum);
  } else {
    static_assert(WM == 1, "wavefronts with rows of their own or with shared rows");
    float* sm_f = reinterpret_cast<float*>(sm);
    __syncthreads();
    if (half == 0) {
      sm_f[(wk * 32 + lane) * 2] = m;
      sm_f[(wk * 32 + lane) * 2 + 1] = z;
    }
    __syncthreads();
    float mm = -INFINITY, zz = 0.f;
#pragma unroll
    for (int w = 0; w < WK; ++w) mm = fmaxf(mm, sm_f[(w * 32 + (lane & 31)) * 2]);
#pragma unroll
    for (int w = 0; w < WK; ++w) {
      const float zw = sm_f[(w * 32 + (lane & 31)) * 2 + 1];
      zz += zw == 0.f ? 0.f : zw * __builtin_amdgcn_exp2f(sm_f[(w * 32 + (lane & 31)) * 2] - mm);
    }
    const float log2_sum = zz == 0.f ? -INFINITY : mm + __builtin_amdgcn_logf(zz);
    const float f = z == 0.f ? 0.f : __builtin_amdgcn_exp2f(m - mm) / zz;
    __syncthreads();
    // [wavefront][row][channel], quads permuted within the row against bank conflicts
    constexpr int kQuads = D / 4;
    floatx4* sm_o = reinterpret_cast<floatx4*>(sm);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        floatx4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = o[dt][4 * j + e] * f;
        const int c = dt * 8 + j * 2 + half, r = lane & 31;
        sm_o[(wk * 32 + r) * kQuads + (c ^ (r & (kQuads - 1)))] = x;
      }
    if (wave == 0 && half == 0 && real) {
      if (kSplit && n_seg > 1)
        state[D] = log2_sum;
      else
        write_lse(log2_sum);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 32 * kQuads; i += Shape::kThreads) {
      const int r = i / kQuads, c = i % kQuads;
      if (tile * Shape::kRows + r >= n_rows) break;
      floatx4 x = sm_o[r * kQuads + (c ^ (r & (kQuads - 1)))];
#pragma unroll
      for (int w = 1; w < WK; ++w) x += sm_o[(w * 32 + r) * kQuads + (c ^ (r & (kQuads - 1)))];
      const int tok = (tile * Shape::kRows + r) / p.group;
      const int h = head * p.group + (tile * Shape::kRows + r) - tok * p.group;
      if (kSplit && n_seg > 1) {
        float* to = p.states + (((int64_t)(rq.state_off + tok) * p.n_heads * p.group + h) * p.n_seg + seg) * kWords;
        *reinterpret_cast<floatx4*>(to + c * 4) = x;
      } else {
        half4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = (_Float16)x[e];
        *reinterpret_cast<half4*>(p.out.data + (int64_t)(rq.row_off + tok) * p.out.token_stride +
                                  (int64_t)h * p.out.head_stride + c * 4) = y;
      }
    }
  }
}

// Rows whose keys were split: the result from the segments' states.  Workgroup = (token of
// the launch, query head), one thread per channel.
template <int D, typename Reqs>
__global__ __launch_bounds__(D) void attention_merge_kernel(AttnParams p, Reqs reqs) {
  const int n_q = p.n_heads * p.group;
  const int t = blockIdx.x / n_q;
  const int h = blockIdx.x - t * n_q;
  int lo = 0, hi = p.n_req - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (reqs.req[mid].state_off <= t)
      lo = mid;
    else
      hi = mid - 1;
  }
  const ChunkReq rq = reqs.req[lo];
  const int n_seg = decode_segments((rq.seq_len + 15) >> 4, p.seg_blocks);
  if (n_seg <= 1) return;  // written by the kernel above
  constexpr int kWords = DecodeParams::state_words(D);
  const float* states = p.states + (int64_t)blockIdx.x * p.n_seg * kWords;
  float mm = -INFINITY, zz = 0.f, o = 0.f;
  for (int i = 0; i < n_seg; ++i) mm = fmaxf(mm, states[(size_t)i * kWords + D]);
#pragma unroll 4
  for (int i = 0; i < n_seg; ++i) {
    const float mi = states[(size_t)i * kWords + D];
    const float f = mi == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mi - mm);
    zz += f;
    o += states[(size_t)i * kWords + threadIdx.x] * f;
  }
  const int token = t - rq.state_off;
  p.out.data[(int64_t)(rq.row_off + token) * p.out.token_stride + (int64_t)h * p.out.head_stride + threadIdx.x] =
      (_Float16)(zz == 0.f ? 0.f : o / zz);
  const int i = p.window - rq.n_new + token;
  if (p.lse && i >= 0 && threadIdx.x == 0)
    p.lse[(int64_t)rq.table_row * p.lse_stride + (int64_t)h * p.window + i] =
        zz == 0.f ? -INFINITY : (mm + __builtin_amdgcn_logf(zz)) * kLn2;
}

template <int D, int WM, int WK, int SRC, typename Reqs>
void launch_one(const AttnParams& p, const Reqs& reqs, hipStream_t s) {
  using Shape = AttnShape<D, WM, WK, SRC>;
  const unsigned grid = (unsigned)p.n_units * p.n_heads;
  if constexpr (SRC != ATTN_ROWS) {
    if (p.n_seg > 1) {
      attention_kernel<D, WM, WK, SRC, true, Reqs><<<grid, Shape::kThreads, Shape::kLdsBytes, s>>>(p, reqs);
      attention_merge_kernel<D, Reqs><<<(unsigned)p.state_rows * p.n_heads * p.group, D, 0, s>>>(p, reqs);
      return;
    }
  }
  attention_kernel<D, WM, WK, SRC, false, Reqs><<<grid, Shape::kThreads, Shape::kLdsBytes, s>>>(p, reqs);
}

template <int D, typename Reqs>
void launch_shape(const AttnParams& p, bool flat, const Reqs& reqs, hipStream_t s) {
  if (p.source == ATTN_ROWS)
    flat ? launch_one<D, 1, 4, ATTN_ROWS>(p, reqs, s) : launch_one<D, 4, 1, ATTN_ROWS>(p, reqs, s);
  else if (p.source == ATTN_F16)
    flat ? launch_one<D, 1, 4, ATTN_F16>(p, reqs, s) : launch_one<D, 4, 1, ATTN_F16>(p, reqs, s);
  else
    flat ? launch_one<D, 1, 4, ATTN_E4M3>(p, reqs, s) : launch_one<D, 4, 1, ATTN_E4M3>(p, reqs, s);
}

}  // namespace

hipError_t launch_attention(const AttnParams& p, bool flat, const ChunkReqs& inline_reqs, hipStream_t s) {
  if (p.n_units == 0) return hipSuccess;
  if ((p.head_dim != 64 && p.head_dim != 128) || p.n_seg < 1 || p.seg_blocks < 1 || (p.source == ATTN_ROWS && p.n_seg > 1))
    return hipErrorInvalidValue;
  auto with = [&](const auto& reqs) {
    if (p.head_dim == 128)
      launch_shape<128>(p, flat, reqs, s);
    else
      launch_shape<64>(p, flat, reqs, s);
  };
  if (p.reqs)
    with(ChunkReqList{p.reqs});
  else
    with(inline_reqs);
  return hipGetLastError();
}

}  // namespace fc
