// Attention of many query rows: whole prompts (K and V as packed rows) and chunks of new
// tokens over the paged cache (fp16, 8-bit or 4-bit), causal, with grouped heads.
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
// Two parts of one launch: many rows (prompts, long chunks; bound by the matrix cores) and few
// rows of a head and request, up to 32 (single tokens, short chunks; bound by memory).  (Two launches:
// a mixed batch of 24 chunks of 1-512 tokens 269 us, one 240, now 230; the few rows' workgroups fill what the
// many rows' leave.)

#include <algorithm>
#include <type_traits>

#include "fc_chunk_plan.h"
#include "fc_e2m1.h"
#include "fc_select_blocks.h"

namespace fc {

namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef __fp16 fp16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) fp16x4* LdsQuad;
typedef int int2v __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) int2v* LdsPair;

constexpr float kSlack = 8.f;
constexpr float kLn2 = 0.69314718055994530942f;

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

// A result as fp16.  The numerators' rounding, up to 2^-11 of each, can carry a mean of values at the
// end of fp16's range past it; infinite is only what was infinite before.
__device__ __forceinline__ float f16_result(float x) {
  const float within = fminf(fmaxf(x, -65504.f), 65504.f);
  return fabsf(x) < INFINITY ? within : x;
}

// The largest magnitudes of two interleaved series of numbers, as bits: infinite or not a
// number from 0x7c00 on.
typedef uint16_t ushort2v __attribute__((ext_vector_type(2)));
__device__ __forceinline__ ushort2v largest(half8 x, ushort2v so_far) {
  const uint4v w = __builtin_bit_cast(uint4v, x);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    so_far = __builtin_elementwise_max(so_far, __builtin_bit_cast(ushort2v, w[i] & 0x7fff7fffu));
  return so_far;
}
__device__ __forceinline__ half8 finite_only(half8 x) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (abs_bits(x[i]) >= 0x7c00u) x[i] = (_Float16)0.f;
  return x;
}

// Loads from memory straight to LDS: lane l's 16 bytes go to to[l].
typedef __amdgpu_buffer_rsrc_t BufferPtr;
__device__ __forceinline__ BufferPtr buffer_of(const void* base, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, bytes, 0x00020000);
}
// kOnce: the line is the first to leave the caches: no other workgroup reads it, but for the tokens of one request that
// select their blocks each for itself (what these share comes from memory again where it has left).
template <bool kOnce>
__device__ __forceinline__ void load_to_lds(BufferPtr from, int lane_offset, half8* to) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, lane_offset, 0, 0,
                                           kOnce ? 2 : 0);
}
__device__ __forceinline__ void load_word_to_lds(BufferPtr from, int lane_offset, void* to) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 4, lane_offset, 0, 0, 0);
}
// V's operand: lane l gets, of the four rows that the sixteen lanes around it point to (four
// lanes a row, 8 bytes each), channel l % 16.  (restrict: without it the compiler waits for
// every load to LDS that is on its way; the waits that are needed are written out.)
__device__ __forceinline__ fp16x4 read_columns(const _Float16* __restrict at) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4f16((LdsQuad)at);
}
// Waits until at most N of the wavefront's vector memory accesses are on their way.
template <int N>
__device__ __forceinline__ void wait_loads() {
  static_assert(N < 64, "six bits");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
  asm volatile("" ::: "memory");
}
// A barrier that leaves vector memory accesses on their way.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// 32-key subtiles of fp16 rows in LDS, from row `at` of tiles k and v.
template <int D>
struct F16Keys {
  static constexpr int kSlabs = 1;  // of K that a lane reads at a time (take_queries)
  const half8 *k, *v;
  int at;
  // A operands: of a slab of K (lane: key, eight channels by half), ...
  __device__ __forceinline__ half8 k_slab(int u, int kk) const {
    const int lane = threadIdx.x & 63;
    return k[k_chunk<D>(at + u * 32 + (lane & 31), 2 * kk + (lane >> 5))];
  }
  // ... and of V^T: keys 16 kk + 4 half + 0..3 and 8 more, rows (lane % 16) / 4 of the transposing reads
  __device__ __forceinline__ half8 v_slab(int u, int kk, int dt) const {
    const int lane = threadIdx.x & 63;
    const int r = at + u * 32 + kk * 16 + (lane >> 5) * 4 + ((lane & 15) >> 2);
    const int c = dt * 4 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
    const fp16x4 lo = read_columns(reinterpret_cast<const _Float16*>(v + v_chunk<D>(r, c)) + (lane & 1) * 4);
    const fp16x4 hi = read_columns(reinterpret_cast<const _Float16*>(v + v_chunk<D>(r + 8, c)) + (lane & 1) * 4);
    return half8{(_Float16)lo[0], (_Float16)lo[1], (_Float16)lo[2], (_Float16)lo[3],
                 (_Float16)hi[0], (_Float16)hi[1], (_Float16)hi[2], (_Float16)hi[3]};
  }
  // whether V holds anything but finite numbers
  template <int kSub>
  __device__ __forceinline__ bool dirty() const {
    ushort2v most = {0, 0};
#pragma unroll
    for (int i = 0; i < kSub * 32 * D / 8 / 64; ++i) most = largest(v[at * (D / 8) + i * 64 + (threadIdx.x & 63)], most);
    return __any(max(most[0], most[1]) >= 0x7c00);
  }
  // four channels of one key, those that are no finite numbers (0 for the others)
  __device__ __forceinline__ floatx4 not_finite(int key, int channel) const {
    const half4 x = *reinterpret_cast<const half4*>(
        reinterpret_cast<const _Float16*>(v + v_chunk<D>(at + key, channel / 8)) + channel % 8);
    floatx4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = abs_bits(x[e]) >= 0x7c00u ? (float)x[e] : 0.f;
    return y;
  }
};

// The 32 rows of a wavefront: operands, result and soft-max state of each lane's row.
template <int D>
struct Rows32 {
  static constexpr int DT = D / 32;  // 32-channel tiles of the result
  static constexpr int KK = D / 16;  // slabs of the first product
  half8 q[KK];                       // B operand (eight channels of a slab by half)
  floatx16 o[DT];
  float m, z;  // running maximum (log2 units), and sum of this lane's keys

  __device__ __forceinline__ void start() {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
    m = -INFINITY;
    z = 0.f;
  }
  // The queries, through `room` in LDS (32 rows of the wavefront's own): read from memory and
  // written there row by row, D / 8 lanes a row.  (A lane's own row straight from memory is 64
  // addresses in 64 lines for each of its loads, which took four wavefronts 2000 cycles of a
  // workgroup's 40000 for a prompt of 1024.)  from(row): where the wavefront's row is.
  template <typename From>
  __device__ __forceinline__ void request_queries(From from) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < KK; ++i) q[i] = load_half8(from((i * 64 + lane) / (D / 8)) + (lane % (D / 8)) * 8);
  }
  // (kSlabs: slabs of K that a lane reads next to each other; the queries' channels follow)
  template <int kSlabs>
  __device__ __forceinline__ void take_queries(half8* room) {
    const int lane = threadIdx.x & 63, half = lane >> 5;
#pragma unroll
    for (int i = 0; i < KK; ++i) room[k_chunk<D>((i * 64 + lane) / (D / 8), lane % (D / 8))] = q[i];
    wave_lds_barrier();
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
      q[kk] = room[k_chunk<D>(lane & 31, kSlabs * (2 * (kk / kSlabs) + half) + kk % kSlabs)];
    wave_lds_barrier();
  }
  // The lane's row times f, as fp16 rows in LDS (32 of the wavefront's own), then row by row to
  // memory.  to(row): where the wavefront's row goes, NULL if nowhere.
  template <typename To>
  __device__ __forceinline__ void write_result(half8* room, float f, To to) {
    const int lane = threadIdx.x & 63, half = lane >> 5;
    // (looked for first: on every number f16_result costs one prompt of 640 tokens 2 %)
    float top = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, fabsf(o[dt][r]));
    if (__any(top * f > 65504.f)) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] = f16_result(o[dt][r] * f);
      f = 1.f;
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        half4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = (_Float16)(o[dt][4 * j + e] * f);
        reinterpret_cast<half4*>(room + k_chunk<D>(lane & 31, dt * 4 + j))[half] = x;
      }
    wave_lds_barrier();
    half8 x[KK];
#pragma unroll
    for (int i = 0; i < KK; ++i) x[i] = room[k_chunk<D>((i * 64 + lane) / (D / 8), lane % (D / 8))];
#pragma unroll
    for (int i = 0; i < KK; ++i) {
      _Float16* row = to((i * 64 + lane) / (D / 8));
      if (row) store_half8(row + (lane % (D / 8)) * 8, x[i]);
    }
  }

  // m follows the maximum when it falls more than kSlack behind: the numerators stay below
  // 2^kSlack, which fp16 and the sums hold as exactly as those below 1.  top: of this lane's
  // logits; returns what numerators are taken relative to.
  __device__ __forceinline__ float follow(float top, float scale_log2e) {
    const float mn = fmaxf(m, other_half_max(top) * scale_log2e);
    if (__any(mn > m + kSlack)) {
      // (nothing seen so far: nothing to rescale, but what was not a number, or infinite, stays)
      const float a = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      z *= a;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] *= a;
      m = mn;
    }
    return m == -INFINITY ? 0.f : m;
  }

  // 64 keys that every row sees, in the tile at `lds`: attend() with its instructions in this
  // order.  Operands are read four products ahead, and the numerators of the next 16 keys are
  // made between the products of these.  (Left to itself the compiler reads an operand, waits
  // for it and multiplies, or does not, as what stands around the loop changes.)
  struct Offsets {  // of the lane's operands in a tile, in bytes
    int k[KK], v[DT];
  };
  __device__ __forceinline__ static Offsets offsets() {
    const int lane = threadIdx.x & 63, half = lane >> 5;
    Offsets at;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) at.k[kk] = k_chunk<D>(lane & 31, 2 * kk + half) * 16;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      at.v[dt] = v_chunk<D>(half * 4 + ((lane & 15) >> 2), dt * 4 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) * 16 +
                 (lane & 1) * 8 + 64 * D * 2;
    return at;
  }
  template <int kTileAt>
  __device__ __forceinline__ void attend_full(const half8* sm, const Offsets& at, float scale_log2e) {
    constexpr int kAhead = 4, kRow = D * 2;
    const char* lds = reinterpret_cast<const char*>(sm) + kTileAt;
    auto k_read = [&](int i) {
      return *reinterpret_cast<const half8*>(lds + at.k[i % KK] + (i / KK) * 32 * kRow);
    };
    auto v_read = [&](int i) {  // product i: 16 keys i / DT, channels 32 (i % DT) and on
      const _Float16* from = reinterpret_cast<const _Float16*>(lds + at.v[i % DT] + (i / DT) * 16 * kRow);
      const fp16x4 lo = read_columns(from), hi = read_columns(from + 8 * D);
      return half8{(_Float16)lo[0], (_Float16)lo[1], (_Float16)lo[2], (_Float16)lo[3],
                   (_Float16)hi[0], (_Float16)hi[1], (_Float16)hi[2], (_Float16)hi[3]};
    };
    half8 a[kAhead + 1];
    floatx16 s[2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[u][r] = 0.f;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) a[i] = k_read(i);
    __builtin_amdgcn_sched_barrier(0);
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 2 * KK; ++i) {
      if (i + kAhead < 2 * KK) a[(i + kAhead) % (kAhead + 1)] = k_read(i + kAhead);
      s[i / KK] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[i % (kAhead + 1)], q[i % KK], s[i / KK], 0, 0, 0);
      if (i >= 2 * KK - 2) {  // (the first half is there by now)
#pragma unroll
        for (int r = 0; r < 8; ++r) top = fmaxf(top, s[0][(i - (2 * KK - 2)) * 8 + r]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) a[i] = v_read(i);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int r = 0; r < 16; ++r) top = fmaxf(top, s[1][r]);
    const float base = follow(top, scale_log2e);
    half8 p[2];
    auto numerator = [&](int i) {  // of the lane's key i of 32
      const float w = __builtin_amdgcn_exp2f(fmaf(s[i / 16][i % 16], scale_log2e, -base));
      z += w;
      p[(i / 8) % 2][i % 8] = (_Float16)w;
    };
#pragma unroll
    for (int i = 0; i < 8; ++i) numerator(i);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 4 * DT; ++i) {
      if (i + kAhead < 4 * DT) a[(i + kAhead) % (kAhead + 1)] = v_read(i + kAhead);
      o[i % DT] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[i % (kAhead + 1)], p[(i / DT) % 2], o[i % DT], 0, 0, 0);
      if (i < 3 * DT) {
#pragma unroll
        for (int j = 0; j < 8 / DT; ++j) numerator(8 * (i / DT + 1) + (i % DT) * (8 / DT) + j);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // kSub * 32 keys, key0: the first one's number.  kMasked: the lane's row sees keys up to
  // last_key only.  after_k: K has been read; before_v: V is needed.
  template <int kSub, bool kMasked, typename Keys, typename AfterK, typename BeforeV>
  __device__ __forceinline__ void attend(const Keys& keys, int key0, int last_key, float scale_log2e, AfterK after_k,
                                         BeforeV before_v) {
    const int half = (threadIdx.x & 63) >> 5;
    floatx16 s[kSub];
#pragma unroll
    for (int u = 0; u < kSub; ++u)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[u][r] = 0.f;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int u = 0; u < kSub; ++u)
        s[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(keys.k_slab(u, kk), q[kk], s[u], 0, 0, 0);
    after_k();
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < kSub; ++u)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if constexpr (kMasked) {
          const int key = key0 + u * 32 + (r >> 2) * 8 + half * 4 + (r & 3);
          if (key > last_key) s[u][r] = -INFINITY;
        }
        top = fmaxf(top, s[u][r]);
      }
    const float base = follow(top, scale_log2e);
    before_v();
    // Where some row does not see some key, 0 * inf and 0 * NaN must not reach it: channels of V
    // that are no finite numbers are added where their key is seen, and are zeros in the product.
    bool dirty = false;
    if constexpr (kMasked) {
      dirty = __any(key0 + kSub * 32 - 1 > last_key) && keys.template dirty<kSub>();
      if (dirty) {
#pragma unroll 1
        for (int key = 0; key < kSub * 32; ++key) {
          const bool seen = key0 + key <= last_key;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const floatx4 x = keys.not_finite(key, dt * 32 + j * 8 + half * 4);
#pragma unroll
              for (int e = 0; e < 4; ++e) o[dt][4 * j + e] += seen ? x[e] : 0.f;
            }
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kSub; ++u) {
      half8 pb[2];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float w = __builtin_amdgcn_exp2f(fmaf(s[u][r], scale_log2e, -base));
        z += w;
        pb[r >> 3][r & 7] = (_Float16)w;
      }
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          half8 v = keys.v_slab(u, kk, dt);
          if constexpr (kMasked) {
            if (dirty) v = finite_only(v);
          }
          o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, pb[kk], o[dt], 0, 0, 0);
        }
    }
  }
};

// row / group, by the inverse 2^31 / group, rounded up (exact for rows below 2^25)
__device__ __forceinline__ int token_of(const AttnParams& p, int row) {
  return (int)__umulhi((uint32_t)row << 1, p.group_inverse);
}

// Where a workgroup is in its request (tile: row tile of kRows) and which keys it walks.
struct Place {
  ChunkReq rq;
  int n_rows, tile, nb, n_seg, seg, key_begin, key_end;
};
template <int kRows, bool kSplit, typename Reqs>
__device__ __forceinline__ Place place_of(const AttnParams& p, const Reqs& reqs, const AttnLaunchView& l, int unit) {
  Place w;
  w.rq = reqs.req[request_of(l.first_req, l.n_req, unit, [&](int i) { return reqs.req[i].unit_start; })];
  w.n_rows = w.rq.n_new * p.group;
  w.nb = (w.rq.seq_len + 15) >> 4;
  w.n_seg = kSplit ? decode_segments(w.nb, l.seg_blocks) : 1;
  const int at = unit - w.rq.unit_start;
  w.seg = kSplit ? at % w.n_seg : 0;
  // (the last rows see most keys: first)
  w.tile = (w.n_rows + kRows - 1) / kRows - 1 - (kSplit ? at / w.n_seg : at);
  w.key_begin = 0;
  w.key_end = w.rq.seq_len - w.rq.n_new + token_of(p, min((w.tile + 1) * kRows, w.n_rows) - 1) + 1;
  if (kSplit) {
    w.key_begin = 16 * decode_segment_begin(w.nb, w.n_seg, w.seg);
    w.key_end = min(w.key_end, 16 * decode_segment_begin(w.nb, w.n_seg, w.seg + 1));
  }
  return w;
}

// A lane's row: its token and query head (rows behind the last one: the last one's).
struct LaneRow {
  int token, in_group;
  bool real;
};
__device__ __forceinline__ LaneRow lane_row(const AttnParams& p, int row, int n_rows) {
  LaneRow r;
  r.real = row < n_rows;
  row = min(row, n_rows - 1);
  r.token = token_of(p, row);
  r.in_group = row - r.token * p.group;
  return r;
}
__device__ __forceinline__ _Float16* row_of(const RowsView& v, const ChunkReq& rq, int token, int head) {
  return v.data + (int64_t)(rq.row_off + token) * v.token_stride + (int64_t)head * v.head_stride;
}
// Rows of a request and of the query heads that share one head of K and V: two products of 32
// bits a row (the strides are limited to that).
struct GroupRows {
  _Float16* base;
  uint32_t token_stride, head_stride;
  __device__ __forceinline__ GroupRows(const RowsView& v, const ChunkReq& rq, const AttnParams& p, int head)
      : base(row_of(v, rq, 0, head * p.group)), token_stride((uint32_t)v.token_stride), head_stride((uint32_t)v.head_stride) {}
  __device__ __forceinline__ _Float16* at(const LaneRow& r) const {
    return base + ((uint64_t)(uint32_t)r.token * token_stride + (uint64_t)(uint32_t)r.in_group * head_stride);
  }
};
template <int D>
__device__ __forceinline__ float* state_of(const AttnParams& p, const AttnLaunchView& l, const ChunkReq& rq, int token,
                                           int q_head, int seg) {
  return l.states + (((int64_t)(rq.state_off + token) * p.n_heads * p.group + q_head) * l.n_seg + seg) *
                        DecodeParams::state_words(D);
}
__device__ __forceinline__ void write_lse(const AttnParams& p, const ChunkReq& rq, int token, int q_head, float log2_sum) {
  const int i = p.window - rq.n_new + token;
  if (p.lse && i >= 0) p.lse[(int64_t)rq.table_row * p.lse_stride + (int64_t)q_head * p.window + i] = log2_sum * kLn2;
}

// Sixteen keys (a pool block) on their way to LDS by one wavefront, K and V in one call each.
// The rows lie in LDS from slot 0 of `to`, which is a multiple of 16 rows into a tile; the
// permutation of the chunks is in the addresses that the lanes read from.
template <int D, bool kOnce>
struct BlockLoader {
  static constexpr int kInstr = 16 * D / 8 / 64;  // wavefront loads of K, and of V
  int k_at[kInstr], v_at[kInstr];                 // byte offset of the lane's chunk, by load
  __device__ __forceinline__ BlockLoader(int k_row_bytes, int v_row_bytes) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < kInstr; ++i) {
      const int r = (i * 64 + lane) / (D / 8), c = lane % (D / 8);
      k_at[i] = r * k_row_bytes + (k_chunk<D>(r, c) - r * (D / 8)) * 16;
      v_at[i] = r * v_row_bytes + (v_chunk<D>(r, c) - r * (D / 8)) * 16;
    }
  }
  __device__ __forceinline__ void k(BufferPtr from, half8* to) const {
#pragma unroll
    for (int i = 0; i < kInstr; ++i) load_to_lds<kOnce>(from, k_at[i], to + i * 64);
  }
  __device__ __forceinline__ void v(BufferPtr from, half8* to) const {
#pragma unroll
    for (int i = 0; i < kInstr; ++i) load_to_lds<kOnce>(from, v_at[i], to + i * 64);
  }
};

// Sixteen keys of an 8-bit pool through registers: codes, exponents; fp16 numbers into LDS.
template <int D>
struct Block8 {
  static constexpr int kLanes = D / 16, kInstr = 16 * kLanes / 64;  // lanes of a row; loads of K, and of V
  uint4v kc[kInstr], vc[kInstr];
  uint32_t ke[kInstr], ve[kInstr];
  __device__ __forceinline__ void request(const uint8_t* block, int n_heads, int head) {
    const int lane = threadIdx.x & 63;
    const size_t v_off = (size_t)n_heads * 16 * D;
#pragma unroll
    for (int i = 0; i < kInstr; ++i) {
      const size_t row = (size_t)head * 16 + (i * 64 + lane) / kLanes;
      const uint8_t* from = block + row * D + (lane % kLanes) * 16;
      kc[i] = *reinterpret_cast<const uint4v*>(from);
      vc[i] = *reinterpret_cast<const uint4v*>(from + v_off);
      ke[i] = block[2 * v_off + row];
      ve[i] = block[2 * v_off + (size_t)n_heads * 16 + row];
    }
  }
  __device__ __forceinline__ void put(half8* sm_k, half8* sm_v, int at) const {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < kInstr; ++i) {
      const int r = at + (i * 64 + lane) / kLanes, c = (lane % kLanes) * 2;
      const float ks = e4m3_scale(ke[i]), vs = e4m3_scale(ve[i]);
      sm_k[k_chunk<D>(r, c)] = e4m3_values(kc[i][0], kc[i][1], ks);
      sm_k[k_chunk<D>(r, c + 1)] = e4m3_values(kc[i][2], kc[i][3], ks);
      sm_v[v_chunk<D>(r, c)] = e4m3_values(vc[i][0], vc[i][1], vs);
      sm_v[v_chunk<D>(r, c + 1)] = e4m3_values(vc[i][2], vc[i][3], vs);
    }
  }
};

// Sixteen keys of a 4-bit pool through registers.  A lane has 16 bytes, a group of 32 channels of one
// row; at 64 channels K's rows are with the first half of the wavefront and V's with the other.
template <int D>
struct Block4 {
  static constexpr int kLanes = D / kE2m1Group;  // lanes of a row
  static constexpr bool kBoth = D == 128;        // every lane has a part of K and one of V
  uint4v c[kBoth ? 2 : 1];
  uint32_t e[kBoth ? 2 : 1];
  __device__ __forceinline__ void request(const uint8_t* block, int n_heads, int head) {
    const int lane = threadIdx.x & 63;
    const size_t codes = (size_t)n_heads * 8 * D, exps = (size_t)n_heads * D / 2;  // of K, and of V
    const int at = kBoth ? lane : lane & 31;  // = row * kLanes + group
    const size_t v = kBoth ? 0 : lane >> 5;
    const uint8_t* c_from = block + v * codes + (size_t)head * 8 * D + at * 16;
    const uint8_t* e_from = block + 2 * codes + v * exps + (size_t)head * D / 2 + at;
#pragma unroll
    for (int i = 0; i < (kBoth ? 2 : 1); ++i) {
      c[i] = __builtin_nontemporal_load(reinterpret_cast<const uint4v*>(c_from + i * codes));
      e[i] = e_from[i * exps];
    }
  }
  __device__ __forceinline__ void put(half8* sm_k, half8* sm_v, int at) const {
    const int lane = threadIdx.x & 63;
    const int r = at + (kBoth ? lane : lane & 31) / kLanes, first = lane % kLanes * 4;
#pragma unroll
    for (int i = 0; i < (kBoth ? 2 : 1); ++i) {
      const float scale = e4m3_scale(e[i]);
      const bool is_v = kBoth ? i == 1 : lane >= 32;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        half8* to = is_v ? sm_v + v_chunk<D>(r, first + w) : sm_k + k_chunk<D>(r, first + w);
        *to = e2m1_values(c[i][w], scale);
      }
    }
  }
};

// The same as codes for a wavefront that works on them alone: they go straight to LDS and
// become fp16 numbers as they are read.  Rows of D bytes, 16-byte chunks permuted for K's
// reads (32 rows at one chunk) and V's transposing ones (eight rows, of two blocks of
// channels).
template <int D>
__device__ __forceinline__ int k8_chunk(int r, int c) {
  return r * (D / 16) + (D == 128 ? c ^ ((r >> 1) & 7) : c ^ ((r >> 2) & 3));
}
template <int D>
__device__ __forceinline__ int v8_chunk(int r, int c) {
  const int swap = D == 128 ? (((r >> 1) & 1) << 1) | (((r >> 3) & 1) << 2) : ((r >> 3) & 1) << 1;
  return r * (D / 16) + (c ^ swap);
}
template <int D>
struct Loader8 {
  static constexpr int kInstr = D / 64;  // wavefront loads of 16 rows of K, and of V
  int k_at[kInstr], v_at[kInstr];
  __device__ __forceinline__ Loader8() {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < kInstr; ++i) {
      const int r = (i * 64 + lane) / (D / 16), c = lane % (D / 16);
      k_at[i] = k8_chunk<D>(r, c) * 16;
      v_at[i] = v8_chunk<D>(r, c) * 16;
    }
  }
  __device__ __forceinline__ void k(BufferPtr from, half8* to) const {
#pragma unroll
    for (int i = 0; i < kInstr; ++i) load_to_lds<true>(from, k_at[i], to + i * 64);
  }
  __device__ __forceinline__ void v(BufferPtr from, half8* to) const {
#pragma unroll
    for (int i = 0; i < kInstr; ++i) load_to_lds<true>(from, v_at[i], to + i * 64);
  }
};
// (lane l: of the eight rows that the sixteen lanes around it point to, two lanes a row, byte l % 16)
__device__ __forceinline__ int2v read_byte_columns(const uint8_t* __restrict at) {
  return __builtin_amdgcn_ds_read_tr8_b64_v2i32((LdsPair)at);
}
constexpr int kExponentBytes = 256;  // of a block, in LDS (what one load of a word a lane fills)
template <int D>
struct E4m3Keys {
  static constexpr int kSlabs = 2;  // a 16-byte read of K is its lane's part of two slabs
  const uint8_t *k, *v;
  float k_scale;         // of the lane's key
  half2v v_scale[2][4];  // of the lane's eight keys of a slab of V
  __device__ __forceinline__ half8 k_slab(int, int kk) const {
    const int lane = threadIdx.x & 63;
    const uint4v c = *reinterpret_cast<const uint4v*>(k + k8_chunk<D>(lane & 31, 2 * (kk / 2) + (lane >> 5)) * 16);
    return e4m3_values(c[2 * (kk % 2)], c[2 * (kk % 2) + 1], k_scale);
  }
  // From the exponents in LDS, 16 of K and 16 of V for each of the two blocks.  Keys behind
  // `last` are seen by no row (and their slots may hold anything): times zero.
  __device__ __forceinline__ void set_k(const uint8_t* exponents) {
    const int lane = threadIdx.x & 63;
    k_scale = e4m3_scale(exponents[((lane & 31) >> 4) * kExponentBytes + (lane & 15)]);
  }
  template <bool kMasked>
  __device__ __forceinline__ void set_v(const uint8_t* exponents, int last) {
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const uint32_t e = *reinterpret_cast<const uint32_t*>(exponents + kk * kExponentBytes + 16 + 8 * w + 4 * half);
        float f[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          f[j] = e4m3_scale((e >> (8 * j)) & 255u);
          if (kMasked && 16 * kk + 8 * w + 4 * half + j > last) f[j] = 0.f;
        }
        v_scale[kk][2 * w] = half2v{(_Float16)f[0], (_Float16)f[1]};
        v_scale[kk][2 * w + 1] = half2v{(_Float16)f[2], (_Float16)f[3]};
      }
  }
  __device__ __forceinline__ half8 v_slab(int, int kk, int dt) const {
    const int lane = threadIdx.x & 63;
    // row (lane % 16) / 2 of the read: keys 4 half + 0..3, then 8 more
    const int i = (lane & 15) >> 1;
    const int r = kk * 16 + (lane >> 5) * 4 + (i & 3) + (i & 4) * 2;
    const int c = dt * 2 + ((lane >> 4) & 1);
    const int2v x = read_byte_columns(v + v8_chunk<D>(r, c) * 16 + (lane & 1) * 8);
    half8 y;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const half2v a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x[w], 1.f, false) * v_scale[kk][2 * w];
      const half2v b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x[w], 1.f, true) * v_scale[kk][2 * w + 1];
      y[4 * w] = a[0];
      y[4 * w + 1] = a[1];
      y[4 * w + 2] = b[0];
      y[4 * w + 3] = b[1];
    }
    return y;
  }
  template <int kSub>
  __device__ __forceinline__ bool dirty() const {
    uint32_t found = 0;
#pragma unroll
    for (int i = 0; i < 32 * D / 16 / 64; ++i) {
      const uint4v x = reinterpret_cast<const uint4v*>(v)[i * 64 + (threadIdx.x & 63)];
#pragma unroll
      for (int w = 0; w < 4; ++w) found |= (x[w] & 0x7f7f7f7fu) + 0x01010101u;
    }
    return __any((found & 0x80808080u) != 0);
  }
  __device__ __forceinline__ floatx4 not_finite(int key, int channel) const {
    const uint32_t x = *reinterpret_cast<const uint32_t*>(v + v8_chunk<D>(key, channel / 16) * 16 + channel % 16);
    floatx4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = ((x >> (8 * e)) & 0x7fu) == 0x7fu ? __builtin_nanf("") : 0.f;
    return y;
  }
};

// 4 bits: codes straight to LDS as well, fp16 numbers as they are read.  A block there: 16 rows of K, 16
// of V, D / 2 bytes each, 16-byte chunks (a group of 32 channels) permuted within the row for K's reads
// (32 rows at one chunk) and V's transposing ones (rows 0-3, 8-11 and so on of a tile, 8 bytes each).
// Through registers, with fp16 rows written to LDS and read from there, the LDS is busy for 1280 of the 1600
// cycles that a SIMD has for a tile at the memory's rate, so for 500.
// (kFew: for Keys16 below, whose transposing reads take rows 0-7 and 16-23, or the others, at a time)
template <int D, bool kFew>
__device__ __forceinline__ int chunk4(int r, int c) {
  if constexpr (kFew) return D == 128 ? c ^ (((r >> 2) & 1) | ((r >> 4) & 1) << 1) : c ^ ((r >> 4) & 1);
  return D == 128 ? c ^ (((r >> 2) & 3) ^ ((r >> 4) & 1)) : c ^ ((r >> 3) & 1);
}
template <int D, bool kFew>
struct Loader4 {
  static constexpr int kRow = D / 2, kHalf = 16 * kRow, kBlock = 2 * kHalf;  // bytes: a row, K's of a block, a block
  static constexpr int kExpWords = D / 8;                                   // of a block's K, and of V
  static constexpr int kLoads = D == 128 ? 3 : 2;                           // wavefront loads of a block
  int at[2];  // the lane's chunk in a tile's first and second block (at 64 channels lanes from 32 on have V's)
  int e_at;
  __device__ __forceinline__ Loader4(int n_heads, int head) {
    const int lane = threadIdx.x & 63;
    const int l = D == 128 ? lane : lane & 31;
    const int r = l / (kRow / 16), c = l % (kRow / 16);
#pragma unroll
    for (int j = 0; j < 2; ++j)
      at[j] = r * kRow + chunk4<D, kFew>(16 * j + r, c) * 16 + (D == 64 && lane >= 32 ? n_heads * kHalf : 0);
    e_at = lane < kExpWords       ? (head * kExpWords + lane) * 4
           : lane < 2 * kExpWords ? ((n_heads + head) * kExpWords + lane - kExpWords) * 4
                                  : 1 << 30;
  }
  // block j of a tile, or nothing; the exponents' room is kExponentBytes
  __device__ __forceinline__ void request(const uint8_t* block, int n_heads, int head, int j, bool wanted, uint8_t* to, uint8_t* to_e) const {
    const uint8_t* k = block + (size_t)head * kHalf;
    const int v_off = n_heads * kHalf;
    load_to_lds<true>(buffer_of(k, wanted ? kHalf + (D == 64 ? v_off : 0) : 0), at[j], reinterpret_cast<half8*>(to));
    if constexpr (D == 128) load_to_lds<true>(buffer_of(k + v_off, wanted ? kHalf : 0), at[j], reinterpret_cast<half8*>(to + kHalf));
    load_word_to_lds(buffer_of(block + 2 * (size_t)v_off, wanted ? 2 * n_heads * kExpWords * 4 : 0), e_at, to_e);
  }
};
typedef __attribute__((address_space(3))) int2v* LdsNibbles;
// (lane l: of the sixteen rows that the sixteen lanes around it point to, 8 bytes each, the code in place l % 16)
__device__ __forceinline__ int2v read_code_columns(const uint8_t* __restrict at) {
  return __builtin_amdgcn_ds_read_tr4_b64_v2i32((LdsNibbles)at);
}
template <int D>
struct E2m1Keys {
  static constexpr int kSlabs = 4;  // a 16-byte read of K is its lane's part of four slabs
  static constexpr int DT = D / 32, G = D / kE2m1Group;
  typedef Loader4<D, false> L;
  const uint8_t* codes;      // two blocks
  const uint8_t* exponents;  // of each
  _Float16* scales;          // V's powers of two [group][half of the wavefront][16 keys], the wavefront's own
  uint4v k_part[G / 2];
  float k_scale[G / 2];
  int2v v_part[DT];
  bool not_finite_seen;
  __device__ __forceinline__ static const uint8_t* row(const uint8_t* codes, int r) { return codes + (r >> 4) * L::kBlock + (r & 15) * L::kRow; }
  // where a key's scale of V lies in its half's sixteen: in the order of the products' keys
  __device__ __forceinline__ static int place(int dt, int key) {
    return (dt * 2 + ((key >> 2) & 1)) * 16 + (key >> 4) * 8 + ((key >> 3) & 1) * 4 + (key & 3);
  }
  __device__ __forceinline__ void set_k() {
    const int lane = threadIdx.x & 63, r = lane & 31, half = lane >> 5;
    const uint8_t* e = exponents + (r >> 4) * kExponentBytes + (r & 15) * G + half;
#pragma unroll
    for (int j = 0; j < G / 2; ++j) {
      k_part[j] = *reinterpret_cast<const uint4v*>(row(codes, r) + chunk4<D, false>(r, 2 * j + half) * 16);
      k_scale[j] = e4m3_scale(e[2 * j]);
    }
  }
  __device__ __forceinline__ half8 k_slab(int, int kk) const { return e2m1_values(k_part[kk / 4][kk % 4], k_scale[kk / 4]); }
  // Keys behind `last` are seen by no row (and their slots may hold anything): times zero.
  template <bool kMasked>
  __device__ __forceinline__ void set_v(int last) {
    const int lane = threadIdx.x & 63, key = lane & 31;
    constexpr int kPer = DT / 2;  // scales that a lane makes
    const uint8_t* e = exponents + (key >> 4) * kExponentBytes + L::kExpWords * 4 + (key & 15) * G + (lane >> 5) * kPer;
    not_finite_seen = false;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const uint32_t x = e[i];
      const bool seen = !kMasked || key <= last;
      // (the code of 1, scaled: 255 << 23 makes it not a number)
      const _Float16 f = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(0x22u, e4m3_scale(x), 0)[0];
      scales[place((lane >> 5) * kPer + i, key)] = seen ? f : (_Float16)0.f;
      if (kMasked && seen && x == kE2m1NotFinite) not_finite_seen = true;
    }
    wave_lds_barrier();
    // row (lane % 16) of the transposing reads: keys in the order of place()
    const int i = lane & 15;
    const int r = (i >> 3) * 16 + ((i >> 2) & 1) * 8 + (lane >> 5) * 4 + (i & 3);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      v_part[dt] = read_code_columns(row(codes, r) + L::kHalf + chunk4<D, false>(r, dt) * 16 + ((lane >> 4) & 1) * 8);
  }
  __device__ __forceinline__ half8 v_slab(int, int kk, int dt) const {
    const half8 scale = *reinterpret_cast<const half8*>(scales + (dt * 2 + ((threadIdx.x & 63) >> 5)) * 16 + kk * 8);
    return e2m1_values(v_part[dt][kk], 1.f) * scale;
  }
  template <int kSub>
  __device__ __forceinline__ bool dirty() const { return __any(not_finite_seen); }
  __device__ __forceinline__ floatx4 not_finite(int key, int channel) const {
    const float x = abs_bits(scales[place(channel / 32, key)]) >= 0x7c00u ? __builtin_nanf("") : 0.f;
    return floatx4{x, x, x, x};
  }
};

// The request's block table, or its head's own one.
__device__ __forceinline__ const int32_t* table_of(const AttnParams& p, const ChunkReq& rq, int head) {
  const int own = p.table_heads > 1 ? head : 0;
  return p.block_tables + ((size_t)rq.table_row * p.table_heads + own) * p.max_blocks;
}
// Block b of the request's cache (behind the last one: the last one, whose rows nobody sees there).
__device__ __forceinline__ int block_id(const AttnParams& p, const int32_t* table, int b, int nb) {
  return clamp_block(load_uniform(table + min(b, nb - 1)), p.n_blocks);
}
template <int D>
__device__ __forceinline__ BufferPtr f16_block(const AttnParams& p, int blk, int head, int which, bool wanted = true) {
  const size_t half_block = (size_t)p.n_heads * 16 * D;
  return buffer_of(static_cast<const _Float16*>(p.kv) + (size_t)blk * 2 * half_block + which * half_block + (size_t)head * 16 * D,
                   wanted ? 16 * D * 2 : 0);
}
// Packed rows from address `from` on, rows_left of them the request's (what is read behind
// them is zeros).
template <int D>
__device__ __forceinline__ BufferPtr rows_at(const _Float16* from, int stride, int rows_left) {
  return buffer_of(from, rows_left > 0 ? (min(rows_left, 16) - 1) * stride * 2 + D * 2 : 0);
}

// ---------------------------------------------------------------------------
// Many rows: four wavefronts of 32 rows over the same keys, 64 at a time.  Two tiles in LDS:
// while one is worked on, each wavefront brings in 16 keys of the next, straight from memory to
// LDS (32 prompts of 600-1200 tokens, 32 heads: 392 us, through registers 741; now 358-397, by
// process and card).  Where its rows see all of a tile, the loop without a mask; the border is the
// wavefront's own (with the workgroup's 373 beside 359).
//
// 64 KB of LDS: two workgroups a CU, the softmax of one beside the products of the other.  Measured,
// 128 channels: prompts of 5900-7040 tokens, 8 heads of K and V and 32 query heads, 0.82-1.04 PFLOP/s by
// card (a library product of 8192^3: 1.09-1.18); 2048 tokens behind 30 000 0.82-1.05, over 8 bits (keys
// through registers) 1.02 beside 1.05; 32 prompts of 600-1200, 32 heads, 0.56-0.61; one of 640, 17-19
// us; 64 channels: the 2048 tokens 0.85.  Long prompts are bound by the card's power: the matrix pipes
// are busy for 60 % of the cycles, at 1.6 GHz, and with zeros for random numbers the same work runs at
// 1.2-1.4 PFLOP/s.  Short ones (34 % of the cycles) by what does not overlap: queries, the first tile,
// the tiles at the mask and the results of two workgroups at a time.
// ---------------------------------------------------------------------------
template <int D, int SRC, bool kSplit, typename Reqs>
__device__ __forceinline__ void attend_tall(const AttnParams& p, const Reqs& reqs, half8* sm, int unit, int head) {
  constexpr int kKeys = 64, kTile = kKeys * D / 8;  // half8s of K, and of V; sm: [2][K, V][kTile]
  const AttnLaunchView& l = p.launch[ATTN_TALL];
  const Place w = place_of<kTallRows, kSplit>(p, reqs, l, unit);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int first_key = w.rq.seq_len - w.rq.n_new;  // what token 0 sees last
  const int row0 = w.tile * kTallRows + wave * 32;
  const LaneRow me = lane_row(p, row0 + (lane & 31), w.n_rows);
  const int q_head = head * p.group + me.in_group;
  const int last_key = min(first_key + me.token, w.key_end - 1);  // (a segment may end inside a tile)
  // the last key that any row of the wavefront sees (none if it has no row)
  const int wave_last = row0 < w.n_rows ? min(first_key + token_of(p, min(row0 + 31, w.n_rows - 1)), w.key_end - 1) : -1;
  const int n_tiles = w.key_end > w.key_begin ? (w.key_end - w.key_begin + kKeys - 1) / kKeys : 0;
  // tiles that every row of the wavefront sees whole (the wavefronts' differ; all meet once a tile)
  const int n_full =
      row0 < w.n_rows ? max(min(first_key + token_of(p, row0), w.key_end - 1) + 1 - w.key_begin, 0) / kKeys : 0;

  Rows32<D> rows;
  rows.start();

  const int32_t* table = SRC == ATTN_ROWS ? nullptr : table_of(p, w.rq, head);
  const int k_stride = SRC == ATTN_ROWS ? (int)p.k.token_stride : D, v_stride = SRC == ATTN_ROWS ? (int)p.v.token_stride : D;
  const BlockLoader<D, false> loader(2 * k_stride, 2 * v_stride);
  half8* to_mine = sm + wave * 16 * D / 8;
  // the next 16 keys that this wavefront brings in
  int block = (w.key_begin >> 4) + wave, next_id = 0;
  int rows_left = w.rq.seq_len - 16 * block;
  const _Float16 *k_from = nullptr, *v_from = nullptr;
  if constexpr (SRC == ATTN_ROWS) {
    k_from = row_of(p.k, w.rq, 16 * block, head);
    v_from = row_of(p.v, w.rq, 16 * block, head);
  } else if (n_tiles > 0) {
    next_id = block_id(p, table, block, w.nb);
  }
  constexpr bool kCodes = SRC == ATTN_E4M3 || SRC == ATTN_E2M1;  // through registers
  std::conditional_t<SRC == ATTN_E2M1, Block4<D>, Block8<D>> b8;
  auto request = [&](int t) {
    half8* to = to_mine + (t & 1) * 2 * kTile;
    if constexpr (SRC == ATTN_ROWS) {
      loader.k(rows_at<D>(k_from, k_stride, rows_left), to);
      loader.v(rows_at<D>(v_from, v_stride, rows_left), to + kTile);
      k_from += (int64_t)kKeys * k_stride;
      v_from += (int64_t)kKeys * v_stride;
      rows_left -= kKeys;
    } else {
      if constexpr (SRC == ATTN_F16) {
        loader.k(f16_block<D>(p, next_id, head, 0), to);
        loader.v(f16_block<D>(p, next_id, head, 1), to + kTile);
      } else {
        const size_t bytes = SRC == ATTN_E2M1 ? e2m1_block_bytes(p.n_heads, D) : e4m3_block_bytes(p.n_heads, D);
        b8.request(static_cast<const uint8_t*>(p.kv) + (size_t)next_id * bytes, p.n_heads, head);
      }
      block += kKeys / 16;
      next_id = block_id(p, table, block, w.nb);
    }
  };
  auto put8 = [&](int t) {
    half8* to = sm + (t & 1) * 2 * kTile;
    b8.put(to, to + kTile, wave * 16);
  };
  // tile t, the next one on its way: work(tile's place in LDS)
  auto step = [&](int t, auto work) {
    if constexpr (!kCodes) wait_loads<0>();
    lds_barrier();  // tile t is there, the one before has been read
    if (t + 1 < n_tiles) request(t + 1);
    work();
    if constexpr (kCodes) {
      if (t + 1 < n_tiles) put8(t + 1);
    }
  };
  const typename Rows32<D>::Offsets operands = Rows32<D>::offsets();
  auto even = [&] { rows.template attend_full<0>(sm, operands, p.scale_log2e); };
  auto odd = [&] { rows.template attend_full<2 * kTile * 16>(sm, operands, p.scale_log2e); };
  if (n_tiles > 0) {
    const GroupRows from(p.q, w.rq, p, head);
    rows.request_queries([&](int r) { return from.at(lane_row(p, row0 + r, w.n_rows)); });
    request(0);
    if constexpr (kCodes) put8(0);
    // (the second tile's room is free until the first barrier)
    rows.template take_queries<F16Keys<D>::kSlabs>(sm + 2 * kTile + wave * 32 * D / 8);
  }
  int t = 0;
  for (; t + 1 < n_full; t += 2) {
    step(t, even);
    step(t + 1, odd);
  }
  if (t < n_full) step(t++, even);
  for (; t < n_tiles; ++t)
    step(t, [&] {
      const half8* sm_k = sm + (t & 1) * 2 * kTile;
      const int key0 = w.key_begin + t * kKeys;
      // 32 keys at a time, those that none of the wavefront's rows sees left out
#pragma unroll 1
      for (int at = 0; at < kKeys && key0 + at <= wave_last; at += 32)
        rows.template attend<1, true>(F16Keys<D>{sm_k, sm_k + kTile, at}, key0 + at, last_key, p.scale_log2e, [] {}, [] {});
    });

  const float z = other_half_sum(rows.z);
  const float inv = z == 0.f ? 0.f : 1.f / z;
  const float log2_sum = z == 0.f ? -INFINITY : rows.m + __builtin_amdgcn_logf(z);
  if (kSplit && w.n_seg > 1) {  // a segment's state: the normalised result and the log2 of the sum
    if (!me.real) return;
    float* state = state_of<D>(p, l, w.rq, me.token, q_head, w.seg);
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        floatx4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = rows.o[dt][4 * j + e] * inv;
        *reinterpret_cast<floatx4*>(state + dt * 32 + j * 8 + half * 4) = x;
      }
    if (half == 0) state[D] = log2_sum;
    return;
  }
  lds_barrier();  // (the last tile has been read)
  const GroupRows to(p.out, w.rq, p, head);
  rows.write_result(sm + wave * 32 * D / 8, inv, [&](int r) -> _Float16* {
    const LaneRow it = lane_row(p, row0 + r, w.n_rows);
    return it.real ? to.at(it) : nullptr;
  });
  if (half == 0 && me.real) write_lse(p, w.rq, me.token, q_head, log2_sum);
}

// ---------------------------------------------------------------------------
// Few rows: four wavefronts over the same 32 rows; each takes every fourth 32 keys, which it
// brings in by itself (no barrier in the loop), and the four states are joined at the end.
// A wavefront has room for one tile: K of the next one is on its way as soon as K has been
// read, V as soon as V has, so that a tile's K or V always is.
//
// Every row of K and V is read once per head, whatever the group.  Measured, 128 channels, fp16:
// single tokens of 48 caches of 1280-7040, 8 heads, 4 query heads each, 5.9 TB/s with the store
// and the merge (135 us, 124 at the card's 6.4 TB/s for reads); 32 heads of their own, 6.4 (491 us).
// 8-bit: 32 heads 6.2 TB/s (259 us), 8 heads of four 4.8 with the merge (84 us of attention and merge,
// 62 at 6.4), the conversion to fp16 beside the loads (16 vector instructions a product, fp16 rows
// 6.6); 5 drafted tokens of 32 caches of 256-1408: 19 us and 6 for the merge, latency.  4-bit, 17 rows and more:
// the same drafts, 8 heads of four, 30.5 us with the store and the merge; a chunk of 2048 behind 30 000 is bound by
// the matrix cores' power as with the other formats (1.05 ms).
// ---------------------------------------------------------------------------

// Bytes of one row of K or V in the LDS of such a wavefront.
template <int D, int SRC>
constexpr int kFlatRowBytes = SRC == ATTN_E4M3 ? D : 2 * D;

// Tiles of a 4-bit pool that such a wavefront has room for, and their bytes with the exponents and V's scales.
constexpr int kStages4 = 3;
constexpr int stage4_bytes(int head_dim) { return 32 * head_dim + 2 * kExponentBytes; }
constexpr int wave4_bytes(int head_dim) { return kStages4 * stage4_bytes(head_dim) + 2 * head_dim; }

// LDS reads before this point have been answered: what they read may be overwritten by loads.
__device__ __forceinline__ void lds_reads_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// id_of(b): number of the request's block b in the pool.
template <int D, int SRC, bool kSplit, typename IdOf>
__device__ __forceinline__ void attend_flat(const AttnParams& p, const Place& w, half8* sm, int head, IdOf id_of) {
  constexpr int kKeys = 32;
  // (codes: two tiles a wavefront fit where one of fp16 rows does; one alone keeps 6 KB on the way
  // on average, and 2048 wavefronts draw 4.2 TB/s with it)
  constexpr int kStages = SRC == ATTN_E4M3 ? 2 : 1;
  constexpr int kTile = kKeys * kFlatRowBytes<D, SRC> / 16;  // sm: [wavefront][stage][K, V][kTile], exponents
  const AttnLaunchView& l = p.launch[ATTN_FLAT];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int first_key = w.rq.seq_len - w.rq.n_new;
  const int row0 = w.tile * kFlatRows;
  const LaneRow me = lane_row(p, row0 + (lane & 31), w.n_rows);
  const int q_head = head * p.group + me.in_group;
  const int last_key = min(first_key + me.token, w.key_end - 1);
  const int first_seen = min(first_key + token_of(p, row0), w.key_end - 1);  // all rows see keys up to this one
  const int n_tiles = w.key_end > w.key_begin ? (w.key_end - w.key_begin + kKeys - 1) / kKeys : 0;
  const int mine = own_tiles(n_tiles, wave, 4);
  // tiles that every row sees whole come first
  const int full = min(mine, own_tiles(max(first_seen + 1 - w.key_begin, 0) / kKeys, wave, 4));

  Rows32<D> rows;
  rows.start();
  const GroupRows from(p.q, w.rq, p, head), to(p.out, w.rq, p, head);
  rows.request_queries([&](int r) { return from.at(lane_row(p, row0 + r, w.n_rows)); });

  half8* sm_k = sm + wave * 2 * kStages * kTile;
  int ids[2] = {0, 0};
  auto block_of = [&](int i, int j) { return (w.key_begin >> 4) + 2 * (wave + 4 * i) + j; };
  auto look_up = [&](int i) {
    if constexpr (SRC != ATTN_ROWS) {
      ids[0] = id_of(block_of(i, 0));
      ids[1] = id_of(block_of(i, 1));
    }
  };
  auto key_of = [&](int i) { return w.key_begin + (wave + 4 * i) * kKeys; };

  // (tiles behind the last one are requested as nothing: every wait counts the same loads)
  if constexpr (SRC == ATTN_E4M3) {
    const Loader8<D> loader;
    uint8_t* sm_e = reinterpret_cast<uint8_t*>(sm + 4 * 2 * kStages * kTile) + wave * kStages * 2 * kExponentBytes;
    const size_t codes = (size_t)2 * p.n_heads * 16 * D;
    // words 0..3 of the exponents: K's, 4..7: V's
    const int e_at = lane < 4 ? head * 16 + lane * 4 : lane < 8 ? (p.n_heads + head) * 16 + (lane - 4) * 4 : 1 << 30;
    auto block_at = [&](int j) {
      return static_cast<const uint8_t*>(p.kv) + (size_t)ids[j] * e4m3_block_bytes(p.n_heads, D);
    };
    auto request_k = [&](int i) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        load_word_to_lds(buffer_of(block_at(j) + codes, i < mine ? 2 * p.n_heads * 16 : 0), e_at,
                         sm_e + ((i % kStages) * 2 + j) * kExponentBytes);
        loader.k(buffer_of(block_at(j) + (size_t)head * 16 * D, i < mine ? 16 * D : 0), sm_k + (i % kStages) * 2 * kTile + j * D);
      }
    };
    auto request_v = [&](int i) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
        loader.v(buffer_of(block_at(j) + codes / 2 + (size_t)head * 16 * D, i < mine ? 16 * D : 0),
                 sm_k + (i % kStages) * 2 * kTile + kTile + j * D);
    };
    constexpr int kV = 2 * Loader8<D>::kInstr, kK = kV + 2;  // loads of a tile
    if (mine > 0) {
#pragma unroll
      for (int i = 0; i < kStages; ++i) {
        look_up(i);
        request_k(i);
        lds_reads_done();  // (K's loads stay ahead of V's, as the waits count on)
        request_v(i);
        lds_reads_done();
        if (i == 0) {  // through the second tile's room
          rows.template take_queries<E4m3Keys<D>::kSlabs>(sm_k + 2 * kTile);
          lds_reads_done();
        }
      }
    }
    auto step = [&](int i, auto masked_) {
      constexpr bool kMasked = decltype(masked_)::value;
      const uint8_t* here = reinterpret_cast<const uint8_t*>(sm_k + (i % kStages) * 2 * kTile);
      const uint8_t* exponents = sm_e + (i % kStages) * 2 * kExponentBytes;
      E4m3Keys<D> keys{here, here + kTile * 16};
      const int key0 = key_of(i);
      look_up(i + kStages);
      wait_loads<(kStages - 1) * (kK + kV) + kV>();
      keys.set_k(exponents);
      keys.template set_v<kMasked>(exponents, w.key_end - 1 - key0);
      rows.template attend<1, kMasked>(
          keys, key0, last_key, p.scale_log2e,
          [&] {
            lds_reads_done();
            request_k(i + kStages);
          },
          [] { wait_loads<(kStages - 1) * (kK + kV) + kK>(); });
      lds_reads_done();
      request_v(i + kStages);
    };
    int i = 0;
    for (; i < full; ++i) step(i, std::false_type());
    for (; i < mine; ++i) step(i, std::true_type());
  } else if constexpr (SRC == ATTN_E2M1) {
    // Two tiles on their way while a third is worked on.
    typedef Loader4<D, false> L;
    const L loader(p.n_heads, head);
    uint8_t* mine4 = reinterpret_cast<uint8_t*>(sm) + wave * wave4_bytes(D);
    auto stage = [&](int i) { return mine4 + (i % kStages4) * stage4_bytes(D); };
    auto request = [&](int i) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
        loader.request(static_cast<const uint8_t*>(p.kv) + (size_t)ids[j] * e2m1_block_bytes(p.n_heads, D), p.n_heads, head, j, i < mine,
                       stage(i) + j * L::kBlock, stage(i) + 2 * L::kBlock + j * kExponentBytes);
    };
    E2m1Keys<D> keys;
    keys.scales = reinterpret_cast<_Float16*>(mine4 + kStages4 * stage4_bytes(D));
    if (mine > 0) {
      static_assert((kStages4 - 1) * stage4_bytes(D) >= 32 * D * 2, "the queries' room");
#pragma unroll
      for (int i = 0; i < kStages4; ++i) {
        look_up(i);
        request(i);
        if (i == 0) {  // through the other tiles' room
          rows.template take_queries<E2m1Keys<D>::kSlabs>(reinterpret_cast<half8*>(stage(1)));
          lds_reads_done();
        }
      }
    }
    auto step = [&](int i, auto masked_) {
      constexpr bool kMasked = decltype(masked_)::value;
      const int key0 = key_of(i);
      look_up(i + kStages4);
      wait_loads<(kStages4 - 1) * 2 * L::kLoads>();
      keys.codes = stage(i);
      keys.exponents = stage(i) + 2 * L::kBlock;
      keys.set_k();
      rows.template attend<1, kMasked>(
          keys, key0, last_key, p.scale_log2e, [] {}, [&] { keys.template set_v<kMasked>(w.key_end - 1 - key0); });
      lds_reads_done();
      request(i + kStages4);
    };
    int i = 0;
    for (; i < full; ++i) step(i, std::false_type());
    for (; i < mine; ++i) step(i, std::true_type());
  } else {
    const BlockLoader<D, SRC == ATTN_F16> loader(SRC == ATTN_ROWS ? (int)p.k.token_stride * 2 : D * 2,
                                                 SRC == ATTN_ROWS ? (int)p.v.token_stride * 2 : D * 2);
    const F16Keys<D> keys{sm_k, sm_k + kTile, 0};
    auto request_k = [&](int i) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int first = 16 * block_of(i, j);
        loader.k(SRC == ATTN_ROWS ? rows_at<D>(row_of(p.k, w.rq, first, head), (int)p.k.token_stride, w.rq.seq_len - first)
                                  : f16_block<D>(p, ids[j], head, 0, i < mine),
                 sm_k + j * 2 * D);
      }
    };
    auto request_v = [&](int i) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int first = 16 * block_of(i, j);
        loader.v(SRC == ATTN_ROWS ? rows_at<D>(row_of(p.v, w.rq, first, head), (int)p.v.token_stride, w.rq.seq_len - first)
                                  : f16_block<D>(p, ids[j], head, 1, i < mine),
                 sm_k + kTile + j * 2 * D);
      }
    };
    constexpr int kLoads = 2 * BlockLoader<D, false>::kInstr;
    if (mine > 0) {
      look_up(0);
      request_k(0);
      lds_reads_done();  // (K's loads stay ahead of V's, as the waits count on)
      rows.template take_queries<F16Keys<D>::kSlabs>(sm_k + kTile);  // through V's room
      lds_reads_done();
      request_v(0);
    }
    auto step = [&](int i, auto masked_) {
      look_up(i + 1);
      wait_loads<kLoads>();  // (V may be on its way)
      rows.template attend<1, decltype(masked_)::value>(
          keys, key_of(i), last_key, p.scale_log2e,
          [&] {
            lds_reads_done();
            request_k(i + 1);
          },
          [] { wait_loads<kLoads>(); });
      lds_reads_done();
      request_v(i + 1);
    };
    int i = 0;
    for (; i < full; ++i) step(i, std::false_type());
    for (; i < mine; ++i) step(i, std::true_type());
  }
  wait_loads<0>();
  const float z = other_half_sum(rows.z), m = rows.m;

  // ---- joining the four states -----------------------------------------------------------
  __shared__ float sm_m[4][32], sm_z[4][32];
  if (half == 0) {
    sm_m[wave][lane] = m;
    sm_z[wave][lane] = z;
  }
  __syncthreads();  // (and every wavefront is done with its keys)
  float mm = -INFINITY, zz = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) mm = fmaxf(mm, sm_m[i][lane & 31]);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float zi = sm_z[i][lane & 31];
    zz += zi == 0.f ? 0.f : zi * __builtin_amdgcn_exp2f(sm_m[i][lane & 31] - mm);
  }
  const float log2_sum = zz == 0.f ? -INFINITY : mm + __builtin_amdgcn_logf(zz);
  const float f = z == 0.f ? 0.f : __builtin_amdgcn_exp2f(m - mm) / zz;
  // [wavefront][row][channel], quads permuted within the row against bank conflicts
  constexpr int kQuads = D / 4;
  floatx4* sm_o = reinterpret_cast<floatx4*>(sm);
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      floatx4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = rows.o[dt][4 * j + e] * f;
      const int c = dt * 8 + j * 2 + half, r = lane & 31;
      sm_o[(wave * 32 + r) * kQuads + (c ^ (r & (kQuads - 1)))] = x;
    }
  if (wave == 0 && half == 0 && me.real) {
    if (kSplit && w.n_seg > 1)
      state_of<D>(p, l, w.rq, me.token, q_head, w.seg)[D] = log2_sum;
    else
      write_lse(p, w.rq, me.token, q_head, log2_sum);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 32 * kQuads; i += 256) {
    const int r = i / kQuads, c = i % kQuads;
    const LaneRow it = lane_row(p, row0 + r, w.n_rows);
    if (!it.real) break;
    floatx4 x = sm_o[r * kQuads + (c ^ (r & (kQuads - 1)))];
#pragma unroll
    for (int k = 1; k < 4; ++k) x += sm_o[(k * 32 + r) * kQuads + (c ^ (r & (kQuads - 1)))];
    if (kSplit && w.n_seg > 1) {
      *reinterpret_cast<floatx4*>(state_of<D>(p, l, w.rq, it.token, head * p.group + it.in_group, w.seg) + c * 4) = x;
    } else {
      half4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = (_Float16)f16_result(x[e]);
      *reinterpret_cast<half4*>(to.at(it) + c * 4) = y;
    }
  }
}

// ---------------------------------------------------------------------------
// Up to 16 rows of a head over 4 bits (single tokens of grouped heads): as the few rows above, on
// v_mfma_f32_16x16x32_f16, a lane a row again, four lanes to each.  With the keys in so few bytes the
// instructions are what a wavefront waits for: of 32 rows' softmax and products most are of rows that
// there are not, and 222 registers leave a SIMD two wavefronts.  Here it has four.  Single tokens of 48 caches of
// 1280-7040, 8 heads of four: the attention 57.6 -> 44 us, 220 MB, 5.0 TB/s with the launch and its ends; between
// them 6.7 (first loads some 5 us, and workgroups that end unevenly: heads are cut into segments of half a share,
// thirds and whole ones take 56-57 for 54 of the whole step).  Rows of 16 keys as f8f6f4 operands, queries in three
// e4m3 parts, saved the conversions and gained nothing (45 us).
//   S^T: a lane reads a group of 32 channels of a key (16 at 64 channels); the queries' channels follow.
//   O^T: a transposing read has eight keys of a lane's column for two tiles of 16 channels, one group.
// ---------------------------------------------------------------------------
constexpr int kFewRows = kFewRows4;
constexpr int kFewStages = 2;
constexpr int few_wave_bytes(int head_dim) { return kFewStages * stage4_bytes(head_dim) + 2 * head_dim; }

__device__ __forceinline__ float quarter_max(float v) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  return other_half_max(v);
}

template <int D>
struct Keys16 {
  static constexpr int KS = D / 32, DT = D / 32, G = D / kE2m1Group;  // slabs of a key that a lane has; groups
  typedef Loader4<D, true> L;
  const uint8_t* codes;      // two blocks
  const uint8_t* exponents;  // of each
  _Float16* scales;          // V's powers of two [group][quarter of the wavefront][8 keys], the wavefront's own
  uint32_t k_part[2][KS];
  float k_scale[2];
  int2v v_part[DT];
  bool not_finite_seen;
  __device__ __forceinline__ static const uint8_t* row(const uint8_t* codes, int r) { return codes + (r >> 4) * L::kBlock + (r & 15) * L::kRow; }
  // where a key's scale of V lies: in the order of the products' keys
  __device__ __forceinline__ static int place(int dt, int key) { return (dt * 4 + ((key >> 2) & 3)) * 8 + (key >> 4) * 4 + (key & 3); }
  __device__ __forceinline__ void set_k() {
    const int lane = threadIdx.x & 63, quarter = lane >> 4;
    const int group = D == 128 ? quarter : quarter >> 1;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int r = 16 * t + (lane & 15);
      const uint8_t* from = row(codes, r) + chunk4<D, true>(r, group) * 16;
      if constexpr (D == 128) {
        const uint4v c = *reinterpret_cast<const uint4v*>(from);
#pragma unroll
        for (int i = 0; i < 4; ++i) k_part[t][i] = c[i];
      } else {
        const uint2v c = *reinterpret_cast<const uint2v*>(from + (quarter & 1) * 8);
#pragma unroll
        for (int i = 0; i < 2; ++i) k_part[t][i] = c[i];
      }
      k_scale[t] = e4m3_scale(exponents[t * kExponentBytes + (lane & 15) * G + group]);
    }
  }
  // Keys behind `last` are seen by no row (and their slots may hold anything): times zero.
  template <bool kMasked>
  __device__ __forceinline__ void set_v(int last) {
    const int lane = threadIdx.x & 63, key = lane & 31;
    constexpr int kPer = DT / 2;  // scales that a lane makes
    const uint8_t* e = exponents + (key >> 4) * kExponentBytes + L::kExpWords * 4 + (key & 15) * G + (lane >> 5) * kPer;
    not_finite_seen = false;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const uint32_t x = e[i];
      const bool seen = !kMasked || key <= last;
      // (the code of 1, scaled: 255 << 23 makes it not a number)
      const _Float16 f = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(0x22u, e4m3_scale(x), 0)[0];
      scales[place((lane >> 5) * kPer + i, key)] = seen ? f : (_Float16)0.f;
      if (kMasked && seen && x == kE2m1NotFinite) not_finite_seen = true;
    }
    wave_lds_barrier();
    // rows of the transposing reads: eight keys, at 16 channels and at the next 16
    const int i = lane & 7, r = (i >> 2) * 16 + (lane >> 4) * 4 + (i & 3);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      v_part[dt] = read_code_columns(row(codes, r) + L::kHalf + chunk4<D, true>(r, dt) * 16 + ((lane >> 3) & 1) * 8);
  }
  __device__ __forceinline__ half8 v_scales(int dt) const {
    return *reinterpret_cast<const half8*>(scales + (dt * 4 + ((threadIdx.x & 63) >> 4)) * 8);
  }
};

template <int D, bool kSplit, typename IdOf>
__device__ __forceinline__ void attend_few4(const AttnParams& p, const Place& w, half8* sm, int head, IdOf id_of) {
  constexpr int kKeys = 32, KS = D / 32, CT = D / 16;
  typedef Loader4<D, true> L;
  const AttnLaunchView& l = p.launch[ATTN_FLAT];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, quarter = lane >> 4;
  const int first_key = w.rq.seq_len - w.rq.n_new;
  const LaneRow me = lane_row(p, lane & 15, w.n_rows);
  const int last_key = min(first_key + me.token, w.key_end - 1);
  const int first_seen = min(first_key, w.key_end - 1);  // all rows see keys up to this one
  const int n_tiles = w.key_end > w.key_begin ? (w.key_end - w.key_begin + kKeys - 1) / kKeys : 0;
  const int mine = own_tiles(n_tiles, wave, 4);
  // tiles that every row sees whole come first
  const int full = min(mine, own_tiles(max(first_seen + 1 - w.key_begin, 0) / kKeys, wave, 4));
  const GroupRows from(p.q, w.rq, p, head), to(p.out, w.rq, p, head);

  half8 q[KS];
#pragma unroll
  for (int i = 0; i < KS; ++i) {
    const int at = i * 64 + lane;
    q[i] = load_half8(from.at(lane_row(p, at / (D / 8), w.n_rows)) + (at % (D / 8)) * 8);
  }
  floatx4 o[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) o[c] = floatx4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, z = 0.f;

  const L loader(p.n_heads, head);
  uint8_t* own = reinterpret_cast<uint8_t*>(sm) + wave * few_wave_bytes(D);
  auto stage = [&](int i) { return own + (i % kFewStages) * stage4_bytes(D); };
  int ids[2] = {0, 0};
  auto look_up = [&](int i) {
    const int b = (w.key_begin >> 4) + 2 * (wave + 4 * i);
    ids[0] = id_of(b);
    ids[1] = id_of(b + 1);
  };
  // (tiles behind the last one are requested as nothing: every wait counts the same loads)
  auto request = [&](int i) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
      loader.request(static_cast<const uint8_t*>(p.kv) + (size_t)ids[j] * e2m1_block_bytes(p.n_heads, D), p.n_heads, head, j, i < mine,
                     stage(i) + j * L::kBlock, stage(i) + 2 * L::kBlock + j * kExponentBytes);
  };
  Keys16<D> keys;
  keys.scales = reinterpret_cast<_Float16*>(own + kFewStages * stage4_bytes(D));
  if (mine > 0) {
    look_up(0);
    request(0);
    look_up(1);
    // the queries through the other tile's room
    static_assert(stage4_bytes(D) >= kFewRows * D * 2, "room");
    half8* room = reinterpret_cast<half8*>(stage(1));
#pragma unroll
    for (int i = 0; i < KS; ++i) room[k_chunk<D>((i * 64 + lane) / (D / 8), lane % (D / 8))] = q[i];
    wave_lds_barrier();
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) q[kk] = room[k_chunk<D>(lane & 15, KS * quarter + kk)];
    lds_reads_done();
    request(1);
  }
  auto step = [&](int i, auto masked_) {
    constexpr bool kMasked = decltype(masked_)::value;
    const int key0 = w.key_begin + (wave + 4 * i) * kKeys;
    look_up(i + kFewStages);
    wait_loads<(kFewStages - 1) * 2 * L::kLoads>();
    keys.codes = stage(i);
    keys.exponents = stage(i) + 2 * L::kBlock;
    keys.set_k();
    keys.template set_v<kMasked>(w.key_end - 1 - key0);
    // (the tile is in registers: two more are on their way while it is worked on)
    lds_reads_done();
    request(i + kFewStages);
    floatx4 s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) s[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kk = 0; kk < KS; ++kk)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(e2m1_values(keys.k_part[t][kk], keys.k_scale[t]), q[kk], s[t], 0, 0, 0);
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if constexpr (kMasked) {
          if (key0 + t * 16 + quarter * 4 + r > last_key) s[t][r] = -INFINITY;
        }
        top = fmaxf(top, s[t][r]);
      }
    // m follows the maximum when that is more than kSlack ahead, as in Rows32
    const float mn = fmaxf(m, quarter_max(top) * p.scale_log2e);
    if (__any(mn > m + kSlack)) {
      const float a = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      z *= a;
#pragma unroll
      for (int c = 0; c < CT; ++c) o[c] *= a;
      m = mn;
    }
    const float base = m == -INFINITY ? 0.f : m;
    half8 pb;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float x = __builtin_amdgcn_exp2f(fmaf(s[t][r], p.scale_log2e, -base));
        z += x;
        pb[t * 4 + r] = (_Float16)x;
      }
    // Where some row does not see some key, 0 * NaN must not reach it: as in Rows32
    bool dirty = false;
    if constexpr (kMasked) {
      dirty = __any(key0 + kKeys - 1 > last_key) && __any(keys.not_finite_seen);
      if (dirty) {
#pragma unroll 1
        for (int key = 0; key < kKeys; ++key) {
          if (key0 + key > last_key) continue;
#pragma unroll
          for (int c = 0; c < CT; ++c)
            if (abs_bits(keys.scales[Keys16<D>::place(c / 2, key)]) >= 0x7c00u) o[c] += __builtin_nanf("");
        }
      }
    }
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) {
      const half8 scale = keys.v_scales(dt);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        half8 v = e2m1_values(keys.v_part[dt][h], 1.f) * scale;
        if constexpr (kMasked) {
          if (dirty) v = finite_only(v);
        }
        o[2 * dt + h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pb, o[2 * dt + h], 0, 0, 0);
      }
    }
  };
  int i = 0;
  for (; i < full; ++i) step(i, std::false_type());
  for (; i < mine; ++i) step(i, std::true_type());
  wait_loads<0>();
  z = quarter_sum(z);

  // ---- joining the four states, as above ---------------------------------------------------
  __shared__ float sm_m[4][kFewRows], sm_z[4][kFewRows];
  if (quarter == 0) {
    sm_m[wave][lane] = m;
    sm_z[wave][lane] = z;
  }
  __syncthreads();  // (and every wavefront is done with its keys)
  float mm = -INFINITY, zz = 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) mm = fmaxf(mm, sm_m[k][lane & 15]);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float zk = sm_z[k][lane & 15];
    zz += zk == 0.f ? 0.f : zk * __builtin_amdgcn_exp2f(sm_m[k][lane & 15] - mm);
  }
  const float log2_sum = zz == 0.f ? -INFINITY : mm + __builtin_amdgcn_logf(zz);
  const float f = z == 0.f ? 0.f : __builtin_amdgcn_exp2f(m - mm) / zz;
  constexpr int kQuads = D / 4;
  floatx4* sm_o = reinterpret_cast<floatx4*>(sm);
  static_assert(4 * kFewRows * kQuads * 16 <= 4 * few_wave_bytes(D), "room");
#pragma unroll
  for (int c = 0; c < CT; ++c)
    sm_o[(wave * kFewRows + (lane & 15)) * kQuads + ((c * 4 + quarter) ^ (lane & 15))] = o[c] * f;
  if (wave == 0 && quarter == 0 && me.real) {
    const int q_head = head * p.group + me.in_group;
    if (kSplit && w.n_seg > 1)
      state_of<D>(p, l, w.rq, me.token, q_head, w.seg)[D] = log2_sum;
    else
      write_lse(p, w.rq, me.token, q_head, log2_sum);
  }
  __syncthreads();
  for (int k = threadIdx.x; k < kFewRows * kQuads; k += 256) {
    const int r = k / kQuads, c = k % kQuads;
    const LaneRow it = lane_row(p, r, w.n_rows);
    if (!it.real) break;
    floatx4 x = sm_o[r * kQuads + (c ^ r)];
#pragma unroll
    for (int n = 1; n < 4; ++n) x += sm_o[(n * kFewRows + r) * kQuads + (c ^ r)];
    if (kSplit && w.n_seg > 1) {
      *reinterpret_cast<floatx4*>(state_of<D>(p, l, w.rq, it.token, head * p.group + it.in_group, w.seg) + c * 4) = x;
    } else {
      half4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = (_Float16)f16_result(x[e]);
      *reinterpret_cast<half4*>(to.at(it) + c * 4) = y;
    }
  }
}

template <int D, bool kSplit, typename Reqs>
__global__ __launch_bounds__(256, 4) void attention_few4_kernel(AttnParams p, Reqs reqs) {
  extern __shared__ __align__(16) half8 sm[];
  const int unit = blockIdx.x / p.n_heads;
  const int head = blockIdx.x - unit * p.n_heads;
  const Place w = place_of<kFlatRows, kSplit>(p, reqs, p.launch[ATTN_FLAT], unit);  // (no more rows than a tile: one a request)
  const int32_t* table = table_of(p, w.rq, head);
  attend_few4<D, kSplit>(p, w, sm, head, [&](int b) { return block_id(p, table, b, w.nb); });
}

// The units with many rows come first: they are the heavy ones.
template <int D, int SRC, bool kSplit, typename Reqs>
__global__ __launch_bounds__(256, 2) void attention_kernel(AttnParams p, Reqs reqs) {
  extern __shared__ __align__(16) half8 sm[];
  const int unit = blockIdx.x / p.n_heads;
  const int head = blockIdx.x - unit * p.n_heads;
  if (unit < p.launch[ATTN_TALL].n_units)
    attend_tall<D, SRC, kSplit>(p, reqs, sm, unit, head);
  else {
    const Place w = place_of<kFlatRows, kSplit>(p, reqs, p.launch[ATTN_FLAT], unit - p.launch[ATTN_TALL].n_units);
    const int32_t* table = SRC == ATTN_ROWS ? nullptr : table_of(p, w.rq, head);
    attend_flat<D, SRC, kSplit>(p, w, sm, head, [&](int b) { return block_id(p, table, b, w.nb); });
  }
}

// A token's head over the blocks that it selects: scores, selection and attention of up to 32 rows by one workgroup.
// The tokens' selections end unevenly, chains of latencies all of them; here a workgroup's streams while another one's
// on its CU selects, and the blocks' numbers stay in LDS.  Single tokens of 48 caches of 1280-7040, 8 heads of four,
// n_select 64, with the bounds before (us, apart / so): fp16 63.5 / 56.6, 8 bits 49 / 42.7, 4 bits 45.5 / 36.8; 256
// blocks of 32 caches 97 / 84; in 4 bits 16 caches of 1000-4000, 32 heads, 43 / 34.
// (4 bits, up to 16 rows, 128 channels: 128 registers would do for four workgroups a CU, its 43 KB of LDS for three;
// 384 heads on 256 CUs are one or two, so that a head's chain shows: 36 us where the bytes take 16.)
constexpr int kSelectedWaves = 4;
template <int D, int SRC, bool kFew4, typename Reqs>
__global__ __launch_bounds__(64 * kSelectedWaves, kFew4 ? 4 : 2) void attention_selected_kernel(SelectParams sp, AttnParams p, Reqs tokens, int ids_at) {
  extern __shared__ __align__(16) half8 sm[];
  const int token = blockIdx.x / p.n_heads;
  const int head = blockIdx.x - token * p.n_heads;
  const ChunkReq rq = tokens.req[token];
  int32_t* ids = reinterpret_cast<int32_t*>(reinterpret_cast<char*>(sm) + ids_at);
  select_for_token<D, kSelectedWaves>(sp, rq, head, Selection(sp, ids, (int64_t)token * p.n_heads + head), reinterpret_cast<char*>(sm));
  __syncthreads();
  Place w;
  w.rq = {token, selected_keys(rq.seq_len, sp.n_select), 1, rq.row_off, 0, 0};
  w.n_rows = p.group;
  w.tile = w.seg = w.key_begin = 0;
  w.n_seg = 1;
  w.nb = (w.rq.seq_len + 15) >> 4;
  w.key_end = w.rq.seq_len;
  auto id_of = [&](int b) { return clamp_block(__builtin_amdgcn_readfirstlane(ids[min(b, w.nb - 1)]), p.n_blocks); };
  if constexpr (kFew4)
    attend_few4<D, false>(p, w, sm, head, id_of);
  else
    attend_flat<D, SRC, false>(p, w, sm, head, id_of);
}

// Rows whose keys were split: the result from the segments' states.  Workgroup = (token of
// the launch, query head); its four wavefronts take every fourth segment, and each finds the
// common maximum and sum by itself, a segment a lane.  Latency bounds it: 4-5 us for 1536 rows of up
// to three segments, 5.5-7 for 5000 rows.
static constexpr int kMaxHeadSegments = kPlanMaxSeqLen / kPlanBlockSize / kPlanMinSegment;
static_assert(kMaxHeadSegments <= 64, "a segment a lane");

template <int D, typename Reqs>
__global__ __launch_bounds__(256) void attention_merge_kernel(AttnParams p, AttnLaunchView l, Reqs reqs) {
  const int n_q = p.n_heads * p.group;
  const int t = blockIdx.x / n_q;
  const int h = blockIdx.x - t * n_q;
  const ChunkReq rq = reqs.req[request_of(l.first_req, l.n_req, t, [&](int i) { return reqs.req[i].state_off; })];
  const int n_seg = decode_segments((rq.seq_len + 15) >> 4, l.seg_blocks);
  if (n_seg <= 1) return;  // written by the kernel above
  constexpr int kWords = DecodeParams::state_words(D);
  constexpr int kPer = D / 64;  // channels of a lane
  const float* states = l.states + (int64_t)blockIdx.x * l.n_seg * kWords;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const float m = lane < n_seg ? states[(size_t)lane * kWords + D] : -INFINITY;
  float mm = m;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) mm = fmaxf(mm, __shfl_xor(mm, d));
  const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mm);
  const float zz = wave_sum(f);
  float o[kPer] = {};
  for (int i = wave; i < n_seg; i += 16)
#pragma unroll
    for (int j = 0; j < 4; ++j) {  // (four loads on their way)
      const int at = min(i + 4 * j, n_seg - 1);
      const float fi = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), at));
#pragma unroll
      for (int c = 0; c < kPer; ++c)
        o[c] += states[(size_t)at * kWords + lane * kPer + c] * (i + 4 * j < n_seg ? fi : 0.f);
    }
  __shared__ float sm_o[4][D];
#pragma unroll
  for (int c = 0; c < kPer; ++c) sm_o[wave][lane * kPer + c] = o[c];
  __syncthreads();
  const int token = t - rq.state_off;
  if (threadIdx.x < D) {
    const float sum = sm_o[0][threadIdx.x] + sm_o[1][threadIdx.x] + sm_o[2][threadIdx.x] + sm_o[3][threadIdx.x];
    row_of(p.out, rq, token, h)[threadIdx.x] = (_Float16)f16_result(zz == 0.f ? 0.f : sum / zz);
  }
  if (threadIdx.x == 0) write_lse(p, rq, token, h, zz == 0.f ? -INFINITY : mm + __builtin_amdgcn_logf(zz));
}

// two tiles of many rows, or four states of few; as much as the keys of few, but for the exponents
constexpr int lds_bytes(int head_dim, int source) {
  const int tiles = 2 * 2 * 64 * head_dim * 2;
  if (source == ATTN_E2M1) return std::max(tiles, 4 * wave4_bytes(head_dim));
  return tiles + (source == ATTN_E4M3 ? 4 * 2 * 2 * kExponentBytes : 0);
}
static_assert(2 * 2 * 64 * 2 == 4 * 32 * 4 && 4 * 2 * 32 * 2 == 4 * 32 * 4, "per channel");

template <int D, int SRC, bool kSplit, typename Reqs>
void launch_kernel(const AttnParams& p, const Reqs& reqs, hipStream_t s) {
  const unsigned grid = (unsigned)(p.launch[0].n_units + p.launch[1].n_units) * p.n_heads;
  if constexpr (SRC == ATTN_E2M1) {
    if (p.launch[ATTN_TALL].n_units == 0 && p.launch[ATTN_FLAT].most_rows <= kFewRows) {
      attention_few4_kernel<D, kSplit, Reqs><<<grid, 256, 4 * few_wave_bytes(D), s>>>(p, reqs);
      return;
    }
  }
  attention_kernel<D, SRC, kSplit, Reqs><<<grid, 256, lds_bytes(D, SRC), s>>>(p, reqs);
}

template <int D, int SRC, typename Reqs>
void launch_source(const AttnParams& p, const Reqs& reqs, hipStream_t s) {
  if constexpr (SRC != ATTN_ROWS) {
    if (p.launch[0].n_seg > 1 || p.launch[1].n_seg > 1) {
      launch_kernel<D, SRC, true>(p, reqs, s);
      for (const AttnLaunchView& l : p.launch)
        if (l.n_seg > 1)
          attention_merge_kernel<D, Reqs><<<(unsigned)l.state_rows * p.n_heads * p.group, 256, 0, s>>>(p, l, reqs);
      return;
    }
  }
  launch_kernel<D, SRC, false>(p, reqs, s);
}

template <int D, typename Reqs>
void launch_shape(const AttnParams& p, const Reqs& reqs, hipStream_t s) {
  if (p.source == ATTN_ROWS)
    launch_source<D, ATTN_ROWS>(p, reqs, s);
  else if (p.source == ATTN_F16)
    launch_source<D, ATTN_F16>(p, reqs, s);
  else if (p.source == ATTN_E4M3)
    launch_source<D, ATTN_E4M3>(p, reqs, s);
  else
    launch_source<D, ATTN_E2M1>(p, reqs, s);
}

template <int D, int SRC, bool kFew4, typename Reqs>
void launch_selected(const SelectParams& sp, const AttnParams& p, const Reqs& tokens, hipStream_t s) {
  const size_t at = std::max<size_t>(kFew4 ? 4 * few_wave_bytes(D) : lds_bytes(D, SRC), (select_bytes(sp, kSelectedWaves) + 15) & ~(size_t)15);
  attention_selected_kernel<D, SRC, kFew4, Reqs>
      <<<(unsigned)sp.n_tokens * sp.n_heads, 64 * kSelectedWaves, at + sp.n_select * sizeof(int32_t), s>>>(sp, p, tokens, (int)at);
}

template <typename Reqs>
hipError_t allow_lds_with() {  // (with the static words more than 64 KB)
  hipError_t e = hipSuccess;
  auto allow = [&](const void* kernel) {
    if (e == hipSuccess)
      e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes(128, ATTN_E4M3) + kMaxKeys * (int)sizeof(int32_t));
  };
  allow(reinterpret_cast<const void*>(&attention_kernel<128, ATTN_ROWS, false, Reqs>));
  allow(reinterpret_cast<const void*>(&attention_kernel<128, ATTN_F16, false, Reqs>));
  allow(reinterpret_cast<const void*>(&attention_kernel<128, ATTN_F16, true, Reqs>));
  allow(reinterpret_cast<const void*>(&attention_kernel<128, ATTN_E4M3, false, Reqs>));
  allow(reinterpret_cast<const void*>(&attention_kernel<128, ATTN_E4M3, true, Reqs>));
  allow(reinterpret_cast<const void*>(&attention_kernel<128, ATTN_E2M1, false, Reqs>));
  allow(reinterpret_cast<const void*>(&attention_kernel<128, ATTN_E2M1, true, Reqs>));
  allow(reinterpret_cast<const void*>(&attention_selected_kernel<128, ATTN_F16, false, Reqs>));
  allow(reinterpret_cast<const void*>(&attention_selected_kernel<128, ATTN_E4M3, false, Reqs>));
  allow(reinterpret_cast<const void*>(&attention_selected_kernel<128, ATTN_E2M1, false, Reqs>));
  return e;
}

}  // namespace

hipError_t attention_one_time_setup() {
  const hipError_t e = allow_lds_with<ChunkReqs>();
  return e == hipSuccess ? allow_lds_with<ChunkReqList>() : e;
}

hipError_t launch_selected_attention(const SelectParams& sp, const AttnParams& p, const ChunkReqs& inline_tokens, hipStream_t s) {
  if (sp.n_tokens == 0) return hipSuccess;
  if ((sp.head_dim != 64 && sp.head_dim != 128) || sp.part_blocks || sp.group > kFlatRows || sp.lds_keys < 1 || sp.lds_keys > kMaxKeys ||
      sp.n_select < 1 || sp.n_select > kMaxKeys || p.source == ATTN_ROWS)
    return hipErrorInvalidValue;
  auto with = [&](auto dim, const auto& tokens) {
    constexpr int D = decltype(dim)::value;
    if (p.source == ATTN_F16)
      launch_selected<D, ATTN_F16, false>(sp, p, tokens, s);
    else if (p.source == ATTN_E4M3)
      launch_selected<D, ATTN_E4M3, false>(sp, p, tokens, s);
    else if (sp.group <= kFewRows)
      launch_selected<D, ATTN_E2M1, true>(sp, p, tokens, s);
    else
      launch_selected<D, ATTN_E2M1, false>(sp, p, tokens, s);
  };
  auto with_tokens = [&](const auto& tokens) {
    if (sp.head_dim == 128)
      with(std::integral_constant<int, 128>(), tokens);
    else
      with(std::integral_constant<int, 64>(), tokens);
  };
  if (sp.tokens)
    with_tokens(ChunkReqList{sp.tokens});
  else
    with_tokens(inline_tokens);
  return hipGetLastError();
}

hipError_t launch_attention(const AttnParams& p, const ChunkReqs& inline_reqs, hipStream_t s) {
  if (p.head_dim != 64 && p.head_dim != 128) return hipErrorInvalidValue;
  for (const AttnLaunchView& l : p.launch)
    if (l.n_seg < 1 || l.n_seg > kMaxHeadSegments || l.seg_blocks < 1 || (p.source == ATTN_ROWS && l.n_seg > 1)) return hipErrorInvalidValue;
  if (p.launch[0].n_units + p.launch[1].n_units == 0) return hipSuccess;
  auto with = [&](const auto& reqs) {
    if (p.head_dim == 128)
      launch_shape<128>(p, reqs, s);
    else
      launch_shape<64>(p, reqs, s);
  };
  if (p.reqs)
    with(ChunkReqList{p.reqs});
  else
    with(inline_reqs);
  return hipGetLastError();
}

}  // namespace fc
