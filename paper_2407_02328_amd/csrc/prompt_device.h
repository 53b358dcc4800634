// What the kernels of attention over whole prompts share: tensors of sequences, tiles in LDS, operands of the matrix
// instructions, and the way from a workgroup to its (sequence, block, head).
//
// All products are 32x32x16 steps (bf16: one instruction; fp32: eight of 32x32x2, whose contraction takes the elements in another
// order, the same one on both sides).  Lane = 32 h + c holds, of an operand, row c and elements 8 h .. 8 h + 7 of the step's 16;
// of a result, column c and rows 8 (r / 4) + 4 h + r % 4, r = 0 .. 15.  A result turned into the next product's operand stays in
// its lane: elements e = 0 .. 7 of step t are its rows r = 8 t + e, and the other operand is read from LDS in that order
// (transposed()).
#pragma once

#include <type_traits>

#include "adore.h"
#include "device_utils.h"

namespace adore {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Rows of a tensor: token t of sequence b, head h starts at p + b seq + (first + t) token + h head (elements); first = start[b], or
// 0 without starts.
template <typename T>
struct Rows {
  T *p;
  int64_t seq, token, head;
};

template <typename T>
inline Rows<T> rows_of(const adore_rows *r) {
  return Rows<T>{static_cast<T *>(r->data), r->seq, r->token, r->head};
}

// A problem's sequences and heads.
struct PromptShape {
  const int32_t *q_start, *k_start;   // [batch + 1], or null: every sequence has q_tokens / k_tokens
  int batch, heads, kv_heads, group, q_tokens, k_tokens;
  float scale, scale_log2;            // and times log2(e)
};

int prompt_shape(const adore_prompt_config *c, const int32_t *q_start, const int32_t *k_start, PromptShape *s);
bool prompt_rows_ok(const adore_rows *r, int dtype);

struct Sequence {
  int b;
  int q_first, k_first;   // first rows in packed tensors (0 in dense ones)
  int nq, nk;
};

// Starts are the caller's device memory: whatever they hold, rows stay within the packed tensors.
__device__ __forceinline__ void span(const int32_t *start, int b, int total, int &first, int &n) {
  const int s = min(max(start[b], 0), total), e = min(max(start[b + 1], 0), total);
  first = s;
  n = max(e - s, 0);
}

__device__ __forceinline__ Sequence sequence_at(const PromptShape &a, int b) {
  Sequence s;
  s.b = b;
  s.q_first = s.k_first = 0;
  s.nq = a.q_tokens;
  s.nk = a.k_tokens;
  if (a.q_start) {
    span(a.q_start, b, a.q_tokens, s.q_first, s.nq);
    span(a.k_start, b, a.k_tokens, s.k_first, s.nk);
  }
  return s;
}

// Blocks of `rows` rows that sequences have together, at most (a grid does not know the starts), and the rows behind the last sequence.
inline long long blocks_at_most(const int32_t *start, int batch, int tokens, int rows) {
  return start ? (long long)tokens / rows + batch + 1 : (long long)batch * ((tokens + rows - 1) / rows);
}

// Block `item` of the sequences' blocks of ROWS rows (of q, or of k), one sequence behind the other.  False: none, and `block` is that
// much behind the last one (tail_rows).  All 64 lanes of a wave call it together.
template <int ROWS, bool OF_Q>
__device__ __forceinline__ bool find_block(const PromptShape &a, int item, Sequence &s, int &block) {
  const int32_t *start = OF_Q ? a.q_start : a.k_start;
  const int tokens = OF_Q ? a.q_tokens : a.k_tokens;
  if (!start) {
    const int per = (tokens + ROWS - 1) / ROWS, b = item / per;
    block = item - b * per;
    s = sequence_at(a, b);
    return true;
  }
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    int n = 0, first;
    if (b0 + lane < a.batch) span(start, b0 + lane, tokens, first, n);
    const int own = (n + ROWS - 1) / ROWS, upto = before + wave_scan(own);
    const uint64_t beyond = __builtin_amdgcn_ballot_w64(upto > item);
    if (beyond) {
      const int at = __builtin_ctzll(beyond);
      block = item - __builtin_amdgcn_readlane(upto - own, at);
      s = sequence_at(a, __builtin_amdgcn_readfirstlane(b0 + at));
      return true;
    }
    before = __builtin_amdgcn_readlane(upto, 63);
  }
  block = item - before;
  return false;
}

// Rows behind the last sequence that the workgroup of a block beyond the sequences' own sees to (it sets what is written there to zero).
template <int ROWS>
__device__ __forceinline__ int tail_rows(const int32_t *start, int batch, int tokens, int block, int &first) {
  const int64_t at = min(max(start[batch], 0), tokens) + int64_t(block) * ROWS;
  first = int(min(at, int64_t(tokens)));
  return min(ROWS, tokens - first);
}

template <typename T, int DH>
__device__ __forceinline__ void zero_rows(const Rows<T> &to, int head, int first, int n, int tid, int threads) {
  constexpr int kChunks = DH * int(sizeof(T)) / 16;
  for (int i = tid; i < n * kChunks; i += threads)
    *reinterpret_cast<u32x4 *>(reinterpret_cast<char *>(to.p + int64_t(first + i / kChunks) * to.token + head * to.head) + i % kChunks * 16) =
        u32x4{0, 0, 0, 0};
}

// Where fp32 values per row of a sequence and head are (lse, scores, ...): [heads][packed rows], or [batch][heads][tokens].
__device__ __forceinline__ size_t row_value(bool packed, int b, int first, int tokens, int heads, int h) {
  return packed ? size_t(h) * tokens + first : (size_t(b) * heads + h) * tokens;
}

// ---- matrix products ------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t pair_bf16(float a, float b) {   // rounded to nearest, ties to even
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

template <typename T>
struct Operand;
template <>
struct Operand<bf16_t> {
  typedef bf16x8 type;
  __device__ static __forceinline__ f32x16 mma(const type &a, const type &b, const f32x16 &c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
  // elements 8 t .. 8 t + 7 of a result, rounded to the storage type
  __device__ static __forceinline__ type of(const f32x16 &p, int t) {
    const u32x4 u = {pair_bf16(p[8 * t], p[8 * t + 1]), pair_bf16(p[8 * t + 2], p[8 * t + 3]), pair_bf16(p[8 * t + 4], p[8 * t + 5]),
                     pair_bf16(p[8 * t + 6], p[8 * t + 7])};
    return __builtin_bit_cast(type, u);
  }
  // ... and what that rounding left of them, rounded
  __device__ static __forceinline__ type rest_of(const f32x16 &p, const type &rounded, int t) {
    const u32x4 u = __builtin_bit_cast(u32x4, rounded);
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      v[i] = pair_bf16(p[8 * t + 2 * i] - __uint_as_float(u[i] << 16), p[8 * t + 2 * i + 1] - __uint_as_float(u[i] & 0xffff0000u));
    return __builtin_bit_cast(type, v);
  }
};
template <>
struct Operand<float> {
  typedef f32x8 type;
  __device__ static __forceinline__ f32x16 mma(const type &a, const type &b, f32x16 c) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
    return c;
  }
  __device__ static __forceinline__ type of(const f32x16 &p, int t) {
    return t == 0 ? __builtin_shufflevector(p, p, 0, 1, 2, 3, 4, 5, 6, 7) : __builtin_shufflevector(p, p, 8, 9, 10, 11, 12, 13, 14, 15);
  }
};

// ---- tiles in LDS -----------------------------------------------------------------------------------------------
// R rows of DH elements, in 16-byte chunks that are permuted within their row so that neither 8 rows x 1 chunk (an operand by rows) nor 4
// rows x 2 neighbouring chunks (transposed) meet in a bank.
template <typename T, int DH>
struct Tile {
  static constexpr int kRow = DH * int(sizeof(T));
  static constexpr int kChunks = kRow / 16;
  __device__ static __forceinline__ int chunk_at(int r, int ch) {
    if constexpr (sizeof(T) == 4) return r * kRow + ((ch ^ (r & 15)) << 4);
    const int x = (r & 3) << 1 | ((r >> 2) & 1);
    return DH == 128 ? r * kRow + ((ch ^ (x | (r & 8))) << 4) : r * kRow + ((ch ^ x) << 4);
  }
  // Row r, elements 16 t + 8 h .. + 7.
  __device__ static __forceinline__ typename Operand<T>::type by_row(const unsigned char *tile, int r, int t, int h) {
    if constexpr (sizeof(T) == 4) {
      const f32x4 lo = *reinterpret_cast<const f32x4 *>(tile + chunk_at(r, 4 * t + 2 * h));
      const f32x4 hi = *reinterpret_cast<const f32x4 *>(tile + chunk_at(r, 4 * t + 2 * h + 1));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      return *reinterpret_cast<const bf16x8 *>(tile + chunk_at(r, 2 * t + h));
    }
  }
  // Column 32 db + c, rows r0 + 16 t + 8 (e / 4) + 4 h + e % 4, e = 0 .. 7 (r0 a multiple of 32).
  __device__ static __forceinline__ typename Operand<T>::type transposed(const unsigned char *tile, int r0, int t, int db, int lane) {
    const int c = lane & 31, h = lane >> 5;
    if constexpr (sizeof(T) == 4) {
      f32x8 v;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int r = r0 + 16 * t + 8 * (e / 4) + 4 * h + e % 4;
        v[e] = *reinterpret_cast<const float *>(tile + chunk_at(r, (32 * db + c) >> 2) + (c & 3) * 4);
      }
      return v;
    } else {
      // 16 lanes read 4 rows x 16 columns, and each gets 4 rows of its column
      const int grp = lane >> 4, row = 4 * (grp >> 1) + ((lane & 15) >> 2), col = 32 * db + (grp & 1) * 16 + (lane & 3) * 4;
      union {
        s16x4 q[2];
        bf16x8 v;
      } u;
#pragma unroll
      for (int e4 = 0; e4 < 2; ++e4) {
        const int at = chunk_at(r0 + 16 * t + 8 * e4 + row, col >> 3) + (col & 4) * 2;
        u.q[e4] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(tile + at));
      }
      return u.v;
    }
  }
};

// A tile's way from memory to LDS: NT threads carry R rows of DH elements, 16 bytes at a time, in registers in between.
template <typename T, int DH, int R, int NT>
struct Carrier {
  typedef Tile<T, DH> L;
  static constexpr int N = R * L::kChunks / NT;
  static_assert(N * NT == R * L::kChunks, "whole chunks per thread");
  u32x4 r[N];
  // Rows first .. first + R - 1 of the row array at `base` (row stride in bytes); rows from `end` on read as row end - 1, or as zeros.
  template <bool ZEROS>
  __device__ __forceinline__ void load(const char *base, int64_t stride, int first, int end, int tid) {
    const char *at = base + int64_t(first) * stride;
    const int row = tid / L::kChunks, col = tid % L::kChunks * 16;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int mine = row + i * (NT / L::kChunks);
      const int there = min(mine, end - 1 - first);
      r[i] = *reinterpret_cast<const u32x4 *>(at + (uint32_t(there) * uint32_t(stride) + uint32_t(col)));
      if (ZEROS && mine != there) r[i] = u32x4{0, 0, 0, 0};
    }
  }
  __device__ __forceinline__ void store(unsigned char *tile, int tid) const {
    const int row = tid / L::kChunks, ch = tid % L::kChunks;
#pragma unroll
    for (int i = 0; i < N; ++i) *reinterpret_cast<u32x4 *>(tile + L::chunk_at(row + i * (NT / L::kChunks), ch)) = r[i];
  }
};

// The wave's transposed result o[db] (row = element 32 db + .., column = row c of 32) to the rows of `to`, through LDS of the wave's
// own (32 rows of DH elements), for whole 16-byte stores.  rest, if given, takes what rounding to bf16 left, rounded.
template <typename T, int DH>
__device__ __forceinline__ void store_rows(const f32x16 (&o)[DH / 32], float factor, unsigned char *own, char *to, int64_t stride, int rows,
                                           char *rest, int64_t rest_stride, int lane) {
  typedef Tile<T, DH> L;
  const int c = lane & 31, h = lane >> 5;
  auto pass = [&](char *dst, int64_t dst_stride, bool what_is_left) {
    wave_lds_fence();
#pragma unroll
    for (int db = 0; db < DH / 32; ++db)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = o[db][4 * j + i] * factor;
        const int e = 32 * db + 8 * j + 4 * h;      // four elements from here
        if constexpr (sizeof(T) == 4) {
          *reinterpret_cast<f32x4 *>(own + L::chunk_at(c, e / 4)) = f32x4{v[0], v[1], v[2], v[3]};
        } else {
          u32x2 u = {pair_bf16(v[0], v[1]), pair_bf16(v[2], v[3])};
          if (what_is_left)
            u = u32x2{pair_bf16(v[0] - __uint_as_float(u[0] << 16), v[1] - __uint_as_float(u[0] & 0xffff0000u)),
                      pair_bf16(v[2] - __uint_as_float(u[1] << 16), v[3] - __uint_as_float(u[1] & 0xffff0000u))};
          *reinterpret_cast<u32x2 *>(own + L::chunk_at(c, e / 8) + (e & 4) * 2) = u;
        }
      }
    wave_lds_fence();
#pragma unroll
    for (int i = 0; i < 32 * L::kChunks / 64; ++i) {
      const int at = i * 64 + lane, r = at / L::kChunks, ch = at % L::kChunks;
      const u32x4 v = *reinterpret_cast<const u32x4 *>(own + L::chunk_at(r, ch));
      if (r < rows) *reinterpret_cast<u32x4 *>(dst + int64_t(r) * dst_stride + ch * 16) = v;
    }
  };
  pass(to, stride, false);
  if constexpr (sizeof(T) == 2) {
    if (rest) pass(rest, rest_stride, true);
  }
}

}  // namespace adore
