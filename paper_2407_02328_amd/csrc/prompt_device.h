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
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

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

// Blocks of `rows` rows that sequences have together, at most (a grid does not know the starts), and the rows that belong to none.
inline long long blocks_at_most(const int32_t *start, int batch, int tokens, int rows) {
  return start ? (long long)tokens / rows + batch + 1 : (long long)batch * ((tokens + rows - 1) / rows);
}

// Block `item` of the sequences' blocks of ROWS rows of q (whose work grows with their index: they see all keys before them) or of k
// (whose work falls).  The order: one sequence behind the other, each with its longest block first, so that what
// one sequence's workgroups share stays in the L2; by_work: the longest of all sequences first, so that a launch of few workgroups
// ends with short ones.  False: there is no such block, and `block` is how far behind the last one (spare_rows).  All 64 lanes of a wave
// call it together.
template <int ROWS, bool OF_Q>
__device__ __forceinline__ bool find_block(const PromptShape &a, int item, bool by_work, Sequence &s, int &block) {
  const int32_t *start = OF_Q ? a.q_start : a.k_start;
  const int tokens = OF_Q ? a.q_tokens : a.k_tokens;
  if (!start) {
    const int per = (tokens + ROWS - 1) / ROWS, b = by_work ? item % a.batch : item / per, i = by_work ? item / a.batch : item - b * per;
    block = OF_Q ? per - 1 - i : i;
    s = sequence_at(a, b);
    return true;
  }
  const int lane = threadIdx.x & 63;
  auto blocks_at = [&](int b) {
    int n = 0, first;
    if (b < a.batch) span(start, b, tokens, first, n);
    return (n + ROWS - 1) / ROWS;
  };
  // by_work: the blocks with more than w in front of them (counted from the sequence's light end) are fewer than or as many as item
  int w = 0;
  if (by_work) {
    auto heavier = [&](int than) {
      int sum = 0;
      for (int b0 = 0; b0 < a.batch; b0 += 64) sum += __builtin_amdgcn_readlane(wave_scan(max(0, blocks_at(b0 + lane) - than)), 63);
      return sum;
    };
    const int all = heavier(0);
    if (item >= all) {
      block = item - all;
      return false;
    }
    int hi = (tokens + ROWS - 1) / ROWS;      // heavier(hi) = 0 <= item < heavier(w)
    while (hi - w > 1) {
      const int mid = (w + hi) >> 1;
      if (heavier(mid) <= item)
        hi = mid;
      else
        w = mid;
    }
    item -= heavier(hi);                      // among the sequences with hi blocks or more, one block each
    w = hi;
  }
  int before = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    const int n = blocks_at(b0 + lane), own = by_work ? (n >= w ? 1 : 0) : n, upto = before + wave_scan(own);
    const uint64_t beyond = __builtin_amdgcn_ballot_w64(upto > item);
    if (beyond) {
      const int at = __builtin_ctzll(beyond), blocks = __builtin_amdgcn_readlane(n, at);
      const int i = by_work ? blocks - w : item - __builtin_amdgcn_readlane(upto - own, at);
      block = OF_Q ? blocks - 1 - i : i;
      s = sequence_at(a, __builtin_amdgcn_readfirstlane(b0 + at));
      return true;
    }
    before = __builtin_amdgcn_readlane(upto, 63);
  }
  block = item - before;
  return false;
}

// Rows of packed tensors that belong to no sequence: those behind the last one, then those in front of the first.  The workgroup of a
// block beyond the sequences' own sees to ROWS of them, at(0) .. at(n - 1) (it sets what is written there to zero).
struct SpareRows {
  int end, behind, first, n;
  __device__ __forceinline__ int at(int i) const {
    const int r = first + i;
    return r < behind ? end + r : r - behind;
  }
};
template <int ROWS>
__device__ __forceinline__ SpareRows spare_rows(const int32_t *start, int batch, int tokens, int block) {
  SpareRows r;
  r.end = min(max(start[batch], 0), tokens);
  r.behind = tokens - r.end;
  const int all = r.behind + min(max(start[0], 0), r.end);
  r.first = int(min(int64_t(block) * ROWS, int64_t(all)));
  r.n = min(ROWS, all - r.first);
  return r;
}

template <typename T, int DH>
__device__ __forceinline__ void zero_rows(const Rows<T> &to, int head, const SpareRows &spare, int tid, int threads) {
  constexpr int kChunks = DH * int(sizeof(T)) / 16;
  for (int i = tid; i < spare.n * kChunks; i += threads)
    *reinterpret_cast<u32x4 *>(reinterpret_cast<char *>(to.p + int64_t(spare.at(i / kChunks)) * to.token + head * to.head) + i % kChunks * 16) =
        u32x4{0, 0, 0, 0};
}

// Where fp32 values per row of a sequence and head are (lse, scores, ...): [heads][packed rows], or [batch][heads][tokens].
__device__ __forceinline__ size_t row_value(bool packed, int b, int first, int tokens, int heads, int h) {
  return packed ? size_t(h) * tokens + first : (size_t(b) * heads + h) * tokens;
}

// Dynamic shared memory beyond what every kernel may have.
template <typename F>
inline hipError_t allow_lds(F *kernel, int bytes) {
  if (bytes <= 64 * 1024) return hipSuccess;
  return hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

// A kernel that is to have N waves a SIMD, no more: the compiler then uses the registers that leaves.
#define ADORE_WAVES(N) __attribute__((amdgpu_waves_per_eu(N, N)))
// What stands before it is issued before what stands behind it.
__device__ __forceinline__ void pin() { __builtin_amdgcn_sched_barrier(0); }

// A row's log-sum-exp as the subtrahend of exponents in base 2: +inf for a row that sees nothing, whose weights are then 0 and not NaN.
__device__ __forceinline__ float subtrahend(float lse) { return lse == -INFINITY ? INFINITY : lse * 1.4426950408889634f; }

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
// R rows of DH elements, in 16-byte chunks that are permuted within their row (an exclusive or with a number that goes by the row) so that
// what one cycle of LDS serves (256 bytes) does not meet in a bank: an operand's 16 rows at one chunk, and transposed 4 rows x 64 bytes
// (two bits of the row choose among four times 64 bytes, the next two within them; at 64 elements two rows share 256 bytes).
template <typename T, int DH>
struct Tile {
  static constexpr int kRow = DH * int(sizeof(T));
  static constexpr int kChunks = kRow / 16;
  static constexpr int kPeriod = sizeof(T) == 2 ? 16 : 8;
  __device__ static __forceinline__ int turn(int r) {
    if constexpr (sizeof(T) == 4) return r & 7;
    return DH == 128 ? (r & 3) << 2 | ((r >> 2) & 3) : (r & 2) << 1 | ((r >> 2) & 3);
  }
  __device__ static __forceinline__ int chunk_at(int r, int ch) { return r * kRow + ((ch ^ turn(r)) << 4); }
};

typedef const __attribute__((address_space(3))) char *LdsPtr;
__device__ __forceinline__ uint32_t lds_offset(const void *p) { return uint32_t(uintptr_t((LdsPtr)(const char *)p)); }
template <typename V>
__device__ __forceinline__ V lds_read(uint32_t at) {
  return *(const __attribute__((address_space(3))) V *)(LdsPtr)uintptr_t(at);
}

// A lane's operands out of tiles.  Everything that goes by the lane is in a few registers made once and moved from stage to stage;
// constant rows and steps are offsets of the instructions (an exclusive or per read would be a third of the vector instructions).
//   by_row(add, r0, t)          row r0 + c, elements 16 t + 8 h .. + 7
//   transposed(add, r0, t, db)  column 32 db + c, rows r0 + 16 t + 8 (e / 4) + 4 h + e % 4, e = 0 .. 7
// of the tile `add` bytes behind the place the reader is at; r0: a multiple of 32.
// FEW: a third of the registers, at an exclusive or a read (tiles then start at multiples of 256 bytes).
template <typename T, int DH, bool FEW = false>
struct Reader {
  typedef Tile<T, DH> L;
  typedef typename Operand<T>::type Frag;
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int NR = F32 ? 4 : FEW ? 1 : DH / 16, NC = F32 ? 4 : DH / 32 * (FEW ? 1 : 2);
  uint32_t row[NR], col[NC];
  __device__ __forceinline__ void move(uint32_t by) {
#pragma unroll
    for (int i = 0; i < NR; ++i) row[i] += by;
#pragma unroll
    for (int i = 0; i < NC; ++i) col[i] += by;
  }
  __device__ __forceinline__ Reader(uint32_t place, int lane) {
    const int c = lane & 31, h = lane >> 5;
    if constexpr (F32) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        row[i] = uint32_t(L::chunk_at(c, 4 * (i >> 1) + 2 * h + (i & 1)));
        col[i] = uint32_t(L::chunk_at(4 * h + i, c >> 2) + (c & 3) * 4);
      }
    } else {
#pragma unroll
      for (int i = 0; i < NR; ++i) row[i] = uint32_t(L::chunk_at(c, 2 * i + h));
      // 16 lanes read 4 rows x 16 columns, and each gets 4 rows of its column
      const int grp = lane >> 4, r = 4 * (grp >> 1) + ((lane & 15) >> 2), x = (grp & 1) * 16 + (lane & 3) * 4;
#pragma unroll
      for (int i = 0; i < NC; ++i) col[i] = uint32_t(L::chunk_at(r + i / (DH / 32) * 8, (32 * (i % (DH / 32)) + x) >> 3) + (x & 4) * 2);
    }
    move(place);
  }
  __device__ __forceinline__ Frag by_row(uint32_t ahead, int r0, int t) const {
    if constexpr (F32) {
      const uint32_t add = ahead + uint32_t(r0 * L::kRow + (t >> 1) * 128);
      const f32x4 lo = lds_read<f32x4>(row[2 * (t & 1)] + add), hi = lds_read<f32x4>(row[2 * (t & 1) + 1] + add);
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      // (step t is bits 1 .. 3 of the chunk, which the permutation turns over one by one)
      return lds_read<bf16x8>((FEW ? row[0] ^ uint32_t(t << 5) : row[FEW ? 0 : t]) + (ahead + uint32_t(r0 * L::kRow)));
    }
  }
  __device__ __forceinline__ Frag transposed(uint32_t ahead, int r0, int t, int db) const {
    if constexpr (F32) {
      f32x8 v;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = lds_read<float>(col[e & 3] + (ahead + uint32_t((r0 + 16 * t + 8 * (e >> 2)) * L::kRow + 128 * db)));
      return v;
    } else {
      union {
        s16x4 q[2];
        bf16x8 v;
      } u;
#pragma unroll
      for (int e4 = 0; e4 < 2; ++e4) {       // (rows 8 further on: another bit of the permutation)
        const uint32_t at = FEW ? (col[db] ^ uint32_t(e4 << 5)) + (ahead + uint32_t((r0 + 16 * t + 8 * e4) * L::kRow))
                                : col[FEW ? 0 : e4 * (DH / 32) + db] + (ahead + uint32_t((r0 + 16 * t) * L::kRow));
        u.q[e4] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(LdsPtr)uintptr_t(at));
      }
      return u.v;
    }
  }
};

// ---- hidden rows that are not finite ----
// A weight of 0 hides a row from a matrix product only where the row is finite.  Rows that some of a workgroup's columns see and others do
// not are all in its few tiles on the diagonal.  Of V, infinities and NaN become 0 there, and when all tiles are done every column takes
// those that it does see (add_not_finite), from memory.  K makes the weights too, so that a tile of it is left as it is: where any is found
// (find_not_finite), the keys from there on are gone over one by one.

// 16 bytes, one of whose elements is an infinity or NaN.
template <typename T>
__device__ __forceinline__ bool chunk_not_finite(const u32x4 &w) {
  constexpr uint32_t kSize = sizeof(T) == 2 ? 0x7fff7fffu : 0x7fffffffu;
  if constexpr (sizeof(T) == 2) {
    u16x2 most = {0, 0};
#pragma unroll
    for (int j = 0; j < 4; ++j) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, w[j] & kSize));
    return most[0] >= 0x7f80 || most[1] >= 0x7f80;
  } else {
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) most = max(most, w[j] & kSize);
    return most >= 0x7f800000u;
  }
}

// The workgroup's tile of R rows; whether this wave found any.  Barriers before and behind are the caller's.
template <typename T, int DH, int R, int NT>
__device__ __forceinline__ bool make_finite(unsigned char *tile) {
  constexpr int N = R * Tile<T, DH>::kChunks / NT;
  static_assert(N * NT == R * Tile<T, DH>::kChunks, "as many chunks for every thread");
  int tid = threadIdx.x;
  asm("" : "+v"(tid));   // (worked out here, not kept in registers)
  u32x4 *const chunk = reinterpret_cast<u32x4 *>(tile) + tid;
  bool found = false;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    u32x4 w = chunk[i * NT];
    if (chunk_not_finite<T>(w)) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if ((w[j] & 0x7f800000u) == 0x7f800000u) w[j] &= sizeof(T) == 2 ? 0xffffu : 0u;
        if (sizeof(T) == 2 && (w[j] & 0x7f80u) == 0x7f80u) w[j] &= 0xffff0000u;
      }
      chunk[i * NT] = w;
      found = true;
    }
  }
  return __builtin_amdgcn_ballot_w64(found) != 0;
}

// ... only looked at.
template <typename T, int DH, int R, int NT>
__device__ __forceinline__ bool find_not_finite(const unsigned char *tile) {
  constexpr int N = R * Tile<T, DH>::kChunks / NT;
  static_assert(N * NT == R * Tile<T, DH>::kChunks, "as many chunks for every thread");
  int tid = threadIdx.x;
  asm("" : "+v"(tid));
  const u32x4 *const chunk = reinterpret_cast<const u32x4 *>(tile) + tid;
  bool found = false;
#pragma unroll
  for (int i = 0; i < N; ++i) found |= chunk_not_finite<T>(chunk[i * NT]);
  return __builtin_amdgcn_ballot_w64(found) != 0;
}

// ---- waves that share rows ----
// Where blocks of 128 rows are too few to fill the chip, a workgroup takes fewer rows and SW of its four waves the same 32: each a part of
// what those rows go over, 32 of a tile's 32 SW.  At the end the first of them adds up the others' sums.  Four times the workgroups, of which
// a unit has room for one (two stages of wide tiles), and none waits four times as long as it must for the longest row.  Both sides
// (128-row blocks / shared rows, us; heads x tokens, bf16 at 128 elements unless said):
//   forward  16 x 300 11.0 / 10.9, 32 x 512 15.6 / 20.0, 8 x 2048 40.7 / 32.5, 12 x 2048 41.4 / 50.3, 2 x 8000 135 / 89, 3 x 8000 140 / 137,
//            4 x 8000 140 / 167, one query of 32 heads behind 4096 keys 72 / 45; fp32 64 elements: 4 x 128 15.0 / 9.0, 64 x 512 45.6 / 46.8,
//            16 x 2048 159 / 111; fp32: 64 x 512 79 / 58
//   dq       as the forward: 16 x 300 13.7 / 13.1, 32 x 512 19.0 / 24.3, 8 x 2048 50.4 / 39.4, 12 x 2048 52.6 / 62.1
//   dk, dv   16 x 300 18.9 / 16.9, 32 x 512 28.9 / 32.8, 8 x 2048 90 / 55, 16 x 2048 108 / 110, 8 of 2 kv heads x 8000 1341 / 548, 4 x 8000
//            381 / 301, 8 kv heads x 2560 behind 512 queries 94 / 120; fp32 64 elements: 4 x 128 23.8 / 12.0, 64 x 512 85 / 79
//   scores   16 x 300 8.5 / 6.0, 64 x 512 12.3 / 12.0, 16 x 2048 36 / 24, 8 of 2 kv heads x 8000 490 / 216; 264 blocks behind 64 queries 9.2 / 17.6
// (fp32 tiles are a quarter as fast and one workgroup of theirs fills a unit either way.)
inline long long length_of(const int32_t *start, int batch, int tokens) { return start ? tokens / batch : tokens; }   // on average
template <typename T>
inline bool share_queries(const PromptShape &s) {
  const int most = sizeof(T) == 4 ? 256 : length_of(s.q_start, s.batch, s.q_tokens) >= 2048 ? 128 : 64;
  return blocks_at_most(s.q_start, s.batch, s.q_tokens, 128) * s.heads <= most;
}
inline long long key_blocks(const PromptShape &s) { return blocks_at_most(s.k_start, s.batch, s.k_tokens, 128) * s.kv_heads; }
template <typename T>
inline bool share_keys(const PromptShape &s) {          // of dk and dv
  const long long queries = length_of(s.q_start, s.batch, s.q_tokens) * s.group;
  return key_blocks(s) <= (sizeof(T) == 4 || queries >= 4096 ? 256 : queries >= 2048 ? 128 : 64);
}
inline bool share_scored_keys(const PromptShape &s) { return key_blocks(s) <= 256; }

template <int SW>
struct Shared {
  static constexpr int kRowWaves = 4 / SW, kRows = 32 * kRowWaves;
  int rows, part;                             // the wave's rows of the workgroup's, its part
  __device__ __forceinline__ explicit Shared(int wave) : rows(wave % kRowWaves), part(wave / kRowWaves) {}
};
// A part's sums, as registers of 64 lanes, to and from LDS.
template <int DB>
__device__ __forceinline__ void put_sums(const f32x16 (&o)[DB], float *to, int lane) {
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) to[(16 * db + r) * 64 + lane] = o[db][r];
}
template <int DB>
__device__ __forceinline__ void add_sums(f32x16 (&o)[DB], const float *from, float factor, int lane) {
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[db][r] = fmaf(from[(16 * db + r) * 64 + lane], factor, o[db][r]);
}

// Whether it holds in any of the workgroup's four waves; s: four words that nothing else uses until the next barrier behind this one.
__device__ __forceinline__ bool any_of_four(bool mine, int *s) {
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = mine;
  __syncthreads();
  return (s[0] | s[1] | s[2] | s[3]) != 0;
}

// acc (element 32 db + .., column c) += what is not finite of rows from .. to - 1 at `rows`, up to the last that the lane's column sees.
template <typename T, int DH>
__device__ __forceinline__ void add_not_finite(f32x16 (&acc)[DH / 32], const char *rows, int64_t stride, int from, int to, int seen, int lane) {
#pragma unroll 1
  for (int i = from; i < to; ++i) {
    if (i > seen) continue;
    const T *row = reinterpret_cast<const T *>(rows + i * stride) + 4 * (lane >> 5);
#pragma unroll
    for (int db = 0; db < DH / 32; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float x = to_float(row[32 * db + 8 * (r >> 2) + (r & 3)]);
        acc[db][r] += fabsf(x) < INFINITY ? 0.f : x;
        if (r % 4 == 3) pin();
      }
  }
}

// 32 rows' way from memory to the wave's own LDS, 16 bytes at a time; rows from `rows` on are zeros.
template <typename T, int DH>
__device__ __forceinline__ void carry_rows(const char *base, int64_t stride, int rows, unsigned char *own, int lane) {
  typedef Tile<T, DH> L;
  constexpr int N = 32 * L::kChunks / 64;
  const int row = lane / L::kChunks, ch = lane % L::kChunks;
  u32x4 r[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int mine = row + i * (64 / L::kChunks);
    r[i] = *reinterpret_cast<const u32x4 *>(base + int64_t(min(mine, rows - 1)) * stride + ch * 16);
    if (mine >= rows) r[i] = u32x4{0, 0, 0, 0};
  }
#pragma unroll
  for (int i = 0; i < N; ++i) *reinterpret_cast<u32x4 *>(own + L::chunk_at(row + i * (64 / L::kChunks), ch)) = r[i];
}

// 32 rows from `base` (zeros from `rows` on) as an operand, through the wave's own LDS, `ahead` of the reader.
template <typename T, int DH, bool FEW>
__device__ __forceinline__ void operand_rows(typename Operand<T>::type (&f)[DH / 16], const Reader<T, DH, FEW> &read, const char *base,
                                             int64_t stride, int rows, unsigned char *own, uint32_t ahead, int lane) {
  wave_lds_fence();
  if (rows > 0) carry_rows<T, DH>(base, stride, rows, own, lane);
  wave_lds_fence();
#pragma unroll
  for (int t = 0; t < DH / 16; ++t) f[t] = read.by_row(ahead, 0, t);
}

// A tile's way from memory straight to LDS (no registers): R rows of DH elements, NT threads.  A wave's load fills 1 KB of LDS in lane
// order, so the lanes read the chunks that the tile's permutation wants there.  Rows from `end` on read as row end - 1.
// `arrived()` behind the loads and ahead of the barrier that hands the tile over: what the compiler does not count.
template <typename T, int DH, int R, int NT>
struct TileLoad {
  typedef Tile<T, DH> L;
  static constexpr int kPer = NT / L::kChunks, N = R / kPer;    // rows of a load of the workgroup's
  static_assert(N * kPer == R && kPer % L::kPeriod == 0, "a thread's chunk has the same place in all of its rows");
  uint32_t at, pitch;        // bytes from the tile's first row to the thread's chunk, from row to row
  int64_t step;              // bytes from one load of the workgroup's to the next
  __device__ __forceinline__ TileLoad(int64_t stride, int tid) : pitch(uint32_t(stride)), step(stride * kPer) {
    at = uint32_t(tid / L::kChunks) * pitch + col_of(tid);
  }
  __device__ static __forceinline__ uint32_t col_of(int tid) { return uint32_t(((tid % L::kChunks) ^ L::turn(tid / L::kChunks)) << 4); }
  // p: the tile's first row; left: rows from there on, at least one; lds: the tile's byte offset in LDS plus the wave's share of a
  // load (wave * 1024)
  __device__ __forceinline__ void operator()(const char *p, int left, uint32_t lds) const {
    if (left >= R) {
#pragma unroll
      for (int i = 0; i < N; ++i, p += step) to_lds(p, at, lds + uint32_t(i * NT * 16));
    } else {
      int tid = threadIdx.x;
      asm("" : "+v"(tid));   // what only a sequence's last tile needs is worked out there, not kept in registers
      const int row = tid / L::kChunks;
#pragma unroll
      for (int i = 0; i < N; ++i) to_lds(p, uint32_t(min(row + i * kPer, left - 1)) * pitch + col_of(tid), lds + uint32_t(i * NT * 16));
    }
  }
  // (As a builtin, the compiler would wait for the load ahead of every LDS read.  It does not look into the block for what the
  // hardware wants between a scalar write of m0 and a load that goes by it: one wait state.  m0 is a register that the compiler
  // never gives out, which it warns of where it is named as overwritten.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
  __device__ static __forceinline__ void to_lds(const char *base, uint32_t off, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory", "m0");
  }
#pragma clang diagnostic pop
};
__device__ __forceinline__ void arrived() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
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
