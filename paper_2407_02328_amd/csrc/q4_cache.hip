// A K/V cache held in 4 bits, evicted by the attention its rows received (paper Sec. 3.1, baseline 6), and single-query attention over
// it (Sec. 2.1, Eq. 1, with grouped heads).
//
// Format: 32 neighbouring elements of a row share a power of two, an element is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6.  gfx950
// turns two of them into bf16, times their power of two, in one instruction, exactly; that is what makes reading 68 bytes per element
// of 64 slots instead of 256 worth while, where shifts and multiplications on 4-bit integers (2 to 3 instructions an element) would
// take longer than the memory.  The power puts the block's largest element into [3.5, 7] of its units: with one step lower from 6
// on instead of 7 the error of Gaussian rows is 11.5 % and not 11.2 %.
//
// Layout of a row's (sequence x kv head) blocks of 64 slots, 68 d bytes each, one behind the other: what a wave needs of a block sits in
// its lanes without an exchange.  Matrix instructions are 16x16x32: lane = 16 quarter + c.
//   K codes   row 16 t + c (32 codes a group of 16 bytes) holds slot 4 c + t: tile t = 0 .. 3 is 16 consecutive rows, a wave's load of
//             it 1 KB in a run (d = 128), and a lane's codes are one scale's
//   V codes   [element][slot]: a lane's 16 slots of an element are 8 bytes, the order in which the weights of tiles 0 .. 3 come out
//             of the first product (row 4 quarter + r of tile t is slot 16 quarter + 4 r + t)
//   scales    K, then V: [group][slot], exponent + 127
#include <hip/hip_runtime.h>

#include <cmath>

#include "prompt_device.h"

namespace adore {

namespace {

constexpr int kSlots = 64;           // slots of a block
constexpr int kMaxQ4Slots = 1 << 20;
constexpr float kLog2e = 1.4426950408889634f;

__host__ __device__ constexpr int blocks_of(int slots) { return (slots + kSlots - 1) / kSlots; }
template <int DH>
struct Block {
  static constexpr int kV = 32 * DH, kKScale = 64 * DH, kVScale = 66 * DH, kBytes = 68 * DH, kGroups = DH / 32;
};

__device__ __forceinline__ float power(uint32_t scale) { return __uint_as_float(scale << 23); }

// Exponent + 127 of a group whose largest magnitude is `big` (not NaN): big / 2^e in (3.5, 7] (large enough that codes stay normal
// numbers, small enough that 6 units are finite).
__device__ __forceinline__ uint32_t scale_of(float big) {
  const int s = int((__float_as_uint(big) + 0x1fffffu) >> 23) - 2;
  return uint32_t(min(max(s, 27), 252));
}
// Codes of eight values, the first in the lowest 4 bits.
__device__ __forceinline__ uint32_t codes_of(const float *x, float unit) {
  uint32_t u = 0;
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[0], x[1], unit, 0);
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[2], x[3], unit, 1);
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[4], x[5], unit, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[6], x[7], unit, 3);
}
// ... and back.
__device__ __forceinline__ void values_of(uint32_t u, float unit, float *x) {
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(u, unit, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(u, unit, 1);
  const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(u, unit, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(u, unit, 3);
  x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1]; x[4] = c[0]; x[5] = c[1]; x[6] = d[0]; x[7] = d[1];
}
__device__ __forceinline__ bf16x8 operand_of(uint32_t u, float unit) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, unit, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, unit, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, unit, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, unit, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ float number(float x) { return x == x ? x : 0.f; }   // a NaN is held as 0

// Order-preserving image of a score; a NaN counts as 0, -0 is 0.
__device__ __forceinline__ uint32_t score_image(float x) {
  const uint32_t b = __float_as_uint(number(x) + 0.f);
  return b ^ (uint32_t(int32_t(b) >> 31) | 0x80000000u);
}

struct Q4Shape {
  int batch, heads, kv_heads, group, slots, blocks, recent;
  float scale_log2;
};

__device__ __forceinline__ uint64_t min_key(uint64_t a, uint64_t b) { return a < b ? a : b; }
__device__ __forceinline__ uint32_t wave_min(uint32_t x) {
  // a lane's neighbours come with the instruction (the row before where there is one, else itself); lane 63 has the result
  auto take = [&](uint32_t y) { x = x < y ? x : y; };
  take(uint32_t(__builtin_amdgcn_update_dpp(int(x), int(x), 0x111, 0xf, 0xf, false)));   // row_shr:1, 2, 4, 8
  take(uint32_t(__builtin_amdgcn_update_dpp(int(x), int(x), 0x112, 0xf, 0xf, false)));
  take(uint32_t(__builtin_amdgcn_update_dpp(int(x), int(x), 0x114, 0xf, 0xf, false)));
  take(uint32_t(__builtin_amdgcn_update_dpp(int(x), int(x), 0x118, 0xf, 0xf, false)));
  take(uint32_t(__builtin_amdgcn_update_dpp(int(x), int(x), 0x142, 0xa, 0xf, false)));   // row_bcast:15 into rows 1 and 3
  take(uint32_t(__builtin_amdgcn_update_dpp(int(x), int(x), 0x143, 0xc, 0xf, false)));   // row_bcast:31 into rows 2 and 3
  return uint32_t(__builtin_amdgcn_readlane(int(x), 63));
}
// Smallest key of the workgroup, in thread 0 (at least); s: one word per wave.  All threads call it.
__device__ __forceinline__ uint64_t workgroup_min(uint64_t key, uint64_t *s) {
  const uint32_t high = wave_min(uint32_t(key >> 32)), low = wave_min(uint32_t(key >> 32) == high ? uint32_t(key) : ~0u);
  key = uint64_t(high) << 32 | low;
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = key;
  __syncthreads();
  if (threadIdx.x == 0)
    for (unsigned w = 1; w < (blockDim.x + 63) / 64; ++w) key = min_key(key, s[w]);
  return key;
}

// ---- which tokens of the prompts stay ----------------------------------------------------------------------------
// A workgroup per row.  Of the tokens before the `recent` last ones the n - K with the lowest scores go, equal scores the lower position
// first: the score with that rank is found by four counts over 8 bits each, then one pass in position order gives the rest their slots.
// 512 rows of 1024 tokens 10 us.
constexpr int kFillThreads = 1024;

struct ChooseArgs {
  Q4Shape s;
  const int32_t *k_start;
  int k_tokens;
  const float *scores;     // or null: all equal
  int32_t *slot_pos;
  float *score;
  int32_t *cursor;
};

__global__ __launch_bounds__(kFillThreads) void q4_choose_kernel(const ChooseArgs a) {
  __shared__ uint32_t s_hist[256];
  __shared__ uint32_t s_pick[2];             // the bin, and the rank within it
  __shared__ int s_wave[2][kFillThreads / 64];
  __shared__ uint64_t s_key[kFillThreads / 64];
  const int row = blockIdx.x, b = row / a.s.kv_heads, hk = row % a.s.kv_heads, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int first = 0, n = a.k_tokens;
  if (a.k_start) span(a.k_start, b, a.k_tokens, first, n);
  const int K = a.s.slots;
  const float *sc = a.scores ? a.scores + row_value(a.k_start != nullptr, b, first, a.k_tokens, a.s.kv_heads, hk) : nullptr;
  int32_t *pos = a.slot_pos + size_t(row) * K;
  float *held = a.score + size_t(row) * K;
  const int old = max(0, n - a.s.recent), gone = max(0, n - K);      // gone <= old: recent < K
  // the image of the last score that goes (prefix), and how many of the tokens that have it go (ties)
  uint32_t prefix = 0;
  int ties = gone;
  if (gone > 0 && sc) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) s_hist[tid] = 0;
      __syncthreads();
      for (int i = tid; i < old; i += kFillThreads) {
        const uint32_t u = score_image(sc[i]);
        if (shift == 24 || (u ^ prefix) >> (shift + 8) == 0) atomicAdd(&s_hist[u >> shift & 255], 1u);
      }
      __syncthreads();
      if (wave == 0) {                        // the bin in which rank `ties` falls, from below: lane l owns bins 4 l .. 4 l + 3
        const int c0 = s_hist[4 * lane], c1 = s_hist[4 * lane + 1], c2 = s_hist[4 * lane + 2], c3 = s_hist[4 * lane + 3];
        const int own = c0 + c1 + c2 + c3, before = wave_scan(own) - own;
        if (before < ties && ties <= before + own) {
          int bin = 4 * lane, rest = ties - before;
          if (rest > c0) { rest -= c0; ++bin;
            if (rest > c1) { rest -= c1; ++bin;
              if (rest > c2) { rest -= c2; ++bin; } } }
          s_pick[0] = bin;
          s_pick[1] = rest;
        }
      }
      __syncthreads();
      prefix |= s_pick[0] << shift;
      ties = int(s_pick[1]);
      __syncthreads();
    }
  } else if (gone > 0) {
    prefix = score_image(0.f);
  }
  // in position order: kept tokens and tied ones before this one
  int kept = 0, tied = 0;
  uint64_t least = ~uint64_t(0);
  for (int i0 = 0; i0 < n; i0 += kFillThreads) {
    const int i = i0 + tid;
    const float x = i < n && sc ? sc[i] : 0.f;
    const uint32_t u = score_image(x);
    const bool is_old = i < old, tie = gone > 0 && is_old && u == prefix;
    const uint64_t tie_lanes = __builtin_amdgcn_ballot_w64(tie);
    if (lane == 0) s_wave[0][wave] = __popcll(tie_lanes);
    __syncthreads();
    int ties_before = tied;
    for (int w = 0; w < kFillThreads / 64; ++w) {
      const int c = s_wave[0][w];
      if (w < wave) ties_before += c;
      tied += c;
    }
    ties_before += __popcll(tie_lanes & ((uint64_t(1) << lane) - 1));
    const bool stays = i < n && !(gone > 0 && is_old && (u < prefix || (tie && ties_before < ties)));
    const uint64_t stay_lanes = __builtin_amdgcn_ballot_w64(stays);
    if (lane == 0) s_wave[1][wave] = __popcll(stay_lanes);
    __syncthreads();
    int slot = kept;
    for (int w = 0; w < kFillThreads / 64; ++w) {
      const int c = s_wave[1][w];
      if (w < wave) slot += c;
      kept += c;
    }
    slot += __popcll(stay_lanes & ((uint64_t(1) << lane) - 1));
    if (stays && slot < K) {
      pos[slot] = i;
      held[slot] = x;
      if (is_old) least = min_key(least, uint64_t(u) << 32 | uint32_t(slot));
    }
  }
  for (int i = min(n, K) + tid; i < K; i += kFillThreads) {
    pos[i] = -1;
    held[i] = 0.f;
  }
  least = workgroup_min(least, s_key);
  if (tid == 0) {
    a.cursor[2 * row] = n < K ? n : int(uint32_t(least));
    a.cursor[2 * row + 1] = n;
  }
}

// ---- the rows of the chosen tokens into the cache -------------------------------------------------------------------
// A workgroup per block; a thread quantises groups of 32 elements.  V goes through LDS to its [element][slot] order.
// Bound by memory: 16 x 32 rows of 512 slots, 134 MB of bf16 in and 36 MB out, 33 us (5.1 TB/s); read back 29 us (5.9).
template <typename T>
struct PackArgs {
  Q4Shape s;
  const int32_t *k_start, *slot_pos;
  int k_tokens;
  Rows<const T> k, v;
  unsigned char *cache;
};

template <typename T, int DH>
__global__ __launch_bounds__(256) void q4_pack_kernel(const PackArgs<T> a) {
  typedef Block<DH> L;
  constexpr int G = L::kGroups, EPL = Vec16<T>::EPL;
  __shared__ __align__(16) unsigned char s_code[kSlots][DH + 16];       // a code per byte
  const int row = blockIdx.x / a.s.blocks, block = blockIdx.x % a.s.blocks, b = row / a.s.kv_heads, hk = row % a.s.kv_heads, tid = threadIdx.x;
  int first = 0, n = a.k_tokens;
  if (a.k_start) span(a.k_start, b, a.k_tokens, first, n);
  unsigned char *out = a.cache + (size_t(row) * a.s.blocks + block) * L::kBytes;
  auto quantised = [&](const Rows<const T> &from, int slot, int g, uint32_t (&code)[4]) {
    float x[32];
    const int at = block * kSlots + slot, pos = at < a.s.slots ? a.slot_pos[size_t(row) * a.s.slots + at] : -1;
    float big = 0.f;
    if (pos >= 0 && pos < n) {
      const T *src = from.p + b * from.seq + (int64_t(first) + pos) * from.token + hk * from.head + 32 * g;
#pragma unroll
      for (int i = 0; i < 32 / EPL; ++i) {
        float y[EPL];
        Vec16<T>::load(src + i * EPL, y);
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
          x[i * EPL + e] = number(y[e]);
          big = fmaxf(big, fabsf(x[i * EPL + e]));
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 32; ++i) x[i] = 0.f;
    }
    const uint32_t scale = scale_of(big);
#pragma unroll
    for (int i = 0; i < 4; ++i) code[i] = codes_of(x + 8 * i, power(scale));
    return scale;
  };
  for (int i = tid; i < kSlots * G; i += 256) {
    const int slot = i / G, g = i % G;
    uint32_t c[4];
    const uint32_t scale = quantised(a.k, slot, g, c);
    *reinterpret_cast<u32x4 *>(out + ((slot & 3) * 16 + (slot >> 2)) * (DH / 2) + g * 16) = u32x4{c[0], c[1], c[2], c[3]};
    out[L::kKScale + g * kSlots + slot] = uint8_t(scale);
  }
  for (int i = tid; i < kSlots * G; i += 256) {
    const int slot = i / G, g = i % G;
    uint32_t c[4];
    const uint32_t scale = quantised(a.v, slot, g, c);
    out[L::kVScale + g * kSlots + slot] = uint8_t(scale);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      // nibbles to bytes, four at a time
      const uint32_t lo = c[w] & 0xffffu, hi = c[w] >> 16;
      auto spread = [](uint32_t u) {
        u = (u | u << 8) & 0x00ff00ffu;
        return (u | u << 4) & 0x0f0f0f0fu;
      };
      *reinterpret_cast<u32x2 *>(&s_code[slot][32 * g + 8 * w]) = u32x2{spread(lo), spread(hi)};
    }
  }
  __syncthreads();
  for (int i = tid; i < DH * 4; i += 256) {           // 16 slots of an element: 8 bytes
    const int e = i % DH, q = i / DH;
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < 16; ++j) w[j >> 3] |= uint32_t(s_code[16 * q + j][e]) << (4 * (j & 7));
    *reinterpret_cast<u32x2 *>(out + L::kV + e * 32 + q * 8) = u32x2{w[0], w[1]};
  }
}

// ---- what the cache holds, in the storage type (zeros in free slots) ----
template <typename T>
struct ReadArgs {
  Q4Shape s;
  const unsigned char *cache;
  const int32_t *slot_pos;
  T *k, *v;                // [batch][kv_heads][slots][DH]
};

template <typename T, int DH>
__global__ __launch_bounds__(256) void q4_read_kernel(const ReadArgs<T> a) {
  typedef Block<DH> L;
  constexpr int EPL = Vec16<T>::EPL;
  __shared__ __align__(16) uint32_t s_v[DH][9];                          // 32 bytes an element, and a word that spreads the banks
  const int row = blockIdx.x / a.s.blocks, block = blockIdx.x % a.s.blocks, tid = threadIdx.x;
  const unsigned char *in = a.cache + (size_t(row) * a.s.blocks + block) * L::kBytes;
  for (int i = tid; i < DH * 2; i += 256) {
    const u32x4 u = *reinterpret_cast<const u32x4 *>(in + L::kV + i * 16);
#pragma unroll
    for (int j = 0; j < 4; ++j) s_v[i >> 1][(i & 1) * 4 + j] = u[j];
  }
  __syncthreads();
  // eight elements a thread: whole lines
  auto put = [&](T *to, uint32_t c, float unit) {
    float x[8];
    values_of(c, unit, x);
#pragma unroll
    for (int i = 0; i < 8 / EPL; ++i) {
      typename Vec16<T>::Raw r;
      T *e = reinterpret_cast<T *>(&r);
#pragma unroll
      for (int j = 0; j < EPL; ++j) store_elem(e + j, x[i * EPL + j]);
      Vec16<T>::store_raw(to + i * EPL, r);
    }
  };
  for (int i = tid; i < kSlots * (DH / 8); i += 256) {
    const int slot = i / (DH / 8), part = i % (DH / 8), g = part / 4, at = block * kSlots + slot;
    if (at >= a.s.slots) continue;
    const bool there = a.slot_pos[size_t(row) * a.s.slots + at] >= 0;
    const size_t to = (size_t(row) * a.s.slots + at) * DH + 8 * part;
    const uint32_t kc = *reinterpret_cast<const uint32_t *>(in + ((slot & 3) * 16 + (slot >> 2)) * (DH / 2) + part * 4);
    uint32_t vc = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) vc |= (s_v[8 * part + j][slot >> 3] >> (4 * (slot & 7)) & 15u) << (4 * j);
    put(a.k + to, there ? kc : 0u, there ? power(in[L::kKScale + g * kSlots + slot]) : 1.f);
    put(a.v + to, there ? vc : 0u, there ? power(in[L::kVScale + g * kSlots + slot]) : 1.f);
  }
}

// ---- a token through the cache ----------------------------------------------------------------------------------------
template <typename T>
struct StepArgs {
  Q4Shape s;
  const T *q, *k_new, *v_new;      // [batch][heads][DH], [batch][kv_heads][DH]
  unsigned char *cache;
  int32_t *slot_pos, *cursor;
  float *score;
  T *out, *k_held, *v_held;        // the latter two or null
  int splits, passes;              // workgroups that share a row's blocks, and passes over its heads (16 at a time at most)
  int extra;                       // 1: a wave of its own for the new token
  float *part_o;                   // several workgroups a row: [row][pass][split][16][DH] unscaled sums,
  float *part_ml;                  // [row][pass][split][16][2] their maximum and sum,
  float *logit;                    // [row][group][64 blocks] the weights' exponents,
  float *part_new;                 // [row][group] the new token's,
  uint64_t *part_key;              // [row][finishing workgroup] and the row's counter
  int32_t *arrived;
};

constexpr int kPassHeads = 16;     // heads of a pass
constexpr int kFinishThreads = 1024;   // of a finishing workgroup, each with 1, 2 or 4 slots

// The token's place and position.  Whatever the cursor holds, the slot is one of the row's.
__device__ __forceinline__ void cursor_of(const int32_t *cursor, int row, int slots, int &slot, int &n) {
  slot = min(max(cursor[2 * row], 0), slots - 1);
  n = cursor[2 * row + 1];
}

// Key of the slot that the next token would rather take: a free one, then the lowest score (equal scores: the lowest slot), never one
// of the `recent` last tokens.
__device__ __forceinline__ uint64_t eviction_key(int pos, float score, int slot, int tokens, int recent) {
  if (pos < 0) return uint32_t(slot);
  return pos >= tokens - recent ? ~uint64_t(0) : uint64_t(score_image(score)) << 32 | uint32_t(slot);
}

// Three bf16 terms of an fp32 value are exact, two leave 2^-16 of it.
template <typename T>
constexpr int kQTerms = sizeof(T) == 2 ? 1 : 3;
template <typename T>
constexpr int kPTerms = sizeof(T) == 2 ? 2 : 3;

template <int N>
__device__ __forceinline__ void terms_of(float (&x)[8], bf16x8 (&t)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    u32x4 u;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      u[e] = pair_bf16(x[2 * e], x[2 * e + 1]);
      if (i + 1 < N) {
        x[2 * e] -= __uint_as_float(u[e] << 16);
        x[2 * e + 1] -= __uint_as_float(u[e] & 0xffff0000u);
      }
    }
    t[i] = __builtin_bit_cast(bf16x8, u);
  }
}

// Reads every code once: 16 sequences, 32 heads, 512 slots 13.5 us (one launch, 2.8 TB/s), 4 sequences, 32 heads over 8, 16384 slots 19 us (4.0 TB/s)
// and 8 for the second launch, one row of 64 slots 5.4 us, which is latency.
// Columns of the matrix instructions.  The second product's left operand (V) has no scales in it: they belong to a slot and a group of 32
// elements, so the weights take them, and every group of elements needs weights of its own.  With few heads (WIDE false: up to
// 16 / groups) a column is a (head, group): a lane scales its weights once, and of the products with all elements keeps its group's.
// With more (WIDE) a column is a head, and a lane makes as many operands as there are groups.
template <typename T, int DH, bool WIDE>
__global__ __launch_bounds__(512) void q4_step_kernel(const StepArgs<T> a) {
  typedef Block<DH> L;
  constexpr int G = L::kGroups, KW = DH / 32, NT = DH / 16, OG = WIDE ? G : 1;   // KW: code words of a lane and tile; NT: tiles of V
  constexpr int HEADS = WIDE ? kPassHeads : 16 / G;
  constexpr int QN = kQTerms<T>, PN = kPTerms<T>;
  extern __shared__ __align__(16) float s_dyn[];    // [waves + 1][HEADS][DH] sums, [waves + 1][HEADS][2]; one workgroup a row: [group][64 blocks] exponents
  __shared__ uint64_t s_key[8];
  __shared__ float s_total[kPassHeads][2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = int(blockDim.x >> 6) - a.extra;
  const int c = lane & 15, quarter = lane >> 4;
  const bool alone = a.splits == 1 && a.passes == 1;
  const int row = blockIdx.x / a.splits, split = blockIdx.x % a.splits, pass = blockIdx.y, b = row / a.s.kv_heads, hk = row % a.s.kv_heads;
  const int K = a.s.slots, KP = a.s.blocks * kSlots;
  const int head0 = pass * kPassHeads, heads = min(HEADS, a.s.group - head0);    // (WIDE false: one pass)
  const int head = WIDE ? c : c / G, mygroup = WIDE ? 0 : c % G;
  float *s_o = s_dyn, *s_ml = s_dyn + (waves + 1) * HEADS * DH, *s_logit = s_ml + (waves + 1) * HEADS * 2;
  int slot, n;
  cursor_of(a.cursor, row, K, slot, n);
  if (!alone && split == 0 && pass == 0 && tid == 0) a.arrived[row] = 0;

  // the query operand: element DH / 4 quarter + 8 s + i of the column's head
  bf16x8 qf[KW][QN];
  {
    const T *q = a.q + (size_t(b) * a.s.heads + hk * a.s.group + head0 + min(head, heads - 1)) * DH + quarter * (DH / 4);
#pragma unroll
    for (int s = 0; s < KW; ++s) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8 / Vec16<T>::EPL; ++i) {
        float y[Vec16<T>::EPL];
        Vec16<T>::load(q + 8 * s + i * Vec16<T>::EPL, y);
#pragma unroll
        for (int e = 0; e < Vec16<T>::EPL; ++e) x[i * Vec16<T>::EPL + e] = y[e];
      }
      terms_of<QN>(x, qf[s]);
    }
  }

  f32x4 o[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  float top = -INFINITY, sum = 0.f;

  struct Raw {
    uint32_t k[4][KW], kscale, v[NT][2];
    u32x4 vscale[OG];
    int pos;                         // of the lane's slot
  };
  unsigned char *cache = a.cache + size_t(row) * a.s.blocks * L::kBytes;
  const int32_t *pos = a.slot_pos + size_t(row) * K;
  auto load_k = [&](int block, Raw &r) {
    const unsigned char *in = cache + size_t(block) * L::kBytes;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const unsigned char *p = in + (16 * t + c) * (DH / 2) + quarter * (DH / 8);
      if constexpr (KW == 4) {
        const u32x4 u = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
        for (int s = 0; s < 4; ++s) r.k[t][s] = u[s];
      } else {
        const u32x2 u = *reinterpret_cast<const u32x2 *>(p);
        r.k[t][0] = u[0];
        r.k[t][1] = u[1];
      }
    }
    r.kscale = *reinterpret_cast<const uint32_t *>(in + L::kKScale + quarter * G / 4 * kSlots + 4 * c);
    r.pos = block * kSlots + lane < K ? pos[block * kSlots + lane] : -1;
  };
  auto load_v = [&](int block, Raw &r) {
    const unsigned char *in = cache + size_t(block) * L::kBytes;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const u32x2 u = *reinterpret_cast<const u32x2 *>(in + L::kV + (16 * t + c) * 32 + quarter * 8);
      r.v[t][0] = u[0];
      r.v[t][1] = u[1];
    }
#pragma unroll
    for (int g = 0; g < OG; ++g) r.vscale[g] = *reinterpret_cast<const u32x4 *>(in + L::kVScale + (WIDE ? g : mygroup) * kSlots + quarter * 16);
  };

  // The wave's next block takes the registers of this one's K as soon as they are free, then those of V.
  auto attend = [&](int block, int next, Raw &r) {
    f32x4 s[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
      const float unit = power(r.kscale >> (8 * t) & 255u);
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        const bf16x8 kf = operand_of(r.k[t][w], unit);
#pragma unroll
        for (int i = QN - 1; i >= 0; --i) s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[w][i], s[t], 0, 0, 0);
      }
      pin();                                       // operands are made as they are needed: all at once they would take 64 registers
    }
    float m = -INFINITY;
    uint64_t there = __builtin_amdgcn_ballot_w64(r.pos >= 0);
    if (next < a.s.blocks) load_k(next, r);
    if (block == slot >> 6) there &= ~(uint64_t(1) << (slot & 63));   // what it held goes; the new token comes in with the sums
    const uint32_t mine = uint32_t((quarter & 2 ? there >> 32 : there) >> (quarter & 1 ? 16 : 0));
#pragma unroll
    for (int i = 0; i < 16; ++i) {                 // slot 16 quarter + i is row i / 4 of tile i % 4
      const float x = mine >> i & 1 ? s[i & 3][i >> 2] * a.s.scale_log2 : -INFINITY;
      s[i & 3][i >> 2] = x;
      m = fmaxf(m, x);
    }
    if ((WIDE || mygroup == 0) && head < heads) {
      const size_t at = size_t(head) * KP + block * kSlots + quarter * 16;
      if (alone) {
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<f32x4 *>(s_logit + at + 4 * j) = f32x4{s[0][j], s[1][j], s[2][j], s[3][j]};
      } else {
        float *to = a.logit + (size_t(row) * a.s.group + head0) * KP + at;
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<f32x4 *>(to + 4 * j) = f32x4{s[0][j], s[1][j], s[2][j], s[3][j]};
      }
    }
    m = fmaxf(top, max_lane_xor<32>(max_lane_xor<16>(m)));
    const float base = m == -INFINITY ? 0.f : m;
    const float fade = __builtin_amdgcn_exp2f(top - base);
    top = m;
    sum *= fade;
#pragma unroll
    for (int t = 0; t < NT; ++t) o[t] *= fade;
    float p[16];
    float part = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      p[i] = __builtin_amdgcn_exp2f(s[i & 3][i >> 2] - base);
      part += p[i];
    }
    sum += part;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      bf16x8 pf[OG][PN];
#pragma unroll
      for (int g = 0; g < OG; ++g) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)            // (0 stays 0 whatever a free slot's scale is, which a product with infinity would not)
          x[i] = __builtin_ldexpf(p[8 * u + i], int(r.vscale[g][2 * u + (i >> 2)] >> (8 * (i & 3)) & 255u) - 127);
        terms_of<PN>(x, pf[g]);
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const bf16x8 vf = operand_of(r.v[t][u], 1.f);
#pragma unroll
        for (int i = PN - 1; i >= 0; --i) o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[WIDE ? t / 2 : 0][i], o[t], 0, 0, 0);
        if (t % 2) pin();
      }
    }
    if (next < a.s.blocks) load_v(next, r);
  };

  // The new token comes in with the waves' sums, as one more of them: its exponent, 1, its V as it is held.  Its codes go to memory
  // meanwhile; what the block's own wave reads of them counts for nothing.  The last wave does it, while its first block is on
  // its way or with nothing else to do.
  auto new_token = [&]() {
    const bool here = (slot >> 6) / waves % a.splits == split, in = lane < DH / 2;
    const size_t src = (size_t(b) * a.s.kv_heads + hk) * DH + 2 * (in ? lane : 0);   // two neighbouring elements a lane (DH = 64: 32 lanes)
    f32x2 held[2] = {f32x2{0.f, 0.f}, f32x2{0.f, 0.f}};
    if (here) {
      unsigned char *to = cache + size_t(slot >> 6) * L::kBytes;
      const int at = slot & 63;
      unsigned char *v = to + L::kV + 64 * (in ? lane : 0) + at / 2;
      // all that it reads at once: a trip to memory takes as long as an attention wave's products
      const T k0 = a.k_new[src], k1 = a.k_new[src + 1], v0 = a.v_new[src], v1 = a.v_new[src + 1];
      const uint32_t old0 = v[0], old1 = v[32];
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        const float x0 = number(to_float(kv ? v0 : k0)), x1 = number(to_float(kv ? v1 : k1));
        float big = fmaxf(fabsf(x0), fabsf(x1));              // of 16 lanes: 32 elements
        big = fmaxf(big, __shfl_xor(big, 1, 64));
        big = fmaxf(big, __shfl_xor(big, 2, 64));
        big = fmaxf(big, __shfl_xor(big, 4, 64));
        big = fmaxf(big, __shfl_xor(big, 8, 64));
        const uint32_t scale = scale_of(big);
        const uint32_t code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x0, x1, power(scale), 0) & 255u;
        held[kv] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, power(scale), 0);
        if (in && pass == 0) {
          if (kv == 0) {
            to[((at & 3) * 16 + (at >> 2)) * (DH / 2) + lane] = uint8_t(code);
          } else {
            const int sh = 4 * (at & 1);
            v[0] = uint8_t((old0 & ~(15u << sh)) | (code & 15u) << sh);
            v[32] = uint8_t((old1 & ~(15u << sh)) | code >> 4 << sh);
          }
          if ((lane & 15) == 0) to[(kv ? L::kVScale : L::kKScale) + (lane >> 4) * kSlots + at] = uint8_t(scale);
          T *out = kv ? a.v_held : a.k_held;
          if (out) {
            store_elem(out + src, held[kv][0]);
            store_elem(out + src + 1, held[kv][1]);
          }
        }
      }
    }
    for (int j = 0; j < heads; ++j) {
      const T *q = a.q + (size_t(b) * a.s.heads + hk * a.s.group + head0 + j) * DH + 2 * (in ? lane : 0);
      float x = in ? fmaf(to_float(q[0]), held[0][0], to_float(q[1]) * held[0][1]) : 0.f;
      x = here ? wave_sum(x) * a.s.scale_log2 : -INFINITY;
      if (lane == 0) {
        s_ml[(waves * HEADS + j) * 2] = x;
        s_ml[(waves * HEADS + j) * 2 + 1] = here ? 1.f : 0.f;
        if (here && !alone) a.part_new[size_t(row) * a.s.group + head0 + j] = x;
      }
      if (in) *reinterpret_cast<f32x2 *>(&s_o[(waves * HEADS + j) * DH + 2 * lane]) = held[1];
    }
  };
  {
    int block = wave < waves ? split * waves + wave : a.s.blocks;
    Raw r;
    if (block < a.s.blocks) {
      load_k(block, r);
      load_v(block, r);
    }
    if (wave == waves - 1 + a.extra) new_token();
    for (const int stride = a.splits * waves; block < a.s.blocks; block += stride) attend(block, block + stride, r);
  }

  // ---- the waves' sums together ----
  // what the end wants of the first slots is on its way meanwhile
  const bool early = alone && tid < K;
  const float early_score = early ? a.score[size_t(row) * K + tid] : 0.f;
  const int early_pos = early ? pos[tid] : -1;
  sum = add_lane_xor<32>(add_lane_xor<16>(sum));
  if (wave < waves && head < heads) {
    if (quarter == 0 && (WIDE || mygroup == 0)) {
      s_ml[(wave * HEADS + head) * 2] = top;
      s_ml[(wave * HEADS + head) * 2 + 1] = sum;
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
      if (WIDE || t / 2 == mygroup) *reinterpret_cast<f32x4 *>(&s_o[(wave * HEADS + head) * DH + 16 * t + 4 * quarter]) = o[t];
  }
  __syncthreads();
  auto total = [&](int j, float &m, float &base, float &l) {
    m = -INFINITY;
    l = 0.f;
    for (int w = 0; w <= waves; ++w) m = fmaxf(m, s_ml[(w * HEADS + j) * 2]);
    base = m == -INFINITY ? 0.f : m;
    for (int w = 0; w <= waves; ++w) l += s_ml[(w * HEADS + j) * 2 + 1] * __builtin_amdgcn_exp2f(s_ml[(w * HEADS + j) * 2] - base);
  };
  if (tid < heads) {
    float m, base, l;
    total(tid, m, base, l);
    s_total[tid][0] = base;
    s_total[tid][1] = 1.f / l;
    if (!alone) {
      float *ml = a.part_ml + (((size_t(row) * a.passes + pass) * a.splits + split) * kPassHeads + tid) * 2;
      ml[0] = m;
      ml[1] = l;
    }
  }
  for (int i = tid; i < heads * DH; i += blockDim.x) {
    const int j = i / DH, e = i % DH;
    float m, base, l, x = 0.f;
    total(j, m, base, l);
    for (int w = 0; w <= waves; ++w) x += s_o[(w * HEADS + j) * DH + e] * __builtin_amdgcn_exp2f(s_ml[(w * HEADS + j) * 2] - base);
    if (alone)
      store_elem(a.out + (size_t(b) * a.s.heads + hk * a.s.group + head0 + j) * DH + e, x / l);
    else
      a.part_o[(((size_t(row) * a.passes + pass) * a.splits + split) * kPassHeads + j) * DH + e] = x;
  }
  if (!alone) return;
  __syncthreads();
  // ---- what the row's slots received, and the next one to go ----
  uint64_t key = ~uint64_t(0);
  for (int i = tid; i < K; i += blockDim.x) {
    float x = i == slot ? 0.f : i == tid ? early_score : a.score[size_t(row) * K + i];
    const int at = i == slot ? n : i == tid ? early_pos : pos[i];
    float p = 0.f;
    for (int j = 0; j < heads; ++j)
      p += __builtin_amdgcn_exp2f((i == slot ? s_ml[(waves * HEADS + j) * 2] : s_logit[size_t(j) * KP + i]) - s_total[j][0]) * s_total[j][1];
    x += p;
    if (at >= 0) a.score[size_t(row) * K + i] = x;
    if (i == slot) a.slot_pos[size_t(row) * K + i] = n;
    key = min_key(key, eviction_key(at, x, i, n + 1, a.s.recent));
  }
  key = workgroup_min(key, s_key);
  if (tid == 0) {
    a.cursor[2 * row] = int(uint32_t(key));
    a.cursor[2 * row + 1] = n + 1;
  }
}

// Several workgroups a row: their sums together, and the slots' share of the attention, OWN to a thread.  The last one to
// arrive looks for the smallest key; keys and the counter go past the L2 (agent scope), nothing else is handed over.
template <typename T, int DH, int OWN>
__global__ __launch_bounds__(kFinishThreads) void q4_finish_kernel(const StepArgs<T> a, int parts) {
  extern __shared__ __align__(16) float s_dyn[];    // [group][2] maximum and 1 / sum, [group][splits] factor of each workgroup's sums
  __shared__ uint64_t s_key[kFinishThreads / 64];
  __shared__ int s_last;
  const int row = blockIdx.x / parts, part = blockIdx.x % parts, b = row / a.s.kv_heads, hk = row % a.s.kv_heads, tid = threadIdx.x;
  const int K = a.s.slots, KP = a.s.blocks * kSlots, group = a.s.group;
  float *s_factor = s_dyn + 2 * group;
  int slot, n;
  cursor_of(a.cursor, row, K, slot, n);
  // the slots' part is on its way while the heads' sums are put together
  constexpr int kOwn = OWN, kEarly = 4;
  const int first = part * (OWN * kFinishThreads) + tid;
  auto exponent = [&](int i, int j) { return i == slot ? a.part_new[size_t(row) * group + j] : a.logit[(size_t(row) * group + j) * KP + i]; };
  float score[kOwn], early[kOwn][kEarly];
  int at[kOwn];
#pragma unroll
  for (int u = 0; u < kOwn; ++u) {
    const int i = first + u * kFinishThreads;
    const bool there = i < K;
    score[u] = there && i != slot ? a.score[size_t(row) * K + i] : 0.f;
    at[u] = i == slot ? n : there ? a.slot_pos[size_t(row) * K + i] : -1;
#pragma unroll
    for (int j = 0; j < kEarly; ++j) early[u][j] = there && j < group ? exponent(i, j) : 0.f;
  }
  // a wave a head
  for (int j = tid >> 6; j < group; j += kFinishThreads / 64) {
    const int lane = tid & 63;
    const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml) + ((size_t(row) * a.passes + j / kPassHeads) * a.splits) * kPassHeads + j % kPassHeads;
    float m = -INFINITY, l = 0.f;
    for (int s = lane; s < a.splits; s += 64) m = fmaxf(m, ml[size_t(s) * kPassHeads].x);
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    const float base = m == -INFINITY ? 0.f : m;
    for (int s = lane; s < a.splits; s += 64) {
      const float2 x = ml[size_t(s) * kPassHeads];
      const float f = __builtin_amdgcn_exp2f(x.x - base);
      s_factor[j * a.splits + s] = f;
      l = fmaf(x.y, f, l);
    }
    l = wave_sum(l);
    if (lane == 0) {
      s_dyn[2 * j] = base;
      s_dyn[2 * j + 1] = 1.f / l;
    }
  }
  __syncthreads();
  for (int i = tid + part * kFinishThreads; i < group * DH; i += parts * kFinishThreads) {
    const int j = i / DH, e = i % DH;
    const float *o = a.part_o + ((size_t(row) * a.passes + j / kPassHeads) * a.splits * kPassHeads + j % kPassHeads) * DH + e;
    float x = 0.f;
#pragma unroll 8
    for (int s = 0; s < a.splits; ++s) x = fmaf(o[size_t(s) * (kPassHeads * DH)], s_factor[j * a.splits + s], x);
    store_elem(a.out + (size_t(b) * a.s.heads + hk * group + j) * DH + e, x * s_dyn[2 * j + 1]);
  }
  uint64_t key = ~uint64_t(0);
#pragma unroll
  for (int u = 0; u < kOwn; ++u) {
    const int i = first + u * kFinishThreads;
    if (i >= K) break;
    float p = 0.f;
#pragma unroll
    for (int j = 0; j < kEarly; ++j)
      if (j < group) p += __builtin_amdgcn_exp2f(early[u][j] - s_dyn[2 * j]) * s_dyn[2 * j + 1];
#pragma unroll 4
    for (int j = kEarly; j < group; ++j) p += __builtin_amdgcn_exp2f(exponent(i, j) - s_dyn[2 * j]) * s_dyn[2 * j + 1];
    const float x = score[u] + p;
    if (at[u] >= 0) a.score[size_t(row) * K + i] = x;
    if (i == slot) a.slot_pos[size_t(row) * K + i] = n;
    key = min_key(key, eviction_key(at[u], x, i, n + 1, a.s.recent));
  }
  key = workgroup_min(key, s_key);
  if (parts == 1) {
    if (tid == 0) {
      a.cursor[2 * row] = int(uint32_t(key));
      a.cursor[2 * row + 1] = n + 1;
    }
    return;
  }
  if (tid == 0) {
    __hip_atomic_store(a.part_key + size_t(row) * parts + part, key, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                 // the key is where the last one will look for it
    s_last = __hip_atomic_fetch_add(a.arrived + row, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == parts - 1;
  }
  __syncthreads();
  if (!s_last) return;
  key = ~uint64_t(0);
  for (int i = tid; i < parts; i += kFinishThreads)
    key = min_key(key, __hip_atomic_load(a.part_key + size_t(row) * parts + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
  key = workgroup_min(key, s_key);
  if (tid == 0) {
    a.cursor[2 * row] = int(uint32_t(key));
    a.cursor[2 * row + 1] = n + 1;
  }
}

// ---- host ----------------------------------------------------------------------------------------------------------------
int q4_shape(const adore_q4_config *c, Q4Shape *s) {
  if (!c || c->batch <= 0 || c->heads <= 0 || c->kv_heads <= 0 || c->heads % c->kv_heads != 0 || c->head_dim <= 0 || c->slots < 2 ||
      c->recent < 1 || c->recent >= c->slots || (c->dtype != ADORE_F32 && c->dtype != ADORE_BF16) || !std::isfinite(c->scale) || c->scale < 0.f)
    return ADORE_E_INVALID;
  if ((c->head_dim != 64 && c->head_dim != 128) || c->slots > kMaxQ4Slots || c->batch > (1 << 16) || c->heads > (1 << 12) ||
      (long long)c->batch * c->kv_heads * blocks_of(c->slots) > (1 << 23) || (long long)c->batch * c->heads > (1 << 20))
    return ADORE_E_UNSUPPORTED;
  s->batch = c->batch;
  s->heads = c->heads;
  s->kv_heads = c->kv_heads;
  s->group = c->heads / c->kv_heads;
  s->slots = c->slots;
  s->blocks = blocks_of(c->slots);
  s->recent = c->recent;
  s->scale_log2 = (c->scale > 0.f ? c->scale : 1.f / sqrtf(float(c->head_dim))) * kLog2e;
  return ADORE_OK;
}

// How a step's work is cut.
struct StepPlan {
  bool wide;
  int passes, splits, waves, extra;
  int own, parts;      // slots of a finishing thread, finishing workgroups of a row
};
constexpr int kMaxLds = 128 * 1024;
int step_lds(const Q4Shape &s, int head_dim, const StepPlan &p) {
  const int heads = p.wide ? kPassHeads : 16 / (head_dim / 32);
  const long long logits = p.splits == 1 && p.passes == 1 ? (long long)s.group * s.blocks * kSlots : 0;
  const long long bytes = ((long long)(p.waves + 1) * heads * (head_dim + 2) + logits) * 4;
  return bytes > kMaxLds ? kMaxLds + 1 : int(bytes);
}
StepPlan plan_step(const Q4Shape &s, int head_dim) {
  StepPlan p;
  p.wide = s.group > 16 / (head_dim / 32);
  p.passes = (s.group + kPassHeads - 1) / kPassHeads;
  const long long rows = (long long)s.batch * s.kv_heads;
  // One workgroup a row wherever that fills the chip, or a wave has few blocks: no second launch.  Few large workgroups, whose waves have
  // their next block on its way, rather than many small ones (4 sequences, 8 kv heads, 16384 slots: 256 workgroups of 8 waves 18 us,
  // 512 20, 1024 28; of 4 waves 22, 25, 30).  With a row for every place (16 x 32 rows of 512 slots) 4 waves each 14 us, 3 15, 8 18.
  // The new token has a wave of its own where a place has waves to spare (long rows 18 us / 20, a single row 5.4 / 6.2; 512 rows 14.9 / 14.0).
  p.splits = 1;
  const long long groups = rows * p.passes;
  p.waves = groups >= 512 ? 4 : 7;
  p.extra = groups >= 512 ? 0 : 1;
  if (s.blocks > 16 && groups < 256) {
    const long long want = (256 + groups - 1) / groups, able = (s.blocks + p.waves - 1) / p.waves;
    p.splits = int(want < able ? want : able);
    if (p.splits > 64) p.splits = 64;
    const int most = 8192 / s.group;      // factors in the finishing workgroups' LDS
    if (p.splits > most) p.splits = most > 1 ? most : 1;
  }
  if (p.waves > s.blocks) p.waves = s.blocks;
  if (p.splits == 1 && step_lds(s, head_dim, p) > kMaxLds) {   // the exponents of all slots are too many for LDS
    p.waves = 4;
    p.splits = 2;
  }
  // Finishing workgroups: as many as have a place each, and one a row where that is enough (slots of a thread 1 / 2 / 4: 4 rows of 8000, 16 heads
  // 23.3 / 26.0 / 31.2 us a step, 16 rows of 4556, 7 heads 18.9 / 20.9 / 24.2; 32 rows of 16384, 4 heads 33.0 / 28.3 / 29.2; 30 of 1335 12.8 / 11.5 / 11.9).
  p.own = s.slots > 2 * kFinishThreads ? 1 : 2;
  auto parts_of = [&](int own) { return (s.slots + own * kFinishThreads - 1) / (own * kFinishThreads); };
  while (p.own < 4 && rows * parts_of(p.own) > 256) p.own *= 2;
  p.parts = parts_of(p.own);
  return p;
}
bool alone(const StepPlan &p) { return p.splits == 1 && p.passes == 1; }

struct StepSpace {
  size_t part_o, part_ml, logit, part_new, part_key, arrived, total;
};
StepSpace step_space(const Q4Shape &s, int head_dim, const StepPlan &p) {
  StepSpace w = {};
  if (alone(p)) {
    w.total = 256;
    return w;
  }
  const size_t rows = size_t(s.batch) * s.kv_heads, parts = rows * p.passes * p.splits * kPassHeads;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) / 256 * 256;
    return here;
  };
  w.part_o = take(parts * head_dim * 4);
  w.part_ml = take(parts * 8);
  w.logit = take(rows * s.group * s.blocks * kSlots * 4);
  w.part_new = take(rows * s.group * 4);
  w.part_key = take(rows * p.parts * 8);
  w.arrived = take(rows * 4);
  w.total = at;
  return w;
}

template <typename T, int DH, bool WIDE>
hipError_t launch_step(const StepArgs<T> &a, const StepPlan &p, hipStream_t st) {
  const int lds = step_lds(a.s, DH, p);
  hipError_t e = allow_lds(&q4_step_kernel<T, DH, WIDE>, lds);
  if (e != hipSuccess) return e;
  const unsigned rows = unsigned(a.s.batch) * unsigned(a.s.kv_heads);
  hipLaunchKernelGGL((q4_step_kernel<T, DH, WIDE>), dim3(rows * unsigned(p.splits), unsigned(p.passes)), dim3(64 * (p.waves + p.extra)), lds, st, a);
  if ((e = hipGetLastError()) != hipSuccess || alone(p)) return e;
  const dim3 grid(rows * unsigned(p.parts)), block(kFinishThreads);
  const int factors = a.s.group * (2 + p.splits) * 4;
  if (p.own == 1)
    hipLaunchKernelGGL((q4_finish_kernel<T, DH, 1>), grid, block, factors, st, a, p.parts);
  else if (p.own == 2)
    hipLaunchKernelGGL((q4_finish_kernel<T, DH, 2>), grid, block, factors, st, a, p.parts);
  else
    hipLaunchKernelGGL((q4_finish_kernel<T, DH, 4>), grid, block, factors, st, a, p.parts);
  return hipGetLastError();
}

template <typename T>
int step_typed(const Q4Shape &s, int head_dim, const void *q, const void *k_new, const void *v_new, void *cache, int32_t *slot_pos, float *score,
               int32_t *cursor, void *out, void *k_held, void *v_held, void *workspace, hipStream_t st) {
  const StepPlan p = plan_step(s, head_dim);
  const StepSpace w = step_space(s, head_dim, p);
  char *ws = static_cast<char *>(workspace);
  StepArgs<T> a;
  a.s = s;
  a.q = static_cast<const T *>(q);
  a.k_new = static_cast<const T *>(k_new);
  a.v_new = static_cast<const T *>(v_new);
  a.cache = static_cast<unsigned char *>(cache);
  a.slot_pos = slot_pos;
  a.cursor = cursor;
  a.score = score;
  a.out = static_cast<T *>(out);
  a.k_held = static_cast<T *>(k_held);
  a.v_held = static_cast<T *>(v_held);
  a.splits = p.splits;
  a.passes = p.passes;
  a.extra = p.extra;
  a.part_o = reinterpret_cast<float *>(ws + w.part_o);
  a.part_ml = reinterpret_cast<float *>(ws + w.part_ml);
  a.logit = reinterpret_cast<float *>(ws + w.logit);
  a.part_new = reinterpret_cast<float *>(ws + w.part_new);
  a.part_key = reinterpret_cast<uint64_t *>(ws + w.part_key);
  a.arrived = reinterpret_cast<int32_t *>(ws + w.arrived);
  hipError_t e;
  if (head_dim == 128)
    e = p.wide ? launch_step<T, 128, true>(a, p, st) : launch_step<T, 128, false>(a, p, st);
  else
    e = p.wide ? launch_step<T, 64, true>(a, p, st) : launch_step<T, 64, false>(a, p, st);
  return e == hipSuccess ? ADORE_OK : ADORE_E_HIP;
}

template <typename T>
int fill_typed(const Q4Shape &s, int head_dim, const int32_t *k_start, int k_tokens, const adore_rows *k, const adore_rows *v, const float *scores,
               void *cache, int32_t *slot_pos, float *score, int32_t *cursor, hipStream_t st) {
  const unsigned rows = unsigned(s.batch) * unsigned(s.kv_heads);
  hipLaunchKernelGGL(q4_choose_kernel, dim3(rows), dim3(kFillThreads), 0, st, ChooseArgs{s, k_start, k_tokens, scores, slot_pos, score, cursor});
  if (hipGetLastError() != hipSuccess) return ADORE_E_HIP;
  PackArgs<T> a;
  a.s = s;
  a.k_start = k_start;
  a.slot_pos = slot_pos;
  a.k_tokens = k_tokens;
  a.k = rows_of<const T>(k);
  a.v = rows_of<const T>(v);
  a.cache = static_cast<unsigned char *>(cache);
  if (head_dim == 128)
    hipLaunchKernelGGL((q4_pack_kernel<T, 128>), dim3(rows * unsigned(s.blocks)), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((q4_pack_kernel<T, 64>), dim3(rows * unsigned(s.blocks)), dim3(256), 0, st, a);
  return hipGetLastError() == hipSuccess ? ADORE_OK : ADORE_E_HIP;
}

template <typename T>
int read_typed(const Q4Shape &s, int head_dim, const void *cache, const int32_t *slot_pos, void *k, void *v, hipStream_t st) {
  const ReadArgs<T> a{s, static_cast<const unsigned char *>(cache), slot_pos, static_cast<T *>(k), static_cast<T *>(v)};
  const unsigned blocks = unsigned(s.batch) * unsigned(s.kv_heads) * unsigned(s.blocks);
  if (head_dim == 128)
    hipLaunchKernelGGL((q4_read_kernel<T, 128>), dim3(blocks), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((q4_read_kernel<T, 64>), dim3(blocks), dim3(256), 0, st, a);
  return hipGetLastError() == hipSuccess ? ADORE_OK : ADORE_E_HIP;
}

bool aligned(const void *p, uintptr_t to) { return p && (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

}  // namespace

}  // namespace adore

extern "C" {

size_t adore_q4_cache_bytes(const adore_q4_config *cfg) {
  adore::Q4Shape s;
  if (adore::q4_shape(cfg, &s) != ADORE_OK) return 0;
  return size_t(s.batch) * s.kv_heads * s.blocks * 68 * cfg->head_dim;
}

size_t adore_q4_workspace_bytes(const adore_q4_config *cfg) {
  adore::Q4Shape s;
  if (adore::q4_shape(cfg, &s) != ADORE_OK) return 0;
  return adore::step_space(s, cfg->head_dim, adore::plan_step(s, cfg->head_dim)).total;
}

int adore_q4_fill(const adore_q4_config *cfg, const int32_t *k_start, int32_t k_tokens, const adore_rows *k, const adore_rows *v,
                  const float *scores, void *cache, int32_t *slot_pos, float *score, int32_t *cursor, void *hip_stream) {
  using namespace adore;
  Q4Shape s;
  const int rc = q4_shape(cfg, &s);
  if (rc != ADORE_OK) return rc;
  if (k_tokens < 0 || !prompt_rows_ok(k, cfg->dtype) || !prompt_rows_ok(v, cfg->dtype) || !aligned(cache, 256) || !aligned(slot_pos, 16) ||
      !aligned(score, 16) || !aligned(cursor, 8))
    return ADORE_E_INVALID;
  if (k_tokens > (1 << 24)) return ADORE_E_UNSUPPORTED;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return cfg->dtype == ADORE_BF16 ? fill_typed<bf16_t>(s, cfg->head_dim, k_start, k_tokens, k, v, scores, cache, slot_pos, score, cursor, st)
                                  : fill_typed<float>(s, cfg->head_dim, k_start, k_tokens, k, v, scores, cache, slot_pos, score, cursor, st);
}

int adore_q4_step(const adore_q4_config *cfg, const void *q, const void *k_new, const void *v_new, void *cache, int32_t *slot_pos, float *score,
                  int32_t *cursor, void *out, void *k_held, void *v_held, void *workspace, size_t workspace_bytes, void *hip_stream) {
  using namespace adore;
  Q4Shape s;
  const int rc = q4_shape(cfg, &s);
  if (rc != ADORE_OK) return rc;
  if (!aligned(q, 16) || !aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(out, 16) || !aligned(cache, 256) || !aligned(slot_pos, 16) ||
      !aligned(score, 16) || !aligned(cursor, 8) || !workspace || (k_held && !aligned(k_held, 16)) || (v_held && !aligned(v_held, 16)))
    return ADORE_E_INVALID;
  if (!aligned(workspace, 256) || workspace_bytes < step_space(s, cfg->head_dim, plan_step(s, cfg->head_dim)).total) return ADORE_E_WORKSPACE;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return cfg->dtype == ADORE_BF16
             ? step_typed<bf16_t>(s, cfg->head_dim, q, k_new, v_new, cache, slot_pos, score, cursor, out, k_held, v_held, workspace, st)
             : step_typed<float>(s, cfg->head_dim, q, k_new, v_new, cache, slot_pos, score, cursor, out, k_held, v_held, workspace, st);
}

int adore_q4_read(const adore_q4_config *cfg, const void *cache, const int32_t *slot_pos, void *k, void *v, void *hip_stream) {
  using namespace adore;
  Q4Shape s;
  const int rc = q4_shape(cfg, &s);
  if (rc != ADORE_OK) return rc;
  if (!aligned(cache, 256) || !aligned(slot_pos, 16) || !aligned(k, 16) || !aligned(v, 16)) return ADORE_E_INVALID;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return cfg->dtype == ADORE_BF16 ? read_typed<bf16_t>(s, cfg->head_dim, cache, slot_pos, k, v, st)
                                  : read_typed<float>(s, cfg->head_dim, cache, slot_pos, k, v, st);
}

}  // extern "C"
