// A K/V cache for attention with a window and first tokens that stay (paper Sec. 3.1, baselines 2 and 5), and single-query attention over it
// (Sec. 2.1, Eq. 1, with grouped heads).  Position p is in slot p if p < sinks, else in slot sinks + (p - sinks) % window: the row that a
// token takes is that of the one that leaves its window.  Which slots hold something, and which one is next, follow from one number.
//
//   out = sum_s softmax_s(scale q . K[s]) V[s] over the slots that are held, the new token's among them
//
// Layout: blocks of 32 slots, K then V, each 32 x DH elements in the order in which the matrix instructions (16x16, lane = 16 quarter + c)
// take them: every load of a wave is 1 KB in a run, straight to the registers of its operand, and V needs no transposition.
//   bf16   K [DH / 32][t = 0, 1][quarter][c][8]: slot 8 (c / 4) + 4 t + c % 4, element 32 i + 8 quarter + e
//          V [DH / 16][quarter][c][8]:           element 16 i + c, slot 8 quarter + e
//   fp32   K [DH / 16][t][quarter][c][4]:        slot 16 t + c, element 16 i + 4 quarter + e
//          V [DH / 16][t][quarter][c][4]:        element 16 i + c, slot 16 t + 4 quarter + e
// S^T = K Q^T leaves lane (quarter, c) the weights of head c and exactly those slots that P^T's operand in O^T += V^T P^T wants of it.
// In bf16 a weight goes in as two terms (within 2^-16); fp32 has its own matrix instructions.
// Bound by memory: every held row is read once for each 16 query heads, and the matrix unit is busy 3 or 4 % of the cycles.  A token of 512 rows of
// up to 512 slots (16 sequences of 32 heads of 128) 20.9 us, 5.1 TB/s, which a large copy reaches; of 32 rows of 16384 slots, 4 heads each,
// 34.6 us at 6.1 TB/s and 4.7 to join.  Prompts of 1024 tokens and fewer into the former 29 us, out of it 38.
// Blocks, and rows in and out, are read past the caches, which a model's other layers would overwrite before the next token: 32 rows of 16384
// slots 46.4 us for 51.1, 512 of 512 25.1 for 27.4, in 29 for 40.  (8 rows of 4096, 16 MB, stepped again and again with nothing between, 10.7
// for 10.1.)  Where a kv head has more than 16 query heads its rows are read more than once, past the caches too: 8 sequences of 64 heads over 2
// and 16384 slots (three caches in turn) 31.9 us, through the caches 33.4; 16 of 48 over 1 and 4096 slots (six caches, which the last level holds
// together) 27.8, through the caches 23.8.
#include <hip/hip_runtime.h>

#include <cmath>

#include "prompt_device.h"

namespace adore {

namespace {

constexpr int kSlots = 32;           // of a block
constexpr int kMaxSlots = 1 << 20;
constexpr int kHeads = 16;           // of a matrix instruction
constexpr float kLog2e = 1.4426950408889634f;

struct RingShape {
  int batch, heads, kv_heads, group;
  int window, sinks, slots, blocks;
  int tiles;                         // of 16 heads that a group has
  float scale_log2;
};

__device__ __forceinline__ int slot_of(int position, int sinks, int window) {
  return position < sinks ? position : sinks + (position - sinks) % window;
}

// A block's chunks: 64 lanes x 16 bytes each.
template <typename T, int DH>
struct Ring {
  static constexpr int kElems = 32 * DH, kChunks = kElems * int(sizeof(T)) / 1024, EPL = 16 / int(sizeof(T));
  // Chunk and element within the block's K (or V) of slot `slot`, element `el`.
  __device__ static __forceinline__ int k_at(int slot, int el) {
    if constexpr (sizeof(T) == 4) return ((el >> 4) * 2 + (slot >> 4)) * 256 + ((el >> 2) & 3) * 64 + (slot & 15) * 4 + (el & 3);
    return ((el >> 5) * 2 + ((slot >> 2) & 1)) * 512 + ((el >> 3) & 3) * 128 + ((slot >> 3) * 4 + (slot & 3)) * 8 + (el & 7);
  }
  __device__ static __forceinline__ int v_at(int slot, int el) {
    if constexpr (sizeof(T) == 4) return ((el >> 4) * 2 + (slot >> 4)) * 256 + ((slot >> 2) & 3) * 64 + (el & 15) * 4 + (slot & 3);
    return (el >> 4) * 512 + (slot >> 3) * 128 + (el & 15) * 8 + (slot & 7);
  }
};

// ---- one token ------------------------------------------------------------------------------------------------------------
template <typename T>
struct StepArgs {
  RingShape s;
  const T *q, *k_new, *v_new;
  T *cache, *out;
  int32_t *cursor;
  float *part_o, *part_ml;           // [row][tile][split][16 heads]: sums [DH], maximum and sum of weights
  int splits;
};

// Waves of a workgroup: 512 rows of 512 slots 25.1 us, 32 of 16384 46.4, 64 of 16384 82.7, 1024 of 256 28.6; eight: 25.3, 49.8, 84.3 and 28.5.
// In fp32 rows of four heads of 128 elements (two to three caches in turn), 128 of 1024 36.5 / 32.3, 32 of 16384 116 / 95, 2 of 4096 19.6 / 23.9; of one
// head 512 of 512 51.0 / 57.0, 1024 of 256 55.6 / 65.4: neither number is best for all.
// A wave has one block in its registers: the next one on its way while it works on one gained nothing (32 of 16384 with loads through the caches
// 52.5 for 51.9) for twice the registers.
constexpr int kStepWaves = 4;
constexpr int kMaxSplits = 64;       // of a row: a lane each where they are joined (splits_of says what that costs)

// The sums of a wave's slots for 16 heads: o[i] (row = element 16 i + 4 quarter + r, column = head c) relative to `top`, and the lane's share
// of the sum of weights.
template <int DH>
struct Sums {
  f32x4 o[DH / 16];
  float top, sum;
};

// A block's 32 slots; `visible` has a bit for each.
template <typename T, int DH>
__device__ __forceinline__ void take_block(Sums<DH> &a, const u32x4 (&qf)[Ring<T, DH>::kChunks / 2], const u32x4 (&kx)[Ring<T, DH>::kChunks],
                                           u32x4 (&vx)[Ring<T, DH>::kChunks], uint32_t visible, float scale, int quarter) {
  constexpr int N = Ring<T, DH>::kChunks;
  f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if constexpr (sizeof(T) == 2) {
      s[i & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kx[i]), __builtin_bit_cast(bf16x8, qf[i >> 1]), s[i & 1], 0, 0, 0);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        s[i & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kx[i][e]), __uint_as_float(qf[i >> 1][e]), s[i & 1], 0, 0, 0);
    }
  }
  if (visible != 0xffffffffu) {
    // (what is hidden may hold anything: a weight of 0 would not hide it from the product)
    uint32_t mine[2];                        // four slots each
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      mine[t] = visible >> (sizeof(T) == 2 ? 8 * quarter + 4 * t : 16 * t + 4 * quarter);
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (!(mine[t] >> r & 1)) s[t][r] = -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t two = mine[j >> 1] >> (2 * (j & 1));
          vx[i][j] &= (two & 1 ? 0xffffu : 0u) | (two & 2 ? 0xffff0000u : 0u);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) vx[i][j] = mine[i & 1] >> j & 1 ? vx[i][j] : 0u;
      }
    }
  }
  float m = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
  m = fmaxf(a.top, max_lane_xor<32>(max_lane_xor<16>(m)));
  if (__builtin_amdgcn_ballot_w64(m > a.top)) {
    const float fade = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((a.top - m) * scale);
    a.sum *= fade;
#pragma unroll
    for (int i = 0; i < DH / 16; ++i) a.o[i] *= fade;
    a.top = m;
  }
  const float base = a.top == -INFINITY ? 0.f : -a.top * scale;
  float part = 0.f;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      s[t][r] = __builtin_amdgcn_exp2f(fmaf(s[t][r], scale, base));
      part += s[t][r];
    }
  a.sum += part;
  if constexpr (sizeof(T) == 2) {
    u32x4 hi, lo;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float x = s[j >> 1][2 * (j & 1)], y = s[j >> 1][2 * (j & 1) + 1];
      hi[j] = pair_bf16(x, y);
      lo[j] = pair_bf16(x - __uint_as_float(hi[j] << 16), y - __uint_as_float(hi[j] & 0xffff0000u));
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      a.o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vx[i]), __builtin_bit_cast(bf16x8, hi), a.o[i], 0, 0, 0);
      a.o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vx[i]), __builtin_bit_cast(bf16x8, lo), a.o[i], 0, 0, 0);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) a.o[i >> 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vx[i][r]), s[i & 1][r], a.o[i >> 1], 0, 0, 0);
  }
}

// A workgroup: a row (sequence x kv head), 16 heads of its group, and a part of the row's blocks, its waves' one after the other.
template <typename T, int DH>
__global__ __launch_bounds__(64 * kStepWaves) void ring_step_kernel(const StepArgs<T> a) {
  typedef Ring<T, DH> L;
  constexpr int N = L::kChunks, EPL = L::EPL, NW = kStepWaves;
  __shared__ __align__(16) float s_o[NW][kHeads][DH + 4];
  __shared__ float s_top[NW][kHeads], s_sum[NW][kHeads];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, quarter = lane >> 4;
  const int split = blockIdx.x % a.splits, item = blockIdx.x / a.splits, tile = item % a.s.tiles, row = item / a.s.tiles;
  const int b = row / a.s.kv_heads, hk = row - b * a.s.kv_heads;
  const int position = max(a.cursor[row], 0), next = slot_of(position, a.s.sinks, a.s.window), held = min(position, a.s.slots);
  const float scale = a.s.scale_log2;
  T *const cache = a.cache + size_t(row) * a.s.blocks * (2 * L::kElems);
  // the queries: column c is head 16 tile + c of the group
  const int head = tile * kHeads + c;
  const T *const qp = a.q + (size_t(b) * a.s.heads + size_t(hk) * a.s.group + min(head, a.s.group - 1)) * DH + quarter * EPL;
  u32x4 qf[N / 2];
#pragma unroll
  for (int i = 0; i < N / 2; ++i) qf[i] = *reinterpret_cast<const u32x4 *>(qp + i * 4 * EPL);
  Sums<DH> sums;
#pragma unroll
  for (int i = 0; i < DH / 16; ++i) sums.o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  sums.top = -INFINITY;
  sums.sum = 0.f;
  u32x4 kx[N], vx[N];
  const int end = (held + kSlots - 1) / kSlots, step = a.splits * NW;
  auto load = [&](int block, u32x4 (&k)[N], u32x4 (&v)[N]) {
    const u32x4 *const p = reinterpret_cast<const u32x4 *>(cache + size_t(block) * (2 * L::kElems)) + lane;
#pragma unroll
    for (int i = 0; i < N; ++i) k[i] = __builtin_nontemporal_load(p + i * 64);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = __builtin_nontemporal_load(p + (N + i) * 64);
  };
  auto take = [&](int block, const u32x4 (&k)[N], u32x4 (&v)[N]) {
    const int left = held - block * kSlots;
    uint32_t visible = left >= kSlots ? 0xffffffffu : (1u << left) - 1u;
    if (next / kSlots == block) visible &= ~(1u << (next % kSlots));    // (its row is about to be another)
    take_block<T, DH>(sums, qf, k, v, visible, scale, quarter);
  };
  for (int block = split * NW + wave; block < end; block += step) {
    load(block, kx, vx);
    take(block, kx, vx);
  }
  if (split == 0 && wave == NW - 1) {
    // the new token: slot 0 of a block of its own, and its place in the ring
    const T *const kn = a.k_new + size_t(row) * DH, *const vn = a.v_new + size_t(row) * DH;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      // (the chunk's elements of slot 0: K's are in one lane's 16 bytes for every quarter, V's the first of quarter 0's lanes)
      kx[i] = vx[i] = u32x4{0, 0, 0, 0};
      if ((i & 1) == 0 && c == 0) kx[i] = *reinterpret_cast<const u32x4 *>(kn + (i >> 1) * 4 * EPL + quarter * EPL);
      if (quarter == 0) {
        if constexpr (sizeof(T) == 2)
          vx[i][0] = vn[16 * i + c].bits;
        else if ((i & 1) == 0)
          vx[i][0] = __float_as_uint(vn[8 * i + c]);
      }
    }
    take_block<T, DH>(sums, qf, kx, vx, 1u, scale, quarter);
    if (tile == 0) {
      T *const to = cache + size_t(next / kSlots) * (2 * L::kElems);
      for (int e = lane; e < DH; e += 64) {
        to[L::k_at(next % kSlots, e)] = kn[e];
        to[L::kElems + L::v_at(next % kSlots, e)] = vn[e];
      }
    }
  }
  // the waves' sums together
  float sum = add_lane_xor<32>(add_lane_xor<16>(sums.sum));
  if (quarter == 0) {
    s_top[wave][c] = sums.top;
    s_sum[wave][c] = sum;
  }
#pragma unroll
  for (int i = 0; i < DH / 16; ++i) *reinterpret_cast<f32x4 *>(&s_o[wave][c][16 * i + 4 * quarter]) = sums.o[i];
  __syncthreads();
  const int heads = min(kHeads, a.s.group - tile * kHeads);
  const bool alone = a.splits == 1;
  for (int i = tid; i < heads * (DH / 4); i += 64 * NW) {
    const int h = i / (DH / 4), e = i % (DH / 4) * 4;
    float top = -INFINITY, total = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, s_top[w][h]);
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = s_top[w][h] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((s_top[w][h] - top) * scale);
      total = fmaf(s_sum[w][h], f, total);
      o += *reinterpret_cast<const f32x4 *>(&s_o[w][h][e]) * f;
    }
    if (alone) {
      const float by = total > 0.f || total != total ? 1.f / total : 0.f;
      T *to = a.out + (size_t(b) * a.s.heads + size_t(hk) * a.s.group + tile * kHeads + h) * DH + e;
#pragma unroll
      for (int j = 0; j < 4; ++j) store_elem(to + j, o[j] * by);
    } else {
      const size_t at = (size_t(blockIdx.x)) * kHeads + h;
      *reinterpret_cast<f32x4 *>(a.part_o + at * DH + e) = o;
      if (e == 0) {
        a.part_ml[2 * at] = top;
        a.part_ml[2 * at + 1] = total;
      }
    }
  }
  if (alone && a.s.tiles == 1 && tid == 0) a.cursor[row] = position + 1;     // (all waves have read it)
}

// Rows that several workgroups shared: their sums together.  A workgroup: a head of a row, a thread: an element.
template <typename T, int DH>
__global__ __launch_bounds__(DH) void ring_join_kernel(const StepArgs<T> a) {
  __shared__ float s_factor[kMaxSplits];
  const int h = blockIdx.x % a.s.group, row = blockIdx.x / a.s.group, e = threadIdx.x, lane = e & 63;
  const size_t first = (size_t(row) * a.s.tiles + h / kHeads) * a.splits * kHeads + h % kHeads;
  if (a.splits > 1) {
    // (every wave for itself: up to 64 parts, one a lane)
    const bool mine = lane < a.splits;
    const size_t at = 2 * (first + size_t(mine ? lane : 0) * kHeads);
    const float top = mine ? a.part_ml[at] : -INFINITY, part = mine ? a.part_ml[at + 1] : 0.f;
    float m = top;
#pragma unroll
    for (int off = 1; off < 64; off *= 2) m = fmaxf(m, __shfl_xor(m, off));
    const float f = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((top - m) * a.s.scale_log2);
    const float total = wave_sum(part * f), by = total > 0.f || total != total ? 1.f / total : 0.f;
    if (e < 64 && mine) s_factor[lane] = f;
    __syncthreads();
    const float *from = a.part_o + first * DH + e;
    float o = 0.f;
#pragma unroll 8
    for (int j = 0; j < a.splits; ++j) o = fmaf(from[size_t(j) * (kHeads * DH)], s_factor[j], o);
    store_elem(a.out + (size_t(row) * a.s.group + h) * DH + e, o * by);
  }
  if (h == 0 && e == 0) a.cursor[row] = max(a.cursor[row], 0) + 1;
}

// ---- rows in and out ---------------------------------------------------------------------------------------------------------
template <typename T>
struct FillArgs {
  RingShape s;
  const int32_t *k_start, *seen;     // either may be null
  int k_tokens;
  Rows<const T> k, v;
  T *cache;
  int32_t *cursor;
};

// A workgroup: a block of a row.  V goes through LDS, where it is turned.
template <typename T, int DH>
__global__ __launch_bounds__(256) void ring_fill_kernel(const FillArgs<T> a) {
  typedef Ring<T, DH> L;
  constexpr int EPL = L::EPL, kRowChunks = DH / EPL;
  __shared__ __align__(16) T s_v[kSlots][DH + EPL];
  // kv head fastest: a token's heads are side by side where prompts are packed
  const int hk = blockIdx.x % a.s.kv_heads, item = blockIdx.x / a.s.kv_heads, block = item % a.s.blocks, b = item / a.s.blocks;
  const int row = b * a.s.kv_heads + hk;
  int first = 0, n = a.k_tokens;
  if (a.k_start) span(a.k_start, b, a.k_tokens, first, n);
  // rows that were left out lie behind the first tokens, and only where the ring has no place for them
  const int seen = a.seen && n >= a.s.slots ? max(a.seen[b], n) : n, held = min(n, a.s.slots);
  if (block == 0 && threadIdx.x == 0) a.cursor[row] = seen;
  if (block * kSlots >= held) return;
  auto token_in = [&](int slot) {            // which of the rows; -1: none
    if (slot >= held) return -1;
    if (slot < a.s.sinks || seen <= a.s.slots) return slot;
    const int last = seen - 1 - a.s.sinks, at = slot - a.s.sinks;      // of the window: positions from the first behind the sinks
    return n - 1 - (last - at) % a.s.window;
  };
  const T *const kp = a.k.p + b * a.k.seq + first * a.k.token + hk * a.k.head, *const vp = a.v.p + b * a.v.seq + first * a.v.token + hk * a.v.head;
  T *const to = a.cache + (size_t(row) * a.s.blocks + block) * (2 * L::kElems);
  for (int i = threadIdx.x; i < kSlots * kRowChunks; i += 256) {
    const int slot = i / kRowChunks, e = i % kRowChunks * EPL, token = token_in(block * kSlots + slot);
    u32x4 k = {0, 0, 0, 0}, v = {0, 0, 0, 0};
    if (token >= 0) {
      k = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(kp + token * a.k.token + e));
      v = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(vp + token * a.v.token + e));
    }
    *reinterpret_cast<u32x4 *>(to + L::k_at(slot, e)) = k;
    *reinterpret_cast<u32x4 *>(&s_v[slot][e]) = v;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < kSlots / EPL * DH; i += 256) {
    const int e = i % 16 + i / (16 * (kSlots / EPL)) * 16, slot = i / 16 % (kSlots / EPL) * EPL;
    T x[EPL];
#pragma unroll
    for (int j = 0; j < EPL; ++j) x[j] = s_v[slot + j][e];
    *reinterpret_cast<u32x4 *>(to + L::kElems + L::v_at(slot, e)) = *reinterpret_cast<const u32x4 *>(x);
  }
}

template <typename T>
struct ReadArgs {
  RingShape s;
  const T *cache;
  const int32_t *cursor;
  T *k, *v;
};

template <typename T, int DH>
__global__ __launch_bounds__(256) void ring_read_kernel(const ReadArgs<T> a) {
  typedef Ring<T, DH> L;
  constexpr int EPL = L::EPL, kRowChunks = DH / EPL;
  __shared__ __align__(16) T s_v[kSlots][DH + EPL];
  const int block = blockIdx.x % a.s.blocks, row = blockIdx.x / a.s.blocks;
  const int position = max(a.cursor[row], 0), held = min(position, a.s.slots);
  const int oldest = position > a.s.slots ? (position - a.s.sinks) % a.s.window : 0;       // of the window's slots
  const T *const from = a.cache + (size_t(row) * a.s.blocks + block) * (2 * L::kElems);
  for (int i = threadIdx.x; i < kSlots / EPL * DH; i += 256) {
    const int e = i % 16 + i / (16 * (kSlots / EPL)) * 16, slot = i / 16 % (kSlots / EPL) * EPL;
    const u32x4 w = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(from + L::kElems + L::v_at(slot, e)));
    T x[EPL];
    *reinterpret_cast<u32x4 *>(x) = w;
#pragma unroll
    for (int j = 0; j < EPL; ++j) s_v[slot + j][e] = x[j];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < kSlots * kRowChunks; i += 256) {
    const int in = i / kRowChunks, slot = block * kSlots + in, e = i % kRowChunks * EPL;
    if (slot >= a.s.slots) continue;
    int place = slot;                        // among the rows in the order of their positions
    if (slot >= a.s.sinks) {
      place = slot - a.s.sinks - oldest;
      if (place < 0) place += a.s.window;
      place += a.s.sinks;
    }
    u32x4 k = {0, 0, 0, 0}, v = {0, 0, 0, 0};
    if (slot < held) {
      k = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(from + L::k_at(in, e)));
      v = *reinterpret_cast<const u32x4 *>(&s_v[in][e]);
    }
    const size_t at = (size_t(row) * a.s.slots + place) * DH + e;
    *reinterpret_cast<u32x4 *>(a.k + at) = k;
    *reinterpret_cast<u32x4 *>(a.v + at) = v;
  }
}

// ---- host ----------------------------------------------------------------------------------------------------------------
int ring_shape(const adore_ring_config *c, RingShape *s) {
  if (!c || c->batch <= 0 || c->heads <= 0 || c->kv_heads <= 0 || c->heads % c->kv_heads != 0 || c->head_dim <= 0 || c->window < 1 || c->sinks < 0 ||
      (c->dtype != ADORE_F32 && c->dtype != ADORE_BF16) || !std::isfinite(c->scale) || c->scale < 0.f)
    return ADORE_E_INVALID;
  if ((c->head_dim != 64 && c->head_dim != 128) || c->window > kMaxSlots || c->sinks > kMaxSlots || c->window + c->sinks > kMaxSlots ||
      c->batch > (1 << 16) || c->heads > (1 << 12) || (long long)c->batch * c->heads > (1 << 20) ||
      (long long)c->batch * c->kv_heads * ((c->window + c->sinks + kSlots - 1) / kSlots) > (1 << 23))
    return ADORE_E_UNSUPPORTED;
  s->batch = c->batch;
  s->heads = c->heads;
  s->kv_heads = c->kv_heads;
  s->group = c->heads / c->kv_heads;
  s->window = c->window;
  s->sinks = c->sinks;
  s->slots = c->window + c->sinks;
  s->blocks = (s->slots + kSlots - 1) / kSlots;
  s->tiles = (s->group + kHeads - 1) / kHeads;
  s->scale_log2 = (c->scale > 0.f ? c->scale : 1.f / sqrtf(float(c->head_dim))) * kLog2e;
  return ADORE_OK;
}

int splits_of(const RingShape &s) {
  const long long groups = (long long)s.batch * s.kv_heads * s.tiles;
  // One workgroup for each unit where rows are few, and two blocks a wave: 4 sequences of 8 kv heads, 16384 slots 46.3 us, with 512
  // workgroups 51.8, 1024 51.8; 1 of 2, 4096 slots 9.9, 9.8 and 10.0; 64 of 8, 1024 slots of 64 elements 23.8, 23.8 and 26.3.
  // A row has kMaxSplits at most, so that fewer than four rows of more than 16384 slots leave units without work: one row of 2^16 slots 23 us
  // (1.5 TB/s), one of 2^20 182 (3.0), two of 2^19 110 (4.9).
  const long long want = (256 + groups - 1) / groups, able = (s.blocks + 2 * kStepWaves - 1) / (2 * kStepWaves);
  const long long n = able <= 1 ? 1 : want < able ? want : able;
  return int(n < kMaxSplits ? n : kMaxSplits);
}

size_t ring_parts(const RingShape &s) { return size_t(s.batch) * s.kv_heads * s.tiles * splits_of(s) * kHeads; }
size_t ring_space(const RingShape &s, int head_dim) {        // never 0: that says "not taken"
  return splits_of(s) == 1 ? 256 : (ring_parts(s) * 2 * 4 + 255) / 256 * 256 + ring_parts(s) * head_dim * 4;
}

template <typename T, int DH>
hipError_t launch_step(const StepArgs<T> &a, hipStream_t st) {
  const unsigned items = unsigned(a.s.batch) * unsigned(a.s.kv_heads) * unsigned(a.s.tiles);
  hipLaunchKernelGGL((ring_step_kernel<T, DH>), dim3(items * unsigned(a.splits)), dim3(64 * kStepWaves), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || (a.splits == 1 && a.s.tiles == 1)) return e;
  hipLaunchKernelGGL((ring_join_kernel<T, DH>), dim3(unsigned(a.s.batch) * unsigned(a.s.heads)), dim3(DH), 0, st, a);
  return hipGetLastError();
}

template <typename T>
int step_typed(const RingShape &s, int head_dim, const void *q, const void *k_new, const void *v_new, void *cache, int32_t *cursor, void *out,
               void *workspace, hipStream_t st) {
  StepArgs<T> a;
  a.s = s;
  a.q = static_cast<const T *>(q);
  a.k_new = static_cast<const T *>(k_new);
  a.v_new = static_cast<const T *>(v_new);
  a.cache = static_cast<T *>(cache);
  a.out = static_cast<T *>(out);
  a.cursor = cursor;
  a.splits = splits_of(s);
  a.part_ml = static_cast<float *>(workspace);
  a.part_o = a.part_ml + (ring_parts(s) * 2 * 4 + 255) / 256 * 64;
  const hipError_t e = head_dim == 128 ? launch_step<T, 128>(a, st) : launch_step<T, 64>(a, st);
  return e == hipSuccess ? ADORE_OK : ADORE_E_HIP;
}

template <typename T>
int fill_typed(const RingShape &s, int head_dim, const int32_t *k_start, int k_tokens, const adore_rows *k, const adore_rows *v, const int32_t *seen,
               void *cache, int32_t *cursor, hipStream_t st) {
  const FillArgs<T> a{s, k_start, seen, k_tokens, rows_of<const T>(k), rows_of<const T>(v), static_cast<T *>(cache), cursor};
  const dim3 grid(unsigned(s.batch) * unsigned(s.kv_heads) * unsigned(s.blocks));
  if (head_dim == 128)
    hipLaunchKernelGGL((ring_fill_kernel<T, 128>), grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((ring_fill_kernel<T, 64>), grid, dim3(256), 0, st, a);
  return hipGetLastError() == hipSuccess ? ADORE_OK : ADORE_E_HIP;
}

template <typename T>
int read_typed(const RingShape &s, int head_dim, const void *cache, const int32_t *cursor, void *k, void *v, hipStream_t st) {
  const ReadArgs<T> a{s, static_cast<const T *>(cache), cursor, static_cast<T *>(k), static_cast<T *>(v)};
  const dim3 grid(unsigned(s.batch) * unsigned(s.kv_heads) * unsigned(s.blocks));
  if (head_dim == 128)
    hipLaunchKernelGGL((ring_read_kernel<T, 128>), grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((ring_read_kernel<T, 64>), grid, dim3(256), 0, st, a);
  return hipGetLastError() == hipSuccess ? ADORE_OK : ADORE_E_HIP;
}

bool aligned(const void *p, uintptr_t to) { return p && (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

}  // namespace

}  // namespace adore

extern "C" {

size_t adore_ring_cache_bytes(const adore_ring_config *cfg) {
  adore::RingShape s;
  if (adore::ring_shape(cfg, &s) != ADORE_OK) return 0;
  return size_t(s.batch) * s.kv_heads * s.blocks * 64 * cfg->head_dim * (cfg->dtype == ADORE_BF16 ? 2 : 4);
}

size_t adore_ring_workspace_bytes(const adore_ring_config *cfg) {
  adore::RingShape s;
  return adore::ring_shape(cfg, &s) == ADORE_OK ? adore::ring_space(s, cfg->head_dim) : 0;
}

int adore_ring_fill(const adore_ring_config *cfg, const int32_t *k_start, int32_t k_tokens, const adore_rows *k, const adore_rows *v,
                    const int32_t *seen, void *cache, int32_t *cursor, void *hip_stream) {
  using namespace adore;
  RingShape s;
  const int rc = ring_shape(cfg, &s);
  if (rc != ADORE_OK) return rc;
  if (k_tokens < 0 || !prompt_rows_ok(k, cfg->dtype) || !prompt_rows_ok(v, cfg->dtype) || !aligned(cache, 256) || !aligned(cursor, 4))
    return ADORE_E_INVALID;
  if (k_tokens > (1 << 24)) return ADORE_E_UNSUPPORTED;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return cfg->dtype == ADORE_BF16 ? fill_typed<bf16_t>(s, cfg->head_dim, k_start, k_tokens, k, v, seen, cache, cursor, st)
                                  : fill_typed<float>(s, cfg->head_dim, k_start, k_tokens, k, v, seen, cache, cursor, st);
}

int adore_ring_step(const adore_ring_config *cfg, const void *q, const void *k_new, const void *v_new, void *cache, int32_t *cursor, void *out,
                    void *workspace, size_t workspace_bytes, void *hip_stream) {
  using namespace adore;
  RingShape s;
  const int rc = ring_shape(cfg, &s);
  if (rc != ADORE_OK) return rc;
  if (!aligned(q, 16) || !aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(out, 16) || !aligned(cache, 256) || !aligned(cursor, 4) || !workspace)
    return ADORE_E_INVALID;
  if (!aligned(workspace, 256) || workspace_bytes < ring_space(s, cfg->head_dim)) return ADORE_E_WORKSPACE;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return cfg->dtype == ADORE_BF16 ? step_typed<bf16_t>(s, cfg->head_dim, q, k_new, v_new, cache, cursor, out, workspace, st)
                                  : step_typed<float>(s, cfg->head_dim, q, k_new, v_new, cache, cursor, out, workspace, st);
}

int adore_ring_read(const adore_ring_config *cfg, const void *cache, const int32_t *cursor, void *k, void *v, void *hip_stream) {
  using namespace adore;
  RingShape s;
  const int rc = ring_shape(cfg, &s);
  if (rc != ADORE_OK) return rc;
  if (!aligned(cache, 256) || !aligned(cursor, 4) || !aligned(k, 16) || !aligned(v, 16)) return ADORE_E_INVALID;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return cfg->dtype == ADORE_BF16 ? read_typed<bf16_t>(s, cfg->head_dim, cache, cursor, k, v, st)
                                  : read_typed<float>(s, cfg->head_dim, cache, cursor, k, v, st);
}

}  // extern "C"
