// Norms of queries and keys per head and the rotation by their tokens' positions, in one pass over a projection's rows; and its gradients.
//
//   r = 1 / sqrt(mean x^2 + eps);  y = x r w        (a tensor without weights: y = x)
//   pair j < R / 2 of a head's first R elements, (j, j + R / 2) or (2 j, 2 j + 1), and t = position f_j:
//     out_a = m (y_a cos t - y_b sin t),  out_b = m (y_a sin t + y_b cos t)         the other elements: out = y
//   g = the same with -t of d_out;  dw = sum over rows of g x r;  dx = r (w g - x r mean(w g x r))
//
// Angles are counted in turns, 2^64 of them a whole one: f_j / 2 pi is a 64-bit fraction made once on the host, position times it is one
// integer product whose overflow is the whole turns that do not matter, and no table has an end.  The product is rounded to 2^-32 turns; the
// fraction's own error, 2^-65 turns and 2^-62 of the frequency, grows with the position: with frequencies of up to a radian less than 2^-32 turns
// at 2^31.  The nearest quarter turn off, sine and cosine are their Taylor series up to pi / 4, within 2^-24, with their argument's two roundings
// within 1.6 of it.
//
// Bound by memory: a row is read once and written once.  A row of DH elements is DH / 16 lanes, 8 elements of each half of the pairs a lane
// (two loads of 16 bytes in bf16), and a wave takes a run of one token's heads, so that sines are made once for up to eight rows.
// 14578 tokens of 32 and 32 heads of 128 in bf16 93 us, 5.1 TB/s, which is what a large copy reaches (75 us where the results' memory was written
// just before and the last level holds it); 29159 of 32 and 8 with norms 109 us (5.5 TB/s), their gradients 195 (4.6: two tensors in, one out,
// vector instructions in 68 % of the cycles) and 4.5 for the weights' sums; 14579 of 32 and 8 with norms in fp32 137 us (4.4 TB/s), their gradients 210 (4.3).
#include <hip/hip_runtime.h>

#include <cmath>

#include "prompt_device.h"

namespace adore {

namespace {

struct RotateShape {
  int batch, heads, kv_heads, tokens;        // (kv_heads may be 0: no k)
  long long all;                             // tokens of all sequences
  int rotary, interleaved;
  float magnitude, eps, sign;                // sign -1: the other way round
  const uint64_t *turns;
  const int32_t *positions;
  int64_t pos_seq, pos_token;
  const float *weight[2];                    // of q and k; either may be null
};

// How a launch is cut: a wave has 1024 / DH groups of lanes, `wide` tokens of them side by side (a power of two), the others are heads;
// a token's heads are cut into `parts` waves.
struct RotatePlan {
  int wide, parts;
  long long waves;
};

// Rows of a group whose loads are under way together, one / two / four (us): 16384 tokens of 64 heads of 128 106.5 / 103.7 / 99.7, as part of a
// layer without a difference; 4096 of 40 18.3 / 17.8 / 18.3; with norms 16384 of 40 heads of 64 41.5 / 41.8 / 44.7, 29159 of 128 115 / 114 / 123.
constexpr int kRowsAtOnce = 2;

template <typename T>
struct Eight;                                // eight elements, as they are
template <>
struct Eight<bf16_t> {
  u32x4 u;
  // Not kept by the caches, which then hold the results for attention: a projection to 32 and 8 heads of 128, rotation and attention of
  // 16384 tokens take 382 us instead of 393, of 32768 767 for 780, of 4096 108 either way.  (With norms 393 for 400; alone, where nothing
  // reads the results, 29159 normed tokens 109 for 101 and their gradients 192 for 200.)  Also where pairs lie side by side or a part of the head
  // is turned, whose lanes' two loads share a line: 16384 tokens of 32 and 8 heads of 128, behind something that has filled the caches, side by
  // side 76.5 us for 89.0, 64 elements turned 75.4 for 88.6; with a projection and attention with a window around them 905 for 900 and 898 for 893.
  __device__ __forceinline__ void load(const bf16_t *p) { u = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p)); }
  __device__ __forceinline__ void none() { u = u32x4{0, 0, 0, 0}; }
  __device__ __forceinline__ void values(float *f) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(u[i] << 16);
      f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
  __device__ static __forceinline__ void store(bf16_t *p, const float *f) {
    *reinterpret_cast<u32x4 *>(p) = u32x4{pair_bf16(f[0], f[1]), pair_bf16(f[2], f[3]), pair_bf16(f[4], f[5]), pair_bf16(f[6], f[7])};
  }
};
template <>
struct Eight<float> {
  f32x4 a, b;
  // In fp32 past the caches loses: 115.7 us, so read 122.7 (14579 tokens of 32 and 8 heads).
  __device__ __forceinline__ void load(const float *p) {
    a = *reinterpret_cast<const f32x4 *>(p);
    b = *reinterpret_cast<const f32x4 *>(p + 4);
  }
  __device__ __forceinline__ void none() { a = b = f32x4{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ void values(float *f) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[i] = a[i];
      f[4 + i] = b[i];
    }
  }
  __device__ static __forceinline__ void store(float *p, const float *f) {
    *reinterpret_cast<f32x4 *>(p) = f32x4{f[0], f[1], f[2], f[3]};
    *reinterpret_cast<f32x4 *>(p + 4) = f32x4{f[4], f[5], f[6], f[7]};
  }
};

// Cosine and sine of t / 2^32 turns.
__device__ __forceinline__ void turn(int32_t t, float &cos_t, float &sin_t) {
  const int32_t quarter = int32_t(uint32_t(t) + (1u << 29)) >> 30;
  const float x = float(int32_t(uint32_t(t) - (uint32_t(quarter) << 30))) * 1.46291807926715968e-9f;   // pi / 2 / 2^30: radians, up to pi / 4
  const float z = x * x;
  float s = fmaf(z, 2.75573192e-6f, -1.98412698e-4f);       // x^9 / 9! ..; the next term is below 2^-28
  s = fmaf(z, s, 8.33333333e-3f);
  s = fmaf(z, s, -1.66666667e-1f);
  s = fmaf(x * z, s, x);
  float c = fmaf(z, -2.75573192e-7f, 2.48015873e-5f);       // x^10 / 10! ..; the next term is below 2^-32
  c = fmaf(z, c, -1.38888889e-3f);
  c = fmaf(z, c, 4.16666667e-2f);
  c = fmaf(z, c, -0.5f);
  c = fmaf(z, c, 1.f);
  const bool odd = quarter & 1;
  const float u = odd ? c : s, v = odd ? s : c;
  sin_t = __uint_as_float(__float_as_uint(u) ^ (uint32_t(quarter & 2) << 30));
  cos_t = __uint_as_float(__float_as_uint(v) ^ (uint32_t((quarter + 1) & 2) << 30));
}

// What a lane has of every row: its place in the row, its eight pairs.
template <int DH>
struct Lane {
  static constexpr int G = DH / 16;          // lanes of a row
  int first, second;                         // its two runs of eight elements
  int pair;                                  // its first pair; -1: elements that are not turned
  __device__ __forceinline__ Lane(const RotateShape &s, int lane) {
    const int l = lane % G, turned = s.rotary / 16;
    pair = l < turned ? 8 * l : -1;
    if (l >= turned || s.interleaved) {
      first = 16 * l;
      second = first + 8;
    } else {
      first = 8 * l;
      second = first + s.rotary / 2;
    }
  }
};

// Cosines and sines of a token's pairs, times the magnitude (1 and 0 for elements that are not turned, whose lanes do not use them: an infinity times
// 0 would be another element's NaN).
__device__ __forceinline__ void angles(const RotateShape &s, int pair, long long token, bool there, float (&cs)[8], float (&sn)[8]) {
  if (pair < 0 || !there) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      cs[i] = 1.f;
      sn[i] = 0.f;
    }
    return;
  }
  const long long b = token / s.tokens, t = token - b * s.tokens;
  const uint64_t position = uint64_t(int64_t(s.positions[b * s.pos_seq + t * s.pos_token]));
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint64_t at = s.turns[pair + i] * position + (1ull << 31);
    turn(int32_t(uint32_t(at >> 32)), cs[i], sn[i]);
    cs[i] *= s.magnitude;
    sn[i] *= s.magnitude * s.sign;
  }
}

// The rotation of a lane's 16 elements: f[0 .. 7] its first run, f[8 .. 15] its second.
__device__ __forceinline__ void rotated(float (&f)[16], const float (&cs)[8], const float (&sn)[8], bool side_by_side) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = side_by_side ? f[2 * i] : f[i], b = side_by_side ? f[2 * i + 1] : f[8 + i];
    const float x = fmaf(a, cs[i], -(b * sn[i])), y = fmaf(a, sn[i], b * cs[i]);
    (side_by_side ? f[2 * i] : f[i]) = x;
    (side_by_side ? f[2 * i + 1] : f[8 + i]) = y;
  }
}

// The mean of a row's squares, of which a lane has 16 elements; all 64 lanes of a wave call it together.  The mean may be a number where the
// sum is beyond fp32, or one of the squares: then once more of sixteenths, whose squares add up to at most half the mean.
template <int DH>
__device__ __forceinline__ float mean_of_squares(const float (&f)[16]) {
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) sum = fmaf(f[i], f[i], sum);
  float mean = group_sum<DH / 16>(sum) * (1.f / DH);
  if (__builtin_amdgcn_ballot_w64(!(mean < INFINITY))) {
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) sum = fmaf(f[i] * 0.0625f, f[i] * 0.0625f, sum);
    sum = group_sum<DH / 16>(sum) * (256.f / DH);
    if (!(mean < INFINITY)) mean = sum;
  }
  return mean;
}

// A wave's item: a token for each lane, and the heads of the wave's groups of lanes: first + mine, then `step` further on.
struct Item {
  long long token;
  int first, mine, step;
  bool there;
};
template <int DH>
__device__ __forceinline__ Item item_of(const RotateShape &s, const RotatePlan &p, long long item, int lane) {
  constexpr int NG = 64 / (DH / 16);
  const int group = lane / (DH / 16), side = NG / p.wide;
  Item it;
  it.token = item / p.parts * p.wide + group / side;
  it.first = int(item % p.parts) * side;
  it.mine = group % side;
  it.step = p.parts * side;
  it.there = it.token < s.all;
  return it;
}

// Rows of q's and k's heads of one token.
template <typename T>
struct TokenRows {
  T *p[2];
  int64_t head[2];
  int heads;
  __device__ __forceinline__ TokenRows(const Rows<T> (&r)[2], const RotateShape &s, const Item &it) : heads(s.heads) {
    const long long b = it.there ? it.token / s.tokens : 0, t = it.there ? it.token - b * s.tokens : 0;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      p[k] = r[k].p + b * r[k].seq + t * r[k].token;
      head[k] = r[k].head;
    }
  }
  __device__ __forceinline__ T *operator()(int h) const { return h < heads ? p[0] + h * head[0] : p[1] + (h - heads) * head[1]; }
};

template <typename T>
struct RotateArgs {
  RotateShape s;
  RotatePlan p;
  Rows<const T> in[2];                       // q, k; the backward pass: gradients of what came of them
  Rows<const T> x[2];                        // the backward pass of norms: q, k
  Rows<T> out[2];
  float *part;                               // ... [workgroup][q, k][DH]: sums of the weights' gradients
};

template <int DH>
__device__ __forceinline__ void lane_weights(const RotateShape &s, const Lane<DH> &mine, float (&w)[2][16]) {
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int i = 0; i < 16; ++i) w[k][i] = s.weight[k] ? s.weight[k][(i < 8 ? mine.first : mine.second - 8) + i] : 1.f;
}

template <typename T, int DH, bool SIDE, bool NORM>
__global__ __launch_bounds__(256) void rotate_heads_kernel(const RotateArgs<T> a) {
  constexpr int U = kRowsAtOnce;
  const int lane = threadIdx.x & 63, all = a.s.heads + a.s.kv_heads;
  const Lane<DH> mine(a.s, lane);
  float w[2][16];
  if constexpr (NORM) lane_weights<DH>(a.s, mine, w);
  for (long long item = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); item < a.p.waves; item += (long long)gridDim.x * 4) {
    const Item it = item_of<DH>(a.s, a.p, item, lane);
    const TokenRows<const T> from(a.in, a.s, it);
    const TokenRows<T> to(a.out, a.s, it);
    float cs[8], sn[8];
    angles(a.s, mine.pair, it.token, it.there, cs, sn);
    for (int h0 = it.first; h0 < all; h0 += U * it.step) {
      Eight<T> x[U][2];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = h0 + u * it.step + it.mine;
        x[u][0].none();
        x[u][1].none();
        if (it.there && h < all) {
          const T *row = from(h);
          x[u][0].load(row + mine.first);
          x[u][1].load(row + mine.second);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = h0 + u * it.step + it.mine, k = h >= a.s.heads;
        float f[16];
        x[u][0].values(f);
        x[u][1].values(f + 8);
        if constexpr (NORM) {
          const float mean = mean_of_squares<DH>(f), r = (k ? a.s.weight[1] : a.s.weight[0]) ? 1.f / sqrtf(mean + a.s.eps) : 1.f;
#pragma unroll
          for (int i = 0; i < 16; ++i) f[i] *= r * (k ? w[1][i] : w[0][i]);
        }
        if (mine.pair >= 0) rotated(f, cs, sn, SIDE);
        if (it.there && h < all) {
          T *row = to(h);
          Eight<T>::store(row + mine.first, f);
          Eight<T>::store(row + mine.second, f + 8);
        }
      }
    }
  }
}

// Rows whose terms a lane adds up one after the other for the weights' gradients, before the wave's lanes are added up and taken over: so
// that what additions lose does not grow with the tokens.  2^20 tokens of 32 equal heads, 2048 rows a lane: worst off by 28 of 2^-24, in one go
// 501; gradients of 29159 tokens of 32 and 8 heads of 128 194 us, in one go 191.5 (128 and 256 rows: 193 to 194 too).
constexpr int kRowsInARow = 64;
constexpr int kRowsOfItem = 8;               // at most

// Gradients where there are norms.  A lane adds up what its elements give the weights over its rows, a wave its lanes, a workgroup its waves, and
// rotate_weights_kernel the workgroups: no atomics, equal inputs give equal bits.
template <typename T, int DH, bool SIDE>
__global__ __launch_bounds__(256) void rotate_backward_kernel(const RotateArgs<T> a) {
  constexpr int U = 1, G = DH / 16;          // (rows at once; two: 76.8 us for 71.4, 16384 tokens of 32 and 8 heads of 64)
  __shared__ __align__(16) float s_sum[4][2][DH];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, all = a.s.heads + a.s.kv_heads;
  const Lane<DH> mine(a.s, lane);
  float w[2][16], dw[2][16];
  lane_weights<DH>(a.s, mine, w);
#pragma unroll
  for (int i = 0; i < 16; ++i) dw[0][i] = dw[1][i] = 0.f;
  float *const sums = s_sum[wave][0];        // (the wave's own lanes' only)
  bool taken = false;                        // whether sums are there already
  int rows = 0;                              // since sums were taken over
  for (long long item = (long long)blockIdx.x * 4 + wave; item < a.p.waves; item += (long long)gridDim.x * 4) {
    const Item it = item_of<DH>(a.s, a.p, item, lane);
    const TokenRows<const T> from(a.in, a.s, it), xs(a.x, a.s, it);
    const TokenRows<T> to(a.out, a.s, it);
    float cs[8], sn[8];
    angles(a.s, mine.pair, it.token, it.there, cs, sn);
    for (int h0 = it.first; h0 < all; h0 += U * it.step) {
      Eight<T> d[U][2], x[U][2];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = h0 + u * it.step + it.mine;
        d[u][0].none();
        d[u][1].none();
        x[u][0].none();
        x[u][1].none();
        if (it.there && h < all) {
          const T *row = from(h);
          d[u][0].load(row + mine.first);
          d[u][1].load(row + mine.second);
          if (h < a.s.heads ? a.s.weight[0] : a.s.weight[1]) {
            row = xs(h);
            x[u][0].load(row + mine.first);
            x[u][1].load(row + mine.second);
          }
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = h0 + u * it.step + it.mine, k = h >= a.s.heads;
        float g[16], f[16];
        d[u][0].values(g);
        d[u][1].values(g + 8);
        if (mine.pair >= 0) rotated(g, cs, sn, SIDE);
        x[u][0].values(f);
        x[u][1].values(f + 8);
        float dot = 0.f;
        const float r = 1.f / sqrtf(mean_of_squares<DH>(f) + a.s.eps);
        const bool some = it.there && h < all, normed = k ? a.s.weight[1] : a.s.weight[0];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          f[i] *= r;                                             // the normed row
          if (some && normed) {
            dw[0][i] += k ? 0.f : g[i] * f[i];
            dw[1][i] += k ? g[i] * f[i] : 0.f;
          }
          g[i] *= k ? w[1][i] : w[0][i];
          dot = fmaf(g[i], f[i], dot);
        }
        dot = group_sum<G>(dot) * (1.f / DH);
        if (normed) {
#pragma unroll
          for (int i = 0; i < 16; ++i) g[i] = r * fmaf(-f[i], dot, g[i]);
        }
        if (some) {
          T *row = to(h);
          Eight<T>::store(row + mine.first, g);
          Eight<T>::store(row + mine.second, g + 8);
        }
      }
      rows += U;
    }
    if (rows <= kRowsInARow - kRowsOfItem && item + (long long)gridDim.x * 4 < a.p.waves) continue;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        dw[k][i] = add_lane_xor<32>(add_lane_xor<16>(add_lane_xor<8>(dw[k][i])));
        if constexpr (G == 4) dw[k][i] = add_lane_xor<4>(dw[k][i]);
      }
    auto fours = [&](auto what) {
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < 16; i += 4) what(*reinterpret_cast<f32x4 *>(sums + k * DH + (i < 8 ? mine.first : mine.second - 8) + i), &dw[k][i]);
    };
    if (lane < G) {
      if (taken)
        fours([](const f32x4 &sum, float *x) {
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] += sum[i];
        });
      fours([](f32x4 &sum, const float *x) { sum = f32x4{x[0], x[1], x[2], x[3]}; });
    }
    fours([](const f32x4 &, float *x) { x[0] = x[1] = x[2] = x[3] = 0.f; });
    rows = 0;
    taken = true;
  }
  if (!taken)
    for (int i = lane; i < 2 * DH; i += 64) sums[i] = 0.f;
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * DH; i += 256) {
    const float *const s = &s_sum[0][0][0] + i;
    a.part[size_t(blockIdx.x) * (2 * DH) + i] = (s[0] + s[2 * DH]) + (s[4 * DH] + s[6 * DH]);
  }
}

// The workgroups' sums added up: 8 columns of the 2 DH a workgroup, 32 threads a column.
template <int DH>
__global__ __launch_bounds__(256) void rotate_weights_kernel(const float *part, int n, float *dq_weight, float *dk_weight) {
  __shared__ float s_sum[32][8];
  const int column = threadIdx.x & 7, row = threadIdx.x >> 3, at = blockIdx.x * 8 + column;
  float sum = 0.f;
#pragma unroll 16
  for (int i = row; i < n; i += 32) sum += part[size_t(i) * (2 * DH) + at];
  s_sum[row][column] = sum;
  __syncthreads();
  for (int half = 16; half > 0; half >>= 1) {
    if (row < half) s_sum[row][column] += s_sum[row + half][column];
    __syncthreads();
  }
  float *const to = at < DH ? dq_weight : dk_weight;
  if (row == 0 && to) to[at < DH ? at : at - DH] = s_sum[0][column];
}

// ---- host ----------------------------------------------------------------------------------------------------------------
constexpr long long kMostParts = 512;        // workgroups whose sums of the weights' gradients are added up: two a unit (a third would have a place)

int rotate_shape(const adore_rotate_config *c, RotateShape *s) {
  if (!c || c->batch <= 0 || c->heads <= 0 || c->kv_heads < 0 || c->tokens < 0 || (c->dtype != ADORE_F32 && c->dtype != ADORE_BF16) ||
      c->head_dim <= 0 || c->rotary_dim < 0 || c->rotary_dim > c->head_dim || !std::isfinite(c->magnitude) || c->magnitude < 0.f ||
      !std::isfinite(c->eps) || c->eps < 0.f)
    return ADORE_E_INVALID;
  if ((c->head_dim != 64 && c->head_dim != 128) || c->rotary_dim % 16 != 0 || c->tokens > (1 << 24) || c->batch > (1 << 16) ||
      c->heads > (1 << 12) || c->kv_heads > (1 << 12))
    return ADORE_E_UNSUPPORTED;
  s->batch = c->batch;
  s->heads = c->heads;
  s->kv_heads = c->kv_heads;
  s->tokens = c->tokens;
  s->all = (long long)c->batch * c->tokens;
  s->rotary = c->rotary_dim;
  s->interleaved = c->interleaved != 0;
  s->magnitude = c->magnitude > 0.f ? c->magnitude : 1.f;
  s->eps = c->eps;
  s->sign = 1.f;
  return ADORE_OK;
}

RotatePlan plan_rotation(const RotateShape &s, int head_dim) {
  const int groups = 64 / (head_dim / 16), all = s.heads + s.kv_heads;
  RotatePlan p;
  int side = groups;
  while (side > 1 && side / 2 >= all) side /= 2;
  p.wide = groups / side;
  const long long steps = (all + side - 1) / side, tokens = (s.all + p.wide - 1) / p.wide;
  // A head of a group each where that leaves units without work, else up to eight, for which sines are made once (us, a head each / up to
  // eight): 64 tokens of 40 heads of 128 4.3 / 5.7, gradients with norms 13.0 / 16.3; 256 5.0 / 5.9 and 15.7 / 16.8; 500 of 64 7.4 / 7.5
  // and 21.2 / 17.8; 1000 of 40 8.4 / 6.9 and 23.3 / 18.4; 4000 23.1 / 15.3 and 69 / 36.
  p.parts = int(tokens * steps <= 2560 ? steps : (steps + kRowsOfItem - 1) / kRowsOfItem);
  p.waves = tokens * p.parts;
  return p;
}

unsigned groups_of(const RotatePlan &p, long long most) {
  const long long n = (p.waves + 3) / 4;
  return unsigned(n < 1 ? 1 : n < most ? n : most);        // (without tokens: one, whose sums are zeros)
}

template <typename T, int DH>
hipError_t launch_rotation(const RotateArgs<T> &a, hipStream_t st) {
  const dim3 grid(groups_of(a.p, 1 << 20)), block(256);
  const bool norm = a.s.weight[0] || a.s.weight[1];
  if (a.s.interleaved) {
    if (norm)
      hipLaunchKernelGGL((rotate_heads_kernel<T, DH, true, true>), grid, block, 0, st, a);
    else
      hipLaunchKernelGGL((rotate_heads_kernel<T, DH, true, false>), grid, block, 0, st, a);
  } else {
    if (norm)
      hipLaunchKernelGGL((rotate_heads_kernel<T, DH, false, true>), grid, block, 0, st, a);
    else
      hipLaunchKernelGGL((rotate_heads_kernel<T, DH, false, false>), grid, block, 0, st, a);
  }
  return hipGetLastError();
}

template <typename T, int DH>
hipError_t launch_rotation_backward(RotateArgs<T> a, float *dq_weight, float *dk_weight, hipStream_t st) {
  a.s.sign = -1.f;
  if (!a.s.weight[0] && !a.s.weight[1]) return launch_rotation<T, DH>(a, st);
  const unsigned n = groups_of(a.p, kMostParts);
  if (a.s.interleaved)
    hipLaunchKernelGGL((rotate_backward_kernel<T, DH, true>), dim3(n), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((rotate_backward_kernel<T, DH, false>), dim3(n), dim3(256), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((rotate_weights_kernel<DH>), dim3(2 * DH / 8), dim3(256), 0, st, a.part, int(n), dq_weight, dk_weight);
  return hipGetLastError();
}

template <typename T>
Rows<T> rows_or_none(const adore_rows *r) {
  return r ? rows_of<T>(r) : Rows<T>{nullptr, 0, 0, 0};
}

template <typename T>
int rotate_typed(const RotateShape &s, int head_dim, const adore_rows *q, const adore_rows *k, const adore_rows *q_out, const adore_rows *k_out,
                 hipStream_t st) {
  RotateArgs<T> a = {};
  a.s = s;
  a.p = plan_rotation(s, head_dim);
  a.in[0] = rows_of<const T>(q);
  a.in[1] = rows_or_none<const T>(k);
  a.out[0] = rows_of<T>(q_out);
  a.out[1] = rows_or_none<T>(k_out);
  const hipError_t e = head_dim == 128 ? launch_rotation<T, 128>(a, st) : launch_rotation<T, 64>(a, st);
  return e == hipSuccess ? ADORE_OK : ADORE_E_HIP;
}

template <typename T>
int backward_typed(const RotateShape &s, int head_dim, const adore_rows *d_q, const adore_rows *d_k, const adore_rows *q, const adore_rows *k,
                   const adore_rows *dq, const adore_rows *dk, float *dq_weight, float *dk_weight, void *workspace, hipStream_t st) {
  RotateArgs<T> a = {};
  a.s = s;
  a.p = plan_rotation(s, head_dim);
  a.in[0] = rows_of<const T>(d_q);
  a.in[1] = rows_or_none<const T>(d_k);
  a.x[0] = rows_or_none<const T>(q);
  a.x[1] = rows_or_none<const T>(k);
  a.out[0] = rows_of<T>(dq);
  a.out[1] = rows_or_none<T>(dk);
  a.part = static_cast<float *>(workspace);
  const hipError_t e = head_dim == 128 ? launch_rotation_backward<T, 128>(a, dq_weight, dk_weight, st)
                                       : launch_rotation_backward<T, 64>(a, dq_weight, dk_weight, st);
  return e == hipSuccess ? ADORE_OK : ADORE_E_HIP;
}

size_t rotate_space(const RotateShape &s, int head_dim) {
  return size_t(groups_of(plan_rotation(s, head_dim), kMostParts)) * 2 * head_dim * sizeof(float) + 256;      // never 0: that says "not taken"
}

bool multiple(const void *p, uintptr_t of) { return (reinterpret_cast<uintptr_t>(p) & (of - 1)) == 0; }

// What both calls look at.
int rotate_inputs(const adore_rotate_config *c, const uint64_t *turns, const int32_t *positions, int64_t pos_seq, int64_t pos_token,
                  const float *q_weight, const float *k_weight, RotateShape *s) {
  const int rc = rotate_shape(c, s);
  if (rc != ADORE_OK) return rc;
  if ((c->rotary_dim > 0 && (!turns || !positions)) || !multiple(turns, 8) || !multiple(positions, 4) || pos_seq < 0 || pos_token < 0 ||
      !multiple(q_weight, 16) || !multiple(k_weight, 16) || (c->kv_heads == 0 && k_weight))
    return ADORE_E_INVALID;
  s->turns = turns;
  s->positions = positions;
  s->pos_seq = pos_seq;
  s->pos_token = pos_token;
  s->weight[0] = q_weight;
  s->weight[1] = k_weight;
  return ADORE_OK;
}

// q's rows, and k's where there are heads of it.
bool both_ok(const adore_rotate_config *c, const adore_rows *q, const adore_rows *k) {
  return prompt_rows_ok(q, c->dtype) && (c->kv_heads == 0 ? k == nullptr : prompt_rows_ok(k, c->dtype));
}

}  // namespace

}  // namespace adore

extern "C" {

int adore_rotary_turns(int32_t rotary_dim, double base, double factor, double original, double low, double high, uint64_t *turns) {
  if (rotary_dim <= 0 || rotary_dim % 2 != 0 || !turns || !std::isfinite(base) || !(base > 0.0) || !std::isfinite(factor) || !(factor > 0.0) ||
      !std::isfinite(original) || original < 0.0)
    return ADORE_E_INVALID;
  const bool by_parts = original > 0.0;
  if (by_parts && (!std::isfinite(low) || !std::isfinite(high) || !(low < high))) return ADORE_E_INVALID;
  const long double two_pi = 6.283185307179586476925286766559005768L;
  for (int j = 0; j < rotary_dim / 2; ++j) {
    const long double f = powl((long double)base, -2.0L * j / rotary_dim);
    long double whole = 0.0L;                  // what share of the frequency is left as it is
    if (by_parts) {
      whole = (original * f / two_pi - low) / ((long double)high - low);
      whole = whole < 0.0L ? 0.0L : whole > 1.0L ? 1.0L : whole;
    }
    const long double t = f * (whole + (1.0L - whole) / factor) / two_pi;
    if (!(t < 4294967296.0L)) return ADORE_E_INVALID;       // (whole turns do not matter, fractions of them have to be there)
    const long double scaled = (t - floorl(t)) * 18446744073709551616.0L;
    turns[j] = scaled >= 18446744073709551615.5L ? 0 : uint64_t(scaled + 0.5L);
  }
  return ADORE_OK;
}

int adore_rotate_heads(const adore_rotate_config *cfg, const uint64_t *turns, const int32_t *positions, int64_t pos_seq, int64_t pos_token,
                       const float *q_weight, const float *k_weight, const adore_rows *q, const adore_rows *k, const adore_rows *q_out,
                       const adore_rows *k_out, void *hip_stream) {
  using namespace adore;
  RotateShape s;
  const int rc = rotate_inputs(cfg, turns, positions, pos_seq, pos_token, q_weight, k_weight, &s);
  if (rc != ADORE_OK) return rc;
  if (!both_ok(cfg, q, k) || !both_ok(cfg, q_out, k_out)) return ADORE_E_INVALID;
  if (s.all == 0) return ADORE_OK;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return cfg->dtype == ADORE_BF16 ? rotate_typed<bf16_t>(s, cfg->head_dim, q, k, q_out, k_out, st)
                                  : rotate_typed<float>(s, cfg->head_dim, q, k, q_out, k_out, st);
}

size_t adore_rotate_backward_workspace_bytes(const adore_rotate_config *cfg) {
  adore::RotateShape s;
  return adore::rotate_shape(cfg, &s) == ADORE_OK ? adore::rotate_space(s, cfg->head_dim) : 0;
}

int adore_rotate_heads_backward(const adore_rotate_config *cfg, const uint64_t *turns, const int32_t *positions, int64_t pos_seq,
                                int64_t pos_token, const float *q_weight, const float *k_weight, const adore_rows *d_q_out,
                                const adore_rows *d_k_out, const adore_rows *q, const adore_rows *k, const adore_rows *dq, const adore_rows *dk,
                                float *dq_weight, float *dk_weight, void *workspace, size_t workspace_bytes, void *hip_stream) {
  using namespace adore;
  RotateShape s;
  const int rc = rotate_inputs(cfg, turns, positions, pos_seq, pos_token, q_weight, k_weight, &s);
  if (rc != ADORE_OK) return rc;
  if (!both_ok(cfg, d_q_out, d_k_out) || !both_ok(cfg, dq, dk) || (q_weight && !prompt_rows_ok(q, cfg->dtype)) ||
      (k_weight && !prompt_rows_ok(k, cfg->dtype)) || (q_weight != nullptr) != (dq_weight != nullptr) ||
      (k_weight != nullptr) != (dk_weight != nullptr) || !multiple(dq_weight, 4) || !multiple(dk_weight, 4))
    return ADORE_E_INVALID;
  const bool norm = q_weight || k_weight;
  if (norm && (!workspace || !multiple(workspace, 256) || workspace_bytes < rotate_space(s, cfg->head_dim))) return ADORE_E_WORKSPACE;
  if (s.all == 0 && !norm) return ADORE_OK;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return cfg->dtype == ADORE_BF16
             ? backward_typed<bf16_t>(s, cfg->head_dim, d_q_out, d_k_out, q, k, dq, dk, dq_weight, dk_weight, workspace, st)
             : backward_typed<float>(s, cfg->head_dim, d_q_out, d_k_out, q, k, dq, dk, dq_weight, dk_weight, workspace, st);
}

}  // extern "C"
