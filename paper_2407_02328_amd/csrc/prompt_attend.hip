// Causal attention over whole prompts (paper Sec. 2.1, Eq. 1 for every token of the prompt) and the attention every key receives
// (Sec. 3.1, baseline 6: what H2O goes by), for packed sequences of any lengths and grouped heads.
//
//   w_ij = scale q_i . k_j,   j <= i + nk - nq;   lse_i = ln sum_j exp w_ij;   out_i = sum_j exp(w_ij - lse_i) v_j
//   received_j = sum over the query heads of j's group and their queries i of exp(w_ij - lse_i)
//
// Forward: a workgroup of four waves takes 128 queries of a head, a wave 32 of them, and goes over the keys once, tile by tile, with
// the running maximum and sum of the softmax (fp32).  S^T = K Q^T leaves a query's weights in two lanes, so the maximum is a tree
// over a lane's registers and one exchange, and P^T is already the right operand of O^T += V^T P^T; V comes out of LDS
// transposed.  P is rounded to the storage type, like every tensor the matrix cores take; its sum is not.
// Bound by the matrix unit and the softmax's vector work, which share a SIMD (a tile of 64 keys and 32 queries: 1024 and some 960 cycles at 128
// elements, 512 and 960 at 64): 2 x 8192 tokens of 32 heads over 4 965 us (1.14 PFLOP/s; a library product of 8192^3 reaches 1.34),
// 16 x 1024 of 32 heads 193 us (0.71), 24 packed sequences of 1 to 2777 tokens at 64 elements 237 us (0.74).  The matrix unit is busy
// 61, 35 and 37 % of these kernels' cycles, vector instructions 57, 45 and 71 %.
//
// With a window (j <= p, and p - j < window or j < sinks, p = i + nk - nq) a workgroup goes over the tiles with first keys and those from
// its first query's window on.  2 x 8192 tokens of 32 heads over 4, window 1020 and 4 first keys, 314 us (0.82 PFLOP/s of what is seen; a wave's 32
// queries go over 18 tiles for the 16 that they see), 24 packed of 1 to 2777 at 64 elements, window 501, 147 us (0.54).  Matrix unit 39 and
// 27 % of the cycles, vector instructions 45 and 67 %; a window of one key takes 85 and 65 us, mostly queries in and outputs out.  Tiles that
// begin with the window's first key instead of a multiple of their length: 337 us for 320, though some windows have one tile less.
#include <hip/hip_runtime.h>

#include <cfloat>
#include <cmath>

#include "prompt_device.h"

namespace adore {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr double kLn2 = 0.6931471805599453;

template <typename T>
struct AttendArgs {
  PromptShape s;
  Rows<const T> q, k, v;
  Rows<T> out, rest;      // rest.p may be null
  float *lse;             // or null
  bool by_work;
};

// Keys of a tile: 16 KB of K and as much of V at head dimension 128.
template <typename T>
constexpr int kKeys = sizeof(T) == 2 ? 64 : 32;

// REST: P goes in as two bf16 terms (within 2^-16) and what rounding out leaves is handed out, for a backward pass whose delta is as good
// as its other terms.
// WIN: with a window (s.window, s.sinks).
template <typename T, int DH, bool REST, int SW, bool WIN>
__global__ __launch_bounds__(256) ADORE_WAVES(sizeof(T) == 4 || SW > 1 ? 1 : DH == 128 ? 2 : REST ? 3 : 4)
void prompt_attend_kernel(const AttendArgs<T> a) {
  constexpr int NT = 256, BQ = Shared<SW>::kRows, KT = SW > 1 ? 32 * SW : kKeys<T>, KB = SW > 1 ? 1 : KT / 32, DB = DH / 32, ST = DH / 16;
  typedef Tile<T, DH> L;
  typedef typename Operand<T>::type Frag;
  constexpr int kTile = KT * L::kRow;
  extern __shared__ __align__(16) unsigned char smem[];   // two stages of K and V; at the end the outputs
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, h = lane >> 5;
  // kv head fastest: with a multiple of eight of them a head's workgroups share an XCD and its L2
  const int hk = blockIdx.x % a.s.kv_heads, item = blockIdx.x / a.s.kv_heads, head = hk * a.s.group + item % a.s.group;
  Sequence sq;
  int block;
  if (!find_block<BQ, true>(a.s, item / a.s.group, a.by_work, sq, block)) {
    const SpareRows spare = spare_rows<BQ>(a.s.q_start, a.s.batch, a.s.q_tokens, block);
    zero_rows<T, DH>(a.out, head, spare, tid, NT);
    if (REST) zero_rows<T, DH>(a.rest, head, spare, tid, NT);
    if (a.lse && tid < spare.n) a.lse[size_t(head) * a.s.q_tokens + spare.at(tid)] = -INFINITY;
    return;
  }
  const Shared<SW> mate(wave);
  const int q0 = block * BQ + mate.rows * 32, off = sq.nk - sq.nq;
  const int rows = min(32, sq.nq - q0);        // may be <= 0
  const char *kp = reinterpret_cast<const char *>(a.k.p + sq.b * a.k.seq + sq.k_first * a.k.token + hk * a.k.head);
  const char *vp = reinterpret_cast<const char *>(a.v.p + sq.b * a.v.seq + sq.k_first * a.v.token + hk * a.v.head);

  const int last = min(block * BQ + BQ, sq.nq) - 1 + off;             // the last key that a query of the workgroup sees
  const int upto = last < 0 ? 0 : last / KT + 1;
  const WindowTiles<KT> win(a.s, block * BQ + off, last, upto);       // (WIN)
  const int tiles = WIN ? win.total : upto;
  const int mine = rows > 0 ? q0 + rows - 1 + off : -1;               // ... of the wave
  const int seen = q0 + c + off;                                      // ... of the lane
  const float scale = a.s.scale_log2;
  const uint32_t base0 = __builtin_amdgcn_readfirstlane(lds_offset(smem)), share = base0 + uint32_t(wave) * 1024u;
  const int64_t ks = KT * a.k.token * int64_t(sizeof(T)), vs = KT * a.v.token * int64_t(sizeof(T));   // from tile to tile
  const TileLoad<T, DH, KT, NT> lk(a.k.token * int64_t(sizeof(T)), tid), lv(a.v.token * int64_t(sizeof(T)), tid);
  if (WIN && win.sinks == 0) {
    kp += win.skip * ks;
    vp += win.skip * vs;
  }
  if (tiles > 0) {
    const int left = sq.nk - (WIN ? win.tile(0) * KT : 0);
    lk(kp, left, share);
    lv(vp, left, share + kTile);
  }
  Reader<T, DH> read(base0 + uint32_t(mate.part * 32 * L::kRow), lane);
  // the query operand, through the wave's share of the second stage
  Frag qf[ST];
  operand_rows<T, DH, false>(qf, read, reinterpret_cast<const char *>(a.q.p + sq.b * a.q.seq + (int64_t(sq.q_first) + q0) * a.q.token + head * a.q.head),
                      a.q.token * int64_t(sizeof(T)), rows, smem + 2 * kTile + wave * (32 * L::kRow),
                      uint32_t(2 * kTile + (wave - mate.part) * (32 * L::kRow)), lane);

  f32x16 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = f32x16{0.f};
  float top = -INFINITY, sum = 0.f;             // of the lane's query: running maximum of the products, sum of its share of the keys
  const float slack = fminf(8.f / scale, FLT_MAX);    // (finite: ahead of the first keys, top + slack has to be less than any product)
  const int hidden = max(block * BQ + off + 1, 0) / KT;               // the first tile that not all of the workgroup's queries see all of
  bool found = false;                           // ... where a value is not finite
  bool careful = !WIN;                          // whether tiles are looked through for those: with a window a third of them would be
  for (int it = 0; it < tiles; ++it) {
    const int tile = WIN ? win.tile(it) : it;
    const int k0 = tile * KT + mate.part * 32;  // the wave's first key of the tile
    arrived();
    __syncthreads();
    if (careful && (tile >= hidden || (WIN && tile * KT < win.partial && tile * KT + KT > a.s.sinks))) {
      found |= make_finite<T, DH, KT, NT>(smem + (it & 1) * 2 * kTile + kTile);
      __syncthreads();
    }
    if (it + 1 < tiles) {
      const uint32_t next = share + uint32_t(~it & 1) * uint32_t(2 * kTile);
      const int following = WIN ? win.tile(it + 1) : it + 1;
      kp += WIN ? (following - tile) * ks : ks;
      vp += WIN ? (following - tile) * vs : vs;
      lk(kp, sq.nk - following * KT, next);
      lv(vp, sq.nk - following * KT, next + kTile);
    }
    if (k0 <= mine && (!WIN || k0 + 32 * KB > q0 + off - a.s.window + 1 || k0 < a.s.sinks)) {
      // Operands are on their way from LDS ahead of the products that take them, and arithmetic stands between products: a wave issues in
      // order, and left to itself the compiler reads, waits and multiplies in turn.
      // While a wave has products to issue it goes ahead of the SIMD's others, which are at their maxima or waiting: 2 % less.
      Frag x[ST], v[DB];
      f32x16 s[KB];
#pragma unroll
      for (int t = 0; t < ST; ++t) x[t] = read.by_row(0, 0, t);
      __builtin_amdgcn_s_setprio(1);
      float m = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        s[kb] = f32x16{0.f};
#pragma unroll
        for (int t = 0; t < ST; ++t) {
          pin();
          s[kb] = Operand<T>::mma(x[t], qf[t], s[kb]);
          if (kb + 1 < KB) x[t] = read.by_row(0, kb * 32 + 32, t);
          if (kb + 1 == KB && t >= ST - DB) v[t - ST + DB] = read.transposed(kTile, 0, 0, t - ST + DB);
        }
      }
      pin();
      __builtin_amdgcn_s_setprio(0);
      if (k0 + 32 * KB - 1 > q0 + off) {        // some of the wave's queries do not see all of these keys
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (k0 + kb * 32 + 8 * (r >> 2) + 4 * h + (r & 3) > seen) s[kb][r] = -INFINITY;
      }
      if (WIN && k0 <= q0 + 31 + off - a.s.window && k0 + 32 * KB > a.s.sinks) {      // ... because they are too far behind
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int key = k0 + kb * 32 + 8 * (r >> 2) + 4 * h + (r & 3);
            if (key <= seen - a.s.window && key >= a.s.sinks) s[kb][r] = -INFINITY;
          }
      }
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) m = fmaxf(m, s[kb][r]);
      // The maximum moves only where some query's has grown by 8 in the exponent: until then its weights are up to 2^8 and not 1, which
      // neither fp32 sums nor bf16 operands mind, and the outputs need not be scaled at every tile.
      m = fmaxf(top, max_lane_xor<32>(m));
      if (__builtin_amdgcn_ballot_w64(m > top + slack)) {
        const float fade = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((top - m) * scale);
        sum *= fade;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[db][r] *= fade;
        top = m;
      }
      const float base = top == -INFINITY ? 0.f : -top * scale;       // (a query that has seen nothing yet)
      float part[4] = {0.f};                    // a tile's weights first, so that few additions round the running sum
      auto weights = [&](int kb, int r0, int n) {
#pragma unroll
        for (int r = r0; r < r0 + n; ++r) {
          s[kb][r] = __builtin_amdgcn_exp2f(fmaf(s[kb][r], scale, base));
          part[r & 3] += s[kb][r];
        }
      };
      Frag pf[2];
      weights(0, 0, 16);
      __builtin_amdgcn_s_setprio(1);
      pf[0] = Operand<T>::of(s[0], 0);
      pf[1] = Operand<T>::of(s[0], 1);
#pragma unroll
      for (int i = 0; i < 2 * KB; ++i) {        // 16 keys a step
        const Frag p = pf[i & 1];
        Frag left;
        if constexpr (REST) left = Operand<T>::rest_of(s[i >> 1], p, i & 1);
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          pin();
          o[db] = Operand<T>::mma(v[db], p, o[db]);
          if constexpr (REST) o[db] = Operand<T>::mma(v[db], left, o[db]);
          if (i + 1 < 2 * KB) v[db] = read.transposed(kTile, (i + 1) / 2 * 32, (i + 1) & 1, db);
          if (i + 2 < 2 * KB) weights((i + 2) >> 1, 8 * (i & 1) + db * (8 / DB), 8 / DB);   // those of the step after the next one
        }
        if (i + 2 < 2 * KB) pf[i & 1] = Operand<T>::of(s[(i + 2) >> 1], i & 1);
      }
      __builtin_amdgcn_s_setprio(0);
      sum += (part[0] + part[1]) + (part[2] + part[3]);
    }
    read.move(it & 1 ? uint32_t(-2 * kTile) : uint32_t(2 * kTile));
    if (WIN && !careful && it + 1 == tiles) {
      // A hidden value that is not finite has made its product with a weight of 0 NaN.  Then all of it once more, carefully.
      float bad = 0.f;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) bad = fmaf(o[db][r], 0.f, bad);
      __syncthreads();
      if (any_of_four(__builtin_amdgcn_ballot_w64(bad != 0.f) != 0, reinterpret_cast<int *>(smem + 4 * 32 * L::kRow))) {
        __syncthreads();
        careful = true;
#pragma unroll
        for (int db = 0; db < DB; ++db) o[db] = f32x16{0.f};
        top = -INFINITY;
        sum = 0.f;
        kp += (win.tile(0) - tile) * ks;
        vp += (win.tile(0) - tile) * vs;
        lk(kp, sq.nk - win.tile(0) * KT, share);
        lv(vp, sq.nk - win.tile(0) * KT, share + kTile);
        if (tiles & 1) read.move(uint32_t(-2 * kTile));
        it = -1;
      }
    }
  }
  __syncthreads();
  found = any_of_four(found, reinterpret_cast<int *>(smem + 4 * 32 * L::kRow));
  if constexpr (SW > 1) {
    constexpr int kFloats = 64 * (16 * DB + 2);
    float *const parts = reinterpret_cast<float *>(smem + 4 * 32 * L::kRow + 256) + mate.rows * kFloats;   // behind any_of_four's words
    constexpr int kPart = Shared<SW>::kRowWaves * kFloats;
    if (mate.part > 0) {
      float *const to = parts + (mate.part - 1) * kPart;
      put_sums(o, to, lane);
      to[16 * DB * 64 + lane] = top;
      to[(16 * DB + 1) * 64 + lane] = sum;
    }
    __syncthreads();
    if (mate.part > 0) return;
    float m = top;
#pragma unroll
    for (int i = 0; i < SW - 1; ++i) m = fmaxf(m, parts[i * kPart + 16 * DB * 64 + lane]);
    auto fade = [&](float t) { return t == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((t - m) * scale); };
    const float mine_fades = fade(top);
    sum *= mine_fades;
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] *= mine_fades;
#pragma unroll
    for (int i = 0; i < SW - 1; ++i) {
      const float f = fade(parts[i * kPart + 16 * DB * 64 + lane]);
      sum = fmaf(parts[i * kPart + (16 * DB + 1) * 64 + lane], f, sum);
      add_sums(o, parts + i * kPart, f, lane);
    }
    top = m;
  }
  if (rows <= 0) return;
  if (found) {
    const char *const v0 = reinterpret_cast<const char *>(a.v.p + sq.b * a.v.seq + sq.k_first * a.v.token + hk * a.v.head);
    const int64_t pitch = a.v.token * int64_t(sizeof(T));
    if constexpr (WIN) {          // (all that the lane's query sees: what is not finite stays so when it is added twice)
      add_not_finite<T, DH>(o, v0, pitch, 0, min(a.s.sinks, mine + 1), 0, seen, lane);
      add_not_finite<T, DH>(o, v0, pitch, win.low, mine + 1, seen - a.s.window + 1, seen, lane);
    } else {
      add_not_finite<T, DH>(o, v0, pitch, hidden * KT, mine + 1, 0, seen, lane);
    }
  }
  sum = add_lane_xor<32>(sum);
  const bool some = sum > 0.f || sum != sum;    // (a query without keys: zeros, and -inf)
  if (a.lse && lane < rows) {
    const size_t at = row_value(a.s.q_start != nullptr, sq.b, sq.q_first, a.s.q_tokens, a.s.heads, head);
    // the exponents are relative to the rounded top * scale; added up in 64 bits, rounded once
    a.lse[at + q0 + lane] = some ? float(double(top * scale) * kLn2 + log(double(sum))) : -INFINITY;
  }
  const int64_t row = int64_t(sq.q_first) + q0;
  char *op = reinterpret_cast<char *>(a.out.p + sq.b * a.out.seq + row * a.out.token + head * a.out.head);
  char *rp = REST ? reinterpret_cast<char *>(a.rest.p + sq.b * a.rest.seq + row * a.rest.token + head * a.rest.head) : nullptr;
  store_rows<T, DH>(o, some ? 1.f / sum : 0.f, smem + wave * (32 * L::kRow), op, a.out.token * int64_t(sizeof(T)), rows, rp,
                    a.rest.token * int64_t(sizeof(T)), lane);
}

template <typename T, int DH, bool REST, int SW, bool WIN>
hipError_t launch_attend_shared(AttendArgs<T> a, hipStream_t st) {
  // a stage, and behind it another one or the waves' 32 queries each
  constexpr int row = Tile<T, DH>::kRow, stage = 2 * (SW > 1 ? 32 * SW : kKeys<T>) * row, waves = 4 * 32 * row, lds = stage + (stage > waves ? stage : waves);
  static_assert(SW == 1 || waves + 256 + 4 * (SW - 1) / SW * 256 * (DH / 2 + 2) <= lds, "the parts' sums");
  const hipError_t e = allow_lds(&prompt_attend_kernel<T, DH, REST, SW, WIN>, lds);
  if (e != hipSuccess) return e;
  const long long blocks = blocks_at_most(a.s.q_start, a.s.batch, a.s.q_tokens, Shared<SW>::kRows) * a.s.heads;
  // Up to two for each place: beyond, what a sequence's blocks share counts for more (4096: 198 / 229 us).  With a unit for each the order is
  // nothing, and finding it 2 us (5 sequences of 17 to 500 tokens 9.8 us / 11.4, gradients 30.2 / 33.2).
  a.by_work = blocks > 256 && blocks < 1024;
  hipLaunchKernelGGL((prompt_attend_kernel<T, DH, REST, SW, WIN>), dim3(unsigned(blocks)), dim3(256), lds, st, a);
  return hipGetLastError();
}

template <typename T, int DH, bool REST, bool WIN>
hipError_t launch_attend_prompt(const AttendArgs<T> &a, hipStream_t st) {
  if (share_queries<T>(a.s))
    return launch_attend_shared<T, DH, REST, DH * sizeof(T) == 512 ? 2 : 4, WIN>(a, st);      // (as many as two stages leave LDS for)
  return launch_attend_shared<T, DH, REST, 1, WIN>(a, st);
}

// ---- the attention every key received -----------------------------------------------------------------------------
// A workgroup takes 128 keys of a kv head, a wave 32 of them, and goes over the queries that see them, of all heads of the group:
// S = Q K^T leaves a key's weights in two lanes, which add them up.  No atomics: the order of the sum is fixed.
// 16 x 1024 tokens of 32 heads 118 us, 3 x 1000 behind 7192, 32 heads over 8, 169 us: vector instructions take 54 and 57 % of the cycles
// and the matrix unit 29 and 36 %, mostly one after the other.  A tile's exponentials are written between the products of its next block,
// but the branch of hide() lets the compiler move them behind the last product, and results lie in accumulation registers, out of
// which they are moved first.
template <typename T>
struct ScoreArgs {
  PromptShape s;
  Rows<const T> q, k;
  const float *lse;
  float *scores;
  bool by_work;
};

template <typename T>
constexpr int kQueries = sizeof(T) == 2 ? 64 : 32;

template <typename T, int DH, int SW>
__global__ __launch_bounds__(256) void prompt_scores_kernel(const ScoreArgs<T> a) {
  constexpr int NT = 256, BK = Shared<SW>::kRows, QT = SW > 1 ? 32 * SW : kQueries<T>, WQ = SW > 1 ? 32 : QT, QB = WQ / 32, ST = DH / 16;
  typedef Tile<T, DH> L;
  typedef typename Operand<T>::type Frag;
  constexpr int kTile = QT * L::kRow;
  extern __shared__ __align__(16) unsigned char smem[];   // Q 0, Q 1
  __shared__ __align__(16) float s_lse[2][QT];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, h = lane >> 5;
  const int hk = blockIdx.x % a.s.kv_heads;
  Sequence sq;
  int block;
  if (!find_block<BK, false>(a.s, blockIdx.x / a.s.kv_heads, a.by_work, sq, block)) {
    const SpareRows spare = spare_rows<BK>(a.s.k_start, a.s.batch, a.s.k_tokens, block);
    if (tid < spare.n) a.scores[size_t(hk) * a.s.k_tokens + spare.at(tid)] = 0.f;
    return;
  }
  const Shared<SW> mate(wave);
  const int k0 = block * BK + mate.rows * 32, off = sq.nk - sq.nq;
  const int rows = min(32, sq.nk - k0);
  const int first = max(block * BK - off, 0) / QT * QT;    // the first tile with a query that sees a key of the workgroup
  const int per = first < sq.nq ? (sq.nq - first + QT - 1) / QT : 0, tiles = per * a.s.group;
  const float scale = a.s.scale_log2;
  const bool packed = a.s.q_start != nullptr;
  const uint32_t base0 = __builtin_amdgcn_readfirstlane(lds_offset(smem)), share = base0 + uint32_t(wave) * 1024u;
  const int64_t qs = a.q.token * int64_t(sizeof(T));
  const TileLoad<T, DH, QT, NT> lq(a.q.token * int64_t(sizeof(T)), tid);
  // the tile after the last one loaded: its head's rows and log-sum-exps, its first query
  const char *qp = reinterpret_cast<const char *>(a.q.p + sq.b * a.q.seq + sq.q_first * a.q.token + hk * a.s.group * a.q.head);
  const float *lp = a.lse + row_value(packed, sq.b, sq.q_first, a.s.q_tokens, a.s.heads, hk * a.s.group);
  int next = first;
  float row_lse = 0.f;
  auto load = [&](int stage) {
    lq(qp + next * qs, sq.nq - next, share + uint32_t(stage * kTile));
    if (tid < QT) row_lse = next + tid < sq.nq ? subtrahend(lp[next + tid]) : INFINITY;
    next += QT;
    if (next >= sq.nq) {
      next = first;
      qp += a.q.head * int64_t(sizeof(T));
      lp += a.s.q_tokens;
    }
  };
  Reader<T, DH> read(base0 + uint32_t(mate.part * 32 * L::kRow), lane);
  Frag kf[ST];                                              // through the wave's quarter of LDS
  operand_rows<T, DH, false>(kf, read, reinterpret_cast<const char *>(a.k.p + sq.b * a.k.seq + (int64_t(sq.k_first) + k0) * a.k.token + hk * a.k.head),
                      a.k.token * int64_t(sizeof(T)), rows, smem + wave * (32 * L::kRow),
                      uint32_t((wave - mate.part) * (32 * L::kRow)), lane);
  __syncthreads();
  if (tiles > 0) load(0);
  if (tid < QT) s_lse[0][tid] = row_lse;
  float sum = 0.f;
  const int mine = mate.part * 32;                          // the wave's first query of a tile's
  int tile = first - QT;
  for (int it = 0; it < tiles; ++it) {
    tile += QT;
    if (tile >= sq.nq) tile = first;
    const int q0 = tile + mine;
    arrived();
    __syncthreads();
    if (it + 1 < tiles) load(~it & 1);
    Frag x[ST];
    float part[4] = {0.f};
    // A hidden query whose log-sum-exp is NaN: its weights are none at all, where the sums below would make them NaN.
    if (q0 + off < k0 + 31 && __builtin_amdgcn_ballot_w64(s_lse[it & 1][mine + lane % WQ] != s_lse[it & 1][mine + lane % WQ])) {
#pragma unroll 1
      for (int qb = 0; qb < QB; ++qb) {
        f32x16 s = {0.f};
#pragma unroll
        for (int t = 0; t < ST; ++t) s = Operand<T>::mma(read.by_row(uint32_t(qb * 32 * L::kRow), 0, t), kf[t], s);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int i = qb * 32 + 8 * (r >> 2) + 4 * h + (r & 3);
          if (k0 + c <= q0 + i + off) part[r & 3] += __builtin_amdgcn_exp2f(fmaf(s[r], scale, -s_lse[it & 1][mine + i]));
        }
      }
      sum += (part[0] + part[1]) + (part[2] + part[3]);
      if (it + 1 < tiles && tid < QT) s_lse[~it & 1][tid] = row_lse;
      read.move(it & 1 ? uint32_t(-kTile) : uint32_t(kTile));
      continue;
    }
#pragma unroll
    for (int t = 0; t < ST; ++t) x[t] = read.by_row(0, 0, t);
    f32x16 s[QB];
    auto weights = [&](int qb, int r4) {
      const f32x4 lse = *reinterpret_cast<const f32x4 *>(&s_lse[it & 1][mine + qb * 32 + 8 * r4 + 4 * h]);
#pragma unroll
      for (int i = 0; i < 4; ++i) part[i] += __builtin_amdgcn_exp2f(fmaf(s[qb][4 * r4 + i], scale, -lse[i]));
    };
    auto hide = [&](int qb) {
      const int qf = q0 + qb * 32 + off;
      if (qf < k0 + 31) {                              // some of these queries do not see some of the wave's keys
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (k0 + c > qf + 8 * (r >> 2) + 4 * h + (r & 3)) s[qb][r] = -INFINITY;
      }
    };
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      s[qb] = f32x16{0.f};
#pragma unroll
      for (int t = 0; t < ST; ++t) {
        pin();
        s[qb] = Operand<T>::mma(x[t], kf[t], s[qb]);
        if (qb + 1 < QB) x[t] = read.by_row(0, qb * 32 + 32, t);
        if (qb > 0 && t % (ST / 4) == ST / 4 - 1) weights(qb - 1, t / (ST / 4));   // the block before (see above for where it ends up)
      }
      pin();
      hide(qb);
    }
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) weights(QB - 1, r4);
    sum += (part[0] + part[1]) + (part[2] + part[3]);
    if (it + 1 < tiles && tid < QT) s_lse[~it & 1][tid] = row_lse;
    read.move(it & 1 ? uint32_t(-kTile) : uint32_t(kTile));
  }
  sum = add_lane_xor<32>(sum);
  if constexpr (SW > 1) {
    float *const sums = reinterpret_cast<float *>(smem);    // [part][rows of the workgroup]
    __syncthreads();
    if (lane < 32) sums[mate.part * BK + mate.rows * 32 + lane] = sum;
    __syncthreads();
    if (mate.part > 0) return;
#pragma unroll
    for (int i = 1; i < SW; ++i) sum += sums[i * BK + mate.rows * 32 + c];
  }
  if (lane < rows) a.scores[row_value(packed, sq.b, sq.k_first, a.s.k_tokens, a.s.kv_heads, hk) + k0 + lane] = sum;
}

template <typename T, int DH, int SW>
hipError_t launch_scores_shared(ScoreArgs<T> a, hipStream_t st) {
  constexpr int tiles = 2 * (SW > 1 ? 32 * SW : kQueries<T>) * Tile<T, DH>::kRow, keys = 128 * Tile<T, DH>::kRow, lds = tiles > keys ? tiles : keys;
  const hipError_t e = allow_lds(&prompt_scores_kernel<T, DH, SW>, lds);
  if (e != hipSuccess) return e;
  const long long blocks = blocks_at_most(a.s.k_start, a.s.batch, a.s.k_tokens, Shared<SW>::kRows) * a.s.kv_heads;
  a.by_work = blocks > 256 && blocks < 1024;      // (as above; 1512: 177 / 197 us)
  hipLaunchKernelGGL((prompt_scores_kernel<T, DH, SW>), dim3(unsigned(blocks)), dim3(256), lds, st, a);
  return hipGetLastError();
}

template <typename T, int DH>
hipError_t launch_scores(const ScoreArgs<T> &a, hipStream_t st) {
  if (share_scored_keys(a.s)) return launch_scores_shared<T, DH, 4>(a, st);
  return launch_scores_shared<T, DH, 1>(a, st);
}

template <typename T, bool WIN>
int attend_typed(const adore_prompt_config &c, const PromptShape &s, const adore_rows *q, const adore_rows *k, const adore_rows *v,
                 const adore_rows *out, float *lse, const adore_rows *rest, hipStream_t st) {
  AttendArgs<T> a;
  a.s = s;
  a.q = rows_of<const T>(q);
  a.k = rows_of<const T>(k);
  a.v = rows_of<const T>(v);
  a.out = rows_of<T>(out);
  a.rest = rest ? rows_of<T>(rest) : Rows<T>{nullptr, 0, 0, 0};
  a.lse = lse;
  hipError_t e;
  if constexpr (sizeof(T) == 2) {
    if (rest)
      e = c.head_dim == 128 ? launch_attend_prompt<T, 128, true, WIN>(a, st) : launch_attend_prompt<T, 64, true, WIN>(a, st);
    else
      e = c.head_dim == 128 ? launch_attend_prompt<T, 128, false, WIN>(a, st) : launch_attend_prompt<T, 64, false, WIN>(a, st);
  } else {
    e = c.head_dim == 128 ? launch_attend_prompt<T, 128, false, WIN>(a, st) : launch_attend_prompt<T, 64, false, WIN>(a, st);
  }
  return e == hipSuccess ? ADORE_OK : ADORE_E_HIP;
}

template <typename T>
int scores_typed(const adore_prompt_config &c, const PromptShape &s, const adore_rows *q, const adore_rows *k, const float *lse,
                 float *scores, hipStream_t st) {
  ScoreArgs<T> a;
  a.s = s;
  a.q = rows_of<const T>(q);
  a.k = rows_of<const T>(k);
  a.lse = lse;
  a.scores = scores;
  const hipError_t e = c.head_dim == 128 ? launch_scores<T, 128>(a, st) : launch_scores<T, 64>(a, st);
  return e == hipSuccess ? ADORE_OK : ADORE_E_HIP;
}

template <bool WIN>
int attend_prompts(const adore_prompt_config *cfg, const PromptShape &s, const adore_rows *q, const adore_rows *k, const adore_rows *v,
                   const adore_rows *out, float *lse, const adore_rows *rest, void *hip_stream) {
  if (!prompt_rows_ok(q, cfg->dtype) || !prompt_rows_ok(k, cfg->dtype) || !prompt_rows_ok(v, cfg->dtype) ||
      !prompt_rows_ok(out, cfg->dtype) || (rest && (cfg->dtype != ADORE_BF16 || !prompt_rows_ok(rest, cfg->dtype))))
    return ADORE_E_INVALID;
  if (s.q_tokens == 0) return ADORE_OK;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return cfg->dtype == ADORE_BF16 ? attend_typed<bf16_t, WIN>(*cfg, s, q, k, v, out, lse, rest, st)
                                  : attend_typed<float, WIN>(*cfg, s, q, k, v, out, lse, rest, st);
}

}  // namespace

// The checks that every call on prompts makes; fills in what the kernels take.
int prompt_shape(const adore_prompt_config *c, const int32_t *q_start, const int32_t *k_start, PromptShape *s) {
  if (!c || (q_start == nullptr) != (k_start == nullptr)) return ADORE_E_INVALID;
  if (c->batch <= 0 || c->heads <= 0 || c->kv_heads <= 0 || c->heads % c->kv_heads != 0 || c->q_tokens < 0 || c->k_tokens < 0 ||
      (c->dtype != ADORE_F32 && c->dtype != ADORE_BF16) || !std::isfinite(c->scale) || c->scale < 0.f || c->head_dim <= 0)
    return ADORE_E_INVALID;
  if (c->head_dim != 64 && c->head_dim != 128) return ADORE_E_UNSUPPORTED;
  // row and workgroup counts far inside 32 bits
  constexpr int kMostTokens = 1 << 24, kMostHeads = 1 << 12, kMostBatch = 1 << 16;
  if (c->q_tokens > kMostTokens || c->k_tokens > kMostTokens || c->heads > kMostHeads || c->batch > kMostBatch) return ADORE_E_UNSUPPORTED;
  const long long rows = c->q_tokens > c->k_tokens ? c->q_tokens : c->k_tokens;
  // fewer than 2^32 threads, 256 a workgroup (with 32 tokens or fewer per sequence there are as many workgroups of 128 as of 32)
  if (blocks_at_most(q_start, c->batch, int(rows), 32) * c->heads >= (1ll << 24)) return ADORE_E_UNSUPPORTED;
  s->q_start = q_start;
  s->k_start = k_start;
  s->batch = c->batch;
  s->heads = c->heads;
  s->kv_heads = c->kv_heads;
  s->group = c->heads / c->kv_heads;
  s->q_tokens = c->q_tokens;
  s->k_tokens = c->k_tokens;
  s->scale = c->scale > 0.f ? c->scale : 1.f / sqrtf(float(c->head_dim));
  s->scale_log2 = s->scale * kLog2e;
  s->window = s->sinks = 0;
  return ADORE_OK;
}

// A window, for a shape that prompt_shape filled in.  No sequence has more than 2^24 tokens: beyond, sums of positions would pass 32 bits.
int window_shape(const adore_window *w, PromptShape *s) {
  constexpr int kMost = 1 << 25;
  if (!w || w->window < 1 || w->sinks < 0) return ADORE_E_INVALID;
  s->window = w->window < kMost ? w->window : kMost;
  s->sinks = w->sinks < kMost ? w->sinks : kMost;
  return ADORE_OK;
}

// A tensor of rows: present, and every row on a 16-byte boundary.
bool prompt_rows_ok(const adore_rows *r, int dtype) {
  if (!r || !r->data || (reinterpret_cast<uintptr_t>(r->data) & 15)) return false;
  const int64_t unit = dtype == ADORE_BF16 ? 8 : 4, most = int64_t(1) << 22;
  return r->seq >= 0 && r->token >= 0 && r->head >= 0 && r->seq % unit == 0 && r->token % unit == 0 && r->head % unit == 0 && r->token <= most;
}

}  // namespace adore

extern "C" {

int adore_prompt_attention(const adore_prompt_config *cfg, const int32_t *q_start, const int32_t *k_start, const adore_rows *q,
                           const adore_rows *k, const adore_rows *v, const adore_rows *out, float *lse, const adore_rows *rest,
                           void *hip_stream) {
  adore::PromptShape s;
  const int rc = adore::prompt_shape(cfg, q_start, k_start, &s);
  return rc != ADORE_OK ? rc : adore::attend_prompts<false>(cfg, s, q, k, v, out, lse, rest, hip_stream);
}

int adore_window_attention(const adore_prompt_config *cfg, const adore_window *window, const int32_t *q_start, const int32_t *k_start,
                           const adore_rows *q, const adore_rows *k, const adore_rows *v, const adore_rows *out, float *lse,
                           const adore_rows *rest, void *hip_stream) {
  adore::PromptShape s;
  int rc = adore::prompt_shape(cfg, q_start, k_start, &s);
  if (rc == ADORE_OK) rc = adore::window_shape(window, &s);
  return rc != ADORE_OK ? rc : adore::attend_prompts<true>(cfg, s, q, k, v, out, lse, rest, hip_stream);
}

int adore_prompt_scores(const adore_prompt_config *cfg, const int32_t *q_start, const int32_t *k_start, const adore_rows *q,
                        const adore_rows *k, const float *lse, float *scores, void *hip_stream) {
  using namespace adore;
  PromptShape s;
  const int rc = prompt_shape(cfg, q_start, k_start, &s);
  if (rc != ADORE_OK) return rc;
  if (!prompt_rows_ok(q, cfg->dtype) || !prompt_rows_ok(k, cfg->dtype) || !lse || !scores) return ADORE_E_INVALID;
  if (s.k_tokens == 0) return ADORE_OK;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return cfg->dtype == ADORE_BF16 ? scores_typed<bf16_t>(*cfg, s, q, k, lse, scores, st) : scores_typed<float>(*cfg, s, q, k, lse, scores, st);
}

}  // extern "C"
