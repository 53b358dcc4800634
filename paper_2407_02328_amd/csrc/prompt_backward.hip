// Gradients of causal attention over whole prompts (prompt_attend.hip), for packed sequences of any lengths and grouped heads.
//
//   p_ij = exp(w_ij - lse_i),  g_ij = p_ij (do_i . v_j - delta_i),  delta_i = do_i . out_i
//   dq_i = scale sum_j g_ij k_j;   dk_j = scale sum_i g_ij q_i,   dv_j = sum_i p_ij do_i   (i over the queries of all heads of j's group)
//
// Two launches without atomics, so that a gradient's bits do not hang on the order of workgroups: delta and dq, whose workgroups own
// queries and go over the keys; dk and dv, whose workgroups own keys and go over the queries of the group.  The weights are made anew
// in both (seven products instead of the five that one pass would need, which would have to add dq up in memory).
// delta wants out as it was before P and it were rounded: from the rounded one a short row's gradients are up to 2.2 times as far off as
// their own rounding, so the forward can take P in two terms and hand out what rounding left (rest): 1.4 times.
// 8 x 2048 tokens of 32 heads over 8, 128 elements: dq 441 us (0.94 PFLOP/s), dk and dv 606 us (0.91).  The matrix unit is busy 46 and
// 43 % of the cycles, vector instructions take 42 and 28 %, LDS 26 and 33 %: nothing bounds alone.  A wave's operands, products and
// arithmetic wait for one another, and the registers leave two waves a SIMD to fill in.
//
// With a window: the same products over what is seen, and the first keys' queries in a launch of their own (Chunks).  8 x 2048 tokens of 32 heads
// over 8, 128 elements, window 508 and 4 first keys: dq 324 us, the first keys 73 (Q and dO once more, 268 MB), dk and dv 359: tiles of 32
// queries as fast as above, 20 a block of 128 keys where 16 would do.  A wave that leaves out the tiles it sees nothing of: 148 registers spilled.
#include <hip/hip_runtime.h>

#include <climits>

#include "prompt_device.h"

namespace adore {

namespace {

template <typename T>
struct BackwardArgs {
  PromptShape s;
  Rows<const T> d_out, q, k, v, out, rest;   // rest.p may be null
  Rows<T> dq, dk, dv;
  const float *lse;
  float *delta;                              // laid out like lse
  bool by_work;
  // With a window, if set: what queries that are further than the window from the first keys give those (SinkPlan).
  float *sink_part;
  int sink_chunk, sink_slots;
};

// The products of 32 rows of dO with those of out (and what its rounding left), as dO goes by on its way to LDS (carry_rows): delta of row
// DH / EPL lanes share comes out in all of them, for rows lane / (DH / EPL) + i * (64 / (DH / EPL)).
template <typename T, int DH, int N>
__device__ __forceinline__ void carry_dots(float (&dot)[N], const char *d_out, int64_t d_stride, const char *out, int64_t o_stride, const char *rest,
                                           int64_t r_stride, int rows, unsigned char *own, int lane) {
  typedef Tile<T, DH> L;
  constexpr int EPL = Vec16<T>::EPL;
  static_assert(N == 32 * L::kChunks / 64, "rows of a lane");
  const int row = lane / L::kChunks, ch = lane % L::kChunks;
  typename Vec16<T>::Raw d[N], o[N], z[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int64_t there = min(row + i * (64 / L::kChunks), rows - 1);
    d[i] = Vec16<T>::load_raw(reinterpret_cast<const T *>(d_out + there * d_stride + ch * 16));
    o[i] = Vec16<T>::load_raw(reinterpret_cast<const T *>(out + there * o_stride + ch * 16));
    if (rest) z[i] = Vec16<T>::load_raw(reinterpret_cast<const T *>(rest + there * r_stride + ch * 16));
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int mine = row + i * (64 / L::kChunks);
    float x[EPL], y[EPL], sum = 0.f;
    Vec16<T>::values(d[i], x);
    Vec16<T>::values(o[i], y);
#pragma unroll
    for (int e = 0; e < EPL; ++e) sum = fmaf(x[e], y[e], sum);
    if (rest) {
      Vec16<T>::values(z[i], y);
#pragma unroll
      for (int e = 0; e < EPL; ++e) sum = fmaf(x[e], y[e], sum);
    }
    dot[i] = group_sum<L::kChunks>(sum);
    Vec16<T>::store_raw(reinterpret_cast<T *>(own + L::chunk_at(mine, ch)), mine < rows ? d[i] : typename Vec16<T>::Raw{});
  }
}

// ---- dq: 128 queries a workgroup, 32 a wave ----
template <typename T>
constexpr int kDqKeys = sizeof(T) == 2 ? 64 : 32;
// Its LDS: a stage of K and V, and behind it another one or every wave's own 32 rows, for the operands at the beginning and the results at
// the end; four words.
template <typename T, int DH, int SW>
constexpr int kDqStage = 2 * (SW > 1 ? 32 * SW : kDqKeys<T>) * Tile<T, DH>::kRow;
template <typename T, int DH, int SW>
constexpr int kDqWords = kDqStage<T, DH, SW> + (kDqStage<T, DH, SW> > 128 * Tile<T, DH>::kRow ? kDqStage<T, DH, SW> : 128 * Tile<T, DH>::kRow);

template <typename T, int DH, int SW, bool WIN>
__global__ __launch_bounds__(256) ADORE_WAVES(sizeof(T) == 4 || SW > 1 ? 1 : DH == 128 ? 2 : 3) void prompt_dq_kernel(const BackwardArgs<T> a) {
  constexpr int NT = 256, BQ = Shared<SW>::kRows, KT = SW > 1 ? 32 * SW : kDqKeys<T>, KB = SW > 1 ? 1 : KT / 32, DB = DH / 32, ST = DH / 16;
  typedef Tile<T, DH> L;
  typedef typename Operand<T>::type Frag;
  constexpr int kTile = KT * L::kRow;
  extern __shared__ __align__(16) unsigned char smem[];   // two stages of K and V
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, h = lane >> 5;
  const int hk = blockIdx.x % a.s.kv_heads, item = blockIdx.x / a.s.kv_heads, head = hk * a.s.group + item % a.s.group;
  Sequence sq;
  int block;
  if (!find_block<BQ, true>(a.s, item / a.s.group, a.by_work, sq, block)) {
    const SpareRows spare = spare_rows<BQ>(a.s.q_start, a.s.batch, a.s.q_tokens, block);
    zero_rows<T, DH>(a.dq, head, spare, tid, NT);
    return;
  }
  const Shared<SW> mate(wave);
  const int q0 = block * BQ + mate.rows * 32, off = sq.nk - sq.nq;
  const int rows = min(32, sq.nq - q0);
  const int64_t row = int64_t(sq.q_first) + q0, es = int64_t(sizeof(T));
  const char *kp = reinterpret_cast<const char *>(a.k.p + sq.b * a.k.seq + sq.k_first * a.k.token + hk * a.k.head);
  const char *vp = reinterpret_cast<const char *>(a.v.p + sq.b * a.v.seq + sq.k_first * a.v.token + hk * a.v.head);
  const int last = min(block * BQ + BQ, sq.nq) - 1 + off, upto = last < 0 ? 0 : last / KT + 1;
  const WindowTiles<KT> win(a.s, block * BQ + off, last, upto);     // (WIN)
  const int tiles = WIN ? win.total : upto;
  const int mine = rows > 0 ? q0 + rows - 1 + off : -1, seen = q0 + c + off;
  const float scale = a.s.scale_log2;
  const uint32_t base0 = __builtin_amdgcn_readfirstlane(lds_offset(smem)), share = base0 + uint32_t(wave) * 1024u;
  Reader<T, DH> read(base0 + uint32_t(mate.part * 32 * L::kRow), lane);
  const TileLoad<T, DH, KT, NT> lk(a.k.token * es, tid), lv(a.v.token * es, tid);
  if (WIN && win.sinks == 0) {
    kp += win.skip * (KT * a.k.token * es);
    vp += win.skip * (KT * a.v.token * es);
  }
  if (tiles > 0) {
    const int left = sq.nk - (WIN ? win.tile(0) * KT : 0);
    lk(kp, left, share);
    lv(vp, left, share + kTile);
  }
  unsigned char *own = smem + 2 * kTile + wave * (32 * L::kRow);    // the wave's share of the second stage
  const uint32_t own_ahead = uint32_t(2 * kTile + (wave - mate.part) * (32 * L::kRow));
  Frag qf[ST], df[ST];
  operand_rows<T, DH, false>(qf, read, reinterpret_cast<const char *>(a.q.p + sq.b * a.q.seq + row * a.q.token + head * a.q.head), a.q.token * es,
                             rows, own, own_ahead, lane);
  // of the lane's query; weights of a query that is not there are 0
  float lse = INFINITY, delta = 0.f;
  {
    constexpr int N = 32 * L::kChunks / 64;
    const size_t at = row_value(a.s.q_start != nullptr, sq.b, sq.q_first, a.s.q_tokens, a.s.heads, head) + q0;
    float dot[N];
    wave_lds_fence();
    if (rows > 0) {
      if (c < rows) lse = subtrahend(a.lse[at + c]);
      carry_dots<T, DH>(dot, reinterpret_cast<const char *>(a.d_out.p + sq.b * a.d_out.seq + row * a.d_out.token + head * a.d_out.head),
                        a.d_out.token * es, reinterpret_cast<const char *>(a.out.p + sq.b * a.out.seq + row * a.out.token + head * a.out.head),
                        a.out.token * es,
                        a.rest.p ? reinterpret_cast<const char *>(a.rest.p + sq.b * a.rest.seq + row * a.rest.token + head * a.rest.head) : nullptr,
                        a.rest.token * es, rows, own, lane);
    }
    wave_lds_fence();
#pragma unroll
    for (int t = 0; t < ST; ++t) df[t] = read.by_row(own_ahead, 0, t);
    wave_lds_fence();
    if (rows > 0) {
      float *const s_delta = reinterpret_cast<float *>(own);
      if (lane % L::kChunks == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) s_delta[lane / L::kChunks + i * (64 / L::kChunks)] = dot[i];
      }
      wave_lds_fence();
      if (c < rows) {
        delta = s_delta[c];
        if (h == 0 && mate.part == 0) a.delta[at + c] = delta;    // for dk and dv
        if (seen < 0) delta = 0.f;                                // (sees no key: weights of 0, whatever dO holds)
      }
    }
  }
  f32x16 dq[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) dq[db] = f32x16{0.f};
  const int hidden = max(block * BQ + off + 1, 0) / KT;    // the first tile that not all of the workgroup's queries see all of
  int from = INT_MAX;                                      // first key of the first such tile where an element of K is not finite
  bool careful = !WIN;                                     // whether tiles are looked through for those: with a window a third of them would be
  for (int it = 0;; ++it) {
    if (it >= tiles) {
      if (careful || tiles == 0) break;
      // A hidden key that is not finite has made its product with a weight of 0 NaN.  Then all of it once more, carefully.
      float bad = 0.f;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) bad = fmaf(dq[db][r], 0.f, bad);
      __syncthreads();
      if (!any_of_four(__builtin_amdgcn_ballot_w64(bad != 0.f) != 0, reinterpret_cast<int *>(smem + kDqWords<T, DH, SW>))) break;
      careful = true;
#pragma unroll
      for (int db = 0; db < DB; ++db) dq[db] = f32x16{0.f};
      kp += (win.tile(0) - win.tile(tiles - 1)) * (KT * a.k.token * es);
      vp += (win.tile(0) - win.tile(tiles - 1)) * (KT * a.v.token * es);
      lk(kp, sq.nk - win.tile(0) * KT, share);
      lv(vp, sq.nk - win.tile(0) * KT, share + kTile);
      if (tiles & 1) read.move(uint32_t(-2 * kTile));
      it = 0;
    }
    const int tile = WIN ? win.tile(it) : it, k0 = tile * KT + mate.part * 32;
    arrived();
    __syncthreads();
    if (careful && (tile >= hidden || (WIN && tile * KT < win.partial && tile * KT + KT > a.s.sinks))) {
      const bool found = any_of_four(find_not_finite<T, DH, KT, NT>(smem + (it & 1) * 2 * kTile), reinterpret_cast<int *>(smem + kDqWords<T, DH, SW>));
      if (__builtin_amdgcn_readfirstlane(found)) from = min(from, tile * KT);
    }
    if (it + 1 < tiles) {
      const uint32_t next = share + uint32_t(~it & 1) * uint32_t(2 * kTile);
      const int following = WIN ? win.tile(it + 1) : it + 1;
      kp += (WIN ? following - tile : 1) * (KT * a.k.token * es);
      vp += (WIN ? following - tile : 1) * (KT * a.v.token * es);
      lk(kp, sq.nk - following * KT, next);
      lv(vp, sq.nk - following * KT, next + kTile);
    }
    if (k0 > mine || tile * KT >= from || (WIN && k0 + 32 * KB <= q0 + off - a.s.window + 1 && k0 >= a.s.sinks)) {
      read.move(it & 1 ? uint32_t(-2 * kTile) : uint32_t(2 * kTile));
      continue;
    }
    // Operands on their way ahead of their products, arithmetic between products (a wave issues in order).
    Frag x[ST], y[DB];
#pragma unroll
    for (int t = 0; t < ST; ++t) x[t] = read.by_row(0, 0, t);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      f32x16 s = {0.f}, g = {0.f};
#pragma unroll
      for (int t = 0; t < ST; ++t) {
        pin();
        s = Operand<T>::mma(x[t], qf[t], s);
        x[t] = read.by_row(kTile, kb * 32, t);
      }
      pin();
      if (k0 + kb * 32 + 31 > q0 + off) {         // some of the wave's queries do not see some of these keys
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (k0 + kb * 32 + 8 * (r >> 2) + 4 * h + (r & 3) > seen) s[r] = -INFINITY;
      }
      const bool behind = WIN && k0 + kb * 32 <= q0 + 31 + off - a.s.window && k0 + kb * 32 + 32 > a.s.sinks;     // ... because they are too far back
      if (behind) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = k0 + kb * 32 + 8 * (r >> 2) + 4 * h + (r & 3);
          if (key <= seen - a.s.window && key >= a.s.sinks) s[r] = -INFINITY;
        }
      }
#pragma unroll
      for (int t = 0; t < ST; ++t) {
        pin();
        g = Operand<T>::mma(x[t], df[t], g);
        if (t >= ST - DB) y[t - ST + DB] = read.transposed(0, kb * 32, 0, t - ST + DB);
#pragma unroll
        for (int r = t * (16 / ST); r < (t + 1) * (16 / ST); ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], scale, -lse));
      }
      pin();
      if (k0 + kb * 32 + 31 > q0 + off) {         // (a hidden row of V may be anything)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (k0 + kb * 32 + 8 * (r >> 2) + 4 * h + (r & 3) > seen) g[r] = delta;
      }
      if (behind) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = k0 + kb * 32 + 8 * (r >> 2) + 4 * h + (r & 3);
          if (key <= seen - a.s.window && key >= a.s.sinks) g[r] = delta;
        }
      }
#pragma unroll
      for (int r = 0; r < 8; ++r) g[r] = s[r] * (g[r] - delta);
      Frag gf = Operand<T>::of(g, 0);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        pin();
        dq[db] = Operand<T>::mma(y[db], gf, dq[db]);
        y[db] = read.transposed(0, kb * 32, 1, db);
#pragma unroll
        for (int r = 8 + db * (8 / DB); r < 8 + (db + 1) * (8 / DB); ++r) g[r] = s[r] * (g[r] - delta);
      }
      gf = Operand<T>::of(g, 1);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        pin();
        dq[db] = Operand<T>::mma(y[db], gf, dq[db]);
        if (kb + 1 < KB) {
#pragma unroll
          for (int t = db * (ST / DB); t < (db + 1) * (ST / DB); ++t) x[t] = read.by_row(0, kb * 32 + 32, t);
        }
      }
      pin();
    }
    read.move(it & 1 ? uint32_t(-2 * kTile) : uint32_t(2 * kTile));
  }
  __syncthreads();
  if constexpr (SW > 1) {
    constexpr int kFloats = 64 * 16 * DB, kPart = Shared<SW>::kRowWaves * kFloats;
    float *const parts = reinterpret_cast<float *>(smem) + mate.rows * kFloats;
    if (mate.part > 0) put_sums(dq, parts + (mate.part - 1) * kPart, lane);
    __syncthreads();
    if (mate.part > 0) return;
#pragma unroll
    for (int i = 0; i < SW - 1; ++i) add_sums(dq, parts + i * kPart, 1.f, lane);
  }
  if (rows <= 0) return;
  // a lane: its query, half of the elements
  const int64_t query = row + min(c, rows - 1);
  const T *const qr = a.q.p + sq.b * a.q.seq + query * a.q.token + head * a.q.head + 4 * h;
  const T *const dr = a.d_out.p + sq.b * a.d_out.seq + query * a.d_out.token + head * a.d_out.head + 4 * h;
#pragma unroll 1
  for (int i = from; i <= mine; ++i) {
    if (WIN && i >= a.s.sinks) i = max(i, win.low);            // (keys in between nobody sees)
    const int64_t key = int64_t(sq.k_first) + i;
    const T *const kr = a.k.p + sq.b * a.k.seq + key * a.k.token + hk * a.k.head + 4 * h;
    const T *const vr = a.v.p + sq.b * a.v.seq + key * a.v.token + hk * a.v.head + 4 * h;
    float w = 0.f, x = 0.f;
#pragma unroll 1
    for (int e = 0; e < DH; e += 8)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        w = fmaf(to_float(qr[e + r]), to_float(kr[e + r]), w);
        x = fmaf(to_float(dr[e + r]), to_float(vr[e + r]), x);
      }
    w = add_lane_xor<32>(w);
    x = add_lane_xor<32>(x);
    x = __builtin_amdgcn_exp2f(fmaf(w, scale, -lse)) * (x - delta);
    if (WIN ? in_window(a.s, i, seen) : i <= seen) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          dq[db][r] = fmaf(x, to_float(kr[32 * db + 8 * (r >> 2) + (r & 3)]), dq[db][r]);
          if (r % 4 == 3) pin();
        }
    }
  }
  store_rows<T, DH>(dq, a.s.scale, own, reinterpret_cast<char *>(a.dq.p + sq.b * a.dq.seq + row * a.dq.token + head * a.dq.head),
                    a.dq.token * es, rows, nullptr, 0, lane);
}

// ---- dk and dv: 128 keys a workgroup, 32 a wave ----
// At 128 elements a wave's K, V and their gradients would be 192 registers, and with the rest more than two waves a SIMD leave room for:
// V stays in LDS (a spilled register in the loop costs a wait for the next tile: loads return in order).
// (fp32 at 128 elements, waves that share keys: LDS has no room for V, one wave a SIMD leaves registers for it)
template <typename T, int DH, int SW>
constexpr bool kValuesInRegisters = SW > 1 && DH * sizeof(T) == 512;

// A place's sequence and first query (Chunks); all 64 lanes of a wave call it together.
__device__ __forceinline__ bool find_chunk(const PromptShape &a, int place, int chunk, Sequence &s, int &query) {
  const int lane = threadIdx.x & 63;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    const int b = min(b0 + lane, a.batch - 1);
    const Chunks mine(a, sequence_at(a, b), chunk);
    const uint64_t here = __builtin_amdgcn_ballot_w64(place >= mine.first && place < mine.first + mine.n);
    if (here) {
      s = sequence_at(a, __builtin_amdgcn_readfirstlane(min(b0 + int(__builtin_ctzll(here)), a.batch - 1)));
      const Chunks found(a, s, chunk);
      query = found.from + (place - found.first) * chunk;
      return true;
    }
  }
  return false;
}

enum { kCausal, kWindow, kSinks };           // every pair; pairs in the window; the others, which the first keys have

template <typename T, int DH, int SW, int MODE>
__global__ __launch_bounds__(256) ADORE_WAVES(sizeof(T) == 2 && SW == 1 ? 2 : 1) void prompt_dkv_kernel(const BackwardArgs<T> a) {
  constexpr int NT = 256, BK = Shared<SW>::kRows, QT = 32 * SW, DB = DH / 32, ST = DH / 16;
  typedef Tile<T, DH> L;
  typedef typename Operand<T>::type Frag;
  constexpr int kTile = QT * L::kRow, kWave = 32 * L::kRow;
  constexpr bool VR = kValuesInRegisters<T, DH, SW>;
  extern __shared__ __align__(16) unsigned char smem[];   // two stages of Q and dO (32 rows a wave besides), the workgroup's V
  float *const s_lse = reinterpret_cast<float *>(smem + 4 * kTile + (VR ? 0 : Shared<SW>::kRowWaves * kWave)), *const s_delta = s_lse + 2 * QT;   // [stage][QT] each, behind V
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, h = lane >> 5;
  const int hk = blockIdx.x % a.s.kv_heads;
  Sequence sq;
  int block, place = 0, chunk = 0;
  if constexpr (MODE == kSinks) {
    const int item = blockIdx.x / a.s.kv_heads;
    block = item / a.sink_slots;
    place = item - block * a.sink_slots;
    if (!find_chunk(a.s, place, a.sink_chunk, sq, chunk)) return;
  } else if (!find_block<BK, false>(a.s, blockIdx.x / a.s.kv_heads, a.by_work, sq, block)) {
    const SpareRows spare = spare_rows<BK>(a.s.k_start, a.s.batch, a.s.k_tokens, block);
    zero_rows<T, DH>(a.dk, hk, spare, tid, NT);
    zero_rows<T, DH>(a.dv, hk, spare, tid, NT);
    return;
  }
  const Shared<SW> mate(wave);
  const int k0 = block * BK + mate.rows * 32, off = sq.nk - sq.nq;
  const int rows = min(32, sq.nk - k0);
  const int64_t row = int64_t(sq.k_first) + k0, es = int64_t(sizeof(T));
  // Tiles of queries begin with the first that sees a key: those before it have no gradient to give, and may hold anything.
  // Queries that some of the block's keys are hidden from, if one of them is not finite, or its weights are not numbers (log-sum-exp or
  // delta tells), are added one by one when the tiles are done.  So are those of a last tile that is not full: the rows it lacks repeat
  // the last query's with weights of 0, which do not hide it where it is not finite.
  // (With a window they are all added one by one then: those that some of the keys are too far behind for too.)
  const int base = max(-off, 0), unseen = block * BK - off - base;       // (of the block's first key, from base on)
  const int sinks = MODE == kWindow ? (a.sink_part ? 0 : a.s.sinks) : a.s.sinks;     // whose queries behind the window are this workgroup's
  const bool all = MODE == kCausal || (MODE == kWindow && block * BK < sinks);     // every query from the diagonal on
  const int diagonal = MODE == kSinks ? chunk + max(block * BK + a.s.window - off - chunk, 0) / QT * QT : base + max(unseen, 0) / QT * QT;
  const int limit = MODE == kSinks ? min(chunk + a.sink_chunk, sq.nq)
                                   : all ? sq.nq : min(sq.nq, max(block * BK + BK - 1 + a.s.window - off, diagonal));     // of those the last one
  const int tiled = MODE == kCausal ? sq.nq : min(diagonal + (max(limit - diagonal, 0) + QT - 1) / QT * QT, sq.nq);    // ... with those that fill its tile
  const int behind = MODE == kCausal ? min(base + (max(unseen + BK - 1, 0) + QT - 1) / QT * QT, sq.nq) : limit;
  const int end = MODE == kCausal ? (sq.nq > behind ? base + (sq.nq - base) / QT * QT : sq.nq) : limit;
  // Of the pairs of the lane's key: those whose query is at least (kSinks), or less than this far behind it.
  const int reach = MODE == kSinks ? (k0 + c < sinks ? a.s.window : INT_MAX) : k0 + c < sinks ? INT_MAX : a.s.window;
  auto hidden = [&](int behind_it) {                        // query's position - key
    if constexpr (MODE == kCausal) return behind_it < 0;
    if constexpr (MODE == kSinks) return behind_it < reach;
    return uint32_t(behind_it) >= uint32_t(reach);
  };
  bool odd = false;
  for (int j = 0; j < a.s.group; ++j) {
    const size_t row0 = row_value(a.s.q_start != nullptr, sq.b, sq.q_first, a.s.q_tokens, a.s.heads, hk * a.s.group + j);
    auto look = [&](int i) { odd |= !(subtrahend(a.lse[row0 + i]) < INFINITY && fabsf(a.delta[row0 + i]) < INFINITY); };
    if constexpr (MODE == kCausal) {
      for (int i = diagonal + tid; i < behind; i += NT) look(i);
      if (end < sq.nq && tid == NT - 1) look(sq.nq - 1);
    } else {
      // on the diagonal, and from the first that is too far from some of the keys
      const int near = MODE == kSinks ? diagonal : min(base + max(unseen + BK - 1, 0), tiled);
      const int far = MODE == kSinks ? diagonal : max(block * BK + a.s.window - off, near);
      for (int i = diagonal + tid; i < near; i += NT) look(i);
      for (int i = far + tid; i < tiled; i += NT) look(i);
      if (tiled == sq.nq && diagonal < tiled && tid == NT - 1) look(sq.nq - 1);
    }
  }
  odd = any_of_four(__builtin_amdgcn_ballot_w64(odd) != 0, reinterpret_cast<int *>(s_delta + 2 * QT));
  const int first = odd ? behind : diagonal, stop = odd ? end : MODE == kCausal ? sq.nq : limit;
  const int per = first < stop ? (stop - first + QT - 1) / QT : 0, tiles = per * a.s.group;
  const float scale = a.s.scale_log2;
  const bool packed = a.s.q_start != nullptr;
  const uint32_t base0 = __builtin_amdgcn_readfirstlane(lds_offset(smem)), share = base0 + uint32_t(wave) * 1024u;
  Reader<T, DH, sizeof(T) == 2> read(base0 + uint32_t(mate.part * kWave), lane);
  const TileLoad<T, DH, QT, NT> lq(a.q.token * es, tid), ld(a.d_out.token * es, tid);
  // The tile after the last one loaded: its head's rows, its first query.  From the last query back to the diagonal: the workgroups of
  // a head start with the same tiles, one reads what the others find in the L2.
  const int final = first + (per - 1) * QT;
  // With a window the workgroups of a head have ranges that overlap: each begins with the tile whose number is a multiple of their length,
  // so that they are at the same tile at the same time all the same (from their last ones on 1027 us a step for 1018, 8 x 2048 tokens of
  // 32 heads over 8, window 508).
  const int begin = MODE == kWindow && per > 0 ? final - (final / QT) % per * QT : final;
  const char *qp = reinterpret_cast<const char *>(a.q.p + sq.b * a.q.seq + sq.q_first * a.q.token + hk * a.s.group * a.q.head);
  const char *dp = reinterpret_cast<const char *>(a.d_out.p + sq.b * a.d_out.seq + sq.q_first * a.d_out.token + hk * a.s.group * a.d_out.head);
  size_t at = row_value(packed, sq.b, sq.q_first, a.s.q_tokens, a.s.heads, hk * a.s.group);
  int next = begin;
  float row_lse = 0.f, row_delta = 0.f;
  auto load = [&](int stage) {
    lq(qp + next * (a.q.token * es), sq.nq - next, share + uint32_t(stage * 2 * kTile));
    ld(dp + next * (a.d_out.token * es), sq.nq - next, share + uint32_t(stage * 2 * kTile + kTile));
    if (tid < QT) {
      const bool there = next + tid < sq.nq;
      row_lse = there ? subtrahend(a.lse[at + next + tid]) : INFINITY;
      row_delta = there ? a.delta[at + next + tid] : 0.f;
    }
    next -= QT;
    if (MODE == kWindow && next < first) next = final;
    if (MODE == kWindow ? next == begin : next < first) {
      next = begin;
      qp += a.q.head * es;
      dp += a.d_out.head * es;
      at += a.s.q_tokens;
    }
  };
  auto hand_over = [&](int stage) {
    if (tid < QT) {
      s_lse[stage * QT + tid] = row_lse;
      s_delta[stage * QT + tid] = row_delta;
    }
  };
  unsigned char *own = smem + wave * kWave;
  constexpr int kVAt = 4 * kTile;
  static_assert(4 * kTile >= 4 * kWave, "the waves' own rows end where V begins, or before");
  Frag kf[ST];
  operand_rows<T, DH, sizeof(T) == 2>(kf, read, reinterpret_cast<const char *>(a.k.p + sq.b * a.k.seq + row * a.k.token + hk * a.k.head), a.k.token * es, rows, own,
                      uint32_t((wave - mate.part) * kWave), lane);
  Frag vf[VR ? ST : 1];
  if constexpr (VR)
    operand_rows<T, DH, sizeof(T) == 2>(vf, read, reinterpret_cast<const char *>(a.v.p + sq.b * a.v.seq + row * a.v.token + hk * a.v.head), a.v.token * es,
                                        rows, own, uint32_t((wave - mate.part) * kWave), lane);
  else if (rows > 0 && mate.part == 0)
    carry_rows<T, DH>(reinterpret_cast<const char *>(a.v.p + sq.b * a.v.seq + row * a.v.token + hk * a.v.head), a.v.token * es, rows,
                      smem + kVAt + mate.rows * kWave, lane);
  __syncthreads();
  if (tiles > 0) load(0);
  hand_over(0);
  const uint32_t v_ahead = uint32_t(kVAt + (mate.rows - mate.part) * kWave);   // of the reader at stage 0
  f32x16 dk[DB], dv[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) dk[db] = dv[db] = f32x16{0.f};
  int tile = begin + QT;
  for (int it = 0; it < tiles; ++it) {
    tile -= QT;
    if (tile < first) tile = final;
    const int q0 = tile + mate.part * 32;                   // the wave's first query of the tile
    arrived();
    __syncthreads();
    if (it + 1 < tiles) load(~it & 1);
    // Operands on their way ahead of their products, arithmetic between products (a wave issues in order).  A tile that none of the wave's
    // keys is seen from is worked on like any other: its weights are zeros.
    const uint32_t va = v_ahead - uint32_t((it & 1) * 2 * kTile);
    const float *const rows_lse = s_lse + (it & 1) * QT + mate.part * 32 + 4 * h, *const rows_delta = rows_lse + 2 * QT;
    Frag x[4], y[4];                                        // rings, four products deep
    f32x16 s = {0.f}, g = {0.f};
#pragma unroll
    for (int t = 0; t < 4; ++t) x[t] = read.by_row(0, 0, t);
#pragma unroll
    for (int t = 0; t < ST; ++t) {
      pin();
      s = Operand<T>::mma(x[t & 3], kf[t], s);
      x[t & 3] = t + 4 < ST ? read.by_row(0, 0, t + 4) : read.by_row(kTile, 0, t + 4 - ST);
      if (!VR && t >= ST - 4) y[t - ST + 4] = read.by_row(va, 0, t - ST + 4);
    }
    pin();
    // some of the queries do not see some of the wave's keys
    const bool partial = MODE == kSinks ? k0 + 31 >= sinks || q0 + off - k0 - 31 < a.s.window
                                        : q0 + off < k0 + 31 || (MODE == kWindow && q0 + off + 31 - k0 >= a.s.window && k0 + 31 >= sinks);
    if (partial) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (hidden(q0 + off - k0 + (4 * h - c) + 8 * (r >> 2) + (r & 3))) s[r] = -INFINITY;
    }
    auto next_of = [&](int i) {                             // columns in the order of the last four groups of products
      const int db = i % DB, t = i / DB;
      return t < 2 ? read.transposed(kTile, 0, t, db) : read.transposed(0, 0, t - 2, db);
    };
#pragma unroll
    for (int t = 0; t < ST; ++t) {
      pin();
      g = Operand<T>::mma(x[t & 3], VR ? vf[VR ? t : 0] : y[t & 3], g);
      x[t & 3] = t + 4 < ST ? read.by_row(kTile, 0, t + 4) : next_of(t + 4 - ST);
      if (!VR && t + 4 < ST) y[t & 3] = read.by_row(va, 0, t + 4);
      if (t % (ST / 4) == 0) {
        const int r4 = t / (ST / 4);
        const f32x4 lse = *reinterpret_cast<const f32x4 *>(rows_lse + 8 * r4);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[4 * r4 + i] = __builtin_amdgcn_exp2f(fmaf(s[4 * r4 + i], scale, -lse[i]));
      }
    }
    pin();
    // dv takes p; meanwhile g becomes p (g - delta)
    auto scaled = [&](int r4) {
      const f32x4 delta = *reinterpret_cast<const f32x4 *>(rows_delta + 8 * r4);
#pragma unroll
      for (int i = 0; i < 4; ++i) g[4 * r4 + i] = s[4 * r4 + i] * (g[4 * r4 + i] - delta[i]);
    };
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const Frag pf = Operand<T>::of(s, t);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const int i = t * DB + db;
        pin();
        dv[db] = Operand<T>::mma(x[i & 3], pf, dv[db]);
        x[i & 3] = next_of(i + 4);
        if (db % (DB / 2) == 0) scaled(2 * t + db / (DB / 2));
      }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const Frag gf = Operand<T>::of(g, t);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const int i = (2 + t) * DB + db;
        pin();
        dk[db] = Operand<T>::mma(x[i & 3], gf, dk[db]);
        if (i + 4 < 4 * DB) x[i & 3] = next_of(i + 4);
      }
    }
    pin();
    if (it + 1 < tiles) hand_over(~it & 1);
    read.move(it & 1 ? uint32_t(-2 * kTile) : uint32_t(2 * kTile));
  }
  __syncthreads();
  if (MODE == kWindow && a.sink_part && block * BK < a.s.sinks) {
    // What the chunks gave the block's first keys: all threads add up 32 keys' sums, in the stages' place, and the wave that has the keys
    // takes them (a wave by itself, whose registers are full, loads one after the other: 568 us for 387 at 8 x 2048 tokens).
    static_assert(64 * DH * 4 <= 4 * kTile, "sums of a wave's keys");
    const Chunks chunks(a.s, sq, a.sink_chunk);
    f32x4 *const total = reinterpret_cast<f32x4 *>(smem);
    const size_t step = sink_sums<DH>(a.s, 1, 0, 0) / 4;
    for (int w = 0; w < BK / 32 && block * BK + 32 * w < min(a.s.sinks, sq.nk); ++w) {
      const f32x4 *const sums = reinterpret_cast<const f32x4 *>(a.sink_part + sink_sums<DH>(a.s, chunks.first, hk, block * (BK / 32) + w));
      const int fours = min((a.s.sinks - block * BK - 32 * w + 3) / 4, 8);       // four keys at a time, those that are first ones
      for (int item = tid; item < 2 * DH * fours; item += NT) {
        const int i = item / fours * 8 + item % fours;
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
        for (int j = 0; j < chunks.n; ++j) sum += sums[i + j * step];
        total[i] = sum;
      }
      __syncthreads();
      if (mate.rows == w && mate.part == 0 && block * BK + 32 * w + c / 4 * 4 < a.s.sinks) {
        add_sums(dk, reinterpret_cast<const float *>(total), 1.f, lane);
        add_sums(dv, reinterpret_cast<const float *>(total) + 32 * DH, 1.f, lane);
      }
      __syncthreads();
    }
  }
  if constexpr (SW > 1) {
    constexpr int kFloats = 64 * 16 * DB * 2, kPart = Shared<SW>::kRowWaves * kFloats;
    static_assert(4 * kWave + (SW - 1) * kPart * 4 <= 4 * kTile, "the parts' sums lie in the stages, behind the waves' own rows");
    float *const parts = reinterpret_cast<float *>(smem + 4 * kWave) + mate.rows * kFloats;
    if (mate.part > 0) {
      put_sums(dk, parts + (mate.part - 1) * kPart, lane);
      put_sums(dv, parts + (mate.part - 1) * kPart + kFloats / 2, lane);
    }
    __syncthreads();
    if (mate.part > 0) return;
#pragma unroll
    for (int i = 0; i < SW - 1; ++i) {
      add_sums(dk, parts + i * kPart, 1.f, lane);
      add_sums(dv, parts + i * kPart + kFloats / 2, 1.f, lane);
    }
  }
  if (rows <= 0) return;
  if (odd) {
    // a lane: its key, half of the elements
    const int64_t key = row + min(c, rows - 1);
    const T *kr = a.k.p + sq.b * a.k.seq + key * a.k.token + hk * a.k.head + 4 * h, *vr = a.v.p + sq.b * a.v.seq + key * a.v.token + hk * a.v.head + 4 * h;
    for (int j = 0; j < a.s.group; ++j) {
      const int head = hk * a.s.group + j;
      const size_t row0 = row_value(packed, sq.b, sq.q_first, a.s.q_tokens, a.s.heads, head);
      for (int i = diagonal < behind ? diagonal : end; i < (MODE == kCausal ? sq.nq : limit); i = i + 1 == behind ? end : i + 1) {
        const int64_t query = int64_t(sq.q_first) + i;
        const T *qr = a.q.p + sq.b * a.q.seq + query * a.q.token + head * a.q.head + 4 * h;
        const T *dr = a.d_out.p + sq.b * a.d_out.seq + query * a.d_out.token + head * a.d_out.head + 4 * h;
        float w = 0.f, x = 0.f;
#pragma unroll 1
        for (int e = 0; e < DH; e += 8)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            w = fmaf(to_float(qr[e + r]), to_float(kr[e + r]), w);
            x = fmaf(to_float(dr[e + r]), to_float(vr[e + r]), x);
          }
        w = add_lane_xor<32>(w);
        x = add_lane_xor<32>(x);
        w = __builtin_amdgcn_exp2f(fmaf(w, scale, -subtrahend(a.lse[row0 + i])));
        x = w * (x - a.delta[row0 + i]);
        if (!hidden(i + off - k0 - c)) {
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int e = 32 * db + 8 * (r >> 2) + (r & 3);
              dv[db][r] = fmaf(w, to_float(dr[e]), dv[db][r]);
              dk[db][r] = fmaf(x, to_float(qr[e]), dk[db][r]);
              if (r % 4 == 3) pin();
            }
        }
      }
    }
  }
  if constexpr (MODE == kSinks) {
    float *const to = a.sink_part + sink_sums<DH>(a.s, place, hk, k0 / 32);
    put_sums(dk, to, lane);
    put_sums(dv, to + 32 * DH, lane);
    return;
  }
  if (MODE == kWindow && k0 + a.s.window <= off && k0 + 31 >= a.s.sinks) {
    // a key that no query sees may hold anything
    const bool seen = k0 + c + a.s.window > off || k0 + c < a.s.sinks;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        dk[db][r] = seen ? dk[db][r] : 0.f;
        dv[db][r] = seen ? dv[db][r] : 0.f;
      }
  }
  store_rows<T, DH>(dk, a.s.scale, own, reinterpret_cast<char *>(a.dk.p + sq.b * a.dk.seq + row * a.dk.token + hk * a.dk.head), a.dk.token * es, rows,
                    nullptr, 0, lane);
  store_rows<T, DH>(dv, 1.f, own, reinterpret_cast<char *>(a.dv.p + sq.b * a.dv.seq + row * a.dv.token + hk * a.dv.head), a.dv.token * es, rows,
                    nullptr, 0, lane);
}

template <typename T, int DH, int SW, bool WIN>
hipError_t launch_dq(BackwardArgs<T> a, hipStream_t st) {
  constexpr int lds = kDqWords<T, DH, SW> + 16;
  static_assert(SW == 1 || 4 * (SW - 1) / SW * 256 * (DH / 2) <= kDqStage<T, DH, SW>, "the parts' sums lie in the first stage");
  const hipError_t e = allow_lds(&prompt_dq_kernel<T, DH, SW, WIN>, lds);
  if (e != hipSuccess) return e;
  const long long blocks = blocks_at_most(a.s.q_start, a.s.batch, a.s.q_tokens, Shared<SW>::kRows) * a.s.heads;
  a.by_work = blocks > 256 && blocks < 1024;      // (as in prompt_attend.hip)
  hipLaunchKernelGGL((prompt_dq_kernel<T, DH, SW, WIN>), dim3(unsigned(blocks)), dim3(256), lds, st, a);
  return hipGetLastError();
}

template <typename T, int DH, int SW, int MODE>
hipError_t launch_dkv(BackwardArgs<T> a, hipStream_t st) {
  // two stages of Q and dO, V, a stage's log-sum-exps and deltas twice, four words
  constexpr int rows = 4 * 32 * SW + (kValuesInRegisters<T, DH, SW> ? 0 : Shared<SW>::kRows), lds = rows * Tile<T, DH>::kRow + 4 * 32 * SW * 4 + 16;
  const hipError_t e = allow_lds(&prompt_dkv_kernel<T, DH, SW, MODE>, lds);
  if (e != hipSuccess) return e;
  const int sinks = a.s.sinks < a.s.k_tokens ? a.s.sinks : a.s.k_tokens;
  const long long items = MODE == kSinks ? (long long)a.sink_slots * ((sinks + Shared<SW>::kRows - 1) / Shared<SW>::kRows)
                                         : blocks_at_most(a.s.k_start, a.s.batch, a.s.k_tokens, Shared<SW>::kRows);
  const long long blocks = items * a.s.kv_heads;
  a.by_work = blocks > 256 && blocks < 2048;   // 1024, with 4 to 64 tiles of 4 heads each: 796 -> 610 us
  hipLaunchKernelGGL((prompt_dkv_kernel<T, DH, SW, MODE>), dim3(unsigned(blocks)), dim3(256), lds, st, a);
  return hipGetLastError();
}

template <typename T, int DH, bool WIN>
hipError_t launch_backward(const BackwardArgs<T> &a, hipStream_t st) {
  constexpr int SW = DH * sizeof(T) == 512 ? 2 : 4;  // (as many as two stages leave LDS for)
  constexpr int MODE = WIN ? kWindow : kCausal;
  hipError_t e = hipSuccess;
  if (a.s.q_tokens > 0) e = share_queries<T>(a.s) ? launch_dq<T, DH, SW, WIN>(a, st) : launch_dq<T, DH, 1, WIN>(a, st);
  if constexpr (WIN) {
    if (e == hipSuccess && a.sink_part) e = launch_dkv<T, DH, SW, kSinks>(a, st);
  }
  if (e == hipSuccess && a.s.k_tokens > 0) e = share_keys<T>(a.s) ? launch_dkv<T, DH, SW, MODE>(a, st) : launch_dkv<T, DH, 1, MODE>(a, st);
  return e;
}

size_t delta_bytes(const adore_prompt_config &c, bool packed) {
  const size_t n = size_t(c.heads) * c.q_tokens * (packed ? 1 : c.batch);
  return (n * sizeof(float) + 255) / 256 * 256 + 256;    // never 0: that says "not taken"
}

template <typename T, bool WIN>
int backward_typed(const adore_prompt_config &c, const PromptShape &s, const adore_rows *d_out, const adore_rows *q, const adore_rows *k,
                   const adore_rows *v, const adore_rows *out, const adore_rows *rest, const float *lse, const adore_rows *dq,
                   const adore_rows *dk, const adore_rows *dv, void *workspace, hipStream_t st) {
  BackwardArgs<T> a;
  a.s = s;
  a.d_out = rows_of<const T>(d_out);
  a.q = rows_of<const T>(q);
  a.k = rows_of<const T>(k);
  a.v = rows_of<const T>(v);
  a.out = rows_of<const T>(out);
  a.rest = rest ? rows_of<const T>(rest) : Rows<const T>{nullptr, 0, 0, 0};
  a.dq = rows_of<T>(dq);
  a.dk = rows_of<T>(dk);
  a.dv = rows_of<T>(dv);
  a.lse = lse;
  a.delta = static_cast<float *>(workspace);
  a.sink_part = nullptr;
  a.sink_chunk = a.sink_slots = 0;
  if constexpr (WIN) {
    const SinkPlan p = plan_sinks(s, c.head_dim, s.q_start != nullptr);
    if (p.slots > 0) {
      a.sink_part = reinterpret_cast<float *>(static_cast<char *>(workspace) + delta_bytes(c, s.q_start != nullptr));
      a.sink_chunk = p.chunk;
      a.sink_slots = p.slots;
    }
  }
  const hipError_t e = c.head_dim == 128 ? launch_backward<T, 128, WIN>(a, st) : launch_backward<T, 64, WIN>(a, st);
  return e == hipSuccess ? ADORE_OK : ADORE_E_HIP;
}

size_t backward_bytes(const adore_prompt_config &c, const PromptShape &s, bool packed, bool window) {
  return delta_bytes(c, packed) + (window ? plan_sinks(s, c.head_dim, packed).bytes : 0);
}

template <bool WIN>
int backward_prompts(const adore_prompt_config *cfg, const PromptShape &s, const adore_rows *d_out, const adore_rows *q, const adore_rows *k,
                     const adore_rows *v, const adore_rows *out, const adore_rows *rest, const float *lse, const adore_rows *dq,
                     const adore_rows *dk, const adore_rows *dv, void *workspace, size_t workspace_bytes, void *hip_stream) {
  for (const adore_rows *r : {d_out, q, k, v, out, dq, dk, dv})
    if (!prompt_rows_ok(r, cfg->dtype)) return ADORE_E_INVALID;
  if (!lse || !workspace || (rest && (cfg->dtype != ADORE_BF16 || !prompt_rows_ok(rest, cfg->dtype)))) return ADORE_E_INVALID;
  if (workspace_bytes < backward_bytes(*cfg, s, s.q_start != nullptr, WIN) || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0)
    return ADORE_E_WORKSPACE;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return cfg->dtype == ADORE_BF16 ? backward_typed<bf16_t, WIN>(*cfg, s, d_out, q, k, v, out, rest, lse, dq, dk, dv, workspace, st)
                                  : backward_typed<float, WIN>(*cfg, s, d_out, q, k, v, out, rest, lse, dq, dk, dv, workspace, st);
}

}  // namespace

}  // namespace adore

extern "C" {

size_t adore_prompt_backward_workspace_bytes(const adore_prompt_config *cfg, int32_t packed) {
  adore::PromptShape s;
  const int32_t some = 0, *start = packed ? &some : nullptr;   // (not read: the checks look at whether there are starts)
  if (adore::prompt_shape(cfg, start, start, &s) != ADORE_OK) return 0;
  return adore::backward_bytes(*cfg, s, packed != 0, false);
}

int adore_prompt_attention_backward(const adore_prompt_config *cfg, const int32_t *q_start, const int32_t *k_start, const adore_rows *d_out,
                                    const adore_rows *q, const adore_rows *k, const adore_rows *v, const adore_rows *out,
                                    const adore_rows *rest, const float *lse, const adore_rows *dq, const adore_rows *dk, const adore_rows *dv,
                                    void *workspace, size_t workspace_bytes, void *hip_stream) {
  adore::PromptShape s;
  const int rc = adore::prompt_shape(cfg, q_start, k_start, &s);
  return rc != ADORE_OK ? rc
                        : adore::backward_prompts<false>(cfg, s, d_out, q, k, v, out, rest, lse, dq, dk, dv, workspace, workspace_bytes, hip_stream);
}

size_t adore_window_backward_workspace_bytes(const adore_prompt_config *cfg, const adore_window *window, int32_t packed) {
  adore::PromptShape s;
  const int32_t some = 0, *start = packed ? &some : nullptr;
  if (adore::prompt_shape(cfg, start, start, &s) != ADORE_OK || adore::window_shape(window, &s) != ADORE_OK) return 0;
  return adore::backward_bytes(*cfg, s, packed != 0, true);
}

int adore_window_attention_backward(const adore_prompt_config *cfg, const adore_window *window, const int32_t *q_start, const int32_t *k_start,
                                    const adore_rows *d_out, const adore_rows *q, const adore_rows *k, const adore_rows *v,
                                    const adore_rows *out, const adore_rows *rest, const float *lse, const adore_rows *dq,
                                    const adore_rows *dk, const adore_rows *dv, void *workspace, size_t workspace_bytes, void *hip_stream) {
  adore::PromptShape s;
  int rc = adore::prompt_shape(cfg, q_start, k_start, &s);
  if (rc == ADORE_OK) rc = adore::window_shape(window, &s);
  return rc != ADORE_OK ? rc
                        : adore::backward_prompts<true>(cfg, s, d_out, q, k, v, out, rest, lse, dq, dk, dv, workspace, workspace_bytes, hip_stream);
}

}  // extern "C"
