// Gradients of causal attention over whole prompts (prompt_attend.hip), for packed sequences of any lengths and grouped heads.
//
//   p_ij = exp(w_ij - lse_i),  g_ij = p_ij (do_i . v_j - delta_i),  delta_i = do_i . out_i
//   dq_i = scale sum_j g_ij k_j;   dk_j = scale sum_i g_ij q_i,   dv_j = sum_i p_ij do_i   (i over the queries of all heads of j's group)
//
// Three launches without atomics, so that a gradient's bits do not hang on the order of workgroups: delta; dq, whose workgroups own
// queries and go over the keys; dk and dv, whose workgroups own keys and go over the queries of the group.  The weights are made anew
// in both (seven products instead of the five that one pass would need, which would have to add dq up in memory).
// delta wants out as it was before P and it were rounded: from the rounded one a short row's gradients are up to 2.2 times as far off as
// their own rounding, so the forward can take P in two terms and hand out what rounding left (rest): 1.4 times.
#include <hip/hip_runtime.h>

#include "prompt_device.h"

namespace adore {

namespace {

constexpr float kLog2e = 1.4426950408889634f;

template <typename T>
struct BackwardArgs {
  PromptShape s;
  Rows<const T> d_out, q, k, v, out, rest;   // rest.p may be null
  Rows<T> dq, dk, dv;
  const float *lse;
  float *delta;                              // laid out like lse
};

// ---- delta: DH / EPL lanes a row, 16 bytes each ----
template <typename T, int DH>
__global__ __launch_bounds__(256) void prompt_delta_kernel(const BackwardArgs<T> a, int rows) {
  constexpr int EPL = Vec16<T>::EPL, LPR = DH / EPL;
  const int64_t i = (int64_t(blockIdx.x) * 256 + threadIdx.x) / LPR;      // token x head, heads fastest
  if (i >= int64_t(rows) * a.s.heads) return;                             // (whole rows leave together)
  const int head = int(i % a.s.heads), row = int(i / a.s.heads), sub = threadIdx.x % LPR;
  const bool packed = a.s.q_start != nullptr;
  const int b = packed ? 0 : row / a.s.q_tokens, t = packed ? row : row - b * a.s.q_tokens;
  float x[EPL], y[EPL], z[EPL], sum = 0.f;
  Vec16<T>::load(a.d_out.p + b * a.d_out.seq + t * a.d_out.token + head * a.d_out.head + sub * EPL, x);
  Vec16<T>::load(a.out.p + b * a.out.seq + t * a.out.token + head * a.out.head + sub * EPL, y);
#pragma unroll
  for (int e = 0; e < EPL; ++e) sum = fmaf(x[e], y[e], sum);
  if (a.rest.p) {
    Vec16<T>::load(a.rest.p + b * a.rest.seq + t * a.rest.token + head * a.rest.head + sub * EPL, z);
#pragma unroll
    for (int e = 0; e < EPL; ++e) sum = fmaf(x[e], z[e], sum);
  }
  sum = group_sum<LPR>(sum);
  if (sub == 0) a.delta[row_value(packed, b, 0, a.s.q_tokens, a.s.heads, head) + t] = sum;
}

// 32 rows from `base` (zeros beyond `rows`) as an operand, through the wave's own LDS.
template <typename T, int DH>
__device__ __forceinline__ void operand_rows(typename Operand<T>::type (&f)[DH / 16], const char *base, int64_t stride, int rows,
                                             unsigned char *own, int lane) {
  Carrier<T, DH, 32, 64> carry;
  wave_lds_fence();
  if (rows > 0) {
    carry.template load<true>(base, stride, 0, rows, lane);
    carry.store(own, lane);
  }
  wave_lds_fence();
#pragma unroll
  for (int t = 0; t < DH / 16; ++t) f[t] = Tile<T, DH>::by_row(own, lane & 31, t, lane >> 5);
}

// ---- dq: 128 queries a workgroup, 32 a wave ----
template <typename T>
constexpr int kDqKeys = sizeof(T) == 2 ? 64 : 32;

template <typename T, int DH>
__global__ __launch_bounds__(256, 2) void prompt_dq_kernel(const BackwardArgs<T> a) {
  constexpr int NT = 256, BQ = 128, KT = kDqKeys<T>, KB = KT / 32, DB = DH / 32, ST = DH / 16;
  typedef Tile<T, DH> L;
  typedef typename Operand<T>::type Frag;
  constexpr int kTile = KT * L::kRow;
  extern __shared__ __align__(16) unsigned char smem[];   // K 0, K 1, V 0, V 1
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, h = lane >> 5;
  const int hk = blockIdx.x % a.s.kv_heads, item = blockIdx.x / a.s.kv_heads, head = hk * a.s.group + item % a.s.group;
  Sequence sq;
  int block;
  if (!find_block<BQ, true>(a.s, item / a.s.group, sq, block)) {
    int first;
    const int n = tail_rows<BQ>(a.s.q_start, a.s.batch, a.s.q_tokens, block, first);
    zero_rows<T, DH>(a.dq, head, first, n, tid, NT);
    return;
  }
  block = (sq.nq + BQ - 1) / BQ - 1 - block;
  const int q0 = block * BQ + wave * 32, off = sq.nk - sq.nq;
  const int rows = min(32, sq.nq - q0);
  const int64_t row = int64_t(sq.q_first) + q0, es = int64_t(sizeof(T));
  const char *kp = reinterpret_cast<const char *>(a.k.p + sq.b * a.k.seq + sq.k_first * a.k.token + hk * a.k.head);
  const char *vp = reinterpret_cast<const char *>(a.v.p + sq.b * a.v.seq + sq.k_first * a.v.token + hk * a.v.head);
  unsigned char *own = smem + wave * (32 * L::kRow);
  Frag qf[ST], df[ST];
  operand_rows<T, DH>(qf, reinterpret_cast<const char *>(a.q.p + sq.b * a.q.seq + row * a.q.token + head * a.q.head), a.q.token * es, rows, own, lane);
  operand_rows<T, DH>(df, reinterpret_cast<const char *>(a.d_out.p + sq.b * a.d_out.seq + row * a.d_out.token + head * a.d_out.head),
                      a.d_out.token * es, rows, own, lane);
  __syncthreads();
  float lse = INFINITY, delta = 0.f;            // of the lane's query; weights of a query that is not there are 0
  if (c < rows) {
    const size_t at = row_value(a.s.q_start != nullptr, sq.b, sq.q_first, a.s.q_tokens, a.s.heads, head) + q0 + c;
    lse = a.lse[at] * kLog2e;
    delta = a.delta[at];
  }
  f32x16 dq[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) dq[db] = f32x16{0.f};
  const int last = min(block * BQ + BQ, sq.nq) - 1 + off, tiles = last < 0 ? 0 : last / KT + 1;
  const int mine = rows > 0 ? q0 + rows - 1 + off : -1, seen = q0 + c + off;
  const float scale = a.s.scale_log2;
  Carrier<T, DH, KT, NT> ck, cv;
  auto load = [&](int k0) {
    ck.template load<true>(kp, a.k.token * es, k0, sq.nk, tid);
    cv.template load<true>(vp, a.v.token * es, k0, sq.nk, tid);
  };
  auto store = [&](unsigned char *to) {
    ck.store(to, tid);
    cv.store(to + 2 * kTile, tid);
  };
  if (tiles > 0) {
    load(0);
    store(smem);
  }
  for (int it = 0; it < tiles; ++it) {
    const unsigned char *kt = smem + (it & 1) * kTile, *vt = kt + 2 * kTile;
    const int k0 = it * KT;
    __syncthreads();
    if (it + 1 < tiles) load(k0 + KT);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const int kf = k0 + kb * 32;
      if (kf > mine) continue;
      f32x16 s = {0.f}, g = {0.f};
#pragma unroll
      for (int t = 0; t < ST; ++t) s = Operand<T>::mma(L::by_row(kt, kb * 32 + c, t, h), qf[t], s);
#pragma unroll
      for (int t = 0; t < ST; ++t) g = Operand<T>::mma(L::by_row(vt, kb * 32 + c, t, h), df[t], g);
      const bool partly = kf + 31 > q0 + off;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float p = __builtin_amdgcn_exp2f(fmaf(s[r], scale, -lse));
        g[r] = (partly && kf + 8 * (r >> 2) + 4 * h + (r & 3) > seen) ? 0.f : p * (g[r] - delta);
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const Frag gf = Operand<T>::of(g, t);
#pragma unroll
        for (int db = 0; db < DB; ++db) dq[db] = Operand<T>::mma(L::transposed(kt, kb * 32, t, db, lane), gf, dq[db]);
      }
    }
    if (it + 1 < tiles) store(smem + (~it & 1) * kTile);
  }
  __syncthreads();
  if (rows <= 0) return;
  store_rows<T, DH>(dq, a.s.scale, own, reinterpret_cast<char *>(a.dq.p + sq.b * a.dq.seq + row * a.dq.token + head * a.dq.head),
                    a.dq.token * es, rows, nullptr, 0, lane);
}

// ---- dk and dv: 128 keys a workgroup, 32 a wave ----
template <typename T>
constexpr int kDkvQueries = 32;

template <typename T, int DH>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void prompt_dkv_kernel(const BackwardArgs<T> a) {
  constexpr int NT = 256, BK = 128, QT = kDkvQueries<T>, QB = QT / 32, DB = DH / 32, ST = DH / 16;
  typedef Tile<T, DH> L;
  typedef typename Operand<T>::type Frag;
  constexpr int kTile = QT * L::kRow;
  extern __shared__ __align__(16) unsigned char smem[];   // Q 0, Q 1, dO 0, dO 1
  __shared__ __align__(16) float s_lse[2][QT], s_delta[2][QT];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, h = lane >> 5;
  const int hk = blockIdx.x % a.s.kv_heads;
  Sequence sq;
  int block;
  if (!find_block<BK, false>(a.s, blockIdx.x / a.s.kv_heads, sq, block)) {
    int first;
    const int n = tail_rows<BK>(a.s.k_start, a.s.batch, a.s.k_tokens, block, first);
    zero_rows<T, DH>(a.dk, hk, first, n, tid, NT);
    zero_rows<T, DH>(a.dv, hk, first, n, tid, NT);
    return;
  }
  const int k0 = block * BK + wave * 32, off = sq.nk - sq.nq;
  const int rows = min(32, sq.nk - k0);
  const int64_t row = int64_t(sq.k_first) + k0, es = int64_t(sizeof(T));
  unsigned char *own = smem + wave * (32 * L::kRow);
  Frag kf[ST], vf[ST];
  operand_rows<T, DH>(kf, reinterpret_cast<const char *>(a.k.p + sq.b * a.k.seq + row * a.k.token + hk * a.k.head), a.k.token * es, rows, own, lane);
  operand_rows<T, DH>(vf, reinterpret_cast<const char *>(a.v.p + sq.b * a.v.seq + row * a.v.token + hk * a.v.head), a.v.token * es, rows, own, lane);
  __syncthreads();
  f32x16 dk[DB], dv[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) dk[db] = dv[db] = f32x16{0.f};
  const int first = max(block * BK - off, 0) / QT * QT;
  const int per = first < sq.nq ? (sq.nq - first + QT - 1) / QT : 0, tiles = per * a.s.group;
  const float scale = a.s.scale_log2;
  const bool packed = a.s.q_start != nullptr;
  Carrier<T, DH, QT, NT> cq, cd;
  float row_lse = 0.f, row_delta = 0.f;
  auto load = [&](int it) {
    const int head = hk * a.s.group + it / per, q0 = first + it % per * QT;
    cq.template load<true>(reinterpret_cast<const char *>(a.q.p + sq.b * a.q.seq + sq.q_first * a.q.token + head * a.q.head), a.q.token * es, q0, sq.nq, tid);
    cd.template load<true>(reinterpret_cast<const char *>(a.d_out.p + sq.b * a.d_out.seq + sq.q_first * a.d_out.token + head * a.d_out.head),
                           a.d_out.token * es, q0, sq.nq, tid);
    if (tid < QT) {
      const bool there = q0 + tid < sq.nq;
      const size_t at = row_value(packed, sq.b, sq.q_first, a.s.q_tokens, a.s.heads, head) + q0 + tid;
      row_lse = there ? a.lse[at] * kLog2e : INFINITY;
      row_delta = there ? a.delta[at] : 0.f;
    }
  };
  auto store = [&](int it) {
    unsigned char *to = smem + (it & 1) * kTile;
    cq.store(to, tid);
    cd.store(to + 2 * kTile, tid);
    if (tid < QT) {
      s_lse[it & 1][tid] = row_lse;
      s_delta[it & 1][tid] = row_delta;
    }
  };
  if (tiles > 0) {
    load(0);
    store(0);
  }
  for (int it = 0; it < tiles; ++it) {
    const unsigned char *qt = smem + (it & 1) * kTile, *dt = qt + 2 * kTile;
    const int q0 = first + it % per * QT;
    __syncthreads();
    if (it + 1 < tiles) load(it + 1);
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const int qf = q0 + qb * 32;
      if (qf + 31 + off < k0) continue;
      f32x16 s = {0.f}, g = {0.f};
#pragma unroll
      for (int t = 0; t < ST; ++t) s = Operand<T>::mma(L::by_row(qt, qb * 32 + c, t, h), kf[t], s);
#pragma unroll
      for (int t = 0; t < ST; ++t) g = Operand<T>::mma(L::by_row(dt, qb * 32 + c, t, h), vf[t], g);
      const bool partly = qf + off < k0 + 31;
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const f32x4 lse = *reinterpret_cast<const f32x4 *>(&s_lse[it & 1][qb * 32 + 8 * r4 + 4 * h]);
        const f32x4 delta = *reinterpret_cast<const f32x4 *>(&s_delta[it & 1][qb * 32 + 8 * r4 + 4 * h]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 4 * r4 + i;
          const bool hidden = partly && k0 + c > qf + 8 * r4 + 4 * h + i + off;
          const float p = __builtin_amdgcn_exp2f(fmaf(s[r], scale, -lse[i]));
          s[r] = hidden ? 0.f : p;
          g[r] = hidden ? 0.f : p * (g[r] - delta[i]);
        }
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const Frag pf = Operand<T>::of(s, t), gf = Operand<T>::of(g, t);
#pragma unroll
        for (int db = 0; db < DB; ++db) dv[db] = Operand<T>::mma(L::transposed(dt, qb * 32, t, db, lane), pf, dv[db]);
#pragma unroll
        for (int db = 0; db < DB; ++db) dk[db] = Operand<T>::mma(L::transposed(qt, qb * 32, t, db, lane), gf, dk[db]);
      }
    }
    if (it + 1 < tiles) store(it + 1);
  }
  __syncthreads();
  if (rows <= 0) return;
  store_rows<T, DH>(dk, a.s.scale, own, reinterpret_cast<char *>(a.dk.p + sq.b * a.dk.seq + row * a.dk.token + hk * a.dk.head), a.dk.token * es, rows,
                    nullptr, 0, lane);
  store_rows<T, DH>(dv, 1.f, own, reinterpret_cast<char *>(a.dv.p + sq.b * a.dv.seq + row * a.dv.token + hk * a.dv.head), a.dv.token * es, rows,
                    nullptr, 0, lane);
}

template <typename F>
hipError_t allow_lds(F *kernel, int bytes) {
  return hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

template <typename T, int DH>
hipError_t launch_backward(const BackwardArgs<T> &a, hipStream_t st) {
  constexpr int row = Tile<T, DH>::kRow, waves = 4 * 32 * row;         // every wave's own 32 rows at the beginning and the end
  constexpr int dq_tiles = 4 * kDqKeys<T> * row, dkv_tiles = 4 * kDkvQueries<T> * row;
  constexpr int dq_lds = dq_tiles > waves ? dq_tiles : waves, dkv_lds = dkv_tiles > waves ? dkv_tiles : waves;
  hipError_t e = allow_lds(&prompt_dq_kernel<T, DH>, dq_lds);
  if (e == hipSuccess) e = allow_lds(&prompt_dkv_kernel<T, DH>, dkv_lds);
  if (e != hipSuccess) return e;
  if (a.s.q_tokens > 0) {
    const int rows = a.s.q_start ? a.s.q_tokens : a.s.batch * a.s.q_tokens, per = 256 / (DH / Vec16<T>::EPL);
    const long long blocks = ((long long)rows * a.s.heads + per - 1) / per;
    hipLaunchKernelGGL((prompt_delta_kernel<T, DH>), dim3(unsigned(blocks)), dim3(256), 0, st, a, rows);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL((prompt_dq_kernel<T, DH>), dim3(unsigned(blocks_at_most(a.s.q_start, a.s.batch, a.s.q_tokens, 128) * a.s.heads)), dim3(256),
                       dq_lds, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.s.k_tokens > 0)
    hipLaunchKernelGGL((prompt_dkv_kernel<T, DH>), dim3(unsigned(blocks_at_most(a.s.k_start, a.s.batch, a.s.k_tokens, 128) * a.s.kv_heads)),
                       dim3(256), dkv_lds, st, a);
  return hipGetLastError();
}

size_t delta_bytes(const adore_prompt_config &c, bool packed) {
  const size_t n = size_t(c.heads) * c.q_tokens * (packed ? 1 : c.batch);
  return (n * sizeof(float) + 255) / 256 * 256 + 256;    // never 0: that says "not taken"
}

template <typename T>
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
  const hipError_t e = c.head_dim == 128 ? launch_backward<T, 128>(a, st) : launch_backward<T, 64>(a, st);
  return e == hipSuccess ? ADORE_OK : ADORE_E_HIP;
}

}  // namespace

}  // namespace adore

extern "C" {

size_t adore_prompt_backward_workspace_bytes(const adore_prompt_config *cfg, int32_t packed) {
  adore::PromptShape s;
  const int32_t some = 0, *start = packed ? &some : nullptr;   // (not read: the checks look at whether there are starts)
  if (adore::prompt_shape(cfg, start, start, &s) != ADORE_OK) return 0;
  return adore::delta_bytes(*cfg, packed != 0);
}

int adore_prompt_attention_backward(const adore_prompt_config *cfg, const int32_t *q_start, const int32_t *k_start, const adore_rows *d_out,
                                    const adore_rows *q, const adore_rows *k, const adore_rows *v, const adore_rows *out,
                                    const adore_rows *rest, const float *lse, const adore_rows *dq, const adore_rows *dk, const adore_rows *dv,
                                    void *workspace, size_t workspace_bytes, void *hip_stream) {
  using namespace adore;
  PromptShape s;
  const int rc = prompt_shape(cfg, q_start, k_start, &s);
  if (rc != ADORE_OK) return rc;
  for (const adore_rows *r : {d_out, q, k, v, out, dq, dk, dv})
    if (!prompt_rows_ok(r, cfg->dtype)) return ADORE_E_INVALID;
  if (!lse || !workspace || (rest && (cfg->dtype != ADORE_BF16 || !prompt_rows_ok(rest, cfg->dtype)))) return ADORE_E_INVALID;
  if (workspace_bytes < delta_bytes(*cfg, q_start != nullptr) || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0) return ADORE_E_WORKSPACE;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return cfg->dtype == ADORE_BF16 ? backward_typed<bf16_t>(*cfg, s, d_out, q, k, v, out, rest, lse, dq, dk, dv, workspace, st)
                                  : backward_typed<float>(*cfg, s, d_out, q, k, v, out, rest, lse, dq, dk, dv, workspace, st);
}

}  // extern "C"
