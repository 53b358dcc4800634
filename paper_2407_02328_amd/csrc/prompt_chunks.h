// Sequences of a call on prompts, and how with a window the queries behind it are cut for the first keys' gradients: which places of the
// workspace a sequence's sums have.  Whole numbers only, and no HIP: what the host plans and the kernels do is the same code, which tests run on
// the host.
#pragma once

#include <cstddef>
#include <cstdint>

#if defined(__HIP__)
#define ADORE_BOTH __host__ __device__ __forceinline__
#else
#define ADORE_BOTH inline
#endif

namespace adore {

ADORE_BOTH int less_of(int a, int b) { return a < b ? a : b; }
ADORE_BOTH int more_of(int a, int b) { return a > b ? a : b; }

// A problem's sequences and heads.
struct PromptShape {
  const int32_t *q_start, *k_start;   // [batch + 1], or null: every sequence has q_tokens / k_tokens
  int batch, heads, kv_heads, group, q_tokens, k_tokens;
  float scale, scale_log2;            // and times log2(e)
  int window, sinks;                  // of kernels with a window: a query sees its last `window` keys and the first `sinks`
};

struct Sequence {
  int b;
  int q_first, k_first;   // first rows in packed tensors (0 in dense ones)
  int nq, nk;
};

// Starts are the caller's device memory: whatever they hold, rows stay within the packed tensors.
ADORE_BOTH void span(const int32_t *start, int b, int total, int &first, int &n) {
  const int s = less_of(more_of(start[b], 0), total), e = less_of(more_of(start[b + 1], 0), total);
  first = s;
  n = more_of(e - s, 0);
}

ADORE_BOTH Sequence sequence_at(const PromptShape &a, int b) {
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

// With a window a block of keys is seen by few queries, but the first keys by all that follow: one workgroup would go over a whole prompt
// while the others go over a window.  So the queries behind the window (p - j >= window) are cut into chunks, each a workgroup's, whose
// sums for 32 first keys (a wave's registers, fp32) go to memory; the workgroup of the block that holds the keys adds them to its own.
// A sequence's chunks: n places from `first` on.
struct Chunks {
  int first, n;
  int from;                                  // the first query that is as far as the window from key 0
  ADORE_BOTH Chunks(const PromptShape &a, const Sequence &s, int chunk) {
    from = more_of(a.window - (s.nk - s.nq), 0);
    n = s.nq > from ? (s.nq - from + chunk - 1) / chunk : 0;
    // packed: of the sequences that have chunks no two are in the same run of window + 1 keys (whatever the starts hold: no place is
    // beyond SinkPlan::slots)
    first = a.q_start ? s.q_first / chunk + less_of(s.b, s.k_first / (a.window + 1)) : s.b * ((a.q_tokens + chunk - 1) / chunk);
  }
};

// The sums of place `place`, kv head hk, for keys 32 i .. 32 i + 31: dk's registers of 64 lanes, then dv's.
template <int DH>
ADORE_BOTH size_t sink_sums(const PromptShape &a, int place, int hk, int i) {
  return ((size_t(place) * a.kv_heads + hk) * ((less_of(a.sinks, a.k_tokens) + 63) / 64 * 2) + i) * (64 * DH);
}

// How the queries behind the window of the first keys are cut (slots 0: not at all, the workgroup of a block of keys goes over them).
struct SinkPlan {
  int chunk, slots;
  size_t bytes;
};
inline SinkPlan plan_sinks(const PromptShape &s, int head_dim, bool packed) {
  SinkPlan p = {0, 0, 0};
  const long long sinks = s.sinks < s.k_tokens ? s.sinks : s.k_tokens, groups = (sinks + 63) / 64 * 2;
  const long long queries = (long long)s.q_tokens * (packed ? 1 : s.batch);
  if (sinks == 0 || s.k_tokens <= s.window) return p;
  // It is a launch more, against one workgroup for each kv head that goes over so many more queries than the others.  Not cut / cut, us
  // (sequences x tokens, heads / kv heads, window; 4 first keys):
  //   64 elements    3 x 128, 4 / 4, 32: 17 / 25;  4 x 256, 8 / 8, 32: 20 / 28;  512, 4 / 2, 64: 32 / 35;  2048, 4 / 4, 1000: 52 / 50;
  //                  2 x 2048, 8 / 2, 100: 133 / 60;  60000, 4 / 4, 1000: 2824 / 408
  //   128 elements   8 x 512, 8 / 2, 64: 69 / 76;  32 x 512, 16 / 4, 128: 249 / 232;  4 x 1000, 4 / 1, 200: 102 / 88;  1024, 8 / 2, 128: 93 / 69;
  //                  4096, 8 / 2, 256: 350 / 105;  16384, 8 / 1, 512: 2669 / 390;  8 x 2048, 32 / 8, 508: 873 / 757
  // Packed lengths are not known here, and one may be nearly all: 8192 tokens before 60 sequences of 100, 8 / 2 heads, 256: 1851 / 198; 2000
  // before 40 of 50, 128: 326 / 83; 8 x 512, 64: 73 / 80.
  if (((long long)s.q_tokens - s.window - 128) * s.group < (packed ? 2048 : 1024)) return p;
  // 256 workgroups, chunks of 128 queries or more (256: 76 us for 69 at 1024 tokens, 109 for 105 at 4096, 748 for 757 at 8 x 2048)
  long long chunk = (queries * s.kv_heads * groups / 2 / 256 + 127) / 128 * 128;
  if (chunk < 128) chunk = 128;
  if (chunk > s.q_tokens) chunk = (s.q_tokens + 127) / 128 * 128;
  const long long long_ones = (long long)s.k_tokens / (s.window + 1);
  const long long slots = packed ? s.q_tokens / chunk + (s.batch < long_ones ? s.batch : long_ones) + 1 : s.batch * ((s.q_tokens + chunk - 1) / chunk);
  const long long bytes = slots * s.kv_heads * groups * 64 * head_dim * 4;
  if (bytes > (256ll << 20)) return p;       // (many short sequences: there is little to cut)
  p.chunk = int(chunk);
  p.slots = int(slots);
  p.bytes = size_t(bytes);
  return p;
}

}  // namespace adore
