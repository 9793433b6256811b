// The best continuations of each request over its beams and the vocabulary: score(b, i, t) = scores[b][i] + x[b][i][t] - lse(x[b][i]), the k largest,
// equal ones in the order of beam and token.
//
// What bounds it: the logits, read once.  beam_rows_kernel: a workgroup has a row or a stretch of it; every wavefront walks over a contiguous part with
// 16-byte loads one round ahead and keeps, per lane, a running maximum and sum of exponentials, and, per wavefront, the best tokens sorted over its
// lanes.  After the first round hardly any logit is above the k-th best one so far: what is goes into a buffer that is sorted in when it is full, so a
// logit costs a maximum, a comparison and an exponential.  beam_pick_kernel: a request's stretches meet; scores are formed and compared in 64 bits, so
// that candidates of different beams that lie next to each other come in their right order.
#include "percache_internal.hpp"

namespace {
typedef unsigned long long u64;
typedef unsigned u32x4_ __attribute__((ext_vector_type(4)));

constexpr int kMaxBest = 64, kMaxBeams = 64, kWaves = 4, kPickThreads = 512;
constexpr int kPickMost = 2048;   // candidates of a request that the second kernel holds
constexpr float kLog2e = 1.44269504088896340736f;

// what a stretch of a row leaves: its maximum, sum of e^(x - maximum), and best tokens, best first (value, token; token -1: none)
struct Stretch { double sum; float top; int32_t pad; };

// a float as an unsigned number in the same order (-0 below 0: they are made equal where a key is formed)
__device__ __forceinline__ unsigned ordered(float x) {
  const unsigned u = __float_as_uint(x);
  return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_ordered(unsigned u) { return __uint_as_float(u ^ ((u >> 31) ? 0x80000000u : 0xffffffffu)); }
// larger logits first, equal ones by the lower token; 0 is below every logit that is one
__device__ __forceinline__ u64 key_of(float x, unsigned token) { return ((u64)ordered(x + 0.f) << 32) | (0xffffffffu - token); }

__device__ __forceinline__ u64 shfl_xor64(u64 x, int m) {
  return ((u64)(unsigned)__shfl_xor((int)(x >> 32), m, 64) << 32) | (unsigned)__shfl_xor((int)x, m, 64);
}
__device__ __forceinline__ u64 shfl64(u64 x, int l) {
  return ((u64)(unsigned)__shfl((int)(x >> 32), l, 64) << 32) | (unsigned)__shfl((int)x, l, 64);
}
// the keys of a wavefront's lanes, largest in lane 0
__device__ __forceinline__ u64 sort64(u64 x, int lane) {
#pragma unroll
  for (int size = 2; size <= 64; size <<= 1)
#pragma unroll
    for (int step = size >> 1; step > 0; step >>= 1) {
      const u64 y = shfl_xor64(x, step);
      const bool larger = ((lane & step) == 0) == ((lane & size) == 0);
      x = larger ? (x > y ? x : y) : (x > y ? y : x);
    }
  return x;
}
// the 64 largest of two sorted lists
__device__ __forceinline__ u64 merge64(u64 a, u64 b, int lane) {
  const u64 r = shfl64(b, 63 - lane);
  u64 x = a > r ? a : r;
#pragma unroll
  for (int step = 32; step > 0; step >>= 1) {
    const u64 y = shfl_xor64(x, step);
    x = (lane & step) == 0 ? (x > y ? x : y) : (x > y ? y : x);
  }
  return x;
}

// e^d for d <= 0.  The difference is taken before the product with log2(e): the sum of a row is compared to the last places of 32 bits, and a reference
// multiplied beforehand would move every term of it by the same 2^-24 of the reference.
__device__ __forceinline__ float exp_below(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }

// NV vectors of 16 bytes a lane and round; T: the logits' type
template <class T>
__global__ __launch_bounds__(64 * kWaves) void beam_rows_kernel(const T *__restrict__ logits, long row_stride, int vocab, int n_stretch, int best, Stretch *__restrict__ st_out,
                                                               u64 *__restrict__ list_out) {
  constexpr int PER = 16 / (int)sizeof(T), NV = 4, EACH = NV * PER;   // logits of a lane and round
  __shared__ u64 buffer[kWaves][128];
  __shared__ u64 lists[kWaves][kMaxBest];
  __shared__ float tops[kWaves];
  __shared__ double sums[kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row = blockIdx.x / n_stretch, stretch = blockIdx.x - row * n_stretch;
  const T *x = logits + (long)row * row_stride;
  // the row as [vectors | tail]; the stretches and wavefronts share the vectors in order, the tail goes to the last of them.  The vectors start with the
  // row, at whatever address (16-byte loads need no alignment here): rows of equal logits have equal sums, to the bit, wherever they lie.
  const int vecs = vocab / PER, tail0 = vecs * PER;
  const int part = stretch * kWaves + wave, parts = n_stretch * kWaves;
  const int v0 = (int)((long)part * vecs / parts), v1 = (int)((long)(part + 1) * vecs / parts);
  typedef unsigned vec_at __attribute__((ext_vector_type(4), aligned(2)));

  u64 list = 0;          // sorted over the lanes; 0: none
  u64 kth = 0;           // the best-th of them
  float bar = -INFINITY; // its logit: what is not above it does not get in (later tokens of this wavefront come after equal ones)
  int held = 0;          // keys in the buffer
  float m = -INFINITY, l = 0.f;

  auto flush = [&]() __attribute__((always_inline)) {
    const u64 fresh = sort64(lane < held ? buffer[wave][lane] : 0ull, lane);
    list = merge64(list, fresh, lane);
    kth = shfl64(list, best - 1);
    if (kth) bar = from_ordered((unsigned)(kth >> 32));
    // (at most 63 keys stay)
    const u64 rest = lane + 64 < held ? buffer[wave][lane + 64] : 0ull;
    buffer[wave][lane] = rest;
    held = max(held - 64, 0);
  };
  auto offer = [&](u64 key) __attribute__((always_inline)) {   // 0: nothing
    const u64 mask = __builtin_amdgcn_ballot_w64(key > kth);
    if (!mask) return;
    if (key > kth) buffer[wave][held + __popcll(mask & ((1ull << lane) - 1))] = key;
    held += __popcll(mask);
    if (held >= 64) flush();
  };
  // Adds EACH logits of a lane to its maximum and sum and offers those that may be among the best.  Logit i is that of token
  // token0 + i / PER * 64 * PER + i % PER.  What is above the bar that the round began with is read again (from cache) when it is offered: rounds in
  // which something is are few, and the values stay in registers under constant indexes only.
  auto take = [&](const float (&v)[EACH], int token0) __attribute__((always_inline)) {
    float top = v[0];
#pragma unroll
    for (int i = 1; i < EACH; ++i) top = fmaxf(top, v[i]);
    const float mn = fmaxf(m, top), ref = mn == -INFINITY ? 0.f : mn;
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int i = 0; i < EACH; i += 2) {
      s0 += exp_below(v[i] - ref);
      s1 += exp_below(v[i + 1] - ref);
    }
    l = (m == -INFINITY ? l : l * exp_below(m - ref)) + (s0 + s1);   // (a sum that is NaN stays)
    m = mn;
    float least = bar;
    const bool unset = kth == 0;
    bool equal_too = false;
    if (unset) {   // the best-th of the lanes' own best ones bounds the best-th of all from below
      const u64 own = sort64(top > -INFINITY ? (u64)ordered(top + 0.f) << 32 | 1u : 0ull, lane), bound = shfl64(own, best - 1);
      if (bound) {
        least = from_ordered((unsigned)(bound >> 32));
        equal_too = true;
      }
    }
    if (!__builtin_amdgcn_ballot_w64(top > least || (equal_too && top == least))) return;
    unsigned wanted = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) wanted |= (unsigned)(v[i] > least || (equal_too && v[i] == least)) << i;
    while (__builtin_amdgcn_ballot_w64(wanted != 0)) {
      const int i = wanted ? __builtin_ctz(wanted) : 0, token = token0 + i / PER * (64 * PER) + i % PER;
      u64 key = 0;
      if (wanted) key = key_of((float)x[token], token);
      wanted &= wanted - 1;
      offer(key);
    }
    if (unset && kth == 0 && held >= best) flush();
  };
  auto load = [&](u32x4_ (&raw)[NV], int v) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < NV; ++j) raw[j] = *(const vec_at *)(x + (long)min(v + j * 64 + lane, v1 - 1) * PER);
  };
  auto few = [&](int from, int n) __attribute__((always_inline)) {   // n < PER logits, one a lane
    const float v = lane < n ? (float)x[from + lane] : -INFINITY, mn = fmaxf(m, v), ref = mn == -INFINITY ? 0.f : mn;
    l = (m == -INFINITY ? l : l * exp_below(m - ref)) + exp_below(v - ref);
    m = mn;
    offer(v > bar ? key_of(v, from + lane) : 0ull);
  };
  if (v0 < v1) {
    u32x4_ raw[NV], next[NV];
    load(raw, v0);
    for (int v = v0; v < v1; v += NV * 64) {
      if (v + NV * 64 < v1) load(next, v + NV * 64);
      float f[EACH];
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const bool in = v + j * 64 + lane < v1;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
          float y;
          if constexpr (sizeof(T) == 2) y = __uint_as_float(e & 1 ? raw[j][e >> 1] & 0xffff0000u : raw[j][e >> 1] << 16);
          else y = __uint_as_float(raw[j][e]);
          f[j * PER + e] = in ? y : -INFINITY;
        }
      }
      take(f, (v + lane) * PER);
#pragma unroll
      for (int j = 0; j < NV; ++j) raw[j] = next[j];
    }
  }
  if (part == parts - 1 && tail0 < vocab) few(tail0, vocab - tail0);
  flush();
  if (held) flush();

  // the wavefront's maximum and sum, then the workgroup's
  float top = m;
#pragma unroll
  for (int sh = 1; sh < 64; sh <<= 1) top = fmaxf(top, __shfl_xor(top, sh, 64));
  double sum = m == -INFINITY ? (l == l ? 0.0 : (double)NAN) : (double)l * (double)exp_below(m - top);
#pragma unroll
  for (int sh = 1; sh < 64; sh <<= 1) sum += __shfl_xor(sum, sh, 64);
  if (lane == 0) {
    tops[wave] = top;
    sums[wave] = sum;
  }
  if (lane < kMaxBest) lists[wave][lane] = list;
  __syncthreads();
  if (wave != 0) return;
#pragma unroll
  for (int w = 1; w < kWaves; ++w) list = merge64(list, lists[w][lane], lane);
  if (lane < best) list_out[(size_t)blockIdx.x * best + lane] = list;
  if (lane == 0) {
    float t = tops[0];
    for (int w = 1; w < kWaves; ++w) t = fmaxf(t, tops[w]);
    double s = 0.0;
    for (int w = 0; w < kWaves; ++w) s += tops[w] == -INFINITY ? (sums[w] == sums[w] ? 0.0 : sums[w]) : sums[w] * exp((double)tops[w] - (double)t);
    st_out[blockIdx.x] = Stretch{s, t, 0};
  }
}

__device__ __forceinline__ u64 ordered64(double x) {
  const u64 u = (u64)__double_as_longlong(x + 0.0);
  return u ^ ((u64)((long long)u >> 63) | 0x8000000000000000ull);
}

// One workgroup a request.  Candidates in the order (beam, stretch, rank), which for equal scores is that of beam and token; those that reach a bound from
// 64 groups' best ones are counted against each other.
__global__ __launch_bounds__(kPickThreads) void beam_pick_kernel(const Stretch *__restrict__ stretches, const u64 *__restrict__ lists, const float *__restrict__ scores,
                                                                 int beams, int n_stretch, int best, int32_t *__restrict__ parent, int32_t *__restrict__ token,
                                                                 float *__restrict__ score) {
  __shared__ double base[kMaxBeams];   // score - lse of every beam, NaN where it has no candidates
  __shared__ u64 total[kPickMost];
  __shared__ u64 few[kPickMost];
  __shared__ uint16_t few_at[kPickMost];
  __shared__ u64 bound;
  __shared__ int n_few;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = beams * n_stretch * best;
  for (int i = wave; i < beams; i += kPickThreads / 64) {
    const Stretch *s = stretches + ((size_t)b * beams + i) * n_stretch;
    double sum = 0.0;
    float top = -INFINITY;
    for (int j = lane; j < n_stretch; j += 64) top = fmaxf(top, s[j].top);
#pragma unroll
    for (int sh = 1; sh < 64; sh <<= 1) top = fmaxf(top, __shfl_xor(top, sh, 64));
    for (int j = lane; j < n_stretch; j += 64) sum += s[j].top == -INFINITY ? s[j].sum : s[j].sum * exp((double)s[j].top - (double)top);
#pragma unroll
    for (int sh = 1; sh < 64; sh <<= 1) sum += __shfl_xor(sum, sh, 64);
    if (lane == 0) {
      const double lse = (double)top + log(sum), at = (double)scores[(size_t)b * beams + i];
      base[i] = isfinite(lse) && isfinite(at) ? at - lse : (double)NAN;
    }
  }
  if (tid == 0) n_few = 0;
  __syncthreads();
  const u64 *mine = lists + (size_t)b * n;
  for (int c = tid; c < n; c += kPickThreads) {
    const u64 key = mine[c];
    const double t = base[c / (n_stretch * best)] + (double)from_ordered((unsigned)(key >> 32));
    total[c] = key && t == t ? ordered64(t) : 0ull;
  }
  __syncthreads();
  // 64 groups of candidates: group g has those at g, g + 64, ...
  {
    u64 top = 0;
    for (int c = wave * 64 + lane; c < n; c += kPickThreads) top = total[c] > top ? total[c] : top;
    few[tid] = top;
  }
  __syncthreads();
  if (wave == 0) {
    u64 top = 0;
#pragma unroll
    for (int w = 0; w < kPickThreads / 64; ++w) top = few[w * 64 + lane] > top ? few[w * 64 + lane] : top;
    const u64 sorted = sort64(top, lane);
    if (lane == best - 1) bound = sorted;
  }
  __syncthreads();
  const u64 least = bound > 0 ? bound : 1ull;
  for (int c = tid; c < n; c += kPickThreads) {
    if (total[c] < least) continue;
    const int at = atomicAdd(&n_few, 1);   // (their order does not matter: each is counted against all of them)
    few[at] = total[c];
    few_at[at] = (uint16_t)c;
  }
  __syncthreads();
  const int count = n_few;
  for (int f = tid; f < count; f += kPickThreads) {
    const u64 t = few[f];
    const int at = few_at[f];
    int rank = 0;
    for (int o = 0; o < count && rank < best; ++o) rank += few[o] > t || (few[o] == t && (int)few_at[o] < at);
    if (rank >= best) continue;
    const u64 key = mine[at];
    const size_t to = (size_t)b * best + rank;
    const int beam = at / (n_stretch * best);
    parent[to] = beam;
    token[to] = (int32_t)(0xffffffffu - (unsigned)key);
    score[to] = (float)(base[beam] + (double)from_ordered((unsigned)(key >> 32)));
  }
  for (int r = count + tid; r < best; r += kPickThreads) {
    const size_t to = (size_t)b * best + r;
    parent[to] = token[to] = -1;
    score[to] = -INFINITY;
  }
}

// Stretches a row is cut into: two workgroups a CU where rows are few, none shorter than 2048 logits, and no more candidates of a request than
// beam_pick_kernel holds.
int stretches_for(int n_cu, long rows, int beams, int vocab, int best) {
  long s = (2L * n_cu + rows - 1) / rows;
  if (s > vocab / 2048) s = vocab / 2048;
  if (s > kPickMost / (beams * best)) s = kPickMost / (beams * best);
  return s < 1 ? 1 : (int)s;
}
}  // namespace

extern "C" {

size_t percache_beam_select_workspace_bytes(const percache_ctx *ctx, int32_t batch, int32_t beams, int32_t vocab, int32_t best) {
  if (!ctx || batch < 1 || beams < 1 || beams > kMaxBeams || vocab < 1 || best < 1 || best > kMaxBest || beams * best > kPickMost) return 0;
  const size_t n = (size_t)batch * beams * stretches_for(ctx->n_cu, (long)batch * beams, beams, vocab, best);
  return pc::align_up(n * sizeof(Stretch)) + pc::align_up(n * best * sizeof(u64));
}

pc_status percache_beam_select(percache_ctx *ctx, const void *logits_dev, int32_t fp32, int64_t row_stride, const float *scores_dev, int32_t batch, int32_t beams,
                               int32_t vocab, int32_t best, int32_t *parent_out_dev, int32_t *token_out_dev, float *score_out_dev, void *workspace_dev,
                               size_t workspace_bytes, void *stream) {
  if (!ctx) return PC_EINVAL;
  if (batch < 0 || (fp32 != 0 && fp32 != 1)) return pc::fail(ctx, PC_EINVAL, "batch is negative or fp32 neither 0 nor 1");
  if (beams < 1 || beams > kMaxBeams) return pc::fail(ctx, PC_ESHAPE, "beams %d outside [1,%d]", beams, kMaxBeams);
  if (best < 1 || best > kMaxBest) return pc::fail(ctx, PC_ESHAPE, "best %d outside [1,%d]", best, kMaxBest);
  if (beams * best > kPickMost) return pc::fail(ctx, PC_ESHAPE, "%d beams with %d best each are more than %d candidates", beams, best, kPickMost);
  if (vocab < 1) return pc::fail(ctx, PC_ESHAPE, "vocab must be positive");
  if (row_stride < vocab) return pc::fail(ctx, PC_EINVAL, "row stride %ld is shorter than a row of %d", (long)row_stride, vocab);
  if (batch == 0) return PC_OK;
  if (!logits_dev || !scores_dev || !parent_out_dev || !token_out_dev || !score_out_dev) return pc::fail(ctx, PC_EINVAL, "NULL tensor pointer");
  if ((uintptr_t)logits_dev % (fp32 ? 4 : 2) || ((uintptr_t)scores_dev | (uintptr_t)parent_out_dev | (uintptr_t)token_out_dev | (uintptr_t)score_out_dev) % 4)
    return pc::fail(ctx, PC_EINVAL, "tensor pointers must be aligned to their elements");
  const size_t need = percache_beam_select_workspace_bytes(ctx, batch, beams, vocab, best);
  if (!workspace_dev || workspace_bytes < need) return pc::fail(ctx, PC_ENOMEM, "workspace has %zu bytes, need %zu", workspace_bytes, need);
  if ((uintptr_t)workspace_dev % pc::kAlign) return pc::fail(ctx, PC_EINVAL, "workspace must be 256-byte aligned");
  const long rows = (long)batch * beams;
  const int ns = stretches_for(ctx->n_cu, rows, beams, vocab, best);
  Stretch *st = (Stretch *)workspace_dev;
  u64 *lists = (u64 *)((char *)workspace_dev + pc::align_up((size_t)rows * ns * sizeof(Stretch)));
  if (rows * ns >= (1L << 31)) return pc::fail(ctx, PC_ESHAPE, "more than 2^31 rows");
  hipStream_t s = (hipStream_t)stream;
  const dim3 grid((unsigned)(rows * ns));
  if (fp32) hipLaunchKernelGGL(beam_rows_kernel<float>, grid, dim3(64 * kWaves), 0, s, (const float *)logits_dev, (long)row_stride, vocab, ns, best, st, lists);
  else hipLaunchKernelGGL(beam_rows_kernel<__bf16>, grid, dim3(64 * kWaves), 0, s, (const __bf16 *)logits_dev, (long)row_stride, vocab, ns, best, st, lists);
  PC_HIP(ctx, hipGetLastError());
  hipLaunchKernelGGL(beam_pick_kernel, dim3((unsigned)batch), dim3(kPickThreads), 0, s, st, lists, scores_dev, beams, ns, best, parent_out_dev, token_out_dev, score_out_dev);
  PC_HIP(ctx, hipGetLastError());
  return PC_OK;
}

}  // extern "C"
