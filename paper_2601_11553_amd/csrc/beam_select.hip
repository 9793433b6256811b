// The best continuations of each request over its beams and the vocabulary: score(b, i, t) = scores[b][i] + x[b][i][t] - lse(x[b][i]), the k largest,
// equal ones in the order of beam and token.
//
// What bounds it: the logits, read once.  beam_rows_kernel: a workgroup has a row or a stretch of it, every lane a share of it, of which it keeps the running
// maximum, the sum of exponentials and the round that the maximum came in -- per logit a maximum, a difference, a product, an exponential and a sum,
// and no list.  64 groups of four lanes have k best tokens at or above the k-th best of their maxima; the lanes that reach it read the round of their maximum
// again (those whose second best round reaches it too all of theirs), and what reaches it, a few more than k as a rule, is put in order by counting.
// 512 rows of 131072 bf16 logits: 29.5 us, of which the stream of 134 MB takes 24 (19 without the exponentials) and what comes behind a stretch's last logit
// 5: the bound 1.3, the second look 2.5, order and the way out (with all of a lane's logits read again 7).
// beam_pick_kernel: a request's stretches meet (5.5 us for 64 requests of 8 x 2 x 16 candidates); scores are formed and compared in 64 bits, so that
// candidates of different beams that lie next to each other come in their right order.
#include "percache_internal.hpp"

namespace {
typedef unsigned long long u64;
typedef unsigned u32x4_ __attribute__((ext_vector_type(4)));

constexpr int kMaxBest = 64, kMaxBeams = 64, kWaves = 4, kThreads = 64 * kWaves, kPickThreads = 512;
constexpr int kFound = 2048;      // tokens that reach the bound of a stretch; more are taken one after the other
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

// over the 64 lanes: data-parallel moves inside 16 of them, then the rows change places
template <int CTRL>
__device__ __forceinline__ float moved(float x) { return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xf, 0xf, true)); }
template <int CTRL>
__device__ __forceinline__ u64 moved(u64 u) {
  const unsigned lo = __builtin_amdgcn_update_dpp(0, (unsigned)u, CTRL, 0xf, 0xf, true), hi = __builtin_amdgcn_update_dpp(0, (unsigned)(u >> 32), CTRL, 0xf, 0xf, true);
  return ((u64)hi << 32) | lo;
}
template <int CTRL>
__device__ __forceinline__ double moved(double x) {
  return __longlong_as_double((long long)moved<CTRL>((u64)__double_as_longlong(x)));
}
template <int CTRL>
__device__ __forceinline__ int moved(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xf, 0xf, true); }
// over 4 or 8 neighbouring lanes
template <int N>
__device__ __forceinline__ int sum_of(int x) {
  x += moved<0xB1>(x);
  x += moved<0x4E>(x);
  return N == 8 ? x + moved<0x141>(x) : x;
}
template <class X, class Op>
__device__ __forceinline__ X over_lanes(X x, Op op) {
  x = op(x, moved<0xB1>(x));     // lane ^ 1
  x = op(x, moved<0x4E>(x));     // lane ^ 2
  x = op(x, moved<0x141>(x));    // mirrored inside 8
  x = op(x, moved<0x140>(x));    // mirrored inside 16
  x = op(x, __shfl_xor(x, 16, 64));
  return op(x, __shfl_xor(x, 32, 64));
}
__device__ __forceinline__ float wave_max(float x) {
  return over_lanes(x, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ double wave_sum(double x) {
  return over_lanes(x, [](double a, double b) { return a + b; });
}

// e^d for d <= 0.  The difference is taken before the product with log2(e): the sum of a row is compared to the last places of 32 bits, and a reference
// multiplied beforehand would move every term of it by the same 2^-24 of the reference.
__device__ __forceinline__ float exp_below(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }

// NV vectors of 16 bytes a lane and round; T: the logits' type
template <class T>
__global__ __launch_bounds__(kThreads) void beam_rows_kernel(const T *__restrict__ logits, long row_stride, int vocab, int n_stretch, int best, Stretch *__restrict__ st_out,
                                                            u64 *__restrict__ list_out) {
  constexpr int PER = 16 / (int)sizeof(T), NV = 4, EACH = NV * PER, ROUND = NV * 64;   // logits of a lane and round; vectors of a wavefront and round
  __shared__ u64 found[kFound];
  __shared__ uint16_t again[kThreads];
  __shared__ float tops[kWaves];
  __shared__ double sums[kWaves];
  __shared__ u64 bound, next_best;
  __shared__ int n_found;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row = blockIdx.x / n_stretch, stretch = blockIdx.x - row * n_stretch;
  const T *x = logits + (long)row * row_stride;
  // the row as [vectors | tail]; the stretches and wavefronts share the vectors in order, the tail goes to the last of them.  The vectors start with the
  // row, at whatever address (16-byte loads need no alignment here): rows of equal logits have equal sums, to the bit, wherever they lie.
  const int vecs = vocab / PER, tail0 = vecs * PER, parts = n_stretch * kWaves;
  auto part_begin = [&](int w) __attribute__((always_inline)) { return (int)((long)(stretch * kWaves + w) * vecs / parts); };
  const int v0 = part_begin(wave), v1 = part_begin(wave + 1);
  const bool has_tail = stretch == n_stretch - 1 && wave == kWaves - 1 && lane < vocab - tail0;
  typedef unsigned vec_at __attribute__((ext_vector_type(4), aligned(2)));
  auto value = [&](const u32x4_ &raw, int e) __attribute__((always_inline)) {
    if constexpr (sizeof(T) == 2) return __uint_as_float(e & 1 ? raw[e >> 1] & 0xffff0000u : raw[e >> 1] << 16);
    else return __uint_as_float(raw[e]);
  };
  auto load = [&](u32x4_ (&raw)[NV], int v) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < NV; ++j) raw[j] = *(const vec_at *)(x + (long)min(v + j * 64 + lane, v1 - 1) * PER);
  };

  float m = -INFINITY, second = -INFINITY, l = 0.f;   // second: the largest in any round but m's
  int when = 0;   // first vector of the round that m came in
  const float tail = has_tail ? (float)x[tail0 + lane] : -INFINITY;
  auto take = [&](const u32x4_ (&raw)[NV], int v, auto whole_c) __attribute__((always_inline)) {
    float f[EACH];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < PER; ++e) f[j * PER + e] = decltype(whole_c)::value || v + j * 64 + lane < v1 ? value(raw[j], e) : -INFINITY;
    float top = f[0];
#pragma unroll
    for (int i = 1; i < EACH; ++i) top = fmaxf(top, f[i]);
    const float mn = fmaxf(m, top), ref = mn == -INFINITY ? 0.f : mn;
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int i = 0; i < EACH; i += 2) {
      s0 += exp_below(f[i] - ref);
      s1 += exp_below(f[i + 1] - ref);
    }
    l = (m == -INFINITY ? l : l * exp_below(m - ref)) + (s0 + s1);   // (a sum that is NaN stays)
    when = top > m ? v : when;
    second = fmaxf(second, fminf(m, top));
    m = mn;
  };
  if (v0 < v1) {
    u32x4_ raw[NV], next[NV];
    load(raw, v0);
    int v = v0;
    for (; v + ROUND <= v1; v += ROUND) {   // whole rounds
      if (v + ROUND < v1) load(next, v + ROUND);
      take(raw, v, std::true_type{});
#pragma unroll
      for (int j = 0; j < NV; ++j) raw[j] = next[j];
    }
    if (v < v1) take(raw, v, std::false_type{});
  }
  // keys that the lane's best token is not below, and not above (0: it has none)
  u64 least = m > -INFINITY ? key_of(m, (unsigned)(when + ROUND - 64 + lane) * PER + PER - 1) : 0ull;
  u64 most = m > -INFINITY ? key_of(m, (unsigned)((when + lane) * PER)) : 0ull;
  if (has_tail) {
    const float mn = fmaxf(m, tail), ref = mn == -INFINITY ? 0.f : mn;
    l = (m == -INFINITY ? l : l * exp_below(m - ref)) + exp_below(tail - ref);
    if (tail > m) least = key_of(tail, (unsigned)(tail0 + lane));
    m = mn;
  }
  // the best token of every group of four neighbouring lanes is not below:
  u64 group = least;
  u64 other = moved<0xB1>(group);
  group = other > group ? other : group;
  other = moved<0x4E>(group);
  group = other > group ? other : group;
  if ((lane & 3) == 0) found[tid >> 2] = group;
  if (tid == 0) {
    n_found = 0;
    bound = ~0ull;
  }
  __syncthreads();
  {   // (a group's lanes count a quarter of the others each)
    int above = 0;
#pragma unroll
    for (int j = 0; j < 16; ++j) above += found[j * 4 + (lane & 3)] > group;
    above = sum_of<4>(above);
    if ((lane & 3) == 0 && above < best) atomicMin(&bound, group ? group : 1ull);   // (fewer than `best` groups with a token: every one of theirs reaches it)
  }
  __syncthreads();
  const u64 reach = bound;
  auto put = [&](u64 key) __attribute__((always_inline)) {
    const int at = atomicAdd(&n_found, 1);   // (in any order: they are counted against each other)
    if (at < kFound) found[at] = key;
  };
  const u64 tail_key = tail > -INFINITY ? key_of(tail, (unsigned)(tail0 + lane)) : 0ull;
  if (tail_key >= reach) put(tail_key);
  // What reaches it is in lanes whose best token does, as a rule in that one's round alone: such a lane reads the round again.
  const float from = reach > 1ull ? from_ordered((unsigned)(reach >> 32)) : -INFINITY;
  const int each = (v1 - v0 + 63) / 64;
  const bool hit = most >= reach, whole = hit && (second >= from || each <= NV);
  auto look = [&](const u32x4_ &raw, int at, auto use) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const float y = value(raw, e);
      if (at < v1 && y >= from && y > -INFINITY) use(key_of(y, (unsigned)(at * PER + e)));
    }
  };
  // the others' vectors, all of them, are dealt out to the wavefront's lanes (and where there is one round: few lanes' are)
  auto enlist = [&](bool mine) __attribute__((always_inline)) {
    const u64 mask = __builtin_amdgcn_ballot_w64(mine);
    __builtin_amdgcn_wave_barrier();
    if (mine) again[wave * 64 + __popcll(mask & ((1ull << lane) - 1))] = (uint16_t)lane;
    __builtin_amdgcn_wave_barrier();
    return __popcll(mask) * each;
  };
  u32x4_ round[NV], more[2];
  int more_at[2];
  auto ask = [&](int item, int items) __attribute__((always_inline)) {   // two of them
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int i = (item + 64 * j) / each;
      more_at[j] = item + 64 * j < items ? v0 + again[wave * 64 + i] + (item + 64 * j - i * each) * 64 : v1;
      more[j] = *(const vec_at *)(x + (long)min(more_at[j], v1 - 1) * PER);
    }
  };
  if (hit && !whole) load(round, when);
  const int rest = enlist(whole);
  if (lane < rest) ask(lane, rest);
  // meanwhile the wavefront's maximum and sum
  const float top = wave_max(m);
  const double sum = wave_sum(m == -INFINITY ? (l == l ? 0.0 : (double)NAN) : (double)l * (double)exp_below(m - top));
  if (lane == 0) {
    tops[wave] = top;
    sums[wave] = sum;
  }
  auto put_if = [&](u64 key) __attribute__((always_inline)) { if (key >= reach) put(key); };
  if (hit && !whole)
#pragma unroll
    for (int j = 0; j < NV; ++j) look(round[j], when + j * 64 + lane, put_if);
  for (int item = lane; item < rest; item += 128) {
    if (item != lane) ask(item, rest);
#pragma unroll
    for (int j = 0; j < 2; ++j) look(more[j], more_at[j], put_if);
  }
  __syncthreads();
  if (wave == kWaves - 1) {
    float t = tops[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) t = fmaxf(t, tops[w]);
    const float mine = tops[lane & (kWaves - 1)];
    const double part = sums[lane & (kWaves - 1)];
    double all = mine == -INFINITY ? (part == part ? 0.0 : part) : part * (double)exp_below(mine - t);
    all += moved<0xB1>(all);
    all += moved<0x4E>(all);
    if (lane == 0) st_out[blockIdx.x] = Stretch{all, t, 0};
  }
  const int count = n_found;
  u64 *out = list_out + (size_t)blockIdx.x * best;
  if (count <= kFound) {
    for (int f = tid >> 2; f < count; f += kThreads / 4) {   // (four lanes a token)
      const u64 key = found[f];
      int above = 0;
#pragma unroll 4
      for (int o = lane & 3; o < count; o += 4) above += found[o] > key;
      above = sum_of<4>(above);
      if ((lane & 3) == 0 && above < best) out[above] = key;
    }
    for (int r = count + tid; r < best; r += kThreads) out[r] = 0;
    return;
  }
  // (the best ones of a stretch lie in few lanes: one after the other)
  const int items = enlist(hit);
  u64 before = ~0ull;
  for (int r = 0; r < best; ++r) {
    if (tid == 0) next_best = 0;
    __syncthreads();
    u64 own = tail_key < before ? tail_key : 0ull;
    for (int item = lane; item < items; item += 128) {
      ask(item, items);
#pragma unroll
      for (int j = 0; j < 2; ++j) look(more[j], more_at[j], [&](u64 key) __attribute__((always_inline)) { own = key < before && key > own ? key : own; });
    }
    atomicMax(&next_best, own);
    __syncthreads();
    before = next_best;
    if (tid == 0) out[r] = before;
    __syncthreads();
  }
}

__device__ __forceinline__ u64 ordered64(double x) {
  const u64 u = (u64)__double_as_longlong(x + 0.0);
  return u ^ ((u64)((long long)u >> 63) | 0x8000000000000000ull);
}

// One workgroup a request.  Candidate c = (list, rank), a list being a beam's stretch, in which order equal scores are those of beam and token.  The
// candidates are dealt out to 64 groups, the ranks of a list and the lists' first ones both to different groups; the best-th of the groups' best ones
// bounds the best-th of all from below, and what reaches it is counted against each other.
// Its time is the launch and one memory latency: the lists are asked for before the beams' log-sum-exps are formed.
__global__ __launch_bounds__(kPickThreads) void beam_pick_kernel(const Stretch *__restrict__ stretches, const u64 *__restrict__ lists, const float *__restrict__ scores,
                                                                 int beams, int n_stretch, int best, int32_t *__restrict__ parent, int32_t *__restrict__ token,
                                                                 float *__restrict__ score) {
  constexpr int EACH = kPickMost / kPickThreads;
  __shared__ double base[kMaxBeams];   // score - lse of every beam, NaN where it has no candidates
  __shared__ u64 groups[64], few[kPickMost], few_key[kPickMost];
  __shared__ uint16_t few_at[kPickMost];
  __shared__ u64 bound;
  __shared__ int n_few;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n_lists = beams * n_stretch, n = n_lists * best;
  const u64 *mine = lists + (size_t)b * n;
  u64 key[EACH];
#pragma unroll
  for (int j = 0; j < EACH; ++j) key[j] = tid + j * kPickThreads < n ? mine[tid + j * kPickThreads] : 0ull;
  if (tid < 64) groups[tid] = 0;
  for (int i = wave; i < beams; i += kPickThreads / 64) {
    const Stretch *s = stretches + ((size_t)b * beams + i) * n_stretch;
    const float from = scores[(size_t)b * beams + i];
    double sum = 0.0;
    float top = -INFINITY;
    for (int j = lane; j < n_stretch; j += 64) {   // (a lane's own stretches, then those of all lanes)
      const Stretch e = s[j];
      const float t = fmaxf(top, e.top);
      sum = (top == -INFINITY ? sum : sum * exp((double)top - (double)t)) + (e.top == -INFINITY ? (e.sum == e.sum ? 0.0 : e.sum) : e.sum * exp((double)e.top - (double)t));
      top = t;
    }
    if (n_stretch > 1) {
      const float t = wave_max(top);
      if (top != -INFINITY) sum *= exp((double)top - (double)t);
      sum = wave_sum(sum);
      top = t;
    }
    if (lane == 0) {
      const double lse = (double)top + log(sum);
      base[i] = isfinite(lse) && isfinite(from) ? (double)from - lse : (double)NAN;
    }
  }
  if (tid == 0) {
    n_few = 0;
    bound = ~0ull;
  }
  __syncthreads();
  u64 total[EACH];
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    const int c = tid + j * kPickThreads, list = c / best;
    const double t = base[min(list / n_stretch, beams - 1)] + (double)from_ordered((unsigned)(key[j] >> 32));
    total[j] = key[j] && t == t ? ordered64(t) : 0ull;
    if (total[j]) atomicMax(&groups[(5 * list + 13 * (c - list * best)) & 63], total[j]);
  }
  __syncthreads();
  {   // (eight lanes a group)
    const u64 top = groups[tid >> 3];
    int above = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) above += groups[j * 8 + (tid & 7)] > top;
    above = sum_of<8>(above);
    if ((tid & 7) == 0 && above < best) atomicMin(&bound, top ? top : 1ull);
  }
  __syncthreads();
  const u64 reach = bound;
#pragma unroll
  for (int j = 0; j < EACH; ++j)
    if (total[j] >= reach) {
      const int to = atomicAdd(&n_few, 1);   // (in any order)
      few[to] = total[j];
      few_key[to] = key[j];
      few_at[to] = (uint16_t)(tid + j * kPickThreads);
    }
  __syncthreads();
  const int count = n_few;
  for (int f = tid >> 3; f < count; f += kPickThreads / 8) {   // (eight lanes a candidate)
    const u64 t = few[f];
    const int c = few_at[f];
    int rank = 0;
#pragma unroll 4
    for (int o = tid & 7; o < count; o += 8) rank += few[o] > t || (few[o] == t && (int)few_at[o] < c);
    rank = sum_of<8>(rank);
    if ((tid & 7) || rank >= best) continue;
    const size_t to = (size_t)b * best + rank;
    const int beam = c / (n_stretch * best);
    parent[to] = beam;
    token[to] = (int32_t)(0xffffffffu - (unsigned)few_key[f]);
    score[to] = (float)(base[beam] + (double)from_ordered((unsigned)(few_key[f] >> 32)));
  }
  for (int r = count + tid; r < best; r += kPickThreads) {
    const size_t to = (size_t)b * best + r;
    parent[to] = token[to] = -1;
    score[to] = -INFINITY;
  }
}

// Stretches a row is cut into: four workgroups a CU (512 rows of 131072 logits: 29.6, 29.5, 31.2 us at two, four, eight; 64 rows 9.6, 8.6, 9.4), none shorter than 2048 logits, and no more
// candidates of a request than beam_pick_kernel holds.
int stretches_for(int n_cu, long rows, int beams, int vocab, int best) {
  long s = (4L * n_cu + rows - 1) / rows;
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
  if ((long)batch * beams >= 1L << 23) return pc::fail(ctx, PC_ESHAPE, "2^23 rows or more");   // (a grid has fewer than 2^32 threads)
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
