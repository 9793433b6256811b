// Verification of drafted tokens: each query brings a tree of t_draft nodes (a node behind its parent), all of them run through a layer at
// once.  Node i sits at position pos0 + depth(i) and attends over [cached chunks ; its ancestors ; itself],
//   o_i = sum_j e^(s_ij - lse_i) v_j,   s_ij = q_i.k_j / sqrt(D),   lse_i = log sum_j e^s_ij.
// The projection is that of qkv_rope_gemm.hip, the attention decode_attention.hip up to 32 rows a kv head and draft_attention.hip above.  Here are
// the host entry points, the lists they take -- positions of the nodes, and for the attention one word of 64 bits per node and 64 nodes that
// says which of them it looks at --, and the merge of the attention's partials with the nodes.
#include "decode_common.hpp"

namespace {

// One workgroup a query: ancestors by pointer doubling, sees[i] |= sees[up[i]], up[i] = up[up[i]], in log2(longest path) rounds, between the lanes of
// a wavefront (up to 64 nodes; 48 nodes 3.6 us through LDS, 2.6 so) or between two LDS buffers.  The parents come packed, two to a word, as a launch
// argument (FROM_ARG; with the words in front of them, which workgroup `batch` then copies) or from device memory.  16 bits of parents a node travel
// instead of 64 bits or more of `sees`: 8 queries of 64 nodes with their chunk list still fit a launch's arguments.
constexpr int kTreeThreads = 256;
template <bool FROM_ARG>
__global__ __launch_bounds__(kTreeThreads) void draft_lists_kernel(int32_t *dst, int n_words, const pc::ListWords lists, const int32_t *packed, int batch, int T,
                                                                   int rounds, uint2 *sees_out) {
  const int b = blockIdx.x, tid = threadIdx.x;
  if (b == (sees_out ? batch : 0)) {
    if constexpr (FROM_ARG) {
      constexpr int EACH = (pc::kListWords + kTreeThreads - 1) / kTreeThreads;
      int32_t w[EACH];   // (asked for together: the launch's arguments are host memory)
#pragma unroll
      for (int k = 0; k < EACH; ++k) w[k] = tid + k * kTreeThreads < n_words ? lists.v[min(tid + k * kTreeThreads, pc::kListWords - 1)] : 0;
#pragma unroll
      for (int k = 0; k < EACH; ++k)
        if (tid + k * kTreeThreads < n_words) dst[tid + k * kTreeThreads] = w[k];
    }
    return;
  }
  auto parent_of = [&](int i) __attribute__((always_inline)) {
    const int at = b * T + i, w = FROM_ARG ? lists.v[n_words + at / 2] : packed[at / 2];
    return (int)(int16_t)(at & 1 ? w >> 16 : w & 0xffff);
  };
  if (T <= 64) {   // one wavefront, a node a lane
    if (tid >= 64) return;
    int up = tid < T ? parent_of(tid) : -2;
    unsigned long long sees = up > -2 ? 1ull << tid : 0ull;
    for (int r = 0; r < rounds; ++r) {
      const unsigned long long theirs = __shfl(sees, max(up, 0), 64);
      const int further = __shfl(up, max(up, 0), 64);
      if (up >= 0) {
        sees |= theirs;
        up = further;
      }
    }
    if (tid < T) sees_out[(size_t)b * T + tid] = make_uint2((unsigned)sees, (unsigned)(sees >> 32));
    return;
  }
  constexpr int N = pc::kMaxNodes;
  __shared__ unsigned long long sees[2][N * (N / 64)];
  __shared__ int up[2][N];
  const int W = (T + 63) / 64;
  for (int i = tid; i < T; i += kTreeThreads) {
    const int p = parent_of(i);
    up[0][i] = p;
    for (int k = 0; k < W; ++k) sees[0][i * W + k] = p > -2 && k == i / 64 ? 1ull << (i & 63) : 0ull;
  }
  __syncthreads();
  int cur = 0;
  for (int r = 0; r < rounds; ++r, cur ^= 1) {
    for (int e = tid; e < T * W; e += kTreeThreads) {
      const int i = e / W, p = up[cur][i];
      sees[cur ^ 1][e] = sees[cur][e] | (p >= 0 ? sees[cur][p * W + e % W] : 0ull);
    }
    for (int i = tid; i < T; i += kTreeThreads) {
      const int p = up[cur][i];
      up[cur ^ 1][i] = p >= 0 ? up[cur][p] : p;
    }
    __syncthreads();
  }
  for (int e = tid; e < T * W; e += kTreeThreads) {
    const unsigned long long v = sees[cur][e];
    sees_out[(size_t)b * T * W + e] = make_uint2((unsigned)v, (unsigned)(v >> 32));
  }
}

#define PC_MOVE(ctrl) __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), ctrl, 0xf, 0xf, true))
// sum over the N = 16 or 8 neighbouring lanes that share a dot product
template <int N>
__device__ __forceinline__ float group_sum(float x) {
  x += PC_MOVE(0xB1);                    // lane ^ 1
  x += PC_MOVE(0x4E);                    // lane ^ 2
  x += PC_MOVE(0x141);                   // mirrored inside 8
  if (N == 16) x += PC_MOVE(0x140);      // mirrored inside 16
  return x;
}
// over the 64 / N groups: lanes l + N k
template <int N, class Op>
__device__ __forceinline__ float over_groups(float x, Op op) {
  if (N == 8) x = op(x, PC_MOVE(0x128)); // lane ^ 8 (rotated by 8 inside 16)
  return pc::dec::over_rows(x, op);
}
// x of the lower half of the lanes (rows of 16: of the even rows), y of the upper half (odd rows), each added over both
__device__ __forceinline__ float halve32(float x, float y) {
  typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
  const u32x2 a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}
__device__ __forceinline__ float halve16(float x, float y) {
  typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
  const u32x2 a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// The merge of a row's partials over the cached keys, and the nodes that the row looks at, a handful of a tree's: each of them is a dot product and
// one more weighted row, which no tile of matrix products would be worth -- and a node that a row does not look at is not read for it, whatever it
// holds.  (In a long plain sequence a row looks at half of the nodes: 4 sequences over 8 x 512 keys each, 16 heads over 8, the merge alone 26 us at
// 128 nodes, 74 at 256, 218 at 512, where percache_attention_reuse takes 44, 54 and 92 for the whole call.)  A wavefront takes one node of the tree
// and H heads of a group, which look at the same nodes: lane (sg, dv) has 8 elements of a head and takes partials sg, sg + SG, ... (NP of them at a
// time) and, 16 nodes of the row at a time, NB of them, dealt out by scalar arithmetic; the SG running (max, sum, output) meet through lane exchanges
// that leave every lane with the elements it writes.  Its time is that of two memory latencies while the rows fit the chip at once -- the first nodes
// are asked for as soon as the row's word of `sees` is there, the partials looked at behind that --, then that of the vector port, hence H. 12288
// rows of 13 nodes and 4 partials: 17.6 us with a row a wavefront, nodes dealt out lane by lane and whole sums exchanged, 13.0 now.
template <int D, int NP, int H>
__global__ __launch_bounds__(256) void draft_merge_kernel(const float *__restrict__ part_o, const float *__restrict__ part_ml, int n_splits, const __bf16 *__restrict__ Q,
                                                          const __bf16 *__restrict__ K, const __bf16 *__restrict__ V, int T, int Hq, int Hkv,
                                                          float scale_log2e, pc::DraftView draft, __bf16 *__restrict__ out) {
  constexpr int VPR = D / 8, SG = 64 / VPR, NB = 16 / SG;
  const int G = Hq / Hkv, R = G * T, groups = (G + H - 1) / H * T, blocks = (groups + 3) / 4;
  const int bg = blockIdx.x / blocks, b = bg / Hkv, g = bg - b * Hkv, lane = threadIdx.x & 63, sg = lane / VPR, dv = lane % VPR;
  const int group = (blockIdx.x - bg * blocks) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (group >= groups) return;
  const int hg = group / T * H, i = group % T, head = g * G + hg, n_heads = min(H, G - hg);

  auto word_of = [&](int w) __attribute__((always_inline)) {
    const unsigned long long x = pc::draft_row(draft, b, T, i, 64 * w);
    return ((unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32) | (unsigned)__builtin_amdgcn_readfirstlane((int)x);
  };
  struct Parts { float2 e[NP]; pc::f32x4 o[NP][2]; };
  auto load = [&](Parts &x, int h, int s0) __attribute__((always_inline)) {
    const size_t prow = (size_t)bg * R + (hg + min(h, n_heads - 1)) * T + i;
    const float2 *ml = (const float2 *)part_ml + prow * n_splits;
    const float *po = part_o + prow * n_splits * D + dv * 8;
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      const int s = s0 + SG * j, sc = min(s, n_splits - 1);
      x.e[j] = ml[sc];
      x.o[j][0] = *(const pc::f32x4 *)(po + (size_t)sc * D);
      x.o[j][1] = *(const pc::f32x4 *)(po + (size_t)sc * D + 4);
      if (s >= n_splits) x.e[j].y = 0.f;
    }
  };
  pc::bf16x8 qv[H];
  if (Q)
#pragma unroll
    for (int h = 0; h < H; ++h) qv[h] = *(const pc::bf16x8 *)(Q + (((size_t)b * Hq + head + min(h, n_heads - 1)) * T + i) * D + dv * 8);
  Parts parts[H];
  if (n_splits > 0)
#pragma unroll
    for (int h = 0; h < H; ++h) load(parts[h], h, sg);

  // nodes: the words of `sees` up to the row's own node
  unsigned long long bits = word_of(0);
  const bool live = i < 64 ? bits >> i & 1 : pc::draft_live(draft, b, T, i);
  const int n_words = live && Q ? i / 64 + 1 : 0;
  const __bf16 *kr = K + (((size_t)b * Hkv + g) * T) * D + dv * 8, *vr = V + (((size_t)b * Hkv + g) * T) * D + dv * 8;
  int word = 0;
  struct Batch { pc::bf16x8 k[NB], v[NB]; bool any, has[NB]; };
  auto next = [&](Batch &x) __attribute__((always_inline)) {   // up to 16 nodes of a word
    while (word < n_words && !bits) {
      ++word;
      if (word < n_words) bits = word_of(word);
    }
    x.any = word < n_words;
    if (!x.any) return;
    const int first = 64 * word + (int)__builtin_ctzll(bits);
    int t[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      t[j] = -1;
#pragma unroll
      for (int y = 0; y < SG; ++y) {
        const int node = bits ? 64 * word + (int)__builtin_ctzll(bits) : -1;
        bits &= bits - 1;
        t[j] = sg == y ? node : t[j];
      }
      x.has[j] = t[j] >= 0;
      t[j] = x.has[j] ? t[j] : first;
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) x.k[j] = *(const pc::bf16x8 *)(kr + (size_t)t[j] * D);
#pragma unroll
    for (int j = 0; j < NB; ++j) x.v[j] = *(const pc::bf16x8 *)(vr + (size_t)t[j] * D);
  };
  Batch batch;
  next(batch);

  struct State {
    float m = -INFINITY, l = 0.f, acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    __device__ __forceinline__ void shift_to(float top) {   // a new reference exponent, never below the old one
      const float a = m == -INFINITY ? (l == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(m - top);   // (a sum that is NaN without a maximum stays)
      m = top;
      l *= a;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] *= a;
    }
  } st[H];
  if (live)
    for (int s0 = sg; s0 - sg < n_splits; s0 += SG * NP)
#pragma unroll
      for (int h = 0; h < H; ++h) {
        if (s0 != sg) load(parts[h], h, s0);
        float top = st[h].m;
#pragma unroll
        for (int j = 0; j < NP; ++j) top = fmaxf(top, parts[h].e[j].y != 0.f ? parts[h].e[j].x : -INFINITY);
        st[h].shift_to(top);
#pragma unroll
        for (int j = 0; j < NP; ++j) {
          // (a partition without a visible key has sum 0, and zeros)
          const float w = parts[h].e[j].y == 0.f ? 0.f : parts[h].e[j].y * __builtin_amdgcn_exp2f(parts[h].e[j].x - st[h].m);
          st[h].l += w;
          // (left out where there is no partition: what was read in its place need not be finite)
          if (parts[h].e[j].y != 0.f)
#pragma unroll
            for (int x = 0; x < 8; ++x) st[h].acc[x] += w * parts[h].o[j][x >> 2][x & 3];
        }
      }
  while (batch.any) {
    // (places that no node fills hold the first one's V, which need not be finite)
#pragma unroll
    for (int j = 0; j < NB; ++j)
      if (!batch.has[j]) batch.v[j] = pc::bf16x8{};
#pragma unroll
    for (int h = 0; h < H; ++h) {
      typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
      float s[NB], top = st[h].m;
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        float d = 0.f;
#pragma unroll
        for (int x = 0; x < 8; x += 2) d = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{qv[h][x], qv[h][x + 1]}, bf16x2{batch.k[j][x], batch.k[j][x + 1]}, d, false);
        d = group_sum<VPR>(d) * scale_log2e;
        s[j] = batch.has[j] ? d : -INFINITY;
        top = fmaxf(top, s[j]);
      }
      st[h].shift_to(top);
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const float w = s[j] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s[j] - st[h].m);
        st[h].l += w;
#pragma unroll
        for (int x = 0; x < 8; ++x) st[h].acc[x] += w * (float)batch.v[j][x];
      }
    }
    next(batch);
  }
#pragma unroll
  for (int h = 0; h < H; ++h) {
    State &z = st[h];
    const float top = over_groups<VPR>(z.m, [](float x, float y) { return fmaxf(x, y); });
    const float a = z.l == 0.f ? 0.f : z.m == top ? 1.f : __builtin_amdgcn_exp2f(z.m - top);
    const float l = over_groups<VPR>(z.l * a, [](float x, float y) { return x + y; }), scale = l == 0.f ? 0.f : a / l;
    // elements 8 dv .. +7 over the groups: halves of them go to halves of the lanes, until a lane has elements 8 dv + at .. of its own
    float x4[4], x2[2];
#pragma unroll
    for (int e = 0; e < 4; ++e) x4[e] = halve32(z.acc[e] * scale, z.acc[e + 4] * scale);
#pragma unroll
    for (int e = 0; e < 2; ++e) x2[e] = halve16(x4[e], x4[e + 2]);
    const int at = 4 * (lane >> 5) + 2 * (lane >> 4 & 1);
    if constexpr (SG == 8) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float x = x2[e];
        x2[e] = x + PC_MOVE(0x128);
      }
    }
    if (h >= n_heads) continue;
    if (draft.lse && lane == 0) draft.lse[((size_t)b * Hq + head + h) * T + i] = pc::lse_of(top, l);
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    if (SG == 4 || (lane & 8) == 0)
      *(bf16x2 *)(out + ((size_t)b * T + i) * ((size_t)Hq * D) + (size_t)(head + h) * D + dv * 8 + at) = bf16x2{(__bf16)x2[0], (__bf16)x2[1]};
  }
}
#undef PC_MOVE

bool aligned16(const void *p) { return (uintptr_t)p % 16 == 0; }

// depth of every node (0: a root; padding counts as one), -1 where there are no parents to take it from
int depth_of(const int32_t *parents, int i, const std::vector<int> &depth) { return parents ? (parents[i] < 0 ? 0 : depth[parents[i]] + 1) : i; }

}  // namespace

namespace pc {

pc_status check_trees(percache_ctx *ctx, int32_t batch, int32_t t_draft, const int32_t *parents) {
  if (!parents) return PC_OK;
  if (t_draft > kMaxNodes) return fail(ctx, PC_ESHAPE, "a tree has %d nodes, at most %d are supported", t_draft, kMaxNodes);
  for (int b = 0; b < batch; ++b) {
    const int32_t *p = parents + (size_t)b * t_draft;
    for (int i = 0; i < t_draft; ++i) {
      if (p[i] < -2 || p[i] >= i) return fail(ctx, PC_EINVAL, "query %d node %d: parent %d outside [-2,%d)", b, i, p[i], i);
      if (p[i] >= 0 && p[p[i]] == -2) return fail(ctx, PC_EINVAL, "query %d node %d: its parent %d is padding", b, i, p[i]);
    }
  }
  return PC_OK;
}

pc_status check_paths(percache_ctx *ctx, int32_t batch, int32_t t_draft, const int32_t *path, const int32_t *n_path, int32_t max_path) {
  if (!n_path) return fail(ctx, PC_EINVAL, "n_path_host is NULL");
  if (max_path < 1 || max_path > t_draft) return fail(ctx, PC_EINVAL, "max_path %d outside [1,%d]", max_path, t_draft);
  for (int b = 0; b < batch; ++b) {
    if (n_path[b] < 0 || n_path[b] > max_path) return fail(ctx, PC_EINVAL, "n_path[%d]=%d outside [0,%d]", b, n_path[b], max_path);
    for (int j = 0; j < n_path[b]; ++j) {
      const int i = path[(size_t)b * max_path + j];
      if (i < 0 || i >= t_draft) return fail(ctx, PC_EINVAL, "query %d: node %d of its path outside [0,%d)", b, i, t_draft);
    }
  }
  return PC_OK;
}

DraftWs carve_draft_ws(const percache_config &c, int n_cu, void *base, int32_t batch, int32_t t_draft, int32_t max_chunks) {
  DraftWs w;
  char *p = (char *)base;
  size_t off = 0;
  auto take = [&](size_t bytes) { char *r = p ? p + off : nullptr; off += align_up(bytes); return r; };
  const size_t B = batch, T = t_draft, ft = (T + kKvTile - 1) / kKvTile, rows = B * c.n_q_heads * T, nc = max_chunks;
  // attention: chunk table, packed parents; projection: positions; weights: entries, users, splits (14 words a chunk and query at most), paths (of at
  // most t_draft nodes), packed parents
  w.words = (int32_t *)take((B * (14 * (nc + 1) + 3 * T + 8) + 16) * sizeof(int32_t));
  w.sees = (uint2 *)take(t_draft <= kMaxNodes ? B * T * ft * sizeof(uint2) : 0);
  const size_t cap = max_splits_for(c, n_cu, batch, t_draft);
  w.part_o = (float *)take(rows * cap * c.head_dim * sizeof(float));
  w.part_ml = (float *)take(rows * cap * 2 * sizeof(float));
  w.total = off;
  return w;
}

pc_status upload_draft(percache_ctx *ctx, std::vector<int32_t> &words, int batch, int t_draft, const int32_t *parents, const DraftWs &ws, hipStream_t stream) {
  const int n = (int)words.size();
  int rounds = 0;
  if (parents) {
    int longest = 1;
    std::vector<int> depth(t_draft);
    words.resize(n + ((size_t)batch * t_draft + 1) / 2, 0);
    for (int b = 0; b < batch; ++b)
      for (int i = 0; i < t_draft; ++i) {
        const size_t at = (size_t)b * t_draft + i;
        words[n + at / 2] |= (int32_t)((uint32_t)(uint16_t)parents[at] << (at & 1 ? 16 : 0));
        depth[i] = depth_of(parents + (size_t)b * t_draft, i, depth);
        if (depth[i] + 1 > longest) longest = depth[i] + 1;
      }
    while ((1 << rounds) < longest) ++rounds;
  }
  ListWords lists;
  uint2 *sees = parents ? ws.sees : nullptr;
  if (words.size() <= (size_t)kListWords) {
    for (size_t i = 0; i < words.size(); ++i) lists.v[i] = words[i];
    hipLaunchKernelGGL(draft_lists_kernel<true>, dim3(sees ? batch + 1 : 1), dim3(kTreeThreads), 0, stream, ws.words, n, lists, nullptr, batch, t_draft, rounds, sees);
  } else {
    const pc_status st = upload_table(ctx, words, ws.words, stream);
    if (st != PC_OK) return st;
    if (!sees) return PC_OK;
    hipLaunchKernelGGL(draft_lists_kernel<false>, dim3(batch), dim3(kTreeThreads), 0, stream, ws.words, n, lists, ws.words + n, batch, t_draft, rounds, sees);
  }
  PC_HIP(ctx, hipGetLastError());
  return PC_OK;
}

pc_status launch_draft_merge(percache_ctx *ctx, const float *part_o, const float *part_ml, int n_splits, const __bf16 *q, const __bf16 *k, const __bf16 *v, int batch, int T,
                             const DraftView &draft, __bf16 *out, hipStream_t stream) {
  const percache_config &c = ctx->cfg;
  const int G = c.n_q_heads / c.n_kv_heads;
  const float scale_log2e = 1.4426950408889634f / sqrtf((float)c.head_dim);
  // Heads of a group together once the rows by themselves, a wavefront each, would be more than the chip holds at once (about 20 a CU).
  const int per = c.head_dim == 128 ? 4 : 8;
  const bool together = n_splits <= per && (long)batch * c.n_q_heads * T > 20L * ctx->n_cu;
  const int H = !together || G == 1 ? 1 : G == 2 ? 2 : G % 3 == 0 ? 3 : G % 4 == 0 || G > 4 ? 4 : 2;
  const long blocks = ((long)((G + H - 1) / H) * T + 3) / 4;
  const dim3 grid((unsigned)(blocks * batch * c.n_kv_heads));
#define PC_MERGE(DD, NN, HH) \
  hipLaunchKernelGGL((draft_merge_kernel<DD, NN, HH>), grid, dim3(256), 0, stream, part_o, part_ml, n_splits, q, k, v, T, c.n_q_heads, c.n_kv_heads, scale_log2e, draft, out)
#define PC_MERGE_D(DD)                                                                                          \
  do {                                                                                                          \
    if (n_splits > per) PC_MERGE(DD, 4, 1);                                                                     \
    else if (H == 1) PC_MERGE(DD, 1, 1);                                                                        \
    else if (H == 2) PC_MERGE(DD, 1, 2);                                                                        \
    else if (H == 3) PC_MERGE(DD, 1, 3);                                                                        \
    else PC_MERGE(DD, 1, 4);                                                                                    \
  } while (0)
  if (c.head_dim == 128) PC_MERGE_D(128); else PC_MERGE_D(64);
#undef PC_MERGE_D
#undef PC_MERGE
  PC_HIP(ctx, hipGetLastError());
  return PC_OK;
}

}  // namespace pc

extern "C" {

size_t percache_draft_workspace_bytes(const percache_ctx *ctx, int32_t batch, int32_t t_draft, int32_t max_chunks) {
  if (!ctx || batch < 1 || t_draft < 1 || max_chunks < 0) return 0;
  return pc::carve_draft_ws(ctx->cfg, ctx->n_cu, nullptr, batch, t_draft, max_chunks).total;
}

pc_status percache_qkv_rope_draft(percache_ctx *ctx, const void *x_dev, const void *wqkv_dev, int32_t batch, int32_t t_draft,
                                  const int32_t *parents_host, const int32_t *pos0_host, void *q_out_dev, void *k_out_dev, void *v_out_dev,
                                  void *workspace_dev, size_t workspace_bytes, void *stream) {
  if (!ctx) return PC_EINVAL;
  const percache_config &c = ctx->cfg;
  if (!x_dev || !wqkv_dev || !q_out_dev || !k_out_dev || !v_out_dev) return pc::fail(ctx, PC_EINVAL, "NULL tensor pointer");
  if (!aligned16(x_dev) || !aligned16(wqkv_dev) || !aligned16(q_out_dev) || !aligned16(k_out_dev) || !aligned16(v_out_dev))
    return pc::fail(ctx, PC_EINVAL, "tensor pointers must be 16-byte aligned");
  if (batch < 1 || t_draft < 1) return pc::fail(ctx, PC_EINVAL, "batch and t_draft must be positive");
  if (!pos0_host) return pc::fail(ctx, PC_EINVAL, "pos0_host is NULL");
  pc_status st = pc::check_trees(ctx, batch, t_draft, parents_host);
  if (st != PC_OK) return st;
  const long F = (long)(c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim, M = (long)batch * t_draft;
  if (F * c.hidden >= (1L << 31) || M * c.hidden >= (1L << 31) || M * F >= (1L << 31)) return pc::fail(ctx, PC_ESHAPE, "operand larger than 2^31 elements");
  const size_t need = percache_draft_workspace_bytes(ctx, batch, t_draft, 0);
  if (!workspace_dev || workspace_bytes < need) return pc::fail(ctx, PC_ENOMEM, "draft workspace has %zu bytes, need %zu", workspace_bytes, need);
  if ((uintptr_t)workspace_dev % pc::kAlign) return pc::fail(ctx, PC_EINVAL, "workspace must be 256-byte aligned");
  // per query a word that the kernels skip, then every node's position less its index
  std::vector<int32_t> words((size_t)batch * (t_draft + 1));
  std::vector<int> depth(t_draft);
  for (int b = 0; b < batch; ++b) {
    int deepest = 0;
    for (int i = 0; i < t_draft; ++i) {
      depth[i] = depth_of(parents_host ? parents_host + (size_t)b * t_draft : nullptr, i, depth);
      if (depth[i] > deepest) deepest = depth[i];
      words[(size_t)b * (t_draft + 1) + 1 + i] = pos0_host[b] + depth[i] - i;
    }
    if (pos0_host[b] < 0 || (long)pos0_host[b] + deepest >= c.max_pos)
      return pc::fail(ctx, PC_ELEN, "query %d: positions %d to %ld outside [0,%d)", b, pos0_host[b], (long)pos0_host[b] + deepest, c.max_pos);
  }
  const pc::DraftWs ws = pc::carve_draft_ws(c, ctx->n_cu, workspace_dev, batch, t_draft, 0);
  hipStream_t s = (hipStream_t)stream;
  st = pc::upload_table(ctx, words, ws.words, s);
  if (st != PC_OK) return st;
  return pc::launch_qkv_rope(ctx, (const __bf16 *)x_dev, (const __bf16 *)wqkv_dev, batch, t_draft, ws.words, t_draft + 1, (__bf16 *)q_out_dev,
                             (__bf16 *)k_out_dev, (__bf16 *)v_out_dev, s, pc::QkvExtras(), nullptr, nullptr, nullptr, 1);
}

pc_status percache_attention_draft(percache_ctx *ctx, int32_t layer, const void *q_dev, const void *k_draft_dev, const void *v_draft_dev, int32_t batch,
                                   int32_t t_draft, const int32_t *slot_ids_host, const int32_t *used_len_host, const int32_t *n_chunks_host,
                                   int32_t max_chunks, const int32_t *parents_host, int32_t n_splits, void *attn_out_dev, float *lse_out_dev,
                                   void *workspace_dev, size_t workspace_bytes, void *stream) {
  if (!ctx) return PC_EINVAL;
  const percache_config &c = ctx->cfg;
  if (!q_dev || !k_draft_dev || !v_draft_dev || !attn_out_dev) return pc::fail(ctx, PC_EINVAL, "NULL tensor pointer");
  if (!aligned16(q_dev) || !aligned16(k_draft_dev) || !aligned16(v_draft_dev) || !aligned16(attn_out_dev))
    return pc::fail(ctx, PC_EINVAL, "tensor pointers must be 16-byte aligned");
  if ((uintptr_t)lse_out_dev % sizeof(float)) return pc::fail(ctx, PC_EINVAL, "lse_out_dev must be 4-byte aligned");
  if (batch < 1 || t_draft < 1) return pc::fail(ctx, PC_EINVAL, "batch and t_draft must be positive");
  const int cap = pc::max_splits_for(c, ctx->n_cu, batch, t_draft);
  if (n_splits < 0 || n_splits > cap) return pc::fail(ctx, PC_EINVAL, "n_splits %d outside [0,%d] for this shape", n_splits, cap);
  pc_status st = pc::check_trees(ctx, batch, t_draft, parents_host);
  if (st != PC_OK) return st;
  if ((long)batch * t_draft * (c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim >= (1L << 31)) return pc::fail(ctx, PC_ESHAPE, "operand larger than 2^31 elements");
  std::vector<int32_t> words;
  st = pc::build_chunk_table(ctx, layer, batch, 1, slot_ids_host, used_len_host, n_chunks_host, max_chunks, words);
  if (st != PC_OK) return st;
  const size_t need = percache_draft_workspace_bytes(ctx, batch, t_draft, max_chunks);
  if (!workspace_dev || workspace_bytes < need) return pc::fail(ctx, PC_ENOMEM, "draft workspace has %zu bytes, need %zu", workspace_bytes, need);
  if ((uintptr_t)workspace_dev % pc::kAlign) return pc::fail(ctx, PC_EINVAL, "workspace must be 256-byte aligned");
  const pc::DraftWs ws = pc::carve_draft_ws(c, ctx->n_cu, workspace_dev, batch, t_draft, max_chunks);
  const int stride = pc::tbl_stride(max_chunks), formats = pc::table_formats(words, stride, batch);
  long tiles = 0;
  for (int b = 0; b < batch; ++b) tiles += words[(size_t)b * stride + 2];
  const int mean_tiles = (int)((tiles + batch - 1) / batch);
  hipStream_t s = (hipStream_t)stream;
  st = pc::upload_draft(ctx, words, batch, t_draft, parents_host, ws, s);
  if (st != PC_OK) return st;
  pc::DraftView draft;
  draft.sees = parents_host ? ws.sees : nullptr;
  draft.lse = lse_out_dev;
  const __bf16 *q = (const __bf16 *)q_dev, *k = (const __bf16 *)k_draft_dev, *v = (const __bf16 *)v_draft_dev;
  __bf16 *out = (__bf16 *)attn_out_dev;
  const bool few = pc::decode_rows(c, t_draft);   // (the decode kernel takes the nodes along as its fresh keys)
  if (!few && mean_tiles == 0) return pc::launch_draft_merge(ctx, nullptr, nullptr, 0, q, k, v, batch, t_draft, draft, out, s);   // (nothing cached)
  pc::prof_begin(ctx, PC_KERNEL_ATTENTION, s);
  st = few ? pc::launch_decode_attention(ctx, layer, q, k, v, nullptr, batch, t_draft, ws.words, stride, mean_tiles, n_splits, 0, out, ws.part_o, ws.part_ml, s, formats, &draft)
           : pc::launch_draft_attention(ctx, layer, q, batch, t_draft, ws.words, stride, mean_tiles, n_splits, ws.part_o, ws.part_ml, s, formats);
  if (st != PC_OK) return st;
  pc::prof_end(ctx, PC_KERNEL_ATTENTION, s);
  if (few && n_splits == 1) return PC_OK;
  return pc::launch_draft_merge(ctx, ws.part_o, ws.part_ml, n_splits, few ? nullptr : q, k, v, batch, t_draft, draft, out, s);
}

}  // extern "C"
