// Verification of drafted tokens: each query brings a tree of t_draft nodes (a node behind its parent), all of them run through a layer at
// once.  Node i sits at position pos0 + depth(i) and attends over [cached chunks ; its ancestors ; itself],
//   o_i = sum_j e^(s_ij - lse_i) v_j,   s_ij = q_i.k_j / sqrt(D),   lse_i = log sum_j e^s_ij.
// The projection and the attention are the kernels of qkv_rope_gemm.hip, reuse_attention.hip and decode_attention.hip; here are the host
// entry points and the lists they take: positions of the nodes, and for the attention one word of 64 bits per node and 64 nodes that
// says which of them it looks at.
#include "percache_internal.hpp"

namespace {

// One workgroup a query: ancestors by pointer doubling, sees[i] |= sees[up[i]], up[i] = up[up[i]], in log2(longest path) rounds between two
// LDS buffers.  The parents come packed, two to a word, as a launch argument (FROM_ARG; with the words in front of them, which workgroup
// `batch` then copies) or from device memory.  16 bits of parents a node travel instead of 64 bits or more of `sees`: 8 queries of 64
// nodes with their chunk list still fit a launch's arguments.
constexpr int kTreeThreads = 256;
template <bool FROM_ARG>
__global__ __launch_bounds__(kTreeThreads) void draft_lists_kernel(int32_t *dst, int n_words, const pc::ListWords lists, const int32_t *packed, int batch, int T,
                                                                   int rounds, uint2 *sees_out) {
  const int b = blockIdx.x, tid = threadIdx.x;
  if (b == (sees_out ? batch : 0)) {
    if constexpr (FROM_ARG)
      for (int i = tid; i < n_words; i += kTreeThreads) dst[i] = lists.v[i];
    return;
  }
  constexpr int N = pc::kMaxNodes;
  __shared__ unsigned long long sees[2][N * (N / 64)];
  __shared__ int up[2][N];
  const int W = (T + 63) / 64;
  for (int i = tid; i < T; i += kTreeThreads) {
    const int at = b * T + i, w = FROM_ARG ? lists.v[n_words + at / 2] : packed[at / 2];
    const int p = (int16_t)(at & 1 ? w >> 16 : w & 0xffff);
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

// over the lanes of a group of 16 (8) neighbours
template <int N>
__device__ __forceinline__ float group_sum(float x) {
#define PC_MOVE(ctrl) __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), ctrl, 0xf, 0xf, true))
  x += PC_MOVE(0xB1);                    // lane ^ 1
  x += PC_MOVE(0x4E);                    // lane ^ 2
  x += PC_MOVE(0x141);                   // mirrored inside 8
  if (N == 16) x += PC_MOVE(0x140);      // mirrored inside 16
#undef PC_MOVE
  return x;
}

// The merge of a row's partials over the cached keys, and the nodes that the row looks at, a handful of a tree's: each of them is a dot product and
// one more weighted row, which no tile of matrix products would be worth -- and a node that a row does not look at is not read for it,
// whatever it holds.  A row is shared by 4 x D/8 lanes: lane (sg, dv) has 8 elements of the head and takes partials sg, sg + 4, ... and the
// nodes j = sg (mod 4), four at a time with all their loads in flight; the four running (max, sum, output) meet through lane shuffles.
template <int D>
__global__ __launch_bounds__(256) void draft_merge_kernel(const float *__restrict__ part_o, const float *__restrict__ part_ml, int n_splits, const __bf16 *__restrict__ Q,
                                                          const __bf16 *__restrict__ K, const __bf16 *__restrict__ V, int T, int Hq, int Hkv, long total_rows,
                                                          float scale_log2e, pc::DraftView draft, __bf16 *__restrict__ out) {
  constexpr int VPR = D / 8, LPR = 4 * VPR;
  const long gid = (long)blockIdx.x * 256 + threadIdx.x, prow = gid / LPR;
  if (prow >= total_rows) return;   // (LPR divides the 64 lanes: a row's lanes stay together)
  const int r = (int)(gid - prow * LPR), sg = r / VPR, dv = r - sg * VPR;
  const int G = Hq / Hkv, R = G * T;
  const long bg = prow / R;
  const int row = (int)(prow - bg * R), b = (int)(bg / Hkv), g = (int)(bg - (long)b * Hkv), hg = row / T, i = row - hg * T, head = g * G + hg;
  const bool live = pc::draft_live(draft, b, T, i);
  float m = -INFINITY, l = 0.f, acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  auto shift_to = [&](float top) __attribute__((always_inline)) {   // a new reference exponent, never below the old one
    const float a = m == -INFINITY ? (l == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(m - top);   // (a sum that is NaN without a maximum stays)
    m = top;
    l *= a;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] *= a;
  };
  if (live) {
    const float2 *ml = (const float2 *)part_ml + prow * n_splits;
    const float *po = part_o + prow * n_splits * D + dv * 8;
    for (int s0 = sg; s0 < n_splits; s0 += 16) {
      float2 e[4];
      pc::f32x4 o[4][2];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int s = s0 + 4 * j, sc = s < n_splits ? s : s0;
        e[j] = ml[sc];
        o[j][0] = *(const pc::f32x4 *)(po + (size_t)sc * D);
        o[j][1] = *(const pc::f32x4 *)(po + (size_t)sc * D + 4);
        if (s >= n_splits) e[j].y = 0.f;
      }
      float top = m;
#pragma unroll
      for (int j = 0; j < 4; ++j) top = fmaxf(top, e[j].y != 0.f ? e[j].x : -INFINITY);
      shift_to(top);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (e[j].y == 0.f) continue;   // (no key of the partition is visible)
        const float w = e[j].y * __builtin_amdgcn_exp2f(e[j].x - m);
        l += w;
#pragma unroll
        for (int x = 0; x < 8; ++x) acc[x] += w * o[j][x >> 2][x & 3];
      }
    }
    if (Q) {
      const pc::bf16x8 qv = *(const pc::bf16x8 *)(Q + (((size_t)b * Hq + head) * T + i) * D + dv * 8);
      const __bf16 *kr = K + ((size_t)b * Hkv + g) * T * D + dv * 8, *vr = V + ((size_t)b * Hkv + g) * T * D + dv * 8;
      for (int t0 = 0; t0 <= i; t0 += 64) {
        unsigned long long bits = pc::draft_row(draft, b, T, i, t0) & (0x1111111111111111ull << sg);
        while (bits) {
          int n = 0, t[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            t[j] = bits ? t0 + (int)__builtin_ctzll(bits) : t[0];
            n += bits != 0;
            bits &= bits - 1;
          }
          pc::bf16x8 kv[4], vv[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            kv[j] = *(const pc::bf16x8 *)(kr + (size_t)t[j] * D);
            vv[j] = *(const pc::bf16x8 *)(vr + (size_t)t[j] * D);
          }
          float s[4], top = m;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float d = 0.f;
#pragma unroll
            for (int x = 0; x < 8; ++x) d += (float)qv[x] * (float)kv[j][x];
            s[j] = group_sum<VPR>(d) * scale_log2e;
            if (j < n) top = fmaxf(top, s[j]);
          }
          shift_to(top);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (j >= n) continue;
            const float w = s[j] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s[j] - m);
            l += w;
#pragma unroll
            for (int x = 0; x < 8; ++x) acc[x] += w * (float)vv[j][x];
          }
        }
      }
    }
  }
#pragma unroll
  for (int sh = VPR; sh < LPR; sh <<= 1) {
    const float m_other = __shfl_xor(m, sh, 64), l_other = __shfl_xor(l, sh, 64), top = fmaxf(m, m_other);
    const float a = l == 0.f ? 0.f : m == top ? 1.f : __builtin_amdgcn_exp2f(m - top);
    const float c = l_other == 0.f ? 0.f : m_other == top ? 1.f : __builtin_amdgcn_exp2f(m_other - top);
    m = top;
    l = l * a + l_other * c;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = acc[e] * a + __shfl_xor(acc[e], sh, 64) * c;
  }
  if (sg != 0) return;
  if (draft.lse && dv == 0) draft.lse[((size_t)b * Hq + head) * T + i] = pc::lse_of(m, l);
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  pc::bf16x8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (__bf16)(acc[e] * inv);
  *(pc::bf16x8 *)(out + ((size_t)b * T + i) * ((size_t)Hq * D) + (size_t)head * D + dv * 8) = v;
}

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
  // attention: chunk table, packed parents; projection: positions; weights: entries, users, paths (of at most t_draft nodes), packed parents
  w.words = (int32_t *)take((B * (8 * (nc + 1) + 3 * T + 8) + 16) * sizeof(int32_t));
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
  const long rows = (long)batch * c.n_q_heads * T;
  const dim3 grid((unsigned)((rows * (c.head_dim / 2) + 255) / 256));
  const float scale_log2e = 1.4426950408889634f / sqrtf((float)c.head_dim);
  if (c.head_dim == 128) hipLaunchKernelGGL(draft_merge_kernel<128>, grid, dim3(256), 0, stream, part_o, part_ml, n_splits, q, k, v, T, c.n_q_heads, c.n_kv_heads, rows, scale_log2e, draft, out);
  else hipLaunchKernelGGL(draft_merge_kernel<64>, grid, dim3(256), 0, stream, part_o, part_ml, n_splits, q, k, v, T, c.n_q_heads, c.n_kv_heads, rows, scale_log2e, draft, out);
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
  return pc::launch_attention(ctx, layer, (const __bf16 *)q_dev, (const __bf16 *)k_draft_dev, (const __bf16 *)v_draft_dev, nullptr, nullptr, batch, t_draft,
                              ws.words, stride, mean_tiles, n_splits, (__bf16 *)attn_out_dev, ws.part_o, ws.part_ml, s, formats, nullptr, &draft);
}

}  // extern "C"
