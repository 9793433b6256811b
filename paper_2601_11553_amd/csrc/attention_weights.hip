// What a layer's query rows pay to every key: w_t = sum over rows of e^(q.k_t / sqrt(D) - lse), from the rows' log-sum-exp that the attention
// handed out.  With it the softmax needs no second pass, so a key's weight is one product and one exponential a row, and the keys are read once.
//
// The keys stay, the rows pass by: a wavefront holds 64 keys of one (slot, kv head) as matrix operands in registers and goes over the rows of
// every query that uses the slot, 32 at a time.  So a slot shared by several queries (a system prompt's chunk) is read once, its sums have one
// owner and one order -- no atomics, no second launch -- and are added to the running sums in place.
#include "decode_common.hpp"

namespace {
using pc::bf16x8;
using pc::f32x16;
using pc::kKvTile;
using pc::dec::codes8;
using pc::dec::fast_exp2;

// Lists of a call (int32 words): n_entries + 1 entries, then the users, then -- with paths -- their n_path [batch] and nodes [batch][max_path].
struct Entry {
  int32_t slot;     // slot id; -1 - b: the draft keys of query b
  int32_t tile0;    // first of its 64-key tiles among all entries'
  int32_t user0;    // first of its users (up to the next entry's)
  int32_t longest;  // keys: the longest used length among its users
};
struct User {
  int32_t query, used;
};

struct Args {
  const __bf16 *q, *k_draft;
  const float *lse;
  const __bf16 *k16;
  const uint8_t *k8;
  const float *k_scale;
  int n_slots16;
  const Entry *entries;
  int n_entries;
  const User *users;
  const int32_t *n_path, *path;  // null: every row counts
  int max_path;
  int T, Hq, Hkv, C;
  float scale_log2e;
  const float *w_in;   // [slots][Hkv][C], may be null (zero) and may be w_out
  float *w_out, *w_draft;
  pc::DraftView draft;
};

template <int D, int FMT>
__global__ __launch_bounds__(64) void attention_weights_kernel(const Args a) {
  constexpr int KS = D / 16;
  const int lane = threadIdx.x, l32 = lane & 31, g2 = lane >> 5;
  const int g = blockIdx.x % a.Hkv, tile = blockIdx.x / a.Hkv, G = a.Hq / a.Hkv, T = a.T;

  // the entry this tile belongs to: the last one that starts at or before it
  int n_before = 0;
  for (int e0 = 0; e0 < a.n_entries; e0 += 64) {
    const bool before = e0 + lane < a.n_entries && a.entries[e0 + lane].tile0 <= tile;
    const int n = __popcll(__ballot(before));
    n_before += n;
    if (n < 64) break;
  }
  const int ei = __builtin_amdgcn_readfirstlane(n_before) - 1;
  const Entry ent = a.entries[ei];
  const int user_end = a.entries[ei + 1].user0, t0 = (tile - ent.tile0) * kKvTile, valid = min(kKvTile, ent.longest - t0);
  const bool is_draft = ent.slot < 0;

  // keys: lane (l32, g2) holds elements 16 ks + 8 g2 .. +7 of key 32 kb + l32 (past a ragged end: the last key's)
  bf16x8 k[2][KS];
  if (is_draft || FMT == 0 || (FMT == 2 && ent.slot < a.n_slots16)) {
    const __bf16 *base = is_draft ? a.k_draft + ((size_t)(-1 - ent.slot) * a.Hkv + g) * T * D : a.k16 + ((size_t)ent.slot * a.Hkv + g) * a.C * D;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const __bf16 *row = base + (size_t)(t0 + min(kb * 32 + l32, valid - 1)) * D + g2 * 8;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) k[kb][ks] = *(const bf16x8 *)(row + ks * 16);
    }
  } else {
    const size_t head = (size_t)(ent.slot - a.n_slots16) * a.Hkv + g;
    const float scale = a.k_scale[head * (a.C / kKvTile) + t0 / kKvTile];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const uint8_t *row = a.k8 + (head * a.C + t0 + min(kb * 32 + l32, valid - 1)) * D + g2 * 8;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) k[kb][ks] = codes8(*(const uint2 *)(row + ks * 16), scale);
    }
  }

  float acc[2][16];
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[kb][r] = 0.f;
  for (int u = ent.user0; u < user_end; ++u) {
    const User user = a.users[u];
    const int b = user.query, left = user.used - t0, n_rows = a.n_path ? a.n_path[b] : T, R = G * n_rows;
    if (left <= 0) continue;
    for (int r0 = 0; r0 < R; r0 += 32) {
      const int row = min(r0 + l32, R - 1), h = row / n_rows, j = row - h * n_rows, i = a.n_path ? a.path[(size_t)b * a.max_path + j] : j;
      const size_t at = ((size_t)b * a.Hq + g * G + h) * T + i;
      const __bf16 *q = a.q + at * D + g2 * 8;
      const float lse = a.lse[at];
      const bool counts = r0 + l32 < R && lse != -INFINITY;
      f32x16 s[2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int x = 0; x < 16; ++x) s[kb][x] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bf16x8 qv = *(const bf16x8 *)(q + ks * 16);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[kb][ks], qv, s[kb], 0, 0, 0);
      }
      const float neg = lse * -1.4426950408889634f;
      const unsigned long long end = left >= kKvTile ? ~0ull : (1ull << left) - 1;
      const unsigned long long sees = !counts ? 0ull : is_draft ? pc::draft_row(a.draft, b, T, i, t0) & end : end;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const int t = kb * 32 + (x >> 2) * 8 + g2 * 4 + (x & 3);
          const float p = fast_exp2(__builtin_fmaf(s[kb][x], a.scale_log2e, neg));
          acc[kb][x] += sees >> t & 1 ? p : 0.f;
        }
    }
  }

  // sums over the 32 lanes of a half: every exchange halves the values a lane keeps; lane l32 ends with value l32 = 16 kb + x
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int v = 0; v < o; ++v) {
      float *flat = &acc[0][0];
      const bool up = l32 & o;
      const float keep = up ? flat[v + o] : flat[v], give = up ? flat[v] : flat[v + o];
      flat[v] = keep + __shfl_xor(give, o, 64);
    }
  const int x = l32 & 15, t = t0 + (l32 >> 4) * 32 + (x >> 2) * 8 + g2 * 4 + (x & 3);
  if (t >= ent.longest) return;
  if (is_draft) {
    a.w_draft[((size_t)(-1 - ent.slot) * a.Hkv + g) * T + t] = acc[0][0];
  } else {
    const size_t at = ((size_t)ent.slot * a.Hkv + g) * a.C + t;
    a.w_out[at] = (a.w_in ? a.w_in[at] : 0.f) + acc[0][0];
  }
}

}  // namespace

extern "C" pc_status percache_attention_weights(percache_ctx *ctx, int32_t layer, const void *q_dev, const void *k_draft_dev, const float *lse_dev,
                                                int32_t batch, int32_t t_draft, const int32_t *slot_ids_host, const int32_t *used_len_host,
                                                const int32_t *n_chunks_host, int32_t max_chunks, const int32_t *parents_host, const int32_t *path_host,
                                                const int32_t *n_path_host, int32_t max_path, const float *weights_in_dev, float *weights_out_dev,
                                                float *draft_weights_out_dev, void *workspace_dev, size_t workspace_bytes, void *stream) {
  if (!ctx) return PC_EINVAL;
  const percache_config &c = ctx->cfg;
  if (!q_dev || !lse_dev || !weights_out_dev || (draft_weights_out_dev && !k_draft_dev)) return pc::fail(ctx, PC_EINVAL, "NULL tensor pointer");
  if (((uintptr_t)q_dev | (uintptr_t)k_draft_dev) % 16) return pc::fail(ctx, PC_EINVAL, "q_dev and k_draft_dev must be 16-byte aligned");
  if (((uintptr_t)lse_dev | (uintptr_t)weights_in_dev | (uintptr_t)weights_out_dev | (uintptr_t)draft_weights_out_dev) % sizeof(float))
    return pc::fail(ctx, PC_EINVAL, "lse and weights must be 4-byte aligned");
  if (batch < 1 || t_draft < 1) return pc::fail(ctx, PC_EINVAL, "batch and t_draft must be positive");
  pc_status st = pc::check_trees(ctx, batch, t_draft, parents_host);
  if (st != PC_OK) return st;
  if (path_host) {
    st = pc::check_paths(ctx, batch, t_draft, path_host, n_path_host, max_path);
    if (st != PC_OK) return st;
  }
  if ((long)batch * t_draft * (c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim >= (1L << 31)) return pc::fail(ctx, PC_ESHAPE, "operand larger than 2^31 elements");
  std::vector<int32_t> rows;
  st = pc::build_chunk_table(ctx, layer, batch, 1, slot_ids_host, used_len_host, n_chunks_host, max_chunks, rows);
  if (st != PC_OK) return st;
  const size_t need = percache_draft_workspace_bytes(ctx, batch, t_draft, max_chunks);
  if (!workspace_dev || workspace_bytes < need) return pc::fail(ctx, PC_ENOMEM, "draft workspace has %zu bytes, need %zu", workspace_bytes, need);
  if ((uintptr_t)workspace_dev % pc::kAlign) return pc::fail(ctx, PC_EINVAL, "workspace must be 256-byte aligned");

  // The slots in the order of their first mention, each with its users in the order of the batch (a query that names a slot twice: two users)
  const int stride = pc::tbl_stride(max_chunks);
  auto alive = [&](int b) { return !path_host || n_path_host[b] > 0; };
  std::vector<Entry> entries;
  std::vector<std::vector<User>> users;
  std::unordered_map<int32_t, int> of_slot;
  for (int b = 0; b < batch; ++b) {
    const int32_t *row = rows.data() + (size_t)b * stride;
    for (int ci = 0; ci < row[0]; ++ci) {
      const int slot = row[pc::kTblHeader + 2 * ci], used = row[pc::kTblHeader + 2 * ci + 1];
      if (used == 0) continue;
      const auto at = of_slot.emplace(slot, (int)entries.size());
      if (at.second) {
        entries.push_back({slot, 0, 0, 0});
        users.emplace_back();
      }
      Entry &e = entries[at.first->second];
      if (used > e.longest) e.longest = used;
      if (alive(b)) users[at.first->second].push_back({b, used});
    }
  }
  if (draft_weights_out_dev)
    for (int b = 0; b < batch; ++b) {
      entries.push_back({-1 - b, 0, 0, t_draft});
      users.emplace_back();
      if (alive(b)) users.back().push_back({b, t_draft});
    }
  if (entries.empty()) return PC_OK;
  std::vector<int32_t> words;
  int tiles = 0, n_users = 0;
  for (size_t e = 0; e <= entries.size(); ++e) {
    const bool last = e == entries.size();
    const int32_t w[4] = {last ? 0 : entries[e].slot, tiles, n_users, last ? 0 : entries[e].longest};
    words.insert(words.end(), w, w + 4);
    if (last) break;
    tiles += (entries[e].longest + kKvTile - 1) / kKvTile;
    n_users += (int)users[e].size();
  }
  const size_t user_at = words.size();
  for (const auto &list : users)
    for (const User &u : list) {
      words.push_back(u.query);
      words.push_back(u.used);
    }
  const size_t n_path_at = words.size(), path_at = n_path_at + batch;
  if (path_host) {
    words.insert(words.end(), n_path_host, n_path_host + batch);
    words.insert(words.end(), path_host, path_host + (size_t)batch * max_path);
  }
  const pc::DraftWs ws = pc::carve_draft_ws(c, ctx->n_cu, workspace_dev, batch, t_draft, max_chunks);
  const int32_t *parents = draft_weights_out_dev ? parents_host : nullptr;   // (nothing else looks at the tree)
  hipStream_t s = (hipStream_t)stream;
  st = pc::upload_draft(ctx, words, batch, t_draft, parents, ws, s);
  if (st != PC_OK) return st;

  Args a;
  a.q = (const __bf16 *)q_dev;
  a.k_draft = (const __bf16 *)k_draft_dev;
  a.lse = lse_dev;
  a.k16 = ctx->k_store + (size_t)layer * ctx->layer_stride;
  a.k8 = ctx->k8_store + (size_t)layer * ctx->layer_stride8;
  a.k_scale = ctx->k_scale + (size_t)layer * ctx->n_slots8 * c.n_kv_heads * (c.slot_capacity / kKvTile);
  a.n_slots16 = ctx->n_slots16;
  a.entries = (const Entry *)ws.words;
  a.n_entries = (int)entries.size();
  a.users = (const User *)(ws.words + user_at);
  a.n_path = path_host ? ws.words + n_path_at : nullptr;
  a.path = ws.words + path_at;
  a.max_path = max_path;
  a.T = t_draft;
  a.Hq = c.n_q_heads;
  a.Hkv = c.n_kv_heads;
  a.C = c.slot_capacity;
  a.scale_log2e = 1.4426950408889634f / sqrtf((float)c.head_dim);
  a.w_in = weights_in_dev;
  a.w_out = weights_out_dev;
  a.w_draft = draft_weights_out_dev;
  a.draft.sees = parents ? ws.sees : nullptr;
  const int formats = pc::table_formats(rows, stride, batch), fmt = !(formats & 1) ? 0 : (formats & 2) ? 2 : 1;
  const dim3 grid((unsigned)(tiles * c.n_kv_heads));
#define PC_WEIGHTS(DD)                                                                                                 \
  do {                                                                                                                 \
    if (fmt == 0) hipLaunchKernelGGL((attention_weights_kernel<DD, 0>), grid, dim3(64), 0, s, a);                       \
    else if (fmt == 1) hipLaunchKernelGGL((attention_weights_kernel<DD, 1>), grid, dim3(64), 0, s, a);                  \
    else hipLaunchKernelGGL((attention_weights_kernel<DD, 2>), grid, dim3(64), 0, s, a);                                \
  } while (0)
  if (c.head_dim == 128) PC_WEIGHTS(128); else PC_WEIGHTS(64);
#undef PC_WEIGHTS
  PC_HIP(ctx, hipGetLastError());
  return PC_OK;
}
