// Slots copied to slots of the same format in many layers: continuations that go on from one prompt, beams that change places.  All copies of a call
// take what the slots held before it, so a list may name a slot as a source and as a destination (a permutation, a rotation).
//
// Slots of one format are laid out alike, so an element's copy is at the same offset in every slot, and the thread that has this offset does all
// copies that depend on each other itself, in an order in which no slot is written before it has been read; a ring of slots keeps its first one in
// registers meanwhile.  Nothing is exchanged between threads and no workspace is needed.  What bounds it: the bytes, a source read once for all of
// its copies (they are neighbours in the list), every copy written once: 4 slots to 12, 1000 tokens of 8 heads of 128, 4 layers, 262 MB in 46 us, 5.7 TB/s.
#include <algorithm>
#include <exception>

#include "launch_lists.hpp"

namespace {
using pc::kKvTile;
using pc::u32x4;
using namespace pc::fork;

// One workgroup copies a block of 64 tokens of one layer and kv head for one list of dependent moves.  ES: bytes per element.
template <int D, int ES>
__global__ __launch_bounds__(256) void kv_fork_kernel(const Moves moves, int blocks, int Hkv, int C, long layer_stride, long scale_stride, char *k, char *v, float *k_scale,
                                                      float *v_scale) {
  constexpr int NP = kKvTile * D * ES / 16 / 256, K_ROW = D * ES, V_ROW = kKvTile * ES, PER = 16 / ES;
  const int tid = threadIdx.x, block = blockIdx.x % blocks, h = blockIdx.x / blocks % Hkv, p = blockIdx.x / blocks / Hkv;
  const long layer = blockIdx.y;
  const int first = moves.start[p], end = moves.start[p + 1];
  u32x4 rk[NP], rv[NP], tk[NP], tv[NP];
  float rs = 0.f, ts = 0.f;
  int held = -1, held_len = 0;   // the slot that rk, rv hold, and how many of its tokens
  for (int at = first; at < end; ++at) {
    const Move m = moves.m[at];
    const int here = m.len - block * kKvTile;   // tokens of this block that are copied
    if (here <= 0 || (m.src == m.dst && here >= kKvTile)) continue;   // (a slot that is cut: zeros behind its last token)
    if (m.src >= 0 && (m.src != held || m.len > held_len)) {
      const size_t base = (size_t)layer * layer_stride + (((size_t)m.src * Hkv + h) * C + (size_t)block * kKvTile) * (D * ES);
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        rk[i] = *(const u32x4 *)(k + base + (tid + 256 * i) * 16);
        rv[i] = *(const u32x4 *)(v + base + (tid + 256 * i) * 16);
      }
      if (ES == 1 && tid < 2) rs = (tid ? v_scale : k_scale)[layer * scale_stride + ((size_t)m.src * Hkv + h) * (C / kKvTile) + block];
      held = m.src;
      held_len = m.len;
    }
    if (m.dst < 0) {
#pragma unroll
      for (int i = 0; i < NP; ++i) { tk[i] = rk[i]; tv[i] = rv[i]; }
      ts = rs;
      continue;
    }
    const size_t base = (size_t)layer * layer_stride + (((size_t)m.dst * Hkv + h) * C + (size_t)block * kKvTile) * (D * ES);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int byte = (tid + 256 * i) * 16;
      u32x4 x = m.src < 0 ? tk[i] : rk[i], y = m.src < 0 ? tv[i] : rv[i];
      if (byte / K_ROW < here) *(u32x4 *)(k + base + byte) = x;
      if (here < kKvTile) {   // zeros behind the last token, as every block of V has them
        const int q0 = byte % V_ROW / ES;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
          const int q = q0 + e, key = ES == 2 ? (q & ~15) + pc::blocked_key(q & 15) : pc::blocked_key8(q);
          if (key >= here) y[e * ES / 4] &= ES == 2 ? ~(0xffffu << (16 * (e & 1))) : ~(0xffu << (8 * (e & 3)));
        }
      }
      *(u32x4 *)(v + base + byte) = y;
    }
    if (ES == 1 && tid < 2)
      (tid ? v_scale : k_scale)[layer * scale_stride + ((size_t)m.dst * Hkv + h) * (C / kKvTile) + block] = m.src < 0 ? ts : rs;
    if (m.dst == held) held = -1;
  }
}

// The moves of a call in an order in which no slot is written before the others have read it; lists[p] are moves that depend on each other (or share their source),
// cut where a launch may end: atoms, none longer than a launch.
typedef std::vector<std::vector<Move>> Atoms;
void order_moves(const std::vector<Move> &all, int n_slots, std::vector<Atoms> &lists) {
  const int n = (int)all.size();
  std::vector<int> parent(n_slots, -1), readers(n_slots, 0), writer(n_slots, -1), next_of(n, -1), first_of(n_slots, -1);
  for (int i = 0; i < n_slots; ++i) parent[i] = i;
  auto find = [&](int x) {
    while (parent[x] != x) x = parent[x] = parent[parent[x]];
    return x;
  };
  for (int i = 0; i < n; ++i) {
    parent[find(all[i].src)] = find(all[i].dst);
    readers[all[i].src] += all[i].src != all[i].dst;   // (a slot that is cut waits for the others that read it)
    writer[all[i].dst] = i;
  }
  for (int i = n - 1; i >= 0; --i) {
    const int root = find(all[i].src);
    next_of[i] = first_of[root];
    first_of[root] = i;
  }
  std::vector<char> done(n, 0);
  std::vector<int> ready;
  for (int root = 0; root < n_slots; ++root) {
    if (first_of[root] < 0) continue;
    Atoms atoms;
    ready.clear();
    for (int i = first_of[root]; i >= 0; i = next_of[i])
      if (readers[all[i].dst] == 0) ready.push_back(i);
    // copies of one source next to each other
    std::stable_sort(ready.begin(), ready.end(), [&](int a, int b) { return all[a].src < all[b].src; });
    for (size_t at = 0; at < ready.size(); ++at) {
      const Move &m = all[ready[at]];
      atoms.push_back({m});
      done[ready[at]] = 1;
      if (m.src != m.dst && --readers[m.src] == 0 && writer[m.src] >= 0) ready.push_back(writer[m.src]);
    }
    for (int i = first_of[root]; i >= 0; i = next_of[i]) {   // what is left is a ring: every slot of it is read once and written once
      if (done[i]) continue;
      std::vector<int> ring;
      for (int j = i; !done[j]; j = writer[all[j].src]) {
        ring.push_back(j);
        done[j] = 1;
      }
      // ring[0] writes a slot that the last one reads.  A ring too long for one launch is two, the first of which leaves the slot that the
      // last move reads where the second one starts.
      const int last_len = all[ring.back()].len, last_dst = all[ring.back()].dst;
      size_t from = 0;
      int saved = all[ring[0]].dst;
      while (true) {
        const size_t left = ring.size() - from, take = std::min(left, (size_t)kMoves - 2);
        std::vector<Move> atom;
        atom.push_back({saved, -1, last_len});
        const bool all_of_it = take == left;
        for (size_t j = from; j < from + take - (all_of_it ? 1 : 0); ++j) atom.push_back(all[ring[j]]);
        const int to = all_of_it ? last_dst : all[ring[from + take - 1]].src;
        atom.push_back({-1, to, last_len});
        atoms.push_back(atom);
        if (all_of_it) break;
        from += take;
        saved = to;
      }
    }
    lists.push_back(std::move(atoms));
  }
}

// A launch: lists of moves of one store, in layers whose copies are equally long.
struct Launch {
  int eight, layer0, n_layers, n_lists, n_moves, longest;
  Moves moves;
  int blocks() const { return (longest + kKvTile - 1) / kKvTile; }
};
pc_status launch_moves(percache_ctx *ctx, const Launch &x, hipStream_t s) {
  const percache_config &c = ctx->cfg;
  const bool eight = x.eight;
  const int blocks = x.blocks();
  const dim3 grid((unsigned)((long)blocks * c.n_kv_heads * x.n_lists), (unsigned)x.n_layers);
  const long layer_bytes = eight ? (long)ctx->layer_stride8 : (long)ctx->layer_stride * 2, scales = (long)ctx->n_slots8 * c.n_kv_heads * (c.slot_capacity / kKvTile);
  char *k = (eight ? (char *)ctx->k8_store : (char *)ctx->k_store) + x.layer0 * layer_bytes, *v = (eight ? (char *)ctx->v8_store : (char *)ctx->v_store) + x.layer0 * layer_bytes;
  float *ks = ctx->k_scale + x.layer0 * scales, *vs = ctx->v_scale + x.layer0 * scales;
#define PC_FORK(DD, EE) hipLaunchKernelGGL((kv_fork_kernel<DD, EE>), grid, dim3(256), 0, s, x.moves, blocks, c.n_kv_heads, c.slot_capacity, layer_bytes, scales, k, v, ks, vs)
  if (c.head_dim == 128) { if (eight) PC_FORK(128, 1); else PC_FORK(128, 2); }
  else { if (eight) PC_FORK(64, 1); else PC_FORK(64, 2); }
#undef PC_FORK
  PC_HIP(ctx, hipGetLastError());
  return PC_OK;
}
}  // namespace

extern "C" pc_status percache_kv_fork(percache_ctx *ctx, int32_t layer0, int32_t n_layers, const int32_t *src_slots_host, const int32_t *dst_slots_host,
                                      const int32_t *n_tokens_host, int32_t n, void *stream) try {
  if (!ctx) return PC_EINVAL;
  const percache_config &c = ctx->cfg;
  if (n < 0 || (n > 0 && (!src_slots_host || !dst_slots_host))) return pc::fail(ctx, PC_EINVAL, "a slot list is NULL or n is negative");
  if (n_layers < 1 || layer0 < 0 || layer0 > c.n_layers - n_layers) return pc::fail(ctx, PC_ESLOT, "layers [%d,%ld) out of range [0,%d)", layer0, (long)layer0 + n_layers, c.n_layers);
  std::vector<char> named(c.n_slots, 0);
  for (int i = 0; i < n; ++i) {
    const int src = src_slots_host[i], dst = dst_slots_host[i];
    if (src < 0 || src >= c.n_slots || dst < 0 || dst >= c.n_slots) return pc::fail(ctx, PC_ESLOT, "copy %d: slot %d or %d out of range [0,%d)", i, src, dst, c.n_slots);
    if (ctx->is8(src) != ctx->is8(dst)) return pc::fail(ctx, PC_ESLOT, "copy %d: slots %d and %d hold different formats", i, src, dst);
    if (named[dst]) return pc::fail(ctx, PC_EINVAL, "slot %d is the destination of two copies", dst);
    named[dst] = 1;
    for (int l = layer0; l < layer0 + n_layers; ++l) {
      const int have = ctx->slot_len[(size_t)l * c.n_slots + src];
      if (have <= 0) return pc::fail(ctx, PC_ESLOT, "copy %d: slot %d of layer %d is empty", i, src, l);
      if (n_tokens_host && (n_tokens_host[i] < 1 || n_tokens_host[i] > have))
        return pc::fail(ctx, PC_ELEN, "copy %d: %d tokens outside [1,%d], what slot %d of layer %d holds", i, n_tokens_host[i], have, src, l);
    }
  }
  if (n == 0) return PC_OK;
  auto len_of = [&](int l, int i) { return n_tokens_host ? n_tokens_host[i] : ctx->slot_len[(size_t)l * c.n_slots + src_slots_host[i]]; };
  // (all launches are put together before the first of them)
  constexpr long kMostBlocks = 1L << 23;   // of a launch: a grid has fewer than 2^32 threads
  std::vector<Launch> launches;
  std::vector<int32_t> lens(n);
  for (int l0 = layer0; l0 < layer0 + n_layers;) {
    int l1 = l0 + 1;   // layers whose copies are equally long share their launches
    for (bool same = true; same && l1 < layer0 + n_layers && l1 - l0 < 65535;) {
      for (int i = 0; same && i < n; ++i) same = len_of(l1, i) == len_of(l0, i);
      l1 += same;
    }
    for (int eight = 0; eight < 2; ++eight) {
      std::vector<Move> all;
      const int off = eight ? ctx->n_slots16 : 0;
      for (int i = 0; i < n; ++i)
        if ((int)ctx->is8(src_slots_host[i]) == eight && (src_slots_host[i] != dst_slots_host[i] || (n_tokens_host && n_tokens_host[i] % kKvTile)))
          all.push_back({src_slots_host[i] - off, dst_slots_host[i] - off, len_of(l0, i)});
      if (all.empty()) continue;
      std::vector<Atoms> lists;
      order_moves(all, eight ? ctx->n_slots8 : ctx->n_slots16, lists);
      const size_t first = launches.size();
      for (const Atoms &atoms : lists) {
        bool open = false;
        for (const std::vector<Move> &atom : atoms) {
          const bool fits = launches.size() > first && launches.back().n_moves + (int)atom.size() <= kMoves &&
                            (open || (launches.back().n_lists + 1L) * ((c.slot_capacity + kKvTile - 1) / kKvTile) * c.n_kv_heads <= kMostBlocks);
          if (!fits) {
            launches.push_back({eight, l0, l1 - l0, 0, 0, 0, {}});
            open = false;
          }
          Launch &x = launches.back();
          if (!open) x.moves.start[x.n_lists++] = (uint16_t)x.n_moves;
          open = true;
          for (const Move &m : atom) {
            x.moves.m[x.n_moves++] = m;
            x.longest = std::max(x.longest, (int)m.len);
          }
          x.moves.start[x.n_lists] = (uint16_t)x.n_moves;
        }
      }
    }
    l0 = l1;
  }
  for (const Launch &x : launches) {
    const pc_status st = launch_moves(ctx, x, (hipStream_t)stream);
    if (st != PC_OK) return st;
  }
  // (lengths all at once: a slot may be a source and a destination)
  for (int l = layer0; l < layer0 + n_layers; ++l) {
    for (int i = 0; i < n; ++i) lens[i] = len_of(l, i);
    for (int i = 0; i < n; ++i) ctx->slot_len[(size_t)l * c.n_slots + dst_slots_host[i]] = lens[i];
  }
  return PC_OK;
} catch (const std::exception &) {   // (before the first launch; the text is short enough to be kept without an allocation)
  return pc::fail(ctx, PC_ENOMEM, "no host memory");
}
