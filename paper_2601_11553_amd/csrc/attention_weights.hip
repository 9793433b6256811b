// What a layer's query rows pay to every key: w_t = sum over rows of e^(q.k_t / sqrt(D) - lse), from the rows' log-sum-exp that the attention
// handed out.  With it the softmax needs no second pass, so a key's weight is one product and one exponential a row, and the keys are read once.
//
// The keys stay, the rows pass by: a slot's keys are matrix operands that go over the rows of every query that uses the slot, 32 rows at a
// time.  So a slot shared by several queries (a system prompt's chunk) is read once, its sums have one owner and one order -- no atomics, no
// second launch -- and are added to the running sums in place.  The rows are on the M side of the product: a lane then has 16 rows of one
// key, whose exponentials it adds up by itself.  The log-sum-exp, which belongs to rows, comes in as one more step of the contraction: -lse sqrt(D) as
// the sum of three bf16 numbers (24 bits) against ones.
//
// With few rows (a decoding step) the key stream bounds it: weights_stream_kernel.  With many the exponentials do (24 clocks of the vector port
// for each 64 of them, where the matrix cores take 18): weights_rows_kernel.
#include <algorithm>

#include "decode_common.hpp"

namespace {
using pc::bf16x8;
using pc::f32x16;
using pc::kKvTile;
using pc::u32x4;
using pc::dec::codes8;
using pc::dec::fast_exp2;

// Lists of a call (int32 words): the entries, the users of those that have not just one, then -- with paths -- their n_path [batch] and nodes [batch][max_path].
struct Entry {
  int32_t slot;     // slot id; -1 - b: the draft keys of query b
  int32_t piece0;   // first of its pieces among all entries'
  int32_t keys;     // 32 x the longest used length among its users, + the 64-key tiles of a piece (at most 31)
  int32_t user;     // its one user, who uses all of its keys; -1 - u: two words per user from word u of the users on, behind their number (two words)
};
constexpr int kMostKeys = 1 << 26;
constexpr int kRowsSpan = 2;   // tiles that weights_rows_kernel holds

struct Args {
  const __bf16 *q, *k_draft;
  const float *lse;
  const __bf16 *k16;
  const uint8_t *k8;
  const float *k_scale;
  int n_slots16;
  const Entry *entries;
  int n_entries;
  const int2 *users;
  const int32_t *n_path, *path;  // null: every row counts
  int max_path;
  int T, Hq, Hkv, C;
  float scale_log2e, sqrt_d;
  const float *w_in;   // [slots][Hkv][C], may be null (zero) and may be w_out
  float *w_out, *w_draft;
  pc::DraftView draft;
};

// The entry of a piece: the last one that starts at or before it.  A lane looks at every 64th entry and hands over the words of the one found.
__device__ __forceinline__ Entry find_entry(const Args &a, int piece, int lane) {
  int4 mine = {0, 0, 0, 0};
  for (int e0 = 0; e0 < a.n_entries; e0 += 64) {
    const int4 e = ((const int4 *)a.entries)[min(e0 + lane, a.n_entries - 1)];
    const unsigned long long before = __ballot(e0 + lane < a.n_entries && e.y <= piece);
    if (!before) break;
    const int at = 63 - __builtin_clzll(before);
    mine = {__builtin_amdgcn_readlane(e.x, at), __builtin_amdgcn_readlane(e.y, at), __builtin_amdgcn_readlane(e.z, at), __builtin_amdgcn_readlane(e.w, at)};
    if (before != ~0ull) break;
  }
  return {mine.x, mine.y, mine.z, mine.w};
}

// The rows that look at an entry's keys, in blocks of 32 (head of the group, counting row) of one user.  A wavefront's view of them.
template <int D>
struct Rows {
  static constexpr int KS = D / 16;
  const Args &a;
  const int g, lane, l32, g2, G;
  const Entry ent;
  const bool is_draft;
  const int longest;
  int n_users;
  const int2 *list;   // (of several users)
  unsigned long long *row_sees;   // [tiles][32] of this wavefront, draft keys: what each row of the block looks at

  struct Cursor { int u, r0, R, n_rows, b, used; };
  // request() only asks for what a block takes; everything that looks at it is in finish(), behind the work on the block before it
  struct Block { bf16x8 q[KS]; float lse; int node, rows, left; };   // rows: counting rows from r0 on; left: keys of the slot that the user uses
  struct Ready { bf16x8 ext; unsigned ok; };

  __device__ __forceinline__ Rows(const Args &args, const Entry &e, int g_, int lane_, unsigned long long *sees)
      : a(args), g(g_), lane(lane_), l32(lane_ & 31), g2(lane_ >> 5), G(args.Hq / args.Hkv), ent(e), is_draft(e.slot < 0), longest(e.keys >> 5), row_sees(sees) {
    n_users = 1;
    list = nullptr;
    if (ent.user < 0) {
      list = a.users + (-1 - ent.user);
      n_users = list[0].x;
      ++list;
    }
  }
  __device__ __forceinline__ void look(Cursor &c) const {
    int2 user = make_int2(ent.user, longest);
    if (list) user = list[c.u];
    c.b = user.x;
    c.used = user.y;
    c.n_rows = a.n_path ? a.n_path[c.b] : a.T;
    c.R = G * c.n_rows;
  }
  __device__ __forceinline__ void settle(Cursor &c) const {   // over users whose rows lie before row r0
    while (c.u < n_users && c.r0 >= c.R) {
      c.r0 -= (c.R + 31) / 32 * 32;
      if (++c.u < n_users) look(c);
    }
  }
  __device__ __forceinline__ Cursor begin(int r0) const {
    Cursor c = {0, r0, 0, 1, 0, 0};
    if (n_users > 0) look(c);
    settle(c);
    return c;
  }
  __device__ __forceinline__ bool done(const Cursor &c) const { return c.u >= n_users; }
  __device__ __forceinline__ void request(const Cursor &c, Block &blk) const {
    const int row = min(c.r0 + l32, c.R - 1), h = row / c.n_rows, j = row - h * c.n_rows, i = a.n_path ? a.path[(size_t)c.b * a.max_path + j] : j;
    const size_t at = ((size_t)c.b * a.Hq + g * G + h) * a.T + i;
    blk.lse = a.lse[at];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) blk.q[ks] = *(const bf16x8 *)(a.q + at * D + g2 * 8 + ks * 16);
    blk.node = i;
    blk.rows = c.R - c.r0;
    blk.left = c.used;
  }
  __device__ __forceinline__ Ready finish(const Block &blk, int tile0, int n_tiles) const {
    const bool ok = l32 < blk.rows && blk.lse != -INFINITY;
    const float x = -blk.lse * a.sqrt_d;
    const __bf16 hi = (__bf16)x, mid = (__bf16)(x - (float)hi), lo = (__bf16)(x - (float)hi - (float)mid);
    const bool split = !(fabsf((float)hi) == INFINITY);
    Ready r = {bf16x8{}, (unsigned)__builtin_amdgcn_ballot_w64(ok)};
    if (g2 == 0 && ok) {
      r.ext[0] = hi;
      r.ext[1] = split ? mid : (__bf16)0.f;
      r.ext[2] = split ? lo : (__bf16)0.f;
    }
    if (is_draft) {
      __builtin_amdgcn_wave_barrier();
      if (g2 == 0) {
#pragma unroll 4
        for (int t = 0; t < n_tiles; ++t) row_sees[t * 32 + l32] = ok ? pc::draft_row(a.draft, -1 - ent.slot, a.T, blk.node, (tile0 + t) * kKvTile) : 0ull;
      }
      __builtin_amdgcn_wave_barrier();
    }
    return r;
  }
  // adds what the block's rows pay to keys t0 .. t0 + 63, the n-th tile of finish(); key operand (kb, ks): elements 16 ks + 8 g2 .. +7 of key 32 kb + l32
  template <class Key>
  __device__ __forceinline__ void pay(Key key, const Block &blk, const Ready &r, int t0, int n, float (&acc)[2][2]) const {
    const int left = blk.left - t0;
    if (left <= 0) return;
    bf16x8 ones = bf16x8{};
    if (g2 == 0) ones[0] = ones[1] = ones[2] = (__bf16)1.f;
    f32x16 s[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int x = 0; x < 16; ++x) s[kb][x] = 0.f;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(r.ext, ones, s[kb], 0, 0, 0);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(blk.q[ks], key(kb, ks), s[kb], 0, 0, 0);
    auto p = [&](int kb, int x) __attribute__((always_inline)) { return fast_exp2(s[kb][x] * a.scale_log2e); };
    // (register x of lane half g2 is row 8 (x / 4) + 4 g2 + x % 4.)  What does not count is selected away, not multiplied by 0: it need not be finite
    auto kept = [](float v, int bits, int at) __attribute__((always_inline)) {
      return __uint_as_float(__float_as_uint(v) & (unsigned)__builtin_amdgcn_sbfe(bits, at, 1));   // (all bits or none)
    };
    if (is_draft) {
#pragma unroll
      for (int x4 = 0; x4 < 4; ++x4) {
        const u32x4 *w = (const u32x4 *)(row_sees + n * 32 + 8 * x4 + 4 * g2);
        const u32x4 w01 = w[0], w23 = w[1];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          acc[kb][0] += kept(p(kb, 4 * x4), (int)w01[kb], l32) + kept(p(kb, 4 * x4 + 2), (int)w23[kb], l32);
          acc[kb][1] += kept(p(kb, 4 * x4 + 1), (int)w01[2 + kb], l32) + kept(p(kb, 4 * x4 + 3), (int)w23[2 + kb], l32);
        }
      }
    } else if (r.ok == ~0u && left >= kKvTile) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int x = 0; x < 16; ++x) acc[kb][x & 1] += p(kb, x);
    } else {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const int rows = kb * 32 + l32 < left ? (int)(r.ok >> (4 * g2)) : 0;
#pragma unroll
        for (int x = 0; x < 16; ++x) acc[kb][x & 1] += kept(p(kb, x), rows, (x >> 2) * 8 + (x & 3));
      }
    }
  }
  // a tile's sums: lane l gets key l's
  __device__ __forceinline__ float total(const float (&acc)[2][2]) const {
    float tot[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      tot[kb] = acc[kb][0] + acc[kb][1];
      tot[kb] += __shfl_xor(tot[kb], 32, 64);
    }
    return g2 ? tot[1] : tot[0];
  }
  __device__ __forceinline__ size_t weight_at(int t0) const {
    return is_draft ? ((size_t)(-1 - ent.slot) * a.Hkv + g) * a.T + t0 + lane : ((size_t)ent.slot * a.Hkv + g) * a.C + t0 + lane;
  }
  // the row of a key, bf16 and (8-bit slots) codes
  __device__ __forceinline__ bool is8(int fmt) const { return fmt != 0 && !is_draft && (fmt == 1 || ent.slot >= a.n_slots16); }
  __device__ __forceinline__ const __bf16 *keys16() const {
    return is_draft ? a.k_draft + ((size_t)(-1 - ent.slot) * a.Hkv + g) * a.T * D : a.k16 + ((size_t)ent.slot * a.Hkv + g) * a.C * D;
  }
  __device__ __forceinline__ size_t head8() const { return (size_t)(ent.slot - a.n_slots16) * a.Hkv + g; }
};

// Few rows: one wavefront walks the tiles of a piece with the keys in registers, the next tile's requested ahead, and its rows -- where they are one block -- loaded
// once.  Up to 2 wavefronts a SIMD, each with 16 KB on the way.  FMT: 0 bf16 slots, 1 8-bit slots, 2 both.
template <int D, int FMT>
__global__ __launch_bounds__(64, 2) void weights_stream_kernel(const Args a) {
  constexpr int KS = D / 16;
  __shared__ __align__(16) unsigned long long row_sees[32];
  const int lane = threadIdx.x, g = blockIdx.x % a.Hkv, piece = blockIdx.x / a.Hkv;
  const Rows<D> rows(a, find_entry(a, piece, lane), g, lane, row_sees);
  const int longest = rows.longest, span = rows.ent.keys & 31, tile0 = (piece - rows.ent.piece0) * span, tile_end = min(tile0 + span, (longest + kKvTile - 1) / kKvTile);
  const bool is8 = rows.is8(FMT);
  u32x4 raw[2][KS];
  float raw_scale = 1.f;
  auto request_keys = [&](int tile) __attribute__((always_inline)) {
    const int t0 = tile * kKvTile, last = min(kKvTile, longest - t0) - 1;   // (past a ragged end: the last key's)
    if (FMT != 0 && is8) {
      const size_t head = rows.head8();
      raw_scale = a.k_scale[head * (a.C / kKvTile) + tile];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const uint8_t *row = a.k8 + (head * a.C + t0 + min(kb * 32 + rows.l32, last)) * D + rows.g2 * 8;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const uint2 w = *(const uint2 *)(row + ks * 16);
          raw[kb][ks] = u32x4{w.x, w.y, 0, 0};
        }
      }
    } else {
      const __bf16 *base = rows.keys16();
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const __bf16 *row = base + (size_t)(t0 + min(kb * 32 + rows.l32, last)) * D + rows.g2 * 8;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) raw[kb][ks] = *(const u32x4 *)(row + ks * 16);
      }
    }
  };
  request_keys(tile0);
  const typename Rows<D>::Cursor first = rows.begin(0);
  typename Rows<D>::Cursor at = first;
  typename Rows<D>::Block blk;
  typename Rows<D>::Ready ready;
  if (!rows.done(at)) {
    rows.request(at, blk);
    ready = rows.finish(blk, tile0, 1);
  }
  for (int tile = tile0; tile < tile_end; ++tile) {
    const int t0 = tile * kKvTile;
    bf16x8 k[2][KS];
    const float scale = raw_scale;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) k[kb][ks] = FMT != 0 && is8 ? codes8(make_uint2(raw[kb][ks][0], raw[kb][ks][1]), scale) : __builtin_bit_cast(bf16x8, raw[kb][ks]);
    if (tile + 1 < tile_end) request_keys(tile + 1);
    const bool mine = t0 + lane < longest;
    const size_t w_at = rows.weight_at(t0);
    float before = 0.f;
    if (mine && !rows.is_draft && a.w_in) before = a.w_in[w_at];
    float acc[2][2] = {{0.f, 0.f}, {0.f, 0.f}};
    auto key = [&](int kb, int ks) __attribute__((always_inline)) { return k[kb][ks]; };
    if (!rows.done(first)) {
      bool again = tile > tile0 && (rows.is_draft || at.u != first.u || at.r0 != first.r0);
      at = first;
      while (true) {
        if (again) {
          rows.request(at, blk);
          ready = rows.finish(blk, tile, 1);
        }
        rows.pay(key, blk, ready, t0, 0, acc);
        typename Rows<D>::Cursor nx = at;
        nx.r0 += 32;
        rows.settle(nx);
        if (rows.done(nx)) break;
        at = nx;
        again = true;
      }
    }
    const float sum = rows.total(acc);
    if (mine) {
      if (rows.is_draft) a.w_draft[w_at] = sum;
      else a.w_out[w_at] = before + sum;
    }
  }
}

// Many rows: a workgroup of four wavefronts keeps the keys of up to two tiles in LDS as bf16 (16-byte pieces XOR-swizzled inside rows of 256 bytes by row & 15, of
// 128 bytes by (row >> 1) & 7); the wavefronts take every fourth block of rows each.  Small pieces of work and four wavefronts a SIMD: while one waits for its lists,
// keys or rows, the others keep the vector port busy.  (Two wavefronts a SIMD with the keys in registers, or four tiles in LDS and the next block's rows requested
// ahead: 4 prompts of 256 rows x 16 heads over 3100 keys 51 and 43 us.)
template <int D, int FMT>
__global__ __launch_bounds__(256, 4) void weights_rows_kernel(const Args a) {
  constexpr int KS = D / 16, ROW = D * 2, TILE = kKvTile * ROW;
  __shared__ __align__(16) char keys[kRowsSpan * TILE];
  __shared__ __align__(16) unsigned long long row_sees[4][kRowsSpan * 32];
  __shared__ float sums[4][kRowsSpan][kKvTile];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = blockIdx.x % a.Hkv, piece = blockIdx.x / a.Hkv;
  const Rows<D> rows(a, find_entry(a, piece, lane), g, lane, row_sees[wave]);
  const int longest = rows.longest, span = rows.ent.keys & 31, tile0 = (piece - rows.ent.piece0) * span;
  const int n_tiles = min(tile0 + span, (longest + kKvTile - 1) / kKvTile) - tile0, first_key = tile0 * kKvTile, n_keys = min(longest - first_key, n_tiles * kKvTile);
  auto swz = [](int row) __attribute__((always_inline)) { return ROW == 256 ? (row & 15) : ((row >> 1) & 7); };
  {
    constexpr int PIECES = D / 8;   // 16-byte pieces of a row (of 8 elements)
    const bool is8 = rows.is8(FMT);
    const size_t head = is8 ? rows.head8() : 0;
    const __bf16 *base = rows.keys16() + (size_t)first_key * D;
    for (int e0 = 0; e0 < n_tiles * kKvTile * PIECES; e0 += 1024) {   // (past a ragged end: the last key's)
      u32x4 w[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int e = e0 + x * 256 + tid, row = min(e / PIECES, n_keys - 1), c = e % PIECES;
        if (FMT != 0 && is8) {
          const uint2 q = *(const uint2 *)(a.k8 + (head * a.C + first_key + row) * D + c * 8);
          w[x] = __builtin_bit_cast(u32x4, codes8(q, a.k_scale[head * (a.C / kKvTile) + tile0 + row / kKvTile]));
        } else {
          w[x] = *(const u32x4 *)(base + (size_t)row * D + c * 8);
        }
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int e = e0 + x * 256 + tid, row = e / PIECES, c = e % PIECES;
        if (row < n_tiles * kKvTile) *(u32x4 *)(keys + row * ROW + ((c ^ swz(row)) * 16)) = w[x];
      }
    }
  }
  __syncthreads();
  float acc[kRowsSpan][2][2];
#pragma unroll
  for (int t = 0; t < kRowsSpan; ++t) acc[t][0][0] = acc[t][0][1] = acc[t][1][0] = acc[t][1][1] = 0.f;
  int k_rd[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) k_rd[ks] = rows.l32 * ROW + (((2 * ks + rows.g2) ^ swz(rows.l32)) * 16);
  for (typename Rows<D>::Cursor at = rows.begin(32 * wave); !rows.done(at);) {
    typename Rows<D>::Block blk;
    rows.request(at, blk);
    const typename Rows<D>::Ready ready = rows.finish(blk, tile0, n_tiles);
#pragma unroll
    for (int t = 0; t < kRowsSpan; ++t)
      if (t < n_tiles)
        rows.pay([&](int kb, int ks) __attribute__((always_inline)) { return *(const bf16x8 *)(keys + t * TILE + kb * 32 * ROW + k_rd[ks]); }, blk, ready,
                 first_key + t * kKvTile, t, acc[t]);
    at.r0 += 4 * 32;
    rows.settle(at);
  }
#pragma unroll
  for (int t = 0; t < kRowsSpan; ++t) sums[wave][t][lane] = rows.total(acc[t]);
  __syncthreads();
  // wavefront t finishes tile t
  const int t0 = first_key + wave * kKvTile;
  if (wave < n_tiles && t0 + lane < longest) {
    const float sum = (sums[0][wave][lane] + sums[1][wave][lane]) + (sums[2][wave][lane] + sums[3][wave][lane]);
    const size_t w_at = rows.weight_at(t0);
    if (rows.is_draft) a.w_draft[w_at] = sum;
    else a.w_out[w_at] = (a.w_in ? a.w_in[w_at] : 0.f) + sum;
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
  if ((long)batch * t_draft * (c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim >= (1L << 31) || c.slot_capacity >= kMostKeys || t_draft >= kMostKeys) return pc::fail(ctx, PC_ESHAPE, "operand larger than 2^31 elements");
  std::vector<int32_t> rows;
  st = pc::build_chunk_table(ctx, layer, batch, 1, slot_ids_host, used_len_host, n_chunks_host, max_chunks, rows);
  if (st != PC_OK) return st;
  const size_t need = percache_draft_workspace_bytes(ctx, batch, t_draft, max_chunks);
  if (!workspace_dev || workspace_bytes < need) return pc::fail(ctx, PC_ENOMEM, "draft workspace has %zu bytes, need %zu", workspace_bytes, need);
  if ((uintptr_t)workspace_dev % pc::kAlign) return pc::fail(ctx, PC_EINVAL, "workspace must be 256-byte aligned");

  // The slots in the order of their first mention, each with its users in the order of the batch (a query that names a slot twice: two users)
  struct Slot { int32_t slot, longest, n_users, blocks, only, only_used, at; };
  const int stride = pc::tbl_stride(max_chunks), G = c.n_q_heads / c.n_kv_heads;
  auto rows_of = [&](int b) { return G * (path_host ? n_path_host[b] : t_draft); };
  std::vector<Slot> slots;
  std::vector<int32_t> of_slot(c.n_slots, -1);
  slots.reserve((size_t)batch * (max_chunks + 1));
  auto use = [&](Slot &sl, int b, int used) {
    if (used > sl.longest) sl.longest = used;
    if (rows_of(b) == 0) return;
    sl.only = b;
    sl.only_used = used;
    sl.blocks += (rows_of(b) + 31) / 32;
    ++sl.n_users;
  };
  bool several = false;
  for (int b = 0; b < batch; ++b) {
    const int32_t *row = rows.data() + (size_t)b * stride;
    for (int ci = 0; ci < row[0]; ++ci) {
      const int slot = row[pc::kTblHeader + 2 * ci], used = row[pc::kTblHeader + 2 * ci + 1];
      if (used == 0) continue;
      if (of_slot[slot] < 0) {
        of_slot[slot] = (int)slots.size();
        slots.push_back({slot, 0, 0, 0, 0, 0, 0});
      } else {
        several = true;
      }
      use(slots[of_slot[slot]], b, used);
    }
  }
  if (draft_weights_out_dev)
    for (int b = 0; b < batch; ++b) {
      slots.push_back({-1 - b, 0, 0, 0, 0, 0, 0});
      use(slots.back(), b, t_draft);
    }
  if (slots.empty()) return PC_OK;
  // Many rows of a query to a key: weights_rows_kernel.  A piece has as many tiles as give every workgroup that the chip holds at once (8 of one wavefront a CU, 4 of four) one
  // of them, fewer where a tile has more blocks of rows than the others; what has more of them comes first.
  int most_rows = 0, least_blocks = INT32_MAX;
  long all_tiles = 0;
  for (int b = 0; b < batch; ++b) most_rows = std::max(most_rows, rows_of(b));
  const bool by_rows = most_rows > 64;
  for (const Slot &sl : slots) {
    all_tiles += (sl.longest + kKvTile - 1) / kKvTile;
    if (sl.blocks) least_blocks = std::min(least_blocks, sl.blocks);
  }
  const long held = (by_rows ? 4L : 8L) * ctx->n_cu, share = (all_tiles * c.n_kv_heads + held - 1) / held;
  const int most = by_rows ? kRowsSpan : 16;
  if (several) {
    std::stable_sort(slots.begin(), slots.end(), [](const Slot &x, const Slot &y) { return x.blocks > y.blocks; });
    for (size_t e = 0; e < slots.size(); ++e)
      if (slots[e].slot >= 0) of_slot[slots[e].slot] = (int)e;
  }
  std::vector<int32_t> words;
  words.reserve(slots.size() * 4 + (several ? (size_t)batch * max_chunks * 2 : 0) + (path_host ? (size_t)batch * (max_path + 1) : 0) + ((size_t)batch * t_draft + 1) / 2 + 2);
  int pieces = 0, n_users = 0;
  for (Slot &sl : slots) {
    const int span = (int)std::max(1L, std::min((long)most, share * least_blocks / std::max(1, sl.blocks)));
    int32_t user = sl.only;
    if (sl.n_users != 1 || sl.only_used != sl.longest) {   // (none or several, or one that uses less than another, none of whose rows counts)
      user = -1 - n_users;
      sl.at = 1 + n_users;
      n_users += sl.n_users + 1;
    }
    const int32_t w[4] = {sl.slot, pieces, sl.longest * 32 + span, user};
    words.insert(words.end(), w, w + 4);
    pieces += ((sl.longest + kKvTile - 1) / kKvTile + span - 1) / span;
  }
  const size_t user_at = words.size();
  words.resize(user_at + 2 * (size_t)n_users, 0);
  if (n_users) {
    for (const Slot &sl : slots)
      if (sl.at) words[user_at + 2 * (size_t)(sl.at - 1)] = sl.n_users;
    std::vector<int32_t> filled(slots.size(), 0);
    for (int b = 0; b < batch; ++b) {
      const int32_t *row = rows.data() + (size_t)b * stride;
      for (int ci = 0; ci < row[0]; ++ci) {
        const int slot = row[pc::kTblHeader + 2 * ci], used = row[pc::kTblHeader + 2 * ci + 1];
        if (used == 0 || rows_of(b) == 0) continue;
        const int e = of_slot[slot];
        if (!slots[e].at) continue;
        int32_t *w = words.data() + user_at + 2 * (size_t)(slots[e].at + filled[e]++);
        w[0] = b;
        w[1] = used;
      }
    }
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
  a.n_entries = (int)slots.size();
  a.users = (const int2 *)(ws.words + user_at);
  a.n_path = path_host ? ws.words + n_path_at : nullptr;
  a.path = ws.words + path_at;
  a.max_path = max_path;
  a.T = t_draft;
  a.Hq = c.n_q_heads;
  a.Hkv = c.n_kv_heads;
  a.C = c.slot_capacity;
  a.scale_log2e = 1.4426950408889634f / sqrtf((float)c.head_dim);
  a.sqrt_d = sqrtf((float)c.head_dim);
  a.w_in = weights_in_dev;
  a.w_out = weights_out_dev;
  a.w_draft = draft_weights_out_dev;
  a.draft.sees = parents ? ws.sees : nullptr;
  const int formats = pc::table_formats(rows, stride, batch), fmt = !(formats & 1) ? 0 : (formats & 2) ? 2 : 1;
  const dim3 grid((unsigned)(pieces * c.n_kv_heads));
#define PC_WEIGHTS_F(DD, FF)                                                                                         \
  do {                                                                                                               \
    if (by_rows) hipLaunchKernelGGL((weights_rows_kernel<DD, FF>), grid, dim3(256), 0, s, a);                         \
    else hipLaunchKernelGGL((weights_stream_kernel<DD, FF>), grid, dim3(64), 0, s, a);                                \
  } while (0)
#define PC_WEIGHTS(DD) do { if (fmt == 0) PC_WEIGHTS_F(DD, 0); else if (fmt == 1) PC_WEIGHTS_F(DD, 1); else PC_WEIGHTS_F(DD, 2); } while (0)
  if (c.head_dim == 128) PC_WEIGHTS(128); else PC_WEIGHTS(64);
#undef PC_WEIGHTS_F
#undef PC_WEIGHTS
  PC_HIP(ctx, hipGetLastError());
  return PC_OK;
}
