// What a layer's query rows pay to every key: w_t = sum over rows of e^(q.k_t / sqrt(D) - lse), from the rows' log-sum-exp that the attention
// handed out.  With it the softmax needs no second pass, so a key's weight is one product and one exponential a row, and the keys are read once.
//
// The keys stay, the rows pass by: a slot's keys are matrix operands that go over the rows of every query that uses the slot, 32 rows at a time.  So
// a slot shared by several queries (a system prompt's chunk) is read once, its sums have one owner and one order -- no atomics -- and are added to
// the running sums in place; only where that would keep one wavefront at work when the others are done are a slot's users split among several, whose
// sums a second launch adds up (weights_join_kernel).  The rows are on the M side of the product: a lane then has 16 rows of one key, whose
// exponentials it adds up by itself.  The log-sum-exp, which belongs to rows, comes in as the last step of the contraction: -lse sqrt(D) as the sum
// of three bf16 numbers (24 bits) against ones.
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

// Lists of a call (int32 words): the entries, the users of those that have not just one, the slots split among several entries, then -- with paths --
// n_path [batch] and the nodes [batch][max_path].
struct Entry {
  int32_t slot;     // slot id; -1 - b: the draft keys of query b
  int32_t piece0;   // first of its pieces among all entries' (few rows: the cost of the entries before it)
  int32_t keys;     // 32 x the longest used length among its users, + the 64-key tiles of a piece (few rows: what a tile costs; at most 31)
  int32_t user;     // its one user, who uses all of its keys; -1 - u: the u-th of the users' records is {their number, of a split slot 1 + the place of its sums}, theirs are behind it
};
struct User {
  int32_t query, used, rows, unused;   // rows: counting rows of a head
};
struct Split {
  int32_t slot, longest, parts, place;   // place: of its first entry's sums in Args::parts, 64 floats each: [entry][kv head][tile]
};
// Few rows: what a tile costs for each block of 32 rows.  A tile of draft keys has its rows and what they look at to load for itself, about three
// tiles' time: eight of them in one share, as a tile each, made a call of 35 us one of 42.
constexpr int kDraftCost = 3, kMostCost = 31;
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
  const User *users;
  const int32_t *n_path, *path;  // null: every row counts
  int max_path;
  int share;                     // few rows: the cost that a wavefront takes
  int T, Hq, Hkv, C;
  float scale_log2e, sqrt_d;
  const float *w_in;   // [slots][Hkv][C], may be null (zero) and may be w_out
  float *w_out, *w_draft, *parts;
  pc::DraftView draft;
};

// The entry of a piece: the last one that starts at or before it (-1: none).  A lane looks at every 64th entry.
__device__ __forceinline__ int find_entry(const Args &a, int piece, int lane) {
  int found = -1;
  for (int e0 = 0; e0 < a.n_entries; e0 += 64) {
    const int at = ((const int4 *)a.entries)[min(e0 + lane, a.n_entries - 1)].y;
    const unsigned long long before = __ballot(e0 + lane < a.n_entries && at <= piece);
    if (!before) break;
    found = e0 + 63 - __builtin_clzll(before);
    if (before != ~0ull) break;
  }
  return found;
}

// The rows that look at an entry's keys, in blocks of 32 (head of the group, counting row) of one user.  A wavefront's view of them.
template <int D>
struct Rows {
  static constexpr int KS = D / 16;
  const Args &a;
  const int g, lane, l32, g2, G;
  Entry ent;
  bool is_draft;
  int longest;
  int n_users, place;   // (place: 1 + that of its sums, a split slot's)
  const User *list;     // (of several users)
  unsigned long long *row_sees;   // [tiles][32] of this wavefront, draft keys: what each row of the block looks at

  struct Cursor { int u, r0, R, n_rows, b, used; };
  // request() only asks for what a block takes; everything that looks at it is in finish(), behind the work on the block before it
  struct Block { bf16x8 q[KS]; float lse; int node, rows, left; };   // rows: counting rows from r0 on; left: keys of the slot that the user uses
  struct Ready { bf16x8 ext; unsigned ok; };

  __device__ __forceinline__ Rows(const Args &args, const Entry &e, int g_, int lane_, unsigned long long *sees)
      : a(args), g(g_), lane(lane_), l32(lane_ & 31), g2(lane_ >> 5), G(args.Hq / args.Hkv), row_sees(sees) {
    set(e);
  }
  __device__ __forceinline__ void set(const Entry &e) {
    ent = e;
    is_draft = e.slot < 0;
    longest = e.keys >> 5;
    n_users = 1;
    place = 0;
    list = nullptr;
    if (ent.user < 0) {
      list = a.users + (-1 - ent.user);
      n_users = __builtin_amdgcn_readfirstlane(list->query);
      place = __builtin_amdgcn_readfirstlane(list->used);
      ++list;
    }
  }
  __device__ __forceinline__ void look(Cursor &c) const {
    if (list) {
      const User user = list[c.u];
      c.b = __builtin_amdgcn_readfirstlane(user.query);
      c.used = __builtin_amdgcn_readfirstlane(user.used);
      c.n_rows = __builtin_amdgcn_readfirstlane(user.rows);
    } else {
      c.b = ent.user;
      c.used = longest;
      c.n_rows = a.n_path ? __builtin_amdgcn_readfirstlane(a.n_path[c.b]) : a.T;
    }
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
  __device__ __forceinline__ Cursor behind(Cursor c) const {
    c.r0 += 32;
    settle(c);
    return c;
  }
  // the node of a lane's row (with paths: a load of its own, which request() waits for)
  __device__ __forceinline__ int node_of(const Cursor &c) const {
    const int row = min(c.r0 + l32, c.R - 1), j = row % c.n_rows;
    return a.n_path ? a.path[(size_t)c.b * a.max_path + j] : j;
  }
  __device__ __forceinline__ void request(const Cursor &c, int i, Block &blk) const {
    const int h = min(c.r0 + l32, c.R - 1) / c.n_rows;
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
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(blk.q[ks], key(kb, ks), s[kb], 0, 0, 0);
    // (the log-sum-exp last: ahead of the others, every step would be rounded at its size)
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(r.ext, ones, s[kb], 0, 0, 0);
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
  // where a tile's sums go, and whether what stands there is added to
  __device__ __forceinline__ bool adds() const { return !is_draft && !place && a.w_in; }
  __device__ __forceinline__ float *sums_at(int t0) const {
    if (place) return a.parts + ((size_t)(place - 1) + (size_t)g * ((longest + kKvTile - 1) / kKvTile) + t0 / kKvTile) * kKvTile + lane;
    return (is_draft ? a.w_draft : a.w_out) + weight_at(t0);
  }
  // the row of a key, bf16 and (8-bit slots) codes
  __device__ __forceinline__ bool is8(int fmt) const { return fmt != 0 && !is_draft && (fmt == 1 || ent.slot >= a.n_slots16); }
  __device__ __forceinline__ const __bf16 *keys16() const {
    return is_draft ? a.k_draft + ((size_t)(-1 - ent.slot) * a.Hkv + g) * a.T * D : a.k16 + ((size_t)ent.slot * a.Hkv + g) * a.C * D;
  }
  __device__ __forceinline__ size_t head8() const { return (size_t)(ent.slot - a.n_slots16) * a.Hkv + g; }
};

// Few rows: one wavefront walks a share of all tiles with the keys in registers, the next tile's requested ahead -- across the end of an entry, too
// --, and its rows -- where they are one block -- loaded once for all tiles of a query.  The shares are equal, so that all end together: a tile
// counts as one, or as what its blocks of rows make of it (Entry::keys), and belongs to the share that it starts in.  Up to 2 wavefronts a SIMD, each
// with 16 KB on the way.  FMT: 0 bf16 slots, 1 8-bit slots, 2 both. 8 queries, 15 rows of a kv head (24 heads over 8) over 12.4k keys each, one chunk
// shared: 195 MB in 37.5 us (5.2 TB/s); 48.6 with the keys loaded as operands and with pieces of at most six tiles of one slot.
template <int D, int FMT>
__global__ __launch_bounds__(64, 2) void weights_stream_kernel(const Args a) {
  constexpr int KS = D / 16;
  __shared__ __align__(16) char stage[kKvTile * D * 2];
  __shared__ __align__(16) unsigned long long row_sees[32];
  const int lane = threadIdx.x, g = blockIdx.x % a.Hkv, lo = blockIdx.x / a.Hkv * a.share, hi = lo + a.share;
  // the first tile that starts in [lo, hi)
  int e = find_entry(a, lo, lane);
  if (e < 0) return;
  auto entry = [&](int at) __attribute__((always_inline)) {
    const int4 w = ((const int4 *)a.entries)[at];
    return Entry{w.x, w.y, w.z, w.w};
  };
  auto tiles_of = [](const Entry &x) __attribute__((always_inline)) { return ((x.keys >> 5) + kKvTile - 1) / kKvTile; };
  auto end_of = [&](const Entry &x) __attribute__((always_inline)) { return min(tiles_of(x), (hi - x.piece0 + (x.keys & 31) - 1) / (x.keys & 31)); };   // behind its tiles in here
  Entry ent = entry(e);
  int tile = (lo - ent.piece0 + (ent.keys & 31) - 1) / (ent.keys & 31);
  if (tile >= tiles_of(ent)) {
    if (++e >= a.n_entries) return;
    ent = entry(e);
    tile = 0;
  }
  int tile_end = end_of(ent);
  if (tile >= tile_end) return;
  Rows<D> rows(a, ent, g, lane, row_sees);
  // A tile comes through LDS: instruction i of its request fills bytes [1024 i, +1024), 16-byte chunks XOR-swizzled inside the rows.  (Loaded as
  // operands, 32 bytes of 32 rows an instruction, a line passes the first-level cache four times: 16 KB of each of 8 wavefronts do not stay in it.)
  auto swz = [](int row_bytes, int row) __attribute__((always_inline)) { return row_bytes == 256 ? (row & 15) : row_bytes == 128 ? ((row >> 1) & 7) : ((row >> 2) & 3); };
  float next_scale = 1.f;
  auto copy = [&](const char *src, auto row_bytes_c, int rows_there) __attribute__((always_inline)) {
    constexpr int RB = decltype(row_bytes_c)::value, LPR = RB / 16, ROWS = 64 / LPR;   // lanes of a row, rows of an instruction
    const int row = lane / LPR, c = lane % LPR;
    auto fill = [&](int i, int from) __attribute__((always_inline)) {
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(src + (unsigned)from), (__attribute__((address_space(3))) void *)(stage + i * 1024), 16, 0, 2);
    };
    if (rows_there >= kKvTile) {
      int base = row * RB + (c ^ swz(RB, row)) * 16;   // (i ROWS reaches the swizzle's upper bits alone)
      asm volatile("" : "+v"(base));                   // (the addresses do not stay in registers over the tiles)
#pragma unroll
      for (int i = 0; i < kKvTile / ROWS; ++i) fill(i, i * 1024 + (base ^ (swz(RB, i * ROWS) * 16)));
    } else {
#pragma unroll 1
      for (int i = 0; i < kKvTile / ROWS; ++i) fill(i, min(i * ROWS + row, rows_there - 1) * RB + (c ^ swz(RB, i * ROWS + row)) * 16);
    }
  };
  // (a slot's block is there to its end, whatever stands behind the used length: no key's sum looks at another key.  Behind the draft keys there is nothing.)
  auto request_keys = [&](const Entry &of, int tile) __attribute__((always_inline)) {
    const int t0 = tile * kKvTile;
    if (FMT != 0 && of.slot >= 0 && (FMT == 1 || of.slot >= a.n_slots16)) {
      const size_t head = (size_t)(of.slot - a.n_slots16) * a.Hkv + g;
      next_scale = a.k_scale[head * (a.C / kKvTile) + tile];
      copy((const char *)(a.k8 + (head * a.C + t0) * D), std::integral_constant<int, D>{}, kKvTile);
    } else {
      const __bf16 *base = of.slot < 0 ? a.k_draft + ((size_t)(-1 - of.slot) * a.Hkv + g) * a.T * D : a.k16 + ((size_t)of.slot * a.Hkv + g) * a.C * D;
      copy((const char *)(base + (size_t)t0 * D), std::integral_constant<int, D * 2>{}, of.slot < 0 ? a.T - t0 : kKvTile);
    }
  };
  request_keys(ent, tile);
  typename Rows<D>::Cursor first, at;
  typename Rows<D>::Block blk;
  typename Rows<D>::Ready ready;
  // (a tile's sums are written under the next one's: before its own keys' wait they would be waited for)
  float *left_at = nullptr, left_sum = 0.f;
  auto put = [&]() __attribute__((always_inline)) { if (left_at) *left_at = left_sum; };
  // Rows are waited for where they are asked for: where the branches meet, the wait would be for everything, the next tile's keys among it.
  auto arrived = [](typename Rows<D>::Block &x) __attribute__((always_inline)) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(x.q[ks]));
  };
  bool same = false;   // the rows held are the entry's first block
  while (true) {
    // (the entry behind this one, looked up early)
    const bool more = e + 1 < a.n_entries;
    const Entry next = entry(more ? e + 1 : e);
    const int next_end = more && next.piece0 < hi ? end_of(next) : 0;
    const int longest = rows.longest;
    const bool is8 = rows.is8(FMT);
    if (!same) {
      first = at = rows.begin(0);
      if (!rows.done(at)) {
        rows.request(at, rows.node_of(at), blk);
        ready = rows.finish(blk, tile, 1);
        arrived(blk);
      }
    } else {
      blk.left = longest;
    }
    bool fresh = true;   // blk is the first block, of this tile
    for (; tile < tile_end; ++tile) {
      const int t0 = tile * kKvTile;
      const float scale = next_scale;
      __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
      asm volatile("" ::: "memory");
      bf16x8 k[2][KS];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const int row = kb * 32 + rows.l32;
          if (FMT != 0 && is8) {
            typedef unsigned u32x2 __attribute__((ext_vector_type(2)));   // (not the struct uint2: its loads are taken to alias the direct loads into LDS)
            const u32x2 w = *(const u32x2 *)(stage + row * D + ((ks ^ swz(D, row)) * 16) + rows.g2 * 8);
            k[kb][ks] = codes8(make_uint2(w[0], w[1]), scale);
          } else {
            k[kb][ks] = *(const bf16x8 *)(stage + row * (D * 2) + (((2 * ks + rows.g2) ^ swz(D * 2, row)) * 16));
          }
        }
      __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0): the stage is free
      asm volatile("" ::: "memory");
      put();
      const bool mine = t0 + lane < longest;
      float before = 0.f;   // (asked for ahead of the next keys: it is waited for first)
      if (mine && rows.adds()) before = a.w_in[rows.weight_at(t0)];
      if (tile + 1 < tile_end) request_keys(ent, tile + 1);
      else if (next_end > 0) request_keys(next, 0);
      float acc[2][2] = {{0.f, 0.f}, {0.f, 0.f}};
      auto key = [&](int kb, int ks) __attribute__((always_inline)) { return k[kb][ks]; };
      if (!rows.done(first)) {
        if (!fresh && (rows.is_draft || at.u != first.u || at.r0 != first.r0)) {
          rows.request(first, rows.node_of(first), blk);
          ready = rows.finish(blk, tile, 1);
          arrived(blk);
        }
        at = first;
        typename Rows<D>::Cursor nx = rows.behind(at);
        int node = 0;
        if (!rows.done(nx)) node = rows.node_of(nx);
        while (true) {   // the next block's rows are on the way during a block's products, and the nodes of the one behind it
          typename Rows<D>::Block ahead;
          const bool more_rows = !rows.done(nx);
          typename Rows<D>::Cursor nx2 = nx;
          int node2 = 0;
          if (more_rows) {
            rows.request(nx, node, ahead);
            nx2 = rows.behind(nx);
            if (!rows.done(nx2)) node2 = rows.node_of(nx2);
          }
          rows.pay(key, blk, ready, t0, 0, acc);
          if (!more_rows) break;
          arrived(ahead);
          blk = ahead;
          ready = rows.finish(blk, tile, 1);
          at = nx;
          nx = nx2;
          node = node2;
        }
      }
      fresh = false;
      left_sum = before + rows.total(acc);
      left_at = mine ? rows.sums_at(t0) : nullptr;
    }
    if (next_end <= 0) break;
    // one query's next slot: its rows are here already
    same = ent.user >= 0 && next.user == ent.user && !rows.is_draft && next.slot >= 0 && at.r0 == first.r0;
    ent = next;
    ++e;
    rows.set(ent);
    tile = 0;
    tile_end = next_end;
  }
  put();
}

// Many rows: a workgroup of four wavefronts keeps the keys of up to two tiles in LDS as bf16 (16-byte pieces XOR-swizzled inside rows of 256 bytes by
// row & 15, of 128 bytes by (row >> 1) & 7); the wavefronts take every fourth block of rows each.  Small pieces of work and four wavefronts a SIMD:
// while one waits for its lists, keys or rows, the others keep the vector port busy.  (Two wavefronts a SIMD with the keys in registers, or four
// tiles in LDS and the next block's rows requested ahead: 4 prompts of 256 rows x 16 heads over 3100 keys 51 and 43 us.)
template <int D, int FMT>
__global__ __launch_bounds__(256, 4) void weights_rows_kernel(const Args a) {
  constexpr int KS = D / 16, ROW = D * 2, TILE = kKvTile * ROW;
  __shared__ __align__(16) char keys[kRowsSpan * TILE];
  __shared__ __align__(16) unsigned long long row_sees[4][kRowsSpan * 32];
  __shared__ float sums[4][kRowsSpan][kKvTile];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = blockIdx.x % a.Hkv, piece = blockIdx.x / a.Hkv;
  const int4 words = ((const int4 *)a.entries)[find_entry(a, piece, lane)];
  const Rows<D> rows(a, Entry{words.x, words.y, words.z, words.w}, g, lane, row_sees[wave]);
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
    rows.request(at, rows.node_of(at), blk);
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
    *rows.sums_at(t0) = (rows.adds() ? a.w_in[rows.weight_at(t0)] : 0.f) + sum;
  }
}

// The sums of split slots, in the order of their parts.  One wavefront a (tile, kv head, slot).
__global__ __launch_bounds__(64) void weights_join_kernel(const Args a, const Split *__restrict__ splits) {
  const Split sp = splits[blockIdx.z];
  const int g = blockIdx.y, tile = blockIdx.x, key = tile * kKvTile + threadIdx.x, tiles = (sp.longest + kKvTile - 1) / kKvTile;
  if (key >= sp.longest) return;
  const float *part = a.parts + ((size_t)sp.place + (size_t)g * tiles + tile) * kKvTile + threadIdx.x;
  const size_t w_at = ((size_t)sp.slot * a.Hkv + g) * a.C + key;
  float sum = a.w_in ? a.w_in[w_at] : 0.f;
#pragma unroll 8
  for (int p = 0; p < sp.parts; ++p) sum += part[(size_t)p * a.Hkv * tiles * kKvTile];
  a.w_out[w_at] = sum;
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
  struct Slot { int32_t slot, longest, n_users, blocks, only, only_used; };
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
        slots.push_back({slot, 0, 0, 0, 0, 0});
      } else {
        several = true;
      }
      use(slots[of_slot[slot]], b, used);
    }
  }
  if (draft_weights_out_dev)
    for (int b = 0; b < batch; ++b) {
      slots.push_back({-1 - b, 0, 0, 0, 0, 0});
      use(slots.back(), b, t_draft);
    }
  if (slots.empty()) return PC_OK;
  // Many rows of a query to a key: weights_rows_kernel, in pieces of two tiles, fewer where a tile has more blocks of rows than the others; what has
  // more of them comes first. Else weights_stream_kernel, in shares of equal cost for all wavefronts that the chip holds at once (8 a CU).  A slot's
  // users are split where a tile would have more blocks of rows than `most`: as many as the others, or four more than a wavefront's share has tiles
  // (a block takes about the time of a tile, the launch that adds the sums up four).  us, 4 prompts of 256 rows (16 heads over 8) over 8 chunks of
  // 384 tokens on average, one of them shared: whole 36.8, split 27.9 and 4.0 for the sums.
  int most_rows = 0, least_blocks = INT32_MAX;
  long all_tiles = 0;
  for (int b = 0; b < batch; ++b) most_rows = std::max(most_rows, rows_of(b));
  const bool by_rows = most_rows > 64;
  const int waves = std::max(1, 8 * ctx->n_cu / c.n_kv_heads);   // (of a kv head)
  auto tiles_of = [](const Slot &sl) { return (sl.longest + kKvTile - 1) / kKvTile; };
  for (const Slot &sl : slots) {
    all_tiles += tiles_of(sl);
    if (sl.blocks) least_blocks = std::min(least_blocks, sl.blocks);
  }
  if (least_blocks == INT32_MAX) least_blocks = 1;   // (no row counts for any slot)
  const int most = by_rows ? least_blocks : (int)std::min<long>(kMostCost, all_tiles / waves + 4);
  if (several) {
    std::stable_sort(slots.begin(), slots.end(), [](const Slot &x, const Slot &y) { return x.blocks > y.blocks; });
    for (size_t e = 0; e < slots.size(); ++e)
      if (slots[e].slot >= 0) of_slot[slots[e].slot] = (int)e;
  }
  // the users of slots that have several, or one that uses less than another, none of whose rows counts
  std::vector<std::vector<std::pair<int32_t, int32_t>>> lists;
  std::vector<int32_t> list_of(slots.size(), -1);
  for (size_t e = 0; e < slots.size(); ++e)
    if (slots[e].n_users != 1 || slots[e].only_used != slots[e].longest) {
      list_of[e] = (int)lists.size();
      lists.emplace_back();
    }
  if (!lists.empty())
    for (int b = 0; b < batch; ++b) {
      const int32_t *row = rows.data() + (size_t)b * stride;
      for (int ci = 0; ci < row[0]; ++ci) {
        const int slot = row[pc::kTblHeader + 2 * ci], used = row[pc::kTblHeader + 2 * ci + 1];
        if (used != 0 && rows_of(b) != 0 && list_of[of_slot[slot]] >= 0) lists[list_of[of_slot[slot]]].push_back({b, used});
      }
    }
  const pc::DraftWs ws = pc::carve_draft_ws(c, ctx->n_cu, workspace_dev, batch, t_draft, max_chunks);
  const size_t room = (size_t)((float *)ws.part_ml - ws.part_o) / kKvTile;   // tiles' sums that the workspace holds
  std::vector<int32_t> words, splits;
  std::vector<User> users;
  words.reserve(slots.size() * 4 + (several ? (size_t)batch * max_chunks * 4 : 0) + (path_host ? (size_t)batch * (max_path + 1) : 0) + ((size_t)batch * t_draft + 1) / 2 + 2);
  long pieces = 0;
  size_t place = 0;
  int most_split = 0;
  for (size_t e = 0; e < slots.size(); ++e) {
    const Slot &sl = slots[e];
    const int tiles = tiles_of(sl);
    auto add = [&](int blocks, int32_t user) {
      const int each = by_rows ? std::max(1, std::min(kRowsSpan, kRowsSpan * least_blocks / std::max(1, blocks))) : std::min(kMostCost, (sl.slot < 0 ? kDraftCost : 1) * std::max(1, blocks));
      const int32_t w[4] = {sl.slot, (int32_t)pieces, sl.longest * 32 + each, user};
      words.insert(words.end(), w, w + 4);
      pieces += by_rows ? (tiles + each - 1) / each : tiles * each;
    };
    if (list_of[e] < 0) {
      add(sl.blocks, sl.only);
      continue;
    }
    const auto &list = lists[list_of[e]];
    // groups of users of at most `most` blocks (or of one user)
    std::vector<size_t> ends;
    std::vector<int> blocks;
    for (size_t u = 0; u < list.size(); ++u) {
      const int n = (rows_of(list[u].first) + 31) / 32;
      if (u == 0 || blocks.back() + n > most) {
        ends.push_back(u);
        blocks.push_back(0);
      }
      ends.back() = u + 1;
      blocks.back() += n;
    }
    const size_t parts = ends.size(), sums = (size_t)c.n_kv_heads * tiles;
    const bool split = parts > 1 && place + parts * sums <= room;
    if (!split) {
      ends.assign(1, list.size());
      blocks.assign(1, sl.blocks);
    } else {
      const int32_t w[4] = {sl.slot, sl.longest, (int32_t)parts, (int32_t)place};
      splits.insert(splits.end(), w, w + 4);
      most_split = std::max(most_split, tiles);
    }
    for (size_t k = 0, u = 0; k < ends.size(); ++k) {
      add(blocks[k], -1 - (int32_t)users.size());
      users.push_back({(int32_t)(ends[k] - u), split ? 1 + (int32_t)place : 0, 0, 0});
      for (; u < ends[k]; ++u) users.push_back({list[u].first, list[u].second, rows_of(list[u].first) / G, 0});
      if (split) place += sums;
    }
  }
  const int n_entries = (int)(words.size() / 4);
  if (pieces * c.n_kv_heads >= (1L << 31)) return pc::fail(ctx, PC_ESHAPE, "too many keys for one call");
  const size_t split_at = words.size();   // (16-byte aligned, as the entries)
  words.insert(words.end(), splits.begin(), splits.end());
  const size_t user_at = words.size();
  if (!users.empty()) words.insert(words.end(), &users[0].query, &users[0].query + 4 * users.size());
  const size_t n_path_at = words.size(), path_at = n_path_at + batch;
  if (path_host) {
    words.insert(words.end(), n_path_host, n_path_host + batch);
    words.insert(words.end(), path_host, path_host + (size_t)batch * max_path);
  }
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
  a.n_entries = n_entries;
  a.users = (const User *)(ws.words + user_at);
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
  a.parts = ws.part_o;
  a.draft.sees = parents ? ws.sees : nullptr;
  const int formats = pc::table_formats(rows, stride, batch), fmt = !(formats & 1) ? 0 : (formats & 2) ? 2 : 1;
  a.share = (int)((pieces + waves - 1) / waves);
  const dim3 grid((unsigned)((by_rows ? pieces : (pieces + a.share - 1) / a.share) * c.n_kv_heads));
#define PC_WEIGHTS_F(DD, FF)                                                                                         \
  do {                                                                                                               \
    if (by_rows) hipLaunchKernelGGL((weights_rows_kernel<DD, FF>), grid, dim3(256), 0, s, a);                         \
    else hipLaunchKernelGGL((weights_stream_kernel<DD, FF>), grid, dim3(64), 0, s, a);                                \
  } while (0)
#define PC_WEIGHTS(DD) do { if (fmt == 0) PC_WEIGHTS_F(DD, 0); else if (fmt == 1) PC_WEIGHTS_F(DD, 1); else PC_WEIGHTS_F(DD, 2); } while (0)
  if (c.head_dim == 128) PC_WEIGHTS(128); else PC_WEIGHTS(64);
#undef PC_WEIGHTS_F
#undef PC_WEIGHTS
  if (!splits.empty())
    hipLaunchKernelGGL(weights_join_kernel, dim3((unsigned)most_split, (unsigned)c.n_kv_heads, (unsigned)(splits.size() / 4)), dim3(64), 0, s, a, (const Split *)(ws.words + split_at));
  PC_HIP(ctx, hipGetLastError());
  return PC_OK;
}
