// Attention of packed rows: request s has T_s fresh rows, one request behind the other, and attends over [its cached chunks ; its own rows up to each]:
//   o_i = sum_j e^(s_ij - lse_i) v_j,   s_ij = q_i.k_j / sqrt(D),   lse_i = log sum_j e^s_ij.
// The arithmetic is that of reuse_attention.hip (transposed scores, bf16 matrix instructions, fp32 softmax state against a lazily refreshed reference
// exponent); what differs is how the work is cut and where the fresh keys come from:
//   - the host cuts every request into blocks of rows and, where the launch would be short of workgroups, the blocks' keys into partitions, and lists
//     them longest first.  A workgroup reads its item from the list; a call of prompts of any lengths and of single tokens is one launch.
//   - the G query heads of a kv head are stacked token by token (row = i G + g), so a block of 256 rows spans 256 / G tokens, all its wavefronts see
//     nearly the same keys, and a token's heads share the rows of a tile;
//   - a fresh tile is taken as it was projected, K and V row by row; V is turned by the LDS transpose reads on its way to the matrix instruction, so
//     there is no launch that lays it out first, and no workspace for it.
// Blocks of up to 32 rows (single tokens, short questions) share a tile by keys instead of rows: eight wavefronts, two tiles, 16 keys each.
//
// A probability is rounded to bf16 for the second product, whose fp32 form has a sixteenth of the rate; its sum is taken unrounded.  Against 64 bits the outputs are off by 0.0023 of their
// size (0.0017 with the output's own rounding alone).
//
// What a row does not see takes no part, whatever stands there: K by the mask on the scores; V behind the end of a chunk or a request by clearing the
// operand; V of a later token of the same tile, where it is not finite, by computing the rows that it made NaN once more, key by key.
//
// What bounds it: prompts the matrix products and the exponentials, whose units overlap in part only.  Head size 128, 256 workgroups of 256 rows over 129 tiles, one a CU: 3620
// cycles a tile on zeros and 3730 on random data, start and end among them, 2048 of them products (0.55 of the cycles); the clock falls from 2.45 to 1.98 GHz
// on random data.  Ten prompts of 574 to 6964 tokens, 32 heads over 8: 890 us, 1.04 PFLOP/s of the scores that count, products in 0.48 of 1.87 M cycles at 2.1 GHz (767 us at 2.4 GHz on
// zeros).  Head size 64 has half of the products and all of the exponentials: 14 heads over 2, the same prompts 246 us, 0.83 PFLOP/s, products in 0.33 of the cycles and
// vector instructions in 0.49.  Single tokens: the key stream (32 tokens over 6100 cached keys each, 700 MB: 120 us, 5.8 TB/s).  Short calls: the launch (5 prompts of 11 to 71
// tokens: 7.8 us).  256 rows a block: fewer would read every tile from LDS and memory more often, a wavefront's 32 are what its registers hold beside the scores of 64
// keys.  With 8-bit tiles at head size 128 they hold them not quite: 9 registers are spilled, none of them on the usual way of the loop.  What reads them back there, the request
// of a tile that ends early and the refresh of the reference exponent, waits for all tiles in flight.
#include <algorithm>
#include <exception>
#include <cmath>
#include <cstddef>
#include <cstring>
#include <functional>

#include "decode_common.hpp"
#include "launch_lists.hpp"

namespace {
using pc::bf16x4;
using pc::bf16x8;
using pc::f32x16;
using pc::f32x4;
using pc::kKvTile;
using pc::u32x4;
using pc::dec::codes4;
using pc::dec::codes8;
using pc::dec::fast_exp2;
using pc::dec::row_max;
using pc::dec::row_sum;
using namespace pc::packed;

constexpr int TK = kKvTile, NW = 8;
constexpr float kSumLimit = 32.f * 256.f;  // 32 probabilities of a lane and tile, each at most 2^8 against the reference
constexpr float kSumLimit4 = 4.f * 256.f;  // 4 of them
constexpr int kMaxPackedSplits = 64;
constexpr int kMoreItems = 16;             // items beyond one a block, per CU

static_assert(sizeof(ArgsAndWords) <= 4096, "the arguments of a launch");
__device__ __forceinline__ const int32_t *words_of_launch() {
  return (const int32_t *)((const char *)__builtin_amdgcn_kernarg_segment_ptr() + offsetof(ArgsAndWords, words));
}

// token (of its request) and query head of a block's row
struct RowAt { int i, head; };
template <class Block>
__device__ __forceinline__ RowAt row_at(const Args &a, const Block &b, int gkv, int local) {
  const int G = a.Hq / a.Hkv, x = b.rem0 + local, q = G == 1 ? x : (int)__umulhi((unsigned)x, a.per_group);
  return {b.i0 + q, gkv * G + x - q * G};
}

// A stage of LDS: a K tile [64][D], rows swizzled by 16-byte chunks, then V: a block [D][64] of the store or, fresh, rows [64][D].
template <int D>
struct Lds {
  static constexpr int K_ROW = D * 2, VB_ROW = TK * 2;
  static constexpr int HALF = TK * D * 2, STAGE = 2 * HALF, NSTAGE = 4;
  static constexpr int O_ROW = D + 4;                                                        // narrow: floats per output row of a wavefront
  static constexpr int MERGE = NW * kNarrowRows * (O_ROW + 2) * 4 + NW * 4;
  static constexpr int BYTES = NSTAGE * STAGE > MERGE ? NSTAGE * STAGE : MERGE;
};
__device__ __forceinline__ int swz(int row_bytes, int row) { return row_bytes == 256 ? (row & 15) : row_bytes == 128 ? ((row >> 1) & 7) : ((row >> 2) & 3); }
// fresh V rows: pairs of chunks stay together, so that the four rows of a transpose read lie in different banks
__device__ __forceinline__ int swz_tr(int row_bytes, int row) { return row_bytes == 256 ? (row & 7) << 1 : ((row >> 1) & 3) << 1; }

#define PC_WAIT_VMCNT(n) __builtin_amdgcn_s_waitcnt(((n) & 0xf) | (7 << 4) | (15 << 8) | ((((n) >> 4) & 3) << 14))

__device__ __forceinline__ float pair_max(float x) { return fmaxf(x, __shfl_xor(x, 32, 64)); }
__device__ __forceinline__ float pair_sum(float x) { return x + __shfl_xor(x, 32, 64); }

__device__ __forceinline__ bf16x8 codes16(unsigned w0, unsigned w1, float scale) { return codes8(make_uint2(w0, w1), scale); }

// four keys of one head-dim index for every lane, from four rows of 16 lanes' 4 x 16 elements (lane i of 16 names row i / 4, elements 4 (i % 4) .. +3,
// and gets element i of the four rows)
__device__ __forceinline__ bf16x4 read_turned(const char *p) {
  typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;
  return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p));
}
// what is left of four bf16 numbers when only the first `left` stay
__device__ __forceinline__ uint2 keep_first(int left) {
  return make_uint2((left > 0 ? 0xffffu : 0u) | (left > 1 ? 0xffff0000u : 0u), (left > 2 ? 0xffffu : 0u) | (left > 3 ? 0xffff0000u : 0u));
}
__device__ __forceinline__ bf16x4 cleared(bf16x4 v, uint2 keep) {
  const uint2 w = __builtin_bit_cast(uint2, v);
  return __builtin_bit_cast(bf16x4, make_uint2(w.x & keep.x, w.y & keep.y));
}
__device__ __forceinline__ bf16x8 cleared(bf16x8 v, uint2 lo, uint2 hi) {
  const u32x4 w = __builtin_bit_cast(u32x4, v);
  return __builtin_bit_cast(bf16x8, (u32x4){w[0] & lo.x, w[1] & lo.y, w[2] & hi.x, w[3] & hi.y});
}
// acc + 0 * v: NaN if one of them is not finite
__device__ __forceinline__ float taint(unsigned two, float acc) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), bf16x2{(__bf16)0.f, (__bf16)0.f}, acc, false);
}

// 16 bytes a lane from src + off to LDS: lane l's to address to + 16 l.  Written out because the compiler would make every transpose read behind it wait
// for all requests in flight; what is read from LDS is waited for where the stages change hands (PC_WAIT_VMCNT).  (m0 is the compiler's own only around
// instructions that need it, of which this file has no others; the wait states are those between a vector instruction that writes a scalar register and
// a memory instruction that reads it.)
template <bool ONCE>   // ONCE: read by this workgroup only, not kept in the caches
__device__ __forceinline__ void to_lds(const char *src, unsigned off, unsigned to) {
  // (all lanes' alike, which a compiler that optimises less does not see)
  const unsigned long at = (unsigned long)src;
  src = (const char *)((unsigned long)(unsigned)__builtin_amdgcn_readfirstlane((int)(at >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)at));
  to = __builtin_amdgcn_readfirstlane((int)to);
  if (ONCE) asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2 nt" : : "s"(to), "v"(off), "s"(src) : "memory");
  else asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(to), "v"(off), "s"(src) : "memory");
}

struct Tile { const char *k, *v; int valid, t0; bool is8; float ks, vs; };   // t0: first fresh token, -1 for a cached tile

// The walk over an item's tiles; every wavefront steps its own, in scalar registers.  Lane c keeps (slot, used length) of entry c of the 64 at hand.
template <int D, bool KV8>
struct Walk {
  const Args &a;
  const Item &it;
  int gkv, lane, my_slot = 0, my_used = 0, ent = 0, left = 0, at = 0, idx = 0;
  const char *ck = nullptr, *cv = nullptr;
  bool c8 = false;
  size_t sc = 0;
  __device__ __forceinline__ Walk(const Args &a_, const Item &it_, int gkv_, int lane_) : a(a_), it(it_), gkv(gkv_), lane(lane_) {
    load();
    if (it.n_cached > 0) {
      enter(it.slot0, it.used0);
      skip(it.tile0);
    }
  }
  __device__ __forceinline__ void load() {   // the 64 entries from ent on (of other requests behind the last one's)
    my_slot = my_used = 0;
    if (it.ent + ent + lane < a.n_ents) {
      const int2 e = *(const int2 *)(a.words + a.ents_at + 2 * (it.ent + ent + lane));
      my_slot = e.x;
      my_used = e.y;
    }
  }
  __device__ __forceinline__ void enter(int slot, int used) {
    left = used;
    at = 0;
    c8 = KV8 && slot >= a.n_slots16;
    const size_t sh = (size_t)(c8 ? slot - a.n_slots16 : slot) * a.Hkv + gkv, base = sh * a.C * D;
    ck = c8 ? (const char *)a.k8 + base : (const char *)a.k16 + base * 2;
    cv = c8 ? (const char *)a.v8 + base : (const char *)a.v16 + base * 2;
    sc = sh * (a.C / TK);
  }
  __device__ __forceinline__ void skip(int n) {
    const size_t bytes = (size_t)n * TK * D * (c8 ? 1 : 2);
    ck += bytes;
    cv += bytes;
    at += n;
    left -= n * TK;
  }
  __device__ __forceinline__ int n() const { return it.n_cached + it.f1 - it.f0; }
  __device__ __forceinline__ Tile next() {
    Tile t;
    t.ks = t.vs = 1.f;
    if (idx < it.n_cached) {
      t.k = ck;
      t.v = cv;
      t.valid = min(TK, left);
      t.t0 = -1;
      t.is8 = c8;
      if (KV8 && c8) {
        // (scalar loads: vector ones would be waited for together with the tiles requested behind them)
        typedef const __attribute__((address_space(4))) float *scalar;
        t.ks = ((scalar)a.k_scale)[sc + at];
        t.vs = ((scalar)a.v_scale)[sc + at];
      }
      skip(1);
      if (left <= 0 && idx + 1 < it.n_cached) {
        ++ent;
        if ((ent & 63) == 0) load();
        enter(__builtin_amdgcn_readlane(my_slot, ent & 63), __builtin_amdgcn_readlane(my_used, ent & 63));
      }
    } else {
      const int f = it.f0 + idx - it.n_cached;
      const size_t at_row = ((size_t)gkv * a.N + it.row0 + (size_t)f * TK) * (D * 2);
      t.k = (const char *)a.k + at_row;
      t.v = (const char *)a.v + at_row;
      t.valid = min(TK, it.T - f * TK);
      t.t0 = f * TK;
      t.is8 = false;
    }
    ++idx;
    return t;
  }
};

// One row of an item once more, key by key, by one wavefront: what the row does not see is not touched.  Rows that need it are those of a tile in which a
// later token's V is not finite.  Their probabilities stay in 32 bits, so they are not, to the last bit, what they are beside finite rows, and nearer to the exact ones.
template <int D, bool KV8>
__device__ __forceinline__ void redo_row(const Args &a, const Item &it, int gkv, int lane, int local, float &m_out, float &l_out, float (&o)[D / 64]) {
  constexpr int E = D / 64;
  const auto [i, head] = row_at(a, it, gkv, local);
  float q[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    q[e] = (float)a.q[((size_t)head * a.N + it.row0 + i) * D + e * 64 + lane];
    o[e] = 0.f;
  }
  float m = -INFINITY, l = 0.f;
  Walk<D, KV8> walk(a, it, gkv, lane);
  for (int t = 0; t < walk.n(); ++t) {
    const Tile x = walk.next();
    const int n = x.t0 < 0 ? x.valid : min(x.valid, i - x.t0 + 1);
    for (int key = 0; key < n; ++key) {
      float kx[E], vx[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int d = e * 64 + lane;
        if (KV8 && x.is8) {
          kx[e] = __builtin_amdgcn_cvt_f32_fp8((int)((const uint8_t *)x.k)[key * D + d], 0) * x.ks;
          vx[e] = __builtin_amdgcn_cvt_f32_fp8((int)((const uint8_t *)x.v)[d * TK + pc::blocked_pos8(key)], 0) * x.vs;
        } else {
          kx[e] = (float)((const __bf16 *)x.k)[key * D + d];
          vx[e] = (float)((const __bf16 *)x.v)[x.t0 < 0 ? d * TK + (key & ~15) + pc::blocked_key(key & 15) : key * D + d];
        }
      }
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) s += q[e] * kx[e];
      s = pc::dec::wave_sum(s) * a.scale_log2e;
      const float top = fmaxf(m, s), w = m == -INFINITY ? 0.f : fast_exp2(m - top), p = s == -INFINITY ? 0.f : fast_exp2(s - top);
      m = top;
      l = l * w + p;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = o[e] * w + p * vx[e];
    }
  }
  m_out = m;
  l_out = l;
  const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] *= inv;
}
template <int D, bool KV8>
__device__ __forceinline__ void redo_and_write(const Args &a, const Item &it, int gkv, int lane, int local) {
  float m, l, o[D / 64];
  redo_row<D, KV8>(a, it, gkv, lane, local, m, l, o);
  const auto [i, head] = row_at(a, it, gkv, local);
  if (it.part < 0) {
#pragma unroll
    for (int e = 0; e < D / 64; ++e) a.out[((size_t)it.row0 + i) * ((size_t)a.Hq * D) + (size_t)head * D + e * 64 + lane] = (__bf16)o[e];
    if (a.lse && lane == 0) a.lse[(size_t)head * a.N + it.row0 + i] = pc::lse_of(m, l);
  } else {
    const size_t prow = (size_t)gkv * a.part_rows + it.part + local;
#pragma unroll
    for (int e = 0; e < D / 64; ++e) a.part_o[prow * D + e * 64 + lane] = o[e];
    if (lane == 0) *(float2 *)(a.part_ml + prow * 2) = make_float2(m, l);
  }
}

// ---- up to 256 rows: a wavefront 32 of them, all wavefronts every tile
template <int D, bool KV8>
__device__ __forceinline__ void wide_item(const Args &a, const Item &it, int gkv, char *lds) {
  using L = Lds<D>;
  constexpr int NLD = 4, NSTAGE = 3, KS = D / 16, DB = D / 32, INSTR = L::HALF / 1024 / NLD;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, g2 = lane >> 5;

  const int local = wave * 32 + l32;
  const bool row_ok = local < it.rows();
  const RowAt mine = row_at(a, it, gkv, min(local, it.rows() - 1));
  const int my_i = mine.i, head = mine.head;
  // first and last token among this wavefront's rows: a fresh tile that reaches past the first is masked, one that starts behind the last skipped
  const bool wave_live = wave * 32 < it.rows();
  const int i_lo = __builtin_amdgcn_readlane(my_i, 0), i_hi = __builtin_amdgcn_readlane(my_i, 31);

  bf16x8 qf[KS];
  {
    const __bf16 *qrow = a.q + ((size_t)head * a.N + it.row0 + my_i) * D;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *(const bf16x8 *)(qrow + ks * 16 + g2 * 8);
  }
  f32x16 o_acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int x = 0; x < 16; ++x) o_acc[db][x] = 0.f;
  float m_ref = -INFINITY, l_run = 0.f, tainted = 0.f;
  bool all_started = false;

  Walk<D, KV8> walk(a, it, gkv, lane);
  const int n = walk.n();

  // ---- requests: wavefronts 0..3 bring in a bf16 tile, instruction i of a half its bytes [1024 i, +1024).  The rows of a wavefront's instructions are 16 (of
  // 256 bytes; of 128 bytes 32) apart and swizzled alike: one offset for all of them, the distance goes into the scalar base.
  constexpr int APART = NLD * 1024;
  static_assert(APART % (16 * 256) == 0, "the instructions' rows are swizzled alike");
  unsigned k_off, vb_off, vf_off;
  {
    const int byte = (wave & (NLD - 1)) * 1024 + lane * 16;
    const int row = byte / L::K_ROW, pc = byte % L::K_ROW / 16, d = byte / L::VB_ROW, pd = byte % L::VB_ROW / 16;
    k_off = row * L::K_ROW + (pc ^ swz(L::K_ROW, row)) * 16;
    vf_off = row * L::K_ROW + (pc ^ swz_tr(L::K_ROW, row)) * 16;
    vb_off = d * L::VB_ROW + (pd ^ swz(L::VB_ROW, d)) * 16;
  }
  const unsigned lds_base = (unsigned)(size_t)(__attribute__((address_space(3))) char *)lds;
  auto request = [&](const Tile &t, int st) __attribute__((always_inline)) {
    const unsigned kb = lds_base + st * L::STAGE + (wave & (NLD - 1)) * 1024, vb = kb + L::HALF;
    if (__builtin_expect(t.valid < TK, 0)) {   // rows past the end repeat the last valid one (masked later); a block of the store is there as a whole
      const int last = t.valid - 1;
#pragma unroll
      for (int j = 0; j < INSTR; ++j) {
        const unsigned ko = k_off + j * APART, vo = vf_off + j * APART;
        to_lds<false>(t.k, min((int)(ko / L::K_ROW), last) * L::K_ROW + ko % L::K_ROW, kb + j * APART);
        to_lds<false>(t.v, t.t0 < 0 ? vb_off + j * APART : min((int)(vo / L::K_ROW), last) * L::K_ROW + vo % L::K_ROW, vb + j * APART);
      }
      return;
    }
    const unsigned v_off = t.t0 < 0 ? vb_off : vf_off;
#pragma unroll
    for (int j = 0; j < INSTR; ++j) to_lds<false>(t.k + j * APART, k_off, kb + j * APART);
#pragma unroll
    for (int j = 0; j < INSTR; ++j) to_lds<false>(t.v + j * APART, v_off, vb + j * APART);
  };
  // 8-bit tiles: codes through registers, 16 of K and of V a thread (D = 64: of the first half of the threads), turned into a bf16 tile one tile
  // ahead of the arithmetic.  The stores are ones that the compiler does not see, for which it would wait for every request in flight.
  constexpr bool ALL = TK * D / 16 == 64 * NW;
  const bool conv = KV8 && (ALL || tid < TK * D / 16);
  const int ck_row = tid * 16 / D, ck_c = tid * 16 % D / 16, cv_row = tid >> 2, cv_m = tid & 3;
  u32x4 kc = {0, 0, 0, 0}, vc = {0, 0, 0, 0};
  auto load_codes = [&](const Tile &t) __attribute__((always_inline)) {
    if (!conv) return;
    kc = *(const u32x4 *)(t.k + min(ck_row, t.valid - 1) * D + ck_c * 16);
    vc = *(const u32x4 *)(t.v + cv_row * TK + cv_m * 16);
  };
  auto store16 = [&](int off, bf16x8 x) __attribute__((always_inline)) {
    const unsigned addr = lds_base + (unsigned)off;
    asm volatile("ds_write_b128 %0, %1" : : "v"(addr), "v"(x) : "memory");
  };
  auto land_codes = [&](const Tile &t, int st) __attribute__((always_inline)) {
    if (!conv) return;
    const int kb = st * L::STAGE + ck_row * L::K_ROW, vb = st * L::STAGE + L::HALF + cv_row * L::VB_ROW, sk = swz(L::K_ROW, ck_row), sv = swz(L::VB_ROW, cv_row);
    store16(kb + ((2 * ck_c) ^ sk) * 16, codes16(kc[0], kc[1], t.ks));
    store16(kb + ((2 * ck_c + 1) ^ sk) * 16, codes16(kc[2], kc[3], t.ks));
    // (bytes 32 J + 16 a + .. of a row of codes: its first 8 are the keys of bf16 chunk 4 J + a, its last 8 those of chunk 4 J + 2 + a)
    store16(vb + ((4 * (cv_m >> 1) + (cv_m & 1)) ^ sv) * 16, codes16(vc[0], vc[1], t.vs));
    store16(vb + ((4 * (cv_m >> 1) + 2 + (cv_m & 1)) ^ sv) * 16, codes16(vc[2], vc[3], t.vs));
  };

  // Operand reads: chunk 2 j + g2 of row l32, swizzled, for j = 0, 1, ...: the first one's address with j in bits 5 and up the other way round.  Kept, or, where
  // registers are short (a tile of codes in flight), formed at each read.
  const int k_rd0 = (g2 ^ swz(L::K_ROW, l32)) * 16 + l32 * L::K_ROW, vb_rd0 = (g2 ^ swz(L::VB_ROW, l32)) * 16 + l32 * L::VB_ROW;
  int vf_rd[DB];
  {
    const int key = 4 * g2 + ((l32 & 15) >> 2);
#pragma unroll
    for (int db = 0; db < DB; ++db) vf_rd[db] = key * L::K_ROW + ((db * 4 + (l32 >> 4) * 2 + ((l32 >> 1) & 1)) ^ swz_tr(L::K_ROW, key)) * 16 + (l32 & 1) * 8;
  }

  auto tile = [&](int st, const Tile &t, auto fresh_c) __attribute__((always_inline)) {
    constexpr bool FRESH = decltype(fresh_c)::value;
    const char *kb = lds + st * L::STAGE, *vb = kb + L::HALF;
    int k_rd = k_rd0, vb_rd = vb_rd0;
    if (KV8) asm volatile("" : "+v"(k_rd), "+v"(vb_rd));
    f32x16 s_acc[2];
#pragma unroll
    for (int kbk = 0; kbk < 2; ++kbk)
#pragma unroll
      for (int x = 0; x < 16; ++x) s_acc[kbk][x] = 0.f;
#pragma unroll
    for (int h = 0; h < KS / 4; ++h) {
      bf16x8 kop[2][4];
#pragma unroll
      for (int k4 = 0; k4 < 4; ++k4)
#pragma unroll
        for (int kbk = 0; kbk < 2; ++kbk) kop[kbk][k4] = *(const bf16x8 *)(kb + kbk * 32 * L::K_ROW + (k_rd ^ (4 * h + k4) * 32));
#pragma unroll
      for (int k4 = 0; k4 < 4; ++k4)
#pragma unroll
        for (int kbk = 0; kbk < 2; ++kbk) s_acc[kbk] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kop[kbk][k4], qf[4 * h + k4], s_acc[kbk], 0, 0, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, 8, 0);
    }
    // V operands of 16 keys: of the first 32-key block now, so that their latency runs under the softmax
    bf16x8 vop[2][DB][2];
    auto v_operands = [&](int half) __attribute__((always_inline)) {
#pragma unroll
      for (int c2 = 0; c2 < 2; ++c2)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const int c4 = 2 * half + c2;
          if constexpr (FRESH) {
            union { bf16x4 p[2]; bf16x8 v; } u;
            u.p[0] = read_turned(vb + 16 * c4 * L::K_ROW + vf_rd[db]);
            u.p[1] = read_turned(vb + (16 * c4 + 8) * L::K_ROW + vf_rd[db]);
            vop[half][db][c2] = u.v;
          } else {
            vop[half][db][c2] = *(const bf16x8 *)(vb + db * 32 * L::VB_ROW + (vb_rd ^ c4 * 32));
          }
        }
    };
    // what stands behind the last key is cleared; whether what is left is finite matters where later rows are among it
    auto clear = [&](int half) __attribute__((always_inline)) {
#pragma unroll
      for (int c2 = 0; c2 < 2; ++c2) {
        const int left = t.valid - (16 * (2 * half + c2) + 4 * g2);
        const uint2 lo = keep_first(left), hi = keep_first(left - 8);
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          vop[half][db][c2] = cleared(vop[half][db][c2], lo, hi);
          if (FRESH) {
            const u32x4 w = __builtin_bit_cast(u32x4, vop[half][db][c2]);
            tainted = taint(w[0], taint(w[1], taint(w[2], taint(w[3], tainted))));
          }
        }
      }
    };
    v_operands(0);
    const bool ragged = t.valid < TK, causal = FRESH && t.t0 + TK - 1 > i_lo;
    if (__builtin_expect(ragged || causal, 0)) {
      clear(0);
      int t_lane = g2 * 4;
      asm volatile("" : "+v"(t_lane));   // (keeps the per-element key indices out of loop-invariant registers)
      const int lim = min(t.valid - 1, FRESH ? my_i - t.t0 : TK) - t_lane;
#pragma unroll
      for (int kbk = 0; kbk < 2; ++kbk)
#pragma unroll
        for (int x = 0; x < 16; ++x) s_acc[kbk][x] = kbk * 32 + (x >> 2) * 8 + (x & 3) <= lim ? s_acc[kbk][x] : -INFINITY;
    }
    bf16x8 pf[2][2];
    auto exponentials = [&](float neg_m) __attribute__((always_inline)) {
      typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
      float sum = 0.f, sum2 = 0.f;
#pragma unroll
      for (int kbk = 0; kbk < 2; ++kbk)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            const float p0 = fast_exp2(__builtin_fmaf(s_acc[kbk][j * 8 + e], a.scale_log2e, neg_m));
            const float p1 = fast_exp2(__builtin_fmaf(s_acc[kbk][j * 8 + e + 1], a.scale_log2e, neg_m));
            const bf16x2 pr = {(__bf16)p0, (__bf16)p1};
            pf[kbk][j][e] = pr[0];
            pf[kbk][j][e + 1] = pr[1];
            sum += p0;
            sum2 += p1;
          }
      return sum + sum2;
    };
    float psum = 0.f;
    bool refresh = !all_started;
    if (__builtin_expect(!refresh, 1)) {
      psum = exponentials(-m_ref);
      refresh = __builtin_amdgcn_ballot_w64(!(psum <= kSumLimit)) != 0;   // also catches inf / nan
    }
    if (__builtin_expect(refresh, 0)) {
      float mx = s_acc[0][0];
#pragma unroll
      for (int kbk = 0; kbk < 2; ++kbk)
#pragma unroll
        for (int x = 0; x < 16; ++x) mx = fmaxf(mx, s_acc[kbk][x]);
      const float mc = pair_max(mx) * a.scale_log2e;
      const bool upd = mc > m_ref;
      const float alpha = upd ? fast_exp2(m_ref - mc) : 1.0f;
      m_ref = upd ? mc : m_ref;
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int x = 0; x < 16; ++x) o_acc[db][x] *= alpha;
      psum = exponentials(m_ref == -INFINITY ? 0.f : -m_ref);
      all_started = __builtin_amdgcn_ballot_w64(m_ref == -INFINITY) == 0;
    }
    l_run += psum;
    v_operands(1);
    if (__builtin_expect(ragged || causal, 0)) clear(1);
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int c2 = 0; c2 < 2; ++c2)
#pragma unroll
        for (int db = 0; db < DB; ++db) o_acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vop[half][db][c2], pf[half][c2], o_acc[db], 0, 0, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, (FRESH ? 4 : 2) * DB, 1);
    __builtin_amdgcn_sched_group_barrier(0x008, 4 * DB, 1);
  };

  // ---- pipeline: tile t is computed from stage t % 3 while tiles t+1 and t+2 are on their way.  At the end of iteration t every wavefront waits for
  // what it has in flight (its share of tile t+1; codes of t+1, which it then turns into their stage), and tile t+2 is requested into the stage
  // that iteration t-1 read; the barrier publishes tile t+1.
  Tile cur = {}, nxt = {}, aft = {};
  auto bring = [&](Tile &t, int st, auto codes_c) __attribute__((always_inline)) {
    t = walk.next();
    if (decltype(codes_c)::value && t.is8) load_codes(t);
    else if (wave < NLD) request(t, st);
  };
  const std::bool_constant<KV8> codes;
  bring(cur, 0, codes);
  if (KV8 && cur.is8) land_codes(cur, 0);
  if (n > 1) bring(nxt, 1, codes);
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[ks]));
  __builtin_amdgcn_s_waitcnt(0);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  // (two loops, one after the other: with both kinds of tiles in one the compiler runs out of registers)
  int st = 0, t = 0;
  auto step = [&](auto codes_c) __attribute__((always_inline)) {
    const int s1 = st + 1 == NSTAGE ? 0 : st + 1, s2 = s1 + 1 == NSTAGE ? 0 : s1 + 1;
    PC_WAIT_VMCNT(0);
    if (decltype(codes_c)::value && t + 1 < n && nxt.is8) {
      land_codes(nxt, s1);
      __builtin_amdgcn_s_waitcnt(0xc07f);   // (lgkmcnt 0)
    }
    if (t + 2 < n) bring(aft, s2, codes_c);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    cur = nxt;
    nxt = aft;
    st = s1;
  };
  for (; t < it.n_cached; ++t) {
    if (wave_live) tile(st, cur, std::false_type{});
    step(codes);
  }
  for (; t < n; ++t) {
    if (wave_live && cur.t0 <= i_hi) tile(st, cur, std::true_type{});
    step(std::false_type{});
  }
  if (!wave_live) return;

  const float l_tot = pair_sum(l_run), inv = l_tot == 0.f ? 0.f : 1.0f / l_tot;
  unsigned again = 0;   // rows whose sums a later token's V has spoilt
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(tainted == 0.f)) != 0, 0)) {
    float bad = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int x = 0; x < 16; ++x) bad += o_acc[db][x] * 0.f;
    const unsigned long long b = __builtin_amdgcn_ballot_w64(row_ok && !(bad == 0.f));
    again = (unsigned)b | (unsigned)(b >> 32);
  }
  if (row_ok && !(again >> l32 & 1)) {
    if (it.part < 0) {
      __bf16 *orow = a.out + ((size_t)it.row0 + my_i) * ((size_t)a.Hq * D) + (size_t)head * D;
      // (lane l has elements 8 x + 0..3, lane l + 32 elements 8 x + 4..7: for every two x they change halves and store 16 bytes each)
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
          uint2 w[2];
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int at = (2 * h + x) * 4;
            w[x] = __builtin_bit_cast(uint2, bf16x4{(__bf16)(o_acc[db][at] * inv), (__bf16)(o_acc[db][at + 1] * inv), (__bf16)(o_acc[db][at + 2] * inv), (__bf16)(o_acc[db][at + 3] * inv)});
          }
          const u32x2 lo = __builtin_amdgcn_permlane32_swap(w[0].x, w[1].x, false, false), hi = __builtin_amdgcn_permlane32_swap(w[0].y, w[1].y, false, false);
          *(u32x4 *)(orow + db * 32 + h * 16 + g2 * 8) = u32x4{lo[0], hi[0], lo[1], hi[1]};
        }
      if (a.lse && g2 == 0) a.lse[(size_t)head * a.N + it.row0 + my_i] = pc::lse_of(m_ref, l_tot);
    } else {
      const size_t prow = (size_t)gkv * a.part_rows + it.part + local;
      float *po = a.part_o + prow * D;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4)
          *(f32x4 *)(po + db * 32 + q4 * 8 + g2 * 4) = f32x4{o_acc[db][q4 * 4] * inv, o_acc[db][q4 * 4 + 1] * inv, o_acc[db][q4 * 4 + 2] * inv, o_acc[db][q4 * 4 + 3] * inv};
      if (g2 == 0) *(float2 *)(a.part_ml + prow * 2) = make_float2(m_ref, l_tot);
    }
  }
  while (again) {
    const int x = __builtin_ctz(again);
    again &= again - 1;
    redo_and_write<D, KV8>(a, it, gkv, lane, wave * 32 + x);
  }
}

// ---- up to 16 NR rows: two tiles at a time, wavefronts 0..3 share the first by keys, 4..7 the second; each has its own running maximum, sum and output
template <int D, bool KV8, int NR>
__device__ __forceinline__ void narrow_item(const Args &a, const Item &it, int gkv, char *lds) {
  using L = Lds<D>;
  constexpr int KS = D / 32, DB = D / 16, I16 = L::HALF / 1024 / 4, I8 = I16 / 2;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g = lane >> 4;
  const int odd = wave >> 2, kq = wave & 3;

  int my_i[NR];
  bf16x8 q[NR][KS];
#pragma unroll
  for (int x = 0; x < NR; ++x) {
    const RowAt r = row_at(a, it, gkv, min(x * 16 + l16, it.rows() - 1));
    my_i[x] = r.i;
    const __bf16 *p = a.q + ((size_t)r.head * a.N + it.row0 + r.i) * D + g * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) q[x][ks] = *(const bf16x8 *)(p + ks * 32);
  }
  f32x4 o[DB][NR];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int x = 0; x < NR; ++x) o[db][x] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_ref[NR], l_run[NR], tainted = 0.f;
#pragma unroll
  for (int x = 0; x < NR; ++x) { m_ref[x] = -INFINITY; l_run[x] = 0.f; }

  Walk<D, KV8> walk(a, it, gkv, lane);
  const int n = walk.n(), pairs = (n + 1) / 2;

  // requests: four wavefronts a tile; 8-bit tiles stay codes (K rows of D bytes, V rows of 64).  The rows of a wavefront's instructions are 4096 bytes apart
  // and swizzled alike; rows past the end repeat the last valid one (masked later).
  const unsigned lds_base = (unsigned)(size_t)(__attribute__((address_space(3))) char *)lds;
  const int byte0 = kq * 1024 + lane * 16;
  auto half = [&](const char *src, unsigned dst, auto row_bytes_c, int instr, int last_row, bool turned) __attribute__((always_inline)) {
    constexpr int RB = decltype(row_bytes_c)::value;
    const int row = byte0 / RB, c = (byte0 % RB / 16 ^ (turned ? swz_tr(RB, row) : swz(RB, row))) * 16;
#pragma unroll
    for (int j = 0; j < I16; ++j) {
      if (j >= instr) break;
      to_lds<true>(src, (unsigned)(min(row + j * (4096 / RB), last_row) * RB + c), dst + kq * 1024 + j * 4096);
    }
  };
  auto request = [&](const Tile &t, int st) __attribute__((always_inline)) {
    const unsigned dst = lds_base + st * L::STAGE;
    if (KV8 && t.is8) {
      half(t.k, dst, std::integral_constant<int, D>{}, I8, t.valid - 1, false);
      half(t.v, dst + L::HALF / 2, std::integral_constant<int, TK>{}, I8, D - 1, false);
    } else {
      half(t.k, dst, std::integral_constant<int, D * 2>{}, I16, t.valid - 1, false);
      if (t.t0 < 0) half(t.v, dst + L::HALF, std::integral_constant<int, TK * 2>{}, I16, D - 1, false);
      else half(t.v, dst + L::HALF, std::integral_constant<int, D * 2>{}, I16, t.valid - 1, true);
    }
  };
  // this wavefront's tile of the next pair; valid 0: there is none
  auto bring = [&](int pair) __attribute__((always_inline)) {
    Tile t = {}, u;
    t.valid = 0;
    if (2 * pair < n) {
      u = walk.next();
      if (!odd) t = u;
    }
    if (2 * pair + 1 < n) {
      u = walk.next();
      if (odd) t = u;
    }
    if (t.valid > 0) request(t, 2 * (pair & 1) + odd);
    return t;
  };

  auto soften = [&](f32x4 &s, int x) __attribute__((always_inline)) {
    f32x4 p;
    auto exponentials = [&](float neg_m) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 4; ++e) p[e] = fast_exp2(__builtin_fmaf(s[e], a.scale_log2e, neg_m));
      return (p[0] + p[1]) + (p[2] + p[3]);
    };
    float sum = 0.f;
    bool refresh = __builtin_amdgcn_ballot_w64(m_ref[x] == -INFINITY) != 0;
    if (!refresh) {
      sum = exponentials(-m_ref[x]);
      refresh = __builtin_amdgcn_ballot_w64(!(sum <= kSumLimit4)) != 0;
    }
    if (refresh) {
      const float mc = row_max(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]))) * a.scale_log2e;
      const bool upd = mc > m_ref[x];
      const float alpha = upd ? fast_exp2(m_ref[x] - mc) : 1.0f;
      m_ref[x] = upd ? mc : m_ref[x];
      l_run[x] *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db][x] *= alpha;
      sum = exponentials(m_ref[x] == -INFINITY ? 0.f : -m_ref[x]);
    }
    l_run[x] += sum;
    return p;
  };

  const int k_row = kq * 16 + l16;
  auto compute = [&](int st, const Tile &t) __attribute__((always_inline)) {
    if (kq * 16 >= t.valid) return;
    const char *kb = lds + st * L::STAGE;
    f32x4 s[NR];
#pragma unroll
    for (int x = 0; x < NR; ++x) s[x] = f32x4{0.f, 0.f, 0.f, 0.f};
    bf16x4 vop[DB];
    if (KV8 && t.is8) {
      const char *vb = kb + L::HALF / 2;
      uint2 raw[KS];
      unsigned vraw[DB];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) raw[ks] = *(const uint2 *)(kb + k_row * D + (((2 * ks + (g >> 1)) ^ swz(D, k_row)) * 16) + (g & 1) * 8);
      // byte p = 32 J + 16 a + 8 j + 4 c + e of a V row holds key 32 J + 16 j + 8 c + 4 a + e
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const int row = db * 16 + l16;
        vraw[db] = *(const unsigned *)(vb + row * TK + (((2 * (kq >> 1) + (g & 1)) ^ swz(TK, row)) * 16) + 8 * (kq & 1) + 4 * (g >> 1));
      }
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bf16x8 k = codes8(raw[ks], t.ks);
#pragma unroll
        for (int x = 0; x < NR; ++x) s[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[x][ks], s[x], 0, 0, 0);
      }
#pragma unroll
      for (int db = 0; db < DB; ++db) vop[db] = codes4(vraw[db], t.vs);
    } else {
      const char *vb = kb + L::HALF;
      bf16x8 kop[KS];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) kop[ks] = *(const bf16x8 *)(kb + k_row * L::K_ROW + (((4 * ks + g) ^ swz(L::K_ROW, k_row)) * 16));
      if (t.t0 < 0) {
        // (keys 4 g .. 4 g + 3 of a group of 16 sit at 8 (g & 1) + 4 (g >> 1))
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const int row = db * 16 + l16;
          vop[db] = *(const bf16x4 *)(vb + row * L::VB_ROW + (((2 * kq + (g & 1)) ^ swz(L::VB_ROW, row)) * 16) + 8 * (g >> 1));
        }
      } else {
        const int key = kq * 16 + 4 * g + (l16 >> 2);
#pragma unroll
        for (int db = 0; db < DB; ++db) vop[db] = read_turned(vb + key * L::K_ROW + ((db * 2 + ((l16 >> 1) & 1)) ^ swz_tr(L::K_ROW, key)) * 16 + (l16 & 1) * 8);
      }
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int x = 0; x < NR; ++x) s[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kop[ks], q[x][ks], s[x], 0, 0, 0);
    }
    if (t.valid < TK || (t.t0 >= 0 && t.t0 + TK - 1 > it.i0)) {
#pragma unroll
      for (int x = 0; x < NR; ++x) {
        const int lim = min(t.valid - 1, t.t0 >= 0 ? my_i[x] - t.t0 : TK) - (kq * 16 + g * 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[x][e] = e <= lim ? s[x][e] : -INFINITY;
      }
      const uint2 keep = keep_first(t.valid - kq * 16 - g * 4);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        vop[db] = cleared(vop[db], keep);
        if (t.t0 >= 0) {
          const uint2 w = __builtin_bit_cast(uint2, vop[db]);
          tainted = taint(w.x, taint(w.y, tainted));
        }
      }
    }
    typedef short s16x4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int x = 0; x < NR; ++x) {
      const f32x4 p = soften(s[x], x);
      const bf16x4 pb = {(__bf16)p[0], (__bf16)p[1], (__bf16)p[2], (__bf16)p[3]};
#pragma unroll
      for (int db = 0; db < DB; ++db)
        o[db][x] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, vop[db]), __builtin_bit_cast(s16x4, pb), o[db][x], 0, 0, 0);
    }
  };

  // ---- pipeline: pair p sits in stages 2 (p & 1) and the next.  The first barrier of an iteration says that it has landed, the second that it has been
  // read, so that its stages take pair p + 2: one to two pairs are on their way while this one is worked on.
  Tile cur = bring(0), nxt = {};
  if (pairs > 1) nxt = bring(1);
#pragma unroll
  for (int x = 0; x < NR; ++x)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(q[x][ks]));
  for (int p = 0; p < pairs; ++p) {
    // (behind this pair's requests are those of the next: of this wavefront 2 I16, 2 I8 of a tile of codes, none past the end)
    if (p + 1 >= pairs || nxt.valid == 0) PC_WAIT_VMCNT(0);
    else if (KV8 && nxt.is8) PC_WAIT_VMCNT(2 * I8);
    else PC_WAIT_VMCNT(2 * I16);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    compute(2 * (p & 1) + odd, cur);
    cur = nxt;
    if (p + 2 < pairs) {
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      nxt = bring(p + 2);
    }
  }

  // ---- merge of the eight wavefronts through LDS (by stores that the compiler does not see: it would make every operand read of this kernel wait for all
  // requests in flight)
  __syncthreads();
  const float *om = (const float *)lds, *ml = om + NW * kNarrowRows * L::O_ROW, *tl = ml + NW * kNarrowRows * 2;   // [wave][row][O_ROW], [wave][row][2], [wave]
  constexpr int VPR = D / 8;
  // (the matrix instructions' results are not waited for by what the compiler does not see)
#pragma unroll
  for (int x = 0; x < NR; ++x)
#pragma unroll
    for (int db = 0; db < DB; ++db) asm volatile("" : "+v"(o[db][x]));
  asm volatile("s_nop 15\n\ts_nop 15");
#pragma unroll
  for (int x = 0; x < NR; ++x) {
    const int row = wave * kNarrowRows + x * 16 + l16;
    const unsigned to = lds_base + (unsigned)((row * L::O_ROW + g * 4) * 4);
#pragma unroll
    for (int db = 0; db < DB; ++db) asm volatile("ds_write_b128 %0, %1 offset:%2" : : "v"(to), "v"(o[db][x]), "n"(db * 64) : "memory");
    const float l = row_sum(l_run[x]);
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    if (g == 0) asm volatile("ds_write_b64 %0, %1" : : "v"(lds_base + (unsigned)((NW * kNarrowRows * L::O_ROW + row * 2) * 4)), "v"(f32x2{m_ref[x], l}) : "memory");
  }
  {
    const float any = __builtin_amdgcn_ballot_w64(!(tainted == 0.f)) ? 1.f : 0.f;
    if (lane == 0) asm volatile("ds_write_b32 %0, %1" : : "v"(lds_base + (unsigned)((NW * kNarrowRows * (L::O_ROW + 2) + wave) * 4)), "v"(any) : "memory");
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  float spoilt = 0.f;
#pragma unroll
  for (int w = 0; w < NW; ++w) spoilt += tl[w];
  const bool any_tainted = __builtin_amdgcn_ballot_w64(spoilt != 0.f) != 0;
  for (int u0 = wave * 64; u0 < it.rows() * VPR; u0 += 64 * NW) {
    const int u = u0 + lane, row = min(u / VPR, it.rows() - 1), dv = u % VPR;
    const bool live = u < it.rows() * VPR;
    float m = -INFINITY, l = 0.f, acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const float2 *const mlr = (const float2 *)ml + row;
#pragma unroll
    for (int w = 0; w < NW; ++w) m = fmaxf(m, mlr[w * kNarrowRows].x);
    // (little code: it runs once a workgroup, from memory rather than from the instruction cache)
#pragma unroll 2
    for (int w = 0; w < NW; ++w) {
      const float2 e = mlr[w * kNarrowRows];
      const float *src = om + (w * kNarrowRows + row) * L::O_ROW + dv * 8;
      const f32x4 lo = *(const f32x4 *)src, hi = *(const f32x4 *)(src + 4);
      if (e.y == 0.f && e.x == -INFINITY) continue;   // (a wavefront that saw no key of the row)
      const float f = e.x == -INFINITY ? 1.f : fast_exp2(e.x - m);   // (a sum that is NaN without a maximum stays)
      l += e.y * f;
#pragma unroll
      for (int x = 0; x < 4; ++x) { acc[x] += lo[x] * f; acc[4 + x] += hi[x] * f; }
    }
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    float bad = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      bad += acc[e] * 0.f;
      acc[e] *= inv;
    }
    const auto [i, head] = row_at(a, it, gkv, row);
    // rows whose sums a later token's V has spoilt (a row's lanes are all in this wavefront)
    unsigned long long redo = __builtin_expect(any_tainted, 0) ? __builtin_amdgcn_ballot_w64(live && !(bad == 0.f)) : 0ull;
    const unsigned long long row_lanes = (1ull << VPR) - 1;
    if (live && !(redo >> (lane / VPR * VPR) & row_lanes)) {
      if (it.part < 0) {
        bf16x8 v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (__bf16)acc[e];
        *(bf16x8 *)(a.out + ((size_t)it.row0 + i) * ((size_t)a.Hq * D) + (size_t)head * D + dv * 8) = v;
        if (a.lse && dv == 0) a.lse[(size_t)head * a.N + it.row0 + i] = pc::lse_of(m, l);
      } else {
        const size_t prow = (size_t)gkv * a.part_rows + it.part + row;
        *(f32x4 *)(a.part_o + prow * D + dv * 8) = f32x4{acc[0], acc[1], acc[2], acc[3]};
        *(f32x4 *)(a.part_o + prow * D + dv * 8 + 4) = f32x4{acc[4], acc[5], acc[6], acc[7]};
        if (dv == 0) *(float2 *)(a.part_ml + prow * 2) = make_float2(m, l);
      }
    }
    while (redo) {
      const int first = __builtin_ctzll(redo) / VPR;
      redo &= ~(row_lanes << (first * VPR));
      redo_and_write<D, KV8>(a, it, gkv, lane, u0 / VPR + first);
    }
  }
}

template <int D, bool KV8>
__device__ __forceinline__ void packed_item(const Args &a) {
  __shared__ __align__(16) char lds[Lds<D>::BYTES];
  // (workgroup ids go round-robin over the XCDs: a kv head's items share one where there are eight heads)
  const int gkv = blockIdx.x % a.Hkv;
  Item it;   // (in scalar registers: every branch on it is the wavefront's)
  {
    int32_t w[kItemWords];
    const int32_t *src = a.words + (size_t)(blockIdx.x / a.Hkv) * kItemWords;
#pragma unroll
    for (int i = 0; i < kItemWords; ++i) w[i] = __builtin_amdgcn_readfirstlane(src[i]);
    it = __builtin_bit_cast(Item, w);
  }
  if (it.kind() == kWide) wide_item<D, KV8>(a, it, gkv, lds);
  else if (it.rows() <= 16) narrow_item<D, KV8, 1>(a, it, gkv, lds);
  else narrow_item<D, KV8, 2>(a, it, gkv, lds);
}
template <int D, bool KV8>
__global__ __launch_bounds__(64 * NW, 2) void packed_attention_kernel(const Args a) { packed_item<D, KV8>(a); }
template <int D, bool KV8>
__global__ __launch_bounds__(64 * NW, 2) void packed_attention_words_kernel(const ArgsAndWords w) {
  Args a = w.a;
  a.words = words_of_launch();
  packed_item<D, KV8>(a);
}

// The partitions of split blocks: D/8 lanes have a row, 8 elements each, and take its partitions four at a time.
template <int D>
__device__ __forceinline__ void packed_merge(const Args &a) {
  constexpr int VPR = D / 8, ROWS = 256 / VPR;
  const Merge m = *(const Merge *)(a.words + a.merges_at + blockIdx.x * kMergeWords);
  const int gkv = blockIdx.z, row = blockIdx.y * ROWS + threadIdx.x / VPR, dv = threadIdx.x % VPR;
  if (row >= m.rows) return;
  const size_t first = (size_t)gkv * a.part_rows + m.part + row;
  float top = -INFINITY, l = 0.f, acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int p0 = 0; p0 < m.n; p0 += 4) {
    float2 e[4];
    f32x4 x[4][2];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const size_t at = first + (size_t)min(p0 + j, m.n - 1) * m.rows;
      e[j] = *(const float2 *)(a.part_ml + at * 2);
      x[j][0] = *(const f32x4 *)(a.part_o + at * D + dv * 8);
      x[j][1] = *(const f32x4 *)(a.part_o + at * D + dv * 8 + 4);
      if (p0 + j >= m.n) e[j] = make_float2(-INFINITY, 0.f);
    }
    float t = top;
#pragma unroll
    for (int j = 0; j < 4; ++j) t = fmaxf(t, e[j].x);
    const float shrink = top == -INFINITY ? (l == 0.f ? 0.f : 1.f) : fast_exp2(top - t);
    top = t;
    l *= shrink;
#pragma unroll
    for (int d = 0; d < 8; ++d) acc[d] *= shrink;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (e[j].y == 0.f) continue;   // (no key of the row in that partition)
      const float w = e[j].x == -INFINITY ? e[j].y : e[j].y * fast_exp2(e[j].x - top);
      l += w;
#pragma unroll
      for (int d = 0; d < 8; ++d) acc[d] += w * x[j][d >> 2][d & 3];
    }
  }
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  const auto [i, head] = row_at(a, m, gkv, row);
  bf16x8 v;
#pragma unroll
  for (int d = 0; d < 8; ++d) v[d] = (__bf16)(acc[d] * inv);
  *(bf16x8 *)(a.out + ((size_t)m.row0 + i) * ((size_t)a.Hq * D) + (size_t)head * D + dv * 8) = v;
  if (a.lse && dv == 0) a.lse[(size_t)head * a.N + m.row0 + i] = pc::lse_of(top, l);
}

template <int D>
__global__ __launch_bounds__(256) void packed_merge_kernel(const Args a) { packed_merge<D>(a); }
template <int D>
__global__ __launch_bounds__(256) void packed_merge_words_kernel(const ArgsAndWords w) {
  Args a = w.a;
  a.words = words_of_launch();
  packed_merge<D>(a);
}

// ---------------------------------------------------------------- host side
struct PackedWs {
  int32_t *words;
  float *part_o, *part_ml;
  long most_items, part_rows;   // of one kv head
  size_t total;
};
long most_blocks(const percache_config &c, int n_seq, int n_rows) { return (long)(c.n_q_heads / c.n_kv_heads) * n_rows / kNarrowRows + n_seq; }
// Partial rows of one kv head.  As many as there are rows, at least two partitions of 256 rows a CU: the longest cut by shares.  No more than kMostCut blocks of 256
// rows a CU have, since more blocks than that are not cut; a larger call asks for as much as that one, so that a workspace is enough for smaller calls too.
constexpr int kMostCut = 8;
long most_part_rows(const percache_config &c, int n_cu, int n_rows) {
  const long rows = (long)(c.n_q_heads / c.n_kv_heads) * n_rows, cut = (long)kMostCut * std::max(1, n_cu / c.n_kv_heads) * kWideRows;
  return std::max(std::min(rows, cut), std::min(rows * kMaxPackedSplits, 2L * n_cu * kWideRows / c.n_kv_heads));
}
PackedWs carve(const percache_config &c, int n_cu, void *base, int n_seq, int n_rows, int max_chunks) {
  PackedWs w;
  char *p = (char *)base;
  size_t off = 0;
  auto take = [&](size_t bytes) { char *r = p ? p + off : nullptr; off += pc::align_up(bytes); return r; };
  const long blocks = most_blocks(c, n_seq, n_rows);
  w.most_items = blocks + (long)kMoreItems * n_cu;
  w.part_rows = most_part_rows(c, n_cu, n_rows);
  w.words = (int32_t *)take(((size_t)w.most_items * kItemWords + (size_t)blocks * kMergeWords + (size_t)n_seq * max_chunks * 2 + 4) * sizeof(int32_t));
  w.part_o = (float *)take((size_t)w.part_rows * c.n_kv_heads * c.head_dim * sizeof(float));
  w.part_ml = (float *)take((size_t)w.part_rows * c.n_kv_heads * 2 * sizeof(float));
  w.total = off;
  return w;
}
int max_splits(const percache_config &c, int n_cu, int n_seq, int n_rows) {
  const long rows = (long)(c.n_q_heads / c.n_kv_heads) * std::max(n_rows, 1), blocks = std::max(most_blocks(c, n_seq, n_rows), 1L);
  const long by_rows = most_part_rows(c, n_cu, n_rows) / rows, by_items = 1 + (long)kMoreItems * n_cu / blocks;
  return (int)std::max(1L, std::min((long)kMaxPackedSplits, std::min(by_rows, by_items)));
}

// The list of a call: items, longest first; merges; chunk entries.
struct Plan {
  std::vector<int32_t> words;
  int n_items = 0, n_merges = 0, merges_at = 0, ents_at = 0, tallest = 0;
};
void plan_items(const percache_ctx *ctx, const std::vector<int32_t> &table, int stride, const int32_t *start, int n_seq, int n_splits, const PackedWs &ws, Plan &plan) {
  const percache_config &c = ctx->cfg;
  const int G = c.n_q_heads / c.n_kv_heads;
  struct Block { int seq, r_first, rows, kind, tiles, n; };   // n: partitions (0: they end where `ends` says)
  std::vector<int32_t> ents, first_ent(n_seq + 1), tiles_before;   // entries with keys; cached tiles before each
  std::vector<int> cached(n_seq);
  long tiles8 = 0, all_tiles = 0;
  for (int s = 0; s < n_seq; ++s) {
    first_ent[s] = (int)ents.size() / 2;
    int tiles = 0;
    if (start[s + 1] > start[s])
      for (int ci = 0; ci < table[(size_t)s * stride]; ++ci) {
        const int slot = table[(size_t)s * stride + pc::kTblHeader + 2 * ci], used = table[(size_t)s * stride + pc::kTblHeader + 2 * ci + 1];
        if (used <= 0) continue;
        ents.push_back(slot);
        ents.push_back(used);
        tiles_before.push_back(tiles);
        tiles += (used + TK - 1) / TK;
        if (ctx->is8(slot)) tiles8 += (used + TK - 1) / TK;
      }
    all_tiles += tiles + (start[s + 1] - start[s] + TK - 1) / TK;
    cached[s] = tiles;
  }
  first_ent[n_seq] = (int)ents.size() / 2;
  // us of a workgroup's start and end, of a MB from memory and of a tile of more than 128 rows, of more than 32, 16, fewer (most of the chip at work on random data: the
  // clock falls; with few workgroups 1.37 and 1.11 of the first two at head size 128, 1.02 and 0.78 at 64), of 8-bit tiles 2.4, 1.57, ..  8-bit tiles cost more because their codes are
  // turned into bf16 ones between the wait for them and the barrier, where no product runs; at head size 64 by half of the threads.
  constexpr float kStart = 6.f, kStartLow = 4.f, kPerMb = 1.f / 5.4f;
  constexpr float kTile[2][2][4] = {{{1.28f, 0.97f, 0.52f, 0.45f}, {1.55f, 1.07f, 0.60f, 0.52f}}, {{1.85f, 1.54f, 0.88f, 0.72f}, {2.40f, 1.57f, 0.76f, 0.65f}}};
  float tile_of[4];
  for (int i = 0; i < 4; ++i) {
    const auto &t = kTile[c.head_dim == 128];
    tile_of[i] = t[0][i] + (t[1][i] - t[0][i]) * (float)tiles8 / (float)std::max(all_tiles, 1L);
  }
  auto class_of = [](const Block &b) { return b.kind == kWide ? b.rows <= kWideRows / 2 : b.rows > 16 ? 2 : 3; };
  auto start_us = [&](const Block &b) { return class_of(b) == 1 ? kStartLow : kStart; };
  auto tile_us = [&](const Block &b) { return tile_of[class_of(b)]; };
  auto cost_of = [&](const Block &b, int tiles) { return start_us(b) + tile_us(b) * (float)tiles; };
  auto cut = [&](int height) {   // blocks of so many rows, the last of a request narrow where 32 rows are left
    std::vector<Block> blocks;
    for (int s = 0; s < n_seq; ++s) {
      const int R = G * (start[s + 1] - start[s]);
      for (int r = 0; r < R;) {
        const int rows = std::min(R - r, R - r <= kNarrowRows ? kNarrowRows : height), kind = rows <= kNarrowRows ? kNarrow : kWide;
        const int tiles = cached[s] + ((r + rows - 1) / G) / TK + 1;
        blocks.push_back({s, r, rows, kind, tiles, 1});
        r += rows;
      }
    }
    return blocks;
  };
  // Partitions: blocks that take longer than a limit, one for each kind, are cut evenly, or all are cut by shares.  A launch is dealt out longest first to the
  // CUs, of which every kv head gets its share; that is played through (while there are few workgroups a CU: many even out by themselves), and what
  // promises 3 % more is taken.  Nothing is faster than its keys come from memory; a merge is a launch and the partial rows.  us at 1, 2, 3, 4
  // partitions, measured (workgroups of all kv heads): 72 wide blocks of 60 tiles at head size 128 95, 64, 53, 60; head size 64, 152 of 36 to 60 tiles (14 heads over 2, seven questions of 43 to
  // 1142 rows behind 2.3k cached keys) 84, 80, 70; 144 narrow ones of 52 tiles (24 heads over 8, 18 single tokens over 3k keys) 53, 62, 53, 59, 32 of them 48, 32, 24, 22; 200 wide ones of 50 to 60
  // tiles (six questions of 118 to 595 rows) beside the 144 134 (cut evenly into 712 workgroups 151).
  auto least_of = [&](const Block &b) { return class_of(b) == 0 ? 6 : 4; };   // tiles of a partition
  const int cus = std::max(1, ctx->n_cu / c.n_kv_heads);
  float mb = 0.f;
  for (int s = 0; s < n_seq; ++s) mb += (float)cached[s] * (float)(TK * c.head_dim * 4 * c.n_kv_heads) * 1e-6f;
  typedef std::vector<std::pair<float, int>> Runs;   // so many workgroups of this cost; so many CUs that are free at this time
  Runs runs, free_at;
  std::vector<float> costs;
  std::vector<int> ends;
  auto play = [&]() {   // us of the runs, longest first
    std::sort(runs.begin(), runs.end(), std::greater<std::pair<float, int>>());
    free_at.assign(1, {0.f, cus});   // (the CUs that are free first at its end)
    for (auto [cost, count] : runs)
      while (count > 0) {
        const auto [at, n] = free_at.back();
        const int m = std::min(n, count);
        count -= m;
        if (m == n) free_at.pop_back();
        else free_at.back().second -= m;
        auto to = free_at.end();
        while (to != free_at.begin() && (to - 1)->first < at + cost) --to;
        if (to != free_at.begin() && (to - 1)->first == at + cost) (to - 1)->second += m;
        else free_at.insert(to, {at + cost, m});
      }
    return free_at.front().first;
  };
  auto merge_us = [&](float rows) { return rows > 0.f ? 5.f + rows * (float)(c.n_kv_heads * c.head_dim) * 1e-6f : 0.f; };
  struct Group { int kind, tiles, count, least; float start, tile, rows; };   // blocks that take equally long
  std::vector<Group> groups;
  auto settle = [&](std::vector<Block> &blocks) {   // chooses the partitions; us
    int most = 0;
    for (const Block &x : blocks) most = std::max(most, x.tiles);
    groups.assign(4 * (size_t)(most + 1), Group{});   // (more than 128 rows; more than 32; more than 16; fewer)
    for (const Block &x : blocks) {
      Group &g = groups[class_of(x) * (size_t)(most + 1) + x.tiles];
      g = {x.kind, x.tiles, g.count + 1, least_of(x), start_us(x), tile_us(x), g.rows + (float)x.rows};
    }
    groups.erase(std::remove_if(groups.begin(), groups.end(), [](const Group &g) { return g.count == 0; }), groups.end());
    float longest[2] = {0.f, 0.f}, whole = 0.f;
    for (const Group &g : groups) {
      const float us = g.start + g.tile * (float)g.tiles;
      longest[g.kind] = std::max(longest[g.kind], us);
      whole += us * (float)g.count;
    }
    auto parts_of = [&](int kind, int least, float start, float tile, int tiles, const float (&limit)[2]) {
      return std::max(1, std::min({(int)(tile * (float)tiles / std::max(limit[kind] - start, 1.f) + 0.99f), tiles / least, kMaxPackedSplits}));
    };
    if (n_splits > 0) {   // the partitions asked for
      float rows = 0.f;
      runs.clear();
      for (const Group &g : groups) {
        const int n = std::min(n_splits, g.tiles);
        runs.push_back({g.start + g.tile * (float)g.tiles / (float)n, n * g.count});
        if (n > 1) rows += (float)n * g.rows;
      }
      for (Block &x : blocks) x.n = std::min(n_splits, x.tiles);
      return std::max(play(), mb * kPerMb) + merge_us(rows);
    }
    // Cut evenly, for limits from the longest block's time down.
    float best = 1e30f, best_limit[2] = {longest[kWide], longest[kNarrow]};
    bool open = true;   // whether finer limits can still be better: their workgroups' time only grows, and there are finer ones
    const float top = std::max(longest[kWide], longest[kNarrow]);
    const bool both = longest[kWide] > 0.f && longest[kNarrow] > 0.f;
    for (float cut = 1.f; open && cut <= (float)kMaxPackedSplits; cut += cut < 6.f ? 1.f : cut < 16.f ? 2.f : 8.f) {   // (the longest block in so many)
      open = false;
      for (float cut2 = 1.f; cut2 <= (both ? 2.f : 1.f); cut2 *= 2.f) {
        const float wide = kStart + (top - kStart) / cut, limit[2] = {wide, std::min(wide, kStart + (longest[kNarrow] - kStart) / cut2)};
        float rows = 0.f, sum = 0.f, end = 0.f;
        int number = 0;
        bool finest = true;
        runs.clear();
        for (const Group &g : groups) {
          const int n = parts_of(g.kind, g.least, g.start, g.tile, g.tiles, limit);
          const float each = g.start + g.tile * (float)g.tiles / (float)n;
          runs.push_back({each, n * g.count});
          number += n * g.count;
          sum += each * (float)(n * g.count);
          end = std::max(end, each);
          finest &= n == std::max(1, std::min(g.tiles / g.least, kMaxPackedSplits));
          if (n > 1) rows += (float)n * g.rows;
        }
        const float more = merge_us(rows);
        if (std::max(sum / (float)cus, mb * kPerMb) + more >= 0.97f * best) continue;
        open |= !finest;
        if (end + more >= 0.97f * best) continue;
        if (number > cus) end = play();
        const float us = std::max(end, mb * kPerMb) + more;
        if (us < 0.97f * best) {
          best = us;
          best_limit[kWide] = limit[kWide];
          best_limit[kNarrow] = limit[kNarrow];
        }
      }
    }
    for (Block &x : blocks) x.n = parts_of(x.kind, least_of(x), start_us(x), tile_us(x), x.tiles, best_limit);
    // The blocks' keys laid end to end and cut where a CU's share ends, the share a little longer from try to try until it is enough: partitions are as long as
    // a share or what is left of one on either side of a block's end, and the launch puts the latter together again, longest with shortest (the 200 wide blocks
    // named above alone, kernel and merge: 131 us cut evenly, 115 so; the 152 of head size 64, half of the chunks 8-bit, 67, 59; the 200 and the 144 narrow ones 131 uncut, 138).
    int tries = (long)blocks.size() <= 4L * cus ? 8 : 0;
    for (float share = std::max(whole / (float)cus + kStart, 2.f * kStart); tries > 0 && std::max(share, mb * kPerMb) + merge_us(1.f) < 0.97f * best; share *= 1.05f, --tries) {
      ends.clear();
      costs.clear();
      int bins = 1;
      float left = share, rows = 0.f;
      for (const Block &x : blocks) {
        const int least = least_of(x);
        const float start = start_us(x), tile = tile_us(x);
        int n = 0;
        for (int t = 0; t < x.tiles; ++n) {
          int can = (int)((left - start) / tile);
          if (can < std::min(least, x.tiles - t)) {
            ++bins;
            left = share;
            can = std::max(least, (int)((left - start) / tile));
          }
          if (can < x.tiles - t && x.tiles - t - can < least) can = x.tiles - t < 2 * least ? x.tiles - t : x.tiles - t - least;
          can = std::min(can, x.tiles - t);
          t += can;
          const float us = start + tile * (float)can;
          left -= us;
          costs.push_back(us);
          ends.push_back(t);
        }
        if (n > 1) rows += (float)(n * x.rows);
        if (bins > cus) break;
      }
      if (bins > cus) continue;
      std::sort(costs.begin(), costs.end());
      runs.clear();
      for (float us : costs)
        if (!runs.empty() && runs.back().first == us) ++runs.back().second;
        else runs.push_back({us, 1});
      const float us = std::max(play(), mb * kPerMb) + merge_us(rows);
      if (us < 0.97f * best) {
        best = us;
        for (Block &x : blocks) x.n = 0;
      }
      break;
    }
    return best;
  };
  // Blocks of 256 rows; where few of them would find the chip half empty, 128 or 32 rows each may be the faster ones (few keys: more workgroups, less of a start
  // and a walk each) or not (many keys: two and eight times as many are walked), whether the partitions are asked for or chosen.  A walk of 20 tiles at
  // head size 128: 8 blocks of 256 rows 37.5 us, 16 of 128 30; 64 and 128 39, 32; 128 and 256 42.3, 36.8.  Seven partitions asked for, 8 heads over 1 of 64, 700 and 430 rows
  // behind 1135 and 575 keys: 84 us a call in blocks of 32 rows, 31 as they are chosen; 8 over 2 of 128, 513 and 300 rows behind 905 and 575: 79, 33.
  std::vector<Block> blocks = cut(kWideRows);
  float best = n_splits > 0 || (long)blocks.size() <= (long)kMostCut * cus ? settle(blocks) : 0.f;   // (more blocks than that even out uncut)
  std::vector<int> best_ends = ends;
  auto lower = [&](int height, long most) {
    std::vector<Block> low = cut(height);
    if ((long)low.size() > most) return;
    const float us = settle(low);
    if (us >= best) return;
    best = us;
    best_ends = ends;
    blocks = std::move(low);
  };
  const long tall = (long)blocks.size();
  if (tall * 2 <= cus) lower(kWideRows / 2, 2L * cus);
  if (tall * 2 <= cus) lower(kNarrowRows, 2L * cus);
  ends = std::move(best_ends);
  struct Unit { int block, begin, end; float cost; int part; };
  std::vector<Unit> units;
  long part_rows = 0, more = ws.most_items - (long)blocks.size();
  const int *end_of = ends.data();
  for (int b = 0; b < (int)blocks.size(); ++b) {
    const Block &x = blocks[b];
    int n = x.n;
    const int *const mine = n ? nullptr : end_of;
    if (mine) {
      while (mine[n] < x.tiles) ++n;
      end_of += ++n;
    }
    if (n - 1 > more || part_rows + (long)n * x.rows > ws.part_rows) n = 1;
    if (n > 1) {
      const Merge m = {start[x.seq], x.r_first / G, x.r_first % G, x.rows, (int32_t)part_rows, n};
      plan.words.insert(plan.words.end(), (const int32_t *)&m, (const int32_t *)&m + kMergeWords);
      ++plan.n_merges;
      plan.tallest = std::max(plan.tallest, x.rows);
    }
    for (int p = 0; p < n; ++p) {
      const int begin = n == 1 ? 0 : mine ? (p ? mine[p - 1] : 0) : (int)((long)p * x.tiles / n), end = n == 1 ? x.tiles : mine ? mine[p] : (int)((long)(p + 1) * x.tiles / n);
      units.push_back({b, begin, end, cost_of(x, end - begin), n > 1 ? (int)part_rows + p * x.rows : -1});
    }
    if (n > 1) part_rows += (long)n * x.rows;
    more -= n - 1;
  }
  std::stable_sort(units.begin(), units.end(), [](const Unit &x, const Unit &y) { return x.cost > y.cost; });
  std::vector<int32_t> items;
  items.reserve(units.size() * kItemWords);
  for (const Unit &u : units) {
    const Block &x = blocks[u.block];
    const int s = x.seq, e0 = first_ent[s], e1 = first_ent[s + 1];
    Item it = {};
    it.row0 = start[s];
    it.T = start[s + 1] - start[s];
    it.i0 = x.r_first / G;
    it.rem0 = (uint16_t)(x.r_first % G);
    it.rows_kind = (uint16_t)(x.rows * 2 + x.kind);
    it.n_cached = std::max(0, std::min(u.end, cached[s]) - u.begin);
    it.f0 = std::max(0, u.begin - cached[s]);
    it.f1 = std::max(it.f0, u.end - cached[s]);
    it.part = u.part;
    if (it.n_cached > 0) {
      const int first = (int)(std::upper_bound(tiles_before.begin() + e0, tiles_before.begin() + e1, u.begin) - tiles_before.begin()) - 1;
      it.ent = first;
      it.tile0 = u.begin - tiles_before[first];
      it.slot0 = ents[2 * first];
      it.used0 = ents[2 * first + 1];
    }
    items.insert(items.end(), (const int32_t *)&it, (const int32_t *)&it + kItemWords);
  }
  plan.n_items = (int)units.size();
  plan.merges_at = (int)items.size();
  items.insert(items.end(), plan.words.begin(), plan.words.end());
  if (items.size() & 1) items.push_back(0);   // (entries are read two words at a time)
  plan.ents_at = (int)items.size();
  items.insert(items.end(), ents.begin(), ents.end());
  plan.words = std::move(items);
}
}  // namespace

extern "C" {

size_t percache_packed_workspace_bytes(const percache_ctx *ctx, int32_t n_seq, int32_t n_rows, int32_t max_chunks) {
  if (!ctx || n_seq < 1 || n_rows < 0 || max_chunks < 0) return 0;
  return carve(ctx->cfg, ctx->n_cu, nullptr, n_seq, n_rows, max_chunks).total;
}

int32_t percache_packed_max_splits(const percache_ctx *ctx, int32_t n_seq, int32_t n_rows) {
  if (!ctx || n_seq < 1 || n_rows < 0) return PC_EINVAL;
  return max_splits(ctx->cfg, ctx->n_cu, n_seq, n_rows);
}

pc_status percache_attention_packed(percache_ctx *ctx, int32_t layer, const void *q_dev, const void *k_dev, const void *v_dev, int32_t n_rows,
                                    const int32_t *start_host, int32_t n_seq, const int32_t *slot_ids_host, const int32_t *used_len_host,
                                    const int32_t *n_chunks_host, int32_t max_chunks, int32_t n_splits, void *attn_out_dev, float *lse_out_dev,
                                    void *workspace_dev, size_t workspace_bytes, void *stream) try {
  if (!ctx) return PC_EINVAL;
  const percache_config &c = ctx->cfg;
  if (n_seq < 1 || n_rows < 0) return pc::fail(ctx, PC_EINVAL, "n_seq must be positive and n_rows not negative");
  if (!start_host) return pc::fail(ctx, PC_EINVAL, "start_host is NULL");
  if (start_host[0] < 0) return pc::fail(ctx, PC_EINVAL, "start[0]=%d is negative", start_host[0]);
  for (int s = 0; s < n_seq; ++s)
    if (start_host[s + 1] < start_host[s]) return pc::fail(ctx, PC_EINVAL, "start[%d]=%d lies before start[%d]=%d", s + 1, start_host[s + 1], s, start_host[s]);
  if (start_host[n_seq] > n_rows) return pc::fail(ctx, PC_EINVAL, "start[%d]=%d lies behind the last of %d rows", n_seq, start_host[n_seq], n_rows);
  if (c.n_q_heads / c.n_kv_heads > 32767) return pc::fail(ctx, PC_ESHAPE, "more than 32767 query heads a kv head");   // (Args::per_group)
  // (stacked rows of a request, and partial rows, are counted in 32 bits)
  if ((long)n_rows * c.n_q_heads >= (1L << 31)) return pc::fail(ctx, PC_ESHAPE, "%d rows of %d heads are 2^31 or more", n_rows, c.n_q_heads);
  const int cap = max_splits(c, ctx->n_cu, n_seq, n_rows);
  if (n_splits < 0 || n_splits > cap) return pc::fail(ctx, PC_EINVAL, "n_splits %d outside [0,%d] for this shape", n_splits, cap);
  std::vector<int32_t> table;
  pc_status st = pc::build_chunk_table(ctx, layer, n_seq, 1, slot_ids_host, used_len_host, n_chunks_host, max_chunks, table);
  if (st != PC_OK) return st;
  const size_t need = percache_packed_workspace_bytes(ctx, n_seq, n_rows, max_chunks);
  if (!workspace_dev || workspace_bytes < need) return pc::fail(ctx, PC_ENOMEM, "packed workspace has %zu bytes, need %zu", workspace_bytes, need);
  if ((uintptr_t)workspace_dev % pc::kAlign) return pc::fail(ctx, PC_EINVAL, "workspace must be 256-byte aligned");
  if (start_host[n_seq] == start_host[0]) return PC_OK;   // (no rows at all)
  if (!q_dev || !k_dev || !v_dev || !attn_out_dev) return pc::fail(ctx, PC_EINVAL, "NULL tensor pointer");
  if (((uintptr_t)q_dev | (uintptr_t)k_dev | (uintptr_t)v_dev | (uintptr_t)attn_out_dev) % 16) return pc::fail(ctx, PC_EINVAL, "tensor pointers must be 16-byte aligned");
  if ((uintptr_t)lse_out_dev % sizeof(float)) return pc::fail(ctx, PC_EINVAL, "lse_out_dev must be 4-byte aligned");
  const int stride = pc::tbl_stride(max_chunks), formats = pc::table_formats(table, stride, n_seq);
  const PackedWs ws = carve(c, ctx->n_cu, workspace_dev, n_seq, n_rows, max_chunks);
  Plan plan;
  plan_items(ctx, table, stride, start_host, n_seq, n_splits, ws, plan);
  if ((long)plan.n_items * c.n_kv_heads >= 1L << 23) return pc::fail(ctx, PC_ESHAPE, "2^23 workgroups or more");   // (a grid has fewer than 2^32 threads)
  hipStream_t s = (hipStream_t)stream;
  const bool in_args = plan.words.size() <= (size_t)kArgWords;
  if (!in_args) {
    // (a replay would find whatever the ring of staging buffers holds by then)
    if (pc::being_captured(s)) return pc::fail(ctx, PC_ESHAPE, "a list of %zu words is too long for a call that is captured (%d)", plan.words.size(), kArgWords);
    st = pc::upload_table(ctx, plan.words, ws.words, s);
    if (st != PC_OK) return st;
  }
  ArgsAndWords aw;
  Args &a = aw.a;
  a.q = (const __bf16 *)q_dev;
  a.k = (const __bf16 *)k_dev;
  a.v = (const __bf16 *)v_dev;
  a.k16 = ctx->k_store + (size_t)layer * ctx->layer_stride;
  a.v16 = ctx->v_store + (size_t)layer * ctx->layer_stride;
  a.k8 = ctx->k8_store + (size_t)layer * ctx->layer_stride8;
  a.v8 = ctx->v8_store + (size_t)layer * ctx->layer_stride8;
  const size_t sc = (size_t)layer * ctx->n_slots8 * c.n_kv_heads * (c.slot_capacity / TK);
  a.k_scale = ctx->k_scale + sc;
  a.v_scale = ctx->v_scale + sc;
  a.words = ws.words;
  a.out = (__bf16 *)attn_out_dev;
  a.lse = lse_out_dev;
  a.part_o = ws.part_o;
  a.part_ml = ws.part_ml;
  a.N = n_rows;
  a.part_rows = ws.part_rows;
  a.merges_at = plan.merges_at;
  a.ents_at = plan.ents_at;
  a.n_ents = (int)(plan.words.size() - plan.ents_at) / 2;
  a.Hq = c.n_q_heads;
  a.Hkv = c.n_kv_heads;
  a.C = c.slot_capacity;
  a.n_slots16 = ctx->n_slots16;
  a.per_group = (unsigned)((0xffffffffull + c.n_q_heads / c.n_kv_heads) / (c.n_q_heads / c.n_kv_heads));
  a.scale_log2e = 1.4426950408889634f / sqrtf((float)c.head_dim);
  const dim3 grid((unsigned)((long)plan.n_items * c.n_kv_heads));
  pc::prof_begin(ctx, PC_KERNEL_ATTENTION, s);
  if (in_args) memcpy(aw.words, plan.words.data(), plan.words.size() * sizeof(int32_t));
#define PC_PACKED(DD, EE)                                                                                                        \
  do {                                                                                                                           \
    if (in_args) hipLaunchKernelGGL((packed_attention_words_kernel<DD, EE>), grid, dim3(64 * NW), 0, s, aw);                      \
    else hipLaunchKernelGGL((packed_attention_kernel<DD, EE>), grid, dim3(64 * NW), 0, s, a);                                     \
  } while (0)
  if (c.head_dim == 128) { if (formats & 1) PC_PACKED(128, true); else PC_PACKED(128, false); }
  else { if (formats & 1) PC_PACKED(64, true); else PC_PACKED(64, false); }
#undef PC_PACKED
  PC_HIP(ctx, hipGetLastError());
  pc::prof_end(ctx, PC_KERNEL_ATTENTION, s);
  if (plan.n_merges) {
    const int per = 256 / (c.head_dim / 8);
    const dim3 mgrid((unsigned)plan.n_merges, (unsigned)((plan.tallest + per - 1) / per), (unsigned)c.n_kv_heads);
#define PC_MERGE(DD)                                                                                          \
  do {                                                                                                        \
    if (in_args) hipLaunchKernelGGL(packed_merge_words_kernel<DD>, mgrid, dim3(256), 0, s, aw);                \
    else hipLaunchKernelGGL(packed_merge_kernel<DD>, mgrid, dim3(256), 0, s, a);                               \
  } while (0)
    if (c.head_dim == 128) PC_MERGE(128); else PC_MERGE(64);
#undef PC_MERGE
    PC_HIP(ctx, hipGetLastError());
  }
  return PC_OK;
} catch (const std::exception &) {   // (before the first launch; the text is short enough to be kept without an allocation)
  return pc::fail(ctx, PC_ENOMEM, "no host memory");
}

}  // extern "C"
