// Attention of the nodes of drafted trees, more than 32 rows a kv head, over the cached keys (the nodes that a row looks at are added in the merge, draft.hip).
//
// What bounds it: 64 to 192 rows share a key, which is about where the key stream and the matrix cores take equally long, and a matrix operand read
// from LDS should serve as many rows as the registers hold outputs for.  The long-context kernel of a prompt (reuse_attention.hip) has 32 rows a
// wavefront: its eight wavefronts read 256 KB of operands for a 32 KB tile, as many clocks of LDS as of the matrix cores, and 192 rows leave two of
// them without work.  Here a workgroup is RG groups of rows x two halves of a 64-key tile, a wavefront NR blocks of 16 rows x 32 keys (16x16x32
// products):
//   - every operand serves NR blocks: 128 KB of LDS a tile whatever NR, and 192 rows are 4 x 3 blocks, nothing idle;
//   - scores come out transposed, S^T = K Q^T, a lane with 4 keys of each of two 16-key blocks of one row, which is the B operand of O^T += V^T P^T
//     as it stands.  Which key is which row of a block is free: the K rows are read in the order in which V lies (the 8 keys of lane group g: 16 (g %
//     2) + 4 (g / 2) + 8 j + e, block j), so that an operand of V is one 16-byte read (8 bytes of codes);
//   - a ring of stages filled by direct global->LDS loads, the scales of a tile of codes among them, one barrier a tile (it says that tile t has
//     landed for every wavefront and that tile t - 1 has been read);
//   - up to 64 rows over codes: RG = 2, half the wavefronts with two blocks each, so that a code is turned into bf16 half as often, and two
//     workgroups on a CU;
//   - the two halves of a row's keys meet once, through LDS, and leave one fp32 partial.
// 8 queries x 8 kv heads, 192 rows over 12.4k keys (bf16, D = 128): 89 us (0.87 PF of products), 106 in a process's first thirty launches, while the
// clock settles.  With a part left out, us a call that took 102: the products of either kind 84, the reads of LDS 88, the exponentials or the
// requests 93; the two wavefronts of a SIMD half a tile apart, and the requests behind the reads, changed nothing.  A wavefront lives four fifths of
// the launch: the longest query has 1.1 times the mean's keys, and there is the first tile to wait for.  6 queries x 8 kv heads, 63 rows over 157
// tiles of codes, one chunk shared: 31 us (3.7 TB/s of codes).
//
// Precision: a probability is rounded to bf16 for the product with V (its sum is taken before), everything else is fp32.
#include "decode_common.hpp"

namespace {
using pc::bf16x8;
using pc::f32x4;
using pc::kKvTile;
using pc::kTblHeader;
using pc::dec::codes8;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
using pc::dec::fast_exp2;
using pc::dec::row_max;
using pc::dec::row_sum;

constexpr int TK = kKvTile;
constexpr float kSumLimit = 8.f * 256.f;   // 8 probabilities of a lane and tile, each at most 2^8 against the reference

#define PC_WAIT_VMCNT(n) __builtin_amdgcn_s_waitcnt(((n) & 0xf) | (7 << 4) | (15 << 8) | ((((n) >> 4) & 3) << 14))

// FMT: 0 every cached chunk of the call sits in a bf16 slot, 1 in an 8-bit slot, 2 some of each.
template <int D, int FMT, int NR, int RG>
struct Lds {
  static constexpr int K16 = TK * D * 2, K8 = TK * D;
  static constexpr int SCALES = FMT == 1 ? 2 * K8 : 2 * K16;               // the two scales of a tile of codes, 256 bytes that repeat them
  static constexpr int STAGE = SCALES + (FMT == 0 ? 0 : 256), NSTG = 4;
  static constexpr int MERGE = RG * (D / 16 * NR * 4 + 2 * NR) * 64 * 4;   // outputs, (m, l) of the second halves, lane by lane
  static constexpr int BYTES = NSTG * STAGE > MERGE ? NSTG * STAGE : MERGE;
};

template <int D, int FMT, int NR, int RG>
__global__ __launch_bounds__(128 * RG, 2) void draft_attention_kernel(
    const __bf16 *__restrict__ Q, const __bf16 *k16, const __bf16 *v16, const uint8_t *__restrict__ k8, const uint8_t *__restrict__ v8,
    const float *__restrict__ k_scale, const float *__restrict__ v_scale, int n_slots16, const int32_t *__restrict__ table, int tbl_stride, int T, int Hq,
    int Hkv, int C, int n_splits, int q_tiles, int n_groups, float scale_log2e, float *__restrict__ part_o, float *__restrict__ part_ml) {
  using L = Lds<D, FMT, NR, RG>;
  constexpr int NW = 2 * RG, KS = D / 32, DB = D / 16, NSTG = L::NSTG, QROWS = RG * NR * 16;
  __shared__ __align__(16) char lds[L::BYTES];
  // the row blocks of one run of keys are consecutive on one XCD (workgroup ids go round-robin over the 8 XCDs)
  const int xcd = blockIdx.x & 7, jj = blockIdx.x >> 3, sg = jj / q_tiles * 8 + xcd, qt = jj % q_tiles;
  if (sg >= n_groups) return;
  const int split = sg % n_splits, bg = sg / n_splits, gkv = bg % Hkv, b = bg / Hkv;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g = lane >> 4;
  const int rg = wave >> 1, kh = wave & 1, G = Hq / Hkv, R = G * T;

  // chunk list: lane c keeps (slot, used length) of chunk c for the first 64 chunks, later ones are read when met
  const int32_t *trow = table + (size_t)b * tbl_stride;
  int my_slot = 0, my_used = 0;
  if (lane < (tbl_stride - kTblHeader) / 2) {
    const int2 e = *(const int2 *)(trow + kTblHeader + 2 * lane);
    my_slot = e.x;
    my_used = e.y;
  }
  const int n_chunks = trow[0], n_tiles = trow[2];
  if (lane >= n_chunks) my_used = 0;
  const unsigned long long live = __ballot(my_used > 0);
  const int tile_begin = (int)((long)split * n_tiles / n_splits), tile_end = (int)((long)(split + 1) * n_tiles / n_splits), n = tile_end - tile_begin;

  // Which 8 of the head dimensions are lane group g's part of product ks: with codes the products come in pairs, whose 16 a lane reads at once.
  auto dim0 = [&](int ks) __attribute__((always_inline)) { return FMT == 0 ? 32 * ks + 8 * g : 64 * (ks >> 1) + 16 * g + 8 * (ks & 1); };
  // this lane's rows (columns of the products): row block r of its group
  const int row0 = qt * QROWS + rg * NR * 16 + l16;
  bf16x8 q[NR][KS];
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    const int row = min(row0 + r * 16, R - 1), hg = row / T;
    const __bf16 *p = Q + (((size_t)b * Hq + gkv * G + hg) * T + (row - hg * T)) * D;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) q[r][ks] = *(const bf16x8 *)(p + dim0(ks));
  }
  f32x4 o[DB][NR];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < NR; ++r) o[db][r] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_ref[NR], l_run[NR];
#pragma unroll
  for (int r = 0; r < NR; ++r) { m_ref[r] = -INFINITY; l_run[r] = 0.f; }
  bool started = false;   // every row of this wavefront has seen a key

  // ---- walk over the tiles of the range: a cursor that only moves on by a tile's size, and the rarely taken step to the next chunk that has keys
  struct Cursor { int chunk, slot, left, off; };   // left: keys of the chunk from the tile on; off: tile inside the chunk
  auto enter = [&](Cursor &c) __attribute__((always_inline)) {   // chunk c.chunk or the next one with keys
    if (c.chunk < 64) {
      const unsigned long long rest = live >> c.chunk;
      c.chunk = rest ? c.chunk + (int)__builtin_ctzll(rest) : min(n_chunks, 64);
    }
    while (c.chunk >= 64 && c.chunk < n_chunks && trow[kTblHeader + 2 * c.chunk + 1] == 0) ++c.chunk;
    if (c.chunk < min(n_chunks, 64)) {
      const int ch = __builtin_amdgcn_readfirstlane(c.chunk);
      c.slot = __builtin_amdgcn_readlane(my_slot, ch);
      c.left = __builtin_amdgcn_readlane(my_used, ch);
    } else if (c.chunk < n_chunks) {
      c.slot = trow[kTblHeader + 2 * c.chunk];
      c.left = trow[kTblHeader + 2 * c.chunk + 1];
    }
    c.off = 0;
  };
  Cursor cur = {0, 0, 0, 0};
  {
    const int my_tiles = (my_used + TK - 1) / TK;
    int incl = my_tiles;
#pragma unroll
    for (int sh = 1; sh < 64; sh <<= 1) {
      const int up = __shfl_up(incl, sh, 64);
      if (lane >= sh) incl += up;
    }
    cur.chunk = __popcll(__ballot(incl <= tile_begin && lane < n_chunks));
    int rem;
    if (cur.chunk < min(n_chunks, 64)) {
      rem = tile_begin - __builtin_amdgcn_readlane(incl - my_tiles, __builtin_amdgcn_readfirstlane(cur.chunk));
    } else {
      rem = tile_begin - __builtin_amdgcn_readlane(incl, 63);
      while (cur.chunk < n_chunks) {
        const int ntc = (trow[kTblHeader + 2 * cur.chunk + 1] + TK - 1) / TK;
        if (rem < ntc) break;
        rem -= ntc;
        ++cur.chunk;
      }
    }
    enter(cur);
    cur.off = rem;
    cur.left -= rem * TK;
  }
  Cursor cmp = cur;   // the tile being computed
  auto is8 = [&](const Cursor &c) __attribute__((always_inline)) { return FMT == 1 || (FMT == 2 && c.slot >= n_slots16); };
  auto advance = [&](Cursor &c) __attribute__((always_inline)) {
    ++c.off;
    c.left -= TK;
    if (__builtin_expect(c.left <= 0, 0)) {
      ++c.chunk;
      enter(c);
    }
  };

  // ---- requests: instruction i of a tile half fills its bytes [1024 i, +1024); 16-byte chunks XOR-swizzled inside a row so that the 16 rows that
  // are read at once fall into different banks (of V 16 consecutive ones, of K rows 0..7 and 16..23, or 8 more): rows of 256 bytes one to a line of
  // all banks, of 128 bytes two, of 64 bytes four
  auto swz = [](int row_bytes, int row) __attribute__((always_inline)) { return row_bytes == 256 ? (row & 15) : row_bytes == 128 ? ((row >> 1) & 7) : ((row >> 2) & 3); };
  auto swz_k = [&](int row_bytes, int row) __attribute__((always_inline)) { return swz(row_bytes, (row & 7) | (row >> 1 & 8)); };
  constexpr int N16 = L::K16 / 1024, N8 = L::K8 / 1024;   // instructions of a tile half (K or V)
  auto half = [&](const char *src, char *dst, auto row_bytes_c, auto n_c, auto swizzle, int last_row) __attribute__((always_inline)) {
    constexpr int RB = decltype(row_bytes_c)::value, N = decltype(n_c)::value;
#pragma unroll
    for (int k = 0; k < (N + NW - 1) / NW; ++k) {
      const int i = N >= NW ? wave + k * NW : wave;
      if (N < NW && i >= N) break;
      const int byte = i * 1024 + lane * 16, row = byte / RB, pc = (byte % RB) / 16;
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(src + (unsigned)(min(row, last_row) * RB + (pc ^ swizzle(RB, row)) * 16)),
                                       (__attribute__((address_space(3))) void *)(dst + i * 1024), 16, 0, 2);
    }
  };
  auto request = [&](int st) __attribute__((always_inline)) {   // the cursor's tile into stage st; steps the cursor
    char *dst = lds + st * L::STAGE;
    const int last = min(TK, cur.left) - 1;       // rows past a ragged end repeat the last valid row (masked later)
    if (FMT != 0 && is8(cur)) {
      const size_t base = (((size_t)(cur.slot - n_slots16) * Hkv + gkv) * C + (size_t)cur.off * TK) * D;
      half((const char *)k8 + base, dst, std::integral_constant<int, D>{}, std::integral_constant<int, N8>{}, swz_k, last);
      half((const char *)v8 + base, dst + L::K8, std::integral_constant<int, TK>{}, std::integral_constant<int, N8>{}, swz, D - 1);
      // the scales go the same way (read as scalars they would be waited for together with the first operands); every wavefront writes the same
      const size_t at = ((size_t)(cur.slot - n_slots16) * Hkv + gkv) * (C / TK) + cur.off;
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)((lane & 1 ? v_scale : k_scale) + at),
                                       (__attribute__((address_space(3))) void *)(dst + L::SCALES), 4, 0, 0);
    } else if (FMT != 1) {
      const size_t base = (((size_t)cur.slot * Hkv + gkv) * C + (size_t)cur.off * TK) * D;
      half((const char *)(k16 + base), dst, std::integral_constant<int, D * 2>{}, std::integral_constant<int, N16>{}, swz_k, last);
      half((const char *)(v16 + base), dst + L::K16, std::integral_constant<int, TK * 2>{}, std::integral_constant<int, N16>{}, swz, D - 1);
    }
    advance(cur);
  };

  // ---- one tile: this wavefront's 32 keys x NR blocks of rows
  const int k_row[2] = {kh * 32 + 16 * (l16 >> 2 & 1) + 4 * (l16 >> 3) + (l16 & 3), kh * 32 + 16 * (l16 >> 2 & 1) + 4 * (l16 >> 3) + 8 + (l16 & 3)};
  const int v_chunk = 2 * (g & 1) + (g >> 1);   // of 16 bytes, inside the 64 of this half's keys
  auto compute = [&](int st, int valid, bool b8) __attribute__((always_inline)) {
    const int mine = valid - kh * 32;   // this half's valid keys
    if (mine <= 0) return;
    const char *kb = lds + st * L::STAGE;
    const bool c8 = FMT == 1 || (FMT == 2 && b8);
    f32x4 s[2][NR];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < NR; ++r) s[j][r] = f32x4{0.f, 0.f, 0.f, 0.f};
    // Operands of V as they lie in LDS (codes: the first two words).  What is read together is held together: everything of K and the first VB of V
    // ahead of the products, the rest of V (where the registers do not hold all of it) ahead of the softmax.  (Codes are read as vectors: a load of
    // the struct uint2 is taken to alias the direct loads into LDS and waits for all of them.)
    constexpr int VB = NR == 3 && D == 128 ? DB / 2 : DB;
    pc::u32x4 v[DB];
    float vs8 = 1.f;
    auto read_v = [&](int from, int to) __attribute__((always_inline)) {
#pragma unroll
      for (int db = from; db < to; ++db) {
        const int row = db * 16 + l16;
        if (c8) {   // byte 32 kh + 16 (g / 2) + 8 (g % 2) + 4 j + e of a row holds the key (blocked_key8)
          const u32x2 w = *(const u32x2 *)(kb + L::K8 + row * TK + (((2 * kh + (g >> 1)) ^ swz(TK, row)) * 16) + 8 * (g & 1));
          v[db] = pc::u32x4{w[0], w[1], 0u, 0u};
        } else {
          v[db] = *(const pc::u32x4 *)(kb + L::K16 + row * (TK * 2) + (((4 * kh + v_chunk) ^ swz(TK * 2, row)) * 16));
        }
      }
    };
    if (c8) {
      pc::u32x4 k[2][KS / 2];
#pragma unroll
      for (int h = 0; h < KS / 2; ++h)
#pragma unroll
        for (int j = 0; j < 2; ++j) k[j][h] = *(const pc::u32x4 *)(kb + k_row[j] * D + (((4 * h + g) ^ swz_k(D, k_row[j])) * 16));
      const float ks8 = *(const float *)(kb + L::SCALES);
      vs8 = *(const float *)(kb + L::SCALES + 4);
      read_v(0, VB);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const bf16x8 a = codes8(make_uint2(k[j][ks >> 1][2 * (ks & 1)], k[j][ks >> 1][2 * (ks & 1) + 1]), ks8);
#pragma unroll
          for (int r = 0; r < NR; ++r) s[j][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, q[r][ks], s[j][r], 0, 0, 0);
        }
    } else {
      bf16x8 k[2][KS];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int j = 0; j < 2; ++j) k[j][ks] = *(const bf16x8 *)(kb + k_row[j] * (D * 2) + (((dim0(ks) >> 3) ^ swz_k(D * 2, k_row[j])) * 16));
      read_v(0, VB);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int r = 0; r < NR; ++r) s[j][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[j][ks], q[r][ks], s[j][r], 0, 0, 0);
    }
    if (VB < DB) {
      __builtin_amdgcn_sched_barrier(0);
      read_v(VB, DB);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (__builtin_expect(mine < 32, 0)) {
      int left = mine - 16 * (g & 1) - 4 * (g >> 1);   // key 8 j + e of this lane's is valid where it is less
      asm volatile("" : "+v"(left));                   // (nothing of this stays in registers over the loop)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[j][r][e] = 8 * j + e < left ? s[j][r][e] : -INFINITY;
      // V of keys past the end cleared: their probabilities are 0, but what stands there need not be finite
      pc::u32x4 keep;
      if (c8) {
#pragma unroll
        for (int j = 0; j < 2; ++j) keep[j] = left >= 8 * j + 4 ? ~0u : left <= 8 * j ? 0u : (1u << 8 * (left & 3)) - 1;
        keep[2] = keep[3] = 0;
      } else {
#pragma unroll
        for (int w = 0; w < 4; ++w) keep[w] = (8 * (w >> 1) + 2 * (w & 1) < left ? 0xffffu : 0u) | (8 * (w >> 1) + 2 * (w & 1) + 1 < left ? 0xffff0000u : 0u);
      }
#pragma unroll
      for (int db = 0; db < DB; ++db) v[db] &= keep;
    }
    // softmax against the lazily refreshed reference exponents: a probability above 2^8 shows in the sums
    bf16x8 p[NR];
    float sum[NR];
    auto exponentials = [&](int r, float neg_m) __attribute__((always_inline)) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = fast_exp2(__builtin_fmaf(s[e >> 2][r][e & 3], scale_log2e, neg_m));
#pragma unroll
      for (int e = 0; e < 8; ++e) p[r][e] = (__bf16)x[e];
      return ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
    };
    bool refresh = !started;
    if (__builtin_expect(!refresh, 1)) {
      bool over = false;
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        sum[r] = exponentials(r, -m_ref[r]);
        over |= !(sum[r] <= kSumLimit);   // (also catches inf / nan)
      }
      refresh = __builtin_amdgcn_ballot_w64(over) != 0;
    }
    if (__builtin_expect(refresh, 0)) {
      bool all = true;
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        float mx = s[0][r][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) mx = fmaxf(mx, s[e >> 2][r][e & 3]);
        const float mc = row_max(mx) * scale_log2e;
        const bool upd = mc > m_ref[r];   // (false for a row whose keys are all masked: mc = -inf)
        const float alpha = upd ? fast_exp2(m_ref[r] - mc) : 1.0f;
        m_ref[r] = upd ? mc : m_ref[r];
        l_run[r] *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db) o[db][r] *= alpha;
        sum[r] = exponentials(r, m_ref[r] == -INFINITY ? 0.f : -m_ref[r]);
        all &= m_ref[r] != -INFINITY;
      }
      started = __builtin_amdgcn_ballot_w64(!all) == 0;
    }
#pragma unroll
    for (int r = 0; r < NR; ++r) l_run[r] += sum[r];
    if (c8) {
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const bf16x8 a = codes8(make_uint2(v[db][0], v[db][1]), vs8);
#pragma unroll
        for (int r = 0; r < NR; ++r) o[db][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, p[r], o[db][r], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < NR; ++r) o[db][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v[db]), p[r], o[db][r], 0, 0, 0);
    }
  };

  // ---- pipeline: tile t sits in stage t % NSTG, NSTG - 1 tiles are requested ahead
#pragma unroll
  for (int k = 0; k < NSTG - 1; ++k)
    if (k < n) request(k);
#pragma unroll
  for (int r = 0; r < NR; ++r)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(q[r][ks]));
  int st = 0;
  for (int t = 0; t < n; ++t) {
    const int valid = min(TK, cmp.left);
    const bool b8 = is8(cmp);
    advance(cmp);
    // what this wavefront has in flight for the tiles behind this one (mixed formats: counted as the smaller kind, which waits for more; a wavefront
    // that a half of a small tile of codes has no instruction for asks for the scales only)
    constexpr int BF16 = 2 * (N16 / NW), CODES = 2 * (N8 >= NW ? N8 / NW : 1) + 1, IPT = FMT == 0 ? BF16 : FMT == 1 ? CODES : BF16 < CODES ? BF16 : CODES;
    const int later = min(NSTG - 2, n - 1 - t);
    if (later <= 0) PC_WAIT_VMCNT(0);
    else if (FMT != 0 && N8 < NW && wave >= N8) { if (later >= 2) PC_WAIT_VMCNT(2); else PC_WAIT_VMCNT(1); }
    else if (later >= 2) PC_WAIT_VMCNT(2 * IPT);
    else PC_WAIT_VMCNT(IPT);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (t + NSTG - 1 < n) request(st == 0 ? NSTG - 1 : st - 1);
    compute(st, valid, b8);
    st = st + 1 == NSTG ? 0 : st + 1;
  }

  // ---- the halves of a row's keys: the second hands its state over lane to lane
  __syncthreads();
  float *mine = (float *)lds + (size_t)rg * (DB * NR * 4 + 2 * NR) * 64 + lane;
  if (kh == 1) {
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      mine[(2 * r) * 64] = m_ref[r];
      mine[(2 * r + 1) * 64] = l_run[r];
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 4; ++e) mine[(2 * NR + (db * NR + r) * 4 + e) * 64] = o[db][r][e];
    }
  }
  __syncthreads();
  if (kh == 1) return;
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    const float m1 = mine[(2 * r) * 64], l1 = mine[(2 * r + 1) * 64], m = fmaxf(m_ref[r], m1);
    const float a0 = m_ref[r] == m ? 1.f : fast_exp2(m_ref[r] - m), a1 = m1 == m ? 1.f : fast_exp2(m1 - m);   // (no key seen: m = -inf, sums of 0)
    const float l = row_sum(l_run[r] * a0 + l1 * a1), inv = l == 0.f ? 0.f : 1.0f / l;
    const int row = row0 + r * 16;
    if (row >= R) continue;
    const size_t prow = ((size_t)bg * R + row) * n_splits + split;
    float *po = part_o + prow * D + 4 * g;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      f32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (o[db][r][e] * a0 + mine[(2 * NR + (db * NR + r) * 4 + e) * 64] * a1) * inv;
      *(f32x4 *)(po + db * 16) = v;
    }
    if (g == 0) {
      part_ml[prow * 2] = m;
      part_ml[prow * 2 + 1] = l;
    }
  }
}

// What a workgroup alone on its CU takes for a 64-key tile, us, with nr blocks of 16 rows a wavefront (see plan_for).
float tile_us(int D, int fmt, int nr) {
  if (fmt == 1 && nr == 1) return D == 128 ? 0.80f : 0.55f;   // (half the wavefronts, two blocks each)
  if (D == 128) return fmt == 0 ? 0.52f + 0.30f * nr : fmt == 1 ? 0.45f + 0.38f * nr : 0.75f + 0.36f * nr;
  return fmt == 0 ? 0.42f + 0.23f * nr : fmt == 1 ? 0.34f + 0.29f * nr : 0.62f + 0.26f * nr;
}
// Row blocks of a wavefront and partitions of the key axis.  Blocks: the least time of all row blocks of a tile, so as many rows share an operand as
// pays (both kinds of tiles in one kernel leave registers for two blocks at D = 128).  Partitions: the least of an estimate that has the rounds in
// which the workgroups go, tiles of 1.7 times the time where two share a CU, 4 us for a workgroup's start and end, and the partials' bytes there and
// back. Over 138 calls (33 to 448 rows, 1 to 16 queries, 22 to 213 tiles, all formats and both head sizes, each timed at up to 19 counts) the counts
// so chosen take 1.01 times the best one's time on average, 1.19 at worst.  us a call, too few | this | too many partitions: 8 kv heads x 8 queries,
// 126 rows over 53 tiles (bf16, D = 128, 4 kv heads 32 | 4) 35 | 29 | 37; blocks of 64 rows against blocks of 192 over the 280 rows of 7 query heads:
// 0.82 us x 5 | 1.42 x 2 a tile.
struct Plan {
  int nr, q_tiles, n_splits;
};
Plan plan_for(int n_cu, int D, int fmt, int R, long n_bg, long rows, int tiles, int n_splits, int cap) {
  Plan p = {1, (R + 63) / 64, n_splits};
  for (int nr = 2; nr <= (D == 128 && fmt == 2 ? 2 : 3); ++nr) {
    const int q_tiles = (R + 64 * nr - 1) / (64 * nr);
    if (q_tiles * tile_us(D, fmt, nr) < p.q_tiles * tile_us(D, fmt, p.nr)) p.nr = nr, p.q_tiles = q_tiles;
  }
  if (n_splits > 0) return p;
  const bool two = (fmt == 1 && p.nr == 1) || (D == 64 && (p.nr == 1 || (fmt == 0 && p.nr == 2)));   // two workgroups fit a CU
  const double us = tile_us(D, fmt, p.nr), per_part = rows * D * 8 / 5.4e6;
  double least = 1e30;
  for (int ns = 1; ns <= cap && ns <= tiles; ++ns) {
    const double share = 0.5 * ((tiles + ns - 1) / ns + (double)tiles / ns);   // (the longest partition, and the mean one)
    const long wgs = ((n_bg * ns + 7) & ~7L) * p.q_tiles, at_once = two ? 2L * n_cu : n_cu;
    const double t = (wgs + at_once - 1) / at_once * (share * us * (wgs > n_cu && two ? 1.7 : 1.0) + 4.0) + 1.2 * ((ns + 15) / 16) + per_part * ns;
    if (t < least - 1e-9) least = t, p.n_splits = ns;
  }
  return p;
}

}  // namespace

namespace pc {

pc_status launch_draft_attention(percache_ctx *ctx, int layer, const __bf16 *q, int batch, int t_draft, const int32_t *table_dev, int tbl_stride, int tiles, int &n_splits,
                                 float *part_o, float *part_ml, hipStream_t stream, int formats) {
  const percache_config &c = ctx->cfg;
  const int R = c.n_q_heads / c.n_kv_heads * t_draft;
  const int fmt = !((formats & 1) && ctx->n_slots8 > 0) ? 0 : (formats & 2) ? 2 : 1;
  const Plan plan = plan_for(ctx->n_cu, c.head_dim, fmt, R, (long)batch * c.n_kv_heads, (long)batch * c.n_q_heads * t_draft, tiles, n_splits,
                             max_splits_for(c, ctx->n_cu, batch, t_draft));
  n_splits = plan.n_splits;
  const int nr = plan.nr, q_tiles = plan.q_tiles, n_groups = batch * c.n_kv_heads * n_splits;
  const __bf16 *k16 = ctx->k_store + (size_t)layer * ctx->layer_stride, *v16 = ctx->v_store + (size_t)layer * ctx->layer_stride;
  const uint8_t *k8 = ctx->k8_store + (size_t)layer * ctx->layer_stride8, *v8 = ctx->v8_store + (size_t)layer * ctx->layer_stride8;
  const size_t sc = (size_t)layer * ctx->n_slots8 * c.n_kv_heads * (c.slot_capacity / TK);
  const float scale_log2e = 1.4426950408889634f / sqrtf((float)c.head_dim);
  const dim3 grid((unsigned)((n_groups + 7) / 8 * 8 * q_tiles));
#define PC_DRAFT(DD, FF, RR, GG)                                                                                                                            \
  hipLaunchKernelGGL((draft_attention_kernel<DD, FF, RR, GG>), grid, dim3(128 * (GG)), 0, stream, q, k16, v16, k8, v8, ctx->k_scale + sc, ctx->v_scale + sc, \
                     ctx->n_slots16, table_dev, tbl_stride, t_draft, c.n_q_heads, c.n_kv_heads, c.slot_capacity, n_splits, q_tiles, n_groups, scale_log2e, part_o, part_ml)
#define PC_DRAFT_R(DD, FF) do { if (nr == 1) PC_DRAFT(DD, FF, (FF == 1 ? 2 : 1), (FF == 1 ? 2 : 4)); else if (nr == 2) PC_DRAFT(DD, FF, 2, 4); else PC_DRAFT(DD, FF, (DD == 128 && FF == 2 ? 2 : 3), 4); } while (0)
#define PC_DRAFT_F(DD) do { if (fmt == 0) PC_DRAFT_R(DD, 0); else if (fmt == 1) PC_DRAFT_R(DD, 1); else PC_DRAFT_R(DD, 2); } while (0)
  if (c.head_dim == 128) PC_DRAFT_F(128); else PC_DRAFT_F(64);
#undef PC_DRAFT_F
#undef PC_DRAFT_R
#undef PC_DRAFT
  PC_HIP(ctx, hipGetLastError());
  return PC_OK;
}

}  // namespace pc
