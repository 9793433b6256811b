// Eviction inside a slot: of the tokens a slot holds, every kv head keeps the first n_first, the last n_last and, of those between, the ones
// that drew the most attention weight; the kept ones stay in order and close up.
//
// Selection is integer work on the order-preserving bits of the weights, so it is exact and the same on every run: a radix search for the
// smallest kept weight, 8 bits a pass over an LDS histogram, then one pass in the order of the tokens that takes everything above it and, of
// those equal to it, the first ones.
#include "fp8_codes.hpp"

namespace {
using pc::kKvTile;

constexpr int kMaxMoves = 64;   // slots of one launch
struct Moves {
  int32_t src[kMaxMoves], dst[kMaxMoves], have[kMaxMoves], keep[kMaxMoves];
};

// Larger weight, larger key: the bits of a float with those of negative ones turned round; -0 counts as 0, NaN below everything.
__device__ __forceinline__ unsigned key_of(float w) {
  if (w != w) return 0u;
  const unsigned u = __float_as_uint(w + 0.f);
  return (u >> 31) ? ~u : u | 0x80000000u;
}

constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64, kSelLds = 8192;
// One workgroup a (kv head, slot).  idx [n][Hkv][idx_stride]: the kept tokens in order, -1 behind them; weights are moved along. Up to four passes
// over a few thousand keys (the last ones mostly spared: few tokens share three digits) and one over the tokens, each a few LDS accesses and
// barriers: a chain of latencies, so the keys are read from memory once, into LDS (slots of up to kSelLds tokens; longer ones are read again from the
// L2).  2048 tokens, 128 workgroups: 14.9 us read in every pass, 9.5 from LDS, 8.6 with the passes spared and the sums of digits taken inside the
// vector pipe.
__global__ __launch_bounds__(kSelThreads) void keep_select_kernel(float *weights, const Moves mv, int Hkv, int C, int n_first, int n_last, int32_t *idx, int idx_stride) {
  __shared__ unsigned keys[kSelLds];
  __shared__ unsigned hist[256];
  __shared__ unsigned found[3];                         // the digit, how many tokens have a larger one, and how many this one
  __shared__ int wave_n[kSelWaves][2];
  const int g = blockIdx.x, z = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int have = mv.have[z], keep = mv.keep[z];
  int32_t *out = idx + ((size_t)z * Hkv + g) * idx_stride;
  const float *w_src = weights + ((size_t)mv.src[z] * Hkv + g) * C;
  float *w_dst = weights + ((size_t)mv.dst[z] * Hkv + g) * C;
  const int lo = n_first, hi = have - n_last;           // the tokens that compete (keep < have: n_first + n_last <= keep < have)
  int need = keep >= have ? 0 : keep - n_first - n_last;
  unsigned top = 0, mask = 0;                           // the digits found so far
  bool whole = false;                                   // every token with these digits is kept: the others need not be found
  const bool in_lds = have <= kSelLds;
  auto key_at = [&](int t) __attribute__((always_inline)) { return in_lds ? keys[t] : key_of(w_src[t]); };
  if (need > 0 && in_lds)
#pragma unroll 4
    for (int t = tid; t < have; t += kSelThreads) keys[t] = key_of(w_src[t]);
  if (keep < have) {
    for (int shift = 24; shift >= 0 && need > 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int t = lo + tid; t < hi; t += kSelThreads) {
        const unsigned k = key_at(t);
        if ((k & mask) == top) atomicAdd(&hist[k >> shift & 255], 1u);
      }
      __syncthreads();
      if (wave == 0) {   // the largest digit at which the tokens from the top reach `need`: lane l counts digits 255 - 4 l .. 252 - 4 l
        unsigned n[4], sum = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) sum += n[j] = hist[255 - 4 * lane - j];
        // sums over the lanes up to this one: inside rows of 16, then over the rows before
        unsigned upto = sum;
#define PC_ADD(ctrl, rows) upto += (unsigned)__builtin_amdgcn_update_dpp(0, (int)upto, ctrl, rows, 0xf, false)
        PC_ADD(0x111, 0xf);
        PC_ADD(0x112, 0xf);
        PC_ADD(0x114, 0xf);
        PC_ADD(0x118, 0xf);
        PC_ADD(0x142, 0xa);
        PC_ADD(0x143, 0xc);
#undef PC_ADD
        unsigned before = upto - sum;
        if (before < (unsigned)need && upto >= (unsigned)need)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (before < (unsigned)need && before + n[j] >= (unsigned)need) {
              found[0] = 255 - 4 * lane - j;
              found[1] = before;
              found[2] = n[j];
            }
            before += n[j];
          }
      }
      __syncthreads();
      top |= found[0] << shift;
      mask |= 255u << shift;
      need -= found[1];   // (hist and found are written again behind the next barriers only)
      whole = (unsigned)need == found[2];
      if (whole) break;
    }
  }
  // `need` tokens with the key `top` are kept, the first ones (whole: every token that starts with its digits), and all with a larger key (keep >=
  // have: every token)
  int at = 0, ties = 0;
  for (int t0 = 0; t0 < have; t0 += kSelThreads) {
    const int t = t0 + tid;
    bool in = false, tie = false;
    float w = 0.f;
    if (t < have) {
      w = w_src[t];
      const bool fixed = keep >= have || t < lo || t >= hi;
      const unsigned k = key_of(w);
      in = fixed || (mask && (whole ? k >= top : k > top));
      tie = !fixed && mask && !whole && k == top;
    }
    const unsigned long long tie_b = __ballot(tie), below = (1ull << lane) - 1;
    if (lane == 0) wave_n[wave][0] = __popcll(tie_b);
    __syncthreads();
    int tie_at = ties;
#pragma unroll
    for (int v = 0; v < kSelWaves; ++v) {
      if (v < wave) tie_at += wave_n[v][0];
      ties += wave_n[v][0];
    }
    tie_at += __popcll(tie_b & below);
    in |= tie && tie_at < need;
    const unsigned long long in_b = __ballot(in);
    if (lane == 0) wave_n[wave][1] = __popcll(in_b);
    __syncthreads();
    int pos = at + __popcll(in_b & below);
#pragma unroll
    for (int v = 0; v < kSelWaves; ++v) {
      if (v < wave) pos += wave_n[v][1];
      at += wave_n[v][1];
    }
    // (in place: pos <= t, and the weights of this round are in registers, those of later ones further on)
    if (in) {
      out[pos] = t;
      w_dst[pos] = w;
    }
  }
  for (int t = at + tid; t < idx_stride; t += kSelThreads) out[t] = -1;
}

// The slots of both formats (layouts: kvstore.hip).
struct Store {
  __bf16 *k16, *v16;
  uint8_t *k8, *v8;
  float *k_scale, *v_scale;
  int n_slots16;
};
// A 64-token block of a slot as it lies in memory: bytes of K and V, then (8-bit) their scales.  In place the blocks go through the workspace: one
// that is written early holds tokens that another one, written late, still has to read.
template <int D>
struct Image {
  static constexpr int HALF = kKvTile * D * 2, BYTES = 2 * HALF + 256;
};

// One workgroup a (slot, kv head, 64 kept tokens): the tokens' K rows are gathered in registers as bf16 (8-bit slots: code * 2^e, exact), V in LDS as
// a bf16 block, and written in the destination's format, an 8-bit block quantised afresh.  K: 16-byte pieces of the tokens' rows.  V: a token is one
// element in each of the D rows of its block, so the blocks that hold kept tokens are read one after the other, 16 bytes of a row a lane (left out
// where none of them is kept), and the kept elements put where they belong; read element by element, two bytes a lane, the addresses took longer than
// the bytes.  16 slots x 8 heads, 1000 of 1536 tokens on average, D = 128, half of either format: 43.6 us element by element, 30.2 so (111 MB).
template <int D>
__global__ __launch_bounds__(256) void keep_move_kernel(Store st, const Moves mv, const int32_t *__restrict__ idx, int idx_stride, int Hkv, int C, char *__restrict__ images,
                                                        int tiles) {
  constexpr int KP = D / 8, KR = kKvTile * KP / 256, V_ROW = kKvTile + 8;     // 16-byte pieces of a K row, and a thread's; elements of a V row in LDS (the last 8 unused)
  __shared__ __align__(16) __bf16 lv[D * V_ROW];
  __shared__ int32_t list[kKvTile], from[kKvTile], rank0[kKvTile];      // kept tokens; source blocks that hold some, and the first of theirs
  __shared__ unsigned long long held[kKvTile];                          // which of a source block's tokens are kept
  __shared__ int n_from;
  __shared__ float red[4][2];
  const int z = blockIdx.z, g = blockIdx.y, tile = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int src = mv.src[z], dst = mv.dst[z], n = min(mv.keep[z], mv.have[z]) - tile * kKvTile;   // kept tokens from this block on
  if (n <= 0) return;
  const bool src8 = src >= st.n_slots16, dst8 = dst >= st.n_slots16;
  const size_t sh = (size_t)(src8 ? src - st.n_slots16 : src) * Hkv + g, dh = (size_t)(dst8 ? dst - st.n_slots16 : dst) * Hkv + g;
  const int bpc = C / kKvTile;
  if (tid < kKvTile) {   // (one wavefront)
    const int t = tid < n ? idx[((size_t)z * Hkv + g) * idx_stride + tile * kKvTile + tid] : -1;
    const int block = t >= 0 ? t / kKvTile : -1, before = __shfl_up(block, 1, 64);
    const bool first = t >= 0 && (lane == 0 || block != before);
    const unsigned long long firsts = __ballot(first);
    const int r = __popcll(firsts & (~0ull >> (63 - lane))) - 1;
    list[lane] = t;
    held[lane] = 0;
    if (first) {
      from[r] = block;
      rank0[r] = lane;
    }
    if (lane == 0) n_from = __popcll(firsts);
    __builtin_amdgcn_wave_barrier();
    if (t >= 0) atomicOr(&held[r], 1ull << (t % kKvTile));
  }
  if (n < kKvTile)   // places that no token fills
    for (int e = tid; e < D * V_ROW / 8; e += 256) *(pc::u32x4 *)(lv + e * 8) = pc::u32x4{0, 0, 0, 0};
  __syncthreads();
  pc::u32x4 kr[KR];
#pragma unroll
  for (int r = 0; r < KR; ++r) {
    const int e = tid + r * 256, t = max(list[e / KP], 0), c = e % KP;
    if (src8) {
      const uint2 q = *(const uint2 *)(st.k8 + (sh * C + t) * D + c * 8);
      kr[r] = pc::u32x4{q.x, q.y, __float_as_uint(st.k_scale[sh * bpc + t / kKvTile]), 0};
    } else {
      kr[r] = *(const pc::u32x4 *)(st.k16 + (sh * C + t) * D + c * 8);
    }
  }
  // V: a thread has the same 16 bytes of every row that it reads of a block, E tokens
  auto gather_v = [&](auto src8_c) __attribute__((always_inline)) {
    constexpr bool S8 = decltype(src8_c)::value;
    constexpr int E = S8 ? 16 : 8, PER = kKvTile / E, N = D * PER / 256;
    const int c = tid % PER, d0 = tid / PER;
    const int nf = n_from;
    for (int f = 0; f < nf; ++f) {
      const unsigned long long m = held[f];
      const int block = from[f];
      // (the keys of these places: the first one's, and steps from it that do not depend on the thread -- see blocked_key, blocked_key8)
      const int key0 = S8 ? 32 * (c >> 1) + 4 * (c & 1) : 16 * (c >> 1) + 4 * (c & 1), r0 = rank0[f] + __popcll(m & ((1ull << key0) - 1));
      const unsigned mine = (unsigned)(m >> key0);
      int to[E];
      bool any = false;
#pragma unroll
      for (int y = 0; y < E; ++y) {
        const int step = (S8 ? 16 * (y >> 3) + 8 * (y >> 2 & 1) : 8 * (y >> 2)) + (y & 3), kept = r0 + __popc(mine & ((1u << step) - 1));
        const bool is = mine >> step & 1;
        to[y] = is ? (kept & ~15) + pc::blocked_key(kept & 15) : kKvTile;   // (the others: into the padding)
        any |= is;
      }
      if (!any) continue;
      const float s = S8 ? st.v_scale[sh * bpc + block] : 1.f;
      const char *p = (S8 ? (const char *)st.v8 : (const char *)st.v16) + ((sh * C + (size_t)block * kKvTile) * D + c * E) * (S8 ? 1 : 2) + d0 * kKvTile * (S8 ? 1 : 2);
      pc::u32x4 w[N];
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = *(const pc::u32x4 *)(p + i * (256 / PER) * kKvTile * (S8 ? 1 : 2));
#pragma unroll
      for (int i = 0; i < N; ++i) {
        __bf16 *row = lv + (d0 + i * (256 / PER)) * V_ROW;
#pragma unroll
        for (int y = 0; y < E; ++y) {
          if (S8) row[to[y]] = (__bf16)(__builtin_amdgcn_cvt_f32_fp8((int)(w[i][y / 4] >> (8 * (y & 3))), 0) * s);
          else row[to[y]] = __builtin_bit_cast(pc::bf16x8, w[i])[y];
        }
      }
    }
  };
  if (src8) gather_v(std::true_type{}); else gather_v(std::false_type{});
  if (src8) {
#pragma unroll
    for (int r = 0; r < KR; ++r) {
      const float s = __uint_as_float(kr[r][2]);
      pc::bf16x8 v;
#pragma unroll
      for (int x = 0; x < 8; ++x) v[x] = (__bf16)(__builtin_amdgcn_cvt_f32_fp8((int)(kr[r][x >> 2] >> (8 * (x & 3))), 0) * s);
      kr[r] = __builtin_bit_cast(pc::u32x4, v);
    }
  }
#pragma unroll
  for (int r = 0; r < KR; ++r)
    if (list[(tid + r * 256) / KP] < 0) kr[r] = pc::u32x4{0, 0, 0, 0};
  __syncthreads();
  char *const image = images ? images + (((size_t)z * Hkv + g) * tiles + tile) * Image<D>::BYTES : nullptr;
  const bool through = src == dst;   // (in place: the block's image)
  if (!dst8) {
    char *const ko = through ? image : (char *)(st.k16 + (dh * C + (size_t)tile * kKvTile) * D), *const vo = through ? image + Image<D>::HALF : (char *)(st.v16 + (dh * C + (size_t)tile * kKvTile) * D);
#pragma unroll
    for (int r = 0; r < kKvTile * KP / 256; ++r) {
      const int e = tid + r * 256;
      if (e / KP < n) *(pc::u32x4 *)(ko + e * 16) = kr[r];
      *(pc::u32x4 *)(vo + e * 16) = *(const pc::u32x4 *)(lv + e / 8 * V_ROW + e % 8 * 8);
    }
    return;
  }
  float amax[2] = {0.f, 0.f};
#pragma unroll
  for (int r = 0; r < kKvTile * KP / 256; ++r) {
    const int e = tid + r * 256;
    const pc::bf16x8 k = __builtin_bit_cast(pc::bf16x8, kr[r]), v = *(const pc::bf16x8 *)(lv + e / 8 * V_ROW + e % 8 * 8);
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      amax[0] = fmaxf(amax[0], fabsf((float)k[x]));
      amax[1] = fmaxf(amax[1], fabsf((float)v[x]));
    }
  }
#pragma unroll
  for (int x = 0; x < 2; ++x) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) amax[x] = fmaxf(amax[x], __shfl_xor(amax[x], o, 64));
    if (lane == 0) red[wave][x] = amax[x];
  }
  __syncthreads();
  int ex[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) ex[x] = pc::fp8::block_exponent(fmaxf(fmaxf(red[0][x], red[1][x]), fmaxf(red[2][x], red[3][x])));
  char *const ko = through ? image : (char *)(st.k8 + (dh * C + (size_t)tile * kKvTile) * D), *const vo = through ? image + Image<D>::HALF : (char *)(st.v8 + (dh * C + (size_t)tile * kKvTile) * D);
  if (tid < 2) {
    const float s = pc::fp8::pow2f(ex[tid]);
    if (through) ((float *)(image + 2 * Image<D>::HALF))[tid] = s;
    else (tid ? st.v_scale : st.k_scale)[dh * bpc + tile] = s;
  }
  auto codes = [&](pc::u32x4 x, float inv) __attribute__((always_inline)) {
    const pc::bf16x8 v = __builtin_bit_cast(pc::bf16x8, x);
    return make_uint2(pc::fp8::encode4((float)v[0] * inv, (float)v[1] * inv, (float)v[2] * inv, (float)v[3] * inv),
                      pc::fp8::encode4((float)v[4] * inv, (float)v[5] * inv, (float)v[6] * inv, (float)v[7] * inv));
  };
  const float ki = pc::fp8::pow2f(-ex[0]), vi = pc::fp8::pow2f(-ex[1]);
#pragma unroll
  for (int r = 0; r < kKvTile * KP / 256; ++r) {
    const int e = tid + r * 256;
    if (e / KP < n) *(uint2 *)(ko + e * 8) = codes(kr[r], ki);
    // bytes 8 c .. of a V row are the bf16 block's elements 8 c' .., c' = c with its two low bits exchanged (blocked_key8, blocked_key)
    const int c = e % 8, at = (c & 4) | (c & 1) << 1 | (c & 2) >> 1;
    *(uint2 *)(vo + e * 8) = codes(*(const pc::u32x4 *)(lv + e / 8 * V_ROW + at * 8), vi);
  }
}

// The images of slots that are cut in place to where they belong.
template <int D>
__global__ __launch_bounds__(256) void keep_place_kernel(Store st, const Moves mv, int Hkv, int C, const char *__restrict__ images, int tiles) {
  const int z = blockIdx.z, g = blockIdx.y, tile = blockIdx.x, slot = mv.dst[z], n = min(mv.keep[z], mv.have[z]) - tile * kKvTile;
  if (n <= 0 || mv.src[z] != slot) return;
  const bool is8 = slot >= st.n_slots16;
  const size_t head = (size_t)(is8 ? slot - st.n_slots16 : slot) * Hkv + g, at = (head * C + (size_t)tile * kKvTile) * D;
  const char *image = images + (((size_t)z * Hkv + g) * tiles + tile) * Image<D>::BYTES;
  const int row = is8 ? D : 2 * D, half = kKvTile * row;
  char *const ko = is8 ? (char *)(st.k8 + at) : (char *)(st.k16 + at), *const vo = is8 ? (char *)(st.v8 + at) : (char *)(st.v16 + at);
  for (int e = threadIdx.x * 16; e < half; e += 4096) {
    const pc::u32x4 k = *(const pc::u32x4 *)(image + e), v = *(const pc::u32x4 *)(image + Image<D>::HALF + e);
    if (e / row < n) *(pc::u32x4 *)(ko + e) = k;
    *(pc::u32x4 *)(vo + e) = v;
  }
  if (is8 && threadIdx.x < 2) (threadIdx.x ? st.v_scale : st.k_scale)[head * (C / kKvTile) + tile] = ((const float *)(image + 2 * Image<D>::HALF))[threadIdx.x];
}

size_t image_bytes(int head_dim) { return head_dim == 128 ? Image<128>::BYTES : Image<64>::BYTES; }

}  // namespace

extern "C" {

size_t percache_kv_keep_workspace_bytes(const percache_ctx *ctx, int32_t n, int32_t max_keep) {
  if (!ctx || n < 1 || max_keep < 1) return 0;
  const percache_config &c = ctx->cfg;
  return pc::align_up((size_t)n * c.n_kv_heads * max_keep * sizeof(int32_t)) + (size_t)n * c.n_kv_heads * ((max_keep + kKvTile - 1) / kKvTile) * image_bytes(c.head_dim);
}

pc_status percache_kv_keep(percache_ctx *ctx, int32_t layer, const int32_t *slots_host, const int32_t *dst_slots_host, int32_t n, const int32_t *keep_host,
                           int32_t n_first, int32_t n_last, float *weights_dev, int32_t *idx_out_dev, void *workspace_dev, size_t workspace_bytes, void *stream) {
  if (!ctx) return PC_EINVAL;
  const percache_config &c = ctx->cfg;
  if (!slots_host || !keep_host || n < 1) return pc::fail(ctx, PC_EINVAL, "slots_host or keep_host is NULL, or n < 1");
  if (!weights_dev) return pc::fail(ctx, PC_EINVAL, "weights_dev is NULL");
  if (((uintptr_t)weights_dev | (uintptr_t)idx_out_dev) % 4) return pc::fail(ctx, PC_EINVAL, "weights_dev and idx_out_dev must be 4-byte aligned");
  if (layer < 0 || layer >= c.n_layers) return pc::fail(ctx, PC_ESLOT, "layer %d out of range [0,%d)", layer, c.n_layers);
  if (n_first < 0 || n_last < 0) return pc::fail(ctx, PC_EINVAL, "n_first and n_last must not be negative");
  const int32_t *dst = dst_slots_host ? dst_slots_host : slots_host;
  std::vector<char> named(c.n_slots, 0);   // 1: source, 2: destination
  int max_keep = 0;
  for (int i = 0; i < n; ++i) {
    for (int slot : {slots_host[i], dst[i]})
      if (slot < 0 || slot >= c.n_slots) return pc::fail(ctx, PC_ESLOT, "slot %d out of range [0,%d)", slot, c.n_slots);
    if (ctx->slot_len[(size_t)layer * c.n_slots + slots_host[i]] <= 0) return pc::fail(ctx, PC_ESLOT, "slot %d of layer %d is empty", slots_host[i], layer);
    if (keep_host[i] < 1 || keep_host[i] > c.slot_capacity) return pc::fail(ctx, PC_ELEN, "keep[%d]=%d outside [1,%d]", i, keep_host[i], c.slot_capacity);
    if ((long)n_first + n_last > keep_host[i]) return pc::fail(ctx, PC_EINVAL, "keep[%d]=%d is less than n_first %d + n_last %d", i, keep_host[i], n_first, n_last);
    if (named[slots_host[i]]) return pc::fail(ctx, PC_EINVAL, "slot %d appears twice", slots_host[i]);
    named[slots_host[i]] = 1;
    if (dst[i] != slots_host[i]) {
      if (named[dst[i]]) return pc::fail(ctx, PC_EINVAL, "slot %d appears twice", dst[i]);
      named[dst[i]] = 2;
    }
    if (keep_host[i] > max_keep) max_keep = keep_host[i];
  }
  if ((long)n * c.n_kv_heads * max_keep * c.head_dim >= (1L << 31)) return pc::fail(ctx, PC_ESHAPE, "more than 2^31 elements are kept");
  const size_t need = percache_kv_keep_workspace_bytes(ctx, n, max_keep);
  if (!workspace_dev || workspace_bytes < need) return pc::fail(ctx, PC_ENOMEM, "workspace has %zu bytes, need %zu", workspace_bytes, need);
  if ((uintptr_t)workspace_dev % pc::kAlign) return pc::fail(ctx, PC_EINVAL, "workspace must be 256-byte aligned");
  char *p = (char *)workspace_dev;
  int32_t *idx = idx_out_dev ? idx_out_dev : (int32_t *)p;
  char *const images = p + pc::align_up((size_t)n * c.n_kv_heads * max_keep * sizeof(int32_t));
  const int tiles = (max_keep + kKvTile - 1) / kKvTile;
  hipStream_t s = (hipStream_t)stream;
  const size_t at16 = (size_t)layer * ctx->layer_stride, at8 = (size_t)layer * ctx->layer_stride8, sc = (size_t)layer * ctx->n_slots8 * c.n_kv_heads * (c.slot_capacity / kKvTile);
  const Store st = {ctx->k_store + at16, ctx->v_store + at16, ctx->k8_store + at8, ctx->v8_store + at8, ctx->k_scale + sc, ctx->v_scale + sc, ctx->n_slots16};
  std::vector<int32_t> left(n);
  for (int i0 = 0; i0 < n; i0 += kMaxMoves) {
    const int cnt = n - i0 < kMaxMoves ? n - i0 : kMaxMoves;
    Moves mv;
    bool in_place = false;
    for (int i = 0; i < cnt; ++i) {
      mv.src[i] = slots_host[i0 + i];
      mv.dst[i] = dst[i0 + i];
      mv.have[i] = ctx->slot_len[(size_t)layer * c.n_slots + mv.src[i]];
      mv.keep[i] = keep_host[i0 + i];
      in_place |= mv.src[i] == mv.dst[i];
      left[i0 + i] = mv.have[i] < mv.keep[i] ? mv.have[i] : mv.keep[i];
    }
    const size_t first = (size_t)i0 * c.n_kv_heads * max_keep;
    hipLaunchKernelGGL(keep_select_kernel, dim3(c.n_kv_heads, cnt), dim3(kSelThreads), 0, s, weights_dev, mv, c.n_kv_heads, c.slot_capacity, n_first, n_last, idx + first, max_keep);
    PC_HIP(ctx, hipGetLastError());
    const dim3 grid(tiles, c.n_kv_heads, cnt);
    char *const im = images + (size_t)i0 * c.n_kv_heads * tiles * image_bytes(c.head_dim);
#define PC_KEEP(DD)                                                                                                                                        \
  do {                                                                                                                                                     \
    hipLaunchKernelGGL(keep_move_kernel<DD>, grid, dim3(256), 0, s, st, mv, idx + first, max_keep, c.n_kv_heads, c.slot_capacity, im, tiles);                \
    if (in_place) hipLaunchKernelGGL(keep_place_kernel<DD>, grid, dim3(256), 0, s, st, mv, c.n_kv_heads, c.slot_capacity, im, tiles);                       \
  } while (0)
    if (c.head_dim == 128) PC_KEEP(128); else PC_KEEP(64);
#undef PC_KEEP
    PC_HIP(ctx, hipGetLastError());
  }
  for (int i = 0; i < n; ++i) ctx->slot_len[(size_t)layer * c.n_slots + dst[i]] = left[i];
  return PC_OK;
}

}  // extern "C"
