// Eviction inside a slot: of the tokens a slot holds, every kv head keeps the first n_first, the last n_last and, of those between, the ones
// that drew the most attention weight; the kept ones stay in order and close up.
//
// Selection is integer work on the order-preserving bits of the weights, so it is exact and the same on every run: a radix search for the
// smallest kept weight, 8 bits a pass over an LDS histogram, then one pass in the order of the tokens that takes everything above it and, of
// those equal to it, the first ones.
#include "percache_internal.hpp"

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

constexpr int kSelThreads = 256;
// One workgroup a (kv head, slot).  idx [n][Hkv][idx_stride]: the kept tokens in order, -1 behind them; weights are moved along.
__global__ __launch_bounds__(kSelThreads) void keep_select_kernel(float *weights, const Moves mv, int Hkv, int C, int n_first, int n_last, int32_t *idx, int idx_stride) {
  __shared__ unsigned hist[256];
  __shared__ unsigned found[2];                         // the digit, and how many tokens have a larger one
  __shared__ int wave_n[kSelThreads / 64][2];
  const int g = blockIdx.x, z = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int have = mv.have[z], keep = mv.keep[z];
  int32_t *out = idx + ((size_t)z * Hkv + g) * idx_stride;
  const float *w_src = weights + ((size_t)mv.src[z] * Hkv + g) * C;
  float *w_dst = weights + ((size_t)mv.dst[z] * Hkv + g) * C;
  const int lo = n_first, hi = have - n_last;           // the tokens that compete (keep < have: n_first + n_last <= keep < have)
  int need = keep >= have ? 0 : keep - n_first - n_last;
  unsigned top = 0, mask = 0;                           // the digits found so far
  if (keep < have) {
    for (int shift = 24; shift >= 0 && need > 0; shift -= 8) {
      hist[tid] = 0;
      __syncthreads();
      for (int t = lo + tid; t < hi; t += kSelThreads) {
        const unsigned k = key_of(w_src[t]);
        if ((k & mask) == top) atomicAdd(&hist[k >> shift & 255], 1u);
      }
      __syncthreads();
      if (wave == 0) {   // the largest digit at which the tokens from the top reach `need`: lane l counts digits 255 - 4 l .. 252 - 4 l
        unsigned n[4], sum = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) sum += n[j] = hist[255 - 4 * lane - j];
        unsigned upto = sum;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
          const unsigned x = __shfl_up(upto, o, 64);
          if (lane >= o) upto += x;
        }
        unsigned before = upto - sum;
        if (before < (unsigned)need && upto >= (unsigned)need)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (before < (unsigned)need && before + n[j] >= (unsigned)need) {
              found[0] = 255 - 4 * lane - j;
              found[1] = before;
            }
            before += n[j];
          }
      }
      __syncthreads();
      top |= found[0] << shift;
      mask |= 255u << shift;
      need -= found[1];
      __syncthreads();
    }
  }
  // `need` tokens with the key `top` are kept, the first ones, and all with a larger key (keep >= have: every token)
  int at = 0, ties = 0;
  for (int t0 = 0; t0 < have; t0 += kSelThreads) {
    const int t = t0 + tid;
    bool in = false, tie = false;
    float w = 0.f;
    if (t < have) {
      w = w_src[t];
      const bool fixed = keep >= have || t < lo || t >= hi;
      const unsigned k = key_of(w);
      in = fixed || (mask && k > top);
      tie = !fixed && mask && k == top;
    }
    const unsigned long long tie_b = __ballot(tie), below = (1ull << lane) - 1;
    if (lane == 0) wave_n[wave][0] = __popcll(tie_b);
    __syncthreads();
    int tie_at = ties;
#pragma unroll
    for (int v = 0; v < kSelThreads / 64; ++v) {
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
    for (int v = 0; v < kSelThreads / 64; ++v) {
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

struct Store {
  const __bf16 *k16, *v16;
  const uint8_t *k8, *v8;
  const float *k_scale, *v_scale;
  int n_slots16;
};
// The kept tokens of every (slot, kv head) as dense rows [n][Hkv][rows][D]: what their slot reads back as (bf16, or code * 2^e).
template <int D>
__global__ __launch_bounds__(256) void keep_gather_kernel(Store st, const Moves mv, const int32_t *idx, int idx_stride, int Hkv, int C, __bf16 *dense_k, __bf16 *dense_v,
                                                          int rows) {
  const int z = blockIdx.z, g = blockIdx.y, slot = mv.src[z], n = min(mv.keep[z], mv.have[z]);
  const int32_t *list = idx + ((size_t)z * Hkv + g) * idx_stride;
  const bool is8 = slot >= st.n_slots16;
  const size_t head = (size_t)(is8 ? slot - st.n_slots16 : slot) * Hkv + g;
  const size_t drow = ((size_t)z * Hkv + g) * rows;
  for (int e = blockIdx.x * 256 + threadIdx.x; e < n * D; e += gridDim.x * 256) {
    const int j = e / D, d = e - j * D, t = list[j], blk = t / kKvTile, in = t % kKvTile;
    const size_t row = head * C + t, block = (head * C + (size_t)blk * kKvTile) * D;
    if (is8) {
      const size_t sc = head * (C / kKvTile) + blk;
      dense_k[(drow + j) * D + d] = (__bf16)(__builtin_amdgcn_cvt_f32_fp8(st.k8[row * D + d], 0) * st.k_scale[sc]);
      dense_v[(drow + j) * D + d] = (__bf16)(__builtin_amdgcn_cvt_f32_fp8(st.v8[block + (size_t)d * kKvTile + pc::blocked_pos8(in)], 0) * st.v_scale[sc]);
    } else {
      dense_k[(drow + j) * D + d] = st.k16[row * D + d];
      dense_v[(drow + j) * D + d] = st.v16[block + (size_t)d * kKvTile + (in & ~15) + pc::blocked_key(in & 15)];
    }
  }
}

}  // namespace

extern "C" {

size_t percache_kv_keep_workspace_bytes(const percache_ctx *ctx, int32_t n, int32_t max_keep) {
  if (!ctx || n < 1 || max_keep < 1) return 0;
  const percache_config &c = ctx->cfg;
  return pc::align_up((size_t)n * c.n_kv_heads * max_keep * sizeof(int32_t)) + 2 * pc::align_up((size_t)n * c.n_kv_heads * max_keep * c.head_dim * 2);
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
  const size_t list = (size_t)n * c.n_kv_heads * max_keep, dense = list * c.head_dim;
  int32_t *idx = idx_out_dev ? idx_out_dev : (int32_t *)p;
  p += pc::align_up(list * sizeof(int32_t));
  __bf16 *dk = (__bf16 *)p, *dv = (__bf16 *)(p + pc::align_up(dense * 2));
  hipStream_t s = (hipStream_t)stream;
  const size_t at16 = (size_t)layer * ctx->layer_stride, at8 = (size_t)layer * ctx->layer_stride8, sc = (size_t)layer * ctx->n_slots8 * c.n_kv_heads * (c.slot_capacity / kKvTile);
  const Store st = {ctx->k_store + at16, ctx->v_store + at16, ctx->k8_store + at8, ctx->v8_store + at8, ctx->k_scale + sc, ctx->v_scale + sc, ctx->n_slots16};
  std::vector<int32_t> bounds(n), left(n);
  for (int i0 = 0; i0 < n; i0 += kMaxMoves) {
    const int cnt = n - i0 < kMaxMoves ? n - i0 : kMaxMoves;
    Moves mv;
    for (int i = 0; i < cnt; ++i) {
      mv.src[i] = slots_host[i0 + i];
      mv.dst[i] = dst[i0 + i];
      mv.have[i] = ctx->slot_len[(size_t)layer * c.n_slots + mv.src[i]];
      mv.keep[i] = keep_host[i0 + i];
      left[i0 + i] = mv.have[i] < mv.keep[i] ? mv.have[i] : mv.keep[i];
    }
    const size_t first = (size_t)i0 * c.n_kv_heads * max_keep;
    hipLaunchKernelGGL(keep_select_kernel, dim3(c.n_kv_heads, cnt), dim3(kSelThreads), 0, s, weights_dev, mv, c.n_kv_heads, c.slot_capacity, n_first, n_last, idx + first, max_keep);
    PC_HIP(ctx, hipGetLastError());
    const dim3 grid((max_keep * c.head_dim + 2047) / 2048, c.n_kv_heads, cnt);
    if (c.head_dim == 128)
      hipLaunchKernelGGL(keep_gather_kernel<128>, grid, dim3(256), 0, s, st, mv, idx + first, max_keep, c.n_kv_heads, c.slot_capacity, dk + first * c.head_dim, dv + first * c.head_dim, max_keep);
    else
      hipLaunchKernelGGL(keep_gather_kernel<64>, grid, dim3(256), 0, s, st, mv, idx + first, max_keep, c.n_kv_heads, c.slot_capacity, dk + first * c.head_dim, dv + first * c.head_dim, max_keep);
    PC_HIP(ctx, hipGetLastError());
  }
  const pc_status put = pc::launch_kv_put_rows(ctx, layer, dst, left.data(), n, dk, dv, max_keep, s);
  if (put != PC_OK) return put;
  for (int i = 0; i < n; ++i) ctx->slot_len[(size_t)layer * c.n_slots + dst[i]] = left[i];
  return PC_OK;
}

}  // extern "C"
