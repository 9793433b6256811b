// Rows of a QKV projection finished in one pass: bias, RMSNorm over each q and k head, rotation of q and k, and out by heads.
//   y = x + bias;  q, k: y <- y / sqrt(mean(y^2) + eps) * gain (where there is a gain), then pair (m, m + D/2) turned by
//   pos[axis(m)] * theta^(-2m/D);  one rounding to bf16.
// Positions come per row and axis (time, height, width of an image patch; one axis for text), axis(m) is the caller's choice, so that axes in
// sections and interleaved ones are the same to the kernel.
//
// What bounds it: the bytes, each read and written once, or the launch.  A group of D/16 lanes has a head of a row at a time, every lane 8 elements of
// its first half and the 8 that they are turned with, so a turn stays inside a lane, the mean takes two or three lane moves, and every access is
// 16 bytes a lane over whole 128-byte lines.  A group takes several heads of its row, which share the row's cosines and sines.
#include "percache_internal.hpp"

namespace {
using pc::bf16x8;

struct NormRopeArgs {
  const __bf16 *x, *bias, *q_norm, *k_norm;
  const int32_t *pos;        // [n_axes][rows]
  const float2 *rope;        // [max_pos][D/2]
  __bf16 *q, *k, *v;         // [heads][rows][D]
  long row_stride;           // elements
  int rows, n_axes, max_pos, Hq, Hkv;
  unsigned long long axis_lo, axis_hi;  // bits of the axis of every pair
  float eps;
};

// sum over the N = 8 or 4 neighbouring lanes of a head
template <int N>
__device__ __forceinline__ float head_sum(float x) {
#define PC_MOVE(ctrl) __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), ctrl, 0xf, 0xf, true))
  x += PC_MOVE(0xB1);                  // lane ^ 1
  x += PC_MOVE(0x4E);                  // lane ^ 2
  if (N == 8) x += PC_MOVE(0x141);     // mirrored inside 8
#undef PC_MOVE
  return x;
}

// HPG heads of a row for every group of lanes, their loads in flight together; ONCE: not kept in the caches
template <int D, int HPG, bool ONCE>
__global__ __launch_bounds__(256) void norm_rope_kernel(const NormRopeArgs a) {
  constexpr int N = D / 16;
  const int heads = a.Hq + 2 * a.Hkv, sets = (heads + HPG - 1) / HPG;
  const long group = ((long)blockIdx.x * 256 + threadIdx.x) / N;
  const int j = threadIdx.x % N;
  const long row = group / sets;
  if (row >= a.rows) return;   // (a group leaves as a whole: the lanes that exchange stay together)
  const int h0 = (int)(group - row * sets) * HPG;
  const __bf16 *x = a.x + row * a.row_stride + j * 8;

  bf16x8 lo[HPG], hi[HPG];
#pragma unroll
  for (int s = 0; s < HPG; ++s) {
    const int h = min(h0 + s, heads - 1);
    const bf16x8 *pl = (const bf16x8 *)(x + (long)h * D), *ph = (const bf16x8 *)(x + (long)h * D + D / 2);
    lo[s] = ONCE ? __builtin_nontemporal_load(pl) : *pl;
    hi[s] = ONCE ? __builtin_nontemporal_load(ph) : *ph;
  }
  float2 cs[8];
  if (h0 < a.Hq + a.Hkv) {
    int p[4];
#pragma unroll
    for (int ax = 0; ax < 4; ++ax) p[ax] = ax < a.n_axes ? a.pos[(size_t)ax * a.rows + row] : 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int m = j * 8 + e, ax = (int)(a.axis_lo >> m & 1) + 2 * (int)(a.axis_hi >> m & 1);
      const int at = ax == 0 ? p[0] : ax == 1 ? p[1] : ax == 2 ? p[2] : p[3];
      const bool in = at >= 0 && at < a.max_pos;
      cs[e] = a.rope[(size_t)(in ? at : 0) * (D / 2) + m];
      if (!in) cs[e] = make_float2(NAN, NAN);
    }
  }
#pragma unroll
  for (int s = 0; s < HPG; ++s) {
    const int h = h0 + s;
    if (h >= heads) return;
    float u[8], w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) { u[e] = (float)lo[s][e]; w[e] = (float)hi[s][e]; }
    if (a.bias) {
      const bf16x8 bl = *(const bf16x8 *)(a.bias + (size_t)h * D + j * 8), bh = *(const bf16x8 *)(a.bias + (size_t)h * D + D / 2 + j * 8);
#pragma unroll
      for (int e = 0; e < 8; ++e) { u[e] += (float)bl[e]; w[e] += (float)bh[e]; }
    }
    __bf16 *dst = h < a.Hq ? a.q + ((size_t)h * a.rows + row) * D : h < a.Hq + a.Hkv ? a.k + ((size_t)(h - a.Hq) * a.rows + row) * D
                                                                                     : a.v + ((size_t)(h - a.Hq - a.Hkv) * a.rows + row) * D;
    if (h < a.Hq + a.Hkv) {
      const __bf16 *gain = h < a.Hq ? a.q_norm : a.k_norm;
      if (gain) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += u[e] * u[e] + w[e] * w[e];
        const float r = 1.0f / sqrtf(head_sum<N>(sum) / (float)D + a.eps);
        const bf16x8 gl = *(const bf16x8 *)(gain + j * 8), gh = *(const bf16x8 *)(gain + D / 2 + j * 8);
#pragma unroll
        for (int e = 0; e < 8; ++e) { u[e] *= r * (float)gl[e]; w[e] *= r * (float)gh[e]; }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float b = u[e], c = w[e];
        u[e] = b * cs[e].x - c * cs[e].y;
        w[e] = c * cs[e].x + b * cs[e].y;
      }
    }
    bf16x8 ol, oh;
#pragma unroll
    for (int e = 0; e < 8; ++e) { ol[e] = (__bf16)u[e]; oh[e] = (__bf16)w[e]; }
    bf16x8 *dl = (bf16x8 *)(dst + j * 8), *dh = (bf16x8 *)(dst + D / 2 + j * 8);
    if (ONCE) {
      __builtin_nontemporal_store(ol, dl);
      __builtin_nontemporal_store(oh, dh);
    } else {
      *dl = ol;
      *dh = oh;
    }
  }
}
}  // namespace

extern "C" pc_status percache_qkv_norm_rope(percache_ctx *ctx, const void *qkv_dev, int64_t row_stride, int32_t n_rows, const int32_t *pos_dev,
                                            int32_t n_axes, const uint8_t *axis_host, const void *qkv_bias_dev, const void *q_norm_dev,
                                            const void *k_norm_dev, float eps, void *q_out_dev, void *k_out_dev, void *v_out_dev, void *stream) {
  if (!ctx) return PC_EINVAL;
  const percache_config &c = ctx->cfg;
  if (n_rows < 0) return pc::fail(ctx, PC_EINVAL, "n_rows is negative");
  if (n_axes < 1 || n_axes > 4) return pc::fail(ctx, PC_ESHAPE, "n_axes %d outside [1,4]", n_axes);
  if (!axis_host && n_axes != 1) return pc::fail(ctx, PC_EINVAL, "axis_host is NULL with %d axes", n_axes);
  const int half = c.head_dim / 2;
  NormRopeArgs a = {};
  for (int m = 0; axis_host && m < half; ++m) {
    if (axis_host[m] >= n_axes) return pc::fail(ctx, PC_EINVAL, "pair %d: axis %d outside [0,%d)", m, axis_host[m], n_axes);
    a.axis_lo |= (unsigned long long)(axis_host[m] & 1) << m;
    a.axis_hi |= (unsigned long long)(axis_host[m] >> 1) << m;
  }
  const long F = (long)(c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim;
  if (row_stride < F || row_stride % 8) return pc::fail(ctx, PC_EINVAL, "row stride %ld: a multiple of 8, at least %ld, is wanted", (long)row_stride, F);
  if (!(eps >= 0.f)) return pc::fail(ctx, PC_EINVAL, "eps must not be negative");
  if (n_rows == 0) return PC_OK;
  if (!qkv_dev || !pos_dev || !q_out_dev || !k_out_dev || !v_out_dev) return pc::fail(ctx, PC_EINVAL, "NULL tensor pointer");
  for (const void *p : {qkv_dev, qkv_bias_dev, q_norm_dev, k_norm_dev, (const void *)q_out_dev, (const void *)k_out_dev, (const void *)v_out_dev})
    if ((uintptr_t)p % 16) return pc::fail(ctx, PC_EINVAL, "tensor pointers must be 16-byte aligned");
  if ((uintptr_t)pos_dev % 4) return pc::fail(ctx, PC_EINVAL, "pos_dev must be 4-byte aligned");
  a.x = (const __bf16 *)qkv_dev;
  a.bias = (const __bf16 *)qkv_bias_dev;
  a.q_norm = (const __bf16 *)q_norm_dev;
  a.k_norm = (const __bf16 *)k_norm_dev;
  a.pos = pos_dev;
  a.rope = (const float2 *)ctx->rope;
  a.q = (__bf16 *)q_out_dev;
  a.k = (__bf16 *)k_out_dev;
  a.v = (__bf16 *)v_out_dev;
  a.row_stride = row_stride;
  a.rows = n_rows;
  a.n_axes = n_axes;
  a.max_pos = c.max_pos;
  a.Hq = c.n_q_heads;
  a.Hkv = c.n_kv_heads;
  a.eps = eps;
  const int heads = c.n_q_heads + 2 * c.n_kv_heads, lanes = c.head_dim / 16;
  hipStream_t s = (hipStream_t)stream;
  // A head for every group of lanes while that fills the chip; then several; past what the last-level cache holds, loads and stores that are not kept (48 heads
  // of 128, 4000 rows 20.4 us kept, 21.6 not; 8000 rows 40.0, 38.9; 16384 rows 84.6, 75.2 and with four heads a group 78: 5.4 TB/s, what a copy of 200 MB reaches).
  const long groups = (long)n_rows * heads;
  const int each = groups * lanes <= 64L * 16 * ctx->n_cu ? 1 : groups * c.head_dim * 4 <= 160L << 20 ? 4 : 2;
  const long blocks = ((long)n_rows * ((heads + each - 1) / each) * lanes + 255) / 256;
  if (blocks >= 1L << 24) return pc::fail(ctx, PC_ESHAPE, "%d rows of %d heads are 2^24 workgroups or more", n_rows, heads);   // (a grid has fewer than 2^32 threads)
#define PC_NR(DD, HH, OO) hipLaunchKernelGGL((norm_rope_kernel<DD, HH, OO>), dim3((unsigned)blocks), dim3(256), 0, s, a)
#define PC_NR_D(DD)                          \
  do {                                       \
    if (each == 1) PC_NR(DD, 1, false);      \
    else if (each == 4) PC_NR(DD, 4, false); \
    else PC_NR(DD, 2, true);                 \
  } while (0)
  if (c.head_dim == 128) PC_NR_D(128); else PC_NR_D(64);
#undef PC_NR_D
#undef PC_NR
  PC_HIP(ctx, hipGetLastError());
  return PC_OK;
}
