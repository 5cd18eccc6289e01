// Norms of the queries and keys of each head and the rotation by their positions, in one pass over both, and the
// gradients.  Bound by HBM: every row is read once and written once.
//
// A row of d values is held by d / 8 lanes, eight values each (one or two 128-bit loads), so that a warp works on two or
// four rows at a time and the mean over a row is a sum over 16 or 8 lanes.  A work item is a token and some of its 2 H
// rows (the q heads, then the k heads): the angles of a token are the same for all of them.  They are formed once per
// item, d / 2 of them spread over the warp's lanes, and passed on through shared memory:
//   turns = p (f / 2 pi) in 64 bits, minus its nearest integer; only that remainder, at most half a turn, goes to fp32
// (in 32 bits a position of 10^6 alone would leave an angle of the first pair wrong by 0.06).
#include "decay.cuh"

namespace la {
namespace nr {

constexpr int kThreads = 256, kWarps = kThreads / 32;

struct Args {
  const float *wq, *wk;
  const double* inv_freq;
  const int64_t* pos;
  float eps, mscale;
  int norm, rot, interleaved;
};

// cos and sin (times mscale) of the item's token, pair m at cs[m].
__device__ __forceinline__ void angles(const Args& a, int b, int t, int lane, float2* cs) {
  const double p = (double)((a.pos ? a.pos[b] : 0) + t);
  __syncwarp();                                    // (the item before has read its angles)
  for (int m = lane; m < a.rot / 2; m += 32) {
    const double turns = p * (a.inv_freq[m] * 0.15915494309189533577);
    float s, c;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
    cs[m] = make_float2(c * a.mscale, s * a.mscale);
  }
  __syncwarp();
}

// Rotates the row whose values 8 l ... 8 l + 7 are in lane l of a group of LPR lanes; sgn = -1: by minus the angle.
template <int LPR>
__device__ __forceinline__ void rotate(const Args& a, const float2* cs, int l, float sgn, float (&x)[8]) {
  const int first = 8 * l;
  if (a.interleaved) {
    if (first < a.rot) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 c = cs[first / 2 + i];
        const float s = sgn * c.y, u = x[2 * i], w = x[2 * i + 1];
        x[2 * i] = fmaf(u, c.x, -w * s);
        x[2 * i + 1] = fmaf(w, c.x, u * s);
      }
    }
    return;
  }
  const int half = a.rot / 16;                     // lanes of half the rotated values
  const int other = l < half ? l + half : l < 2 * half ? l - half : l;
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = __shfl_sync(0xffffffffu, x[i], other, LPR);
  if (l < 2 * half) {
    const float2* c = cs + 8 * (l < half ? l : other);
    const float sg = l < half ? -sgn : sgn;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = fmaf(x[i], c[i].x, y[i] * (sg * c[i].y));
  }
}

template <int LPR> __device__ __forceinline__ float row_sum(float x) {
#pragma unroll
  for (int o = LPR / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o, LPR);
  return x;
}
__device__ __forceinline__ int64_t at(const la_view& v, int b, int h, int t) { return b * v.sb + h * v.sh + t * v.st; }
__device__ __forceinline__ void weights(const float* w, int l, float (&x)[8]) {
  if (w) {
    Io8<float>::load(w + 8 * l, x);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 1.f;
  }
}

// parts: a token's rows are shared out over this many items
template <typename T, int D>
__global__ void __launch_bounds__(kThreads)
norm_rope_kernel(const Args a, const la_view q, const la_view k, const la_view qo, const la_view ko, int H, int Tlen,
                 int64_t items, int parts) {
  constexpr int LPR = D / 8, RPW = 32 / LPR;       // lanes per row, rows per warp
  __shared__ float2 cs_all[kWarps][D / 2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane % LPR, r0 = lane / LPR;
  float2* cs = cs_all[warp];
  pdl_wait();
  pdl_trigger();
  const int per = (2 * H + parts - 1) / parts;
  for (int64_t it = (int64_t)blockIdx.x * kWarps + warp; it < items; it += (int64_t)gridDim.x * kWarps) {
    const int64_t tok = it / parts;
    const int b = (int)(tok / Tlen), t = (int)(tok % Tlen), lo = (int)(it % parts) * per, hi = min(2 * H, lo + per);
    angles(a, b, t, lane, cs);
    for (int base = lo; base < hi; base += RPW) {
      const int row = base + r0;
      const bool live = row < hi, isk = row >= H;
      const int h = isk ? row - H : row;
      float x[8], w[8];
      if (live) {
        const la_view& v = isk ? k : q;
        Io8<T>::load((const T*)v.p + at(v, b, h, t) + 8 * l, x);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = 0.f;
      }
      if (a.norm) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(x[i], x[i], s);
        const float rs = 1.f / sqrtf(row_sum<LPR>(s) * (1.f / D) + a.eps);
        weights(isk ? a.wk : a.wq, l, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= rs * w[i];
      }
      rotate<LPR>(a, cs, l, 1.f, x);
      if (live) {
        const la_view& v = isk ? ko : qo;
        Io8<T>::store((T*)v.p + at(v, b, h, t) + 8 * l, x);
      }
    }
  }
}

// u = the rotation undone (its transpose, mscale included), xh = x rs:
//   dw += u xh,   dx = rs (w u - xh mean(w u xh)).
// Each warp keeps its part of dw in registers, the q rows and the k rows apart; a block adds up its warps' parts and
// writes them to its place in `part`.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads)
norm_rope_backward_kernel(const Args a, const la_view q, const la_view k, const la_view gq, const la_view gk, const la_view dq,
                          const la_view dk, float* __restrict__ part, int H, int Tlen, int64_t items, int parts) {
  constexpr int LPR = D / 8, RPW = 32 / LPR;
  __shared__ float2 cs_all[kWarps][D / 2];
  __shared__ float sums[kWarps][2][D];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane % LPR, r0 = lane / LPR;
  float2* cs = cs_all[warp];
  pdl_wait();
  pdl_trigger();
  float dw[2][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) dw[0][i] = dw[1][i] = 0.f;
  const int per = (2 * H + parts - 1) / parts;
  for (int64_t it = (int64_t)blockIdx.x * kWarps + warp; it < items; it += (int64_t)gridDim.x * kWarps) {
    const int64_t tok = it / parts;
    const int b = (int)(tok / Tlen), t = (int)(tok % Tlen), lo = (int)(it % parts) * per, hi = min(2 * H, lo + per);
    angles(a, b, t, lane, cs);
    for (int base = lo; base < hi; base += RPW) {
      const int row = base + r0;
      const bool live = row < hi, isk = row >= H;
      const int h = isk ? row - H : row;
      float x[8], u[8], w[8];
      if (live) {
        const la_view &v = isk ? k : q, &gv = isk ? gk : gq;
        Io8<T>::load((const T*)v.p + at(v, b, h, t) + 8 * l, x);
        Io8<T>::load((const T*)gv.p + at(gv, b, h, t) + 8 * l, u);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = u[i] = 0.f;
      }
      rotate<LPR>(a, cs, l, -1.f, u);
      if (a.norm) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(x[i], x[i], s);
        s = row_sum<LPR>(s);
        const float rs = live ? 1.f / sqrtf(s * (1.f / D) + a.eps) : 0.f;
        weights(isk ? a.wk : a.wq, l, w);
        float m = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[i] *= rs;
          const float d = u[i] * x[i];
          if (isk) dw[1][i] += d;
          else dw[0][i] += d;
          m = fmaf(w[i], d, m);
        }
        m = row_sum<LPR>(m) * (1.f / D);
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = rs * fmaf(w[i], u[i], -x[i] * m);
      }
      if (live) {
        const la_view& v = isk ? dk : dq;
        Io8<T>::store((T*)v.p + at(v, b, h, t) + 8 * l, u);
      }
    }
  }
  if (!part) return;
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float x = dw[s][i];
#pragma unroll
      for (int o = LPR; o < 32; o <<= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
      if (r0 == 0) sums[warp][s][8 * l + i] = x;
    }
  __syncthreads();
  if (threadIdx.x < 2 * D) {
    float x = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) x += (&sums[w][0][0])[threadIdx.x];
    part[(size_t)blockIdx.x * 2 * D + threadIdx.x] = x;
  }
}

// dwq, dwk = the blocks' parts added up, in the same order whatever ran when: 32 columns per block, a part in 8 per warp.
template <int D>
__global__ void __launch_bounds__(kThreads)
dw_sum_kernel(const float* __restrict__ part, int n, float* __restrict__ dwq, float* __restrict__ dwk) {
  __shared__ float sums[kWarps][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
  pdl_wait();
  pdl_trigger();
  float x = 0.f;
#pragma unroll 8
  for (int i = warp; i < n; i += kWarps) x += part[(size_t)i * 2 * D + col];
  sums[warp][lane] = x;
  __syncthreads();
  if (warp == 0) {
    x = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) x += sums[w][lane];
    if (col < D) dwq[col] = x;
    else dwk[col - D] = x;
  }
}

}  // namespace nr

namespace {

constexpr int kBlocksPerSm = 4;                    // of the backward kernel, each with a part of dw of its own

nr::Args pack(const la_norm_rope_args& a) {
  return {a.wq, a.wk, a.inv_freq, a.pos, a.eps, a.mscale, a.norm, a.rot, a.interleaved};
}
// A token's rows are shared out until every warp of the GPU has an item, or an item is down to as many rows as a warp
// takes at a time.
int share(const la_ctx* ctx, int64_t tokens, int rows_at_once) {
  const int64_t want = (int64_t)ctx->sm_count * 32;
  int parts = 1;
  while (parts * tokens < want && parts * rows_at_once < 2 * ctx->cfg.H) parts *= 2;
  return parts;
}

template <typename T, int D>
cudaError_t launch_fwd(la_ctx* ctx, int B, int T_, const la_norm_rope_args& a, const la_view& q, const la_view& k,
                       const la_view& qo, const la_view& ko, cudaStream_t s) {
  const int parts = share(ctx, (int64_t)B * T_, 256 / D);
  const int64_t items = (int64_t)B * T_ * parts, blocks = (items + nr::kWarps - 1) / nr::kWarps;
  ctx->launches += 1;
  return launch_pdl(nr::norm_rope_kernel<T, D>, dim3((unsigned)(blocks < ctx->sm_count * 8 ? blocks : ctx->sm_count * 8)), dim3(nr::kThreads), 0, s,
                    pack(a), q, k, qo, ko, ctx->cfg.H, T_, items, parts);
}

template <typename T, int D>
cudaError_t launch_bwd(la_ctx* ctx, int B, int T_, const la_norm_rope_args& a, const la_view& q, const la_view& k,
                       const la_view& gq, const la_view& gk, const la_view& dq, const la_view& dk, float* dwq, float* dwk,
                       float* scratch, cudaStream_t s) {
  const int parts = share(ctx, (int64_t)B * T_, 256 / D);
  const int64_t items = (int64_t)B * T_ * parts;
  int64_t blocks = (items + nr::kWarps - 1) / nr::kWarps;
  if (blocks > ctx->sm_count * kBlocksPerSm) blocks = ctx->sm_count * kBlocksPerSm;
  ctx->launches += 1;
  cudaError_t e = launch_pdl(nr::norm_rope_backward_kernel<T, D>, dim3((unsigned)blocks), dim3(nr::kThreads), 0, s, pack(a), q, k, gq,
                             gk, dq, dk, dwq ? scratch : nullptr, ctx->cfg.H, T_, items, parts);
  if (e != cudaSuccess || !dwq) return e;
  ctx->launches += 1;
  return launch_pdl(nr::dw_sum_kernel<D>, dim3(2 * D / 32), dim3(nr::kThreads), 0, s, (const float*)scratch, (int)blocks, dwq, dwk);
}

}  // namespace

size_t norm_rope_scratch_bytes(const la_ctx* ctx) { return (size_t)ctx->sm_count * kBlocksPerSm * 2 * ctx->cfg.d * sizeof(float); }

cudaError_t launch_norm_rope(la_ctx* ctx, int B, int T, const la_norm_rope_args& a, const la_view& q, const la_view& k,
                             const la_view& qo, const la_view& ko, cudaStream_t s) {
  if (ctx->cfg.io_dtype == LA_F32)
    return ctx->cfg.d == 64 ? launch_fwd<float, 64>(ctx, B, T, a, q, k, qo, ko, s) : launch_fwd<float, 128>(ctx, B, T, a, q, k, qo, ko, s);
  return ctx->cfg.d == 64 ? launch_fwd<__nv_bfloat16, 64>(ctx, B, T, a, q, k, qo, ko, s)
                          : launch_fwd<__nv_bfloat16, 128>(ctx, B, T, a, q, k, qo, ko, s);
}

cudaError_t launch_norm_rope_backward(la_ctx* ctx, int B, int T, const la_norm_rope_args& a, const la_view& q,
                                      const la_view& k, const la_view& gq, const la_view& gk, const la_view& dq,
                                      const la_view& dk, float* dwq, float* dwk, float* scratch, cudaStream_t s) {
  if (ctx->cfg.io_dtype == LA_F32)
    return ctx->cfg.d == 64 ? launch_bwd<float, 64>(ctx, B, T, a, q, k, gq, gk, dq, dk, dwq, dwk, scratch, s)
                            : launch_bwd<float, 128>(ctx, B, T, a, q, k, gq, gk, dq, dk, dwq, dwk, scratch, s);
  return ctx->cfg.d == 64 ? launch_bwd<__nv_bfloat16, 64>(ctx, B, T, a, q, k, gq, gk, dq, dk, dwq, dwk, scratch, s)
                          : launch_bwd<__nv_bfloat16, 128>(ctx, B, T, a, q, k, gq, gk, dq, dk, dwq, dwk, scratch, s);
}

}  // namespace la
