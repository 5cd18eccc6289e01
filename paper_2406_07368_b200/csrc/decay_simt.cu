// The recurrence with a decay in fp32 on the CUDA cores, chunkwise, for fp32 inputs: chunks of 64 tokens, every product an
// fp32 multiply-add on register tiles fed by 128-bit shared-memory loads (twelve loads for 128 multiply-adds).  Per chunk of n
// tokens, X the state before it (Fade: lam^n):
//   P_ij = r upd lam^(i-j) q_i . k_j  (j <= i),   o_i = r lam^(i+1) q_i^T X + sum_j P_ij v_j
//   k_j <- upd lam^(n-1-j) k_j,                   X <- lam^n X + sum_j k_j v_j^T
// Rows are loaded in the order of the sweep, so that a sweep backwards in time is a sweep forwards in here.  X stays in
// registers, with a copy in shared memory for Q X.  Bound by the multiply-adds (of P only the blocks that the mask leaves
// are formed; P V stops at the diagonal, which also keeps a v that is not finite away from earlier tokens).
// Few chains of a long sequence are cut over a cluster of up to 8 blocks, as in the tensor-core kernel: each block first
// forms the sum of its own segment, and those before it are read through distributed shared memory.
#include "decay.cuh"

namespace la {
namespace dsm {

constexpr int C = 64, kMaxSeg = 8;
constexpr int R = 8;                                 // rows of P and o per thread
template <int D> __host__ __device__ constexpr int threads() { return C / R * (D / 4); }
constexpr int PS = C + 4;                            // row stride of P; of q, k, v: D + 4 (eight rows in a row lie on different banks)
template <int D> struct Smem {
  float q[C][D + 4], k[C][D + 4], v[C][D + 4], p[C][PS];
  float X[D][D];
  float pw[C + 1];                                   // lam^n
};

__device__ __forceinline__ void cluster_sync() { asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ float4 ld_cluster(const void* p, int rank) {
  uint32_t a = (uint32_t)__cvta_generic_to_shared(p), r;
  float4 v;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(r) : "memory");
  return v;
}
__device__ __forceinline__ void get4(const float* p, float (&x)[4]) {
  const float4 v = *reinterpret_cast<const float4*>(p);
  x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
}

// y += f x for four columns: two packed multiply-adds (each half rounds as the scalar instruction does).
__device__ __forceinline__ void add4(float2 (&y)[2], float f, const float (&x)[4]) {
  const float2 ff = make_float2(f, f);
  y[0] = __ffma2_rn(ff, make_float2(x[0], x[1]), y[0]);
  y[1] = __ffma2_rn(ff, make_float2(x[2], x[3]), y[1]);
}

template <int D>
__global__ void __launch_bounds__(threads<D>(), D == 64 ? 2 : 1)
decay_simt_kernel(const DecayPasses ps, const float* __restrict__ log_decay, const int32_t* __restrict__ lens,
                  int64_t* __restrict__ pos, int* status, int H, int Tlen, int nseg) {
  constexpr int NT = threads<D>(), TC = D / 4;       // threads; groups of 4 columns
  constexpr int S = C / R;                           // groups of rows; a thread's rows lie S apart
  constexpr int UJ = C / TC;                         // P: columns tc + TC u of a thread
  constexpr int XR = D * D / NT / 4;                 // rows of X per thread (4 columns each)
  extern __shared__ unsigned char smem_raw[];
  Smem<D>& sm = *reinterpret_cast<Smem<D>*>(smem_raw);
  const int tid = threadIdx.x;
  const int rank = (int)blockIdx.x % nseg, chain = (int)blockIdx.x / nseg, bh = chain / ps.n, b = bh / H, h = bh % H;
  const DecayPass& p = ps.p[chain % ps.n];
  pdl_wait();
  pdl_trigger();
  const float g = log_decay[h];
  const int L = seq_len(lens, b, Tlen);
  const bool bad = L < 0 || !decay_ok(g);            // (such a block still takes part in the cluster's barriers)
  if (pos && L > 0 && chain % ps.n == 0 && rank == 0 && h == 0 && tid == 0) pos[b] += L;
  if (bad && tid == 0) report(status, LA_ERR_INVALID_ARG);
  const int chunks = bad ? 0 : (L + C - 1) / C, seg = (chunks + nseg - 1) / nseg * C;
  const int n0 = min(max(L, 0), rank * seg), n1 = min(max(L, 0), n0 + seg);
  const float* q = (const float*)p.q.p + b * p.q.sb + h * p.q.sh;
  const float* k = (const float*)p.k.p + b * p.k.sb + h * p.k.sh;
  const float* v = (const float*)p.v.p + b * p.v.sb + h * p.v.sh;
  float* o = (float*)p.o.p + b * p.o.sb + h * p.o.sh;
  const size_t sbase = (size_t)bh * D * D;
  if (tid <= C) sm.pw[tid] = bad ? 0.f : decay_pow(g, tid);
  const Fade fade_c = decay_fade(bad ? 0.f : g, C);

  // A thread's place: 4 x 8 of them in a warp.
  // X: rows XR ti ..., columns 4 tc ...;  o: rows ti + C / R u, columns 4 tc ...;  P: rows ti + C / R u, columns tc + TC u.
  const int w = tid / 32, ti = w / (TC / 8) * 4 + tid % 32 / 8, tc = w % (TC / 8) * 8 + tid % 8;
  float2 X[XR][2];
#pragma unroll
  for (int i = 0; i < XR; ++i) X[i][0] = X[i][1] = make_float2(0.f, 0.f);

  auto row = [&](int n) { return (int64_t)(p.rev ? L - 1 - n : n); };
  auto load = [&](const float* x, int64_t st, float (*to)[D + 4], int at, int n) {   // asynchronous; rows from n on: zeros
#pragma unroll
    for (int i = 0; i < C * TC / NT; ++i) {
      const int r = i * (NT / TC) + tid / TC, c = tid % TC * 4;
      const uint32_t dst = (uint32_t)__cvta_generic_to_shared(&to[r][c]);
      const float* src = r < n ? x + row(at + r) * st + c : x;
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(r < n ? 16 : 0) : "memory");
    }
  };
  auto landed = [&] {
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
  };
  auto scale_k = [&](int n) {
#pragma unroll
    for (int i = 0; i < C * TC / NT; ++i) {
      const int r = i * (NT / TC) + tid / TC, c = tid % TC * 4;
      const float f = r < n ? p.upd * sm.pw[n - 1 - r] : 0.f;
      float4 x = *reinterpret_cast<float4*>(&sm.k[r][c]);
      *reinterpret_cast<float4*>(&sm.k[r][c]) = make_float4(x.x * f, x.y * f, x.z * f, x.w * f);
    }
  };
  auto add_kv = [&](const Fade& f) {                 // X = lam^n X + K^T V
#pragma unroll
    for (int i = 0; i < XR; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) X[i][j] = make_float2(f(X[i][j].x), f(X[i][j].y));
#pragma unroll 4
    for (int j = 0; j < C; ++j) {
      float kv[XR], vv[4];
#pragma unroll
      for (int i = 0; i < XR; i += 4) get4(&sm.k[j][XR * ti + i], *reinterpret_cast<float(*)[4]>(&kv[i]));
      get4(&sm.v[j][4 * tc], vv);
#pragma unroll
      for (int i = 0; i < XR; ++i) add4(X[i], kv[i], vv);
    }
  };
  auto put_x = [&] {
#pragma unroll
    for (int i = 0; i < XR; ++i) *reinterpret_cast<float4*>(&sm.X[XR * ti + i][4 * tc]) = make_float4(X[i][0].x, X[i][0].y, X[i][1].x, X[i][1].y);
  };

  // ---- the sum of the segment, and X before it ----
  if (nseg > 1) {
    if (rank < nseg - 1)
      for (int at = n0; at < n1; at += C) {
        const int n = min(C, n1 - at);
        __syncthreads();
        load(k, p.k.st, sm.k, at, n);
        load(v, p.v.st, sm.v, at, n);
        landed();
        scale_k(n);
        __syncthreads();
        add_kv(n == C ? fade_c : decay_fade(g, n));
      }
    put_x();
    cluster_sync();
  }
  if (p.S_in && !bad) {
#pragma unroll
    for (int i = 0; i < XR; ++i) {
      float y[4];
      if (p.trans) {
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = p.S_in[sbase + (size_t)(4 * tc + j) * D + XR * ti + i];
      } else {
        get4(p.S_in + sbase + (size_t)(XR * ti + i) * D + 4 * tc, y);
      }
      X[i][0] = make_float2(y[0], y[1]);
      X[i][1] = make_float2(y[2], y[3]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < XR; ++i) X[i][0] = X[i][1] = make_float2(0.f, 0.f);
  }
  if (nseg > 1) {
    for (int s = 0; s < rank; ++s) {
      const int ls = bad ? 0 : min(L, (s + 1) * seg) - min(L, s * seg);
      const Fade f = decay_fade(bad ? 0.f : g, ls > 0 ? ls - (s == 0 ? p.rev : 0) : 0);   // (backwards: the gradient as it is)
#pragma unroll
      for (int i = 0; i < XR; ++i) {
        const float4 y = ld_cluster(&sm.X[XR * ti + i][4 * tc], s);
        X[i][0] = make_float2(f(X[i][0].x) + y.x, f(X[i][0].y) + y.y);
        X[i][1] = make_float2(f(X[i][1].x) + y.z, f(X[i][1].y) + y.w);
      }
    }
    cluster_sync();                                  // everybody has read: the copies may change
  }

  for (int at = n0; at < n1; at += C) {
    const int n = min(C, n1 - at), e = p.rev && at == 0;
    put_x();
    if (at == n0) load(q, p.q.st, sm.q, at, n);
    load(k, p.k.st, sm.k, at, n);
    load(v, p.v.st, sm.v, at, n);
    landed();
    // ---- P; blocks of 8 rows and TC columns that lie behind the diagonal are not formed ----
    {
      float acc[R][UJ];
#pragma unroll
      for (int a = 0; a < R; ++a)
#pragma unroll
        for (int c = 0; c < UJ; ++c) acc[a][c] = 0.f;
#pragma unroll 2
      for (int d = 0; d < D; d += 4) {
        float qa[R][4], kc[UJ][4];
#pragma unroll
        for (int a = 0; a < R; ++a) get4(&sm.q[ti + S * a][d], qa[a]);
#pragma unroll
        for (int c = 0; c < UJ; ++c) get4(&sm.k[tc + TC * c][d], kc[c]);
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int a = 0; a < R; ++a)
#pragma unroll
            for (int c = 0; c < UJ; ++c)
              if (TC * c < S * a + S) acc[a][c] = fmaf(qa[a][x], kc[c][x], acc[a][c]);
      }
#pragma unroll
      for (int a = 0; a < R; ++a)
#pragma unroll
        for (int c = 0; c < UJ; ++c) {
          const int i = ti + S * a, j = tc + TC * c;
          if (TC * c < S * a + S) sm.p[i][j] = j <= i ? acc[a][c] * (p.r * p.upd * sm.pw[i - j]) : 0.f;
        }
    }
    __syncthreads();
    // ---- outputs: r lam^(i+1) Q X, then P V up to the diagonal ----
    {
      float2 acc[R][2];
#pragma unroll
      for (int u = 0; u < R; ++u) acc[u][0] = acc[u][1] = make_float2(0.f, 0.f);
#pragma unroll 2
      for (int a = 0; a < D; a += 4) {
        float qi[R][4], x[4][4];
#pragma unroll
        for (int u = 0; u < R; ++u) get4(&sm.q[ti + S * u][a], qi[u]);
#pragma unroll
        for (int j = 0; j < 4; ++j) get4(&sm.X[a + j][4 * tc], x[j]);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int u = 0; u < R; ++u) add4(acc[u], qi[u][j], x[j]);
      }
#pragma unroll
      for (int u = 0; u < R; ++u) {
        const float f = p.r * sm.pw[ti + S * u + 1 - e];
#pragma unroll
        for (int c = 0; c < 2; ++c) acc[u][c] = make_float2(acc[u][c].x * f, acc[u][c].y * f);
      }
      // 8 tokens at a time: rows of the same 8 as far as the diagonal, the rows behind them all
#pragma unroll
      for (int s = 0; s < R; ++s)
#pragma unroll
        for (int j0 = 0; j0 < S; j0 += 4) {
          float pu[R][4], x[4][4];
#pragma unroll
          for (int u = s; u < R; ++u) get4(&sm.p[ti + S * u][S * s + j0], pu[u]);
#pragma unroll
          for (int j = 0; j < 4; ++j) get4(&sm.v[S * s + j0 + j][4 * tc], x[j]);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (j0 + j <= ti) add4(acc[s], pu[s][j], x[j]);
#pragma unroll
            for (int u = s + 1; u < R; ++u) add4(acc[u], pu[u][j], x[j]);
          }
        }
#pragma unroll
      for (int u = 0; u < R; ++u)
        if (ti + S * u < n) *reinterpret_cast<float4*>(o + row(at + ti + S * u) * p.o.st + 4 * tc) = make_float4(acc[u][0].x, acc[u][0].y, acc[u][1].x, acc[u][1].y);
    }
    scale_k(n);                                      // (P has been formed: K as it was is not wanted any more)
    __syncthreads();
    if (at + C < n1) load(q, p.q.st, sm.q, at + C, min(C, n1 - at - C));   // (Q of this chunk has been read)
    add_kv(n - e == C ? fade_c : decay_fade(g, n - e));
    __syncthreads();
  }
  if (bad) return;
  for (int64_t i = (int64_t)L * TC + rank * NT + tid; i < (int64_t)Tlen * TC; i += (int64_t)nseg * NT)
    *reinterpret_cast<float4*>(o + i / TC * p.o.st + i % TC * 4) = make_float4(0.f, 0.f, 0.f, 0.f);   // rows behind the sequence
  if (p.S_out && rank == nseg - 1) {
    const Fade f = decay_fade(g, p.rev && L > 0 ? 1 : 0);
#pragma unroll
    for (int i = 0; i < XR; ++i)
      *reinterpret_cast<float4*>(p.S_out + sbase + (size_t)(XR * ti + i) * D + 4 * tc) = make_float4(f(X[i][0].x), f(X[i][0].y), f(X[i][1].x), f(X[i][1].y));
  }
}

}  // namespace dsm

cudaError_t launch_decay_simt(la_ctx* ctx, int B, int T, const DecayPasses& ps, const float* log_decay, const int32_t* lens,
                              int64_t* pos, cudaStream_t s) {
  const la_config& c = ctx->cfg;
  const int64_t chains = (int64_t)B * c.H * ps.n;
  const int chunks = (T + dsm::C - 1) / dsm::C, places = ctx->sm_count * (c.d == 64 ? 2 : 1);
  // (a segment's sum costs a third of its outputs)
  // (48 chains, d = 64, us, whole / 2 / 4: 128 tokens 19.9 / 15.8 / -, 256 37 / 28 / 25, 1000 143 / 99 / 74.)
  int nseg = 1;
  while (nseg < dsm::kMaxSeg && chains * nseg * 2 <= places && chunks >= nseg * 2) nseg *= 2;
  if (chains * nseg > INT32_MAX) return cudaErrorInvalidValue;
  auto kern = c.d == 64 ? dsm::decay_simt_kernel<64> : dsm::decay_simt_kernel<128>;
  const size_t smem = c.d == 64 ? sizeof(dsm::Smem<64>) : sizeof(dsm::Smem<128>);
  const cudaError_t e = allow_smem((const void*)kern, ctx->device);
  if (e != cudaSuccess) return e;
  ctx->launches += 1;
  return launch_cluster(nseg, true, kern, dim3((unsigned)(chains * nseg)), dim3(c.d == 64 ? dsm::threads<64>() : dsm::threads<128>()), smem, s, ps, log_decay, lens, pos,
                        ctx->d_status, c.H, T, nseg);
}

}  // namespace la
