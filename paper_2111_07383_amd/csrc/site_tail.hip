// Tail of a residual block, forward and backward (formulas in include/ssconv.h): the norm of the convolution's output,
// the gate, the residual scale and sum, and the norm in front of the next block, in one pass over the rows.
//
// Bound: memory. Every array is read or written once, 16 bytes a lane (site_row.hpp says how rows lie in registers);
// what a gate's lane owes its field's lanes goes through LDS, and back in the gradient.
#include "site_row.hpp"

namespace ssconv {
namespace {

constexpr f8 kZero = {0, 0, 0, 0, 0, 0, 0, 0}, kOne = {1, 1, 1, 1, 1, 1, 1, 1};

template <typename T, int L, int K, int RAG>
__global__ __launch_bounds__(kSiteNT, tail_fwd_per_cu(L, K, RAG)) void tail_fwd_kernel(SiteTab t, TailArgs a, int lds_row) {
  extern __shared__ __attribute__((aligned(32))) float lds[];
  using R = Row<L, K, RAG>;
  R w;
  Gates<L, K, RAG> gates;
  w.init(t, t.n);
  float unused[R::Q];
  gates.init(t, w.i, nullptr, unused);
  const int C = t.C, S = t.ch0[t.n], By = t.b0[t.n], Bh = t.b0[t.n_regular], G = t.G;
  float* buf = lds + ((threadIdx.x >> 6) * R::R + w.sub) * lds_row;
  f8 gp[K], sc[K], gn[K];
  w.params(a.gain_post, gp, t.f0[t.n]);
  w.params(a.scale, sc, t.f0[t.n_regular]);
  w.params(a.gain_next, gn, t.f0[t.n_regular]);
  bool main[K];  // a chunk of the fields, not of the gates
  int at[K];     // its place in a matrix without the gates
  float least[K];  // what is at most this becomes 0: relu of the scalars; nothing is at most NaN
#pragma unroll
  for (int k = 0; k < K; ++k) {
    main[k] = w.hi[k] > 0 && w.e < t.n_regular;
    at[k] = main[k] ? w.start[k] : 0;
    least[k] = w.scalar ? 0.f : __builtin_nanf("");
    if (G && main[k] && w.scalar) lds_put(w, k, buf, kOne);  // a scalar's factor, which nothing overwrites
  }
  const int64_t step = (int64_t)gridDim.x * (kSiteNT / L);
  for (int64_t r0 = first_row<R::R>(); r0 < a.n; r0 += step) {
    const bool on = w.sub < a.n - r0;
    const int row = w.row_of(a.n - r0);
    f8 y[K], h[K];
    float r, sig[R::Q];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      y[k] = w.template load<T>((const T*)a.y.data + r0 * S, row, S, k, w.start[k]);
      h[k] = kZero;
      if (RAG < 3 || main[k]) h[k] = w.template load<T>((const T*)a.h.data + r0 * C, row, C, k, at[k]);
    }
    if (a.yq) w.pack(y, a.yq + r0 * S, a.ye + r0 * By, row, S, By, t.n, on);
    w.norm(y, r, a.eps);
    if (G) {
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (w.hi[k] > 0 && !main[k]) lds_put(w, k, buf, y[k] * gp[k]);
      wave_lds_fence();
      gates.open(buf, S, sig);
      wave_lds_fence();
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const f8 f = G ? lds_get(w, k, buf) : kOne;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const float u = y[k][c] * gp[k][c], g = u <= least[k] ? 0.f : f[c] * u;  // NaN stays
        h[k][c] = fmaf(sc[k][c], g, h[k][c]);
      }
      h[k] = round8<T>(h[k]);
      if (on && main[k]) w.template store<T>((T*)a.h_out + r0 * C, row, C, k, h[k]);
    }
    if (G) wave_lds_fence();
    if (a.hq) w.pack(h, a.hq + r0 * C, a.he + r0 * Bh, row, C, Bh, t.n_regular, on);
    if (a.x_out) {
      w.norm(h, r, a.eps);
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (on && main[k]) w.template store<T>((T*)a.x_out + r0 * C, row, C, k, h[k] * gn[k]);
    }
  }
}

// With e = dh times the gate's factor (1 or 0 for a scalar; a gate channel's own gradient there), the gradients of both
// parameters of the block's output are the same sum over the rows: dscale = gain_post sum(e yhat),
// dgain_post = scale sum(e yhat); and what goes on behind the norm is scale gain_post e.  The components of a field
// share both parameters, so its gate's lane multiplies their sum of dh u by the scale.
template <typename T, int L, int K, int RAG, bool PK>
__global__ __launch_bounds__(kSiteNT, tail_bwd_per_cu(L, K, RAG)) void tail_bwd_kernel(SiteTab t, TailArgs a, int lds_row) {
  extern __shared__ __attribute__((aligned(32))) float lds[];
  using R = Row<L, K, RAG>;
  R w;
  Gates<L, K, RAG> gates;
  w.init(t, t.n);
  float gate_scale[R::Q];
  gates.init(t, w.i, a.scale, gate_scale);
  const int C = t.C, S = t.ch0[t.n], By = t.b0[t.n], Bh = t.b0[t.n_regular], G = t.G;
  float* buf = lds + ((threadIdx.x >> 6) * R::R + w.sub) * lds_row;
  f8 gp[K], sc[K], gn[K], acc[K], acc_n[K];
  w.params(a.gain_post, gp, t.f0[t.n]);
  w.params(a.scale, sc, t.f0[t.n_regular]);
  w.params(a.gain_next, gn, t.f0[t.n_regular]);
  bool main[K];
  int at[K], blk[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    main[k] = w.hi[k] > 0 && w.e < t.n_regular;
    at[k] = main[k] ? w.start[k] : 0;
    blk[k] = main[k] ? w.blk[k] : 0;
    sc[k] = main[k] ? sc[k] * gp[k] : gp[k];
    acc[k] = acc_n[k] = kZero;
    if (G && main[k] && w.scalar) lds_put(w, k, buf, kOne);  // a scalar's factor, which nothing overwrites
  }
  const int64_t step = (int64_t)gridDim.x * (kSiteNT / L);
  for (int64_t r0 = first_row<R::R>(); r0 < a.n; r0 += step) {
    const bool on = w.sub < a.n - r0;
    const int row = w.row_of(a.n - r0);
    f8 y[K], e[K], h[K], dx[K];
    float r, ys[K], hs[K], sig[R::Q];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      y[k] = w.template load_rows<T, PK>(a.y, r0, row, S, By, k, w.start[k], w.blk[k], ys[k]);
      e[k] = h[k] = dx[k] = kZero;
      hs[k] = 1.f;
      if (RAG == 3 && !main[k]) continue;
      e[k] = w.template load<T>((const T*)a.dh + r0 * C, row, C, k, at[k]);
      if (!a.dx) continue;
      dx[k] = w.template load<T>((const T*)a.dx + r0 * C, row, C, k, at[k]);
      h[k] = w.template load_rows<T, PK>(a.h, r0, row, C, Bh, k, at[k], blk[k], hs[k]);
    }
    const bool part = a.n - r0 < R::R;  // a row read a second time adds nothing to the parameters' gradients
    if (part && !on)
#pragma unroll
      for (int k = 0; k < K; ++k) e[k] = dx[k] = kZero;
    if (a.dx) {
      w.norm(h, hs, r, a.eps);
#pragma unroll
      for (int k = 0; k < K; ++k) {
#pragma unroll
        for (int c = 0; c < 8; ++c) acc_n[k][c] = fmaf(dx[k][c], h[k][c], acc_n[k][c]);
        dx[k] *= gn[k];
      }
      w.norm_back(h, r, dx);
#pragma unroll
      for (int k = 0; k < K; ++k) e[k] += dx[k];
    }
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (on && main[k]) w.template store<T>((T*)a.dh_in + r0 * C, row, C, k, e[k]);
    w.norm(y, ys, r, a.eps);
    if (G) {
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (w.hi[k] > 0 && !main[k]) lds_put(w, k, buf, y[k] * gp[k]);
      wave_lds_fence();
      gates.open(buf, S, sig);
      wave_lds_fence();
    }
    // All factors are read before the first product is written: a chunk moved back shares channels with its neighbour,
    // which is another lane's where a lane has one chunk, and no lane's own addresses keep the compiler from starting a
    // lane's writes between its reads.  Chunks that are whole share nothing with another lane's.
    f8 f[K];
#pragma unroll
    for (int k = 0; k < K; ++k) f[k] = G ? lds_get(w, k, buf) : kOne;
    if (K > 1 || RAG) wave_lds_fence();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      f8 prod;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const float u = y[k][c] * gp[k][c];
        prod[c] = e[k][c] * u;
        e[k][c] = u > 0.f || !w.scalar ? e[k][c] * f[k][c] : 0.f;  // a closed relu stops infinities and NaN too
      }
      if (G && main[k] && !w.scalar) lds_put(w, k, buf, prod);
    }
    if (G) {
      wave_lds_fence();
      gates.close(buf, sig, gate_scale);
      wave_lds_fence();
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (w.hi[k] > 0 && !main[k]) e[k] = lds_get(w, k, buf);
      wave_lds_fence();
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
      for (int c = 0; c < 8; ++c) acc[k][c] = fmaf(e[k][c], y[k][c], acc[k][c]);
      e[k] *= sc[k];
    }
    w.norm_back(y, r, e);
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (on) w.template store<T>((T*)a.dy + r0 * S, row, S, k, e[k]);
  }
  if (a.part || a.grad[0] || a.grad[1] || a.grad[2]) {
    float* out = a.part ? a.part + (int64_t)blockIdx.x * (S + 2 * C) : nullptr;
    f8 s[K];
    w.params(a.scale, s, t.f0[t.n_regular]);
#pragma unroll
    for (int k = 0; k < K; ++k) s[k] = main[k] ? s[k] * acc[k] : acc[k], acc[k] *= gp[k];
    sum_rows<L, K, RAG>(w, s, S, lds, out, t, t.n, a.grad[0]);
    sum_rows<L, K, RAG>(w, acc, C, lds, out ? out + S : nullptr, t, t.n_regular, a.grad[1]);
    sum_rows<L, K, RAG>(w, acc_n, C, lds, out ? out + S + C : nullptr, t, t.n_regular, a.grad[2]);
  }
}

}  // namespace

int launch_tail_fwd(const SiteTab& t, ssconv_dtype dt, const TailArgs& a, hipStream_t st) {
  const unsigned nb = site_blocks(t, a.n, tail_fwd_per_cu);
  const int lds_row = site_lds_row(t);
  const size_t lds = t.G ? (size_t)site_rows(t) * lds_row * 4 : 0;
  auto go = [&](auto kernel) {
    kernel<<<nb, kSiteNT, lds, st>>>(t, a, lds_row);
    SSC_HIP(hipGetLastError());
    return (int)SSCONV_OK;
  };
#define SSK_GO(L_, K_, R_) \
  return dt == SSCONV_F32 ? go(tail_fwd_kernel<float, L_, K_, R_>) : go(tail_fwd_kernel<uint16_t, L_, K_, R_>)
  SSK_SITE_DISPATCH(t, SSK_GO);
#undef SSK_GO
}

int launch_tail_bwd(const SiteTab& t, ssconv_dtype dt, const TailArgs& a, hipStream_t st) {
  const unsigned nb = bwd_blocks(t, a.n, tail_bwd_per_cu);
  const int lds_row = site_lds_row(t);
  const size_t lds = (size_t)site_rows(t) * lds_row * 4;
  auto go = [&](auto kernel) {
    kernel<<<nb, kSiteNT, lds, st>>>(t, a, lds_row);
    SSC_HIP(hipGetLastError());
    return (int)SSCONV_OK;
  };
#define SSK_GO(L_, K_, R_) \
  return a.y.exps ? dt == SSCONV_F32 ? go(tail_bwd_kernel<float, L_, K_, R_, true>)       \
                                     : go(tail_bwd_kernel<uint16_t, L_, K_, R_, true>)    \
         : dt == SSCONV_F32 ? go(tail_bwd_kernel<float, L_, K_, R_, false>)                \
                            : go(tail_bwd_kernel<uint16_t, L_, K_, R_, false>)
  SSK_SITE_DISPATCH(t, SSK_GO);
#undef SSK_GO
}

}  // namespace ssconv
