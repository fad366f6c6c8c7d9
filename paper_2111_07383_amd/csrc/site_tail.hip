// Tail of a residual block, forward and backward (formulas in include/ssconv.h): the norm of the convolution's output,
// the gate, the residual scale and sum, and the norm in front of the next block, in one pass over the rows.
//
// Bound: memory. Every array is read or written once, 16 bytes a lane (site_row.hpp says how rows lie in registers);
// what a gate's lane owes its field's lanes goes through LDS, and back in the gradient.
#include "site_row.hpp"

namespace ssconv {
namespace {

template <typename T, int L, int K, bool RAG>
__global__ __launch_bounds__(kSiteNT) void tail_fwd_kernel(SiteTab t, TailArgs a) {
  extern __shared__ float lds[];
  using R = Row<L, K, RAG>;
  R w;
  w.init(t, t.n);
  const int C = t.C, S = t.ch0[t.n], By = t.b0[t.n], Bh = t.b0[t.n_regular], G = t.G;
  float* sig = lds + ((threadIdx.x >> 6) * R::R + w.sub) * G;  // the row's gates
  f8 gp[K], sc[K], gn[K];
  w.params(a.gain_post, gp, t.n);
  w.params(a.scale, sc, t.n_regular);
  w.params(a.gain_next, gn, t.n_regular);
  bool main[K];  // a chunk of the fields, not of the gates
#pragma unroll
  for (int k = 0; k < K; ++k) main[k] = w.hi[k] > 0 && w.e[k] < t.n_regular;
  const int64_t step = (int64_t)gridDim.x * (kSiteNT / L);
  for (int64_t r0 = ((int64_t)blockIdx.x * (kSiteNT / 64) + (threadIdx.x >> 6)) * R::R; r0 < a.n; r0 += step) {
    const bool on = r0 + w.sub < a.n;
    const int64_t row = on ? r0 + w.sub : a.n - 1;
    f8 y[K], h[K];
    float r[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      y[k] = w.template load<T>((const T*)a.y.data + row * S, k);
      h[k] = f8{0, 0, 0, 0, 0, 0, 0, 0};
      if (main[k]) h[k] = w.template load<T>((const T*)a.h.data + row * C, k);
    }
    if (a.yq) w.pack(y, a.yq + row * S, a.ye + row * By, t.n, on);
    w.norm(y, r, a.eps);
#pragma unroll
    for (int k = 0; k < K; ++k) y[k] *= gp[k];
    if (G) {
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (w.hi[k] > 0 && !main[k])
#pragma unroll
          for (int c = 0; c < 8; ++c)
            if (c < w.hi[k]) sig[w.start[k] - C + c] = sigmoid_of(y[k][c]);
      wave_lds_fence();
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (!main[k]) continue;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        float g = y[k][c];
        if (w.scalar[k])
          g = g <= 0.f ? 0.f : g;  // NaN stays
        else if (!RAG || c < w.hi[k])
          g *= sig[w.gate[k] + w.field(k, c)];
        h[k][c] = fmaf(sc[k][c], g, h[k][c]);
      }
      h[k] = round8<T>(h[k]);
      if (on) w.template store<T>((T*)a.h_out + row * C, k, h[k]);
    }
    if (G) wave_lds_fence();
    if (a.hq) w.pack(h, a.hq + row * C, a.he + row * Bh, t.n_regular, on);
    if (a.x_out) {
      w.norm(h, r, a.eps);
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (on && main[k]) w.template store<T>((T*)a.x_out + row * C, k, h[k] * gn[k]);
    }
  }
}

template <typename T, int L, int K, bool RAG>
__global__ __launch_bounds__(kSiteNT) void tail_bwd_kernel(SiteTab t, TailArgs a) {
  extern __shared__ float lds[];
  using R = Row<L, K, RAG>;
  R w;
  w.init(t, t.n);
  const int C = t.C, S = t.ch0[t.n], By = t.b0[t.n], Bh = t.b0[t.n_regular], G = t.G;
  float* sig = lds + ((threadIdx.x >> 6) * R::R + w.sub) * S;  // the row's gates, and behind them dg * u by channel
  float* prod = sig + G;
  f8 gp[K], sc[K], gn[K], acc_p[K], acc_s[K], acc_n[K];
  w.params(a.gain_post, gp, t.n);
  w.params(a.scale, sc, t.n_regular);
  w.params(a.gain_next, gn, t.n_regular);
  const f8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
  bool main[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    main[k] = w.hi[k] > 0 && w.e[k] < t.n_regular;
    acc_p[k] = acc_s[k] = acc_n[k] = zero;
  }
  const int64_t step = (int64_t)gridDim.x * (kSiteNT / L);
  for (int64_t r0 = ((int64_t)blockIdx.x * (kSiteNT / 64) + (threadIdx.x >> 6)) * R::R; r0 < a.n; r0 += step) {
    const bool on = r0 + w.sub < a.n;
    const int64_t row = on ? r0 + w.sub : a.n - 1;
    f8 y[K], h[K], dh[K], dx[K];
    float r[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      y[k] = a.y.exps ? w.load_packed((const int8_t*)a.y.data + row * S, a.y.exps + row * By, k)
                      : w.template load<T>((const T*)a.y.data + row * S, k);
      h[k] = dh[k] = dx[k] = zero;
      if (!main[k]) continue;
      dh[k] = w.template load<T>((const T*)a.dh + row * C, k);
      if (!a.dx) continue;
      dx[k] = w.template load<T>((const T*)a.dx + row * C, k);
      h[k] = a.h.exps ? w.load_packed((const int8_t*)a.h.data + row * C, a.h.exps + row * Bh, k)
                      : w.template load<T>((const T*)a.h.data + row * C, k);
    }
    if (a.dx) {
      w.norm(h, r, a.eps);
#pragma unroll
      for (int k = 0; k < K; ++k) {
        if (on) acc_n[k] += dx[k] * h[k];
        dx[k] *= gn[k];
      }
      w.norm_back(h, r, dx);
#pragma unroll
      for (int k = 0; k < K; ++k) dh[k] += dx[k];
    }
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (on && main[k]) w.template store<T>((T*)a.dh_in + row * C, k, dh[k]);
    w.norm(y, r, a.eps);
    if (G) {
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (w.hi[k] > 0 && !main[k])
#pragma unroll
          for (int c = 0; c < 8; ++c)
            if (c < w.hi[k]) sig[w.start[k] - C + c] = sigmoid_of(y[k][c] * gp[k][c]);
      wave_lds_fence();
    }
    f8 du[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      du[k] = zero;
      if (!main[k]) continue;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const float u = y[k][c] * gp[k][c];
        float f = u > 0.f ? 1.f : 0.f;
        if (!w.scalar[k] && (!RAG || c < w.hi[k])) f = sig[w.gate[k] + w.field(k, c)];
        const float dg = sc[k][c] * dh[k][c];
        if (on) acc_s[k][c] = fmaf(dh[k][c], f * u, acc_s[k][c]);
        du[k][c] = dg * f;
        if (!w.scalar[k] && (!RAG || c < w.hi[k])) prod[w.start[k] + c] = dg * u;
      }
    }
    if (G) {
      // a field's products make its gate's gradient; the fields of the row are shared out over its lanes
      wave_lds_fence();
      for (int e = 0; e < t.n_regular; ++e) {
        if (t.l[e] == 0) continue;
        const int d = 2 * t.l[e] + 1;
        for (int f = w.i; f < t.mult[e]; f += L) {
          float s = 0.f;
          for (int c = 0; c < d; ++c) s += prod[t.ch0[e] + f * d + c];
          const float sg = sig[t.gate0[e] + f];
          sig[t.gate0[e] + f] = s * (sg * (1.f - sg));
        }
      }
      wave_lds_fence();
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (w.hi[k] > 0 && !main[k])
#pragma unroll
          for (int c = 0; c < 8; ++c)
            if (c < w.hi[k]) du[k][c] = sig[w.start[k] - C + c];
      wave_lds_fence();
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (on) acc_p[k] += du[k] * y[k];
      du[k] *= gp[k];
    }
    w.norm_back(y, r, du);
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (on) w.template store<T>((T*)a.dy + row * S, k, du[k]);
  }
  if (a.part) {
    float* out = a.part + (int64_t)blockIdx.x * (S + 2 * C);
    sum_rows<L, K, RAG>(w, acc_p, S, lds, out);
    sum_rows<L, K, RAG>(w, acc_s, C, lds, out + S);
    sum_rows<L, K, RAG>(w, acc_n, C, lds, out + S + C);
  }
}

}  // namespace

int launch_tail_fwd(const SiteTab& t, ssconv_dtype dt, const TailArgs& a, hipStream_t st) {
  const unsigned nb = site_blocks(t, a.n, kFwdPerCu);
  const size_t lds = (size_t)site_rows(t) * t.G * 4;
  auto go = [&](auto kernel) {
    kernel<<<nb, kSiteNT, lds, st>>>(t, a);
    SSC_HIP(hipGetLastError());
    return (int)SSCONV_OK;
  };
#define SSK_GO(L_, K_, R_) \
  return dt == SSCONV_F32 ? go(tail_fwd_kernel<float, L_, K_, R_>) : go(tail_fwd_kernel<uint16_t, L_, K_, R_>)
  SSK_SITE_DISPATCH(t, SSK_GO);
#undef SSK_GO
}

int launch_tail_bwd(const SiteTab& t, ssconv_dtype dt, const TailArgs& a, hipStream_t st) {
  const unsigned nb = site_blocks(t, a.n, kBwdPerCu);
  const size_t lds = (size_t)site_rows(t) * t.ch0[t.n] * 4;
  auto go = [&](auto kernel) {
    kernel<<<nb, kSiteNT, lds, st>>>(t, a);
    SSC_HIP(hipGetLastError());
    return (int)SSCONV_OK;
  };
#define SSK_GO(L_, K_, R_) \
  return dt == SSCONV_F32 ? go(tail_bwd_kernel<float, L_, K_, R_>) : go(tail_bwd_kernel<uint16_t, L_, K_, R_>)
  SSK_SITE_DISPATCH(t, SSK_GO);
#undef SSK_GO
}

}  // namespace ssconv
