// Norm of a site, forward and backward (formulas in include/ssconv.h), and the 8-bit checkpoints.
//
// Bound: memory. A row is read and written once, 16 bytes a lane (site_row.hpp says how rows lie in registers).
#include "site_row.hpp"

namespace ssconv {
namespace {

__device__ __forceinline__ void clear_words(const SplitFlags& f) {
  if (f.w && blockIdx.x == 0 && threadIdx.x < SplitFlags::kBytes / 4) f.w[threadIdx.x] = 0;
}

template <typename T, int L, int K, int RAG, bool PK>
__global__ __launch_bounds__(kSiteNT, norm_fwd_per_cu(L, K, RAG)) void norm_fwd_kernel(SiteTab t, NormArgs a) {
  using R = Row<L, K, RAG>;
  R w;
  clear_words(a.clear);
  w.init(t, t.n);
  const int C = t.ch0[t.n], B = t.b0[t.n];
  f8 g[K];
  w.params(a.gain, g, t.f0[t.n]);
  const int64_t step = (int64_t)gridDim.x * (kSiteNT / L);
  for (int64_t r0 = first_row<R::R>(); r0 < a.n; r0 += step) {
    const bool on = w.sub < a.n - r0;
    const int row = w.row_of(a.n - r0);
    f8 x[K];
    float r, xs[K];
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] = w.template load_rows<T, PK>(a.x, r0, row, C, B, k, w.start[k], w.blk[k], xs[k]);
    if (a.q) w.pack(x, a.q + r0 * C, a.exps + r0 * B, row, C, B, t.n, on);
    w.norm(x, xs, r, a.eps);
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (on) w.template store<T>((T*)a.out + r0 * C, row, C, k, x[k] * g[k]);
  }
}

template <typename T, int L, int K, int RAG, bool PK>
__global__ __launch_bounds__(kSiteNT, norm_bwd_per_cu(L, K, RAG)) void norm_bwd_kernel(SiteTab t, NormArgs a) {
  extern __shared__ float lds[];
  using R = Row<L, K, RAG>;
  R w;
  w.init(t, t.n);
  const int C = t.ch0[t.n], B = t.b0[t.n];
  f8 g[K], acc[K];
  w.params(a.gain, g, t.f0[t.n]);
#pragma unroll
  for (int k = 0; k < K; ++k) acc[k] = f8{0, 0, 0, 0, 0, 0, 0, 0};
  const int64_t step = (int64_t)gridDim.x * (kSiteNT / L);
  for (int64_t r0 = first_row<R::R>(); r0 < a.n; r0 += step) {
    const bool on = w.sub < a.n - r0;
    const int row = w.row_of(a.n - r0);
    f8 x[K], d[K], res[K];
    float r, xs[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      x[k] = w.template load_rows<T, PK>(a.x, r0, row, C, B, k, w.start[k], w.blk[k], xs[k]);
      d[k] = w.template load<T>((const T*)a.dy + r0 * C, row, C, k, w.start[k]);
      res[k] = f8{0, 0, 0, 0, 0, 0, 0, 0};
      if (a.dres) res[k] = w.template load<T>((const T*)a.dres + r0 * C, row, C, k, w.start[k]);
    }
    if (a.n - r0 < R::R)  // a row read a second time adds nothing
#pragma unroll
      for (int k = 0; k < K; ++k) d[k] = on ? d[k] : f8{0, 0, 0, 0, 0, 0, 0, 0};
    w.norm(x, xs, r, a.eps);
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
      for (int c = 0; c < 8; ++c) acc[k][c] = fmaf(d[k][c], x[k][c], acc[k][c]);
      d[k] *= g[k];
    }
    w.norm_back(x, r, d);
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (on) w.template store<T>((T*)a.out + r0 * C, row, C, k, d[k] + res[k]);
  }
  if (a.part || a.dgain)
    sum_rows<L, K, RAG>(w, acc, C, lds, a.part ? a.part + (int64_t)blockIdx.x * C : nullptr, t, t.n, a.dgain);
}

template <typename T, int L, int K, int RAG>
__global__ __launch_bounds__(kSiteNT, norm_fwd_per_cu(L, K, RAG)) void pack_kernel(SiteTab t, const T* x, int64_t n,
                                                                                   int8_t* q, uint8_t* exps) {
  using R = Row<L, K, RAG>;
  R w;
  w.init(t, t.n);
  const int C = t.ch0[t.n], B = t.b0[t.n];
  const int64_t step = (int64_t)gridDim.x * (kSiteNT / L);
  for (int64_t r0 = first_row<R::R>(); r0 < n; r0 += step) {
    const bool on = w.sub < n - r0;
    const int row = w.row_of(n - r0);
    f8 v[K];
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = w.template load<T>(x + r0 * C, row, C, k, w.start[k]);
    w.pack(v, q + r0 * C, exps + r0 * B, row, C, B, t.n, on);
  }
}

template <typename T, int L, int K, int RAG>
__global__ __launch_bounds__(kSiteNT, norm_fwd_per_cu(L, K, RAG)) void unpack_kernel(SiteTab t, const int8_t* q,
                                                                                     const uint8_t* exps, int64_t n, T* x,
                                                                                     SplitFlags clear) {
  using R = Row<L, K, RAG>;
  R w;
  clear_words(clear);
  w.init(t, t.n);
  const int C = t.ch0[t.n], B = t.b0[t.n];
  const int64_t step = (int64_t)gridDim.x * (kSiteNT / L);
  for (int64_t r0 = first_row<R::R>(); r0 < n; r0 += step) {
    if (w.sub < n - r0)
#pragma unroll
      for (int k = 0; k < K; ++k) {
        float s;
        const f8 v = w.load_packed(q + r0 * C, exps + r0 * B, w.sub, C, B, k, w.start[k], w.blk[k], s);
        w.template store<T>(x + r0 * C, w.sub, C, k, v * s);
      }
  }
}

}  // namespace

int launch_norm_fwd(const SiteTab& t, ssconv_dtype dt, const NormArgs& a, hipStream_t st) {
  const unsigned nb = site_blocks(t, a.n, norm_fwd_per_cu);
  auto go = [&](auto kernel) {
    kernel<<<nb, kSiteNT, 0, st>>>(t, a);
    SSC_HIP(hipGetLastError());
    return (int)SSCONV_OK;
  };
#define SSK_GO(L_, K_, R_) \
  return a.x.exps ? dt == SSCONV_F32 ? go(norm_fwd_kernel<float, L_, K_, R_, true>)       \
                                     : go(norm_fwd_kernel<uint16_t, L_, K_, R_, true>)    \
         : dt == SSCONV_F32 ? go(norm_fwd_kernel<float, L_, K_, R_, false>)                \
                            : go(norm_fwd_kernel<uint16_t, L_, K_, R_, false>)
  SSK_SITE_DISPATCH(t, SSK_GO);
#undef SSK_GO
}

int launch_norm_bwd(const SiteTab& t, ssconv_dtype dt, const NormArgs& a, hipStream_t st) {
  const unsigned nb = bwd_blocks(t, a.n, norm_bwd_per_cu);
  const size_t lds = a.part || a.dgain ? (size_t)site_rows(t) * t.ch0[t.n] * 4 : 0;
  auto go = [&](auto kernel) {
    kernel<<<nb, kSiteNT, lds, st>>>(t, a);
    SSC_HIP(hipGetLastError());
    return (int)SSCONV_OK;
  };
#define SSK_GO(L_, K_, R_) \
  return a.x.exps ? dt == SSCONV_F32 ? go(norm_bwd_kernel<float, L_, K_, R_, true>)       \
                                     : go(norm_bwd_kernel<uint16_t, L_, K_, R_, true>)    \
         : dt == SSCONV_F32 ? go(norm_bwd_kernel<float, L_, K_, R_, false>)                \
                            : go(norm_bwd_kernel<uint16_t, L_, K_, R_, false>)
  SSK_SITE_DISPATCH(t, SSK_GO);
#undef SSK_GO
}

int launch_pack(const SiteTab& t, ssconv_dtype dt, const void* x, int64_t n, int8_t* q, uint8_t* exps,
                hipStream_t st) {
  const unsigned nb = site_blocks(t, n, norm_fwd_per_cu);
  auto go = [&](auto kernel, auto* p) {
    kernel<<<nb, kSiteNT, 0, st>>>(t, p, n, q, exps);
    SSC_HIP(hipGetLastError());
    return (int)SSCONV_OK;
  };
#define SSK_GO(L_, K_, R_)                                                              \
  return dt == SSCONV_F32 ? go(pack_kernel<float, L_, K_, R_>, (const float*)x)         \
                          : go(pack_kernel<uint16_t, L_, K_, R_>, (const uint16_t*)x)
  SSK_SITE_DISPATCH(t, SSK_GO);
#undef SSK_GO
}

int launch_unpack(const SiteTab& t, ssconv_dtype dt, const int8_t* q, const uint8_t* exps, int64_t n, void* x,
                  const SplitFlags& clear, hipStream_t st) {
  const unsigned nb = site_blocks(t, n, norm_fwd_per_cu);
  auto go = [&](auto kernel, auto* p) {
    kernel<<<nb, kSiteNT, 0, st>>>(t, q, exps, n, p, clear);
    SSC_HIP(hipGetLastError());
    return (int)SSCONV_OK;
  };
#define SSK_GO(L_, K_, R_)                                                      \
  return dt == SSCONV_F32 ? go(unpack_kernel<float, L_, K_, R_>, (float*)x)     \
                          : go(unpack_kernel<uint16_t, L_, K_, R_>, (uint16_t*)x)
  SSK_SITE_DISPATCH(t, SSK_GO);
#undef SSK_GO
}

}  // namespace ssconv
