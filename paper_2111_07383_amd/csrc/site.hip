// Norm of a site and the tail of a residual block (norm, gate, residual scale and sum, next norm), forward and
// backward, from rows or from their 8-bit checkpoints.
//
// A site is one wavefront's: its row lies in LDS in fp32, the lanes take an entry's channels in turn, and a group's
// sums are butterflies over the wavefront.
#include <algorithm>

#include "site.hpp"

namespace ssconv {

int make_sitetab(const ssconv_fields* f, bool gated, SiteTab* t) {
  FieldTab ft;
  SSC_TRY(make_fieldtab(f, &ft));
  *t = SiteTab{};
  t->C = ft.ch0[ft.n];
  for (int e = 0; e < ft.n; ++e) {
    t->l[e] = ft.l[e];
    t->mult[e] = ft.mult[e];
    t->gate0[e] = t->G;
    if (ft.l[e] > 0) t->G += ft.mult[e];
  }
  t->n = ft.n;
  if (gated && t->G > 0) {
    if (ft.n >= SSCONV_MAX_ENTRIES) return fail(SSCONV_E_INVALID, "the gates need an entry of their own: at most %d entries", SSCONV_MAX_ENTRIES - 1);
    t->l[t->n] = 0;
    t->mult[t->n] = t->G;
    ++t->n;
  }
  int64_t ch = 0, fi = 0, b = 0;
  for (int e = 0; e < t->n; ++e) {
    const int64_t w = (int64_t)t->mult[e] * (2 * t->l[e] + 1);
    if (ch + w > kSiteMaxC) return fail(SSCONV_E_INVALID, "a row has at most %d channels", kSiteMaxC);
    t->ch0[e] = (int)ch;
    t->f0[e] = (int)fi;
    t->b0[e] = (int)b;
    ch += w;
    fi += t->mult[e];
    b += (w + kPackBlock - 1) / kPackBlock;
  }
  for (int e = t->n; e <= SSCONV_MAX_ENTRIES; ++e) t->ch0[e] = (int)ch, t->f0[e] = (int)fi, t->b0[e] = (int)b;
  return SSCONV_OK;
}

namespace {

constexpr int kSiteBlocks = 2048;  // workgroups of a backward call at most; each leaves a row of partial sums

__device__ __forceinline__ float sigmoidf(float x) { return 1.f / (1.f + __expf(-x)); }

__device__ __forceinline__ float wave_sum(float v) {
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// One row of a matrix of n_ch channels into LDS as fp32, values of a checkpoint where it is one.
template <typename T>
__device__ void load_row(const SiteTab& t, const ssconv_rows& x, int64_t row, float* v) {
  const int S = t.ch0[t.n];
  if (!x.exps) {
    const T* p = (const T*)x.data + row * S;
    for (int c = threadIdx.x; c < S; c += 64) v[c] = DT<T>::to_f(p[c]);
  } else {
    const int8_t* p = (const int8_t*)x.data + row * S;
    const uint8_t* b = x.exps + row * t.b0[t.n];
    for (int e = 0; e < t.n; ++e)
      for (int i = threadIdx.x; i < t.ch0[e + 1] - t.ch0[e]; i += 64)
        v[t.ch0[e] + i] = (float)p[t.ch0[e] + i] * pack_scale(b[t.b0[e] + i / kPackBlock]);
  }
  __syncthreads();
}

template <typename T>
__device__ void store_row(const float* v, int C, T* p) {
  for (int c = threadIdx.x; c < C; c += 64) p[c] = DT<T>::from_f(v[c]);
}

// The checkpoint of a row in LDS: a block of 32 channels is half a wavefront's.
__device__ void pack_row(const SiteTab& t, const float* v, int64_t row, int8_t* q, uint8_t* exps) {
  const int S = t.ch0[t.n];
  for (int e = 0; e < t.n; ++e) {
    const int w = t.ch0[e + 1] - t.ch0[e];
    for (int i0 = 0; i0 < w; i0 += 64) {
      const int i = i0 + threadIdx.x;
      const float x = i < w ? v[t.ch0[e] + i] : 0.f;
      uint32_t amax = __float_as_uint(x) & 0x7fffffffu;
      for (int d = 16; d > 0; d >>= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, d));
      const int byte = pack_byte(amax);
      if (i < w) q[row * S + t.ch0[e] + i] = byte == 255 ? 0 : (int8_t)(int)rintf(x * pack_inverse(byte));
      if (i < w && (i & 31) == 0) exps[row * t.b0[t.n] + t.b0[e] + i / kPackBlock] = (uint8_t)byte;
    }
  }
}

// v becomes xhat of its entry e; returns 1 / sqrt(variance + eps).
__device__ float norm_entry(const SiteTab& t, int e, float* v, float eps) {
  const int c0 = t.ch0[e], w = t.ch0[e + 1] - c0;
  const float m = (float)t.mult[e];
  float mu = 0.f;
  if (t.l[e] == 0) {
    float s = 0.f;
    for (int i = threadIdx.x; i < w; i += 64) s += v[c0 + i];
    mu = wave_sum(s) / m;
  }
  float s = 0.f;
  for (int i = threadIdx.x; i < w; i += 64) {
    const float d = v[c0 + i] - mu;
    s = fmaf(d, d, s);
  }
  const float r = 1.f / sqrtf(wave_sum(s) / m + eps);
  for (int i = threadIdx.x; i < w; i += 64) v[c0 + i] = (v[c0 + i] - mu) * r;
  return r;
}

__device__ __forceinline__ float param(const float* p, int f) { return p ? p[f] : 1.f; }

// dy becomes the gradient behind the norm of entry e, from xhat and r; the gain's products are added to acc.
__device__ void norm_entry_back(const SiteTab& t, int e, const float* xhat, float r, float* dy, const float* gain,
                                float* acc) {
  const int c0 = t.ch0[e], w = t.ch0[e + 1] - c0, d = 2 * t.l[e] + 1;
  const float m = (float)t.mult[e];
  float a = 0.f, b = 0.f;
  for (int i = threadIdx.x; i < w; i += 64) {
    const float g = dy[c0 + i], x = xhat[c0 + i];
    if (acc) acc[c0 + i] += g * x;
    const float tv = g * param(gain, t.f0[e] + i / d);
    dy[c0 + i] = tv;
    a += tv;
    b = fmaf(tv, x, b);
  }
  a = t.l[e] == 0 ? wave_sum(a) / m : 0.f;
  b = wave_sum(b) / m;
  for (int i = threadIdx.x; i < w; i += 64) dy[c0 + i] = r * (dy[c0 + i] - a - xhat[c0 + i] * b);
}

template <typename T>
__global__ __launch_bounds__(64) void site_norm_fwd(SiteTab t, ssconv_rows x, int64_t n, float eps,
                                                    const float* __restrict__ gain, T* y, int8_t* q, uint8_t* exps) {
  extern __shared__ float lds[];
  float* v = lds;
  const int C = t.ch0[t.n];
  for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
    load_row<T>(t, x, row, v);
    if (q) pack_row(t, v, row, q, exps);
    for (int e = 0; e < t.n; ++e) {
      norm_entry(t, e, v, eps);
      for (int i = threadIdx.x; i < t.ch0[e + 1] - t.ch0[e]; i += 64)
        v[t.ch0[e] + i] *= param(gain, t.f0[e] + i / (2 * t.l[e] + 1));
    }
    __syncthreads();
    store_row(v, C, y + row * C);
    __syncthreads();
  }
}

template <typename T>
__global__ __launch_bounds__(64) void site_norm_bwd(SiteTab t, ssconv_rows x, const T* dy, const T* dres, int64_t n,
                                                    float eps, const float* __restrict__ gain, T* dx,
                                                    float* __restrict__ part) {
  extern __shared__ float lds[];
  const int C = t.ch0[t.n];
  float *v = lds, *g = lds + C, *acc = lds + 2 * C;
  for (int c = threadIdx.x; c < C; c += 64) acc[c] = 0.f;
  __syncthreads();
  for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
    load_row<T>(t, x, row, v);
    load_row<T>(t, ssconv_rows{dy, nullptr}, row, g);
    for (int e = 0; e < t.n; ++e) {
      const float r = norm_entry(t, e, v, eps);
      norm_entry_back(t, e, v, r, g, gain, acc);
    }
    __syncthreads();
    for (int c = threadIdx.x; c < C; c += 64)
      dx[row * C + c] = DT<T>::from_f(dres ? g[c] + DT<T>::to_f(dres[row * C + c]) : g[c]);
    __syncthreads();
  }
  if (part)
    for (int c = threadIdx.x; c < C; c += 64) part[(int64_t)blockIdx.x * C + c] = acc[c];
}

template <typename T>
__global__ __launch_bounds__(64) void residual_fwd(SiteTab ty, SiteTab th, const T* y, const T* h, int64_t n, float eps,
                                                   const float* __restrict__ gain_post, const float* __restrict__ scale,
                                                   const float* __restrict__ gain_next, T* h_out, T* x_out, int8_t* yq,
                                                   uint8_t* ye, int8_t* hq, uint8_t* he) {
  extern __shared__ float lds[];
  const int C = ty.C, S = ty.ch0[ty.n];
  float *u = lds, *v = lds + S;
  for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
    load_row<T>(ty, ssconv_rows{y, nullptr}, row, u);
    load_row<T>(th, ssconv_rows{h, nullptr}, row, v);
    if (yq) pack_row(ty, u, row, yq, ye);
    for (int e = 0; e < ty.n; ++e) {
      norm_entry(ty, e, u, eps);
      for (int i = threadIdx.x; i < ty.ch0[e + 1] - ty.ch0[e]; i += 64)
        u[ty.ch0[e] + i] *= param(gain_post, ty.f0[e] + i / (2 * ty.l[e] + 1));
    }
    __syncthreads();
    for (int e = 0; e < th.n; ++e)
      for (int i = threadIdx.x; i < th.ch0[e + 1] - th.ch0[e]; i += 64) {
        const int f = i / (2 * th.l[e] + 1), c = th.ch0[e] + i;
        const float uc = u[c];
        const float g = th.l[e] == 0 ? (uc <= 0.f ? 0.f : uc) : sigmoidf(u[C + th.gate0[e] + f]) * uc;
        v[c] = DT<T>::to_f(DT<T>::from_f(fmaf(param(scale, th.f0[e] + f), g, v[c])));
      }
    __syncthreads();
    store_row(v, C, h_out + row * C);
    if (hq) pack_row(th, v, row, hq, he);
    __syncthreads();
    if (x_out) {
      for (int e = 0; e < th.n; ++e) {
        norm_entry(th, e, v, eps);
        for (int i = threadIdx.x; i < th.ch0[e + 1] - th.ch0[e]; i += 64)
          v[th.ch0[e] + i] *= param(gain_next, th.f0[e] + i / (2 * th.l[e] + 1));
      }
      __syncthreads();
      store_row(v, C, x_out + row * C);
    }
    __syncthreads();
  }
}

template <typename T>
__global__ __launch_bounds__(64) void residual_bwd(SiteTab ty, SiteTab th, ssconv_rows y, ssconv_rows h, const T* dh,
                                                   const T* dx, int64_t n, float eps,
                                                   const float* __restrict__ gain_post, const float* __restrict__ scale,
                                                   const float* __restrict__ gain_next, T* dy, T* dh_in,
                                                   float* __restrict__ part) {
  extern __shared__ float lds[];
  const int C = ty.C, S = ty.ch0[ty.n];
  float *u = lds, *du = u + S, *a = du + S, *b = a + C, *acc_post = b + C, *acc_scale = acc_post + S,
        *acc_next = acc_scale + C;
  float* rs = acc_next + C;
  for (int c = threadIdx.x; c < S + 2 * C; c += 64) acc_post[c] = 0.f;
  __syncthreads();
  for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
    load_row<T>(ty, y, row, u);
    load_row<T>(th, ssconv_rows{dh, nullptr}, row, b);
    if (dx) {
      load_row<T>(th, h, row, a);
      load_row<T>(th, ssconv_rows{dx, nullptr}, row, du);
      for (int e = 0; e < th.n; ++e) {
        const float r = norm_entry(th, e, a, eps);
        norm_entry_back(th, e, a, r, du, gain_next, acc_next);
        for (int i = threadIdx.x; i < th.ch0[e + 1] - th.ch0[e]; i += 64) b[th.ch0[e] + i] += du[th.ch0[e] + i];
      }
    }
    __syncthreads();
    store_row(b, C, dh_in + row * C);
    for (int e = 0; e < ty.n; ++e) {
      const float r = norm_entry(ty, e, u, eps);
      if (threadIdx.x == 0) rs[e] = r;
    }
    __syncthreads();
    for (int e = 0; e < th.n; ++e) {
      const int d = 2 * th.l[e] + 1;
      for (int f = threadIdx.x; f < th.mult[e]; f += 64) {
        const int c0 = th.ch0[e] + f * d, fi = th.f0[e] + f;
        const float sc = param(scale, fi), gp = param(gain_post, fi);
        if (d == 1) {
          const float uc = u[c0] * gp;
          acc_scale[c0] += b[c0] * (uc <= 0.f ? 0.f : uc);
          du[c0] = uc > 0.f ? sc * b[c0] : 0.f;
        } else {
          const int gc = C + th.gate0[e] + f;
          const float sg = sigmoidf(u[gc] * param(gain_post, ty.f0[ty.n - 1] + th.gate0[e] + f));
          float dot = 0.f;
          for (int i = 0; i < d; ++i) {
            const float uc = u[c0 + i] * gp;
            dot = fmaf(sc * b[c0 + i], uc, dot);
            acc_scale[c0 + i] += b[c0 + i] * (sg * uc);
            du[c0 + i] = sc * b[c0 + i] * sg;
          }
          du[gc] = dot * sg * (1.f - sg);
        }
      }
    }
    __syncthreads();
    for (int e = 0; e < ty.n; ++e) norm_entry_back(ty, e, u, rs[e], du, gain_post, acc_post);
    __syncthreads();
    store_row(du, S, dy + row * S);
    __syncthreads();
  }
  if (part)
    for (int c = threadIdx.x; c < S + 2 * C; c += 64) part[(int64_t)blockIdx.x * (S + 2 * C) + c] = acc_post[c];
}

// out[f] = sum over the workgroups' partials (in their order) and the components of field f.
__global__ void site_reduce(SiteTab t, const float* __restrict__ part, int blocks, int stride, float* __restrict__ out) {
  const int f = blockIdx.x * blockDim.x + threadIdx.x;
  if (f >= t.f0[t.n]) return;
  int e = 0;
  while (f >= t.f0[e + 1]) ++e;
  const int d = 2 * t.l[e] + 1, c0 = t.ch0[e] + (f - t.f0[e]) * d;
  float s = 0.f;
  for (int b = 0; b < blocks; ++b)
    for (int i = 0; i < d; ++i) s += part[(int64_t)b * stride + c0 + i];
  out[f] = s;
}

template <typename T>
__global__ __launch_bounds__(64) void pack_kernel(SiteTab t, const T* x, int64_t n, int8_t* q, uint8_t* exps) {
  extern __shared__ float lds[];
  for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
    load_row<T>(t, ssconv_rows{x, nullptr}, row, lds);
    pack_row(t, lds, row, q, exps);
    __syncthreads();
  }
}

template <typename T>
__global__ __launch_bounds__(64) void unpack_kernel(SiteTab t, ssconv_rows x, int64_t n, T* y) {
  extern __shared__ float lds[];
  for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
    load_row<T>(t, x, row, lds);
    store_row(lds, t.ch0[t.n], y + row * t.ch0[t.n]);
    __syncthreads();
  }
}

unsigned site_blocks(int64_t n) { return (unsigned)std::min<int64_t>(n, kSiteBlocks); }

int check_site(const ssconv_fields* fields, bool gated, ssconv_dtype dt, int64_t n, SiteTab* t) {
  if (dt != SSCONV_F32 && dt != SSCONV_BF16) return fail(SSCONV_E_DTYPE, "unsupported dtype %d", (int)dt);
  if (n < 0) return fail(SSCONV_E_INVALID, "negative row count");
  return make_sitetab(fields, gated, t);
}

int check_eps(double eps) {
  if (!(eps > 0.0) || !((float)eps > 0.f) || !(eps < 1e30)) return fail(SSCONV_E_INVALID, "eps must be positive and finite in fp32");
  return SSCONV_OK;
}

int check_workspace(const void* ws, size_t bytes, size_t need) {
  if (!ws || bytes < need || (reinterpret_cast<uintptr_t>(ws) & 255))
    return fail(SSCONV_E_INVALID, "workspace must be 256-byte aligned and hold %zu bytes", need);
  return SSCONV_OK;
}

size_t ws_bytes_of(int64_t n, int floats) { return (size_t)site_blocks(n) * floats * 4; }

}  // namespace

int launch_site_norm_fwd(const SiteTab& t, const ssconv_rows& x, ssconv_dtype dt, int64_t n, float eps,
                         const float* gain, void* y, int8_t* q, uint8_t* exps, hipStream_t st) {
  const size_t lds = t.ch0[t.n] * 4;
  if (dt == SSCONV_F32)
    site_norm_fwd<float><<<site_blocks(n), 64, lds, st>>>(t, x, n, eps, gain, (float*)y, q, exps);
  else
    site_norm_fwd<uint16_t><<<site_blocks(n), 64, lds, st>>>(t, x, n, eps, gain, (uint16_t*)y, q, exps);
  SSC_HIP(hipGetLastError());
  return SSCONV_OK;
}

int launch_unpack(const SiteTab& t, const int8_t* q, const uint8_t* exps, int64_t n, ssconv_dtype dt, void* x,
                  hipStream_t st) {
  const size_t lds = t.ch0[t.n] * 4;
  const ssconv_rows r{q, exps};
  if (dt == SSCONV_F32)
    unpack_kernel<float><<<site_blocks(n), 64, lds, st>>>(t, r, n, (float*)x);
  else
    unpack_kernel<uint16_t><<<site_blocks(n), 64, lds, st>>>(t, r, n, (uint16_t*)x);
  SSC_HIP(hipGetLastError());
  return SSCONV_OK;
}

}  // namespace ssconv

using namespace ssconv;

extern "C" int64_t ssconv_packed_blocks(const ssconv_fields* fields) {
  SiteTab t;
  return make_sitetab(fields, false, &t) == SSCONV_OK ? t.b0[t.n] : 0;
}

extern "C" int ssconv_pack(const ssconv_fields* fields, const void* x, ssconv_dtype dtype, int64_t n, int8_t* q,
                           uint8_t* exps, hipStream_t stream) {
  SiteTab t;
  SSC_TRY(check_site(fields, false, dtype, n, &t));
  if (n == 0) return SSCONV_OK;
  if (!x || !q || !exps) return fail(SSCONV_E_INVALID, "NULL feature or checkpoint buffer");
  const size_t lds = t.ch0[t.n] * 4;
  if (dtype == SSCONV_F32)
    pack_kernel<float><<<site_blocks(n), 64, lds, stream>>>(t, (const float*)x, n, q, exps);
  else
    pack_kernel<uint16_t><<<site_blocks(n), 64, lds, stream>>>(t, (const uint16_t*)x, n, q, exps);
  SSC_HIP(hipGetLastError());
  return SSCONV_OK;
}

extern "C" int ssconv_unpack(const ssconv_fields* fields, const int8_t* q, const uint8_t* exps, int64_t n,
                             ssconv_dtype dtype, void* x, hipStream_t stream) {
  SiteTab t;
  SSC_TRY(check_site(fields, false, dtype, n, &t));
  if (n == 0) return SSCONV_OK;
  if (!x || !q || !exps) return fail(SSCONV_E_INVALID, "NULL feature or checkpoint buffer");
  return launch_unpack(t, q, exps, n, dtype, x, stream);
}

extern "C" int ssconv_site_norm_forward(const ssconv_fields* fields, const ssconv_rows* x, ssconv_dtype dtype,
                                        int64_t n, double eps, const float* gain, void* y, int8_t* q, uint8_t* exps,
                                        hipStream_t stream) {
  SiteTab t;
  SSC_TRY(check_site(fields, false, dtype, n, &t));
  SSC_TRY(check_eps(eps));
  if ((q != nullptr) != (exps != nullptr)) return fail(SSCONV_E_INVALID, "a checkpoint is both of q and exps");
  if (!x) return fail(SSCONV_E_INVALID, "NULL rows");
  if (q && x->exps) return fail(SSCONV_E_INVALID, "x is a checkpoint already");
  if (n == 0) return SSCONV_OK;
  if (!x->data || !y) return fail(SSCONV_E_INVALID, "NULL feature buffer");
  return launch_site_norm_fwd(t, *x, dtype, n, (float)eps, gain, y, q, exps, stream);
}

extern "C" size_t ssconv_site_norm_workspace_size(const ssconv_fields* fields, int64_t n) {
  SiteTab t;
  if (n < 0 || make_sitetab(fields, false, &t) != SSCONV_OK) return 0;
  return ws_bytes_of(n, t.C);
}

extern "C" int ssconv_site_norm_backward(const ssconv_fields* fields, const ssconv_rows* x, const void* dy,
                                         const void* dres, ssconv_dtype dtype, int64_t n, double eps,
                                         const float* gain, void* dx, float* dgain, void* workspace, size_t ws_bytes,
                                         hipStream_t stream) {
  SiteTab t;
  SSC_TRY(check_site(fields, false, dtype, n, &t));
  SSC_TRY(check_eps(eps));
  if (n > 0 && (!x || !x->data || !dy || !dx)) return fail(SSCONV_E_INVALID, "NULL feature buffer");
  if (dgain && n > 0) SSC_TRY(check_workspace(workspace, ws_bytes, ws_bytes_of(n, t.C)));
  const int F = t.f0[t.n];
  float* part = dgain ? (float*)workspace : nullptr;
  if (n > 0) {
    const size_t lds = 3 * t.C * 4;
    if (dtype == SSCONV_F32)
      site_norm_bwd<float><<<site_blocks(n), 64, lds, stream>>>(t, *x, (const float*)dy, (const float*)dres, n,
                                                                (float)eps, gain, (float*)dx, part);
    else
      site_norm_bwd<uint16_t><<<site_blocks(n), 64, lds, stream>>>(t, *x, (const uint16_t*)dy, (const uint16_t*)dres, n,
                                                                   (float)eps, gain, (uint16_t*)dx, part);
  }
  if (dgain) site_reduce<<<cdiv(F, 64), 64, 0, stream>>>(t, part, (int)site_blocks(n), t.C, dgain);
  SSC_HIP(hipGetLastError());
  return SSCONV_OK;
}

extern "C" int ssconv_residual_forward(const ssconv_fields* fields, const void* y, const void* h, ssconv_dtype dtype,
                                       int64_t n, double eps, const float* gain_post, const float* scale,
                                       const float* gain_next, void* h_out, void* x_out, int8_t* y_q, uint8_t* y_exps,
                                       int8_t* h_q, uint8_t* h_exps, hipStream_t stream) {
  SiteTab ty, th;
  SSC_TRY(check_site(fields, true, dtype, n, &ty));
  SSC_TRY(make_sitetab(fields, false, &th));
  SSC_TRY(check_eps(eps));
  if ((y_q != nullptr) != (y_exps != nullptr) || (h_q != nullptr) != (h_exps != nullptr))
    return fail(SSCONV_E_INVALID, "a checkpoint is both of q and exps");
  if (gain_next && !x_out && n > 0) return fail(SSCONV_E_INVALID, "gain_next without x_out");
  if (n == 0) return SSCONV_OK;
  if (!y || !h || !h_out) return fail(SSCONV_E_INVALID, "NULL feature buffer");
  const size_t lds = (ty.ch0[ty.n] + ty.C) * 4;
  if (dtype == SSCONV_F32)
    residual_fwd<float><<<site_blocks(n), 64, lds, stream>>>(ty, th, (const float*)y, (const float*)h, n, (float)eps,
                                                             gain_post, scale, gain_next, (float*)h_out, (float*)x_out,
                                                             y_q, y_exps, h_q, h_exps);
  else
    residual_fwd<uint16_t><<<site_blocks(n), 64, lds, stream>>>(
        ty, th, (const uint16_t*)y, (const uint16_t*)h, n, (float)eps, gain_post, scale, gain_next, (uint16_t*)h_out,
        (uint16_t*)x_out, y_q, y_exps, h_q, h_exps);
  SSC_HIP(hipGetLastError());
  return SSCONV_OK;
}

extern "C" size_t ssconv_residual_workspace_size(const ssconv_fields* fields, int64_t n) {
  SiteTab t;
  if (n < 0 || make_sitetab(fields, true, &t) != SSCONV_OK) return 0;
  return ws_bytes_of(n, t.ch0[t.n] + 2 * t.C);
}

extern "C" int ssconv_residual_backward(const ssconv_fields* fields, const ssconv_rows* y, const ssconv_rows* h_out,
                                        const void* dh, const void* dx, ssconv_dtype dtype, int64_t n, double eps,
                                        const float* gain_post, const float* scale, const float* gain_next, void* dy,
                                        void* dh_in, float* dgain_post, float* dscale, float* dgain_next,
                                        void* workspace, size_t ws_bytes, hipStream_t stream) {
  SiteTab ty, th;
  SSC_TRY(check_site(fields, true, dtype, n, &ty));
  SSC_TRY(make_sitetab(fields, false, &th));
  SSC_TRY(check_eps(eps));
  if (n > 0 && (!y || !y->data || !dh || !dy || !dh_in)) return fail(SSCONV_E_INVALID, "NULL feature buffer");
  if (n > 0 && dx && (!h_out || !h_out->data)) return fail(SSCONV_E_INVALID, "dx needs h_out");
  if (n > 0 && !dx && (gain_next || dgain_next)) return fail(SSCONV_E_INVALID, "a next norm without dx");
  const int S = ty.ch0[ty.n], C = ty.C, stride = S + 2 * C;
  float* part = nullptr;
  if (n > 0 && (dgain_post || dscale || dgain_next)) {
    SSC_TRY(check_workspace(workspace, ws_bytes, ws_bytes_of(n, stride)));
    part = (float*)workspace;
  }
  const unsigned nb = site_blocks(n);
  if (n > 0) {
    const ssconv_rows hr = dx ? *h_out : ssconv_rows{nullptr, nullptr};
    const size_t lds = (3 * S + 4 * C + SSCONV_MAX_ENTRIES) * 4;
    if (dtype == SSCONV_F32)
      residual_bwd<float><<<nb, 64, lds, stream>>>(ty, th, *y, hr, (const float*)dh, (const float*)dx, n, (float)eps,
                                                   gain_post, scale, gain_next, (float*)dy, (float*)dh_in, part);
    else
      residual_bwd<uint16_t><<<nb, 64, lds, stream>>>(ty, th, *y, hr, (const uint16_t*)dh, (const uint16_t*)dx, n,
                                                      (float)eps, gain_post, scale, gain_next, (uint16_t*)dy,
                                                      (uint16_t*)dh_in, part);
  }
  if (dgain_post) site_reduce<<<cdiv(ty.f0[ty.n], 64), 64, 0, stream>>>(ty, part, (int)nb, stride, dgain_post);
  if (dscale) site_reduce<<<cdiv(th.f0[th.n], 64), 64, 0, stream>>>(th, part + S, (int)nb, stride, dscale);
  if (dgain_next) site_reduce<<<cdiv(th.f0[th.n], 64), 64, 0, stream>>>(th, part + S + C, (int)nb, stride, dgain_next);
  SSC_HIP(hipGetLastError());
  return SSCONV_OK;
}
