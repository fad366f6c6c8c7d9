// Entry points of the norm of a site, the tail of a residual block and the 8-bit checkpoints: tables, checks, launches.
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
  t->n = t->n_regular = ft.n;
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
    t->inv[e] = 65536 / (2 * t->l[e] + 1) + 1;
    t->m[e] = (float)t->mult[e];
    t->rm[e] = 1.f / t->m[e];
    ch += w;
    fi += t->mult[e];
    b += (w + kPackBlock - 1) / kPackBlock;
  }
  for (int e = t->n; e <= SSCONV_MAX_ENTRIES; ++e)
    t->ch0[e] = (int)ch, t->f0[e] = (int)fi, t->b0[e] = (int)b;
  for (t->K = 1;; t->K *= 2) {  // K = 4 fits: at most 1024 / 32 lanes and one more an entry
    int lanes = 0;
    t->ragged = 0;
    for (int e = 0; e < t->n; ++e) {
      const int w = t->ch0[e + 1] - t->ch0[e], per = kChunk * t->K;
      t->t0[e] = lanes;
      lanes += (w + per - 1) / per;
      if (w % per) t->ragged = std::max(t->ragged, w < kChunk ? 2 : 1);
    }
    for (int e = t->n; e <= SSCONV_MAX_ENTRIES; ++e) t->t0[e] = lanes;
    if (lanes <= 64) break;
  }
  if (t->C < kChunk) t->ragged = 3;
  return SSCONV_OK;
}

namespace {

struct ReduceArgs {
  float* out[3];
  int at[3];   // first channel of each in a row of partials
  int end[3];  // workgroups up to this one are its groups of fields
};

// Gradients of up to three parameters: out[f] = sum of the workgroups' partial sums over the components of field f, in
// fp64 and a fixed order.  A workgroup takes as many fields of an entry as 16 channels hold: 64 slices of the rows of
// partials (up to 1536, which lie in the L2s) are read side by side, 64 bytes a row: 6.2 us for 1536 rows of 208
// channels (one workgroup a field and a component at a time, a cache line for 4 bytes: 13.6 us for 2048 rows).
constexpr int kReduceNT = 1024, kReduceC = 16;
inline int fields_per_group(int l) { return kReduceC / (2 * l + 1); }

__global__ __launch_bounds__(kReduceNT) void site_reduce(SiteTab t, const float* __restrict__ part, int blocks,
                                                         int stride, ReduceArgs a) {
  __shared__ double wave[kReduceNT / 64][kReduceC];
  __shared__ double total[kReduceC];
  const int p = blockIdx.x < a.end[0] ? 0 : blockIdx.x < a.end[1] ? 1 : 2;
  int g = blockIdx.x - (p ? a.end[p - 1] : 0), e = 0, d = 1, per = kReduceC;
  for (;; ++e) {  // the host has counted the groups of the entries of this parameter
    d = 2 * t.l[e] + 1;
    per = kReduceC / d;
    const int groups = (t.mult[e] + per - 1) / per;
    if (g < groups || e + 1 == t.n) break;
    g -= groups;
  }
  const int fields = min(per, t.mult[e] - g * per), c = threadIdx.x & (kReduceC - 1);
  const float* src = part + a.at[p] + t.ch0[e] + g * per * d + min(c, fields * d - 1);
  double s = 0.0;
#pragma unroll 8
  for (int b = threadIdx.x / kReduceC; b < blocks; b += kReduceNT / kReduceC) s += (double)src[(int64_t)b * stride];
  s += __shfl_xor(s, 16);
  s += __shfl_xor(s, 32);
  if ((threadIdx.x & 63) < kReduceC) wave[threadIdx.x >> 6][c] = s;
  __syncthreads();
  if (threadIdx.x < kReduceC) {
    s = 0.0;
    for (int w = 0; w < kReduceNT / 64; ++w) s += wave[w][threadIdx.x];
    total[threadIdx.x] = s;
  }
  __syncthreads();
  if (threadIdx.x < fields) {
    s = 0.0;
    for (int i = 0; i < d; ++i) s += total[threadIdx.x * d + i];
    a.out[p][t.f0[e] + g * per + threadIdx.x] = (float)s;
  }
}

int reduce_groups(const SiteTab& t, int entries) {
  int n = 0;
  for (int e = 0; e < entries; ++e) n += (t.mult[e] + fields_per_group(t.l[e]) - 1) / fields_per_group(t.l[e]);
  return n;
}

// t: the entries of the longest list among the parameters; the others are its beginning.
int reduce_fields(const SiteTab& t, const float* part, unsigned blocks, int stride, const ReduceArgs& a,
                  hipStream_t st) {
  if (a.end[2] == 0) return SSCONV_OK;
  site_reduce<<<a.end[2], kReduceNT, 0, st>>>(t, part, (int)blocks, stride, a);
  SSC_HIP(hipGetLastError());
  return SSCONV_OK;
}

int check_site(const ssconv_fields* fields, bool gated, ssconv_dtype dt, int64_t n, SiteTab* t) {
  if (dt != SSCONV_F32 && dt != SSCONV_BF16) return fail(SSCONV_E_DTYPE, "unsupported dtype %d", (int)dt);
  if (n < 0) return fail(SSCONV_E_INVALID, "negative row count");
  return make_sitetab(fields, gated, t);
}

int check_workspace(const void* ws, size_t bytes, size_t need) {
  if (need == 0) return SSCONV_OK;
  if (!ws || bytes < need || (reinterpret_cast<uintptr_t>(ws) & 255))
    return fail(SSCONV_E_INVALID, "workspace must be 256-byte aligned and hold %zu bytes", need);
  return SSCONV_OK;
}

// A row of partial sums of every workgroup; none where there is one.
size_t part_bytes(unsigned blocks, int floats) { return blocks <= 1 ? 0 : (size_t)blocks * floats * 4; }
size_t norm_ws_bytes(const SiteTab& t, int64_t n) { return part_bytes(bwd_blocks(t, n, norm_bwd_per_cu), t.C); }
size_t tail_ws_bytes(const SiteTab& t, int64_t n) {
  return part_bytes(bwd_blocks(t, n, tail_bwd_per_cu), t.ch0[t.n] + 2 * t.C);
}

}  // namespace

int check_site_eps(double eps) {
  if (!(eps >= 1.1754944e-38) || !(eps < 1e30)) return fail(SSCONV_E_INVALID, "eps must be a positive normal number of fp32 under 1e30");
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
  return launch_pack(t, dtype, x, n, q, exps, stream);
}

extern "C" int ssconv_unpack(const ssconv_fields* fields, const int8_t* q, const uint8_t* exps, int64_t n,
                             ssconv_dtype dtype, void* x, hipStream_t stream) {
  SiteTab t;
  SSC_TRY(check_site(fields, false, dtype, n, &t));
  if (n == 0) return SSCONV_OK;
  if (!x || !q || !exps) return fail(SSCONV_E_INVALID, "NULL feature or checkpoint buffer");
  return launch_unpack(t, dtype, q, exps, n, x, SplitFlags{}, stream);
}

extern "C" int ssconv_site_norm_forward(const ssconv_fields* fields, const ssconv_rows* x, ssconv_dtype dtype,
                                        int64_t n, double eps, const float* gain, void* y, int8_t* q, uint8_t* exps,
                                        hipStream_t stream) {
  SiteTab t;
  SSC_TRY(check_site(fields, false, dtype, n, &t));
  SSC_TRY(check_site_eps(eps));
  if ((q != nullptr) != (exps != nullptr)) return fail(SSCONV_E_INVALID, "a checkpoint is both of q and exps");
  if (!x) return fail(SSCONV_E_INVALID, "NULL rows");
  if (q && x->exps) return fail(SSCONV_E_INVALID, "x is a checkpoint already");
  if (n == 0) return SSCONV_OK;
  if (!x->data || !y) return fail(SSCONV_E_INVALID, "NULL feature buffer");
  NormArgs a{};
  a.x = *x;
  a.n = n;
  a.eps = (float)eps;
  a.gain = gain;
  a.out = y;
  a.q = q;
  a.exps = exps;
  return launch_norm_fwd(t, dtype, a, stream);
}

extern "C" size_t ssconv_site_norm_workspace_size(const ssconv_fields* fields, int64_t n) {
  SiteTab t;
  if (n < 0 || make_sitetab(fields, false, &t) != SSCONV_OK) return 0;
  return norm_ws_bytes(t, n);
}

extern "C" int ssconv_site_norm_backward(const ssconv_fields* fields, const ssconv_rows* x, const void* dy,
                                         const void* dres, ssconv_dtype dtype, int64_t n, double eps,
                                         const float* gain, void* dx, float* dgain, void* workspace, size_t ws_bytes,
                                         hipStream_t stream) {
  SiteTab t;
  SSC_TRY(check_site(fields, false, dtype, n, &t));
  SSC_TRY(check_site_eps(eps));
  if (n > 0 && (!x || !x->data || !dy || !dx)) return fail(SSCONV_E_INVALID, "NULL feature buffer");
  if (dgain && n > 0) SSC_TRY(check_workspace(workspace, ws_bytes, norm_ws_bytes(t, n)));
  float* part = dgain && n > 0 ? (float*)workspace : nullptr;
  if (n > 0) {
    NormArgs a{};
    a.x = *x;
    a.dy = dy;
    a.dres = dres;
    a.n = n;
    a.eps = (float)eps;
    a.gain = gain;
    a.out = dx;
    const bool one = bwd_blocks(t, n, norm_bwd_per_cu) == 1;
    a.part = one ? nullptr : part;
    a.dgain = one ? dgain : nullptr;
    SSC_TRY(launch_norm_bwd(t, dtype, a, stream));
    if (one) return SSCONV_OK;
  }
  const int F = dgain ? reduce_groups(t, t.n) : 0;
  return reduce_fields(t, part, bwd_blocks(t, n, norm_bwd_per_cu), t.C, ReduceArgs{{dgain}, {0}, {F, F, F}}, stream);
}

extern "C" int ssconv_residual_forward(const ssconv_fields* fields, const void* y, const void* h, ssconv_dtype dtype,
                                       int64_t n, double eps, const float* gain_post, const float* scale,
                                       const float* gain_next, void* h_out, void* x_out, int8_t* y_q, uint8_t* y_exps,
                                       int8_t* h_q, uint8_t* h_exps, hipStream_t stream) {
  SiteTab ty;
  SSC_TRY(check_site(fields, true, dtype, n, &ty));
  SSC_TRY(check_site_eps(eps));
  if ((y_q != nullptr) != (y_exps != nullptr) || (h_q != nullptr) != (h_exps != nullptr))
    return fail(SSCONV_E_INVALID, "a checkpoint is both of q and exps");
  if (gain_next && !x_out && n > 0) return fail(SSCONV_E_INVALID, "gain_next without x_out");
  if (n == 0) return SSCONV_OK;
  if (!y || !h || !h_out) return fail(SSCONV_E_INVALID, "NULL feature buffer");
  TailArgs a{};
  a.y = ssconv_rows{y, nullptr};
  a.h = ssconv_rows{h, nullptr};
  a.n = n;
  a.eps = (float)eps;
  a.gain_post = gain_post;
  a.scale = scale;
  a.gain_next = gain_next;
  a.h_out = h_out;
  a.x_out = x_out;
  a.yq = y_q;
  a.ye = y_exps;
  a.hq = h_q;
  a.he = h_exps;
  return launch_tail_fwd(ty, dtype, a, stream);
}

extern "C" size_t ssconv_residual_workspace_size(const ssconv_fields* fields, int64_t n) {
  SiteTab t;
  if (n < 0 || make_sitetab(fields, true, &t) != SSCONV_OK) return 0;
  return tail_ws_bytes(t, n);
}

extern "C" int ssconv_residual_backward(const ssconv_fields* fields, const ssconv_rows* y, const ssconv_rows* h_out,
                                        const void* dh, const void* dx, ssconv_dtype dtype, int64_t n, double eps,
                                        const float* gain_post, const float* scale, const float* gain_next, void* dy,
                                        void* dh_in, float* dgain_post, float* dscale, float* dgain_next,
                                        void* workspace, size_t ws_bytes, hipStream_t stream) {
  SiteTab ty;
  SSC_TRY(check_site(fields, true, dtype, n, &ty));
  SSC_TRY(check_site_eps(eps));
  if (n > 0 && (!y || !y->data || !dh || !dy || !dh_in)) return fail(SSCONV_E_INVALID, "NULL feature buffer");
  if (n > 0 && dx && (!h_out || !h_out->data)) return fail(SSCONV_E_INVALID, "dx needs h_out");
  if (n > 0 && dx && !y->exps != !h_out->exps)
    return fail(SSCONV_E_INVALID, "y and h_out are rows, or both are checkpoints");
  if (n > 0 && !dx && (gain_next || dgain_next)) return fail(SSCONV_E_INVALID, "a next norm without dx");
  const int S = ty.ch0[ty.n], C = ty.C, stride = S + 2 * C;
  float* part = nullptr;
  if (n > 0 && (dgain_post || dscale || dgain_next)) {
    SSC_TRY(check_workspace(workspace, ws_bytes, tail_ws_bytes(ty, n)));
    part = (float*)workspace;
  }
  if (n > 0) {
    TailArgs a{};
    a.y = *y;
    a.h = dx ? *h_out : ssconv_rows{nullptr, nullptr};
    a.dh = dh;
    a.dx = dx;
    a.n = n;
    a.eps = (float)eps;
    a.gain_post = gain_post;
    a.scale = scale;
    a.gain_next = gain_next;
    a.dy = dy;
    a.dh_in = dh_in;
    const bool one = bwd_blocks(ty, n, tail_bwd_per_cu) == 1;
    a.part = one ? nullptr : part;
    a.grad[0] = one ? dgain_post : nullptr;
    a.grad[1] = one ? dscale : nullptr;
    a.grad[2] = one ? dgain_next : nullptr;
    SSC_TRY(launch_tail_bwd(ty, dtype, a, stream));
    if (one) return SSCONV_OK;
  }
  const int F = reduce_groups(ty, ty.n_regular), FS = reduce_groups(ty, ty.n);
  ReduceArgs r{{dgain_post, dscale, dgain_next}, {0, S, S + C}, {}};
  r.end[0] = dgain_post ? FS : 0;
  r.end[1] = r.end[0] + (dscale ? F : 0);
  r.end[2] = r.end[1] + (dgain_next ? F : 0);
  return reduce_fields(ty, part, bwd_blocks(ty, n, tail_bwd_per_cu), stride, r, stream);
}
