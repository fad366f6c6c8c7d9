// Norm of a site, tail of a residual block, 8-bit checkpoints: what the kernels and the entry points share.
#pragma once

#include <algorithm>

#include "common.hpp"
#include "split_guard.hpp"

namespace ssconv {

constexpr int kPackBlock = 32;  // channels that share an exponent
constexpr int kSiteMaxC = 1024;
constexpr int kChunk = 8;       // channels that a lane holds at a time
constexpr int kSiteNT = 256;

// Entries of a row (those of a field list, and behind them the gates of a residual block as one more).  Every entry is
// cut into chunks of 8 channels of its own, K of which a lane holds: 1, 2 or 4, the least that fits 64 lanes.  (Two chunks
// on half the lanes share out the sums over more channels, but take twice the registers and leave gaps between the
// lanes' loads: backward of a tail of 100k rows of 104 channels 39 us with one, 77 with two; of 208 channels 68 and 80.)
struct SiteTab {
  int n;                            // entries
  int l[SSCONV_MAX_ENTRIES];
  int mult[SSCONV_MAX_ENTRIES];     // fields per entry
  int ch0[SSCONV_MAX_ENTRIES + 1];  // first channel of each entry, ch0[n] = channels
  int f0[SSCONV_MAX_ENTRIES + 1];   // first field
  int b0[SSCONV_MAX_ENTRIES + 1];   // first checkpoint block, b0[n] = blocks of a row
  int K;                            // chunks of a lane
  int t0[SSCONV_MAX_ENTRIES + 1];   // first lane, t0[n] = lanes that a row needs
  int gate0[SSCONV_MAX_ENTRIES];    // gate of the first field of each entry (entries of order > 0)
  int inv[SSCONV_MAX_ENTRIES];      // 65536 / components + 1: channel -> field without a division
  float m[SSCONV_MAX_ENTRIES], rm[SSCONV_MAX_ENTRIES];  // fields, and 1 / fields
  int C, G;                         // channels without the gates, gates
  int n_regular;                    // entries without the gates'
  int ragged;                       // 1: some entry is no multiple of 8 K channels, 2: fewer than 8, 3: the whole row has
};

// gated: the gates of the fields of order > 0 as one more entry.
int make_sitetab(const ssconv_fields* f, bool gated, SiteTab* t);

// Lanes per row: the fewest that hold a row with one chunk each, or 64 with two or four.  Twice as many leave half of a
// wavefront idle (backward of a residual tail, bf16: 150k rows of 36 channels on 8 lanes 53 us, on 16 86; 100k of 104 on
// 16 38, on 32 55).  K is doubled only where 64 lanes are too few (SiteTab has both sides).
inline int site_lanes(const SiteTab& t) {
  const int c = t.t0[t.n];
  return c <= 8 ? 8 : c <= 16 ? 16 : c <= 32 ? 32 : 64;
}
// Floats of LDS per row of the residual tail: the row, and 8 that a chunk moved off it may read.
inline int site_lds_row(const SiteTab& t) { return (t.ch0[t.n] + 8 + 7) / 8 * 8; }
// Rows that a workgroup takes at a time.
inline int site_rows(const SiteTab& t) { return kSiteNT / site_lanes(t); }

// Workgroups of a compute unit at a time, by a kernel's registers (their launch bounds); a workgroup is one wavefront
// per SIMD.  All loop over the rows, so a grid of more would run in rounds of which the last is part empty (backward of
// a 208-channel tail: 1024 workgroups of 144 registers, of which 768 fit, 235 us; the next version, 1024 of 128
// registers, 127).  The norm's backward would hold 8; its partial sums then cost more (191.8k rows of 208 channels
// forward and backward with 8 97 us, 6 94, 4 101).  Backward of a tail of 60k rows of 312 channels: 3 85 us, 4 73.
constexpr int norm_fwd_per_cu(int L, int K, int rag) { return K == 4 ? 2 : K == 2 || rag ? 5 : 8; }
constexpr int norm_bwd_per_cu(int L, int K, int rag) { return K == 4 ? 1 : K == 2 ? 3 : rag || L == 64 ? 5 : 6; }
constexpr int tail_fwd_per_cu(int L, int K, int rag) { return K == 4 ? 1 : K == 2 ? 3 : rag ? 4 : L == 64 ? 5 : 6; }
constexpr int tail_bwd_per_cu(int L, int K, int rag) { return K == 4 ? 1 : K == 2 ? 2 : L == 64 && rag ? 3 : 4; }
inline unsigned site_blocks(const SiteTab& t, int64_t n, int (*per_cu)(int, int, int)) {
  const int64_t rows = site_rows(t);
  return (unsigned)std::min<int64_t>((n + rows - 1) / rows,
                                     256 * per_cu(site_lanes(t), t.K, t.ragged));
}

// The backward's, whose workgroups each leave a row of partial sums of the parameters' gradients for a second launch.  Up
// to two turns of one workgroup are left to one, which writes the gradients itself (backward of a tail of 8 rows of 104
// channels, in passes that wait for the host: 22.4 us with the second launch and its workspace, 17.4 without).
inline unsigned bwd_blocks(const SiteTab& t, int64_t n, int (*per_cu)(int, int, int)) {
  return n <= 2 * site_rows(t) ? (n > 0 ? 1u : 0u) : site_blocks(t, n, per_cu);
}

struct NormArgs {
  ssconv_rows x;
  const void *dy, *dres;
  int64_t n;
  float eps;
  const float* gain;
  void* out;       // y, or dx
  int8_t* q;       // checkpoint of x (forward)
  uint8_t* exps;
  float* part;     // [workgroups][C] (backward); one workgroup writes dgain
  float* dgain;
  SplitFlags clear;  // words to clear, if any (forward)
};
struct TailArgs {
  ssconv_rows y, h;  // h: h_out in the backward
  const void *dh, *dx;
  int64_t n;
  float eps;
  const float *gain_post, *scale, *gain_next;
  void *h_out, *x_out;  // forward
  int8_t *yq, *hq;
  uint8_t *ye, *he;
  void *dy, *dh_in;  // backward
  float* part;       // [workgroups][S + 2 C]: post, scale, next; one workgroup writes grad
  float* grad[3];
};

int launch_norm_fwd(const SiteTab& t, ssconv_dtype dt, const NormArgs& a, hipStream_t st);
int launch_norm_bwd(const SiteTab& t, ssconv_dtype dt, const NormArgs& a, hipStream_t st);
int launch_tail_fwd(const SiteTab& t, ssconv_dtype dt, const TailArgs& a, hipStream_t st);
int launch_tail_bwd(const SiteTab& t, ssconv_dtype dt, const TailArgs& a, hipStream_t st);
int launch_pack(const SiteTab& t, ssconv_dtype dt, const void* x, int64_t n, int8_t* q, uint8_t* exps, hipStream_t st);
int launch_unpack(const SiteTab& t, ssconv_dtype dt, const int8_t* q, const uint8_t* exps, int64_t n, void* x,
                  const SplitFlags& clear, hipStream_t st);

// Rows of a checkpoint, or their site norm, for the gradient of a convolution (checked arguments; n > 0), which also
// clears that call's words, so that small calls need a launch less.
inline int expand_packed(const SiteTab& t, ssconv_dtype dt, const int8_t* q, const uint8_t* exps, int64_t n, bool norm,
                         float eps, const float* gain, void* rows, const SplitFlags& clear, hipStream_t st) {
  if (!norm) return launch_unpack(t, dt, q, exps, n, rows, clear, st);
  NormArgs a{};
  a.x = ssconv_rows{q, exps};
  a.n = n;
  a.eps = eps;
  a.gain = gain;
  a.out = rows;
  a.clear = clear;
  return launch_norm_fwd(t, dt, a, st);
}

int check_site_eps(double eps);

}  // namespace ssconv
