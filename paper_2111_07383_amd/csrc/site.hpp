// Norm of a site, tail of a residual block, 8-bit checkpoints: what the kernels and the entry points share.
#pragma once

#include "common.hpp"

namespace ssconv {

constexpr int kPackBlock = 32;  // channels that share an exponent
constexpr int kSiteMaxC = 1024;

// Entries of a row (those of a field list, and behind them the gates of a residual block as one more).
struct SiteTab {
  int n;                            // entries
  int l[SSCONV_MAX_ENTRIES];
  int mult[SSCONV_MAX_ENTRIES];     // fields per entry
  int ch0[SSCONV_MAX_ENTRIES + 1];  // first channel of each entry, ch0[n] = channels
  int f0[SSCONV_MAX_ENTRIES + 1];   // first field
  int b0[SSCONV_MAX_ENTRIES + 1];   // first checkpoint block, b0[n] = blocks of a row
  int gate0[SSCONV_MAX_ENTRIES];    // gate of the first field of each entry (entries of order > 0)
  int C, G;                         // channels without the gates, gates
};

// gated: the gates of the fields of order > 0 as one more entry.
int make_sitetab(const ssconv_fields* f, bool gated, SiteTab* t);

// Exponent byte of a block with this largest magnitude (as bits), and its scale and the scale's inverse.
__device__ __forceinline__ int pack_byte(uint32_t amax_bits) {
  if (amax_bits >= 0x7f800000u) return 255;
  const int k = (int)(amax_bits >> 23) - 127 - 6 + ((amax_bits & 0x7fffffu) > 0x7e0000u ? 1 : 0);  // 127/64 = 1 + 63/64
  return (k < -126 ? -126 : k) + 127;
}
__device__ __forceinline__ float pack_scale(int byte) {
  return byte == 255 ? __uint_as_float(0x7fc00000u) : __uint_as_float((uint32_t)byte << 23);
}
__device__ __forceinline__ float pack_inverse(int byte) {  // 2^-k; of a block with no value to keep 0
  return byte == 255 ? 0.f : __uint_as_float((uint32_t)(254 - byte) << 23);
}

// Rows of the site norm of a checkpoint, for the gradient of the convolution behind it (checked arguments).
int launch_site_norm_fwd(const SiteTab& t, const ssconv_rows& x, ssconv_dtype dt, int64_t n, float eps,
                         const float* gain, void* y, int8_t* q, uint8_t* exps, hipStream_t st);
int launch_unpack(const SiteTab& t, const int8_t* q, const uint8_t* exps, int64_t n, ssconv_dtype dt, void* x,
                  hipStream_t st);

}  // namespace ssconv
