// Rows of sites in registers: what the kernels of the site norm, the residual tail and the checkpoints share.
//
// A row is L lanes' of a wavefront (64 / L rows each), every lane holding K chunks of 8 channels of one entry each.
// Loads and stores are one 16-byte access a chunk (bf16; two in fp32, 8 bytes of a checkpoint) at whatever alignment
// the row has, so nothing passes through LDS but what lanes owe each other.  RAG = 1: an entry that is no multiple of 8
// ends in a chunk moved back to its end: its first `lo` channels are the previous chunk's too, take part in no sum and are
// computed and stored twice, with the same bits.  RAG = 2: entries under 8 channels have one chunk of `hi` channels, moved
// element by element, which every chunk then has branches for (backward of a tail of 60k rows of 303 channels without
// narrow entries: 126 us with them, 94 without).
//
// With K = 1 an entry is a run of lanes, and its sums are a segmented prefix sum (3 to 6 DPP additions, whatever the
// number of entries) of which the run's last lane is read back; with K = 2 or 3 (rows over 64 or 128 chunks) they are sums
// over the wavefront entry by entry.
#pragma once

#include "site.hpp"

namespace ssconv {

typedef float f8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef u4 u4_any __attribute__((aligned(2)));
typedef f8 f8_any __attribute__((aligned(4)));
typedef u2 u2_any __attribute__((aligned(1)));

// Exponent byte of a block with this largest magnitude (as bits), and its scale and the scale's inverse.
__device__ __forceinline__ int pack_byte(uint32_t amax_bits) {
  const int k = (int)(amax_bits >> 23) - 127 - 6 + ((amax_bits & 0x7fffffu) > 0x7e0000u ? 1 : 0);  // 127/64 = 1 + 63/64
  return amax_bits >= 0x7f800000u ? 255 : (k < -126 ? -126 : k) + 127;
}
__device__ __forceinline__ float pack_scale(int byte) {
  return __uint_as_float(byte == 255 ? 0x7fc00000u : (uint32_t)byte << 23);
}
__device__ __forceinline__ float pack_inverse(int byte) {  // 2^-k; 0 for a block that keeps no value
  return __uint_as_float(byte == 255 ? 0u : (uint32_t)(254 - byte) << 23);
}

// Order of LDS accesses of the lanes of one wavefront (the LDS itself serves a wavefront in order).
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ float sigmoid_of(float x) { return __builtin_amdgcn_rcpf(1.f + __expf(-x)); }

template <int CTRL>
__device__ __forceinline__ float dpp_or_0(float v) {  // the value of another lane, 0 where there is none
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}

// Sum over the wavefront, in a scalar register.
__device__ __forceinline__ float wave_total(float v) {
  v += dpp_or_0<0x111>(v);  // the lane 1, 2, 4, 8 before
  v += dpp_or_0<0x112>(v);
  v += dpp_or_0<0x114>(v);
  v += dpp_or_0<0x118>(v);
  v += dpp_or_0<0x142>(v);  // lane 15 of the 16 before
  v += dpp_or_0<0x143>(v);  // lane 31
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

__device__ __forceinline__ float read_lane(float v, int addr) {
  return __int_as_float(__builtin_amdgcn_ds_bpermute(addr, __float_as_int(v)));
}

template <typename T>
__device__ __forceinline__ f8 load8(const T* p);
template <>
__device__ __forceinline__ f8 load8<float>(const float* p) {
  return *reinterpret_cast<const f8_any*>(p);
}
template <>
__device__ __forceinline__ f8 load8<uint16_t>(const uint16_t* p) {
  const u4 v = *reinterpret_cast<const u4_any*>(p);
  f8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r[2 * i] = __uint_as_float(v[i] << 16);
    r[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
  }
  return r;
}
// The values as they are stored (rounded to nearest even), written to p where full.
template <typename T>
__device__ __forceinline__ f8 round8(f8 v);
template <>
__device__ __forceinline__ f8 round8<float>(f8 v) { return v; }
template <>
__device__ __forceinline__ f8 round8<uint16_t>(f8 v) {
  return __builtin_convertvector(__builtin_convertvector(v, bf8), f8);
}
__device__ __forceinline__ void store8(float* p, f8 v) { *reinterpret_cast<f8_any*>(p) = v; }
__device__ __forceinline__ void store8(uint16_t* p, f8 v) {
  *reinterpret_cast<u4_any*>(p) = __builtin_bit_cast(u4, __builtin_convertvector(v, bf8));
}

// First row of a wavefront that takes ROWS at a time, in scalar registers.
template <int ROWS>
__device__ __forceinline__ int64_t first_row() {
  return ((int64_t)blockIdx.x * (kSiteNT / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * ROWS;
}

template <int L, int K, int RAG>
struct Row {
  static constexpr int R = 64 / L;            // rows of a wavefront
  static constexpr int Q = K == 1 ? 2 : 4;    // gates of a lane: a row of 8 L K channels has at most 2 L K of them
  int i, sub;                       // lane of the row, row of the wavefront
  int start[K];                     // first channel of the chunk
  int lo[K], hi[K];                 // its channels that count: [lo, hi); those under hi exist; hi = 0: no chunk
  int e[K];                         // entry
  int rel[K], f0[K], inv[K];        // first channel within the entry, first field of the entry, 65536 / components + 1
  int blk[K], blk_lo[K], quad[K];   // exponent byte, that of the channels under lo, place of the chunk in its block
  float m[K], rm[K];                // fields of the entry, and 1 / m
  bool scalar[K];
  bool any_scalar;                  // uniform
  int n;
  int last;                         // ds_bpermute address of the last lane of the run (K = 1)
  int mate[3];                      // and of the lanes of the same block
  float m1, m2, m4, m8, m15, m31;   // 1 where the lane that many places before belongs to the run

  __device__ __forceinline__ void init(const SiteTab& t, int entries) {
    const int lane = threadIdx.x & 63;
    i = lane & (L - 1);
    sub = lane / L;
    n = entries;
    any_scalar = false;
    int seg0 = i, seg1 = i;  // a lane without a chunk is a run of its own
#pragma unroll
    for (int k = 0; k < K; ++k) {
      start[k] = lo[k] = hi[k] = rel[k] = f0[k] = blk[k] = blk_lo[k] = quad[k] = 0;
      e[k] = -1;
      inv[k] = 65537;
      m[k] = rm[k] = 1.f;
      scalar[k] = false;
    }
#pragma unroll
    for (int en = 0; en < SSCONV_MAX_ENTRIES; ++en) {
      if (en >= entries) break;
      const int t0 = t.t0[en], t1 = t.t0[en + 1], ch0 = t.ch0[en], w = t.ch0[en + 1] - ch0;
      any_scalar |= t.l[en] == 0;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int c = i + k * L, j = c - t0, at = 8 * j;
        const bool in = c >= t0 && c < t1;
        int s = at, first = 0, end = 8;
        if (RAG) {
          const bool over = at + 8 > w;
          s = over ? (RAG == 2 ? max(w - 8, 0) : w - 8) : at;
          first = at - s;
          if (RAG == 2) end = min(w, 8);
        }
        start[k] = in ? ch0 + s : start[k];
        rel[k] = in ? s : rel[k];
        lo[k] = in ? first : lo[k];
        hi[k] = in ? end : hi[k];
        e[k] = in ? en : e[k];
        inv[k] = in ? t.inv[en] : inv[k];
        f0[k] = in ? t.f0[en] : f0[k];
        blk[k] = in ? t.b0[en] + j / 4 : blk[k];
        blk_lo[k] = in ? t.b0[en] + max(j - 1, 0) / 4 : blk_lo[k];
        quad[k] = in ? j & 3 : quad[k];
        m[k] = in ? t.m[en] : m[k];
        rm[k] = in ? t.rm[en] : rm[k];
        scalar[k] = in ? t.l[en] == 0 : scalar[k];
        if (k == 0) seg0 = in ? t0 : seg0, seg1 = in ? t1 - 1 : seg1;
      }
    }
    if (K == 1) {
      const int base = lane - i;
      last = 4 * (base + seg1);
      m1 = i - 1 >= seg0 ? 1.f : 0.f;
      m2 = i - 2 >= seg0 ? 1.f : 0.f;
      m4 = i - 4 >= seg0 ? 1.f : 0.f;
      m8 = i - 8 >= seg0 ? 1.f : 0.f;
      m15 = (i & 16) && seg0 < (i & ~15) ? 1.f : 0.f;
      m31 = i >= 32 && seg0 < 32 ? 1.f : 0.f;
#pragma unroll
      for (int b = 0; b < 3; ++b) mate[b] = 4 * (base + min(i - quad[0] + ((quad[0] + b + 1) & 3), seg1));
    }
  }

  __device__ __forceinline__ int field(int k, int v) const {  // of channel v of the chunk, in its entry; < 1024 channels
    return ((rel[k] + v) * inv[k]) >> 16;
  }

  // Every matrix is addressed from the wavefront's first row (scalar registers) by 32-bit offsets of the lanes.  Rows
  // past the last are read at the last.
  __device__ __forceinline__ int row_of(int64_t left) const { return min(sub, (int)min(left, (int64_t)R) - 1); }

  // The channels of a chunk, of row r of a matrix of C channels, from channel s on (start[k], or 0 where the chunk lies
  // past a matrix without the gates).  Without narrow entries a lane with no chunk there reads the row's first channels,
  // which nothing uses; else it has zeros.
  template <typename T>
  __device__ __forceinline__ f8 load(const void* p, int r, int C, int k, int s) const {
    f8 v = {0, 0, 0, 0, 0, 0, 0, 0};
    const T* q = reinterpret_cast<const T*>((const char*)p + (__umul24(r, C) + s) * (uint32_t)sizeof(T));
    if (RAG < 2 || hi[k] == 8) {
      v = load8<T>(q);
    } else {
#pragma unroll
      for (int c = 0; c < 7; ++c)
        if (c < hi[k]) v[c] = DT<T>::to_f(q[c]);
    }
    return v;
  }

  // The same of a checkpoint of C channels and B blocks: the int8 values and the exponent bytes.  The values are scale
  // times what is returned; a chunk of two blocks (ragged) has them multiplied here.
  __device__ __forceinline__ f8 load_packed(const void* p, const uint8_t* b, int r, int C, int B, int k, int s, int bl,
                                            float& scale) const {
    f8 v = {0, 0, 0, 0, 0, 0, 0, 0};
    scale = 1.f;
    if (RAG == 2 && hi[k] == 0) return v;
    const int8_t* at = (const int8_t*)p + (uint32_t)(__umul24(r, C) + s);
    u2 q = {0, 0};
    if (RAG < 2 || hi[k] == 8) {
      q = *reinterpret_cast<const u2_any*>(at);
    } else {
#pragma unroll
      for (int c = 0; c < 7; ++c)
        if (c < hi[k]) q[c / 4] |= (uint32_t)(uint8_t)at[c] << (8 * (c & 3));
    }
    const float x = pack_scale(b[(uint32_t)(__umul24(r, B) + bl)]);
#pragma unroll
    for (int c = 0; c < 8; ++c) v[c] = (float)(int8_t)(q[c / 4] >> (8 * (c & 3)));
    if (!RAG) {
      scale = x;
      return v;
    }
    const int to_lo = s == start[k] ? blk_lo[k] : bl;  // a lane that reads elsewhere uses nothing of it
    const float x_lo = pack_scale(b[(uint32_t)(__umul24(r, B) + to_lo)]);
#pragma unroll
    for (int c = 0; c < 8; ++c) v[c] *= c < lo[k] ? x_lo : x;
    if (RAG == 2 && hi[k] < 8)  // 0 * NaN
#pragma unroll
      for (int c = 1; c < 8; ++c)
        if (c >= hi[k]) v[c] = 0.f;
    return v;
  }

  // Rows, or (PK) a checkpoint of them, from row r0 on.  Which it is belongs to the kernel: with a branch here every
  // matrix would be waited for before the next is asked for.
  template <typename T, bool PK>
  __device__ __forceinline__ f8 load_rows(const ssconv_rows& x, int64_t r0, int r, int C, int B, int k, int s, int bl,
                                          float& scale) const {
    if constexpr (PK) return load_packed((const int8_t*)x.data + r0 * C, x.exps + r0 * B, r, C, B, k, s, bl, scale);
    scale = 1.f;
    return load<T>((const T*)x.data + r0 * C, r, C, k, s);
  }

  template <typename T>
  __device__ __forceinline__ void store(void* p, int r, int C, int k, f8 v) const {
    T* q = reinterpret_cast<T*>((char*)p + (__umul24(r, C) + start[k]) * (uint32_t)sizeof(T));
    if (RAG < 2 || hi[k] == 8) {
      if (hi[k]) store8(q, v);
    } else {
#pragma unroll
      for (int c = 0; c < 7; ++c)
        if (c < hi[k]) q[c] = DT<T>::from_f(v[c]);
    }
  }

  __device__ __forceinline__ bool counts(int k, int c) const { return !RAG || (c >= lo[k] && (RAG == 1 || c < hi[k])); }

  __device__ __forceinline__ float of(f8 v, int k) const {  // sum of the chunk's channels that count
    float s[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) s[c] = counts(k, c) ? v[c] : 0.f;
    return ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
  }
  __device__ __forceinline__ float dot(f8 a, f8 b, int k) const {
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int c = 0; c < 8; c += 2) {
      s0 = counts(k, c) ? fmaf(a[c], b[c], s0) : s0;
      s1 = counts(k, c + 1) ? fmaf(a[c + 1], b[c + 1], s1) : s1;
    }
    return s0 + s1;
  }

  // Sums over the entry of every chunk, of one or two values a chunk.  A step of the prefix sum is one instruction: the
  // value of the lane before, times 1 or 0 by whether it belongs to the run.  0 times an infinity or a NaN of another
  // entry would not be 0, so sums that are not finite are taken again with selections (the branch is uniform).  A lane
  // read by DPP has to be written two wait states before, hence the s_nop.
  template <int N>
  __device__ __forceinline__ void sums(float (&v)[N][K]) const {
    if constexpr (K == 1) {
      float s[N];
      bool fine = true;
#pragma unroll
      for (int a = 0; a < N; ++a) s[a] = v[a][0];
      if constexpr (N == 1) {
#define SSK_STEP(CTRL) "s_nop 1\n\tv_fmac_f32_dpp %0, %0, %" CTRL " row_mask:0xf bank_mask:0xf bound_ctrl:1\n\t"
        if constexpr (L == 8)
          asm(SSK_STEP("1 row_shr:1") SSK_STEP("2 row_shr:2") SSK_STEP("3 row_shr:4")
              : "+v"(s[0]) : "v"(m1), "v"(m2), "v"(m4));
        if constexpr (L == 16)
          asm(SSK_STEP("1 row_shr:1") SSK_STEP("2 row_shr:2") SSK_STEP("3 row_shr:4") SSK_STEP("4 row_shr:8")
              : "+v"(s[0]) : "v"(m1), "v"(m2), "v"(m4), "v"(m8));
        if constexpr (L == 32)  // row_bcast:15: lane 15 of the 16 before
          asm(SSK_STEP("1 row_shr:1") SSK_STEP("2 row_shr:2") SSK_STEP("3 row_shr:4") SSK_STEP("4 row_shr:8")
              SSK_STEP("5 row_bcast:15") : "+v"(s[0]) : "v"(m1), "v"(m2), "v"(m4), "v"(m8), "v"(m15));
        if constexpr (L == 64)  // row_bcast:31: lane 31
          asm(SSK_STEP("1 row_shr:1") SSK_STEP("2 row_shr:2") SSK_STEP("3 row_shr:4") SSK_STEP("4 row_shr:8")
              SSK_STEP("5 row_bcast:15") SSK_STEP("6 row_bcast:31")
              : "+v"(s[0]) : "v"(m1), "v"(m2), "v"(m4), "v"(m8), "v"(m15), "v"(m31));
#undef SSK_STEP
      } else {
#define SSK_STEP(CTRL)                                                                  \
  "s_nop 1\n\tv_fmac_f32_dpp %0, %0, %" CTRL " row_mask:0xf bank_mask:0xf bound_ctrl:1\n\t" \
  "v_fmac_f32_dpp %1, %1, %" CTRL " row_mask:0xf bank_mask:0xf bound_ctrl:1\n\t"
        if constexpr (L == 8)
          asm(SSK_STEP("2 row_shr:1") SSK_STEP("3 row_shr:2") SSK_STEP("4 row_shr:4")
              : "+v"(s[0]), "+v"(s[N - 1]) : "v"(m1), "v"(m2), "v"(m4));
        if constexpr (L == 16)
          asm(SSK_STEP("2 row_shr:1") SSK_STEP("3 row_shr:2") SSK_STEP("4 row_shr:4") SSK_STEP("5 row_shr:8")
              : "+v"(s[0]), "+v"(s[N - 1]) : "v"(m1), "v"(m2), "v"(m4), "v"(m8));
        if constexpr (L == 32)
          asm(SSK_STEP("2 row_shr:1") SSK_STEP("3 row_shr:2") SSK_STEP("4 row_shr:4") SSK_STEP("5 row_shr:8")
              SSK_STEP("6 row_bcast:15") : "+v"(s[0]), "+v"(s[N - 1]) : "v"(m1), "v"(m2), "v"(m4), "v"(m8), "v"(m15));
        if constexpr (L == 64)
          asm(SSK_STEP("2 row_shr:1") SSK_STEP("3 row_shr:2") SSK_STEP("4 row_shr:4") SSK_STEP("5 row_shr:8")
              SSK_STEP("6 row_bcast:15") SSK_STEP("7 row_bcast:31")
              : "+v"(s[0]), "+v"(s[N - 1]) : "v"(m1), "v"(m2), "v"(m4), "v"(m8), "v"(m15), "v"(m31));
#undef SSK_STEP
      }
#pragma unroll
      for (int a = 0; a < N; ++a) fine = fine && fabsf(s[a]) <= 3.4028235e38f;
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(!fine) != 0, 0)) {
#pragma unroll
        for (int a = 0; a < N; ++a) s[a] = v[a][0];
#define SSK_STEP(CTRL, M)                              \
  _Pragma("unroll") for (int a = 0; a < N; ++a) {      \
    const float o_ = dpp_or_0<CTRL>(s[a]);             \
    s[a] += (M) != 0.f ? o_ : 0.f;                     \
  }
        SSK_STEP(0x111, m1)
        SSK_STEP(0x112, m2)
        SSK_STEP(0x114, m4)
        if constexpr (L >= 16) { SSK_STEP(0x118, m8) }
        if constexpr (L >= 32) { SSK_STEP(0x142, m15) }
        if constexpr (L >= 64) { SSK_STEP(0x143, m31) }
#undef SSK_STEP
      }
#pragma unroll
      for (int a = 0; a < N; ++a) v[a][0] = read_lane(s[a], last);
    } else {
      float out[N][K] = {};
      for (int en = 0; en < n; ++en)
#pragma unroll
        for (int a = 0; a < N; ++a) {
          float s = 0.f;
#pragma unroll
          for (int k = 0; k < K; ++k) s += e[k] == en ? v[a][k] : 0.f;
          const float all = wave_total(s);
#pragma unroll
          for (int k = 0; k < K; ++k) out[a][k] = e[k] == en ? all : out[a][k];
        }
#pragma unroll
      for (int a = 0; a < N; ++a)
#pragma unroll
        for (int k = 0; k < K; ++k) v[a][k] = out[a][k];
    }
  }

  // s / m with one correction step: exact where the quotient is a value of fp32 (a mean that equals one of its
  // values gives a difference of exactly zero, on which a relu turns).
  __device__ __forceinline__ float over_m(float s, int k) const {
    const float q = s * rm[k];
    const float r = fmaf(fmaf(-q, m[k], s), rm[k], q);
    return fabsf(q) < 3e38f ? r : q;
  }

  // xhat in place of x, whose values are scale times x; r = 1 / sqrt(v + eps).
  __device__ __forceinline__ void norm(f8 (&x)[K], const float (&scale)[K], float (&r)[K], float eps) const {
    float mu[K];
#pragma unroll
    for (int k = 0; k < K; ++k) mu[k] = 0.f;
    if (any_scalar) {
      float s[1][K];
#pragma unroll
      for (int k = 0; k < K; ++k) s[0][k] = of(x[k], k) * scale[k];
      sums(s);
#pragma unroll
      for (int k = 0; k < K; ++k) mu[k] = scalar[k] ? over_m(s[0][k], k) : 0.f;
    }
    float s[1][K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
      for (int c = 0; c < 8; ++c) x[k][c] = fmaf(x[k][c], scale[k], -mu[k]);
      s[0][k] = dot(x[k], x[k], k);
    }
    sums(s);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      r[k] = __builtin_amdgcn_rsqf(fmaf(s[0][k], rm[k], eps));
      x[k] *= r[k];
    }
  }
  __device__ __forceinline__ void norm(f8 (&x)[K], float (&r)[K], float eps) const {
    float one[K];
#pragma unroll
    for (int k = 0; k < K; ++k) one[k] = 1.f;
    norm(x, one, r, eps);
  }

  // Gradient behind a norm in place of t = gain * dy, from xhat and r: r t - r mean(t) - xhat r sum(t xhat) / m.
  __device__ __forceinline__ void norm_back(const f8 (&xhat)[K], const float (&r)[K], f8 (&t)[K]) const {
    float s[2][K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      s[0][k] = of(t[k], k);
      s[1][k] = dot(t[k], xhat[k], k);
    }
    sums(s);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const float rr = r[k] * rm[k], a = scalar[k] ? s[0][k] * rr : 0.f, b = s[1][k] * rr;
#pragma unroll
      for (int c = 0; c < 8; ++c) t[k][c] = fmaf(t[k][c], r[k], fmaf(-xhat[k][c], b, -a));
    }
  }

  // A parameter of `fields` values, one per field, as one per channel of the chunks; ones without it.  Chunks past its
  // fields (the gates of a parameter of the fields) get its last value: looking at them here would wait for the loads,
  // which the first row's overlap.
  __device__ __forceinline__ void params(const float* p, f8 (&v)[K], int fields) const {
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int c = 0; c < 8; ++c) v[k][c] = p ? p[min(f0[k] + field(k, c), fields - 1)] : 1.f;
  }

  // The checkpoint of row r: int8 values at q, exponent bytes at b; of the chunks of the first `entries` entries.
  __device__ __forceinline__ void pack(const f8 (&x)[K], int8_t* q0, uint8_t* b0, int r, int C, int B, int entries,
                                       bool on) const {
    uint32_t amax[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      amax[k] = 0;
#pragma unroll
      for (int c = 0; c < 8; ++c)
        if (counts(k, c)) amax[k] = max(amax[k], __float_as_uint(x[k][c]) & 0x7fffffffu);
    }
    // the chunks of a block lie in up to four neighbouring lanes
    if constexpr (K == 1) {
      uint32_t o[3];
#pragma unroll
      for (int a = 0; a < 3; ++a) o[a] = (uint32_t)__builtin_amdgcn_ds_bpermute(mate[a], (int)amax[0]);
      amax[0] = max(max(amax[0], o[0]), max(o[1], o[2]));
    } else {  // lane i of chunk row k is chunk i + 64 k of the row
      uint32_t all[K];
#pragma unroll
      for (int k = 0; k < K; ++k) all[k] = amax[k];
#pragma unroll
      for (int s = -3; s <= 3; ++s) {
        if (s == 0) continue;
        uint32_t far[K];
        int blk_far[K];
        const int to = (i + s) & 63;
#pragma unroll
        for (int k = 0; k < K; ++k) {
          far[k] = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * to, (int)amax[k]);
          blk_far[k] = __builtin_amdgcn_ds_bpermute(4 * to, hi[k] ? blk[k] : -1);
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
          const int kk = k + (i + s < 0 ? -1 : i + s > 63 ? 1 : 0);
#pragma unroll
          for (int o = 0; o < K; ++o)
            if (o == kk && blk_far[o] == blk[k]) all[k] = max(all[k], far[o]);
        }
      }
#pragma unroll
      for (int k = 0; k < K; ++k) amax[k] = all[k];
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (!on || hi[k] == 0 || e[k] >= entries) continue;
      int8_t* q = q0 + (uint32_t)(__umul24(r, C) + start[k]);
      const int byte = pack_byte(amax[k]);
      const float scale = pack_inverse(byte);
      // 1.5 2^23 + v has v, rounded to nearest even, in its low bits
      uint32_t w[8];
#pragma unroll
      for (int c = 0; c < 8; ++c) w[c] = byte == 255 ? 0u : __float_as_uint(fmaf(x[k][c], scale, 12582912.f));
      if (!RAG || (lo[k] == 0 && hi[k] == 8)) {
        u2 p;
#pragma unroll
        for (int a = 0; a < 2; ++a) {
          const uint32_t l16 = __builtin_amdgcn_perm(w[4 * a + 1], w[4 * a], 0x0c0c0400u);
          const uint32_t h16 = __builtin_amdgcn_perm(w[4 * a + 3], w[4 * a + 2], 0x04000c0cu);
          p[a] = l16 | h16;
        }
        *reinterpret_cast<u2_any*>(q) = p;
      } else {
#pragma unroll
        for (int c = 0; c < 8; ++c)
          if (counts(k, c)) q[c] = (int8_t)w[c];
      }
      if (quad[k] == 0) b0[(uint32_t)(__umul24(r, B) + blk[k])] = (uint8_t)byte;
    }
  }
};

// The gates of a row, shared out over its lanes: gate i + q L of the row has components [c0, c0 + d) of the fields.
template <int L, int K, int RAG>
struct Gates {
  static constexpr int Q = Row<L, K, RAG>::Q;
  int c0[Q], d[Q], at[Q];  // d = 0: none; at: the gate's own channel
  int most;                // components of the largest order (uniform)

  // d[q] for a comparison made where it stands: hoisted out of the loop over the rows, the comparisons' masks take more
  // scalar registers than there are (60 v_readlane a row).
  __device__ __forceinline__ int comps(int q) const {
    int v = d[q];
    asm volatile("" : "+v"(v));
    return v;
  }

  // scale (optional): v[q] = the parameter of the field that a gate opens.
  __device__ __forceinline__ void init(const SiteTab& t, int i, const float* p, float (&v)[Q]) {
    int f0[Q];
    most = 0;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      c0[q] = d[q] = f0[q] = 0;
      at[q] = t.C + i + q * L;
      v[q] = 1.f;
    }
#pragma unroll
    for (int en = 0; en < SSCONV_MAX_ENTRIES; ++en) {
      if (en >= t.n_regular) break;
      const int dd = 2 * t.l[en] + 1;
      most = max(most, dd);
      if (dd == 1) continue;
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const int f = i + q * L - t.gate0[en];
        const bool in = f >= 0 && f < t.mult[en];
        c0[q] = in ? t.ch0[en] + f * dd : c0[q];
        f0[q] = in ? t.f0[en] + f : f0[q];
        d[q] = in ? dd : d[q];
      }
    }
    if (p)
#pragma unroll
      for (int q = 0; q < Q; ++q) v[q] = p[f0[q]];
  }

  // buf[channel], of a row that ends at `end`: from the gates' inputs in their channels, their sigmoids in all components of what they gate.
  __device__ __forceinline__ void open(float* buf, int end, float (&s)[Q]) const {
#pragma unroll
    for (int q = 0; q < Q; ++q) s[q] = buf[min(at[q], end)];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int n = comps(q);
      s[q] = sigmoid_of(s[q]);
      if (n == 0) continue;
      float* b = buf + c0[q];
      b[0] = b[1] = b[2] = s[q];
      if (n > 3) b[3] = b[4] = s[q];
      if (most > 5 && n > 5) b[5] = b[6] = s[q];
      if (most > 7 && n > 7) b[7] = b[8] = s[q];
    }
  }

  // From the products dh * u in the components, the gates' gradients in their channels.
  __device__ __forceinline__ void close(float* buf, const float (&s)[Q], const float (&scale)[Q]) const {
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int n = comps(q);
      if (n == 0) continue;
      const float* b = buf + c0[q];
      float v = (b[0] + b[1]) + b[2];
      if (n > 3) v += b[3] + b[4];
      if (most > 5 && n > 5) v += b[5] + b[6];
      if (most > 7 && n > 7) v += b[7] + b[8];
      buf[at[q]] = v * (scale[q] * (s[q] * (1.f - s[q])));
    }
  }
};

// 8 channels of a row in LDS; those past hi (where the chunk is no whole one) are left alone.
template <int L, int K, int RAG>
__device__ __forceinline__ void lds_put(const Row<L, K, RAG>& w, int k, float* buf, f8 v) {
  if constexpr (!RAG) {
    *reinterpret_cast<f8*>(buf + w.start[k]) = v;
  } else if (RAG == 1 || w.hi[k] == 8) {
    *reinterpret_cast<f8_any*>(buf + w.start[k]) = v;
  } else {
#pragma unroll
    for (int c = 0; c < 7; ++c)
      if (c < w.hi[k]) buf[w.start[k] + c] = v[c];
  }
}
template <int L, int K, int RAG>
__device__ __forceinline__ f8 lds_get(const Row<L, K, RAG>& w, int k, const float* buf) {  // the buffer ends 8 past the row
  if constexpr (!RAG) return *reinterpret_cast<const f8*>(buf + w.start[k]);
  return *reinterpret_cast<const f8_any*>(buf + w.start[k]);
}

// Sums of a per-channel value over the rows that the workgroup's lanes have taken, in a fixed order; lds holds one row of
// floats per row that the workgroup takes at a time.  All threads call it.  part: to part[channels]; else (the only
// workgroup of its call) to grad, summed over the components of the fields of `entries` entries.
template <int L, int K, int RAG>
__device__ __forceinline__ void sum_rows(const Row<L, K, RAG>& w, const f8 (&acc)[K], int channels, float* lds,
                                         float* part, const SiteTab& t, int entries, float* grad) {
  constexpr int ROWS = kSiteNT / L;
  __syncthreads();
  float* mine = lds + ((threadIdx.x >> 6) * (64 / L) + w.sub) * channels;
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int c = 0; c < 8; ++c)
      if (w.hi[k] > 0 && w.counts(k, c) && w.start[k] + c < channels) mine[w.start[k] + c] = acc[k][c];
  __syncthreads();
  for (int c = threadIdx.x; c < channels; c += kSiteNT) {
    float s = 0.f;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) s += lds[r * channels + c];
    if (part)
      part[c] = s;
    else
      lds[c] = s;  // its column is this thread's
  }
  if (part || !grad) return;
  __syncthreads();
  for (int e = 0; e < entries; ++e) {
    const int d = 2 * t.l[e] + 1;
    for (int f = threadIdx.x; f < t.mult[e]; f += kSiteNT) {
      float s = 0.f;
      for (int i = 0; i < d; ++i) s += lds[t.ch0[e] + f * d + i];
      grad[t.f0[e] + f] = s;
    }
  }
}

// GO_(L, K, RAG) for a table.
#define SSK_SITE_DISPATCH(t_, GO_)               \
  do {                                           \
    const int chunks_ = (t_).t0[(t_).n];         \
    if ((t_).ragged == 2) SSK_SITE_MODE(GO_, 2); \
    if ((t_).ragged == 1) SSK_SITE_MODE(GO_, 1); \
    SSK_SITE_MODE(GO_, 0);                       \
  } while (0)
#define SSK_SITE_MODE(GO_, R_)                \
  do {                                        \
    if (chunks_ <= 8) GO_(8, 1, R_);          \
    if (chunks_ <= 16) GO_(16, 1, R_);        \
    if (chunks_ <= 32) GO_(32, 1, R_);        \
    if (chunks_ <= 64) GO_(64, 1, R_);        \
    if (chunks_ <= 128) GO_(64, 2, R_);       \
    GO_(64, 3, R_);                           \
  } while (0)

}  // namespace ssconv
