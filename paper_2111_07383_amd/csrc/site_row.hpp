// Rows of sites in registers: what the kernels of the site norm, the residual tail and the checkpoints share.
//
// A row is L lanes' of a wavefront (64 / L rows each), every lane holding K chunks of 8 channels of one entry each.
// Loads and stores are one 16-byte access a chunk (bf16; two in fp32, 8 bytes of a checkpoint) at whatever alignment
// the row has, so nothing passes through LDS but what lanes owe each other.  RAG = 1: an entry that is no multiple of 8
// ends in a chunk moved back to its end: its first `lo` channels are the previous chunk's too, take part in no sum and are
// computed and stored twice, with the same bits.  RAG = 2: an entry under 8 channels has one chunk, which reads its
// neighbours' channels too, so that all loads are alike, and stores the entry's element by element (150k rows of 36
// channels in four entries: backward of a tail 52 us with loads by element, 39 so).  RAG = 3: rows under 8 channels, where
// that would leave the row: all element by element.
//
// An entry begins with a lane, so it is a run of lanes; what its last lane has no chunk for is left empty.  Its sums are
// a segmented prefix sum (3 to 6 DPP additions, whatever the number of entries) of which the run's last lane is read
// back.  (With two chunks a lane, summing over the wavefront entry by entry made the tail of 60k rows of 480 channels
// 87 us forward and 211 backward; this way 69 and 149.)
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

// Exponent byte of a block with this largest magnitude (as bits), and its scale and the scale's inverse.  At the types'
// end k stays 121: at 122 the values above 127 2^121 would be 64 2^122 = 2^128, which is infinity.  They are 127 2^121
// instead, less than 2^121 away, and that is under amax / 127 like everywhere.
constexpr int kPackTop = 121 + 127;
__device__ __forceinline__ int pack_byte(uint32_t amax_bits) {
  const int byte = (int)(amax_bits >> 23) - 6 + ((amax_bits & 0x7fffffu) > 0x7e0000u ? 1 : 0);  // 127/64 = 1 + 63/64
  return amax_bits >= 0x7f800000u ? 255 : min(max(byte, 1), kPackTop);
}
__device__ __forceinline__ float pack_hold(float x) {  // to -127 2^121 .. 127 2^121
  return __builtin_amdgcn_fmed3f(x, -0x1.fcp127f, 0x1.fcp127f);
}
__device__ __forceinline__ u2 low_bytes(const uint32_t (&w)[8]) {
  u2 p;
#pragma unroll
  for (int a = 0; a < 2; ++a) {
    const uint32_t l16 = __builtin_amdgcn_perm(w[4 * a + 1], w[4 * a], 0x0c0c0400u);
    const uint32_t h16 = __builtin_amdgcn_perm(w[4 * a + 3], w[4 * a + 2], 0x04000c0cu);
    p[a] = l16 | h16;
  }
  return p;
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
  static constexpr int Q = 2 * K;             // gates of a lane: a row of 8 L K channels has at most 2 L K of them
  static constexpr int M = 4 / K;             // lanes of a checkpoint's block
  int i, sub;                       // lane of the row, row of the wavefront
  int start[K];                     // first channel of the chunk
  int lo[K], hi[K];                 // its channels that count: [lo, hi); those under hi exist; hi = 0: no chunk
  int rel[K];                       // first channel within the entry
  int blk[K], blk_lo[K];            // exponent byte, that of the channels under lo
  int e, f0, inv;                   // entry, its first field, 65536 / components + 1
  float m, rm;                      // fields of the entry, and 1 / m
  bool scalar;
  bool any_scalar;                  // uniform
  bool narrow;                      // the entry has less than 8 channels, all in the first chunk
  bool first;                       // of the lanes of its block
  int last;                         // ds_bpermute address of the last lane of the run
  int mate[3];                      // and of the other lanes of the block
  float m1, m2, m4, m8, m15, m31;   // 1 where the lane that many places before belongs to the run

  __device__ __forceinline__ void init(const SiteTab& t, int entries) {
    const int lane = threadIdx.x & 63;
    i = lane & (L - 1);
    sub = lane / L;
    any_scalar = scalar = narrow = false;
    int seg0 = i, seg1 = i;  // a lane without an entry is a run of its own
    e = -1;
    f0 = 0;
    inv = 65537;
    m = rm = 1.f;
#pragma unroll
    for (int k = 0; k < K; ++k) start[k] = hi[k] = rel[k] = blk[k] = blk_lo[k] = 0, lo[k] = 8;
#pragma unroll
    for (int en = 0; en < SSCONV_MAX_ENTRIES; ++en) {
      if (en >= entries) break;
      const int t0 = t.t0[en], t1 = t.t0[en + 1], ch0 = t.ch0[en], w = t.ch0[en + 1] - ch0;
      any_scalar |= t.l[en] == 0;
      const bool in = i >= t0 && i < t1;
      e = in ? en : e;
      inv = in ? t.inv[en] : inv;
      f0 = in ? t.f0[en] : f0;
      m = in ? t.m[en] : m;
      rm = in ? t.rm[en] : rm;
      scalar = in ? t.l[en] == 0 : scalar;
      seg0 = in ? t0 : seg0;
      seg1 = in ? t1 - 1 : seg1;
      if (RAG == 2) narrow = in ? w < 8 : narrow;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int j = (i - t0) * K + k, at = 8 * j;
        const bool here = RAG ? in && at < w : in;
        int s = at, skip = 0, end = 8;
        if (RAG == 3) {
          end = w;
        } else if (RAG == 2 && w < 8) {
          s = min(0, (en < t.n_regular ? t.C : t.ch0[t.n]) - 8 - ch0);
          skip = -s;
          end = skip + w;
        } else if (RAG) {
          s = min(at, w - 8);
          skip = at - s;
        }
        start[k] = here ? ch0 + s : start[k];
        rel[k] = here ? s : rel[k];
        lo[k] = here ? skip : lo[k];
        hi[k] = here ? end : hi[k];
        blk[k] = here ? t.b0[en] + j / 4 : blk[k];
        blk_lo[k] = here ? t.b0[en] + max(j - 1, 0) / 4 : blk_lo[k];
      }
    }
    const int base = lane - i, in_block = (i - seg0) & (M - 1);
    first = in_block == 0;
    last = 4 * (base + seg1);
    m1 = i - 1 >= seg0 ? 1.f : 0.f;
    m2 = i - 2 >= seg0 ? 1.f : 0.f;
    m4 = i - 4 >= seg0 ? 1.f : 0.f;
    m8 = i - 8 >= seg0 ? 1.f : 0.f;
    m15 = (i & 16) && seg0 < (i & ~15) ? 1.f : 0.f;
    m31 = i >= 32 && seg0 < 32 ? 1.f : 0.f;
#pragma unroll
    for (int b = 0; b < 3; ++b) mate[b] = 4 * (base + min(i - in_block + ((in_block + b + 1) & (M - 1)), seg1));
  }

  __device__ __forceinline__ int field(int k, int v) const {  // of channel v of the chunk, in its entry; < 1024 channels
    return ((RAG == 2 ? max(rel[k] + v, 0) : rel[k] + v) * inv) >> 16;
  }

  // Every matrix is addressed from the wavefront's first row (scalar registers) by 32-bit offsets of the lanes.  Rows
  // past the last are read at the last.
  __device__ __forceinline__ int row_of(int64_t left) const { return min(sub, (int)min(left, (int64_t)R) - 1); }

  // The channels of a chunk, of row r of a matrix of C channels, from channel s on (start[k], or 0 where the chunk lies
  // past a matrix without the gates).  A lane with no chunk there reads the row's first channels, which nothing
  // uses; in rows under 8 channels it has zeros.
  template <typename T>
  __device__ __forceinline__ f8 load(const void* p, int r, int C, int k, int s) const {
    f8 v = {0, 0, 0, 0, 0, 0, 0, 0};
    const T* q = reinterpret_cast<const T*>((const char*)p + (__umul24(r, C) + s) * (uint32_t)sizeof(T));
    if (RAG < 3) {
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
    if (RAG == 3 && hi[k] == 0) return v;
    const int8_t* at = (const int8_t*)p + (uint32_t)(__umul24(r, C) + s);
    u2 q = {0, 0};
    if (RAG < 3) {
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
    if (RAG == 3)  // 0 * NaN
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
    if (!by_element(k)) {
      if (hi[k]) store8(q, v);
    } else {
#pragma unroll
      for (int c = 0; c < 8; ++c)
        if (counts(k, c)) q[c] = DT<T>::from_f(v[c]);
    }
  }

  // A chunk whose channels are stored one by one.
  __device__ __forceinline__ bool by_element(int k) const { return RAG == 3 || (RAG == 2 && k == 0 && narrow); }

  __device__ __forceinline__ bool counts(int k, int c) const { return !RAG || (c >= lo[k] && (RAG == 1 || c < hi[k])); }

  __device__ __forceinline__ float of(const f8 (&v)[K]) const {  // sum of the lane's channels that count
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float s[8];
#pragma unroll
      for (int c = 0; c < 8; ++c) s[c] = counts(k, c) ? v[k][c] : 0.f;
      const float all = ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
      sum = k ? sum + all : all;
    }
    return sum;
  }
  __device__ __forceinline__ float dot(const f8 (&a)[K], const f8 (&b)[K]) const {
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int c = 0; c < 8; c += 2) {
        s0 = counts(k, c) ? fmaf(a[k][c], b[k][c], s0) : s0;
        s1 = counts(k, c + 1) ? fmaf(a[k][c + 1], b[k][c + 1], s1) : s1;
      }
    return s0 + s1;
  }

  // Sums over the entry of every lane, of one or two values a lane.  A step of the prefix sum is one instruction: the
  // value of the lane before, times 1 or 0 by whether it belongs to the run.  0 times an infinity or a NaN of another
  // entry would not be 0, so sums that are not finite are taken again with selections (the branch is uniform).  A lane
  // read by DPP has to be written two wait states before, hence the s_nop.
  template <int N>
  __device__ __forceinline__ void sums(float (&v)[N]) const {
    float s[N];
    bool fine = true;
#pragma unroll
    for (int a = 0; a < N; ++a) s[a] = v[a];
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
      for (int a = 0; a < N; ++a) s[a] = v[a];
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
    for (int a = 0; a < N; ++a) v[a] = read_lane(s[a], last);
  }

  // s / m with one correction step: exact where the quotient is a value of fp32 (a mean that equals one of its
  // values gives a difference of exactly zero, on which a relu turns).
  __device__ __forceinline__ float over_m(float s) const {
    const float q = s * rm;
    const float r = fmaf(fmaf(-q, m, s), rm, q);
    return fabsf(q) < 3e38f ? r : q;
  }

  // xhat in place of x, whose values are scale times x; r = 1 / sqrt(v + eps).
  __device__ __forceinline__ void norm(f8 (&x)[K], const float (&scale)[K], float& r, float eps) const {
    float mu = 0.f;
    if (any_scalar) {
      float s[1];
      if constexpr (K == 1) {
        s[0] = of(x) * scale[0];
      } else {
        f8 v[K];
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = x[k] * scale[k];
        s[0] = of(v);
      }
      sums(s);
      mu = scalar ? over_m(s[0]) : 0.f;
    }
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int c = 0; c < 8; ++c) x[k][c] = fmaf(x[k][c], scale[k], -mu);
    float s[1] = {dot(x, x)};
    sums(s);
    r = __builtin_amdgcn_rsqf(fmaf(s[0], rm, eps));
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] *= r;
  }
  __device__ __forceinline__ void norm(f8 (&x)[K], float& r, float eps) const {
    float one[K];
#pragma unroll
    for (int k = 0; k < K; ++k) one[k] = 1.f;
    norm(x, one, r, eps);
  }

  // Gradient behind a norm in place of t = gain * dy, from xhat and r: r t - r mean(t) - xhat r sum(t xhat) / m.
  __device__ __forceinline__ void norm_back(const f8 (&xhat)[K], float r, f8 (&t)[K]) const {
    float s[2] = {of(t), dot(t, xhat)};
    sums(s);
    const float rr = r * rm, a = scalar ? s[0] * rr : 0.f, b = s[1] * rr;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int c = 0; c < 8; ++c) t[k][c] = fmaf(t[k][c], r, fmaf(-xhat[k][c], b, -a));
  }

  // A parameter of `fields` values, one per field, as one per channel of the chunks; ones without it.  Chunks past its
  // fields (the gates of a parameter of the fields) get its last value: looking at them here would wait for the loads,
  // which the first row's overlap.  0 for an entry of one scalar, whose norm is 0 whatever it is: its gradient, a
  // difference of two equal terms, would be their rounding, times 1 / sqrt(eps).
  __device__ __forceinline__ void params(const float* p, f8 (&v)[K], int fields) const {
    const bool zero = scalar && m == 1.f;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int c = 0; c < 8; ++c) v[k][c] = zero ? 0.f : p ? p[min(f0 + field(k, c), fields - 1)] : 1.f;
  }

  // The checkpoint of row r: int8 values at q, exponent bytes at b; of the chunks of the first `entries` entries.
  __device__ __forceinline__ void pack(const f8 (&x)[K], int8_t* q0, uint8_t* b0, int r, int C, int B, int entries,
                                       bool on) const {
    uint32_t amax = 0;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int c = 0; c < 8; ++c)
        if (counts(k, c)) amax = max(amax, __float_as_uint(x[k][c]) & 0x7fffffffu);
    uint32_t o[3] = {};  // the other lanes of the block
#pragma unroll
    for (int a = 0; a < M - 1; ++a) o[a] = (uint32_t)__builtin_amdgcn_ds_bpermute(mate[a], (int)amax);
    amax = max(max(amax, o[0]), max(o[1], o[2]));
    if (!on || e < 0 || e >= entries) return;
    const int byte = pack_byte(amax);
    const float scale = pack_inverse(byte);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (RAG && hi[k] == 0) continue;
      int8_t* q = q0 + (uint32_t)(__umul24(r, C) + start[k]);
      // 1.5 2^23 + v has v, rounded to nearest even, in its low bits
      uint32_t w[8];
#pragma unroll
      for (int c = 0; c < 8; ++c) w[c] = byte == 255 ? 0u : __float_as_uint(fmaf(x[k][c], scale, 12582912.f));
      if (!RAG || (lo[k] == 0 && hi[k] == 8)) {
        u2 p = low_bytes(w);
        if (__builtin_expect(byte == kPackTop, 0)) {  // taken again from held values: a clamp of w would keep all of it
          uint32_t held[8];
#pragma unroll
          for (int c = 0; c < 8; ++c) held[c] = __float_as_uint(fmaf(pack_hold(x[k][c]), scale, 12582912.f));
          p = low_bytes(held);
        }
        *reinterpret_cast<u2_any*>(q) = p;
      } else {
#pragma unroll
        for (int c = 0; c < 8; ++c)
          if (counts(k, c))
            q[c] = (int8_t)(byte == 255 ? 0u : __float_as_uint(fmaf(pack_hold(x[k][c]), scale, 12582912.f)));
      }
    }
    if (first) b0[(uint32_t)(__umul24(r, B) + blk[0])] = (uint8_t)byte;
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

  // buf[channel], of a row that ends at `end`: from the gates' inputs in their channels, their sigmoids in all components
  // of what they gate.
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

// The channels of a chunk in a row in LDS.
template <int L, int K, int RAG>
__device__ __forceinline__ void lds_put(const Row<L, K, RAG>& w, int k, float* buf, f8 v) {
  if constexpr (!RAG) {
    *reinterpret_cast<f8*>(buf + w.start[k]) = v;
  } else if (!w.by_element(k)) {
    *reinterpret_cast<f8_any*>(buf + w.start[k]) = v;
  } else {
#pragma unroll
    for (int c = 0; c < 8; ++c)
      if (w.counts(k, c)) buf[w.start[k] + c] = v[c];
  }
}
template <int L, int K, int RAG>
__device__ __forceinline__ f8 lds_get(const Row<L, K, RAG>& w, int k, const float* buf) {  // the buffer ends 8 past the row
  if constexpr (!RAG) return *reinterpret_cast<const f8*>(buf + w.start[k]);
  return *reinterpret_cast<const f8_any*>(buf + w.start[k]);
}

// Sums of a per-channel value over the rows that the workgroup's lanes have taken, in a fixed order; lds holds one row of
// floats per row that the workgroup takes at a time.  All threads call it.  part: to part[channels], for a second launch
// that adds the workgroups up; else (the only workgroup of its call) to grad, summed over the components of the fields of
// `entries` entries.  A lane has added the rows that it took in fp32 (of 200k rows 6 on 8 lanes, 24 on 32, 200 where a
// compute unit holds one workgroup of four rows): 64 bits there would take eight registers more a chunk, which the kernels
// do not have.  From here on sums are in fp64; a workgroup's is rounded once more, to its partial.
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
    double s = 0.0;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) s += (double)lds[r * channels + c];
    if (part) {
      part[c] = (float)s;
    } else {  // its column is this thread's: the halves of s take the first two rows of it
      lds[c] = __int_as_float(__double2hiint(s));
      lds[channels + c] = __int_as_float(__double2loint(s));
    }
  }
  if (part || !grad) return;
  __syncthreads();
  for (int e = 0; e < entries; ++e) {
    const int d = 2 * t.l[e] + 1;
    for (int f = threadIdx.x; f < t.mult[e]; f += kSiteNT) {
      double s = 0.0;
      for (int i = 0; i < d; ++i) {
        const float* at = lds + t.ch0[e] + f * d + i;
        s += __hiloint2double(__float_as_int(at[0]), __float_as_int(at[channels]));
      }
      grad[t.f0[e] + f] = (float)s;
    }
  }
}

// GO_(L, K, RAG) for a table.
#define SSK_SITE_DISPATCH(t_, GO_)                                    \
  do {                                                                \
    const int lanes_ = site_lanes(t_);                                \
    if ((t_).ragged == 3) GO_(8, 1, 3); /* at most 8 entries */       \
    if ((t_).K == 4) { /* K = 2 would do without empty chunks */      \
      if ((t_).ragged == 2) GO_(64, 4, 2);                            \
      GO_(64, 4, 1);                                                  \
    }                                                                 \
    if ((t_).ragged == 2) SSK_SITE_MODE(GO_, (t_).K, lanes_, 2);      \
    if ((t_).ragged == 1) SSK_SITE_MODE(GO_, (t_).K, lanes_, 1);      \
    SSK_SITE_MODE(GO_, (t_).K, lanes_, 0);                            \
  } while (0)
#define SSK_SITE_MODE(GO_, K_, lanes_, R_) \
  do {                                     \
    if ((K_) == 2) GO_(64, 2, R_);         \
    if ((lanes_) == 8) GO_(8, 1, R_);      \
    if ((lanes_) == 16) GO_(16, 1, R_);    \
    if ((lanes_) == 32) GO_(32, 1, R_);    \
    GO_(64, 1, R_);                        \
  } while (0)

}  // namespace ssconv
