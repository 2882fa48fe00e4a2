// Device helpers of the token operators (laud_norm.hip, laud_matmul8.hip, laud_moe.hip): lane reductions, pieces of eight
// elements, 8-bit floating point (e4m3) in blocks of 128.
#pragma once

#include "laud_tile_util.h"

namespace laud {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef unsigned int tok_u4 __attribute__((ext_vector_type(4)));  // (compiler's own vectors: see laud_tile_util.h)
typedef unsigned int tok_u2 __attribute__((ext_vector_type(2)));

constexpr int kScaleBlock = 128;       // elements that share a scale along a row
constexpr float kE4m3Max = 448.f;

inline __host__ __device__ int scale_blocks(int n) { return n / kScaleBlock + (n % kScaleBlock != 0); }  // (no sum past 2^31)

// ---- reductions whose result every lane gets; data-parallel moves inside a row of sixteen lanes, swaps across rows ---------
template <int CTRL>
__device__ __forceinline__ unsigned dpp_mov(unsigned v) {
  return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
template <int CTRL>
__device__ __forceinline__ float dpp_movf(float v) { return __uint_as_float(dpp_mov<CTRL>(__float_as_uint(v))); }

__device__ __forceinline__ float lanes16_sum(float v) {
  v += dpp_movf<0xB1>(v);   // lane ^ 1
  v += dpp_movf<0x4E>(v);   // lane ^ 2
  v += dpp_movf<0x141>(v);  // the other four of eight
  v += dpp_movf<0x140>(v);  // the other eight of sixteen
  return v;
}
__device__ __forceinline__ unsigned lanes16_max(unsigned v) {
  v = max(v, dpp_mov<0xB1>(v));
  v = max(v, dpp_mov<0x4E>(v));
  v = max(v, dpp_mov<0x141>(v));
  return max(v, dpp_mov<0x140>(v));
}
__device__ __forceinline__ float lanes64_sum(float v) {
  v = lanes16_sum(v);
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ unsigned lanes64_max(unsigned v) {
  v = lanes16_max(v);
  auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(r[0], r[1]);
  r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max(r[0], r[1]);
}

// ---- eight consecutive elements of a row ------------------------------------------------------------------------------------
template <typename ET> struct piece8;
template <> struct piece8<bf16_t> {
  tok_u4 v;
  __device__ __forceinline__ void load(const void* row, int i) { v = reinterpret_cast<const tok_u4*>(row)[i]; }
  __device__ __forceinline__ void store(void* row, int i) const { reinterpret_cast<tok_u4*>(row)[i] = v; }
  __device__ __forceinline__ void get(float (&f)[8]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f[2 * e] = __uint_as_float(v[e] << 16);
      f[2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void put(const float (&f)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = pack_bf16(f[2 * e], f[2 * e + 1]);  // nearest even
  }
};
template <> struct piece8<float> {
  tok_u4 v[2];
  __device__ __forceinline__ void load(const void* row, int i) {
    v[0] = reinterpret_cast<const tok_u4*>(row)[2 * i];
    v[1] = reinterpret_cast<const tok_u4*>(row)[2 * i + 1];
  }
  __device__ __forceinline__ void store(void* row, int i) const {
    reinterpret_cast<tok_u4*>(row)[2 * i] = v[0];
    reinterpret_cast<tok_u4*>(row)[2 * i + 1] = v[1];
  }
  __device__ __forceinline__ void get(float (&f)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(v[e / 4][e % 4]);
  }
  __device__ __forceinline__ void put(const float (&f)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e / 4][e % 4] = __float_as_uint(f[e]);
  }
};

// ---- e4m3 -----------------------------------------------------------------------------------------------------------------
// Largest magnitude of eight values as its bit pattern: patterns of non-negative floats order like the floats, infinity above
// every number and NaN above that, so a NaN is what a maximum over a block ends with.
__device__ __forceinline__ unsigned top_bits(const float (&f)[8]) {
  unsigned m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(f[e]) & 0x7fffffffu);
  return m;
}
// The block's scale from its largest magnitude.  2^-126 keeps quotients of subnormal blocks and of zeros finite.
__device__ __forceinline__ float block_scale(unsigned top) {
  const float s = __uint_as_float(top) / kE4m3Max;
  return s < 0x1p-126f ? 0x1p-126f : s;  // (NaN stays)
}
// Codes of f / s, nearest even.  The quotient by the rounded reciprocal and one correction of its remainder is the rounded quotient
// (a division for every element took twice the instructions of all the rest of a norm); where s is infinite or NaN it is NaN.  What
// a quotient of 2^-10 (half the least code) leaves over is as small as 2^-56 s: where that is no float, both are taken 2^64 times.
__device__ __forceinline__ float quotient(float f, float s, float inv) {
  const float q = f * inv;
  return fmaf(fmaf(-q, s, f), inv, q);
}
__device__ __forceinline__ tok_u2 codes8(float (&f)[8], float s) {
  if (s < 0x1p-60f) {
    s *= 0x1p64f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] *= 0x1p64f;
  }
  const float inv = 1.f / s;
  tok_u2 q;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(f[4 * h], s, inv), quotient(f[4 * h + 1], s, inv), 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(f[4 * h + 2], s, inv), quotient(f[4 * h + 3], s, inv), w, true);
    q[h] = (unsigned)w;
  }
  return q;
}

__device__ __forceinline__ bf16x8 widen8(unsigned lo, unsigned hi) {  // eight e4m3 codes, exact in bf16
  union { bf16x2 h[4]; bf16x8 v; } u;
  u.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
  u.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
  u.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
  u.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
  return u.v;
}
__device__ __forceinline__ f32x4 mma_bf16_16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// ---- memory through descriptors ---------------------------------------------------------------------------------------------
constexpr unsigned kOutside = 0xfffffff0u;  // an offset past every descriptor: reads zeros
__device__ __forceinline__ __amdgpu_buffer_rsrc_t bytes_of(const void* base, long long bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)(unsigned)min(bytes, 0xffffffe0ll), 0x00020000);
}
__device__ __forceinline__ tok_u4 load16(__amdgpu_buffer_rsrc_t r, unsigned off) {
  return __builtin_bit_cast(tok_u4, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0));
}
// Four consecutive results of a row.
template <typename OT>
__device__ __forceinline__ void store4(OT* out, const f32x4& v) {
  if constexpr (sizeof(OT) == 4) {
    *reinterpret_cast<f32x4*>(out) = v;
  } else {
    *reinterpret_cast<tok_u2*>(out) = tok_u2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
  }
}

// ---- host side: argument checks the token operators share ------------------------------------------------------------------
// whether a launch of so many workgroups has less than 2^32 threads, the most that one takes along a dimension
inline bool launchable(double groups, int threads) { return groups * threads < 4294967296.0; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool good_ld(int64_t ld, int cols, int step) { return ld >= cols && ld % step == 0; }
inline bool float_type(int dtype) { return dtype == LAUD_F32 || dtype == LAUD_BF16; }
// bytes from the first to behind the last element of `rows` rows
inline size_t span_bytes(int rows, int64_t ld, int cols, size_t eb) { return rows > 0 ? ((size_t)(rows - 1) * (size_t)ld + (size_t)cols) * eb : 0; }
inline bool ranges_meet(const void* a, size_t na, const void* b, size_t nb) {
  const char *p = (const char*)a, *q = (const char*)b;
  return p && q && na && nb && p < q + nb && q < p + na;
}
// whether n bytes share one with a row array; they may lie between its rows
inline bool range_meets_rows(const void* p, size_t n, const void* a, int64_t lda, size_t eb, int rows, int cols) {
  if (!ranges_meet(p, n, a, span_bytes(rows, lda, cols, eb))) return false;
  if ((uintptr_t)p < (uintptr_t)a) return true;  // (they reach the first row)
  const size_t pitch = (size_t)lda * eb, d = (size_t)((uintptr_t)p - (uintptr_t)a) % pitch;
  return d < (size_t)cols * eb || d + n > pitch;
}
// whether two row arrays of `rows` rows share a byte; rows at the same distance may lie side by side (columns of one wider array)
inline bool rows_meet(const void* a, int64_t lda, size_t ea, const void* b, int64_t ldb, size_t eb, int rows, int cols) {
  if (!a || !b || !ranges_meet(a, span_bytes(rows, lda, cols, ea), b, span_bytes(rows, ldb, cols, eb))) return false;
  const size_t pitch = (size_t)lda * ea;
  if (pitch != (size_t)ldb * eb) return true;
  const size_t d = (size_t)((uintptr_t)a < (uintptr_t)b ? (uintptr_t)b - (uintptr_t)a : (uintptr_t)a - (uintptr_t)b) % pitch;
  const bool a_first = (uintptr_t)a < (uintptr_t)b;
  const size_t lower = (size_t)cols * (a_first ? ea : eb), upper = (size_t)cols * (a_first ? eb : ea);
  return d < lower || d + upper > pitch;
}
// ... or are the same array (base, type and distance of rows) or apart
inline bool same_or_apart(const void* a, int64_t lda, size_t ea, const void* b, int64_t ldb, size_t eb, int rows, int cols) {
  return (a == b && lda == ldb && ea == eb) || !rows_meet(a, lda, ea, b, ldb, eb, rows, cols);
}

}  // namespace laud
