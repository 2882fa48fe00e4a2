// What the attention kernels (laud_attend.hip, laud_cache.hip, laud_cached.hip) share: sequences of packed rows, pages, pieces of the
// softmax, and the host's checks.
#pragma once

#include "laud_token.h"

namespace laud {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kMaxHeadWidth = 128;
constexpr int64_t kMaxRowDistance = 1 << 22;  // elements: 64 rows stay below the 2 GiB a descriptor addresses

// ---- sequences ------------------------------------------------------------------------------------------------------------
// Offsets are device data: whatever they hold, rows stay within 0 .. T.
__device__ __forceinline__ int row_at(const int32_t* offsets, int i, int T) { return min(max(offsets[i], 0), T); }

// Tiles of `tile` rows (a token counts as `per` of them): sequence b's begin at number row_at(b) * per / tile + b, which leaves room
// for all of them whatever the lengths are, so that a launch's size follows from T and B alone and no tile's place from a sum over
// the sequences before it.
inline __host__ __device__ long long tiles_of(long long T, int B, int per, int tile) { return T * per / tile + B; }
__device__ __forceinline__ long long first_tile(int row, int b, int per, int tile) { return (long long)row * per / tile + b; }
// The last sequence that begins at or before something (below(its first row, its number); the first one if none does), its rows and, of a
// batch, its length.  A whole wave asks, 64 sequences at a time, and has all of it after one trip to memory.
struct Sequence { int b, row0, next, len; };
template <typename F>
__device__ __forceinline__ Sequence sequence_at(const int32_t* offsets, const int32_t* lens, int B, int T, F&& below) {
  int lo = 0, hi = B;  // the answer lies in [lo, hi)
  while (hi - lo > kWave) {
    const int mid = lo + (hi - lo) / 2;
    if (below(row_at(offsets, mid, T), mid)) lo = mid;
    else hi = mid;
  }
  const int i = min(lo + lane_id(), B - 1);
  const int row = row_at(offsets, i, T), next = row_at(offsets, i + 1, T), len = lens ? lens[i] : 0;
  const unsigned long long m = __ballot(lo + lane_id() < hi && below(row, i));
  const int at = __builtin_amdgcn_readfirstlane(max(__popcll(m), 1) - 1);
  return {lo + at, __builtin_amdgcn_readlane(row, at), __builtin_amdgcn_readlane(next, at), __builtin_amdgcn_readlane(len, at)};
}

// a pointer that is the same for the wave, in scalar registers (what descriptors are made of)
template <typename T>
__device__ __forceinline__ const T* scalar_pointer(const T* p) {
  const unsigned long long at = (unsigned long long)(uintptr_t)p;
  const unsigned lo = __builtin_amdgcn_readfirstlane((int)at), hi = __builtin_amdgcn_readfirstlane((int)(at >> 32));
  return reinterpret_cast<const T*>((uintptr_t)((unsigned long long)hi << 32 | lo));
}

// ---- softmax --------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
constexpr float kNoScore = -__builtin_inff();
// Weights are exp2(c * score - top), c = scale * log2(e) and top the largest c * score so far as it was rounded, so that sums taken
// relative to an earlier top are carried over by exp2(top - later top) with nothing left over.  What is subtracted: a row without
// a score yet subtracts 0, and its weights exp2(-inf) are 0.
__device__ __forceinline__ float shift_of(float top) { return top == kNoScore ? 0.f : top; }

// The exponent, its product rounded before the difference: what a fused operation would leave of the rounding is any number where the largest product is
// beyond 2^24, and the largest score's weight 0 or infinite instead of 1.
__device__ __forceinline__ float rounded_exponent(float score, float c, float shift) {
#pragma clang fp contract(off)
  const float product = score * c;
  return product - shift;
}
// Whether that may be so for a lane of the wave: tiles of many rows, which feel the second instruction, ask.
constexpr float kLargeTop = 0x1p24f;
__device__ __forceinline__ bool any_large(float shift) { return __ballot(fabsf(shift) > kLargeTop) != 0; }

__device__ __forceinline__ float other_half_max(float v) {  // over lanes l and l + 32
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float other_half_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float quarters_max(float v) {  // over lanes l, l ^ 16, l ^ 32, l ^ 48
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return other_half_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float quarters_sum(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return other_half_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// Two weights as bf16 operands in two parts each: the leading eight bits, cut off, and the rest, rounded (2^-15 of the weight).  Nothing is rounded up
// to an infinity.  The weight is lowered a little before it is cut, so that the rest of one that fits in eight bits is not 0 either: 0 * infinity is NaN,
// and an infinite value is infinite for every weight that is not 0.
__device__ __forceinline__ void two_parts(float a, float b, unsigned& lead, unsigned& rest) {
  constexpr float kLower = 1.f - 0x1p-16f;
  const unsigned ua = __float_as_uint(a * kLower), ub = __float_as_uint(b * kLower);
  lead = __builtin_amdgcn_perm(ub, ua, 0x07060302u);
  rest = pack_bf16(a - __uint_as_float(ua & 0xffff0000u), b - __uint_as_float(ub & 0xffff0000u));
}

// ---- values that are no numbers ---------------------------------------------------------------------------------------------
// A matrix instruction multiplies every weight with every value, and 0 * NaN is NaN: where some queries of a tile do not see all of a
// step's keys, values that are not finite become zeros in front of the product, and are added to the queries that see them one by one,
// from memory.
__device__ __forceinline__ bool not_finite2(unsigned v) { return (v & 0x7f800000u) == 0x7f800000u || (v & 0x7f80u) == 0x7f80u; }
__device__ __forceinline__ bool not_finite(float v) { return (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ unsigned finite2(unsigned v) {  // of two bf16
  if ((v & 0x7f80u) == 0x7f80u) v &= 0xffff0000u;
  if ((v & 0x7f800000u) == 0x7f800000u) v &= 0xffffu;
  return v;
}
// bytes of e4m3 codes that are NaN (0x7f, 0xff) become zero
__device__ __forceinline__ unsigned nan_codes(unsigned v) { return ((v & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
__device__ __forceinline__ unsigned finite4(unsigned v) { return v & ~((nan_codes(v) >> 7) * 0xffu); }

// ---- host side ------------------------------------------------------------------------------------------------------------
// whether two row arrays of as many rows, of different widths, share a byte; at the same distance they may lie side by side
inline bool rows_overlap(const void* a, int64_t lda, size_t ea, int ca, const void* b, int64_t ldb, size_t eb, int cb, int rows) {
  if (!ranges_meet(a, span_bytes(rows, lda, ca, ea), b, span_bytes(rows, ldb, cb, eb))) return false;
  const size_t pitch = (size_t)lda * ea, wa = (size_t)ca * ea, wb = (size_t)cb * eb;
  if (pitch != (size_t)ldb * eb) return true;
  const uintptr_t pa = (uintptr_t)a, pb = (uintptr_t)b;
  const size_t d = (pa < pb ? pb - pa : pa - pb) % pitch, lower = pa < pb ? wa : wb, upper = pa < pb ? wb : wa;
  return d < lower || d + upper > pitch;
}
inline int check_heads(const laud_heads* p) {
  if (!p || p->heads <= 0 || p->kv_heads <= 0 || p->heads % p->kv_heads || p->D <= 0 || !float_type(p->dtype) || !(p->scale > 0.f) ||
      !(p->scale * kLog2e <= 3.402823466e38f))
    return LAUD_ERR_INVALID_ARG;
  if (p->D % 8 || p->D > kMaxHeadWidth || p->heads > 65535) return LAUD_ERR_UNSUPPORTED;
  return LAUD_OK;
}
// a cache and the parts of a batch that every call reads from the host
inline int check_cache(const laud_cache* c, const laud_batch* b) {
  if (!c || !b || c->pages <= 0 || c->page <= 0 || c->kv_heads <= 0 || c->D <= 0 || b->B < 0) return LAUD_ERR_INVALID_ARG;
  if (!float_type(c->dtype) && c->dtype != LAUD_E4M3) return LAUD_ERR_INVALID_ARG;
  if ((c->page & (c->page - 1)) || c->page < 16 || c->page > 256 || c->D % (c->dtype == LAUD_E4M3 ? 16 : 8) || c->D > kMaxHeadWidth ||
      c->kv_heads > 65535 || (int64_t)c->pages * c->page > INT32_MAX)
    return LAUD_ERR_UNSUPPORTED;
  if (!c->k || !c->v || !aligned16(c->k) || !aligned16(c->v) ||
      (c->dtype == LAUD_E4M3 && (!c->k_scale || !c->v_scale || !aligned16(c->k_scale) || !aligned16(c->v_scale))))
    return LAUD_ERR_INVALID_ARG;
  if (b->B && (b->table_ld <= 0 || (int64_t)b->table_ld * c->page > 1 << 30)) return LAUD_ERR_INVALID_ARG;
  return LAUD_OK;
}
inline int page_bits(const laud_cache* c) { return __builtin_ctz((unsigned)c->page); }
// laud_attention by the kernel of few rows (laud_cached.hip): 16 query rows a workgroup, keys straight into registers
int attend_few(const laud_heads& p, int B, const int32_t* offsets, int T, const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v,
               int64_t ldv, const uint8_t* keep, void* out, int64_t ldo, hipStream_t st);
inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
inline bool check_batch(const laud_batch* b) {
  return b->offsets && b->lens && b->table && aligned4(b->offsets) && aligned4(b->lens) && aligned4(b->table);
}
inline size_t cache_rows_of(const laud_cache* c) { return (size_t)c->pages * c->page * c->kv_heads; }
inline size_t cache_bytes(const laud_cache* c) { return cache_rows_of(c) * c->D * (c->dtype == LAUD_E4M3 ? 1 : elem_bytes(c->dtype)); }
inline bool rows_meet_cache(const laud_cache* c, const void* p, int64_t ld, size_t eb, int C, int rows) {
  return range_meets_rows(c->k, cache_bytes(c), p, ld, eb, rows, C) || range_meets_rows(c->v, cache_bytes(c), p, ld, eb, rows, C) ||
         (c->dtype == LAUD_E4M3 && (range_meets_rows(c->k_scale, cache_rows_of(c) * 4, p, ld, eb, rows, C) ||
                                    range_meets_rows(c->v_scale, cache_rows_of(c) * 4, p, ld, eb, rows, C)));
}
inline bool cache_meets(const laud_cache* c, const void* p, size_t n) {
  const size_t scales = c->dtype == LAUD_E4M3 ? cache_rows_of(c) * 4 : 0;
  return ranges_meet(p, n, c->k, cache_bytes(c)) || ranges_meet(p, n, c->v, cache_bytes(c)) || ranges_meet(p, n, c->k_scale, scales) ||
         ranges_meet(p, n, c->v_scale, scales);
}
struct Span { const void* p; size_t n; };
// what the calls read of a batch
struct BatchSpans {
  Span s[3];
  explicit BatchSpans(const laud_batch* b)
      : s{{b->offsets, 4 * ((size_t)b->B + 1)}, {b->lens, 4 * (size_t)b->B}, {b->table, 4 * (size_t)b->B * b->table_ld}} {}
};
inline bool rows_meet_batch(const laud_batch* b, const void* p, int64_t ld, size_t eb, int rows, int cols) {
  for (const Span& s : BatchSpans(b).s)
    if (range_meets_rows(s.p, s.n, p, ld, eb, rows, cols)) return true;
  return false;
}
// whether the cache's parts meet each other or the batch (what a call writes shares no byte with anything else of it)
inline bool cache_meets_batch(const laud_cache* c, const laud_batch* b) {
  const bool c8 = c->dtype == LAUD_E4M3;
  const size_t scales = c8 ? cache_rows_of(c) * 4 : 0;
  const Span part[4] = {{c->k, cache_bytes(c)}, {c->v, cache_bytes(c)}, {c->k_scale, scales}, {c->v_scale, scales}};
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < i; ++j)
      if (ranges_meet(part[i].p, part[i].n, part[j].p, part[j].n)) return true;
    for (const Span& s : BatchSpans(b).s)
      if (ranges_meet(part[i].p, part[i].n, s.p, s.n)) return true;
  }
  return false;
}

}  // namespace laud
