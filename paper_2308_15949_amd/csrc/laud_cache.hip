// Rows of keys and values into a paged cache and back, quantised on the way where the cache is in 8 bits.
#include "laud_heads.h"

namespace laud {
namespace {

struct CacheArgs {
  int T, B, kv_heads, D, pages, page_bits, table_ld;  // page_bits: a page holds 2^page_bits tokens
  const int32_t *offsets, *lens, *table;
  uint8_t* k;  // the cache
  uint8_t* v;
  float *ks, *vs;
  uint8_t* rk;  // the rows
  uint8_t* rv;
  int64_t ldk, ldv;
};

// Sixteen lanes a token and head: eight elements each of its key and of its value.  Bound by memory (12 prompts of up to 2000 tokens, 8 heads of
// 128: written in 8 bits 15 us, 4.0 TB/s, read back 10.6 us, 4.8); a few rows by the launch and three trips to memory, one behind the other:
// offsets, length, page (4 tokens 2.3 us).
// The sequence of a token is the number of sequences that end at or before it: sixteen lanes look at 64 at a time.
__device__ __forceinline__ int sequence_of(const CacheArgs& a, int token, int lane16) {
  int lo = 0, hi = a.B;
  while (hi - lo > kWave) {
    const int mid = lo + (hi - lo) / 2;
    if (row_at(a.offsets, mid, a.T) <= token) lo = mid;
    else hi = mid;
  }
  float count = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int i = lo + 16 * j + lane16;
    if (i < hi && row_at(a.offsets, i + 1, a.T) <= token) count += 1.f;
  }
  return lo + (int)lanes16_sum(count);
}

template <typename ET, bool C8, bool WRITE>
__global__ __launch_bounds__(256) void k_cache_rows(CacheArgs a) {
  const int lane16 = threadIdx.x % 16;
  const unsigned rows = (unsigned)a.T * (unsigned)a.kv_heads;  // (below 2^31, a step below 2^25)
  for (unsigned r = blockIdx.x * 16 + threadIdx.x / 16; r < rows; r += gridDim.x * 16) {
    const int token = (int)(r / (unsigned)a.kv_heads), head = (int)(r - (unsigned)token * a.kv_heads);
    const bool in = lane16 < a.D / 8;
    ET* const rk = reinterpret_cast<ET*>(a.rk) + token * a.ldk + head * a.D;
    ET* const rv = reinterpret_cast<ET*>(a.rv) + token * a.ldv + head * a.D;
    piece8<ET> pk, pv;
    if (WRITE && in) {  // (asked for before it is known whether they are wanted)
      pk.load(rk, lane16);
      pv.load(rv, lane16);
    }
    const int b = sequence_of(a, token, lane16);
    if (b >= a.B) continue;
    const int first = row_at(a.offsets, b, a.T), next = row_at(a.offsets, b + 1, a.T);
    if (token < first) continue;
    const long long before = (long long)a.lens[b] - (next - token);
    const int pos = (int)max(before, -1ll);
    int page = -1;
    if (pos >= 0 && pos >> a.page_bits < a.table_ld) page = a.table[(long long)b * a.table_ld + (pos >> a.page_bits)];
    const bool there = (unsigned)page < (unsigned)a.pages;
    if (WRITE && !there) continue;
    const long long at = there ? ((((long long)page * a.kv_heads + head) << a.page_bits) | (pos & ((1 << a.page_bits) - 1))) : 0;
    float f[2][8] = {};
    if constexpr (WRITE) {
      if constexpr (C8) {
        if (in) {
          pk.get(f[0]);
          pv.get(f[1]);
        }
        const float sk = block_scale(lanes16_max(top_bits(f[0]))), sv = block_scale(lanes16_max(top_bits(f[1])));
        if (in) {
          *reinterpret_cast<tok_u2*>(a.k + at * a.D + lane16 * 8) = codes8(f[0], sk);
          *reinterpret_cast<tok_u2*>(a.v + at * a.D + lane16 * 8) = codes8(f[1], sv);
        }
        if (lane16 == 0) {
          a.ks[at] = sk;
          a.vs[at] = sv;
        }
      } else if (in) {
        pk.store(reinterpret_cast<ET*>(a.k) + at * a.D, lane16);
        pv.store(reinterpret_cast<ET*>(a.v) + at * a.D, lane16);
      }
    } else if (in) {
      pk.put(f[0]);
      pv.put(f[0]);
      if (there) {
        if constexpr (C8) {
          const tok_u2 ck = *reinterpret_cast<const tok_u2*>(a.k + at * a.D + lane16 * 8);
          const tok_u2 cv = *reinterpret_cast<const tok_u2*>(a.v + at * a.D + lane16 * 8);
          const float sk = a.ks[at], sv = a.vs[at];
          piece8<bf16_t> w;
          w.v = __builtin_bit_cast(tok_u4, widen8(ck[0], ck[1]));
          w.get(f[0]);
          w.v = __builtin_bit_cast(tok_u4, widen8(cv[0], cv[1]));
          w.get(f[1]);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            f[0][e] *= sk;
            f[1][e] *= sv;
          }
          pk.put(f[0]);
          pv.put(f[1]);
        } else {
          pk.load(reinterpret_cast<const ET*>(a.k) + at * a.D, lane16);
          pv.load(reinterpret_cast<const ET*>(a.v) + at * a.D, lane16);
        }
      }
      pk.store(rk, lane16);
      pv.store(rv, lane16);
    }
  }
}

template <bool WRITE>
int cache_rows(const laud_cache* c, const laud_batch* b, int T, void* k, int64_t ldk, void* v, int64_t ldv, int dtype, void* stream) {
  const int bad = check_cache(c, b);
  if (bad) return bad;
  if (T < 0 || !float_type(dtype) || (c->dtype != LAUD_E4M3 && c->dtype != dtype)) return LAUD_ERR_INVALID_ARG;
  if (b->B == 0 || T == 0) return LAUD_OK;
  if ((int64_t)T * c->kv_heads > INT32_MAX) return LAUD_ERR_UNSUPPORTED;
  const int64_t C = (int64_t)c->kv_heads * c->D;
  if (!check_batch(b) || !k || !v || !good_ld(ldk, (int)C, 8) || !good_ld(ldv, (int)C, 8) || !aligned16(k) || !aligned16(v))
    return LAUD_ERR_INVALID_ARG;
  const size_t eb = elem_bytes(dtype);
  if (rows_meet_cache(c, k, ldk, eb, (int)C, T) || rows_meet_cache(c, v, ldv, eb, (int)C, T)) return LAUD_ERR_INVALID_ARG;
  if (!WRITE && (rows_meet(k, ldk, eb, v, ldv, eb, T, (int)C) || rows_meet_batch(b, k, ldk, eb, T, (int)C) ||
                 rows_meet_batch(b, v, ldv, eb, T, (int)C)))
    return LAUD_ERR_INVALID_ARG;
  if (WRITE && cache_meets_batch(c, b)) return LAUD_ERR_INVALID_ARG;
  CacheArgs a{};
  a.T = T; a.B = b->B; a.kv_heads = c->kv_heads; a.D = c->D; a.pages = c->pages; a.page_bits = page_bits(c); a.table_ld = b->table_ld;
  a.offsets = b->offsets; a.lens = b->lens; a.table = b->table;
  a.k = (uint8_t*)c->k; a.v = (uint8_t*)c->v; a.ks = c->k_scale; a.vs = c->v_scale;
  a.rk = (uint8_t*)k; a.rv = (uint8_t*)v; a.ldk = ldk; a.ldv = ldv;
  const long long groups = ((long long)T * c->kv_heads + 15) / 16;
  const dim3 grid((unsigned)std::min(groups, 1ll << 20));
  hipStream_t st = (hipStream_t)stream;
  clear_stale_error();
  const bool c8 = c->dtype == LAUD_E4M3;
  if (dtype == LAUD_BF16) {
    if (c8) hipLaunchKernelGGL((k_cache_rows<bf16_t, true, WRITE>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_cache_rows<bf16_t, false, WRITE>), grid, dim3(256), 0, st, a);
  } else {
    if (c8) hipLaunchKernelGGL((k_cache_rows<float, true, WRITE>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_cache_rows<float, false, WRITE>), grid, dim3(256), 0, st, a);
  }
  return check_launch();
}

}  // namespace
}  // namespace laud

extern "C" int laud_cache_write(const laud_cache* c, const laud_batch* b, int T, const void* k, int64_t ldk, const void* v, int64_t ldv,
                                int dtype, void* stream) {
  return laud::cache_rows<true>(c, b, T, const_cast<void*>(k), ldk, const_cast<void*>(v), ldv, dtype, stream);
}

extern "C" int laud_cache_read(const laud_cache* c, const laud_batch* b, int T, void* k, int64_t ldk, void* v, int64_t ldv, int dtype,
                               void* stream) {
  return laud::cache_rows<false>(c, b, T, k, ldk, v, ldv, dtype, stream);
}
