// Attention of new tokens over a paged cache: parts of the keys by workgroup, joined where there are several.
#include "laud_cached.h"

namespace laud {

constexpr int kWaves = kCachedWaves;

// ---- operands ---------------------------------------------------------------------------------------------------------------
// CT: the cache's type.  A step has GROUPS times sixteen keys; lane l holds key l % 16 of each for the scores (keys * queries: a lane's
// results are keys 4 * (l / 16) .. +3 of its query, l % 16), and of the values keys 4 * (l / 16) .. +3, elements kEach * (l % 16) .. of
// each: all of a row's bytes come in one piece a lane, straight into registers, and with element e of every lane the matrix instruction
// makes channels kEach * m + e, m = 0 .. 15.  Nothing has to change lanes between the two products.
template <typename CT, int DP, int GROUPS> struct CacheOperands;

template <int DP, int GROUPS>
struct CacheOperands<bf16_t, DP, GROUPS> {
  static constexpr int kGroups = GROUPS, kEach = DP / 16, kPieces = DP / 32, kQuery = DP / 32;
  static constexpr int kBytes = 2;
  tok_u4 k[kGroups][kPieces];
  unsigned v[kGroups][4][kEach / 2];
  __device__ __forceinline__ void load_keys(int u, __amdgpu_buffer_rsrc_t rk, int D, unsigned pitch, unsigned there, int r16, int quarter) {
#pragma unroll
    for (int s = 0; s < kPieces; ++s) {
      const int d = 32 * s + 8 * quarter;
      k[u][s] = load16(rk, d < D && (there >> r16 & 1) ? (r16 * pitch + d) * 2u : kOutside);
    }
  }
  __device__ __forceinline__ void load_values(int u, __amdgpu_buffer_rsrc_t rv, int D, unsigned pitch, unsigned there, int r16, int quarter) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned at = r16 * kEach < D && (there >> (4 * quarter + j) & 1) ? ((4 * quarter + j) * pitch + r16 * kEach) * 2u : kOutside;
      if constexpr (kEach == 8) {
        const tok_u4 w = load16(rv, at);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[u][j][e] = w[e];
      } else {
        const tok_u2 w = load8(rv, at);
        v[u][j][0] = w[0];
        v[u][j][1] = w[1];
      }
    }
  }
  static __device__ __forceinline__ int query_at(int s, int quarter) { return 32 * s + 8 * quarter; }  // eight elements
  __device__ __forceinline__ bf16x8 key(int u, int s) const { return __builtin_bit_cast(bf16x8, k[u][s]); }
  // element e of the lane's eight keys of groups 2 h and 2 h + 1
  __device__ __forceinline__ tok_u4 value(int h, int e) const {
    tok_u4 r;
#pragma unroll
    for (int p = 0; p < 4; ++p)
      r[p] = __builtin_amdgcn_perm(v[2 * h + p / 2][p % 2 * 2 + 1][e / 2], v[2 * h + p / 2][p % 2 * 2][e / 2], e % 2 ? 0x07060302u : 0x05040100u);
    return r;
  }
  __device__ __forceinline__ bool take_out() {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kGroups * 4 * (kEach / 2); ++i) {
      unsigned& x = v[i / (2 * kEach)][i / (kEach / 2) % 4][i % (kEach / 2)];
      bad |= not_finite2(x);
      x = finite2(x);
    }
    return bad;
  }
  static __device__ __forceinline__ float value_at(const uint8_t* p, int i) { return bf16_to_f32(reinterpret_cast<const bf16_t*>(p)[i]); }
};

template <int DP, int GROUPS>
struct CacheOperands<uint8_t, DP, GROUPS> {
  static constexpr int kGroups = GROUPS, kEach = DP / 16, kPieces = DP / 64, kQuery = DP / 32;
  static constexpr int kBytes = 1;
  tok_u4 k[kGroups][kPieces];
  unsigned v[kGroups][4][kEach / 4];
  __device__ __forceinline__ void load_keys(int u, __amdgpu_buffer_rsrc_t rk, int D, unsigned pitch, unsigned there, int r16, int quarter) {
#pragma unroll
    for (int s = 0; s < kPieces; ++s) {
      const int d = 64 * s + 16 * quarter;
      k[u][s] = load16(rk, d < D && (there >> r16 & 1) ? r16 * pitch + d : kOutside);
    }
  }
  __device__ __forceinline__ void load_values(int u, __amdgpu_buffer_rsrc_t rv, int D, unsigned pitch, unsigned there, int r16, int quarter) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned at = r16 * kEach < D && (there >> (4 * quarter + j) & 1) ? (4 * quarter + j) * pitch + r16 * kEach : kOutside;
      if constexpr (kEach == 8) {
        const tok_u2 w = load8(rv, at);
        v[u][j][0] = w[0];
        v[u][j][1] = w[1];
      } else {
        v[u][j][0] = load4(rv, at);
      }
    }
  }
  static __device__ __forceinline__ int query_at(int s, int quarter) { return 64 * (s / 2) + 16 * quarter + 8 * (s % 2); }
  __device__ __forceinline__ bf16x8 key(int u, int s) const { return widen8(k[u][s / 2][s % 2 * 2], k[u][s / 2][s % 2 * 2 + 1]); }
  __device__ __forceinline__ tok_u4 value(int h, int e) const {
    tok_u4 r;
#pragma unroll
    for (int p = 0; p < 4; ++p) {  // codes e and its neighbour of two keys, the asked one widened
      const unsigned w = __builtin_amdgcn_perm(v[2 * h + p / 2][p % 2 * 2 + 1][e / 4], v[2 * h + p / 2][p % 2 * 2][e / 4], e % 4 / 2 ? 0x07030602u : 0x05010400u);
      bf16x2 h;
      if (e % 2) h = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true);
      else h = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false);
      r[p] = __builtin_bit_cast(unsigned, h);
    }
    return r;
  }
  __device__ __forceinline__ bool take_out() {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kGroups * 4 * (kEach / 4); ++i) {
      unsigned& x = v[i / kEach][i / (kEach / 4) % 4][i % (kEach / 4)];
      bad |= nan_codes(x) != 0;
      x = finite4(x);
    }
    return bad;
  }
  static __device__ __forceinline__ float value_at(const uint8_t* p, int i) { return (p[i] & 0x7f) == 0x7f ? __builtin_nanf("") : 0.f; }
};

template <int DP, int GROUPS>
struct CacheOperands<float, DP, GROUPS> {
  static constexpr int kGroups = GROUPS, kEach = DP / 16, kPieces = DP / 16, kQuery = DP / 16;
  static constexpr int kBytes = 4;
  tok_u4 k[kGroups][kPieces];
  float v[kGroups][4][kEach];
  __device__ __forceinline__ void load_keys(int u, __amdgpu_buffer_rsrc_t rk, int D, unsigned pitch, unsigned there, int r16, int quarter) {
#pragma unroll
    for (int s = 0; s < kPieces; ++s) {
      const int d = 16 * s + 4 * quarter;
      k[u][s] = load16(rk, d < D && (there >> r16 & 1) ? (r16 * pitch + d) * 4u : kOutside);
    }
  }
  __device__ __forceinline__ void load_values(int u, __amdgpu_buffer_rsrc_t rv, int D, unsigned pitch, unsigned there, int r16, int quarter) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int h = 0; h < kEach / 4; ++h) {
        const tok_u4 w = load16(rv, r16 * kEach < D && (there >> (4 * quarter + j) & 1) ? ((4 * quarter + j) * pitch + r16 * kEach + 4 * h) * 4u : kOutside);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[u][j][4 * h + e] = __uint_as_float(w[e]);
      }
  }
  static __device__ __forceinline__ int query_at(int s, int quarter) { return 16 * s + 4 * quarter; }  // four elements
  __device__ __forceinline__ bool take_out() {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4 * kEach; ++i) {
      float& x = v[0][i / kEach][i % kEach];
      bad |= not_finite(x);
      if (not_finite(x)) x = 0.f;
    }
    return bad;
  }
  static __device__ __forceinline__ float value_at(const uint8_t* p, int i) { return reinterpret_cast<const float*>(p)[i]; }
};

__device__ __forceinline__ f32x4 mma4(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// the values of four lanes in a row, in each of them
__device__ __forceinline__ f32x4 of_four(float v) { return f32x4{dpp_movf<0x00>(v), dpp_movf<0x55>(v), dpp_movf<0xAA>(v), dpp_movf<0xFF>(v)}; }

// Sixteen query rows a row tile (RT of them a workgroup): the tokens of a sequence times the query heads of a key head, so that a key is
// fetched once for all of them.  Four waves share a part's keys, each takes every fourth step of 16 or 32 keys; their sums are joined through LDS.
// The softmax runs along: sums are relative to the largest score so far and scaled when a larger one comes.  Weights meet values of 8 or 16 bits in two
// parts: memory bounds these shapes, and a third product costs little (one token over 32767 32.5 -> 32.8 us, 64 in 8 bits 117.1, 32 behind 16384 42.5 -> 44,
// 5 x 100 over 6000 in 8 bits 154 -> 171) for results whose error is that of their own rounding.
//
// Bound by memory: one token over 32767 (32 heads of 128 over 8, bf16) 22.4 us, 6 TB/s, and 4.6 for the join; 64 tokens over up to 8000 in 8 bits
// 106 us, 4.2 TB/s: half the bytes are in flight with the same registers for what they are widened to.  32 tokens behind 16384 36 us: the prefix is
// multiplied for 32 rows a fetch (64 rows: 86 to 114 us, sums in memory).  ROWS, the keys are rows of this call: 5 x 197 tokens, 16 heads of 64
// in float32 19 to 21 us, of which 9 pass before the first step and behind the last one (1040 workgroups), then 2.7 a step of 64 keys.
template <typename ET, typename CT, int DP, int RT, bool ROWS>
__global__ __launch_bounds__(kWaves * kWave, 2) void k_cached(CachedArgs a) {
  typedef CacheOperands<CT, DP, (sizeof(CT) == 4 ? 1 : 2)> O;
  constexpr bool kWide = sizeof(CT) == 4;  // float32 instructions
  constexpr int kGroups = O::kGroups, kKeys = 16 * kGroups, kRows = 16 * RT, kEach = O::kEach, kLdRow = DP + 4;
  extern __shared__ __align__(16) unsigned char lds[];
  float* const sums = reinterpret_cast<float*>(lds);                    // [wave][16][kLdRow]
  float* const stats = sums + kWaves * 16 * kLdRow;                     // [wave][kRows][2]
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), r16 = lane % 16, quarter = lane / 16;

  // Which rows, key head and part.  Where several tiles read the same keys they go to one XCD, one behind the other.
  const bool shared = blockIdx.x < a.prefix_groups;  // the prefix: every token's rows over the same keys
  const unsigned id = shared ? blockIdx.x : blockIdx.x - a.prefix_groups;
  const unsigned tiles = shared ? a.prefix_tiles : a.tiles, splits = shared ? a.prefix_splits : a.splits;
  int tile, hk, split;
  if (shared ? a.prefix_by_xcd : a.by_xcd) {
    const unsigned j = id / 8;
    const unsigned g = j / tiles * 8 + id % 8;
    tile = j % tiles;
    hk = g % a.kv_heads;
    split = g / a.kv_heads;
  } else {
    split = id % splits;
    const unsigned j = id / splits;
    hk = j % a.kv_heads;
    tile = j / a.kv_heads;
  }
  int row0 = 0, n = a.T, len = a.prefix_len, whole_len = len;
  const int32_t* table = a.prefix;
  if (!shared) {
    const Sequence s = sequence_at(a.offsets, ROWS ? nullptr : a.lens, a.B, a.T, [&](int row, int i) { return first_tile(row, i, a.group, kRows) <= tile; });
    row0 = s.row0;
    n = s.next - s.row0;
    whole_len = s.len;
    const long long before = first_tile(s.row0, s.b, a.group, kRows);
    if ((long long)tile < before) return;
    tile -= (int)before;
    len = ROWS ? max(n, 0) : cached_tokens(a, s.len);
    table = a.table + (long long)s.b * a.table_ld;
  }
  if (n <= 0) return;
  const unsigned rows = (unsigned)n * (unsigned)a.group, first_row = (unsigned)tile * kRows;  // (T * heads is below 2^31)
  if (first_row >= rows) return;
  const int there = (int)min((unsigned)kRows, rows - first_row);  // rows of this tile
  const int each = part_keys(len, splits);
  if (split > 0 && (long long)split * each >= len) return;
  const long long past = (long long)(ROWS ? len : whole_len) - n;  // position of the first token
  const bool causal = a.causal && !shared;
  auto limit_of = [&](unsigned row) -> int {  // keys that a row sees
    return causal ? (int)min(max(past + token_of(a, row) + 1, 0ll), (long long)len) : len;
  };
  const int begin = split * each;
  const int end = __builtin_amdgcn_readfirstlane(min(min(begin + each, len), limit_of(first_row + there - 1)));
  const uint8_t* const keep = ROWS && a.keep ? a.keep + row0 : nullptr;
  const int all_see = keep ? 0 : __builtin_amdgcn_readfirstlane(limit_of(first_row));  // keys that every row sees

  // Queries: one row tile stays in registers; several lie in LDS, where every wave reads them step by step (in registers as well they
  // would push sums out into memory).
  constexpr bool kQueryLds = RT > 1;
  constexpr int kQueryRow = DP * (int)sizeof(ET) + 16;
  static_assert(kRows * kQueryRow <= kWaves * 16 * kLdRow * 4, "queries lie where the waves' sums come later");
  int limit[RT];
  tok_u4 q[O::kQuery];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const unsigned row = first_row + t * 16 + r16, token = token_of(a, row);
    const bool in = t * 16 + r16 < there;
    limit[t] = in && (!keep || keep[token] != 0) ? limit_of(row) : 0;
    if (kQueryLds && t % kWaves != wave) continue;
    const ET* const from = reinterpret_cast<const ET*>(a.q) + (long long)(row0 + token) * a.ldq + (hk * a.group + (row - token * a.group)) * a.D;
#pragma unroll
    for (int s = 0; s < O::kQuery; ++s) {
      const int d = O::query_at(s, quarter);
      q[s] = tok_u4{0, 0, 0, 0};
      if (in && d < a.D) q[s] = *reinterpret_cast<const tok_u4*>(from + d);
      if constexpr (kQueryLds) *reinterpret_cast<tok_u4*>(lds + (t * 16 + r16) * kQueryRow + d * (int)sizeof(ET)) = q[s];
    }
  }
  if constexpr (kQueryLds) __syncthreads();
  auto query = [&](int t, int i) {
    if constexpr (kQueryLds) return *reinterpret_cast<const tok_u4*>(lds + (t * 16 + r16) * kQueryRow + O::query_at(i, quarter) * (int)sizeof(ET));
    else return q[i];
  };

  f32x4 acc[RT][kEach];
  float top[RT], sum[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    top[t] = kNoScore;
    sum[t] = 0.f;
#pragma unroll
    for (int e = 0; e < kEach; ++e) acc[t][e] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // Where a step's keys are: of each sixteen how many (a page that is none has none), and the first one's row of the cache.
  // Where the keys are rows of this call: which of the sixteen the masker kept.
  struct Place {
    int valid[kGroups];
    unsigned there[kGroups];
    long long at[kGroups];
  };
  auto place_of = [&](int key) {
    Place s;
#pragma unroll
    for (int u = 0; u < kGroups; ++u) {
      const int pos = key + 16 * u;
      s.there[u] = 0xffffu;
      if constexpr (ROWS) {
        s.valid[u] = min(16, max(end - pos, 0));
        s.at[u] = row0 + pos;
        if (keep) s.there[u] = (unsigned)__ballot(r16 < s.valid[u] && keep[min(pos + r16, n - 1)] != 0) & 0xffffu;
        continue;
      }
      const int pg = pos < end ? __builtin_amdgcn_readfirstlane(table[pos >> a.page_bits]) : -1;
      const bool ok = (unsigned)pg < (unsigned)a.pages;
      s.valid[u] = ok ? min(16, end - pos) : 0;
      s.at[u] = ok ? (((long long)pg * a.kv_heads + hk) << a.page_bits) + (pos & ((1 << a.page_bits) - 1)) : 0;
    }
    return s;
  };
  // bytes from a row to the next, of keys and of values, and to the row that a place begins with
  const long long pitch_k = ROWS ? a.ldk : a.D, pitch_v = ROWS ? a.ldv : a.D, skip = ROWS ? hk * a.D : 0;
  auto row_of = [&](const uint8_t* base, long long at, long long pitch) { return base + (at * pitch + skip) * O::kBytes; };
  auto rows_in = [&](const uint8_t* base, const Place& s, int u, long long pitch) {
    return bytes_of(scalar_pointer(row_of(base, s.at[u], pitch)), s.valid[u] ? ((s.valid[u] - 1) * pitch + a.D) * O::kBytes : 0);
  };
  O o;
  float ks[kGroups], vs[kGroups];  // scales: of four lanes in a row each has one of their four keys'
  auto load_keys = [&](const Place& s) {
#pragma unroll
    for (int u = 0; u < kGroups; ++u) {
      o.load_keys(u, rows_in(a.k, s, u, pitch_k), a.D, (unsigned)pitch_k, s.there[u], r16, quarter);
      if constexpr (O::kBytes == 1)  // (all of a page's scales are there)
        ks[u] = __uint_as_float(load4(bytes_of(scalar_pointer(a.ks + s.at[u]), s.valid[u] ? 64 : 0), quarter * 16 + r16 % 4 * 4));
    }
  };
  auto load_values = [&](const Place& s) {
#pragma unroll
    for (int u = 0; u < kGroups; ++u) {
      o.load_values(u, rows_in(a.v, s, u, pitch_v), a.D, (unsigned)pitch_v, s.there[u], r16, quarter);
      if constexpr (O::kBytes == 1)
        vs[u] = __uint_as_float(load4(bytes_of(scalar_pointer(a.vs + s.at[u]), s.valid[u] ? 64 : 0), quarter * 16 + r16 % 4 * 4));
    }
  };

  // A step's keys are asked for when the last step's are used up, its values likewise: something is always under way.
  constexpr int kStride = kWaves * kKeys;
  int key = begin + wave * kKeys;
  Place here = place_of(key);
  if (key < end) {
    load_keys(here);
    load_values(here);
  }
#pragma unroll 1
  for (; key < end; key += kStride) {
    const Place next = place_of(key + kStride);  // (past the end: no keys)
    bool whole = key + kKeys <= all_see;
#pragma unroll
    for (int u = 0; u < kGroups; ++u) whole = whole && here.valid[u] == 16;
    f32x4 sc[RT][kGroups];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      if (t * 16 >= there) break;
#pragma unroll
      for (int u = 0; u < kGroups; ++u) {
        sc[t][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < O::kQuery; ++i) {
          const tok_u4 qf = query(t, i);
          if constexpr (kWide) {
#pragma unroll
            for (int j = 0; j < 4; ++j) sc[t][u] = mma4(__uint_as_float(o.k[u][i][j]), __uint_as_float(qf[j]), sc[t][u]);
          } else {
            sc[t][u] = mma_bf16_16(o.key(u, i), __builtin_bit_cast(bf16x8, qf), sc[t][u]);
          }
        }
        if constexpr (O::kBytes == 1) sc[t][u] *= of_four(ks[u]);
      }
      if constexpr (kQueryLds) __builtin_amdgcn_sched_barrier(0);  // (no reads of all row tiles at once)
    }
    load_keys(next);
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      if (t * 16 >= there) break;
      unsigned unseen = 0;  // keys that the lane's row does not see
      if (!whole) {
#pragma unroll
        for (int u = 0; u < kGroups; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int at = 4 * quarter + i;
            if (!(at < here.valid[u] && key + 16 * u + at < limit[t] && (here.there[u] >> at & 1))) {
              sc[t][u][i] = kNoScore;
              unseen |= 1u << (4 * u + i);
            }
          }
      }
      float most = sc[t][0][0];
#pragma unroll
      for (int u = 0; u < kGroups; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) most = fmaxf(most, sc[t][u][i]);
      most = fmaxf(top[t], quarters_max(most) * a.c);
      const float shift = shift_of(most);
      if (__ballot(most > top[t])) {
        const float shrink = exp2_fast(top[t] - shift);
        sum[t] *= shrink;
#pragma unroll
        for (int e = 0; e < kEach; ++e) acc[t][e] *= shrink;
        top[t] = most;
      }
#pragma unroll
      for (int u = 0; u < kGroups; ++u) {
        f32x4 scales = {1.f, 1.f, 1.f, 1.f};
        if constexpr (O::kBytes == 1) {
          scales = of_four(vs[u]);  // (all lanes take part)
          if (!whole) {             // what a value's scale holds where there is no key, or an unseen one, is nobody's business
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (unseen >> (4 * u + i) & 1) scales[i] = 0.f;
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          sc[t][u][i] = exp2_fast(rounded_exponent(sc[t][u][i], a.c, shift));
          sum[t] += sc[t][u][i];
          if constexpr (O::kBytes == 1) sc[t][u][i] *= scales[i];
        }
      }
    }
    bool bad = false;
    if (all_see < min(key + kKeys, end)) bad = __ballot(o.take_out()) != 0;  // some rows see fewer keys of the step than others
    if constexpr (kWide) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < kEach; ++e)
#pragma unroll
          for (int t = 0; t < RT; ++t)
            if (t * 16 < there) acc[t][e] = mma4(o.v[0][i][e], sc[t][0][i], acc[t][e]);
    } else {
#pragma unroll
      for (int h = 0; h < kGroups / 2; ++h) {
        tok_u4 w[RT], rest[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t)
          if (t * 16 < there)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              unsigned lead, last;
              two_parts(sc[t][2 * h + j / 2][j % 2 * 2], sc[t][2 * h + j / 2][j % 2 * 2 + 1], lead, last);
              w[t][j] = lead;
              rest[t][j] = last;
            }
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
          const tok_u4 v = o.value(h, e);
#pragma unroll
          for (int t = 0; t < RT; ++t)
            if (t * 16 < there) {
              acc[t][e] = mma_bf16_16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, w[t]), acc[t][e]);
              acc[t][e] = mma_bf16_16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, rest[t]), acc[t][e]);
            }
        }
      }
    }
    load_values(next);
    if (bad) {
#pragma unroll
      for (int u = 0; u < kGroups; ++u)
#pragma unroll 1
        for (int j = 0; j < here.valid[u]; ++j) {
          if (!(here.there[u] >> j & 1)) continue;
          const uint8_t* const row = row_of(a.v, here.at[u] + j, pitch_v);
#pragma unroll 1
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
              const float v = O::value_at(row, min(kEach * (4 * quarter + i) + e, a.D - 1));
#pragma unroll
              for (int t = 0; t < RT; ++t) {
                const float add = key + 16 * u + j < limit[t] && not_finite(v) ? v : 0.f;
#pragma unroll
                for (int x = 0; x < 4; ++x) acc[t][e][x] += x == i ? add : 0.f;
              }
            }
        }
    }
    here = next;
  }

  // The waves' parts: each row's maximum over them, their sums relative to it.
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const float all = quarters_sum(sum[t]);
    if (quarter == 0) {
      stats[(wave * kRows + t * 16 + r16) * 2] = top[t];
      stats[(wave * kRows + t * 16 + r16) * 2 + 1] = all;
    }
  }
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    if (t * 16 >= there) break;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < kEach; e += 4)
        *reinterpret_cast<f32x4*>(sums + (wave * 16 + r16) * kLdRow + kEach * (4 * quarter + i) + e) =
            f32x4{acc[t][e][i], acc[t][e + 1][i], acc[t][e + 2][i], acc[t][e + 3][i]};
    __syncthreads();
    // sixteen threads a row, kEach channels each
    const int r = threadIdx.x / 16, d = threadIdx.x % 16 * kEach;
    float most = kNoScore, total = 0.f, f[kEach] = {};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) most = fmaxf(most, stats[(w * kRows + t * 16 + r) * 2]);
    const float shift = shift_of(most);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float by = exp2_fast(stats[(w * kRows + t * 16 + r) * 2] - shift);
      total = fmaf(stats[(w * kRows + t * 16 + r) * 2 + 1], by, total);
#pragma unroll
      for (int e = 0; e < kEach; ++e) f[e] = fmaf(sums[(w * 16 + r) * kLdRow + d + e], by, f[e]);
    }
    if (t * 16 + r >= there) continue;
    const unsigned row = first_row + t * 16 + r;
    const unsigned token = token_of(a, row);
    const long long tok = row0 + token;
    const int h = hk * a.group + (int)(row - token * a.group);
    if (a.splits + a.prefix_splits > 1) {
      const long long at = ((long long)(shared ? a.splits + split : split) * a.T + tok) * a.heads + h;
      if (d < a.D)
#pragma unroll
        for (int e = 0; e < kEach; e += 4) *reinterpret_cast<f32x4*>(a.part_out + at * a.D + d + e) = f32x4{f[e], f[e + 1], f[e + 2], f[e + 3]};
      if (d == 0) {
        a.part_stat[2 * at] = most;
        a.part_stat[2 * at + 1] = total;
      }
    } else if (d < a.D) {
      const float inv = 1.f / total;
      ET* const out = reinterpret_cast<ET*>(a.out) + tok * a.ldo + h * a.D + d;
#pragma unroll
      for (int e = 0; e < kEach; e += 4) {
        f32x4 o = {f[e] * inv, f[e + 1] * inv, f[e + 2] * inv, f[e + 3] * inv};
        if (total == 0.f) o = f32x4{0.f, 0.f, 0.f, 0.f};
        store4(out + e, o);
      }
    }
  }
}

// Joins the parts of a row, 32 threads each of which has four channels: SLOTS groups of them a row, each takes every SLOTSth part, eight at
// most.  What a thread reads of the sums does not depend on the row's statistics (parts that do not count are dropped behind their loads), so
// that the trips to memory overlap.  One row a workgroup where there are few (8 slots; 32 rows 4.7 us, 2048 rows 6.0), eight where there are many.
template <typename ET, int SLOTS>
__global__ __launch_bounds__(256) void k_join(CachedArgs a) {
  constexpr int kRows = 8 / SLOTS, kHalf = kWave / 2;
  __shared__ f32x4 part[8][kHalf];
  const int lane = lane_id(), r32 = lane % kHalf, slot = threadIdx.x / kHalf % SLOTS, d = r32 * 4, parts = a.splits + a.prefix_splits;
  const long long rows = (long long)a.T * a.heads;
  const unsigned mine = blockIdx.x * kRows + threadIdx.x / (kHalf * SLOTS);
  const unsigned row = (unsigned)min((long long)mine, rows - 1);  // (below 2^31)
  const int token = (int)(row / (unsigned)a.heads), head = (int)(row - (unsigned)token * a.heads);
  f32x4 v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i * SLOTS + slot < parts && d < a.D) v[i] = *reinterpret_cast<const f32x4*>(a.part_out + ((long long)(i * SLOTS + slot) * rows + row) * a.D + d);
  // statistics: a lane has parts r32 and r32 + 32 (more than 32 where a row has all of a workgroup only)
  float top[2], sum[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int p = r32 + j * kHalf;
    float2 s = {kNoScore, 0.f};
    if (p < parts) s = *reinterpret_cast<const float2*>(a.part_stat + 2 * ((long long)p * rows + row));
    top[j] = s.x;
    sum[j] = s.y;
  }
  // the halves of a wave may have rows of two tokens
  const int first = __builtin_amdgcn_readlane(token, 0), second = __builtin_amdgcn_readlane(token, kHalf);
  Sequence seq = sequence_at(a.offsets, a.lens, a.B, a.T, [&](int r, int) { return r <= first; });
  if (SLOTS == 1 && second != first) {
    const Sequence s = sequence_at(a.offsets, a.lens, a.B, a.T, [&](int r, int) { return r <= second; });
    if (lane >= kHalf) seq = s;
  }
  const int own = parts_of(cached_tokens(a, seq.len), a.splits), shared = a.prefix_splits ? parts_of(a.prefix_len, a.prefix_splits) : 0;
  const bool wanted = mine < rows && token >= seq.row0 && token < seq.next;
  float most = kNoScore;
  bool there[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int p = r32 + j * kHalf;
    there[j] = p < a.splits ? p < own : p - a.splits < shared;  // (else nobody wrote the part)
    if (there[j]) most = fmaxf(most, top[j]);
  }
#pragma unroll
  for (int o = 1; o < kHalf; o <<= 1) most = fmaxf(most, __shfl_xor(most, o, kWave));
  float by[2], total = 0.f;
  unsigned counts[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const bool c = there[j] && sum[j] != 0.f;  // (has a weight; scores that are all NaN leave a NaN for a sum, and no maximum)
    by[j] = c ? exp2_fast(top[j] - most) : 0.f;
    total += c ? sum[j] * by[j] : 0.f;
    counts[j] = (unsigned)(__ballot(there[j]) >> (lane / kHalf * kHalf));  // (without a weight: sums of 0, or NaN of values that are no numbers)
  }
#pragma unroll
  for (int o = 1; o < kHalf; o <<= 1) total += __shfl_xor(total, o, kWave);
  f32x4 f = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int p = i * SLOTS + slot, j = i * SLOTS / kHalf;
    const float w = __shfl(by[j], lane / kHalf * kHalf + p % kHalf, kWave);
    if ((counts[j] >> (p % kHalf)) & 1)
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] = fmaf(v[i][e], w, f[e]);
  }
  if constexpr (SLOTS > 1) {
    if (!wanted) return;  // (all of the workgroup)
    part[slot][r32] = f;
    __syncthreads();
    if (slot != 0) return;
#pragma unroll
    for (int i = 1; i < SLOTS; ++i) f += part[i][r32];
  }
  if (!wanted || d >= a.D) return;
  const float inv = 1.f / total;
  f *= inv;
  if (total == 0.f) f = f32x4{0.f, 0.f, 0.f, 0.f};
  store4(reinterpret_cast<ET*>(a.out) + token * a.ldo + head * a.D + d, f);
}

namespace {

// group_by, group_shift: with 2^l the next power of two, the least multiple m / 2^(31 + l) not below 1 / group is off by less than
// 2^l / 2^(31 + l) / group, which 2^31 rows do not raise to another whole number.
void set_group(CachedArgs& a, int group) {
  int l = 0;
  while ((1 << l) < group) ++l;
  a.group = group;
  a.group_shift = 31 + l;
  a.group_by = (unsigned)(((1ull << (31 + l)) + group - 1) / group);
}

// ---- plan -------------------------------------------------------------------------------------------------------------------
struct Plan {
  int rt;                   // row tiles of a workgroup; 0: the kernel of many rows
  int own, shared;          // parts of the sequences' own keys, and of the prefix
  long long tiles, prefix_tiles;
  size_t stat_at, bytes;    // workspace: sums, then statistics
};
// Which kernel: a workgroup of sixteen rows, of 32, or of 128 with its keys through LDS.  The last two, in us (sequences x new tokens + cached
// ones, 32 heads of 128 over 8, bf16): 1 x 512 + 8000 179, 109;  2 x 200 + 4000 96, 77;  4 x 128 + 4000 105, 71;  8 x 64 + 4000 105, 107;  16 x 12 + 4000
// 75, 94.  In float32 32 rows are the faster ones (4 x 300 + 2000, 16 heads of 64: 157, 187), and behind a prefix (32 x 1 + 500 behind 16384: 41, 47).
// The rows of a sequence are the mean of all: many new tokens of one among single ones of the others go by 32 rows.
inline int row_tiles(double rows, double of_a_sequence, int type) {
  return type == LAUD_BF16 && of_a_sequence >= 512 ? 0 : rows <= 16 ? 1 : 2;
}

// Parts: as many as stay within so many workgroups, none of fewer than 128 keys.  1024 where a few rows wait for memory, 512 where many rows keep
// the matrix cores busy; with a prefix 256 each for it and for the sequences' own keys (32 x 1 + 500 behind 16384: 52 us with 1024, 46 with
// 512, 41 with 256, 59 with 128: whatever is split is joined again).  But none of more than 2048 keys of a row of the table while that stays within 1024
// workgroups (33 x 316 new tokens of 4286, 8 heads of 32 in 8 bits: 116 -> 76 us; 43 x 121 of 25845 behind 30: 259 -> 177); and two parts of as many
// keys where one makes 512 to 819 workgroups (65 x 1 of up to 8192, 32 heads of 128 over 8: 224 -> 182 us, 100 x 1 of 32768 in 8 bits 1423 -> 1295; of more
// workgroups it does not pay: 127 x 1 1391 -> 1418).
// Rounded up, a last part of few workgroups waits for nearly as long as the others (1 x 512 new tokens of 8512: 109 us with 4 parts, 145 with 5; 48 x 1 of
// 32768 1063 -> 1092; 20 x 1 of 500 behind 5000 26 -> 31; but 33 x 1 820 -> 796); sixty drawn caches take as long either way.
// A part of the sums costs its way to memory and back, c = rows * D * 8 bytes / 5 TB/s, a key 16 ns of a workgroup's time: p parts 16 ns * keys
// / p + c * p, least at p = sqrt(16 ns * keys / c); and splitting at all costs another launch, 4 us (9 x 398 new tokens, 8 heads of 80: 43 -> 13 us with one
// part in place of five; 3 x 115 of 4304 in 8 bits, 32 heads of 128: 31.5 -> 12.5; 33 x 1 of 108, 16 heads of 64: 12.8 -> 5.6).
// All of this takes the sequences for about as long as the table has room for: parts of one long sequence among short ones are as many as theirs.
inline int parts_for(double workgroups, double groups, long long keys, double sums, bool joined, int most) {
  const double all = 0.016 * keys, part = sums * 8 / 5e6;  // us
  if (!joined && all / 2 < 4 + 2 * part) return 1;
  double filled = 1024 / groups;
  if (filled >= 1.25 && filled < 2) filled = 2;
  const double want = std::min(std::max(workgroups / groups, std::min(filled, keys / 2048.0)), std::sqrt(all / part));
  const long long room = (keys + kPartStep - 1) / kPartStep;
  return (int)std::max(1ll, std::min({(long long)want, room, (long long)most}));
}

Plan plan_of(const laud_heads* p, const laud_cache* c, const laud_batch* b, int T) {
  Plan s{};
  const int group = p->heads / p->kv_heads;
  const bool prefix = b->prefix_len > 0;
  const double rows = (double)T * group;
  s.rt = row_tiles(prefix ? rows : rows / b->B, rows / b->B, c->dtype);
  const int per = s.rt ? 16 * s.rt : kManyRows;
  s.tiles = tiles_of(T, b->B, group, per);
  const double busy = std::max((double)b->B, rows / per) * p->kv_heads;
  const double sums = (double)T * p->heads * p->D;
  s.own = parts_for(prefix ? 256 : s.rt ? 1024 : 512, busy, (long long)b->table_ld * c->page, sums, prefix, prefix ? kMaxParts / 2 : kMaxParts);
  if (prefix) {
    s.prefix_tiles = ((long long)T * group - 1) / per + 1;
    s.shared = parts_for(256, (double)s.prefix_tiles * p->kv_heads, b->prefix_len, sums, true, kMaxParts / 2);
  }
  if (s.own + s.shared > 1) {
    const size_t all = (size_t)(s.own + s.shared) * T * p->heads;
    s.stat_at = align_up(all * p->D * 4, 256);
    s.bytes = s.stat_at + all * 8;
  }
  return s;
}

template <typename ET, typename CT, int DP, int RT, bool ROWS>
void launch_cached(const CachedArgs& a, unsigned groups, hipStream_t st) {
  constexpr int kLds = kWaves * 16 * (DP + 4) * 4 + kWaves * 16 * RT * 8;
  hipLaunchKernelGGL((k_cached<ET, CT, DP, RT, ROWS>), dim3(groups), dim3(kWaves * kWave), kLds, st, a);
}
template <typename ET, typename CT>
void launch_rows(const CachedArgs& a, int rt, unsigned groups, hipStream_t st) {
  if (a.D <= 64) {
    if (rt == 1) launch_cached<ET, CT, 64, 1, false>(a, groups, st);
    else launch_cached<ET, CT, 64, 2, false>(a, groups, st);
  } else {
    if (rt == 1) launch_cached<ET, CT, 128, 1, false>(a, groups, st);
    else launch_cached<ET, CT, 128, 2, false>(a, groups, st);
  }
}
template <typename ET>
void launch_join(const CachedArgs& a, hipStream_t st) {
  const unsigned rows = (unsigned)a.T * (unsigned)a.heads;
  if (rows >= 4096 && a.splits + a.prefix_splits <= 8) hipLaunchKernelGGL((k_join<ET, 1>), dim3((rows + 7) / 8), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((k_join<ET, 8>), dim3(rows), dim3(256), 0, st, a);
}
void launch_types(const CachedArgs& a, int cache_type, int rt, unsigned groups, hipStream_t st) {
  if (cache_type == LAUD_F32) launch_rows<float, float>(a, rt, groups, st);
  else if (cache_type == LAUD_BF16) launch_rows<bf16_t, bf16_t>(a, rt, groups, st);
  else launch_rows<bf16_t, uint8_t>(a, rt, groups, st);
}

}  // namespace

int attend_few(const laud_heads& p, int B, const int32_t* offsets, int T, const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v,
               int64_t ldv, const uint8_t* keep, void* out, int64_t ldo, hipStream_t st) {
  CachedArgs a{};
  set_group(a, p.heads / p.kv_heads);
  a.heads = p.heads; a.kv_heads = p.kv_heads; a.D = p.D; a.causal = p.causal; a.B = B; a.T = T;
  a.splits = 1; a.c = p.scale * kLog2e;
  a.offsets = offsets; a.k = (const uint8_t*)k; a.v = (const uint8_t*)v; a.ldk = ldk; a.ldv = ldv; a.keep = keep;
  a.q = q; a.out = out; a.ldq = ldq; a.ldo = ldo;
  const long long tiles = tiles_of(T, B, a.group, 16);  // (as many as a launch takes: laud_attention has looked)
  a.tiles = (int)tiles;
  const unsigned groups = (unsigned)(tiles * a.kv_heads);
  if (p.dtype == LAUD_F32) {
    if (p.D <= 64) launch_cached<float, float, 64, 1, true>(a, groups, st);
    else launch_cached<float, float, 128, 1, true>(a, groups, st);
  } else {
    if (p.D <= 64) launch_cached<bf16_t, bf16_t, 64, 1, true>(a, groups, st);
    else launch_cached<bf16_t, bf16_t, 128, 1, true>(a, groups, st);
  }
  return check_launch();
}

namespace {

// The arguments that the host sees, all but the rows and the workspace.
int check_cached(const laud_heads* p, const laud_cache* c, const laud_batch* b, int T) {
  int bad = check_heads(p);
  if (!bad) bad = check_cache(c, b);
  if (bad) return bad;
  if (T < 0 || p->kv_heads != c->kv_heads || p->D != c->D || b->prefix_len < 0 || b->prefix_len > 1 << 30 ||
      (b->prefix_len > 0 && (!b->prefix || !aligned4(b->prefix))) ||
      !(c->dtype == p->dtype || (c->dtype == LAUD_E4M3 && p->dtype == LAUD_BF16)))
    return LAUD_ERR_INVALID_ARG;
  if ((int64_t)T * p->heads > INT32_MAX) return LAUD_ERR_UNSUPPORTED;
  return LAUD_OK;
}

}  // namespace
}  // namespace laud

extern "C" size_t laud_cache_attention_workspace(const laud_heads* p, const laud_cache* c, const laud_batch* b, int T) {
  using namespace laud;
  if (check_cached(p, c, b, T) || T == 0 || b->B == 0) return 0;
  return plan_of(p, c, b, T).bytes;
}

extern "C" int laud_cache_attention(const laud_heads* p, const laud_cache* c, const laud_batch* b, int T, const void* q, int64_t ldq, void* out,
                                    int64_t ldo, void* ws, size_t ws_bytes, void* stream) {
  using namespace laud;
  const int bad = check_cached(p, c, b, T);
  if (bad) return bad;
  if (b->B == 0 || T == 0) return LAUD_OK;
  const int C = p->heads * p->D;
  if (!check_batch(b) || !q || !out || !good_ld(ldq, C, 8) || !good_ld(ldo, C, 8) || !aligned16(q) || !aligned16(out)) return LAUD_ERR_INVALID_ARG;
  const size_t eb = elem_bytes(p->dtype), prefix_bytes = ((size_t)b->prefix_len + c->page - 1) / c->page * 4;
  if (!same_or_apart(q, ldq, eb, out, ldo, eb, T, C) || rows_meet_cache(c, out, ldo, eb, C, T) || rows_meet_batch(b, out, ldo, eb, T, C) ||
      range_meets_rows(b->prefix_len ? b->prefix : nullptr, prefix_bytes, out, ldo, eb, T, C))
    return LAUD_ERR_INVALID_ARG;
  const Plan s = plan_of(p, c, b, T);
  if (s.bytes) {
    if (!ws || ws_bytes < s.bytes) return LAUD_ERR_WORKSPACE;
    if (!aligned16(ws) || range_meets_rows(ws, s.bytes, q, ldq, eb, T, C) || range_meets_rows(ws, s.bytes, out, ldo, eb, T, C) ||
        cache_meets(c, ws, s.bytes) || (b->prefix_len && ranges_meet(ws, s.bytes, b->prefix, prefix_bytes)))
      return LAUD_ERR_INVALID_ARG;
    for (const Span& x : BatchSpans(b).s)
      if (ranges_meet(ws, s.bytes, x.p, x.n)) return LAUD_ERR_INVALID_ARG;
  }
  if (s.rt == 0 && attend_init_device() != LAUD_OK) return LAUD_ERR_HIP;
  const double own = (double)s.tiles * p->kv_heads * s.own, shared = (double)s.prefix_tiles * p->kv_heads * s.shared;
  if (!launchable(own + shared, kWaves * kWave) || (s.bytes && !launchable((double)T * p->heads, 256))) return LAUD_ERR_UNSUPPORTED;
  CachedArgs a{};
  set_group(a, p->heads / p->kv_heads);
  a.heads = p->heads; a.kv_heads = p->kv_heads; a.D = p->D; a.causal = p->causal; a.B = b->B; a.T = T;
  a.pages = c->pages; a.page_bits = page_bits(c); a.table_ld = b->table_ld;
  a.tiles = (int)s.tiles; a.splits = s.own; a.prefix_tiles = (int)s.prefix_tiles; a.prefix_splits = s.shared;
  a.prefix_groups = (unsigned)shared; a.prefix_len = b->prefix_len;
  a.by_xcd = s.rt != 1 && (long long)p->kv_heads * s.own % 8 == 0;
  a.prefix_by_xcd = (long long)p->kv_heads * s.shared % 8 == 0;
  a.c = p->scale * kLog2e;
  a.offsets = b->offsets; a.lens = b->lens; a.table = b->table; a.prefix = b->prefix;
  a.k = (const uint8_t*)c->k; a.v = (const uint8_t*)c->v; a.ks = c->k_scale; a.vs = c->v_scale;
  a.q = q; a.out = out; a.ldq = ldq; a.ldo = ldo;
  a.part_out = s.bytes ? (float*)ws : nullptr;
  a.part_stat = s.bytes ? (float*)((char*)ws + s.stat_at) : nullptr;
  clear_stale_error();
  hipStream_t st = (hipStream_t)stream;
  if (s.rt == 0) launch_many_rows(a, (unsigned)(own + shared), st);
  else launch_types(a, c->dtype, s.rt, (unsigned)(own + shared), st);
  if (s.own + s.shared > 1) {
    if (p->dtype == LAUD_BF16) launch_join<bf16_t>(a, st);
    else launch_join<float>(a, st);
  }
  return check_launch();
}
