// Attention of new tokens over a paged cache: parts of the keys by workgroup, joined where there are several.
#include "laud_heads.h"

namespace laud {
namespace {

struct CachedArgs {
  int heads, group, kv_heads, D, causal, B, T, pages, page_bits, table_ld, prefix_len;
  int tiles, splits;      // tiles of query rows; parts that a tile's keys are shared out over
  int parts, first_part;  // all parts that are joined; the first of this launch
  int shared;             // the prefix: every token's rows over the same keys
  int by_xcd;
  float c;                // scale * log2(e)
  const int32_t *offsets, *lens, *table;
  const uint8_t *k, *v;
  const float *ks, *vs;
  const void* q;
  void* out;
  float *part_out, *part_stat;  // [parts][T * heads][D] and [parts][T * heads][2]: maximum and sum
  int64_t ldq, ldo;
};

constexpr int kWaves = 4, kMaxParts = 64, kPartStep = 128;
// Keys of a part: the same for every tile of a sequence, so that whoever joins the parts knows how many there are.
__device__ __forceinline__ int part_keys(int len, int splits) {
  const int each = (len + splits - 1) / splits;
  return max((each + kPartStep - 1) / kPartStep * kPartStep, kPartStep);
}
__device__ __forceinline__ int cached_tokens(const CachedArgs& a, int b) {
  const long long room = (long long)a.table_ld << a.page_bits;
  return (int)min((long long)max(a.lens[b], 0), room);
}

// ---- operands ---------------------------------------------------------------------------------------------------------------
// CT: the cache's type.  A step has GROUPS times sixteen keys; lane l holds key l % 16 of each for the scores (keys * queries: a lane's
// results are keys 4 * (l / 16) .. +3 of its query, l % 16), and of the values keys 4 * (l / 16) .. +3, elements kEach * (l % 16) .. of
// each: all of a row's bytes come in one piece a lane, straight into registers, and with element e of every lane the matrix instruction
// makes channels kEach * m + e, m = 0 .. 15.  Nothing has to change lanes between the two products.
template <typename CT, int DP> struct Operands;

template <int DP>
struct Operands<bf16_t, DP> {
  static constexpr int kGroups = 2, kEach = DP / 16, kPieces = DP / 32, kQuery = DP / 32;
  static constexpr int kBytes = 2;
  tok_u4 k[kGroups][kPieces];
  unsigned v[kGroups][4][kEach / 2];
  __device__ __forceinline__ void load(int u, __amdgpu_buffer_rsrc_t rk, __amdgpu_buffer_rsrc_t rv, int D, int r16, int quarter) {
#pragma unroll
    for (int s = 0; s < kPieces; ++s) {
      const int d = 32 * s + 8 * quarter;
      k[u][s] = load16(rk, d < D ? (unsigned)(r16 * D + d) * 2u : kOutside);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned at = r16 * kEach < D ? (unsigned)((4 * quarter + j) * D + r16 * kEach) * 2u : kOutside;
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
  // element e of the lane's eight keys
  __device__ __forceinline__ tok_u4 value(int e) const {
    tok_u4 r;
#pragma unroll
    for (int p = 0; p < 4; ++p)
      r[p] = __builtin_amdgcn_perm(v[p / 2][p % 2 * 2 + 1][e / 2], v[p / 2][p % 2 * 2][e / 2], e % 2 ? 0x07060302u : 0x05040100u);
    return r;
  }
};

template <int DP>
struct Operands<uint8_t, DP> {
  static constexpr int kGroups = 2, kEach = DP / 16, kPieces = DP / 64, kQuery = DP / 32;
  static constexpr int kBytes = 1;
  tok_u4 k[kGroups][kPieces];
  unsigned v[kGroups][4][kEach / 4];
  __device__ __forceinline__ void load(int u, __amdgpu_buffer_rsrc_t rk, __amdgpu_buffer_rsrc_t rv, int D, int r16, int quarter) {
#pragma unroll
    for (int s = 0; s < kPieces; ++s) {
      const int d = 64 * s + 16 * quarter;
      k[u][s] = load16(rk, d < D ? (unsigned)(r16 * D + d) : kOutside);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned at = r16 * kEach < D ? (unsigned)((4 * quarter + j) * D + r16 * kEach) : kOutside;
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
  __device__ __forceinline__ tok_u4 value(int e) const {
    tok_u4 r;
#pragma unroll
    for (int p = 0; p < 4; ++p) {  // codes e and its neighbour of two keys, the asked one widened
      const unsigned w = __builtin_amdgcn_perm(v[p / 2][p % 2 * 2 + 1][e / 4], v[p / 2][p % 2 * 2][e / 4], e % 4 / 2 ? 0x07030602u : 0x05010400u);
      bf16x2 h;
      if (e % 2) h = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true);
      else h = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false);
      r[p] = __builtin_bit_cast(unsigned, h);
    }
    return r;
  }
};

template <int DP>
struct Operands<float, DP> {
  static constexpr int kGroups = 1, kEach = DP / 16, kPieces = DP / 16, kQuery = DP / 16;
  static constexpr int kBytes = 4;
  tok_u4 k[kGroups][kPieces];
  float v[kGroups][4][kEach];
  __device__ __forceinline__ void load(int u, __amdgpu_buffer_rsrc_t rk, __amdgpu_buffer_rsrc_t rv, int D, int r16, int quarter) {
#pragma unroll
    for (int s = 0; s < kPieces; ++s) {
      const int d = 16 * s + 4 * quarter;
      k[u][s] = load16(rk, d < D ? (unsigned)(r16 * D + d) * 4u : kOutside);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int h = 0; h < kEach / 4; ++h) {
        const tok_u4 w = load16(rv, r16 * kEach < D ? (unsigned)((4 * quarter + j) * D + r16 * kEach + 4 * h) * 4u : kOutside);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[u][j][4 * h + e] = __uint_as_float(w[e]);
      }
  }
  static __device__ __forceinline__ int query_at(int s, int quarter) { return 16 * s + 4 * quarter; }  // four elements
};

__device__ __forceinline__ f32x4 mma4(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// Sixteen query rows a row tile (RT of them a workgroup): the tokens of a sequence times the query heads of a key head, so that a key is
// fetched once for all of them.  Four waves share a part's keys, each takes every fourth step of 16 or 32 keys; their sums are joined through LDS.
template <typename ET, typename CT, int DP, int RT>
__global__ __launch_bounds__(kWaves * kWave, (RT > 2 ? 1 : 2)) void k_cached(CachedArgs a) {
  typedef Operands<CT, DP> O;
  constexpr bool kWide = sizeof(CT) == 4;  // float32 instructions
  constexpr int kGroups = O::kGroups, kKeys = 16 * kGroups, kRows = 16 * RT, kEach = O::kEach, kLdRow = DP + 4;
  extern __shared__ __align__(16) unsigned char lds[];
  float* const sums = reinterpret_cast<float*>(lds);                    // [wave][16][kLdRow]
  float* const stats = sums + kWaves * 16 * kLdRow;                     // [wave][kRows][2]
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), r16 = lane % 16, quarter = lane / 16;

  // Which rows, key head and part.  Where several tiles read the same keys they go to one XCD, one behind the other.
  int tile, hk, split;
  if (a.by_xcd) {
    const unsigned j = blockIdx.x / 8;
    const unsigned g = j / a.tiles * 8 + blockIdx.x % 8;
    tile = j % a.tiles;
    hk = g % a.kv_heads;
    split = g / a.kv_heads;
  } else {
    split = blockIdx.x % a.splits;
    const unsigned j = blockIdx.x / a.splits;
    hk = j % a.kv_heads;
    tile = j / a.kv_heads;
  }
  int b = 0, row0 = 0, n = a.T, len = a.prefix_len;
  const int32_t* table = a.table;
  if (!a.shared) {
    b = last_not_above(a.B, [&](int i) { return first_tile(a.offsets, i, a.T, a.group, kRows) <= tile; });
    row0 = row_at(a.offsets, b, a.T);
    n = row_at(a.offsets, b + 1, a.T) - row0;
    if ((long long)tile < first_tile(a.offsets, b, a.T, a.group, kRows)) return;
    tile -= (int)first_tile(a.offsets, b, a.T, a.group, kRows);
    len = cached_tokens(a, b);
    table += (long long)b * a.table_ld;
  }
  if (n <= 0) return;
  const unsigned rows = (unsigned)n * (unsigned)a.group, first_row = (unsigned)tile * kRows;  // (T * heads is below 2^31)
  if (first_row >= rows) return;
  const int there = (int)min((unsigned)kRows, rows - first_row);  // rows of this tile
  const int each = part_keys(len, a.splits);
  if (split > 0 && (long long)split * each >= len) return;
  const long long past = (long long)(a.shared ? len : a.lens[b]) - n;  // position of the first token
  const bool causal = a.causal && !a.shared;
  auto limit_of = [&](unsigned row) -> int {  // keys that a row sees
    return causal ? (int)min(max(past + row / (unsigned)a.group + 1, 0ll), (long long)len) : len;
  };
  const int begin = split * each;
  const int end = min(min(begin + each, len), limit_of(first_row + there - 1)), all_see = limit_of(first_row);

  // queries, for good
  int limit[RT];
  tok_u4 q[RT][O::kQuery];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const unsigned row = first_row + t * 16 + r16, token = row / (unsigned)a.group;
    const bool in = t * 16 + r16 < there;
    limit[t] = in ? limit_of(row) : 0;
    const ET* const from = reinterpret_cast<const ET*>(a.q) + (long long)(row0 + token) * a.ldq + (hk * a.group + (row - token * a.group)) * a.D;
#pragma unroll
    for (int s = 0; s < O::kQuery; ++s) {
      const int d = O::query_at(s, quarter);
      q[t][s] = tok_u4{0, 0, 0, 0};
      if (in && d < a.D) q[t][s] = *reinterpret_cast<const tok_u4*>(from + d);
    }
  }

  f32x4 acc[RT][kEach];
  float top[RT], sum[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    top[t] = kNoScore;
    sum[t] = 0.f;
#pragma unroll
    for (int e = 0; e < kEach; ++e) acc[t][e] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // A step's operands, and how many keys of each sixteen there are (a page that is none has none).
  struct Step {
    O o;
    f32x4 ks[kGroups], vs[kGroups];
    int valid[kGroups];
  };
  auto page_at = [&](int key, int u) {
    const int pos = key + 16 * u;
    return pos < end ? table[pos >> a.page_bits] : -1;
  };
  auto load = [&](Step& s, int key, const int (&page)[kGroups]) {
#pragma unroll
    for (int u = 0; u < kGroups; ++u) {
      const int pos = key + 16 * u, pg = __builtin_amdgcn_readfirstlane(page[u]);
      const bool ok = pos < end && (unsigned)pg < (unsigned)a.pages;
      s.valid[u] = ok ? min(16, end - pos) : 0;
      const long long at = ok ? (((long long)pg * a.kv_heads + hk) << a.page_bits) + (pos & ((1 << a.page_bits) - 1)) : 0;
      const int bytes = s.valid[u] * a.D * O::kBytes;
      s.o.load(u, bytes_of(a.k + at * a.D * O::kBytes, bytes), bytes_of(a.v + at * a.D * O::kBytes, bytes), a.D, r16, quarter);
      if constexpr (O::kBytes == 1) {
        const __amdgpu_buffer_rsrc_t rks = bytes_of(a.ks + at, ok ? 64 : 0), rvs = bytes_of(a.vs + at, ok ? 64 : 0);  // (all of a page's scales are there)
        s.ks[u] = __builtin_bit_cast(f32x4, load16(rks, quarter * 16));
        s.vs[u] = __builtin_bit_cast(f32x4, load16(rvs, quarter * 16));
      }
    }
  };
  auto compute = [&](const Step& s, int key) {
    bool whole = key + kKeys <= all_see;
#pragma unroll
    for (int u = 0; u < kGroups; ++u) whole = whole && s.valid[u] == 16;
    float p[RT][kGroups][4];
    unsigned seen[RT];  // bits 4 u + i: the lane's query sees key i of the lane's four
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      if (t * 16 >= there) break;
      f32x4 sc[kGroups];
#pragma unroll
      for (int u = 0; u < kGroups; ++u) {
        sc[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < O::kQuery; ++i) {
          if constexpr (kWide) {
#pragma unroll
            for (int j = 0; j < 4; ++j) sc[u] = mma4(__uint_as_float(s.o.k[u][i][j]), __uint_as_float(q[t][i][j]), sc[u]);
          } else {
            sc[u] = mma_bf16_16(s.o.key(u, i), __builtin_bit_cast(bf16x8, q[t][i]), sc[u]);
          }
        }
        if constexpr (O::kBytes == 1) sc[u] *= s.ks[u];
      }
      seen[t] = (1u << (4 * kGroups)) - 1;
      if (!whole) {
        seen[t] = 0;
#pragma unroll
        for (int u = 0; u < kGroups; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int at = 4 * quarter + i;
            const bool sees = at < s.valid[u] && key + 16 * u + at < limit[t];
            seen[t] |= sees ? 1u << (4 * u + i) : 0u;
            if (!sees) sc[u][i] = kNoScore;
          }
      }
      float most = sc[0][0];
#pragma unroll
      for (int u = 0; u < kGroups; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) most = fmaxf(most, sc[u][i]);
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
      for (int u = 0; u < kGroups; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[t][u][i] = exp2_fast(fmaf(sc[u][i], a.c, -shift));
          sum[t] += p[t][u][i];
          if constexpr (O::kBytes == 1) p[t][u][i] = (seen[t] >> (4 * u + i)) & 1 ? p[t][u][i] * s.vs[u][i] : 0.f;
        }
    }
    const bool mixed = all_see < min(key + kKeys, end);  // some rows see fewer keys of the step than others
    if constexpr (kWide) {
      bool clean = true;
      if (mixed) {
        bool bad = false;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < kEach; ++e) bad |= not_finite(s.o.v[0][i][e]);
        clean = __ballot(bad) == 0;
      }
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        if (t * 16 >= there) break;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < kEach; ++e) {
            const float v = s.o.v[0][i][e];
            acc[t][e] = mma4(clean || !not_finite(v) ? v : 0.f, p[t][0][i], acc[t][e]);
          }
        if (!clean) {
#pragma unroll
          for (int e = 0; e < kEach; ++e)
#pragma unroll
            for (int sign = 0; sign < 2; ++sign) {
              f32x4 found = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int i = 0; i < 4; ++i) found = mma4(endless(s.o.v[0][i][e], sign), (seen[t] >> i) & 1 ? 1.f : 0.f, found);
              add_endless(acc[t][e], found, sign);
            }
        }
      }
    } else {
      tok_u4 w[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t)
        if (t * 16 < there)
#pragma unroll
          for (int j = 0; j < 4; ++j) w[t][j] = pack_bf16(p[t][j / 2][j % 2 * 2], p[t][j / 2][j % 2 * 2 + 1]);
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        tok_u4 v = s.o.value(e);
        bool bad = false;
        if (mixed) {
#pragma unroll
          for (int j = 0; j < 4; ++j) bad |= not_finite2(v[j]);
          bad = __ballot(bad) != 0;
        }
        if (bad) {
#pragma unroll
          for (int sign = 0; sign < 2; ++sign) {
            tok_u4 x;
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = endless2(v[j], sign);
#pragma unroll
            for (int t = 0; t < RT; ++t) {
              if (t * 16 >= there) break;
              tok_u4 sees;
#pragma unroll
              for (int j = 0; j < 4; ++j) sees[j] = ((seen[t] >> (2 * j)) & 1 ? 0x3f80u : 0u) | ((seen[t] >> (2 * j)) & 2 ? 0x3f800000u : 0u);
              const f32x4 found = mma_bf16_16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, sees), f32x4{0.f, 0.f, 0.f, 0.f});
              add_endless(acc[t][e], found, sign);
            }
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] = finite2(v[j]);
        }
#pragma unroll
        for (int t = 0; t < RT; ++t)
          if (t * 16 < there) acc[t][e] = mma_bf16_16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, w[t]), acc[t][e]);
      }
    }
  };

  constexpr int kStride = kWaves * kKeys;
  for (int key = begin + wave * kKeys; key < end; key += kStride) {
    int page[kGroups];
#pragma unroll
    for (int u = 0; u < kGroups; ++u) page[u] = page_at(key, u);
    Step s;
    load(s, key, page);
    compute(s, key);
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
    const long long tok = row0 + row / (unsigned)a.group;
    const int h = hk * a.group + (int)(row % (unsigned)a.group);
    if (a.parts > 1) {
      const long long at = ((long long)(a.first_part + split) * a.T + tok) * a.heads + h;
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

// Joins the parts of a row: a wave a row, its lanes first the parts' statistics, then the channels.
template <typename ET>
__global__ __launch_bounds__(256) void k_join(CachedArgs a, int own, int shared) {
  const int lane = lane_id();
  const unsigned row = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const long long rows = (long long)a.T * a.heads;
  if (row >= rows) return;
  const int token = (int)(row / (unsigned)a.heads), head = (int)(row - (unsigned)token * a.heads);
  const int b = last_not_above(a.B, [&](int i) { return row_at(a.offsets, i, a.T) <= token; });
  if (token < row_at(a.offsets, b, a.T) || token >= row_at(a.offsets, b + 1, a.T)) return;
  const int len = cached_tokens(a, b), each = part_keys(len, own), used = max((len + each - 1) / each, 1);
  // part i of the workspace: of the sequence's own, then of the prefix
  const bool in = lane < own + shared && (lane < used || lane >= own);
  float top = kNoScore, sum = 0.f;
  if (in) {
    const long long at = (long long)lane * rows + row;
    top = a.part_stat[2 * at];
    sum = a.part_stat[2 * at + 1];
  }
  float most = top;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) most = fmaxf(most, __shfl_xor(most, o, kWave));
  const float by = exp2_fast(top - shift_of(most));
  const float total = lanes64_sum(in ? sum * by : 0.f);
  const unsigned long long counts = __ballot(in && top != kNoScore);  // (the others' sums were not written, or are zero)
  float f[2] = {0.f, 0.f};
  const int d = lane * 2;
  for (int i = 0; i < own + shared; ++i) {
    if (!((counts >> i) & 1)) continue;
    const float w = __shfl(by, i, kWave);
    if (d < a.D) {
      const float2 v = *reinterpret_cast<const float2*>(a.part_out + ((long long)i * rows + row) * a.D + d);
      f[0] = fmaf(v.x, w, f[0]);
      f[1] = fmaf(v.y, w, f[1]);
    }
  }
  if (d >= a.D) return;
  const float inv = 1.f / total;
  const float x = total == 0.f ? 0.f : f[0] * inv, y = total == 0.f ? 0.f : f[1] * inv;
  ET* const out = reinterpret_cast<ET*>(a.out) + token * a.ldo + head * a.D + d;
  if constexpr (sizeof(ET) == 4) *reinterpret_cast<float2*>(out) = make_float2(x, y);
  else *reinterpret_cast<unsigned*>(out) = pack_bf16(x, y);
}

// ---- plan -------------------------------------------------------------------------------------------------------------------
struct Plan {
  int rt, prefix_rt;        // row tiles of a workgroup
  int own, shared;          // parts of the sequences' own keys, and of the prefix
  long long tiles, prefix_tiles;
  size_t stat_at, bytes;    // workspace: sums, then statistics
};
inline int row_tiles(double rows, bool wide) { return rows <= 16 ? 1 : rows <= 32 || wide ? 2 : 4; }

// Parts: as many workgroups as keep the card's 256 compute units busy for a few rounds, none of fewer than 256 keys.
inline int parts_for(double groups, long long keys, int most) {
  const double want = 1024.0 / groups;
  const long long room = (keys + 255) / 256;
  return (int)max(1ll, min(min((long long)(want + 0.999), room), (long long)most));
}

Plan plan_of(const laud_heads* p, const laud_cache* c, const laud_batch* b, int T) {
  Plan s{};
  const int group = p->heads / p->kv_heads;
  const bool wide = c->dtype == LAUD_F32;
  const double rows = (double)T * group;
  s.rt = row_tiles(rows / b->B, wide);
  s.tiles = tiles_of(T, b->B, group, 16 * s.rt);
  const double busy = max((double)b->B, rows / (16 * s.rt)) * p->kv_heads;
  const bool prefix = b->prefix_len > 0;
  s.own = parts_for(busy, (long long)b->table_ld * c->page, prefix ? kMaxParts / 2 : kMaxParts);
  if (prefix) {
    s.prefix_rt = row_tiles(rows, wide);
    s.prefix_tiles = ((long long)T * group - 1) / (16 * s.prefix_rt) + 1;
    s.shared = parts_for((double)s.prefix_tiles * p->kv_heads, b->prefix_len, kMaxParts / 2);
  }
  if (s.own + s.shared > 1) {
    const size_t all = (size_t)(s.own + s.shared) * T * p->heads;
    s.stat_at = align_up(all * p->D * 4, 256);
    s.bytes = s.stat_at + all * 8;
  }
  return s;
}

template <typename ET, typename CT, int DP, int RT>
int launch_cached(const CachedArgs& a, hipStream_t st) {
  constexpr int kLds = kWaves * 16 * (DP + 4) * 4 + kWaves * 16 * RT * 8;
  const double groups = (double)a.tiles * a.kv_heads * a.splits;
  if (!launchable(groups, kWaves * kWave)) return LAUD_ERR_UNSUPPORTED;
  hipLaunchKernelGGL((k_cached<ET, CT, DP, RT>), dim3((unsigned)groups), dim3(kWaves * kWave), kLds, st, a);
  return LAUD_OK;
}
template <typename ET, typename CT, int DP>
int launch_rows(const CachedArgs& a, int rt, hipStream_t st) {
  if (rt == 1) return launch_cached<ET, CT, DP, 1>(a, st);
  if (rt == 2) return launch_cached<ET, CT, DP, 2>(a, st);
  if constexpr (sizeof(CT) < 4) return launch_cached<ET, CT, DP, 4>(a, st);
  return LAUD_ERR_UNSUPPORTED;
}
int launch_types(const CachedArgs& a, int cache_type, int rt, hipStream_t st) {
  if (cache_type == LAUD_F32) return a.D <= 64 ? launch_rows<float, float, 64>(a, rt, st) : launch_rows<float, float, 128>(a, rt, st);
  if (cache_type == LAUD_BF16) return a.D <= 64 ? launch_rows<bf16_t, bf16_t, 64>(a, rt, st) : launch_rows<bf16_t, bf16_t, 128>(a, rt, st);
  return a.D <= 64 ? launch_rows<bf16_t, uint8_t, 64>(a, rt, st) : launch_rows<bf16_t, uint8_t, 128>(a, rt, st);
}

// The arguments that the host sees, all but the rows and the workspace.
int check_cached(const laud_heads* p, const laud_cache* c, const laud_batch* b, int T) {
  int bad = check_heads(p);
  if (!bad) bad = check_cache(c, b);
  if (bad) return bad;
  if (T < 0 || p->kv_heads != c->kv_heads || p->D != c->D || b->prefix_len < 0 || (b->prefix_len > 0 && (!b->prefix || !aligned4(b->prefix))) ||
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
  const double most = 2147483648.0;
  if (s.tiles >= most || !launchable((double)s.tiles * p->kv_heads * s.own, kWaves * kWave) ||
      !launchable((double)s.prefix_tiles * p->kv_heads * s.shared, kWaves * kWave) || !launchable(((double)T * p->heads + 3) / 4, 256))
    return LAUD_ERR_UNSUPPORTED;
  CachedArgs a{};
  a.heads = p->heads; a.group = p->heads / p->kv_heads; a.kv_heads = p->kv_heads; a.D = p->D; a.causal = p->causal; a.B = b->B; a.T = T;
  a.pages = c->pages; a.page_bits = page_bits(c); a.table_ld = b->table_ld;
  a.parts = s.own + s.shared;
  a.c = p->scale * kLog2e;
  a.offsets = b->offsets; a.lens = b->lens;
  a.k = (const uint8_t*)c->k; a.v = (const uint8_t*)c->v; a.ks = c->k_scale; a.vs = c->v_scale;
  a.q = q; a.out = out; a.ldq = ldq; a.ldo = ldo;
  a.part_out = (float*)ws;
  a.part_stat = s.bytes ? (float*)((char*)ws + s.stat_at) : nullptr;
  clear_stale_error();
  hipStream_t st = (hipStream_t)stream;
  CachedArgs o = a;
  o.tiles = (int)s.tiles; o.splits = s.own; o.table = b->table;
  o.by_xcd = s.rt > 1 && (long long)p->kv_heads * s.own % 8 == 0;
  int status = launch_types(o, c->dtype, s.rt, st);
  if (status) return status;
  if (s.shared) {
    o = a;
    o.tiles = (int)s.prefix_tiles; o.splits = s.shared; o.first_part = s.own; o.table = b->prefix; o.prefix_len = b->prefix_len; o.shared = 1;
    o.by_xcd = (long long)p->kv_heads * s.shared % 8 == 0;
    status = launch_types(o, c->dtype, s.prefix_rt, st);
    if (status) return status;
  }
  if (a.parts > 1) {
    const dim3 grid((unsigned)(((long long)T * p->heads + 3) / 4));
    if (p->dtype == LAUD_BF16) hipLaunchKernelGGL((k_join<bf16_t>), grid, dim3(256), 0, st, a, s.own, s.shared);
    else hipLaunchKernelGGL((k_join<float>), grid, dim3(256), 0, st, a, s.own, s.shared);
  }
  return check_launch();
}
