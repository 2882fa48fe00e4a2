// Attention over the tokens of packed sequences: one pass over keys and values with the running maximum and sum of each query's softmax.
#include "laud_heads.h"

namespace laud {
namespace {

struct AttendArgs {
  int heads, group, D, causal, B, T, tiles;  // group: query heads of a key head; tiles: of queries, over all sequences (tiles_of)
  float c;                                   // scale * log2(e)
  const int32_t* offsets;
  const void *q, *k, *v;
  const uint8_t* keep;
  void* out;
  int64_t ldq, ldk, ldv, ldo;  // elements
};

// A workgroup has a tile of 32 queries a wave of one head and goes over their keys, KN at a time.  Keys and values come by LDS-direct
// loads into two stages that take turns: one barrier a step, the next step's loads under way while this one is multiplied.  A wave
// multiplies keys * queries (32 x 32: a lane has 16 keys of its query, the other half wave the other 16), so that a query's maximum and
// sum are a lane's own business but for one swap, and the weights lie as the second product, values^T * weights, takes them: its order
// of keys within 16 is the first product's (lane half h: 4 h .. 4 h + 3 and those 8 behind), and the values are read to match -
// transposed on their way from LDS where they are bf16.
template <typename ET, int DP>
struct Tile {
  static constexpr bool kHalf = sizeof(ET) == 2;
  static constexpr int kKeys = kHalf ? 64 : 32;     // KN
  static constexpr int kRow = DP * (int)sizeof(ET);  // bytes of a row in LDS
  static constexpr int kChunks = kRow / 16;
  static constexpr int kPart = kKeys * kRow;  // keys, or values, of a stage
  static constexpr int kStage = 2 * kPart, kBytes = 2 * kStage;
  // A row's 16-byte chunk c lies at position c ^ swizzle: sixteen lanes that read a chunk of sixteen rows, or a transposed read's four
  // rows of four chunks, meet all banks.
  static __device__ __forceinline__ int key_swizzle(int row) { return kChunks == 8 ? (row >> 1) & 7 : row & 15; }
  static __device__ __forceinline__ int value_swizzle(int row) {
    return !kHalf ? 0 : kChunks == 8 ? ((row >> 1) & 1) << 2 : (row & 3) << 2;
  }
};

typedef short tok_s4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ tok_u2 read_transposed(const unsigned char* at) {
  return __builtin_bit_cast(tok_u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) tok_s4*)at));
}
__device__ __forceinline__ f32x16 mma32(const tok_u4& a, const tok_u4& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma32(float a, float b, const f32x16& c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }

template <typename ET, int DP, int NW>
__global__ __launch_bounds__(NW * kWave, 2) void k_attend(AttendArgs a) {
  typedef Tile<ET, DP> L;
  constexpr bool kHalf = L::kHalf;
  constexpr int kKeys = L::kKeys, kBlocks = kKeys / 32, kRows = NW * 32, kDt = DP / 32;
  constexpr int kLoads = L::kPart / 1024 / NW, kLanesRow = L::kChunks;  // LDS-direct loads a wave of keys; lanes that bring a row
  static_assert(kLoads * NW * 1024 == L::kPart, "loads shared evenly");
  extern __shared__ __align__(16) unsigned char lds[];
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), r32 = lane % 32, half = lane / 32;

  // Workgroups go round-robin over the eight XCDs: each takes a run of heads, whose keys its L2 then serves, the tiles of several heads
  // side by side; the last tiles, which see the most keys, first.
  const long long total = (long long)a.heads * a.tiles, per = (total + 7) / 8;
  const long long id = (long long)(blockIdx.x % 8) * per + blockIdx.x / 8;
  if (blockIdx.x / 8 >= per || id >= total) return;
  const int band = a.heads % 8 == 0 ? a.heads / 8 : 1;
  const long long in_band = id % ((long long)band * a.tiles);
  const int head = (int)(id / ((long long)band * a.tiles)) * band + (int)(in_band % band);
  const long long tile = a.tiles - 1 - in_band / band;
  const int b = last_not_above(a.B, [&](int i) { return first_tile(a.offsets, i, a.T, 1, kRows) <= tile; });
  const int row0 = row_at(a.offsets, b, a.T), n = row_at(a.offsets, b + 1, a.T) - row0;  // (n may be negative: no rows)
  const long long q_first = (tile - first_tile(a.offsets, b, a.T, 1, kRows)) * kRows;
  if (q_first < 0 || q_first >= n) return;
  const int q0 = (int)q_first, qw = q0 + wave * 32, qr = qw + r32;  // the tile's first row in its sequence, the wave's, the lane's
  const int end = a.causal ? min(n, q0 + kRows) : n, steps = (end + kKeys - 1) / kKeys;

  // the wave's queries, for good: lane = query, sixteen-byte pieces 2 s + half
  constexpr int kPieces = L::kChunks / 2, kPer = 16 / (int)sizeof(ET);
  tok_u4 qf[kPieces];
  {
    const __amdgpu_buffer_rsrc_t rq = bytes_of(reinterpret_cast<const ET*>(a.q) + (row0 + (long long)q0) * a.ldq + head * a.D,
                                               ((long long)(min(kRows, n - q0) - 1) * a.ldq + a.D) * (long long)sizeof(ET));
#pragma unroll
    for (int s = 0; s < kPieces; ++s) {
      const int d = (2 * s + half) * kPer;
      qf[s] = load16(rq, qr < n && d < a.D ? (unsigned)((qr - q0) * a.ldq + d) * (unsigned)sizeof(ET) : kOutside);
    }
  }
  const ET* const kp = reinterpret_cast<const ET*>(a.k) + (long long)row0 * a.ldk + head / a.group * a.D;
  const ET* const vp = reinterpret_cast<const ET*>(a.v) + (long long)row0 * a.ldv + head / a.group * a.D;
  const uint8_t* const keep = a.keep ? a.keep + row0 : nullptr;

  // which of a step's keys are there: rows of the sequence that the masker kept
  auto kept_byte = [&](int step) -> unsigned {
    const long long r = (long long)step * kKeys + lane;
    return lane < kKeys && r < n ? (keep ? (unsigned)keep[r] : 1u) : 0u;
  };
  // LDS-direct loads of a step: rows that are not there come as zeros (their weights are 0, and so are not 0 * NaN)
  unsigned vk[kLoads], vv[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int at = (wave * kLoads + i) * kWave + lane, row = at / kLanesRow, pos = at % kLanesRow;
    const int ck = (pos ^ L::key_swizzle(row)) * kPer, cv = (pos ^ L::value_swizzle(row)) * kPer;
    vk[i] = ck < a.D ? (unsigned)(row * a.ldk + ck) * (unsigned)sizeof(ET) : kOutside;
    vv[i] = cv < a.D ? (unsigned)(row * a.ldv + cv) * (unsigned)sizeof(ET) : kOutside;
  }
  auto request = [&](int step, unsigned long long there) {
    const unsigned stage = (step & 1) * L::kStage;
    const __amdgpu_buffer_rsrc_t rk = bytes_of(kp + (long long)step * kKeys * a.ldk, 0x7fffffff);
    const __amdgpu_buffer_rsrc_t rv = bytes_of(vp + (long long)step * kKeys * a.ldv, 0x7fffffff);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int row = ((wave * kLoads + i) * kWave + lane) / kLanesRow;
      const bool in = (there >> row) & 1;
      dma16(rk, in ? vk[i] : kOutside, 0, stage + (wave * kLoads + i) * 1024);
      dma16(rv, in ? vv[i] : kOutside, 0, stage + L::kPart + (wave * kLoads + i) * 1024);
    }
  };

  f32x16 acc[kDt];
#pragma unroll
  for (int t = 0; t < kDt; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[t][e] = 0.f;
  float top = kNoScore, sum = 0.f;
  const bool asks = qr < n && (!keep || keep[min(qr, n - 1)] != 0);

  unsigned long long there = __ballot(kept_byte(0) != 0);
  request(0, there);
  unsigned kept_next = steps > 1 ? kept_byte(1) : 0;
  for (int step = 0; step < steps; ++step) {
    vm_wait<0>();
    __syncthreads();  // the step's rows are there, and nobody reads the other stage any more
    const unsigned long long there_next = __ballot(kept_next != 0);
    if (step + 1 < steps) request(step + 1, there_next);
    if (step + 2 < steps) kept_next = kept_byte(step + 2);
    const int k0 = step * kKeys;
    const unsigned long long here = there;
    there = there_next;
    if (a.causal && k0 > qw + 31) continue;  // (the wave's queries see none of them)
    const unsigned char *ks = lds + (step & 1) * L::kStage, *vs = ks + L::kPart;

    // scores: key 32 u + 8 * (e / 4) + 4 * half + e % 4 with the lane's query
    f32x16 s[kBlocks];
#pragma unroll
    for (int u = 0; u < kBlocks; ++u) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[u][e] = 0.f;
      const unsigned char* const row = ks + (u * 32 + r32) * L::kRow;
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
        const tok_u4 kf = *reinterpret_cast<const tok_u4*>(row + (((2 * i + half) ^ L::key_swizzle(r32)) << 4));
        if constexpr (kHalf) {
          s[u] = mma32(kf, qf[i], s[u]);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) s[u] = mma32(__uint_as_float(kf[j]), __uint_as_float(qf[i][j]), s[u]);
        }
      }
    }
    const bool diagonal = a.causal && k0 + kKeys - 1 > qw;
    const unsigned long long all = kKeys == 64 ? ~0ull : 0xffffffffull;
    const bool masked = diagonal || here != all || keep;
    unsigned long long seen = all;
    if (masked) {
      seen = asks ? here : 0;
      if (a.causal) {
        const int last = qr - k0;  // the last key that the query sees
        seen &= last < 0 ? 0 : last >= 63 ? ~0ull : (2ull << last) - 1;
      }
      seen >>= 4 * half;
#pragma unroll
      for (int u = 0; u < kBlocks; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (!((seen >> (32 * u + 8 * (e / 4) + e % 4)) & 1)) s[u][e] = kNoScore;
    }
    float most = s[0][0];
#pragma unroll
    for (int u = 0; u < kBlocks; ++u)
#pragma unroll
      for (int e = 0; e < 16; ++e) most = fmaxf(most, s[u][e]);
    most = fmaxf(top, other_half_max(most) * a.c);
    const float shift = shift_of(most);
    if (__ballot(most > top)) {
      const float shrink = exp2_fast(top - shift);
      sum *= shrink;
#pragma unroll
      for (int t = 0; t < kDt; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[t][e] *= shrink;
      top = most;
    }
#pragma unroll
    for (int u = 0; u < kBlocks; ++u)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[u][e] = exp2_fast(fmaf(s[u][e], a.c, -shift));
        sum += s[u][e];
      }

    // out^T += values^T * weights
    bool clean = true;
    if (diagonal) {  // values that some of the queries do not see: numbers?
      bool bad = false;
      for (int i = lane; i < L::kPart / 16; i += kWave) {
        const tok_u4 v = reinterpret_cast<const tok_u4*>(vs)[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) bad |= kHalf ? not_finite2(v[j]) : not_finite(__uint_as_float(v[j]));
      }
      clean = __ballot(bad) == 0;
    }
    if constexpr (kHalf) {
      tok_u4 w[kBlocks * 2];
#pragma unroll
      for (int t = 0; t < kBlocks * 2; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) w[t][j] = pack_bf16(s[t / 2][8 * (t % 2) + 2 * j], s[t / 2][8 * (t % 2) + 2 * j + 1]);
      const int i16 = lane % 16, low = (lane / 16) % 2 * 2 + i16 % 4 / 2;
      const unsigned char* const from = vs + (4 * half + i16 / 4) * L::kRow + i16 % 2 * 8;
      auto values = [&](int t, int dt) {
        const unsigned char* const at = from + 16 * t * L::kRow + (((4 * dt + low) ^ L::value_swizzle(i16 / 4)) << 4);
        const tok_u2 lo = read_transposed(at), hi = read_transposed(at + 8 * L::kRow);
        return tok_u4{lo[0], lo[1], hi[0], hi[1]};
      };
      if (clean) {
#pragma unroll
        for (int t = 0; t < kBlocks * 2; ++t)
#pragma unroll
          for (int dt = 0; dt < kDt; ++dt) acc[dt] = mma32(values(t, dt), w[t], acc[dt]);
      } else {
#pragma unroll
        for (int t = 0; t < kBlocks * 2; ++t)
#pragma unroll
          for (int dt = 0; dt < kDt; ++dt) {
            tok_u4 v = values(t, dt);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = finite2(v[j]);
            acc[dt] = mma32(v, w[t], acc[dt]);
          }
#pragma unroll 1
        for (int i = 0; i < 2 * kDt; ++i) {  // infinities of either sign
          f32x16 found;
#pragma unroll
          for (int e = 0; e < 16; ++e) found[e] = 0.f;
#pragma unroll 1
          for (int t = 0; t < kBlocks * 2; ++t) {
            tok_u4 v = values(t, i / 2), sees;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              v[j] = endless2(v[j], i % 2);
              const int key = 16 * t + 8 * (j / 2) + j % 2 * 2;  // (of seen, which is shifted by the lane's half)
              sees[j] = ((seen >> key) & 1 ? 0x3f80u : 0u) | ((seen >> key) & 2 ? 0x3f800000u : 0u);
            }
            found = mma32(v, sees, found);
          }
#pragma unroll
          for (int t = 0; t < kDt; ++t)
            if (t == i / 2) add_endless(acc[t], found, i % 2);
        }
      }
    } else {
      const float* const from = reinterpret_cast<const float*>(vs) + 4 * half * DP + r32;
      auto value = [&](int e, int dt) { return from[(8 * (e / 4) + e % 4) * DP + 32 * dt]; };
      if (clean) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
#pragma unroll
          for (int dt = 0; dt < kDt; ++dt) acc[dt] = mma32(value(e, dt), s[0][e], acc[dt]);
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e)
#pragma unroll
          for (int dt = 0; dt < kDt; ++dt) {
            const float v = value(e, dt);
            acc[dt] = mma32(not_finite(v) ? 0.f : v, s[0][e], acc[dt]);
          }
#pragma unroll 1
        for (int i = 0; i < 2 * kDt; ++i) {  // infinities of either sign
          f32x16 found;
#pragma unroll
          for (int e = 0; e < 16; ++e) found[e] = 0.f;
#pragma unroll 1
          for (int e = 0; e < 16; ++e)
            found = mma32(endless(value(e, i / 2), i % 2), (seen >> (8 * (e / 4) + e % 4)) & 1 ? 1.f : 0.f, found);
#pragma unroll
          for (int t = 0; t < kDt; ++t)
            if (t == i / 2) add_endless(acc[t], found, i % 2);
        }
      }
    }
  }

  // out: the lane's query, channels 32 t + 16 * half .. + 15
  sum = other_half_sum(sum);
  const bool none = sum == 0.f;
  const float inv = 1.f / sum;
  ET* const out = reinterpret_cast<ET*>(a.out) + (row0 + (long long)qr) * a.ldo + head * a.D;
#pragma unroll
  for (int t = 0; t < kDt; ++t) {
    float v[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = none ? 0.f : acc[t][e] * inv;
    to_consecutive_channels(v);
    // (the swaps leave channels 0-3, 8-11 of a half in v[0..7] and 4-7, 12-15 in v[8..15])
    float f[2][8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f[0][e] = v[e];
      f[0][4 + e] = v[8 + e];
      f[1][e] = v[4 + e];
      f[1][4 + e] = v[12 + e];
    }
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int d = 32 * t + 16 * half + 8 * g;
      if (qr < n && d < a.D) {
        piece8<ET> p;
        p.put(f[g]);
        p.store(out, d / 8);
      }
    }
  }
}

template <typename ET, int DP>
int launch_attend(AttendArgs a, hipStream_t st) {
  constexpr int kWaves = 4, kRows = kWaves * 32;
  const long long tiles = tiles_of(a.T, a.B, 1, kRows), groups = (tiles * a.heads + 7) / 8 * 8;
  if (!launchable((double)groups, kWaves * kWave)) return LAUD_ERR_UNSUPPORTED;
  a.tiles = (int)tiles;
  hipLaunchKernelGGL((k_attend<ET, DP, kWaves>), dim3((unsigned)groups), dim3(kWaves * kWave), (Tile<ET, DP>::kBytes), st, a);
  return check_launch();
}

}  // namespace
}  // namespace laud

extern "C" int laud_attention(const laud_heads* p, int B, const int32_t* offsets, int T, const void* q, int64_t ldq, const void* k, int64_t ldk,
                              const void* v, int64_t ldv, const uint8_t* keep, void* out, int64_t ldo, void* stream) {
  using namespace laud;
  const int bad = check_heads(p);
  if (bad) return bad;
  if (B < 0 || T < 0) return LAUD_ERR_INVALID_ARG;
  if (B == 0 || T == 0) return LAUD_OK;
  const int C = p->heads * p->D, Ck = p->kv_heads * p->D;
  if (!offsets || !q || !k || !v || !out || !good_ld(ldq, C, 8) || !good_ld(ldk, Ck, 8) || !good_ld(ldv, Ck, 8) || !good_ld(ldo, C, 8) ||
      !aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || (reinterpret_cast<uintptr_t>(offsets) & 3u))
    return LAUD_ERR_INVALID_ARG;
  if (ldq > kMaxRowDistance || ldk > kMaxRowDistance || ldv > kMaxRowDistance || ldo > kMaxRowDistance) return LAUD_ERR_UNSUPPORTED;
  // a tile's queries are read by the workgroup that writes their results, keys and values by others
  const size_t eb = elem_bytes(p->dtype);
  if (!same_or_apart(q, ldq, eb, out, ldo, eb, T, C) || rows_overlap(out, ldo, eb, C, k, ldk, eb, Ck, T) ||
      rows_overlap(out, ldo, eb, C, v, ldv, eb, Ck, T) || range_meets_rows(offsets, 4 * ((size_t)B + 1), out, ldo, eb, T, C) ||
      range_meets_rows(keep, (size_t)T, out, ldo, eb, T, C))
    return LAUD_ERR_INVALID_ARG;
  AttendArgs a{};
  a.heads = p->heads; a.group = p->heads / p->kv_heads; a.D = p->D; a.causal = p->causal; a.B = B; a.T = T;
  a.c = p->scale * kLog2e;
  a.offsets = offsets; a.q = q; a.k = k; a.v = v; a.keep = keep; a.out = out;
  a.ldq = ldq; a.ldk = ldk; a.ldv = ldv; a.ldo = ldo;
  clear_stale_error();
  hipStream_t st = (hipStream_t)stream;
  if (p->dtype == LAUD_BF16) return p->D <= 64 ? launch_attend<bf16_t, 64>(a, st) : launch_attend<bf16_t, 128>(a, st);
  return p->D <= 64 ? launch_attend<float, 64>(a, st) : launch_attend<float, 128>(a, st);
}
