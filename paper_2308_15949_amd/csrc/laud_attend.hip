// Attention over the tokens of packed sequences: one pass over keys and values with the running maximum and sum of each query's softmax.
#include <type_traits>

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

// A workgroup has a tile of NW * 32 queries of one head, 32 a wave, and goes over their keys, KK at a time; KG groups of waves share the
// steps, each with stages of its own, and join their sums at the end.  Keys and values come by LDS-direct loads into two stages that take
// turns: one barrier a step, the next step's loads under way while this one is multiplied.  A wave multiplies keys * queries (32 x 32: a
// lane has 16 keys of its query, the other half wave the other 16), so that a query's maximum and sum are a lane's own business but for
// one swap, and the weights lie as the second product, values^T * weights, takes them: its order of keys within 16 is the first product's
// (lane half h: 4 h .. 4 h + 3 and those 8 behind), and the values are read to match - transposed on their way from LDS where they are
// bf16.
template <typename ET, int DP, int KK>
struct Tile {
  static constexpr bool kHalf = sizeof(ET) == 2;
  static constexpr int kRow = DP * (int)sizeof(ET);  // bytes of a row in LDS
  static constexpr int kChunks = kRow / 16;
  static constexpr int kPart = KK * kRow;  // keys, or values, of a stage
  static constexpr int kStage = 2 * kPart, kGroup = 2 * kStage;
  static constexpr int kSums = DP / 32 * 4 * kWave;  // of a wave's 32 queries, in f32x4
  // LDS of a workgroup: the groups' stages, in whose place all groups' but the first's sums, maxima and sums of weights come
  static constexpr int bytes(int NW, int KG) {
    const int stages = KG * kGroup, sums = (KG - 1) * NW * (kSums * 16 + 2 * kWave * 4);
    return stages > sums ? stages : sums;
  }
  // A row's 16-byte chunk c lies at position c ^ swizzle: sixteen lanes that read a chunk of sixteen rows, or a transposed read's four
  // rows of four chunks, meet all banks (no bank conflict counted).
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

// Sums are relative to a maximum that is let grow by this much (as an exponent of 2) before they are taken anew: the largest weight is
// 2^8 instead of 1, which costs float32 nothing, and most steps are spared the scaling of all sums (64 instructions).
constexpr float kSlack = 8.f;

template <typename ET, int DP, int NW, int KG, int KK>
__global__ __launch_bounds__(NW * KG * kWave, (NW * KG > 4 ? 1 : 2)) void k_attend(AttendArgs a) {
  typedef Tile<ET, DP, KK> L;
  constexpr bool kHalf = L::kHalf;
  constexpr int kBlocks = KK / 32, kRows = NW * 32, kDt = DP / 32, kEb = (int)sizeof(ET);
  constexpr int kLanesRow = L::kChunks, kRowsLoad = kWave / kLanesRow;  // lanes that bring a row, rows of an LDS-direct load
  constexpr int kLoads = L::kPart / 1024 / NW;                          // loads a wave of a step's keys
  static_assert(kLoads * NW * 1024 == L::kPart, "loads shared evenly");
  extern __shared__ __align__(16) unsigned char lds[];
  const int lane = lane_id(), r32 = lane % 32, half = lane / 32;
  const int group = __builtin_amdgcn_readfirstlane(threadIdx.x / (NW * kWave));
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) - group * NW;

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
  const int end = a.causal ? min(n, q0 + kRows) : n, steps = (end + KK - 1) / KK, rounds = (steps + KG - 1) / KG;
  const uint8_t* const keep = a.keep ? a.keep + row0 : nullptr;
  // rounds whose keys are all there, and seen by all queries of the tile
  const int whole_steps = keep ? 0 : (a.causal ? min(n, q0 + 1) : n) / KK, whole = whole_steps / KG;

  // the wave's queries, for good: lane = query, sixteen-byte pieces 2 s + half
  constexpr int kPieces = L::kChunks / 2, kPer = 16 / kEb;
  tok_u4 qf[kPieces];
  {
    const __amdgpu_buffer_rsrc_t rq = bytes_of(reinterpret_cast<const ET*>(a.q) + (row0 + (long long)q0) * a.ldq + head * a.D,
                                               ((long long)(min(kRows, n - q0) - 1) * a.ldq + a.D) * kEb);
#pragma unroll
    for (int s = 0; s < kPieces; ++s) {
      const int d = (2 * s + half) * kPer;
      qf[s] = load16(rq, qr < n && d < a.D ? (unsigned)((qr - q0) * a.ldq + d) * kEb : kOutside);
    }
  }
  const ET* const kp = reinterpret_cast<const ET*>(a.k) + (long long)row0 * a.ldk + head / a.group * a.D;
  const ET* const vp = reinterpret_cast<const ET*>(a.v) + (long long)row0 * a.ldv + head / a.group * a.D;

  // Which of a step's keys are there, a bit each: rows of the sequence that the masker kept (asked for a round ahead).
  auto kept_byte = [&](int step) -> unsigned {
    const long long r = (long long)step * KK + lane;
    return lane < KK && r < n ? (unsigned)keep[r] : 0u;
  };
  auto rows_there = [&](int step) -> unsigned long long {
    const long long rows = n - (long long)step * KK;
    return rows >= 64 ? ~0ull : rows <= 0 ? 0ull : (1ull << rows) - 1;
  };
  // LDS-direct loads of a step: load i brings rows i * NW * kRowsLoad + wave * kRowsLoad .., of which a lane has one chunk, the same of
  // each where the swizzles' periods (16 rows) allow.
  constexpr bool kSame = NW * kRowsLoad % (kHalf ? 16 : 16) == 0;
  constexpr int kOffsets = kSame ? 1 : kLoads;
  unsigned vk[kOffsets], vv[kOffsets];
#pragma unroll
  for (int i = 0; i < kOffsets; ++i) {
    const int row = (i * NW + wave) * kRowsLoad + lane / kLanesRow, pos = lane % kLanesRow;
    const int ck = (pos ^ L::key_swizzle(row)) * kPer, cv = (pos ^ L::value_swizzle(row)) * kPer;
    vk[i] = ck < a.D ? (unsigned)(row * a.ldk + ck) * kEb : kOutside;
    vv[i] = cv < a.D ? (unsigned)(row * a.ldv + cv) * kEb : kOutside;
  }
  const unsigned stage0 = group * L::kGroup;
  auto request = [&](int round, int step, bool all, unsigned long long there) {
    const unsigned stage = stage0 + (round & 1) * L::kStage + wave * 1024;
    const __amdgpu_buffer_rsrc_t rk = bytes_of(kp + (long long)step * KK * a.ldk, 0x7fffffff);
    const __amdgpu_buffer_rsrc_t rv = bytes_of(vp + (long long)step * KK * a.ldv, 0x7fffffff);
    if (all) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const unsigned skip = kSame ? (unsigned)i * NW * kRowsLoad * kEb : 0u;
        dma16(rk, vk[kSame ? 0 : i], skip * (unsigned)a.ldk, stage + i * NW * 1024);
        dma16(rv, vv[kSame ? 0 : i], skip * (unsigned)a.ldv, stage + L::kPart + i * NW * 1024);
      }
    } else {  // rows that are not there come as zeros (their weights are 0, and so are not 0 * NaN)
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int row = (i * NW + wave) * kRowsLoad + lane / kLanesRow;
        const unsigned skip = kSame ? (unsigned)i * NW * kRowsLoad * kEb : 0u, ok = vk[kSame ? 0 : i], ov = vv[kSame ? 0 : i];
        const bool in = (there >> row) & 1;
        dma16(rk, in && ok != kOutside ? ok + skip * (unsigned)a.ldk : kOutside, 0, stage + i * NW * 1024);
        dma16(rv, in && ov != kOutside ? ov + skip * (unsigned)a.ldv : kOutside, 0, stage + L::kPart + i * NW * 1024);
      }
    }
  };

  f32x16 acc[kDt];
#pragma unroll
  for (int t = 0; t < kDt; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[t][e] = 0.f;
  float top = kNoScore, sum = 0.f;

  auto multiply = [&](auto some, int round, int k0, unsigned long long here, bool asks) {
    constexpr bool kSome = decltype(some)::value;  // some keys are not there, or not seen by every query
    const unsigned char *ks = lds + stage0 + (round & 1) * L::kStage, *vs = ks + L::kPart;
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
    unsigned long long seen = 0;
    if constexpr (kSome) {
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
    most = other_half_max(most) * a.c;
    if (__ballot(most > top + kSlack)) {  // (the first score: more than -infinity)
      most = fmaxf(top, most);
      const float shrink = exp2_fast(top - shift_of(most));
      sum *= shrink;
#pragma unroll
      for (int t = 0; t < kDt; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[t][e] *= shrink;
      top = most;
    }
    const float shift = shift_of(top);
#pragma unroll
    for (int u = 0; u < kBlocks; ++u)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[u][e] = exp2_fast(fmaf(s[u][e], a.c, -shift));
        sum += s[u][e];
      }

    // out^T += values^T * weights
    bool clean = true;
    if constexpr (kSome) {  // values that some of the queries do not see: numbers?
      if (a.causal) {
        bool bad = false;
        for (int i = lane; i < L::kPart / 16; i += kWave) {
          const tok_u4 v = reinterpret_cast<const tok_u4*>(vs)[i];
#pragma unroll
          for (int j = 0; j < 4; ++j) bad |= kHalf ? not_finite2(v[j]) : not_finite(__uint_as_float(v[j]));
        }
        clean = __ballot(bad) == 0;
      }
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
#pragma unroll
      for (int t = 0; t < kBlocks * 2; ++t)
#pragma unroll
        for (int dt = 0; dt < kDt; ++dt) {
          tok_u4 v = values(t, dt);
          if (kSome && !clean) {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = finite2(v[j]);
          }
          acc[dt] = mma32(v, w[t], acc[dt]);
        }
      if (kSome && !clean) {
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
#pragma unroll
      for (int e = 0; e < 16; ++e)
#pragma unroll
        for (int dt = 0; dt < kDt; ++dt) {
          float v = value(e, dt);
          if (kSome && !clean) v = not_finite(v) ? 0.f : v;
          acc[dt] = mma32(v, s[0][e], acc[dt]);
        }
      if (kSome && !clean) {
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
  };

  // Rounds of whole steps, then those of which some keys are not there or not seen.
  unsigned kept = 0;
  unsigned long long there = 0;
  auto ask = [&](int round) {  // a round's loads; its step may be past the last one: nothing is fetched
    const int step = round * KG + group;
    there = keep ? __ballot(kept != 0) : rows_there(step);
    request(round, step, !keep && round < whole, there);
    if (keep) kept = kept_byte(step + KG);
  };
  if (keep) kept = kept_byte(group);
  ask(0);
  int round = 0;
  for (; round < whole; ++round) {
    vm_wait<0>();
    __syncthreads();  // the step's rows are there, and nobody reads the other stage any more
    if (round + 1 < rounds) ask(round + 1);
    multiply(std::false_type(), round, 0, 0, true);
  }
  if (round < rounds) {
    const bool asks = qr < n && (!keep || keep[min(qr, n - 1)] != 0);
    for (; round < rounds; ++round) {
      const unsigned long long here = there;
      vm_wait<0>();
      __syncthreads();
      if (round + 1 < rounds) ask(round + 1);
      const int k0 = (round * KG + group) * KK;
      if (k0 >= end || (a.causal && k0 > qw + 31)) continue;  // (no keys, or none that the wave's queries see)
      multiply(std::true_type(), round, k0, here, asks);
    }
  }
  sum = other_half_sum(sum);

  if constexpr (KG > 1) {  // the other groups' sums through LDS to the first, in their order
    constexpr int kSums = L::kSums;
    f32x4* const sums = reinterpret_cast<f32x4*>(lds);
    float* const stats = reinterpret_cast<float*>(lds + (KG - 1) * NW * kSums * 16);
    __syncthreads();
    if (group != 0) {
      const int at = (group - 1) * NW + wave;
#pragma unroll
      for (int t = 0; t < kDt; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          sums[at * kSums + (t * 4 + e) * kWave + lane] = f32x4{acc[t][4 * e], acc[t][4 * e + 1], acc[t][4 * e + 2], acc[t][4 * e + 3]};
      stats[(2 * at) * kWave + lane] = top;
      stats[(2 * at + 1) * kWave + lane] = sum;
    }
    __syncthreads();
    if (group != 0) return;
    float most = top;
#pragma unroll
    for (int g = 0; g < KG - 1; ++g) most = fmaxf(most, stats[2 * (g * NW + wave) * kWave + lane]);
    const float shift = shift_of(most), mine = exp2_fast(top - shift);
    sum *= mine;
#pragma unroll
    for (int t = 0; t < kDt; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[t][e] *= mine;
#pragma unroll
    for (int g = 0; g < KG - 1; ++g) {
      const int at = g * NW + wave;
      const float by = exp2_fast(stats[2 * at * kWave + lane] - shift);
      sum = fmaf(stats[(2 * at + 1) * kWave + lane], by, sum);
#pragma unroll
      for (int t = 0; t < kDt; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const f32x4 v = sums[at * kSums + (t * 4 + e) * kWave + lane];
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[t][4 * e + j] = fmaf(v[j], by, acc[t][4 * e + j]);
        }
    }
  }

  // out: the lane's query, channels 32 t + 16 * half .. + 15
  const bool none = sum == 0.f;
  const float inv = 1.f / sum;
  ET* const out = reinterpret_cast<ET*>(a.out) + (row0 + (long long)qr) * a.ldo + head * a.D;
#pragma unroll
  for (int t = 0; t < kDt; ++t) {
    float v[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = none ? 0.f : acc[t][e] * inv;
    to_consecutive_channels(v);
    // (the swaps leave the first eight in v[0..3] and v[8..11])
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

template <typename ET, int DP, int NW, int KG, int KK>
int ask_tile_lds() {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(&k_attend<ET, DP, NW, KG, KK>), hipFuncAttributeMaxDynamicSharedMemorySize,
                             (Tile<ET, DP, KK>::bytes(NW, KG))) == hipSuccess ? LAUD_OK : LAUD_ERR_HIP;
}
template <typename ET, int DP, int NW, int KG, int KK>
int launch_tiles(AttendArgs a, hipStream_t st) {
  const long long tiles = tiles_of(a.T, a.B, 1, NW * 32), groups = (tiles * a.heads + 7) / 8 * 8;
  if (!launchable((double)groups, NW * KG * kWave)) return LAUD_ERR_UNSUPPORTED;
  a.tiles = (int)tiles;
  if (Tile<ET, DP, KK>::bytes(NW, KG) > 65536 && ask_tile_lds<ET, DP, NW, KG, KK>() != LAUD_OK) return LAUD_ERR_HIP;
  hipLaunchKernelGGL((k_attend<ET, DP, NW, KG, KK>), dim3((unsigned)groups), dim3(NW * KG * kWave), (Tile<ET, DP, KK>::bytes(NW, KG)), st, a);
  return check_launch();
}

template <typename ET, int DP>
int launch_attend(const AttendArgs& a, hipStream_t st) {
  constexpr bool kHalf = sizeof(ET) == 2;
#ifdef LAUD_VARIANT
  constexpr int v = LAUD_VARIANT;
#else
  const int v = 0;
#endif
  if constexpr (kHalf) {
    if (v == 1) return launch_tiles<ET, DP, 4, 2, 32>(a, st);
    if (v == 2) return launch_tiles<ET, DP, 2, 2, 32>(a, st);
    return launch_tiles<ET, DP, 4, 1, 64>(a, st);
  } else {
    return launch_tiles<ET, DP, 4, 1, 32>(a, st);
  }
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
