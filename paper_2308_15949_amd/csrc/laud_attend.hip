// Attention over the tokens of packed sequences, and of many new tokens over a cache: one pass over keys and values with the running
// maximum and sum of each query's softmax.
#include <atomic>

#include "laud_cached.h"

namespace laud {

struct AttendArgs {
  int heads, group, D, causal, B, T, tiles;  // group: query heads of a key head; tiles: of queries, over all sequences (tiles_of)
  float c;                                   // scale * log2(e)
  const int32_t* offsets;
  const void *q, *k, *v;
  const uint8_t* keep;
  void* out;
  int64_t ldq, ldk, ldv, ldo;  // elements
};

// A workgroup has a tile of 128 queries of one head, 32 a wave, and goes over their keys, a step of KK at a time.  Keys and values come by
// LDS-direct loads into two stages that take turns: one barrier a step, the next step's loads under way while this one is multiplied.  A
// wave multiplies keys * queries (32 x 32: a lane has 16 keys of its query, the other half wave the other 16), so that a query's maximum
// and sum are a lane's own business but for one swap, and the weights lie as the second product, values^T * weights, takes them: its order
// of keys within 16 is the first product's (lane half h: 4 h .. 4 h + 3 and those 8 behind), and the values are read to match - transposed
// on their way from LDS where they are bf16.
//
// Bound by the matrix cores: 16384 causal tokens, 16 heads of 128 in bf16, take 990 to 1050 us on five machines, 1.05 to 1.1 PFLOP/s of the
// products that the mask leaves (a library product of 8192^3: 1.20); their cores are busy for 55 % of the clocks, of which the load leaves
// 1.8 to 1.9 GHz.
// Short prompts (12 of up to 2000 tokens, 145 to 152 us, 0.65 PFLOP/s) pay 5 us a workgroup for its start, queries and results, 2 for the next one.
// Float32 rows of more than 96 channels under a mask keep 6 registers a lane in memory; the other instances none.
// A weight is rounded to bf16 where it meets bf16 values: in two parts, as k_cached has it, it would be off by 2^-15 instead of 2^-8 and the result by its
// own rounding (16384 tokens: 1.5e-3 of its size from 64 bits instead of 2.0e-3), but the third product of every two takes 1025 -> 1382 us,
// 12 prompts 147 -> 182, 3 x 577 masked tokens 18.4 -> 20.0.
// Tiles: 256 queries by eight waves 1023 and 180 us, 64 queries 1210 and 196, two groups
// of waves that share the keys 1203 and 210, all at a time when this tile had 1040 and 161.
constexpr int kAttendWaves = 4, kAttendRows = kAttendWaves * 32;
static_assert(kAttendRows == kManyRows, "the rows that a cache's tiles are counted in");
// Where keys come from: the call's rows; those of them that the masker kept, by a list (3 x 577 tokens, 12 heads of 80, 0.66 kept: 24.4 us with
// the skipped ones' weights set to 0, 16.8 without them); a cache.
enum { kRowsAll, kRowsKept, kRowsCached };
// The list: rows of kept tokens in order, as a ring.  It is filled kScan rows at a time, whenever it ends less than four steps ahead.
constexpr int kListed = 2048, kScan = 1024;
template <typename ET, int DC>
struct AttendTile {
  static constexpr int KK = sizeof(ET) == 2 ? 64 : 32;  // keys of a step
  static constexpr int DP = DC <= 64 ? 64 : 128;  // channels of a row in LDS; the first DC of them are multiplied
  static constexpr bool kHalf = sizeof(ET) == 2;
  static constexpr int kRow = DP * (int)sizeof(ET);  // bytes of a row in LDS
  static constexpr int kChunks = kRow / 16;
  static constexpr int kPart = KK * kRow;  // keys, or values, of a stage
  // LDS of a workgroup: two stages of keys, two of values, a flag for each of two steps; of kept rows their list and the tile's queries
  static constexpr int kValues = 2 * kPart, kFlags = 4 * kPart, kList = kFlags + 2 * 4, kQueries = kList + kListed * 4;
  static constexpr int bytes(int FROM) { return FROM == kRowsKept ? kQueries + kAttendRows * 4 : kList; }
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

template <typename ET, int DC, int FROM>
__global__ __launch_bounds__(kAttendWaves * kWave, 2) void k_attend(AttendArgs a, CachedArgs cache) {
  typedef AttendTile<ET, DC> L;
  constexpr int DP = L::DP, KK = L::KK, NW = kAttendWaves;
  constexpr bool kHalf = L::kHalf, KEPT = FROM == kRowsKept, PAGED = FROM == kRowsCached;
  constexpr int kBlocks = KK / 32, kRows = kAttendRows, kDt = DC / 32, kEb = (int)sizeof(ET);
  constexpr int kLanesRow = L::kChunks, kRowsLoad = kWave / kLanesRow;  // lanes that bring a row, rows of an LDS-direct load
  constexpr int kLoads = L::kPart / 1024 / NW;                          // loads a wave of a step's keys
  static_assert(kLoads * NW * 1024 == L::kPart, "loads shared evenly");
  extern __shared__ __align__(16) unsigned char lds[];
  const int lane = lane_id(), r32 = lane % 32, half = lane / 32;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);

  // Rows first .. first + kScan - 1 of n, of which the masker kept some: put(number, row) for each, numbers from `number` on; the number
  // after them.  Every wave looks at all of them, and puts every fourth sixty-four.
  auto scan = [&](const uint8_t* keep, int n, int first, int number, auto&& put) {
    bool here[kScan / kWave];
#pragma unroll
    for (int j = 0; j < kScan / kWave; ++j) {
      const int row = first + j * kWave + lane;
      here[j] = row < n && keep[min(row, n - 1)] != 0;
    }
#pragma unroll
    for (int j = 0; j < kScan / kWave; ++j) {
      const unsigned long long m = __ballot(here[j]);
      if (here[j] && j % NW == wave) put(number + __popcll(m & ((1ull << lane) - 1)), first + j * kWave + lane);
      number += __popcll(m);
    }
    return number;
  };

  // The tile's queries and their keys.  Keys are counted from the first that this workgroup looks at: there are `end` of them, a query sees
  // those below its limit, every query of the tile those below all_see.
  int head, hk, n, end, all_see, limit = 0;
  long long my_row;  // the lane's query among all rows
  bool in;
  const uint8_t* keep = nullptr;  // of the sequence's rows
  int first_row = 0, first_query = 0, rows_of_sequence = 0, listed = 0, scanned = 0;  // kept rows in the list, rows that were looked at for them
  int* const list = reinterpret_cast<int*>(lds + L::kList);
  unsigned long long skipped = 0;  // lanes whose row of the output the masker skipped, two a row
  auto put_zeros = [&](long long row, int head) {
    if (!(skipped >> lane & 1)) return;
    piece8<ET> zero;
    const float f[8] = {};
    zero.put(f);
    for (int d = lane % 2; d < a.D / 8; d += 2) zero.store(reinterpret_cast<ET*>(a.out) + row * a.ldo + head * a.D, d);
  };
  const ET *kp = nullptr, *vp = nullptr;
  CachedTile part;
  if constexpr (PAGED) {
    if (!cached_tile<kRows>(part, cache)) return;
    const unsigned row = part.first_row + wave * 32 + r32, token = token_of(cache, row);
    in = row < part.rows;
    hk = part.hk;
    head = hk * cache.group + (int)(row - token * cache.group);
    my_row = (long long)part.row0 + token;
    n = end = max(part.end - part.begin, 0);
    all_see = min(max(part.all_see - part.begin, 0), end);
    if (in) limit = min(max(part.limit_of(cache, row) - part.begin, 0), end);
  } else {
    // Workgroups go round-robin over the eight XCDs: each takes a run of heads, whose keys its L2 then serves, the tiles of several heads
    // side by side; the last tiles, which see the most keys, first.
    const unsigned total = (unsigned)a.heads * (unsigned)a.tiles, per = (total + 7) / 8;  // (a launch has less than 2^32 threads)
    const unsigned id = blockIdx.x % 8 * per + blockIdx.x / 8;
    if (blockIdx.x / 8 >= per || id >= total) return;
    const unsigned band = a.heads % 8 == 0 ? a.heads / 8 : 1, in_band = id % (band * a.tiles);
    head = (int)(id / (band * a.tiles) * band + in_band % band);
    hk = head / a.group;
    const int tile = a.tiles - 1 - (int)(in_band / band);
    const Sequence s = sequence_at(a.offsets, nullptr, a.B, a.T, [&](int row, int i) { return first_tile(row, i, 1, kRows) <= tile; });
    const int row0 = s.row0;
    n = rows_of_sequence = s.next - row0;  // (may be negative: no rows)
    const long long q_first = (tile - first_tile(row0, s.b, 1, kRows)) * kRows;
    if (q_first < 0 || q_first >= n) return;
    const int q0 = __builtin_amdgcn_readfirstlane((int)q_first), qr = q0 + wave * 32 + r32;
    kp = reinterpret_cast<const ET*>(a.k) + (long long)row0 * a.ldk + hk * a.D;
    vp = reinterpret_cast<const ET*>(a.v) + (long long)row0 * a.ldv + hk * a.D;
    my_row = row0 + (long long)qr;
    if constexpr (KEPT) {
      // Kept tokens are numbered in order, and the tile has the queries of numbers q0 .. q0 + 127: what the masker skipped is neither
      // fetched nor multiplied.  Of the skipped rows, those of numbers q0 .. q0 + 127 among all get their zeros here.
      keep = a.keep + row0;
      const int here = q0 + threadIdx.x / 2;
      const bool skip = here < n && keep[min(here, n - 1)] == 0;
      int* const queries = reinterpret_cast<int*>(lds + L::kQueries);
      int kept = 0;
      bool open = true;
      for (int first = 0; first < n && !(a.causal && kept >= q0 + kRows); first += kScan) {
        open = open && kept <= kListed - kScan;
        kept = scan(keep, n, first, kept, [&](int number, int row) {
          if (open) list[number % kListed] = row;
          if ((unsigned)(number - q0) < (unsigned)kRows) queries[number - q0] = row;
        });
        if (open) {
          listed = kept;
          scanned = first + kScan;
        }
      }
      n = kept;
      skipped = __ballot(skip);
      if (q0 >= n) {
        put_zeros(row0 + (long long)here, head);
        return;
      }
      first_row = row0;
      first_query = q0;
      __syncthreads();
      in = qr < n;
      if (in) my_row = row0 + (long long)queries[qr - q0];
    } else {
      in = qr < n;
    }
    end = a.causal ? min(n, q0 + kRows) : n;
    all_see = a.causal ? min(n, q0 + 1) : n;
    if (in) limit = a.causal ? qr + 1 : n;
  }
  const int steps = (end + KK - 1) / KK;
  const int whole = all_see / KK;  // steps whose keys are all there, and seen by all queries of the tile
  const int wave_sees = __builtin_amdgcn_readfirstlane((int)lanes64_max((unsigned)limit));

  // the wave's queries, for good: lane = query, sixteen-byte pieces 2 s + half
  constexpr int kPieces = DC * kEb / 32, kPer = 16 / kEb;
  tok_u4 qf[kPieces];
#pragma unroll
  for (int s = 0; s < kPieces; ++s) {
    const int d = (2 * s + half) * kPer;
    qf[s] = tok_u4{0, 0, 0, 0};
    if (in && d < a.D) qf[s] = *reinterpret_cast<const tok_u4*>(reinterpret_cast<const ET*>(a.q) + my_row * a.ldq + head * a.D + d);
  }

  // Sixteen keys of a cache lie in one page: a step's pages, and which of its keys are there.
  constexpr int kSixteens = KK / 16;
  struct Pages {
    long long at[kSixteens];  // the first one's row of the cache
    unsigned long long there;
  };
  int ahead[kSixteens];  // page numbers of the step that is asked for next
  auto look_up = [&](int step) {
    if constexpr (PAGED) {
#pragma unroll
      for (int g = 0; g < kSixteens; ++g) {
        const int key = step * KK + 16 * g;
        ahead[g] = key < end ? part.table[(part.begin + key) >> cache.page_bits] : -1;
      }
    }
  };
  auto pages_of = [&](int step) {
    Pages s{};
    if constexpr (PAGED) {
#pragma unroll
      for (int g = 0; g < kSixteens; ++g) {
        const int key = step * KK + 16 * g, page = __builtin_amdgcn_readfirstlane(ahead[g]);
        if ((unsigned)page < (unsigned)cache.pages) {  // (-1 past the end)
          s.at[g] = (((long long)page * cache.kv_heads + hk) << cache.page_bits) + ((part.begin + key) & ((1 << cache.page_bits) - 1));
          s.there |= ((1ull << min(16, end - key)) - 1) << (16 * g);
        }
      }
    }
    return s;
  };

  // which of a step's keys are there, a bit each
  auto rows_there = [&](int step) -> unsigned long long {
    const long long rows = n - (long long)step * KK;
    return rows >= 64 ? ~0ull : rows <= 0 ? 0 : (1ull << rows) - 1;
  };
  // LDS-direct loads of a step: load i brings rows i * NW * kRowsLoad + wave * kRowsLoad .., of which a lane has one chunk, the same of
  // each where the swizzles' periods (16 rows) allow.
  constexpr bool kSame = NW * kRowsLoad % 16 == 0;
  constexpr int kOffsets = kSame ? 1 : kLoads;
  unsigned vk[kOffsets], vv[kOffsets];
#pragma unroll
  for (int i = 0; i < kOffsets; ++i) {
    const int row = (i * NW + wave) * kRowsLoad + lane / kLanesRow, pos = lane % kLanesRow;
    const int ck = (pos ^ L::key_swizzle(row)) * kPer, cv = (pos ^ L::value_swizzle(row)) * kPer;
    const int from = KEPT ? 0 : PAGED ? lane / kLanesRow : row;  // (a load of a cache begins with its first row)
    vk[i] = ck < a.D ? (unsigned)(from * a.ldk + ck) * kEb : kOutside;
    vv[i] = cv < a.D ? (unsigned)(from * a.ldv + cv) * kEb : kOutside;
  }
  auto request = [&](const ET* from, int64_t ld, const unsigned (&off)[kOffsets], unsigned to, bool all, unsigned long long there) {
    const unsigned stage = __builtin_amdgcn_readfirstlane(to + wave * 1024);
    const __amdgpu_buffer_rsrc_t r = bytes_of(scalar_pointer(from), 0x7fffffff);
    if (all) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        dma16(r, off[kSame ? 0 : i], kSame ? (unsigned)(i * NW * kRowsLoad * kEb) * (unsigned)ld : 0u, stage + i * NW * 1024);
    } else {  // rows that are not there come as zeros (their weights are 0, and so are not 0 * NaN)
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const unsigned skip = kSame ? (unsigned)(i * NW * kRowsLoad * kEb) * (unsigned)ld : 0u, o = off[kSame ? 0 : i];
        const bool in = (unsigned)(there >> (i * NW + wave) * kRowsLoad) >> lane / kLanesRow & 1;
        dma16(r, in && o != kOutside ? o + skip : kOutside, 0, stage + i * NW * 1024);
      }
    }
  };
  auto request_pages = [&](const uint8_t* base, const unsigned (&off)[kOffsets], unsigned to, const Pages& s) {
    const unsigned stage = __builtin_amdgcn_readfirstlane(to + wave * 1024);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int row = (i * NW + wave) * kRowsLoad, bits = (int)(s.there >> row & ((1u << kRowsLoad) - 1));
      long long at = 0;
#pragma unroll
      for (int g = 0; g < kSixteens; ++g)
        if (row / 16 == g) at = s.at[g] + row % 16;
      dma16(bytes_of(scalar_pointer(base + at * a.D * kEb), __popc((unsigned)bits) * a.D * kEb), off[kSame ? 0 : i], 0, stage + i * NW * 1024);
    }
  };
  // Kept rows, by the list: a lane's row of each load, from the wave's first one on.  Where that is too far for one descriptor, row by row.
  constexpr int kOfList = KEPT ? kLoads : 1;
  int row_of[kOfList];  // of the keys that were asked for last
  auto look_at_list = [&](int step) {
    const int k0 = step * KK, rows = min(KK, end - k0);
#pragma unroll
    for (int i = 0; i < kOfList; ++i)
      row_of[i] = list[(k0 + min((i * NW + wave) * kRowsLoad + lane / kLanesRow, max(rows - 1, 0))) % kListed];
  };
  auto request_kept = [&](const ET* base, int64_t ld, const unsigned (&off)[kOffsets], unsigned to, int step) {
    const unsigned stage = __builtin_amdgcn_readfirstlane(to + wave * 1024);
    const int rows = min(KK, end - step * KK);  // (none, past the end)
    const int first = rows > 0 ? __builtin_amdgcn_readlane(row_of[0], 0) : 0;
    const int last = rows > 0 ? __builtin_amdgcn_readlane(row_of[kOfList - 1], kWave - 1) : 0;
    if (((long long)(last - first) * ld + a.D) * kEb <= 0x7fffffff) {
      const __amdgpu_buffer_rsrc_t r = bytes_of(scalar_pointer(base + first * ld), 0x7fffffff);
#pragma unroll
      for (int i = 0; i < kOfList; ++i) {
        const bool there = (i * NW + wave) * kRowsLoad + lane / kLanesRow < rows;
        const unsigned o = off[kSame ? 0 : i];
        dma16(r, there && o != kOutside ? (unsigned)(row_of[i] - first) * ((unsigned)ld * kEb) + o : kOutside, 0, stage + i * NW * 1024);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kOfList; ++i)
#pragma unroll 1
        for (int j = 0; j < kRowsLoad; ++j) {
          const bool there = (i * NW + wave) * kRowsLoad + j < rows;
          const int row = there ? __builtin_amdgcn_readlane(row_of[i], j * kLanesRow) : 0;
          const __amdgpu_buffer_rsrc_t r = bytes_of(scalar_pointer(base + row * ld), there ? a.D * kEb : 0);
          if (lane / kLanesRow == j) dma16(r, off[kSame ? 0 : i], 0, stage + i * NW * 1024);
        }
    }
  };
  Pages asked;  // of the keys that were asked for last
  auto ask_keys = [&](int step) {
    const unsigned to = (step & 1) * L::kPart;
    if constexpr (PAGED) {
      asked = pages_of(step);
      look_up(step + 1);
      request_pages(cache.k, vk, to, asked);
    } else if constexpr (KEPT) {
      look_at_list(step);
      request_kept(kp, a.ldk, vk, to, step);
    } else {
      request(kp + (long long)step * KK * a.ldk, a.ldk, vk, to, step < whole, step < whole ? 0 : rows_there(step));
    }
  };
  auto ask_values = [&](int step) {  // (of a cache: of the keys that were asked for last)
    const unsigned to = L::kValues + (step & 1) * L::kPart;
    if constexpr (PAGED) request_pages(cache.v, vv, to, asked);
    else if constexpr (KEPT) request_kept(vp, a.ldv, vv, to, step);
    else request(vp + (long long)step * KK * a.ldv, a.ldv, vv, to, step < whole, step < whole ? 0 : rows_there(step));
  };

  f32x16 acc[kDt];
#pragma unroll
  for (int t = 0; t < kDt; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[t][e] = 0.f;
  float top = kNoScore, sum = 0.f;

  // which of the keys that are there the lane's query sees
  auto seen_of = [&](int k0, unsigned long long here) -> unsigned long long {
    const int sees = limit - k0;
    return sees <= 0 ? 0 : sees >= 64 ? here : here & ((1ull << sees) - 1);
  };
  const int i16 = lane % 16, low = (lane / 16) % 2 * 2 + i16 % 4 / 2;
  // keys 32 u + 8 * (e / 4) + 4 * half + e % 4 of a step with the lane's query
  auto scores_part = [&](f32x16 (&s)[kBlocks], const unsigned char* ks, int i) {
#pragma unroll
    for (int u = 0; u < kBlocks; ++u) {
      const tok_u4 kf = *reinterpret_cast<const tok_u4*>(ks + (u * 32 + r32) * L::kRow + (((2 * i + half) ^ L::key_swizzle(r32)) << 4));
      if constexpr (kHalf) {
        s[u] = mma32(kf, qf[i], s[u]);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) s[u] = mma32(__uint_as_float(kf[j]), __uint_as_float(qf[i][j]), s[u]);
      }
    }
  };
  auto clear = [&](f32x16 (&s)[kBlocks]) {
#pragma unroll
    for (int u = 0; u < kBlocks; ++u)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[u][e] = 0.f;
  };
  auto hide = [&](f32x16 (&s)[kBlocks], unsigned long long seen) {  // what the lane's query does not see
    seen >>= 4 * half;
#pragma unroll
    for (int u = 0; u < kBlocks; ++u) {
      const unsigned bits = (unsigned)(seen >> (32 * u));
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const unsigned m = (unsigned)((int)(bits << (31 - 8 * (e / 4) - e % 4)) >> 31);  // all bits, or none
        s[u][e] = __uint_as_float((__float_as_uint(s[u][e]) & m) | (__float_as_uint(kNoScore) & ~m));
      }
    }
  };
  // whether a score has grown past the maximum that the sums are relative to
  auto most_of = [&](const f32x16 (&s)[kBlocks]) {
    float most[2] = {s[0][0], s[0][1]};
#pragma unroll
    for (int u = 0; u < kBlocks; ++u)
#pragma unroll
      for (int e = 0; e < 16; ++e) most[e % 2] = fmaxf(most[e % 2], s[u][e]);
    return other_half_max(fmaxf(most[0], most[1])) * a.c;
  };
  auto raise = [&](float most) {
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
  };

  // 0 * NaN is NaN, so where some queries of a tile do not see all of a step's keys, values that are not finite must not meet the matrix
  // instructions.  They become zeros in LDS, and are added to the queries that see them one by one, from memory.
  int* const found = reinterpret_cast<int*>(lds + L::kFlags);  // of two steps in turn
  auto take_out = [&](int turn) {
    tok_u4* const vs = reinterpret_cast<tok_u4*>(lds + L::kValues + turn * L::kPart);
    bool bad = false;
#pragma unroll
    for (int i = 0; i < L::kPart / 16 / (NW * kWave); ++i) {
      const int at = (i * NW + wave) * kWave + lane;
      tok_u4 v = vs[at];
      bool here = false;
#pragma unroll
      for (int j = 0; j < 4; ++j) here |= kHalf ? not_finite2(v[j]) : not_finite(__uint_as_float(v[j]));
      if (here) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = kHalf ? finite2(v[j]) : not_finite(__uint_as_float(v[j])) ? 0u : v[j];
        vs[at] = v;
        bad = true;
      }
    }
    if (__ballot(bad) && lane == 0) found[turn] = 1;
  };
  auto add_back = [&](int k0, unsigned long long here) {
    const unsigned long long seen = seen_of(k0, here);
#pragma unroll 1
    for (int j = 0; j < KK; ++j) {
      if (!((here >> j) & 1)) continue;
      const uint8_t* from = reinterpret_cast<const uint8_t*>(vp + (long long)(KEPT ? list[(k0 + j) % kListed] : k0 + j) * a.ldv);
      if constexpr (PAGED) {
        const int key = part.begin + k0 + j, page = __builtin_amdgcn_readfirstlane(part.table[key >> cache.page_bits]);
        const long long at = (((long long)page * cache.kv_heads + hk) << cache.page_bits) + (key & ((1 << cache.page_bits) - 1));
        from = cache.v + at * a.D * kEb;
      }
      const __amdgpu_buffer_rsrc_t row = bytes_of(scalar_pointer(from), a.D * kEb);
      const bool sees = (seen >> j) & 1;
#pragma unroll
      for (int t = 0; t < kDt; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          float v[4];
          if constexpr (kHalf) {
            const tok_u2 x = load8(row, half * 8 + (32 * t + 8 * g) * 2);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(e % 2 ? x[e / 2] & 0xffff0000u : x[e / 2] << 16);
          } else {
            const tok_u4 x = load16(row, half * 16 + (32 * t + 8 * g) * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(x[e]);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[t][4 * g + e] += sees && not_finite(v[e]) ? v[e] : 0.f;
        }
    }
  };

  // A step's scores are made while the step before becomes weights: matrix and vector instructions of one wave side by side.  Keys are
  // asked for two steps ahead, values one.
  const bool mixed = all_see < end;  // some queries see fewer keys than others
  if (mixed && threadIdx.x < 2) found[threadIdx.x] = 0;
  look_up(0);
  ask_keys(0);
  ask_values(0);
  const unsigned long long there_first = PAGED ? asked.there : 0;
  ask_keys(1);
  // of a step's keys, those that are there (of a cache: as they were asked for)
  auto there_of = [&](int step, unsigned long long pages) { return PAGED ? pages : rows_there(step); };
  constexpr unsigned long long kAll = KK == 64 ? ~0ull : 0xffffffffull;
  auto hidden = [&](f32x16 (&s)[kBlocks], int step, unsigned long long pages) {
    if (step >= whole || (PAGED && pages != kAll)) hide(s, seen_of(step * KK, there_of(step, pages)));
  };
  f32x16 s0[kBlocks], s1[kBlocks];
  vm_wait<2 * kLoads>();
  __syncthreads();
  clear(s0);
#pragma unroll
  for (int i = 0; i < kPieces; ++i) scores_part(s0, lds, i);
  hidden(s0, 0, there_first);
  raise(most_of(s0));
  unsigned long long there_now = there_first;
  auto body = [&](int step, f32x16 (&s)[kBlocks], f32x16 (&next)[kBlocks]) {
    const int k0 = step * KK, turn = step & 1;
    vm_wait<0>();
    __syncthreads();  // the next keys and the values are there, and nobody reads the stages that are filled now any more
    if constexpr (KEPT)  // (for the next step; in the place of rows that steps before this one had)
      for (; listed < min(end, k0 + 4 * KK) && scanned < rows_of_sequence; scanned += kScan)
        listed = scan(keep, rows_of_sequence, scanned, listed, [&](int number, int row) { list[number % kListed] = row; });
    ask_values(step + 1);
    const unsigned long long there_next = PAGED ? asked.there : 0, there = there_now;
    there_now = there_next;
    ask_keys(step + 2);
    const bool partly = mixed && step >= whole;
    if (partly) {
      take_out(turn);
      __syncthreads();
      if (threadIdx.x == 0) found[turn ^ 1] = 0;  // (the next step's, whose last reader has passed this barrier)
    }
    if (k0 >= wave_sees) return;  // (no keys that the wave's queries see, from here on)
    const unsigned char *ks = lds + (turn ^ 1) * L::kPart, *vs = lds + L::kValues + turn * L::kPart;
    float shift = shift_of(top), by = a.c;
    if (any_large(shift)) {  // (exponents in the place of scores)
#pragma unroll
      for (int u = 0; u < kBlocks; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[u][e] = rounded_exponent(s[u][e], by, shift);
      shift = 0.f;
      by = 1.f;
    }
    clear(next);
    float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      scores_part(next, ks, i);
#pragma unroll
      for (int e = i * 16 * kBlocks / kPieces; e < (i + 1) * 16 * kBlocks / kPieces; ++e) {
        s[e / 16][e % 16] = exp2_fast(fmaf(s[e / 16][e % 16], by, -shift));
        part[e % 4] += s[e / 16][e % 16];
      }
    }
    sum += (part[0] + part[1]) + (part[2] + part[3]);
    // out^T += values^T * weights
    if constexpr (kHalf) {
      tok_u4 w[kBlocks * 2];
#pragma unroll
      for (int t = 0; t < kBlocks * 2; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) w[t][j] = pack_bf16(s[t / 2][8 * (t % 2) + 2 * j], s[t / 2][8 * (t % 2) + 2 * j + 1]);
      const unsigned char* const from = vs + (4 * half + i16 / 4) * L::kRow + i16 % 2 * 8;
#pragma unroll
      for (int t = 0; t < kBlocks * 2; ++t)
#pragma unroll
        for (int dt = 0; dt < kDt; ++dt) {
          const unsigned char* const at = from + 16 * t * L::kRow + (((4 * dt + low) ^ L::value_swizzle(i16 / 4)) << 4);
          const tok_u2 lo = read_transposed(at), hi = read_transposed(at + 8 * L::kRow);
          acc[dt] = mma32(tok_u4{lo[0], lo[1], hi[0], hi[1]}, w[t], acc[dt]);
        }
    } else {
      const float* const from = reinterpret_cast<const float*>(vs) + 4 * half * DP + r32;
#pragma unroll
      for (int e = 0; e < 16; ++e)
#pragma unroll
        for (int dt = 0; dt < kDt; ++dt) acc[dt] = mma32(from[(8 * (e / 4) + e % 4) * DP + 32 * dt], s[0][e], acc[dt]);
    }
    hidden(next, step + 1, there_next);
    const float most = most_of(next);
    if (partly && found[turn]) add_back(k0, there_of(step, there));
    raise(most);
  };
  for (int step = 0; step < steps;) {
    body(step++, s0, s1);
    if (step >= steps) break;
    body(step++, s1, s0);
  }
  vm_wait<0>();  // (no load into LDS is left behind)
  sum = other_half_sum(sum);

  if constexpr (KEPT) put_zeros(first_row + (long long)first_query + threadIdx.x / 2, head);
  // out: the lane's query, channels 32 t + 16 * half .. + 15; of a part of the keys its sums as they are, maximum and sum of weights beside
  const bool parts = PAGED && cache.splits + cache.prefix_splits > 1, none = !parts && sum == 0.f;
  const float inv = parts ? 1.f : 1.f / sum;
  long long at = 0;
  if constexpr (PAGED) {
    at = ((long long)(part.shared ? cache.splits + part.split : part.split) * cache.T + my_row) * a.heads + head;
    if (parts && in && half == 0) {
      cache.part_stat[2 * at] = top;
      cache.part_stat[2 * at + 1] = sum;
    }
  }
  ET* const out = reinterpret_cast<ET*>(a.out) + my_row * a.ldo + head * a.D;
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
      if (!in || d >= a.D) continue;
      if (parts) {
        piece8<float> p;
        p.put(f[g]);
        p.store(cache.part_out + at * a.D, d / 8);
      } else {
        piece8<ET> p;
        p.put(f[g]);
        p.store(out, d / 8);
      }
    }
  }
}

// With 64 channels a row a compute unit has room for four workgroups, and a launch of few is spread unevenly: a workgroup then asks for half
// of the LDS.  4 x 16 x 1024 tokens of float32 211 -> 154 us, 4 x 32 x 512 114 -> 85, 32 x 16 x 197 94 -> 83, of bf16 and 32 channels 4 x 16 x
// 1024 29 -> 23; with 1024 tiles (1 x 64 x 2048) it costs 2 to 6 %.
constexpr int kSpreadBytes = 80 * 1024, kSpreadTiles = 1024;
template <typename ET, int DC, int FROM>
int ask_tile_lds() {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(&k_attend<ET, DC, FROM>), hipFuncAttributeMaxDynamicSharedMemorySize,
                             kSpreadBytes) == hipSuccess ? LAUD_OK : LAUD_ERR_HIP;
}
template <typename ET, int DC, int FROM>
void launch_tiles(const AttendArgs& a, const CachedArgs& cache, unsigned groups, hipStream_t st) {
  constexpr int kBytes = AttendTile<ET, DC>::bytes(FROM);
  static_assert(kBytes <= kSpreadBytes, "two workgroups a compute unit");
  hipLaunchKernelGGL((k_attend<ET, DC, FROM>), dim3(groups), dim3(kAttendWaves * kWave),
                     ((long long)a.T * a.heads / kAttendRows < kSpreadTiles ? kSpreadBytes : kBytes), st, a, cache);
}

template <typename ET, int DC>
int launch_attend(AttendArgs a, hipStream_t st) {
  const long long tiles = tiles_of(a.T, a.B, 1, kAttendRows), groups = (tiles * a.heads + 7) / 8 * 8;
  if (!launchable((double)groups, kAttendWaves * kWave)) return LAUD_ERR_UNSUPPORTED;
  if (attend_init_device() != LAUD_OK) return LAUD_ERR_HIP;
  a.tiles = (int)tiles;
  if (a.keep) launch_tiles<ET, DC, kRowsKept>(a, CachedArgs{}, (unsigned)groups, st);
  else launch_tiles<ET, DC, kRowsAll>(a, CachedArgs{}, (unsigned)groups, st);
  return check_launch();
}
template <typename ET>
int launch_width(const AttendArgs& a, hipStream_t st) {
  if (a.D <= 32) return launch_attend<ET, 32>(a, st);
  if (a.D <= 64) return launch_attend<ET, 64>(a, st);
  if (a.D <= 96) return launch_attend<ET, 96>(a, st);
  return launch_attend<ET, 128>(a, st);
}

// LDS of every instance (more than the 64 KB that a launch may take unasked)
template <typename ET, int DC>
int ask_lds_of_width() {
  const int rc = ask_tile_lds<ET, DC, kRowsAll>();
  return rc != LAUD_OK ? rc : ask_tile_lds<ET, DC, kRowsKept>();
}
int attend_init_device() {
  static std::atomic<unsigned> done{0};  // one bit per device ordinal (ordinals >= 32 repeat the request)
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return LAUD_ERR_HIP;
  const unsigned bit = dev >= 0 && dev < 32 ? 1u << dev : 0u;
  if (bit && (done.load(std::memory_order_acquire) & bit)) return LAUD_OK;
  for (int rc : {ask_lds_of_width<bf16_t, 32>(), ask_lds_of_width<bf16_t, 64>(), ask_lds_of_width<bf16_t, 96>(), ask_lds_of_width<bf16_t, 128>(),
                 ask_lds_of_width<float, 32>(), ask_lds_of_width<float, 64>(), ask_lds_of_width<float, 96>(), ask_lds_of_width<float, 128>(),
                 ask_tile_lds<bf16_t, 64, kRowsCached>(), ask_tile_lds<bf16_t, 128, kRowsCached>()})
    if (rc != LAUD_OK) return rc;
  done.fetch_or(bit, std::memory_order_release);
  return LAUD_OK;
}

void launch_many_rows(const CachedArgs& c, unsigned groups, hipStream_t st) {
  AttendArgs a{};
  a.heads = c.heads; a.group = c.group; a.D = c.D; a.c = c.c; a.T = c.T;
  a.q = c.q; a.out = c.out; a.ldq = c.ldq; a.ldo = c.ldo;
  a.ldk = a.ldv = c.D;
  if (c.D <= 64) launch_tiles<bf16_t, 64, kRowsCached>(a, c, groups, st);
  else launch_tiles<bf16_t, 128, kRowsCached>(a, c, groups, st);
}

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
  if (T > 1 << 30 || ldq > kMaxRowDistance || ldk > kMaxRowDistance || ldv > kMaxRowDistance || ldo > kMaxRowDistance) return LAUD_ERR_UNSUPPORTED;
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
  // Few rows leave these tiles without enough workgroups; 16 rows a workgroup with its waves sharing the keys fill the card sooner, but
  // fetch the keys more often.  Both, in us (causal; sequences x heads x tokens, widths of 64 float32 and 128 bf16):
  //   1 x 8 x 64  10.8, 5.4    4 x 16 x 128  18, 10    8 x 16 x 200  34, 24      1 x 16 x 1024  80, 38       1 x 32 x 512  45, 23     4 x 32 x 512  65, 73
  //   1 x 8 x 64   7.5, 7.1    4 x 16 x 128  11, 11    1 x 16 x 256  12.6, 9.6   1 x 16 x 512   17.8, 15.8   16 x 16 x 64  11, 17     1 x 32 x 512  18, 25
  // where every query sees all of its sequence:
  //   8 x 16 x 200  39, 28     1 x 16 x 1024  79, 53    1 x 16 x 2048  154, 177    4 x 32 x 512  80, 106
  //   4 x 16 x 128  9.3, 9.4   1 x 16 x 256  10.7, 8.5   1 x 16 x 512  16.2, 17.6   1 x 8 x 1024  24.6, 26.5
  // Many short sequences leave most of a tile's rows without a query.  Both, in us (sequences x tokens; 16 heads of 64 and 32 of 128 over 8):
  //   float32  128 x 16  42, 23 and 133, 61    128 x 33  67, 40 and 203, 128    128 x 48  70, 54 and 207, 178    128 x 64  65, 60 and 214, 242
  //   bf16     256 x 8   43, 27 and 109, 54    256 x 14  46, 30 and 112, 101    256 x 16  44, 43 and 113, 105    128 x 33  26, 34 and  63, 111
  //   bf16, 12 heads of 80 and 16 of 128: 256 x 14  44, 44 and 64, 64    256 x 16  42, 53 and 61, 100
  // Both rules take the sequences for about as long as each other: a long one among many short ones goes their way.
  const bool few = (int64_t)p->heads * T <= (p->dtype == LAUD_F32 ? 28000 : 8192), brief = T <= (int64_t)B * (p->dtype == LAUD_F32 ? 48 : 14);
  if ((few || brief) && launchable((double)tiles_of(T, B, a.group, 16) * p->kv_heads, kAttendWaves * kWave))
    return attend_few(*p, B, offsets, T, q, ldq, k, ldk, v, ldv, keep, out, ldo, st);
  return p->dtype == LAUD_BF16 ? launch_width<bf16_t>(a, st) : launch_width<float>(a, st);
}
