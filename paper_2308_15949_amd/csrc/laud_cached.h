// Attention over a cache: the arguments of its kernels, and which rows and keys a workgroup has (laud_cached.hip, laud_attend.hip).
#pragma once

#include "laud_heads.h"

namespace laud {

struct CachedArgs {
  int heads, group, kv_heads, D, causal, B, T, pages, page_bits, table_ld, prefix_len;
  // of the sequences' own keys, and of the prefix, whose workgroups come first: tiles of query rows, and parts that a tile's keys are
  // shared out over; all parts of a row are joined, its own first
  int tiles, splits, prefix_tiles, prefix_splits;
  unsigned prefix_groups;
  int by_xcd, prefix_by_xcd;
  // rows of this call in place of a cache: how far apart, and which the masker kept
  int64_t ldk, ldv;
  const uint8_t* keep;
  float c;                // scale * log2(e)
  unsigned group_by, group_shift;  // x / group = x * group_by >> group_shift (x below 2^31)
  const int32_t *offsets, *lens, *table, *prefix;
  const uint8_t *k, *v;
  const float *ks, *vs;
  const void* q;
  void* out;
  float *part_out, *part_stat;  // [parts][T * heads][D] and [parts][T * heads][2]: maximum and sum
  int64_t ldq, ldo;
};

constexpr int kCachedWaves = 4, kMaxParts = 64, kPartStep = 128;
// Keys of a part: the same for every tile of a sequence, so that whoever joins the parts knows how many there are.
__device__ __forceinline__ int part_keys(int len, int splits) {
  const int each = (len + splits - 1) / splits;
  return max((each + kPartStep - 1) / kPartStep * kPartStep, kPartStep);
}
__device__ __forceinline__ int parts_of(int len, int splits) {  // how many of them have keys; one where there are none
  const int each = part_keys(len, splits);
  return max((len + each - 1) / each, 1);
}
__device__ __forceinline__ int cached_tokens(const CachedArgs& a, int len) {  // of a sequence's length, those that its table has room for
  const long long room = (long long)a.table_ld << a.page_bits;
  return (int)min((long long)max(len, 0), room);
}

__device__ __forceinline__ unsigned token_of(const CachedArgs& a, unsigned row) {
  return (unsigned)((unsigned long long)row * a.group_by >> a.group_shift);
}

// A workgroup's rows - tokens of a sequence (of the prefix' workgroups: all tokens) times the query heads of a key head - and the
// part of the keys that it looks at.
struct CachedTile {
  bool shared, causal;             // the prefix
  int hk, split, row0, n, len;     // key head, part; the sequence's first row, its rows, its keys
  int begin, end, all_see;         // the part's keys: from begin to end, of which every row of the tile sees those below all_see
  unsigned first_row, rows;        // the tile's first row, and the sequence's
  int there;                       // rows of the tile
  long long past;                  // position of the first token
  const int32_t* table;
  __device__ __forceinline__ int limit_of(const CachedArgs& a, unsigned row) const {  // keys that a row sees
    return causal ? (int)min(max(past + token_of(a, row) + 1, 0ll), (long long)len) : len;
  }
};
template <int ROWS_TILE>
__device__ __forceinline__ bool cached_tile(CachedTile& t, const CachedArgs& a) {
  // Where several tiles read the same keys they go to one XCD, one behind the other.
  t.shared = blockIdx.x < a.prefix_groups;
  const unsigned id = t.shared ? blockIdx.x : blockIdx.x - a.prefix_groups;
  const unsigned tiles = t.shared ? a.prefix_tiles : a.tiles, splits = t.shared ? a.prefix_splits : a.splits;
  int tile;
  if (t.shared ? a.prefix_by_xcd : a.by_xcd) {
    const unsigned j = id / 8;
    const unsigned g = j / tiles * 8 + id % 8;
    tile = j % tiles;
    t.hk = g % a.kv_heads;
    t.split = g / a.kv_heads;
  } else {
    t.split = id % splits;
    const unsigned j = id / splits;
    t.hk = j % a.kv_heads;
    tile = j / a.kv_heads;
  }
  int len = a.prefix_len;
  t.row0 = 0; t.n = a.T; t.len = len;
  t.table = a.prefix;
  if (!t.shared) {
    const Sequence s = sequence_at(a.offsets, a.lens, a.B, a.T, [&](int row, int i) { return first_tile(row, i, a.group, ROWS_TILE) <= tile; });
    t.row0 = s.row0;
    t.n = s.next - s.row0;
    len = s.len;
    const long long before = first_tile(s.row0, s.b, a.group, ROWS_TILE);
    if ((long long)tile < before) return false;
    tile = __builtin_amdgcn_readfirstlane(tile - (int)before);
    t.len = __builtin_amdgcn_readfirstlane(cached_tokens(a, s.len));
    t.table = a.table + (long long)s.b * a.table_ld;
  }
  if (t.n <= 0) return false;
  t.rows = (unsigned)t.n * (unsigned)a.group;  // (T * heads is below 2^31)
  t.first_row = (unsigned)tile * ROWS_TILE;
  if (t.first_row >= t.rows) return false;
  t.there = (int)min((unsigned)ROWS_TILE, t.rows - t.first_row);
  const int each = part_keys(t.len, splits);
  if (t.split > 0 && (long long)t.split * each >= t.len) return false;
  t.past = (long long)len - t.n;
  t.causal = a.causal && !t.shared;
  t.begin = __builtin_amdgcn_readfirstlane(t.split * each);
  t.hk = __builtin_amdgcn_readfirstlane(t.hk);
  t.split = __builtin_amdgcn_readfirstlane(t.split);
  t.there = __builtin_amdgcn_readfirstlane(t.there);
  t.first_row = (unsigned)__builtin_amdgcn_readfirstlane((int)t.first_row);
  t.table = scalar_pointer(t.table);
  t.end = __builtin_amdgcn_readfirstlane(min(min(t.begin + each, t.len), t.limit_of(a, t.first_row + t.there - 1)));
  t.all_see = __builtin_amdgcn_readfirstlane(t.limit_of(a, t.first_row));
  return true;
}

// the kernel of many rows (laud_attend.hip), for bf16: 128 a workgroup, keys through LDS
constexpr int kManyRows = 128;
void launch_many_rows(const CachedArgs& a, unsigned groups, hipStream_t st);

}  // namespace laud
