// Matrix product of e4m3 operands with a scale for each block of 128.
#include <atomic>
#include <cmath>

#include "laud_token.h"

namespace laud {

struct Mm8Args {
  const uint8_t *a, *b;
  const float *sa, *sb;
  void* out;
  int M, N, K, kb;           // kb: blocks of 128 along K
  int64_t lda, ldb, ldo;
};

constexpr double kComputeUnits = 256;
constexpr int64_t kMaxLd = 1 << 22;    // elements from row to row: 256 rows of a tile stay below the 2 GiB a descriptor addresses
// Sixteen rows of the first operand times sixteen of the second over a block of 128: lane l holds row l % 16, bytes 16 * (l / 16)
// and 64 behind them (any order of K serves as long as both operands have the same).  Result: row 4 * (l / 16) + i of the first,
// row l % 16 of the second.  The codes are widened to bf16, which holds them exactly, for every result: the 8-bit matrix
// instructions take half the time, but they add groups of eight products with 14 bits below the group's largest (2^16 + 2^2 in one
// group is 2^16, and 2^16 - 2^16 + 2^2 nothing; measured 1.5e-5 of a result's norm, against 3e-7 here).
typedef int i32x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ i32x8 join(const tok_u4& a, const tok_u4& b) {
  return __builtin_bit_cast(i32x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}
__device__ __forceinline__ f32x4 mma_block(const i32x8& a, const i32x8& b) {
  f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int h = 0; h < 8; h += 2)
    c = mma_bf16_16(widen8((unsigned)a[h], (unsigned)a[h + 1]), widen8((unsigned)b[h], (unsigned)b[h + 1]), c);
  return c;
}

// Up to 16 rows: the weights are read once, for all of them.  A workgroup has 16 columns, its waves share the reduction, their sums are
// added in the waves' order.  Bound by memory and the launch: one row of 4096 x 4096 in 5.2 us back to back, 5.0 to 6.6 by itself (back
// to back 5.6 with all of a wave's blocks asked for at once, 5.2 to 5.3 with sixteen waves).
constexpr int kSplit = 8, kSplitRows = 16;
template <typename OT>
__global__ __launch_bounds__(kSplit * kWave) void k_mm8_split(Mm8Args g) {
  extern __shared__ __align__(16) unsigned char lds[];  // (LDS-direct loads of the other kernels: no static LDS in this file)
  f32x4(*part)[kWave] = reinterpret_cast<f32x4(*)[kWave]>(lds);
  const int lane = lane_id(), wave = threadIdx.x / kWave, r16 = lane % 16, quarter = lane / 16;
  const int n0 = blockIdx.x * 16, nrows = min(16, g.N - n0);
  const __amdgpu_buffer_rsrc_t rb = bytes_of(g.b + n0 * g.ldb, (nrows - 1) * g.ldb + g.K);
  const __amdgpu_buffer_rsrc_t ra = bytes_of(g.a, (g.M - 1) * g.lda + g.K);
  const unsigned off_b = (unsigned)(min(r16, nrows - 1) * g.ldb), off_a = (unsigned)(min(r16, g.M - 1) * g.lda);
  const float* sa = g.sa + (long long)min(r16, g.M - 1) * g.kb;
  const float* sb = g.sb + (long long)(n0 / kScaleBlock) * g.kb;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int kb = wave; kb < g.kb; kb += kSplit) {
    tok_u4 w[2], x[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = kb * kScaleBlock + h * 64 + quarter * 16;
      w[h] = load16(rb, k < g.K ? off_b + (unsigned)k : kOutside);
      x[h] = load16(ra, k < g.K ? off_a + (unsigned)k : kOutside);
    }
    const float f = sb[kb] * sa[kb];
    const f32x4 p = mma_block(join(w[0], w[1]), join(x[0], x[1]));
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = fmaf(p[i], f, acc[i]);
  }
  part[wave][lane] = acc;
  __syncthreads();
  if (wave != 0) return;
#pragma unroll
  for (int w = 1; w < kSplit; ++w) acc += part[w][lane];
  const int n = n0 + quarter * 4;
  if (r16 < g.M && n < g.N) store4(reinterpret_cast<OT*>(g.out) + r16 * g.ldo + n, acc);
}

// ---- tiles ------------------------------------------------------------------------------------------------------------------
// BM x BN results a workgroup, WM x WN a wave; KG groups of waves share the blocks of K.  Both operands go into LDS by LDS-direct
// loads, a block of 128 along K at a time, into NS stages that take turns: one barrier a block, the next blocks' loads are under way
// while this one is multiplied.  A row's eight 16-byte chunks lie XOR-swizzled (chunk ^ row % 8; the swizzle is applied to the global
// side).  The first operand of the matrix instructions is b: a lane's results are consecutive columns, its row of a - and that row's
// scale - is one for all of them.  Bound by the matrix cores at their bf16 rate: 8192 x 8192 x 4096 in 412 to 444 us, 1.2 to 1.3
// PFLOP/s, where a large bf16 product of the vendor's library reaches 1.1.
template <int BM, int BN, int NS, int KG> struct TileLds {
  static constexpr int kB = 0, kA = BN * kScaleBlock, kSa = kA + BM * kScaleBlock, kSb = kSa + BM * 4, kStage = kSb + 256;
  static constexpr int kGroup = NS * kStage, kBytes = KG * kGroup;
};

template <typename OT, int BM, int BN, int WM, int WN, int NS, int KG>
__global__ __launch_bounds__(KG * BM / WM * (BN / WN) * kWave) void k_mm8_tile(Mm8Args g, int mtiles, int ntiles) {
  typedef TileLds<BM, BN, NS, KG> L;
  constexpr int kWaves = BM / WM * (BN / WN), kMT = WM / 16, kNT = WN / 16;
  constexpr int kLoadsB = BN / 8 / kWaves, kLoadsA = BM / 8 / kWaves;
  static_assert(kLoadsB * 8 * kWaves == BN && kLoadsA * 8 * kWaves == BM && BM < kWaves * kWave && BM % kWave == 0 && kMT % 2 == 0,
                "rows shared evenly");
  extern __shared__ __align__(16) unsigned char lds[];
  const int lane = lane_id(), r16 = lane % 16, quarter = lane / 16;
  const int group = __builtin_amdgcn_readfirstlane(threadIdx.x / (kWaves * kWave));
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) - group * kWaves;
  uint8_t* const stages = lds + group * L::kGroup;  // a group's own
  const unsigned lds0 = group * L::kGroup;          // ... from the start of the workgroup's LDS (there is no static LDS)
  // Workgroups go round-robin over the eight XCDs: each takes a run of tiles, in bands of eight rows of tiles, so that its L2 serves
  // a block of them.
  const int tiles = mtiles * ntiles, per = (tiles + 7) / 8;
  const int id = (int)(blockIdx.x % 8) * per + (int)(blockIdx.x / 8);
  if ((int)(blockIdx.x / 8) >= per || id >= tiles) return;
  const int band = id / (8 * ntiles), in_band = id - band * 8 * ntiles, high = min(8, mtiles - band * 8);
  const int mt = band * 8 + in_band % high, nt = in_band / high;
  const long long m0 = (long long)mt * BM;
  const int n0 = nt * BN, mrows = (int)min((long long)BM, g.M - m0), nrows = min(BN, g.N - n0);

  const int chunk = (lane % 8) ^ (lane / 8);  // of the row whose chunk this lane brings (rows come eight at a time)
  unsigned vb[kLoadsB], va[kLoadsA];
#pragma unroll
  for (int i = 0; i < kLoadsB; ++i) vb[i] = (unsigned)(min((wave * kLoadsB + i) * 8 + lane / 8, nrows - 1) * g.ldb) + chunk * 16;
#pragma unroll
  for (int i = 0; i < kLoadsA; ++i) va[i] = (unsigned)(min((wave * kLoadsA + i) * 8 + lane / 8, mrows - 1) * g.lda) + chunk * 16;
  // the first waves bring the rows' scales, 64 each, the others the one or two of the columns (all to the same place)
  const bool rows_scales = wave < BM / kWave;
  const unsigned vs = rows_scales ? (unsigned)(min(wave * kWave + lane, mrows - 1) * (long long)g.kb * 4)
                                  : lane < (nrows - 1) / kScaleBlock + 1 ? (unsigned)(lane * g.kb * 4) : kOutside;
  const unsigned to_s = rows_scales ? L::kSa + wave * 256 : L::kSb;
  const uint8_t *pa = g.a + m0 * g.lda, *pb = g.b + (long long)n0 * g.ldb;
  const float* ps = rows_scales ? g.sa + m0 * g.kb : g.sb + (long long)(n0 / kScaleBlock) * g.kb;

  // The loads of block kb, kPer of them behind each row tile's matrix instructions.  Behind the last block they fetch nothing: the loop
  // over the blocks has no branch, across which the compiler would gather the scalings.
  constexpr bool kDeep = kMT * kNT <= 8;
  constexpr int kLoads = kLoadsB + kLoadsA + 1, kPer = kDeep ? (kLoads - 1) / kMT + 1 : (kLoads - 1) / (kMT - 1) + 1;
  static_assert(kPer * kMT >= kLoads, "all of a block's loads before its last row tile");
  auto request = [&](int step, unsigned stage, int from, int to) {
    const int kb = step * KG + group;
    const bool in = kb * kScaleBlock + chunk * 16 < g.K;
#pragma unroll
    for (int i = from; i < to; ++i) {
      if (i == 0) dma4(bytes_of(ps + kb, 0x7fffffff), kb < g.kb ? vs : kOutside, 0, stage + to_s);
      else if (i <= kLoadsB)
        dma16(bytes_of(pb + kb * kScaleBlock, 0x7fffffff), in ? vb[i - 1] : kOutside, 0, stage + L::kB + (wave * kLoadsB + i - 1) * 1024);
      else if (i < kLoads)
        dma16(bytes_of(pa + kb * kScaleBlock, 0x7fffffff), in ? va[i - 1 - kLoadsB] : kOutside, 0,
              stage + L::kA + (wave * kLoadsA + i - 1 - kLoadsB) * 1024);
    }
  };

  const int wm = wave % (BM / WM) * WM, wn = wave / (BM / WM) * WN;
  const unsigned frag = (unsigned)(r16 * kScaleBlock + ((quarter ^ (lane & 7)) << 4));
  auto operand = [&](const uint8_t* at) {
    return join(*reinterpret_cast<const tok_u4*>(at + frag), *reinterpret_cast<const tok_u4*>(at + (frag ^ 64)));
  };
  float acc[kNT][kMT][4];  // (plain floats: as vectors the compiler moves them about in fours)
  f32x4 p[kNT];
  float f = 0.f;
#pragma unroll
  for (int i = 0; i < kNT; ++i) {
#pragma unroll
    for (int j = 0; j < kMT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i][j][e] = 0.f;
    p[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  if constexpr (kDeep) {
    // Few row tiles a wave: all of a block's operands are in registers, and the next block's come from LDS behind the barrier, while
    // this one is multiplied.
    struct Operands {
      i32x8 n[kNT], m[kMT];
      float s[kMT], sb;
    };
    auto read = [&](Operands& o, const uint8_t* at) {
      o.sb = *reinterpret_cast<const float*>(at + L::kSb + wn / kScaleBlock * 4);
#pragma unroll
      for (int i = 0; i < kNT; ++i) o.n[i] = operand(at + L::kB + (wn + i * 16) * kScaleBlock);
#pragma unroll
      for (int j = 0; j < kMT; ++j) {
        o.s[j] = *reinterpret_cast<const float*>(at + L::kSa + (wm + j * 16 + r16) * 4);
        o.m[j] = operand(at + L::kA + (wm + j * 16) * kScaleBlock);
      }
    };
    int now = 0;
    auto step = [&](int kb, const Operands& o, Operands& ahead) {
      const int next = now + 1 < NS ? now + 1 : 0;
      lds_wait();
      vm_wait<(NS - 2) * kLoads>();
      __syncthreads();
      read(ahead, stages + next * L::kStage);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < kMT; ++j) {
        const float f_old = f;
        f = o.sb * o.s[j];
        request(kb + NS, lds0 + now * L::kStage, j * kPer, (j + 1) * kPer);
#pragma unroll
        for (int i = 0; i < kNT; ++i) {
          const f32x4 old = p[i];
          p[i] = mma_block(o.n[i], o.m[j]);
          __builtin_amdgcn_sched_barrier(0);
          float(&c)[4] = acc[i][(j + kMT - 1) % kMT];
#pragma unroll
          for (int e = 0; e < 4; ++e) c[e] = fmaf(old[e], f_old, c[e]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      now = next;
    };
#pragma unroll
    for (int s = 0; s < NS; ++s) request(s, lds0 + s * L::kStage, 0, kLoads);
    vm_wait<(NS - 1) * kLoads>();
    __syncthreads();
    Operands even, odd;
    read(even, stages);
    for (int kb = 0; kb * KG < g.kb; kb += 2) {  // (past the last block: zeros)
      step(kb, even, odd);
      step(kb + 1, odd, even);
    }
  } else {
    i32x8 nf[kNT];
    tok_u4 mf[2];  // the two halves of a row tile's operand
    bf16x8 n8[kNT][4];
    float s[2], sb;
    auto read_s = [&](const uint8_t* at, int j) { s[j & 1] = *reinterpret_cast<const float*>(at + L::kSa + (wm + j * 16 + r16) * 4); };
    auto read_m = [&](const uint8_t* at, int j, int half) {
      mf[half] = *reinterpret_cast<const tok_u4*>(at + L::kA + (wm + j * 16) * kScaleBlock + (half ? frag ^ 64 : frag));
    };
    auto read_n = [&](const uint8_t* at, int i) { nf[i] = operand(at + L::kB + (wn + i * 16) * kScaleBlock); };
    auto read_sb = [&](const uint8_t* at) { sb = *reinterpret_cast<const float*>(at + L::kSb + wn / kScaleBlock * 4); };
#pragma unroll
    for (int s = 0; s < NS - 1; ++s) request(s, lds0 + s * L::kStage, 0, kLoads);
    vm_wait<(NS - 2) * kLoads>();
    __syncthreads();
    request(NS - 1, lds0 + (NS - 1) * L::kStage, 0, kPer);
    read_m(stages, 0, 0);
    read_m(stages, 0, 1);
    read_s(stages, 0);
    read_sb(stages);
#pragma unroll
    for (int i = 0; i < kNT; ++i) read_n(stages, i);
    // The column tiles' operands stay in registers, widened, for the block; a row tile's is widened a quarter at a time, each time
    // for all column tiles (with a tile's four instructions one behind the other both were held whole: 23 registers in memory at
    // 256 x 256, 4096 x 4096 x 4096 149 us against 104).  A product's scaling stands behind the matrix instructions of the next row
    // tile (in the last of a block: of the next block's first), in this order and no other: a result is there long before it is
    // asked for.  The barrier stands in front of a block's last row tile, whose operands have been read by then: behind it the next
    // block's first ones come from LDS, and the loads of the block after that may overwrite this one's stage.  (Behind the last block
    // it reads what is there, unused.)
    int now = 0, fill = NS - 1;  // stages of this block and of the one being requested
    for (int kb = 0; kb * KG < g.kb; ++kb) {
      const int next = now + 1 < NS ? now + 1 : 0;
      const uint8_t *at = stages + now * L::kStage, *ahead = stages + next * L::kStage;
#pragma unroll
      for (int j = 0; j < kMT; ++j) {
        const float f_old = f;
        f = sb * s[j & 1];
        if (j == kMT - 1) {
          lds_wait();
          vm_wait<(NS - 2) * kLoads>();
          __syncthreads();
          read_s(ahead, 0);
          read_sb(ahead);
          fill = now;
          request(kb + NS, lds0 + fill * L::kStage, 0, kPer);
        } else {
          request(kb + NS - 1, lds0 + fill * L::kStage, (j + 1) * kPer, (j + 2) * kPer);
          read_s(at, j + 1);
        }
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          const bf16x8 m8 = widen8(mf[h / 2][h % 2 * 2], mf[h / 2][h % 2 * 2 + 1]);
#pragma unroll
          for (int i = 0; i < kNT; ++i) {
            if (j == 0) n8[i][h] = widen8((unsigned)nf[i][2 * h], (unsigned)nf[i][2 * h + 1]);
            if (h == 0) {
              float(&c)[4] = acc[i][(j + kMT - 1) % kMT];
#pragma unroll
              for (int e = 0; e < 4; ++e) c[e] = fmaf(p[i][e], f_old, c[e]);
              p[i] = mma_bf16_16(n8[i][h], m8, f32x4{0.f, 0.f, 0.f, 0.f});
            } else {
              p[i] = mma_bf16_16(n8[i][h], m8, p[i]);
            }
            __builtin_amdgcn_sched_barrier(0);
            if (i == 0 && h % 2 == 1) {
              if (j == kMT - 1) read_m(ahead, 0, h / 2);
              else read_m(at, j + 1, h / 2);
            }
            if (j == kMT - 1 && h == 3) read_n(ahead, i);
            if (h == 0 && i == 0) __builtin_amdgcn_s_setprio(1);
            if (h == 3 && i == kNT - 1) __builtin_amdgcn_s_setprio(0);
          }
        }
      }
      now = next;
    }
  }
  vm_wait<0>();  // (no load into LDS is left behind)
#pragma unroll
  for (int i = 0; i < kNT; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[i][kMT - 1][e] = fmaf(p[i][e], f, acc[i][kMT - 1][e]);
  if constexpr (KG > 1) {  // the other groups' sums through LDS to the first, in their order
    static_assert((KG - 1) * BM * BN * 4 <= L::kBytes, "sums fit");
    constexpr int kTile = BM * BN / 4;  // in f32x4
    f32x4* const sums = reinterpret_cast<f32x4*>(lds) + threadIdx.x % (kWaves * kWave);
    __syncthreads();
    if (group != 0) {
#pragma unroll
      for (int i = 0; i < kNT; ++i)
#pragma unroll
        for (int j = 0; j < kMT; ++j)
          sums[(group - 1) * kTile + (i * kMT + j) * kWaves * kWave] = f32x4{acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
    }
    __syncthreads();
    if (group != 0) return;
#pragma unroll
    for (int o = 0; o < KG - 1; ++o)
#pragma unroll
      for (int i = 0; i < kNT; ++i)
#pragma unroll
        for (int j = 0; j < kMT; ++j) {
          const f32x4 v = sums[o * kTile + (i * kMT + j) * kWaves * kWave];
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][j][e] += v[e];
        }
  }
  // Lane (row r16 of a, quarter) holds columns 4 * quarter .. +3 of every 16: after a swap of neighbouring quarters between two
  // column tiles it holds eight in a row, and four lanes 64 bytes of a row of bf16 results.
#pragma unroll
  for (int j = 0; j < kMT; ++j) {
    const int m = wm + j * 16 + r16;
    OT* out = reinterpret_cast<OT*>(g.out) + (m0 + m) * g.ldo + n0;
#pragma unroll
    for (int i = 0; i < kNT; i += 2) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(acc[i][j][e]), __float_as_uint(acc[i + 1][j][e]), false, false);
        v[e] = __uint_as_float(r[0]);
        v[4 + e] = __uint_as_float(r[1]);
      }
      const int n = wn + (i + quarter % 2) * 16 + quarter / 2 * 8;
      if (m < mrows && n < nrows) {
        piece8<OT> q;
        q.put(v);
        q.store(out + n, 0);
      }
    }
  }
}

inline double tile_count(const Mm8Args& g, int bm, int bn) { return (double)((g.M - 1) / bm + 1) * ((g.N - 1) / bn + 1); }

template <typename OT, int BM, int BN, int WM, int WN, int NS, int KG = 1>
int ask_tile_lds() {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(&k_mm8_tile<OT, BM, BN, WM, WN, NS, KG>), hipFuncAttributeMaxDynamicSharedMemorySize,
                             TileLds<BM, BN, NS, KG>::kBytes) == hipSuccess ? LAUD_OK : LAUD_ERR_HIP;
}
template <typename OT, int BM, int BN, int WM, int WN, int NS, int KG = 1>
int launch_tile(const Mm8Args& g, hipStream_t st) {
  constexpr int kThreads = KG * BM / WM * (BN / WN) * kWave;
  if (!launchable(tile_count(g, BM, BN) + 7, kThreads)) return LAUD_ERR_UNSUPPORTED;  // (so that their number is an int's)
  if (matmul8_init_device() != LAUD_OK) return LAUD_ERR_HIP;
  const int mtiles = (g.M - 1) / BM + 1, ntiles = (g.N - 1) / BN + 1;
  hipLaunchKernelGGL((k_mm8_tile<OT, BM, BN, WM, WN, NS, KG>), dim3((unsigned)((mtiles * ntiles + 7) / 8 * 8)), dim3(kThreads),
                     (TileLds<BM, BN, NS, KG>::kBytes), st, g, mtiles, ntiles);
  return check_launch();
}

// Which tile: a launch takes rounds of one tile a compute unit, a round the blocks of K times the tile's time for one and its two
// ends, in us.  Launches as measured, in us; the rule takes the least, or one within 3 % of it:
//   bf16 results         64 x 64   64 x 128   128 x 128   128 x 256   256 x 256     float32   64 x 64   64 x 128   128 x 128
//    256 x 4096 x 4096     17.1       22.0        29.7        53.5        91.3                  17.8       22.8        42.9
//    512 x 4096 x 4096     32.4       24.1        31.2        53.9        91.8                  32.9       25.3        43.4
//   1024 x 4096 x 4096     62.6       46.2        34.4        55.2        91.7                  61.2       47.2        46.5
//   2048 x 4096 x 4096    119.4       87.4        66.3        61.8        94.0                 119.0       89.8        89.0
//   4096 x 4096 x 4096    229.6      169.5       124.4       117.7       104.8                 235.6      180.5       173.7
//   1003 x 2120 x 2000     28.6       26.8        18.2        29.7        49.3                  29.9       27.9        25.3
//   3000 x 1000 x  512     11.3       11.8         8.4        10.8        16.4                  13.1       14.2        11.9
//   4000 x 4008 x  272     52.8       44.3        31.3        22.0        19.1
// The smaller ones share the blocks of K between two groups of waves (128 x 128 for bf16 results only), and short reductions on
// 64 x 64 tiles take two stages instead of four, two workgroups a compute unit (197 x 2048 x 1024).
// Where there is a compute unit for each, tiles are 64 x 32: two groups of waves and two stages up to 12 blocks of K, four and three
// beyond.  64 x 64 and these two, float32 results (bf16 ones take 0 to 0.5 us less):
//   64 x 4096 x  512      4.7,  3.9,  5.2         197 x 2048 x 1024     6.1,  5.0,  5.4
//   64 x 4096 x 2048      9.7,  7.3,  6.9          64 x 4096 x 8192    27.2, 25.2, 16.7
// and with two tiles a compute unit, 128 x 8192 x 2048, 10.7, 11.1, 14.2.
struct TileTime {
  int bm, bn;
  float block, ends;
};
inline float tile_time(const Mm8Args& g, const TileTime& t) {
  return (float)(std::ceil(tile_count(g, t.bm, t.bn) / kComputeUnits) * (g.kb * t.block + t.ends));
}

template <typename OT>
int launch_mm8(const Mm8Args& g, hipStream_t st) {
  if (g.M <= kSplitRows) {
    const int ntiles = (g.N - 1) / 16 + 1;
    if (!launchable(ntiles, kSplit * kWave)) return LAUD_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((k_mm8_split<OT>), dim3(ntiles), dim3(kSplit * kWave), kSplit * kWave * sizeof(f32x4), st, g);
    return check_launch();
  }
  constexpr bool kBf16 = sizeof(OT) == 2;
  constexpr TileTime kTimes[5] = {{64, 64, 0.45f, 2.0f}, {64, 128, 0.61f, 3.4f},
                                  {128, 128, kBf16 ? 0.93f : 1.18f, kBf16 ? 4.2f : 6.2f}, {128, 256, 1.66f, 5.5f}, {256, 256, 2.9f, 10.6f}};
  int best = 0;
  for (int i = 1; i < (kBf16 ? 5 : 3); ++i)
    if (tile_time(g, kTimes[i]) < tile_time(g, kTimes[best])) best = i;
  if constexpr (kBf16) {
    if (best == 4) return launch_tile<OT, 256, 256, 128, 64, 2>(g, st);
    if (best == 3) return launch_tile<OT, 128, 256, 64, 64, 3>(g, st);
    if (best == 2) return launch_tile<OT, 128, 128, 64, 64, 2, 2>(g, st);
  } else {
    if (best == 2) return launch_tile<OT, 128, 128, 64, 64, 4>(g, st);
  }
  if (best == 1) return launch_tile<OT, 64, 128, 32, 64, 3, 2>(g, st);
  if (tile_count(g, 64, 32) <= kComputeUnits) {
    if (g.kb <= 12) return launch_tile<OT, 64, 32, 32, 32, 2, 2>(g, st);
    return launch_tile<OT, 64, 32, 32, 32, 3, 4>(g, st);
  }
  if (g.kb <= 10) return launch_tile<OT, 64, 64, 32, 32, 2, 2>(g, st);
  return launch_tile<OT, 64, 64, 32, 32, 4, 2>(g, st);
}

int matmul8_init_device() {
  static std::atomic<unsigned> done{0};  // one bit per device ordinal (ordinals >= 32 repeat the request)
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return LAUD_ERR_HIP;
  const unsigned bit = dev >= 0 && dev < 32 ? 1u << dev : 0u;
  if (bit && (done.load(std::memory_order_acquire) & bit)) return LAUD_OK;
  for (int rc : {ask_tile_lds<bf16_t, 256, 256, 128, 64, 2>(), ask_tile_lds<bf16_t, 128, 256, 64, 64, 3>(),
                 ask_tile_lds<bf16_t, 128, 128, 64, 64, 2, 2>(), ask_tile_lds<bf16_t, 64, 128, 32, 64, 3, 2>(),
                 ask_tile_lds<bf16_t, 64, 64, 32, 32, 2, 2>(), ask_tile_lds<bf16_t, 64, 64, 32, 32, 4, 2>(),
                 ask_tile_lds<bf16_t, 64, 32, 32, 32, 2, 2>(), ask_tile_lds<bf16_t, 64, 32, 32, 32, 3, 4>(),
                 ask_tile_lds<float, 64, 32, 32, 32, 2, 2>(), ask_tile_lds<float, 64, 32, 32, 32, 3, 4>(),
                 ask_tile_lds<float, 128, 128, 64, 64, 4>(), ask_tile_lds<float, 64, 128, 32, 64, 3, 2>(),
                 ask_tile_lds<float, 64, 64, 32, 32, 2, 2>(), ask_tile_lds<float, 64, 64, 32, 32, 4, 2>()})
    if (rc != LAUD_OK) return rc;
  done.fetch_or(bit, std::memory_order_release);
  return LAUD_OK;
}

}  // namespace laud

extern "C" size_t laud_matmul_e4m3_workspace(int M, int N, int K) {
  (void)M; (void)N; (void)K;
  return 0;
}

extern "C" int laud_matmul_e4m3(const void* a, int64_t lda, const float* sa, const void* b, int64_t ldb, const float* sb, int M, int N,
                                int K, void* out, int64_t ldo, int out_dtype, void* ws, size_t ws_bytes, void* stream) {
  using namespace laud;
  (void)ws; (void)ws_bytes;
  if (M < 0 || N <= 0 || K <= 0 || !float_type(out_dtype)) return LAUD_ERR_INVALID_ARG;
  if (N % 8 || K % 16) return LAUD_ERR_UNSUPPORTED;
  if (M == 0) return LAUD_OK;
  if (!a || !sa || !b || !sb || !out || !good_ld(lda, K, 16) || !good_ld(ldb, K, 16) || !good_ld(ldo, N, 8)) return LAUD_ERR_INVALID_ARG;
  if (!aligned16(a) || !aligned16(b) || !aligned16(out)) return LAUD_ERR_INVALID_ARG;
  if (lda > kMaxLd || ldb > kMaxLd) return LAUD_ERR_UNSUPPORTED;
  const size_t ob = span_bytes(M, ldo, N, elem_bytes(out_dtype));
  if (ranges_meet(a, span_bytes(M, lda, K, 1), out, ob) || ranges_meet(b, span_bytes(N, ldb, K, 1), out, ob)) return LAUD_ERR_INVALID_ARG;
  const size_t kb = (size_t)scale_blocks(K) * 4, eb = elem_bytes(out_dtype);
  if (range_meets_rows(sa, M * kb, out, ldo, eb, M, N) || range_meets_rows(sb, scale_blocks(N) * kb, out, ldo, eb, M, N))
    return LAUD_ERR_INVALID_ARG;
  Mm8Args g{(const uint8_t*)a, (const uint8_t*)b, sa, sb, out, M, N, K, scale_blocks(K), lda, ldb, ldo};
  clear_stale_error();
  return out_dtype == LAUD_BF16 ? launch_mm8<bf16_t>(g, (hipStream_t)stream) : launch_mm8<float>(g, (hipStream_t)stream);
}
