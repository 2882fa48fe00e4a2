// Mixture-of-experts layer for a few tokens: routing, the chosen experts' two products, the weighted sum.
#include "laud_token.h"

namespace laud {
namespace {

constexpr int kMaxExperts = 1024, kMaxTopK = 32;

struct MoeArgs {
  int T, C, F, E, top_k, renormalise;
  int Fp;               // F rounded up to whole blocks of 128
  float scale;
  const void *x, *router, *up, *down;
  const float *s_up, *s_down;
  const uint8_t* keep;
  void* out;
  int64_t ldx, ldo;
  int32_t* experts;     // [T][top_k], the caller's or the workspace's
  float* weights;       // [T][top_k]
  void* h;              // [T * top_k][Fp] float32, or three planes of it in bf16 (by_token)
  int by_token;         // the last product is k_moe_down_few's
  float* y;             // [T * top_k][C]: an entry's weighted result
  float* logits;        // [E], of a single token
};

constexpr int kColumns = 32;  // output channels of a workgroup of the last product

// ---- routing ----------------------------------------------------------------------------------------------------------------
// Floats as unsigned integers in their order; a NaN lies below all.
__device__ __forceinline__ unsigned order_key(float f) {
  const unsigned u = __float_as_uint(f);
  return f != f ? 0u : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

constexpr int kRouteThreads = 1024, kLogitWaves = 4;

// The logits of N experts from e0 on, by one wave, D pieces of 16 bytes a lane of every row at a time, whose loads are all under way
// together (one piece of each row at a time: one token through 2 of 8 experts of 4096 x 2048, bf16, 33.3 us against 30.3).
template <typename ET, int N, int D>
__device__ __forceinline__ void router_logits(const MoeArgs& a, const ET* x, int e0, float* logits) {
  const int lane = lane_id();
  constexpr int kElems = 16 / (int)sizeof(ET);
  const long long row_bytes = (long long)a.C * (int)sizeof(ET);
  const __amdgpu_buffer_rsrc_t rx = bytes_of(x, row_bytes);  // (behind its end: zeros)
  float s[N] = {};
  for (int u0 = 0; u0 < a.C / kElems; u0 += kWave * D) {
    tok_u4 p[D], q[N][D];
#pragma unroll
    for (int d = 0; d < D; ++d) {
      const unsigned off = (unsigned)(u0 + d * kWave + lane) * 16;
      p[d] = load16(rx, off);
#pragma unroll
      for (int i = 0; i < N; ++i)
        q[i][d] = load16(bytes_of(reinterpret_cast<const ET*>(a.router) + (long long)min(e0 + i, a.E - 1) * a.C, row_bytes), off);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int d = 0; d < D; ++d)
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          if constexpr (sizeof(ET) == 4) {
            s[i] = fmaf(__uint_as_float(p[d][u]), __uint_as_float(q[i][d][u]), s[i]);
          } else {
            s[i] = fmaf(__uint_as_float(p[d][u] << 16), __uint_as_float(q[i][d][u] << 16), s[i]);
            s[i] = fmaf(__uint_as_float(p[d][u] & 0xffff0000u), __uint_as_float(q[i][d][u] & 0xffff0000u), s[i]);
          }
        }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    s[i] = lanes64_sum(s[i]);
    if (lane == 0 && e0 + i < a.E) logits[e0 + i] = s[i];
  }
}

// The choice of one token by a workgroup of THREADS from logits [E] in LDS, and its weights: an expert is chosen if fewer than top_k
// come before it, and sixteen lanes count those of one expert.  The first wave writes both.
template <int THREADS>
__device__ __forceinline__ void choose_experts(const MoeArgs& a, const float* logits, uint8_t* chosen, int32_t* experts, float* weights) {
  const int lane = lane_id(), E = a.E;
  for (int e0 = 0; e0 < E; e0 += THREADS / 16) {
    const int e = e0 + (int)threadIdx.x / 16;
    if (e >= E) continue;  // (sixteen lanes at a time)
    const unsigned key = order_key(logits[e]);
    int before = 0;
    for (int j = (int)threadIdx.x % 16; j < E; j += 16) {
      const unsigned k = order_key(logits[j]);
      before += k > key || (k == key && j < e);
    }
    const float n = lanes16_sum((float)before);
    if (threadIdx.x % 16 == 0) chosen[e] = n < (float)a.top_k;
  }
  __syncthreads();
  if ((int)threadIdx.x >= kWave) return;
  float top = -INFINITY;
  for (int e = lane; e < E; e += kWave) top = fmaxf(top, logits[e]);
  {
    const unsigned k = lanes64_max(order_key(top));
    top = __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k);
  }
  float sum = 0.f;
  for (int e = lane; e < E; e += kWave) {
    const float p = expf(logits[e] - top);
    if (!a.renormalise || chosen[e] || p != p) sum += p;  // (a NaN anywhere is in every softmax value)
  }
  sum = lanes64_sum(sum);
  int before = 0;
  for (int e0 = 0; e0 < E; e0 += kWave) {
    const bool mine = e0 + lane < E && chosen[e0 + lane];
    const unsigned long long b = __ballot(mine);
    if (mine) {
      const int at = before + ballot_prefix(b);
      experts[at] = e0 + lane;
      weights[at] = expf(logits[e0 + lane] - top) / sum * a.scale;
    }
    before += __popcll(b);
  }
}

// One workgroup a token.
template <typename ET>
__global__ __launch_bounds__(kRouteThreads) void k_moe_route(MoeArgs a) {
  __shared__ float logits[kMaxExperts];
  __shared__ uint8_t chosen[kMaxExperts];
  const int t = blockIdx.x, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  int32_t* experts = a.experts + (long long)t * a.top_k;
  float* weights = a.weights + (long long)t * a.top_k;
  if (a.keep && a.keep[t] == 0) {
    if ((int)threadIdx.x < a.top_k) { experts[threadIdx.x] = -1; weights[threadIdx.x] = 0.f; }
    return;
  }
  constexpr int kAtOnce = 4;  // experts a wave takes at a time, so that their loads are under way together
  for (int e0 = wave * kAtOnce; e0 < a.E; e0 += kRouteThreads / kWave * kAtOnce)
    router_logits<ET, kAtOnce, 4>(a, reinterpret_cast<const ET*>(a.x) + t * a.ldx, e0, logits);
  __syncthreads();
  choose_experts<kRouteThreads>(a, logits, chosen, experts, weights);
}

// A single token's logits, an expert a wave over many workgroups, where one workgroup would wait for its share of the memory's rate;
// the workgroups of the first product then choose, each for itself.  (One token, 8 of 64 experts of 2048 x 1024, bf16:
// 28.9 us against 31.3 routed by one workgroup.)
template <typename ET>
__global__ __launch_bounds__(kLogitWaves * kWave) void k_moe_logits(MoeArgs a) {
  const int e = blockIdx.x * kLogitWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  if (e < a.E && !(a.keep && a.keep[0] == 0)) router_logits<ET, 1, 8>(a, reinterpret_cast<const ET*>(a.x), e, a.logits);
}

// ---- products -----------------------------------------------------------------------------------------------------------------
// The matrix instructions take sixteen rows of weights and sixteen token rows; lane l holds a piece of row l % 16 of both.
// W: how the experts' weights are stored.  A block of 128 along the reduction is kPieces pieces of 16 bytes a lane; the elements
// of piece p start at first(p, l / 16), and the token side reads the same ones.
enum { W_BF16, W_F32, W_E4M3 };
template <int W> struct Weights {
  static constexpr int kBytes = W == W_BF16 ? 2 : W == W_F32 ? 4 : 1;
  static constexpr int kElems = 16 / kBytes;
  static constexpr int kPieces = 128 * kBytes / 64;
  __device__ static __forceinline__ int first(int p, int quarter) { return (p * 4 + quarter) * kElems; }
};

// c += one piece of weights times the token values of the same elements: x (bf16 or float32, as stored) ...
template <int W>
__device__ __forceinline__ f32x4 mma_stored(const tok_u4& w, const tok_u4 (&x)[W == W_E4M3 ? 2 : 1], f32x4 c) {
  if constexpr (W == W_BF16) {
    return mma_bf16_16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x[0]), c);
  } else if constexpr (W == W_F32) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[i]), __uint_as_float(x[0][i]), c, 0, 0, 0);
    return c;
  } else {
    c = mma_bf16_16(widen8(w[0], w[1]), __builtin_bit_cast(bf16x8, x[0]), c);
    return mma_bf16_16(widen8(w[2], w[3]), __builtin_bit_cast(bf16x8, x[1]), c);
  }
}
// Hidden values are float32.  Through bf16 instructions they go as a sum of three: the eight leading bits (not rounded: a finite value
// stays finite), the eight behind them and the rest, which hold all 24 (rounded to bf16 alone they would add an error as large as
// the result's own rounding, in two parts one of 2^-17 of theirs).  k_moe_down splits them in registers, beside its loads of weights
// (three planes read instead: 64 tokens 187.6 us against 178.7); k_moe_down_few, whose lanes hold a part each, finds them split in
// three planes (split there: one token 34.9 us against 29.5).  Where
// the leading parts' sum is infinite or NaN it is the result: an infinite weight times a part that is zero, or the parts behind an
// infinity, are none of the formula's.
__device__ __forceinline__ unsigned leading(float a, float b) {  // of two values, as two bf16
  return (__float_as_uint(a) >> 16) | (__float_as_uint(b) & 0xffff0000u);
}
__device__ __forceinline__ float behind(float a) { return a - __uint_as_float(__float_as_uint(a) & 0xffff0000u); }
__device__ __forceinline__ void split8(const tok_u4& x, const tok_u4& y, bf16x8 (&part)[3]) {
  float f[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(e < 4 ? x[e] : y[e - 4]);
#pragma unroll
  for (int n = 0; n < 3; ++n) {
    tok_u4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = leading(f[2 * e], f[2 * e + 1]);
      f[2 * e] = behind(f[2 * e]);
      f[2 * e + 1] = behind(f[2 * e + 1]);
    }
    part[n] = __builtin_bit_cast(bf16x8, v);
  }
}
__device__ __forceinline__ float joined(float lead, float rest) { return fabsf(lead) < INFINITY ? lead + rest : lead; }
template <int W> constexpr int kHiddenParts = W == W_F32 ? 1 : 3;
// Eight codes of a piece of weights (of bf16 ones: all of it).
template <int W>
__device__ __forceinline__ bf16x8 eight(const tok_u4& w, int g) {
  if constexpr (W == W_E4M3) return widen8(w[2 * g], w[2 * g + 1]);
  else return __builtin_bit_cast(bf16x8, w);
}

// The products run for (tile of channels, slot): a slot is an expert, or, where the entries (token, choice) are fewer than the
// experts, an entry, whose workgroups take its expert if no earlier entry has the same.
struct Slot {
  int expert, entries;
  bool by_entry;
};
__device__ __forceinline__ Slot slot_of(const MoeArgs& a) {
  Slot s;
  s.entries = a.T * a.top_k;
  s.by_entry = s.entries < a.E;
  s.expert = s.by_entry ? a.experts[blockIdx.y] : (int)blockIdx.y;
  return s;
}
// The slot's entries in `list` (in any order: no entry's value depends on it) and their number, 0 if it has none or an earlier slot
// has its expert.  Called by a whole workgroup.
__device__ __forceinline__ int find_entries(const MoeArgs& a, const Slot& s, int* list, int* counts) {
  if (threadIdx.x < 2) counts[threadIdx.x] = 0;
  __syncthreads();
  if (s.expert >= 0) {
    for (int i = threadIdx.x; i < s.entries; i += blockDim.x) {
      if (a.experts[i] != s.expert) continue;
      if (s.by_entry && i < (int)blockIdx.y) counts[1] = 1;
      list[atomicAdd(&counts[0], 1)] = i;
    }
  }
  __syncthreads();
  return counts[1] ? 0 : counts[0];
}

// Sums of the S waves' parts of N row tiles, in the waves' order, for the first wave.
template <int S, int N>
__device__ __forceinline__ void join_waves(f32x4 (&v)[N], f32x4 (*part)[N][kWave], int wave, int lane) {
#pragma unroll
  for (int n = 0; n < N; ++n) part[wave][n][lane] = v[n];
  __syncthreads();
  if (wave == 0) {
#pragma unroll
    for (int w = 1; w < S; ++w)
#pragma unroll
      for (int n = 0; n < N; ++n) v[n] += part[w][n][lane];
  }
  __syncthreads();
}

// Waves of a workgroup, which share the reduction by blocks of 128.  Few waves leave room for more workgroups, which wait for their
// entries, their weights and each other at different times (16 / 64 tokens, 8 of 64 experts of 2048 x 1024, bf16, eight / four / two
// waves: 156 / 143 / 153 and 189 / 179 / 189 us; 16 tokens, 6 of 64 of 2048 x 1424, 8 bits, 115 / 111 / 118); float32 blocks need the
// registers of the longer ones (32 tokens, 2 of 16 experts of 1024 x 1024, eight / four: 61.3 / 62.9).  A single token's workgroups,
// one or two a compute unit, have eight (29.9 against 31.1 us with four).
template <int W> constexpr int kSplit = W == W_F32 ? 8 : 4;
constexpr int kSplitOne = 8;

// h of one expert's entries for 16 hidden channels; ONE: of one entry of the single token.  Bound by memory: 64 experts of 2048 x 1024
// in bf16, 537 MB, in 108 us, 5.0 TB/s.
template <int W, bool ONE>
__global__ __launch_bounds__((ONE ? kSplitOne : kSplit<W>) * kWave) void k_moe_up(MoeArgs a) {
  typedef Weights<W> WT;
  constexpr int S = ONE ? kSplitOne : kSplit<W>, kXP = W == W_E4M3 ? 2 : 1, xb = W == W_F32 ? 4 : 2;
  __shared__ int list[LAUD_MOE_MAX_TOKENS], counts[2];
  __shared__ f32x4 part[S][2][kWave];
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), r16 = lane % 16, quarter = lane / 16;
  Slot slot;
  if constexpr (ONE) {
    __shared__ float logits[kMaxExperts], weights[kMaxTopK];
    __shared__ uint8_t chosen[kMaxExperts];
    const bool dropped = a.keep && a.keep[0] == 0;
    if (!dropped) {
      for (int e = threadIdx.x; e < a.E; e += S * kWave) logits[e] = a.logits[e];
      __syncthreads();
      choose_experts<S * kWave>(a, logits, chosen, list, weights);
      __syncthreads();
    }
    if (blockIdx.x == 0 && blockIdx.y == 0 && (int)threadIdx.x < a.top_k) {
      a.experts[threadIdx.x] = dropped ? -1 : list[threadIdx.x];
      a.weights[threadIdx.x] = dropped ? 0.f : weights[threadIdx.x];
    }
    if (dropped) return;
    slot.expert = __builtin_amdgcn_readfirstlane(list[blockIdx.y]);
  } else {
    slot = slot_of(a);
  }
  const int f0 = blockIdx.x * 16, rows = min(16, a.F - f0);  // (from F to the end of its block of 128 h is 0: rows may be none)
  const int kb_all = scale_blocks(a.C);
  const long long row_bytes = (long long)a.C * WT::kBytes;
  const uint8_t* base = reinterpret_cast<const uint8_t*>(a.up) + ((long long)max(slot.expert, 0) * 2 * a.F + f0) * row_bytes;
  const __amdgpu_buffer_rsrc_t rg = bytes_of(base, max(rows, 0) * row_bytes);
  const __amdgpu_buffer_rsrc_t ru = bytes_of(base + a.F * row_bytes, max(rows, 0) * row_bytes);
  tok_u4 wg[WT::kPieces], wu[WT::kPieces];
  auto request = [&](int kb) {
#pragma unroll
    for (int p = 0; p < WT::kPieces; ++p) {
      const int k = kb * kScaleBlock + WT::first(p, quarter);
      const unsigned off = k < a.C && r16 < rows ? (unsigned)(r16 * row_bytes) + (unsigned)k * WT::kBytes : kOutside;
      wg[p] = load16(rg, off);
      wu[p] = load16(ru, off);
    }
  };
  const int len = ONE ? 1 : find_entries(a, slot, list, counts);
  if (len == 0) return;
  const __amdgpu_buffer_rsrc_t rx = bytes_of(a.x, ((a.T - 1) * a.ldx + a.C) * xb);
  const int fb = scale_blocks(a.F);
  const float* s = W == W_E4M3 && rows > 0 ? a.s_up + ((long long)slot.expert * 2 * fb + f0 / kScaleBlock) * kb_all : nullptr;
  for (int l0 = 0; l0 < len; l0 += 16) {
    const int entry = ONE ? (int)blockIdx.y : list[min(l0 + r16, len - 1)];
    const bool real = l0 + r16 < len;  // (of the other rows nothing is fetched)
    const unsigned xoff = (unsigned)(entry / a.top_k * a.ldx * xb);
    f32x4 v[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    for (int kb = wave; kb < kb_all; kb += S) {
      request(kb);
      const float fg = s ? s[kb] : 1.f, fu = s ? s[fb * kb_all + kb] : 1.f;
      tok_u4 x[WT::kPieces][kXP];
#pragma unroll
      for (int p = 0; p < WT::kPieces; ++p) {
        const int k = kb * kScaleBlock + WT::first(p, quarter);
#pragma unroll
        for (int i = 0; i < kXP; ++i) x[p][i] = load16(rx, k < a.C && real ? xoff + (unsigned)(k + 8 * i) * xb : kOutside);
      }
      __builtin_amdgcn_sched_barrier(0);  // (all loads are under way before the first product waits for one)
      f32x4 pg = {0.f, 0.f, 0.f, 0.f}, pu = pg;
#pragma unroll
      for (int p = 0; p < WT::kPieces; ++p) {
        pg = mma_stored<W>(wg[p], x[p], pg);
        pu = mma_stored<W>(wu[p], x[p], pu);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[0][i] = fmaf(pg[i], fg, v[0][i]);
        v[1][i] = fmaf(pu[i], fu, v[1][i]);
      }
    }
    join_waves<S>(v, part, wave, lane);
    if (wave == 0 && real) {
      f32x4 h;
#pragma unroll
      for (int i = 0; i < 4; ++i) h[i] = quarter * 4 < rows ? v[0][i] / (1.f + expf(-v[0][i])) * v[1][i] : 0.f;
      const long long at = (long long)entry * a.Fp + f0 + quarter * 4;
      if (W == W_F32 || !a.by_token) {
        *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(a.h) + at) = h;
      } else {
        bf16_t* plane = reinterpret_cast<bf16_t*>(a.h) + at;
#pragma unroll
        for (int n = 0; n < 3; ++n, plane += (long long)a.T * a.top_k * a.Fp) {
          *reinterpret_cast<tok_u2*>(plane) = tok_u2{leading(h[0], h[1]), leading(h[2], h[3])};
#pragma unroll
          for (int i = 0; i < 4; ++i) h[i] = behind(h[i]);
        }
      }
    }
  }
}

// One expert's entries for 32 output channels, weighted; k_moe_sum adds each token's entries up.  Bound by memory and, at two blocks of
// the reduction a wave, by a workgroup's start and end: 64 experts of 2048 x 1024 in bf16, 268 MB, in 65 us, 4.1 TB/s.
template <int W>
__global__ __launch_bounds__(kSplit<W> * kWave) void k_moe_down(MoeArgs a) {
  typedef Weights<W> WT;
  constexpr int N = kColumns / 16, S = kSplit<W>, kXP = WT::kElems / 4;
  __shared__ int list[LAUD_MOE_MAX_TOKENS], counts[2];
  __shared__ f32x4 part[S][N][kWave];
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), r16 = lane % 16, quarter = lane / 16;
  const Slot slot = slot_of(a);
  const int c0 = blockIdx.x * kColumns, rows = min(kColumns, a.C - c0);
  const int kb_all = scale_blocks(a.F);
  const long long row_bytes = (long long)a.F * WT::kBytes;
  const __amdgpu_buffer_rsrc_t rw =
      bytes_of(reinterpret_cast<const uint8_t*>(a.down) + ((long long)max(slot.expert, 0) * a.C + c0) * row_bytes, rows * row_bytes);
  tok_u4 w[N][WT::kPieces];
  auto request = [&](int kb) {
#pragma unroll
    for (int p = 0; p < WT::kPieces; ++p) {
      const int k = kb * kScaleBlock + WT::first(p, quarter);
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const int row = n * 16 + r16;
        w[n][p] = load16(rw, k < a.F && row < rows ? (unsigned)(row * row_bytes) + (unsigned)k * WT::kBytes : kOutside);
      }
    }
  };
  const int len = find_entries(a, slot, list, counts);
  if (len == 0) return;
  const __amdgpu_buffer_rsrc_t rh = bytes_of(a.h, (long long)a.T * a.top_k * a.Fp * 4);
  const float* s = W == W_E4M3 ? a.s_down + ((long long)slot.expert * scale_blocks(a.C) + c0 / kScaleBlock) * kb_all : nullptr;
  for (int l0 = 0; l0 < len; l0 += 16) {
    const int entry = list[min(l0 + r16, len - 1)];
    const bool real = l0 + r16 < len;
    const unsigned at = (unsigned)entry * (unsigned)a.Fp * 4;
    const float share = a.weights[entry];
    f32x4 v[N] = {};
    for (int kb = wave; kb < kb_all; kb += S) {
      request(kb);
      const float f = s ? s[kb] : 1.f;
      tok_u4 x[WT::kPieces][kXP];
#pragma unroll
      for (int p = 0; p < WT::kPieces; ++p) {
        const int k = kb * kScaleBlock + WT::first(p, quarter);
#pragma unroll
        for (int u = 0; u < kXP; ++u) x[p][u] = load16(rh, real ? at + (unsigned)(k + 4 * u) * 4 : kOutside);
      }
      __builtin_amdgcn_sched_barrier(0);  // (as above)
      f32x4 lead[N] = {}, rest[N] = {};
#pragma unroll
      for (int p = 0; p < WT::kPieces; ++p) {
        if constexpr (W == W_F32) {
#pragma unroll
          for (int n = 0; n < N; ++n) lead[n] = mma_stored<W>(w[n][p], x[p], lead[n]);
        } else {
#pragma unroll
          for (int g = 0; g < kXP / 2; ++g) {
            bf16x8 h[3];
            split8(x[p][2 * g], x[p][2 * g + 1], h);
#pragma unroll
            for (int n = 0; n < N; ++n) {
              const bf16x8 wv = eight<W>(w[n][p], g);
              lead[n] = mma_bf16_16(wv, h[0], lead[n]);
              rest[n] = mma_bf16_16(wv, h[1], rest[n]);
              rest[n] = mma_bf16_16(wv, h[2], rest[n]);
            }
          }
        }
      }
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[n][i] = fmaf(joined(lead[n][i], rest[n][i]), f, v[n][i]);
    }
    join_waves<S>(v, part, wave, lane);
    if (wave == 0 && real) {
      float* y = a.y + (long long)entry * a.C + c0;
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (i * 16 + quarter * 4 < rows) *reinterpret_cast<f32x4*>(y + i * 16 + quarter * 4) = v[i] * share;
    }
  }
}

// A token's entries, in the order of its experts: four channels a thread.  (A launch of its own costs less than a sum by the last of
// the workgroups of a tile of channels, each of which then waits for its stores and a count: 64 tokens 183.6 against 187.1 us.)
template <typename OT>
__global__ __launch_bounds__(256) void k_moe_sum(MoeArgs a) {
  const int t = blockIdx.y, c = ((int)blockIdx.x * 256 + (int)threadIdx.x) * 4;
  if (c >= a.C) return;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  if (!a.keep || a.keep[t] != 0) {
    const float* y = a.y + (long long)t * a.top_k * a.C + c;
#pragma unroll 8
    for (int j = 0; j < a.top_k; ++j) sum += *reinterpret_cast<const f32x4*>(y + (long long)j * a.C);
  }
  store4(reinterpret_cast<OT*>(a.out) + t * a.ldo + c, sum);
}

// One token's entries for 8 output channels, weighted and added up by one workgroup: where the entries are no more than the experts, so
// that tokens seldom share one, nothing is gained by joining theirs and nothing has to be handed from workgroup to workgroup.  All
// of a wave's loads are under way together.  The waves share the entries' blocks of the reduction, two at a time, as the two halves
// of a matrix instruction's sixteen rows of weights; of the token side, column 0 is the even block and column 1 the odd one, columns
// 2 to 5 the parts behind the leading ones of both; a half's results stand in its columns.  Sums are added in the waves' order.
// The layer, with k_moe_down / with this kernel, in us:
//   8 of 64 experts of 2048 x 1024, bf16    1 token 32.6 / 29.9    4 tokens 84.2 / 82.7    8 tokens 119.2 / 127.9    16 tokens 148.2 / 190.6
//   6 of 64 experts of 2048 x 1424, e4m3            27.0 / 22.3             62.7 / 57.5              88.0 /  86.9             111.3 / 126.4
//   2 of  8 experts of 4096 x 2048, bf16            34.3 / 29.6             74.1 / 73.9              91.3 / 105.4
//   2 of 16 experts of 1024 x 1024, float32                                 32.8 / 28.2              51.2 /  45.9              59.2 /  61.0
// (Two pairs of blocks at a time take 78 registers in bf16, four took 140 and leave room for one workgroup of 8 waves a compute unit
// instead of two: 54.6 against 62.5 us for two tokens of the last one.)
constexpr int kFewColumns = 8;
template <int W> constexpr int kPairs = W == W_F32 ? 1 : 2;  // pairs whose loads a wave has under way together
template <int W, typename OT, int S>
__global__ __launch_bounds__(S * kWave) void k_moe_down_few(MoeArgs a) {
  typedef Weights<W> WT;
  constexpr unsigned kHb = W == W_F32 ? 4 : 2;  // bytes of a hidden value in a plane
  constexpr int kXP = W == W_E4M3 ? 2 : 1, P = kHiddenParts<W>, kAtOnce = kPairs<W>;
  __shared__ f32x4 part[S][4][P];
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), r16 = lane % 16, quarter = lane / 16;
  const int t = blockIdx.y, c0 = blockIdx.x * kFewColumns;
  const int kb_all = scale_blocks(a.F), pairs = (kb_all + 1) / 2, items = a.keep && a.keep[t] == 0 ? 0 : a.top_k * pairs;
  const long long row_bytes = (long long)a.F * WT::kBytes;
  const unsigned plane = (unsigned)(a.T * a.top_k) * (unsigned)a.Fp * kHb;  // (three of them: below 2^32)
  const __amdgpu_buffer_rsrc_t rh = bytes_of(a.h, (long long)P * plane);
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = wave; i0 < items; i0 += S * kAtOnce) {
    tok_u4 w[kAtOnce][WT::kPieces], x[kAtOnce][WT::kPieces][kXP];
    int expert[kAtOnce], entry[kAtOnce], kb[kAtOnce];
    float f[kAtOnce];
    auto live = [&](int n) { return i0 + n * S < items; };  // (behind the last pair: zeros)
#pragma unroll
    for (int n = 0; n < kAtOnce; ++n) {
      const int i = min(i0 + n * S, items - 1);
      entry[n] = t * a.top_k + i / pairs;
      kb[n] = i % pairs * 2;
      expert[n] = a.experts[entry[n]];
    }
#pragma unroll
    for (int n = 0; n < kAtOnce; ++n) {
      const int e = __builtin_amdgcn_readfirstlane(expert[n]);
      const __amdgpu_buffer_rsrc_t rw =
          bytes_of(reinterpret_cast<const uint8_t*>(a.down) + ((long long)e * a.C + c0) * row_bytes, kFewColumns * row_bytes);
#pragma unroll
      for (int p = 0; p < WT::kPieces; ++p) {
        const int k = (kb[n] + r16 / 8) * kScaleBlock + WT::first(p, quarter);
        w[n][p] = load16(rw, k < a.F && live(n) ? (unsigned)(r16 % 8 * row_bytes) + (unsigned)k * WT::kBytes : kOutside);
      }
      f[n] = live(n) ? a.weights[entry[n]] : 0.f;
      if constexpr (W == W_E4M3) {
        const bool in = live(n) && kb[n] + quarter / 2 < kb_all;
        f[n] *= in ? a.s_down[((long long)e * scale_blocks(a.C) + c0 / kScaleBlock) * kb_all + kb[n] + quarter / 2] : 0.f;
      }
    }
#pragma unroll
    for (int n = 0; n < kAtOnce; ++n)
#pragma unroll
      for (int p = 0; p < WT::kPieces; ++p) {
        const unsigned k = (unsigned)((kb[n] + r16 % 2) * kScaleBlock + WT::first(p, quarter));
        const unsigned at = r16 / 2 * plane + ((unsigned)entry[n] * (unsigned)a.Fp + k) * kHb;
#pragma unroll
        for (int u = 0; u < kXP; ++u) x[n][p][u] = load16(rh, r16 < 2 * P && (int)k < a.Fp && live(n) ? at + 8 * u * kHb : kOutside);
      }
    __builtin_amdgcn_sched_barrier(0);  // (the loads stay in front of the products)
#pragma unroll
    for (int n = 0; n < kAtOnce; ++n) {
      f32x4 r = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int p = 0; p < WT::kPieces; ++p) r = mma_stored<W>(w[n][p], x[n][p], r);
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = fmaf(r[q], f[n], v[q]);
    }
  }
  if (r16 < 2 * P && r16 % 2 == quarter / 2) part[wave][quarter][r16 / 2] = v;
  __syncthreads();
  if ((int)threadIdx.x >= kFewColumns / 4) return;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f}, rest = sum;
#pragma unroll
  for (int n = 0; n < S; ++n) {
    sum += part[n][threadIdx.x][0] + part[n][threadIdx.x + 2][0];
#pragma unroll
    for (int p = 1; p < P; ++p) rest += part[n][threadIdx.x][p] + part[n][threadIdx.x + 2][p];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) sum[i] = joined(sum[i], rest[i]);
  store4(reinterpret_cast<OT*>(a.out) + t * a.ldo + c0 + threadIdx.x * 4, sum);
}

template <int W, typename ET>
void launch_moe(MoeArgs& a, hipStream_t st) {
  const long long entries = (long long)a.T * a.top_k;
  a.by_token = entries <= a.E;
  const dim3 up(a.Fp / 16, (unsigned)std::min((long long)a.E, entries));
  if (a.T == 1) {
    hipLaunchKernelGGL((k_moe_logits<ET>), dim3((a.E - 1) / kLogitWaves + 1), dim3(kLogitWaves * kWave), 0, st, a);
    hipLaunchKernelGGL((k_moe_up<W, true>), up, dim3(kSplitOne * kWave), 0, st, a);
  } else {
    hipLaunchKernelGGL((k_moe_route<ET>), dim3(a.T), dim3(kRouteThreads), 0, st, a);
    hipLaunchKernelGGL((k_moe_up<W, false>), up, dim3(kSplit<W> * kWave), 0, st, a);
  }
  if (!a.by_token) {
    hipLaunchKernelGGL((k_moe_down<W>), dim3((a.C - 1) / kColumns + 1, a.E), dim3(kSplit<W> * kWave), 0, st, a);
    hipLaunchKernelGGL((k_moe_sum<ET>), dim3((a.C - 1) / 1024 + 1, a.T), dim3(256), 0, st, a);
  } else {
    const dim3 down(a.C / kFewColumns, a.T);
    // Eight waves where four would take more than two rounds: one token of the layers above with 32 and 36 pairs, four waves / eight,
    // 33.1 / 32.0 and 25.8 / 24.7 us; 4 of 30 experts of 1024 x 512, e4m3, 8 pairs, 8 tokens 19.2 / 20.8.
    if (a.top_k * ((scale_blocks(a.F) + 1) / 2) > 2 * 4 * kPairs<W>)
      hipLaunchKernelGGL((k_moe_down_few<W, ET, 8>), down, dim3(8 * kWave), 0, st, a);
    else hipLaunchKernelGGL((k_moe_down_few<W, ET, 4>), down, dim3(4 * kWave), 0, st, a);
  }
}

struct MoeWs { size_t experts, weights, h, y, logits, bytes; };
MoeWs moe_ws(const laud_moe_layer* p, int T) {
  MoeWs w;
  const size_t n = (size_t)T * p->top_k;
  w.experts = 0;
  w.weights = align_up(n * 4, 256);
  w.h = w.weights + align_up(n * 4, 256);
  // three planes of bf16, or one of float32
  w.y = align_up(w.h + n * (size_t)scale_blocks(p->F) * kScaleBlock * 6, 256);
  w.logits = align_up(w.y + n * (size_t)p->C * 4, 256);
  w.bytes = w.logits + (size_t)p->E * 4;
  return w;
}

// Whether what a call writes (out, its routing, the workspace) lies over what it reads or over each other; out may be x.
bool moe_overlaps(const laud_moe_layer* p, int T, const void* x, int64_t ldx, const uint8_t* keep, const void* out, int64_t ldo,
                  const int32_t* experts, const float* weights, const void* ws, size_t ws_bytes) {
  struct Range { const void* p; size_t n; };
  const size_t E = p->E, C = p->C, F = p->F, eb = elem_bytes(p->dtype), wb = p->w_dtype == LAUD_E4M3 ? 1 : eb;
  const size_t scales = p->w_dtype == LAUD_E4M3 ? E * scale_blocks(p->F) * scale_blocks(p->C) * 4 : 0, chosen = (size_t)T * p->top_k * 4;
  const Range written[] = {{experts, chosen}, {weights, chosen}, {ws, ws_bytes}};
  for (const Range& r : {Range{p->router, E * C * eb}, Range{p->up, E * 2 * F * C * wb}, Range{p->down, E * C * F * wb},
                         Range{p->s_up, 2 * scales}, Range{p->s_down, scales}, Range{keep, (size_t)T}}) {
    if (range_meets_rows(r.p, r.n, out, ldo, eb, T, p->C)) return true;
    for (const Range& w : written)
      if (ranges_meet(r.p, r.n, w.p, w.n)) return true;
  }
  for (int i = 0; i < 3; ++i) {
    const Range& w = written[i];
    if (range_meets_rows(w.p, w.n, x, ldx, eb, T, p->C) || range_meets_rows(w.p, w.n, out, ldo, eb, T, p->C)) return true;
    for (int j = 0; j < i; ++j)
      if (ranges_meet(w.p, w.n, written[j].p, written[j].n)) return true;
  }
  return false;
}

int validate_moe(const laud_moe_layer* p, int T) {
  if (!p || T < 0 || p->C <= 0 || p->F <= 0 || p->E <= 0 || p->top_k <= 0 || p->top_k > p->E || !float_type(p->dtype))
    return LAUD_ERR_INVALID_ARG;
  if (p->w_dtype != p->dtype && p->w_dtype != LAUD_E4M3) return LAUD_ERR_INVALID_ARG;
  if (p->w_dtype == LAUD_E4M3 && p->dtype != LAUD_BF16) return LAUD_ERR_UNSUPPORTED;
  const int step = p->w_dtype == LAUD_E4M3 ? 16 : 8;
  if (p->C % step || p->F % step || p->C > (1 << 20) || p->F > (1 << 20) || p->E > kMaxExperts || p->top_k > kMaxTopK ||
      T > LAUD_MOE_MAX_TOKENS || (long long)T * p->top_k * (scale_blocks(p->F) * kScaleBlock) * 4 > 0x7fffffffll)
    return LAUD_ERR_UNSUPPORTED;
  return LAUD_OK;
}

}  // namespace
}  // namespace laud

extern "C" size_t laud_moe_workspace(const laud_moe_layer* p, int T) {
  return T > 0 && laud::validate_moe(p, T) == LAUD_OK ? laud::moe_ws(p, T).bytes : 0;
}

extern "C" int laud_moe(const laud_moe_layer* p, int T, const void* x, int64_t ldx, const uint8_t* keep, void* out, int64_t ldo,
                        int32_t* experts, float* weights, void* ws, size_t ws_bytes, void* stream) {
  using namespace laud;
  const int rc = validate_moe(p, T);
  if (rc != LAUD_OK) return rc;
  if (T == 0) return LAUD_OK;
  if (!x || !out || !p->router || !p->up || !p->down || !good_ld(ldx, p->C, 8) || !good_ld(ldo, p->C, 8)) return LAUD_ERR_INVALID_ARG;
  if (p->w_dtype == LAUD_E4M3 && (!p->s_up || !p->s_down)) return LAUD_ERR_INVALID_ARG;
  if (!aligned16(x) || !aligned16(out) || !aligned16(p->router) || !aligned16(p->up) || !aligned16(p->down) || !aligned16(ws))
    return LAUD_ERR_INVALID_ARG;
  const size_t eb = elem_bytes(p->dtype);
  if (span_bytes(T, ldx, p->C, eb) > 0x7fffffffull) return LAUD_ERR_UNSUPPORTED;
  if (!same_or_apart(x, ldx, eb, out, ldo, eb, T, p->C)) return LAUD_ERR_INVALID_ARG;
  if (!ws || ws_bytes < laud_moe_workspace(p, T)) return LAUD_ERR_WORKSPACE;
  const MoeWs w = moe_ws(p, T);
  if (moe_overlaps(p, T, x, ldx, keep, out, ldo, experts, weights, ws, w.bytes)) return LAUD_ERR_INVALID_ARG;
  MoeArgs a{};
  a.T = T; a.C = p->C; a.F = p->F; a.E = p->E; a.top_k = p->top_k; a.renormalise = p->renormalise;
  a.Fp = scale_blocks(p->F) * kScaleBlock;
  a.scale = p->scale;
  a.x = x; a.router = p->router; a.up = p->up; a.down = p->down; a.s_up = p->s_up; a.s_down = p->s_down;
  a.keep = keep; a.out = out; a.ldx = ldx; a.ldo = ldo;
  a.experts = experts ? experts : (int32_t*)((char*)ws + w.experts);
  a.weights = weights ? weights : (float*)((char*)ws + w.weights);
  a.h = (char*)ws + w.h;
  a.y = (float*)((char*)ws + w.y);
  a.logits = (float*)((char*)ws + w.logits);
  clear_stale_error();
  hipStream_t st = (hipStream_t)stream;
  if (p->w_dtype == LAUD_E4M3) launch_moe<W_E4M3, bf16_t>(a, st);
  else if (p->dtype == LAUD_BF16) launch_moe<W_BF16, bf16_t>(a, st);
  else launch_moe<W_F32, float>(a, st);
  return check_launch();
}
