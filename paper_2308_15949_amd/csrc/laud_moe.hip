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
  float* h;             // [T * top_k][Fp]
  float* y;             // [T * top_k][C]: an entry's weighted result
  unsigned* arrived;    // [column tiles of the last product]: workgroups that are done, 0 behind the routing
};

constexpr int kColumns = 32;  // output channels of a workgroup of the last product
__host__ __device__ inline int column_tiles(int C) { return (C - 1) / kColumns + 1; }

// ---- routing ----------------------------------------------------------------------------------------------------------------
// Floats as unsigned integers in their order; a NaN lies below all.
__device__ __forceinline__ unsigned order_key(float f) {
  const unsigned u = __float_as_uint(f);
  return f != f ? 0u : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// The choice of one token by one wave from logits [E] in LDS.
__device__ __forceinline__ void choose_experts(const float* logits, int E, int top_k, bool renormalise, float scale, int32_t* experts,
                                               float* weights) {
  const int lane = lane_id();
  unsigned chosen = 0;  // bit j: expert 64 j + lane
  float top = -INFINITY;
  for (int e = lane; e < E; e += kWave) top = fmaxf(top, logits[e]);
  {
    const unsigned k = lanes64_max(order_key(top));
    top = __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k);
  }
  for (int n = 0; n < top_k; ++n) {
    unsigned key = 0, id = 0;  // id: bits of 2^31 - 1 - expert, so that the lower expert is the larger one
    for (int e = lane, j = 0; e < E; e += kWave, ++j) {
      if (chosen >> j & 1u) continue;
      const unsigned k = order_key(logits[e]);
      if (k > key || id == 0) { key = k; id = 0x7fffffffu - (unsigned)e; }
    }
    const unsigned best = lanes64_max(key);
    const unsigned e = 0x7fffffffu - lanes64_max(key == best ? id : 0u);
    if ((e & 63u) == (unsigned)lane) chosen |= 1u << (e >> 6);
  }
  float sum = 0.f;
  for (int e = lane, j = 0; e < E; e += kWave, ++j) {
    const float p = expf(logits[e] - top);
    if (!renormalise || (chosen >> j & 1u) || p != p) sum += p;  // (a NaN anywhere is in every softmax value)
  }
  sum = lanes64_sum(sum);
  int before = 0;
  for (int e0 = 0, j = 0; e0 < E; e0 += kWave, ++j) {
    const bool mine = chosen >> j & 1u;
    const unsigned long long b = __ballot(mine);
    if (mine) {
      const int at = before + ballot_prefix(b);
      experts[at] = e0 + lane;
      weights[at] = expf(logits[e0 + lane] - top) / sum * scale;
    }
    before += __popcll(b);
  }
}

// One workgroup a token: the waves take the experts' logits in turn, the first one chooses.
constexpr int kRouteThreads = 1024;
template <typename ET>
__global__ __launch_bounds__(kRouteThreads) void k_moe_route(MoeArgs a) {
  __shared__ float logits[kMaxExperts];
  const int t = blockIdx.x, lane = lane_id(), wave = threadIdx.x / kWave;
  if (t == 0)
    for (int i = threadIdx.x; i < column_tiles(a.C); i += kRouteThreads) a.arrived[i] = 0;
  int32_t* experts = a.experts + (long long)t * a.top_k;
  float* weights = a.weights + (long long)t * a.top_k;
  if (a.keep && a.keep[t] == 0) {
    if ((int)threadIdx.x < a.top_k) { experts[threadIdx.x] = -1; weights[threadIdx.x] = 0.f; }
    return;
  }
  const ET* x = reinterpret_cast<const ET*>(a.x) + t * a.ldx;
  constexpr int kAtOnce = 4;  // experts a wave takes at a time, so that their loads are under way together
  for (int e0 = wave * kAtOnce; e0 < a.E; e0 += kRouteThreads / kWave * kAtOnce) {
    float s[kAtOnce] = {};
#pragma unroll 2
    for (int c = lane; c < a.C / 8; c += kWave) {
      piece8<ET> p, q[kAtOnce];
      float f[8], g[8];
      p.load(x, c);
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) q[i].load(reinterpret_cast<const ET*>(a.router) + (long long)min(e0 + i, a.E - 1) * a.C, c);
      p.get(f);
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        q[i].get(g);
#pragma unroll
        for (int u = 0; u < 8; ++u) s[i] = fmaf(f[u], g[u], s[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      s[i] = lanes64_sum(s[i]);
      if (lane == 0 && e0 + i < a.E) logits[e0 + i] = s[i];
    }
  }
  __syncthreads();
  if (wave == 0) choose_experts(logits, a.E, a.top_k, a.renormalise != 0, a.scale, experts, weights);
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
// ... or float32 values, which go through bf16 instructions as a sum of two: the part bf16 holds and its remainder, 16 bits
// together (a hidden value rounded to bf16 alone would add an error as large as the result's own rounding).
template <int W>
__device__ __forceinline__ f32x4 mma_wide(const tok_u4& w, const f32x4* v, f32x4 c) {
  if constexpr (W == W_F32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[i]), v[0][i], c, 0, 0, 0);
  } else {
#pragma unroll
    for (int u = 0; u < (W == W_E4M3 ? 2 : 1); ++u) {
      union { bf16x2 p[4]; bf16x8 v; } hi, lo;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x2 f = {v[2 * u + i / 2][i % 2 * 2], v[2 * u + i / 2][i % 2 * 2 + 1]};
        hi.p[i] = __builtin_convertvector(f, bf16x2);
        const f32x2 rest = {f[0] - (float)hi.p[i][0], f[1] - (float)hi.p[i][1]};
        lo.p[i] = __builtin_convertvector(rest, bf16x2);
      }
      const bf16x8 a = W == W_E4M3 ? widen8(w[2 * u], w[2 * u + 1]) : __builtin_bit_cast(bf16x8, w);
      c = mma_bf16_16(a, hi.v, c);
      c = mma_bf16_16(a, lo.v, c);
    }
  }
  return c;
}

// The products run for (tile of channels, slot): a slot is an expert, or, where the entries (token, choice) are fewer than the
// experts, an entry, whose workgroups take its expert if no earlier entry has the same.  Returns the expert and in `list` its
// entries (in any order: no entry's value depends on it), or no entries.  Called by a whole workgroup.
constexpr int kSplit = 8;  // waves of a workgroup, which share the reduction by blocks of 128
__device__ __forceinline__ int slot_entries(const int32_t* experts, int entries, int E, int slot, int* list, int* counts, int& len) {
  const bool by_entry = entries < E;
  if (threadIdx.x < 2) counts[threadIdx.x] = 0;
  const int e = by_entry ? experts[slot] : slot;
  __syncthreads();
  if (e >= 0) {
    for (int i = threadIdx.x; i < entries; i += kSplit * kWave) {
      if (experts[i] != e) continue;
      if (by_entry && i < slot) counts[1] = 1;
      list[atomicAdd(&counts[0], 1)] = i;
    }
  }
  __syncthreads();
  len = counts[1] ? 0 : counts[0];
  return e;
}

// Sums of the waves' parts of two row tiles, in the waves' order, for the first wave.
__device__ __forceinline__ void join_waves(f32x4 (&v)[2], f32x4 (*part)[2][kWave], int wave, int lane) {
  part[wave][0][lane] = v[0];
  part[wave][1][lane] = v[1];
  __syncthreads();
  if (wave == 0) {
#pragma unroll
    for (int w = 1; w < kSplit; ++w) {
      v[0] += part[w][0][lane];
      v[1] += part[w][1][lane];
    }
  }
  __syncthreads();
}

// h of one expert's entries for 16 hidden channels.
template <int W>
__global__ __launch_bounds__(kSplit * kWave) void k_moe_up(MoeArgs a) {
  typedef Weights<W> WT;
  constexpr int kXP = W == W_E4M3 ? 2 : 1;
  __shared__ int list[LAUD_MOE_MAX_TOKENS], counts[2];
  __shared__ f32x4 part[kSplit][2][kWave];
  const int lane = lane_id(), wave = threadIdx.x / kWave, r16 = lane % 16, quarter = lane / 16;
  int len;
  const int e = slot_entries(a.experts, a.T * a.top_k, a.E, blockIdx.y, list, counts, len);
  if (len == 0) return;
  const int f0 = blockIdx.x * 16, rows = min(16, a.F - f0);  // (from F to the end of its block of 128 h is 0: rows may be none)
  const int kb_all = scale_blocks(a.C);
  const long long row_bytes = (long long)a.C * WT::kBytes;
  const uint8_t* base = reinterpret_cast<const uint8_t*>(a.up) + ((long long)e * 2 * a.F + f0) * row_bytes;
  const __amdgpu_buffer_rsrc_t rg = bytes_of(base, max(rows, 0) * row_bytes);
  const __amdgpu_buffer_rsrc_t ru = bytes_of(base + a.F * row_bytes, max(rows, 0) * row_bytes);
  const int xb = W == W_F32 ? 4 : 2;
  const __amdgpu_buffer_rsrc_t rx = bytes_of(a.x, ((a.T - 1) * a.ldx + a.C) * xb);
  const float *sg = nullptr, *su = nullptr;
  if (W == W_E4M3 && rows > 0) {
    const int fb = scale_blocks(a.F);
    sg = a.s_up + ((long long)e * 2 * fb + f0 / kScaleBlock) * kb_all;
    su = sg + (long long)fb * kb_all;
  }
  for (int l0 = 0; l0 < len; l0 += 16) {
    const int entry = list[min(l0 + r16, len - 1)];
    const unsigned xoff = (unsigned)(entry / a.top_k * a.ldx * xb);
    f32x4 v[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    for (int kb = wave; kb < kb_all; kb += kSplit) {
      f32x4 pg = {0.f, 0.f, 0.f, 0.f}, pu = pg;
#pragma unroll
      for (int p = 0; p < WT::kPieces; ++p) {
        const int k = kb * kScaleBlock + WT::first(p, quarter);
        const bool in = k < a.C;
        const unsigned woff = in && r16 < rows ? (unsigned)(r16 * row_bytes) + (unsigned)k * WT::kBytes : kOutside;
        const tok_u4 wg = load16(rg, woff), wu = load16(ru, woff);
        tok_u4 x[kXP];
#pragma unroll
        for (int i = 0; i < kXP; ++i) x[i] = load16(rx, in ? xoff + (unsigned)(k + 8 * i) * xb : kOutside);
        pg = mma_stored<W>(wg, x, pg);
        pu = mma_stored<W>(wu, x, pu);
      }
      const float fg = sg ? sg[kb] : 1.f, fu = su ? su[kb] : 1.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[0][i] = fmaf(pg[i], fg, v[0][i]);
        v[1][i] = fmaf(pu[i], fu, v[1][i]);
      }
    }
    join_waves(v, part, wave, lane);
    if (wave == 0 && l0 + r16 < len) {
      f32x4 h;
#pragma unroll
      for (int i = 0; i < 4; ++i) h[i] = quarter * 4 < rows ? v[0][i] / (1.f + expf(-v[0][i])) * v[1][i] : 0.f;
      *reinterpret_cast<f32x4*>(a.h + (long long)entry * a.Fp + f0 + quarter * 4) = h;
    }
  }
}

// Values that workgroups on different XCDs hand over within a launch go past the XCDs' caches, which do not see each other (a
// release and an acquire by every workgroup instead, which write back and drop a whole cache, made the launch three times as long).
__device__ __forceinline__ void shared_store(float* p, float v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ float shared_load(const float* p) {
  return __hip_atomic_load(const_cast<float*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// One expert's entries for 32 output channels, weighted; the last workgroup of a tile of channels to get here adds each token's
// entries up, in the order of its experts.
template <int W, typename OT>
__global__ __launch_bounds__(kSplit * kWave) void k_moe_down(MoeArgs a) {
  typedef Weights<W> WT;
  __shared__ int list[LAUD_MOE_MAX_TOKENS], counts[2];
  __shared__ f32x4 part[kSplit][2][kWave];
  __shared__ unsigned place;
  const int lane = lane_id(), wave = threadIdx.x / kWave, r16 = lane % 16, quarter = lane / 16;
  int len;
  const int e = slot_entries(a.experts, a.T * a.top_k, a.E, blockIdx.y, list, counts, len);
  const int c0 = blockIdx.x * kColumns, rows = min(kColumns, a.C - c0);
  if (len > 0) {
    const int kb_all = scale_blocks(a.F);
    const long long row_bytes = (long long)a.F * WT::kBytes;
    const __amdgpu_buffer_rsrc_t rw =
        bytes_of(reinterpret_cast<const uint8_t*>(a.down) + ((long long)e * a.C + c0) * row_bytes, rows * row_bytes);
    const float* sw = W == W_E4M3 ? a.s_down + ((long long)e * scale_blocks(a.C) + c0 / kScaleBlock) * kb_all : nullptr;
    for (int l0 = 0; l0 < len; l0 += 16) {
      const int entry = list[min(l0 + r16, len - 1)];
      const float* h = a.h + (long long)entry * a.Fp;
      f32x4 v[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
      for (int kb = wave; kb < kb_all; kb += kSplit) {
        f32x4 p0 = {0.f, 0.f, 0.f, 0.f}, p1 = p0;
#pragma unroll
        for (int p = 0; p < WT::kPieces; ++p) {
          const int k = kb * kScaleBlock + WT::first(p, quarter);
          const unsigned off = (unsigned)(r16 * row_bytes) + (unsigned)k * WT::kBytes;
          const tok_u4 w0 = load16(rw, k < a.F && r16 < rows ? off : kOutside);
          const tok_u4 w1 = load16(rw, k < a.F && 16 + r16 < rows ? off + (unsigned)(16 * row_bytes) : kOutside);
          f32x4 x[WT::kElems / 4];
#pragma unroll
          for (int i = 0; i < WT::kElems / 4; ++i) x[i] = *reinterpret_cast<const f32x4*>(h + k + 4 * i);
          p0 = mma_wide<W>(w0, x, p0);
          p1 = mma_wide<W>(w1, x, p1);
        }
        const float f = sw ? sw[kb] : 1.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[0][i] = fmaf(p0[i], f, v[0][i]);
          v[1][i] = fmaf(p1[i], f, v[1][i]);
        }
      }
      join_waves(v, part, wave, lane);
      if (wave == 0 && l0 + r16 < len) {
        const float w = a.weights[entry];
        float* y = a.y + (long long)entry * a.C + c0;
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (i * 16 + quarter * 4 < rows)
#pragma unroll
            for (int n = 0; n < 4; ++n) shared_store(y + i * 16 + quarter * 4 + n, v[i][n] * w);
      }
    }
  }
  vm_wait<0>();  // (the stores have arrived before the workgroup counts as done)
  __syncthreads();
  if (threadIdx.x == 0)
    place = __hip_atomic_fetch_add(a.arrived + blockIdx.x, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (place + 1 != gridDim.y) return;
  for (int i = threadIdx.x; i < a.T * (kColumns / 4); i += kSplit * kWave) {
    const int t = i / (kColumns / 4), c = i % (kColumns / 4) * 4;
    if (c >= rows) continue;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    if (!a.keep || a.keep[t] != 0) {
      const float* y = a.y + (long long)t * a.top_k * a.C + c0 + c;
      for (int j = 0; j < a.top_k; ++j)
#pragma unroll
        for (int n = 0; n < 4; ++n) s[n] += shared_load(y + (long long)j * a.C + n);
    }
    store4(reinterpret_cast<OT*>(a.out) + t * a.ldo + c0 + c, s);
  }
}

template <int W, typename ET>
void launch_moe(const MoeArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((k_moe_route<ET>), dim3(a.T), dim3(kRouteThreads), 0, st, a);
  const unsigned slots = (unsigned)min((long long)a.E, (long long)a.T * a.top_k);
  hipLaunchKernelGGL((k_moe_up<W>), dim3(a.Fp / 16, slots), dim3(kSplit * kWave), 0, st, a);
  hipLaunchKernelGGL((k_moe_down<W, ET>), dim3(column_tiles(a.C), slots), dim3(kSplit * kWave), 0, st, a);
}

struct MoeWs { size_t experts, weights, h, y, arrived, bytes; };
MoeWs moe_ws(const laud_moe_layer* p, int T) {
  MoeWs w;
  const size_t n = (size_t)T * p->top_k;
  w.experts = 0;
  w.weights = align_up(n * 4, 256);
  w.h = w.weights + align_up(n * 4, 256);
  w.y = align_up(w.h + n * (size_t)scale_blocks(p->F) * kScaleBlock * 4, 256);
  w.arrived = align_up(w.y + n * (size_t)p->C * 4, 256);
  w.bytes = w.arrived + (size_t)column_tiles(p->C) * 4;
  return w;
}

int validate_moe(const laud_moe_layer* p, int T) {
  if (!p || T < 0 || p->C <= 0 || p->F <= 0 || p->E <= 0 || p->top_k <= 0 || p->top_k > p->E || !float_type(p->dtype))
    return LAUD_ERR_INVALID_ARG;
  if (p->w_dtype != p->dtype && p->w_dtype != LAUD_E4M3) return LAUD_ERR_INVALID_ARG;
  if (p->w_dtype == LAUD_E4M3 && p->dtype != LAUD_BF16) return LAUD_ERR_UNSUPPORTED;
  const int step = p->w_dtype == LAUD_E4M3 ? 16 : 8;
  if (p->C % step || p->F % step || p->C > (1 << 20) || p->F > (1 << 20) || p->E > kMaxExperts || p->top_k > kMaxTopK ||
      T > LAUD_MOE_MAX_TOKENS)
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
  MoeArgs a{};
  a.T = T; a.C = p->C; a.F = p->F; a.E = p->E; a.top_k = p->top_k; a.renormalise = p->renormalise;
  a.Fp = scale_blocks(p->F) * kScaleBlock;
  a.scale = p->scale;
  a.x = x; a.router = p->router; a.up = p->up; a.down = p->down; a.s_up = p->s_up; a.s_down = p->s_down;
  a.keep = keep; a.out = out; a.ldx = ldx; a.ldo = ldo;
  a.experts = experts ? experts : (int32_t*)((char*)ws + w.experts);
  a.weights = weights ? weights : (float*)((char*)ws + w.weights);
  a.h = (float*)((char*)ws + w.h);
  a.y = (float*)((char*)ws + w.y);
  a.arrived = (unsigned*)((char*)ws + w.arrived);
  clear_stale_error();
  hipStream_t st = (hipStream_t)stream;
  if (p->w_dtype == LAUD_E4M3) launch_moe<W_E4M3, bf16_t>(a, st);
  else if (p->dtype == LAUD_BF16) launch_moe<W_BF16, bf16_t>(a, st);
  else launch_moe<W_F32, float>(a, st);
  return check_launch();
}
