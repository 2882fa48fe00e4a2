// The seam between two residual blocks of a token list (norm after a block, gate, residual add, norm before the next block, its
// result optionally in 8 bits) and the quantisation in blocks of 128.
#include "laud_token.h"

namespace laud {
namespace {

// Bound by memory: x and y are read once, out and z written once.  A row belongs to TPR threads, which keep it in registers from its
// only read to its last write: chunk j of a thread is eight elements, chunks of neighbouring threads lie side by side.  A workgroup
// goes from row to row with the norms' vectors in registers and requests the next row's x and y before it finishes a row, four waves
// a SIMD (128 registers): 16384 x 4096 bf16 to 8 bits, a quarter of the rows skipped, 109 -> 86 us, 5.1 TB/s of a copy's 5.2.  Bf16
// rows up to 4096 channels fit; float32 rows of two pieces a thread keep up to 32 registers of a lane in memory and rows of four pieces
// 32 to 93: 8192 x 4096 float32 at 5.2 TB/s, 4.5 to 8 bits, 4096 x 8192 4.0; 2048 x 16384 bf16 at 4.5, 1024 x 32768 at 3.0.  More
// threads a row for few rows: 4 x 2048 in 2.8 us with 256, 3.2 with 128, 4.3 with 64 threads; 8192 x 2048 26.1 / 26.9 / 34.6.
constexpr int kMaxC = 32768;
constexpr int kMostGroups = 1 << 20;   // workgroups of a launch (threads are counted in 32 bits); longer lists loop
constexpr int kNormThreads = 1 << 20;  // threads of a norm's launch, four times what is resident: a thread has rows to look ahead to

struct NormArgs {
  int rows, C, kind, rows_per_gate;
  float eps, alpha, beta, inv_c;
  const float *post_w, *post_b, *pre_w, *pre_b, *gate;
  const uint8_t* keep;
  const void *x, *y;
  void *out, *z;
  float* z_scale;
  int64_t ldx, ldy, ldo, ldz;  // elements
};

// Sum over the threads of a row.  The waves' sums meet in `part`, whose two halves take turns: who writes a half again has passed
// the barrier of the call between, which every wave reaches only after it has read that half.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float (*part)[TPR / kWave], int& turn) {
  v = lanes64_sum(v);
  if constexpr (TPR > kWave) {
    constexpr int kWaves = TPR / kWave;
    float* const at = part[turn];
    turn ^= 1;
    if (lane_id() == 0) at[threadIdx.x / kWave] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) v += at[w];
  }
  return v;
}

__device__ __forceinline__ void load8(float (&f)[8], const float* p, int chunk) {
  piece8<float> q;
  q.load(p, chunk);
  q.get(f);
}

// A vector over the channels: a thread's pieces in registers for all its rows, or, where a row takes four pieces a thread, read
// again for each row.
template <int TPR, int VPT>
struct Channels {
  static constexpr bool kHeld = VPT <= 2;
  const float* p;
  float held[kHeld ? VPT : 1][8];
  __device__ __forceinline__ Channels(const float* from, int t, int chunks) : p(from) {
    if constexpr (kHeld) {
#pragma unroll
      for (int j = 0; j < VPT; ++j)
        if (p && t + j * TPR < chunks) load8(held[j], p, t + j * TPR);
    }
  }
  __device__ __forceinline__ void get(float (&f)[8], int t, int j) const {
    if constexpr (kHeld) {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = held[j][e];
    } else {
      load8(f, p, t + j * TPR);
    }
  }
};

// v <- norm(v) * w + b
template <int TPR, int VPT>
__device__ __forceinline__ void norm_row(float (&v)[VPT][8], const NormArgs& a, const Channels<TPR, VPT>& w, const float* b, int t,
                                         float (*part)[TPR / kWave], int& turn) {
  const int chunks = a.C / 8;
  if (a.kind == LAUD_NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < VPT; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) s += v[j][e];  // (chunks past the row hold zeros)
    const float mean = row_sum<TPR>(s, part, turn) * a.inv_c;
#pragma unroll
    for (int j = 0; j < VPT; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[j][e] = t + j * TPR < chunks ? v[j][e] - mean : 0.f;
  }
  float s = 0.f;
#pragma unroll
  for (int j = 0; j < VPT; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(v[j][e], v[j][e], s);
  const float r = 1.f / sqrtf(row_sum<TPR>(s, part, turn) * a.inv_c + a.eps);
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int c = t + j * TPR;
    if (c >= chunks) continue;
    float f[8];
    w.get(f, t, j);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[j][e] = v[j][e] * r * f[e];
    if (b) {
      load8(f, b, c);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[j][e] += f[e];
    }
  }
}

// A row's pieces of x and y on their way.
template <typename ET, int TPR, int VPT>
struct Row {
  piece8<ET> x[VPT], y[VPT];
  bool kept;
  __device__ __forceinline__ void request(const NormArgs& a, long long row, bool keep, int t) {
    const int chunks = a.C / 8;
    kept = keep;
    const ET *xr = reinterpret_cast<const ET*>(a.x) + row * a.ldx, *yr = reinterpret_cast<const ET*>(a.y) + row * a.ldy;
#pragma unroll
    for (int j = 0; j < VPT; ++j)
      if (t + j * TPR < chunks) x[j].load(xr, t + j * TPR);
    if (kept) {
#pragma unroll
      for (int j = 0; j < VPT; ++j)
        if (t + j * TPR < chunks) y[j].load(yr, t + j * TPR);
    }
  }
};

template <typename ET, bool Z8, int TPR, int VPT>
__global__ __launch_bounds__(TPR == kWave ? 256 : TPR, 4) void k_norm_residual(NormArgs a) {
  constexpr int kRows = TPR == kWave ? 256 / TPR : 1;  // rows of a workgroup; more than one only where a row is a wave's
  static_assert(kRows == 1 || TPR == kWave, "rows that share a workgroup need no barrier");
  __shared__ float part[2][TPR / kWave];
  int turn = 0;
  const int t = threadIdx.x % TPR, chunks = a.C / 8;
  const long long step = (long long)gridDim.x * kRows;
  long long row = (long long)blockIdx.x * kRows + threadIdx.x / TPR;
  auto is_kept = [&](long long r) { return r < a.rows && a.y && (!a.keep || a.keep[r] != 0); };
  if (row >= a.rows) return;
  bool kept_next = is_kept(row + step);
  Row<ET, TPR, VPT> in;
  in.request(a, row, is_kept(row), t);
  const Channels<TPR, VPT> post(a.post_w, t, chunks), pre(a.pre_w, t, chunks);
  for (; row < a.rows; row += step) {
    float r[VPT][8];
    piece8<ET> o[VPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) r[j][e] = 0.f;
    if (in.kept) {
#pragma unroll
      for (int j = 0; j < VPT; ++j)
        if (t + j * TPR < chunks) in.y[j].get(r[j]);
      if (a.post_w) norm_row<TPR, VPT>(r, a, post, a.post_b, t, part, turn);
      const float* g = a.gate ? a.gate + row / a.rows_per_gate * a.C : nullptr;
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        if (t + j * TPR >= chunks) continue;
        float x[8];
        in.x[j].get(x);
        if (g) {
          float f[8];
          load8(f, g, t + j * TPR);
#pragma unroll
          for (int e = 0; e < 8; ++e) r[j][e] *= f[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) r[j][e] = fmaf(a.beta, r[j][e], a.alpha * x[e]);
        o[j].put(r[j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        o[j] = in.x[j];
        if (t + j * TPR < chunks) in.x[j].get(r[j]);
      }
    }
    // the next row is under way while this one is finished
    if (row + step < a.rows) {
      in.request(a, row + step, kept_next, t);
      kept_next = is_kept(row + 2 * step);
    }
    if (a.out) {
      ET* out = reinterpret_cast<ET*>(a.out) + row * a.ldo;
#pragma unroll
      for (int j = 0; j < VPT; ++j)
        if (t + j * TPR < chunks) o[j].store(out, t + j * TPR);
    }
    if (!a.z) continue;
    norm_row<TPR, VPT>(r, a, pre, a.pre_b, t, part, turn);
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int c = t + j * TPR;
      if constexpr (Z8) {
        const float s = block_scale(lanes16_max(c < chunks ? top_bits(r[j]) : 0u));  // sixteen lanes: one block
        if (c < chunks) {
          reinterpret_cast<tok_u2*>(reinterpret_cast<uint8_t*>(a.z) + row * a.ldz)[c] = codes8(r[j], s);
          if (c % 16 == 0) a.z_scale[row * scale_blocks(a.C) + c / 16] = s;
        }
      } else if (c < chunks) {
        o[j].put(r[j]);
        o[j].store(reinterpret_cast<ET*>(a.z) + row * a.ldz, c);
      }
    }
  }
}

template <typename ET, bool Z8>
void launch_norm(const NormArgs& a, hipStream_t st) {
  const int chunks = a.C / 8;
#define LAUD_NORM(TPR, VPT)                                                                                               \
  do {                                                                                                                    \
    constexpr int kThreads = TPR == kWave ? 256 : TPR, kRows = kThreads / TPR;                                            \
    hipLaunchKernelGGL((k_norm_residual<ET, Z8, TPR, VPT>), dim3(min((a.rows - 1) / kRows + 1, kNormThreads / kThreads)), \
                       dim3(kThreads), 0, st, a);                                                                         \
  } while (0)
  if (chunks <= 64) LAUD_NORM(64, 1);
  else if (chunks <= 128) LAUD_NORM(64, 2);
  else if (chunks <= 256) LAUD_NORM(256, 1);
  else if (chunks <= 512) LAUD_NORM(256, 2);
  else if (chunks <= 1024) LAUD_NORM(512, 2);
  else if (chunks <= 2048) LAUD_NORM(1024, 2);
  else LAUD_NORM(1024, 4);
#undef LAUD_NORM
}

// ---- quantisation ---------------------------------------------------------------------------------------------------------
// One scale for 128 elements of a row: sixteen lanes a block, one read of x.  Bound by memory: 16384 x 4096 bf16 in 38.7 us, 5.2 TB/s.
template <typename ET>
__global__ __launch_bounds__(256) void k_quant_rows(const ET* __restrict__ x, int64_t ldx, long long blocks, int kb, int cols,
                                                    uint8_t* __restrict__ q, int64_t ldq, float* __restrict__ scale) {
  for (long long b = (long long)blockIdx.x * 16 + threadIdx.x / 16; b < blocks; b += (long long)gridDim.x * 16) {
    const long long row = b / kb;
    const int c = (int)(b - row * kb) * 16 + threadIdx.x % 16;
    const bool in = c < cols / 8;
    float f[8] = {};
    if (in) {
      piece8<ET> p;
      p.load(x + row * ldx, c);
      p.get(f);
    }
    const float s = block_scale(lanes16_max(top_bits(f)));
    if (in) reinterpret_cast<tok_u2*>(q + row * ldq)[c] = codes8(f, s);
    if (threadIdx.x % 16 == 0) scale[b] = s;
  }
}

// One scale for 128 rows of 128 elements: a workgroup a block, which stays in registers between its maximum and its codes.  Bound by
// memory: 8192 x 4096 bf16 in 21 us, 4.7 TB/s, float32 in 33, 5.1.
template <typename ET>
__global__ __launch_bounds__(256) void k_quant_square(const ET* __restrict__ x, int64_t ldx, int rows, int kb, int cols,
                                                      uint8_t* __restrict__ q, int64_t ldq, float* __restrict__ scale) {
  __shared__ unsigned part[4];
  const long long rb = blockIdx.y + (long long)blockIdx.z * gridDim.y;
  if (rb * 128 >= rows) return;
  const int cb = blockIdx.x;
  const int c = cb * 16 + threadIdx.x % 16;
  piece8<ET> p[8];
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const long long r = rb * 128 + i * 16 + threadIdx.x / 16;
    if (r < rows && c < cols / 8) {
      p[i].load(x + r * ldx, c);
    } else {
      const float zero[8] = {};
      p[i].put(zero);
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float f[8];
    p[i].get(f);
    top = max(top, top_bits(f));
  }
  top = lanes64_max(top);
  if (lane_id() == 0) part[threadIdx.x / kWave] = top;
  __syncthreads();
  const float s = block_scale(max(max(part[0], part[1]), max(part[2], part[3])));
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const long long r = rb * 128 + i * 16 + threadIdx.x / 16;
    if (r < rows && c < cols / 8) {
      float f[8];
      p[i].get(f);
      reinterpret_cast<tok_u2*>(q + r * ldq)[c] = codes8(f, s);
    }
  }
  if (threadIdx.x == 0) scale[rb * kb + cb] = s;
}

template <typename ET>
void launch_quant(const void* x, int64_t ldx, int rows, int cols, int block_rows, void* q, int64_t ldq, float* scale, hipStream_t st) {
  const int kb = scale_blocks(cols);
  if (block_rows == 1) {
    const long long blocks = (long long)rows * kb;
    hipLaunchKernelGGL((k_quant_rows<ET>), dim3((unsigned)std::min((blocks + 15) / 16, (long long)kMostGroups)), dim3(256), 0, st, (const ET*)x, ldx,
                       blocks, kb, cols, (uint8_t*)q, ldq, scale);
  } else {
    const int rbs = scale_blocks(rows), per = min(rbs, 32768);
    hipLaunchKernelGGL((k_quant_square<ET>), dim3((unsigned)kb, (unsigned)per, (unsigned)((rbs + per - 1) / per)), dim3(256), 0, st,
                       (const ET*)x, ldx, rows, kb, cols, (uint8_t*)q, ldq, scale);
  }
}

}  // namespace
}  // namespace laud

extern "C" int laud_norm_residual(const laud_norm_block* p, int rows, const void* x, int64_t ldx, const void* y, int64_t ldy,
                                  const uint8_t* keep, const float* gate, int rows_per_gate, void* out, int64_t ldo, void* z,
                                  int64_t ldz, int z_dtype, float* z_scale, void* stream) {
  using namespace laud;
  if (!p || rows < 0 || p->C <= 0 || !float_type(p->dtype) || (p->kind != LAUD_NORM_RMS && p->kind != LAUD_NORM_LAYER) || !(p->eps >= 0.f))
    return LAUD_ERR_INVALID_ARG;
  if (p->C % 8 || p->C > kMaxC) return LAUD_ERR_UNSUPPORTED;
  if (rows == 0) return LAUD_OK;
  if (!x || (!out && !z) || !good_ld(ldx, p->C, 8) || (y && !good_ld(ldy, p->C, 8)) || (out && !good_ld(ldo, p->C, 8)) ||
      (z && !good_ld(ldz, p->C, 8)))
    return LAUD_ERR_INVALID_ARG;
  if ((!y && (keep || gate)) || (gate && rows_per_gate <= 0)) return LAUD_ERR_INVALID_ARG;
  const bool z8 = z && z_dtype == LAUD_E4M3;
  if (z && (!p->pre_w || (!z8 && z_dtype != p->dtype) || (z8 && !z_scale))) return LAUD_ERR_INVALID_ARG;
  if (!aligned16(x) || !aligned16(y) || !aligned16(out) || !aligned16(z) || !aligned16(gate) || !aligned16(p->post_w) ||
      !aligned16(p->post_b) || !aligned16(p->pre_w) || !aligned16(p->pre_b))
    return LAUD_ERR_INVALID_ARG;
  // a row's results are written after all of that row has been read, so a result may take its row's place and no other's
  const size_t eb = elem_bytes(p->dtype), zb = z8 ? 1 : eb;
  if ((out && (!same_or_apart(x, ldx, eb, out, ldo, eb, rows, p->C) || (y && !same_or_apart(y, ldy, eb, out, ldo, eb, rows, p->C)))) ||
      (z && (!same_or_apart(x, ldx, eb, z, ldz, zb, rows, p->C) || (y && !same_or_apart(y, ldy, eb, z, ldz, zb, rows, p->C)))) ||
      (out && z && rows_meet(out, ldo, eb, z, ldz, zb, rows, p->C)))
    return LAUD_ERR_INVALID_ARG;
  // ... and over nothing that every row reads; the scales over nothing at all
  const size_t scales = z8 ? (size_t)rows * scale_blocks(p->C) * 4 : 0, vector = (size_t)p->C * 4;
  const auto over_result = [&](const void* q, size_t n) {
    return range_meets_rows(q, n, out, ldo, eb, rows, p->C) || range_meets_rows(q, n, z, ldz, zb, rows, p->C);
  };
  for (const void* v : {y ? p->post_w : nullptr, y && p->post_w ? p->post_b : nullptr, z ? p->pre_w : nullptr, z ? p->pre_b : nullptr})
    if (over_result(v, vector) || ranges_meet(v, vector, z_scale, scales)) return LAUD_ERR_INVALID_ARG;
  const size_t gates = gate ? ((size_t)(rows - 1) / rows_per_gate + 1) * vector : 0;
  if (over_result(keep, rows) || over_result(gate, gates) || over_result(z_scale, scales) || ranges_meet(keep, rows, z_scale, scales) ||
      ranges_meet(gate, gates, z_scale, scales) || range_meets_rows(z_scale, scales, x, ldx, eb, rows, p->C) ||
      range_meets_rows(z_scale, scales, y, ldy, eb, rows, p->C))
    return LAUD_ERR_INVALID_ARG;
  NormArgs a{};
  a.rows = rows; a.C = p->C; a.kind = p->kind; a.rows_per_gate = rows_per_gate;
  a.eps = p->eps; a.alpha = p->alpha; a.beta = p->beta; a.inv_c = 1.f / (float)p->C;
  a.post_w = p->post_w; a.post_b = p->post_b; a.pre_w = p->pre_w; a.pre_b = p->pre_b;
  a.gate = gate; a.keep = keep; a.x = x; a.y = y; a.out = out; a.z = z; a.z_scale = z_scale;
  a.ldx = ldx; a.ldy = ldy; a.ldo = ldo; a.ldz = ldz;
  clear_stale_error();
  hipStream_t st = (hipStream_t)stream;
  if (p->dtype == LAUD_BF16) {
    if (z8) launch_norm<bf16_t, true>(a, st);
    else launch_norm<bf16_t, false>(a, st);
  } else {
    if (z8) launch_norm<float, true>(a, st);
    else launch_norm<float, false>(a, st);
  }
  return check_launch();
}

extern "C" int laud_quantize_e4m3(const void* x, int64_t ldx, int rows, int cols, int dtype, int block_rows, void* q, int64_t ldq,
                                  float* scale, void* stream) {
  using namespace laud;
  if (rows < 0 || cols <= 0 || !float_type(dtype) || (block_rows != 1 && block_rows != kScaleBlock)) return LAUD_ERR_INVALID_ARG;
  if (cols % 8 || (block_rows != 1 && !launchable(scale_blocks(cols), 256))) return LAUD_ERR_UNSUPPORTED;
  if (rows == 0) return LAUD_OK;
  if (!x || !q || !scale || !good_ld(ldx, cols, 8) || !good_ld(ldq, cols, 8) || !aligned16(x) || !aligned16(q)) return LAUD_ERR_INVALID_ARG;
  const size_t scales = ((size_t)(rows - 1) / block_rows + 1) * scale_blocks(cols) * 4;
  if (rows_meet(x, ldx, elem_bytes(dtype), q, ldq, 1, rows, cols) || range_meets_rows(scale, scales, x, ldx, elem_bytes(dtype), rows, cols) ||
      range_meets_rows(scale, scales, q, ldq, 1, rows, cols))
    return LAUD_ERR_INVALID_ARG;
  clear_stale_error();
  if (dtype == LAUD_BF16) launch_quant<bf16_t>(x, ldx, rows, cols, block_rows, q, ldq, scale, (hipStream_t)stream);
  else launch_quant<float>(x, ldx, rows, cols, block_rows, q, ldq, scale, (hipStream_t)stream);
  return check_launch();
}
