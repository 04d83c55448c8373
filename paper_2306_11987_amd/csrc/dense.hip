// Dense (unquantised) linear layer: how each product is run, the products of few tokens, the
// activation's gradient, operands with unaligned rows, and the sums of a K that was split.
#include "dense_kernel.h"

#include <algorithm>

namespace hqlss {

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------- small products
// Few rows (a serving batch: the weight's bytes bound it) or few outputs (a small layer: a
// chain of latencies bounds it): operands go from memory straight into the registers as MFMA
// fragments, with no stage to fill first.  A wave holds 16 MT x 16 outputs and a part of K; the
// waves of a workgroup share the outputs and add their sums through LDS in a fixed order.  Rows
// may be unaligned, K anything: a unit of K that is not whole is read element by element.

// The fragments of one operand: 16 rows from r0 on, unit u of K (64 bytes of a row).
template <int DT, bool KM>
struct Direct {
  static constexpr int ES = Elem<DT>::bytes, E = kPer<DT>;
  const char* p;
  int64_t step;  // bytes of a unit
  int64_t ld, K;
  int c;
  __device__ __forceinline__ void init(const void* src, int64_t ld_, int64_t row, int64_t rows, int64_t K_, int c_) {
    row = min(row, rows - 1);
    ld = ld_ * ES;
    K = K_;
    c = c_;
    p = static_cast<const char*>(src) + (KM ? c * E * ld + row * ES : row * ld + c * 16);
    step = KM ? 4 * E * ld : 64;
  }
  __device__ __forceinline__ uint4 whole(int u) const {
    const char* const q = p + u * step;
    if constexpr (!KM) return ld_loose<DT>(q);
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (ES == 4) {
        w[j] = *reinterpret_cast<const uint32_t*>(q + j * ld);
      } else {
        w[j] = *reinterpret_cast<const uint16_t*>(q + 2 * j * ld) |
               (uint32_t)*reinterpret_cast<const uint16_t*>(q + (2 * j + 1) * ld) << 16;
      }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  // (a loop that stays one: what a short kernel runs once is mostly the fetching of its code)
  __device__ __forceinline__ uint4 part(int u) const {
    const int64_t k = ((int64_t)u * 4 + c) * E;  // this lane's first k
    const char* q = p + u * step;
    uint64_t w[2] = {0, 0};
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll 1
      for (int j = 0; j < E / 2; ++j) {
        if (k + h * (E / 2) + j < K) {
          uint64_t v;
          if constexpr (ES == 4) v = *reinterpret_cast<const uint32_t*>(q);
          else v = *reinterpret_cast<const uint16_t*>(q);
          w[h] |= v << (8 * ES * j);
        }
        q += KM ? ld : ES;
      }
    return make_uint4((uint32_t)w[0], (uint32_t)(w[0] >> 32), (uint32_t)w[1], (uint32_t)(w[1] >> 32));
  }
};

template <int DT, int MT, bool TRA, bool TRB>
__device__ __forceinline__ void direct_body(const DenseArgs& g, float* red) {  // red: [waves][16 MT rows][16]
  constexpr int E = kPer<DT>;
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nw = blockDim.x >> 6;
  const int64_t n0 = (int64_t)blockIdx.x * 16, m0 = (int64_t)blockIdx.y * (16 * MT);
  const int r = lane & 15, c = lane >> 4;
  const int units = (int)((g.K + 4 * E - 1) / (4 * E)), per = (units + nw - 1) / nw;
  const int u0 = wid * per, u1 = min(units, u0 + per);
  Direct<DT, TRB> w;
  Direct<DT, TRA> x[MT];
  w.init(g.B, g.ldb, n0 + r, g.N, g.K, c);
#pragma unroll
  for (int t = 0; t < MT; ++t) x[t].init(g.A, g.lda, m0 + 16 * t + r, g.M, g.K, c);
  v4f acc[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) acc[t] = v4f{0.f, 0.f, 0.f, 0.f};
  auto product = [&](const uint4& a, const uint4 (&b)[MT]) {
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      if constexpr (DT == kF32) {
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.x), __uint_as_float(b[t].x), acc[t], 0, 0, 0);
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.y), __uint_as_float(b[t].y), acc[t], 0, 0, 0);
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.z), __uint_as_float(b[t].z), acc[t], 0, 0, 0);
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w), __uint_as_float(b[t].w), acc[t], 0, 0, 0);
      } else if constexpr (DT == kF16) {
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b[t]), acc[t], 0, 0, 0);
      } else {
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, a), __builtin_bit_cast(v8b, b[t]), acc[t], 0, 0, 0);
      }
    }
  };
  const int full = min(u1, (int)(g.K / (4 * E)));  // whole units: their loads need no limits
  constexpr int UN = (TRA || TRB) && DT != kF32 ? 2 : MT == 1 ? 8 : 4;
  for (int u = u0; u < full; u += UN) {
    uint4 a[UN], b[UN][MT];
#pragma unroll
    for (int k = 0; k < UN; ++k) {
      if (u + k >= full) break;  // uniform: all loads of a batch go out before its first product
      a[k] = w.whole(u + k);
#pragma unroll
      for (int t = 0; t < MT; ++t) b[k][t] = x[t].whole(u + k);
    }
#pragma unroll
    for (int k = 0; k < UN; ++k) {
      if (u + k >= full) break;
      product(a[k], b[k]);
    }
  }
  if (full < u1 && u0 < u1) {
    uint4 b[MT];
    const uint4 a = w.part(full);
#pragma unroll
    for (int t = 0; t < MT; ++t) b[t] = x[t].part(full);
    product(a, b);
  }
  // a lane holds row 16 t + r, outputs 4 c ..
#pragma unroll
  for (int t = 0; t < MT; ++t)
    *reinterpret_cast<float4*>(red + ((wid * MT + t) * 16 + r) * 16 + 4 * c) = make_float4(acc[t][0], acc[t][1], acc[t][2], acc[t][3]);
  __syncthreads();
  for (int i = threadIdx.x; i < MT * 256; i += blockDim.x) {
    const int64_t m = m0 + (i >> 4), n = n0 + (i & 15);
    if (m >= g.M || n >= g.N) continue;
    float z[1] = {0.f};
    for (int q = 0; q < nw; ++q) z[0] += red[q * MT * 256 + i];
    if (g.bias) z[0] += ld1<DT>(g.bias, n);
    if (g.Z) st1<DT>(g.Z, m * g.N + n, z[0]);
    act_all(g.act, z);
    if (g.res) z[0] += ld1<DT>(g.res, m * g.N + n);
    st1<DT>(g.out, m * g.N + n, z[0]);
  }
}

template <int DT, int MT, bool TRA, bool TRB>
__global__ __launch_bounds__(1024) void direct_kernel(DenseArgs g) {
  extern __shared__ float red[];
  direct_body<DT, MT, TRA, TRB>(g, red);
}
// Both gradients of a small layer in one launch: z = 0 the input's, z = 1 the weight's.
template <int DT, int MT>
__global__ __launch_bounds__(1024) void direct_grads_kernel(DenseArgs dx, DenseArgs dw) {
  extern __shared__ float red[];
  const DenseArgs& g = blockIdx.z ? dw : dx;
  if ((int64_t)blockIdx.x * 16 >= g.N || (int64_t)blockIdx.y * 16 * MT >= g.M) return;
  if (blockIdx.z) direct_body<DT, MT, true, true>(dw, red);
  else direct_body<DT, MT, false, true>(dx, red);
}

// Rows of a workgroup / 16, its waves: about 2048 waves in flight, two units of K each at least.
struct DirectShape { int mt, nw; int64_t blocks_n, blocks_m, units; };
DirectShape direct_shape(int dt, int64_t M, int64_t N, int64_t K) {
  DirectShape d;
  d.mt = M > 16 ? 2 : 1;
  d.nw = 4;
  d.blocks_n = (N + 15) / 16;
  d.blocks_m = (M + 16 * d.mt - 1) / (16 * d.mt);
  d.units = dt == kF32 ? (K + 15) / 16 : (K + 31) / 32;
  while (d.nw < 16 && d.blocks_n * d.blocks_m * d.nw < 2048 && d.units >= 4 * d.nw) d.nw *= 2;
  return d;
}

template <int DT, int MT>
hipError_t run_direct_mt(hipStream_t s, const DenseArgs& g, const DirectShape& d) {
  const dim3 grid((unsigned)d.blocks_n, (unsigned)d.blocks_m);
  const size_t lds = (size_t)d.nw * MT * 1024;
  timing_begin(s);
  if (!g.b_kmajor) direct_kernel<DT, MT, false, false><<<grid, 64 * d.nw, lds, s>>>(g);
  else if (!g.a_kmajor) direct_kernel<DT, MT, false, true><<<grid, 64 * d.nw, lds, s>>>(g);
  else direct_kernel<DT, MT, true, true><<<grid, 64 * d.nw, lds, s>>>(g);
  timing_end(s, kKDense);
  return hipGetLastError();
}
template <int DT, int MT>
hipError_t run_direct_grads(hipStream_t s, const DenseArgs& dx, const DenseArgs& dw, const DirectShape& a, const DirectShape& b) {
  const int nw = std::max(a.nw, b.nw);
  timing_begin(s);
  direct_grads_kernel<DT, MT><<<dim3((unsigned)std::max(a.blocks_n, b.blocks_n), (unsigned)std::max(a.blocks_m, b.blocks_m), 2u),
                                64 * nw, (size_t)nw * MT * 1024, s>>>(dx, dw);
  timing_end(s, kKDense);
  return hipGetLastError();
}

template <int DT>
hipError_t run_direct(hipStream_t s, const DenseArgs& g) {
  const DirectShape d = direct_shape(DT, g.M, g.N, g.K);
  return d.mt == 1 ? run_direct_mt<DT, 1>(s, g, d) : run_direct_mt<DT, 2>(s, g, d);
}

// ---------------------------------------------------------------- split K
// out = epilogue(sum of the S partials): eight outputs a thread.
template <int DT>
__global__ __launch_bounds__(256) void dense_reduce_kernel(DenseArgs g, int S) {
  const int64_t pieces = (g.N + 7) / 8, total = g.M * pieces, plane = g.M * g.N;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t m = total >> 32 ? i / pieces : (int64_t)((uint32_t)i / (uint32_t)pieces), n = (i - m * pieces) * 8;
    const char* const base = reinterpret_cast<const char*>(g.part + m * g.N + n);
    const int left = (int)(g.N - n < 8 ? g.N - n : 8);
    float z[8], b[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      z[j] = 0.f;
      b[j] = g.bias && j < left ? ld1<DT>(g.bias, n + j) : 0.f;
    }
    for (int p = 0; p < S; p += 4) {
      float v[4][8];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (p + k < S) ld8<kF32>(base + (int64_t)(p + k) * plane * 4, 0, left, v[k]);
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (p + k < S) {
#pragma unroll
          for (int j = 0; j < 8; ++j) z[j] += v[k][j];
        }
    }
    dense_epilogue<DT>(g, m, n, z, b);
  }
}

// ---------------------------------------------------------------- unaligned rows
// dst [rows][pitch] = src [rows][cols] of 16-bit values, zeros past cols; up to two matrices a
// launch.  (The loads into LDS take 4 or 16 aligned bytes: fp32 rows always suit them.)
struct PadJob { const void* src; void* dst; int64_t rows, cols, pitch; };
__global__ __launch_bounds__(256) void pad_kernel(PadJob a, PadJob b) {
  const PadJob j = blockIdx.y ? b : a;
  const int64_t pieces = j.pitch / 8, total = j.rows * pieces;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / pieces, p = i - r * pieces;
    *reinterpret_cast<uint4*>(static_cast<char*>(j.dst) + i * 16) =
        ld_piece<kF16>(static_cast<const char*>(j.src) + r * j.cols * 2, p, j.cols);
  }
}

// ---------------------------------------------------------------- the activation's gradient
// HBM bounds it.  T lanes (a power of two) share a row's pieces of 16 bytes, or 64 of them a
// strip; a workgroup's 16 waves take 16 (64 / T) rows at a time.  Column sums are held in the
// lanes and added over the workgroup's rows through LDS.
constexpr int kAgWaves = 16;
template <int DT>
__global__ __launch_bounds__(64 * kAgWaves) void act_grad_kernel(const void* dY, const void* Z, void* G, int64_t pitch,
                                                                 void* db, float* part, int64_t N, int64_t C, int act, int T) {
  constexpr int E = kPer<DT>, ES = Elem<DT>::bytes;
  __shared__ float red[kAgWaves][64 * E];
  const int col = threadIdx.x % T, sub = threadIdx.x / T, rows = 64 * kAgWaves / T;
  const int64_t p = (int64_t)blockIdx.x * T + col, step = (int64_t)gridDim.y * rows;
  float s[E];
#pragma unroll
  for (int j = 0; j < E; ++j) s[j] = 0.f;
  int64_t r = (int64_t)blockIdx.y * rows + sub;
  // two rows ahead: nothing else moves a load above the store of the row before it
  uint4 y[2], z[2];
  auto fetch = [&](int k, int64_t row) {
    if (row >= N) return;
    y[k] = ld_piece<DT>(static_cast<const char*>(dY) + row * C * ES, p, C);
    if (act != kActNone) z[k] = ld_piece<DT>(static_cast<const char*>(Z) + row * C * ES, p, C);
  };
  auto work = [&](int k, int64_t row) {
    float v[E], w[E];
    widen_piece<DT>(y[k], v);
    if (act != kActNone) {
      widen_piece<DT>(z[k], w);
#pragma unroll
      for (int j = 0; j < E; ++j) v[j] *= act_slope(act, w[j]);
    }
    fetch(k, row + 2 * step);
    if (G) st_piece<DT>(static_cast<char*>(G) + row * pitch * ES, p, pitch, v);
#pragma unroll
    for (int j = 0; j < E; ++j) s[j] += v[j];
  };
  if (p * E < C) {
    fetch(0, r);
    fetch(1, r + step);
    for (; r < N; r += 2 * step) {
      work(0, r);
      if (r + step < N) work(1, r + step);
    }
  }
  if (!db) return;
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  for (int o = T; o < 64; o <<= 1)
#pragma unroll
    for (int j = 0; j < E; ++j) s[j] += __shfl_xor(s[j], o);
  if (lane < T) {
#pragma unroll
    for (int j = 0; j < E; ++j) red[wv][lane * E + j] = s[j];
  }
  __syncthreads();
  for (int c = threadIdx.x; c < T * E; c += 64 * kAgWaves) {
    float v = 0.f;
#pragma unroll
    for (int q = 0; q < kAgWaves; ++q) v += red[q][c];
    const int64_t n = (int64_t)blockIdx.x * T * E + c;
    if (n >= C) continue;
    if (gridDim.y == 1) st1<DT>(db, n, v);
    else part[(int64_t)blockIdx.y * C + n] = v;
  }
}

// Lanes of a row: 64, or all its pieces; few rows take fewer lanes, so that a workgroup covers
// more of them at a time and more workgroups share the columns.
int ag_lanes(int dt, int64_t N, int64_t C) {
  const int64_t P = (C * (dt == kF32 ? 4 : 2) + 15) / 16;
  int T = 1;
  while (T < 64 && T < P) T *= 2;
  while (T > 8 && 64 * kAgWaves / T < N && (P + T - 1) / T < 128 && N <= 8 * 64 * kAgWaves / 8) T /= 2;
  return T;
}

// ---------------------------------------------------------------- how a product runs
constexpr int kDirect = -1;
struct Plan { int tile, splits; };  // tile: kTile*, or kDirect

// A tile: its size, the workgroups of it that a CU holds, and in us the time that a stage (128
// bytes of K) of one takes when it is alone on its CU, the share of a CU's time it takes when it is
// not, and everything besides the stages.  Measured on full devices of 4096- and 8192-wide products.
struct TileCost { int bm, bn, per_cu; double alone, shared, fixed; };
constexpr TileCost kCost16[5] = {{256, 256, 1, 1.33, 1.33, 10.0}, {256, 128, 1, 0.74, 0.76, 5.8}, {128, 128, 2, 0.72, 0.465, 3.8},
                                 {64, 64, 3, 0.35, 0.2, 2.5}, {}};
constexpr TileCost kCost32[5] = {{}, {}, {128, 128, 2, 1.95, 1.87, 5.0}, {64, 64, 3, 0.62, 0.52, 3.0}, {32, 64, 4, 0.42, 0.26, 2.5}};

double tile_us(const TileCost& c, int64_t tiles, int64_t stages) {
  const int64_t slots = (int64_t)kCUs * c.per_cu, full = tiles / slots, rest = tiles % slots;
  auto round = [&](int64_t n) {
    const double st = (double)n * c.shared;
    return (double)stages * (st > c.alone ? st : c.alone) + c.fixed;
  };
  return (double)full * round(c.per_cu) + (rest ? round((rest + kCUs - 1) / kCUs) : 0.0);
}

// The way that is estimated to take the least.  Besides the rounds of resident workgroups a split
// of K costs a launch and its fp32 sums written and read; operands with unaligned rows a launch and
// their copy; a small product, which loads no stage, what its fragments take out of the L2.
Plan plan_of(int dt, bool a_kmajor, bool b_kmajor, int64_t M, int64_t N, int64_t K) {
  const int64_t es = dt == kF32 ? 4 : 2, ke = 128 / es, stages = (K + ke - 1) / ke;
  const DirectShape d = direct_shape(dt, M, N, K);
  Plan best{kDirect, 1};
  const bool gather = es == 2 && (a_kmajor || b_kmajor);  // two-byte loads
  const double blocks = (double)((d.blocks_n * d.blocks_m + kCUs - 1) / kCUs), at_once = 32.0 / d.nw;
  double least = 2.2 + (gather ? 3.4 : 2.0) * (blocks > at_once ? blocks / at_once : 1.0) +
                 blocks * (double)K * (double)es * 16.0 * (1 + d.mt) / (gather ? 3.0e4 : 4.2e4);
  const int64_t ra = a_kmajor ? M : K, rb = b_kmajor ? N : K;
  const double pad = es == 4 || (ra % 8 == 0 && rb % 8 == 0) ? 0.0
                     : 3.0 + (double)((ra % 8 ? M * K : 0) + (rb % 8 ? N * K : 0)) * 4.0 / 4e6;
  for (int t = dt == kF32 ? kTileMid : kTileLarge; t <= (dt == kF32 ? kTileTiny : kTileSmall); ++t) {
    const TileCost& c = dt == kF32 ? kCost32[t] : kCost16[t];
    const int64_t tiles = ((M + c.bm - 1) / c.bm) * ((N + c.bn - 1) / c.bn);
    for (int sp = 1; sp <= 16 && (sp == 1 || stages >= 4 * sp); ++sp) {
      double us = 2.0 + tile_us(c, tiles * sp, (stages + sp - 1) / sp) + pad;
      if (sp > 1) us += 4.0 + 0.3 * sp + (double)M * (double)N * 4.0 * (2 * sp) / 5.0e6;
      if (us < least) {
        least = us;
        best = {t, sp};
      }
    }
  }
  return best;
}

size_t round256(size_t x) { return (x + 255) & ~size_t(255); }
// bytes of an operand's padded copy (0: its rows are aligned)
size_t pad_bytes(int dt, int64_t rows, int64_t cols) {
  const int64_t p = dense_pitch(dt, cols);
  return p == cols ? 0 : round256((size_t)rows * p * 2);
}

template <int DT>
hipError_t reduce_t(hipStream_t s, const DenseArgs& g, int S) {
  const int64_t n = (g.M * ((g.N + 7) / 8) + 255) / 256;
  timing_begin(s);
  dense_reduce_kernel<DT><<<(unsigned)(n < 4096 ? n : 4096), 256, 0, s>>>(g, S);
  timing_end(s, kKDenseReduce);
  return hipGetLastError();
}

hipError_t run_pad(hipStream_t s, const PadJob& a, const PadJob& b) {
  const int64_t w = std::max(a.rows * a.pitch, b.rows * b.pitch) / 8, n = (w + 255) / 256;
  timing_begin(s);
  pad_kernel<<<dim3((unsigned)(n < 2048 ? n : 2048), b.rows ? 2u : 1u), 256, 0, s>>>(a, b);
  timing_end(s, kKDensePad);
  return hipGetLastError();
}

}  // namespace

int64_t dense_pitch(int dt, int64_t cols) { return dt == kF32 ? cols : (cols + 7) / 8 * 8; }

size_t dense_scratch_bytes(int dt, bool a_kmajor, bool b_kmajor, bool a_padded, int64_t M, int64_t N, int64_t K) {
  const Plan p = plan_of(dt, a_kmajor, b_kmajor, M, N, K);
  if (p.tile == kDirect) return 0;
  const size_t parts = p.splits > 1 ? round256((size_t)p.splits * M * N * sizeof(float)) : 0;
  return parts + (a_padded ? 0 : a_kmajor ? pad_bytes(dt, K, M) : pad_bytes(dt, M, K)) + (b_kmajor ? pad_bytes(dt, K, N) : pad_bytes(dt, N, K));
}

hipError_t launch_dense(hipStream_t s, int dt, const DenseArgs& args, void* scratch) {
  DenseArgs g = args;
  const Plan p = plan_of(dt, g.a_kmajor, g.b_kmajor, g.M, g.N, g.K);
  if (p.tile == kDirect) return dt == kF32 ? run_direct<kF32>(s, g) : dt == kF16 ? run_direct<kF16>(s, g) : run_direct<kBF16>(s, g);
  char* at = static_cast<char*>(scratch);
  PadJob jobs[2] = {};
  int nj = 0;
  auto pad = [&](const void*& src, int64_t& ld, int64_t rows, int64_t cols) {
    const int64_t pitch = dense_pitch(dt, cols);
    if (ld == pitch) return;  // aligned rows, or padded ones already
    jobs[nj++] = PadJob{src, at, rows, cols, pitch};
    src = at;
    ld = pitch;
    at += pad_bytes(dt, rows, cols);
  };
  pad(g.A, g.lda, g.a_kmajor ? g.K : g.M, g.a_kmajor ? g.M : g.K);
  pad(g.B, g.ldb, g.b_kmajor ? g.K : g.N, g.b_kmajor ? g.N : g.K);
  hipError_t e = hipSuccess;
  if (nj) e = run_pad(s, jobs[0], jobs[1]);
  if (e != hipSuccess) return e;
  g.part = p.splits > 1 ? reinterpret_cast<float*>(at) : nullptr;
  e = dt == kF32 ? run_dense_f32(s, g, p.tile, p.splits) : dt == kF16 ? run_dense_f16(s, g, p.tile, p.splits) : run_dense_bf16(s, g, p.tile, p.splits);
  if (e != hipSuccess || !g.part) return e;
  return dt == kF32 ? reduce_t<kF32>(s, g, p.splits) : dt == kF16 ? reduce_t<kF16>(s, g, p.splits) : reduce_t<kBF16>(s, g, p.splits);
}

hipError_t launch_dense_grads(hipStream_t s, int dt, const DenseArgs* dx, const DenseArgs* dw, void* scratch) {
  if (dx && dw && plan_of(dt, false, true, dx->M, dx->N, dx->K).tile == kDirect &&
      plan_of(dt, true, true, dw->M, dw->N, dw->K).tile == kDirect) {
    const DirectShape a = direct_shape(dt, dx->M, dx->N, dx->K), b = direct_shape(dt, dw->M, dw->N, dw->K);
    if (a.mt == 2 && b.mt == 2) {
      if (dt == kF32) return run_direct_grads<kF32, 2>(s, *dx, *dw, a, b);
      if (dt == kF16) return run_direct_grads<kF16, 2>(s, *dx, *dw, a, b);
      return run_direct_grads<kBF16, 2>(s, *dx, *dw, a, b);
    }
  }
  hipError_t e = dx ? launch_dense(s, dt, *dx, scratch) : hipSuccess;
  if (e == hipSuccess && dw) e = launch_dense(s, dt, *dw, scratch);
  return e;
}

int act_grad_parts(int dt, int64_t N, int64_t C) {
  const int T = ag_lanes(dt, N, C);
  const int64_t rows = 64 * kAgWaves / T, P = (C * (dt == kF32 ? 4 : 2) + 15) / 16, strips = (P + T - 1) / T;
  if (N <= 8 * rows) return 1;  // a chain of eight loads costs less than a second launch
  const int64_t most = strips < 512 ? 512 / strips : 1, want = (N + 4 * rows - 1) / (4 * rows);
  return (int)(want < most ? want : most);
}

hipError_t launch_act_grad(hipStream_t s, int dt, const void* dY, const void* Z, void* G, int64_t pitch, void* db,
                           float* part, int64_t N, int64_t C, int act) {
  const int T = ag_lanes(dt, N, C), parts = act_grad_parts(dt, N, C);
  const int64_t P = (C * (dt == kF32 ? 4 : 2) + 15) / 16;
  const dim3 grid((unsigned)((P + T - 1) / T), (unsigned)parts);
  timing_begin(s);
  if (dt == kF32) act_grad_kernel<kF32><<<grid, 64 * kAgWaves, 0, s>>>(dY, Z, G, pitch, db, part, N, C, act, T);
  else if (dt == kF16) act_grad_kernel<kF16><<<grid, 64 * kAgWaves, 0, s>>>(dY, Z, G, pitch, db, part, N, C, act, T);
  else act_grad_kernel<kBF16><<<grid, 64 * kAgWaves, 0, s>>>(dY, Z, G, pitch, db, part, N, C, act, T);
  timing_end(s, kKActGrad);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !db || parts == 1) return e;
  return launch_column_reduce(s, dt, part, parts, C, 1, db, nullptr);
}

}  // namespace hqlss
