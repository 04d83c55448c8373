// Dense (unquantised) linear layer: how each product is run, the products of few tokens, the
// activation's gradient, operands with unaligned rows, and the sums of a K that was split.
#include "dense_kernel.h"

namespace hqlss {

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------- products of few rows
// M <= 16 MT rows: the weight's bytes bound them, so they go from memory straight into the
// registers as MFMA fragments, once.  A wave holds 16 of the N outputs and a part of K; the
// waves of a workgroup share the 16 outputs and add their sums through LDS in a fixed order.
// Rows may be unaligned, K anything: the last piece of a row is read element by element.
template <int DT, int MT>
__global__ __launch_bounds__(1024) void skinny_kernel(DenseArgs g) {
  constexpr int ES = Elem<DT>::bytes, E = kPer<DT>;
  extern __shared__ float red[];  // [waves][16 MT rows][16]
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nw = blockDim.x >> 6;
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const int r = lane & 15, c = lane >> 4;
  const int units = (int)((g.K + 4 * E - 1) / (4 * E)), per = (units + nw - 1) / nw;
  const int u0 = wid * per, u1 = min(units, u0 + per);
  const char* const wrow = static_cast<const char*>(g.B) + min(n0 + r, g.N - 1) * g.ldb * ES;
  const char* xrow[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t)
    xrow[t] = static_cast<const char*>(g.A) + min((int64_t)(16 * t + r), g.M - 1) * g.lda * ES;
  v4f acc[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) acc[t] = v4f{0.f, 0.f, 0.f, 0.f};
  auto product = [&](const uint4& w, const uint4 (&x)[MT]) {
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      if constexpr (DT == kF32) {
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w.x), __uint_as_float(x[t].x), acc[t], 0, 0, 0);
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w.y), __uint_as_float(x[t].y), acc[t], 0, 0, 0);
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w.z), __uint_as_float(x[t].z), acc[t], 0, 0, 0);
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w.w), __uint_as_float(x[t].w), acc[t], 0, 0, 0);
      } else if constexpr (DT == kF16) {
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, w), __builtin_bit_cast(v8h, x[t]), acc[t], 0, 0, 0);
      } else {
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, w), __builtin_bit_cast(v8b, x[t]), acc[t], 0, 0, 0);
      }
    }
  };
  const int full = min(u1, (int)(g.K / (4 * E)));  // whole units: their loads need no limits
  constexpr int UN = MT == 1 ? 8 : 4;
  int u = u0;
  for (; u + UN <= full; u += UN) {
    uint4 w[UN], x[UN][MT];
#pragma unroll
    for (int k = 0; k < UN; ++k) {
      const int64_t at = ((int64_t)(u + k) * 4 + c) * 16;
      w[k] = ld_loose<DT>(wrow + at);
#pragma unroll
      for (int t = 0; t < MT; ++t) x[k][t] = ld_loose<DT>(xrow[t] + at);
    }
#pragma unroll
    for (int k = 0; k < UN; ++k) product(w[k], x[k]);
  }
  for (; u < u1; ++u) {
    uint4 x[MT];
    const uint4 w = ld_piece<DT>(wrow, (int64_t)u * 4 + c, g.K);
#pragma unroll
    for (int t = 0; t < MT; ++t) x[t] = ld_piece<DT>(xrow[t], (int64_t)u * 4 + c, g.K);
    product(w, x);
  }
  // a lane holds row 16 t + r, outputs 4 c ..
#pragma unroll
  for (int t = 0; t < MT; ++t)
    *reinterpret_cast<float4*>(red + ((wid * MT + t) * 16 + r) * 16 + 4 * c) = make_float4(acc[t][0], acc[t][1], acc[t][2], acc[t][3]);
  __syncthreads();
  for (int i = threadIdx.x; i < MT * 32; i += blockDim.x) {
    const int64_t m = i >> 1, n = n0 + 8 * (i & 1);
    if (m >= g.M || n >= g.N) continue;
    float z[8], b[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      z[j] = 0.f;
      b[j] = g.bias && n + j < g.N ? ld1<DT>(g.bias, n + j) : 0.f;
    }
    for (int w = 0; w < nw; ++w) {
      const float* const p = red + ((w * MT) * 16 + m) * 16 + 8 * (i & 1);
#pragma unroll
      for (int j = 0; j < 8; ++j) z[j] += p[j];
    }
    dense_epilogue<DT>(g, m, n, z, b);
  }
}

template <int DT, int MT>
hipError_t run_skinny(hipStream_t s, const DenseArgs& g) {
  const int64_t blocks = (g.N + 15) / 16, units = (g.K + 4 * kPer<DT> - 1) / (4 * kPer<DT>);
  int nw = 4;  // waves: about 2048 in flight, two units of K each at least
  while (nw < 16 && blocks * nw < 2048 && units >= 4 * nw) nw *= 2;
  timing_begin(s);
  skinny_kernel<DT, MT><<<(unsigned)blocks, 64 * nw, (size_t)nw * MT * 1024, s>>>(g);
  timing_end(s, kKDense);
  return hipGetLastError();
}

// ---------------------------------------------------------------- split K
// out = epilogue(sum of the S partials): eight outputs a thread.
template <int DT>
__global__ __launch_bounds__(256) void dense_reduce_kernel(DenseArgs g, int S) {
  const int64_t pieces = (g.N + 7) / 8, total = g.M * pieces;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t m = i / pieces, n = (i - m * pieces) * 8;
    float z[8], b[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      z[j] = 0.f;
      b[j] = g.bias && n + j < g.N ? ld1<DT>(g.bias, n + j) : 0.f;
    }
#pragma unroll 4
    for (int p = 0; p < S; ++p) {
      float v[8];
      ld_row8<kF32>(g.part + (int64_t)p * g.M * g.N, m, n, g.N, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) z[j] += v[j];
    }
    dense_epilogue<DT>(g, m, n, z, b);
  }
}

// ---------------------------------------------------------------- unaligned rows
// dst [rows][pitch] = src [rows][cols], zeros past cols; up to two matrices a launch.
struct PadJob { const void* src; void* dst; int64_t rows, cols, pitch; };
template <int DT>
__global__ __launch_bounds__(256) void pad_kernel(PadJob a, PadJob b) {
  const PadJob j = blockIdx.y ? b : a;
  constexpr int E = kPer<DT>, ES = Elem<DT>::bytes;
  const int64_t pieces = j.pitch / E, total = j.rows * pieces;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / pieces, p = i - r * pieces;
    *reinterpret_cast<uint4*>(static_cast<char*>(j.dst) + i * 16) =
        ld_piece<DT>(static_cast<const char*>(j.src) + r * j.cols * ES, p, j.cols);
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
  __shared__ float red[64 * kAgWaves * E];
  const int col = threadIdx.x % T, sub = threadIdx.x / T, rows = 64 * kAgWaves / T;
  const int64_t p = (int64_t)blockIdx.x * T + col;
  const bool mine = p * E < C;
  float s[E];
#pragma unroll
  for (int j = 0; j < E; ++j) s[j] = 0.f;
  if (mine) {
#pragma unroll 2
    for (int64_t r = (int64_t)blockIdx.y * rows + sub; r < N; r += (int64_t)gridDim.y * rows) {
      float v[E], z[E];
      widen_piece<DT>(ld_piece<DT>(static_cast<const char*>(dY) + r * C * ES, p, C), v);
      if (act != kActNone) {
        widen_piece<DT>(ld_piece<DT>(static_cast<const char*>(Z) + r * C * ES, p, C), z);
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] *= act_slope(act, z[j]);
      }
      if (G) st_piece<DT>(static_cast<char*>(G) + r * pitch * ES, p, pitch, v);
#pragma unroll
      for (int j = 0; j < E; ++j) s[j] += v[j];
    }
  }
  if (!db) return;
#pragma unroll
  for (int j = 0; j < E; ++j) red[(sub * T + col) * E + j] = s[j];
  __syncthreads();
  for (int c = threadIdx.x; c < T * E; c += 64 * kAgWaves) {
    float v = 0.f;
    for (int q = 0; q < rows; ++q) v += red[q * T * E + c];
    const int64_t n = (int64_t)blockIdx.x * T * E + c;
    if (n >= C) continue;
    if (gridDim.y == 1) st1<DT>(db, n, v);
    else part[(int64_t)blockIdx.y * C + n] = v;
  }
}

int ag_lanes(int dt, int64_t C) {
  const int64_t P = (C * (dt == kF32 ? 4 : 2) + 15) / 16;
  int T = 1;
  while (T < 64 && T < P) T *= 2;
  return T;
}

// ---------------------------------------------------------------- how a product runs
struct Plan { int tile, splits; };  // tile < 0: the kernel of few rows

// Times in us of a workgroup's stage (128 bytes of K) and of what it does besides, on a full
// device, and the workgroups resident at once; measured on 16-bit products.
struct TileCost { int bm, bn, slots; double stage, fixed; };
constexpr TileCost kCost16[3] = {{256, 256, 256, 1.25, 9.0}, {128, 128, 512, 0.9, 5.0}, {64, 64, 512, 0.45, 3.5}};
constexpr TileCost kCost32[3] = {{0, 0, 0, 0, 0}, {128, 128, 512, 7.2, 5.0}, {64, 64, 512, 1.9, 3.5}};

// The tile and the number of parts of K that are estimated to take the least: rounds of the
// resident workgroups, and where K is split, its fp32 sums written and read again.
Plan plan_of(int dt, bool a_kmajor, bool b_kmajor, int64_t M, int64_t N, int64_t K) {
  if (M <= 32 && !a_kmajor && !b_kmajor) return {-1, 1};
  const int64_t ke = dt == kF32 ? 32 : 64, stages = (K + ke - 1) / ke;
  Plan best{kTileMid, 1};
  double least = 1e300;
  for (int t = dt == kF32 ? kTileMid : kTileLarge; t <= kTileSmall; ++t) {
    const TileCost& c = dt == kF32 ? kCost32[t] : kCost16[t];
    const int64_t tiles = ((M + c.bm - 1) / c.bm) * ((N + c.bn - 1) / c.bn);
    for (int sp = 1; sp <= 16 && (sp == 1 || stages >= 4 * sp); ++sp) {
      const int64_t rounds = (tiles * sp + c.slots - 1) / c.slots, per = (stages + sp - 1) / sp;
      double us = (double)rounds * ((double)per * c.stage + c.fixed);
      if (sp > 1) us += 4.0 + (double)M * (double)N * 4.0 * (sp * 2) / 4.0e6;
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
  return p == cols ? 0 : round256((size_t)rows * p * (dt == kF32 ? 4 : 2));
}

template <int DT>
hipError_t reduce_t(hipStream_t s, const DenseArgs& g, int S) {
  const int64_t n = (g.M * ((g.N + 7) / 8) + 255) / 256;
  timing_begin(s);
  dense_reduce_kernel<DT><<<(unsigned)(n < 4096 ? n : 4096), 256, 0, s>>>(g, S);
  timing_end(s, kKDenseReduce);
  return hipGetLastError();
}

template <int DT>
hipError_t pad_t(hipStream_t s, const PadJob& a, const PadJob& b) {
  const int64_t w = (a.rows * a.pitch > b.rows * b.pitch ? a.rows * a.pitch : b.rows * b.pitch) / kPer<DT>;
  const int64_t n = (w + 255) / 256;
  timing_begin(s);
  pad_kernel<DT><<<dim3((unsigned)(n < 2048 ? n : 2048), b.rows ? 2u : 1u), 256, 0, s>>>(a, b);
  timing_end(s, kKDensePad);
  return hipGetLastError();
}

}  // namespace

int64_t dense_pitch(int dt, int64_t cols) {
  const int64_t e = dt == kF32 ? 4 : 8;
  return (cols + e - 1) / e * e;
}

size_t dense_scratch_bytes(int dt, bool a_kmajor, bool b_kmajor, bool a_padded, int64_t M, int64_t N, int64_t K) {
  const Plan p = plan_of(dt, a_kmajor, b_kmajor, M, N, K);
  if (p.tile < 0) return 0;
  const size_t parts = p.splits > 1 ? round256((size_t)p.splits * M * N * sizeof(float)) : 0;
  return parts + (a_padded ? 0 : a_kmajor ? pad_bytes(dt, K, M) : pad_bytes(dt, M, K)) + (b_kmajor ? pad_bytes(dt, K, N) : pad_bytes(dt, N, K));
}

hipError_t launch_dense(hipStream_t s, int dt, const DenseArgs& args, void* scratch) {
  DenseArgs g = args;
  const Plan p = plan_of(dt, g.a_kmajor, g.b_kmajor, g.M, g.N, g.K);
  if (p.tile < 0) {
    const bool two = g.M > 16;
    if (dt == kF32) return two ? run_skinny<kF32, 2>(s, g) : run_skinny<kF32, 1>(s, g);
    if (dt == kF16) return two ? run_skinny<kF16, 2>(s, g) : run_skinny<kF16, 1>(s, g);
    return two ? run_skinny<kBF16, 2>(s, g) : run_skinny<kBF16, 1>(s, g);
  }
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
  if (nj) e = dt == kF32 ? pad_t<kF32>(s, jobs[0], jobs[1]) : dt == kF16 ? pad_t<kF16>(s, jobs[0], jobs[1]) : pad_t<kBF16>(s, jobs[0], jobs[1]);
  if (e != hipSuccess) return e;
  g.part = p.splits > 1 ? reinterpret_cast<float*>(at) : nullptr;
  e = dt == kF32 ? run_dense_f32(s, g, p.tile, p.splits) : dt == kF16 ? run_dense_f16(s, g, p.tile, p.splits) : run_dense_bf16(s, g, p.tile, p.splits);
  if (e != hipSuccess || !g.part) return e;
  return dt == kF32 ? reduce_t<kF32>(s, g, p.splits) : dt == kF16 ? reduce_t<kF16>(s, g, p.splits) : reduce_t<kBF16>(s, g, p.splits);
}

int act_grad_parts(int dt, int64_t N, int64_t C) {
  const int T = ag_lanes(dt, C);
  const int64_t rows = 64 * kAgWaves / T, P = (C * (dt == kF32 ? 4 : 2) + 15) / 16, strips = (P + T - 1) / T;
  if (N <= 8 * rows) return 1;  // a chain of eight loads costs less than a second launch
  const int64_t most = strips < 512 ? 512 / strips : 1, want = (N + 4 * rows - 1) / (4 * rows);
  return (int)(want < most ? want : most);
}

hipError_t launch_act_grad(hipStream_t s, int dt, const void* dY, const void* Z, void* G, int64_t pitch, void* db,
                           float* part, int64_t N, int64_t C, int act) {
  const int T = ag_lanes(dt, C), parts = act_grad_parts(dt, N, C);
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
