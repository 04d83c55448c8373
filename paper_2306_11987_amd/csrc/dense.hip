// Dense (unquantised) linear layer: products in fp32, fp16 or bf16 on the MFMA with fp32
// accumulation, bias, activation and residual in the epilogue; the activation's gradient.
#include "common.h"
#include "launch.h"

namespace hqlss {

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));

template <int DT>
__device__ __forceinline__ float ld1(const void* p, int64_t i) {
  if constexpr (DT == kF32) return static_cast<const float*>(p)[i];
  else if constexpr (DT == kF16) return h2f(static_cast<const uint16_t*>(p)[i]);
  else return bf2f(static_cast<const uint16_t*>(p)[i]);
}

__device__ __forceinline__ float act_of(int act, float z) {
  switch (act) {
    case kActRelu: return z > 0.f ? z : (z != z ? z : 0.f);
    case kActGelu: return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
    case kActGeluTanh: return 0.5f * z * (1.f + tanhf(0.79788456080286536f * (z + 0.044715f * z * z * z)));
    case kActSilu: return z / (1.f + expf(-z));
    case kActTanh: return tanhf(z);
  }
  return z;
}
__device__ __forceinline__ float act_slope(int act, float z) {
  switch (act) {
    case kActRelu: return z > 0.f ? 1.f : (z != z ? z : 0.f);
    case kActGelu:
      return 0.5f * (1.f + erff(z * 0.70710678118654752f)) + z * expf(-0.5f * z * z) * 0.39894228040143268f;
    case kActGeluTanh: {
      const float t = tanhf(0.79788456080286536f * (z + 0.044715f * z * z * z));
      return 0.5f * (1.f + t) + 0.5f * z * (1.f - t * t) * (0.79788456080286536f * (1.f + 0.134145f * z * z));
    }
    case kActSilu: {
      const float p = 1.f / (1.f + expf(-z));
      return p * (1.f + z * (1.f - p));
    }
    case kActTanh: {
      const float t = tanhf(z);
      return 1.f - t * t;
    }
  }
  return 1.f;
}

// 64 x 64 tile of a workgroup of four waves (16 rows x 64 columns each), 32 k a stage, elements
// staged one by one: any layout, any size.
template <int DT>
__global__ __launch_bounds__(256) void dense_kernel(DenseArgs g) {
  using Raw = typename std::conditional<DT == kF32, uint32_t, uint16_t>::type;
  constexpr int KS = 32, PITCH = KS + 16 / (int)sizeof(Raw);
  __shared__ Raw sa[64 * PITCH], sb[64 * PITCH];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int64_t m0 = (int64_t)blockIdx.y * 64, n0 = (int64_t)blockIdx.x * 64;
  v4f acc[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) acc[j] = v4f{0.f, 0.f, 0.f, 0.f};
  const Raw* const A = static_cast<const Raw*>(g.A);
  const Raw* const B = static_cast<const Raw*>(g.B);
  for (int64_t k0 = 0; k0 < g.K; k0 += KS) {
    for (int i = tid; i < 64 * KS; i += 256) {
      const int ra = g.a_kmajor ? i % 64 : i / KS, ka = g.a_kmajor ? i / 64 : i % KS;
      const int rb = g.b_kmajor ? i % 64 : i / KS, kb = g.b_kmajor ? i / 64 : i % KS;
      const int64_t m = m0 + ra, n = n0 + rb;
      sa[ra * PITCH + ka] = m < g.M && k0 + ka < g.K ? A[g.a_kmajor ? (k0 + ka) * g.lda + m : m * g.lda + k0 + ka] : Raw(0);
      sb[rb * PITCH + kb] = n < g.N && k0 + kb < g.K ? B[g.b_kmajor ? (k0 + kb) * g.ldb + n : n * g.ldb + k0 + kb] : Raw(0);
    }
    __syncthreads();
    if constexpr (DT == kF32) {
#pragma unroll
      for (int k = 0; k < KS; k += 4) {
        const float a = __uint_as_float(sa[(16 * w + (lane & 15)) * PITCH + k + (lane >> 4)]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float b = __uint_as_float(sb[(16 * j + (lane & 15)) * PITCH + k + (lane >> 4)]);
          acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, acc[j], 0, 0, 0);
        }
      }
    } else {
      const v8s a = *reinterpret_cast<const v8s*>(sa + (16 * w + (lane & 15)) * PITCH + 8 * (lane >> 4));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const v8s b = *reinterpret_cast<const v8s*>(sb + (16 * j + (lane & 15)) * PITCH + 8 * (lane >> 4));
        if constexpr (DT == kF16)
          acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), acc[j], 0, 0, 0);
        else
          acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, a), __builtin_bit_cast(v8b, b), acc[j], 0, 0, 0);
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t m = m0 + 16 * w + 4 * (lane >> 4) + r, n = n0 + 16 * j + (lane & 15);
      if (m >= g.M || n >= g.N) continue;
      float z = acc[j][r];
      if (g.bias) z += ld1<DT>(g.bias, n);
      if (g.Z) store1<DT>(g.Z, m * g.N + n, z);
      z = act_of(g.act, z);
      if (g.res) z += ld1<DT>(g.res, m * g.N + n);
      store1<DT>(g.out, m * g.N + n, z);
    }
}

constexpr int kActRows = 64;  // rows of a workgroup at least
template <int DT>
__global__ __launch_bounds__(256) void act_grad_kernel(const void* dY, const void* Z, void* G, float* part, int64_t N,
                                                       int64_t C, int act) {
  __shared__ float red[4][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t c = (int64_t)blockIdx.x * 64 + lane;
  float s = 0.f;
  if (c < C)
    for (int64_t r = (int64_t)blockIdx.y * 4 + w; r < N; r += (int64_t)gridDim.y * 4) {
      float v = ld1<DT>(dY, r * C + c);
      if (act != kActNone) v *= act_slope(act, ld1<DT>(Z, r * C + c));
      if (G) store1<DT>(G, r * C + c, v);
      s += v;
    }
  if (!part) return;
  red[w][lane] = s;
  __syncthreads();
  if (w == 0 && c < C) part[(int64_t)blockIdx.y * C + c] = (red[0][lane] + red[1][lane]) + (red[2][lane] + red[3][lane]);
}

}  // namespace

hipError_t launch_dense(hipStream_t s, int dt, const DenseArgs& g) {
  const dim3 grid((unsigned)((g.N + 63) / 64), (unsigned)((g.M + 63) / 64));
  timing_begin(s);
  if (dt == kF32) dense_kernel<kF32><<<grid, 256, 0, s>>>(g);
  else if (dt == kF16) dense_kernel<kF16><<<grid, 256, 0, s>>>(g);
  else dense_kernel<kBF16><<<grid, 256, 0, s>>>(g);
  timing_end(s, kKDense);
  return hipGetLastError();
}

int act_grad_parts(int64_t N, int64_t C) {
  (void)C;
  const int64_t p = (N + kActRows - 1) / kActRows;
  return (int)(p < 128 ? p : 128);
}

hipError_t launch_act_grad(hipStream_t s, int dt, const void* dY, const void* Z, void* G, float* part, int64_t N,
                           int64_t C, int act) {
  const dim3 grid((unsigned)((C + 63) / 64), (unsigned)act_grad_parts(N, C));
  timing_begin(s);
  if (dt == kF32) act_grad_kernel<kF32><<<grid, 256, 0, s>>>(dY, Z, G, part, N, C, act);
  else if (dt == kF16) act_grad_kernel<kF16><<<grid, 256, 0, s>>>(dY, Z, G, part, N, C, act);
  else act_grad_kernel<kBF16><<<grid, 256, 0, s>>>(dY, Z, G, part, N, C, act);
  timing_end(s, kKActGrad);
  return hipGetLastError();
}

}  // namespace hqlss
