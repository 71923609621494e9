// Float32 contraction on CUDA cores for the scoring and distillation calls with float32 operands that are too small for the
// tensor cores' planes to pay, or ask for this path:
//   C[m, n] (+)= sum_k A(m, k) B(k, n)
// with either operand contiguous along k or along its own index.  Blocks of 256 threads compute 128 x 128 outputs,
// 8 x 8 a thread in two-element multiply-adds, from 16-deep slices of both operands that are double-buffered in shared
// memory ([k][index], so that a thread's eight values are two 128-bit loads); the next slice is in registers while
// one is multiplied.  Few output tiles and a long k (d_hidden: 8 tiles over 4096 vocabulary entries at the test size)
// are cut over k into parts that a second kernel adds in order.
// 512 x 4096 outputs, k 256: 29 us, 37 TFLOP/s, half of what the float32 units can do: 128 tiles on 148 multiprocessors, and
// two warps a scheduler hide neither the 16 slices' barriers nor the start.  128 x 64 tiles took 32 us, 512 threads 35,
// scalar multiply-adds 33, values of the next k fetched ahead into registers 30.
#pragma once

#include "common.cuh"
#include "simt.cuh"
#include "umma_gemm.cuh"

namespace ulorl {

constexpr int kSgTile = 128;
constexpr int kSgK = 16;
constexpr int kSgThreads = 256;
constexpr int kSgPad = 4;

struct SgemmArgs {
  const float* A;
  const float* B;
  float* C;
  size_t lda, ldb, ldc;     // elements between consecutive values of the operand's non-contiguous index; multiples of 4
  int M, N, K;
  int k_part;               // k values a part covers (multiple of kSgK); part blockIdx.z writes at C + z * part_stride
  size_t part_stride;
  int accumulate;
};

// One slice of an operand, 128 x 16: two float4 a thread.  kAlongK: rows of the index, 4 values of k; else rows of k,
// 4 values of the index.  Rows are padded to a multiple of 4 values in memory, so a vector that starts inside one may
// be read; values of k at or beyond k_end count as zero.
template <bool kAlongK>
__device__ __forceinline__ void sg_load(const float* __restrict__ X, size_t ld, int i0, int n_index, int k0, int k_end,
                                        float4 (&v)[2]) {
  const int tid = threadIdx.x;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    v[q] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (kAlongK) {
      const int i = i0 + (tid >> 2) + 64 * q, k = k0 + (tid & 3) * 4;
      if (i < n_index && k < k_end) {
        v[q] = *reinterpret_cast<const float4*>(X + (size_t)i * ld + k);
        if (k + 1 >= k_end) v[q].y = 0.f;
        if (k + 2 >= k_end) v[q].z = 0.f;
        if (k + 3 >= k_end) v[q].w = 0.f;
      }
    } else {
      const int k = k0 + (tid >> 5) + 8 * q, i = i0 + (tid & 31) * 4;
      if (i < n_index && k < k_end) v[q] = *reinterpret_cast<const float4*>(X + (size_t)k * ld + i);
    }
  }
}
template <bool kAlongK>
__device__ __forceinline__ void sg_store(float (*S)[kSgTile + kSgPad], const float4 (&v)[2]) {
  const int tid = threadIdx.x;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    if (kAlongK) {
      const int i = (tid >> 2) + 64 * q, k = (tid & 3) * 4;
      S[k][i] = v[q].x; S[k + 1][i] = v[q].y; S[k + 2][i] = v[q].z; S[k + 3][i] = v[q].w;
    } else {
      *reinterpret_cast<float4*>(&S[(tid >> 5) + 8 * q][(tid & 31) * 4]) = v[q];
    }
  }
}

template <bool kAAlongK, bool kBAlongK>
__global__ void __launch_bounds__(kSgThreads)
sgemm_kernel(const SgemmArgs a) {
  __shared__ __align__(16) float As[2][kSgK][kSgTile + kSgPad];
  __shared__ __align__(16) float Bs[2][kSgK][kSgTile + kSgPad];
  int m0, n0;
  tile_of_block(a.N, kSgTile, m0, n0);
  const int k_begin = blockIdx.z * a.k_part, k_end = min(a.K, k_begin + a.k_part);
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float2 acc[8][4] = {};
  float4 ra[2], rb[2];
  sg_load<kAAlongK>(a.A, a.lda, m0, a.M, k_begin, k_end, ra);
  sg_load<kBAlongK>(a.B, a.ldb, n0, a.N, k_begin, k_end, rb);
  sg_store<kAAlongK>(As[0], ra);
  sg_store<kBAlongK>(Bs[0], rb);
  __syncthreads();
  int buf = 0;
  for (int k0 = k_begin; k0 < k_end; k0 += kSgK, buf ^= 1) {
    const bool more = k0 + kSgK < k_end;
    if (more) {
      sg_load<kAAlongK>(a.A, a.lda, m0, a.M, k0 + kSgK, k_end, ra);
      sg_load<kBAlongK>(a.B, a.ldb, n0, a.N, k0 + kSgK, k_end, rb);
    }
#pragma unroll
    for (int k = 0; k < kSgK; ++k) {
      float x[8];
      float2 y[4];
      *reinterpret_cast<float4*>(&x[0]) = *reinterpret_cast<const float4*>(&As[buf][k][ty * 4]);
      *reinterpret_cast<float4*>(&x[4]) = *reinterpret_cast<const float4*>(&As[buf][k][64 + ty * 4]);
      *reinterpret_cast<float4*>(&y[0]) = *reinterpret_cast<const float4*>(&Bs[buf][k][tx * 4]);
      *reinterpret_cast<float4*>(&y[2]) = *reinterpret_cast<const float4*>(&Bs[buf][k][64 + tx * 4]);
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fma2(make_float2(x[i], x[i]), y[j], acc[i][j]);
    }
    if (more) {
      sg_store<kAAlongK>(As[buf ^ 1], ra);
      sg_store<kBAlongK>(Bs[buf ^ 1], rb);
    }
    __syncthreads();
  }
  float* C = a.C + (size_t)blockIdx.z * a.part_stride;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int m = m0 + (i < 4 ? ty * 4 + i : 64 + ty * 4 + i - 4);
    if (m >= a.M) continue;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int n = n0 + 64 * h + tx * 4;
      float* dst = C + (size_t)m * a.ldc + n;
      float4 v = make_float4(acc[i][2 * h].x, acc[i][2 * h].y, acc[i][2 * h + 1].x, acc[i][2 * h + 1].y);
      if (n + 3 < a.N) {
        if (a.accumulate) {
          const float4 o = *reinterpret_cast<const float4*>(dst);
          v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
        }
        *reinterpret_cast<float4*>(dst) = v;
      } else {
        const float w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (n + j < a.N) dst[j] = a.accumulate ? dst[j] + w[j] : w[j];
      }
    }
  }
}

// out[i] (+)= sum of the parts' values, in the order of the parts; n a multiple of 4.
__global__ void sgemm_parts_kernel(const float* __restrict__ parts, int n_parts, size_t part_stride, size_t n,
                                   float* __restrict__ out, int accumulate) {
  const size_t i = ((size_t)blockIdx.x * blockDim.x + threadIdx.x) * 4;
  if (i >= n) return;
  float4 s = accumulate ? *reinterpret_cast<const float4*>(out + i) : make_float4(0.f, 0.f, 0.f, 0.f);
  for (int p = 0; p < n_parts; ++p) {
    const float4 x = *reinterpret_cast<const float4*>(parts + (size_t)p * part_stride + i);
    s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
  }
  *reinterpret_cast<float4*>(out + i) = s;
}

}  // namespace ulorl
