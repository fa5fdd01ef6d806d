// stb_gemm_i8: the linear layer in 8 bits, Y[t][i] = x_scale[t] w_scale[i] sum_j W[i][j] X[t][j] (+ bias[i]).
// The sums are whole numbers in int32, so every order of them, every split of K and every kernel gives the same bits.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/stb.h"
#include "stb_ptx.cuh"

namespace cg = cooperative_groups;

namespace stb {

struct I8Args {
  const int8_t *W, *X;
  const float *w_scale, *bias, *x_scale;
  void* Y;
  size_t ldw, ldx, ldy;
  int n, m, T, ydt;
};

__device__ __forceinline__ float i8_value(int sum, float xs, float ws, float bias, bool with_bias) {
  const float v = __fmul_rn(__fmul_rn(__int2float_rn(sum), xs), ws);
  return with_bias ? __fadd_rn(v, bias) : v;
}
__device__ __forceinline__ void i8_store(void* Y, size_t at, int ydt, float v) {
  if (ydt == STB_F32) static_cast<float*>(Y)[at] = v;
  else if (ydt == STB_F16) static_cast<__half*>(Y)[at] = __float2half_rn(v);
  else static_cast<__nv_bfloat16*>(Y)[at] = __float2bfloat16_rn(v);
}

// D(16x8, int32) += A(16x32, int8, row) * B(32x8, int8, col)
__device__ __forceinline__ void mma_i8(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 16 bytes of weights, which this call reads once
__device__ __forceinline__ uint4 ldg_stream_v4(const void* p) {
  uint4 v;
  asm("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
// The bytes [at, at + 16) of a row of m, zeros behind its end (nothing there is read).
__device__ __noinline__ uint4 row_end(const int8_t* row, int at, int m) {
  uint32_t w[4] = {0, 0, 0, 0};
  for (int i = 0; i < 16 && at + i < m; ++i) w[i >> 2] |= (uint32_t)(uint8_t)row[at + i] << (8 * (i & 3));
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Few tokens: the weights are read once and the tensor cores take them as they come.  16 rows of W and up to 8 NB tokens per CTA; its
// eight warps take every eighth 64 columns of the CTA's part of K.  Lane 4 g + t reads 16 bytes at column 16 t of the rows g and g + 8 and of token
// g: the same columns of both operands are then in the same place of two instructions, which is all that an order of K has to satisfy.
// The sums of the warps meet in shared memory, those of the `ksplit` CTAs of a cluster in that of its first.
constexpr int kI8Warps = 8, kI8Rows = 16, kI8Step = 64;
template <int NB>
__global__ void __launch_bounds__(32 * kI8Warps)
gemv_i8_kernel(const I8Args args, int ksplit) {
  __shared__ int part[kI8Warps][NB][4][32];
  __shared__ int whole[8][NB][4][32];
  const int8_t *W = args.W, *X = args.X;
  const float *w_scale = args.w_scale, *x_scale = args.x_scale, *bias = args.bias;
  if (ksplit > 1) cluster_arrive();          // (before a CTA writes into another's shared memory, that one has started)
  begin_after(W, X, w_scale, x_scale, bias);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int kz = (int)blockIdx.x % ksplit, row0 = (int)(blockIdx.x / ksplit) * kI8Rows, tok0 = (int)blockIdx.y * 8 * NB;
  const int m = args.m, steps = (m + kI8Step - 1) / kI8Step;
  const bool r0 = row0 + g < args.n, r1 = row0 + g + 8 < args.n;
  const int8_t *w0 = W + (size_t)(r0 ? row0 + g : 0) * args.ldw, *w1 = W + (size_t)(r1 ? row0 + g + 8 : 0) * args.ldw;
  int acc[NB][4];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[b][k] = 0;
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll 4
  for (int s = kz * kI8Warps + warp; s < steps; s += ksplit * kI8Warps) {
    const int at = s * kI8Step + 16 * t;
    const bool full = at + 16 <= m;
    const uint4 a0 = !r0 ? zero : (full ? ldg_stream_v4(w0 + at) : row_end(w0, at, m)), a1 = !r1 ? zero : (full ? ldg_stream_v4(w1 + at) : row_end(w1, at, m));
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int tok = tok0 + 8 * b + g;
      uint4 x = zero;
      if (tok < args.T) {
        const int8_t* xr = X + (size_t)tok * args.ldx;
        x = full ? ldg_nc_v4(xr + at) : row_end(xr, at, m);
      }
      mma_i8(acc[b], a0.x, a1.x, a0.y, a1.y, x.x, x.y);
      mma_i8(acc[b], a0.z, a1.z, a0.w, a1.w, x.z, x.w);
    }
  }
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int k = 0; k < 4; ++k) part[warp][b][k][lane] = acc[b][k];
  __syncthreads();
  if (ksplit > 1) cluster_wait();
  for (int i = threadIdx.x; i < NB * 128; i += 32 * kI8Warps) {
    int sum = 0;
#pragma unroll
    for (int w = 0; w < kI8Warps; ++w) sum += part[w][i >> 7][(i >> 5) & 3][i & 31];
    if (ksplit == 1) part[0][i >> 7][(i >> 5) & 3][i & 31] = sum;
    else cg::this_cluster().map_shared_rank(&whole[0][0][0][0], 0)[(kz * NB * 128) + i] = sum;
  }
  if (ksplit > 1) {
    cluster_arrive();
    cluster_wait();
    if (kz != 0) return;
  } else {
    __syncthreads();
  }
  // accumulator k of lane 4 g + t is row g + 8 (k / 2), token 2 t + k % 2
  for (int i = threadIdx.x; i < NB * 128; i += 32 * kI8Warps) {
    const int row = i & 15, tl = i >> 4, tok = tok0 + tl;
    const int b = tl >> 3, k = ((row >> 3) << 1) | (tl & 1), ln = 4 * (row & 7) + ((tl & 7) >> 1);
    if (row0 + row >= args.n || tok >= args.T) continue;
    int sum = 0;
    if (ksplit == 1) sum = part[0][b][k][ln];
    else for (int z = 0; z < ksplit; ++z) sum += whole[z][b][k][ln];
    const int r = row0 + row;
    i8_store(args.Y, (size_t)tok * args.ldy + r, args.ydt, i8_value(sum, x_scale[tok], w_scale[r], bias ? bias[r] : 0.0f, bias != nullptr));
  }
}

template <int NB>
static cudaError_t launch_gemv_i8(const I8Args& a, cudaStream_t s) {
  const int groups = (a.n + kI8Rows - 1) / kI8Rows, steps = (a.m + kI8Step - 1) / kI8Step;
  int ksplit = 1;
  while (ksplit < 8 && groups * ksplit < 148 * 2 && steps / (2 * ksplit) >= 2 * kI8Warps) ksplit *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(groups * ksplit), (unsigned)((a.T + 8 * NB - 1) / (8 * NB)));
  cfg.blockDim = dim3(32 * kI8Warps);
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)ksplit; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
  cfg.attrs = at; cfg.numAttrs = ksplit > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, gemv_i8_kernel<NB>, a, ksplit);
}

}  // namespace stb

extern "C" int stb_gemm_i8(const int8_t* W, size_t ldw, const float* w_scale, const float* bias, int n, int m, const int8_t* X, size_t ldx,
                           const float* x_scale, int T, void* Y, stb_dtype ydt, size_t ldy, int* dev_status, void* stream) {
  (void)dev_status;
  if (!W || !w_scale || !X || !x_scale || !Y) return STB_ERR_ARG;
  if (n < 1 || m < 1 || T < 1 || m > 131071) return STB_ERR_SHAPE;
  if (ydt != STB_F32 && ydt != STB_F16 && ydt != STB_BF16) return STB_ERR_UNSUPPORTED;
  if (ldw < (size_t)m || ldx < (size_t)m || ldy < (size_t)n || (ldw % 16) != 0 || (ldx % 16) != 0) return STB_ERR_ARG;
  const uintptr_t small = ydt == STB_F32 ? 3u : 1u;
  if (((reinterpret_cast<uintptr_t>(W) | reinterpret_cast<uintptr_t>(X)) & 15u) || (reinterpret_cast<uintptr_t>(Y) & small) ||
      ((reinterpret_cast<uintptr_t>(w_scale) | reinterpret_cast<uintptr_t>(x_scale) | reinterpret_cast<uintptr_t>(bias)) & 3u))
    return STB_ERR_ARG;
  const stb::I8Args a = {W, X, w_scale, bias, x_scale, Y, ldw, ldx, ldy, n, m, T, ydt};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = T <= 8 ? stb::launch_gemv_i8<1>(a, s) : (T <= 16 ? stb::launch_gemv_i8<2>(a, s) : stb::launch_gemv_i8<4>(a, s));
  return e == cudaSuccess ? STB_OK : STB_ERR_CUDA;
}
