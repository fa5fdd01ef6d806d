// stb_gemm_i8: the linear layer in 8 bits, Y[t][i] = x_scale[t] w_scale[i] sum_j W[i][j] X[t][j] (+ bias[i]).
// The sums are whole numbers in int32, so every order of them, every split of K and every kernel gives the same bits.
#include <cooperative_groups.h>
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/stb.h"
#include "stb_ptx.cuh"
#include "stb_tcgen05.cuh"

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


// ---- the 5th-generation tensor cores ------------------------------------------------------------------------------------------------
// kind::i8 of tcgen05.mma: signed bytes, int32 in tensor memory.  W is the M side (128 rows of a CTA, the lanes of tensor memory), the
// tokens are the N side, K comes in stages of 128 columns = one swizzled row of 128 bytes: four instructions of K = 32 each.  Both operands arrive by
// TMA as they lie in memory; what a box has beyond n, m or T is zeros.
constexpr int kI8M = 128, kI8K = 128;
constexpr uint32_t kI8StageA = kI8M * kI8K;
constexpr uint32_t kI8SmemMax = 232448;
// Instruction descriptor: D int32 (2), A and B signed (1), both K-major.
__host__ __device__ inline uint32_t i8_idesc(int M, int bn) { return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(bn >> 3) << 17) | ((uint32_t)(M >> 4) << 24); }

template <int kGroup>
__device__ __forceinline__ void umma_i8(uint32_t d_tmem, uint32_t adesc_lo, uint32_t bdesc_lo, uint32_t desc_hi, uint32_t idesc, uint32_t accumulate) {
  if (kGroup == 1)
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
                 "tcgen05.mma.cta_group::1.kind::i8 [%0], da, db, %4, p;\n\t}"
                 ::"r"(d_tmem), "r"(adesc_lo), "r"(bdesc_lo), "r"(desc_hi), "r"(idesc), "r"(accumulate) : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
                 "tcgen05.mma.cta_group::2.kind::i8 [%0], da, db, %4, p;\n\t}"
                 ::"r"(d_tmem), "r"(adesc_lo), "r"(bdesc_lo), "r"(desc_hi), "r"(idesc), "r"(accumulate) : "memory");
}
// the same place in the shared memory of another CTA of the cluster
__device__ __forceinline__ uint32_t smem_of_rank(uint32_t a, uint32_t rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
  return r;
}

// Four channels side by side, from `r` on: their scales, and where a token's results go.
struct I8Channels {
  float ws[4], b[4];
  int r;
  bool whole;             // all four exist and their results can be stored at once
  __device__ __forceinline__ I8Channels(const I8Args& a, const float* w_scale, const float* bias, int r_) : r(r_) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      ws[e] = r + e < a.n ? w_scale[r + e] : 0.0f;
      b[e] = bias && r + e < a.n ? bias[r + e] : 0.0f;
    }
    const uintptr_t unit = a.ydt == STB_F32 ? 16 : 8;
    whole = r + 4 <= a.n && a.ldy % 4 == 0 && (reinterpret_cast<uintptr_t>(a.Y) & (unit - 1)) == 0;
  }
  __device__ __forceinline__ void store(const I8Args& a, int tok, float xs, const int4& sum) const {
    const int s[4] = {sum.x, sum.y, sum.z, sum.w};
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = i8_value(s[e], xs, ws[e], b[e], a.bias != nullptr);
    const size_t at = (size_t)tok * a.ldy + r;
    if (!whole) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (r + e < a.n) i8_store(a.Y, at + e, a.ydt, v[e]);
    } else if (a.ydt == STB_F32) {
      *reinterpret_cast<float4*>(static_cast<float*>(a.Y) + at) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
      uint2 w;
      if (a.ydt == STB_F16) {
        const __half2 lo = __floats2half2_rn(v[0], v[1]), hi = __floats2half2_rn(v[2], v[3]);
        w = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
      } else {
        const __nv_bfloat162 lo = __floats2bfloat162_rn(v[0], v[1]), hi = __floats2bfloat162_rn(v[2], v[3]);
        w = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
      }
      *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.Y) + at) = w;
    }
  }
};

// Some tokens (a decode batch, a short prompt): one CTA per 128 channels, `bn` tokens and part of K; the `ks` parts of a tile are a cluster.
//   warp 0 brings the stages by TMA, warp 1 issues the products (it also owns tensor memory), warps 4 to 7 read the sums out.
// Every CTA hands the sums of every eighth-of-tokens chunk to the CTA of the cluster that owns the chunk (chunk mod ks), in that one's shared memory,
// where the ring was; the owner adds them, scales and stores rows of 128 channels.
struct I8Batch { int ks, per, stages, ttiles, bn, ring, own; uint32_t stage_bytes, tmem; };
constexpr int kI8BatchThreads = 256;
constexpr uint32_t kI8BatchScale = 1024, kI8BatchRing = 2048;     // the tokens' scales; the ring
constexpr int kI8MaxRing = 12;
__global__ void __launch_bounds__(kI8BatchThreads, 1)
gemm_i8_batch_kernel(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap xmap, const I8Args args, const __grid_constant__ I8Batch sh,
                     int* dev_status) {
  extern __shared__ __align__(1024) uint8_t smem[];
  const int warp = __shfl_sync(0xFFFFFFFFu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int ks = sh.ks, kz = (int)blockIdx.x % ks, tile = (int)blockIdx.x / ks, tt = tile % sh.ttiles, mt = tile / sh.ttiles;
  const int s0 = kz * sh.per, count = max(0, min(sh.stages, s0 + sh.per) - s0);
  const uint32_t sbase = smem_u32(smem), bar_full = sbase, bar_empty = sbase + 8 * kI8MaxRing, bar_accum = sbase + 16 * kI8MaxRing;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + 16 * kI8MaxRing + 8);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + 16 * kI8MaxRing + 16);
  if (threadIdx.x == 0) {
    for (int i = 0; i < sh.ring; ++i) { mbar_init(bar_full + 8 * i, 1); mbar_init(bar_empty + 8 * i, 1); }
    mbar_init(bar_accum, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
    asm volatile("prefetch.tensormap [%0];" ::"l"(&wmap) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&xmap) : "memory");
  }
  if (warp == 1) tmem_alloc(smem_u32(tmem_slot), sh.tmem);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_d = *tmem_slot;
  const float *w_scale = args.w_scale, *x_scale = args.x_scale, *bias = args.bias;
  begin_after(w_scale, x_scale, bias);
  if (warp >= 2)
    for (int i = (int)threadIdx.x - 64; i < sh.bn; i += kI8BatchThreads - 64)
      reinterpret_cast<float*>(smem + kI8BatchScale)[i] = tt * sh.bn + i < args.T ? x_scale[tt * sh.bn + i] : 0.0f;

  if (warp == 0) {
    const bool leader = elect_one();
    int s = 0;
    uint32_t parity = 1;
    for (int it = 0; it < count; ++it) {
      if (!__all_sync(0xFFFFFFFFu, gemm_wait(bar_empty + 8 * s, parity, abort_flag))) break;
      if (leader) {
        const uint32_t at = sbase + kI8BatchRing + (uint32_t)s * sh.stage_bytes, full = bar_full + 8 * s;
        mbar_expect_tx(full, sh.stage_bytes);
        tma_load_2d(at, &wmap, (s0 + it) * kI8K, mt * kI8M, full);
        tma_load_2d(at + kI8StageA, &xmap, (s0 + it) * kI8K, tt * sh.bn, full);
      }
      __syncwarp();
      if (++s == sh.ring) { s = 0; parity ^= 1u; }
    }
    if (*abort_flag) {       // let copies in flight land before the CTA gives its shared memory up
      const long long t0 = clock64();
      while (clock64() - t0 < 200000) {}
    }
  } else if (warp == 1) {
    const bool leader = elect_one();
    const uint32_t desc_hi = (uint32_t)(umma_desc(0u) >> 32), lo0 = (uint32_t)umma_desc(sbase + kI8BatchRing), idesc = i8_idesc(kI8M, sh.bn);
    const uint32_t tmem_u = __shfl_sync(0xFFFFFFFFu, tmem_d, 0);
    int s = 0;
    uint32_t parity = 0;
    for (int it = 0; it < count; ++it) {
      if (!__all_sync(0xFFFFFFFFu, gemm_wait(bar_full + 8 * s, parity, abort_flag))) break;
      tc_fence_after();
      const uint32_t a_lo = lo0 + (uint32_t)s * (sh.stage_bytes >> 4), b_lo = a_lo + (kI8StageA >> 4);
      if (leader) {
#pragma unroll
        for (int k = 0; k < kI8K / 32; ++k) umma_i8<1>(tmem_u, a_lo + 2u * k, b_lo + 2u * k, desc_hi, idesc, (it | k) != 0);
        umma_commit(bar_empty + 8 * s);
      }
      __syncwarp();
      if (++s == sh.ring) { s = 0; parity ^= 1u; }
    }
    if (leader) umma_commit(bar_accum);
    __syncwarp();
  }
  // every CTA of the cluster has read its ring to the end before sums are written where it was
  const bool have = __all_sync(0xFFFFFFFFu, gemm_wait(bar_accum, 0u, abort_flag));
  if (ks > 1) { cluster_arrive(); cluster_wait(); } else __syncthreads();
  const uint32_t sums = sbase + kI8BatchRing;                          // [rank][token of the owner][channel]
  if (warp >= 4 && have) {
    tc_fence_after();
    const int row = 32 * (warp - 4) + lane;
    for (int c0 = 0; c0 < sh.bn; c0 += 32) {
      uint32_t r[32];
      if (count > 0) tmem_ld32(tmem_d + ((uint32_t)(32 * (warp - 4)) << 16) + (uint32_t)c0, r);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int chunk = (c0 >> 3) + j;
        if (chunk * 8 >= sh.bn) break;
        const uint32_t at = sums + (uint32_t)(((kz * sh.own + chunk / ks) * 8) * kI8M + row) * 4u, to = ks > 1 ? smem_of_rank(at, (uint32_t)(chunk % ks)) : at;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(to + (uint32_t)i * (kI8M * 4u)), "r"(count > 0 ? r[8 * j + i] : 0u) : "memory");
      }
    }
    tc_fence_before();
  }
  if (ks > 1) { cluster_arrive(); cluster_wait(); } else __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_d, sh.tmem);
  }
  // four channels of a token per lane: 16 bytes of sums at a time, one 8- or 16-byte store
  const int r = mt * kI8M + 4 * lane;
  if (have && r < args.n) {
    const float* scales = reinterpret_cast<const float*>(smem + kI8BatchScale);
    const I8Channels ch(args, w_scale, bias, r);
    for (int lt = warp; lt < 8 * sh.own; lt += kI8BatchThreads / 32) {
      const int local = 8 * ((lt >> 3) * ks + kz) + (lt & 7), tok = tt * sh.bn + local;
      if (local >= sh.bn || tok >= args.T) break;
      int4 v = make_int4(0, 0, 0, 0);
      for (int z = 0; z < ks; ++z) {
        const int4 p = *reinterpret_cast<const int4*>(smem + kI8BatchRing + (size_t)(z * sh.own * 8 + lt) * (kI8M * 4) + 16 * lane);
        v.x += p.x; v.y += p.y; v.z += p.z; v.w += p.w;
      }
      ch.store(args, tok, scales[local], v);
    }
  }
  if (threadIdx.x == 0 && *abort_flag && dev_status) *dev_status = STB_ERR_TIMEOUT;
}

// Rows of bytes as a tensor map: boxes of 128 columns x `box_rows` rows, swizzled, zeros beyond the matrix.
static bool i8_map(EncodeTiledFn enc, CUtensorMap* map, const int8_t* p, int rows, int m, size_t ld, int box_rows) {
  const cuuint64_t dims[2] = {(cuuint64_t)m, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld};
  const cuuint32_t box[2] = {(cuuint32_t)kI8K, (cuuint32_t)box_rows}, estr[2] = {1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<int8_t*>(p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
static cudaError_t allow_smem(const void* kernel, bool* done, uint32_t bytes) {      // the shared-memory limit of a kernel is a per-device setting
  int dev = 0;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 0 && dev < 64 && done[dev]) return cudaSuccess;
  const cudaError_t f = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (f == cudaSuccess && dev >= 0 && dev < 64) done[dev] = true;
  return f;
}
static cudaError_t launch_cluster(const void* kernel, unsigned grid, unsigned cluster, unsigned threads, uint32_t smem, cudaStream_t s, void** params) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = cluster; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
  cfg.attrs = at; cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelExC(&cfg, kernel, params);
}

static int launch_i8_batch(const I8Args& a, int* dev_status, cudaStream_t s) {
  EncodeTiledFn enc = encode_tiled_fn();
  if (!enc) return STB_ERR_CUDA;
  I8Batch sh;
  sh.stages = (a.m + kI8K - 1) / kI8K;
  const int mtiles = (a.n + kI8M - 1) / kI8M, least = (a.T + 255) / 256;
  sh.bn = ((a.T + least - 1) / least + 15) / 16 * 16;
  sh.ttiles = (a.T + sh.bn - 1) / sh.bn;
  const long long tiles = (long long)mtiles * sh.ttiles;
  sh.ks = 1;
  while (sh.ks < 8 && tiles * sh.ks * 2 <= 148 && sh.stages >= 8 * sh.ks) sh.ks *= 2;
  sh.per = (sh.stages + sh.ks - 1) / sh.ks;
  sh.stage_bytes = kI8StageA + (uint32_t)sh.bn * kI8K;
  sh.ring = (int)((kI8SmemMax - kI8BatchRing) / sh.stage_bytes);
  if (sh.ring > kI8MaxRing) sh.ring = kI8MaxRing;
  sh.own = (sh.bn / 8 + sh.ks - 1) / sh.ks;
  sh.tmem = sh.bn <= 32 ? 32 : (sh.bn <= 64 ? 64 : (sh.bn <= 128 ? 128 : 256));
  const uint32_t sums = (uint32_t)(sh.ks * sh.own * 8) * kI8M * 4u, ring = (uint32_t)sh.ring * sh.stage_bytes;
  const uint32_t smem = kI8BatchRing + (ring > sums ? ring : sums);
  CUtensorMap wmap, xmap;
  if (!i8_map(enc, &wmap, a.W, a.n, a.m, a.ldw, kI8M) || !i8_map(enc, &xmap, a.X, a.T, a.m, a.ldx, sh.bn)) return STB_ERR_ARG;
  static bool done[64] = {};
  if (allow_smem(reinterpret_cast<const void*>(gemm_i8_batch_kernel), done, kI8SmemMax) != cudaSuccess) return STB_ERR_CUDA;
  I8Args args = a;
  void* params[] = {&wmap, &xmap, &args, &sh, &dev_status};
  return launch_cluster(reinterpret_cast<const void*>(gemm_i8_batch_kernel), (unsigned)(tiles * sh.ks), (unsigned)sh.ks, kI8BatchThreads, smem, s, params) == cudaSuccess ? STB_OK : STB_ERR_CUDA;
}

// ---- many tokens ----------------------------------------------------------------------------------------------------------------------
// Two CTAs of a cluster compute a tile of 256 channels x `bn` tokens together (cta_group::2): each holds 128 rows of W and half of the tokens'
// rows, the first one's issuing lane multiplies for both, and each has the sums of its 128 channels for all tokens in its tensor memory.  The
// clusters stay for the whole call and take every so-many-th tile (tokens fastest, so that W is read from HBM once); two accumulators of 256 columns,
// so that a tile is read out while the next one is multiplied.  Per 128 columns of K a CTA fetches 16 KB + bn / 2 rows for 256 x bn x 128
// multiply-adds of the pair: at bn = 256 64 bytes per clock of the tensor core, what an SM gets from L2.
//   warp 0 brings the stages, warp 1 issues the products, warps 4 to 7 read the sums out: 32 tokens at a time through shared memory, from where they leave
//   as rows of 128 channels by TMA (or by plain stores where rows of Y are on no 16-byte boundary).
struct I8Prefill { int stages, ttiles, tiles, bn, ring, tma_out; uint32_t stage_bytes; };
constexpr int kI8PrefillThreads = 256, kI8PrefillMaxRing = 10, kI8OutTokens = 32;
constexpr uint32_t kI8OutBytes = kI8OutTokens * kI8M * 4u;
constexpr uint32_t kI8PrefillScale = 512, kI8PrefillOut = 2048, kI8PrefillRing = kI8PrefillOut + 2u * kI8OutBytes;      // (a tile's scales: 256 floats)
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {      // the barrier may be the other CTA's
  asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void umma_commit_pair(uint32_t bar) {      // arrives on the barrier of both CTAs
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_wait_cluster(uint32_t bar, uint32_t parity, volatile int* abort_flag) {      // gemm_wait for arrivals of the other CTA
  const long long t0 = clock64();
  for (;;) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    if (ok) return true;
    if (*abort_flag) return false;
    if (clock64() - t0 > kGemmWaitLimit) { *abort_flag = 1; return false; }
  }
}
// the barrier of the warps 4 to 7: whether all of their threads say yes
__device__ __forceinline__ bool barrier_and(bool yes) {
  uint32_t all;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(all) : "r"((uint32_t)yes) : "memory");
  return all != 0;
}
__global__ void __launch_bounds__(kI8PrefillThreads, 1)
gemm_i8_prefill_kernel(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CUtensorMap ymap, const I8Args args,
                       const __grid_constant__ I8Prefill sh, int* dev_status) {
  extern __shared__ __align__(1024) uint8_t smem[];
  const int warp = __shfl_sync(0xFFFFFFFFu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int rank = (int)(blockIdx.x & 1u), first = (int)(blockIdx.x >> 1), step = (int)(gridDim.x >> 1);
  const uint32_t sbase = smem_u32(smem);
  const uint32_t bar_full = sbase, bar_empty = bar_full + 8 * kI8PrefillMaxRing, bar_acc_full = bar_empty + 8 * kI8PrefillMaxRing, bar_acc_empty = bar_acc_full + 16;
  constexpr uint32_t kBars = 8 * (2 * kI8PrefillMaxRing + 4);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + kBars);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + kBars + 8);
  if (threadIdx.x == 0) {
    for (int i = 0; i < sh.ring; ++i) { mbar_init(bar_full + 8 * i, 1); mbar_init(bar_empty + 8 * i, 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(bar_acc_full + 8 * i, 1); mbar_init(bar_acc_empty + 8 * i, 8); }      // (four warps of either CTA)
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
    asm volatile("prefetch.tensormap [%0];" ::"l"(&wmap) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&xmap) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_arrive();                        // both CTAs' barriers are there before either signals the other's
  cluster_wait();
  tc_fence_after();
  const uint32_t tmem_d = *tmem_slot;
  const float *w_scale = args.w_scale, *x_scale = args.x_scale, *bias = args.bias;
  begin_after(w_scale, x_scale, bias);

  if (warp == 0) {
    const bool leader = elect_one();
    const uint32_t full0 = smem_of_rank(bar_full, 0u);
    int s = 0;
    uint32_t parity = 1;
    bool ok = true;
    for (int tile = first; tile < sh.tiles && ok; tile += step) {
      const int wrow = (tile / sh.ttiles) * 2 * kI8M + rank * kI8M, xrow = (tile % sh.ttiles) * sh.bn + rank * (sh.bn >> 1);
      for (int it = 0; it < sh.stages; ++it) {
        ok = __all_sync(0xFFFFFFFFu, gemm_wait(bar_empty + 8 * s, parity, abort_flag));
        if (!ok) break;
        if (leader) {
          const uint32_t at = sbase + kI8PrefillRing + (uint32_t)s * sh.stage_bytes;
          if (rank == 0) mbar_expect_tx(bar_full + 8 * s, 2u * sh.stage_bytes);
          tma_load_2d_pair(at, &wmap, it * kI8K, wrow, full0 + 8 * s);
          tma_load_2d_pair(at + kI8StageA, &xmap, it * kI8K, xrow, full0 + 8 * s);
        }
        __syncwarp();
        if (++s == sh.ring) { s = 0; parity ^= 1u; }
      }
    }
    // the first CTA's products signal this one's barriers: all of that has arrived before the CTA may leave
    for (int i = 0; i < sh.ring && ok; ++i) {
      ok = __all_sync(0xFFFFFFFFu, gemm_wait(bar_empty + 8 * s, parity, abort_flag));
      if (++s == sh.ring) { s = 0; parity ^= 1u; }
    }
    if (*abort_flag) {       // let copies in flight land before the CTA gives its shared memory up
      const long long t0 = clock64();
      while (clock64() - t0 < 200000) {}
    }
  } else if (warp == 1 && rank == 0) {
    const bool leader = elect_one();
    const uint32_t desc_hi = (uint32_t)(umma_desc(0u) >> 32), lo0 = (uint32_t)umma_desc(sbase + kI8PrefillRing), idesc = i8_idesc(2 * kI8M, sh.bn);
    const uint32_t tmem_u = __shfl_sync(0xFFFFFFFFu, tmem_d, 0);
    int s = 0, use = 0;
    uint32_t parity = 0;
    bool ok = true;
    for (int tile = first; tile < sh.tiles && ok; tile += step, ++use) {
      const int acc = use & 1;
      ok = __all_sync(0xFFFFFFFFu, mbar_wait_cluster(bar_acc_empty + 8 * acc, ((uint32_t)(use >> 1) & 1u) ^ 1u, abort_flag));
      if (!ok) break;
      tc_fence_after();
      for (int it = 0; it < sh.stages; ++it) {
        ok = __all_sync(0xFFFFFFFFu, gemm_wait(bar_full + 8 * s, parity, abort_flag));
        if (!ok) break;
        tc_fence_after();
        const uint32_t a_lo = lo0 + (uint32_t)s * (sh.stage_bytes >> 4), b_lo = a_lo + (kI8StageA >> 4);
        if (leader) {
#pragma unroll
          for (int k = 0; k < kI8K / 32; ++k) umma_i8<2>(tmem_u + 256u * acc, a_lo + 2u * k, b_lo + 2u * k, desc_hi, idesc, (it | k) != 0);
          umma_commit_pair(bar_empty + 8 * s);
        }
        __syncwarp();
        if (++s == sh.ring) { s = 0; parity ^= 1u; }
      }
      if (leader) umma_commit_pair(bar_acc_full + 8 * acc);      // (also where the loop was left early: the sums are then not used)
      __syncwarp();
    }
  } else if (warp >= 4) {
    const int q = warp - 4, row = 32 * q + lane, t128 = (int)threadIdx.x - 128;
    const uint32_t acc_empty0 = smem_of_rank(bar_acc_empty, 0u);
    const int elem = args.ydt == STB_F32 ? 4 : 2;
    float* scales = reinterpret_cast<float*>(smem + kI8PrefillScale);
    int use = 0, buf = 0;
    for (int tile = first; tile < sh.tiles; tile += step, ++use) {
      const int acc = use & 1, r0 = (tile / sh.ttiles) * 2 * kI8M + rank * kI8M, r = r0 + row, tok0 = (tile % sh.ttiles) * sh.bn;
      const float ws = r < args.n ? w_scale[r] : 0.0f, b = bias && r < args.n ? bias[r] : 0.0f;
      asm volatile("bar.sync 1, 128;" ::: "memory");             // the last tile's scales have been read
      for (int i = t128; i < sh.bn; i += 128) scales[i] = tok0 + i < args.T ? x_scale[tok0 + i] : 0.0f;
      if (!barrier_and(gemm_wait(bar_acc_full + 8 * acc, (uint32_t)(use >> 1) & 1u, abort_flag))) break;      // (one verdict for the four warps)
      tc_fence_after();
      for (int c0 = 0; c0 < sh.bn; c0 += kI8OutTokens, buf ^= 1) {
        uint32_t v[32];
        tmem_ld32(tmem_d + ((uint32_t)(32 * q) << 16) + (uint32_t)(256 * acc + c0), v);
        const uint32_t out = sbase + kI8PrefillOut + (uint32_t)buf * kI8OutBytes;
        if (t128 == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");       // the store before last has read this buffer
        asm volatile("bar.sync 1, 128;" ::: "memory");
#pragma unroll
        for (int i = 0; i < kI8OutTokens; ++i) {
          const float f = i8_value((int)v[i], scales[c0 + i], ws, b, bias != nullptr);
          if (elem == 4) asm volatile("st.shared.f32 [%0], %1;" ::"r"(out + (uint32_t)(i * kI8M + row) * 4u), "f"(f) : "memory");
          else {
            const uint16_t h = args.ydt == STB_F16 ? __half_as_ushort(__float2half_rn(f)) : __bfloat16_as_ushort(__float2bfloat16_rn(f));
            asm volatile("st.shared.u16 [%0], %1;" ::"r"(out + (uint32_t)(i * kI8M + row) * 2u), "h"(h) : "memory");
          }
        }
        if (sh.tma_out) fence_async_smem();
        asm volatile("bar.sync 1, 128;" ::: "memory");
        if (r0 >= args.n || tok0 + c0 >= args.T) continue;
        if (sh.tma_out) {
          if (t128 == 0) {
            asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];" ::"l"(&ymap), "r"(out), "r"(r0), "r"(tok0 + c0) : "memory");
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
          }
        } else if (r < args.n) {
          for (int i = 0; i < kI8OutTokens && tok0 + c0 + i < args.T; ++i) {
            const size_t at = (size_t)(tok0 + c0 + i) * args.ldy + r;
            const uint8_t* p = smem + kI8PrefillOut + (size_t)buf * kI8OutBytes + (size_t)(i * kI8M + row) * elem;
            if (elem == 4) static_cast<float*>(args.Y)[at] = *reinterpret_cast<const float*>(p);
            else static_cast<uint16_t*>(args.Y)[at] = *reinterpret_cast<const uint16_t*>(p);
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(acc_empty0 + 8 * acc);
    }
    if (t128 == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_arrive();                        // nobody leaves while the other CTA's products read its operands or its barriers are signalled
  cluster_wait();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_d), "r"(512) : "memory");
  }
  if (threadIdx.x == 0 && *abort_flag && dev_status) *dev_status = STB_ERR_TIMEOUT;
}

static int launch_i8_prefill(const I8Args& a, int* dev_status, cudaStream_t s) {
  EncodeTiledFn enc = encode_tiled_fn();
  if (!enc) return STB_ERR_CUDA;
  I8Prefill sh;
  sh.stages = (a.m + kI8K - 1) / kI8K;
  const int least = (a.T + 255) / 256;
  sh.bn = ((a.T + least - 1) / least + 31) / 32 * 32;
  sh.ttiles = (a.T + sh.bn - 1) / sh.bn;
  const long long tiles = (long long)((a.n + 2 * kI8M - 1) / (2 * kI8M)) * sh.ttiles;
  if (tiles > 0x7FFFFFFF) return STB_ERR_SHAPE;
  sh.tiles = (int)tiles;
  sh.stage_bytes = kI8StageA + (uint32_t)sh.bn * (kI8K / 2);
  sh.ring = (int)((kI8SmemMax - kI8PrefillRing) / sh.stage_bytes);
  if (sh.ring > kI8PrefillMaxRing) sh.ring = kI8PrefillMaxRing;
  const uint32_t smem = kI8PrefillRing + (uint32_t)sh.ring * sh.stage_bytes;
  CUtensorMap wmap, xmap, ymap = {};
  if (!i8_map(enc, &wmap, a.W, a.n, a.m, a.ldw, kI8M) || !i8_map(enc, &xmap, a.X, a.T, a.m, a.ldx, sh.bn / 2)) return STB_ERR_ARG;
  const int elem = a.ydt == STB_F32 ? 4 : 2;
  sh.tma_out = (a.ldy * (size_t)elem) % 16 == 0 && (reinterpret_cast<uintptr_t>(a.Y) & 15u) == 0;
  if (sh.tma_out) {
    const cuuint64_t dims[2] = {(cuuint64_t)a.n, (cuuint64_t)a.T}, strides[1] = {(cuuint64_t)a.ldy * (cuuint64_t)elem};
    const cuuint32_t box[2] = {(cuuint32_t)kI8M, (cuuint32_t)kI8OutTokens}, estr[2] = {1, 1};
    const CUtensorMapDataType dt = a.ydt == STB_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : (a.ydt == STB_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16);
    sh.tma_out = enc(&ymap, dt, 2, a.Y, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  }
  static bool done[64] = {};
  if (allow_smem(reinterpret_cast<const void*>(gemm_i8_prefill_kernel), done, kI8SmemMax) != cudaSuccess) return STB_ERR_CUDA;
  I8Args args = a;
  void* params[] = {&wmap, &xmap, &ymap, &args, &sh, &dev_status};
  const int pairs = sh.tiles < 74 ? sh.tiles : 74;
  return launch_cluster(reinterpret_cast<const void*>(gemm_i8_prefill_kernel), 2u * (unsigned)pairs, 2u, kI8PrefillThreads, smem, s, params) == cudaSuccess ? STB_OK : STB_ERR_CUDA;
}

}  // namespace stb

extern "C" int stb_gemm_i8(const int8_t* W, size_t ldw, const float* w_scale, const float* bias, int n, int m, const int8_t* X, size_t ldx,
                           const float* x_scale, int T, void* Y, stb_dtype ydt, size_t ldy, int* dev_status, void* stream) {
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
  if (T > 256 && (long long)((n + 255) / 256) * ((T + 255) / 256) >= 37) return stb::launch_i8_prefill(a, dev_status, s);
  if (T > 16) return stb::launch_i8_batch(a, dev_status, s);
  const cudaError_t e = T <= 8 ? stb::launch_gemv_i8<1>(a, s) : stb::launch_gemv_i8<2>(a, s);
  return e == cudaSuccess ? STB_OK : STB_ERR_CUDA;
}
