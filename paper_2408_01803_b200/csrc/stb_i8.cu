// stb_gemm_i8: the linear layer in 8 bits, Y[t][i] = x_scale[t] w_scale[i] sum_j W[i][j] X[t][j] (+ bias[i]).
// The sums are whole numbers in int32, so every order of them, every split of K and every kernel gives the same bits.
#include <cooperative_groups.h>
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/stb.h"
#include "stb_ptx.cuh"
#include "stb_tcgen05.cuh"

namespace cg = cooperative_groups;

namespace stb {

// A wait that runs out ends its CTA's part of the call: the results that are then not known become NaN, so that nobody takes them for results, and *dev_status, where
// there is one, STB_ERR_TIMEOUT.  Self-test: copies off for some of the CTAs or tiles, and a limit of about 50 microseconds.
constexpr long long kI8SelftestLimit = 100000;
constexpr int kI8MaxSide = 1 << 30;      // of n and T: tiles and what lies behind the last one are counted in 32 bits

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
// the arrival that says only that this CTA has started (cluster_arrive also waits for what it has written)
__device__ __forceinline__ void cluster_arrive_relaxed() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
// Asks for a piece of memory to be brought into L2 (16-byte aligned, a multiple of 16 bytes).  It is read by nobody yet: a kernel may ask for
// what the one before it is still writing.
__device__ __forceinline__ void prefetch_l2(const void* p, uint32_t bytes) {
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p), "r"(bytes) : "memory");
}
__device__ __forceinline__ void prefetch_l2_box(const CUtensorMap* map, int x, int y) {
  asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(map), "r"(x), "r"(y) : "memory");
}
// A few tokens (up to 8) and few weights: the tensor cores take the weights as they come.  16 rows of W per CTA; its eight warps take every eighth
// 64 columns of the CTA's part of K.  Lane 4 g + t reads 16 bytes at column 16 t of the rows g and g + 8 and of token g: the same columns of both
// operands are then in the same place of two instructions, which is all that an order of K has to satisfy (m is a multiple of 16).  The sums of
// the warps meet in shared memory, those of the `ksplit` CTAs of a cluster in that of its first.
constexpr int kI8Warps = 8, kI8Rows = 16, kI8Step = 64, kI8FewTokens = 8;
constexpr int kI8PrefetchRow = 4096;       // bytes of a row asked for ahead: 4096 x 4096, one token, 6.5 -> 5.1 us (1 KB 5.6, 16 KB 5.2)
__global__ void __launch_bounds__(32 * kI8Warps)
gemv_i8_kernel(const I8Args args, int ksplit, int prefetch) {
  __shared__ int part[kI8Warps][4][32];
  __shared__ int whole[8][4][32];
  const int8_t *W = args.W, *X = args.X;
  const float *w_scale = args.w_scale, *x_scale = args.x_scale, *bias = args.bias;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int kz = (int)blockIdx.x % ksplit, row0 = (int)(blockIdx.x / ksplit) * kI8Rows;
  const int m = args.m, steps = (m + kI8Step - 1) / kI8Step, per = (steps + ksplit - 1) / ksplit, end = min(steps, (kz + 1) * per);
  if (ksplit > 1) cluster_arrive_relaxed();  // (before a CTA writes into another's shared memory, that one has started)
  if (warp == 0 && lane < kI8Rows && row0 + lane < args.n) {      // while what is before this kernel still runs: the weights, into L2
    const int from = kz * per * kI8Step, bytes = min(min(end * kI8Step, m) - from, prefetch);
    if (bytes > 0) prefetch_l2(W + (size_t)(row0 + lane) * args.ldw + from, (uint32_t)bytes);
  }
  begin_after(W, X, w_scale, x_scale, bias);
  const bool r0 = row0 + g < args.n, r1 = row0 + g + 8 < args.n, tok = g < args.T;
  const int8_t *w0 = W + (size_t)(r0 ? row0 + g : 0) * args.ldw, *w1 = W + (size_t)(r1 ? row0 + g + 8 : 0) * args.ldw, *xr = X + (size_t)(tok ? g : 0) * args.ldx;
  int acc[4] = {0, 0, 0, 0};
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll 4
  for (int s = kz * per + warp; s < end; s += kI8Warps) {
    const int at = s * kI8Step + 16 * t;
    const bool in = at < m;
    const uint4 a0 = r0 && in ? ldg_stream_v4(w0 + at) : zero, a1 = r1 && in ? ldg_stream_v4(w1 + at) : zero, x = tok && in ? ldg_nc_v4(xr + at) : zero;
    mma_i8(acc, a0.x, a1.x, a0.y, a1.y, x.x, x.y);
    mma_i8(acc, a0.z, a1.z, a0.w, a1.w, x.z, x.w);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) part[warp][k][lane] = acc[k];
  __syncthreads();
  if (ksplit > 1) cluster_wait();
  const int i = threadIdx.x;
  if (i < 128) {
    int sum = 0;
#pragma unroll
    for (int w = 0; w < kI8Warps; ++w) sum += part[w][i >> 5][i & 31];
    cg::this_cluster().map_shared_rank(&whole[0][0][0], 0)[kz * 128 + i] = sum;
  }
  if (ksplit > 1) {
    cluster_arrive();
    cluster_wait();
    if (kz != 0) return;
  } else {
    __syncthreads();
  }
  // accumulator k of lane 4 g + t is row g + 8 (k / 2), token 2 t + k % 2
  const int row = i & 15, to = i >> 4, k = ((row >> 3) << 1) | (to & 1), ln = 4 * (row & 7) + ((to & 7) >> 1), r = row0 + row;
  if (i < 128 && r < args.n && to < args.T) {
    int sum = 0;
    for (int z = 0; z < ksplit; ++z) sum += whole[z][k][ln];
    i8_store(args.Y, (size_t)to * args.ldy + r, args.ydt, i8_value(sum, x_scale[to], w_scale[r], bias ? bias[r] : 0.0f, bias != nullptr));
  }
}

// Whether these calls are for gemv_i8_kernel, and the CTAs of a cluster if so (else 0).  Its grid is one wave of up to four CTAs per SM, which gemm_i8_batch_kernel,
// whose CTAs take longer to set up, cannot beat below some 20 million weights: 1024 x 8192, one token, 3.9 us against 4.7; 4096 x 4096 5.1 against 5.9;
// 966 x 20352 5.4 against 7.1.  Beyond, bulk copies into deep rings win: 12434 x 1536, eight tokens, 6.7 against 5.8; 11008 x 4096 10.5 against 10.2.
static int gemv_i8_split(int n, int m, int T) {
  const int groups = (n + kI8Rows - 1) / kI8Rows, steps = (m + kI8Step - 1) / kI8Step, slots = 4 * 148;
  if (T > kI8FewTokens || m % 16 != 0 || groups > slots || (long long)n * m > 20000000) return 0;
  int ksplit = 1;
  while (ksplit < 8 && groups * ksplit * 2 <= slots && steps >= 10 * ksplit && steps > 16) ksplit *= 2;
  return ksplit;
}
static cudaError_t launch_gemv_i8(const I8Args& a, int ksplit, cudaStream_t s) {
  const int groups = (a.n + kI8Rows - 1) / kI8Rows;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(groups * ksplit));
  cfg.blockDim = dim3(32 * kI8Warps);
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)ksplit; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
  cfg.attrs = at; cfg.numAttrs = ksplit > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, gemv_i8_kernel, a, ksplit, kI8PrefetchRow);
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
// 32 columns of a warp's lanes: asked for, and waited for (all that was asked for; the registers pass through the wait, so that none is used before it)
__device__ __forceinline__ void tmem_ask32(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
               "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                 "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
                 "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
                 "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
               : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_wait32(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                 "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]),
                 "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]),
                 "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31]) :: "memory");
}
// the same place in the shared memory of another CTA of the cluster
__device__ __forceinline__ uint32_t smem_of_rank(uint32_t a, uint32_t rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
  return r;
}

// Results of one channel for up to kCount tokens from `tok` on (`live` of them exist).  The lanes of a warp hold channels side by side.
template <int kCount>
__device__ __forceinline__ void i8_channel_out(const I8Args& a, const uint32_t (&sum)[kCount], const float* scales, float ws, float b, bool with_bias, int tok, int live, int r) {
  const size_t at = (size_t)tok * a.ldy + r;
#pragma unroll
  for (int i = 0; i < kCount; ++i) {
    if (i >= live) break;
    const float f = i8_value((int)sum[i], scales[i], ws, b, with_bias);
    if (a.ydt == STB_F32) static_cast<float*>(a.Y)[at + i * a.ldy] = f;
    else if (a.ydt == STB_F16) static_cast<__half*>(a.Y)[at + i * a.ldy] = __float2half_rn(f);
    else static_cast<__nv_bfloat16*>(a.Y)[at + i * a.ldy] = __float2bfloat16_rn(f);
  }
}

// Some tokens (a decode batch, a short prompt): one CTA per 128 channels, `bn` tokens and part of K; the `ks` parts of a tile are a cluster.
//   warp 0 brings the stages by TMA, warp 1 issues the products (it also owns tensor memory); then all eight warps read the sums out.
// ks = 1: straight to Y.  Else eight tokens at a time belong to one CTA of the cluster (group of eight mod ks), which gets everybody's sums of them
// into its shared memory (32 bytes per channel and CTA), adds, scales and stores.  Bound by HBM where W is large (28672 x 8192, one token 38.7 us, 94 % of its
// bytes' time; 4096 x 11008, 64 tokens, 11.1 us: 64 %, the rest the way from the launch to the first stage and the sum of the cluster).
// A CTA without its sums hands over kI8Lost in their place, which no sum of a part of K is (|sum| < 2^31).
// `off`: the part of K that is not copied (self-test), else -1.
struct I8Batch { int lks, per, stages, ttiles, bn, ring, prefetch, off; uint32_t stage_bytes, tmem; long long limit; };
constexpr uint32_t kI8Lost = 0x80000000u;
constexpr int kI8BatchThreads = 256;
constexpr uint32_t kI8BatchScale = 1024, kI8BatchRing = 2048;     // the tokens' scales; the ring, and behind it the sums that the CTAs hand over
constexpr int kI8MaxRing = 12;
__global__ void __launch_bounds__(kI8BatchThreads, 1)
gemm_i8_batch_kernel(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap xmap, const I8Args args, const __grid_constant__ I8Batch sh,
                     int* dev_status) {
  extern __shared__ __align__(1024) uint8_t smem[];
  const int warp = __shfl_sync(0xFFFFFFFFu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int lks = sh.lks, ks = 1 << lks, kz = (int)blockIdx.x & (ks - 1), tile = (int)blockIdx.x >> lks, tt = tile % sh.ttiles, mt = tile / sh.ttiles;
  const int s0 = kz * sh.per, count = max(0, min(sh.stages, s0 + sh.per) - s0);
  if (ks > 1) cluster_arrive_relaxed();    // (before a CTA writes into another's shared memory, that one has started)
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
    // while what is before this kernel still runs: the first weights, into L2
    for (int it = 0; it < count && it < sh.prefetch; ++it) prefetch_l2_box(&wmap, (s0 + it) * kI8K, mt * kI8M);
  }
  if (warp == 1) tmem_alloc(smem_u32(tmem_slot), sh.tmem);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_d = *tmem_slot;
  const float *w_scale = args.w_scale, *x_scale = args.x_scale, *bias = args.bias;
  begin_after(w_scale, x_scale, bias);
  const int row = 32 * (warp & 3) + lane, r = mt * kI8M + row, half = warp >> 2;       // the channel that this thread reads out
  const float ws = r < args.n ? w_scale[r] : 0.0f, b = bias && r < args.n ? bias[r] : 0.0f;
  if (warp >= 2)
    for (int i = (int)threadIdx.x - 64; i < sh.bn; i += kI8BatchThreads - 64)
      reinterpret_cast<float*>(smem + kI8BatchScale)[i] = tt * sh.bn + i < args.T ? x_scale[tt * sh.bn + i] : 0.0f;

  if (warp == 0) {
    const bool leader = elect_one();
    int s = 0;
    uint32_t parity = 1;
    for (int it = 0; it < count; ++it) {
      if (!__all_sync(0xFFFFFFFFu, gemm_wait(bar_empty + 8 * s, parity, abort_flag, sh.limit))) break;
      if (leader && kz != sh.off) {
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
    int s = 0, it = 0;
    uint32_t parity = 0;
    for (; it < count; ++it) {
      if (!__all_sync(0xFFFFFFFFu, gemm_wait(bar_full + 8 * s, parity, abort_flag, sh.limit))) break;
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
    if (leader && it >= count) umma_commit(bar_accum);                  // (sums of fewer stages are nobody's: the waits for them run out)
    __syncwarp();
  }
  const bool have = __all_sync(0xFFFFFFFFu, gemm_wait(bar_accum, 0u, abort_flag, sh.limit));
  tc_fence_after();
  const uint32_t from = tmem_d + ((uint32_t)(32 * (warp & 3)) << 16);
  const float* scales = reinterpret_cast<const float*>(smem + kI8BatchScale);
  const int live = min(sh.bn, args.T - tt * sh.bn);                    // tokens of the tile
  if (ks == 1) {
    __syncthreads();                                                   // (the scales)
    for (int c0 = 32 * half; c0 < live; c0 += 64) {
      uint32_t v[32];
      if (have) {
        tmem_ask32(from + (uint32_t)c0, v);
        tmem_wait32(v);
      } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = 0u;
      }
      if (r < args.n) i8_channel_out<32>(args, v, scales + c0, have ? ws : __uint_as_float(0x7FC00000u), b, bias != nullptr, tt * sh.bn + c0, live - c0, r);
    }
  } else {
    cluster_wait();
    const uint32_t mine = sbase + kI8BatchRing + (uint32_t)sh.ring * sh.stage_bytes + (uint32_t)(kz * kI8M) * 32u + (uint32_t)row * 16u;
    for (int c0 = 32 * half; c0 < live; c0 += 64) {
      uint32_t v[32];
      if (have && count > 0) {
        tmem_ask32(from + (uint32_t)c0, v);
        tmem_wait32(v);
      } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = have ? 0u : kI8Lost;       // (have: no columns of K were left for this CTA)
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int g = (c0 >> 3) + j;
        if (8 * g >= live) break;
        const uint32_t to = smem_of_rank(mine + (uint32_t)((g >> lks << lks) * kI8M) * 32u, (uint32_t)(g & (ks - 1)));
        asm volatile("st.shared::cluster.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(to), "r"(v[8 * j]), "r"(v[8 * j + 1]), "r"(v[8 * j + 2]), "r"(v[8 * j + 3]) : "memory");
        asm volatile("st.shared::cluster.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(to + 16u * kI8M), "r"(v[8 * j + 4]), "r"(v[8 * j + 5]), "r"(v[8 * j + 6]), "r"(v[8 * j + 7]) : "memory");
      }
    }
    cluster_arrive();
    cluster_wait();
    if (r < args.n) {
      const uint8_t* sums = smem + kI8BatchRing + (size_t)sh.ring * sh.stage_bytes + (size_t)row * 16;
      for (int g = half * ks + kz; 8 * g < live; g += 2 * ks) {
        uint32_t v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        bool lost = false;
#pragma unroll 4
        for (int z = 0; z < ks; ++z) {
          const uint4* p = reinterpret_cast<const uint4*>(sums + (size_t)((g >> lks << lks) + z) * (kI8M * 32));
          const uint4 lo = p[0], hi = p[kI8M];
          lost = lost || lo.x == kI8Lost;
          v[0] += lo.x; v[1] += lo.y; v[2] += lo.z; v[3] += lo.w; v[4] += hi.x; v[5] += hi.y; v[6] += hi.z; v[7] += hi.w;
        }
        i8_channel_out<8>(args, v, scales + 8 * g, lost ? __uint_as_float(0x7FC00000u) : ws, b, bias != nullptr, tt * sh.bn + 8 * g, live - 8 * g, r);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_d, sh.tmem);
  }
  if (threadIdx.x == 0 && *abort_flag && dev_status) *dev_status = STB_ERR_TIMEOUT;
}

// ---- which kernel, which tile ---------------------------------------------------------------------------------------------------------
// pair: gemm_i8_prefill_kernel.  half: the CTAs of gemm_i8_batch_kernel take half of an SM's shared memory, so that two fit (and the first CTAs of the
// call after this one can be set up beside the last ones of this one).
struct I8Plan { bool pair, half; int bn, ttiles, lks; };
constexpr uint32_t kI8HalfSmem = 115000;
__host__ inline uint32_t i8_stage_bytes(int bn) { return kI8StageA + (uint32_t)bn * kI8K; }
__host__ inline uint32_t i8_sum_bytes(int bn, int ks) { return ks > 1 ? (uint32_t)((bn / 8 + ks - 1) / ks * ks) * (kI8M * 32u) : 0u; }
__host__ inline int i8_ring(int bn, int ks, bool half) {
  const uint32_t room = half ? kI8HalfSmem : kI8SmemMax, taken = kI8BatchRing + i8_sum_bytes(bn, ks);
  const int ring = room > taken ? (int)((room - taken) / i8_stage_bytes(bn)) : 0;
  return ring > kI8MaxRing ? kI8MaxRing : ring;
}
// The layout whose estimated time is smallest.  In microseconds, fitted to 4200 timed calls of 450 shapes (n, m of 64 to 28672, T of 1 to 4096); over them the choice
// is 1.0 % behind the fastest layout of each shape on average, 4 % in one of ten.  (The estimates rank layouts; as times they can be a third off: 33 for 24.7 at 5120 x 13824 and
// 333 tokens.)
//   gemm_i8_batch_kernel:   a stage of 128 columns 0.12 + 0.0014 bn (0.023 more where two CTAs share an SM), times the stages of the fullest SM; the bytes at
//                           6.3 TB/s / 0.95, the tokens' rows counting 2.2 times (they are read by every row of tiles); the root of the sum of the two squared;
//                           1.9 for the call, 0.019 bn per wave for reading the sums out, 0.7 for a cluster's sum, 2.5 per further wave
//   gemm_i8_prefill_kernel: a stage 0.134 + 0.00053 bn times the stages of a cluster; 2.0 for the call, 0.057 bn for the last tile, 3.1 and 0.0047 bn per further tile
// A cluster lies within one of the GPU's partitions: of four CTAs 33 fit at once, of eight 15.
static I8Plan i8_plan(int n, int m, int T) {
  I8Plan best = {};
  float best_cost = 3.4e38f;
  const int stages = (m + kI8K - 1) / kI8K, least = (T + 255) / 256, mtiles = (n + kI8M - 1) / kI8M;
  const float weights = (float)n * (float)m, tokens = (float)T * (float)m, out = 2.0f * (float)T * (float)n;
  if (T <= 700) {
    const float bytes = (weights + 2.2f * tokens + out) * (0.95f / 6.3e6f);
    for (int tt = least; tt < least + 8; ++tt) {
      const int bn = ((T + tt - 1) / tt + 15) / 16 * 16;
      if (bn > 256 || (tt > least && (bn < 48 || (tt - 1) * bn >= T))) continue;
      for (int lks = 0; lks < 4; ++lks) {
        const int ks = 1 << lks, one = lks == 0 || lks == 1 ? 148 : (lks == 2 ? 132 : 120);
        const long long ctas = (long long)mtiles * tt * ks;
        if (lks > 0 && (stages < 2 * ks || ctas > 600)) break;
        for (int half = 0; half < 2; ++half) {
          if (i8_ring(bn, ks, half != 0) < 3) continue;
          const long long at_once = (long long)one << half, full = ctas / at_once, rest = ctas % at_once;
          const float per_sm = (float)((full << half) + (rest > one ? 2 : (rest > 0 ? 1 : 0))), waves = (float)(full + (rest > 0));
          const float sm = per_sm * (float)((stages + ks - 1) / ks) * (0.122f + 0.00137f * (float)bn + (half ? 0.023f : 0.0f));
          const float cost = 1.93f + sqrtf(sm * sm + bytes * bytes) + 0.0193f * (float)bn * waves + (ks > 1 ? 0.71f + 0.001f * (float)bn : 0.0f) + 2.53f * (waves - 1.0f);
          if (cost < best_cost) { best_cost = cost; best = {false, half != 0, bn, tt, lks}; }
        }
      }
    }
  }
  if (T > 48) {
    const float bytes = (weights + tokens + out) * (0.82f / 6.3e6f);
    for (int bn = 256; bn >= 64; bn -= 32) {        // (seven choices however many tokens there are)
      const int tt = (T + bn - 1) / bn;
      const float turns = (float)(((long long)((mtiles + 1) / 2) * tt + 73) / 74), sm = turns * (float)stages * (0.1336f + 0.000532f * (float)bn);
      const float cost = 2.0f + sqrtf(sm * sm + bytes * bytes) + 0.0567f * (float)bn + (turns - 1.0f) * (3.07f + 0.0047f * (float)bn);
      if (cost < best_cost) { best_cost = cost; best = {true, false, bn, tt, 0}; }
    }
  }
  return best;
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

static int launch_i8_batch(const I8Args& a, const I8Plan& plan, int* dev_status, cudaStream_t s, bool selftest) {
  EncodeTiledFn enc = encode_tiled_fn();
  if (!enc) return STB_ERR_CUDA;
  I8Batch sh;
  const int ks = 1 << plan.lks;
  sh.lks = plan.lks; sh.bn = plan.bn; sh.ttiles = plan.ttiles;
  sh.stages = (a.m + kI8K - 1) / kI8K;
  sh.per = (sh.stages + ks - 1) / ks;
  const long long ctas = (long long)((a.n + kI8M - 1) / kI8M) * sh.ttiles * ks;
  if (ctas > 0x7FFFFFFF) return STB_ERR_SHAPE;
  sh.stage_bytes = i8_stage_bytes(sh.bn);
  const uint32_t sums = i8_sum_bytes(sh.bn, ks);
  sh.ring = i8_ring(sh.bn, ks, plan.half);
  sh.prefetch = ctas <= (plan.half ? 296 : 148) ? 4 : 0;       // (a CTA that starts late has nobody to hide behind)
  sh.tmem = sh.bn <= 32 ? 32 : (sh.bn <= 64 ? 64 : (sh.bn <= 128 ? 128 : 256));
  sh.off = selftest ? (sh.stages - 1) / sh.per : -1;           // (the last part that has columns)
  sh.limit = selftest ? kI8SelftestLimit : kGemmWaitLimit;
  const uint32_t smem = kI8BatchRing + (uint32_t)sh.ring * sh.stage_bytes + sums;
  CUtensorMap wmap, xmap;
  if (!i8_map(enc, &wmap, a.W, a.n, a.m, a.ldw, kI8M) || !i8_map(enc, &xmap, a.X, a.T, a.m, a.ldx, sh.bn)) return STB_ERR_ARG;
  static bool done[64] = {};
  if (allow_smem(reinterpret_cast<const void*>(gemm_i8_batch_kernel), done, kI8SmemMax) != cudaSuccess) return STB_ERR_CUDA;
  I8Args args = a;
  void* params[] = {&wmap, &xmap, &args, &sh, &dev_status};
  return launch_cluster(reinterpret_cast<const void*>(gemm_i8_batch_kernel), (unsigned)ctas, (unsigned)ks, kI8BatchThreads, smem, s, params) == cudaSuccess ? STB_OK : STB_ERR_CUDA;
}

// ---- many tokens ----------------------------------------------------------------------------------------------------------------------
// Two CTAs of a cluster compute a tile of 256 channels x `bn` tokens together (cta_group::2): each holds 128 rows of W and half of the tokens'
// rows, the first one's issuing lane multiplies for both, and each has the sums of its 128 channels for all tokens in its tensor memory.  The
// clusters stay for the whole call and take every so-many-th tile (tokens fastest, so that W is read from HBM once); two accumulators of 256 columns,
// so that a tile is read out while the next one is multiplied.  Per 128 columns of K a CTA fetches 16 KB + bn / 2 rows for 256 x bn x 128
// multiply-adds of the pair: at bn = 256 64 bytes per clock of the tensor core, what an SM gets from L2.  28672 x 8192, 2048 tokens, 282 us: 3.4 POP/s (3.0 once the
// GPU is at its power limit).
//   warp 0 brings the stages, warp 1 issues the products, warps 4 to 7 read the sums out: 32 tokens at a time through shared memory, from where they leave
//   as rows of 128 channels by TMA, or by plain stores where rows of Y are on no 16-byte boundary or n ends inside a piece of 16 bytes (TMA writes whole pieces: what lies
//   behind the n-th value would become zeros).
// `copied`: the tiles from this one on are not copied (self-test).
struct I8Prefill { int stages, ttiles, tiles, bn, ring, tma_out, copied; uint32_t stage_bytes; long long limit; };
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
__device__ __forceinline__ bool mbar_wait_cluster(uint32_t bar, uint32_t parity, volatile int* abort_flag, long long limit) {      // gemm_wait for arrivals of the other CTA
  const long long t0 = clock64();
  for (;;) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    if (ok) return true;
    if (*abort_flag) return false;
    if (clock64() - t0 > limit) { *abort_flag = 1; return false; }
  }
}
// A channel's results for 32 tokens, into rows of 128 channels in shared memory.
template <int kType>
__device__ __forceinline__ void i8_rows_out(const uint32_t (&sum)[32], const float* scales, float ws, float b, bool with_bias, uint32_t out, int row) {
#pragma unroll
  for (int i = 0; i < kI8OutTokens; i += 4) {
    const float4 xs = *reinterpret_cast<const float4*>(scales + i);
    float f[4] = {i8_value((int)sum[i], xs.x, ws, b, false), i8_value((int)sum[i + 1], xs.y, ws, b, false), i8_value((int)sum[i + 2], xs.z, ws, b, false), i8_value((int)sum[i + 3], xs.w, ws, b, false)};
    if (with_bias) {
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] = __fadd_rn(f[e], b);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (kType == STB_F32) {
        asm volatile("st.shared.f32 [%0], %1;" ::"r"(out + (uint32_t)((i + e) * kI8M + row) * 4u), "f"(f[e]) : "memory");
      } else {
        const uint16_t h = kType == STB_F16 ? __half_as_ushort(__float2half_rn(f[e])) : __bfloat16_as_ushort(__float2bfloat16_rn(f[e]));
        asm volatile("st.shared.u16 [%0], %1;" ::"r"(out + (uint32_t)((i + e) * kI8M + row) * 2u), "h"(h) : "memory");
      }
    }
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
        ok = __all_sync(0xFFFFFFFFu, gemm_wait(bar_empty + 8 * s, parity, abort_flag, sh.limit));
        if (!ok) break;
        if (leader && tile < sh.copied) {
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
      ok = __all_sync(0xFFFFFFFFu, gemm_wait(bar_empty + 8 * s, parity, abort_flag, sh.limit));
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
      ok = __all_sync(0xFFFFFFFFu, mbar_wait_cluster(bar_acc_empty + 8 * acc, ((uint32_t)(use >> 1) & 1u) ^ 1u, abort_flag, sh.limit));
      if (!ok) break;
      tc_fence_after();
      for (int it = 0; it < sh.stages; ++it) {
        ok = __all_sync(0xFFFFFFFFu, gemm_wait(bar_full + 8 * s, parity, abort_flag, sh.limit));
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
      if (leader && ok) umma_commit_pair(bar_acc_full + 8 * acc);      // (sums of fewer stages are nobody's: the waits for them run out)
      __syncwarp();
    }
  } else if (warp >= 4) {
    const int q = warp - 4, row = 32 * q + lane, t128 = (int)threadIdx.x - 128;
    const uint32_t acc_empty0 = smem_of_rank(bar_acc_empty, 0u);
    const int elem = args.ydt == STB_F32 ? 4 : 2;
    float* scales = reinterpret_cast<float*>(smem + kI8PrefillScale);
    int use = 0, buf = 0, tile = first;
    for (; tile < sh.tiles; tile += step, ++use) {
      const int acc = use & 1, r0 = (tile / sh.ttiles) * 2 * kI8M + rank * kI8M, r = r0 + row, tok0 = (tile % sh.ttiles) * sh.bn;
      const float ws = r < args.n ? w_scale[r] : 0.0f, b = bias && r < args.n ? bias[r] : 0.0f;
      asm volatile("bar.sync 1, 128;" ::: "memory");             // the last tile's scales have been read
      for (int i = t128; i < sh.bn; i += 128) scales[i] = tok0 + i < args.T ? x_scale[tok0 + i] : 0.0f;
      if (!barrier_and(gemm_wait(bar_acc_full + 8 * acc, (uint32_t)(use >> 1) & 1u, abort_flag, sh.limit))) break;      // (one verdict for the four warps)
      tc_fence_after();
      uint32_t v[2][32];
      const uint32_t from = tmem_d + ((uint32_t)(32 * q) << 16) + 256u * acc;
      tmem_ask32(from, v[0]);
      // Each chunk of 32 tokens takes the other buffer and closes one group of stores, an empty one where it lies behind the last token or channel: "all but the newest
      // group" is then every earlier use of the chunk's buffer, from tile to tile too.
#pragma unroll 2
      for (int c0 = 0; c0 < sh.bn; c0 += kI8OutTokens, buf ^= 1) {
        uint32_t(&now)[32] = v[(c0 / kI8OutTokens) & 1];
        tmem_wait32(now);
        if (c0 + kI8OutTokens < sh.bn) tmem_ask32(from + (uint32_t)(c0 + kI8OutTokens), v[((c0 / kI8OutTokens) & 1) ^ 1]);
        const uint32_t out = sbase + kI8PrefillOut + (uint32_t)buf * kI8OutBytes;
        if (t128 == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");       // the group before last, this buffer's, has been read
        asm volatile("bar.sync 1, 128;" ::: "memory");             // (plain stores: each thread reads back what it alone has written)
        switch (args.ydt) {
          case STB_F32: i8_rows_out<STB_F32>(now, scales + c0, ws, b, bias != nullptr, out, row); break;
          case STB_F16: i8_rows_out<STB_F16>(now, scales + c0, ws, b, bias != nullptr, out, row); break;
          default: i8_rows_out<STB_BF16>(now, scales + c0, ws, b, bias != nullptr, out, row); break;
        }
        if (sh.tma_out) fence_async_smem();
        asm volatile("bar.sync 1, 128;" ::: "memory");
        if (r0 >= args.n || tok0 + c0 >= args.T) {
          if (t128 == 0) asm volatile("cp.async.bulk.commit_group;" ::: "memory");
          continue;
        }
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
    for (; tile < sh.tiles; tile += step) {                      // tiles without their sums
      const int r = (tile / sh.ttiles) * 2 * kI8M + rank * kI8M + row, tok0 = (tile % sh.ttiles) * sh.bn;
      if (r < args.n)
        for (int t = tok0; t < min(tok0 + sh.bn, args.T); ++t) i8_store(args.Y, (size_t)t * args.ldy + r, args.ydt, __uint_as_float(0x7FC00000u));
    }
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

static int launch_i8_prefill(const I8Args& a, const I8Plan& plan, int* dev_status, cudaStream_t s, bool selftest) {
  EncodeTiledFn enc = encode_tiled_fn();
  if (!enc) return STB_ERR_CUDA;
  I8Prefill sh;
  sh.stages = (a.m + kI8K - 1) / kI8K;
  sh.bn = plan.bn; sh.ttiles = plan.ttiles;
  const long long tiles = (long long)((a.n + 2 * kI8M - 1) / (2 * kI8M)) * sh.ttiles;
  if (tiles > 0x7FFFFFFF) return STB_ERR_SHAPE;
  sh.tiles = (int)tiles;
  const int pairs = sh.tiles < 74 ? sh.tiles : 74;
  sh.copied = !selftest ? sh.tiles : (sh.tiles > pairs ? pairs : 0);      // (self-test: a pair's first tile, where it has more)
  sh.limit = selftest ? kI8SelftestLimit : kGemmWaitLimit;
  sh.stage_bytes = kI8StageA + (uint32_t)sh.bn * (kI8K / 2);
  sh.ring = (int)((kI8SmemMax - kI8PrefillRing) / sh.stage_bytes);
  if (sh.ring > kI8PrefillMaxRing) sh.ring = kI8PrefillMaxRing;
  const uint32_t smem = kI8PrefillRing + (uint32_t)sh.ring * sh.stage_bytes;
  CUtensorMap wmap, xmap, ymap = {};
  if (!i8_map(enc, &wmap, a.W, a.n, a.m, a.ldw, kI8M) || !i8_map(enc, &xmap, a.X, a.T, a.m, a.ldx, sh.bn / 2)) return STB_ERR_ARG;
  const int elem = a.ydt == STB_F32 ? 4 : 2;
  sh.tma_out = (a.ldy * (size_t)elem) % 16 == 0 && ((size_t)a.n * (size_t)elem) % 16 == 0 && (reinterpret_cast<uintptr_t>(a.Y) & 15u) == 0;
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
  return launch_cluster(reinterpret_cast<const void*>(gemm_i8_prefill_kernel), 2u * (unsigned)pairs, 2u, kI8PrefillThreads, smem, s, params) == cudaSuccess ? STB_OK : STB_ERR_CUDA;
}

}  // namespace stb

static int gemm_i8_impl(const int8_t* W, size_t ldw, const float* w_scale, const float* bias, int n, int m, const int8_t* X, size_t ldx,
                        const float* x_scale, int T, void* Y, stb_dtype ydt, size_t ldy, int* dev_status, void* stream, bool selftest) {
  if (!W || !w_scale || !X || !x_scale || !Y) return STB_ERR_ARG;
  if (n < 1 || m < 1 || T < 1 || m > 131071 || n > stb::kI8MaxSide || T > stb::kI8MaxSide) return STB_ERR_SHAPE;
  if (ydt != STB_F32 && ydt != STB_F16 && ydt != STB_BF16) return STB_ERR_UNSUPPORTED;
  if (ldw < (size_t)m || ldx < (size_t)m || ldy < (size_t)n || (ldw % 16) != 0 || (ldx % 16) != 0) return STB_ERR_ARG;
  const uintptr_t small = ydt == STB_F32 ? 3u : 1u;
  if (((reinterpret_cast<uintptr_t>(W) | reinterpret_cast<uintptr_t>(X)) & 15u) || (reinterpret_cast<uintptr_t>(Y) & small) ||
      ((reinterpret_cast<uintptr_t>(w_scale) | reinterpret_cast<uintptr_t>(x_scale) | reinterpret_cast<uintptr_t>(bias)) & 3u))
    return STB_ERR_ARG;
  const stb::I8Args a = {W, X, w_scale, bias, x_scale, Y, ldw, ldx, ldy, n, m, T, ydt};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (const int ksplit = stb::gemv_i8_split(n, m, T)) return selftest ? STB_ERR_UNSUPPORTED : stb::launch_gemv_i8(a, ksplit, s) == cudaSuccess ? STB_OK : STB_ERR_CUDA;
  const stb::I8Plan plan = stb::i8_plan(n, m, T);
  return plan.pair ? stb::launch_i8_prefill(a, plan, dev_status, s, selftest) : stb::launch_i8_batch(a, plan, dev_status, s, selftest);
}

extern "C" int stb_gemm_i8(const int8_t* W, size_t ldw, const float* w_scale, const float* bias, int n, int m, const int8_t* X, size_t ldx,
                           const float* x_scale, int T, void* Y, stb_dtype ydt, size_t ldy, int* dev_status, void* stream) {
  return gemm_i8_impl(W, ldw, w_scale, bias, n, m, X, ldx, x_scale, T, Y, ydt, ldy, dev_status, stream, false);
}

extern "C" int stb_gemm_i8_wait_selftest(const int8_t* W, size_t ldw, const float* w_scale, const float* bias, int n, int m, const int8_t* X, size_t ldx,
                                         const float* x_scale, int T, void* Y, stb_dtype ydt, size_t ldy, int* dev_status, void* stream) {
  if (!dev_status) return STB_ERR_ARG;
  return gemm_i8_impl(W, ldw, w_scale, bias, n, m, X, ldx, x_scale, T, Y, ydt, ldy, dev_status, stream, true);
}
