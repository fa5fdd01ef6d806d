// Rows between the linears of a decoder block: stb_quantize_i8 (rows in 8 bits, one scale each, the gated activation formed on the way)
// and stb_block_norm (the norms before and after a block with its gate, residual scale and residual sum).
//
// Both are bound by memory: every value is read once, kept in registers as fp32 (8 per thread and piece, up to four pieces), and every
// output is written once, whatever happens in between.  A row of up to 1024 values belongs to one warp, a longer one to one CTA of up to
// 1024 threads; row sums and maxima go through shuffles and, per CTA, one barrier each.
//
// 8 bits: s = max|v| / 127, q = the whole number nearest to 127 v / max|v| (ties to even), decided as in exact arithmetic: the product with
// the rounded reciprocal is within 127 * 2^-22 of the quotient, so only a value that near to a border (one in 10^4) is decided by the exact
// products 254 |v| and (2 k + 1) max|v| in float64.  The result therefore does not depend on how it is computed.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/stb.h"
#include "stb_ptx.cuh"

namespace stb {

constexpr int kPiece = 8;                 // values of a thread in a row, side by side
constexpr int kMaxPieces = 4;
constexpr int kMaxRowThreads = 1024;
constexpr int kMaxRow = kPiece * kMaxPieces * kMaxRowThreads;
constexpr float kSmallestMax = 3.0092655e-36f;      // 2^-118: below it 127 / max would overflow; such a row is zeros with scale 0

__host__ __device__ inline int dtype_bytes(int dt) { return dt == STB_F32 ? 4 : 2; }

// ---- eight values of a row ---------------------------------------------------------------------------------------------------------
// Where a thread's values of a row lie: piece p of thread `lane` of `width` is the eight values at 8 (p width + lane) where rows may be
// read in 16-byte pieces, else every value is width behind the one before it, so that a warp's loads stay together.
template <bool kVec>
struct RowPlace {
  int lane, width, m;
  __device__ __forceinline__ int at(int p, int k) const { return kVec ? (p * width + lane) * kPiece + k : (p * kPiece + k) * width + lane; }
};
__device__ __forceinline__ float load_one(const void* p, size_t i, int dt) {
  if (dt == STB_F32) return static_cast<const float*>(p)[i];
  const unsigned short u = static_cast<const unsigned short*>(p)[i];
  return dt == STB_F16 ? __half2float(__ushort_as_half(u)) : __bfloat162float(__ushort_as_bfloat16(u));
}
__device__ __forceinline__ void unpack_two(uint32_t w, int dt, float& a, float& b) {
  if (dt == STB_F16) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    a = f.x; b = f.y;
  } else {
    a = __uint_as_float(w << 16);
    b = __uint_as_float(w & 0xFFFF0000u);
  }
}
// v[p][k] = value at(p, k) of the row that starts at `row`, 0 behind its end.  All loads of a row are issued before the first is used.
template <int P, bool kVec>
__device__ __forceinline__ void load_row(const RowPlace<kVec>& pl, const void* row, int dt, float (&v)[P][kPiece]) {
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int i = pl.at(p, 0);
    if (kVec && i + kPiece <= pl.m) {
      if (dt == STB_F32) {
        const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(row) + i);
        const float4 a = q[0], b = q[1];
        v[p][0] = a.x; v[p][1] = a.y; v[p][2] = a.z; v[p][3] = a.w; v[p][4] = b.x; v[p][5] = b.y; v[p][6] = b.z; v[p][7] = b.w;
      } else {
        const uint4 a = *reinterpret_cast<const uint4*>(static_cast<const unsigned short*>(row) + i);
        unpack_two(a.x, dt, v[p][0], v[p][1]); unpack_two(a.y, dt, v[p][2], v[p][3]);
        unpack_two(a.z, dt, v[p][4], v[p][5]); unpack_two(a.w, dt, v[p][6], v[p][7]);
      }
    } else {
#pragma unroll
      for (int k = 0; k < kPiece; ++k) {
        const int e = pl.at(p, k);
        v[p][k] = e < pl.m ? load_one(row, (size_t)e, dt) : 0.0f;
      }
    }
  }
}
__device__ __forceinline__ unsigned short to_sixteen(float v, int dt) {
  return dt == STB_F16 ? __half_as_ushort(__float2half_rn(v)) : __bfloat16_as_ushort(__float2bfloat16_rn(v));
}
__device__ __forceinline__ uint32_t pack_two(float a, float b, int dt) {
  if (dt == STB_F16) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <int P, bool kVec>
__device__ __forceinline__ void store_row(const RowPlace<kVec>& pl, void* row, int dt, const float (&v)[P][kPiece]) {
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int i = pl.at(p, 0);
    if (kVec && i + kPiece <= pl.m) {
      if (dt == STB_F32) {
        float4* q = reinterpret_cast<float4*>(static_cast<float*>(row) + i);
        q[0] = make_float4(v[p][0], v[p][1], v[p][2], v[p][3]);
        q[1] = make_float4(v[p][4], v[p][5], v[p][6], v[p][7]);
      } else {
        *reinterpret_cast<uint4*>(static_cast<unsigned short*>(row) + i) =
            make_uint4(pack_two(v[p][0], v[p][1], dt), pack_two(v[p][2], v[p][3], dt), pack_two(v[p][4], v[p][5], dt), pack_two(v[p][6], v[p][7], dt));
      }
    } else {
#pragma unroll
      for (int k = 0; k < kPiece; ++k) {
        const int e = pl.at(p, k);
        if (e >= pl.m) continue;
        if (dt == STB_F32) static_cast<float*>(row)[e] = v[p][k];
        else static_cast<unsigned short*>(row)[e] = to_sixteen(v[p][k], dt);
      }
    }
  }
}

// ---- sums and maxima over the threads of a row ----------------------------------------------------------------------------------------
// kWarp: the row belongs to this warp.  Else to the CTA: every reduction of a kernel has a `slot` of its own in shared memory, so that one
// barrier does for each.  All orders are fixed.
constexpr int kSlots = 5;
struct RowShared { float part[kSlots][32]; };
template <bool kWarp>
__device__ __forceinline__ float row_sum(float v, RowShared& sh, int slot) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  if (kWarp) return v;
  const int lane = threadIdx.x & 31;
  if (lane == 0) sh.part[slot][threadIdx.x >> 5] = v;
  __syncthreads();
  v = lane < (int)(blockDim.x >> 5) ? sh.part[slot][lane] : 0.0f;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}
// of the magnitudes' bit patterns: an infinity is above every number and a NaN above that
template <bool kWarp>
__device__ __forceinline__ uint32_t row_max(uint32_t v, RowShared& sh, int slot) {
  v = __reduce_max_sync(0xFFFFFFFFu, v);
  if (kWarp) return v;
  const int lane = threadIdx.x & 31;
  if (lane == 0) sh.part[slot][threadIdx.x >> 5] = __uint_as_float(v);
  __syncthreads();
  v = lane < (int)(blockDim.x >> 5) ? __float_as_uint(sh.part[slot][lane]) : 0u;
  return __reduce_max_sync(0xFFFFFFFFu, v);
}
template <int P>
__device__ __forceinline__ uint32_t max_bits(const float (&v)[P][kPiece]) {
  uint32_t b = 0;
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int k = 0; k < kPiece; ++k) b = max(b, __float_as_uint(v[p][k]) & 0x7FFFFFFFu);
  return b;
}

// ---- a row in 8 bits --------------------------------------------------------------------------------------------------------------
struct RowScale { float largest, inverse, scale; };
__device__ __forceinline__ RowScale row_scale(uint32_t bits) {
  RowScale s;
  s.largest = __uint_as_float(bits);
  const bool broken = bits >= 0x7F800000u, live = !broken && s.largest >= kSmallestMax;
  s.scale = broken ? __uint_as_float(0x7FC00000u) : (live ? __fdiv_rn(s.largest, 127.0f) : 0.0f);
  s.inverse = live ? __fdiv_rn(127.0f, s.largest) : 0.0f;
  return s;
}
// The exact decision between two neighbours where v inverse lies next to the border between them.
__device__ __noinline__ float border_i8(float v, float t, float largest) {
  const float k = floorf(fabsf(t));
  const double a = 254.0 * (double)fabsf(v), c = (2.0 * (double)k + 1.0) * (double)largest;      // both exact
  const float r = a > c ? k + 1.0f : (a < c ? k : 2.0f * rintf(0.5f * (k + 0.25f)));              // the even one of k, k + 1 on the border itself
  return copysignf(r, v);
}
constexpr float kRoundBias = 12582912.0f;           // 1.5 * 2^23: adding it rounds to the nearest whole number, whose low byte is the sum's
// q of one value, in the low byte
__device__ __forceinline__ uint32_t value_i8(float v, const RowScale& s) {
  const float t = v * s.inverse;
  float u = t + kRoundBias;
  if (fabsf(t - (u - kRoundBias)) > 0.4999f) u = border_i8(v, t, s.largest) + kRoundBias;
  return __float_as_uint(u);
}
template <int P, bool kVec>
__device__ __forceinline__ void store_row_i8(const RowPlace<kVec>& pl, int8_t* row, const float (&v)[P][kPiece], const RowScale& s) {
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int i = pl.at(p, 0);
    if (i >= pl.m) break;
    uint32_t q[kPiece];
#pragma unroll
    for (int k = 0; k < kPiece; ++k) q[k] = s.inverse == 0.0f ? 0u : value_i8(v[p][k], s);
    if (kVec && i + kPiece <= pl.m) {
      const uint32_t lo = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
      const uint32_t hi = __byte_perm(__byte_perm(q[4], q[5], 0x0040), __byte_perm(q[6], q[7], 0x0040), 0x5410);
      *reinterpret_cast<uint2*>(row + i) = make_uint2(lo, hi);
    } else {
#pragma unroll
      for (int k = 0; k < kPiece; ++k)
        if (pl.at(p, k) < pl.m) row[pl.at(p, k)] = (int8_t)(q[k] & 0xFFu);
    }
  }
}

// ---- the gated activation ---------------------------------------------------------------------------------------------------------
// silu(a) b rounded to fp32 and then to the 16-bit type, as exact arithmetic would: evaluated in fp32 within 2^-21 (expf one unit in the
// last place, __fdividef two, the sum and the product half a one each), and where both ends of a band of 1.5 times that do not round to
// the same 16-bit value, in float64.  Products too small for a relative bound in fp32 go that way as well.
__device__ __noinline__ float gated_exact(float a, float b) {
  const double d = (double)a;
  return (float)(d / (1.0 + exp(-d)) * (double)b);
}
__device__ __forceinline__ void gated_two(float& a0, float& a1, float b0, float b1, int dt) {
  constexpr float kBand = 1.5f / 2097152.0f;
  const float h0 = __fdividef(a0, 1.0f + expf(-a0)) * b0, h1 = __fdividef(a1, 1.0f + expf(-a1)) * b1;
  const uint32_t lo = pack_two(h0 * (1.0f - kBand), h1 * (1.0f - kBand), dt), hi = pack_two(h0 * (1.0f + kBand), h1 * (1.0f + kBand), dt);
  constexpr float kTiny = 7.8886091e-31f;           // 2^-100
  const bool tiny0 = fabsf(h0) < kTiny && a0 != 0.0f && b0 != 0.0f, tiny1 = fabsf(h1) < kTiny && a1 != 0.0f && b1 != 0.0f;
  uint32_t w = lo;
  if (lo != hi || tiny0 || tiny1) w = pack_two(gated_exact(a0, b0), gated_exact(a1, b1), dt);
  unpack_two(w, dt, a0, a1);
}
template <int P>
__device__ __forceinline__ void gated_row(float (&a)[P][kPiece], const float (&b)[P][kPiece], int dt) {
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int k = 0; k < kPiece; k += 2) gated_two(a[p][k], a[p][k + 1], b[p][k], b[p][k + 1], dt);
}

// ---- stb_quantize_i8 ----------------------------------------------------------------------------------------------------------------
struct QuantI8Args {
  const void *x, *x2;
  int dt, rows, m;
  size_t ldx, ldx2, ldq;
  int8_t* q;
  float* scale;
};
// kLong: the row does not fit the registers of a CTA; it is read twice.
template <int P, bool kVec, bool kWarp, bool kGated, bool kLong>
__global__ void __launch_bounds__(kMaxRowThreads)
quantize_i8_kernel(const QuantI8Args args) {
  __shared__ RowShared sh;
  const void *x = args.x, *x2 = args.x2;
  begin_after(x, x2);
  const int row = kWarp ? (int)(blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5)) : (int)blockIdx.x;
  if (kWarp && row >= args.rows) return;
  const int bytes = dtype_bytes(args.dt);
  const char *xr = static_cast<const char*>(x) + (size_t)row * args.ldx * (size_t)bytes, *xr2 = static_cast<const char*>(x2) + (size_t)row * args.ldx2 * (size_t)bytes;
  int8_t* qr = args.q + (size_t)row * args.ldq;
  RowPlace<kVec> pl{kWarp ? (int)(threadIdx.x & 31) : (int)threadIdx.x, kWarp ? 32 : (int)blockDim.x, args.m};
  const int span = pl.width * kPiece * P;
  auto read = [&](int base, float (&v)[P][kPiece]) {
    pl.m = args.m - base;
    load_row<P, kVec>(pl, xr + (size_t)base * bytes, args.dt, v);
    if (kGated) {
      float b[P][kPiece];
      load_row<P, kVec>(pl, xr2 + (size_t)base * bytes, args.dt, b);
      gated_row<P>(v, b, args.dt);
    }
  };
  float v[P][kPiece];
  uint32_t bits = 0;
  if (kLong) {
    for (int base = 0; base < args.m; base += span) { read(base, v); bits = max(bits, max_bits<P>(v)); }
  } else {
    read(0, v);
    bits = max_bits<P>(v);
  }
  const RowScale s = row_scale(row_max<kWarp>(bits, sh, 0));
  if (pl.lane == 0) args.scale[row] = s.scale;
  if (kLong) {
    for (int base = 0; base < args.m; base += span) { read(base, v); store_row_i8<P, kVec>(pl, qr + base, v, s); }
  } else {
    store_row_i8<P, kVec>(pl, qr, v, s);
  }
}

// ---- stb_block_norm -----------------------------------------------------------------------------------------------------------------
template <int P, bool kVec, bool kWarp>
__device__ __forceinline__ void norm_row(const RowPlace<kVec>& pl, float (&v)[P][kPiece], int kind, float eps, RowShared& sh, int slot) {
  const float per = __fdiv_rn(1.0f, (float)pl.m);
  if (kind == STB_NORM_LAYER) {
    float sum = 0.0f;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int k = 0; k < kPiece; ++k) sum += v[p][k];
    const float mean = __fdiv_rn(row_sum<kWarp>(sum, sh, slot), (float)pl.m);
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int k = 0; k < kPiece; ++k) v[p][k] = pl.at(p, k) < pl.m ? v[p][k] - mean : 0.0f;
  }
  float squares = 0.0f;
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int k = 0; k < kPiece; ++k) squares = fmaf(v[p][k], v[p][k], squares);
  const float inv = rsqrtf(fmaf(row_sum<kWarp>(squares, sh, slot + 1), per, eps));
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int k = 0; k < kPiece; ++k) v[p][k] *= inv;
}
template <int P, bool kVec>
__device__ __forceinline__ void times_row(const RowPlace<kVec>& pl, float (&v)[P][kPiece], const void* w, int dt) {
  float f[P][kPiece];
  load_row<P, kVec>(pl, w, dt, f);
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int k = 0; k < kPiece; ++k) v[p][k] *= f[p][k];
}
template <int P, bool kVec>
__device__ __forceinline__ void plus_row(const RowPlace<kVec>& pl, float (&v)[P][kPiece], const void* w, int dt) {
  float f[P][kPiece];
  load_row<P, kVec>(pl, w, dt, f);
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int k = 0; k < kPiece; ++k) v[p][k] += f[p][k];
}
template <int P, bool kVec, bool kWarp>
__global__ void __launch_bounds__(kMaxRowThreads)
block_norm_kernel(const stb_norm a) {
  __shared__ RowShared sh;
  const void *x = a.x, *resid = a.resid, *pw = a.post_weight, *pb = a.post_bias, *gate = a.gate, *w = a.weight, *b = a.bias;
  begin_after(x, resid, pw, pb, gate, w, b);
  const int row = kWarp ? (int)(blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5)) : (int)blockIdx.x;
  if (kWarp && row >= a.tokens) return;
  const RowPlace<kVec> pl{kWarp ? (int)(threadIdx.x & 31) : (int)threadIdx.x, kWarp ? 32 : (int)blockDim.x, a.h};
  auto row_of = [&](const void* base, size_t r, size_t ld, int dt) { return static_cast<const char*>(base) + r * ld * (size_t)dtype_bytes(dt); };
  float v[P][kPiece], r[P][kPiece];
  load_row<P, kVec>(pl, row_of(x, row, a.ldx, a.xdt), a.xdt, v);
  if (resid) load_row<P, kVec>(pl, row_of(resid, row, a.ldr, a.rdt), a.rdt, r);
  if (a.post) {
    norm_row<P, kVec, kWarp>(pl, v, a.kind, a.eps, sh, 0);
    if (pw) times_row<P, kVec>(pl, v, pw, a.wdt);
    if (pb) plus_row<P, kVec>(pl, v, pb, a.wdt);
  }
  if (gate) times_row<P, kVec>(pl, v, row_of(gate, row / a.tokens_per_gate, a.ldgate, a.wdt), a.wdt);
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int k = 0; k < kPiece; ++k) v[p][k] = resid ? fmaf(a.alpha, v[p][k], r[p][k]) : a.alpha * v[p][k];
  if (a.resid_out) store_row<P, kVec>(pl, const_cast<char*>(row_of(a.resid_out, row, a.ldro, a.rdt)), a.rdt, v);
  if (!a.y && !a.q) return;
  norm_row<P, kVec, kWarp>(pl, v, a.kind, a.eps, sh, 2);
  if (w) times_row<P, kVec>(pl, v, w, a.wdt);
  if (b) plus_row<P, kVec>(pl, v, b, a.wdt);
  if (a.y) store_row<P, kVec>(pl, const_cast<char*>(row_of(a.y, row, a.ldy, a.ydt)), a.ydt, v);
  if (a.q) {
    const RowScale s = row_scale(row_max<kWarp>(max_bits<P>(v), sh, 4));
    if (pl.lane == 0) a.q_scale[row] = s.scale;
    store_row_i8<P, kVec>(pl, a.q + (size_t)row * a.ldq, v, s);
  }
}

// How rows of `m` values are dealt out.  Few rows: one piece per thread, for the shortest way through a row; many: two, which halves the
// warps that wait at a barrier.
struct RowShape { int pieces, threads, rows_per_cta; bool warp, long_row; };
static RowShape row_shape(int m, int rows) {
  RowShape s;
  s.long_row = m > kMaxRow;
  s.warp = m <= 32 * kPiece * kMaxPieces && (rows > 148 || m <= 32 * kPiece);
  if (s.warp) {
    s.pieces = m <= 32 * kPiece ? 1 : (m <= 64 * kPiece ? 2 : 4);
    s.rows_per_cta = rows >= 148 * 8 ? 8 : (rows >= 148 * 2 ? 2 : 1);
    s.threads = 32 * s.rows_per_cta;
    return s;
  }
  s.rows_per_cta = 1;
  const int pieces = (m + kPiece - 1) / kPiece;
  s.pieces = rows > 148 ? 2 : 1;
  while (s.pieces < kMaxPieces && pieces > s.pieces * kMaxRowThreads) s.pieces *= 2;
  s.threads = ((pieces + s.pieces - 1) / s.pieces + 31) / 32 * 32;
  if (s.threads > kMaxRowThreads) s.threads = kMaxRowThreads;
  return s;
}

static bool rows_aligned(const void* p, size_t ld, int bytes, size_t to) { return !p || ((reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0 && (ld * (size_t)bytes) % to == 0); }
static bool element_aligned(const void* p, int dt) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(dtype_bytes(dt) - 1)) == 0; }
static bool known_dtype(int dt) { return dt == STB_F16 || dt == STB_BF16 || dt == STB_F32; }

template <bool kGated>
static cudaError_t launch_quantize(const QuantI8Args& a, const RowShape& s, bool vec, cudaStream_t st) {
  const dim3 grid((unsigned)((a.rows + s.rows_per_cta - 1) / s.rows_per_cta)), block((unsigned)s.threads);
  auto go = [&](auto kernel) { return launch_after(kernel, grid, block, 0, st, a); };
  if (s.long_row) return vec ? go(quantize_i8_kernel<2, true, false, kGated, true>) : go(quantize_i8_kernel<2, false, false, kGated, true>);
  if (s.warp) {
    if (s.pieces == 1) return vec ? go(quantize_i8_kernel<1, true, true, kGated, false>) : go(quantize_i8_kernel<1, false, true, kGated, false>);
    if (s.pieces == 2) return vec ? go(quantize_i8_kernel<2, true, true, kGated, false>) : go(quantize_i8_kernel<2, false, true, kGated, false>);
    return vec ? go(quantize_i8_kernel<4, true, true, kGated, false>) : go(quantize_i8_kernel<4, false, true, kGated, false>);
  }
  if (s.pieces == 1) return vec ? go(quantize_i8_kernel<1, true, false, kGated, false>) : go(quantize_i8_kernel<1, false, false, kGated, false>);
  if (s.pieces == 2) return vec ? go(quantize_i8_kernel<2, true, false, kGated, false>) : go(quantize_i8_kernel<2, false, false, kGated, false>);
  return vec ? go(quantize_i8_kernel<4, true, false, kGated, false>) : go(quantize_i8_kernel<4, false, false, kGated, false>);
}

}  // namespace stb

extern "C" int stb_quantize_i8(const void* x, size_t ldx, const void* x2, size_t ldx2, stb_dtype xdt, int rows, int m, int8_t* q, size_t ldq,
                               float* scale, void* stream) {
  if (!x || !q || !scale) return STB_ERR_ARG;
  if (rows < 1 || m < 1) return STB_ERR_SHAPE;
  if (!stb::known_dtype(xdt) || (x2 && xdt == STB_F32)) return STB_ERR_UNSUPPORTED;      // the gated activation is one of 16 bits
  if (ldx < (size_t)m || (x2 && ldx2 < (size_t)m) || ldq < (size_t)m) return STB_ERR_ARG;
  if (!stb::element_aligned(x, xdt) || !stb::element_aligned(x2, xdt) || !stb::element_aligned(scale, STB_F32)) return STB_ERR_ARG;
  const int bytes = stb::dtype_bytes(xdt);
  const bool vec = stb::rows_aligned(x, ldx, bytes, 16) && stb::rows_aligned(x2, ldx2, bytes, 16) && stb::rows_aligned(q, ldq, 1, 8);
  const stb::QuantI8Args a = {x, x2, xdt, rows, m, ldx, ldx2, ldq, q, scale};
  stb::RowShape s = stb::row_shape(m, rows);
  if (s.long_row) s.threads = stb::kMaxRowThreads;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return (x2 ? stb::launch_quantize<true>(a, s, vec, st) : stb::launch_quantize<false>(a, s, vec, st)) == cudaSuccess ? STB_OK : STB_ERR_CUDA;
}

extern "C" int stb_block_norm(const stb_norm* args, void* stream) {
  if (!args) return STB_ERR_ARG;
  stb_norm a = *args;
  if (!a.x || (!a.resid_out && !a.y && !a.q) || (a.q && !a.q_scale)) return STB_ERR_ARG;
  if (a.tokens < 1 || a.h < 1) return STB_ERR_SHAPE;
  if (a.h > stb::kMaxRow) return STB_ERR_SIZE;
  if (a.kind != STB_NORM_RMS && a.kind != STB_NORM_LAYER) return STB_ERR_UNSUPPORTED;
  const bool vectors = a.post_weight || a.post_bias || a.gate || a.weight || a.bias, residual = a.resid || a.resid_out;
  if (!stb::known_dtype(a.xdt) || (residual && !stb::known_dtype(a.rdt)) || (vectors && !stb::known_dtype(a.wdt)) || (a.y && !stb::known_dtype(a.ydt)))
    return STB_ERR_UNSUPPORTED;
  if (!(a.eps >= 0.0f) || a.eps > 3.4e38f || !(a.alpha >= -3.4e38f && a.alpha <= 3.4e38f)) return STB_ERR_ARG;
  if ((a.post_weight || a.post_bias) && !a.post) return STB_ERR_ARG;
  if ((a.weight || a.bias) && !a.y && !a.q) return STB_ERR_ARG;
  const size_t h = (size_t)a.h;
  if (a.ldx < h || (a.resid && a.ldr < h) || (a.resid_out && a.ldro < h) || (a.y && a.ldy < h) || (a.q && a.ldq < h)) return STB_ERR_ARG;
  if (a.gate && (a.tokens_per_gate < 1 || (a.tokens > a.tokens_per_gate && a.ldgate < h))) return STB_ERR_ARG;
  if (!stb::element_aligned(a.x, a.xdt) || !stb::element_aligned(a.resid, a.rdt) || !stb::element_aligned(a.resid_out, a.rdt) || !stb::element_aligned(a.y, a.ydt) ||
      !stb::element_aligned(a.q_scale, STB_F32) || !stb::element_aligned(a.post_weight, a.wdt) || !stb::element_aligned(a.post_bias, a.wdt) ||
      !stb::element_aligned(a.gate, a.wdt) || !stb::element_aligned(a.weight, a.wdt) || !stb::element_aligned(a.bias, a.wdt))
    return STB_ERR_ARG;
  const int xb = stb::dtype_bytes(a.xdt), rb = stb::dtype_bytes(a.rdt), wb = stb::dtype_bytes(a.wdt), yb = stb::dtype_bytes(a.ydt);
  const bool vec = stb::rows_aligned(a.x, a.ldx, xb, 16) && stb::rows_aligned(a.resid, a.ldr, rb, 16) && stb::rows_aligned(a.resid_out, a.ldro, rb, 16) &&
                   stb::rows_aligned(a.y, a.ldy, yb, 16) && stb::rows_aligned(a.q, a.ldq, 1, 8) && stb::rows_aligned(a.gate, a.tokens > a.tokens_per_gate ? a.ldgate : 0, wb, 16) &&
                   stb::rows_aligned(a.post_weight, 0, wb, 16) && stb::rows_aligned(a.post_bias, 0, wb, 16) && stb::rows_aligned(a.weight, 0, wb, 16) &&
                   stb::rows_aligned(a.bias, 0, wb, 16);
  const stb::RowShape s = stb::row_shape(a.h, a.tokens);
  const dim3 grid((unsigned)((a.tokens + s.rows_per_cta - 1) / s.rows_per_cta)), block((unsigned)s.threads);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  auto go = [&](auto kernel) { return stb::launch_after(kernel, grid, block, 0, st, a) == cudaSuccess ? STB_OK : STB_ERR_CUDA; };
  if (s.warp) {
    if (s.pieces == 1) return vec ? go(stb::block_norm_kernel<1, true, true>) : go(stb::block_norm_kernel<1, false, true>);
    if (s.pieces == 2) return vec ? go(stb::block_norm_kernel<2, true, true>) : go(stb::block_norm_kernel<2, false, true>);
    return vec ? go(stb::block_norm_kernel<4, true, true>) : go(stb::block_norm_kernel<4, false, true>);
  }
  if (s.pieces == 1) return vec ? go(stb::block_norm_kernel<1, true, false>) : go(stb::block_norm_kernel<1, false, false>);
  if (s.pieces == 2) return vec ? go(stb::block_norm_kernel<2, true, false>) : go(stb::block_norm_kernel<2, false, false>);
  return vec ? go(stb::block_norm_kernel<4, true, false>) : go(stb::block_norm_kernel<4, false, false>);
}
